"""Features of requests from their tokens, for a length predictor: what `LengthPredictor` takes where a request is its prompt.

A token's row of a table is multiplied into a gate and a value for every channel; a gated recurrence goes along the tokens of a
request; its last state is what the request is to the predictor.  While a request runs every token that it generates moves its state on by one
step, so that its remaining length can be predicted anew (Sec. 3.4's periodic re-check) without reading it again.

Rows, products, the recurrence, dropout and all their gradients are kernels of the library; torch holds the memory, draws the first weights and
adds up the update.

    python -m paper_2605_16867_amd.reader        # trains on synthetic prompts, routes a fleet's arrivals, re-checks what runs
"""
from __future__ import annotations

import math
from typing import Optional, Tuple

import torch

from . import binding


class PromptReader:
    """Weights, gradients and the buffers of up to `max_tokens` tokens and `max_rows` requests a call, on the current device."""

    def __init__(self, n_vocab: int, n_out: int, width: int = 256, max_tokens: int = 1 << 16, max_rows: int = 4096, drop: float = 0.1,
                 dtype: torch.dtype = torch.bfloat16, max_norm: float = 1.0, seed: int = 0):
        self.n_vocab, self.n_out, self.width, self.drop, self.dtype, self.max_norm, self.seed = n_vocab, n_out, width, drop, dtype, max_norm, seed
        self.h = binding.Tokens(max_tokens, n_vocab, max(width, n_out))
        self.products = binding.Experts(1, max_tokens, 1)
        self.dev = torch.device("cuda", torch.cuda.current_device())
        g = torch.Generator(device=self.dev)
        g.manual_seed(seed)
        self.scale = math.sqrt(width)
        self.table = (torch.randn(n_vocab, width, generator=g, device=self.dev) / self.scale).to(dtype)
        self.w = (torch.randn(2 * n_out, width, generator=g, device=self.dev) / self.scale).to(dtype)
        # channels remember 2 to 500 tokens at first: that many of them are a gate of log(tokens - 1)
        far = torch.logspace(math.log10(2), math.log10(500), n_out, device=self.dev)
        self.b = torch.cat([torch.log(far - 1 + 1e-3), torch.zeros(n_out, device=self.dev)]).to(dtype)
        self.dtable, self.dw, self.db = (torch.empty_like(t) for t in (self.table, self.w, self.b))
        T, R, f32 = max_tokens, max_rows, torch.float32
        self.rows, self.both = self._empty(T, width), self._empty(T, 2 * n_out)
        # a batch's own, which wait for its gradient while others are read
        self.batch_rows, self.batch_both, self.y = self._empty(T, width), self._empty(T, 2 * n_out), self._empty(T, n_out)
        self.drows, self.dboth = self._empty(T, width), self._empty(T, 2 * n_out)
        self.last, self.dlast, self.features = self._empty(R, n_out, of=f32), self._empty(R, n_out, of=f32), self._empty(R, n_out)
        self.norm = self._empty(1, of=f32)
        self.step = torch.zeros(1, dtype=torch.int64, device=self.dev)      # of training: what dropout draws by

    def _empty(self, *shape, of=None):
        return torch.empty(*shape, dtype=of or self.dtype, device=self.dev)

    def _gates(self, token: torch.Tensor, rows: torch.Tensor, both: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
        """Gates and values of tokens, the halves of one product's result."""
        n = token.numel()
        self.h.gr_token_embed(token, self.table, rows[:n], scale=self.scale)
        self.products.gr_expert_linear(rows[:n], self.w, both[:n], bias=self.b)
        return both[:n, :self.n_out], both[:n, self.n_out:]

    # ---- reading ------------------------------------------------------------------------------

    def read(self, token: torch.Tensor, off: torch.Tensor, start: Optional[torch.Tensor] = None) -> torch.Tensor:
        """States [requests, n_out] (float32) after the tokens of every request: token int32 [tokens], request r's at off[r] .. off[r+1]-1.  start:
        the states that they go on from (of what was read of them before).  The caller's to keep."""
        out = self._empty(off.numel() - 1, self.n_out, of=torch.float32)
        self.h.gr_gated_scan(*self._gates(token, self.rows, self.both), off=off, h0=start, out_h=out)
        return out

    def advance(self, token: torch.Tensor, state: torch.Tensor) -> None:
        """A generated token of every running request: states [requests, n_out] move on in place."""
        self.h.gr_gated_scan(*self._gates(token, self.rows, self.both), h0=state, out_h=state)

    def features_of(self, state: torch.Tensor) -> torch.Tensor:
        """What a length predictor takes of states (in single precision the states themselves, which `advance` moves on)."""
        return state.to(self.dtype)

    # ---- training -----------------------------------------------------------------------------

    def train_forward(self, token: torch.Tensor, off: torch.Tensor) -> torch.Tensor:
        """Features [requests, n_out] of a batch, some of them dropped; valid until the next batch's."""
        n, R = token.numel(), off.numel() - 1
        self.step.add_(1)
        self.h.gr_gated_scan(*self._gates(token, self.batch_rows, self.batch_both), out_y=self.y[:n], off=off, out_h=self.last[:R])
        self.features[:R].copy_(self.last[:R])
        self.h.gr_dropout(self.features[:R], self.features[:R], self.drop, self.seed, offset_add=self.step)
        return self.features[:R]

    def backward(self, token: torch.Tensor, off: torch.Tensor, dfeatures: torch.Tensor) -> None:
        """Gradients of the weights from that of the features of the last `train_forward`, which is overwritten.  What was read since does not matter."""
        n, R, C = token.numel(), off.numel() - 1, self.n_out
        self.h.gr_dropout(dfeatures, dfeatures, self.drop, self.seed, offset_add=self.step)
        self.dlast[:R].copy_(dfeatures)
        both, d = self.batch_both[:n], self.dboth[:n]
        self.h.gr_gated_scan_backward(both[:, :C], both[:, C:], self.y[:n], d[:, :C], d[:, C:], off=off, dh=self.dlast[:R])
        self.products.gr_expert_linear_backward(self.batch_rows[:n], self.w, d, out_dx=self.drows[:n], out_dw=self.dw, out_db=self.db)
        self.h.gr_token_embed_backward(token, self.drows[:n], self.dtable, scale=self.scale)

    def update(self, rate: float) -> None:
        gradients = [self.dtable, self.dw, self.db]
        self.products.gr_clip_gradients(gradients, self.max_norm, self.norm)
        for p, g in zip((self.table, self.w, self.b), gradients):
            p.add_(g, alpha=-rate)


def train(reader: PromptReader, predictor, token, off, target, expert, rate: float, reader_rate: float) -> torch.Tensor:
    """A step of the predictor's first phase with the reader in front of it: prompts with logarithms of lengths `target`, each given to
    expert [requests].  Returns the loss."""
    x = reader.train_forward(token, off)
    dx = torch.empty_like(x)
    loss = predictor.train_experts(x, target, expert, rate, out_dx=dx)
    reader.backward(token, off, dx)
    reader.update(reader_rate)
    return loss


def synthetic_prompts(rows: int, n_vocab: int, n_kind: int, mean_tokens: int, seed: int, kinds_seed: int = 0):
    """Prompts of n_kind kinds, whose tokens come from a part of the vocabulary of their own half of the time: token [tokens], off [rows + 1],
    logarithms of lengths [rows], kinds [rows].  A length hangs on the kind and on the share of some telling tokens in the prompt."""
    dev = torch.device("cuda", torch.cuda.current_device())
    of_kinds, g = torch.Generator(device=dev), torch.Generator(device=dev)
    of_kinds.manual_seed(kinds_seed)
    g.manual_seed(seed + 1)
    base = 3 + 4 * torch.rand(n_kind, generator=of_kinds, device=dev)
    kind = torch.randint(n_kind, (rows,), generator=g, device=dev)
    length = (torch.rand(rows, generator=g, device=dev).neg_().log1p_().neg_() * mean_tokens).long() + 1
    off = torch.cat([torch.zeros(1, dtype=torch.long, device=dev), length.cumsum(0)])
    of = torch.repeat_interleave(torch.arange(rows, device=dev), length)
    n, part = of.numel(), n_vocab // n_kind
    own = torch.rand(n, generator=g, device=dev) < 0.5
    token = torch.where(own, kind[of] * part + torch.randint(max(part, 1), (n,), generator=g, device=dev),
                        torch.randint(n_vocab, (n,), generator=g, device=dev))
    telling = torch.zeros(rows, device=dev).index_add_(0, of, (token % 16 == 0).float()) / length
    return token.int(), off.int(), base[kind] + 4 * telling, kind.int()


def main() -> None:
    from . import predictor, workloads
    n_vocab, n_out, rows = 4096, 256, 1024
    reader = PromptReader(n_vocab, n_out, width=128, max_tokens=1 << 18, max_rows=8192)
    p = predictor.LengthPredictor(n_out, hidden=(256, 128, 64), router_hidden=128, max_rows=8192)
    for step in range(200):
        token, off, target, kind = synthetic_prompts(rows, n_vocab, p.n_expert, 64, seed=step)
        loss = train(reader, p, token, off, target, kind, 0.05, 0.5)
        if step % 50 == 0 or step == 199:
            print(f"reader and experts, step {step}: mean squared error of the logarithm {float(loss):.3f}, gradient norms {float(reader.norm):.2f} "
                  f"and {float(p.norm):.2f}", flush=True)
    for step in range(100):
        token, off, target, kind = synthetic_prompts(rows, n_vocab, p.n_expert, 64, seed=step)
        loss = p.train_router(reader.features_of(reader.read(token, off)), target, 0.2)
    print(f"router: mean squared error of the logarithm {float(loss):.3f}", flush=True)

    # the arrivals of a fleet, routed by what is predicted of their prompts
    fl = workloads.make_fleet(workloads.spec("mid"))
    up = lambda a: torch.from_numpy(a).to(reader.dev)
    max_len = int(fl.spec.max_len)
    h = binding.Fleet(*(fl.coef[k] for k in ("delta", "alpha", "beta", "gamma")), fl.inst_class, fl.spec.n_active + fl.spec.n_queued, max_len,
                      max(len(fl.in_prompt), len(fl.act_prompt)))
    lists = [up(a) for a in (fl.act_off, fl.act_prompt, fl.act_gen, fl.act_rem, fl.q_off, fl.q_prompt, fl.q_len)]
    finish = torch.empty(len(fl.act_prompt), dtype=torch.float32, device=reader.dev)
    h.gr_build_status(*lists, finish)
    token, off, _, _ = synthetic_prompts(len(fl.in_prompt), n_vocab, p.n_expert, 48, seed=10_000)
    length = p.predict(reader.features_of(reader.read(token, off)), max_len)
    inst, slack = torch.empty_like(length), torch.empty(len(length), dtype=torch.float32, device=reader.dev)
    h.gr_score_route(off[1:] - off[:-1], length, up(fl.in_budget), inst, slack)
    print(f"{len(length)} arrivals of {token.numel()} tokens sent to {int(inst.unique().numel())} instances, {float((slack >= 0).float().mean()):.0%} "
          "expected in time")

    # what runs has generated some tokens more: its states move on, its remaining lengths are predicted anew
    n = len(fl.act_prompt)
    token, off, _, _ = synthetic_prompts(n, n_vocab, p.n_expert, 24, seed=20_000)
    state = reader.read(token, off)
    for step in range(8):
        reader.advance(torch.randint(n_vocab, (n,), device=reader.dev, dtype=torch.int32), state)
    lists[3] = torch.cat([p.predict(reader.features_of(s), max_len) for s in state.split(p.max_rows)])
    flag, target = torch.empty(n, dtype=torch.uint8, device=reader.dev), torch.empty(n, dtype=torch.int32, device=reader.dev)
    target_slack = torch.empty(n, dtype=torch.float32, device=reader.dev)
    h.gr_risk_scan(*lists, up(fl.act_budget), flag, finish, target, target_slack)
    print(f"{n} running requests re-checked: {int(flag.sum())} at risk, {int(((target >= 0) & (target_slack >= 0)).sum())} in time elsewhere")


if __name__ == "__main__":
    main()
