"""A length predictor of the paper's kind (Sec. 3.2) from the library's operators: where the predicted lengths of
`gr_score_route` and the refreshed ones of `gr_risk_scan` come from.

A two-layer network scores the experts of a request; every expert is a network of four layers with one result; the results of the
`top_k` best (the paper: all nine) are added up by their shares.  Results are logarithms of lengths.  Trained as in the paper in two
phases: the experts, each on requests given to it, then the router with the experts as they are.

Every product, choice, sum, gradient and clipping is a kernel of the library; torch holds the memory, draws the first weights, and
does the elementwise arithmetic of the loss, the update and the rounding to whole tokens.

    python -m paper_2605_16867_amd.predictor        # trains on synthetic requests, routes a fleet's arrivals by what it predicts
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import torch

from . import binding


class LengthPredictor:
    """Weights, gradients and the buffers of up to `max_rows` requests a call, on the current device."""

    def __init__(self, n_in: int, n_expert: int = 9, hidden: Sequence[int] = (1024, 512, 128), router_hidden: int = 512,
                 top_k: Optional[int] = None, max_rows: int = 4096, dtype: torch.dtype = torch.bfloat16, max_norm: float = 1.0,
                 seed: int = 0):
        self.n_expert, self.top_k = n_expert, top_k or n_expert
        self.max_rows, self.dtype, self.max_norm = max_rows, dtype, max_norm
        self.h = binding.Experts(n_expert, max_rows, self.top_k)
        self.dev = torch.device("cuda", torch.cuda.current_device())
        g = torch.Generator(device=self.dev)
        g.manual_seed(seed)

        def weights(*shape):
            return (torch.randn(*shape, generator=g, device=self.dev) * (2.0 / shape[-1]) ** 0.5).to(dtype)

        widths = [n_in, *hidden, 1]
        self.widths = widths
        self.w = [weights(n_expert, o, i) for i, o in zip(widths, widths[1:])]
        self.b = [self._empty(n_expert, o).zero_() for o in widths[1:]]
        self.router_w = [weights(router_hidden, n_in), weights(n_expert, router_hidden)]
        self.router_b = [self._empty(router_hidden).zero_(), self._empty(n_expert).zero_()]
        self.dw, self.db = [torch.empty_like(w) for w in self.w], [torch.empty_like(b) for b in self.b]
        self.router_dw, self.router_db = [torch.empty_like(w) for w in self.router_w], [torch.empty_like(b) for b in self.router_b]
        # what a call works in: a row per request, or per request and expert
        T, S, i32, f32 = max_rows, max_rows * self.top_k, torch.int32, torch.float32
        self.off, self.slot = self._empty(n_expert + 1, of=i32), self._empty(S, of=i32)
        self.pos, self.expert = self._empty(T, self.top_k, of=i32), self._empty(T, self.top_k, of=i32)
        self.weight, self.dweight = self._empty(T, self.top_k, of=f32), self._empty(T, self.top_k, of=f32)
        self.y = [self._empty(S, o) for o in widths[1:]]
        self.router_y = [self._empty(T, router_hidden), self._empty(T, n_expert)]
        self.out, self.dlogits = self._empty(T, 1), self._empty(T, n_expert)
        self.dy = [self._empty(S, o) for o in widths[1:]]
        self.router_dy = self._empty(T, router_hidden)
        self.norm = self._empty(1, of=f32)

    def _empty(self, *shape, of=None):
        return torch.empty(*shape, dtype=of or self.dtype, device=self.dev)

    def parameters(self) -> int:
        return sum(t.numel() for t in (*self.w, *self.b, *self.router_w, *self.router_b))

    # ---- forward ------------------------------------------------------------------------------

    def _experts(self, x, n, top_k) -> torch.Tensor:
        """Results of the experts, by position, from the order that self.off and self.slot[:n] hold."""
        off, slot, last = self.off, self.slot[:n], len(self.w) - 1
        for i, (w, b) in enumerate(zip(self.w, self.b)):
            first = dict(slot=slot, top_k=top_k) if i == 0 else {}
            self.h.gr_expert_linear(x if i == 0 else self.y[i - 1][:n], w, self.y[i][:n], bias=b, off=off, relu=i < last, **first)
        return self.y[last][:n]

    def _route(self, x):
        T, k = x.shape[0], self.top_k
        hidden, logits = self.router_y[0][:T], self.router_y[1][:T]
        self.h.gr_expert_linear(x, self.router_w[0], hidden, bias=self.router_b[0], relu=True)
        self.h.gr_expert_linear(hidden, self.router_w[1], logits, bias=self.router_b[1])
        self.h.gr_expert_route(logits, self.weight[:T], self.expert[:T], self.off, self.slot[:T * k], self.pos[:T], renormalise=True)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """Logarithms of the lengths of requests x [rows, n_in], [rows, 1]; valid until the next call."""
        T = x.shape[0]
        self._route(x)
        y = self._experts(x, T * self.top_k, self.top_k)
        self.h.gr_expert_combine(y, self.pos[:T], self.out[:T], weight=self.weight[:T])
        return self.out[:T]

    def predict(self, x: torch.Tensor, max_len: int) -> torch.Tensor:
        """Predicted decode lengths, int32 [rows], in [1, max_len]; max_len where a result is no number."""
        n = self.forward(x).float().exp_().round_().double()      # (single precision has no room for every max_len)
        return n.nan_to_num_(nan=max_len).clamp_(1, max_len).to(torch.int32).view(-1)

    # ---- training -----------------------------------------------------------------------------

    def _loss(self, out, target, like, counts=None):
        """Mean squared error of the logarithms, and its gradient in `like`; of those rows that `counts` says (None: all)."""
        error = out.float().view(-1) - target
        if counts is None:
            return (error * error).mean(), (error * (2.0 / error.numel())).to(self.dtype).view_as(like)
        error = torch.where(counts, error, torch.zeros_like(error))
        n = counts.sum().clamp(min=1)
        return (error * error).mean() * (error.numel() / n), (error * (2.0 / n)).to(self.dtype).view_as(like)

    def _update(self, parameters: List[torch.Tensor], gradients: List[torch.Tensor], rate: float) -> None:
        self.h.gr_clip_gradients(gradients, self.max_norm, self.norm)
        for p, g in zip(parameters, gradients):
            p.add_(g, alpha=-rate)

    def train_experts(self, x: torch.Tensor, target: torch.Tensor, expert: torch.Tensor, rate: float,
                      out_dx: Optional[torch.Tensor] = None) -> torch.Tensor:
        """A step of the first phase: requests x with logarithms of lengths `target` [rows], each given to expert [rows] (int32; a request
        whose expert there is not is left out).  out_dx, as x: the gradient by the features, for what makes them.  Returns the loss."""
        T = x.shape[0]
        off, slot, h = self.off, self.slot[:T], self.h
        pos = self.pos.view(-1)[:T].view(T, 1)
        h.gr_expert_plan(expert.view(T, 1), off, slot, pos)
        by_position = None if out_dx is None else torch.empty_like(out_dx)
        y = self._experts(x, T, 1)
        loss, d = self._loss(y, target[torch.where(slot < 0, -1 - slot, slot).long()], self.dy[-1][:T], counts=slot >= 0)
        for i in range(len(self.w) - 1, -1, -1):
            relu = i < len(self.w) - 1
            source = x if i == 0 else self.y[i - 1][:T]
            h.gr_expert_linear_backward(source, self.w[i], d, out_dx=self.dy[i - 1][:T] if i else by_position, out_dw=self.dw[i], out_db=self.db[i],
                                        y=self.y[i][:T] if relu else None, out_dz=d if relu else None, off=off,
                                        slot=slot if i == 0 else None)
            d = self.dy[i - 1][:T]
        if out_dx is not None:
            h.gr_expert_combine(by_position, pos, out_dx)
        self._update(self.w + self.b, self.dw + self.db, rate)
        return loss

    def train_router(self, x: torch.Tensor, target: torch.Tensor, rate: float) -> torch.Tensor:
        """A step of the second phase: the experts stay as they are.  Returns the loss."""
        T, h = x.shape[0], self.h
        loss, dout = self._loss(self.forward(x), target, self.out[:T])
        S = T * self.top_k
        h.gr_expert_combine_backward(dout, self.y[-1][:S], self.slot[:S], weight=self.weight[:T], out_dweight=self.dweight[:T])
        h.gr_expert_route_backward(self.router_y[1][:T], self.expert[:T], self.dweight[:T], self.dlogits[:T], renormalise=True)
        hidden, dhidden = self.router_y[0][:T], self.router_dy[:T]
        h.gr_expert_linear_backward(hidden, self.router_w[1], self.dlogits[:T], out_dx=dhidden, out_dw=self.router_dw[1], out_db=self.router_db[1])
        h.gr_expert_linear_backward(x, self.router_w[0], dhidden, out_dw=self.router_dw[0], out_db=self.router_db[0], y=hidden, out_dz=dhidden)
        self._update(self.router_w + self.router_b, self.router_dw + self.router_db, rate)
        return loss


def synthetic_requests(rows: int, n_in: int, n_kind: int, seed: int, dtype=torch.bfloat16, kinds_seed: int = 0):
    """Requests of n_kind kinds: features [rows, n_in] (a kind's own part stands out), logarithms of lengths [rows], kinds [rows].  A length hangs
    on its kind and, differently from kind to kind, on the features."""
    dev = torch.device("cuda", torch.cuda.current_device())
    of_kinds, g = torch.Generator(device=dev), torch.Generator(device=dev)
    of_kinds.manual_seed(kinds_seed)
    g.manual_seed(seed + 1)
    centre = torch.randn(n_kind, n_in, generator=of_kinds, device=dev)
    slope = torch.randn(n_kind, n_in, generator=of_kinds, device=dev) / n_in ** 0.5
    base = 3 + 4 * torch.rand(n_kind, generator=of_kinds, device=dev)
    kind = torch.randint(n_kind, (rows,), generator=g, device=dev)
    own = torch.randn(rows, n_in, generator=g, device=dev)
    x = (0.5 * centre[kind] + own).to(dtype)
    return x, base[kind] + 0.5 * (own * slope[kind]).sum(1), kind.to(torch.int32)


def main() -> None:
    from . import workloads
    n_in, rows = 512, 2048
    p = LengthPredictor(n_in, hidden=(256, 128, 64), router_hidden=128, max_rows=8192)
    print(f"{p.parameters() / 1e6:.1f} M parameters")
    for phase, rate in (("experts", 0.05), ("router", 0.2)):
        for step in range(150):
            x, target, kind = synthetic_requests(rows, n_in, p.n_expert, seed=step)
            loss = p.train_experts(x, target, kind, rate) if phase == "experts" else p.train_router(x, target, rate)
            if step % 50 == 0 or step == 149:
                print(f"{phase} step {step}: mean squared error of the logarithm {float(loss):.3f}, gradient norm {float(p.norm):.2f}", flush=True)
    # the arrivals of a fleet, routed by what is predicted of them
    fl = workloads.make_fleet(workloads.spec("mid"))
    up = lambda a: torch.from_numpy(a).to(p.dev)
    h = binding.Fleet(*(fl.coef[k] for k in ("delta", "alpha", "beta", "gamma")), fl.inst_class, fl.spec.n_active + fl.spec.n_queued,
                      int(fl.spec.max_len), len(fl.in_prompt))
    finish = torch.empty(len(fl.act_prompt), dtype=torch.float32, device=p.dev)
    h.gr_build_status(*(up(a) for a in (fl.act_off, fl.act_prompt, fl.act_gen, fl.act_rem, fl.q_off, fl.q_prompt, fl.q_len)), finish)
    x, target, _ = synthetic_requests(len(fl.in_prompt), n_in, p.n_expert, seed=10_000)
    length = p.predict(x, int(fl.spec.max_len))
    inst, slack = torch.empty_like(length), torch.empty(len(length), dtype=torch.float32, device=p.dev)
    h.gr_score_route(up(fl.in_prompt), length, up(fl.in_budget), inst, slack)
    off = (length.float().log() - target).abs().mean()
    print(f"{len(length)} arrivals: lengths off by a factor of {float(off.exp()):.2f} on average, sent to {int(inst.unique().numel())} instances, "
          f"{float((slack >= 0).float().mean()):.0%} expected in time")


if __name__ == "__main__":
    main()
