"""Binding of libgoodroute: same names as the C interface, argument
marshalling only (natively, by csrc/marshal.cpp, for the calls of a serving loop and those of a length
predictor; by ctypes for the others, and for all of them where that module is not built or is of another
torch: 7 to 9 us a call).  `Fleet` has the calls on a fleet, `Experts` those of a length predictor, `Tokens`
those that read a request's tokens.
Tensors are torch tensors on the GPU (device memory and the current stream come from torch; every step
of the path runs in the library's kernels).  There is no fallback for those: without the built library every call raises.
"""
from __future__ import annotations

import ctypes as C
import operator
import os
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "csrc", "libgoodroute.so")
MARSHAL_PATH = os.path.join(_HERE, "csrc", "goodroute_marshal.so")

EXPORTS = ("gr_create", "gr_destroy", "gr_build_status", "gr_score_route", "gr_score_route_noalloc", "gr_score_route_cached", "gr_route_feedback",
           "gr_risk_scan", "gr_observe", "gr_set_blend", "gr_set_batch_cap", "gr_set_small_batch_pairs", "gr_set_feedback_wait", "gr_set_feedback_units", "gr_set_feedback_team", "gr_feedback_team",
           "gr_device_status", "gr_strerror", "gr_profile_enable", "gr_profile_select", "gr_profile_read",
           "gr_profile_read_launches", "gr_profile_kernel_count", "gr_profile_kernel_name",
           "gr_experts_create", "gr_experts_destroy", "gr_expert_route", "gr_expert_route_backward", "gr_expert_plan",
           "gr_expert_linear", "gr_expert_linear_backward", "gr_expert_combine", "gr_expert_combine_backward",
           "gr_clip_gradients",
           "gr_tokens_create", "gr_tokens_destroy", "gr_token_embed", "gr_token_embed_backward", "gr_gated_scan", "gr_gated_scan_backward",
           "gr_dropout")

_lib = None
_marshal = None


class GoodRouteError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} ({code})")


def lib() -> C.CDLL:
    """Load libgoodroute.so (built by paper_2605_16867_amd.build / __graft_entry__.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2605_16867_amd.build`")
        l = C.CDLL(LIB_PATH)
        p, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        l.gr_create.restype = C.c_int
        l.gr_create.argtypes = [C.POINTER(p), i32, i32, p, p, p, p, p, i32, i32, i64]
        l.gr_destroy.restype = C.c_int
        l.gr_destroy.argtypes = [p]
        l.gr_build_status.restype = C.c_int
        l.gr_build_status.argtypes = [p, p, p, p, p, i64, p, p, p, i64, p, p, p, p, p]
        l.gr_score_route.restype = C.c_int
        l.gr_score_route.argtypes = [p, i64, p, p, p, p, p, p, p, p, p]
        l.gr_score_route_noalloc.restype = C.c_int
        l.gr_score_route_noalloc.argtypes = [p, i64, p, p, p, p, p, p, p, p]
        l.gr_score_route_cached.restype = C.c_int
        l.gr_score_route_cached.argtypes = [p, i64, p, p, p, p, p, p, p, i64, p, p, p, p, p]
        l.gr_route_feedback.restype = C.c_int
        l.gr_route_feedback.argtypes = [p, i64, i64, p, p, p, p, p, p, p, p]
        l.gr_risk_scan.restype = C.c_int
        l.gr_risk_scan.argtypes = [p, p, p, p, p, i64, p, p, p, i64, p, p, p, p, p, p, p]
        l.gr_observe.restype = C.c_int
        l.gr_observe.argtypes = [p, C.c_double, p, p, p, p]
        l.gr_set_blend.restype = C.c_int
        l.gr_set_blend.argtypes = [p, C.c_double]
        l.gr_set_small_batch_pairs.restype = C.c_int
        l.gr_set_small_batch_pairs.argtypes = [p, C.c_int64]
        l.gr_set_feedback_wait.restype = C.c_int
        l.gr_set_feedback_wait.argtypes = [p, i32]
        l.gr_set_feedback_units.restype = C.c_int
        l.gr_set_feedback_units.argtypes = [p, i32]
        l.gr_set_feedback_team.restype = C.c_int
        l.gr_set_feedback_team.argtypes = [p, i32]
        l.gr_feedback_team.restype = C.c_int
        l.gr_feedback_team.argtypes = [p, C.POINTER(i32)]
        l.gr_set_batch_cap.restype = C.c_int
        l.gr_set_batch_cap.argtypes = [p, p]
        l.gr_device_status.restype = C.c_int
        l.gr_device_status.argtypes = [p, C.POINTER(i32)]
        l.gr_profile_enable.restype = C.c_int
        l.gr_profile_enable.argtypes = [p, i32]
        l.gr_profile_select.restype = C.c_int
        l.gr_profile_select.argtypes = [p, C.c_uint64]
        l.gr_profile_read.restype = C.c_int
        l.gr_profile_read.argtypes = [p, i32, p, p]
        l.gr_profile_read_launches.restype = C.c_int
        l.gr_profile_read_launches.argtypes = [p, i32, p, p, p]
        l.gr_profile_kernel_count.restype = i32
        l.gr_profile_kernel_count.argtypes = []
        l.gr_profile_kernel_name.restype = C.c_char_p
        l.gr_profile_kernel_name.argtypes = [i32]
        f32 = C.c_float
        for name, args in {
                "gr_experts_create": [C.POINTER(p), i32, i64, i32], "gr_experts_destroy": [p],
                "gr_expert_route": [p, i64, i32, p, i32, p, i32, i32, i32, i32, f32, p, p, p, p, p, p],
                "gr_expert_route_backward": [p, i64, i32, p, i32, i32, i32, f32, p, p, p, p],
                "gr_expert_plan": [p, i64, i32, p, p, p, p, p],
                "gr_expert_linear": [p, i64, i32, i32, i32, p, p, i32, p, p, p, i32, p, p],
                "gr_expert_linear_backward": [p, i64, i32, i32, i32, p, p, i32, p, p, p, p, p, p, p, p, p],
                "gr_expert_combine": [p, i64, i32, i32, i32, p, p, p, p, p],
                "gr_expert_combine_backward": [p, i64, i32, i32, i32, p, p, p, p, p, p, p],
                "gr_clip_gradients": [p, i32, p, p, p, p, f32, p, p],
                "gr_tokens_create": [C.POINTER(p), i64, i32, i32], "gr_tokens_destroy": [p],
                "gr_token_embed": [p, i64, i32, i32, i32, p, p, f32, p, p],
                "gr_token_embed_backward": [p, i64, i32, i32, i32, p, p, f32, p, p],
                "gr_gated_scan": [p, i64, i64, i32, i32, p, p, i64, p, i64, p, p, p, p],
                "gr_gated_scan_backward": [p, i64, i64, i32, i32, p, p, i64, p, i64, p, p, p, p, p, i64, p, i64, p, p],
                "gr_dropout": [p, i64, i32, p, p, C.c_double, C.c_uint64, C.c_uint64, p, p, p]}.items():
            getattr(l, name).restype, getattr(l, name).argtypes = C.c_int, args
        l.gr_strerror.restype = C.c_char_p
        l.gr_strerror.argtypes = [C.c_int]
        _lib = l
    return _lib


def marshal():
    """The marshalling of the serving calls, connected to the library's entry points: native, or by ctypes where the
    native module is not there."""
    global _marshal
    if _marshal is None:
        l = lib()
        try:
            _marshal = _native(l)
        except ImportError as e:
            import warnings
            warnings.warn(f"arguments are marshalled by ctypes: {e}", RuntimeWarning, stacklevel=2)
            _marshal = _Ctypes
    return _marshal


def _native(l):
    if not os.path.exists(MARSHAL_PATH):
        raise ImportError(f"{MARSHAL_PATH} is not built; run `python -m paper_2605_16867_amd.build`")
    import importlib.machinery
    import importlib.util

    import torch  # noqa: F401  (its libraries come first)
    loader = importlib.machinery.ExtensionFileLoader("goodroute_marshal", MARSHAL_PATH)
    m = importlib.util.module_from_spec(importlib.util.spec_from_loader("goodroute_marshal", loader))
    loader.exec_module(m)
    m.connect(_check_slowly, *[C.cast(getattr(l, n), C.c_void_p).value for n in (
        "gr_build_status", "gr_score_route", "gr_score_route_noalloc", "gr_score_route_cached", "gr_route_feedback",
        "gr_risk_scan", "gr_expert_route", "gr_expert_route_backward", "gr_expert_plan", "gr_expert_linear",
        "gr_expert_linear_backward", "gr_expert_combine", "gr_expert_combine_backward", "gr_clip_gradients",
        "gr_token_embed", "gr_token_embed_backward", "gr_gated_scan", "gr_gated_scan_backward", "gr_dropout")])
    return m


def _check_slowly(t, code, name, n):
    """What the native marshalling asks about a tensor that is not plainly right: its address, or an error."""
    import torch
    p = _dev(t, {"i": torch.int32, "f": torch.float32, "d": torch.float64, "B": torch.uint8}[code], name, n)
    return None if p is None else p.value


def strerror(code: int) -> str:
    return lib().gr_strerror(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != 0:
        raise GoodRouteError(code, where)


def _dev(t, dtype, name: str, n: Optional[int] = None):
    """Device pointer of a contiguous GPU tensor of the given dtype (None -> NULL)."""
    if t is None:
        return None
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name}: need a contiguous {dtype} GPU tensor, got {t.dtype} on {t.device}")
    if n is not None and t.numel() < n:
        raise ValueError(f"{name}: {t.numel()} elements, need {n}")
    return C.c_void_p(t.data_ptr())


def _stream():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


class _Ctypes:
    """The functions of csrc/marshal.cpp by ctypes: the same arguments, the same refusals."""

    @staticmethod
    def _lists(M, act_off, act_prompt, act_gen, act_rem, q_off, q_prompt, q_len, rem="act_rem"):
        import torch
        i32, na, nq = torch.int32, act_prompt.numel(), q_prompt.numel()
        return na, nq, (_dev(act_off, i32, "act_off", M + 1), _dev(act_prompt, i32, "act_prompt"),
                        _dev(act_gen, i32, "act_gen", na), _dev(act_rem, i32, rem, na), na,
                        _dev(q_off, i32, "q_off", M + 1), _dev(q_prompt, i32, "q_prompt"), _dev(q_len, i32, "q_len", nq), nq)

    @staticmethod
    def _requests(ctx0, pred_len, budget, exclude):
        import torch
        n = ctx0.numel()
        return n, (_dev(ctx0, torch.int32, "ctx0"), _dev(pred_len, torch.int32, "pred_len", n),
                   _dev(budget, torch.float32, "budget", n), _dev(exclude, torch.int32, "exclude_inst", n))

    @staticmethod
    def _choices(n, inst, slack, fallback):
        import torch
        return (_dev(inst, torch.int32, "out_inst", n), _dev(slack, torch.float32, "out_slack", n),
                _dev(fallback, torch.uint8, "out_fallback", n))

    @classmethod
    def build_status(cls, h, M, *args):
        import torch
        finish, q_finish, d, rank = args[7:]
        na, nq, lists = cls._lists(M, *args[:7])
        return lib().gr_build_status(h, *lists, _dev(finish, torch.float32, "out_act_finish", na),
                                     _dev(q_finish, torch.float32, "out_q_finish", nq), _dev(d, torch.float64, "out_d", M),
                                     _dev(rank, torch.int32, "out_rank", M), _stream())

    @classmethod
    def score_route(cls, h, M, ctx0, pred_len, budget, exclude, inst, slack, fallback, T):
        import torch
        n, requests = cls._requests(ctx0, pred_len, budget, exclude)
        return lib().gr_score_route(h, n, *requests, *cls._choices(n, inst, slack, fallback),
                                    _dev(T, torch.float32, "out_T", n * M), _stream())

    @classmethod
    def score_route_noalloc(cls, h, ctx0, pred_len, budget, exclude, inst, slack, fallback):
        n, requests = cls._requests(ctx0, pred_len, budget, exclude)
        return lib().gr_score_route_noalloc(h, n, *requests, *cls._choices(n, inst, slack, fallback), _stream())

    @classmethod
    def score_route_cached(cls, h, M, ctx0, pred_len, budget, exclude, off, hit_inst, hit_len, inst, slack, fallback, T):
        import torch
        i32, nh = torch.int32, hit_inst.numel()
        n, requests = cls._requests(ctx0, pred_len, budget, exclude)
        hits = (_dev(off, i32, "hit_off", n + 1), _dev(hit_inst, i32, "hit_inst"), _dev(hit_len, i32, "hit_len", nh), nh)
        return lib().gr_score_route_cached(h, n, *requests, *hits, *cls._choices(n, inst, slack, fallback),
                                           _dev(T, torch.float32, "out_T", n * M), _stream())

    @classmethod
    def route_feedback(cls, h, chunk, ctx0, pred_len, budget, exclude, inst, slack, fallback):
        n, requests = cls._requests(ctx0, pred_len, budget, exclude)
        return lib().gr_route_feedback(h, n, chunk, *requests, *cls._choices(n, inst, slack, fallback), _stream())

    @classmethod
    def risk_scan(cls, h, M, *args):
        import torch
        f32, i32 = torch.float32, torch.int32
        budget, flag, finish, target, slack, n_flagged = args[7:]
        na, nq, lists = cls._lists(M, *args[:7], rem="act_rem_refreshed")
        return lib().gr_risk_scan(h, *lists, _dev(budget, f32, "act_budget", na), _dev(flag, torch.uint8, "out_flag", na),
                                  _dev(finish, f32, "out_finish", na), _dev(target, i32, "out_target", na),
                                  _dev(slack, f32, "out_target_slack", na), _dev(n_flagged, i32, "out_n_flagged", 1), _stream())


class Fleet:
    """Owns a gr_fleet handle on the current device."""

    def __init__(self, delta, alpha, beta, gamma, inst_class, max_entries_per_inst: int,
                 max_len: int, max_requests: int):
        import numpy as np
        self._h, self._at = C.c_void_p(), None
        self._m = marshal()
        co = [np.ascontiguousarray(x, dtype=np.float64) for x in (delta, alpha, beta, gamma)]
        ic = np.ascontiguousarray(inst_class, dtype=np.int32)
        self.n_inst = int(ic.shape[0])
        _check(lib().gr_create(C.byref(self._h), self.n_inst, int(co[0].shape[0]),
                               *[c.ctypes.data_as(C.c_void_p) for c in co],
                               ic.ctypes.data_as(C.c_void_p), int(max_entries_per_inst),
                               int(max_len), int(max_requests)), "gr_create")
        self._at = self._h.value

    def close(self) -> None:
        if self._h:
            h, self._h, self._at = self._h, C.c_void_p(), None
            _check(lib().gr_destroy(h), "gr_destroy")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def gr_build_status(self, act_off, act_prompt, act_gen, act_rem, q_off, q_prompt, q_len,
                        out_act_finish, out_q_finish=None, out_d=None, out_rank=None) -> None:
        rc = self._m.build_status(self._at, self.n_inst, act_off, act_prompt, act_gen, act_rem, q_off, q_prompt, q_len,
                                  out_act_finish, out_q_finish, out_d, out_rank)
        if rc:
            _check(rc, "gr_build_status")

    def gr_score_route(self, ctx0, pred_len, budget, out_inst, out_slack, exclude_inst=None,
                       out_fallback=None, out_T=None) -> None:
        rc = self._m.score_route(self._at, self.n_inst, ctx0, pred_len, budget, exclude_inst, out_inst, out_slack,
                                 out_fallback, out_T)
        if rc:
            _check(rc, "gr_score_route")

    def gr_score_route_noalloc(self, ctx0, pred_len, budget, out_inst, out_slack, exclude_inst=None,
                               out_fallback=None) -> None:
        rc = self._m.score_route_noalloc(self._at, ctx0, pred_len, budget, exclude_inst, out_inst, out_slack, out_fallback)
        if rc:
            _check(rc, "gr_score_route_noalloc")

    def gr_score_route_cached(self, ctx0, pred_len, budget, hit_off, hit_inst, hit_len, out_inst, out_slack,
                              exclude_inst=None, out_fallback=None, out_T=None) -> None:
        rc = self._m.score_route_cached(self._at, self.n_inst, ctx0, pred_len, budget, exclude_inst, hit_off, hit_inst,
                                        hit_len, out_inst, out_slack, out_fallback, out_T)
        if rc:
            _check(rc, "gr_score_route_cached")

    def gr_route_feedback(self, chunk: int, ctx0, pred_len, budget, out_inst, out_slack, exclude_inst=None,
                          out_fallback=None) -> None:
        rc = self._m.route_feedback(self._at, int(chunk), ctx0, pred_len, budget, exclude_inst, out_inst, out_slack,
                                    out_fallback)
        if rc:
            _check(rc, "gr_route_feedback")

    def gr_risk_scan(self, act_off, act_prompt, act_gen, act_rem_refreshed, q_off, q_prompt, q_len,
                     act_budget, out_flag, out_finish, out_target, out_target_slack,
                     out_n_flagged=None) -> None:
        rc = self._m.risk_scan(self._at, self.n_inst, act_off, act_prompt, act_gen, act_rem_refreshed, q_off, q_prompt, q_len,
                               act_budget, out_flag, out_finish, out_target, out_target_slack, out_n_flagged)
        if rc:
            _check(rc, "gr_risk_scan")

    def gr_observe(self, weight: float, obs_wait=None, obs_prefill=None, obs_decode=None) -> None:
        import torch
        f32, M = torch.float32, self.n_inst
        _check(lib().gr_observe(self._h, float(weight), _dev(obs_wait, f32, "obs_wait", M),
                                _dev(obs_prefill, f32, "obs_prefill", M),
                                _dev(obs_decode, f32, "obs_decode", M), _stream()), "gr_observe")

    def gr_set_blend(self, black_box_weight: float) -> None:
        _check(lib().gr_set_blend(self._h, float(black_box_weight)), "gr_set_blend")

    def gr_set_feedback_wait(self, looks: int) -> None:
        _check(lib().gr_set_feedback_wait(self._h, int(looks)), "gr_set_feedback_wait")

    def gr_set_feedback_units(self, units: int) -> None:
        _check(lib().gr_set_feedback_units(self._h, int(units)), "gr_set_feedback_units")

    def gr_set_feedback_team(self, workgroups: int) -> None:
        _check(lib().gr_set_feedback_team(self._h, int(workgroups)), "gr_set_feedback_team")

    def gr_feedback_team(self) -> int:
        v = C.c_int32(0)
        _check(lib().gr_feedback_team(self._h, C.byref(v)), "gr_feedback_team")
        return v.value

    def gr_set_small_batch_pairs(self, max_pairs: int) -> None:
        _check(lib().gr_set_small_batch_pairs(self._h, int(max_pairs)), "gr_set_small_batch_pairs")

    def gr_set_batch_cap(self, cap) -> None:
        """cap: host int array of n_inst entries, or None to remove the caps."""
        import numpy as np
        if cap is None:
            _check(lib().gr_set_batch_cap(self._h, None), "gr_set_batch_cap")
            return
        c = np.ascontiguousarray(cap, dtype=np.int32)
        if c.shape != (self.n_inst,):
            raise ValueError(f"cap: need {self.n_inst} entries")
        _check(lib().gr_set_batch_cap(self._h, c.ctypes.data_as(C.c_void_p)), "gr_set_batch_cap")

    def gr_profile_enable(self, max_launches: int) -> None:
        _check(lib().gr_profile_enable(self._h, int(max_launches)), "gr_profile_enable")

    def gr_profile_select(self, names=None) -> None:
        """Time only the kernels whose name starts with one of `names` (None: all)."""
        n = int(lib().gr_profile_kernel_count())
        mask = 0
        for k in range(n):
            nm = lib().gr_profile_kernel_name(k).decode()
            if names is None or any(nm.startswith(x) for x in names):
                mask |= 1 << k
        _check(lib().gr_profile_select(self._h, mask), "gr_profile_select")

    def gr_profile_read(self) -> dict:
        """{kernel name: (total milliseconds, launches)} since the last read."""
        n = int(lib().gr_profile_kernel_count())
        ms = (C.c_double * n)()
        cnt = (C.c_int64 * n)()
        _check(lib().gr_profile_read(self._h, n, ms, cnt), "gr_profile_read")
        return {lib().gr_profile_kernel_name(k).decode(): (float(ms[k]), int(cnt[k])) for k in range(n)}

    def gr_profile_read_launches(self, max_launches: int) -> dict:
        """{kernel name: [milliseconds of each recorded launch, in launch order]} since the last read."""
        ids = (C.c_int32 * max(max_launches, 1))()
        ms = (C.c_float * max(max_launches, 1))()
        n = C.c_int32(0)
        _check(lib().gr_profile_read_launches(self._h, int(max_launches), ids, ms, C.byref(n)), "gr_profile_read_launches")
        out = {}
        for i in range(int(n.value)):
            out.setdefault(lib().gr_profile_kernel_name(ids[i]).decode(), []).append(float(ms[i]))
        return out

    def gr_device_status(self) -> int:
        bits = C.c_int32(0)
        _check(lib().gr_device_status(self._h, C.byref(bits)), "gr_device_status")
        return int(bits.value)


_SCORING = {"softmax": 0, "sigmoid": 1}


def _dtype(t, name: str) -> int:
    import torch
    code = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: need float32, bfloat16 or float16, got {t.dtype}")
    return code


def _done(code: int, where: str) -> None:
    if code:
        _check(code, where)


class _Unclear:
    """In the place of the native marshalling where that is not built: every call is for the binding to marshal."""

    def __getattr__(self, name):
        return lambda *args: None


_Unclear = _Unclear()


class _Workspace:
    """A handle of the library's on the current device, with its checks of tensors."""

    _destroy = None      # name of the entry point

    def _create(self, entry, *sizes):
        self._h, self._at = C.c_void_p(), None
        self._m = marshal()
        if self._m is _Ctypes:
            self._m = _Unclear
        _check(getattr(lib(), entry)(C.byref(self._h), *sizes), entry)
        import torch
        self._device = torch.cuda.current_device()
        self._at = (self._h.value, self._device)

    def close(self) -> None:
        if self._h:
            h, self._h, self._at = self._h, C.c_void_p(), None
            _check(getattr(lib(), self._destroy)(h), self._destroy)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _dev(self, t, dtype, name: str, n: Optional[int] = None):
        if t is not None and t.is_cuda and t.device.index != self._device:
            raise ValueError(f"{name}: on {t.device}, need the handle's device, cuda:{self._device}")
        return _dev(t, dtype, name, n)

    def _stream(self):
        import torch
        if torch.cuda.current_device() != self._device:
            raise ValueError(f"the current device is cuda:{torch.cuda.current_device()}, need the handle's, cuda:{self._device}")
        return _stream()

    @staticmethod
    def _shape(t, name, *shape):
        """A tensor's shape, as far as it is asked for (None: any)."""
        if t.dim() != len(shape) or any(w is not None and w != g for w, g in zip(shape, t.shape)):
            raise ValueError(f"{name}: shape {tuple(t.shape)}, need {tuple('any' if w is None else w for w in shape)}")
        return t.shape


class Experts(_Workspace):
    """Owns a gr_experts handle on the current device: the workspace of a length predictor's operators.

    Shapes are taken from the tensors: logits [rows, experts], choices and weights [rows, top_k], x [rows or positions, n_in], w [experts,
    n_out, n_in], y [positions, n_out]; all contiguous and on the handle's device, which has to be the current one; x, w and y of one type.
    Outputs are tensors of the caller's, and nothing is recorded for torch's automatic differentiation: a gradient is a call of its own."""

    _destroy = "gr_experts_destroy"

    def __init__(self, n_expert: int, max_rows: int, max_top_k: int):
        self.n_expert = int(n_expert)
        self._create("gr_experts_create", self.n_expert, int(max_rows), int(max_top_k))

    def _plan(self, n, off, slot, pos):
        import torch
        i32 = torch.int32
        return self._dev(off, i32, "out_off", self.n_expert + 1), self._dev(slot, i32, "out_slot", n), self._dev(pos, i32, "out_pos", n)

    def gr_expert_route(self, logits, out_weight, out_expert, out_off=None, out_slot=None, out_pos=None, bias=None,
                        scoring="softmax", n_group=1, n_group_kept=1, renormalise=False, scale=1.0) -> None:
        rc = self._m.expert_route(self._at, self.n_expert, logits, out_weight, out_expert, out_off, out_slot, out_pos, bias,
                                  _SCORING[scoring], n_group, n_group_kept, renormalise, scale)
        if rc is not None:
            return _done(rc, "gr_expert_route")
        import torch
        T, _ = self._shape(logits, "logits", None, self.n_expert)
        _, k = self._shape(out_expert, "out_expert", T, None)
        _check(lib().gr_expert_route(
            self._h, T, k, self._dev(logits, logits.dtype, "logits"), _dtype(logits, "logits"),
            self._dev(bias, torch.float32, "bias", self.n_expert), _SCORING[scoring], int(n_group), int(n_group_kept), int(renormalise),
            float(scale), self._dev(out_weight, torch.float32, "out_weight", T * k), self._dev(out_expert, torch.int32, "out_expert"),
            *self._plan(T * k, out_off, out_slot, out_pos), self._stream()), "gr_expert_route")

    def gr_expert_route_backward(self, logits, expert, dweight, out_dlogits, scoring="softmax", renormalise=False, scale=1.0) -> None:
        rc = self._m.expert_route_backward(self._at, self.n_expert, logits, expert, dweight, out_dlogits, _SCORING[scoring], renormalise,
                                           scale)
        if rc is not None:
            return _done(rc, "gr_expert_route_backward")
        import torch
        T, E = self._shape(logits, "logits", None, self.n_expert)
        _, k = self._shape(expert, "expert", T, None)
        _check(lib().gr_expert_route_backward(
            self._h, T, k, self._dev(logits, logits.dtype, "logits"), _dtype(logits, "logits"), _SCORING[scoring], int(renormalise),
            float(scale), self._dev(expert, torch.int32, "expert"), self._dev(dweight, torch.float32, "dweight", T * k),
            self._dev(out_dlogits, logits.dtype, "out_dlogits", T * E), self._stream()), "gr_expert_route_backward")

    def gr_expert_plan(self, expert, out_off, out_slot, out_pos) -> None:
        rc = self._m.expert_plan(self._at, self.n_expert, expert, out_off, out_slot, out_pos)
        if rc is not None:
            return _done(rc, "gr_expert_plan")
        import torch
        T, k = self._shape(expert, "expert", None, None)
        _check(lib().gr_expert_plan(self._h, T, k, self._dev(expert, torch.int32, "expert"), *self._plan(T * k, out_off, out_slot, out_pos),
                                    self._stream()), "gr_expert_plan")

    def _layer(self, x, w, off, slot, top_k, n):
        """Arguments that a layer's forward and backward share, from `off` to `w`, behind the sizes."""
        import torch
        E = 1 if off is None else self.n_expert
        _, O, I = self._shape(w, "w", E, None, None) if w.dim() == 3 or off is not None else (1, *self._shape(w, "w", None, None))
        self._shape(x, "x", n if slot is None else (n + top_k - 1) // top_k if top_k > 0 else None, I)
        i32 = torch.int32
        return E, I, O, (n, I, O, _dtype(x, "x"), self._dev(off, i32, "off", self.n_expert + 1), self._dev(slot, i32, "slot", n), int(top_k),
                         self._dev(x, x.dtype, "x"), self._dev(w, x.dtype, "w"))

    def gr_expert_linear(self, x, w, out_y, bias=None, off=None, slot=None, top_k=1, relu=False) -> None:
        rc = self._m.expert_linear(self._at, self.n_expert, x, w, out_y, bias, off, slot, top_k, relu)
        if rc is not None:
            return _done(rc, "gr_expert_linear")
        n, O = self._shape(out_y, "out_y", None, w.shape[-2])
        E, I, O, layer = self._layer(x, w, off, slot, int(top_k), n)
        _check(lib().gr_expert_linear(self._h, *layer, self._dev(bias, x.dtype, "bias", E * O), int(relu), self._dev(out_y, x.dtype, "out_y"),
                                      self._stream()), "gr_expert_linear")

    def gr_expert_linear_backward(self, x, w, dy, out_dx=None, out_dw=None, out_db=None, y=None, out_dz=None, off=None,
                                  slot=None, top_k=1) -> None:
        rc = self._m.expert_linear_backward(self._at, self.n_expert, x, w, dy, out_dx, out_dw, out_db, y, out_dz, off, slot, top_k)
        if rc is not None:
            return _done(rc, "gr_expert_linear_backward")
        n, O = self._shape(dy, "dy", None, w.shape[-2])
        E, I, O, layer = self._layer(x, w, off, slot, int(top_k), n)
        t = x.dtype
        _check(lib().gr_expert_linear_backward(
            self._h, *layer, self._dev(y, t, "y", n * O), self._dev(dy, t, "dy"), self._dev(out_dz, t, "out_dz", n * O),
            self._dev(out_dx, t, "out_dx", n * I), self._dev(out_dw, t, "out_dw", E * O * I), self._dev(out_db, t, "out_db", E * O), self._stream()),
            "gr_expert_linear_backward")

    def gr_expert_combine(self, y, pos, out, weight=None) -> None:
        rc = self._m.expert_combine(self._at, y, pos, out, weight)
        if rc is not None:
            return _done(rc, "gr_expert_combine")
        import torch
        T, k = self._shape(pos, "pos", None, None)
        _, O = self._shape(out, "out", T, None)
        _check(lib().gr_expert_combine(self._h, T, k, O, _dtype(out, "out"), self._dev(weight, torch.float32, "weight", T * k),
                                       self._dev(pos, torch.int32, "pos"), self._dev(y, out.dtype, "y", T * k * O), self._dev(out, out.dtype, "out"),
                                       self._stream()), "gr_expert_combine")

    def gr_expert_combine_backward(self, dout, y, slot, out_dy=None, weight=None, out_dweight=None) -> None:
        rc = self._m.expert_combine_backward(self._at, dout, y, slot, out_dy, weight, out_dweight)
        if rc is not None:
            return _done(rc, "gr_expert_combine_backward")
        import torch
        T, O = self._shape(dout, "dout", None, None)
        if T and slot.numel() % T:
            raise ValueError(f"slot: {slot.numel()} elements, need a multiple of {T}")
        S = slot.numel()
        t, f32 = dout.dtype, torch.float32
        _check(lib().gr_expert_combine_backward(
            self._h, T, S // T if T else 1, O, _dtype(dout, "dout"), self._dev(weight, f32, "weight", S), self._dev(slot, torch.int32, "slot"),
            self._dev(y, t, "y", S * O), self._dev(dout, t, "dout"), self._dev(out_dy, t, "out_dy", S * O),
            self._dev(out_dweight, f32, "out_dweight", S), self._stream()), "gr_expert_combine_backward")

    def gr_clip_gradients(self, grads, max_norm, out_norm=None, out=None) -> None:
        """grads: a list of tensors, scaled in place unless `out` names as many others."""
        rc = self._m.clip_gradients(self._at, grads, max_norm, out_norm, grads if out is None else out)
        if rc is not None:
            return _done(rc, "gr_clip_gradients")
        import torch
        out = grads if out is None else out
        n = len(grads)
        if len(out) != n:
            raise ValueError(f"out: {len(out)} tensors, need {n}")
        _check(lib().gr_clip_gradients(
            self._h, n, (C.c_void_p * n)(*[self._dev(g, g.dtype, "grads") for g in grads]),
            (C.c_void_p * n)(*[self._dev(o, g.dtype, "out", g.numel()) for o, g in zip(out, grads)]),
            (C.c_int64 * n)(*[g.numel() for g in grads]), (C.c_int32 * n)(*[_dtype(g, "grads") for g in grads]),
            float(max_norm), self._dev(out_norm, torch.float32, "out_norm", 1), self._stream()), "gr_clip_gradients")


class Tokens(_Workspace):
    """Owns a gr_tokens handle on the current device: the workspace of the operators that read a request's tokens.

    Shapes are taken from the tensors: token [tokens], table [vocab, width], out, gate, x, y [tokens, width], off [sequences + 1], states h
    [sequences, width]; tokens and offsets int32, states float32, all others of one type; all on the handle's device, which has to be the
    current one.  gate, x and their gradients may be rows of something wider (a distance from row to row of at least their width); everything else is
    contiguous.  Outputs are tensors of the caller's, and nothing is recorded for torch's automatic differentiation: a gradient is a call of its own."""

    _destroy = "gr_tokens_destroy"

    def __init__(self, max_tokens: int, max_vocab: int, max_width: int):
        self._create("gr_tokens_create", int(max_tokens), int(max_vocab), int(max_width))

    def _rows(self, t, dtype, name: str, n: int, width: int):
        """Address and distance of rows that need not be next to each other."""
        self._shape(t, name, n, width)
        if not t.is_cuda or t.dtype != dtype or (width > 1 and t.numel() and t.stride(1) != 1):
            raise TypeError(f"{name}: need a {dtype} GPU tensor of contiguous rows, got {t.dtype} on {t.device}")
        stride = t.stride(0) if n > 1 else width
        if stride < width:
            raise ValueError(f"{name}: rows {stride} elements apart, need {width}")
        return self._dev(t[:1], dtype, name) if n else None, stride

    def gr_token_embed(self, token, table, out, scale=1.0) -> None:
        rc = self._m.token_embed(self._at, token, table, out, scale)
        if rc is not None:
            return _done(rc, "gr_token_embed")
        import torch
        V, W = self._shape(table, "table", None, None)
        n, = self._shape(token, "token", None)
        self._shape(out, "out", n, W)
        _check(lib().gr_token_embed(self._h, n, V, W, _dtype(table, "table"), self._dev(token, torch.int32, "token"),
                                    self._dev(table, table.dtype, "table"), float(scale), self._dev(out, table.dtype, "out"), self._stream()),
               "gr_token_embed")

    def gr_token_embed_backward(self, token, dout, out_dtable, scale=1.0) -> None:
        rc = self._m.token_embed_backward(self._at, token, dout, out_dtable, scale)
        if rc is not None:
            return _done(rc, "gr_token_embed_backward")
        import torch
        V, W = self._shape(out_dtable, "out_dtable", None, None)
        n, = self._shape(token, "token", None)
        self._shape(dout, "dout", n, W)
        _check(lib().gr_token_embed_backward(
            self._h, n, V, W, _dtype(dout, "dout"), self._dev(token, torch.int32, "token"), self._dev(dout, dout.dtype, "dout"), float(scale),
            self._dev(out_dtable, dout.dtype, "out_dtable"), self._stream()), "gr_token_embed_backward")

    def _sequences(self, gate, off, states, name):
        """Tokens, sequences and width; the sequences are those of `off`, without it the tokens."""
        import torch
        n, W = self._shape(gate, "gate", None, None)
        S = n
        if off is not None:
            S = self._shape(off, "off", None)[0] - 1
            if S < 0:
                raise ValueError("off: 0 elements, need one at least")
        for t, what in zip(states, name):
            if t is not None:
                self._shape(t, what, S, W)
        return n, S, W, self._dev(off, torch.int32, "off")

    def gr_gated_scan(self, gate, x, out_y=None, off=None, h0=None, out_h=None) -> None:
        rc = self._m.gated_scan(self._at, gate, x, out_y, off, h0, out_h)
        if rc is not None:
            return _done(rc, "gr_gated_scan")
        import torch
        f32, t = torch.float32, gate.dtype
        n, S, W, off = self._sequences(gate, off, (h0, out_h), ("h0", "out_h"))
        if out_y is not None:
            self._shape(out_y, "out_y", n, W)
        _check(lib().gr_gated_scan(
            self._h, n, S, W, _dtype(gate, "gate"), off, *self._rows(gate, t, "gate", n, W), *self._rows(x, t, "x", n, W),
            self._dev(h0, f32, "h0"), self._dev(out_y, t, "out_y"), self._dev(out_h, f32, "out_h"), self._stream()), "gr_gated_scan")

    def gr_gated_scan_backward(self, gate, x, y, out_dgate, out_dx, off=None, h0=None, dy=None, dh=None, out_dh0=None) -> None:
        rc = self._m.gated_scan_backward(self._at, gate, x, y, out_dgate, out_dx, off, h0, dy, dh, out_dh0)
        if rc is not None:
            return _done(rc, "gr_gated_scan_backward")
        import torch
        f32, t = torch.float32, gate.dtype
        n, S, W, off = self._sequences(gate, off, (h0, dh, out_dh0), ("h0", "dh", "out_dh0"))
        for v, name in ((y, "y"), (dy, "dy")):
            if v is not None:
                self._shape(v, name, n, W)
        _check(lib().gr_gated_scan_backward(
            self._h, n, S, W, _dtype(gate, "gate"), off, *self._rows(gate, t, "gate", n, W), *self._rows(x, t, "x", n, W),
            self._dev(y, t, "y"), self._dev(h0, f32, "h0"), self._dev(dy, t, "dy"), self._dev(dh, f32, "dh"),
            *self._rows(out_dgate, t, "out_dgate", n, W), *self._rows(out_dx, t, "out_dx", n, W), self._dev(out_dh0, f32, "out_dh0"),
            self._stream()), "gr_gated_scan_backward")

    def gr_dropout(self, x, out, rate, seed, offset=0, residual=None, offset_add=None) -> None:
        """seed, offset: in [0, 2^64); offset_add: an int64 tensor of one element, whose bits are added to offset when the kernel runs."""
        rc = self._m.dropout(self._at, x, out, rate, seed, offset, residual, offset_add)
        if rc is not None:
            return _done(rc, "gr_dropout")
        import torch
        n, t = x.numel(), x.dtype
        for v, name in ((out, "out"), (residual, "residual")):
            if v is not None:
                self._shape(v, name, *x.shape)
        for v, name in ((seed, "seed"), (offset, "offset")):
            if not 0 <= operator.index(v) < 1 << 64:
                raise ValueError(f"{name}: {v}, need 64 bits without a sign")
        _check(lib().gr_dropout(self._h, n, _dtype(x, "x"), self._dev(x, t, "x"), self._dev(residual, t, "residual"), float(rate), int(seed),
                                int(offset), self._dev(offset_add, torch.int64, "offset_add", 1), self._dev(out, t, "out"), self._stream()),
               "gr_dropout")
