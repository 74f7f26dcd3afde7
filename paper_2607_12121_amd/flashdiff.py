"""Python binding of libflashdiff.so (the region-sparse DiT step's C ABI).

Argument marshalling only: every function below passes device pointers, sizes
and torch's current HIP stream to the C entry point of the same name; all
computation runs in the library's HIP kernels.  torch provides device memory
and streams.  If the library is missing this module raises on import of the
library (there is no fallback path).
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass
from typing import Dict, Optional, Sequence

import numpy as np
import torch

LIB_PATH = os.environ.get("FLASHDIFF_LIB") or os.path.join(os.path.dirname(os.path.abspath(__file__)),
                                                            "libflashdiff.so")

FD_SKIP_FREEZE = 0
FD_SKIP_REUSE_DRIFT = 1

KERNELS = {"score": 1, "select": 2, "gather": 3, "embed": 4, "adaln": 5, "ln": 6, "gemm_qkv": 7,
           "attn": 8, "gemm_o": 9, "gemm_mlp1": 10, "gemm_mlp2": 11, "final": 12, "scatter": 13,
           "importance": 14, "partition": 15, "quant": 16, "rms": 17, "rope": 18, "linear": 19,
           "int_rows": 20, "int_linear": 21, "norm_residual": 22, "cache_write": 23, "cache_attn": 24}

_p = ctypes.c_void_p
_i32 = ctypes.c_int32


class FdPlan(ctypes.Structure):
    _fields_ = [("n_tokens", _i32), ("n_regions", _i32), ("n_requests", _i32),
                ("max_region_tokens", _i32), ("max_request_tokens", _i32),
                ("region_ptr", _p), ("region_tokens", _p), ("region_req", _p),
                ("token_region", _p), ("req_tok_off", _p), ("req_reg_off", _p)]


class FdDims(ctypes.Structure):
    _fields_ = [("C", _i32), ("D", _i32), ("H", _i32), ("dh", _i32), ("F", _i32)]


class FdBlockWeights(ctypes.Structure):
    _fields_ = [(n, _p) for n in ("w_qkv", "b_qkv", "w_o", "b_o", "w_1", "b_1", "w_2", "b_2",
                                  "w_ada", "b_ada", "mod")]


class FdFinalWeights(ctypes.Structure):
    _fields_ = [(n, _p) for n in ("w_ada", "b_ada", "w_out", "b_out")]


class FdGate(ctypes.Structure):
    _fields_ = [("eta", ctypes.c_double), ("max_skip", _i32)]


_Axes, _Reals = _i32 * 4, ctypes.c_double * 4


class FdRope(ctypes.Structure):
    _fields_ = [("n_axes", _i32), ("pairing", _i32), ("dim", _Axes), ("theta", _Reals), ("step", _Reals)]


class FdScaledWeights(ctypes.Structure):
    _fields_ = [(n, _p) for n in ("w_qkv", "s_qkv", "b_qkv", "w_o", "s_o", "b_o", "w_1", "s_1", "b_1", "w_2", "s_2", "b_2",
                                  "norm_1", "norm_2", "mod")]


class FlashDiffError(RuntimeError):
    pass


_lib: Optional[ctypes.CDLL] = None


def lib() -> ctypes.CDLL:
    """Load libflashdiff.so (built by paper_2607_12121_amd.build); raise if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FlashDiffError(f"{LIB_PATH} is missing: build it with `python -m paper_2607_12121_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    P = ctypes.POINTER
    sig = {
        "fd_last_error": ([], ctypes.c_char_p),
        "fd_version": ([], ctypes.c_char_p),
        "fd_plan_build": ([_i32, _i32, _i32, _p, _p, _p, _p, _p, _p, _p, _p], _i32),
        "fd_region_score_ws_size": ([P(FdPlan), _i32], ctypes.c_size_t),
        "fd_region_score": ([P(FdPlan), _i32, _p, _p, _p, _p, ctypes.c_size_t, _p], _i32),
        "fd_region_score_noalloc": ([P(FdPlan), _i32, _p, _p, _p, _p], _i32),
        "fd_select": ([P(FdPlan), _p, _p, FdGate, _p, _p, _p, _p, _p, _p, _p, _p], _i32),
        "fd_gather": ([P(FdPlan), _i32, _p, _p, _p, _p, _p], _i32),
        "fd_embed": ([P(FdPlan), P(FdDims), _p, _p, _p, _p, _p, _p, _p, _p], _i32),
        "fd_adaln": ([P(FdDims), _i32, _i32, _i32, _p, _p, _p, _p, _p], _i32),
        "fd_block_ws_size": ([P(FdPlan), P(FdDims)], ctypes.c_size_t),
        "fd_block_forward": ([P(FdPlan), P(FdDims), P(FdBlockWeights), _p, _p, _p, _p, _p, _p, _p, _p,
                              ctypes.c_size_t, _p], _i32),
        "fd_final": ([P(FdPlan), P(FdDims), P(FdFinalWeights), _p, _p, _p, _p, _p, _p, ctypes.c_size_t, _p],
                     _i32),
        "fd_scatter_update": ([P(FdPlan), _i32, _p, _p, _p, _p, _p, _p, _p, _i32, _p], _i32),
        "fd_importance_ws_size": ([P(FdPlan), P(FdDims)], ctypes.c_size_t),
        "fd_region_importance": ([P(FdPlan), P(FdDims), _p, ctypes.c_size_t, _p, _p, _p, _p, _p, _p, _p, _p,
                                  ctypes.c_size_t, _p], _i32),
        "fd_partition_ws_size": ([_i32, _i32], ctypes.c_size_t),
        "fd_partition": ([_i32, _p, _p, _p, _p, _p, ctypes.c_size_t, _p], _i32),
        "fd_scale_stride": ([_i32], _i32),
        "fd_quant_blocks": ([_i32, _i32, _i32, _p, _p, _p, _p, _p], _i32),
        "fd_rms_quant": ([_i32, _i32, _i32, _p, _p, _p, _p, _p, _p, _i32, ctypes.c_float, _p, _p, _p, _p, _p], _i32),
        "fd_rope_axes": ([_i32, _i32, P(FdRope), _i32, _i32, _i32, _p, _p, _p, _p, _p, _p, _p, _p], _i32),
        "fd_scaled_linear": ([_i32, _i32, _i32, _p, _p, _p, _p, _p, _i32, _p, _p, _p, _p, _p, _p], _i32),
        "fd_scaled_block_ws_size": ([P(FdPlan), P(FdDims)], ctypes.c_size_t),
        "fd_scaled_block_forward": ([P(FdPlan), P(FdDims), P(FdScaledWeights), P(FdRope), _p, _p, _p, _p, _p, _p, _p, _p,
                                     ctypes.c_size_t, _p], _i32),
        "fd_int_rows": ([_i32, _i32, _p, _p, _p, _p, _p], _i32),
        "fd_int_linear": ([_i32, _i32, _i32, _p, _p, _p, _p, _p, _i32, _p, _p, _p, _p], _i32),
        "fd_norm_residual": ([_i32, _i32, _i32, _p, _p, ctypes.c_float, _p, _p, _p, _p, _p, _i32, ctypes.c_float, _p, _p, _p, _p, _p,
                              _p, _p, _p], _i32),
        "fd_cache_write": ([_i32, _i32, P(FdRope), _i32, _i32, _i32, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p], _i32),
        "fd_cache_attention_ws_size": ([_i32, _i32, _i32, _i32], ctypes.c_size_t),
        "fd_cache_attention": ([_i32, _i32, _i32, _i32, _i32, _i32, _i32, ctypes.c_float, _p, _p, _p, _p, _p, _p, _p, _p, _p,
                                ctypes.c_size_t, _p], _i32),
        "fd_timer_arm": ([_i32, _i32], _i32),
        "fd_timer_read": ([_p, _i32], _i32),
        "fd_timer_disarm": ([], None),
    }
    for name, (args, res) in sig.items():
        f = getattr(L, name)
        f.argtypes = args
        f.restype = res
    _lib = L
    return L


def exported_symbols() -> Sequence[str]:
    return ("fd_last_error", "fd_version", "fd_plan_build", "fd_region_score_ws_size", "fd_region_score",
            "fd_region_score_noalloc",
            "fd_select", "fd_gather", "fd_embed", "fd_adaln", "fd_block_ws_size", "fd_block_forward", "fd_final",
            "fd_scatter_update", "fd_importance_ws_size", "fd_region_importance", "fd_partition_ws_size",
            "fd_partition", "fd_scale_stride", "fd_quant_blocks", "fd_rms_quant", "fd_rope_axes", "fd_scaled_linear",
            "fd_scaled_block_ws_size", "fd_scaled_block_forward", "fd_int_rows", "fd_int_linear", "fd_norm_residual",
            "fd_cache_write", "fd_cache_attention_ws_size", "fd_cache_attention", "fd_timer_arm", "fd_timer_read", "fd_timer_disarm")


def _check(name: str, status: int) -> None:
    if status != 0:
        msg = lib().fd_last_error().decode(errors="replace")
        raise FlashDiffError(f"{name} failed with status {status}: {msg}")


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_contiguous():
        raise FlashDiffError("tensor arguments must be contiguous")
    return t.data_ptr()


_DT = {"f32": (torch.float32,), "f64": (torch.float64,), "i32": (torch.int32,), "u8": (torch.uint8,),
       "b16": (torch.bfloat16, torch.int16, torch.uint16), "bytes": None,
       "code": (torch.float8_e4m3fn, torch.uint8), "scale": (torch.uint8, torch.float8_e8m0fnu), "i8": (torch.int8,)}


def _need(name: str, t: Optional[torch.Tensor], kind: str, numel: int, exact: bool = False,
          optional: bool = False) -> None:
    """Host-side check of one tensor argument before its pointer reaches the library:
    on a GPU, contiguous, of the element type the C entry point reads (`kind`;
    "b16" = any 2-byte bf16 bit pattern, "bytes" = any type) and with at least
    (or, with exact=True, exactly) `numel` elements."""
    if t is None:
        if optional:
            return
        raise FlashDiffError(f"{name} is required")
    if not t.is_cuda:
        raise FlashDiffError(f"{name} must be a device tensor")
    allowed = _DT[kind]
    if allowed is not None and t.dtype not in allowed:
        raise FlashDiffError(f"{name} must be {kind}, got {t.dtype}")
    n = t.numel() if kind != "bytes" else t.numel() * t.element_size()
    if (n != numel) if exact else (n < numel):
        raise FlashDiffError(f"{name} holds {n} elements, needs {'exactly ' if exact else ''}{numel}")


def _stream(stream: Optional[torch.cuda.Stream] = None) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def version() -> str:
    return lib().fd_version().decode()


# ------------------------------------------------------------------ plan

@dataclass
class Plan:
    """Region plan uploaded to the device, with its C descriptor."""

    c: FdPlan
    tensors: Dict[str, torch.Tensor]
    host: Dict[str, np.ndarray]

    @property
    def n_tokens(self) -> int:
        return self.c.n_tokens

    @property
    def n_regions(self) -> int:
        return self.c.n_regions

    @property
    def n_requests(self) -> int:
        return self.c.n_requests


def fd_plan_build(token_region: np.ndarray, req_tok_off: np.ndarray, n_regions: int) -> Dict[str, np.ndarray]:
    """Host CSR plan (calls the C builder)."""
    tr = np.ascontiguousarray(token_region, dtype=np.int32)
    to = np.ascontiguousarray(req_tok_off, dtype=np.int32)
    N, B = len(tr), len(to) - 1
    out = {"region_ptr": np.zeros(n_regions + 1, np.int32), "region_tokens": np.zeros(N, np.int32),
           "region_req": np.zeros(n_regions, np.int32), "req_reg_off": np.zeros(B + 1, np.int32)}
    mx_r, mx_b = _i32(0), _i32(0)
    st = lib().fd_plan_build(N, n_regions, B, tr.ctypes.data, to.ctypes.data, out["region_ptr"].ctypes.data,
                             out["region_tokens"].ctypes.data, out["region_req"].ctypes.data,
                             out["req_reg_off"].ctypes.data, ctypes.addressof(mx_r), ctypes.addressof(mx_b))
    _check("fd_plan_build", st)
    out["token_region"] = tr
    out["req_tok_off"] = to
    out["max_region_tokens"] = np.int32(mx_r.value)
    out["max_request_tokens"] = np.int32(mx_b.value)
    return out


def make_plan(token_region: np.ndarray, req_tok_off: np.ndarray, n_regions: int, device="cuda") -> Plan:
    host = fd_plan_build(token_region, req_tok_off, n_regions)
    keys = ("region_ptr", "region_tokens", "region_req", "token_region", "req_tok_off", "req_reg_off")
    t = {k: torch.from_numpy(host[k]).to(device) for k in keys}
    c = FdPlan(len(host["token_region"]), n_regions, len(host["req_tok_off"]) - 1,
               int(host["max_region_tokens"]), int(host["max_request_tokens"]),
               *[t[k].data_ptr() for k in keys])
    return Plan(c, t, host)


def dims(C: int, D: int, H: int, dh: int, F: int) -> FdDims:
    return FdDims(C, D, H, dh, F)


# ------------------------------------------------------------------ entry points

def fd_region_score_ws_size(plan: Plan, C: int) -> int:
    return int(lib().fd_region_score_ws_size(ctypes.byref(plan.c), C))


def fd_region_score(plan: Plan, C: int, x_cur, x_prev, score, ws, stream=None) -> None:
    N, R = plan.n_tokens, plan.n_regions
    _need("x_cur", x_cur, "f32", N * C)
    _need("x_prev", x_prev, "f32", N * C)
    _need("score", score, "f64", R)
    _need("ws", ws, "bytes", fd_region_score_ws_size(plan, C))
    _check("fd_region_score", lib().fd_region_score(ctypes.byref(plan.c), C, _ptr(x_cur), _ptr(x_prev),
                                                    _ptr(score), _ptr(ws), ws.numel() * ws.element_size(),
                                                    _stream(stream)))


def fd_region_score_noalloc(plan: Plan, C: int, x_cur, x_prev, score, stream=None) -> None:
    """fd_region_score with the library's built-in scratch (no workspace argument)."""
    N, R = plan.n_tokens, plan.n_regions
    _need("x_cur", x_cur, "f32", N * C)
    _need("x_prev", x_prev, "f32", N * C)
    _need("score", score, "f64", R)
    _check("fd_region_score_noalloc", lib().fd_region_score_noalloc(ctypes.byref(plan.c), C, _ptr(x_cur), _ptr(x_prev),
                                                                    _ptr(score), _stream(stream)))


def fd_select(plan: Plan, score, eps, eta: float, max_skip: int, s_tilde, skip_run, prev_active, active,
              idx, cu_q, m, stream=None) -> None:
    N, R, B = plan.n_tokens, plan.n_regions, plan.n_requests
    for n_, t_, k_, c_ in (("score", score, "f64", R), ("eps", eps, "f64", B), ("s_tilde", s_tilde, "f64", R),
                           ("skip_run", skip_run, "i32", R), ("prev_active", prev_active, "u8", R),
                           ("active", active, "u8", R), ("idx", idx, "i32", N), ("cu_q", cu_q, "i32", B + 1),
                           ("m", m, "i32", 1)):
        _need(n_, t_, k_, c_)
    _check("fd_select", lib().fd_select(ctypes.byref(plan.c), _ptr(score), _ptr(eps), FdGate(eta, max_skip),
                                        _ptr(s_tilde), _ptr(skip_run), _ptr(prev_active), _ptr(active),
                                        _ptr(idx), _ptr(cu_q), _ptr(m), _stream(stream)))


def fd_gather(plan: Plan, C: int, x_cur, idx, m, xa, stream=None) -> None:
    N = plan.n_tokens
    _need("x_cur", x_cur, "f32", N * C)
    _need("idx", idx, "i32", N)
    _need("m", m, "i32", 1)
    _need("xa", xa, "b16", N * C)
    _check("fd_gather", lib().fd_gather(ctypes.byref(plan.c), C, _ptr(x_cur), _ptr(idx), _ptr(m), _ptr(xa),
                                        _stream(stream)))


def fd_embed(plan: Plan, d: FdDims, xa, w_e, b_e, pos, idx, m, h, stream=None) -> None:
    N = plan.n_tokens
    for n_, t_, k_, c_ in (("xa", xa, "b16", N * d.C), ("w_e", w_e, "b16", d.D * d.C), ("b_e", b_e, "f32", d.D),
                           ("pos", pos, "f32", N * d.D), ("idx", idx, "i32", N), ("m", m, "i32", 1),
                           ("h", h, "f32", N * d.D)):
        _need(n_, t_, k_, c_)
    _check("fd_embed", lib().fd_embed(ctypes.byref(plan.c), ctypes.byref(d), _ptr(xa), _ptr(w_e), _ptr(b_e),
                                      _ptr(pos), _ptr(idx), _ptr(m), _ptr(h), _stream(stream)))


def fd_block_ws_size(plan: Plan, d: FdDims) -> int:
    return int(lib().fd_block_ws_size(ctypes.byref(plan.c), ctypes.byref(d)))


def fd_adaln(d: FdDims, n_blocks: int, n_out: int, n_requests: int, w_ada, b_ada, cond, mod, stream=None) -> None:
    _need("w_ada", w_ada, "b16", n_blocks * n_out * d.D)
    _need("b_ada", b_ada, "f32", n_blocks * n_out)
    _need("cond", cond, "f32", n_requests * d.D)
    _need("mod", mod, "f32", n_blocks * n_requests * n_out)
    _check("fd_adaln", lib().fd_adaln(ctypes.byref(d), n_blocks, n_out, n_requests, _ptr(w_ada), _ptr(b_ada),
                                      _ptr(cond), _ptr(mod), _stream(stream)))


def block_weights(params: Dict[str, torch.Tensor], l: int, mod: Optional[torch.Tensor] = None) -> FdBlockWeights:
    """Weights of block l; `mod` ([B, 6D] fp32, from fd_adaln) replaces the block's own adaLN."""
    names = ("w_qkv", "b_qkv", "w_o", "b_o", "w_1", "b_1", "w_2", "b_2", "w_ada", "b_ada")
    return FdBlockWeights(*[_ptr(params[n][l]) for n in names], _ptr(mod))


def final_weights(params: Dict[str, torch.Tensor]) -> FdFinalWeights:
    return FdFinalWeights(_ptr(params["w_adaf"]), _ptr(params["b_adaf"]), _ptr(params["w_out"]),
                          _ptr(params["b_out"]))


def fd_block_forward(plan: Plan, d: FdDims, w: FdBlockWeights, cond, h, idx, cu_q, m, k_cache, v_cache, ws,
                     stream=None) -> None:
    N, B = plan.n_tokens, plan.n_requests
    _need("cond", cond, "f32", B * d.D, optional=bool(w.mod))
    for n_, t_, k_, c_ in (("h", h, "f32", N * d.D), ("idx", idx, "i32", N), ("cu_q", cu_q, "i32", B + 1),
                           ("m", m, "i32", 1), ("k_cache", k_cache, "b16", N * d.D),
                           ("v_cache", v_cache, "b16", N * d.D), ("ws", ws, "bytes", fd_block_ws_size(plan, d))):
        _need(n_, t_, k_, c_)
    _check("fd_block_forward", lib().fd_block_forward(
        ctypes.byref(plan.c), ctypes.byref(d), ctypes.byref(w), _ptr(cond), _ptr(h), _ptr(idx), _ptr(cu_q),
        _ptr(m), _ptr(k_cache), _ptr(v_cache), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def fd_final(plan: Plan, d: FdDims, w: FdFinalWeights, cond, h, cu_q, m, v, ws, stream=None) -> None:
    N, B = plan.n_tokens, plan.n_requests
    for n_, t_, k_, c_ in (("cond", cond, "f32", B * d.D), ("h", h, "f32", N * d.D), ("cu_q", cu_q, "i32", B + 1),
                           ("m", m, "i32", 1), ("v", v, "f32", N * d.C), ("ws", ws, "bytes", fd_block_ws_size(plan, d))):
        _need(n_, t_, k_, c_)
    _check("fd_final", lib().fd_final(ctypes.byref(plan.c), ctypes.byref(d), ctypes.byref(w), _ptr(cond), _ptr(h),
                                      _ptr(cu_q), _ptr(m), _ptr(v), _ptr(ws), ws.numel() * ws.element_size(),
                                      _stream(stream)))


def fd_scatter_update(plan: Plan, C: int, x, v, idx, m, dt, vcache, active, skip_mode: int, stream=None) -> None:
    N, R, B = plan.n_tokens, plan.n_regions, plan.n_requests
    for n_, t_, k_, c_ in (("x", x, "f32", N * C), ("v", v, "f32", N * C), ("idx", idx, "i32", 1), ("m", m, "i32", 1),
                           ("dt", dt, "f32", B), ("vcache", vcache, "f32", N * C), ("active", active, "u8", R)):
        _need(n_, t_, k_, c_)
    _check("fd_scatter_update", lib().fd_scatter_update(ctypes.byref(plan.c), C, _ptr(x), _ptr(v), _ptr(idx),
                                                        _ptr(m), _ptr(dt), _ptr(vcache), _ptr(active),
                                                        skip_mode, _stream(stream)))


def fd_importance_ws_size(plan: Plan, d: FdDims) -> int:
    return int(lib().fd_importance_ws_size(ctypes.byref(plan.c), ctypes.byref(d)))


def fd_region_importance(plan: Plan, d: FdDims, block_ws, k_cache, idx, m, active, r_bar, delta, importance, ws,
                         stream=None) -> None:
    N, R = plan.n_tokens, plan.n_regions
    for n_, t_, k_, c_ in (("block_ws", block_ws, "bytes", fd_block_ws_size(plan, d)),
                           ("k_cache", k_cache, "b16", N * d.D), ("idx", idx, "i32", N), ("m", m, "i32", 1),
                           ("active", active, "u8", R), ("r_bar", r_bar, "f64", R), ("delta", delta, "f64", R),
                           ("ws", ws, "bytes", fd_importance_ws_size(plan, d))):
        _need(n_, t_, k_, c_)
    _need("importance", importance, "f64", R, optional=True)
    _check("fd_region_importance", lib().fd_region_importance(
        ctypes.byref(plan.c), ctypes.byref(d), _ptr(block_ws), block_ws.numel() * block_ws.element_size(),
        _ptr(k_cache), _ptr(idx), _ptr(m), _ptr(active), _ptr(r_bar), _ptr(delta), _ptr(importance), _ptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)))


def fd_partition_ws_size(n_tokens: int, n_requests: int) -> int:
    return int(lib().fd_partition_ws_size(n_tokens, n_requests))


def fd_partition(req_tok_off, req_reg_off, saliency, token_region, ws, stream=None) -> None:
    """Patch partitioner.  req_tok_off, req_reg_off: host int sequences [B+1];
    saliency: device 2-byte tensor [N] holding uint16 values; token_region:
    device int32 [N] (output); ws: device bytes of fd_partition_ws_size(N, B)."""
    to = np.ascontiguousarray(req_tok_off, dtype=np.int32)
    ro = np.ascontiguousarray(req_reg_off, dtype=np.int32)
    if to.shape != ro.shape or to.ndim != 1 or len(to) < 2:
        raise FlashDiffError("req_tok_off and req_reg_off must both have B + 1 entries")
    if saliency.element_size() != 2 or token_region.dtype != torch.int32:
        raise FlashDiffError("saliency must hold 16-bit values and token_region int32")
    n = int(to[-1])
    _need("saliency", saliency, "bytes", 2 * n, exact=True)
    _need("token_region", token_region, "i32", n, exact=True)
    _need("ws", ws, "bytes", fd_partition_ws_size(n, len(to) - 1))
    _check("fd_partition", lib().fd_partition(len(to) - 1, to.ctypes.data, ro.ctypes.data, _ptr(saliency),
                                              _ptr(token_region), _ptr(ws), ws.numel() * ws.element_size(),
                                              _stream(stream)))


def partition(saliency: torch.Tensor, req_tok_off, req_reg_off, stream=None) -> torch.Tensor:
    """fd_partition with its output and workspace allocated here: the global
    region id of every token (device int32 [N])."""
    N, B = int(saliency.numel()), len(req_tok_off) - 1
    out = torch.empty(N, dtype=torch.int32, device=saliency.device)
    ws = torch.empty(max(fd_partition_ws_size(N, B), 256), dtype=torch.uint8, device=saliency.device)
    if stream is not None:
        # the buffers come from the current stream's pool and the saliency may still be
        # written there: the launch stream waits for that work, and both buffers are
        # marked as used on it (ws is freed here while the kernel may still run)
        stream.wait_stream(torch.cuda.current_stream())
    fd_partition(req_tok_off, req_reg_off, saliency, out, ws, stream)
    if stream is not None:
        ws.record_stream(stream)
        out.record_stream(stream)
    return out


# ------------------------------------------------------------------ 8-bit rows

def fd_scale_stride(cols: int) -> int:
    """Bytes of a row of block scales: ceil(cols / 128) rounded up to a multiple of 4."""
    return lib().fd_scale_stride(cols)


def _stride(cols: int) -> int:
    """fd_scale_stride without the call into the library (0.2 us)."""
    return (cols + 511) // 512 * 4


def _rows(name: str, t: Optional[torch.Tensor]) -> Sequence[int]:
    if t is None:
        raise FlashDiffError(f"{name} is required")
    s = t.shape
    if len(s) != 2 or s[0] > 1 << 30 or s[1] > 1 << 30:
        raise FlashDiffError(f"{name} must have two dimensions of at most 2^30, got {tuple(s)}")
    return s


_KIND = {k: frozenset(v) for k, v in _DT.items() if v is not None}


# The handle of a device's current stream: without the stream object that torch.cuda.current_stream builds (2.7 us) where
# this torch has that.
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _pointers(stream: Optional[torch.cuda.Stream], *args) -> list:
    """Checks (name, tensor, kind, elements) tuples as _need does, and that every tensor and the stream are on
    the current device, the one the call runs on; returns the tensors' addresses and the stream's handle.  One
    pass of cheap tests, as these calls take microseconds on the GPU; what fails is named by the slow path.
    An element count below 0 marks an optional tensor of minus that many elements."""
    cur, out, kinds = None, [], _KIND
    put = out.append
    for name, t, kind, n in args:
        if t is None:
            if n >= 0:
                raise FlashDiffError(f"{name} is required")
            put(None)
            continue
        if n < 0:
            n = -n
        if cur is None:
            if not t.is_cuda:
                _need(name, t, kind, n)
            cur = torch.cuda.current_device()
        if t.get_device() != cur or t.dtype not in kinds[kind] or t.numel() < n or not t.is_contiguous():
            _need(name, t, kind, n)
            if t.get_device() != cur:
                raise FlashDiffError(f"{name} is on {t.device}, the current device is {cur}")
            _ptr(t)
        put(t.data_ptr())
    if stream is None:
        out.append(_current_stream(cur))
    elif stream.device.index != cur:
        raise FlashDiffError(f"the stream is on {stream.device}, the current device is {cur}")
    else:
        out.append(stream.cuda_stream)
    return out


def fd_quant_blocks(x, block_rows: int, q, scale, m=None, stream=None) -> None:
    """bf16 x [rows, cols] to e4m3 codes q [rows, cols] and scale bytes
    [ceil(rows / block_rows), fd_scale_stride(cols)]; block_rows 1 (activations, `m` of
    the rows when given) or 128 (weights)."""
    rows, cols = _rows("x", x)
    p = _pointers(stream, ("x", x, "b16", rows * cols), ("m", m, "i32", -1), ("q", q, "code", rows * cols),
                  ("scale", scale, "scale", -(-rows // max(block_rows, 1)) * _stride(cols)))
    _check("fd_quant_blocks", lib().fd_quant_blocks(rows, cols, block_rows, *p))


def _modulation(h, B: int, D: int, *parts):
    """(row stride, addresses) of a request's gate, shift and scale: fp32 [B, D] on h's device, or None."""
    stride, mod = None, []
    for t in parts:
        if t is None:
            mod.append(None)
            continue
        steps = t.stride()
        if stride is None:
            stride, dev, want = steps[0], h.get_device(), (B, D)
        if t.shape != want or steps != (stride, 1) or stride > 1 << 30 or t.dtype is not torch.float32 or t.get_device() != dev:
            raise FlashDiffError(f"gate, shift and mod_scale must be fp32 [{B}, {D}] with contiguous rows of one stride, on {h.device}")
        mod.append(t.data_ptr())
    return stride or 0, mod


def fd_rms_quant(h, q, scale, cu_q, m, y=None, gate=None, weight=None, shift=None, mod_scale=None, eps: float = 1e-6,
                 stream=None) -> None:
    """h [rows, D] fp32 += gate * y (with y), then its RMS norm times weight, modulated, as codes q
    [rows, D] and scale bytes [rows, fd_scale_stride(D)]; q and scale None: h's update alone.  cu_q None: one
    request.  gate, shift and mod_scale: fp32 [requests, D], which may be column ranges of one modulation tensor
    (equal row strides)."""
    rows, D = _rows("h", h)
    B = 1 if cu_q is None else cu_q.numel() - 1
    stride, mod = _modulation(h, B, D, gate, shift, mod_scale)
    n = rows * D
    h_, y_, w_, cu_, m_, q_, s_, st = _pointers(
        stream, ("h", h, "f32", n), ("y", y, "b16", -n), ("weight", weight, "f32", -D), ("cu_q", cu_q, "i32", -2 if B == 1 else 2), ("m", m, "i32", 1),
        ("q", q, "code", n if scale is not None else -n), ("scale", scale, "scale", rows * _stride(D) * (1 if q is not None else -1)))
    _check("fd_rms_quant", lib().fd_rms_quant(rows, D, B, h_, y_, mod[0], w_, mod[1], mod[2], stride, eps, cu_, m_, q_, s_, st))


def rope_axes(dims: Sequence[int], theta=10000.0, step=1.0, halves: bool = False) -> FdRope:
    """Descriptor of rotary positions: the head's values per axis, theta and step of each axis (or
    one for all), pairs (j, j + dim / 2) with halves, else (2j, 2j + 1)."""
    n = len(dims)
    if not 1 <= n <= 4:
        raise FlashDiffError(f"{n} axes, not 1 to 4")
    r = FdRope(n, int(bool(halves)))    # the rest zeros
    r.dim[:n] = tuple(dims)
    for field, v in ((r.theta, theta), (r.step, step)):
        per = (v,) * n if isinstance(v, (int, float)) else [float(u) for u in v]
        if len(per) != n:
            raise FlashDiffError("dims, theta and step must have one entry per axis")
        field[:n] = per
    return r


def fd_rope_axes(qkv, coord, idx, m, q, k_cache, v_cache, heads: int, kv_heads: int, head_dim: int, dims=None, theta=10000.0,
                 step=1.0, halves: bool = False, rope: Optional[FdRope] = None, stream=None) -> None:
    """q | k | v rows qkv [rows, (heads + 2 kv_heads) head_dim]: q and k turned by the token's
    coord [tokens, axes]; q to [rows, heads head_dim], k and v to the caches' rows idx.  The axes
    are given by dims, theta, step and halves, or by a descriptor from rope_axes."""
    if rope is None and dims is None:
        raise FlashDiffError("the axes are required: dims or rope")
    r = rope if rope is not None else rope_axes(dims, theta, step, halves)
    (rows, cols), (tokens, axes) = _rows("qkv", qkv), _rows("coord", coord)
    if cols != (heads + 2 * kv_heads) * head_dim or axes != r.n_axes:
        raise FlashDiffError(f"qkv has {cols} columns and coord {axes} axes, needs {(heads + 2 * kv_heads) * head_dim} and {r.n_axes}")
    kv = tokens * kv_heads * head_dim
    p = _pointers(stream, ("coord", coord, "i32", tokens * axes), ("qkv", qkv, "b16", rows * cols), ("idx", idx, "i32", -rows),
                  ("m", m, "i32", 1), ("q", q, "b16", rows * heads * head_dim), ("k_cache", k_cache, "b16", kv), ("v_cache", v_cache, "b16", kv))
    _check("fd_rope_axes", lib().fd_rope_axes(rows, tokens, ctypes.byref(r), heads, kv_heads, head_dim, *p))


def fd_scaled_linear(a, a_scale, w, w_scale, y, y_scale=None, bias=None, gelu: bool = False, m=None, stream=None) -> None:
    """y = act(a w^T + bias) of codes a [rows, n_in] and w [n_out, n_in] with their scale bytes.
    y's type chooses the output: bf16, fp32, or codes (with y_scale [rows, fd_scale_stride(n_out)])."""
    (rows, k), (n, kw) = _rows("a", a), _rows("w", w)
    if k != kw:
        raise FlashDiffError(f"a has {k} columns, w {kw}")
    if y is None:
        raise FlashDiffError("y is required")
    dt, ld = y.dtype, _stride(k)
    codes, wide = dt in _KIND["code"], dt == torch.float32
    *ptrs, y_, ys_, st = _pointers(
        stream, ("a", a, "code", rows * k), ("a_scale", a_scale, "scale", rows * ld), ("w", w, "code", n * k),
        ("w_scale", w_scale, "scale", -(-n // 128) * ld), ("bias", bias, "f32", -n), ("m", m, "i32", -1),
        ("y", y, "code" if codes else "f32" if wide else "b16", rows * n),
        ("y_scale", y_scale if codes else None, "scale", rows * _stride(n) if codes else -1))
    a_, as_, w_, ws_, b_, m_ = ptrs
    _check("fd_scaled_linear", lib().fd_scaled_linear(rows, n, k, a_, as_, w_, ws_, b_, int(gelu), m_, None if codes or wide else y_,
                                                      y_ if wide else None, y_ if codes else None, ys_, st))


_SCALED = ("w_qkv", "w_o", "w_1", "w_2")


def scaled_params(params: Dict[str, torch.Tensor]) -> Dict[str, torch.Tensor]:
    """The block parameters of a model for 8-bit products, laid out once: every bf16 weight stack
    [L, out, in] as codes with 128 x 128 scales (s_* for w_*), the rest as it is.  norm_1 and norm_2
    ([L, D] fp32), where the model has them, are the weights of its RMS norms."""
    out = {k: v for k, v in params.items() if k not in _SCALED}
    for k in _SCALED:
        w = params[k]
        L, n, c = w.shape
        q = torch.empty((L, n, c), dtype=torch.float8_e4m3fn, device=w.device)
        s = torch.zeros((L, -(-n // 128), fd_scale_stride(c)), dtype=torch.uint8, device=w.device)
        for l in range(L):
            fd_quant_blocks(w[l], 128, q[l], s[l])
        out[k], out["s" + k[1:]] = q, s
    return out


def scaled_weights(params: Dict[str, torch.Tensor], l: int, mod: torch.Tensor) -> FdScaledWeights:
    """Weights of block l of scaled_params' tensors; mod: the block's [B, 6D] fp32 from fd_adaln."""
    D, F = params["w_o"].shape[1], params["w_1"].shape[1]
    block, kinds = [], []
    for n, out, cols in (("qkv", 3 * D, D), ("o", D, D), ("1", F, D), ("2", D, F)):
        block += [params["w_" + n][l], params["s_" + n][l], params["b_" + n][l]]
        kinds += [("w_" + n, "code", out * cols), ("s_" + n, "scale", -(-out // 128) * _stride(cols)), ("b_" + n, "f32", out)]
    for n in ("norm_1", "norm_2"):
        block.append(params[n][l] if n in params else None)
        kinds.append((n, "f32", D))
    for t, (name, kind, numel) in zip(block, kinds):
        _need(name, t, kind, numel, exact=True, optional=kind == "f32" and name.startswith("norm"))
    _need("mod", mod, "f32", 6 * D)
    return FdScaledWeights(*[_ptr(t) for t in block], _ptr(mod))


def fd_scaled_block_ws_size(plan: Plan, d: FdDims) -> int:
    return int(lib().fd_scaled_block_ws_size(ctypes.byref(plan.c), ctypes.byref(d)))


def fd_scaled_block_forward(plan: Plan, d: FdDims, w: FdScaledWeights, rope: Optional[FdRope], coord, h, idx, cu_q, m, k_cache,
                            v_cache, ws, stream=None) -> None:
    """fd_block_forward with RMS norms, rotary positions (rope from rope_axes and coord [tokens, axes], or
    both None) and 8-bit products; ws of fd_scaled_block_ws_size bytes."""
    N, B = plan.n_tokens, plan.n_requests
    p = _pointers(stream, ("h", h, "f32", N * d.D), ("idx", idx, "i32", N), ("cu_q", cu_q, "i32", B + 1), ("m", m, "i32", 1),
                  ("k_cache", k_cache, "b16", N * d.D), ("v_cache", v_cache, "b16", N * d.D),
                  ("coord", coord, "i32", -1 if rope is None else N * rope.n_axes))
    _need("ws", ws, "bytes", fd_scaled_block_ws_size(plan, d))
    if ws.device != h.device:
        raise FlashDiffError(f"ws is on {ws.device}, h on {h.device}")
    h_, idx_, cu_, m_, k_, v_, c_, st = p
    _check("fd_scaled_block_forward", lib().fd_scaled_block_forward(
        ctypes.byref(plan.c), ctypes.byref(d), ctypes.byref(w), None if rope is None else ctypes.byref(rope), c_, h_, idx_, cu_, m_,
        k_, v_, _ptr(ws), ws.numel() * ws.element_size(), st))


# ------------------------------------------------------------------ 8-bit integers

def fd_int_rows(x, q, scale, m=None, stream=None) -> None:
    """bf16 x [rows, cols] to int8 q [rows, cols] and fp32 scale [rows]: activations (`m` of the rows when given), or
    weights with a scale per output channel."""
    rows, cols = _rows("x", x)
    p = _pointers(stream, ("x", x, "b16", rows * cols), ("m", m, "i32", -1), ("q", q, "i8", rows * cols), ("scale", scale, "f32", rows))
    _check("fd_int_rows", lib().fd_int_rows(rows, cols, *p))


def fd_int_linear(a, a_scale, w, w_scale, y, bias=None, gelu: bool = False, m=None, stream=None) -> None:
    """y = act((a w^T) * w_scale * a_scale + bias) of int8 a [rows, n_in] and w [n_out, n_in] with fp32 scales per row
    and per output channel; y bf16 or fp32."""
    (rows, k), (n, kw) = _rows("a", a), _rows("w", w)
    if k != kw:
        raise FlashDiffError(f"a has {k} columns, w {kw}")
    if y is None:
        raise FlashDiffError("y is required")
    wide = y.dtype == torch.float32
    a_, as_, w_, ws_, b_, m_, y_, st = _pointers(
        stream, ("a", a, "i8", rows * k), ("a_scale", a_scale, "f32", rows), ("w", w, "i8", n * k), ("w_scale", w_scale, "f32", n),
        ("bias", bias, "f32", -n), ("m", m, "i32", -1), ("y", y, "f32" if wide else "b16", rows * n))
    _check("fd_int_linear", lib().fd_int_linear(rows, n, k, a_, as_, w_, ws_, b_, int(gelu), m_, None if wide else y_, y_ if wide else None, st))


def fd_norm_residual(h, a, cu_q, m, y=None, post_weight=None, gate=None, residual: float = 1.0, weight=None, shift=None, mod_scale=None,
                     a_scale=None, eps: float = 1e-6, stream=None) -> None:
    """h [rows, D] fp32 = residual * h + gate * RMS(y) post_weight (with y), then a = RMS(h) * weight, modulated.  a's type
    chooses the result: bf16 rows, e4m3 codes with a_scale bytes [rows, fd_scale_stride(D)], or int8 with a_scale fp32
    [rows]; None: h's update alone.  cu_q None: one request; gate, shift and mod_scale as for fd_rms_quant."""
    rows, D = _rows("h", h)
    B = 1 if cu_q is None else cu_q.numel() - 1
    stride, mod = _modulation(h, B, D, gate, shift, mod_scale)
    n, dt = rows * D, None if a is None else a.dtype
    kind, per = ("i8", rows) if dt == torch.int8 else ("code", rows * _stride(D)) if dt in _KIND["code"] else ("b16", 0)
    if a_scale is not None and not per:
        raise FlashDiffError("a_scale belongs to 8-bit rows")
    h_, y_, p_, w_, cu_, m_, a_, s_, st = _pointers(
        stream, ("h", h, "f32", n), ("y", y, "b16", -n), ("post_weight", post_weight, "f32", -D), ("weight", weight, "f32", -D),
        ("cu_q", cu_q, "i32", -2 if B == 1 else 2), ("m", m, "i32", 1), ("a", a, kind, -n),
        ("a_scale", a_scale, "f32" if kind == "i8" else "scale", per if per else -1))
    bf, codes, ints = kind == "b16", kind == "code", kind == "i8"
    _check("fd_norm_residual", lib().fd_norm_residual(
        rows, D, B, h_, y_, residual, p_, mod[0], w_, mod[1], mod[2], stride, eps, cu_, m_, a_ if bf else None, a_ if codes else None,
        s_ if codes else None, a_ if ints else None, s_ if ints else None, st))


# ------------------------------------------------------------------ 8-bit cache

def _cache(k, k_scale, v, v_scale, kv_heads: int, head_dim: int) -> int:
    """Tokens of an 8-bit cache: k and v [tokens, kv_heads * head_dim] with scales [kv_heads, tokens]."""
    tokens, cols = _rows("k", k)
    want = (kv_heads, tokens)
    for name, t, scale in (("k", k, k_scale), ("v", v, v_scale)):
        if t is None or scale is None:
            raise FlashDiffError(f"{name if t is None else name + '_scale'} is required")
        if t.shape != (tokens, kv_heads * head_dim):
            raise FlashDiffError(f"{name} has {t.shape[-1]} columns, needs {kv_heads * head_dim}" if t.shape[-1:] != (kv_heads * head_dim,)
                                 else "k and v must have the same tokens")
        if scale.shape != want:
            raise FlashDiffError(f"{name}_scale must be [{kv_heads}, {tokens}], got {tuple(scale.shape)}")
    return tokens


def fd_cache_write(qkv, coord, idx, m, q, k, k_scale, v, v_scale, heads: int, kv_heads: int, head_dim: int, dims=None, theta=10000.0,
                   step=1.0, halves: bool = False, rope: Optional[FdRope] = None, stream=None) -> None:
    """fd_rope_axes to an 8-bit cache: k and v e4m3 [tokens, kv_heads head_dim] with scale bytes [kv_heads, tokens].  coord
    None (with no dims or rope): q and k are not turned."""
    r = rope if rope is not None else rope_axes(dims, theta, step, halves) if dims is not None else None
    if (r is None) != (coord is None):
        raise FlashDiffError("rotary positions need both coord and the axes (dims or rope)")
    rows, cols = _rows("qkv", qkv)
    if cols != (heads + 2 * kv_heads) * head_dim:
        raise FlashDiffError(f"qkv has {cols} columns, needs {(heads + 2 * kv_heads) * head_dim}")
    tokens = _cache(k, k_scale, v, v_scale, kv_heads, head_dim)
    if coord is not None and coord.shape != (tokens, r.n_axes):
        raise FlashDiffError(f"coord must be [{tokens}, {r.n_axes}], got {tuple(coord.shape)}")
    kv = tokens * kv_heads
    p = _pointers(stream, ("coord", coord, "i32", -1 if r is None else tokens * r.n_axes), ("qkv", qkv, "b16", rows * cols), ("idx", idx, "i32", -rows),
                  ("m", m, "i32", 1), ("q", q, "b16", rows * heads * head_dim), ("k", k, "code", kv * head_dim), ("k_scale", k_scale, "scale", kv),
                  ("v", v, "code", kv * head_dim), ("v_scale", v_scale, "scale", kv))
    _check("fd_cache_write", lib().fd_cache_write(rows, tokens, None if r is None else ctypes.byref(r), heads, kv_heads, head_dim, *p))


def fd_cache_attention_ws_size(n_rows: int, heads: int, kv_heads: int, head_dim: int) -> int:
    return int(lib().fd_cache_attention_ws_size(n_rows, heads, kv_heads, head_dim))


def fd_cache_attention(q, k, k_scale, v, v_scale, o, cu_q, req_tok_off, heads: int, kv_heads: int, head_dim: int, ws,
                       max_request_tokens: Optional[int] = None, scale: Optional[float] = None, stream=None) -> None:
    """Attention of q's rows [rows, heads head_dim] (request b's are cu_q[b] .. cu_q[b + 1] - 1) over their request's
    tokens (req_tok_off) in an 8-bit cache, to o [rows, heads head_dim] bf16; scale None: 1 / sqrt(head_dim).  ws of
    fd_cache_attention_ws_size bytes, its own for calls that overlap."""
    rows, cols = _rows("q", q)
    if cols != heads * head_dim:
        raise FlashDiffError(f"q has {cols} columns, needs {heads * head_dim}")
    tokens = _cache(k, k_scale, v, v_scale, kv_heads, head_dim)
    if cu_q is None or req_tok_off is None or cu_q.numel() < 2 or cu_q.numel() != req_tok_off.numel():
        raise FlashDiffError("cu_q and req_tok_off must both have requests + 1 entries")
    B, kv = cu_q.numel() - 1, tokens * kv_heads
    if ws is None or not ws.is_cuda or not ws.is_contiguous() or ws.get_device() != q.get_device():
        raise FlashDiffError("ws must be a contiguous tensor on q's device")
    q_, k_, ks_, v_, vs_, cu_, to_, o_, st = _pointers(
        stream, ("q", q, "b16", rows * cols), ("k", k, "code", kv * head_dim), ("k_scale", k_scale, "scale", kv), ("v", v, "code", kv * head_dim),
        ("v_scale", v_scale, "scale", kv), ("cu_q", cu_q, "i32", B + 1), ("req_tok_off", req_tok_off, "i32", B + 1), ("o", o, "b16", rows * cols))
    _check("fd_cache_attention", lib().fd_cache_attention(
        rows, tokens, B, tokens if max_request_tokens is None else max_request_tokens, heads, kv_heads, head_dim,
        head_dim ** -0.5 if scale is None else scale, q_, k_, ks_, v_, vs_, cu_, to_, o_, ws.data_ptr(), ws.numel() * ws.element_size(), st))


def fd_timer_arm(kernel: str, capacity: int) -> None:
    _check("fd_timer_arm", lib().fd_timer_arm(KERNELS[kernel], capacity))


def fd_timer_read(capacity: int) -> np.ndarray:
    out = np.zeros(capacity, np.float32)
    n = lib().fd_timer_read(out.ctypes.data, capacity)
    return out[:n]


def fd_timer_disarm() -> None:
    lib().fd_timer_disarm()


# ------------------------------------------------------------------ step state

class SparseStep:
    """Device buffers of one batch and the call sequence of one region-sparse step.

    Holds the plan, model parameters (device tensors from workloads.make_params),
    per-block K/V caches, the gate state and the row workspaces; `step()` issues
    fd_region_score, fd_select, fd_gather, fd_embed, fd_adaln (the modulation of
    all L blocks in one pass), L x fd_block_forward, fd_final and
    fd_scatter_update on the current stream.  With the importance signal the
    gate thresholds `delta` (carried from the previous step) instead of the
    region score, and fd_region_importance runs after the chosen block.

    With `scaled` (scaled_params of the model) the blocks are fd_scaled_block_forward's: RMS norms
    and 8-bit products, and rotary positions where `rope` (rope_axes) and `coord` (int32
    [N, axes], the tokens' positions) are given.
    """

    def __init__(self, plan: Plan, d: FdDims, params: Dict[str, torch.Tensor], n_layers: int,
                 k_cache: Optional[torch.Tensor] = None, v_cache: Optional[torch.Tensor] = None,
                 device: str = "cuda", scaled: Optional[Dict[str, torch.Tensor]] = None, rope: Optional[FdRope] = None,
                 coord: Optional[torch.Tensor] = None):
        if scaled is None and (rope is not None or coord is not None):
            raise FlashDiffError("rotary positions belong to the 8-bit blocks: give `scaled` too")
        if (rope is None) != (coord is None):
            raise FlashDiffError("rotary positions need both `rope` and `coord`")
        if coord is not None:
            if tuple(coord.shape) != (plan.n_tokens, rope.n_axes):
                raise FlashDiffError(f"coord must be [{plan.n_tokens}, {rope.n_axes}], got {tuple(coord.shape)}")
            _need("coord", coord, "i32", coord.numel())
            _ptr(coord)
        self.plan, self.d, self.params, self.L = plan, d, params, n_layers
        N, R, B, C, D = plan.n_tokens, plan.n_regions, plan.n_requests, d.C, d.D
        dev = torch.device(device)
        self.k_cache = k_cache if k_cache is not None else torch.zeros((n_layers, N, D), dtype=torch.bfloat16,
                                                                        device=dev)
        self.v_cache = v_cache if v_cache is not None else torch.zeros((n_layers, N, D), dtype=torch.bfloat16,
                                                                        device=dev)
        self.score = torch.zeros(R, dtype=torch.float64, device=dev)
        self.s_tilde = torch.zeros(R, dtype=torch.float64, device=dev)
        self.skip_run = torch.zeros(R, dtype=torch.int32, device=dev)
        self.active = torch.ones(R, dtype=torch.uint8, device=dev)
        self.all_active = torch.ones(R, dtype=torch.uint8, device=dev)
        self.idx = torch.zeros(N, dtype=torch.int32, device=dev)
        self.cu_q = torch.zeros(B + 1, dtype=torch.int32, device=dev)
        self.m = torch.zeros(1, dtype=torch.int32, device=dev)
        self.xa = torch.zeros((N, C), dtype=torch.bfloat16, device=dev)
        self.h = torch.zeros((N, D), dtype=torch.float32, device=dev)
        self.v = torch.zeros((N, C), dtype=torch.float32, device=dev)
        self.vcache = torch.zeros((N, C), dtype=torch.float32, device=dev)
        self.ws_score = torch.empty(max(fd_region_score_ws_size(plan, C), 256), dtype=torch.uint8, device=dev)
        ws_block = fd_block_ws_size(plan, d) if scaled is None else fd_scaled_block_ws_size(plan, d)
        self.ws_block = torch.empty(ws_block, dtype=torch.uint8, device=dev)
        self.mod = torch.zeros((n_layers, B, 6 * D), dtype=torch.float32, device=dev)
        self.scaled, self.rope, self.coord = scaled, rope, coord
        if scaled is None:
            self.block_w = [block_weights(params, l, self.mod[l]) for l in range(n_layers)]
        else:
            self.block_w = [scaled_weights(scaled, l, self.mod[l]) for l in range(n_layers)]
        self.final_w = final_weights(params)
        self.r_bar = torch.zeros(R, dtype=torch.float64, device=dev)
        self.delta = torch.zeros(R, dtype=torch.float64, device=dev)
        self.importance = torch.zeros(R, dtype=torch.float64, device=dev)
        self.ws_imp = torch.empty(max(fd_importance_ws_size(plan, d), 256), dtype=torch.uint8, device=dev)

    def reset_gate(self) -> None:
        self.s_tilde.zero_()
        self.skip_run.zero_()
        self.active.fill_(1)
        self.r_bar.zero_()
        self.delta.zero_()

    def step(self, x: torch.Tensor, x_prev: torch.Tensor, eps: torch.Tensor, dt: torch.Tensor,
             cond: torch.Tensor, eta: float = 0.0, max_skip: int = 0, skip_mode: int = FD_SKIP_FREEZE,
             stateless: bool = False, stream=None, signal: str = "delta",
             importance_block: Optional[int] = None) -> None:
        """One step on the latent x (updated in place); eps fp64 [B], dt fp32 [B], cond fp32 [B, D].

        stateless=True gates on fresh scores only (every region counts as
        executed at the previous step).  signal="importance" gates on `delta`;
        importance_block (a block index) updates r_bar and delta from that
        block's self-attention for the next step."""
        p, d, C = self.plan, self.d, self.d.C
        prev = self.all_active if stateless else self.active
        if signal == "importance":
            score = self.delta
        else:
            fd_region_score(p, C, x, x_prev, self.score, self.ws_score, stream)
            score = self.score
        fd_select(p, score, eps, eta, max_skip, self.s_tilde, self.skip_run, prev, self.active,
                  self.idx, self.cu_q, self.m, stream)
        fd_gather(p, C, x, self.idx, self.m, self.xa, stream)
        fd_embed(p, d, self.xa, self.params["w_e"], self.params["b_e"], self.params["pos"], self.idx, self.m,
                 self.h, stream)
        fd_adaln(d, self.L, 6 * d.D, p.n_requests, self.params["w_ada"], self.params["b_ada"], cond, self.mod,
                 stream)
        for l in range(self.L):
            if self.scaled is None:
                fd_block_forward(p, d, self.block_w[l], cond, self.h, self.idx, self.cu_q, self.m, self.k_cache[l],
                                 self.v_cache[l], self.ws_block, stream)
            else:
                fd_scaled_block_forward(p, d, self.block_w[l], self.rope, self.coord, self.h, self.idx, self.cu_q, self.m,
                                        self.k_cache[l], self.v_cache[l], self.ws_block, stream)
            if importance_block == l:
                fd_region_importance(p, d, self.ws_block, self.k_cache[l], self.idx, self.m, self.active, self.r_bar,
                                     self.delta, self.importance, self.ws_imp, stream)
        fd_final(p, d, self.final_w, cond, self.h, self.cu_q, self.m, self.v, self.ws_block, stream)
        fd_scatter_update(p, C, x, self.v, self.idx, self.m, dt, self.vcache, self.active, skip_mode, stream)

    def capture(self, x: torch.Tensor, x_prev: torch.Tensor, eps: torch.Tensor, dt: torch.Tensor,
                cond: torch.Tensor, **kw) -> "torch.cuda.CUDAGraph":
        """Records one step on these tensors into a HIP graph (nothing runs during the
        capture); each replay() runs the step on whatever the tensors then hold, with
        the same state buffers as step().  The step makes no host round trip and no
        allocation, and no kernel keeps state from one launch to the next, so replays
        are independent of each other.  Keyword arguments are those of step() except
        `stream`."""
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            self.step(x, x_prev, eps, dt, cond, **kw)
        return g
