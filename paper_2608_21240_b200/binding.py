"""Thin ctypes binding of libspice.so: argument marshalling only.

Every function named spice_* forwards to the C entry point of the same name (include/spice.h)
with torch tensors turned into device pointers; nothing of the layer is computed in Python.
`SpiceLayer` bundles a context with output allocation for convenience.  torch is used for
device memory and streams only.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("SPICE_LIB") or os.path.join(_PKG, "libspice.so")   # SPICE_LIB: an instrumented or older build

SPICE_OK = 0
HIT, MISS_EXACT, LOWCONF = 0, 1, 2


class SpiceError(RuntimeError):
    pass


class LayerCfg(C.Structure):
    """Mirror of spice_layer_cfg."""
    _fields_ = [("d", C.c_int32), ("n_experts", C.c_int32), ("top_k", C.c_int32), ("inter", C.c_int32),
                ("inter_shared", C.c_int32), ("lore_rank", C.c_int32), ("n_slots", C.c_int32),
                ("norm_topk", C.c_int32), ("conf_stride", C.c_int32), ("tau", C.c_float)]


class LayerWeightsC(C.Structure):
    """Mirror of spice_layer_weights (device pointers)."""
    _fields_ = [("w_router", C.c_void_p), ("slot_w_gate_up", C.c_void_p), ("slot_w_down", C.c_void_p),
                ("slot_of_expert", C.c_void_p), ("shared_w_gate_up", C.c_void_p), ("shared_w_down", C.c_void_p),
                ("lore_A", C.c_void_p), ("lore_B", C.c_void_p)]


class LayerWeightsFp8C(C.Structure):
    """Mirror of spice_layer_weights_fp8 (device pointers)."""
    _fields_ = [("w_router", C.c_void_p), ("slot_q_gate_up", C.c_void_p), ("slot_s_gate_up", C.c_void_p),
                ("slot_q_down", C.c_void_p), ("slot_s_down", C.c_void_p), ("slot_of_expert", C.c_void_p),
                ("shared_q_gate_up", C.c_void_p), ("shared_s_gate_up", C.c_void_p), ("shared_q_down", C.c_void_p),
                ("shared_s_down", C.c_void_p), ("lore_A", C.c_void_p), ("lore_B", C.c_void_p)]


_lib = None


def lib() -> C.CDLL:
    """Load libspice.so.  Raises if it has not been built: there is no fallback path."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise SpiceError(f"{LIB_PATH} is missing: build it with `python -m paper_2608_21240_b200.build` "
                             "(needs nvcc); the library has no CPU or PyTorch fallback")
        L = C.CDLL(LIB_PATH)
        L.spice_status_string.restype = C.c_char_p
        L.spice_version.restype = C.c_int32
        for name in ("spice_create", "spice_destroy", "spice_workspace_bytes", "spice_route_topk",
                     "spice_classify_misses", "spice_grouped_expert_ffn", "spice_lore_surrogate",
                     "spice_moe_layer_fwd", "spice_get_device_status", "spice_launch_count", "spice_set_option",
                     "spice_grouped_expert_ffn_static", "spice_draft_confidence", "spice_prefetch_rollout",
                     "spice_quantize_e4m3_rows", "spice_moe_layer_fwd_fp8"):
            getattr(L, name).restype = C.c_int
        i32, i64, f32, ptr = C.c_int32, C.c_int64, C.c_float, C.c_void_p
        for name, args in (("spice_residual_rmsnorm", [ptr, ptr, ptr, ptr, f32, i32, i32, ptr, ptr, ptr, ptr]),
                           ("spice_quantize_i8_rows", [ptr, i64, i32, ptr, ptr, ptr]),
                           ("spice_gemm_i8", [ptr, ptr, ptr, ptr, i32, i32, i32, i32, ptr, ptr, ptr]),
                           ("spice_swiglu_i8", [ptr, ptr, ptr, ptr, i32, i32, i32, ptr, ptr, ptr]),
                           ("spice_sort_tokens", [ptr, i32, i32, i32, ptr, ptr, ptr, ptr, i32, ptr, ptr, i32, ptr, ptr]),
                           ("spice_combine_tokens", [ptr, i32, i32, ptr, ptr, i32, i32, i32, i32, ptr, ptr]),
                           ("spice_combine_tokens_grad", [ptr, i32, ptr, i32, i32, ptr, ptr, i32, i32, i32, ptr, ptr, ptr]),
                           ("spice_quantize_e4m3_blocks", [ptr, i64, i64, i32, i32, ptr, ptr, ptr]),
                           ("spice_gemm_e4m3_blocks", [ptr, ptr, ptr, ptr, ptr, i32, i32, i32, i32, i32, ptr, ptr, ptr]),
                           ("spice_swiglu_e4m3_blocks", [ptr, ptr, ptr, ptr, ptr, i32, i32, i32, i32, ptr, ptr, ptr, ptr]),
                           ("spice_route_scored", [ptr, ptr, i32, i32, i32, i32, i32, i32, i32, i32, f32, ptr, ptr, ptr])):
            getattr(L, name).argtypes, getattr(L, name).restype = args, C.c_int
        L.spice_static_scratch_bytes.restype = C.c_size_t
        L.spice_lore_calibrate.restype = C.c_int
        L.spice_lore_calibrate_workspace_bytes.restype = C.c_size_t
        _lib = L
    return _lib


def _check(code: int, what: str) -> None:
    if code != SPICE_OK:
        raise SpiceError(f"{what}: {lib().spice_status_string(code).decode()} (status {code})")


def _ptr(t: Optional[torch.Tensor], dtype=None) -> C.c_void_p:
    if t is None:
        return C.c_void_p(0)
    # (pinned host memory is device-accessible under unified addressing: a caller may let the kernels write small
    # results straight into it instead of copying them back)
    if not (t.is_cuda or t.is_pinned()) or not t.is_contiguous():
        raise SpiceError("tensors passed to libspice must be contiguous CUDA tensors (or pinned host tensors)")
    if dtype is not None and t.dtype != dtype:
        raise SpiceError(f"expected dtype {dtype}, got {t.dtype}")
    return C.c_void_p(t.data_ptr())


def _stream(stream) -> C.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


# ------------------------------------------------------------------ C entry points, same names
def spice_create(cfg: LayerCfg, max_tokens: int, device: int = 0) -> C.c_void_p:
    ctx = C.c_void_p()
    _check(lib().spice_create(C.byref(ctx), C.c_int32(device), C.byref(cfg), C.c_int32(max_tokens)), "spice_create")
    return ctx


def spice_destroy(ctx) -> None:
    _check(lib().spice_destroy(ctx), "spice_destroy")


def spice_workspace_bytes(ctx) -> int:
    n = C.c_size_t()
    _check(lib().spice_workspace_bytes(ctx, C.byref(n)), "spice_workspace_bytes")
    return n.value


def spice_launch_count(ctx) -> int:
    n = C.c_int64()
    _check(lib().spice_launch_count(ctx, C.byref(n)), "spice_launch_count")
    return n.value


OPT_PATH, OPT_SPIN_LIMIT, OPT_TC_WAIT_LIMIT, OPT_I8_WAIT_LIMIT, OPT_E4M3_WAIT_LIMIT = 0, 1, 2, 3, 4


def spice_set_option(ctx, option: int, value: int) -> None:
    _check(lib().spice_set_option(ctx, C.c_int32(option), C.c_int64(value)), "spice_set_option")


def spice_get_device_status(ctx) -> int:
    v = C.c_int32()
    _check(lib().spice_get_device_status(ctx, C.byref(v)), "spice_get_device_status")
    return v.value


def spice_route_topk(ctx, h, w_router, T, idx, gate, logits=None, stream=None) -> None:
    _check(lib().spice_route_topk(ctx, _ptr(h, torch.bfloat16), _ptr(w_router, torch.bfloat16), C.c_int32(T),
                                  _ptr(idx, torch.int32), _ptr(gate, torch.float32), _ptr(logits, torch.float32),
                                  _stream(stream)), "spice_route_topk")


def spice_draft_confidence(ctx, h_hat, w_draft_router, T, idx_hat, conf, pi_hat=None, stream=None) -> None:
    _check(lib().spice_draft_confidence(ctx, _ptr(h_hat, torch.bfloat16), _ptr(w_draft_router, torch.bfloat16), C.c_int32(T),
                                        _ptr(idx_hat, torch.int32), _ptr(pi_hat, torch.float32), _ptr(conf, torch.float32),
                                        _stream(stream)), "spice_draft_confidence")


def spice_min_lookahead_depth(n_prefetch, expert_bytes, pcie_bytes_per_s, t_comp_s) -> int:
    f = lib().spice_min_lookahead_depth
    f.restype = C.c_int32
    return int(f(C.c_int32(n_prefetch), C.c_double(expert_bytes), C.c_double(pcie_bytes_per_s), C.c_double(t_comp_s)))


def spice_prefetch_rollout(ctx, weights, x_current, T, l_min, l_max, tau, idx_hat, conf, depth, h_final=None,
                           prefetch_mask=None, stream=None) -> None:
    """weights: sequence of l_max LayerWeightsC structs (depth 1 first)."""
    arr = (LayerWeightsC * l_max)(*weights)
    _check(lib().spice_prefetch_rollout(ctx, arr, _ptr(x_current, torch.bfloat16), C.c_int32(T), C.c_int32(l_min),
                                        C.c_int32(l_max), C.c_float(tau), _ptr(idx_hat, torch.int32),
                                        _ptr(conf, torch.float32), _ptr(depth, torch.int32), _ptr(h_final, torch.bfloat16),
                                        _ptr(prefetch_mask, torch.uint8), _stream(stream)), "spice_prefetch_rollout")


def spice_lore_calibrate(h_cal, resid, rank, ridge=0.0, iterations=100, stream=None):
    """Fit the LoRE factors of one expert on the device.  h_cal [n,d] bf16, resid [n,d] fp32 (device tensors).
    Returns (A [rank,d] bf16, B [d,rank] bf16, loss tensor [2] = (objective, sum resid^2), status tensor [1])."""
    n, d = h_cal.shape
    dev = h_cal.device
    nbytes = int(lib().spice_lore_calibrate_workspace_bytes(C.c_int32(d), C.c_int32(n), C.c_int32(rank)))
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    A = torch.empty(rank, d, dtype=torch.bfloat16, device=dev)
    Bm = torch.empty(d, rank, dtype=torch.bfloat16, device=dev)
    loss = torch.empty(2, dtype=torch.float32, device=dev)
    status = torch.empty(1, dtype=torch.int32, device=dev)
    with torch.cuda.device(dev):
        _check(lib().spice_lore_calibrate(C.c_int32(d), C.c_int32(n), C.c_int32(rank), C.c_float(ridge), C.c_int32(iterations),
                                          _ptr(h_cal, torch.bfloat16), _ptr(resid, torch.float32), _ptr(A, torch.bfloat16),
                                          _ptr(Bm, torch.bfloat16), _ptr(loss, torch.float32), _ptr(status, torch.int32),
                                          C.c_void_p(ws.data_ptr()), C.c_size_t(nbytes), _stream(stream)),
               "spice_lore_calibrate")
    return A, Bm, loss, status


def spice_classify_misses(ctx, idx, gate, slot_of_expert, conf, T, cls, slot, counts, resid_tok=None, resid_k=None,
                          resid_expert=None, resid_gate=None, stream=None) -> None:
    _check(lib().spice_classify_misses(ctx, _ptr(idx, torch.int32), _ptr(gate, torch.float32),
                                       _ptr(slot_of_expert, torch.int32), _ptr(conf, torch.float32), C.c_int32(T),
                                       _ptr(cls, torch.uint8), _ptr(slot, torch.int32), _ptr(counts, torch.int32),
                                       _ptr(resid_tok, torch.int32), _ptr(resid_k, torch.int32),
                                       _ptr(resid_expert, torch.int32), _ptr(resid_gate, torch.float32),
                                       _stream(stream)), "spice_classify_misses")


def spice_grouped_expert_ffn(ctx, weights: LayerWeightsC, h, idx, gate, cls, slot, T, y, stream=None) -> None:
    _check(lib().spice_grouped_expert_ffn(ctx, C.byref(weights), _ptr(h, torch.bfloat16), _ptr(idx, torch.int32),
                                          _ptr(gate, torch.float32), _ptr(cls, torch.uint8), _ptr(slot, torch.int32),
                                          C.c_int32(T), _ptr(y, torch.float32), _stream(stream)),
           "spice_grouped_expert_ffn")


def spice_grouped_expert_ffn_static(cfg: LayerCfg, weights: LayerWeightsC, h, idx, gate, cls, slot, T, y,
                                    device_status=None, stream=None) -> None:
    """The resident-expert FFN without a ctx and without any allocation (for hosts that may not call
    cudaMalloc): scratch lives in a fixed 8 MiB device array inside the library.  Calls on one GPU must
    not overlap; the first call on a GPU should precede any stream capture."""
    _check(lib().spice_grouped_expert_ffn_static(C.byref(cfg), C.byref(weights), _ptr(h, torch.bfloat16),
                                                 _ptr(idx, torch.int32), _ptr(gate, torch.float32),
                                                 _ptr(cls, torch.uint8), _ptr(slot, torch.int32), C.c_int32(T),
                                                 _ptr(y, torch.float32), _ptr(device_status, torch.int32),
                                                 _stream(stream)), "spice_grouped_expert_ffn_static")


def spice_static_scratch_bytes() -> int:
    return int(lib().spice_static_scratch_bytes())


def spice_lore_surrogate(ctx, weights: LayerWeightsC, h, idx, gate, cls, T, y, stream=None) -> None:
    _check(lib().spice_lore_surrogate(ctx, C.byref(weights), _ptr(h, torch.bfloat16), _ptr(idx, torch.int32),
                                      _ptr(gate, torch.float32), _ptr(cls, torch.uint8), C.c_int32(T),
                                      _ptr(y, torch.float32), _stream(stream)), "spice_lore_surrogate")


def spice_moe_layer_fwd(ctx, weights: LayerWeightsC, h, conf, T, y, y_cpu_residual=None, x_resid=None, idx=None,
                        gate=None, cls=None, counts=None, resid_tok=None, resid_k=None, resid_expert=None,
                        resid_gate=None, stream=None) -> None:
    _check(lib().spice_moe_layer_fwd(ctx, C.byref(weights), _ptr(h, torch.bfloat16), _ptr(conf, torch.float32),
                                     C.c_int32(T), _ptr(y_cpu_residual, torch.float32),
                                     _ptr(x_resid, torch.bfloat16), _ptr(y, torch.bfloat16), _ptr(idx, torch.int32),
                                     _ptr(gate, torch.float32), _ptr(cls, torch.uint8), _ptr(counts, torch.int32),
                                     _ptr(resid_tok, torch.int32), _ptr(resid_k, torch.int32),
                                     _ptr(resid_expert, torch.int32), _ptr(resid_gate, torch.float32),
                                     _stream(stream)), "spice_moe_layer_fwd")


def spice_quantize_e4m3_rows(w, q, scale, stream=None) -> None:
    """w [..., cols] bf16 -> q (uint8, same shape) and scale (fp32, shape without the last axis): E4M3 codes with one
    power-of-two scale per row."""
    cols = w.shape[-1]
    rows = w.numel() // cols
    with torch.cuda.device(w.device):
        _check(lib().spice_quantize_e4m3_rows(_ptr(w, torch.bfloat16), C.c_int64(rows), C.c_int32(cols), _ptr(q, torch.uint8),
                                              _ptr(scale, torch.float32), _stream(stream)), "spice_quantize_e4m3_rows")


def spice_moe_layer_fwd_fp8(ctx, weights: "LayerWeightsFp8C", h, conf, T, y, y_cpu_residual=None, x_resid=None, idx=None,
                            gate=None, cls=None, counts=None, resid_tok=None, resid_k=None, resid_expert=None,
                            resid_gate=None, stream=None) -> None:
    _check(lib().spice_moe_layer_fwd_fp8(ctx, C.byref(weights), _ptr(h, torch.bfloat16), _ptr(conf, torch.float32),
                                         C.c_int32(T), _ptr(y_cpu_residual, torch.float32),
                                         _ptr(x_resid, torch.bfloat16), _ptr(y, torch.bfloat16), _ptr(idx, torch.int32),
                                         _ptr(gate, torch.float32), _ptr(cls, torch.uint8), _ptr(counts, torch.int32),
                                         _ptr(resid_tok, torch.int32), _ptr(resid_k, torch.int32),
                                         _ptr(resid_expert, torch.int32), _ptr(resid_gate, torch.float32),
                                         _stream(stream)), "spice_moe_layer_fwd_fp8")


# ---- steps next to the layer: no ctx; shapes are read off the tensors and checked, the call goes to the tensors' device
SCORE_SOFTMAX, SCORE_SIGMOID = 0, 1
GROUP_MAX, GROUP_TOP2 = 0, 1
OUT_BF16, OUT_F32, OUT_F32_ADD = 0, 1, 2


def _addr(what: str, t: Optional[torch.Tensor], dtype, shape, dev: int, pinned: bool = True) -> Optional[int]:
    """Address of a tensor of this type and shape on CUDA device `dev` (or, with `pinned`, in pinned host memory); None for
    None."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.is_contiguous() and (t.get_device() == dev or (pinned and t.is_pinned())):
        return t.data_ptr()
    raise SpiceError(f"{what}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on cuda:{dev}, got {t.dtype} "
                     f"{tuple(t.shape)} on {t.device}{'' if t.is_contiguous() else ', not contiguous'}")


def _rows_of(what: str, t: torch.Tensor):
    """(rows, columns, device index) of the 2-D CUDA tensor that gives a call its sizes."""
    shape = t.shape
    if len(shape) != 2 or not t.is_cuda:
        raise SpiceError(f"{what}: expected a 2-D CUDA tensor, got shape {tuple(shape)} on {t.device}")
    rows, cols = shape
    if rows > 0x7fffffff or cols > 0x7fffffff:
        raise SpiceError(f"{what}: too many rows or columns: {tuple(shape)}")
    return rows, cols, t.get_device()


# The raw handle of a device's current stream without a Stream object around it (2 us less per call, as much as the launch
# itself); the public way where this build of torch does not have it.
_current_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call_on(dev: int, name: str, stream, *args) -> None:
    """The entry point on the tensors' device, whatever the current one is."""
    st = _current_raw_stream(dev) if stream is None else stream.cuda_stream
    f = getattr(_lib or lib(), name)
    if dev == _current_device():
        code = f(*args, st)
    else:
        with torch.cuda.device(dev):
            code = f(*args, st)
    if code != SPICE_OK:
        _check(code, name)


def spice_residual_rmsnorm(x_resid, weight, eps, q=None, scale=None, h=None, delta=None, stream=None) -> None:
    """x_resid [T,d] bf16 (in/out), delta [T,d] bf16 or fp32 or None, weight [d] bf16 -> h [T,d] bf16 and / or q [T,d] int8
    with scale [T] fp32."""
    f = "spice_residual_rmsnorm"
    T, d, dev = _rows_of(f, x_resid)
    bf, f32 = torch.bfloat16, torch.float32
    wide = delta is not None and delta.dtype == f32
    if (q is None) != (scale is None):
        raise SpiceError(f"{f}: q and scale are given together")
    _call_on(dev, f, stream, _addr(f, x_resid, bf, (T, d), dev), None if wide else _addr(f, delta, bf, (T, d), dev),
             _addr(f, delta, f32, (T, d), dev) if wide else None, _addr(f, weight, bf, (d,), dev), eps, T, d,
             _addr(f, h, bf, (T, d), dev), _addr(f, q, torch.int8, (T, d), dev), _addr(f, scale, f32, (T,), dev))


def spice_quantize_i8_rows(w, q, scale, stream=None) -> None:
    """w [..., cols] bf16 -> q (int8, same shape) and scale (fp32, shape without the last axis)."""
    f = "spice_quantize_i8_rows"
    if w.dim() < 1 or not w.is_cuda:
        raise SpiceError(f"{f}: expected a CUDA tensor, got shape {tuple(w.shape)} on {w.device}")
    cols, dev = w.shape[-1], w.get_device()
    if cols < 1 or cols > 0x7fffffff:
        raise SpiceError(f"{f}: unsupported row length {cols}")
    _call_on(dev, f, stream, _addr(f, w, torch.bfloat16, w.shape, dev), w.numel() // cols, cols,
             _addr(f, q, torch.int8, w.shape, dev), _addr(f, scale, torch.float32, w.shape[:-1], dev))


def spice_gemm_i8(x_q, x_scale, w_q, w_scale, y, accumulate=False, device_status=None, stream=None) -> None:
    """x_q [T,k] int8, x_scale [T] fp32, w_q [n,k] int8, w_scale [n] fp32 -> y [T,n] bf16 or fp32; accumulate: y fp32 is
    added to.  x_q and w_q live on the device (the kernels' bulk copies read them).  device_status: zeroed int32 tensor of one
    element that receives an expired wait."""
    f = "spice_gemm_i8"
    T, k, dev = _rows_of(f, x_q)
    n = min(w_q.shape[0], 0x7fffffff) if w_q.dim() else 0   # (its shape is checked with its address)
    i8, f32 = torch.int8, torch.float32
    out = (OUT_F32_ADD if accumulate else OUT_F32) if y.dtype == f32 else OUT_BF16
    if accumulate and out == OUT_BF16:
        raise SpiceError(f"{f}: only an fp32 y is added to")
    _call_on(dev, f, stream, _addr(f, x_q, i8, (T, k), dev), _addr(f, x_scale, f32, (T,), dev),
             _addr(f, w_q, i8, (n, k), dev, False), _addr(f, w_scale, f32, (n,), dev), T, n, k, out,
             _addr(f, y, torch.bfloat16 if out == OUT_BF16 else f32, (T, n), dev), _addr(f, device_status, torch.int32, (1,), dev))


def spice_swiglu_i8(x_q, x_scale, w_gate_up_q, w_scale, act, device_status=None, stream=None) -> None:
    """x_q [T,k] int8, x_scale [T] fp32, w_gate_up_q [2 inter,k] int8 (gate rows, then up rows), w_scale [2 inter] fp32 ->
    act [T,inter] bf16.  x_q and w_gate_up_q live on the device."""
    f = "spice_swiglu_i8"
    T, k, dev = _rows_of(f, x_q)
    n2 = min(w_gate_up_q.shape[0], 0x7ffffffe) if w_gate_up_q.dim() else 0
    if n2 % 2:
        raise SpiceError(f"{f}: w_gate_up_q has an odd number of rows")
    i8, f32 = torch.int8, torch.float32
    _call_on(dev, f, stream, _addr(f, x_q, i8, (T, k), dev), _addr(f, x_scale, f32, (T,), dev),
             _addr(f, w_gate_up_q, i8, (n2, k), dev, False), _addr(f, w_scale, f32, (n2,), dev), T, n2 // 2, k,
             _addr(f, act, torch.bfloat16, (T, n2 // 2), dev), _addr(f, device_status, torch.int32, (1,), dev))


def spice_route_scored(logits, idx, gate, bias=None, score=SCORE_SOFTMAX, n_groups=1, top_groups=1, group_score=GROUP_MAX,
                       norm_topk=True, scale=1.0, stream=None) -> None:
    """logits [T,N] fp32 (and bias [N] fp32) -> idx [T,K] int32, gate [T,K] fp32."""
    f = "spice_route_scored"
    T, N, dev = _rows_of(f, logits)
    K = min(idx.shape[-1], 0x7fffffff) if idx.dim() else 0
    f32 = torch.float32
    _call_on(dev, f, stream, _addr(f, logits, f32, (T, N), dev), _addr(f, bias, f32, (N,), dev), T, N, K, score, n_groups,
             top_groups, group_score, int(norm_topk), scale, _addr(f, idx, torch.int32, (T, K), dev),
             _addr(f, gate, f32, (T, K), dev))


# ---- experts of one's own: tokens sorted by expert and back, products in E4M3 with a scale for each block of 128
def spice_sort_tokens(idx, offset, pos, entry, x=None, rows=None, x_scale=None, rows_scale=None, stream=None) -> None:
    """idx [T,K] int32 -> offset [n_experts + 1], pos [T,K], entry [T*K] int32; with x [T,d] (any type, rows of a multiple of 16
    bytes) rows [T*K,d] of the same type, with x_scale [T,c] fp32 rows_scale [T*K,c]."""
    f = "spice_sort_tokens"
    T, K, dev = _rows_of(f, idx)
    i32, f32 = torch.int32, torch.float32
    if offset.dim() != 1 or offset.shape[0] < 2:
        raise SpiceError(f"{f}: offset has an element for each expert and one more")
    if (x is None) != (rows is None) or (x_scale is None) != (rows_scale is None) or (x is None and x_scale is not None):
        raise SpiceError(f"{f}: x and rows, x_scale and rows_scale are given together, scales with rows")
    d = row_bytes = cols = 0
    if x is not None:
        d = _rows_of(f, x)[1]
        row_bytes = min(d * x.element_size(), 0x7fffffff)
    if x_scale is not None:
        cols = _rows_of(f, x_scale)[1]
    _call_on(dev, f, stream, _addr(f, idx, i32, (T, K), dev), T, K, offset.shape[0] - 1, _addr(f, offset, i32, offset.shape, dev),
             _addr(f, pos, i32, (T, K), dev), _addr(f, entry, i32, (T * K,), dev),
             None if x is None else _addr(f, x, x.dtype, (T, d), dev), row_bytes,
             None if x is None else _addr(f, rows, x.dtype, (T * K, d), dev), _addr(f, x_scale, f32, (T, cols), dev), cols,
             _addr(f, rows_scale, f32, (T * K, cols), dev))


def _row_type(what: str, t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return OUT_F32
    if t.dtype == torch.bfloat16:
        return OUT_BF16
    raise SpiceError(f"{what}: expected rows of bfloat16 or float32, got {t.dtype}")


def spice_combine_tokens(rows, pos, y, gate=None, accumulate=False, stream=None) -> None:
    """rows [R,d] bf16 or fp32, pos [T,K] int32, gate [T,K] fp32 or None -> y [T,d] bf16 or fp32; accumulate: y fp32 is added to."""
    f = "spice_combine_tokens"
    R, d, dev = _rows_of(f, rows)
    T, K, _ = _rows_of(f, pos)
    f32 = torch.float32
    out = _row_type(f, y)
    if accumulate and out == OUT_BF16:
        raise SpiceError(f"{f}: only an fp32 y is added to")
    _call_on(dev, f, stream, _addr(f, rows, rows.dtype, (R, d), dev), _row_type(f, rows), R, _addr(f, pos, torch.int32, (T, K), dev),
             _addr(f, gate, f32, (T, K), dev), T, K, d, OUT_F32_ADD if accumulate else out, _addr(f, y, y.dtype, (T, d), dev))


def spice_combine_tokens_grad(dy, rows, pos, gate=None, d_rows=None, d_gate=None, stream=None) -> None:
    """dy [T,d] bf16 or fp32, rows [R,d] bf16 or fp32 (None without d_gate), pos [T,K] int32, gate [T,K] fp32 or None -> d_rows
    [R,d] bf16 or fp32 (the type of rows) and / or d_gate [T,K] fp32."""
    f = "spice_combine_tokens_grad"
    T, d, dev = _rows_of(f, dy)
    K = _rows_of(f, pos)[1]
    like = rows if rows is not None else d_rows
    if like is None or (d_rows is None and d_gate is None) or (d_gate is not None and rows is None):
        raise SpiceError(f"{f}: nothing is asked for, or d_gate without rows")
    R = _rows_of(f, like)[0]
    f32 = torch.float32
    _call_on(dev, f, stream, _addr(f, dy, dy.dtype, (T, d), dev), _row_type(f, dy), _addr(f, rows, like.dtype, (R, d), dev),
             _row_type(f, like), R, _addr(f, pos, torch.int32, (T, K), dev), _addr(f, gate, f32, (T, K), dev), T, K, d,
             _addr(f, d_rows, like.dtype, (R, d), dev), _addr(f, d_gate, f32, (T, K), dev))


def spice_quantize_e4m3_blocks(w, q, scale, block_rows=1, stream=None) -> None:
    """w [..., rows, cols] bf16 -> q (uint8 E4M3 codes, same shape) and scale [..., ceil(rows / block_rows), ceil(cols / 128)] fp32;
    block_rows 1 (activations) or 128 (weights)."""
    f = "spice_quantize_e4m3_blocks"
    if w.dim() < 2 or not w.is_cuda:
        raise SpiceError(f"{f}: expected a CUDA tensor of matrices, got shape {tuple(w.shape)} on {w.device}")
    if block_rows not in (1, 128):
        raise SpiceError(f"{f}: blocks have 1 or 128 rows")
    (rows, cols), dev = w.shape[-2:], w.get_device()
    if cols < 1 or cols > 0x7fffffff:
        raise SpiceError(f"{f}: unsupported row length {cols}")
    lead = w.shape[:-2]
    _call_on(dev, f, stream, _addr(f, w, torch.bfloat16, w.shape, dev), lead.numel(), rows, cols, block_rows,
             _addr(f, q, torch.uint8, w.shape, dev),
             _addr(f, scale, torch.float32, (*lead, -(-rows // block_rows), -(-cols // 128)), dev))


def _block_operands(f, x_q, x_scale, w_q, w_scale, offset):
    """What the two products check alike: (addresses of the operands and offsets, groups, T, rows of a weight matrix, k, device)."""
    T, k, dev = _rows_of(f, x_q)
    u8, f32, kb = torch.uint8, torch.float32, -(-k // 128)
    lead = () if offset is None else (min(w_q.shape[0] if w_q.dim() else 0, 0x7fffffff),)
    n = min(w_q.shape[len(lead)], 0x7ffffffe) if w_q.dim() > len(lead) else 0   # (its shape is checked with its address)
    G = lead[0] if lead else 1
    return ((_addr(f, x_q, u8, (T, k), dev, False), _addr(f, x_scale, f32, (T, kb), dev), _addr(f, w_q, u8, (*lead, n, k), dev, False),
             _addr(f, w_scale, f32, (*lead, -(-n // 128), kb), dev), _addr(f, offset, torch.int32, (G + 1,), dev)), G, T, n, k, dev)


def spice_gemm_e4m3_blocks(x_q, x_scale, w_q, w_scale, y, offset=None, accumulate=False, device_status=None, stream=None) -> None:
    """x_q [T,k] uint8, x_scale [T,ceil(k/128)] fp32, w_q [n,k] uint8 with w_scale [ceil(n/128),ceil(k/128)], or with offset [G+1]
    int32 w_q [G,n,k] and w_scale [G,...] -> y [T,n] bf16 or fp32; accumulate: y fp32 is added to.  x_q, w_q and y live on the
    device (bulk copies).  device_status: zeroed int32 tensor of one element that receives bad offsets and an expired wait."""
    f = "spice_gemm_e4m3_blocks"
    ptrs, G, T, n, k, dev = _block_operands(f, x_q, x_scale, w_q, w_scale, offset)
    out = _row_type(f, y)
    if accumulate and out == OUT_BF16:
        raise SpiceError(f"{f}: only an fp32 y is added to")
    _call_on(dev, f, stream, *ptrs, G, T, n, k, OUT_F32_ADD if accumulate else out, _addr(f, y, y.dtype, (T, n), dev, False),
             _addr(f, device_status, torch.int32, (1,), dev))


def spice_swiglu_e4m3_blocks(x_q, x_scale, w_gate_up_q, w_scale, act_q, act_scale, offset=None, device_status=None, stream=None) -> None:
    """As spice_gemm_e4m3_blocks with w_gate_up_q [(G,) 2 inter, k] (gate rows, then up rows) -> act_q [T,inter] uint8 E4M3 codes with
    act_scale [T, inter / 128] fp32."""
    f = "spice_swiglu_e4m3_blocks"
    ptrs, G, T, n2, k, dev = _block_operands(f, x_q, x_scale, w_gate_up_q, w_scale, offset)
    if n2 % 256:
        raise SpiceError(f"{f}: w_gate_up_q has {n2} rows, not two times a multiple of 128")
    inter = n2 // 2
    _call_on(dev, f, stream, *ptrs, G, T, inter, k, _addr(f, act_q, torch.uint8, (T, inter), dev),
             _addr(f, act_scale, torch.float32, (T, inter // 128), dev), _addr(f, device_status, torch.int32, (1,), dev))


# ------------------------------------------------------------------ convenience wrappers
@dataclass
class LayerWeights:
    """Device tensors of one layer (bf16 unless noted); see spice_layer_weights."""
    w_router: torch.Tensor          # [N,d]
    slot_w_gate_up: torch.Tensor    # [S,2I,d]
    slot_w_down: torch.Tensor       # [S,d,I]
    slot_of_expert: torch.Tensor    # [N] int32
    shared_w_gate_up: torch.Tensor  # [2Is,d]
    shared_w_down: torch.Tensor     # [d,Is]
    lore_A: torch.Tensor            # [N,r,d]
    lore_B: torch.Tensor            # [N,d,r]

    def c_struct(self) -> LayerWeightsC:
        return LayerWeightsC(_ptr(self.w_router, torch.bfloat16), _ptr(self.slot_w_gate_up, torch.bfloat16),
                             _ptr(self.slot_w_down, torch.bfloat16), _ptr(self.slot_of_expert, torch.int32),
                             _ptr(self.shared_w_gate_up, torch.bfloat16), _ptr(self.shared_w_down, torch.bfloat16),
                             _ptr(self.lore_A, torch.bfloat16), _ptr(self.lore_B, torch.bfloat16))


@dataclass
class LayerWeightsFp8:
    """Device tensors of one layer at the 8-bit weight precision; see spice_layer_weights_fp8."""
    w_router: torch.Tensor          # [N,d] bf16
    slot_q_gate_up: torch.Tensor    # [S,2I,d] uint8 (E4M3)
    slot_s_gate_up: torch.Tensor    # [S,2I] fp32
    slot_q_down: torch.Tensor       # [S,d,I] uint8
    slot_s_down: torch.Tensor       # [S,d] fp32
    slot_of_expert: torch.Tensor    # [N] int32
    shared_q_gate_up: torch.Tensor  # [2Is,d] uint8
    shared_s_gate_up: torch.Tensor  # [2Is] fp32
    shared_q_down: torch.Tensor     # [d,Is] uint8
    shared_s_down: torch.Tensor     # [d] fp32
    lore_A: torch.Tensor            # [N,r,d] bf16
    lore_B: torch.Tensor            # [N,d,r] bf16

    def c_struct(self) -> LayerWeightsFp8C:
        u8, f32, bf = torch.uint8, torch.float32, torch.bfloat16
        return LayerWeightsFp8C(_ptr(self.w_router, bf), _ptr(self.slot_q_gate_up, u8), _ptr(self.slot_s_gate_up, f32),
                                _ptr(self.slot_q_down, u8), _ptr(self.slot_s_down, f32), _ptr(self.slot_of_expert, torch.int32),
                                _ptr(self.shared_q_gate_up, u8), _ptr(self.shared_s_gate_up, f32),
                                _ptr(self.shared_q_down, u8), _ptr(self.shared_s_down, f32), _ptr(self.lore_A, bf),
                                _ptr(self.lore_B, bf))


def quantize_layer(w: "LayerWeights") -> LayerWeightsFp8:
    """The 8-bit form of a bf16 weight set: four calls of spice_quantize_e4m3_rows (allocation of the outputs only)."""
    def qz(t):
        q = torch.empty(t.shape, dtype=torch.uint8, device=t.device)
        s = torch.empty(t.shape[:-1], dtype=torch.float32, device=t.device)
        spice_quantize_e4m3_rows(t, q, s)
        return q, s
    sgu, ssgu = qz(w.slot_w_gate_up)
    sd, ssd = qz(w.slot_w_down)
    hgu, shgu = qz(w.shared_w_gate_up)
    hd, shd = qz(w.shared_w_down)
    return LayerWeightsFp8(w.w_router, sgu, ssgu, sd, ssd, w.slot_of_expert, hgu, shgu, hd, shd, w.lore_A, w.lore_B)


@dataclass
class SharedExpertI8:
    """Device tensors of the shared expert (or a dense FFN) in 8-bit integers with a scale per output channel."""
    q_gate_up: torch.Tensor    # [2Is,d] int8
    s_gate_up: torch.Tensor    # [2Is] fp32
    q_down: torch.Tensor       # [d,Is] int8
    s_down: torch.Tensor       # [d] fp32


def quantize_shared_i8(w: "LayerWeights") -> SharedExpertI8:
    """The shared expert of a bf16 weight set in 8-bit integers: two calls of spice_quantize_i8_rows."""
    def qz(t):
        q = torch.empty(t.shape, dtype=torch.int8, device=t.device)
        s = torch.empty(t.shape[:-1], dtype=torch.float32, device=t.device)
        spice_quantize_i8_rows(t, q, s)
        return q, s
    return SharedExpertI8(*qz(w.shared_w_gate_up), *qz(w.shared_w_down))


def shared_expert_i8(w: SharedExpertI8, x_q, x_scale, y, accumulate=False, device_status=None, stream=None) -> torch.Tensor:
    """y (bf16 or fp32, or added to fp32) = the SwiGLU FFN of the 8-bit rows that spice_residual_rmsnorm wrote: three calls
    (gate/up products with the activation, the activations' 8-bit rows, the down product) and the buffers between them.
    S(h) once: a layer in which entries are LOWCONF needs it once more for each of them and takes spice_lore_surrogate (bf16
    weights) instead."""
    T, dev = x_q.shape[0], x_q.device
    with torch.cuda.stream(stream):
        act = torch.empty(T, w.q_down.shape[1], dtype=torch.bfloat16, device=dev)
        q, s = torch.empty_like(act, dtype=torch.int8), torch.empty(T, dtype=torch.float32, device=dev)
    spice_swiglu_i8(x_q, x_scale, w.q_gate_up, w.s_gate_up, act, device_status, stream)
    spice_quantize_i8_rows(act, q, s, stream)
    spice_gemm_i8(q, s, w.q_down, w.s_down, y, accumulate, device_status, stream)
    return y


@dataclass
class ExpertsE4M3:
    """Device tensors of SwiGLU experts in E4M3 with a scale for each block of 128 x 128."""
    q_gate_up: torch.Tensor    # [G,2I,d] uint8
    s_gate_up: torch.Tensor    # [G,2I/128,ceil(d/128)] fp32
    q_down: torch.Tensor       # [G,d,I] uint8
    s_down: torch.Tensor       # [G,ceil(d/128),I/128] fp32


def quantize_experts_e4m3(w_gate_up: torch.Tensor, w_down: torch.Tensor) -> ExpertsE4M3:
    """Experts [G,2I,d] and [G,d,I] bf16 (the slot pool of a LayerWeights) in E4M3: two calls of spice_quantize_e4m3_blocks."""
    def qz(t):
        q = torch.empty(t.shape, dtype=torch.uint8, device=t.device)
        s = torch.empty(*t.shape[:-2], -(-t.shape[-2] // 128), -(-t.shape[-1] // 128), dtype=torch.float32, device=t.device)
        spice_quantize_e4m3_blocks(t, q, s, block_rows=128)
        return q, s
    return ExpertsE4M3(*qz(w_gate_up), *qz(w_down))


def routed_experts_e4m3(w: ExpertsE4M3, h, idx, gate, y, accumulate=False, device_status=None, stream=None) -> torch.Tensor:
    """y (bf16 or fp32, or added to fp32) = sum_k gate[t,k] E_{idx[t,k]}(h[t]) over the entries with 0 <= idx < G, for any batch: five calls
    (8-bit rows of h, sort, gate/up products with the activation, down products, weighted sum) and the buffers between them.
    idx: the routing's idx, or the slot array of spice_classify_misses for the experts of a slot pool."""
    (T, K), (G, d, inter), dev = idx.shape, w.q_down.shape, h.device
    f32, i32, u8 = torch.float32, torch.int32, torch.uint8
    with torch.cuda.stream(stream):
        new = lambda *shape, dtype: torch.empty(*shape, dtype=dtype, device=dev)  # noqa: E731
        q, s = new(T, d, dtype=u8), new(T, -(-d // 128), dtype=f32)
        offset, pos, entry = new(G + 1, dtype=i32), new(T, K, dtype=i32), new(T * K, dtype=i32)
        rows, rows_s = new(T * K, d, dtype=u8), new(T * K, -(-d // 128), dtype=f32)
        act, act_s = new(T * K, inter, dtype=u8), new(T * K, inter // 128, dtype=f32)
        down = new(T * K, d, dtype=torch.bfloat16)
    spice_quantize_e4m3_blocks(h, q, s, 1, stream)
    spice_sort_tokens(idx, offset, pos, entry, q, rows, s, rows_s, stream)
    spice_swiglu_e4m3_blocks(rows, rows_s, w.q_gate_up, w.s_gate_up, act, act_s, offset, device_status, stream)
    spice_gemm_e4m3_blocks(act, act_s, w.q_down, w.s_down, down, offset, False, device_status, stream)
    spice_combine_tokens(down, pos, y, gate, accumulate, stream)
    return y


@dataclass
class LayerOutputs:
    y: torch.Tensor
    idx: torch.Tensor
    gate: torch.Tensor
    cls: torch.Tensor
    counts: torch.Tensor
    resid_tok: torch.Tensor
    resid_k: torch.Tensor
    resid_expert: torch.Tensor
    resid_gate: torch.Tensor


def make_cfg(d, n_experts, top_k, inter, inter_shared, lore_rank, n_slots, tau, norm_topk=1, conf_per_expert=True):
    return LayerCfg(d, n_experts, top_k, inter, inter_shared, lore_rank, n_slots, norm_topk,
                    n_experts if conf_per_expert else 0, tau)


class SpiceLayer:
    """A spice_ctx plus output buffers; every method is one C call."""

    def __init__(self, cfg: LayerCfg, max_tokens: int, device: int = 0):
        self.cfg, self.max_tokens, self.device = cfg, max_tokens, device
        torch.cuda.set_device(device)
        self.ctx = spice_create(cfg, max_tokens, device)
        self.dev = torch.device("cuda", device)

    def close(self):
        if self.ctx is not None:
            spice_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _empty(self, shape, dtype):
        return torch.empty(shape, dtype=dtype, device=self.dev)

    def route_topk(self, h, w_router, want_logits=False, stream=None):
        T, K, N = h.shape[0], self.cfg.top_k, self.cfg.n_experts
        idx, gate = self._empty((T, K), torch.int32), self._empty((T, K), torch.float32)
        logits = self._empty((T, N), torch.float32) if want_logits else None
        spice_route_topk(self.ctx, h, w_router, T, idx, gate, logits, stream)
        return (idx, gate, logits) if want_logits else (idx, gate)

    def draft_confidence(self, h_hat, w_draft_router, want_pi=False, stream=None):
        T, K, N = h_hat.shape[0], self.cfg.top_k, self.cfg.n_experts
        idx, conf = self._empty((T, K), torch.int32), self._empty((T,), torch.float32)
        pi = self._empty((T, N), torch.float32) if want_pi else None
        spice_draft_confidence(self.ctx, h_hat, w_draft_router, T, idx, conf, pi, stream)
        return (idx, conf, pi) if want_pi else (idx, conf)

    def prefetch_rollout(self, weights, x_current, l_min, l_max, tau, stream=None):
        """weights: list of l_max LayerWeights (depth 1 first).  Returns (idx_hat, conf, depth, h_final)."""
        T, K = x_current.shape[0], self.cfg.top_k
        idx = self._empty((l_max, T, K), torch.int32)
        conf = self._empty((l_max, T), torch.float32)
        depth = self._empty((T,), torch.int32)
        h_final = self._empty((T, self.cfg.d), torch.bfloat16)
        self.prefetch_mask = self._empty((l_max, self.cfg.n_experts), torch.uint8)
        spice_prefetch_rollout(self.ctx, [w.c_struct() for w in weights], x_current, T, l_min, l_max, tau, idx, conf,
                               depth, h_final, self.prefetch_mask, stream)
        return idx, conf, depth, h_final

    def classify_misses(self, idx, gate, slot_of_expert, conf, stream=None):
        T, K = idx.shape
        cls, slot = self._empty((T, K), torch.uint8), self._empty((T, K), torch.int32)
        counts = torch.zeros(3, dtype=torch.int32, device=self.dev)
        n = max(T * K, 1)
        rt, rk, re_ = (self._empty((n,), torch.int32) for _ in range(3))
        rg = self._empty((n,), torch.float32)
        spice_classify_misses(self.ctx, idx, gate, slot_of_expert, conf, T, cls, slot, counts, rt, rk, re_, rg, stream)
        return cls, slot, counts, (rt, rk, re_, rg)

    def grouped_expert_ffn(self, w: LayerWeights, h, idx, gate, cls, slot, y, stream=None):
        spice_grouped_expert_ffn(self.ctx, w.c_struct(), h, idx, gate, cls, slot, h.shape[0], y, stream)
        return y

    def lore_surrogate(self, w: LayerWeights, h, idx, gate, cls, y, stream=None):
        spice_lore_surrogate(self.ctx, w.c_struct(), h, idx, gate, cls, h.shape[0], y, stream)
        return y

    def moe_layer_fwd(self, w: LayerWeights, h, conf, y_cpu_residual=None, x_resid=None, stream=None) -> LayerOutputs:
        T, K, d = h.shape[0], self.cfg.top_k, self.cfg.d
        n = max(T * K, 1)
        o = LayerOutputs(self._empty((T, d), torch.bfloat16), self._empty((T, K), torch.int32),
                         self._empty((T, K), torch.float32), self._empty((T, K), torch.uint8),
                         torch.zeros(3, dtype=torch.int32, device=self.dev), self._empty((n,), torch.int32),
                         self._empty((n,), torch.int32), self._empty((n,), torch.int32),
                         self._empty((n,), torch.float32))
        spice_moe_layer_fwd(self.ctx, w.c_struct(), h, conf, T, o.y, y_cpu_residual, x_resid, o.idx, o.gate, o.cls,
                            o.counts, o.resid_tok, o.resid_k, o.resid_expert, o.resid_gate, stream)
        return o

    def moe_layer_fwd_fp8(self, w: LayerWeightsFp8, h, conf, y_cpu_residual=None, x_resid=None, stream=None) -> LayerOutputs:
        T, K, d = h.shape[0], self.cfg.top_k, self.cfg.d
        n = max(T * K, 1)
        o = LayerOutputs(self._empty((T, d), torch.bfloat16), self._empty((T, K), torch.int32),
                         self._empty((T, K), torch.float32), self._empty((T, K), torch.uint8),
                         torch.zeros(3, dtype=torch.int32, device=self.dev), self._empty((n,), torch.int32),
                         self._empty((n,), torch.int32), self._empty((n,), torch.int32),
                         self._empty((n,), torch.float32))
        spice_moe_layer_fwd_fp8(self.ctx, w.c_struct(), h, conf, T, o.y, y_cpu_residual, x_resid, o.idx, o.gate, o.cls,
                                o.counts, o.resid_tok, o.resid_k, o.resid_expert, o.resid_gate, stream)
        return o

    def set_option(self, option: int, value: int) -> None:
        spice_set_option(self.ctx, option, value)

    def device_status(self) -> int:
        return spice_get_device_status(self.ctx)

    def launch_count(self) -> int:
        return spice_launch_count(self.ctx)


# ------------------------------------------------------------------ workload marshalling
def bf16_tensor(x_f32, dev="cuda") -> torch.Tensor:
    """fp32 numpy array holding bf16-representable values -> bf16 device tensor (bit exact)."""
    import numpy as np
    from . import workloads as W
    bits = W.bf16_bits(x_f32)
    return torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16).to(dev)


def bits_tensor(bits, dev="cuda") -> torch.Tensor:
    import numpy as np
    return torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16).to(dev)


def cfg_of(s, tau=None, norm_topk=None, conf_per_expert=True) -> LayerCfg:
    """spice_layer_cfg of a workloads.LayerShape."""
    return make_cfg(s.d, s.n_experts, s.top_k, s.inter, s.inter_shared, s.lore_rank, s.n_slots,
                    s.tau if tau is None else tau, s.norm_topk if norm_topk is None else norm_topk, conf_per_expert)


def upload(wl, dev="cuda", only=None) -> LayerWeights:
    """Copy a workloads.LayerWorkload's weights to the device in the library's layout.

    only: experts whose slot contents matter (see LayerWorkload.slot_pool_bits)."""
    gu, dn = wl.slot_pool_bits(only)
    sg, su, sd = wl.shared()
    A, Bm = wl.lore()
    return LayerWeights(
        w_router=bf16_tensor(wl.w_router, dev),
        slot_w_gate_up=bits_tensor(gu, dev),
        slot_w_down=bits_tensor(dn, dev),
        slot_of_expert=torch.from_numpy(wl.slot_of_expert.copy()).to(dev),
        shared_w_gate_up=torch.cat([bf16_tensor(sg, dev), bf16_tensor(su, dev)], 0).contiguous(),
        shared_w_down=bf16_tensor(sd, dev),
        lore_A=bf16_tensor(A, dev),
        lore_B=bf16_tensor(Bm, dev),
    )
