"""Thin ctypes binding of libquaff.so: the same entry points as include/quaff.h, taking torch device tensors.

Argument marshalling only - every step of the path runs in the HIP kernels behind the C ABI.  PyTorch is used
for device memory (`tensor.data_ptr()`) and the current HIP stream.  The library must have been built
(`python -m paper_2505_14742_amd.build`); loading fails loudly otherwise - there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libquaff.so")

OK, ERR_NULL, ERR_SHAPE, ERR_WORKSPACE, ERR_ALIGN, ERR_HIP = 0, -1, -2, -3, -4, -5

_vp, _i64, _i32, _f32, _sz = C.c_void_p, C.c_int64, C.c_int32, C.c_float, C.c_size_t

SIGNATURES = {
    "quaff_status_string": (C.c_char_p, [C.c_int]),
    "quaff_last_hip_error": (C.c_int, []),
    "quaff_padded_outliers": (_i32, [_i32]),
    "quaff_packed_weight_bytes": (_sz, [_i64, _i64]),
    "quaff_packed_weight_offset": (_i64, [_i64, _i64, _i64, _i64]),
    "quaff_prepare_workspace_bytes": (_sz, [_i64, _i64]),
    "quaff_workspace_bytes": (_sz, [_i64, _i64, _i64, _i32, _i32]),
    "quaff_prepare_weight": (C.c_int, [_vp, _i64, _i64, _i64, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "quaff_scale_update": (C.c_int, [_vp, _i64, _i64, _i64, _vp, _i32, _vp, _vp, _i64, _f32, _vp, _vp, _vp, _vp, _vp,
                                     _vp, _sz, _vp]),
    "quaff_check_outliers": (C.c_int, [_vp, _i32, _i64, _vp, _vp]),
    "quaff_scale_update_static_max_outliers": (_i32, []),
    "quaff_scale_update_static": (C.c_int, [_vp, _i64, _i64, _i64, _vp, _i32, _vp, _vp, _i64, _f32, _vp, _vp, _vp, _vp,
                                            _vp, _vp]),
    "quaff_quant_act": (C.c_int, [_vp, _i64, _i64, _i64, _vp, _vp, _i32, _vp, _vp, _vp, _vp]),
    "quaff_linear_fwd": (C.c_int, [_vp, _vp, _vp, _i64, _vp, _vp, _i64, _i64, _vp, _vp, _i32, _vp, _i64, _vp, _vp,
                                   _i32, _f32, _vp, _i64, _vp, _sz, _vp]),
    "quaff_linear_fwd_bf16": (C.c_int, [_vp, _vp, _vp, _i64, _vp, _vp, _i64, _i64, _vp, _vp, _i32, _vp, _i64, _vp, _vp,
                                   _i32, _f32, _vp, _i64, _vp, _sz, _vp]),
    "quaff_linear_fwd_acc": (C.c_int, [_vp, _vp, _i64, _vp, _i64, _i64, _vp, _i32, _vp, _vp, _vp]),
    "quaff_linear_bwd_dx": (C.c_int, [_vp, _i64, _i64, _vp, _vp, _i64, _i64, _vp, _vp, _i32, _f32, _vp, _i64, _vp,
                                      _sz, _vp]),
    "quaff_linear_bwd_dx_bf16": (C.c_int, [_vp, _i64, _i64, _vp, _vp, _i64, _i64, _vp, _vp, _i32, _f32, _vp, _i64, _vp,
                                      _sz, _vp]),
    "quaff_linear_bwd_dx_acc": (C.c_int, [_vp, _i64, _i64, _vp, _vp, _i64, _i64, _vp, _vp, _vp, _vp]),
    "quaff_lora_bwd_workspace_bytes": (_sz, [_i64, _i64, _i64, _i32]),
    "quaff_bwd_step_workspace_bytes": (_sz, [_i64, _i64, _i64, _i32]),
    "quaff_linear_bwd_step": (C.c_int, [_vp, _i64, _i64, _vp, _i64, _vp, _vp, _i64, _i64, _vp, _vp, _i32, _f32, _vp,
                                        _i64, _vp, _vp, _vp, _sz, _vp, _vp, _vp, _vp]),
    "quaff_lora_bwd_weights": (C.c_int, [_vp, _i64, _vp, _i64, _i64, _i64, _i64, _vp, _vp, _i32, _f32, _vp, _vp, _vp,
                                         _sz, _vp]),
    "quaff_bwd_dx_outlier_workspace_bytes": (_sz, [_i64, _i64]),
    "quaff_bwd_dx_outlier_exact": (C.c_int, [_vp, _i64, _i64, _i64, _i64, _vp, _i32, _vp, _vp, _vp, _i32, _f32, _vp,
                                             _i64, _vp, _sz, _vp]),
    "quaff_calibrate_workspace_bytes": (_sz, [_i64, _i32]),
    "quaff_calibrate_outliers": (C.c_int, [_vp, _i64, _i64, _i64, _vp, _i32, C.c_double, _i32, _vp, _vp, _vp, _vp, _sz,
                                           _vp]),
    "quaff_fwd_step_workspace_bytes": (_sz, [_i64, _i64, _i64, _i32, _i32]),
    "quaff_linear_fwd_step": (C.c_int, [_vp, _i64, _i64, _i64, _vp, _i32, _vp, _vp, _i64, _f32, _vp, _vp, _vp, _vp, _vp,
                                        _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i32, _f32, _vp, _i64, _vp, _sz, _vp]),
    "quaff_mx4_padded": (_i64, [_i64]),
    "quaff_mx4_quantize": (C.c_int, [_vp, _i64, _i64, _i64, _vp, _vp, _vp]),
    "quaff_mx4_dequantize": (C.c_int, [_vp, _vp, _i64, _i64, _vp, _i64, _vp]),
    "quaff_mx4_prepare_weight": (C.c_int, [_vp, _i32, _i64, _i64, _i64, _vp, _vp, _vp, _vp, _vp]),
    "quaff_check_group_offsets": (C.c_int, [_vp, _i32, _i64, _vp, _vp]),
    "quaff_mx4_linear_workspace_bytes": (_sz, [_i64, _i64, _i64, _i32, _i32]),
    **{name: (C.c_int, [_vp, _i64, _i64, _vp, _i32, _vp, _vp, _i64, _i64, _vp, _vp, _i32, _f32, _vp, _i64, _vp, _sz, _vp])
       for name in ("quaff_mx4_linear_fwd", "quaff_mx4_linear_fwd_bf16", "quaff_mx4_linear_bwd_dx", "quaff_mx4_linear_bwd_dx_bf16")},
    "quaff_grouped_linear_workspace_bytes": (_sz, [_i64, _i64, _i64, _i32]),
    **{name: (C.c_int, [_vp, _i64, _i64, _vp, _i32, _vp, _i64, _i64, _f32, C.c_int, _vp, _i64, _vp, _sz, _vp])
       for name in ("quaff_grouped_linear_fwd", "quaff_grouped_linear_bwd_dx")},
    **{name: (C.c_int, [_vp, _i64, _i64, _vp, _i32, _vp, _i64, _i64, _f32, _vp, _i64, _vp, _sz, _vp])
       for name in ("quaff_grouped_linear_fwd_bf16", "quaff_grouped_linear_bwd_dx_bf16")},
    "quaff_grouped_linear_bwd_dw": (C.c_int, [_vp, _i64, _vp, _i64, _i64, _vp, _i32, _i64, _i64, _f32, _vp, _vp, _sz, _vp]),
    "quaff_debug_group_form": (C.c_char_p, [C.c_int, _i64, _i64, _i64, _i32]),
    "quaff_debug_grid_wait_ticks": (C.c_longlong, [C.c_longlong]),
    "quaff_debug_product_form": (C.c_char_p, [_i64, _i64, _i64, _i32, _i32, C.c_int]),
    "quaff_profile_enable": (C.c_int, [C.c_int]),
    "quaff_profile_collect": (_i64, []),
    "quaff_profile_launch": (C.c_int, [_i64, C.POINTER(C.c_int), C.POINTER(C.c_float)]),
    "quaff_profile_kind_name": (C.c_char_p, [C.c_int]),
    "quaff_microbench_mfma_i8": (C.c_int, [C.c_int, C.POINTER(C.c_double), C.POINTER(C.c_double)]),
    "quaff_microbench_copy": (C.c_int, [_sz, C.POINTER(C.c_double)]),
}

_lib = None


class QuaffError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        msg = lib().quaff_status_string(status).decode()
        if status == ERR_HIP:
            msg += " (hipError %d)" % lib().quaff_last_hip_error()
        super().__init__(msg)


def lib():
    """The loaded C-ABI library.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libquaff.so is not built: run `python -m paper_2505_14742_amd.build` "
                               "(there is no CPU or PyTorch fallback for this path)")
        # PyTorch ships its own copy of the HIP runtime.  The tensors handed to this library live in that runtime's
        # context, so it must be the one libquaff.so binds to: load torch first (a process that loaded libquaff.so
        # before torch got two runtimes and "no device" from the first launch).
        import torch  # noqa: F401
        l = C.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(l, name)
            fn.restype, fn.argtypes = res, args
        _lib = l
    return _lib


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    """Handle of the current stream of the current device.  torch's own accessor of the handle spares the Stream object that
    torch.cuda.current_stream() makes of it (3.1 us a call, half of a small call's host time) and is no public name: where it is missing, the
    Stream object it is."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return torch.cuda.current_stream().cuda_stream if raw is None else raw(torch.cuda.current_device())


def _check(status):
    if status != OK:
        raise QuaffError(status)


def padded_outliers(n: int) -> int:
    return int(lib().quaff_padded_outliers(n))


def packed_weight_bytes(c_in: int, c_out: int) -> int:
    return int(lib().quaff_packed_weight_bytes(c_in, c_out))


def packed_weight_offset(c_in: int, c_out: int, k: int, j: int) -> int:
    return int(lib().quaff_packed_weight_offset(c_in, c_out, k, j))


def prepare_workspace_bytes(c_in: int, c_out: int) -> int:
    return int(lib().quaff_prepare_workspace_bytes(c_in, c_out))


def workspace_bytes(t: int, c_in: int, c_out: int, n_outlier: int, lora_rank: int) -> int:
    return int(lib().quaff_workspace_bytes(t, c_in, c_out, n_outlier, lora_rank))


def prepare_weight(W, O, Wq_packed, delta_w, W_O, wmax_O, Wq_plain, workspace):
    c_in, c_out = W.shape
    n = 0 if O is None else O.numel()
    _check(lib().quaff_prepare_weight(_ptr(W), c_in, c_out, W.stride(0), _ptr(O), n, _ptr(Wq_packed), _ptr(delta_w),
                                      _ptr(W_O), _ptr(wmax_O), _ptr(Wq_plain), _ptr(workspace),
                                      workspace.numel() * workspace.element_size(), _stream()))


def scale_update(X, O, W_O, wmax_O, c_out, gamma, s_O, colscale, what_int, delta_what, cmax_out, workspace):
    t, c_in = X.shape
    n = 0 if O is None else O.numel()
    _check(lib().quaff_scale_update(_ptr(X), t, c_in, X.stride(0), _ptr(O), n, _ptr(W_O), _ptr(wmax_O), c_out,
                                    float(gamma), _ptr(s_O), _ptr(colscale), _ptr(what_int), _ptr(delta_what),
                                    _ptr(cmax_out), _ptr(workspace),
                                    0 if workspace is None else workspace.numel() * workspace.element_size(),
                                    _stream()))


def check_outliers(O, c_in, result):
    """Enqueue the validity scan of O; `result` is a one-element int32 device tensor (0 = valid, else 1 + position)."""
    n = 0 if O is None else O.numel()
    _check(lib().quaff_check_outliers(_ptr(O), n, c_in, _ptr(result), _stream()))


def scale_update_static_max_outliers() -> int:
    return int(lib().quaff_scale_update_static_max_outliers())


def scale_update_static(X, O, W_O, wmax_O, c_out, gamma, s_O, colscale, what_int, delta_what, cmax_out):
    t, c_in = X.shape
    n = 0 if O is None else O.numel()
    _check(lib().quaff_scale_update_static(_ptr(X), t, c_in, X.stride(0), _ptr(O), n, _ptr(W_O), _ptr(wmax_O), c_out,
                                           float(gamma), _ptr(s_O), _ptr(colscale), _ptr(what_int), _ptr(delta_what),
                                           _ptr(cmax_out), _stream()))


def quant_act(X, colscale, O, Xq, delta, xq_O):
    t, c = X.shape
    n = 0 if O is None else O.numel()
    _check(lib().quaff_quant_act(_ptr(X), t, c, X.stride(0), _ptr(colscale), _ptr(O), n, _ptr(Xq), _ptr(delta),
                                 _ptr(xq_O), _stream()))


def linear_fwd(Xq, delta_x, xq_O, Wq_packed, delta_w, c_in, c_out, what_int, delta_what, n_outlier, X, lora_A, lora_B,
               lora_rank, lora_scale, Y, workspace, bf16_out=False):
    t = Xq.shape[0]
    fn = lib().quaff_linear_fwd_bf16 if bf16_out else lib().quaff_linear_fwd
    _check(fn(_ptr(Xq), _ptr(delta_x), _ptr(xq_O), t, _ptr(Wq_packed), _ptr(delta_w), c_in, c_out,
                                  _ptr(what_int), _ptr(delta_what), n_outlier, _ptr(X),
                                  0 if X is None else X.stride(0), _ptr(lora_A), _ptr(lora_B), lora_rank,
                                  float(lora_scale), _ptr(Y), Y.stride(0), _ptr(workspace),
                                  0 if workspace is None else workspace.numel() * workspace.element_size(), _stream()))


def linear_fwd_acc(Xq, xq_O, Wq_packed, c_in, c_out, what_int, n_outlier, acc1, acc2):
    t = Xq.shape[0]
    _check(lib().quaff_linear_fwd_acc(_ptr(Xq), _ptr(xq_O), t, _ptr(Wq_packed), c_in, c_out, _ptr(what_int),
                                      n_outlier, _ptr(acc1), _ptr(acc2), _stream()))


def linear_bwd_dx(dY, Wq_packed, delta_w, c_in, c_out, lora_A, lora_B, lora_rank, lora_scale, dX, workspace,
                  bf16_out=False):
    t = dY.shape[0]
    fn = lib().quaff_linear_bwd_dx_bf16 if bf16_out else lib().quaff_linear_bwd_dx
    _check(fn(_ptr(dY), t, dY.stride(0), _ptr(Wq_packed), _ptr(delta_w), c_in, c_out,
                                     _ptr(lora_A), _ptr(lora_B), lora_rank, float(lora_scale), _ptr(dX), dX.stride(0),
                                     _ptr(workspace),
                                     0 if workspace is None else workspace.numel() * workspace.element_size(),
                                     _stream()))


def lora_bwd_workspace_bytes(t, c_in, c_out, lora_rank) -> int:
    return int(lib().quaff_lora_bwd_workspace_bytes(t, c_in, c_out, lora_rank))


def lora_bwd_weights(X, dY, lora_A, lora_B, lora_rank, lora_scale, dA, dB, workspace):
    t, c_in, c_out = X.shape[0], X.shape[1], dY.shape[1]
    _check(lib().quaff_lora_bwd_weights(_ptr(X), X.stride(0), _ptr(dY), dY.stride(0), t, c_in, c_out, _ptr(lora_A),
                                        _ptr(lora_B), lora_rank, float(lora_scale), _ptr(dA), _ptr(dB),
                                        _ptr(workspace),
                                        0 if workspace is None else workspace.numel() * workspace.element_size(),
                                        _stream()))


def bwd_step_workspace_bytes(t, c_in, c_out, lora_rank) -> int:
    return int(lib().quaff_bwd_step_workspace_bytes(t, c_in, c_out, lora_rank))


class SideStream:
    """A second stream and two events (timing disabled) for quaff_linear_bwd_step, owned by the caller."""

    def __init__(self):
        import torch
        self.stream = torch.cuda.Stream()
        self.fork, self.join = torch.cuda.Event(), torch.cuda.Event()
        for ev in (self.fork, self.join):   # torch creates the underlying event at its first record
            ev.record(self.stream)
        self.stream.synchronize()

    def handles(self):
        return self.stream.cuda_stream, self.fork.cuda_event, self.join.cuda_event


def linear_bwd_step(dY, X, Wq_packed, delta_w, c_in, c_out, lora_A, lora_B, lora_rank, lora_scale, dX, dA, dB, workspace,
                    side=None):
    """side: a SideStream (the weight gradients then run beside the input-gradient product) or None."""
    t = dY.shape[0]
    hs, hf, hj = side.handles() if side is not None else (None, None, None)
    _check(lib().quaff_linear_bwd_step(_ptr(dY), t, dY.stride(0), _ptr(X), X.stride(0), _ptr(Wq_packed), _ptr(delta_w),
                                       c_in, c_out, _ptr(lora_A), _ptr(lora_B), lora_rank, float(lora_scale), _ptr(dX),
                                       dX.stride(0), _ptr(dA), _ptr(dB), _ptr(workspace),
                                       0 if workspace is None else workspace.numel() * workspace.element_size(),
                                       _stream(), hs, hf, hj))


def bwd_dx_outlier_workspace_bytes(t, c_out) -> int:
    return int(lib().quaff_bwd_dx_outlier_workspace_bytes(t, c_out))


def bwd_dx_outlier_exact(dY, c_in, O, W_O, lora_A, lora_B, lora_rank, lora_scale, dX, workspace):
    t, c_out = dY.shape[0], dY.shape[1]
    n = 0 if O is None else O.numel()
    _check(lib().quaff_bwd_dx_outlier_exact(_ptr(dY), t, dY.stride(0), c_in, c_out, _ptr(O), n, _ptr(W_O),
                                            _ptr(lora_A), _ptr(lora_B), lora_rank, float(lora_scale), _ptr(dX),
                                            dX.stride(0), _ptr(workspace),
                                            0 if workspace is None else workspace.numel() * workspace.element_size(),
                                            _stream()))


def calibrate_workspace_bytes(c_in, n_samples) -> int:
    return int(lib().quaff_calibrate_workspace_bytes(c_in, n_samples))


def calibrate_outliers(X, sample_offsets, ratio, budget, xi, O, n_outlier, workspace):
    t_total, c_in = X.shape[0], X.shape[1]
    _check(lib().quaff_calibrate_outliers(_ptr(X), t_total, c_in, X.stride(0), _ptr(sample_offsets),
                                          sample_offsets.numel() - 1, float(ratio), budget, _ptr(xi), _ptr(O),
                                          _ptr(n_outlier), _ptr(workspace),
                                          0 if workspace is None else workspace.numel() * workspace.element_size(),
                                          _stream()))


def fwd_step_workspace_bytes(t, c_in, c_out, n_outlier, lora_rank) -> int:
    return int(lib().quaff_fwd_step_workspace_bytes(t, c_in, c_out, n_outlier, lora_rank))


def linear_fwd_step(X, O, W_O, wmax_O, c_out, gamma, s_O, colscale, what_int, delta_what, cmax_out, Xq, delta_x, xq_O,
                    Wq_packed, delta_w, lora_A, lora_B, lora_rank, lora_scale, Y, workspace):
    t, c_in = X.shape[0], X.shape[1]
    n = 0 if O is None else O.numel()
    _check(lib().quaff_linear_fwd_step(_ptr(X), t, c_in, X.stride(0), _ptr(O), n, _ptr(W_O), _ptr(wmax_O), c_out,
                                       float(gamma), _ptr(s_O), _ptr(colscale), _ptr(what_int), _ptr(delta_what),
                                       _ptr(cmax_out), _ptr(Xq), _ptr(delta_x), _ptr(xq_O), _ptr(Wq_packed),
                                       _ptr(delta_w), _ptr(lora_A), _ptr(lora_B), lora_rank, float(lora_scale),
                                       _ptr(Y), Y.stride(0), _ptr(workspace),
                                       0 if workspace is None else workspace.numel() * workspace.element_size(),
                                       _stream()))


# ---- 4-bit microscaled layers and products grouped by expert -------------------------------------------------------

def _need(ok: bool):
    """A tensor that does not fit the call (its size or type; the library sees pointers only)."""
    if not ok:
        raise QuaffError(ERR_SHAPE)


def _where(t):
    """Index of the device that t lies on: the current one, whose stream the call uses."""
    import torch
    d = t.get_device()
    _need(d >= 0 and d == torch.cuda.current_device())
    return d


def _fits(t, d, dtype, numel):
    """t holds at least `numel` elements of that type one after the other, on device d."""
    return t is not None and t.dtype == dtype and t.get_device() == d and t.numel() >= numel and t.is_contiguous()


def _rows(t, d, dtype, cols, rows=None):
    """t is a matrix of `cols` columns (and `rows` rows) whose rows are contiguous, on device d."""
    if t.dtype != dtype or t.dim() != 2 or t.get_device() != d:
        return False
    n, c = t.shape
    return c == cols and (rows is None or n == rows) and (n == 0 or t.stride(1) == 1)


def _ld(t):
    """Leading dimension (what a matrix of at most one row says of it means nothing)."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _room(ws, d):
    _need(ws is None or (ws.get_device() == d and ws.is_contiguous()))
    return 0 if ws is None else ws.numel() * ws.element_size()


def _matrix(t):
    _need(t.dim() == 2)
    return t.shape


def _groups(offsets, d):
    import torch
    if offsets is None:
        return 0
    _need(offsets.dtype == torch.int64 and offsets.get_device() == d and offsets.dim() == 1 and offsets.is_contiguous())
    return offsets.numel() - 1


def mx4_padded(k: int) -> int:
    """As quaff_mx4_padded."""
    return 0 if k <= 0 else (k + 255) // 256 * 256


def mx4_quantize(X, codes, scales):
    import torch
    (rows, k), d = _matrix(X), _where(X)
    kp = mx4_padded(k)
    _need(_rows(X, d, torch.bfloat16, k) and _fits(codes, d, torch.uint8, rows * kp // 2) and _fits(scales, d, torch.uint8, rows * kp // 32))
    _check(lib().quaff_mx4_quantize(_ptr(X), rows, k, _ld(X), _ptr(codes), _ptr(scales), _stream()))


def mx4_dequantize(codes, scales, out):
    import torch
    (rows, k), d = _matrix(out), _where(out)
    kp = mx4_padded(k)
    _need(_rows(out, d, torch.bfloat16, k) and _fits(codes, d, torch.uint8, rows * kp // 2) and _fits(scales, d, torch.uint8, rows * kp // 32))
    _check(lib().quaff_mx4_dequantize(_ptr(codes), _ptr(scales), rows, k, _ptr(out), _ld(out), _stream()))


def mx4_prepare_weight(W, codes_fwd, scales_fwd, codes_bwd, scales_bwd):
    """W [c_in x c_out] or [groups x c_in x c_out] fp32, contiguous; either pair of copies may be None."""
    import torch
    _need(W.dim() in (2, 3))
    (c_in, c_out), d = W.shape[-2:], _where(W)
    n = W.shape[0] if W.dim() == 3 else 1
    _need(_fits(W, d, torch.float32, n * c_in * c_out))
    for codes, scales, rows, k in ((codes_fwd, scales_fwd, n * c_out, c_in), (codes_bwd, scales_bwd, n * c_in, c_out)):
        kp = mx4_padded(k)
        _need(codes is None or _fits(codes, d, torch.uint8, rows * kp // 2))
        _need(scales is None or _fits(scales, d, torch.uint8, rows * kp // 32))
    _check(lib().quaff_mx4_prepare_weight(_ptr(W), n, c_in, c_out, c_out, _ptr(codes_fwd), _ptr(scales_fwd), _ptr(codes_bwd), _ptr(scales_bwd),
                                          _stream()))


def check_group_offsets(offsets, t, result):
    """Enqueue the validity scan; `result` is a one-element int32 device tensor (0 = valid, else 1 + position)."""
    import torch
    _need(offsets is not None)
    d = _where(offsets)
    n = _groups(offsets, d)
    _need(_fits(result, d, torch.int32, 1))
    _check(lib().quaff_check_group_offsets(_ptr(offsets), n, t, _ptr(result), _stream()))


def mx4_linear_workspace_bytes(t, c_in, c_out, n_groups, lora_rank) -> int:
    return int(lib().quaff_mx4_linear_workspace_bytes(t, c_in, c_out, n_groups, lora_rank))


def _mx4_linear(fn, X, offsets, codes, scales, c_in, c_out, k, n, lora_A, lora_B, lora_rank, lora_scale, Y, workspace, bf16_out):
    import torch
    (t, _), d, bf16, u8 = _matrix(X), _where(X), torch.bfloat16, torch.uint8
    groups = _groups(offsets, d)
    e, kp = groups or 1, mx4_padded(k)
    _need(_rows(X, d, bf16, k) and _rows(Y, d, bf16 if bf16_out else torch.float32, n, t) and _fits(codes, d, u8, e * n * kp // 2) and
          _fits(scales, d, u8, e * n * kp // 32))
    _need(lora_rank == 0 or (_fits(lora_A, d, bf16, e * c_in * lora_rank) and _fits(lora_B, d, bf16, e * c_out * lora_rank)))
    _check(fn(_ptr(X), t, _ld(X), _ptr(offsets), groups, _ptr(codes), _ptr(scales), c_in, c_out, _ptr(lora_A), _ptr(lora_B), lora_rank,
              lora_scale, _ptr(Y), _ld(Y), _ptr(workspace), _room(workspace, d), _stream()))


def mx4_linear_fwd(X, offsets, codes, scales, c_in, c_out, lora_A, lora_B, lora_rank, lora_scale, Y, workspace, bf16_out=False):
    """offsets: int64 [groups + 1] device tensor, or None for a dense layer."""
    l = lib()
    _mx4_linear(l.quaff_mx4_linear_fwd_bf16 if bf16_out else l.quaff_mx4_linear_fwd, X, offsets, codes, scales, c_in, c_out, c_in, c_out,
                lora_A, lora_B, lora_rank, lora_scale, Y, workspace, bf16_out)


def mx4_linear_bwd_dx(dY, offsets, codes, scales, c_in, c_out, lora_A, lora_B, lora_rank, lora_scale, dX, workspace, bf16_out=False):
    l = lib()
    _mx4_linear(l.quaff_mx4_linear_bwd_dx_bf16 if bf16_out else l.quaff_mx4_linear_bwd_dx, dY, offsets, codes, scales, c_in, c_out, c_out, c_in,
                lora_A, lora_B, lora_rank, lora_scale, dX, workspace, bf16_out)


def grouped_linear_workspace_bytes(t, c_in, c_out, n_groups) -> int:
    return int(lib().quaff_grouped_linear_workspace_bytes(t, c_in, c_out, n_groups))


def _grouped_rows(fn, X, offsets, W, gradient, scale, Y, workspace, bf16_out, accumulate):
    import torch
    (t, _), d = _matrix(X), _where(X)
    groups = _groups(offsets, d)
    _need(W.dim() == 3 and W.shape[0] == groups and _fits(W, d, torch.bfloat16, 0))
    _, c_in, c_out = W.shape
    k, n = (c_out, c_in) if gradient else (c_in, c_out)
    _need(_rows(X, d, torch.bfloat16, k) and _rows(Y, d, torch.bfloat16 if bf16_out else torch.float32, n, t) and not (bf16_out and accumulate))
    how = () if bf16_out else (1 if accumulate else 0,)
    _check(fn(_ptr(X), t, _ld(X), _ptr(offsets), groups, _ptr(W), c_in, c_out, scale, *how, _ptr(Y), _ld(Y), _ptr(workspace),
              _room(workspace, d), _stream()))


def grouped_linear_fwd(X, offsets, W, scale, Y, workspace, bf16_out=False, accumulate=False):
    """W [groups x c_in x c_out] bf16; accumulate adds to an fp32 Y."""
    l = lib()
    _grouped_rows(l.quaff_grouped_linear_fwd_bf16 if bf16_out else l.quaff_grouped_linear_fwd, X, offsets, W, False, scale, Y, workspace,
                  bf16_out, accumulate)


def grouped_linear_bwd_dx(dY, offsets, W, scale, dX, workspace, bf16_out=False, accumulate=False):
    l = lib()
    _grouped_rows(l.quaff_grouped_linear_bwd_dx_bf16 if bf16_out else l.quaff_grouped_linear_bwd_dx, dY, offsets, W, True, scale, dX, workspace,
                  bf16_out, accumulate)


def grouped_linear_bwd_dw(X, dY, offsets, scale, dW, workspace):
    """dW [groups x c_in x c_out] fp32, overwritten."""
    import torch
    (t, c_in), (_, c_out), d = _matrix(X), _matrix(dY), _where(X)
    groups = _groups(offsets, d)
    _need(_rows(X, d, torch.bfloat16, c_in) and _rows(dY, d, torch.bfloat16, c_out, t) and tuple(dW.shape) == (groups, c_in, c_out) and
          _fits(dW, d, torch.float32, 0))
    _check(lib().quaff_grouped_linear_bwd_dw(_ptr(X), _ld(X), _ptr(dY), _ld(dY), t, _ptr(offsets), groups, c_in, c_out, scale, _ptr(dW),
                                             _ptr(workspace), _room(workspace, d), _stream()))


def debug_group_form(what: str, t: int, c_in: int, c_out: int, n_groups: int) -> str:
    """Kernel form of "mx4_fwd", "mx4_dx", "fwd", "dx" or "dw" at these sizes (n_groups 0: a dense 4-bit layer)."""
    return lib().quaff_debug_group_form(("mx4_fwd", "mx4_dx", "fwd", "dx", "dw").index(what), t, c_in, c_out, n_groups).decode()


def debug_grid_wait_ticks(ticks: int) -> int:
    """Set (ticks >= 0) or read (ticks < 0) the bound of the one-launch forward preparation's grid-wide wait."""
    return int(lib().quaff_debug_grid_wait_ticks(ticks))


def debug_product_form(t: int, c_in: int, c_out: int, n_outlier: int, lora_rank: int, how: int) -> str:
    """Kernel form of a layer's product at these sizes (how: 0 forward, 1 with the smallest workspace; 2, 3 the input
    gradient; 4 the input gradient beside a second stream)."""
    return lib().quaff_debug_product_form(t, c_in, c_out, n_outlier, lora_rank, how).decode()


def linear_bwd_dx_acc(dY, Wq_packed, delta_w, c_in, c_out, Gq, delta_g, acc):
    t = dY.shape[0]
    _check(lib().quaff_linear_bwd_dx_acc(_ptr(dY), t, dY.stride(0), _ptr(Wq_packed), _ptr(delta_w), c_in, c_out,
                                         _ptr(Gq), _ptr(delta_g), _ptr(acc), _stream()))


def profile_enable(on: bool):
    _check(lib().quaff_profile_enable(1 if on else 0))


def profile_launches():
    """[(kernel kind name, milliseconds), ...] of every launch recorded since profile_enable(True), in order."""
    n = int(lib().quaff_profile_collect())
    if n < 0:
        raise QuaffError(ERR_HIP)
    out = []
    kind, ms = C.c_int(), C.c_float()
    for i in range(n):
        _check(lib().quaff_profile_launch(i, C.byref(kind), C.byref(ms)))
        out.append((lib().quaff_profile_kind_name(kind.value).decode(), float(ms.value)))
    return out


def microbench_mfma_i8(random_operands: bool):
    """(TOP/s, shader clock MHz) of a register-only INT8 MFMA loop on the whole chip."""
    tops, mhz = C.c_double(), C.c_double()
    _check(lib().quaff_microbench_mfma_i8(1 if random_operands else 0, C.byref(tops), C.byref(mhz)))
    return tops.value, mhz.value


def microbench_copy(nbytes: int = 1 << 30) -> float:
    """GB/s (read + write) of a streaming device copy."""
    gbs = C.c_double()
    _check(lib().quaff_microbench_copy(nbytes, C.byref(gbs)))
    return gbs.value
