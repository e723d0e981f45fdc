"""ctypes binding of libnq_binlr.so -- argument marshalling only.

Every function has the name of the C entry point it calls (see
``include/nq_binlr.h``).  Device buffers are passed as ``torch`` CUDA tensors
(or raw integer addresses); the stream defaults to torch's current stream.
Nothing is computed here, and there is no fallback: if the shared library has
not been built, importing symbols from it raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence

import numpy as np

NQ_OK = 0
NQ_E_INVALID_ARG, NQ_E_SHAPE, NQ_E_ALIGN, NQ_E_NULL, NQ_E_UNSUPPORTED, NQ_E_HIP, NQ_E_TIMEOUT = -1, -2, -3, -4, -5, -6, -7
NQ_I8, NQ_F32, NQ_F16, NQ_BF16, NQ_F64 = 0, 1, 2, 3, 4
NQ_FLAG_DEFAULT, NQ_FLAG_DECODE_VALU, NQ_FLAG_NO_PREFILL = 0, 1, 2
NQ_MAX_DIM = 65536
NQ_DECODE_MAX_BATCH = 8
NQ_PREFILL_MIN_BATCH = 9
NQ_STATIC_SCRATCH_BYTES = 2 << 20

DTYPE_BY_NAME = {"f32": NQ_F32, "f16": NQ_F16, "bf16": NQ_BF16, "i8": NQ_I8}

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libnq_binlr.so")
_lib = None


class NQError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"nq status {status}: {message}")
        self.status = status


def lib() -> ctypes.CDLL:
    """The loaded shared library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2602_06694_amd.build` "
                              "(there is no CPU fallback)")
        # torch first: it brings its own copy of the HIP runtime, and a process must hold one.  Loaded the other way
        # round (this library, then torch) the system's copy comes in first and torch then finds no GPU.
        import torch  # noqa: F401
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, ci, u32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_uint32
        L.nq_packed_words.argtypes = [i64, i64]; L.nq_packed_words.restype = ctypes.c_size_t
        L.nq_pack_signs.argtypes = [vp, ci, i64, i64, vp]; L.nq_pack_signs.restype = ci
        L.nq_unpack_signs.argtypes = [vp, i64, i64, vp]; L.nq_unpack_signs.restype = ci
        L.nq_binlr_create.argtypes = [ctypes.POINTER(vp), i64, i64, i64, vp, vp, vp, vp, ci, ci, u32]
        L.nq_binlr_create.restype = ci
        L.nq_pack_signs_device.argtypes = [vp, ci, i64, i64, vp, vp, vp]; L.nq_pack_signs_device.restype = ci
        L.nq_binlr_create_from_device.argtypes = [ctypes.POINTER(vp), i64, i64, i64, vp, vp, vp, vp, ci, ci, u32]
        L.nq_binlr_create_from_device.restype = ci
        L.nq_binlr_reserve.argtypes = [vp, ci]; L.nq_binlr_reserve.restype = ci
        L.nq_binlr_reserved.argtypes = [vp, ctypes.POINTER(ci), ctypes.POINTER(ctypes.c_size_t)]; L.nq_binlr_reserved.restype = ci
        L.nq_binlr_forward.argtypes = [vp, vp, vp, ci, vp]; L.nq_binlr_forward.restype = ci
        L.nq_binlr_forward_static.argtypes = [vp, vp, vp, ci, vp]; L.nq_binlr_forward_static.restype = ci
        L.nq_binlr_forward_exact.argtypes = [vp, vp, vp, ci, vp]; L.nq_binlr_forward_exact.restype = ci
        L.nq_set_option.argtypes = [ctypes.c_char_p, ci]; L.nq_set_option.restype = ci
        L.nq_get_option.argtypes = [ctypes.c_char_p, ctypes.POINTER(ci)]; L.nq_get_option.restype = ci
        L.nq_binlr_forward_many.argtypes = [vp, vp, vp, ci, ci, vp]; L.nq_binlr_forward_many.restype = ci
        L.nq_plan_create.argtypes = [ctypes.POINTER(vp), vp, vp, vp, ci, ci]; L.nq_plan_create.restype = ci
        L.nq_plan_forward.argtypes = [vp, vp]; L.nq_plan_forward.restype = ci
        L.nq_plan_forward_timed.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_float)]; L.nq_plan_forward_timed.restype = ci
        L.nq_binlr_forward_unscaled.argtypes = [vp, vp, vp, ci, vp]; L.nq_binlr_forward_unscaled.restype = ci
        L.nq_binlr_forward_transposed_unscaled.argtypes = [vp, vp, vp, ci, vp]; L.nq_binlr_forward_transposed_unscaled.restype = ci
        L.nq_binlr_backward_input.argtypes = [vp, vp, vp, ci, vp]; L.nq_binlr_backward_input.restype = ci
        L.nq_scale_grad.argtypes = [vp, ci, vp, ci, ci, ctypes.c_int64, vp, vp]; L.nq_scale_grad.restype = ci
        L.nq_binlr_set_mid_scale.argtypes = [vp, vp]; L.nq_binlr_set_mid_scale.restype = ci
        L.nq_probe_hbm_read.argtypes = [ctypes.c_size_t, ci, ci, ctypes.POINTER(ctypes.c_double)]; L.nq_probe_hbm_read.restype = ci
        L.nq_probe_mfma.argtypes = [ci, ctypes.POINTER(ctypes.c_double)]; L.nq_probe_mfma.restype = ci
        L.nq_plan_schedules.argtypes = [vp, ctypes.POINTER(ctypes.c_int)]; L.nq_plan_schedules.restype = ci
        L.nq_plan_destroy.argtypes = [vp]; L.nq_plan_destroy.restype = ci
        L.nq_binlr_destroy.argtypes = [vp]; L.nq_binlr_destroy.restype = ci
        L.nq_binlr_weight_bytes.argtypes = [vp]; L.nq_binlr_weight_bytes.restype = ctypes.c_size_t
        L.nq_binlr_export_words.argtypes = [vp, vp, vp]; L.nq_binlr_export_words.restype = ci
        L.nq_binlr_read_intermediate.argtypes = [vp, vp, ci]; L.nq_binlr_read_intermediate.restype = ci
        L.nq_exec_create.argtypes = [ctypes.POINTER(vp), vp, vp, vp, vp, ci]; L.nq_exec_create.restype = ci
        L.nq_exec_forward.argtypes = [vp, vp]; L.nq_exec_forward.restype = ci
        L.nq_exec_status.argtypes = [vp, vp]; L.nq_exec_status.restype = ci
        L.nq_exec_info.argtypes = [vp, ctypes.POINTER(ci), ctypes.POINTER(ci), ctypes.POINTER(ctypes.c_size_t)]; L.nq_exec_info.restype = ci
        L.nq_exec_destroy.argtypes = [vp]; L.nq_exec_destroy.restype = ci
        for f in (L.nq_exec_plan_tasks, L.nq_exec_plan_lists):
            f.argtypes = [vp, vp, vp, vp, ci, ci, vp, ci, ctypes.POINTER(ci)]; f.restype = ci
        L.nq_debug_slab_count.argtypes = []; L.nq_debug_slab_count.restype = ci
        dbl, szp = ctypes.c_double, ctypes.POINTER(ctypes.c_size_t)
        L.nq_lb_admm_workspace_bytes.argtypes = [i64, i64, i64, szp]; L.nq_lb_admm_workspace_bytes.restype = ci
        L.nq_lb_admm.argtypes = [vp, i64, i64, i64, vp, vp, ci, dbl, dbl, dbl, ci, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.nq_lb_admm.restype = ci
        L.nq_lb_admm_balance.argtypes = [vp, vp, i64, vp, vp, i64, i64, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.nq_lb_admm_balance.restype = ci
        L.nq_dgemm.argtypes = [ci, ci, i64, i64, i64, dbl, vp, i64, vp, i64, dbl, vp, i64, vp]; L.nq_dgemm.restype = ci
        vpp = ctypes.POINTER(vp)
        L.nq_kv_create.argtypes = [vpp, vp, vp, ci, ci, ci, ci, i64, i64, i64, i64]
        L.nq_kv_copy_pages.argtypes = [vp, ci, vp, vp, ci, vp]
        L.nq_kv_compact.argtypes = [vp, ci, vp, vp, i64, vp, i64, vp, ci, vp]
        L.nq_rope_freqs.argtypes = [ci, ci, dbl, dbl, dbl, dbl, dbl, vp, ctypes.POINTER(dbl)]
        L.nq_rope_create.argtypes = [vpp, ci, ci, ci, ci, ci, vp, dbl, dbl, dbl, ci, ci]
        L.nq_rope_forward.argtypes = [vp, vp, i64, vp, i64, vp, vp, vp, ci, vp, i64, vp, i64, vp]
        L.nq_rope_cache.argtypes = [vp, vp, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, ci, vp, i64, vp]
        L.nq_rope_backward_workspace_bytes.argtypes = [vp, ci, szp]
        L.nq_rope_backward.argtypes = [vp, vp, i64, vp, i64, vp, vp, vp, ci, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, ctypes.c_size_t, vp]
        L.nq_attn_create.argtypes = [vpp, vp, ci, dbl, dbl, ci]
        L.nq_attn_workspace_bytes.argtypes = [vp, ci, ci, szp]
        L.nq_attn_forward.argtypes = [vp, vp, i64, vp, vp, vp, i64, vp, ci, ci, ci, vp, i64, vp, vp, ctypes.c_size_t, vp]
        L.nq_sample_workspace_bytes.argtypes = [ci, i64, szp]
        L.nq_sample.argtypes = [vp, ci, ci, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        for f in (L.nq_kv_destroy, L.nq_rope_destroy, L.nq_attn_destroy):
            f.argtypes = [vp]
        for f in (L.nq_kv_create, L.nq_kv_copy_pages, L.nq_kv_compact, L.nq_kv_destroy, L.nq_rope_freqs, L.nq_rope_create, L.nq_rope_forward, L.nq_rope_cache,
                  L.nq_rope_backward_workspace_bytes, L.nq_rope_backward, L.nq_rope_destroy, L.nq_attn_create, L.nq_attn_workspace_bytes, L.nq_attn_forward,
                  L.nq_attn_destroy, L.nq_sample_workspace_bytes, L.nq_sample):
            f.restype = ci
        L.nq_status_string.argtypes = [ci]; L.nq_status_string.restype = ctypes.c_char_p
        L.nq_last_error_string.argtypes = []; L.nq_last_error_string.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _check(status: int) -> None:
    if status != NQ_OK:
        L = lib()
        raise NQError(status, f"{L.nq_status_string(status).decode()}: {L.nq_last_error_string().decode()}")


def _np_ptr(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(ctypes.c_void_p)


def _dev_ptr(t) -> Optional[int]:
    """Address of a device buffer: torch tensor, int, or None."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("expected a device (cuda) tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return t.data_ptr()


# (current stream's address of a device, current device) once torch's CUDA side is up; a forked child starts over, as torch does
_raw_stream = None


def _forget_raw_stream() -> None:
    global _raw_stream
    _raw_stream = None


os.register_at_fork(after_in_child=_forget_raw_stream)


def _current_stream() -> Optional[int]:
    """torch.cuda.current_stream() builds a stream object on every call: 2.9 us, as much as a launch costs.  The address alone takes 0.2
    (a lone 1024 x 1024 layer, two launches: 8.8 -> 6.3 us of host time per call).  The first call goes the public way, which initialises CUDA."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        s = torch.cuda.current_stream().cuda_stream
        raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        if raw is not None and device is not None and raw(device()) == s:
            _raw_stream = (raw, device)
        return s or None
    return _raw_stream[0](_raw_stream[1]()) or None


def _stream(stream) -> Optional[int]:
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def nq_status_string(status: int) -> str:
    return lib().nq_status_string(status).decode()


def nq_last_error_string() -> str:
    return lib().nq_last_error_string().decode()


def nq_packed_words(rows: int, cols: int) -> int:
    return int(lib().nq_packed_words(rows, cols))


def nq_pack_signs(signs: np.ndarray, dtype: Optional[int] = None) -> np.ndarray:
    """signs: host [rows, cols]; int8 (+-1), float32, float16, or uint16 holding bf16 bits
    (then pass dtype=NQ_BF16).  Returns canonical uint32 [rows, ceil(cols/32)]."""
    if signs.ndim != 2:
        raise ValueError("signs must be 2-D")
    if dtype is None:
        dtype = {np.dtype(np.int8): NQ_I8, np.dtype(np.float32): NQ_F32, np.dtype(np.float16): NQ_F16}.get(signs.dtype)
        if dtype is None:
            raise ValueError(f"cannot infer NQ dtype from {signs.dtype}")
    a = np.ascontiguousarray(signs)
    rows, cols = a.shape
    out = np.empty((rows, (cols + 31) // 32), dtype=np.uint32)
    _check(lib().nq_pack_signs(_np_ptr(a), dtype, rows, cols, _np_ptr(out)))
    return out


def nq_unpack_signs(words: np.ndarray, cols: int) -> np.ndarray:
    w = np.ascontiguousarray(words, dtype=np.uint32)
    rows = w.shape[0]
    if w.shape != (rows, (cols + 31) // 32):
        raise ValueError("words has the wrong shape")
    out = np.empty((rows, cols), dtype=np.int8)
    _check(lib().nq_unpack_signs(_np_ptr(w), rows, cols, _np_ptr(out)))
    return out


def nq_binlr_create(d_out: int, d_in: int, r: int, U_words: np.ndarray, V_words: np.ndarray,
                    s_out: np.ndarray, s_in: np.ndarray, x_dtype: int, y_dtype: int = NQ_F32,
                    flags: int = NQ_FLAG_DEFAULT) -> int:
    """Returns the opaque handle (an integer address)."""
    wpr = (r + 31) // 32
    U = np.ascontiguousarray(U_words, dtype=np.uint32)
    V = np.ascontiguousarray(V_words, dtype=np.uint32)
    so = np.ascontiguousarray(s_out, dtype=np.float16)
    si = np.ascontiguousarray(s_in, dtype=np.float16)
    if U.shape != (d_out, wpr) or V.shape != (d_in, wpr) or so.shape != (d_out,) or si.shape != (d_in,):
        raise ValueError("argument shapes do not match d_out, d_in, r")
    h = ctypes.c_void_p()
    _check(lib().nq_binlr_create(ctypes.byref(h), d_out, d_in, r, _np_ptr(U), _np_ptr(V), _np_ptr(so), _np_ptr(si),
                                 x_dtype, y_dtype, flags))
    return h.value


def nq_pack_signs_device(d_signs, dtype: int, rows: int, cols: int, d_words, d_invalid=None, stream=None) -> None:
    """d_signs / d_words / d_invalid: device arrays (anything with data_ptr()) or raw addresses."""
    _check(lib().nq_pack_signs_device(_dev_ptr(d_signs), dtype, rows, cols, _dev_ptr(d_words),
                                      _dev_ptr(d_invalid) if d_invalid is not None else None, _stream(stream)))


def nq_binlr_create_from_device(d_out: int, d_in: int, r: int, d_U_words, d_V_words, d_s_out, d_s_in,
                                x_dtype: int, y_dtype: int = NQ_F32, flags: int = NQ_FLAG_DEFAULT) -> int:
    """All four inputs are device arrays: canonical words (uint32 / int32 storage) and fp16 scales."""
    h = ctypes.c_void_p()
    _check(lib().nq_binlr_create_from_device(ctypes.byref(h), d_out, d_in, r, _dev_ptr(d_U_words), _dev_ptr(d_V_words),
                                             _dev_ptr(d_s_out), _dev_ptr(d_s_in), x_dtype, y_dtype, flags))
    return h.value


def nq_binlr_set_mid_scale(h: int, s_mid: Optional[np.ndarray]) -> None:
    """s_mid: r fp16 values (numpy float16 or their uint16 bits), or None to remove the scale."""
    if s_mid is None:
        _check(lib().nq_binlr_set_mid_scale(h, None))
        return
    a = np.ascontiguousarray(s_mid)
    if a.dtype == np.float16:
        a = a.view(np.uint16)
    if a.dtype != np.uint16:
        raise TypeError("s_mid must be float16 (or uint16 bits)")
    _check(lib().nq_binlr_set_mid_scale(h, a.ctypes.data_as(ctypes.c_void_p)))


def nq_binlr_reserve(h: int, max_batch: int) -> None:
    _check(lib().nq_binlr_reserve(h, max_batch))


def nq_binlr_reserved(h: int):
    """(largest batch that allocates nothing, bytes of the dense path's workspace)."""
    b, n = ctypes.c_int(), ctypes.c_size_t()
    _check(lib().nq_binlr_reserved(h, ctypes.byref(b), ctypes.byref(n)))
    return int(b.value), int(n.value)


def nq_binlr_forward(h: int, x, y, batch: int, stream=None) -> None:
    _check(lib().nq_binlr_forward(h, _dev_ptr(x), _dev_ptr(y), batch, _stream(stream)))


def nq_binlr_forward_static(h: int, x, y, batch: int, stream=None) -> None:
    _check(lib().nq_binlr_forward_static(h, _dev_ptr(x), _dev_ptr(y), batch, _stream(stream)))


def nq_binlr_forward_exact(h: int, x, y, batch: int, stream=None) -> None:
    _check(lib().nq_binlr_forward_exact(h, _dev_ptr(x), _dev_ptr(y), batch, _stream(stream)))


def nq_set_option(name: str, value: Optional[int]) -> None:
    """value None (or negative) restores the option's default."""
    _check(lib().nq_set_option(name.encode(), -1 if value is None else int(value)))


def nq_get_option(name: str) -> int:
    v = ctypes.c_int()
    _check(lib().nq_get_option(name.encode(), ctypes.byref(v)))
    return int(v.value)


def nq_binlr_forward_unscaled(h: int, x, z, batch: int, stream=None) -> None:
    _check(lib().nq_binlr_forward_unscaled(h, _dev_ptr(x), _dev_ptr(z), batch, _stream(stream)))


def nq_binlr_forward_transposed_unscaled(h: int, g, w, batch: int, stream=None) -> None:
    _check(lib().nq_binlr_forward_transposed_unscaled(h, _dev_ptr(g), _dev_ptr(w), batch, _stream(stream)))


def nq_binlr_backward_input(h: int, g, dx, batch: int, stream=None) -> None:
    _check(lib().nq_binlr_backward_input(h, _dev_ptr(g), _dev_ptr(dx), batch, _stream(stream)))


def nq_scale_grad(a, a_dtype: int, b, b_dtype: int, batch: int, n: int, out, stream=None) -> None:
    _check(lib().nq_scale_grad(_dev_ptr(a), a_dtype, _dev_ptr(b), b_dtype, batch, n, _dev_ptr(out), _stream(stream)))


def _ptr_array(vals: Sequence[Optional[int]]):
    arr = (ctypes.c_void_p * len(vals))(*vals)
    return arr


def nq_binlr_forward_many(hs: Sequence[int], xs: Sequence, ys: Sequence, batch: int, stream=None) -> None:
    n = len(hs)
    if len(xs) != n or len(ys) != n:
        raise ValueError("hs, xs, ys must have the same length")
    _check(lib().nq_binlr_forward_many(_ptr_array(list(hs)), _ptr_array([_dev_ptr(x) for x in xs]),
                                       _ptr_array([_dev_ptr(y) for y in ys]), n, batch, _stream(stream)))


def nq_plan_create(hs: Sequence[int], xs: Sequence, ys: Sequence, batch: int) -> int:
    n = len(hs)
    if len(xs) != n or len(ys) != n:
        raise ValueError("hs, xs, ys must have the same length")
    p = ctypes.c_void_p()
    _check(lib().nq_plan_create(ctypes.byref(p), _ptr_array(list(hs)), _ptr_array([_dev_ptr(x) for x in xs]),
                                _ptr_array([_dev_ptr(y) for y in ys]), n, batch))
    return p.value


def nq_exec_create(hs: Sequence[int], xs: Sequence, ys: Sequence, level_of: Sequence[int]) -> int:
    n = len(hs)
    if len(xs) != n or len(ys) != n or len(level_of) != n:
        raise ValueError("hs, xs, ys, level_of must have the same length")
    e = ctypes.c_void_p()
    lv = (ctypes.c_int * n)(*[int(v) for v in level_of])
    _check(lib().nq_exec_create(ctypes.byref(e), _ptr_array(list(hs)), _ptr_array([_dev_ptr(x) for x in xs]),
                                _ptr_array([_dev_ptr(y) for y in ys]), lv, n))
    return e.value


def nq_exec_forward(e: int, stream=None) -> None:
    _check(lib().nq_exec_forward(e, _stream(stream)))


def nq_exec_status(e: int, stream=None) -> None:
    """Waits for the stream; raises NQError(NQ_E_TIMEOUT) if a wait inside a launch gave up."""
    _check(lib().nq_exec_status(e, _stream(stream)))


def nq_exec_info(e: int):
    """(workgroups, tasks, LDS bytes per workgroup)."""
    a, b, c = ctypes.c_int(), ctypes.c_int(), ctypes.c_size_t()
    _check(lib().nq_exec_info(e, ctypes.byref(a), ctypes.byref(b), ctypes.byref(c)))
    return int(a.value), int(b.value), int(c.value)


def nq_exec_destroy(e: Optional[int]) -> None:
    _check(lib().nq_exec_destroy(e))


def _exec_plan(call, words: int, d_out, d_in, r, level_of, n_workgroups: int) -> np.ndarray:
    n = len(d_out)
    a = [np.ascontiguousarray(v, dtype=np.int64) for v in (d_out, d_in, r)]
    lv = np.ascontiguousarray(level_of, dtype=np.int32)
    cnt = ctypes.c_int()
    _check(call(_np_ptr(a[0]), _np_ptr(a[1]), _np_ptr(a[2]), _np_ptr(lv), n, n_workgroups, None, 0, ctypes.byref(cnt)))
    out = np.zeros((cnt.value, words), dtype=np.int32)
    _check(call(_np_ptr(a[0]), _np_ptr(a[1]), _np_ptr(a[2]), _np_ptr(lv), n, n_workgroups, _np_ptr(out), cnt.value, ctypes.byref(cnt)))
    return out


def nq_exec_plan_lists(d_out: Sequence[int], d_in: Sequence[int], r: Sequence[int], level_of: Sequence[int],
                       n_workgroups: int) -> np.ndarray:
    """Host only: int32 [n_tasks, 9] = workgroup, phase, layer, stage, first row block, row blocks, waves per row block, first bit plane,
    bit planes (0: whole row blocks): the lists that nq_exec_create builds."""
    return _exec_plan(lib().nq_exec_plan_lists, 9, d_out, d_in, r, level_of, n_workgroups)


def nq_exec_plan_tasks(d_out: Sequence[int], d_in: Sequence[int], r: Sequence[int], level_of: Sequence[int],
                       n_workgroups: int) -> np.ndarray:
    """Host only: int32 [n_tasks, 7] = workgroup, phase, layer, stage, first row block, row blocks, waves per row block; a row block
    that is dealt out by bit planes once."""
    return _exec_plan(lib().nq_exec_plan_tasks, 7, d_out, d_in, r, level_of, n_workgroups)


def nq_plan_forward(p: int, stream=None) -> None:
    _check(lib().nq_plan_forward(p, _stream(stream)))


def nq_plan_forward_timed(p: int, stream=None) -> List[float]:
    ms = (ctypes.c_float * 4)()
    _check(lib().nq_plan_forward_timed(p, _stream(stream), ms))
    return [float(v) for v in ms]


def nq_plan_schedules(p: int) -> List[int]:
    w = (ctypes.c_int * 2)()
    _check(lib().nq_plan_schedules(p, w))
    return [int(v) for v in w]


def nq_probe_hbm_read(nbytes: int, iters: int = 10, prewarm_ms: int = 50) -> float:
    out = ctypes.c_double()
    _check(lib().nq_probe_hbm_read(nbytes, iters, prewarm_ms, ctypes.byref(out)))
    return float(out.value)


def nq_probe_mfma(dtype: int) -> float:
    out = ctypes.c_double()
    _check(lib().nq_probe_mfma(dtype, ctypes.byref(out)))
    return float(out.value)


def nq_plan_destroy(p: Optional[int]) -> None:
    _check(lib().nq_plan_destroy(p))


def nq_binlr_destroy(h: Optional[int]) -> None:
    _check(lib().nq_binlr_destroy(h))


def nq_debug_slab_count() -> int:
    return int(lib().nq_debug_slab_count())


def nq_binlr_weight_bytes(h: Optional[int]) -> int:
    return int(lib().nq_binlr_weight_bytes(h))


def nq_binlr_export_words(h: int, d_out: int, d_in: int, r: int):
    wpr = (r + 31) // 32
    U = np.empty((d_out, wpr), dtype=np.uint32)
    V = np.empty((d_in, wpr), dtype=np.uint32)
    _check(lib().nq_binlr_export_words(h, _np_ptr(U), _np_ptr(V)))
    return U, V


def nq_binlr_read_intermediate(h: int, r: int, batch: int) -> np.ndarray:
    t = np.empty((batch, r), dtype=np.float32)
    _check(lib().nq_binlr_read_intermediate(h, _np_ptr(t), batch))
    return t


# ---- latent-binary ADMM (include/nq_lb_admm.h) ----

NQ_ADMM_MAX_RANK = 8192
NQ_ADMM_MAX_DIM = 65536


def nq_lb_admm_workspace_bytes(n: int, m: int, r: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().nq_lb_admm_workspace_bytes(n, m, r, ctypes.byref(out)))
    return out.value


def nq_lb_admm(W, n: int, m: int, r: int, U0, V0, n_iters: int, rho_start: float, rho_end: float, lam: float, power_iters: int,
               U, V, Z_U, Z_V, Lambda_U, Lambda_V, workspace, workspace_bytes: int, stream=None) -> None:
    _check(lib().nq_lb_admm(_dev_ptr(W), n, m, r, _dev_ptr(U0), _dev_ptr(V0), n_iters, rho_start, rho_end, lam, power_iters,
                            _dev_ptr(U), _dev_ptr(V), _dev_ptr(Z_U), _dev_ptr(Z_V), _dev_ptr(Lambda_U), _dev_ptr(Lambda_V),
                            _dev_ptr(workspace), workspace_bytes, _stream(stream)))


def nq_lb_admm_balance(U, Lambda_U, n: int, V, Lambda_V, m: int, r: int, U_words, V_words, s1, s2, eta, workspace,
                       workspace_bytes: int, stream=None) -> None:
    _check(lib().nq_lb_admm_balance(_dev_ptr(U), _dev_ptr(Lambda_U), n, _dev_ptr(V), _dev_ptr(Lambda_V), m, r, _dev_ptr(U_words),
                                    _dev_ptr(V_words), _dev_ptr(s1), _dev_ptr(s2), _dev_ptr(eta), _dev_ptr(workspace), workspace_bytes,
                                    _stream(stream)))


def nq_dgemm(trans_a: int, trans_b: int, M: int, N: int, K: int, alpha: float, A, lda: int, B, ldb: int, beta: float, C, ldc: int,
             stream=None) -> None:
    _check(lib().nq_dgemm(trans_a, trans_b, M, N, K, alpha, _dev_ptr(A), lda, _dev_ptr(B), ldb, beta, _dev_ptr(C), ldc, _stream(stream)))


# ---- between the layers (include/nq_decoder.h) ----
# Tokens' tensors are [n_tokens, heads * head_dim] (or [n_tokens, heads, head_dim]) and may be columns of a wider tensor; numbers of
# tokens, sequences, rows and strides are read off the tensors, whose element types are checked against the calls'.

NQ_MAX_HEAD_DIM = 256
NQ_MAX_VOCAB = 1 << 20
NQ_ROPE_HALF, NQ_ROPE_INTERLEAVED = 0, 1
NQ_ROPE_PLAIN, NQ_ROPE_LINEAR, NQ_ROPE_BASE, NQ_ROPE_YARN, NQ_ROPE_BANDED = 0, 1, 2, 3, 4

_types = None


def _typed(t, kind: str, what: str) -> Optional[int]:
    """Address of a contiguous device tensor of one element type (or None)."""
    global _types
    if t is None:
        return None
    if _types is None:
        import torch
        _types = {"i32": (torch.int32, torch.uint32), "i64": (torch.int64,), "f32": (torch.float32,)}
    if t.dtype in _types[kind] and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    if t.dtype not in _types[kind]:
        raise ValueError(f"{what}: expected {kind}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{what}: expected a device (cuda) tensor")
    raise ValueError(f"{what}: expected a contiguous tensor")


def _rows(t, n_tokens: int, what: str):
    """(address, stride between tokens) of a tensor whose tokens' elements are contiguous."""
    if not t.is_cuda:
        raise ValueError(f"{what}: expected a device (cuda) tensor")
    shape, stride = t.shape, t.stride()
    if shape[0] != n_tokens:
        raise ValueError(f"{what}: {shape[0]} tokens, expected {n_tokens}")
    width = shape[-1]
    if len(shape) == 3:
        if stride[1] != width and shape[1] > 1:
            raise ValueError(f"{what}: the heads of a token must be contiguous")
        width *= shape[1]
    elif len(shape) != 2:
        raise ValueError(f"{what}: expected [tokens, heads * head_dim] or [tokens, heads, head_dim]")
    if stride[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{what}: the elements of a token must be contiguous")
    return t.data_ptr(), (stride[0] if n_tokens > 1 else width), width


def _extent(t) -> int:
    """Elements from a tensor's first to its last."""
    return 1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride())) if t.numel() else 0


_WIDTHS = {}            # handle of a cache, rope or attention -> widths and types that the tensors of a call have to match
_TORCH_TYPES = {}


def _torch_type(dtype: int):
    if not _TORCH_TYPES:
        import torch
        _TORCH_TYPES.update({NQ_F32: torch.float32, NQ_F16: torch.float16, NQ_BF16: torch.bfloat16})
    return _TORCH_TYPES.get(dtype)


def _tokens(t, n_tokens: int, width: int, dtype, what: str):
    """(address, stride between tokens), checked against the handle's head layout and type."""
    if t.dim() == 2 and t.dtype is dtype and t.is_cuda:                    # the usual tensor in as few calls as it takes
        (n, w), (stride, one) = t.shape, t.stride()
        if n == n_tokens and w == width and one == 1:
            return t.data_ptr(), (stride if n > 1 else w)
    p, stride, w = _rows(t, n_tokens, what)
    if w != width:
        raise ValueError(f"{what}: {w} elements a token, expected {width}")
    if t.dtype != dtype:
        raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
    return p, stride


def _same_length(n: int, what: str, *tensors) -> None:
    for t in tensors:
        if t is not None and t.numel() != n:
            raise ValueError(f"{what}: {t.numel()} values, expected {n}")


def nq_kv_create(k, v, dtype: int, kv_heads: int, head_dim: int, page_size: int, n_pages: int, page_stride: int = 0, slot_stride: int = 0,
                 head_stride: int = 0) -> int:
    """k, v: device tensors (or addresses) that hold the pages; strides in elements, 0, 0, 0: [n_pages][kv_heads][page_size][head_dim], for which tensors have to be
    contiguous.  Tensors have to hold all pages."""
    h = ctypes.c_void_p()
    kind, at, tensors = _torch_type(dtype), [], []
    for t in (k, v):
        if t is not None and not isinstance(t, int):
            if t.dtype != kind:
                raise ValueError(f"k, v: expected {kind}, got {t.dtype}")
            if not t.is_cuda:
                raise ValueError("k, v: expected device (cuda) tensors")
            tensors.append(t)
            t = t.data_ptr()
        at.append(t)
    _check(lib().nq_kv_create(ctypes.byref(h), at[0], at[1], dtype, kv_heads, head_dim, page_size, n_pages, page_stride, slot_stride, head_stride))
    packed = not (page_stride or slot_stride or head_stride)
    need = n_pages * kv_heads * page_size * head_dim if packed else \
        (n_pages - 1) * page_stride + (page_size - 1) * slot_stride + (kv_heads - 1) * head_stride + head_dim
    for t in tensors:
        whole = t.is_contiguous()
        if need > (t.numel() if whole else _extent(t)) or (packed and not whole):
            lib().nq_kv_destroy(h)
            raise ValueError(f"k, v: the pages take {need} elements, {tuple(t.shape)} of strides {t.stride()} are no room for them")
    _WIDTHS[h.value] = (head_dim, kind)
    return h.value


def nq_kv_destroy(kv: Optional[int]) -> None:
    _WIDTHS.pop(kv, None)
    _check(lib().nq_kv_destroy(kv))


def nq_kv_copy_pages(kvs: Sequence[int], src, dst, stream=None) -> None:
    n = src.numel()
    _same_length(n, "dst", dst)
    _check(lib().nq_kv_copy_pages(_ptr_array(kvs), len(kvs), _typed(src, "i32", "src"), _typed(dst, "i32", "dst"), n, _stream(stream)))


def nq_kv_compact(kvs: Sequence[int], ctx_len, page_table, path, path_len, stream=None) -> None:
    """page_table: [n_seqs, table_stride]; path: [n_seqs, path_stride]."""
    n = ctx_len.numel()
    _same_length(n, "path_len", path_len)
    if page_table.shape[0] != n or path.shape[0] != n:
        raise ValueError("page_table and path need a row for every sequence")
    _check(lib().nq_kv_compact(_ptr_array(kvs), len(kvs), _typed(ctx_len, "i32", "ctx_len"), _typed(page_table, "i32", "page_table"), page_table.shape[1],
                               _typed(path, "i32", "path"), path.shape[1], _typed(path_len, "i32", "path_len"), n, _stream(stream)))


def nq_rope_freqs(kind: int, rot_dim: int, base: float, factor: float = 1.0, trained_len: float = 1.0, low: float = 1.0, high: float = 32.0):
    """(binary64 frequencies [rot_dim / 2], magnitude)."""
    out, mag = np.empty(max(1, rot_dim // 2), dtype=np.float64), ctypes.c_double()
    _check(lib().nq_rope_freqs(kind, rot_dim, base, factor, trained_len, low, high, _np_ptr(out), ctypes.byref(mag)))
    return out, mag.value


def nq_rope_create(q_heads: int, kv_heads: int, head_dim: int, rot_dim: int, layout: int, inv_freq: Optional[np.ndarray], magnitude: float, eps: float,
                   weight_offset: float, in_dtype: int, out_dtype: int) -> int:
    f = None if inv_freq is None else np.ascontiguousarray(inv_freq, dtype=np.float64)
    if f is not None and f.size != rot_dim // 2:
        raise ValueError("inv_freq must hold rot_dim / 2 values")
    h = ctypes.c_void_p()
    _check(lib().nq_rope_create(ctypes.byref(h), q_heads, kv_heads, head_dim, rot_dim, layout, _np_ptr(f), magnitude, eps, weight_offset, in_dtype, out_dtype))
    _WIDTHS[h.value] = (q_heads * head_dim, kv_heads * head_dim, _torch_type(in_dtype), _torch_type(out_dtype), head_dim)
    return h.value


def nq_rope_destroy(r: Optional[int]) -> None:
    _WIDTHS.pop(r, None)
    _check(lib().nq_rope_destroy(r))


def nq_rope_forward(r: int, q, k, q_weight, k_weight, positions, q_out, k_out, stream=None) -> None:
    n = positions.numel()
    qw, kw, tin, tout, d = _WIDTHS[r]
    _same_length(d, "weight", q_weight, k_weight)
    _check(lib().nq_rope_forward(r, *_tokens(q, n, qw, tin, "q"), *_tokens(k, n, kw, tin, "k"), _typed(q_weight, "f32", "q_weight"), _typed(k_weight, "f32", "k_weight"),
                                 _typed(positions, "i32", "positions"), n, *_tokens(q_out, n, qw, tout, "q_out"), *_tokens(k_out, n, kw, tout, "k_out"), _stream(stream)))


def nq_rope_cache(r: int, kv: int, q, k, v, q_weight, k_weight, positions, slots, q_out, stream=None) -> None:
    n = positions.numel()
    qw, kw, tin, tout, d = _WIDTHS[r]
    _same_length(d, "weight", q_weight, k_weight)
    _same_length(n, "slots", slots)
    _check(lib().nq_rope_cache(r, kv, *_tokens(q, n, qw, tin, "q"), *_tokens(k, n, kw, tin, "k"), *_tokens(v, n, kw, tin, "v"), _typed(q_weight, "f32", "q_weight"),
                               _typed(k_weight, "f32", "k_weight"), _typed(positions, "i32", "positions"), _typed(slots, "i64", "slots"), n,
                               *_tokens(q_out, n, qw, tout, "q_out"), _stream(stream)))


def nq_rope_backward_workspace_bytes(r: int, n_tokens: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().nq_rope_backward_workspace_bytes(r, n_tokens, ctypes.byref(out)))
    return out.value


def nq_rope_backward(r: int, q, k, q_weight, k_weight, positions, dq_out, dk_out, dq, dk, dq_weight, dk_weight, workspace, workspace_bytes: int, stream=None) -> None:
    n = positions.numel()
    qw, kw, tin, tout, d = _WIDTHS[r]
    _same_length(d, "weight", q_weight, k_weight, dq_weight, dk_weight)
    _check(lib().nq_rope_backward(r, *_tokens(q, n, qw, tin, "q"), *_tokens(k, n, kw, tin, "k"), _typed(q_weight, "f32", "q_weight"), _typed(k_weight, "f32", "k_weight"),
                                  _typed(positions, "i32", "positions"), n, *_tokens(dq_out, n, qw, tout, "dq_out"), *_tokens(dk_out, n, kw, tout, "dk_out"),
                                  *_tokens(dq, n, qw, tin, "dq"), *_tokens(dk, n, kw, tin, "dk"), _typed(dq_weight, "f32", "dq_weight"),
                                  _typed(dk_weight, "f32", "dk_weight"), _dev_ptr(workspace), workspace_bytes, _stream(stream)))


def nq_attn_create(kv: int, q_heads: int, scale: float, cap: float, out_dtype: int) -> int:
    h = ctypes.c_void_p()
    _check(lib().nq_attn_create(ctypes.byref(h), kv, q_heads, scale, cap, out_dtype))
    head_dim, dtype = _WIDTHS[kv]
    _WIDTHS[h.value] = (q_heads * head_dim, dtype, _torch_type(out_dtype), q_heads)
    return h.value


def nq_attn_destroy(a: Optional[int]) -> None:
    _WIDTHS.pop(a, None)
    _check(lib().nq_attn_destroy(a))


def nq_attn_workspace_bytes(a: int, n_seqs: int, n_tokens: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().nq_attn_workspace_bytes(a, n_seqs, n_tokens, ctypes.byref(out)))
    return out.value


def nq_attn_forward(a: int, q, new_begin, ctx_len, page_table, tree, out, lse, workspace, workspace_bytes: int, stream=None) -> None:
    """page_table: [n_seqs, table_stride]; tree: int32 or uint32 [n_tokens, tree_words] or None."""
    n_seqs, n = ctx_len.numel(), q.shape[0]
    _same_length(n_seqs + 1, "new_begin", new_begin)
    if page_table.shape[0] != n_seqs:
        raise ValueError("page_table needs a row for every sequence")
    if tree is not None and tree.shape[0] != n:
        raise ValueError("tree needs a row for every new token")
    width, tin, tout, heads = _WIDTHS[a]
    _same_length(n * heads, "lse", lse)
    qp, qs = _tokens(q, n, width, tin, "q")
    op, os_ = _tokens(out, n, width, tout, "out")
    _check(lib().nq_attn_forward(a, qp, qs, _typed(new_begin, "i32", "new_begin"), _typed(ctx_len, "i32", "ctx_len"), _typed(page_table, "i32", "page_table"),
                                 page_table.shape[1], _typed(tree, "i32", "tree"), 0 if tree is None else tree.shape[1], n_seqs, n, op, os_, _typed(lse, "f32", "lse"),
                                 _dev_ptr(workspace), workspace_bytes, _stream(stream)))


def nq_sample_workspace_bytes(n_rows: int, vocab: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().nq_sample_workspace_bytes(n_rows, vocab, ctypes.byref(out)))
    return out.value


def nq_sample(logits, dtype: int, temperature, top_k, top_p, min_p, uniform, tokens, logprobs, workspace, workspace_bytes: int, stream=None) -> None:
    """logits: [n_rows, vocab], rows may be strided."""
    n, vocab = logits.shape
    p, stride, _ = _rows(logits, n, "logits")
    if logits.dtype != _torch_type(dtype):
        raise ValueError(f"logits: expected {_torch_type(dtype)}, got {logits.dtype}")
    _same_length(n, "one value per row", temperature, top_k, top_p, min_p, uniform, tokens, logprobs)
    _check(lib().nq_sample(p, dtype, n, vocab, stride, _typed(temperature, "f32", "temperature"), _typed(top_k, "i32", "top_k"), _typed(top_p, "f32", "top_p"),
                           _typed(min_p, "f32", "min_p"), _typed(uniform, "f32", "uniform"), _typed(tokens, "i32", "tokens"), _typed(logprobs, "f32", "logprobs"),
                           _dev_ptr(workspace), workspace_bytes, _stream(stream)))
