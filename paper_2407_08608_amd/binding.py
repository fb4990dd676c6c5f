"""ctypes binding over libfa_mi355.so: same names as the C ABI, argument marshalling only.

Every step of the attention path runs in the library's HIP kernels; PyTorch is used here
for device memory and streams.  There is no fallback: if the library has not been built
(`python -m paper_2407_08608_amd.build`), importing a symbol raises.

The calls that programs make over and over go through csrc/fa_binding.cpp when its arguments are plain ones (that file
says which): the same checks, outputs and library call in native code.  The Python below is the definition; it takes
everything else, and all of it where the native part has not been built for this Python and torch.
"""
import ctypes
import os

import torch

try:
    from . import _fa_binding as _native
except ImportError:
    _native = None

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfa_mi355.so")

FA_OK = 0
FA_F32, FA_BF16, FA_F16, FA_FP8_E4M3, FA_FP4_E2M1 = 0, 1, 2, 3, 4
_DTYPE_CODE = {torch.float32: FA_F32, torch.bfloat16: FA_BF16, torch.float16: FA_F16}

EXPORTS = ("fa_fwd", "fa_fwd_fp8", "fa_fp8_quant_hadamard", "fa_bwd_workspace_bytes", "fa_bwd",
           "fa_fwd_schedule", "fa_fwd_gqa", "fa_fwd_fp8_gqa", "fa_bwd_gqa", "fa_bwd_noalloc", "fa_fwd_kernel_name",
           "fa_probe_mfma_flops", "fa_probe_mfma", "fa_status_string", "fa_rope", "fa_rope_bwd", "fa_rope_frequencies",
           "fa_cache_write", "fa_cache_read", "fa_fwd_cache_workspace_bytes", "fa_fwd_cache", "fa_rope_axes", "fa_rope_axes_bwd",
           "fa_cache_pages_workspace_bytes", "fa_cache_fork", "fa_cache_extend", "fa_cache_compact", "fa_cache_copy")

_lib = None


class FaError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__(f"{what}: fa_status {status} ({status_string(status)})")


def lib():
    """The loaded shared library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2407_08608_amd.build`; "
                               "there is no fallback path")
        L = ctypes.CDLL(LIB_PATH)
        vp, fp, ci, cf = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_float
        L.fa_fwd.argtypes = [vp, vp, vp, vp, fp, ci, ci, ci, ci, cf, ci, ci, vp]
        L.fa_fwd.restype = ci
        L.fa_fwd_fp8.argtypes = [vp, vp, vp, fp, fp, fp, vp, fp, ci, ci, ci, ci, ci, cf, ci, vp]
        L.fa_fwd_fp8.restype = ci
        L.fa_fp8_quant_hadamard.argtypes = [vp, ci, vp, fp, ci, ci, ci, ci, ci, vp, ci, vp]
        L.fa_fp8_quant_hadamard.restype = ci
        L.fa_bwd_workspace_bytes.argtypes = [ci, ci, ci, ci, ci]
        L.fa_bwd_workspace_bytes.restype = ctypes.c_size_t
        L.fa_bwd.argtypes = [vp] * 10 + [ctypes.c_size_t, ci, ci, ci, ci, cf, ci, ci, vp]
        L.fa_bwd.restype = ci
        L.fa_fwd_schedule.argtypes = [vp, vp, vp, vp, fp, ci, ci, ci, ci, cf, ci, ci, ci, vp]
        L.fa_fwd_schedule.restype = ci
        L.fa_fwd_gqa.argtypes = [vp, vp, vp, vp, fp, ci, ci, ci, ci, ci, cf, ci, ci, vp]
        L.fa_fwd_gqa.restype = ci
        L.fa_fwd_fp8_gqa.argtypes = [vp, vp, vp, fp, fp, fp, vp, fp, ci, ci, ci, ci, ci, ci, cf, ci, vp]
        L.fa_fwd_fp8_gqa.restype = ci
        L.fa_bwd_gqa.argtypes = [vp] * 10 + [ctypes.c_size_t, ci, ci, ci, ci, ci, cf, ci, ci, vp]
        L.fa_bwd_gqa.restype = ci
        L.fa_bwd_noalloc.argtypes = [vp] * 9 + [ci, ci, ci, ci, cf, ci, ci, vp]
        L.fa_bwd_noalloc.restype = ci
        L.fa_fwd_kernel_name.argtypes = [ci, ci, ci, ci]
        L.fa_fwd_kernel_name.restype = ctypes.c_char_p
        L.fa_probe_mfma_flops.argtypes = [ci, ci]
        L.fa_probe_mfma_flops.restype = ctypes.c_double
        L.fa_probe_mfma.argtypes = [vp, ctypes.c_size_t, fp, ci, ci, vp]
        L.fa_probe_mfma.restype = ci
        cd, ip, sp = ctypes.c_double, ctypes.c_void_p, ctypes.c_void_p  # int32 and stride arrays
        L.fa_rope.argtypes = L.fa_rope_bwd.argtypes = [vp, sp] * 4 + [vp, ip] + [ci] * 6 + [cf, ci, ci, vp]
        L.fa_rope.restype = L.fa_rope_bwd.restype = ci
        L.fa_rope_frequencies.argtypes = [vp, vp, ci, cd, ci, cd, cd]
        L.fa_rope_frequencies.restype = ci
        L.fa_cache_write.argtypes = [vp, sp, vp, sp, vp, vp, fp, fp, ip, ip, ip] + [ci] * 9 + [vp]
        L.fa_cache_write.restype = ci
        L.fa_cache_read.argtypes = [vp, vp, fp, fp, ip, ip, vp, vp] + [ci] * 9 + [vp]
        L.fa_cache_read.restype = ci
        L.fa_fwd_cache_workspace_bytes.argtypes = [ci] * 7
        L.fa_fwd_cache_workspace_bytes.restype = ctypes.c_size_t
        L.fa_fwd_cache.argtypes = [vp, sp, vp, vp, fp, fp, ip, ip, ip, ip, ci, vp, sp, fp, vp, ctypes.c_size_t] + [ci] * 9 + [cf, ci, ci, vp]
        L.fa_fwd_cache.restype = ci
        L.fa_rope_axes.argtypes = L.fa_rope_axes_bwd.argtypes = [vp, sp] * 4 + [vp, ip, ip] + [ci] * 7 + [cf, ci, ci, vp]
        L.fa_rope_axes.restype = L.fa_rope_axes_bwd.restype = ci
        L.fa_cache_pages_workspace_bytes.argtypes = [ci] * 2
        L.fa_cache_pages_workspace_bytes.restype = ctypes.c_size_t
        L.fa_cache_fork.argtypes = [ip] * 9 + [vp, ctypes.c_size_t] + [ci] * 5 + [vp]
        L.fa_cache_extend.argtypes = [ip] * 5 + [vp, ctypes.c_size_t] + [ci] * 5 + [vp]
        L.fa_cache_compact.argtypes = [ip] * 6 + [vp, ctypes.c_size_t] + [ci] * 4 + [vp]
        L.fa_cache_copy.argtypes = [vp] * 4 + [ip] * 2 + [ci] * 6 + [vp]
        L.fa_cache_fork.restype = L.fa_cache_extend.restype = L.fa_cache_compact.restype = L.fa_cache_copy.restype = ci
        L.fa_status_string.argtypes = [ci]
        L.fa_status_string.restype = ctypes.c_char_p
        _lib = L
        if _native is not None:
            _native.bind(*(ctypes.cast(f, vp).value for f in (L.fa_fwd_gqa, L.fa_fwd_fp8_gqa, L.fa_fp8_quant_hadamard,
                                                              L.fa_bwd_workspace_bytes, L.fa_bwd_gqa, L.fa_rope, L.fa_rope_bwd,
                                                              L.fa_cache_write, L.fa_cache_read, L.fa_fwd_cache_workspace_bytes,
                                                              L.fa_fwd_cache, L.fa_rope_axes, L.fa_rope_axes_bwd,
                                                              L.fa_cache_pages_workspace_bytes, L.fa_cache_fork, L.fa_cache_extend,
                                                              L.fa_cache_compact, L.fa_cache_copy)))
    return _lib


def status_string(status):
    return lib().fa_status_string(int(status)).decode()


def _stream():
    """The current stream of the current device as a hipStream_t.  (The raw handle: building a torch.cuda.Stream
    object around it costs 2.9 us a call against 0.2, a quarter of a small forward's host time.)"""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _empty_like(t, dtype):
    """An uninitialised contiguous tensor of t's shape and device."""
    return torch.empty_like(t, dtype=dtype, memory_format=torch.contiguous_format)


def _outputs(result, what):
    """What a native call that was made came to: its outputs, or the refusal as an exception."""
    if type(result) is int:
        raise FaError(result, what)
    return result


def _check_dev(*ts):
    for t in ts:
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise ValueError("tensors must be contiguous device tensors")


def fa_fwd(q, k, v, scale, causal, o=None, lse=None, dtype=None):
    """O, L = attention forward.  q, k, v: [B,H,N,d] device tensors of one dtype
    (float32 / bfloat16 / float16, or uint8 e4m3 codes with dtype=FA_FP8_E4M3)."""
    if _native is not None and dtype is None:
        r = _native.fwd(q, k, v, scale, causal, o, lse, False, _stream)
        if r is not None:
            return _outputs(r, "fa_fwd")
    _check_dev(q, k, v, o, lse)
    B, H, N, d = q.shape
    code = dtype if dtype is not None else _DTYPE_CODE[q.dtype]
    if o is None:
        o = _empty_like(q, torch.bfloat16 if code == FA_FP8_E4M3 else q.dtype)
    if lse is None:
        lse = torch.empty((B, H, N), device=q.device, dtype=torch.float32)
    st = lib().fa_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), B, H, N, d,
                      float(scale), int(bool(causal)), code, _stream())
    if st != FA_OK:
        raise FaError(st, "fa_fwd")
    return o, lse


def fa_fp8_quant_hadamard(x, signs=None, block_rows=128, per_tensor=False, x8=None, scales=None):
    """codes (uint8 e4m3) and per-block scales of x [B,H,N,d]; signs: int8 [d] device tensor or None."""
    if _native is not None and block_rows == 128:
        r = _native.quant(x, signs, per_tensor, x8, scales, _stream)
        if r is not None:
            return _outputs(r, "fa_fp8_quant_hadamard")
    _check_dev(x, signs, x8, scales)
    B, H, N, d = x.shape
    nb = -(-N // block_rows)
    if x8 is None:
        x8 = _empty_like(x, torch.uint8)
    if scales is None:
        scales = torch.empty((B, H, nb), device=x.device, dtype=torch.float32)
    st = lib().fa_fp8_quant_hadamard(x.data_ptr(), _DTYPE_CODE[x.dtype], x8.data_ptr(), scales.data_ptr(), B, H, N, d,
                                     int(block_rows), None if signs is None else signs.data_ptr(),
                                     int(bool(per_tensor)), _stream())
    if st != FA_OK:
        raise FaError(st, "fa_fp8_quant_hadamard")
    return x8, scales


def fa_fwd_fp8(q8, k8, v8, q_scale, k_scale, v_scale, scale, causal, block_rows=128, o=None, lse=None):
    """O (bf16), L from e4m3 codes with per-block scales."""
    if _native is not None and block_rows == 128:
        r = _native.fwd_fp8(q8, k8, v8, q_scale, k_scale, v_scale, scale, causal, o, lse, False, _stream)
        if r is not None:
            return _outputs(r, "fa_fwd_fp8")
    _check_dev(q8, k8, v8, q_scale, k_scale, v_scale, o, lse)
    B, H, N, d = q8.shape
    if o is None:
        o = _empty_like(q8, torch.bfloat16)
    if lse is None:
        lse = torch.empty((B, H, N), device=q8.device, dtype=torch.float32)
    st = lib().fa_fwd_fp8(q8.data_ptr(), k8.data_ptr(), v8.data_ptr(), q_scale.data_ptr(), k_scale.data_ptr(),
                          v_scale.data_ptr(), o.data_ptr(), lse.data_ptr(), B, H, N, d, int(block_rows),
                          float(scale), int(bool(causal)), _stream())
    if st != FA_OK:
        raise FaError(st, "fa_fwd_fp8")
    return o, lse


def fa_bwd_workspace_bytes(B, H, N, d, dtype=FA_BF16):
    return int(lib().fa_bwd_workspace_bytes(B, H, N, d, dtype))


def fa_bwd(q, k, v, o, lse, dout, scale, causal, dq=None, dk=None, dv=None, workspace=None):
    """dQ, dK, dV from the forward's inputs, O, L and dO."""
    if _native is not None:
        r = _native.bwd(q, k, v, o, lse, dout, scale, causal, dq, dk, dv, workspace, False, _stream)
        if r is not None:
            return _outputs(r, "fa_bwd")
    _check_dev(q, k, v, o, lse, dout, dq, dk, dv, workspace)
    B, H, N, d = q.shape
    code = _DTYPE_CODE[q.dtype]
    need = fa_bwd_workspace_bytes(B, H, N, d, code)
    if workspace is None:
        workspace = torch.empty((max(need, 16),), device=q.device, dtype=torch.uint8)
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    st = lib().fa_bwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), dout.data_ptr(),
                      dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), workspace.data_ptr(), workspace.numel(),
                      B, H, N, d, float(scale), int(bool(causal)), code, _stream())
    if st != FA_OK:
        raise FaError(st, "fa_bwd")
    return dq, dk, dv


FA_BWD_NOALLOC_MAX_ROWS = 1048576


def fa_bwd_noalloc(q, k, v, o, lse, dout, scale, causal, dq, dk, dv):
    """fa_bwd on the library's fixed scratch: the caller passes every tensor, outputs included, and the
    call allocates nothing (neither here nor in the library)."""
    _check_dev(q, k, v, o, lse, dout, dq, dk, dv)
    B, H, N, d = q.shape
    st = lib().fa_bwd_noalloc(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), dout.data_ptr(),
                              dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), B, H, N, d, float(scale),
                              int(bool(causal)), _DTYPE_CODE[q.dtype], _stream())
    if st != FA_OK:
        raise FaError(st, "fa_bwd_noalloc")
    return dq, dk, dv


FA_SCHED_AUTO, FA_SCHED_LOCKSTEP_4W, FA_SCHED_LOCKSTEP_8W, FA_SCHED_PINGPONG = 0, 1, 2, 3


def fa_fwd_schedule(q, k, v, scale, causal, schedule, o=None, lse=None):
    """fa_fwd with the kernel schedule forced (ablation)."""
    _check_dev(q, k, v, o, lse)
    B, H, N, d = q.shape
    o = torch.empty_like(q) if o is None else o
    if lse is None:
        lse = torch.empty((B, H, N), device=q.device, dtype=torch.float32)
    st = lib().fa_fwd_schedule(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), B, H, N, d,
                               float(scale), int(bool(causal)), _DTYPE_CODE[q.dtype], int(schedule), _stream())
    if st != FA_OK:
        raise FaError(st, "fa_fwd_schedule")
    return o, lse


def fa_fwd_gqa(q, k, v, scale, causal, o=None, lse=None, dtype=None):
    """Grouped-query forward: q [B,H,N,d]; k, v [B,H_kv,N,d] with H_kv dividing H."""
    if _native is not None and dtype is None:
        r = _native.fwd(q, k, v, scale, causal, o, lse, True, _stream)
        if r is not None:
            return _outputs(r, "fa_fwd_gqa")
    _check_dev(q, k, v, o, lse)
    B, H, N, d = q.shape
    H_kv = k.shape[1]
    code = dtype if dtype is not None else _DTYPE_CODE[q.dtype]
    if o is None:
        o = _empty_like(q, torch.bfloat16 if code == FA_FP8_E4M3 else q.dtype)
    if lse is None:
        lse = torch.empty((B, H, N), device=q.device, dtype=torch.float32)
    st = lib().fa_fwd_gqa(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), B, H, H_kv, N, d,
                          float(scale), int(bool(causal)), code, _stream())
    if st != FA_OK:
        raise FaError(st, "fa_fwd_gqa")
    return o, lse


def fa_fwd_fp8_gqa(q8, k8, v8, q_scale, k_scale, v_scale, scale, causal, block_rows=128, o=None, lse=None):
    """Grouped-query FP8 forward: q8 [B,H,N,d]; k8, v8 [B,H_kv,N,d] and their scales [B,H_kv,blocks]."""
    if _native is not None and block_rows == 128:
        r = _native.fwd_fp8(q8, k8, v8, q_scale, k_scale, v_scale, scale, causal, o, lse, True, _stream)
        if r is not None:
            return _outputs(r, "fa_fwd_fp8_gqa")
    _check_dev(q8, k8, v8, q_scale, k_scale, v_scale, o, lse)
    B, H, N, d = q8.shape
    H_kv = k8.shape[1]
    if o is None:
        o = _empty_like(q8, torch.bfloat16)
    if lse is None:
        lse = torch.empty((B, H, N), device=q8.device, dtype=torch.float32)
    st = lib().fa_fwd_fp8_gqa(q8.data_ptr(), k8.data_ptr(), v8.data_ptr(), q_scale.data_ptr(), k_scale.data_ptr(),
                              v_scale.data_ptr(), o.data_ptr(), lse.data_ptr(), B, H, H_kv, N, d, int(block_rows),
                              float(scale), int(bool(causal)), _stream())
    if st != FA_OK:
        raise FaError(st, "fa_fwd_fp8_gqa")
    return o, lse


def fa_bwd_gqa(q, k, v, o, lse, dout, scale, causal, dq=None, dk=None, dv=None, workspace=None):
    """Grouped-query backward: dQ [B,H,N,d]; dK, dV [B,H_kv,N,d] (summed over each group's query heads)."""
    if _native is not None:
        r = _native.bwd(q, k, v, o, lse, dout, scale, causal, dq, dk, dv, workspace, True, _stream)
        if r is not None:
            return _outputs(r, "fa_bwd_gqa")
    _check_dev(q, k, v, o, lse, dout, dq, dk, dv, workspace)
    B, H, N, d = q.shape
    H_kv = k.shape[1]
    code = _DTYPE_CODE[q.dtype]
    need = fa_bwd_workspace_bytes(B, H, N, d, code)
    if workspace is None:
        workspace = torch.empty((max(need, 16),), device=q.device, dtype=torch.uint8)
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    st = lib().fa_bwd_gqa(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), dout.data_ptr(),
                          dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), workspace.data_ptr(), workspace.numel(),
                          B, H, H_kv, N, d, float(scale), int(bool(causal)), code, _stream())
    if st != FA_OK:
        raise FaError(st, "fa_bwd_gqa")
    return dq, dk, dv


FA_ROPE_PLAIN, FA_ROPE_LINEAR, FA_ROPE_NTK, FA_ROPE_BY_PARTS = 0, 1, 2, 3
FA_CACHE_MAX_TOKENS = 256


def _check(what, t, shape, dtypes, strided=False):
    """A tensor of this shape and one of these dtypes on the current device, contiguous or (strided) with contiguous rows."""
    if not t.is_cuda or t.get_device() != torch._C._cuda_getDevice():
        raise ValueError(f"{what} must be on the current device")
    if t.dtype not in dtypes or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} must be {list(shape)} of {' or '.join(str(d) for d in dtypes)}, not {list(t.shape)} of {t.dtype}")
    if not (t.is_contiguous() or (strided and t.stride(-1) == 1)):
        raise ValueError(f"{what} must {'have contiguous rows' if strided else 'be contiguous'}")


def _strides(t):
    """The batch, head and token strides of a [B,H,N,d] tensor for the library (None: contiguous)"""
    return None if t.is_contiguous() else (ctypes.c_longlong * 3)(*t.stride()[:3])


def _ptr(t):
    return None if t is None else t.data_ptr()


def fa_rope_frequencies(rot_dim, base=10000.0, scaling=FA_ROPE_PLAIN, factor=1.0, trained_len=0.0, device="cuda"):
    """inv_freq (fp64 [rot_dim / 2] on `device`) and amplitude of rotary positions, as fa_rope takes them."""
    f, amplitude = torch.empty((max(int(rot_dim), 0) // 2,), dtype=torch.float64), ctypes.c_float()
    st = lib().fa_rope_frequencies(f.data_ptr() or 1, ctypes.byref(amplitude), int(rot_dim), float(base), int(scaling), float(factor),
                                   float(trained_len))
    if st != FA_OK:
        raise FaError(st, "fa_rope_frequencies")
    return f.to(device), amplitude.value


def _rope(name, q, inv_freq, k, positions, rot_dim, interleaved, amplitude, q_out, k_out, axis=None, several=False):
    if _native is not None:
        if several:
            r = _native.rope_axes(name == "fa_rope_axes_bwd", q, inv_freq, k, positions, rot_dim, interleaved, amplitude, q_out, k_out, _stream, axis)
        else:
            r = _native.rope(name == "fa_rope_bwd", q, inv_freq, k, positions, rot_dim, interleaved, amplitude, q_out, k_out, _stream)
        if r is not None:
            return _outputs(r, name)
    if q.dim() != 4 or (k is not None and k.dim() != 4):
        raise ValueError("q and k must be [B,H,N,d] and [B,H_kv,N,d]")
    B, H, N, d = q.shape
    H_kv = 0 if k is None else k.shape[1]
    rot_dim = d if rot_dim is None else int(rot_dim)
    dtypes = (q.dtype,) if q.dtype in _DTYPE_CODE else tuple(_DTYPE_CODE)
    _check("q", q, q.shape, dtypes, strided=True)
    _check("inv_freq", inv_freq, (rot_dim // 2,), (torch.float64,))
    if several:
        if positions.dim() != 3:
            raise ValueError("positions must be [axes,B,N]")
        _check("axis", axis, (rot_dim // 2,), (torch.int32,))
        _check("positions", positions, (positions.shape[0], B, N), (torch.int32,))
    elif positions is not None:
        _check("positions", positions, (B, N), (torch.int32,))
    if q_out is None:
        q_out = _empty_like(q, q.dtype)
    _check("q_out", q_out, q.shape, dtypes, strided=True)
    if k is not None:
        _check("k", k, (B, H_kv, N, d), dtypes, strided=True)
        if k_out is None:
            k_out = _empty_like(k, k.dtype)
        _check("k_out", k_out, k.shape, dtypes, strided=True)
    else:
        k_out = None
    turns = (_ptr(axis), _ptr(positions), positions.shape[0]) if several else (_ptr(positions),)
    st = getattr(lib(), name)(q.data_ptr(), _strides(q), _ptr(k), None if k is None else _strides(k), q_out.data_ptr(), _strides(q_out),
                              _ptr(k_out), None if k is None else _strides(k_out), inv_freq.data_ptr(), *turns, B, H, H_kv, N, d,
                              rot_dim, float(amplitude), int(bool(interleaved)), _DTYPE_CODE[q.dtype], _stream())
    if st != FA_OK:
        raise FaError(st, name)
    return q_out, k_out


def fa_rope(q, inv_freq, k=None, positions=None, rot_dim=None, interleaved=False, amplitude=1.0, q_out=None, k_out=None):
    """q [B,H,N,d] and k [B,H_kv,N,d] (or None) with the first rot_dim (None: d) elements of every row rotated by its token's
    position: positions int32 [B,N], or None for 0 .. N-1.  Any strides with contiguous rows; outputs contiguous unless given
    (q_out may be q, k_out may be k)."""
    return _rope("fa_rope", q, inv_freq, k, positions, rot_dim, interleaved, amplitude, q_out, k_out)


def fa_rope_bwd(dq, inv_freq, k=None, positions=None, rot_dim=None, interleaved=False, amplitude=1.0, q_out=None, k_out=None):
    """Gradients by the rotated q (and k, given as `k`) taken back to gradients by fa_rope's inputs; arguments as there."""
    return _rope("fa_rope_bwd", dq, inv_freq, k, positions, rot_dim, interleaved, amplitude, q_out, k_out)


def fa_rope_axes(q, inv_freq, axis, positions, k=None, rot_dim=None, interleaved=False, amplitude=1.0, q_out=None, k_out=None):
    """fa_rope with several axes: pair i goes by positions[axis[i]] (positions int32 [axes,B,N], axis int32 [rot_dim / 2])."""
    return _rope("fa_rope_axes", q, inv_freq, k, positions, rot_dim, interleaved, amplitude, q_out, k_out, axis, True)


def fa_rope_axes_bwd(dq, inv_freq, axis, positions, k=None, rot_dim=None, interleaved=False, amplitude=1.0, q_out=None, k_out=None):
    """Gradients by the rotated q (and k, given as `k`) taken back to gradients by fa_rope_axes' inputs; arguments as there."""
    return _rope("fa_rope_axes_bwd", dq, inv_freq, k, positions, rot_dim, interleaved, amplitude, q_out, k_out, axis, True)


_CACHE_CODE = {torch.bfloat16: FA_BF16, torch.float16: FA_F16, torch.uint8: FA_FP8_E4M3, torch.float8_e4m3fn: FA_FP8_E4M3}


# (Not every torch has these types; bytes it always takes.)
_POWERS = tuple(t for t in (torch.uint8, getattr(torch, "float8_e8m0fnu", None)) if t is not None)
_CODES4 = getattr(torch, "float4_e2m1fn_x2", None)


def _in_four_bits(k_pages, k_scales):
    """Whether the last dimension of pages is half of d: two e2m1 codes to a byte, which their type says, or that of the scales does"""
    return (_CODES4 is not None and k_pages.dtype is _CODES4) or (k_pages.dtype is torch.uint8 and k_scales is not None and k_scales.dtype in _POWERS)


def _check_pages(H_kv, d, k_pages, v_pages, k_scales, v_scales):
    """(page_size, n_pages, dtype code) of pages and scales that belong together"""
    if k_pages.dim() != 4:
        raise ValueError("pages must be [n_pages,H_kv,page_size,d]")
    n_pages, _, page_size, _ = k_pages.shape
    four = _in_four_bits(k_pages, k_scales)
    dtypes = (k_pages.dtype,) if four or k_pages.dtype in _CACHE_CODE else tuple(_CACHE_CODE)
    for name, t in (("k_pages", k_pages), ("v_pages", v_pages)):
        _check(name, t, (n_pages, H_kv, page_size, d // 2 if four else d), dtypes)
    code = FA_FP4_E2M1 if four else _CACHE_CODE[k_pages.dtype]
    for name, t in (("k_scales", k_scales), ("v_scales", v_scales)):
        if (t is not None) != (code in (FA_FP8_E4M3, FA_FP4_E2M1)):
            raise ValueError("an e4m3 or e2m1 cache has k_scales and v_scales, a 16-bit one has none")
        if four:
            _check(name, t, (n_pages, H_kv, page_size, d // 32), _POWERS)
        elif t is not None:
            _check(name, t, (n_pages, H_kv, page_size), (torch.float32,))
    return page_size, n_pages, code


def _check_cache(B, H_kv, d, k_pages, v_pages, block_table, lens, counts, k_scales, v_scales):
    """(page_size, n_pages, max_pages, dtype code) of a cache whose tensors belong together"""
    if k_pages.dim() != 4 or block_table.dim() != 2:
        raise ValueError("pages must be [n_pages,H_kv,page_size,d] and the block table [B,max_pages]")
    page_size, n_pages, code = _check_pages(H_kv, d, k_pages, v_pages, k_scales, v_scales)
    _check("block_table", block_table, (B, block_table.shape[1]), (torch.int32,))
    _check("lens", lens, (B,), (torch.int32,))
    if counts is not None:
        _check("counts", counts, (B,), (torch.int32,))
    return page_size, n_pages, block_table.shape[1], code


def fa_cache_write(k, v, k_pages, v_pages, block_table, lens, counts=None, k_scales=None, v_scales=None):
    """k, v [B,H_kv,T,d] (contiguous rows) into the cache behind the lens[b] tokens that it holds: T of every sequence, or
    counts[b] of them.  Pages [n_pages,H_kv,page_size,d]: 16-bit, or e4m3 codes (uint8 or float8_e4m3fn) with scales; or
    [n_pages,H_kv,page_size,d / 2] of two e2m1 codes each (uint8 or float4_e2m1fn_x2), with scales [n_pages,H_kv,page_size,d / 32]
    that are powers of two (uint8 or float8_e8m0fnu)."""
    if _native is not None:
        r = _native.cache_write(k, v, k_pages, v_pages, block_table, lens, counts, k_scales, v_scales, _stream)
        if r is not None:
            return _outputs(r, "fa_cache_write")
    if k.dim() != 4:
        raise ValueError("k and v must be [B,H_kv,T,d]")
    B, H_kv, T, d = k.shape
    dtypes = (k.dtype,) if k.dtype in _DTYPE_CODE else tuple(_DTYPE_CODE)
    _check("k", k, k.shape, dtypes, strided=True)
    _check("v", v, k.shape, dtypes, strided=True)
    page_size, n_pages, max_pages, code = _check_cache(B, H_kv, d, k_pages, v_pages, block_table, lens, counts, k_scales, v_scales)
    st = lib().fa_cache_write(k.data_ptr(), _strides(k), v.data_ptr(), _strides(v), k_pages.data_ptr(), v_pages.data_ptr(), _ptr(k_scales),
                              _ptr(v_scales), block_table.data_ptr(), lens.data_ptr(), _ptr(counts), B, H_kv, T, d, page_size, n_pages,
                              max_pages, _DTYPE_CODE[k.dtype], code, _stream())
    if st != FA_OK:
        raise FaError(st, "fa_cache_write")
    return k_pages, v_pages


def fa_cache_read(k_pages, v_pages, block_table, lens, N=None, dtype=None, k_scales=None, v_scales=None, k=None, v=None):
    """The first min(lens[b], N) cached tokens of every sequence as k, v [B,H_kv,N,d]; the other rows stay as they are (in a tensor
    allocated here: uninitialised).  `dtype`: of allocated outputs (None: the cache's own 16-bit type, bfloat16 for codes)."""
    if _native is not None:
        r = _native.cache_read(k_pages, v_pages, block_table, lens, N, dtype, k_scales, v_scales, k, v, _stream)
        if r is not None:
            return _outputs(r, "fa_cache_read")
    if k_pages.dim() != 4 or block_table.dim() != 2:
        raise ValueError("pages must be [n_pages,H_kv,page_size,d] and the block table [B,max_pages]")
    B, (_, H_kv, _, d) = block_table.shape[0], k_pages.shape
    if _in_four_bits(k_pages, k_scales):
        d *= 2
    given = k if k is not None else v
    if given is not None:
        N, dtype = given.shape[2] if N is None else int(N), given.dtype if dtype is None else dtype
    elif N is None:
        raise ValueError("N is needed where neither k nor v is given")
    if dtype is None:
        dtype = k_pages.dtype if k_pages.dtype in _DTYPE_CODE else torch.bfloat16
    if dtype not in _DTYPE_CODE:
        raise ValueError(f"the cache is not read as {dtype}")
    page_size, n_pages, max_pages, code = _check_cache(B, H_kv, d, k_pages, v_pages, block_table, lens, None, k_scales, v_scales)
    shape = (B, H_kv, int(N), d)
    k = torch.empty(shape, device=k_pages.device, dtype=dtype) if k is None else k
    v = torch.empty(shape, device=k_pages.device, dtype=dtype) if v is None else v
    _check("k", k, shape, (dtype,))
    _check("v", v, shape, (dtype,))
    st = lib().fa_cache_read(k_pages.data_ptr(), v_pages.data_ptr(), _ptr(k_scales), _ptr(v_scales), block_table.data_ptr(),
                             lens.data_ptr(), k.data_ptr(), v.data_ptr(), B, H_kv, int(N), d, page_size, n_pages, max_pages, code,
                             _DTYPE_CODE[dtype], _stream())
    if st != FA_OK:
        raise FaError(st, "fa_cache_read")
    return k, v


def _new(t, shape):
    return torch.empty(shape, device=t.device, dtype=torch.int32)


def _together(like, *sized):
    """The given tensors, and new ones of these sizes for those that are not, in one allocation"""
    new = iter(_new(like, (sum(n for n, t in sized if t is None),)).split([n for n, t in sized if t is None]))
    return [next(new) if t is None else t for _, t in sized]


def fa_cache_pages_workspace_bytes(B, n_pages):
    return int(lib().fa_cache_pages_workspace_bytes(B, n_pages))


def _pages_workspace(workspace, B, n_pages, like):
    """(pointer, bytes, what keeps them) of the given workspace, or a new one where there has to be one"""
    if workspace is None:
        need = fa_cache_pages_workspace_bytes(B, n_pages)
        workspace = torch.empty((need,), device=like.device, dtype=torch.uint8) if need else None
    else:
        _check("workspace", workspace, (workspace.numel(),), (torch.uint8,))
    return _ptr(workspace), 0 if workspace is None else workspace.numel(), workspace


def _check_ints(*named):
    for name, t, shape in named:
        if t is not None:
            _check(name, t, shape, (torch.int32,))


def _check_table(block_table):
    if block_table.dim() != 2:
        raise ValueError("the block table must be [B,max_pages]")
    _check("block_table", block_table, block_table.shape, (torch.int32,))


def fa_cache_fork(block_table, lens, parents, page_size, n_pages, held=None, new_table=None, new_lens=None, src=None, dst=None, missing=None,
                  workspace=None):
    """The batch of the next step: new_table [B_new,max_pages] and new_lens of sequences that continue parents[i] (int32 [B_new]; none: -1),
    sharing whole pages; what fa_cache_copy has to copy for them (src, dst: last pages that are not full and have another reader, or are held);
    and how many pages were missing."""
    if _native is not None:
        r = _native.cache_fork(block_table, lens, parents, page_size, n_pages, held, new_table, new_lens, src, dst, missing, workspace, _stream)
        if r is not None:
            return _outputs(r, "fa_cache_fork")
    _check_table(block_table)
    if parents.dim() != 1:
        raise ValueError("parents must be [B_new]")
    (B, max_pages), B_new, n_pages = block_table.shape, parents.shape[0], int(n_pages)
    _check_ints(("lens", lens, (B,)), ("parents", parents, (B_new,)), ("held", held, (n_pages,)))
    new_table = _new(block_table, (B_new, max_pages)) if new_table is None else new_table
    new_lens, src, dst, missing = _together(block_table, (B_new, new_lens), (B_new, src), (B_new, dst), (1, missing))
    _check_ints(("new_table", new_table, (B_new, max_pages)), ("new_lens", new_lens, (B_new,)), ("src", src, (B_new,)), ("dst", dst, (B_new,)),
                ("missing", missing, (1,)))
    space, bytes, workspace = _pages_workspace(workspace, B_new, n_pages, block_table)
    st = lib().fa_cache_fork(block_table.data_ptr(), lens.data_ptr(), parents.data_ptr(), _ptr(held), new_table.data_ptr(), new_lens.data_ptr(),
                             src.data_ptr(), dst.data_ptr(), missing.data_ptr(), space, bytes, B, B_new, int(page_size),
                             n_pages, max_pages, _stream())
    if st != FA_OK:
        raise FaError(st, "fa_cache_fork")
    return new_table, new_lens, src, dst, missing


def fa_cache_extend(block_table, lens, T, page_size, n_pages, counts=None, held=None, missing=None, workspace=None):
    """Free pages for the next T (or counts[b]) tokens of every sequence, where block_table, which is changed in place, has none.  Returns
    it, and how many were missing."""
    if _native is not None:
        r = _native.cache_extend(block_table, lens, T, page_size, n_pages, counts, held, missing, workspace, _stream)
        if r is not None:
            return _outputs(r, "fa_cache_extend")
    _check_table(block_table)
    (B, max_pages), n_pages = block_table.shape, int(n_pages)
    missing = _new(block_table, (1,)) if missing is None else missing
    _check_ints(("lens", lens, (B,)), ("counts", counts, (B,)), ("held", held, (n_pages,)), ("missing", missing, (1,)))
    space, bytes, workspace = _pages_workspace(workspace, B, n_pages, block_table)
    st = lib().fa_cache_extend(block_table.data_ptr(), lens.data_ptr(), _ptr(counts), _ptr(held), missing.data_ptr(), space, bytes, B, int(T), int(page_size), n_pages, max_pages, _stream())
    if st != FA_OK:
        raise FaError(st, "fa_cache_extend")
    return block_table, missing


def fa_cache_compact(block_table, n_pages, moves=None, held=None, new_table=None, src=None, dst=None, top=None, workspace=None):
    """Pages in use moved to the lowest numbers, `moves` of them at most (None: n_pages / 2, which is always enough): the table by the new
    numbers (new_table may be block_table), what fa_cache_copy has to copy (src, dst [moves]), and one more than the highest page in use."""
    if _native is not None:
        r = _native.cache_compact(block_table, n_pages, moves, held, new_table, src, dst, top, workspace, _stream)
        if r is not None:
            return _outputs(r, "fa_cache_compact")
    _check_table(block_table)
    (B, max_pages), n_pages = block_table.shape, int(n_pages)
    moves = max(n_pages // 2, 1) if moves is None else int(moves)
    _check_ints(("held", held, (n_pages,)))
    new_table = _new(block_table, (B, max_pages)) if new_table is None else new_table
    src, dst, top = _together(block_table, (moves, src), (moves, dst), (1, top))
    _check_ints(("new_table", new_table, (B, max_pages)), ("src", src, (moves,)), ("dst", dst, (moves,)), ("top", top, (1,)))
    space, bytes, workspace = _pages_workspace(workspace, B, n_pages, block_table)
    st = lib().fa_cache_compact(block_table.data_ptr(), _ptr(held), new_table.data_ptr(), src.data_ptr(), dst.data_ptr(), top.data_ptr(),
                                space, bytes, B, moves, n_pages, max_pages, _stream())
    if st != FA_OK:
        raise FaError(st, "fa_cache_compact")
    return new_table, src, dst, top


def fa_cache_copy(k_pages, v_pages, src, dst, k_scales=None, v_scales=None):
    """Page src[i] of a cache (any that fa_cache_write takes) copied to page dst[i], K and V with their scales; pairs of -1 are left out."""
    if _native is not None:
        r = _native.cache_copy(k_pages, v_pages, src, dst, k_scales, v_scales, _stream)
        if r is not None:
            return _outputs(r, "fa_cache_copy")
    if k_pages.dim() != 4 or src.dim() != 1:
        raise ValueError("pages must be [n_pages,H_kv,page_size,d], src and dst [n]")
    H_kv, d = k_pages.shape[1], k_pages.shape[3] * (2 if _in_four_bits(k_pages, k_scales) else 1)
    page_size, n_pages, code = _check_pages(H_kv, d, k_pages, v_pages, k_scales, v_scales)
    _check_ints(("src", src, (src.shape[0],)), ("dst", dst, (src.shape[0],)))
    st = lib().fa_cache_copy(k_pages.data_ptr(), v_pages.data_ptr(), _ptr(k_scales), _ptr(v_scales), src.data_ptr(), dst.data_ptr(), src.shape[0],
                             H_kv, d, page_size, n_pages, code, _stream())
    if st != FA_OK:
        raise FaError(st, "fa_cache_copy")
    return k_pages, v_pages


def fa_tree_words(visible):
    """The `tree` of fa_fwd_cache, int32 [..., T, ceil(T / 32)], from visible[..., t, u]: whether (not zero) new token t sees new token u."""
    T = visible.shape[-1]
    bits = torch.nn.functional.pad((visible != 0).to(torch.int64), (0, -T % 32)).unflatten(-1, (-1, 32))
    words = (bits << torch.arange(32, device=visible.device)).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def fa_fwd_cache_workspace_bytes(B, H, H_kv, T, d, max_len, cache_dtype=FA_BF16):
    return int(lib().fa_fwd_cache_workspace_bytes(B, H, H_kv, T, d, max_len, cache_dtype))


def fa_fwd_cache(q, k_pages, v_pages, block_table, lens, scale, tree=None, counts=None, k_scales=None, v_scales=None, max_len=0,
                 o=None, lse=None, workspace=None):
    """O, L of T new tokens of every sequence, q [B,H,T,d] (contiguous rows), over the cache, which holds them behind lens[b]
    others.  tree: int32 [B or 1, T, ceil(T / 32)] (fa_tree_words), None: a chain.  Rows from counts[b] on stay as they are (in
    tensors allocated here: uninitialised).  max_len: what lens[b] + T reaches at most, 0: the width of the block table."""
    if _native is not None:
        r = _native.fwd_cache(q, k_pages, v_pages, block_table, lens, scale, tree, counts, k_scales, v_scales, max_len, o, lse, workspace,
                              _stream)
        if r is not None:
            return _outputs(r, "fa_fwd_cache")
    if q.dim() != 4 or k_pages.dim() != 4:
        raise ValueError("q must be [B,H,T,d] and pages [n_pages,H_kv,page_size,d]")
    B, H, T, d = q.shape
    H_kv = k_pages.shape[1]
    dtypes = (q.dtype,) if q.dtype in (torch.bfloat16, torch.float16) else (torch.bfloat16, torch.float16)
    _check("q", q, q.shape, dtypes, strided=True)
    page_size, n_pages, max_pages, code = _check_cache(B, H_kv, d, k_pages, v_pages, block_table, lens, counts, k_scales, v_scales)
    if tree is not None:
        batches = tree.shape[0] if tree.dim() == 3 and tree.shape[0] == B else 1
        _check("tree", tree, (batches, T, -(-T // 32)), (torch.int32,))
    else:
        batches = 0
    if o is None:
        o = _empty_like(q, q.dtype)
    if lse is None:
        lse = torch.empty((B, H, T), device=q.device, dtype=torch.float32)
    _check("o", o, q.shape, dtypes, strided=True)
    _check("lse", lse, (B, H, T), (torch.float32,))
    need = lib().fa_fwd_cache_workspace_bytes(B, H, H_kv, T, d, int(max_len) or max_pages * page_size, code)
    if workspace is None:
        if need:
            workspace = torch.empty((need,), device=q.device, dtype=torch.uint8)
    else:
        _check("workspace", workspace, (workspace.numel(),), (torch.uint8,))
    st = lib().fa_fwd_cache(q.data_ptr(), _strides(q), k_pages.data_ptr(), v_pages.data_ptr(), _ptr(k_scales), _ptr(v_scales),
                            block_table.data_ptr(), lens.data_ptr(), _ptr(counts), _ptr(tree), batches, o.data_ptr(), _strides(o),
                            lse.data_ptr(), _ptr(workspace), 0 if workspace is None else workspace.numel(), B, H, H_kv, T, d, page_size,
                            n_pages, max_pages, int(max_len), float(scale), _DTYPE_CODE[q.dtype], code, _stream())
    if st != FA_OK:
        raise FaError(st, "fa_fwd_cache")
    return o, lse


def fa_probe_mfma_flops(dtype, iters):
    return float(lib().fa_probe_mfma_flops(int(dtype), int(iters)))


def fa_probe_mfma(operands, dtype, iters, sink=None):
    """One launch of the MFMA-only rate probe on the raw operand bits in `operands` (uint8)."""
    _check_dev(operands, sink)
    if sink is None:
        sink = torch.empty((512,), device=operands.device, dtype=torch.float32)
    st = lib().fa_probe_mfma(operands.data_ptr(), operands.numel() * operands.element_size(), sink.data_ptr(),
                             int(dtype), int(iters), _stream())
    if st != FA_OK:
        raise FaError(st, "fa_probe_mfma")
    return sink


def fa_fwd_kernel_name(dtype, N, d, causal):
    """Profiler name of the kernel that serves this forward request (None if unsupported)."""
    name = lib().fa_fwd_kernel_name(int(dtype), int(N), int(d), int(bool(causal)))
    return None if name is None else name.decode()
