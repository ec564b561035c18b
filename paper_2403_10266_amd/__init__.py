"""Python binding of libdsp: one GPU's share of a Dynamic Sequence Parallelism
spatial-temporal block on MI355X.

Argument marshalling only.  Every computation runs in the HIP kernels of
``libdsp.so`` (built in-tree by ``paper_2403_10266_amd.build``); this module
turns torch tensors into device pointers, sizes and the current HIP stream,
calls the C entry point of the same name and raises ``DspError`` on a nonzero
status.  There is no fallback: if the library is missing, importing the
binding's functions raises.

Entry points (see ``include/dsp.h`` for the exact contracts):
``dsp_switch``, ``dsp_exchange_unpack``, ``dsp_split``, ``dsp_gather``,
``dsp_spatial_attn``, ``dsp_temporal_attn``, ``dsp_attn_strided``,
``dsp_attn_fwd_lse``, ``dsp_attn_bwd``, ``dsp_attn_general``, ``dsp_attn_general_bwd``, ``dsp_attn_relpos``, ``dsp_attn_relpos_bwd``, ``dsp_relpos_buckets``, ``dsp_qk_norm_rope``, ``dsp_qk_norm_rope_bwd``, ``dsp_layernorm_bwd``, ``dsp_linear_bwd_data``, ``dsp_linear_bwd_weight``,
``dsp_layernorm``, ``dsp_linear``, ``dsp_st_block_forward``.
"""
from __future__ import annotations

import ctypes
import os
from pathlib import Path

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libdsp.so"

# status codes and enums of include/dsp.h
DSP_OK, DSP_ERR_NULL, DSP_ERR_DIM, DSP_ERR_SHAPE, DSP_ERR_DTYPE, DSP_ERR_ALIGN, DSP_ERR_HIP, \
    DSP_ERR_WORKSPACE, DSP_ERR_ARG = range(9)
DSP_F32, DSP_BF16 = 0, 1
DSP_EPI_NONE, DSP_EPI_GELU, DSP_EPI_RESID, DSP_EPI_F32, DSP_EPI_RELU = 0, 1, 2, 3, 4
DSP_BLOCK_NO_MLP_LN, DSP_BLOCK_ATTN_ONLY, DSP_BLOCK_POST_LN, DSP_BLOCK_RELU = 1, 2, 4, 8
DSP_ROPE_ADJACENT = 1
DSP_RELPOS_CAUSAL = 1
DSP_GRAD_EPI_F32, DSP_GRAD_EPI_BF16, DSP_GRAD_EPI_GELU_BWD, DSP_GRAD_EPI_RELU_BWD = 0, 1, 2, 3

BLOCK_WEIGHT_FIELDS = ("wqkv_s", "bqkv_s", "wo_s", "bo_s", "wqkv_t", "bqkv_t", "wo_t", "bo_t",
                       "w1", "b1", "w2", "b2")


class DspError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_str(status)} (status {status})")


class BlockWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in BLOCK_WEIGHT_FIELDS]


class BlockGrads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in BLOCK_WEIGHT_FIELDS]


_lib = None

_c = ctypes
_P, _I, _I64, _F, _SZ = _c.c_void_p, _c.c_int, _c.c_int64, _c.c_float, _c.c_size_t
_SIGNATURES = {
    "dsp_status_str": (_c.c_char_p, [_I]),
    "dsp_version": (_I, []),
    "dsp_switch": (_I, [_P, _P, _c.POINTER(_I64), _I, _I, _I, _I, _I, _P]),
    "dsp_switch_variant": (_I, [_P, _P, _c.POINTER(_I64), _I, _I, _I, _I, _I, _I, _P]),
    "dsp_exchange_unpack": (_I, [_c.POINTER(_P), _c.POINTER(_P), _c.POINTER(_I64), _I, _P]),
    "dsp_split": (_I, [_P, _P, _c.POINTER(_I64), _I, _I, _I, _I, _I, _P]),
    "dsp_gather": (_I, [_c.POINTER(_P), _P, _c.POINTER(_I64), _I, _I, _I, _I, _P]),
    "dsp_spatial_attn": (_I, [_P, _P, _P, _P, _I64, _I64, _I64, _I, _I, _I64, _I64, _F, _I, _P]),
    "dsp_temporal_attn": (_I, [_P, _P, _P, _P, _I64, _I64, _I64, _I, _I, _I64, _I64, _F, _I, _P]),
    "dsp_attn_strided": (_I, [_P, _P, _P, _P, _I64, _I64, _I64, _I, _I, _c.POINTER(_I64),
                              _c.POINTER(_I64), _F, _I, _P]),
    "dsp_attn_fwd_lse": (_I, [_P, _P, _P, _P, _P, _I64, _I64, _I64, _I, _I, _c.POINTER(_I64),
                              _c.POINTER(_I64), _F, _I, _P]),
    "dsp_attn_bwd": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _I, _I,
                          _c.POINTER(_I64), _c.POINTER(_I64), _F, _I, _P]),
    "dsp_attn_bwd_noalloc_max_rows": (_I64, []),
    "dsp_attn_bwd_noalloc": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _I, _I,
                                  _c.POINTER(_I64), _c.POINTER(_I64), _F, _I, _P]),
    "dsp_relpos_buckets": (_I, [_P, _I, _I, _I]),
    "dsp_attn_relpos_workspace_bytes": (_SZ, [_I64] * 4 + [_I] * 4),
    "dsp_attn_relpos": (_I, [_P] * 7 + [_I, _I, _P, _P, _I, _P, _SZ] + [_I64] * 4 + [_I] * 3
                        + [_c.POINTER(_I64)] * 3 + [_F, _I, _P]),
    "dsp_attn_relpos_bwd_workspace_bytes": (_SZ, [_I64] * 4 + [_I] * 5),
    "dsp_attn_relpos_bwd": (_I, [_P] * 12 + [_I, _I, _P, _P, _I, _P, _SZ] + [_I64] * 4 + [_I] * 3
                            + [_c.POINTER(_I64)] * 3 + [_F, _I, _P]),
    "dsp_qk_norm_rope": (_I, [_P] * 9 + [_I64, _I, _I, _I64, _I64, _I64, _I, _I, _I] + [_c.POINTER(_I64)] * 4
                         + [_F, _I, _P]),
    "dsp_qk_norm_rope_bwd_workspace_bytes": (_SZ, [_I64, _I64, _I64, _I, _I, _I]),
    "dsp_qk_norm_rope_bwd": (_I, [_P] * 13 + [_I64, _I, _I, _P, _SZ, _I64, _I64, _I64, _I, _I, _I]
                             + [_c.POINTER(_I64)] * 6 + [_F, _I, _P]),
    "dsp_layernorm": (_I, [_P, _I, _P, _I, _I64, _I, _F, _P]),
    "dsp_attn_general": (_I, [_P, _P, _P, _P, _P, _I64, _I64, _I64, _I64, _I, _I, _I, _c.POINTER(_I64),
                              _c.POINTER(_I64), _c.POINTER(_I64), _F, _I, _P]),
    "dsp_attn_general_bwd": (_I, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I64, _I64, _I64, _I64, _I, _I, _I,
                                  _c.POINTER(_I64), _c.POINTER(_I64), _c.POINTER(_I64), _F, _I, _P]),
    "dsp_layernorm_bwd": (_I, [_P, _I, _P, _I, _P, _P, _I64, _I, _F, _P]),
    "dsp_linear_bwd_data": (_I, [_P, _P, _P, _P, _I64, _I, _I, _I, _I, _P]),
    "dsp_linear_bwd_weight_workspace_bytes": (_SZ, [_I64, _I, _I, _I]),
    "dsp_linear_bwd_weight": (_I, [_P, _P, _P, _P, _P, _SZ, _I64, _I, _I, _I, _P]),
    "dsp_linear": (_I, [_P, _P, _P, _P, _P, _I64, _I, _I, _I, _I, _P]),
    "dsp_st_block_workspace_bytes": (_SZ, [_I64, _I64, _I64, _I, _I, _I, _I]),
    "dsp_st_block_train_saved_bytes": (_SZ, [_I64, _I64, _I64, _I, _I, _I, _I, _I]),
    "dsp_probe_mfma_workspace_bytes": (_SZ, []),
    "dsp_probe_mfma_flops": (_c.c_double, [_I]),
    "dsp_probe_mfma": (_I, [_P, _SZ, _I, _P]),
    "dsp_st_block_backward_workspace_bytes": (_SZ, [_I64, _I64, _I64, _I, _I, _I, _I]),
    "dsp_st_block_forward_train": (_I, [_P, _P, _c.POINTER(BlockWeights), _P, _SZ, _I64, _I64, _I64, _I, _I,
                                        _I, _F, _I, _I, _P]),
    "dsp_st_block_backward": (_I, [_P, _P, _c.POINTER(BlockWeights), _P, _SZ, _P, _SZ, _P,
                                   _c.POINTER(BlockGrads), _I64, _I64, _I64, _I, _I, _I, _F, _I, _I, _P]),
    "dsp_st_block_forward": (_I, [_P, _P, _c.POINTER(BlockWeights), _P, _SZ, _I64, _I64, _I64, _I,
                                  _I, _I, _F, _I, _I, _P]),
}


def lib() -> ctypes.CDLL:
    """The loaded libdsp.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise RuntimeError(f"libdsp.so not found at {LIB_PATH}; build it with "
                               "`python -m paper_2403_10266_amd.build`")
        L = ctypes.CDLL(str(LIB_PATH))
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def status_str(status: int) -> str:
    return lib().dsp_status_str(int(status)).decode()


def _check_status(status: int, where: str) -> None:
    if status != DSP_OK:
        raise DspError(status, where)


# --------------------------------------------------------------------------- torch marshalling
#
# Every wrapper validates the tensors it is given (device, dtype, shape and
# strides) and raises before anything is launched: the library reads and
# writes them in place, so a tensor that does not have the layout the C entry
# point assumes is an error here, never silently copied.  New outputs and
# workspaces are allocated, and the call is enqueued, on `stream` (default:
# the current stream), so the caching allocator orders their reuse after the
# kernels that use them.

def _torch():
    import torch
    return torch


def _dtype_code(t) -> int:
    torch = _torch()
    if t.dtype == torch.float32:
        return DSP_F32
    if t.dtype == torch.bfloat16:
        return DSP_BF16
    raise TypeError(f"unsupported dtype {t.dtype}; use float32 or bfloat16")


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


class _on:
    """Context that makes `stream` current (None: leaves the current stream of the
    current device) and yields it as a ctypes handle."""
    __slots__ = ("guard", "handle")

    def __init__(self, stream):
        torch = _torch()
        if stream is None:
            # the handle alone where torch offers it (an internal function): building a
            # torch.cuda.Stream object costs 2.6 us, a sixth of a small call's host time
            self.guard = None
            device = torch.cuda.current_device()
            raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
            self.handle = raw(device) if raw else torch.cuda.current_stream(device).cuda_stream
        else:
            self.guard = torch.cuda.stream(stream)
            self.handle = stream.cuda_stream

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return ctypes.c_void_p(self.handle)

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)
        return False


_I3 = ctypes.c_int64 * 3


class _on_device(_on):
    """`_on` for calls whose tensors may be on another device than the current one: that
    device is current meanwhile (its current stream, or the given `stream` of it).
    Yields the stream's handle as a number."""
    __slots__ = ("device",)

    def __init__(self, t, stream):
        torch = _torch()
        if stream is not None and stream.device != t.device:
            raise ValueError(f"the stream is on {stream.device}, the tensors on {t.device}")
        dev = t.get_device()
        if stream is not None or dev == torch.cuda.current_device():
            self.device = None
            super().__init__(stream)
            return
        self.device = torch.cuda.device(dev)
        self.device.__enter__()
        try:
            super().__init__(None)
        except BaseException:
            self.device.__exit__(None, None, None)
            raise

    def __enter__(self):
        super().__enter__()
        return self.handle

    def __exit__(self, *exc):
        super().__exit__(*exc)
        if self.device is not None:
            self.device.__exit__(*exc)
        return False


def _as(t, dtype, shape, device) -> bool:
    """Whether t has this dtype, shape and device index: most of `_check` at a third of
    its time, for calls of a few microseconds (`_check` then says what is wrong)."""
    return t is not None and t.dtype is dtype and t.shape == shape and t.get_device() == device


def _at(t):
    """A tensor's address for an argument of pointer type, None for None."""
    return None if t is None else t.data_ptr()


def _check(where, name, t, *, dtype=None, shape=None, numel=None, contiguous=True, like=None, strides=None):
    """Raise ValueError unless tensor `t` is on the device of `like` (if given)
    and has the given dtype, shape / element count, strides or contiguity."""
    if t is None:
        raise ValueError(f"{where}: {name} is required")
    if not t.is_cuda:
        raise ValueError(f"{where}: {name} must be a device tensor")
    if like is not None and t.device != like.device:
        raise ValueError(f"{where}: {name} is on {t.device}, the inputs on {like.device}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{where}: {name} must be {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{where}: {name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{where}: {name} must have {numel} elements, got {t.numel()}")
    if strides is not None and tuple(t.stride()) != tuple(strides):
        raise ValueError(f"{where}: {name} must have strides {tuple(strides)}, got {tuple(t.stride())}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{where}: {name} must be contiguous (the library works on it in place; "
                         "pass a contiguous tensor)")
    return t


def _float_dtype(where, t):
    torch = _torch()
    if t.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError(f"{where}: unsupported dtype {t.dtype}; use float32 or bfloat16")
    return t.dtype


def _nbytes(t) -> int:
    return t.numel() * t.element_size()


def _switch_out_shape(dims, from_dim, to_dim, n_chunks):
    nd = len(dims)
    if from_dim == to_dim or not (1 <= from_dim <= nd - 2 and 1 <= to_dim <= nd - 2):
        return tuple(dims)
    others = [k for k in range(1, nd - 1) if k != from_dim]
    mid = [dims[k] // max(n_chunks, 1) if k == to_dim else dims[k] for k in others]
    return (n_chunks, dims[0], *mid, dims[from_dim], dims[-1])


def dsp_switch(x, from_dim: int, to_dim: int, n_chunks: int, out=None, variant: int = 0,
               stream=None):
    """Permute + pack of a contiguous [B, S_1, .., S_K, C] shard, K = 2 or 3 (see
    dsp.h).  Returns ``out``: a tensor of shape [n_chunks, B, (the other sequence
    dims, the to-dim cut to D_to/n_chunks), D_from, C] (or x's shape when
    from_dim == to_dim); a given ``out`` needs x's dtype and element count."""
    torch = _torch()
    w = "dsp_switch"
    _check(w, "x", x)
    dt = _float_dtype(w, x)
    if x.dim() not in (4, 5):
        raise ValueError(f"{w}: x must be [B, S_1, .., S_K, C] with K = 2 or 3")
    dims = list(x.shape)
    with _on(stream) as s:
        if out is None:
            out = torch.empty(_switch_out_shape(dims, from_dim, to_dim, n_chunks), dtype=dt, device=x.device)
        _check(w, "out", out, dtype=dt, numel=x.numel(), like=x)
        shape = (ctypes.c_int64 * x.dim())(*dims)
        _check_status(lib().dsp_switch_variant(_ptr(x), _ptr(out), shape, x.dim(), from_dim, to_dim, n_chunks,
                                               _dtype_code(x), variant, s), w)
    return out


def dsp_split(x, dim: int, n_chunks: int, rank: int, out=None, stream=None):
    """Split (primitive table, s^ -> s_i): rank ``rank``'s slice of the replicated
    contiguous tensor x [B, S_1, .., S_K, C] along sequence dimension ``dim``."""
    torch = _torch()
    w = "dsp_split"
    _check(w, "x", x)
    dt = _float_dtype(w, x)
    if x.dim() not in (4, 5):
        raise ValueError(f"{w}: x must be [B, S_1, .., S_K, C] with K = 2 or 3")
    dims = list(x.shape)
    oshape = list(dims)
    if 1 <= dim < x.dim() - 1 and n_chunks >= 1:
        oshape[dim] //= n_chunks
    with _on(stream) as s:
        if out is None:
            out = torch.empty(oshape, dtype=dt, device=x.device)
        _check(w, "out", out, dtype=dt, shape=oshape, like=x)
        shape = (ctypes.c_int64 * x.dim())(*dims)
        _check_status(lib().dsp_split(_ptr(x), _ptr(out), shape, x.dim(), dim, n_chunks, rank, _dtype_code(x), s), w)
    return out


def dsp_gather(shards, dim: int, out=None, stream=None):
    """Gather (primitive table, s_i -> s^): the concatenation along sequence
    dimension ``dim`` of N equal contiguous shards [B, S_1, .., S_K, C], in rank
    order; the receiving side of the all-gather, every rank's shard on one GPU."""
    torch = _torch()
    w = "dsp_gather"
    shards = list(shards)
    if not shards:
        raise ValueError(f"{w}: at least one shard")
    x0 = shards[0]
    _check(w, "shards[0]", x0)
    dt = _float_dtype(w, x0)
    for i, t in enumerate(shards):
        _check(w, f"shards[{i}]", t, dtype=dt, shape=x0.shape, like=x0)
    if x0.dim() not in (4, 5):
        raise ValueError(f"{w}: shards must be [B, S_1, .., S_K, C] with K = 2 or 3")
    dims = list(x0.shape)
    oshape = list(dims)
    if 1 <= dim < x0.dim() - 1:
        oshape[dim] *= len(shards)
    with _on(stream) as s:
        if out is None:
            out = torch.empty(oshape, dtype=dt, device=x0.device)
        _check(w, "out", out, dtype=dt, shape=oshape, like=x0)
        ptrs = (ctypes.c_void_p * len(shards))(*[t.data_ptr() for t in shards])
        shape = (ctypes.c_int64 * x0.dim())(*dims)
        _check_status(lib().dsp_gather(ptrs, _ptr(out), shape, x0.dim(), dim, len(shards), _dtype_code(x0), s), w)
    return out


def _row_views(w, q, k, v, C, ld_in):
    """q, k, v: 4-D views [B, X, L, >= C] whose (B, X, L) rows follow each other
    at stride ld_in (a dense tensor, or a column slice of a packed one)."""
    for name, t in (("q", q), ("k", k), ("v", v)):
        _check(w, name, t, contiguous=False, like=q, dtype=q.dtype)
        if t.dim() != 4 or tuple(t.shape[:3]) != tuple(q.shape[:3]) or t.shape[3] < C:
            raise ValueError(f"{w}: {name} must be a 4-D view [B, X, L, >= {C}] like q")
        B, X, L = t.shape[:3]
        want = (X * L * ld_in, L * ld_in, ld_in, 1)
        if any(n > 1 and st != ws for n, st, ws in zip(t.shape, t.stride(), want)):
            raise ValueError(f"{w}: {name} must have row stride {ld_in} with rows packed densely "
                             f"(strides {want}), got {tuple(t.stride())}")
    _float_dtype(w, q)


def _attn(name, q, k, v, B, X, L, H, out, ld_in, ld_out, scale, stream, C):
    torch = _torch()
    if C % H:
        raise ValueError(f"{name}: C = {C} is not a multiple of H = {H}")
    _row_views(name, q, k, v, C, ld_in)
    with _on(stream) as s:
        if out is None:
            if ld_out is not None and ld_out != C:
                raise ValueError(f"{name}: pass `out` for an output row stride other than C")
            out = torch.empty((B, X, L, C), dtype=q.dtype, device=q.device)
        if ld_out is None:
            ld_out = out.stride(2)
        _row_views(name, out, out, out, C, ld_out)
        _check(name, "out", out, dtype=q.dtype, like=q, contiguous=False)
        if tuple(out.shape[:3]) != (B, X, L):
            raise ValueError(f"{name}: out must be [B, X, L, >= C] like q")
        fn = getattr(lib(), name)
        _check_status(fn(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, X, L, H, C // H, ld_in, ld_out, float(scale),
                         _dtype_code(q), s), name)
    return out


def dsp_exchange_unpack(packed, out=None, stream=None):
    """Exchange + unpack of N ranks' packed switch outputs on one GPU (see
    dsp.h).  ``packed``: N contiguous tensors of shape [N, B, P, F, C] (same
    dtype).  Returns N tensors of shape [B, P, N*F, C]: rank n's result."""
    torch = _torch()
    w = "dsp_exchange_unpack"
    packed = list(packed)
    N = len(packed)
    if N == 0:
        raise ValueError(f"{w}: no ranks")
    p0 = packed[0]
    _check(w, "packed[0]", p0)
    dt = _float_dtype(w, p0)
    shape = tuple(p0.shape)
    if len(shape) != 5 or shape[0] != N:
        raise ValueError(f"{w}: packed[0] has shape {shape}, want [N={N}, B, P, F, C]")
    for i, t in enumerate(packed):
        _check(w, f"packed[{i}]", t, dtype=dt, shape=shape, like=p0)
    _, B, P, F, C = shape
    with _on(stream) as s:
        if out is None:
            out = [torch.empty((B, P, N * F, C), dtype=dt, device=p0.device) for _ in range(N)]
        out = list(out)
        if len(out) != N:
            raise ValueError(f"{w}: out must hold N = {N} tensors")
        for i, o in enumerate(out):
            _check(w, f"out[{i}]", o, dtype=dt, shape=(B, P, N * F, C), like=p0)
        src = (ctypes.c_void_p * N)(*[t.data_ptr() for t in packed])
        dst = (ctypes.c_void_p * N)(*[o.data_ptr() for o in out])
        shp = (ctypes.c_int64 * 5)(N, B, P, F, C)
        _check_status(lib().dsp_exchange_unpack(src, dst, shp, _dtype_code(p0), s), w)
    return out


def dsp_spatial_attn(q, k, v, H: int, out=None, scale: float = 0.0, C: int | None = None,
                     ld_in: int | None = None, ld_out: int | None = None, stream=None):
    """Attention over S within each frame.  q, k, v: (B, T, S, ld_in) views whose
    first C = H*D columns hold the heads (pass C explicitly for packed QKV views)."""
    B, T, S = q.shape[0], q.shape[1], q.shape[2]
    C = C if C is not None else q.shape[3]
    ld_in = ld_in if ld_in is not None else q.stride(2)
    return _attn("dsp_spatial_attn", q, k, v, B, T, S, H, out, ld_in, ld_out, scale, stream, C)


def dsp_temporal_attn(q, k, v, H: int, out=None, scale: float = 0.0, C: int | None = None,
                      ld_in: int | None = None, ld_out: int | None = None, stream=None):
    """Attention over T at each spatial location.  q, k, v: (B, S, T, ld_in) views."""
    B, S, T = q.shape[0], q.shape[1], q.shape[2]
    C = C if C is not None else q.shape[3]
    ld_in = ld_in if ld_in is not None else q.stride(2)
    return _attn("dsp_temporal_attn", q, k, v, B, S, T, H, out, ld_in, ld_out, scale, stream, C)


def _qkv_views(where, q, k, v, H):
    for name, t in (("q", q), ("k", k), ("v", v)):
        _check(where, name, t, contiguous=False, like=q, dtype=q.dtype)
    _float_dtype(where, q)
    if q.dim() != 4 or q.shape != k.shape or q.shape != v.shape:
        raise ValueError(f"{where}: q, k, v must be 4-D views of one shape [B, X, L, C]")
    if q.stride() != k.stride() or q.stride() != v.stride() or q.stride(3) != 1:
        raise ValueError(f"{where}: q, k, v must share strides, with a unit last stride")
    B, X, L, C = q.shape
    if C % H:
        raise ValueError(f"{where}: C must be a multiple of H")
    return B, X, L, C


def _like_view(where, t, like, name):
    _check(where, name, t, contiguous=False, like=like, dtype=like.dtype)
    if t.shape != like.shape or t.stride(3) != 1:
        raise ValueError(f"{where}: {name} must be a view of shape {tuple(like.shape)} with a unit last stride")


def dsp_attn_strided(q, k, v, H: int, out=None, scale: float = 0.0, stream=None):
    """Attention over dim 2 of the 4-D views q, k, v [B, X, L, >=H*D] (any
    strides, last one 1, the same for q, k and v), per (b, x, head): e.g.
    temporal attention on a (B, T, S, C) tensor x is ``q = x.permute(0, 2, 1, 3)``.
    The output is a new contiguous [B, X, L, C] tensor, or ``out`` (any 4-D
    view with last stride 1)."""
    torch = _torch()
    w = "dsp_attn_strided"
    B, X, L, C = _qkv_views(w, q, k, v, H)
    with _on(stream) as s:
        if out is None:
            out = torch.empty((B, X, L, C), dtype=q.dtype, device=q.device)
        _like_view(w, out, q, "out")
        ins = (ctypes.c_int64 * 3)(*q.stride()[:3])
        outs = (ctypes.c_int64 * 3)(*out.stride()[:3])
        _check_status(lib().dsp_attn_strided(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, X, L, H, C // H, ins, outs,
                                             float(scale), _dtype_code(q), s), w)
    return out


def dsp_attn_fwd_lse(q, k, v, H: int, out=None, lse=None, scale: float = 0.0, stream=None):
    """dsp_attn_strided that also returns the row log-sum-exp: (out, lse) with
    lse a float32 tensor [B, X, H, L]."""
    torch = _torch()
    w = "dsp_attn_fwd_lse"
    B, X, L, C = _qkv_views(w, q, k, v, H)
    with _on(stream) as s:
        if out is None:
            out = torch.empty((B, X, L, C), dtype=q.dtype, device=q.device)
        _like_view(w, out, q, "out")
        if lse is None:
            lse = torch.empty((B, X, H, L), dtype=torch.float32, device=q.device)
        _check(w, "lse", lse, dtype=torch.float32, numel=B * X * H * L, like=q)
        ins = (ctypes.c_int64 * 3)(*q.stride()[:3])
        outs = (ctypes.c_int64 * 3)(*out.stride()[:3])
        _check_status(lib().dsp_attn_fwd_lse(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), B, X, L, H, C // H,
                                             ins, outs, float(scale), _dtype_code(q), s), w)
    return out, lse


def dsp_attn_bwd(q, k, v, o, dout, lse, H: int, dq=None, dk=None, dv=None, delta=None,
                 scale: float = 0.0, stream=None):
    """Gradients (dq, dk, dv) of attention over dim 2 of the 4-D views q, k, v
    (as dsp_attn_strided), given its output o, the row log-sum-exp ``lse``
    from dsp_attn_fwd_lse and the output gradient ``dout`` (o and dout share
    one layout).  New contiguous gradients unless dq/dk/dv (views with the
    strides of q) are given.  ``delta``: optional float32 workspace of
    B*X*H*L elements (holds rowsum(dout * o) on return)."""
    torch = _torch()
    w = "dsp_attn_bwd"
    B, X, L, C = _qkv_views(w, q, k, v, H)
    _like_view(w, o, q, "o")
    _like_view(w, dout, q, "dout")
    if dout.stride() != o.stride():
        raise ValueError(f"{w}: dout must have the strides of o")
    _check(w, "lse", lse, dtype=torch.float32, numel=B * X * H * L, like=q)
    with _on(stream) as s:
        if dq is None or dk is None or dv is None:
            if not q.is_contiguous():
                raise ValueError(f"{w}: for a non-contiguous q pass dq, dk, dv views with its strides")
            dq, dk, dv = (torch.empty_like(q) if g is None else g for g in (dq, dk, dv))
        for g, name in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
            _like_view(w, g, q, name)
            if tuple(g.stride()) != tuple(q.stride()):
                raise ValueError(f"{w}: {name} must have the strides of q, k, v")
        if delta is None:
            delta = torch.empty(B * X * H * L, dtype=torch.float32, device=q.device)
        _check(w, "delta", delta, dtype=torch.float32, numel=B * X * H * L, like=q)
        qs = (ctypes.c_int64 * 3)(*q.stride()[:3])
        os_ = (ctypes.c_int64 * 3)(*o.stride()[:3])
        _check_status(lib().dsp_attn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(dout), _ptr(lse), _ptr(dq),
                                         _ptr(dk), _ptr(dv), _ptr(delta), B, X, L, H, C // H, qs, os_,
                                         float(scale), _dtype_code(q), s), w)
    return dq, dk, dv


def attn_bwd_noalloc_max_rows() -> int:
    """Largest B*X*H*L that dsp_attn_bwd_noalloc accepts."""
    return int(lib().dsp_attn_bwd_noalloc_max_rows())


def dsp_attn_bwd_noalloc(q, k, v, o, dout, lse, H: int, dq, dk, dv, scale: float = 0.0, stream=None):
    """dsp_attn_bwd for callers that cannot allocate: no Delta workspace (the
    library keeps Delta in a static per-device array; calls overlapping on one
    GPU race) and caller-given dq, dk, dv (views with the strides of q)."""
    torch = _torch()
    w = "dsp_attn_bwd_noalloc"
    B, X, L, C = _qkv_views(w, q, k, v, H)
    _like_view(w, o, q, "o")
    _like_view(w, dout, q, "dout")
    if dout.stride() != o.stride():
        raise ValueError(f"{w}: dout must have the strides of o")
    _check(w, "lse", lse, dtype=torch.float32, numel=B * X * H * L, like=q)
    for g, name in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
        _like_view(w, g, q, name)
        if tuple(g.stride()) != tuple(q.stride()):
            raise ValueError(f"{w}: {name} must have the strides of q, k, v")
    with _on(stream) as s:
        qs = (ctypes.c_int64 * 3)(*q.stride()[:3])
        os_ = (ctypes.c_int64 * 3)(*o.stride()[:3])
        _check_status(lib().dsp_attn_bwd_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(dout), _ptr(lse),
                                                 _ptr(dq), _ptr(dk), _ptr(dv), B, X, L, H, C // H, qs, os_,
                                                 float(scale), _dtype_code(q), s), w)
    return dq, dk, dv


def dsp_layernorm(x, eps: float = 1e-6, out=None, out_dtype=None, stream=None):
    """y = (x - mean) / sqrt(var + eps) over the last dimension of the
    contiguous x; y in out_dtype (default x's), or into ``out``."""
    torch = _torch()
    w = "dsp_layernorm"
    _check(w, "x", x)
    _float_dtype(w, x)
    C = x.shape[-1]
    rows = x.numel() // C if C else 0
    with _on(stream) as s:
        if out is None:
            out = torch.empty(x.shape, dtype=out_dtype or x.dtype, device=x.device)
        _check(w, "out", out, shape=x.shape, like=x)
        _float_dtype(w, out)
        _check_status(lib().dsp_layernorm(_ptr(x), _dtype_code(x), _ptr(out), _dtype_code(out), rows, C,
                                          float(eps), s), w)
    return out


def _same_layout(a, b) -> bool:
    """Whether a and b, of one shape, have the same strides where a dimension has more than
    one element (the others' say nothing)."""
    return a.stride() == b.stride() or a.numel() == 0 or all(
        n < 2 or s == t for n, s, t in zip(a.shape, a.stride(), b.stride()))


def _st3(t):
    return (ctypes.c_int64 * 3)(*t.stride()[:3])


def _general_views(w, q, k, v, H, Hkv, same=lambda a, b: a.stride() == b.stride()):
    for name, t in (("q", q), ("k", k), ("v", v)):
        _check(w, name, t, contiguous=False, like=q, dtype=q.dtype)
    _float_dtype(w, q)
    if q.dim() != 4 or k.dim() != 4 or k.shape != v.shape or not same(k, v) or q.stride(3) != 1 or k.stride(3) != 1:
        raise ValueError(f"{w}: q [B, X, Lq, C] and k, v [B, X, Lk, Ckv] views of one layout")
    B, X, Lq, C = q.shape
    if H < 1 or Hkv < 1 or C % H or tuple(k.shape[:2]) != (B, X):
        raise ValueError(f"{w}: shapes do not match")
    D = C // H
    if k.shape[3] != Hkv * D:
        raise ValueError(f"{w}: k and v must hold Hkv heads of the query head width")
    return B, X, Lq, k.shape[2], C, D


def dsp_attn_general(q, k, v, H: int, Hkv: int, out=None, lse=None, with_lse: bool = False,
                     scale: float = 0.0, stream=None):
    """Grouped-query / multi-query / cross-attention over dim 2 of 4-D views:
    q [B, X, Lq, H*D], k and v [B, X, Lk, Hkv*D] (same strides; a 0 stride
    broadcasts).  Returns out [B, X, Lq, H*D] (and lse [B, X, H, Lq] fp32 when
    with_lse or lse is given)."""
    torch = _torch()
    w = "dsp_attn_general"
    B, X, Lq, Lk, C, D = _general_views(w, q, k, v, H, Hkv)
    with _on(stream) as s:
        if out is None:
            out = torch.empty((B, X, Lq, C), dtype=q.dtype, device=q.device)
        _like_view(w, out, q, "out")
        if with_lse and lse is None:
            lse = torch.empty((B, X, H, Lq), dtype=torch.float32, device=q.device)
        if lse is not None:
            _check(w, "lse", lse, dtype=torch.float32, numel=B * X * H * Lq, like=q)
        _check_status(lib().dsp_attn_general(_ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), B, X, Lq, Lk, H,
                                             Hkv, D, _st3(q), _st3(k), _st3(out), float(scale), _dtype_code(q), s), w)
    return (out, lse) if lse is not None else out


def dsp_attn_general_bwd(q, k, v, o, dout, lse, H: int, Hkv: int, dq=None, dk=None, dv=None, delta=None,
                         scale: float = 0.0, stream=None):
    """Gradients of dsp_attn_general: (dq like q, dk and dv like k and v)."""
    torch = _torch()
    w = "dsp_attn_general_bwd"
    B, X, Lq, Lk, C, D = _general_views(w, q, k, v, H, Hkv)
    _like_view(w, o, q, "o")
    _like_view(w, dout, q, "dout")
    if dout.stride() != o.stride():
        raise ValueError(f"{w}: dout must have the strides of o")
    _check(w, "lse", lse, dtype=torch.float32, numel=B * X * H * Lq, like=q)
    with _on(stream) as s:
        dq = torch.empty_like(q) if dq is None else dq
        dk = torch.empty_like(k) if dk is None else dk
        dv = torch.empty_like(v) if dv is None else dv
        _check(w, "dq", dq, dtype=q.dtype, shape=q.shape, strides=q.stride(), contiguous=False, like=q)
        _check(w, "dk", dk, dtype=q.dtype, shape=k.shape, strides=k.stride(), contiguous=False, like=q)
        _check(w, "dv", dv, dtype=q.dtype, shape=k.shape, strides=k.stride(), contiguous=False, like=q)
        if delta is None:
            delta = torch.empty(B * X * H * Lq, dtype=torch.float32, device=q.device)
        _check(w, "delta", delta, dtype=torch.float32, numel=B * X * H * Lq, like=q)
        _check_status(lib().dsp_attn_general_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(dout), _ptr(lse),
                                                 _ptr(dq), _ptr(dk), _ptr(dv), _ptr(delta), B, X, Lq, Lk, H, Hkv, D,
                                                 _st3(q), _st3(k), _st3(o), float(scale), _dtype_code(q), s), w)
    return dq, dk, dv


def dsp_relpos_buckets(max_dist: int, n_buckets: int, bidirectional: bool = True):
    """The usual map of distances -max_dist .. max_dist to buckets (see dsp.h): int32
    [2 * max_dist + 1] on the CPU, for `.cuda()` once."""
    torch = _torch()
    w = "dsp_relpos_buckets"
    if max_dist < 0:
        raise ValueError(f"{w}: max_dist must not be negative")
    out = torch.empty(2 * max_dist + 1, dtype=torch.int32)
    _check_status(lib().dsp_relpos_buckets(_ptr(out), max_dist, n_buckets, 1 if bidirectional else 0), w)
    return out


def _relpos_args(w, q, k, v, H, Hkv, bias, buckets, q_pos, kv_len):
    torch = _torch()
    dims = _general_views(w, q, k, v, H, Hkv, _same_layout)
    dev = q.get_device()
    if not (_as(bias, q.dtype, (bias.shape[0] if bias is not None and bias.dim() else 0, H), dev)
            and bias.shape[0] > 0 and bias.is_contiguous()):
        _check(w, "bias", bias, dtype=q.dtype, like=q)
        raise ValueError(f"{w}: bias must be [n_buckets, H = {H}]")
    if not (_as(buckets, torch.int32, (buckets.numel() | 1 if buckets is not None else 0,), dev)
            and buckets.is_contiguous()):
        _check(w, "buckets", buckets, dtype=torch.int32, like=q)
        raise ValueError(f"{w}: buckets must be [2 * max_dist + 1]")
    for name, t in (("q_pos", q_pos), ("kv_len", kv_len)):
        if t is not None and not (_as(t, torch.int32, dims[:1], dev) and t.is_contiguous()):
            _check(w, name, t, dtype=torch.int32, shape=dims[:1], like=q)
    return dims


def _workspace(w, need, workspace, like):
    """The given workspace, or a new one of `need` bytes (None where none is needed)."""
    torch = _torch()
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=like.device) if need else None
    return _check(w, "workspace", workspace, like=like)


def dsp_attn_relpos(q, k, v, H: int, Hkv: int, bias, buckets, causal: bool = False, q_pos=None, kv_len=None, out=None,
                    lse=None, with_lse: bool = False, scale: float = 0.0, workspace=None, stream=None):
    """Attention with a learned relative position bias (see dsp.h) over dim 2 of 4-D
    views q [B, X, Lq, H*D], k and v [B, X, Lk, Hkv*D].  ``bias`` [n_buckets, H] of
    q's dtype, ``buckets`` int32 [2 * max_dist + 1] (dsp_relpos_buckets), ``q_pos``
    and ``kv_len`` int32 [B]: the key index of the first query and the keys of each
    sequence (default 0 and Lk).  Returns out [B, X, Lq, H*D] (and lse
    [B, X, H, Lq] fp32 when with_lse or lse is given)."""
    torch = _torch()
    w = "dsp_attn_relpos"
    B, X, Lq, Lk, C, D = _relpos_args(w, q, k, v, H, Hkv, bias, buckets, q_pos, kv_len)
    with _on_device(q, stream) as s:
        if out is None:
            out = torch.empty((B, X, Lq, C), dtype=q.dtype, device=q.device)
        _like_view(w, out, q, "out")
        if with_lse and lse is None:
            lse = torch.empty((B, X, H, Lq), dtype=torch.float32, device=q.device)
        if lse is not None:
            _check(w, "lse", lse, dtype=torch.float32, numel=B * X * H * Lq, like=q)
        dt = _dtype_code(q)
        L = lib()
        ws = _workspace(w, L.dsp_attn_relpos_workspace_bytes(B, X, Lq, Lk, H, Hkv, D, dt), workspace, q)
        _check_status(L.dsp_attn_relpos(
            q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), _at(lse), bias.data_ptr(), buckets.data_ptr(),
            bias.shape[0], buckets.numel() // 2, _at(q_pos), _at(kv_len), DSP_RELPOS_CAUSAL if causal else 0, _at(ws),
            _nbytes(ws) if ws is not None else 0, B, X, Lq, Lk, H, Hkv, D, _I3(*q.stride()[:3]), _I3(*k.stride()[:3]),
            _I3(*out.stride()[:3]), scale, dt, s), w)
    return (out, lse) if lse is not None else out


def _relpos_grads(w, q, k, v, dq, dk, dv):
    """The gradients given, and new ones laid out like their inputs for the others; for
    columns of packed rows ([Q | K | V]) without any, the columns of one new buffer."""
    torch = _torch()
    ins, grads = (q, k, v), [dq, dk, dv]
    for i, (name, t) in enumerate(zip("qkv", ins)):
        if grads[i] is None:
            if any(n > 1 and s == 0 for n, s in zip(t.shape, t.stride())):
                raise ValueError(f"{w}: {name} broadcasts, so its rows have no gradient of their own; pass a copy")
            if t.is_contiguous():
                grads[i] = torch.empty_like(t)
    if all(g is None for g in grads) and q.shape[:3] == k.shape[:3] and _same_layout(q[..., :1], k[..., :1]) \
            and len({t.untyped_storage().data_ptr() for t in ins}) == 1:
        pitch = min((s for n, s in zip(q.shape[:3], q.stride()) if n > 1), default=0)
        first = min(t.storage_offset() for t in ins)
        cols = [(t.storage_offset() - first, t.storage_offset() - first + t.shape[3]) for t in ins]
        order = sorted(cols)
        if order[2][1] <= pitch and all(a[1] <= b[0] for a, b in zip(order, order[1:])):
            row = torch.empty_strided((*q.shape[:3], order[2][1]), q.stride(), dtype=q.dtype, device=q.device)
            return [row[..., a:b] for a, b in cols]
    return [torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=t.device) if g is None else g
            for t, g in zip(ins, grads)]


def dsp_attn_relpos_bwd(q, k, v, o, dout, lse, H: int, Hkv: int, bias, buckets, causal: bool = False, q_pos=None,
                        kv_len=None, dq=None, dk=None, dv=None, dbias=None, scale: float = 0.0, workspace=None,
                        stream=None):
    """Gradients of dsp_attn_relpos, given its o and lse and the gradient dout (o's
    strides): (dq like q, dk and dv like k and v, dbias like bias), each with its input's
    strides.  New ones for columns of a packed projection are columns of one buffer."""
    torch = _torch()
    w = "dsp_attn_relpos_bwd"
    B, X, Lq, Lk, C, D = _relpos_args(w, q, k, v, H, Hkv, bias, buckets, q_pos, kv_len)
    _like_view(w, o, q, "o")
    _like_view(w, dout, q, "dout")
    if not _same_layout(dout, o):
        raise ValueError(f"{w}: dout must have the strides of o")
    _check(w, "lse", lse, dtype=torch.float32, numel=B * X * H * Lq, like=q)
    with _on_device(q, stream) as s:
        dq, dk, dv = _relpos_grads(w, q, k, v, dq, dk, dv)
        for name, g, x in (("dq", dq, q), ("dk", dk, k), ("dv", dv, k)):
            _check(w, name, g, dtype=q.dtype, shape=x.shape, contiguous=False, like=q)
            if not _same_layout(g, x):
                raise ValueError(f"{w}: {name} must have the strides of its input, {x.stride()}, got {g.stride()}")
        dbias = torch.empty_like(bias) if dbias is None else dbias
        _check(w, "dbias", dbias, dtype=q.dtype, shape=bias.shape, like=q)
        dt, M = _dtype_code(q), buckets.numel() // 2
        L = lib()
        ws = _workspace(w, L.dsp_attn_relpos_bwd_workspace_bytes(B, X, Lq, Lk, H, Hkv, D, M, dt), workspace, q)
        _check_status(L.dsp_attn_relpos_bwd(
            q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), dout.data_ptr(), lse.data_ptr(), dq.data_ptr(),
            dk.data_ptr(), dv.data_ptr(), dbias.data_ptr(), bias.data_ptr(), buckets.data_ptr(), bias.shape[0], M,
            _at(q_pos), _at(kv_len), DSP_RELPOS_CAUSAL if causal else 0, _at(ws),
            _nbytes(ws) if ws is not None else 0, B, X, Lq, Lk, H, Hkv, D, _I3(*q.stride()[:3]), _I3(*k.stride()[:3]),
            _I3(*o.stride()[:3]), scale, dt, s), w)
    return dq, dk, dv, dbias


def _norm_rope_args(w, q, k, H, Hkv, gq, gk, cos, sin, pos):
    """Checks what dsp_qk_norm_rope and its gradient share; returns (B, X, L, D, P, rot)."""
    torch = _torch()
    x, n = (q, H) if q is not None else (k, Hkv)
    _check(w, "q" if q is not None else "k", x, contiguous=False)
    dt, dev = _float_dtype(w, x), x.get_device()
    if (q is None) != (H == 0) or (k is None) != (Hkv == 0):
        raise ValueError(f"{w}: q has H heads and k has Hkv heads (None: 0)")
    if x.dim() != 4 or n < 1 or x.shape[3] % n:
        raise ValueError(f"{w}: q and k must be 4-D views [B, X, L, heads * D]")
    B, X, L, C = x.shape
    D = C // n
    for name, t, heads, g in (("q", q, H, gq), ("k", k, Hkv, gk)):
        if t is None:
            continue
        if not _as(t, dt, (B, X, L, heads * D), dev):
            _check(w, name, t, dtype=dt, shape=(B, X, L, heads * D), contiguous=False, like=x)
        if t.stride(3) != 1:
            raise ValueError(f"{w}: {name} must have a unit last stride")
        if g is not None and not (_as(g, dt, (D,), dev) and g.is_contiguous()):
            _check(w, "g" + name, g, dtype=dt, shape=(D,), like=x)
    if (cos is None) != (sin is None):
        raise ValueError(f"{w}: cos and sin come together")
    P = rot = 0
    if cos is not None:
        shape, f32 = cos.shape, torch.float32
        if len(shape) != 2:
            raise ValueError(f"{w}: cos must be [P, rot / 2]")
        for name, t in (("cos", cos), ("sin", sin)):
            if not (_as(t, f32, shape, dev) and t.is_contiguous()):
                _check(w, name, t, dtype=f32, shape=shape, like=x)
        P, rot = shape[0], 2 * shape[1]
    if pos is not None and not (_as(pos, torch.int32, (B, L), dev) and pos.is_contiguous()):
        _check(w, "pos", pos, dtype=torch.int32, shape=(B, L), like=x)
    return B, X, L, D, P, rot


def _norm_rope_out(w, name, o, t):
    """The given output for t, checked, or a new one; None without t."""
    if t is None:
        return None
    if o is None:
        return _torch().empty(t.shape, dtype=t.dtype, device=t.device)
    if not (_as(o, t.dtype, t.shape, t.get_device()) and o.stride(3) == 1):
        _like_view(w, o, t, name)
    return o


def _strides(t):
    return None if t is None else _I3(*t.stride()[:3])


def dsp_qk_norm_rope(q, k, H: int, Hkv: int, gq=None, gk=None, cos=None, sin=None, pos=None,
                     interleaved: bool = False, eps: float = 1e-6, out_q=None, out_k=None, stream=None):
    """Norm of queries and keys for each head and the rotation by position in one
    pass (see dsp.h): q [B, X, L, H*D] and k [B, X, L, Hkv*D], 4-D views with any
    strides (columns of a packed projection among them) and a unit last one; either
    may be None with 0 heads.  ``gq``, ``gk``: gains [D] of q's dtype.  ``cos``,
    ``sin``: float32 [P, rot/2]; the first rot elements of a head turn, in pairs
    (i, i + rot/2) or, ``interleaved``, (2i, 2i + 1).  ``pos``: int32 [B, L], the
    table's row of each token (default: its place l; without a row: NaN).  Returns
    (yq, yk): new contiguous tensors, or ``out_q`` and ``out_k`` (q and k
    themselves: in place)."""
    torch = _torch()
    w = "dsp_qk_norm_rope"
    B, X, L, D, P, rot = _norm_rope_args(w, q, k, H, Hkv, gq, gk, cos, sin, pos)
    like = q if q is not None else k
    with _on_device(like, stream) as s:
        yq, yk = _norm_rope_out(w, "out_q", out_q, q), _norm_rope_out(w, "out_k", out_k, k)
        _check_status(lib().dsp_qk_norm_rope(
            _at(q), _at(k), _at(yq), _at(yk), _at(gq), _at(gk), _at(cos), _at(sin), _at(pos), P, rot,
            DSP_ROPE_ADJACENT if interleaved else 0, B, X, L, H, Hkv, D, _strides(q), _strides(k), _strides(yq),
            _strides(yk), eps, _dtype_code(like), s), w)
    return yq, yk


def dsp_qk_norm_rope_bwd(q, k, dyq, dyk, H: int, Hkv: int, gq=None, gk=None, cos=None, sin=None, pos=None,
                         interleaved: bool = False, eps: float = 1e-6, dq=None, dk=None, gains: bool = True,
                         workspace=None, stream=None):
    """Gradient of dsp_qk_norm_rope at its inputs q and k: (dq, dk, dgq, dgk) from
    the gradients dyq, dyk of its outputs (views of any strides).  dq and dk are new
    contiguous tensors, or views given (dyq and dyk themselves: in place); dgq and
    dgk are float32 [D], None without ``gains`` or without the side."""
    torch = _torch()
    w = "dsp_qk_norm_rope_bwd"
    B, X, L, D, P, rot = _norm_rope_args(w, q, k, H, Hkv, gq, gk, cos, sin, pos)
    like = q if q is not None else k
    with _on_device(like, stream) as s:
        dg = []
        for t, dy, name in ((q, dyq, "dyq"), (k, dyk, "dyk")):
            if t is None:
                if dy is not None:
                    raise ValueError(f"{w}: {name} without its input")
            elif not (_as(dy, t.dtype, t.shape, t.get_device()) and dy.stride(3) == 1):
                _like_view(w, dy, t, name)
            dg.append(torch.empty(D, dtype=torch.float32, device=like.device) if gains and t is not None else None)
        dq, dk = _norm_rope_out(w, "dq", dq, q), _norm_rope_out(w, "dk", dk, k)
        need = lib().dsp_qk_norm_rope_bwd_workspace_bytes(B, X, L, H, Hkv, D) if gains else 0
        workspace = _workspace(w, need, workspace, like)
        _check_status(lib().dsp_qk_norm_rope_bwd(
            _at(q), _at(k), _at(dyq), _at(dyk), _at(dq), _at(dk), _at(dg[0]), _at(dg[1]), _at(gq), _at(gk), _at(cos),
            _at(sin), _at(pos), P, rot, DSP_ROPE_ADJACENT if interleaved else 0, _at(workspace),
            _nbytes(workspace) if workspace is not None else 0, B, X, L, H, Hkv, D, _strides(q), _strides(k),
            _strides(dyq), _strides(dyk), _strides(dq), _strides(dk), eps, _dtype_code(like), s), w)
    return dq, dk, dg[0], dg[1]


def dsp_layernorm_bwd(x, dy, eps: float = 1e-6, dres=None, out=None, stream=None):
    """dx (fp32) = dres + the LayerNorm backward of dy at x (contiguous rows of C)."""
    torch = _torch()
    w = "dsp_layernorm_bwd"
    _check(w, "x", x)
    _float_dtype(w, x)
    _check(w, "dy", dy, shape=x.shape, like=x)
    _float_dtype(w, dy)
    if dres is not None:
        _check(w, "dres", dres, dtype=torch.float32, shape=x.shape, like=x)
    C = x.shape[-1]
    rows = x.numel() // C if C else 0
    with _on(stream) as s:
        if out is None:
            out = torch.empty(x.shape, dtype=torch.float32, device=x.device)
        _check(w, "out", out, dtype=torch.float32, shape=x.shape, like=x)
        _check_status(lib().dsp_layernorm_bwd(_ptr(x), _dtype_code(x), _ptr(dy), _dtype_code(dy), _ptr(dres),
                                              _ptr(out), rows, C, float(eps), s), w)
    return out


def dsp_linear(a, w, bias=None, residual=None, epilogue: int = DSP_EPI_NONE, out=None,
               stream=None):
    """out = epilogue(a @ w.T + bias); a [..., K] and w [N, K] contiguous, one dtype."""
    torch = _torch()
    where = "dsp_linear"
    _check(where, "a", a)
    dt = _float_dtype(where, a)
    K = a.shape[-1]
    M = a.numel() // K if K else 0
    _check(where, "w", w, dtype=dt, like=a)
    if w.dim() != 2 or w.shape[1] != K:
        raise ValueError(f"{where}: w must be [N, K = {K}]")
    N = w.shape[0]
    if bias is not None:
        _check(where, "bias", bias, dtype=dt, numel=N, like=a)
    oshape = (*a.shape[:-1], N)
    if residual is not None:
        _check(where, "residual", residual, dtype=torch.float32, numel=M * N, like=a)
    odt = torch.float32 if epilogue in (DSP_EPI_RESID, DSP_EPI_F32) else dt
    with _on(stream) as s:
        if out is None:
            out = torch.empty(oshape, dtype=odt, device=a.device)
        _check(where, "out", out, dtype=odt, numel=M * N, like=a)
        _check_status(lib().dsp_linear(_ptr(a), _ptr(w), _ptr(bias), _ptr(residual), _ptr(out), M, N, K,
                                       epilogue, _dtype_code(a), s), where)
    return out


def dsp_linear_bwd_data(dy, w, u=None, epilogue: int = DSP_GRAD_EPI_F32, out=None, stream=None):
    """dx = epilogue(dy @ w) for y = x @ w.T (w stored [N, K]); u: the saved
    pre-activation [..., K] for the GELU/ReLU backward epilogues."""
    torch = _torch()
    where = "dsp_linear_bwd_data"
    _check(where, "dy", dy)
    dt = _float_dtype(where, dy)
    _check(where, "w", w, dtype=dt, like=dy)
    if w.dim() != 2 or w.shape[0] != dy.shape[-1]:
        raise ValueError(f"{where}: w must be [N = {dy.shape[-1]}, K]")
    N, K = w.shape
    M = dy.numel() // N if N else 0
    if u is not None:
        _check(where, "u", u, dtype=dt, numel=M * K, like=dy)
    odt = torch.float32 if epilogue == DSP_GRAD_EPI_F32 else dt
    with _on(stream) as s:
        if out is None:
            out = torch.empty((*dy.shape[:-1], K), dtype=odt, device=dy.device)
        _check(where, "out", out, dtype=odt, numel=M * K, like=dy)
        _check_status(lib().dsp_linear_bwd_data(_ptr(dy), _ptr(w), _ptr(u), _ptr(out), M, N, K, epilogue,
                                                _dtype_code(dy), s), where)
    return out


def dsp_linear_bwd_weight(dy, x, with_bias: bool = False, dw=None, db=None, workspace=None, stream=None):
    """(dw [N, K] fp32, db [N] fp32 or None) for y = x @ w.T + b: dw = dy^T x."""
    torch = _torch()
    where = "dsp_linear_bwd_weight"
    _check(where, "dy", dy)
    dt = _float_dtype(where, dy)
    _check(where, "x", x, dtype=dt, like=dy)
    N, K = dy.shape[-1], x.shape[-1]
    M = dy.numel() // N if N else 0
    if K == 0 or x.numel() != M * K:
        raise ValueError(f"{where}: x must hold the same {M} rows as dy")
    with _on(stream) as s:
        if dw is None:
            dw = torch.empty((N, K), dtype=torch.float32, device=dy.device)
        _check(where, "dw", dw, dtype=torch.float32, numel=N * K, like=dy)
        if with_bias and db is None:
            db = torch.empty(N, dtype=torch.float32, device=dy.device)
        if db is not None:
            _check(where, "db", db, dtype=torch.float32, numel=N, like=dy)
        need = int(lib().dsp_linear_bwd_weight_workspace_bytes(M, N, K, _dtype_code(dy)))
        if workspace is None and need:
            workspace = torch.empty(need, dtype=torch.uint8, device=dy.device)
        if workspace is not None:
            _check(where, "workspace", workspace, like=dy)
        ws_bytes = _nbytes(workspace) if workspace is not None else 0
        _check_status(lib().dsp_linear_bwd_weight(_ptr(dy), _ptr(x), _ptr(dw), _ptr(db), _ptr(workspace), ws_bytes,
                                                  M, N, K, _dtype_code(dy), s), where)
    return dw, db


def block_workspace_bytes(B, T, S, C, H, F, dtype_code) -> int:
    return int(lib().dsp_st_block_workspace_bytes(B, T, S, C, H, F, dtype_code))


def _block_args(where, x, weights, H, flags, dtype, need_mlp=True):
    """Validate x (B, T, S, C) fp32 and the weights; returns (B, T, S, C, F, code, wt)."""
    torch = _torch()
    _check(where, "x", x, dtype=torch.float32)
    if x.dim() != 4:
        raise ValueError(f"{where}: x must be (B, T, S, C)")
    B, T, S, C = x.shape
    w0 = weights.get("wqkv_s")
    if w0 is None:
        raise ValueError(f"{where}: wqkv_s is required")
    wdt = dtype or w0.dtype
    if wdt not in (torch.float32, torch.bfloat16):
        raise ValueError(f"{where}: unsupported weight dtype {wdt}")
    w1 = weights.get("w1")
    mlp = need_mlp and not (flags & DSP_BLOCK_ATTN_ONLY)
    if mlp and w1 is None:
        raise ValueError(f"{where}: w1 and w2 are required unless DSP_BLOCK_ATTN_ONLY")
    F = w1.shape[0] if w1 is not None else 0
    shapes = {"wqkv_s": (3 * C, C), "bqkv_s": (3 * C,), "wo_s": (C, C), "bo_s": (C,),
              "wqkv_t": (3 * C, C), "bqkv_t": (3 * C,), "wo_t": (C, C), "bo_t": (C,),
              "w1": (F, C), "b1": (F,), "w2": (C, F), "b2": (C,)}
    required = {"wqkv_s", "wo_s", "wqkv_t", "wo_t"} | ({"w1", "w2"} if mlp else set())
    for n in BLOCK_WEIGHT_FIELDS:
        t = weights.get(n)
        if t is None:
            if n in required:
                raise ValueError(f"{where}: {n} is required")
            continue
        _check(where, n, t, dtype=wdt, shape=shapes[n], like=x)
    code = DSP_BF16 if wdt == torch.bfloat16 else DSP_F32
    got = [weights.get(n) for n in BLOCK_WEIGHT_FIELDS]
    wt = BlockWeights(*[None if t is None else t.data_ptr() for t in got])
    return B, T, S, C, F, code, wt


def dsp_st_block_forward(x, weights: dict, H: int, eps: float = 1e-6, flags: int = 0,
                         out=None, workspace=None, dtype=None, stream=None):
    """One spatial-temporal block on x (B, T, S, C) fp32; returns (B, S, T, C) fp32.
    ``weights`` maps the dsp_block_weights_t field names to device tensors (or None)."""
    torch = _torch()
    where = "dsp_st_block_forward"
    B, T, S, C, F, code, wt = _block_args(where, x, weights, H, flags, dtype)
    with _on(stream) as s:
        if out is None:
            out = torch.empty((B, S, T, C), dtype=torch.float32, device=x.device)
        _check(where, "out", out, dtype=torch.float32, shape=(B, S, T, C), like=x)
        need = block_workspace_bytes(B, T, S, C, H, F, code)
        if workspace is None:
            workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=x.device)
        _check(where, "workspace", workspace, like=x)
        _check_status(lib().dsp_st_block_forward(_ptr(x), _ptr(out), ctypes.byref(wt), _ptr(workspace),
                                                 _nbytes(workspace), B, T, S, C, H, F, float(eps), flags, code, s),
                      where)
    return out


def dsp_st_block_forward_train(x, weights: dict, H: int, eps: float = 1e-6, flags: int = 0, out=None,
                               saved=None, dtype=None, stream=None):
    """dsp_st_block_forward that also keeps the activations the backward needs:
    returns (y (B, S, T, C) fp32, saved: a uint8 device tensor)."""
    torch = _torch()
    where = "dsp_st_block_forward_train"
    B, T, S, C, F, code, wt = _block_args(where, x, weights, H, flags, dtype)
    with _on(stream) as s:
        if out is None:
            out = torch.empty((B, S, T, C), dtype=torch.float32, device=x.device)
        _check(where, "out", out, dtype=torch.float32, shape=(B, S, T, C), like=x)
        need = int(lib().dsp_st_block_train_saved_bytes(B, T, S, C, H, F, flags, code))
        if saved is None:
            saved = torch.empty(max(need, 1), dtype=torch.uint8, device=x.device)
        _check(where, "saved", saved, like=x)
        _check_status(lib().dsp_st_block_forward_train(_ptr(x), _ptr(out), ctypes.byref(wt), _ptr(saved),
                                                       _nbytes(saved), B, T, S, C, H, F, float(eps), flags, code, s),
                      where)
    return out, saved


def dsp_st_block_backward(x, dy, weights: dict, saved, H: int, eps: float = 1e-6, flags: int = 0, dx=None,
                          grads=None, with_bias: bool = False, workspace=None, dtype=None, stream=None):
    """Backward of the block: returns (dx (B, T, S, C) fp32, grads: dict of fp32
    tensors shaped like the weights, plus the biases when with_bias)."""
    torch = _torch()
    where = "dsp_st_block_backward"
    B, T, S, C, F, code, wt = _block_args(where, x, weights, H, flags, dtype)
    _check(where, "dy", dy, dtype=torch.float32, shape=(B, S, T, C), like=x)
    _check(where, "saved", saved, like=x)
    shapes = {"wqkv_s": (3 * C, C), "wo_s": (C, C), "wqkv_t": (3 * C, C), "wo_t": (C, C), "w1": (F, C),
              "w2": (C, F), "bqkv_s": (3 * C,), "bo_s": (C,), "bqkv_t": (3 * C,), "bo_t": (C,), "b1": (F,),
              "b2": (C,)}
    with _on(stream) as s:
        if dx is None:
            dx = torch.empty((B, T, S, C), dtype=torch.float32, device=x.device)
        _check(where, "dx", dx, dtype=torch.float32, shape=(B, T, S, C), like=x)
        if grads is None:
            names = [n for n in BLOCK_WEIGHT_FIELDS if n.startswith("w") or with_bias]
            grads = {n: torch.empty(shapes[n], dtype=torch.float32, device=x.device) for n in names}
        for n, g in grads.items():
            if n not in shapes:
                raise ValueError(f"{where}: unknown gradient {n}")
            if g is not None:
                _check(where, f"grads[{n}]", g, dtype=torch.float32, shape=shapes[n], like=x)
        need = int(lib().dsp_st_block_backward_workspace_bytes(B, T, S, C, H, F, code))
        if workspace is None:
            workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=x.device)
        _check(where, "workspace", workspace, like=x)
        gt = BlockGrads(**{n: (grads[n].data_ptr() if grads.get(n) is not None else None)
                           for n in BLOCK_WEIGHT_FIELDS})
        _check_status(lib().dsp_st_block_backward(_ptr(x), _ptr(dy), ctypes.byref(wt), _ptr(saved), _nbytes(saved),
                                                  _ptr(workspace), _nbytes(workspace), _ptr(dx), ctypes.byref(gt),
                                                  B, T, S, C, H, F, float(eps), flags, code, s), where)
    return dx, grads


def probe_mfma_workspace_bytes() -> int:
    return int(lib().dsp_probe_mfma_workspace_bytes())


def probe_mfma_flops(iters: int) -> float:
    """Flops one dsp_probe_mfma launch of `iters` iterations issues."""
    return float(lib().dsp_probe_mfma_flops(iters))


def dsp_probe_mfma(iters: int, workspace, stream=None):
    """Launch the sustained-MFMA-rate probe (a measurement aid): time it with
    events on `stream` and divide probe_mfma_flops(iters) by the time."""
    _check("dsp_probe_mfma", "workspace", workspace)
    with _on(stream) as s:
        _check_status(lib().dsp_probe_mfma(_ptr(workspace), _nbytes(workspace), iters, s), "dsp_probe_mfma")


__all__ = ["lib", "status_str", "DspError", "BlockWeights", "dsp_switch", "dsp_spatial_attn",
           "dsp_temporal_attn", "dsp_layernorm", "dsp_linear", "dsp_st_block_forward",
           "dsp_st_block_forward_train", "dsp_st_block_backward", "block_workspace_bytes", "LIB_PATH"]
