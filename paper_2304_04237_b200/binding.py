"""ctypes binding of libslide_attn.so: the same entry points as include/slide_attn.h.

Argument marshalling only -- every step of the forward runs in the library's CUDA kernels.
PyTorch appears here for device memory and streams alone.  There is no fallback: if the
library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libslide_attn.so")

F32, BF16 = 0, 1
VARIANT_AUTO, VARIANT_DIRECT, VARIANT_MMA, VARIANT_UMMA_TS, VARIANT_STRIP, VARIANT_TILE, VARIANT_MMA_WIDE = 0, 1, 2, 5, 6, 8, 9
VARIANT_UMMA_SPLIT = 11
OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_ALIGNMENT, ERR_ALLOC, ERR_CUDA, ERR_ARCH, ERR_TIMEOUT = range(8)
ERR_TOO_LARGE = 8
ERR_NOT_FIXED_SHIFT = 9
ACT_NONE, ACT_SILU, ACT_GELU = range(3)
DROP_ELEMENTS, DROP_IMAGES = range(2)

EXPORTS = ("slide_attn_create", "slide_attn_forward", "slide_attn_forward_host", "slide_attn_backward",
           "slide_attn_forward_noalloc", "slide_attn_project", "slide_attn_block_forward",
           "slide_attn_set_variant", "slide_attn_get_variant", "slide_attn_launches_per_forward",
           "slide_attn_set_fixed_shift", "slide_attn_detect_fixed_shift",
           "slide_attn_profile_begin", "slide_attn_profile_end",
           "slide_attn_group_norm_forward", "slide_attn_group_norm_backward", "slide_attn_group_norm_workspace",
           "slide_attn_dropout_forward", "slide_attn_dropout_backward",
           "slide_attn_select_blocks", "slide_attn_select_workspace",
           "slide_attn_sparse_forward", "slide_attn_sparse_backward", "slide_attn_sparse_workspace",
           "slide_attn_query_status", "slide_attn_destroy", "slide_attn_status_string")

_lib = None

# the current stream's handle and device without the objects around them, where this torch gives them out
_raw_stream, _raw_device = (getattr(torch._C, n, None) for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))


class SlideAttnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {slide_attn_status_string(status)} (status {status})")


def load() -> ctypes.CDLL:
    """Loads the shared library; raises if it is missing (build it with
    `python -m paper_2304_04237_b200.build`)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} not found: build the CUDA library first "
                               "(python -m paper_2304_04237_b200.build); there is no fallback path")
        lib = ctypes.CDLL(LIB_PATH)
        vp, i = ctypes.c_void_p, ctypes.c_int
        lib.slide_attn_create.argtypes = [ctypes.POINTER(vp), i, i, i, i, i, i, i, i]
        lib.slide_attn_forward.argtypes = [vp] * 9
        lib.slide_attn_forward_host.argtypes = [vp] * 9
        lib.slide_attn_backward.argtypes = [vp] * 15
        lib.slide_attn_forward_noalloc.argtypes = [vp] * 7 + [i] * 7 + [vp]
        lib.slide_attn_project.argtypes = [vp, vp, vp, i, vp, vp, vp, vp]
        lib.slide_attn_block_forward.argtypes = [vp] * 9
        lib.slide_attn_set_variant.argtypes = [vp, i]
        lib.slide_attn_get_variant.argtypes = [vp, ctypes.POINTER(i)]
        lib.slide_attn_set_fixed_shift.argtypes = [vp, i]
        lib.slide_attn_detect_fixed_shift.argtypes = [vp, vp, vp, ctypes.POINTER(i), vp]
        lib.slide_attn_launches_per_forward.argtypes = [vp, ctypes.POINTER(i)]
        lib.slide_attn_profile_begin.argtypes = [vp]
        lib.slide_attn_profile_end.argtypes = [vp, ctypes.POINTER(ctypes.c_double),
                                               ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i)]
        ll, f, sz = ctypes.c_longlong, ctypes.c_float, ctypes.c_size_t
        lib.slide_attn_group_norm_forward.argtypes = [vp] * 6 + [i] * 5 + [f, i, i, vp, sz, vp]
        lib.slide_attn_group_norm_backward.argtypes = [vp] * 9 + [i] * 7 + [vp, sz, vp]
        lib.slide_attn_group_norm_workspace.argtypes = [i] * 7 + [ctypes.POINTER(sz)]
        lib.slide_attn_dropout_forward.argtypes = [vp] * 3 + [ll, ll, f, i, vp, i, vp]
        lib.slide_attn_dropout_backward.argtypes = [vp] * 2 + [ll, ll, f, i, vp, i, vp]
        lib.slide_attn_select_blocks.argtypes = [vp] * 3 + [i] * 9 + [vp, sz, vp]
        lib.slide_attn_select_workspace.argtypes = [i] * 7 + [ctypes.POINTER(sz)]
        lib.slide_attn_sparse_forward.argtypes = [vp] * 6 + [i] * 9 + [vp]
        lib.slide_attn_sparse_backward.argtypes = [vp] * 10 + [i] * 9 + [vp, sz, vp]
        lib.slide_attn_sparse_workspace.argtypes = [i] * 8 + [ctypes.POINTER(sz)]
        lib.slide_attn_query_status.argtypes = [vp, vp]
        lib.slide_attn_destroy.argtypes = [vp]
        lib.slide_attn_status_string.argtypes = [i]
        lib.slide_attn_status_string.restype = ctypes.c_char_p
        for name in EXPORTS[:-1]:
            getattr(lib, name).restype = i
        _lib = lib
    return _lib


def slide_attn_status_string(status: int) -> str:
    return load().slide_attn_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != OK:
        raise SlideAttnError(status, where)


def slide_attn_create(B, H, W, heads, head_dim, ksize, dtype, has_bias) -> int:
    """Returns the context handle (an integer address).  dtype: F32 / BF16 or a torch dtype."""
    if isinstance(dtype, torch.dtype):
        dtype = {torch.float32: F32, torch.bfloat16: BF16}[dtype]
    h = ctypes.c_void_p()
    _check(load().slide_attn_create(ctypes.byref(h), B, H, W, heads, head_dim, ksize, int(dtype),
                                    int(bool(has_bias))), "slide_attn_create")
    return h.value


def _dev_ptr(t):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("slide_attn_forward takes contiguous CUDA tensors")
    return t.data_ptr()


def _host_ptr(t):
    if t is None:
        return None
    if t.is_cuda or not t.is_contiguous():
        raise ValueError("slide_attn_forward_host takes contiguous CPU tensors")
    return t.data_ptr()


def _stream_ptr(stream):
    if stream is None:
        # torch.cuda.current_stream() builds a stream object, 3 of the 13 us that a small call takes; the raw handle costs 0.3
        if _raw_stream and _raw_device and torch.cuda.is_initialized():
            return _raw_stream(_raw_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def slide_attn_forward(ctx, q, k, v, wk, wv, bias, out, stream=None) -> None:
    """Device tensors in, result written to `out`; asynchronous on `stream`
    (default: torch's current stream)."""
    _check(load().slide_attn_forward(ctx, *map(_dev_ptr, (q, k, v, wk, wv, bias, out)),
                                     _stream_ptr(stream)), "slide_attn_forward")


def slide_attn_backward(ctx, q, k, v, wk, wv, bias, dout, dq, dk, dv, dwk, dwv, dbias, stream=None) -> None:
    """Gradients of the forward's inputs for dout = d(loss)/d(out); device tensors, asynchronous on
    `stream`.  dq, dk, dv: shape and dtype of q; dwk, dwv: float32 like wk; dbias: float32 like bias or None."""
    _check(load().slide_attn_backward(ctx, *map(_dev_ptr, (q, k, v, wk, wv, bias, dout, dq, dk, dv, dwk, dwv, dbias)),
                                      _stream_ptr(stream)), "slide_attn_backward")


def slide_attn_project(ctx, x, w, ys, stream=None) -> None:
    """Eq. 1 / Eq. 3: ys[i] = x w[i] over the tokens of the context's shape.  x and every ys[i]: bf16 device
    tensors [B, H, W, C]; w: float32 device tensor [len(ys), C, C] (input channel, output channel)."""
    ys = list(ys)
    ptrs = [_dev_ptr(y) for y in ys] + [None] * (3 - len(ys))
    _check(load().slide_attn_project(ctx, _dev_ptr(x), _dev_ptr(w), len(ys), *ptrs, _stream_ptr(stream)),
           "slide_attn_project")


def slide_attn_block_forward(ctx, x, w_qkv, w_o, wk, wv, bias, out, stream=None) -> None:
    """A whole block: projections (Eq. 1, w_qkv float32 [3, C, C]), the local attention, output projection
    (Eq. 3, w_o float32 [C, C]); x and out bf16 device tensors [B, H, W, C]."""
    _check(load().slide_attn_block_forward(ctx, *map(_dev_ptr, (x, w_qkv, w_o, wk, wv, bias, out)),
                                           _stream_ptr(stream)), "slide_attn_block_forward")


def slide_attn_forward_host(ctx, q, k, v, wk, wv, bias, out, stream=None) -> None:
    """CPU tensors in and out (pinned for best speed); returns when `out` is filled."""
    _check(load().slide_attn_forward_host(ctx, *map(_host_ptr, (q, k, v, wk, wv, bias, out)),
                                          _stream_ptr(stream)), "slide_attn_forward_host")


def slide_attn_forward_noalloc(q, k, v, wk, wv, bias, out, ksize, stream=None) -> None:
    """Forward for callers that must not allocate device memory: no context, the library's
    fixed scratch is used instead (bf16, head_dim 32, ksize 3, at most 16 heads).  The shape is
    taken from `q` ([B, H, W, heads, head_dim]).  Calls that overlap on the GPU race on the
    shared scratch; keep them on one stream."""
    B, H, W, heads, head_dim = q.shape
    dtype = {torch.float32: F32, torch.bfloat16: BF16}[q.dtype]
    _check(load().slide_attn_forward_noalloc(*map(_dev_ptr, (q, k, v, wk, wv, bias, out)),
                                             B, H, W, heads, head_dim, int(ksize), dtype,
                                             _stream_ptr(stream)), "slide_attn_forward_noalloc")


def slide_attn_set_variant(ctx, variant: int) -> None:
    _check(load().slide_attn_set_variant(ctx, int(variant)), "slide_attn_set_variant")


def slide_attn_set_fixed_shift(ctx, enable: bool) -> None:
    """Declares that later forwards get exactly the one-hot shift kernels as wk and wv (checked on
    the device in every forward); they then run the fixed-shift kernel."""
    _check(load().slide_attn_set_fixed_shift(ctx, int(bool(enable))), "slide_attn_set_fixed_shift")


def slide_attn_detect_fixed_shift(ctx, wk, wv, stream=None) -> bool:
    """True if the device tensors wk and wv are exactly the one-hot shift kernels (synchronises)."""
    r = ctypes.c_int()
    _check(load().slide_attn_detect_fixed_shift(ctx, _dev_ptr(wk), _dev_ptr(wv), ctypes.byref(r), _stream_ptr(stream)),
           "slide_attn_detect_fixed_shift")
    return bool(r.value)


def slide_attn_get_variant(ctx) -> int:
    v = ctypes.c_int()
    _check(load().slide_attn_get_variant(ctx, ctypes.byref(v)), "slide_attn_get_variant")
    return v.value


def slide_attn_launches_per_forward(ctx) -> int:
    n = ctypes.c_int()
    _check(load().slide_attn_launches_per_forward(ctx, ctypes.byref(n)), "slide_attn_launches_per_forward")
    return n.value


def slide_attn_profile_begin(ctx) -> None:
    _check(load().slide_attn_profile_begin(ctx), "slide_attn_profile_begin")


def slide_attn_profile_end(ctx):
    """Returns (mean ms per forward, mean ms of the main kernel, forwards averaged)."""
    f, m, n = ctypes.c_double(), ctypes.c_double(), ctypes.c_int()
    _check(load().slide_attn_profile_end(ctx, ctypes.byref(f), ctypes.byref(m), ctypes.byref(n)),
           "slide_attn_profile_end")
    return f.value, m.value, n.value


def slide_attn_query_status(ctx, stream=None) -> int:
    """Synchronises the stream; returns OK or ERR_TIMEOUT (does not raise on timeout)."""
    st = load().slide_attn_query_status(ctx, _stream_ptr(stream))
    if st not in (OK, ERR_TIMEOUT, ERR_NOT_FIXED_SHIFT):
        raise SlideAttnError(st, "slide_attn_query_status")
    return st


def slide_attn_destroy(ctx) -> None:
    _check(load().slide_attn_destroy(ctx), "slide_attn_destroy")


# ---- operators around and beside the local attention: sizes from the tensors, scratch memory from torch unless it is given ----------

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


def _device_ptrs(where, *tensors):
    """Addresses of contiguous CUDA tensors (None stays None), all on the current device."""
    device = _raw_device() if _raw_device and torch.cuda.is_initialized() else None
    ptrs = []
    for t in tensors:
        if t is None:
            ptrs.append(None)
        elif t.get_device() == device and t.is_contiguous():
            ptrs.append(t.data_ptr())
        elif not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{where} takes contiguous CUDA tensors")
        elif t.get_device() != torch.cuda.current_device():
            raise ValueError(f"{where}: a tensor is on device {t.get_device()}, the current device is {torch.cuda.current_device()}")
        else:
            ptrs.append(t.data_ptr())
    return ptrs


def _dtype_of(where, x):
    dtype = _DTYPES.get(x.dtype)
    if dtype is None:
        raise ValueError(f"{where} takes float32 or bfloat16 maps, not {x.dtype}")
    return dtype


def _expect(where, name, t, shape, dtype):
    if t is not None and (t.dtype != dtype or t.shape != shape):
        raise ValueError(f"{where}: {name} has to be {dtype} {tuple(shape)}, not {t.dtype} {tuple(t.shape)}")


@functools.lru_cache(maxsize=256)
def _workspace_bytes(where, size, *args):
    need = ctypes.c_size_t()
    _check(getattr(load(), size)(*args, ctypes.byref(need)), where)
    return need.value


def _workspace(where, given, stream, size, *args):
    """(tensor, address, bytes) of the scratch memory that the library's function `size` asks for.  Without one of the caller's it is torch's, taken from the pool
    of the stream that the call runs on, so that it can be handed back as soon as the call is made."""
    need = _workspace_bytes(where, size, *args)
    if given is None and need == 0:
        return None, None, 0
    if given is None:
        if stream is None:
            given = torch.empty(need, dtype=torch.uint8, device="cuda")
        else:
            handle = _stream_ptr(stream)
            with torch.cuda.stream(torch.cuda.ExternalStream(handle) if handle else torch.cuda.default_stream()):
                given = torch.empty(need, dtype=torch.uint8, device="cuda")
    return given, _device_ptrs(where, given)[0], given.numel() * given.element_size()


def slide_attn_group_norm_forward(x, gamma, beta, groups, eps, act, y, mean, rstd, stream=None, workspace=None) -> None:
    """y = act(group norm of x * gamma + beta) over [B, H, W, C] maps; act: ACT_NONE, ACT_SILU or ACT_GELU; gamma, beta: float32 [C] or None;
    mean, rstd: float32 [B, groups], written for the backward.  Asynchronous on `stream`."""
    where = "slide_attn_group_norm_forward"
    dtype = _dtype_of(where, x)
    B, H, W, C = x.shape
    _expect(where, "y", y, x.shape, x.dtype)
    for name, t in (("gamma", gamma), ("beta", beta)):
        _expect(where, name, t, (C,), torch.float32)
    for name, t in (("mean", mean), ("rstd", rstd)):
        _expect(where, name, t, (B, groups), torch.float32)
    lib = load()
    ptrs = _device_ptrs(where, x, gamma, beta, y, mean, rstd)
    workspace, at, size = _workspace(where, workspace, stream, "slide_attn_group_norm_workspace", B, H, W, C, groups, dtype, 0)
    _check(lib.slide_attn_group_norm_forward(*ptrs, B, H, W, C, groups, eps, act, dtype, at, size, _stream_ptr(stream)), where)


def slide_attn_group_norm_backward(x, gamma, beta, groups, act, mean, rstd, dy, dx, dgamma, dbeta, stream=None, workspace=None) -> None:
    """Gradients of the forward's x, gamma and beta for dy = d(loss)/d(y); dgamma and dbeta: float32 [C], or both None."""
    where = "slide_attn_group_norm_backward"
    dtype = _dtype_of(where, x)
    B, H, W, C = x.shape
    for name, t in (("dy", dy), ("dx", dx)):
        _expect(where, name, t, x.shape, x.dtype)
    for name, t in (("gamma", gamma), ("beta", beta), ("dgamma", dgamma), ("dbeta", dbeta)):
        _expect(where, name, t, (C,), torch.float32)
    for name, t in (("mean", mean), ("rstd", rstd)):
        _expect(where, name, t, (B, groups), torch.float32)
    lib = load()
    ptrs = _device_ptrs(where, x, gamma, beta, mean, rstd, dy, dx, dgamma, dbeta)
    workspace, at, size = _workspace(where, workspace, stream, "slide_attn_group_norm_workspace", B, H, W, C, groups, dtype, 1)
    _check(lib.slide_attn_group_norm_backward(*ptrs, B, H, W, C, groups, act, dtype, at, size, _stream_ptr(stream)), where)


def _dropout_sizes(where, x, rng, **others):
    for name, t in others.items():
        _expect(where, name, t, x.shape, x.dtype)
    if rng.dtype not in (torch.int64, torch.uint64) or rng.numel() != 2:
        raise ValueError(f"{where}: rng has to be two 64-bit integers (seed, offset)")
    if x.numel() == 0:
        raise ValueError(f"{where}: x is empty")
    return x.shape[0] if x.dim() else 1, x.numel() // (x.shape[0] if x.dim() else 1)


def slide_attn_dropout_forward(x, residual, p, unit, rng, y, stream=None) -> None:
    """y = residual + (kept ? x / (1 - p) : 0); residual may be None, y may be x or residual.  unit: DROP_ELEMENTS, or DROP_IMAGES for all of
    an image (x's first dimension) or nothing of it.  rng: device tensor of two 64-bit integers, seed and offset, read when the call runs."""
    where = "slide_attn_dropout_forward"
    dtype = _dtype_of(where, x)
    images, per_image = _dropout_sizes(where, x, rng, residual=residual, y=y)
    px, pr, py, prng = _device_ptrs(where, x, residual, y, rng)
    _check(load().slide_attn_dropout_forward(px, pr, py, images, per_image, p, unit, prng, dtype, _stream_ptr(stream)), where)


def slide_attn_dropout_backward(dy, p, unit, rng, dx, stream=None) -> None:
    """dx = kept ? dy / (1 - p) : 0 with the mask of a forward of the same p, unit and rng; dx may be dy."""
    where = "slide_attn_dropout_backward"
    dtype = _dtype_of(where, dy)
    images, per_image = _dropout_sizes(where, dy, rng, dx=dx)
    pdy, pdx, prng = _device_ptrs(where, dy, dx, rng)
    _check(load().slide_attn_dropout_backward(pdy, pdx, images, per_image, p, unit, prng, dtype, _stream_ptr(stream)), where)


def _lists(where, q, idx, block):
    """Blocks and entries of the lists of a call on [B, H, W, heads, head_dim] maps."""
    B, H, W, heads, _ = q.shape
    bh, bw = block
    if bh < 1 or bw < 1:
        raise ValueError(f"{where}: a block has at least one pixel")
    _expect(where, "idx", idx, (B, heads, -(-H // bh) * -(-W // bw), idx.shape[-1]), torch.int32)
    return bh, bw, idx.shape[-1]


def slide_attn_select_blocks(q, k, block, idx, stream=None, workspace=None) -> None:
    """Writes, for every block of queries and every head, the numbers of the idx.shape[-1] blocks of keys with the largest scores (pooled
    query times pooled key).  block: (height, width) in pixels; idx: int32 [B, heads, blocks, top]."""
    where = "slide_attn_select_blocks"
    dtype = _dtype_of(where, q)
    B, H, W, heads, d = q.shape
    _expect(where, "k", k, q.shape, q.dtype)
    bh, bw, top = _lists(where, q, idx, block)
    lib = load()
    ptrs = _device_ptrs(where, q, k, idx)
    workspace, at, size = _workspace(where, workspace, stream, "slide_attn_select_workspace", B, H, W, heads, d, bh, bw)
    _check(lib.slide_attn_select_blocks(*ptrs, B, H, W, heads, d, bh, bw, top, dtype, at, size, _stream_ptr(stream)), where)


def slide_attn_sparse_forward(q, k, v, idx, block, out, lse, stream=None) -> None:
    """Attention of every query to the pixels of the blocks that idx (int32 [B, heads, blocks, top]) lists for its own block; lse: float32
    [B, H, W, heads], written for the backward."""
    where = "slide_attn_sparse_forward"
    dtype = _dtype_of(where, q)
    B, H, W, heads, d = q.shape
    for name, t in (("k", k), ("v", v), ("out", out)):
        _expect(where, name, t, q.shape, q.dtype)
    _expect(where, "lse", lse, (B, H, W, heads), torch.float32)
    bh, bw, top = _lists(where, q, idx, block)
    _check(load().slide_attn_sparse_forward(*_device_ptrs(where, q, k, v, idx, out, lse), B, H, W, heads, d, bh, bw, top, dtype,
                                            _stream_ptr(stream)), where)


def slide_attn_sparse_backward(q, k, v, idx, block, out, lse, dout, dq, dk, dv, stream=None, workspace=None) -> None:
    """Gradients of the forward's q, k and v for dout = d(loss)/d(out); the lists are constants."""
    where = "slide_attn_sparse_backward"
    dtype = _dtype_of(where, q)
    B, H, W, heads, d = q.shape
    for name, t in (("k", k), ("v", v), ("out", out), ("dout", dout), ("dq", dq), ("dk", dk), ("dv", dv)):
        _expect(where, name, t, q.shape, q.dtype)
    _expect(where, "lse", lse, (B, H, W, heads), torch.float32)
    bh, bw, top = _lists(where, q, idx, block)
    lib = load()
    ptrs = _device_ptrs(where, q, k, v, idx, out, lse, dout, dq, dk, dv)
    workspace, at, size = _workspace(where, workspace, stream, "slide_attn_sparse_workspace", B, H, W, heads, d, bh, bw, top)
    _check(lib.slide_attn_sparse_backward(*ptrs, B, H, W, heads, d, bh, bw, top, dtype, at, size, _stream_ptr(stream)), where)
