"""Thin ctypes binding of libpsa.so: argument marshalling only.

Every step of the path runs inside the CUDA library; torch is used for device memory
and streams.  Importing this module without a built library, or calling it without a
CUDA device, raises -- there is no CPU fallback.  Attention is forward only: its outputs carry no
gradient.  Norm and rotation (psa_qk_norm_rope) have one.

With ``stream=`` a call runs there instead of on the current stream: its inputs have to be ready there, and what it
returns is memory of that stream, which the current one may use once it waits for it, and drop while it still does.
"""
from __future__ import annotations

import ctypes
import os
import struct
from contextlib import nullcontext
from itertools import chain
from typing import List, Optional, Sequence, Tuple

import torch
from torch.autograd.function import once_differentiable

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpsa.so")

PSA_OK = 0
PSA_ERR_INVALID_ARG = -1
PSA_ERR_UNSUPPORTED = -2
PSA_ERR_CAPACITY = -3
PSA_ERR_CUDA = -4
PSA_ERR_TIMEOUT = -5
PSA_ERR_INTERNAL = -6


class PsaError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} ({status})")


class HeadParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("Tw", "To", "Ts", "Sw", "So", "Ss")]


class Tile(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("bt", "bh", "bw")]


class Problem(ctypes.Structure):
    _fields_ = [("n_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("tile", Tile),
                ("scale", ctypes.c_float), ("stride_head", ctypes.c_int64), ("stride_token", ctypes.c_int64)]


_lib = None


def lib() -> ctypes.CDLL:
    """Loads libpsa.so (built by paper_2609_37001_b200.build); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2609_37001_b200.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64p = ctypes.c_void_p, ctypes.c_int, ctypes.POINTER(ctypes.c_int64)
        hp, pp = ctypes.POINTER(HeadParams), vp   # (a problem travels as packed bytes or by reference)
        L.psa_status_string.restype = ctypes.c_char_p
        L.psa_status_string.argtypes = [i32]
        L.psa_launch_count.restype = ctypes.c_int64
        L.psa_launch_count.argtypes = []
        L.psa_mask_sizes.argtypes = [hp, pp, i32, i32, i32, i64p, i64p]
        L.psa_mask_build.argtypes = [hp, pp, i32, i32, i32, vp, vp, vp, ctypes.c_int64, vp]
        L.psa_attn_fwd.argtypes = [vp, vp, vp, vp, vp, hp, pp, i32, i32, i32, vp]
        L.psa_attn_fwd_host.argtypes = [vp] * 10 + [hp, pp, i32, i32, i32, vp]
        L.psa_attn_fwd_noalloc.argtypes = [vp, vp, vp, vp, vp, hp, pp, i32, i32, i32, vp, ctypes.POINTER(ctypes.c_int32)]
        L.psa_attn_fwd_noalloc.restype = ctypes.c_int
        L.psa_attn_fwd_batched.argtypes = [vp, vp, vp, vp, vp, hp, pp, i32, ctypes.c_int64, i32, i32, i32, vp]
        L.psa_attn_fwd_joint.argtypes = [vp, vp, vp, vp, vp, hp, pp, ctypes.c_int64, i32, i32, i32, vp]
        L.psa_search_scratch_bytes.argtypes = [i32, i32, i32, i32]
        L.psa_search_scratch_bytes.restype = ctypes.c_int64
        L.psa_search_losses.argtypes = [vp, vp, vp, hp, i32, pp, i32, i32, i32, vp, vp, vp]
        L.psa_search_losses.restype = ctypes.c_int
        L.psa_search_select.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_float), i32, ctypes.c_float]
        L.psa_search_select.restype = ctypes.c_int
        L.psa_search_select_at_sparsity.argtypes = L.psa_search_select.argtypes
        L.psa_search_select_at_sparsity.restype = ctypes.c_int
        L.psa_select_scratch_bytes.argtypes = [vp, i32, i32, i32]
        L.psa_select_scratch_bytes.restype = ctypes.c_int64
        L.psa_select_blocks.argtypes = [vp, vp, vp, i32, i32, i32, vp, i32, vp, vp, ctypes.c_int64, vp, vp]
        L.psa_select_blocks.restype = ctypes.c_int
        L.psa_attn_fwd_lists_scratch_bytes.argtypes = [vp, ctypes.c_int64, i32, i32, i32]
        L.psa_attn_fwd_lists_scratch_bytes.restype = ctypes.c_int64
        L.psa_attn_fwd_lists.argtypes = [vp] * 7 + [ctypes.c_int64, vp, ctypes.c_int64, i32, i32, i32, vp, vp]
        L.psa_attn_fwd_lists.restype = ctypes.c_int
        L.psa_qk_norm_rope.argtypes = [vp] * 8 + [i32, i32, i32, vp]
        L.psa_qk_norm_rope.restype = ctypes.c_int
        L.psa_qk_norm_rope_bwd_scratch_bytes.argtypes = [vp]
        L.psa_qk_norm_rope_bwd_scratch_bytes.restype = ctypes.c_int64
        L.psa_qk_norm_rope_bwd.argtypes = [vp] * 12 + [i32, i32, i32, vp, vp]
        L.psa_qk_norm_rope_bwd.restype = ctypes.c_int
        L.psa_last_device_status.argtypes = [ctypes.POINTER(ctypes.c_int32)]
        L.psa_last_attn_launch.argtypes = [ctypes.POINTER(ctypes.c_int32)] * 2
        L.psa_last_attn_launch.restype = ctypes.c_int
        L.psa_last_attn_grid.argtypes = [ctypes.POINTER(ctypes.c_int32)] * 2
        L.psa_last_attn_grid.restype = ctypes.c_int
        L.psa_last_attn_class.argtypes = [i32] + [ctypes.POINTER(ctypes.c_int32)] * 3
        L.psa_last_attn_class.restype = ctypes.c_int
        L.psa_shutdown.argtypes = []
        L.psa_selftest_wait_timeout.argtypes = [i32, vp]
        L.psa_selftest_wait_timeout.restype = ctypes.c_int
        L.psa_profile_events.argtypes = [vp, vp]
        L.psa_profile_events.restype = ctypes.c_int
        for f in (L.psa_mask_sizes, L.psa_mask_build, L.psa_attn_fwd, L.psa_attn_fwd_host,
                  L.psa_last_device_status, L.psa_shutdown):
            f.restype = ctypes.c_int
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().psa_status_string(int(status)).decode()


def _check(status: int, what: str) -> None:
    if status != PSA_OK:
        raise PsaError(status, what)


_PARAMS_CACHE: dict = {}


def _params_array(head_params: Sequence[Sequence[int]]):
    """ctypes array of the per-head parameters, memoised by value: a model calls with the same few sets of masks, and
    looking 40 heads up takes 1 us where converting them takes 15 (40 with one structure per head).  Entries are stored
    under tuples of ints only, so what is given finds one by being equal to it; rows that hash by identity (tensors) are
    equal to none of them and are converted on every call.  (The rows as given where they are such tuples: finding the
    same objects again takes half the time of comparing equal ones.)"""
    given = tuple(head_params)
    try:
        arr = _PARAMS_CACHE.get(given)
    except TypeError:   # rows without a hash: lists, arrays
        arr = None
    if arr is not None:
        return arr
    n, packed = len(given), None
    try:
        if set(map(len, given)) == {6}:
            flat = tuple(chain.from_iterable(given))
            packed = struct.pack("%di" % (6 * n), *flat)
            plain = set(map(type, given)) == {tuple} and set(map(type, flat)) == {int}
            key = given if plain else tuple(struct.iter_unpack("6i", packed))
    except (TypeError, struct.error):   # floats and the like
        packed = None
    if packed is None:
        key = tuple([tuple([int(x) for x in p]) for p in given])
    arr = _PARAMS_CACHE.get(key)
    if arr is None:
        if packed is not None:
            arr = (HeadParams * n).from_buffer_copy(packed)
        else:   # (a row of fewer values leaves the others 0, one of more is an error)
            arr = (HeadParams * n)()
            for i, p in enumerate(key):
                arr[i] = HeadParams(*p)
        if len(_PARAMS_CACHE) >= 64:
            _PARAMS_CACHE.clear()
        _PARAMS_CACHE[key] = arr
    return arr


def make_problem(n_heads: int, tile: Sequence[int], scale: float, stride_head: int, stride_token: int,
                 head_dim: int = 128) -> Problem:
    bt, bh, bw = tile
    return Problem(int(n_heads), int(head_dim), Tile(int(bt), int(bh), int(bw)), float(scale),
                   int(stride_head), int(stride_token))


_pack_problem = struct.Struct("iiiiifqq").pack   # the layout of Problem
assert struct.calcsize("iiiiifqq") == ctypes.sizeof(Problem)


def _problem(n_heads, tile, scale, stride_head, stride_token, head_dim=128) -> bytes:
    """make_problem as packed bytes (0.5 instead of 1.6 us)."""
    bt, bh, bw = tile
    return _pack_problem(n_heads, head_dim, int(bt), int(bh), int(bw), scale, stride_head, stride_token)


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    if stream is not None:
        return stream.cuda_stream
    # the current stream's handle without building a torch.cuda.Stream around it (0.3 instead of 3 us)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


_CURRENT = nullcontext()


def _memory_of(stream: Optional[torch.cuda.Stream]):
    """Context for the allocations of a call on `stream`: memory of that stream.  (Memory of the current stream may have been dropped while
    kernels there still use it, behind which nothing orders the call's.)"""
    return _CURRENT if stream is None else torch.cuda.stream(stream)


def _used_here(stream: Optional[torch.cuda.Stream], *tensors: Optional[torch.Tensor]) -> None:
    """Tensors allocated for a call on `stream` and returned: the current stream may read them until they are dropped, before `stream` gets
    their memory again."""
    if stream is not None:
        here = torch.cuda.current_stream()
        if stream != here:
            for t in tensors:
                if t is not None:
                    t.record_stream(here)


def _new_scratch(need: int, like: torch.Tensor, stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    if stream is None:
        return torch.empty(need, dtype=torch.uint8, device=like.device)
    with _memory_of(stream):
        return torch.empty(need, dtype=torch.uint8, device=like.device)


def _require_cuda(*tensors: torch.Tensor) -> None:
    for t in tensors:
        if not t.is_cuda:
            raise ValueError("device tensors required")


def psa_mask_sizes(head_params, grid: Sequence[int], tile: Sequence[int]) -> Tuple[int, int]:
    """(NB, nnz) for psa_mask_build's outputs.  Host arithmetic only."""
    prob = _problem(len(head_params), tile, 1.0, 0, 128)
    nb, nnz = ctypes.c_int64(0), ctypes.c_int64(0)
    T, H, W = map(int, grid)
    _check(lib().psa_mask_sizes(_params_array(head_params), prob, T, H, W,
                                ctypes.byref(nb), ctypes.byref(nnz)), "psa_mask_sizes")
    return nb.value, nnz.value


def psa_mask_build(head_params, grid: Sequence[int], tile: Sequence[int], device="cuda",
                   out: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor]] = None,
                   stream: Optional[torch.cuda.Stream] = None):
    """Block mask uint8[heads, NB, NB], row_ptr int32[heads*NB+1], col_idx int32[nnz] on the device."""
    nh = len(head_params)
    T, H, W = map(int, grid)
    if out is None:
        nb, nnz = psa_mask_sizes(head_params, grid, tile)
        with _memory_of(stream):
            mask = torch.empty((nh, nb, nb), dtype=torch.uint8, device=device)
            row_ptr = torch.empty(nh * nb + 1, dtype=torch.int32, device=device)
            col_idx = torch.empty(max(nnz, 1), dtype=torch.int32, device=device)
        _used_here(stream, mask, row_ptr, col_idx)
    else:
        mask, row_ptr, col_idx = out
        nnz = None
    _require_cuda(mask, row_ptr, col_idx)
    prob = _problem(nh, tile, 1.0, 0, 128)
    _check(lib().psa_mask_build(_params_array(head_params), prob, T, H, W, mask.data_ptr(),
                                row_ptr.data_ptr(), col_idx.data_ptr(), col_idx.numel(), _stream_ptr(stream)),
           "psa_mask_build")
    if nnz is not None:
        col_idx = col_idx[:nnz]
    return mask, row_ptr, col_idx


def _device_call(q, k, v, out, lse, lse_shape, stream):
    """Checks the tensors of a device call and allocates the outputs that were not given.
    Returns (out, lse, q's strides)."""
    _require_cuda(q, k, v)
    bf16 = torch.bfloat16
    if q.dtype != bf16 or k.dtype != bf16 or v.dtype != bf16:
        raise ValueError("bf16 tensors required")
    st = q.stride()
    if st != k.stride() or st != v.stride() or st[-1] != 1:
        raise ValueError("q, k, v must share strides with a contiguous last dimension")
    if stream is not None and (out is None or lse is None):
        mine = out, lse
        with _memory_of(stream):
            out, lse, _ = _device_call(q, k, v, out, lse, lse_shape, None)
        _used_here(stream, *(new for new, given in zip((out, lse), mine) if given is None))
    if out is None:
        out = q.new_empty_strided(q.shape, st)
    elif out.stride() != st:
        raise ValueError("out must share q's strides; lse must be contiguous")
    if lse is None:
        lse = q.new_empty(lse_shape, dtype=torch.float32)
    elif not lse.is_contiguous():
        raise ValueError("out must share q's strides; lse must be contiguous")
    return out, lse, st


def psa_attn_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, head_params, grid: Sequence[int],
                 tile: Sequence[int], scale: float, out: Optional[torch.Tensor] = None,
                 lse: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """q, k, v: bf16 device tensors [heads, L, 128] (any head/token strides, last dim contiguous,
    shared by all three).  Returns (out bf16 like q, lse fp32 [heads, L])."""
    nh, L, d = q.shape
    T, H, W = map(int, grid)
    if L != T * H * W or k.shape != q.shape or v.shape != q.shape:
        raise ValueError("shape mismatch")
    out, lse, st = _device_call(q, k, v, out, lse, (nh, L), stream)
    prob = _problem(nh, tile, scale, st[0], st[1], d)
    _check(lib().psa_attn_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                              _params_array(head_params), prob, T, H, W, _stream_ptr(stream)),
           "psa_attn_fwd")
    return out, lse


def psa_attn_fwd_batched(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, head_params, grid: Sequence[int],
                         tile: Sequence[int], scale: float, out: Optional[torch.Tensor] = None,
                         lse: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Batched call: q, k, v are bf16 device tensors [batch, heads, L, 128] sharing strides (last dim
    contiguous); every sample uses the same per-head masks.  Returns (out like q, lse fp32
    [batch, heads, L])."""
    nb, nh, L, d = q.shape
    T, H, W = map(int, grid)
    if L != T * H * W or k.shape != q.shape or v.shape != q.shape or len(head_params) != nh:
        raise ValueError("shape mismatch")
    out, lse, st = _device_call(q, k, v, out, lse, (nb, nh, L), stream)
    prob = _problem(nh, tile, scale, st[1], st[2], d)
    _check(lib().psa_attn_fwd_batched(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                      _params_array(head_params), prob, nb, st[0], T, H, W,
                                      _stream_ptr(stream)), "psa_attn_fwd_batched")
    return out, lse


def psa_attn_fwd_joint(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, head_params, grid: Sequence[int],
                       tile: Sequence[int], scale: float, n_text: int, out: Optional[torch.Tensor] = None,
                       lse: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Joint video + text sequence: q, k, v are bf16 device tensors [heads, L + n_text, 128] with the
    video tokens first.  The stripe mask applies between video tokens; text keys are attended by every
    query and text queries attend every key.  Returns (out like q, lse fp32 [heads, L + n_text])."""
    nh, Lt, d = q.shape
    T, H, W = map(int, grid)
    if Lt != T * H * W + int(n_text) or k.shape != q.shape or v.shape != q.shape:
        raise ValueError("shape mismatch")
    out, lse, st = _device_call(q, k, v, out, lse, (nh, Lt), stream)
    prob = _problem(nh, tile, scale, st[0], st[1], d)
    _check(lib().psa_attn_fwd_joint(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                    _params_array(head_params), prob, int(n_text), T, H, W,
                                    _stream_ptr(stream)), "psa_attn_fwd_joint")
    return out, lse


def psa_attn_fwd_noalloc(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor,
                         head_params, grid: Sequence[int], tile: Sequence[int], scale: float,
                         stream: Optional[torch.cuda.Stream] = None, check: bool = True) -> int:
    """psa_attn_fwd through the entry point that never allocates device memory: for callers whose device
    memory is owned by someone else's pool, or who cannot afford the device-wide synchronisation of
    cudaMalloc.  The caller supplies ``out`` and ``lse`` (nothing is allocated here either); the library's
    scratch is a fixed array inside the library image, so the problem must fit its limits (see psa.h).
    With ``check`` the call synchronises the stream and raises on a device-side timeout; it returns the
    diagnostic word."""
    _require_cuda(q, k, v, out, lse)
    nh, L, d = q.shape
    T, H, W = map(int, grid)
    if L != T * H * W or k.shape != q.shape or v.shape != q.shape or out.shape != q.shape:
        raise ValueError("shape mismatch")
    if q.stride() != k.stride() or q.stride() != v.stride() or q.stride() != out.stride() or q.stride(2) != 1:
        raise ValueError("q, k, v, out must share strides with a contiguous last dimension")
    if not lse.is_contiguous() or tuple(lse.shape) != (nh, L):
        raise ValueError("lse must be a contiguous [heads, L] tensor")
    prob = _problem(nh, tile, scale, q.stride(0), q.stride(1), d)
    detail = ctypes.c_int32(0)
    _check(lib().psa_attn_fwd_noalloc(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                      _params_array(head_params), prob, T, H, W, _stream_ptr(stream),
                                      ctypes.byref(detail) if check else None), "psa_attn_fwd_noalloc")
    return detail.value


def psa_attn_fwd_host(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor,
                      staging: Sequence[torch.Tensor], head_params, grid: Sequence[int], tile: Sequence[int],
                      scale: float, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Host-tensor variant: q, k, v, out (bf16 [heads, L, 128], contiguous) and lse (fp32 [heads, L])
    live in host memory; ``staging`` = (d_q, d_k, d_v, d_out, d_lse) are device buffers of the same
    shapes.  Copies in, runs, copies out and synchronises the stream."""
    d_q, d_k, d_v, d_out, d_lse = staging
    _require_cuda(d_q, d_k, d_v, d_out, d_lse)
    for t in (q, k, v, out, lse):
        if t.is_cuda or not t.is_contiguous():
            raise ValueError("contiguous host tensors required")
    nh, L, d = q.shape
    T, H, W = map(int, grid)
    prob = _problem(nh, tile, scale, q.stride(0), q.stride(1), d)
    _check(lib().psa_attn_fwd_host(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                   d_q.data_ptr(), d_k.data_ptr(), d_v.data_ptr(), d_out.data_ptr(),
                                   d_lse.data_ptr(), _params_array(head_params), prob, T, H, W,
                                   _stream_ptr(stream)), "psa_attn_fwd_host")


def psa_search_scratch_bytes(n_cand: int, grid: Sequence[int]) -> int:
    """Bytes of device scratch psa_search_losses needs for ``n_cand`` candidates on this token grid."""
    T, H, W = map(int, grid)
    n = int(lib().psa_search_scratch_bytes(int(n_cand), T, H, W))
    if n < 0:
        _check(n, "psa_search_scratch_bytes")
    return n


def psa_search_losses(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, candidates, grid: Sequence[int],
                      tile: Sequence[int], scale: float, scratch: Optional[torch.Tensor] = None,
                      stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Inner loop of PSA-Search for one head (Algorithm 3): q, k, v are bf16 [L, 128] device tensors of
    that head, ``candidates`` a sequence of six-integer masks.  Returns the fp32 loss of every candidate
    against full attention (device tensor).  ``scratch`` (uint8, psa_search_scratch_bytes long) is
    allocated when not given."""
    _require_cuda(q, k, v)
    L, d = q.shape
    T, H, W = map(int, grid)
    if L != T * H * W or k.shape != q.shape or v.shape != q.shape:
        raise ValueError("shape mismatch")
    if q.stride() != k.stride() or q.stride() != v.stride() or q.stride(1) != 1:
        raise ValueError("q, k, v must share strides with a contiguous last dimension")
    n_cand = len(candidates)
    need = psa_search_scratch_bytes(n_cand, grid)
    if scratch is not None and (scratch.numel() * scratch.element_size() < need or not scratch.is_contiguous()):
        raise ValueError("scratch too small")
    with _memory_of(stream):
        if scratch is None:
            scratch = torch.empty(need, dtype=torch.uint8, device=q.device)
        losses = torch.empty(n_cand, dtype=torch.float32, device=q.device)
    _used_here(stream, losses)
    prob = _problem(1, tile, scale, 0, q.stride(0), d)
    _check(lib().psa_search_losses(q.data_ptr(), k.data_ptr(), v.data_ptr(), _params_array(candidates), n_cand,
                                   prob, T, H, W, scratch.data_ptr(), losses.data_ptr(),
                                   _stream_ptr(stream)), "psa_search_losses")
    return losses


def psa_search_select(losses: Sequence[float], sparsity: Sequence[float], alpha: float) -> int:
    """Selection step of PSA-Search (Algorithm 3) on host arrays; returns the chosen candidate's index."""
    n = len(losses)
    if len(sparsity) != n:
        raise ValueError("losses and sparsity differ in length")
    la = (ctypes.c_float * n)(*[float(x) for x in losses])
    sa = (ctypes.c_float * n)(*[float(x) for x in sparsity])
    r = int(lib().psa_search_select(la, sa, n, float(alpha)))
    if r < 0:
        _check(r, "psa_search_select")
    return r


def psa_search_select_at_sparsity(losses: Sequence[float], sparsity: Sequence[float], target: float) -> int:
    """Second interface of PSA-Search: minimal-loss candidate among those at least ``target`` sparse;
    -1 when none is."""
    n = len(losses)
    if len(sparsity) != n:
        raise ValueError("losses and sparsity differ in length")
    la = (ctypes.c_float * n)(*[float(x) for x in losses])
    sa = (ctypes.c_float * n)(*[float(x) for x in sparsity])
    r = int(lib().psa_search_select_at_sparsity(la, sa, n, float(target)))
    if r == -3:  # PSA_ERR_CAPACITY: no candidate reaches the target
        return -1
    if r < 0:
        _check(r, "psa_search_select_at_sparsity")
    return r


def _on_current_device(*tensors: Optional[torch.Tensor]) -> None:
    """Device tensors of the current device (kernels are launched there)."""
    here = -2
    for t in tensors:
        if t is not None:
            index = t.get_device()   # (-1: host memory)
            if index != here:
                if index < 0:
                    raise ValueError("device tensors required")
                if here < 0:
                    here = torch._C._cuda_getDevice()
                if index != here:
                    raise ValueError("tensors must be on the current device")


_DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_NORMS = {"none": 0, "head": 1, "token": 2}
_PAIRS = {"interleaved": 0, "halves": 1}
_pack_qk = struct.Struct("8ifi12q").pack     # the layout of psa_qk
_pack_rope = struct.Struct("4i7d").pack      # the layout of psa_rope


def _strides4(t: torch.Tensor) -> Tuple[int, int, int]:
    """Strides of batch, head and token of [(batch,) heads, tokens, channels]; the channels must be contiguous."""
    st = t.stride()
    if st[-1] != 1:
        raise ValueError("a contiguous last dimension is required")
    return (0, st[0], st[1]) if len(st) == 3 else st[:3]


def _new_outputs(x: torch.Tensor, dtype: Optional[torch.dtype], two: bool) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """New tensors of x's shape and strides, gaps included, as attention asks of q, k and v together (v may still lie in the projection that
    x is a view of).  Without gaps where elements of x share memory, which those of an output must not."""
    y = torch.empty_like(x, dtype=dtype)
    st = x.stride()
    if y.stride() != st:   # (x has either)
        span = 1
        for s, n in sorted(zip(st, x.shape)):
            if n > 1:
                if s < span:
                    break
                span += s * (n - 1)
        else:
            y = x.new_empty_strided(x.shape, st, dtype=dtype)
            return y, y.new_empty_strided(x.shape, st) if two else None
    return y, torch.empty_like(y) if two else None


def _norm_rope_call(first: torch.Tensor, out: torch.Tensor, grad: Optional[torch.Tensor], dtype: torch.dtype, q_weight, k_weight, two: bool,
                    dims, theta, norm, eps, pairs, origin, step, n_text, first_token) -> Tuple[bytes, bytes, int]:
    """psa_qk and psa_rope of a call as packed bytes, and the heads that the weights are of (0: no weights)."""
    shape = first.shape
    if len(shape) not in (3, 4):
        raise ValueError("[heads, tokens, channels] or [batch, heads, tokens, channels] required")
    batch, heads, tokens, d = shape if len(shape) == 4 else (1, *shape)
    if norm not in _NORMS or pairs not in _PAIRS:
        raise ValueError("norm is one of %s, pairs one of %s" % (", ".join(_NORMS), ", ".join(_PAIRS)))
    if dtype not in _DTYPES or out.dtype not in _DTYPES:
        raise ValueError("bf16, fp16 or fp32 tensors required")
    weight_heads, weight_dtype = 0, torch.float32
    for w in (q_weight, k_weight):
        if w is None:
            continue
        if tuple(w.shape) not in ((d,), (heads, d)) or not w.is_contiguous() or w.dtype not in _DTYPES:
            raise ValueError("weights are contiguous [channels] or [heads, channels] tensors of bf16, fp16 or fp32")
        n = 1 if w.dim() == 1 else heads
        if weight_heads and (n, w.dtype) != (weight_heads, weight_dtype):
            raise ValueError("both weights must be alike")
        weight_heads, weight_dtype = n, w.dtype
    if norm == "none" and weight_heads:
        raise ValueError("there are no weights without a norm")
    if two and norm != "none" and (q_weight is None) != (k_weight is None):
        raise ValueError("weights for both tensors or for none")
    if not two and k_weight is not None:
        raise ValueError("a weight for k without k")
    prob = _pack_qk(batch, heads, d, _DTYPES[dtype], _DTYPES[out.dtype], _NORMS[norm], _DTYPES[weight_dtype], max(weight_heads, 1), eps, 0, tokens,
                    int(first_token), int(n_text), *_strides4(first), *_strides4(out), *(_strides4(grad) if grad is not None else (0, 0, 0)))
    dt, dh, dw = dims
    rope = _pack_rope(int(dt), int(dh), int(dw), _PAIRS[pairs], theta, *origin, *step)
    return prob, rope, weight_heads


_SIZES: dict = {}


def _scratch_bytes(what: str, n_heads: int, grid, tile, n_text: int = 0) -> int:
    """Scratch of psa_select_blocks or psa_attn_fwd_lists, remembered by the call's sizes (asking takes 2 us)."""
    key = (what, n_heads, tuple(grid), tuple(tile), n_text)
    need = _SIZES.get(key)
    if need is None:
        need = psa_select_scratch_bytes(n_heads, grid, tile) if what == "select" else psa_attn_fwd_lists_scratch_bytes(n_heads, grid, tile, n_text)
        if len(_SIZES) >= 256:
            _SIZES.clear()
        _SIZES[key] = need
    return need


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def psa_qk_norm_rope(q: torch.Tensor, k: Optional[torch.Tensor], grid: Sequence[int], dims: Sequence[int] = (44, 42, 42), theta: float = 10000.0,
                     norm: str = "head", q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                     pairs: str = "interleaved", origin: Sequence[float] = (0.0, 0.0, 0.0), step: Sequence[float] = (1.0, 1.0, 1.0),
                     n_text: int = 0, first_token: int = 0, out: Optional[Sequence[Optional[torch.Tensor]]] = None,
                     out_dtype: Optional[torch.dtype] = None, stream: Optional[torch.cuda.Stream] = None):
    """Root-mean-square norm and rotary positions of queries and keys (see psa.h), in one pass.

    q, k: bf16, fp16 or fp32 device tensors [heads, tokens, 128] or [batch, heads, tokens, 128] sharing shape, strides and type (the
    last dimension contiguous; views of a fused projection will do); k may be None.  They hold tokens ``first_token`` .. of the sequence
    of T*H*W video tokens and ``n_text`` text tokens, which are normed and not rotated.
    ``dims``: channels that turn with the frame, the row and the column.  ``norm``: "head", "token" (over all heads) or "none"; weights
    [128] or [heads, 128].  Positions are ``origin + step * index``.  ``out``: (q_out, k_out), which may be (q, k); by default new
    tensors with q's strides, as attention's ``out`` (q, k and v of one projection still share strides then), of ``out_dtype`` (q's
    type, or bf16).  Returns (q_out, k_out).

    Where q, k or a weight requires a gradient, the new tensors have one, by psa_qk_norm_rope_bwd (first derivatives; into ``out`` the
    call takes no part in autograd).  As everywhere in autograd, a backward pass is captured into a CUDA graph only while no graph of the same
    leaves from outside the capture is alive."""
    if out is None and torch.is_grad_enabled() and (
            q.requires_grad or (k is not None and k.requires_grad) or (q_weight is not None and q_weight.requires_grad) or
            (k_weight is not None and k_weight.requires_grad)):
        how = dict(dims=dims, theta=theta, norm=norm, eps=eps, pairs=pairs, origin=origin, step=step, n_text=n_text, first_token=first_token, stream=stream)
        return _NormRope.apply(q, k, q_weight, k_weight, grid, out_dtype, how)
    two = k is not None
    if two and (k.shape != q.shape or k.stride() != q.stride() or k.dtype != q.dtype):
        raise ValueError("q and k must share shape, strides and type")
    if out is None:
        if stream is None:
            q_out, k_out = _new_outputs(q, out_dtype, two)
        else:
            with _memory_of(stream):
                q_out, k_out = _new_outputs(q, out_dtype, two)
            _used_here(stream, q_out, k_out)
    else:
        q_out, k_out = out
        if q_out.shape != q.shape or (k_out is not None) != two or (out_dtype is not None and q_out.dtype != out_dtype):
            raise ValueError("out must be (q_out, k_out) of q's shape")
    if two and (k_out.shape != q_out.shape or k_out.stride() != q_out.stride() or k_out.dtype != q_out.dtype):
        raise ValueError("q_out and k_out must share shape, strides and type")
    _on_current_device(q, k, q_out, k_out, q_weight, k_weight)
    prob, rope, _ = _norm_rope_call(q, q_out, None, q.dtype, q_weight, k_weight, two, dims, theta, norm, eps, pairs, origin, step, n_text, first_token)
    T, H, W = map(int, grid)
    _check(lib().psa_qk_norm_rope(q.data_ptr(), _ptr(k), q_out.data_ptr(), _ptr(k_out), _ptr(q_weight), _ptr(k_weight), prob, rope, T, H, W,
                                  _stream_ptr(stream)), "psa_qk_norm_rope")
    return q_out, k_out


def psa_qk_norm_rope_bwd(dq_out: torch.Tensor, dk_out: Optional[torch.Tensor], q: Optional[torch.Tensor], k: Optional[torch.Tensor],
                         grid: Sequence[int], dims: Sequence[int] = (44, 42, 42), theta: float = 10000.0, norm: str = "head",
                         q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
                         pairs: str = "interleaved", origin: Sequence[float] = (0.0, 0.0, 0.0), step: Sequence[float] = (1.0, 1.0, 1.0),
                         n_text: int = 0, first_token: int = 0, stream: Optional[torch.cuda.Stream] = None):
    """Gradient of psa_qk_norm_rope: from the gradients of its outputs (sharing shape, strides and type) and its inputs, which norm
    "none" does not need (None).  Returns (dq, dk, dq_weight, dk_weight): of q's type and layout without gaps, and fp32; None for
    what there is no input for."""
    two = dk_out is not None
    if two and (dk_out.shape != dq_out.shape or dk_out.stride() != dq_out.stride() or dk_out.dtype != dq_out.dtype):
        raise ValueError("dq_out and dk_out must share shape, strides and type")
    if q is None and (k is not None or norm != "none"):
        raise ValueError("q and k are needed with a norm")
    like = dq_out if q is None else q
    if q is not None:
        if q.shape != dq_out.shape or (k is not None) != two:
            raise ValueError("q and k must be those of the outputs")
        if two and (k.shape != q.shape or k.stride() != q.stride() or k.dtype != q.dtype):
            raise ValueError("q and k must share shape, strides and type")
    with _memory_of(stream):
        dq = torch.empty_like(like)
        dk = torch.empty_like(like) if two else None
    _on_current_device(dq_out, dk_out, q, k, q_weight, k_weight)
    prob, rope, weight_heads = _norm_rope_call(like, dq_out, dq, like.dtype, q_weight, k_weight, two, dims, theta, norm, eps, pairs, origin, step,
                                               n_text, first_token)
    dq_weight = dk_weight = scratch = None
    if weight_heads:
        with _memory_of(stream):
            dq_weight = torch.empty(q_weight.shape, dtype=torch.float32, device=q.device)
            dk_weight = torch.empty_like(dq_weight) if two else None
            scratch = torch.empty(int(lib().psa_qk_norm_rope_bwd_scratch_bytes(prob)), dtype=torch.uint8, device=q.device)
    _used_here(stream, dq, dk, dq_weight, dk_weight)
    T, H, W = map(int, grid)
    _check(lib().psa_qk_norm_rope_bwd(dq_out.data_ptr(), _ptr(dk_out), _ptr(q), _ptr(k), dq.data_ptr(), _ptr(dk), _ptr(q_weight), _ptr(k_weight),
                                      _ptr(dq_weight), _ptr(dk_weight), prob, rope, T, H, W, _ptr(scratch), _stream_ptr(stream)),
           "psa_qk_norm_rope_bwd")
    return dq, dk, dq_weight, dk_weight


def _as_it_lies(t: torch.Tensor) -> bool:
    """Whether the kernels can read a tensor of [..., tokens, 128] as it lies in memory."""
    st = t.stride()
    return st[-1] == 1 and t.data_ptr() % 16 == 0 and all(n <= 1 or (s >= 128 and s % 8 == 0) for n, s in zip(t.shape[:-1], st[:-1]))


class _NormRope(torch.autograd.Function):
    """psa_qk_norm_rope and its gradient, psa_qk_norm_rope_bwd."""

    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, grid, out_dtype, how):
        q_out, k_out = psa_qk_norm_rope(q, k, grid, q_weight=q_weight, k_weight=k_weight, out_dtype=out_dtype, **how)
        needed = how["norm"] != "none" or q.dtype != q_out.dtype   # (a rotation's gradient needs their type, if it is another one)
        ctx.save_for_backward(*((q, k) if needed else (None, None)), q_weight, k_weight)
        ctx.call = grid, how
        return q_out, k_out

    @staticmethod
    @once_differentiable
    def backward(ctx, dq_out, dk_out):
        q, k, q_weight, k_weight = ctx.saved_tensors
        grid, how = ctx.call
        grads = [g for g in (dq_out, dk_out) if g is not None]
        if not all(_as_it_lies(g) for g in grads) or grads[0].stride() != grads[-1].stride():   # (of a sum, say: one value for all)
            grads = [g.clone(memory_format=torch.contiguous_format) for g in grads]
        stream, here = how["stream"], None
        if stream is not None:   # q and k are ready there, the gradients here
            here = torch.cuda.current_stream()
            stream.wait_stream(here)
            for g in grads:
                g.record_stream(stream)
        dq, dk, dq_weight, dk_weight = psa_qk_norm_rope_bwd(grads[0], grads[1] if len(grads) > 1 else None, q, k, grid, q_weight=q_weight,
                                                            k_weight=k_weight, **how)
        if stream is not None:
            here.wait_stream(stream)
        if dq_weight is not None:
            dq_weight = dq_weight.to(q_weight.dtype)
        if dk_weight is not None:
            dk_weight = dk_weight.to(k_weight.dtype)
        return dq, dk, dq_weight, dk_weight, None, None, None


def psa_select_scratch_bytes(n_heads: int, grid: Sequence[int], tile: Sequence[int]) -> int:
    """Bytes of device scratch that psa_select_blocks needs."""
    T, H, W = map(int, grid)
    n = int(lib().psa_select_scratch_bytes(_problem(n_heads, tile, 1.0, 0, 128), T, H, W))
    if n < 0:
        _check(n, "psa_select_scratch_bytes")
    return n


def psa_select_blocks(q: torch.Tensor, k: torch.Tensor, grid: Sequence[int], tile: Sequence[int], keep, keep_self: bool = False,
                      out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, scratch: Optional[torch.Tensor] = None,
                      stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Key blocks with the largest pooled scores for every query block (see psa.h): q, k are bf16 device tensors [heads, T*H*W, 128]
    sharing strides (of a joint sequence: its video tokens, q[:, :T*H*W]), ``keep`` the number of blocks, one for all heads or one
    each.  Returns (row_ptr int32 [heads * blocks + 1], col_idx int32), in ``out`` if given; ``scratch`` (uint8,
    psa_select_scratch_bytes long) is allocated when not given."""
    nh, L, d = q.shape
    T, H, W = map(int, grid)
    if L != T * H * W or k.shape != q.shape:
        raise ValueError("shape mismatch")
    _on_current_device(q, k, scratch, *(out or ()))
    if q.dtype != torch.bfloat16 or k.dtype != torch.bfloat16:
        raise ValueError("bf16 tensors required")
    st = q.stride()
    if st != k.stride() or st[2] != 1:
        raise ValueError("q and k must share strides with a contiguous last dimension")
    bt, bh, bw = tile
    if bt < 1 or bh < 1 or bw < 1:
        raise ValueError("tile extents must be positive")
    nb = -(-T // bt) * -(-H // bh) * -(-W // bw)
    each = [keep] * nh if type(keep) is int else [int(x) for x in (keep if hasattr(keep, "__len__") else [keep] * nh)]
    if len(each) != nh or min(each, default=1) < 1 or max(each, default=1) > nb:
        raise ValueError("keep: between 1 and the number of blocks, one for all heads or one each")
    prob = _problem(nh, tile, 1.0, st[0], st[1], d)
    need = _scratch_bytes("select", nh, grid, tile)
    if out is None:
        with _memory_of(stream):
            out = (torch.empty(nh * nb + 1, dtype=torch.int32, device=q.device), torch.empty(sum(each) * nb, dtype=torch.int32, device=q.device))
        _used_here(stream, *out)
    elif any(x.dtype != torch.int32 or not x.is_contiguous() for x in out) or out[0].numel() != nh * nb + 1 or out[1].numel() < sum(each) * nb:
        raise ValueError("row_ptr (heads * blocks + 1 entries) and col_idx must be contiguous int32 tensors")
    row_ptr, col_idx = out
    if scratch is None:
        scratch = _new_scratch(need, q, stream)
    elif scratch.numel() * scratch.element_size() < need or not scratch.is_contiguous():
        raise ValueError("scratch too small")
    _check(lib().psa_select_blocks(q.data_ptr(), k.data_ptr(), prob, T, H, W, struct.pack("%di" % nh, *each), 1 if keep_self else 0, row_ptr.data_ptr(),
                                   col_idx.data_ptr(), col_idx.numel(), scratch.data_ptr(), _stream_ptr(stream)), "psa_select_blocks")
    return row_ptr, col_idx


def psa_attn_fwd_lists_scratch_bytes(n_heads: int, grid: Sequence[int], tile: Sequence[int], n_text: int = 0) -> int:
    """Bytes of device scratch that psa_attn_fwd_lists needs."""
    T, H, W = map(int, grid)
    n = int(lib().psa_attn_fwd_lists_scratch_bytes(_problem(n_heads, tile, 1.0, 0, 128), int(n_text), T, H, W))
    if n < 0:
        _check(n, "psa_attn_fwd_lists_scratch_bytes")
    return n


def psa_attn_fwd_lists(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, row_ptr: torch.Tensor, col_idx: torch.Tensor, grid: Sequence[int],
                       tile: Sequence[int], scale: float, n_text: int = 0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                       scratch: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """Attention over lists of key blocks (see psa.h): q, k, v are bf16 device tensors [heads, T*H*W + n_text, 128] sharing strides, the
    video tokens first; query block i of head h attends the blocks ``col_idx[row_ptr[h*NB + i]:row_ptr[h*NB + i + 1]]`` (int32,
    ascending), as psa_mask_build and psa_select_blocks write them, and all of the text.  ``scratch`` (uint8,
    psa_attn_fwd_lists_scratch_bytes long) is allocated when not given.  Returns (out like q, lse fp32 [heads, tokens]).

    How work is handed out goes by an average list of ``col_idx.numel() / row_ptr.numel()`` blocks: of a larger buffer pass the entries in use
    (``col_idx[:n]``), or a launch of few blocks may be slower than it needs to be."""
    nh, Lt, d = q.shape
    T, H, W = map(int, grid)
    n_text = int(n_text)
    if Lt != T * H * W + n_text or k.shape != q.shape or v.shape != q.shape:
        raise ValueError("shape mismatch")
    _on_current_device(q, k, v, row_ptr, col_idx, out, lse, scratch)
    bt, bh, bw = tile
    if bt < 1 or bh < 1 or bw < 1:
        raise ValueError("tile extents must be positive")
    nb = -(-T // bt) * -(-H // bh) * -(-W // bw)
    i32 = torch.int32
    if row_ptr.dtype != i32 or col_idx.dtype != i32 or not row_ptr.is_contiguous() or not col_idx.is_contiguous() or row_ptr.numel() != nh * nb + 1:
        raise ValueError("row_ptr (heads * blocks + 1 entries) and col_idx must be contiguous int32 tensors")
    if (out is not None and (out.shape != q.shape or out.dtype != q.dtype)) or (lse is not None and (tuple(lse.shape) != (nh, Lt) or lse.dtype != torch.float32)):
        raise ValueError("out must be like q, lse fp32 [heads, tokens]")
    out, lse, st = _device_call(q, k, v, out, lse, (nh, Lt), stream)
    prob = _problem(nh, tile, scale, st[0], st[1], d)
    need = _scratch_bytes("lists", nh, grid, tile, n_text)
    if scratch is None:
        scratch = _new_scratch(need, q, stream)
    elif scratch.numel() * scratch.element_size() < need or not scratch.is_contiguous():
        raise ValueError("scratch too small")
    _check(lib().psa_attn_fwd_lists(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(), row_ptr.data_ptr(), col_idx.data_ptr(),
                                    col_idx.numel(), prob, n_text, T, H, W, scratch.data_ptr(), _stream_ptr(stream)), "psa_attn_fwd_lists")
    return out, lse


LAUNCH_MODES = ("ticket", "direct", "shared", "shared_direct", "ticket_edge", "ticket_short")


def psa_last_attn_launch() -> Tuple[int, str, int]:
    """(work items, mode, CTAs per item) of the last attention kernel launched, see psa.h."""
    mode, ctas = ctypes.c_int32(0), ctypes.c_int32(0)
    items = lib().psa_last_attn_launch(ctypes.byref(mode), ctypes.byref(ctas))
    return items, LAUNCH_MODES[mode.value], ctas.value


GRID_KINDS = ("whole", "padded", "cut")


def psa_last_attn_grid() -> Tuple[str, int, int]:
    """(kind of grid, key slabs per block, keys of a block's last slab) of the last attention kernel launched, see psa.h."""
    slabs, keys = ctypes.c_int32(0), ctypes.c_int32(0)
    kind = lib().psa_last_attn_grid(ctypes.byref(slabs), ctypes.byref(keys))
    return GRID_KINDS[kind], slabs.value, keys.value


def psa_last_attn_classes() -> Tuple[int, List[Tuple[int, int, int]]]:
    """(axes whose last blocks were told apart, per class (query slabs, keys, blocks that share these)) of the last attention
    kernel launched, see psa.h: psa_last_attn_class."""
    got, axes = [], 0
    for c in range(8):
        x = [ctypes.c_int32(0) for _ in range(3)]
        axes = lib().psa_last_attn_class(c, *map(ctypes.byref, x))
        got.append(tuple(v.value for v in x))
    return axes, got


def psa_last_device_status() -> Tuple[int, int]:
    """Synchronises the device; returns (status, detail) left by the last psa_attn_fwd."""
    detail = ctypes.c_int32(0)
    st = lib().psa_last_device_status(ctypes.byref(detail))
    return st, detail.value


def psa_profile_events(start: Optional[torch.cuda.Event], stop: Optional[torch.cuda.Event]) -> None:
    """Record ``start``/``stop`` around the attention kernel of every later psa_attn_fwd (None, None: off).
    The events must have been created with enable_timing=True and recorded once (so that they exist)."""
    a = None if start is None else ctypes.c_void_p(start.cuda_event)
    b = None if stop is None else ctypes.c_void_p(stop.cuda_event)
    _check(lib().psa_profile_events(a, b), "psa_profile_events")


def psa_selftest_wait_timeout(limit_ms: int = 20, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Launches the bounded-wait self-test kernel (see psa.h); read the outcome with psa_last_device_status()."""
    _check(lib().psa_selftest_wait_timeout(int(limit_ms), _stream_ptr(stream)), "psa_selftest_wait_timeout")


def psa_launch_count() -> int:
    return int(lib().psa_launch_count())


def psa_shutdown() -> None:
    _check(lib().psa_shutdown(), "psa_shutdown")
