"""Python binding of the C ABI in include/block_attn.h: attention over selected blocks and over an
8-bit cache (argument marshalling, checks and workspaces only).

The functions named as in the header take device tensors or addresses and the header's arguments.
The torch wrappers below them (block_means, block_lists, block_attn, block_attn_grad, cache_write,
cache_attn) check shapes, types and devices, allocate outputs and workspaces and run on the current
stream of the tensors' device.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import warnings

from ._lib import lib
from .api import _check, _ptr, _stream

try:
    import torch
except ImportError:  # the functions of the C ABI take addresses and do without
    torch = None

BLOCK_TOKENS = 128
_HERE = contextlib.nullcontext()


def block_attn_means(x, means, B: int, H: int, S: int, d: int, lens=None, stream=None) -> None:
    """block_attn_means of the C ABI."""
    _check(lib.block_attn_means(_ptr(x), _ptr(means), B, H, S, d, _ptr(lens), _stream(stream)), "block_attn_means")


def block_attn_lists(q, kmeans, lists, B: int, H: int, Hkv: int, Sq: int, Skv: int, d: int, n_list: int,
                     sink: int, local: int, causal, lens=None, stream=None) -> None:
    """block_attn_lists of the C ABI."""
    _check(lib.block_attn_lists(_ptr(q), _ptr(kmeans), _ptr(lists), B, H, Hkv, Sq, Skv, d, n_list, sink, local,
                                int(causal), _ptr(lens), _stream(stream)), "block_attn_lists")


def _bytes_of(fn, name: str, *sizes: int) -> int:
    n = ctypes.c_size_t(0)
    _check(fn(*sizes, ctypes.byref(n)), name)
    return n.value


@functools.lru_cache(maxsize=1024)
def block_attn_fwd_workspace(B: int, H: int, Hkv: int, Sq: int, Skv: int, d: int, n_list: int) -> int:
    """Bytes of workspace that block_attn_fwd needs for these sizes."""
    return _bytes_of(lib.block_attn_fwd_workspace, "block_attn_fwd_workspace", B, H, Hkv, Sq, Skv, d, n_list)


def block_attn_fwd(q, k, v, lists, out, lse, B: int, H: int, Hkv: int, Sq: int, Skv: int, d: int, n_list: int,
                   causal, lens, scale: float, workspace=None, workspace_bytes: int = 0, stream=None) -> None:
    """block_attn_fwd of the C ABI."""
    _check(lib.block_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(lists), _ptr(out), _ptr(lse), B, H, Hkv, Sq, Skv, d,
                              n_list, int(causal), _ptr(lens), float(scale), _ptr(workspace), workspace_bytes,
                              _stream(stream)), "block_attn_fwd")


@functools.lru_cache(maxsize=1024)
def block_attn_bwd_workspace(B: int, H: int, Hkv: int, Sq: int, Skv: int, d: int, n_list: int) -> int:
    """Bytes of workspace that block_attn_bwd needs for these sizes."""
    return _bytes_of(lib.block_attn_bwd_workspace, "block_attn_bwd_workspace", B, H, Hkv, Sq, Skv, d, n_list)


def block_attn_bwd(q, k, v, lists, out, dout, lse, dq, dk, dv, B: int, H: int, Hkv: int, Sq: int, Skv: int, d: int,
                   n_list: int, causal, lens, scale: float, workspace=None, workspace_bytes: int = 0,
                   stream=None) -> None:
    """block_attn_bwd of the C ABI."""
    _check(lib.block_attn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(lists), _ptr(out), _ptr(dout), _ptr(lse), _ptr(dq),
                              _ptr(dk), _ptr(dv), B, H, Hkv, Sq, Skv, d, n_list, int(causal), _ptr(lens),
                              float(scale), _ptr(workspace), workspace_bytes, _stream(stream)), "block_attn_bwd")


def cache_attn_write(k, v, k_pages, v_pages, k_scales, v_scales, table, lens, n_new, B: int, Hkv: int, N: int, d: int,
                     max_pages: int, n_pages: int, stream=None) -> None:
    """cache_attn_write of the C ABI."""
    _check(lib.cache_attn_write(_ptr(k), _ptr(v), _ptr(k_pages), _ptr(v_pages), _ptr(k_scales), _ptr(v_scales),
                                _ptr(table), _ptr(lens), _ptr(n_new), B, Hkv, N, d, max_pages, n_pages,
                                _stream(stream)), "cache_attn_write")


@functools.lru_cache(maxsize=1024)
def cache_attn_fwd_workspace(B: int, H: int, Hkv: int, N: int, d: int, max_pages: int) -> int:
    """Bytes of workspace that cache_attn_fwd needs for these sizes."""
    return _bytes_of(lib.cache_attn_fwd_workspace, "cache_attn_fwd_workspace", B, H, Hkv, N, d, max_pages)


def cache_attn_fwd(q, k_pages, v_pages, k_scales, v_scales, table, lens, per_head, out, lse, B: int, H: int, Hkv: int,
                   N: int, d: int, max_pages: int, n_pages: int, scale: float, workspace=None,
                   workspace_bytes: int = 0, stream=None) -> None:
    """cache_attn_fwd of the C ABI."""
    _check(lib.cache_attn_fwd(_ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(k_scales), _ptr(v_scales), _ptr(table),
                              _ptr(lens), int(per_head), _ptr(out), _ptr(lse), B, H, Hkv, N, d, max_pages, n_pages,
                              float(scale), _ptr(workspace), workspace_bytes, _stream(stream)), "cache_attn_fwd")


# ---------------------------------------------------------------------------------------------
# torch wrappers


def _want(t, name: str, shape, dtype, device) -> None:
    """t is a contiguous tensor of this shape and type on this GPU: checked before anything is
    launched, since the kernels read and write that many elements."""
    if t.shape == shape and t.dtype is dtype and t.device == device and t.is_contiguous():
        return
    if t.shape != shape:
        raise ValueError(f"{name} must have the shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} must be on the GPU {device}, got {t.device}")
    raise ValueError(f"{name} must be contiguous")


def _unrecorded(name: str, instead: str) -> None:
    """Called where an input requires a gradient: says that the outputs carry no graph, if autograd
    would have recorded the call."""
    if torch.is_grad_enabled():
        warnings.warn(f"{name} is not recorded by autograd, its inputs get no gradient from it: {instead}", stacklevel=3)


def _out(out, shape, dtype, device):
    """The output that the caller gave, or a new one."""
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _want(out, "out", shape, dtype, device)
    return out


def _on(device):
    """The context in which `device` is the current one."""
    return _HERE if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def _current(device) -> int:
    """The handle of the device's current stream."""
    return torch._C._cuda_getCurrentRawStream(device.index)


def _heads(q, k):
    """(B, H, Hkv, Sq, Skv, d) of q [B, H, Sq, d] and k [B, Hkv, Skv, d]."""
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("expected [B, H, S, d] tensors")
    if not q.is_cuda:
        raise ValueError("tensors must be on a GPU")
    B, H, Sq, d = q.shape
    return B, H, k.shape[1], Sq, k.shape[2], d


def _lens(lens, shape, device) -> None:
    if lens is not None:
        _want(lens, "lens", shape, torch.int32, device)


def _workspace(n: int, device):
    """Scratch of n bytes from torch's allocator, which hands it on in stream order and gives calls
    that are captured into a graph memory of that graph's own."""
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def block_means(x, lens=None, out=None):
    """Means of every block of 128 tokens: x [B, H, S, d] bf16 -> [B, H, ceil(S / 128), d] bf16; lens
    (int32 [B]) leaves out the tokens behind a sequence's end."""
    if x.dim() != 4 or not x.is_cuda:
        raise ValueError("x must be a [B, H, S, d] tensor on a GPU")
    B, H, S, d = x.shape
    _want(x, "x", x.shape, torch.bfloat16, x.device)
    shape = (B, H, -(-S // BLOCK_TOKENS), d)
    with _on(x.device):
        out = _out(out, shape, torch.bfloat16, x.device)
        _lens(lens, (B,), x.device)
        block_attn_means(x, out, B, H, S, d, lens, _current(x.device))
    return out


def block_lists(q, kmeans, Skv: int, n_list: int, causal=False, sink: int = 0, local: int = 1, lens=None, out=None):
    """The key blocks that each block of 128 query rows attends to, chosen by the product of the
    block means: q [B, H, Sq, d], kmeans [B, Hkv, ceil(Skv / 128), d] (block_means of the keys) ->
    int32 [B, Hkv, ceil(Sq / 128), n_list], ascending, -1 behind the end. The first `sink` blocks
    and the rows' own (with local - 1 more beside them; local = 0: none) are always chosen. The rows
    are the last Sq of Skv positions, the same in every sequence: with lens, a query block whose rows
    are all padding gets an empty list. One list serves all rows of a query block, chosen by the mean
    of them all: with causal too, which blocks a row gets depends on rows up to 127 later (Sq = 1
    chooses by the token alone, as a program that decodes does)."""
    B, H, Hkv, Sq, nb, d = _heads(q, kmeans)
    if nb != -(-Skv // BLOCK_TOKENS):
        raise ValueError(f"kmeans must hold {-(-Skv // BLOCK_TOKENS)} blocks for Skv = {Skv}, got {nb}")
    _want(q, "q", q.shape, torch.bfloat16, q.device)
    _want(kmeans, "kmeans", (B, Hkv, nb, d), torch.bfloat16, q.device)
    shape = (B, Hkv, -(-Sq // BLOCK_TOKENS), n_list)
    with _on(q.device):
        out = _out(out, shape, torch.int32, q.device)
        _lens(lens, (B,), q.device)
        block_attn_lists(q, kmeans, out, B, H, Hkv, Sq, Skv, d, n_list, sink, local, causal, lens,
                         _current(q.device))
    return out


def _check_qkv(q, k, v, lists):
    B, H, Hkv, Sq, Skv, d = _heads(q, k)
    _want(q, "q", q.shape, torch.bfloat16, q.device)
    _want(k, "k", (B, Hkv, Skv, d), torch.bfloat16, q.device)
    _want(v, "v", (B, Hkv, Skv, d), torch.bfloat16, q.device)
    if lists.dim() != 4:
        raise ValueError("lists must be [B, Hkv, ceil(Sq / 128), n_list]")
    _want(lists, "lists", (B, Hkv, -(-Sq // BLOCK_TOKENS), lists.shape[3]), torch.int32, q.device)
    return B, H, Hkv, Sq, Skv, d, lists.shape[3]


def block_attn(q, k, v, lists, causal=False, scale: float | None = None, lens=None, out=None, return_lse=False):
    """Attention over the listed blocks: q [B, H, Sq, d], k and v [B, Hkv, Skv, d], lists as
    block_lists gives them. The rows are the last Sq of Skv positions, the same in every sequence: with
    lens, rows from lens[b] on are padding and give zeros, so decoding sequences of different lengths
    takes a call for each (cache_attn takes them together). Autograd does not record it (it warns where
    it would have): block_attn_grad gives the gradients. Returns out, or (out, lse)."""
    sizes = _check_qkv(q, k, v, lists)
    if q.requires_grad or k.requires_grad or v.requires_grad:
        _unrecorded("block_attn", "block_attn_grad gives the gradients")
    B, H, _, Sq, _, d, _ = sizes
    with _on(q.device):
        if out is None:
            out = torch.empty_like(q)
        else:
            _want(out, "out", q.shape, torch.bfloat16, q.device)
        _lens(lens, (B,), q.device)
        lse = torch.empty((B, H, Sq), dtype=torch.float32, device=q.device) if return_lse else None
        n = block_attn_fwd_workspace(*sizes)
        block_attn_fwd(q, k, v, lists, out, lse, *sizes, causal, lens, d ** -0.5 if scale is None else scale,
                       _workspace(n, q.device), n, _current(q.device))
    return (out, lse) if return_lse else out


def block_attn_grad(q, k, v, lists, out, dout, lse, causal=False, scale: float | None = None, lens=None):
    """(dq, dk, dv) of block_attn: out and lse are what it returned for the same arguments, dout is
    the gradient of out."""
    sizes = _check_qkv(q, k, v, lists)
    B, H, _, Sq, _, d, _ = sizes
    _want(out, "out", q.shape, torch.bfloat16, q.device)
    _want(dout, "dout", q.shape, torch.bfloat16, q.device)
    _want(lse, "lse", (B, H, Sq), torch.float32, q.device)
    _lens(lens, (B,), q.device)
    with _on(q.device):
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        n = block_attn_bwd_workspace(*sizes)
        block_attn_bwd(q, k, v, lists, out, dout, lse, dq, dk, dv, *sizes, causal, lens,
                       d ** -0.5 if scale is None else scale, _workspace(n, q.device), n, _current(q.device))
    return dq, dk, dv


def _check_cache(k_pages, v_pages, k_scales, v_scales, device):
    """(pages, key heads, d) of the cache's tensors."""
    if k_pages.dim() != 4:
        raise ValueError("k_pages must be [n_pages, Hkv, 128, d]")
    pages, Hkv, _, d = k_pages.shape
    _want(k_pages, "k_pages", (pages, Hkv, BLOCK_TOKENS, d), torch.float8_e4m3fn, device)
    _want(v_pages, "v_pages", (pages, Hkv, d, BLOCK_TOKENS), torch.float8_e4m3fn, device)
    _want(k_scales, "k_scales", (pages, Hkv), torch.float32, device)
    _want(v_scales, "v_scales", (pages, Hkv), torch.float32, device)
    return pages, Hkv, d


def cache_write(k, v, k_pages, v_pages, k_scales, v_scales, table, lens, n_new=None) -> None:
    """Puts k, v [B, Hkv, N, d] bf16 behind the lens[b] tokens that the sequences hold in the cache:
    k_pages [n_pages, Hkv, 128, d] and v_pages [n_pages, Hkv, d, 128] float8_e4m3fn, scales fp32
    [n_pages, Hkv], table int32 [B, max_pages], lens int32 [B] (left as it is). n_new (int32 [B]):
    how many of the N tokens each sequence takes."""
    if k.dim() != 4 or not k.is_cuda:
        raise ValueError("k must be a [B, Hkv, N, d] tensor on a GPU")
    pages, Hkv, d = _check_cache(k_pages, v_pages, k_scales, v_scales, k.device)
    B, _, N, _ = k.shape
    _want(k, "k", (B, Hkv, N, d), torch.bfloat16, k.device)
    _want(v, "v", (B, Hkv, N, d), torch.bfloat16, k.device)
    if table.dim() != 2:
        raise ValueError("table must be [B, max_pages]")
    _want(table, "table", (B, table.shape[1]), torch.int32, k.device)
    _want(lens, "lens", (B,), torch.int32, k.device)
    if n_new is not None:
        _want(n_new, "n_new", (B,), torch.int32, k.device)
    with _on(k.device):
        cache_attn_write(k, v, k_pages, v_pages, k_scales, v_scales, table, lens, n_new, B, Hkv, N, d,
                         table.shape[1], pages, _current(k.device))


def cache_attn(q, k_pages, v_pages, k_scales, v_scales, table, lens, scale: float | None = None, out=None,
               return_lse=False):
    """Attention of q [B, H, N, d], the last N tokens of each sequence, over the cache; lens counts
    them. table [B, max_pages] with lens [B], or, for pages chosen per key head, [B, Hkv, max_pages]
    with [B, Hkv]. It has no gradient (and warns where autograd would have recorded it). Returns out,
    or (out, lse)."""
    if q.dim() != 4 or not q.is_cuda:
        raise ValueError("q must be a [B, H, N, d] tensor on a GPU")
    if q.requires_grad:
        _unrecorded("cache_attn", "it has no gradient")
    pages, Hkv, d = _check_cache(k_pages, v_pages, k_scales, v_scales, q.device)
    B, H, N, _ = q.shape
    _want(q, "q", (B, H, N, d), torch.bfloat16, q.device)
    per_head = table.dim() == 3
    if table.dim() not in (2, 3):
        raise ValueError("table must be [B, max_pages] or [B, Hkv, max_pages]")
    lead = (B, Hkv) if per_head else (B,)
    width = table.shape[-1]
    _want(table, "table", (*lead, width), torch.int32, q.device)
    _want(lens, "lens", lead, torch.int32, q.device)
    with _on(q.device):
        if out is None:
            out = torch.empty_like(q)
        else:
            _want(out, "out", q.shape, torch.bfloat16, q.device)
        lse = torch.empty((B, H, N), dtype=torch.float32, device=q.device) if return_lse else None
        n = cache_attn_fwd_workspace(B, H, Hkv, N, d, width)
        cache_attn_fwd(q, k_pages, v_pages, k_scales, v_scales, table, lens, per_head, out, lse, B, H, Hkv, N, d,
                       width, pages, d ** -0.5 if scale is None else scale, _workspace(n, q.device), n,
                       _current(q.device))
    return (out, lse) if return_lse else out
