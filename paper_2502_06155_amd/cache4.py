"""Python binding of the C ABI in include/cache4_attn.h: the cache in 4 bits (argument marshalling, checks and
workspaces only).

The functions named as in the header take device tensors or addresses and the header's arguments. The
torch wrappers below them (cache4_new, cache4_write, cache4_read, cache4_attn) check shapes, types and devices,
allocate outputs and workspaces and run on the current stream of the tensors' device.
"""
from __future__ import annotations

import functools

from ._lib import lib
from .api import _check, _ptr, _stream
from .blocks import BLOCK_TOKENS, _bytes_of, _current, _on, _unrecorded, _want, _workspace

try:
    import torch
except ImportError:  # the functions of the C ABI take addresses and do without
    torch = None

CACHE4_GROUP = 32


def cache4_attn_write(k, v, k_pages, v_pages, k_scales, v_scales, table, lens, n_new, k_held, v_held, B: int, Hkv: int,
                      N: int, d: int, max_pages: int, n_pages: int, stream=None) -> None:
    """cache4_attn_write of the C ABI."""
    _check(lib.cache4_attn_write(_ptr(k), _ptr(v), _ptr(k_pages), _ptr(v_pages), _ptr(k_scales), _ptr(v_scales),
                                 _ptr(table), _ptr(lens), _ptr(n_new), _ptr(k_held), _ptr(v_held), B, Hkv, N, d,
                                 max_pages, n_pages, _stream(stream)), "cache4_attn_write")


def cache4_attn_read(k_pages, v_pages, k_scales, v_scales, table, lens, k_out, v_out, B: int, Hkv: int, N: int, d: int,
                     max_pages: int, n_pages: int, first: int, stream=None) -> None:
    """cache4_attn_read of the C ABI."""
    _check(lib.cache4_attn_read(_ptr(k_pages), _ptr(v_pages), _ptr(k_scales), _ptr(v_scales), _ptr(table), _ptr(lens),
                                _ptr(k_out), _ptr(v_out), B, Hkv, N, d, max_pages, n_pages, first,
                                _stream(stream)), "cache4_attn_read")


@functools.lru_cache(maxsize=1024)
def cache4_attn_fwd_workspace(B: int, H: int, Hkv: int, N: int, d: int, max_pages: int) -> int:
    """Bytes of workspace that cache4_attn_fwd needs for these sizes."""
    return _bytes_of(lib.cache4_attn_fwd_workspace, "cache4_attn_fwd_workspace", B, H, Hkv, N, d, max_pages)


def cache4_attn_fwd(q, k_pages, v_pages, k_scales, v_scales, table, lens, per_head, out, lse, B: int, H: int, Hkv: int,
                    N: int, d: int, max_pages: int, n_pages: int, scale: float, workspace=None,
                    workspace_bytes: int = 0, stream=None) -> None:
    """cache4_attn_fwd of the C ABI."""
    _check(lib.cache4_attn_fwd(_ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(k_scales), _ptr(v_scales), _ptr(table),
                               _ptr(lens), int(per_head), _ptr(out), _ptr(lse), B, H, Hkv, N, d, max_pages, n_pages,
                               float(scale), _ptr(workspace), workspace_bytes, _stream(stream)), "cache4_attn_fwd")


# ---------------------------------------------------------------------------------------------
# torch wrappers


def cache4_new(n_pages: int, Hkv: int, d: int, device="cuda"):
    """(k_pages, v_pages, k_scales, v_scales) of a cache of n_pages pages, not initialised."""
    codes = (n_pages, Hkv, BLOCK_TOKENS, d // 2)
    scales = (n_pages, Hkv, d // CACHE4_GROUP, BLOCK_TOKENS)
    return tuple(torch.empty(s, dtype=torch.uint8, device=device) for s in (codes, codes, scales, scales))


def _check_cache(k_pages, v_pages, k_scales, v_scales):
    """(pages, key heads, d, device) of the cache's tensors."""
    if k_pages.dim() != 4 or not k_pages.is_cuda:
        raise ValueError("k_pages must be a [n_pages, Hkv, 128, d / 2] tensor on a GPU")
    pages, Hkv, _, half = shape = k_pages.shape
    device, u8 = k_pages.device, torch.uint8
    codes, scales = (pages, Hkv, BLOCK_TOKENS, half), (pages, Hkv, half // (CACHE4_GROUP // 2), BLOCK_TOKENS)
    # One comparison chain where all is well: four tensors a call.
    if not (shape == codes == v_pages.shape and scales == k_scales.shape == v_scales.shape
            and k_pages.dtype is u8 and v_pages.dtype is u8 and k_scales.dtype is u8 and v_scales.dtype is u8
            and device == v_pages.device == k_scales.device == v_scales.device and k_pages.is_contiguous()
            and v_pages.is_contiguous() and k_scales.is_contiguous() and v_scales.is_contiguous()):
        _want(k_pages, "k_pages", codes, u8, device)
        _want(v_pages, "v_pages", codes, u8, device)
        _want(k_scales, "k_scales", scales, u8, device)
        _want(v_scales, "v_scales", scales, u8, device)
    return pages, Hkv, 2 * half, device


def _check_table(table, lens, B: int, device) -> int:
    """Pages of a row of a table that all heads share."""
    if table.dim() != 2:
        raise ValueError("table must be [B, max_pages]")
    _want(table, "table", (B, table.shape[1]), torch.int32, device)
    _want(lens, "lens", (B,), torch.int32, device)
    return table.shape[1]


def cache4_write(k, v, k_pages, v_pages, k_scales, v_scales, table, lens, n_new=None, return_held=False):
    """Puts k, v [B, Hkv, N, d] bf16 behind the lens[b] tokens that the sequences hold in the cache: k_pages, v_pages
    uint8 [n_pages, Hkv, 128, d / 2] and k_scales, v_scales uint8 [n_pages, Hkv, d / 32, 128] (cache4_new), table int32
    [B, max_pages], lens int32 [B] (left as it is). n_new (int32 [B]): how many of the N tokens each sequence takes.
    With return_held it returns (k, v) as the cache holds them, zeros for tokens that were not written: what later
    tokens will attend to, for the attention of the tokens themselves, without a gradient (it warns where autograd
    would have recorded one)."""
    pages, Hkv, d, device = _check_cache(k_pages, v_pages, k_scales, v_scales)
    if k.dim() != 4:
        raise ValueError("k must be a [B, Hkv, N, d] tensor on a GPU")
    B, _, N, _ = k.shape
    _want(k, "k", (B, Hkv, N, d), torch.bfloat16, device)
    _want(v, "v", (B, Hkv, N, d), torch.bfloat16, device)
    width = _check_table(table, lens, B, device)
    if n_new is not None:
        _want(n_new, "n_new", (B,), torch.int32, device)
    if return_held:
        _unrecorded("cache4_write", "what it returns is rounded to the cache's numbers", (k, v))
    with _on(device):
        held = (torch.empty_like(k), torch.empty_like(v)) if return_held else (None, None)
        _check(lib.cache4_attn_write(k.data_ptr(), v.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
                                     k_scales.data_ptr(), v_scales.data_ptr(), table.data_ptr(), lens.data_ptr(),
                                     _ptr(n_new), *map(_ptr, held), B, Hkv, N, d, width, pages, _current(device)),
               "cache4_attn_write")
    return held if return_held else None


def cache4_read(k_pages, v_pages, k_scales, v_scales, table, lens, N: int, first: int = 0):
    """(k, v) bf16 [B, Hkv, N, d]: tokens first .. first + N - 1 of every sequence of the cache, exactly; zeros from
    lens[b] on."""
    pages, Hkv, d, device = _check_cache(k_pages, v_pages, k_scales, v_scales)
    B = lens.shape[0] if lens.dim() == 1 else 0
    width = _check_table(table, lens, B, device)
    if N < 1:
        raise ValueError(f"N must be at least 1, got {N}")
    if not -(1 << 31) <= first < 1 << 31:  # (a C int would take what is left of it)
        raise ValueError(f"first must be a token below 2^31, got {first}")
    with _on(device):
        k = torch.empty((B, Hkv, N, d), dtype=torch.bfloat16, device=device)
        out = (k, torch.empty_like(k))
        _check(lib.cache4_attn_read(k_pages.data_ptr(), v_pages.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(),
                                    table.data_ptr(), lens.data_ptr(), k.data_ptr(), out[1].data_ptr(), B, Hkv, N, d,
                                    width, pages, first, _current(device)), "cache4_attn_read")
    return out


def cache4_attn(q, k_pages, v_pages, k_scales, v_scales, table, lens, scale: float | None = None, out=None,
                return_lse=False):
    """Attention of q [B, H, N, d], the last N tokens of each sequence, over the 4-bit cache; lens counts them.
    table [B, max_pages] with lens [B], or, for pages chosen per key head, [B, Hkv, max_pages] with [B, Hkv]. It has
    no gradient (and warns where autograd would have recorded it). Returns out, or (out, lse)."""
    pages, Hkv, d, device = _check_cache(k_pages, v_pages, k_scales, v_scales)
    if q.dim() != 4:
        raise ValueError("q must be a [B, H, N, d] tensor on a GPU")
    _unrecorded("cache4_attn", "it has no gradient", (q,))
    B, H, N, _ = q.shape
    _want(q, "q", (B, H, N, d), torch.bfloat16, device)
    per_head = table.dim() == 3
    if table.dim() not in (2, 3):
        raise ValueError("table must be [B, max_pages] or [B, Hkv, max_pages]")
    lead = (B, Hkv) if per_head else (B,)
    width = table.shape[-1]
    _want(table, "table", (*lead, width), torch.int32, device)
    _want(lens, "lens", lead, torch.int32, device)
    with _on(device):
        if out is None:
            out = torch.empty_like(q)
        else:
            _want(out, "out", q.shape, torch.bfloat16, device)
        lse = q.new_empty((B, H, N), dtype=torch.float32) if return_lse else None
        n = cache4_attn_fwd_workspace(B, H, Hkv, N, d, width)
        workspace = _workspace(n, device)
        _check(lib.cache4_attn_fwd(q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), k_scales.data_ptr(),
                                   v_scales.data_ptr(), table.data_ptr(), lens.data_ptr(), per_head, out.data_ptr(),
                                   lse.data_ptr() if return_lse else None, B, H, Hkv, N, d, width, pages,
                                   d ** -0.5 if scale is None else scale, workspace.data_ptr() if n else None, n,
                                   _current(device)), "cache4_attn_fwd")
    return (out, lse) if return_lse else out
