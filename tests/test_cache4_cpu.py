"""Host-side checks of the 4-bit cache's entry points that need no GPU: exports, argument errors (found before any
HIP call, so nothing is enqueued), workspace sizes, and the torch wrappers' checks."""
import ctypes
import os
import re

import pytest

import paper_2502_06155_amd as ta
from paper_2502_06155_amd._lib import lib
from tests.conftest import ROOT

NULL, SHAPE, DIM, ALIGN, SCALE, OVERLAP = 1, 2, 3, 5, 6, 7
M = 1 << 20  # addresses a MiB apart: every tensor below is smaller


def test_every_declared_symbol_is_exported_and_bound():
    src = open(os.path.join(ROOT, "include", "cache4_attn.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    names = sorted(set(re.findall(r"^\s*int\s+(\w+)\s*\(", src, flags=re.M)))
    assert len(names) == 4
    for name in names:
        assert hasattr(lib, name) and hasattr(ta, name), name
    assert f"#define TA_CACHE4_GROUP {ta.CACHE4_GROUP}" in src


def _write(**kw):
    a = dict(k=M, v=2 * M, kp=3 * M, vp=4 * M, ks=5 * M, vs=6 * M, table=7 * M, lens=8 * M, n_new=None, kh=9 * M,
             vh=10 * M, B=2, Hkv=2, N=3, d=64, max_pages=4, n_pages=8)
    a.update(kw)
    return lib.cache4_attn_write(*a.values(), None)


def _read(**kw):
    a = dict(kp=3 * M, vp=4 * M, ks=5 * M, vs=6 * M, table=7 * M, lens=8 * M, k=9 * M, v=10 * M, B=2, Hkv=2, N=3, d=64,
             max_pages=4, n_pages=8, first=0)
    a.update(kw)
    return lib.cache4_attn_read(*a.values(), None)


def _attn(**kw):
    a = dict(q=M, kp=2 * M, vp=3 * M, ks=4 * M, vs=5 * M, table=6 * M, lens=7 * M, per_head=0, out=8 * M, lse=9 * M, B=2,
             H=4, Hkv=2, N=3, d=64, max_pages=40, n_pages=8, scale=0.1, ws=16 * M, bytes=1 << 30)
    a.update(kw)
    return lib.cache4_attn_fwd(*a.values(), None)


@pytest.mark.parametrize("call,pointers", [(_write, "k v kp vp ks vs table lens"), (_read, "kp vp ks vs table lens"),
                                           (_attn, "q kp vp ks vs table lens out")])
def test_null_pointers(call, pointers):
    for p in pointers.split():
        assert call(**{p: None}) == NULL, p
    assert _read(k=None, v=None) == NULL


@pytest.mark.parametrize("call", [_write, _read, _attn])
def test_shapes(call):
    for kw in (dict(B=0), dict(Hkv=0), dict(N=0), dict(max_pages=0), dict(n_pages=0), dict(max_pages=1 << 24),
               dict(B=65536), dict(B=65535, Hkv=1, max_pages=1 << 20)):
        if call is _attn and "Hkv" in kw:
            kw = {**kw, "H": 4}
        assert call(**kw) == SHAPE, kw
    for d in (0, 32, 80, 256):
        assert call(d=d) == DIM


def test_write_errors():
    for p in ("k", "v", "kp", "vp", "ks", "vs", "kh", "vh"):
        assert _write(**{p: 11 * M + 8}) == ALIGN, p
    assert _write(table=7 * M + 2) == ALIGN and _write(lens=8 * M + 1) == ALIGN and _write(n_new=11 * M + 2) == ALIGN
    for kw in (dict(kp=M), dict(vp=3 * M + 1024), dict(ks=3 * M), dict(vs=7 * M), dict(kp=8 * M), dict(kh=M),
               dict(vh=9 * M), dict(kh=4 * M), dict(vh=8 * M), dict(ks=5 * M, n_new=5 * M)):
        assert _write(**kw) == OVERLAP, kw


@pytest.mark.parametrize("d,most", [(64, 32), (96, 20), (128, 16)])
def test_more_tokens_than_the_grid_holds(d, most):
    """256 threads a workgroup and 2^32 in a grid; `most` tokens a workgroup. What fits goes on to the next check."""
    far = dict(k=1 << 50, v=1 << 51, kh=1 << 52, vh=1 << 53, B=1, Hkv=1, d=d, max_pages=1 << 23)
    limit = ((1 << 32) // 256 - 9) * most
    assert limit >= 2 ** 28 - 256
    for call, kw in ((_write, far), (_read, {**far, "k": 1 << 50, "v": 1 << 51})):
        kw = {n: x for n, x in kw.items() if call is _write or n not in ("kh", "vh")}
        assert call(**kw, N=limit + 2 * most) == SHAPE
        assert call(**kw, N=limit - most, lens=8 * M + 1) == ALIGN


def test_read_errors():
    assert _read(first=-1) == SHAPE and _read(first=2 ** 31 - 3) == SHAPE
    for p in ("kp", "vp", "ks", "vs", "k", "v"):
        assert _read(**{p: 11 * M + 8}) == ALIGN, p
    assert _read(lens=8 * M + 2) == ALIGN
    for kw in (dict(k=3 * M), dict(v=9 * M), dict(v=6 * M), dict(k=7 * M), dict(v=8 * M)):
        assert _read(**kw) == OVERLAP, kw


def test_attention_errors():
    assert _attn(H=3) == SHAPE and _attn(H=0) == SHAPE and _attn(N=1 << 20) == SHAPE
    assert _attn(scale=float("nan")) == SCALE and _attn(scale=float("-inf")) == SCALE
    for p in ("q", "kp", "vp", "ks", "vs", "out"):
        assert _attn(**{p: 11 * M + 8}) == ALIGN, p
    assert _attn(lse=9 * M + 2) == ALIGN
    for kw in (dict(out=M), dict(out=2 * M), dict(lse=8 * M), dict(out=6 * M), dict(ws=4 * M), dict(lse=7 * M)):
        assert _attn(**kw) == OVERLAP, kw
    n = ta.cache4_attn_fwd_workspace(2, 4, 2, 3, 64, 40)
    assert n > 0 and ta.cache4_attn_fwd_workspace(2, 4, 2, 3, 64, 4) == 0
    assert _attn(bytes=n - 1) == SHAPE and _attn(ws=None) == SHAPE and _attn(ws=16 * M + 8) == ALIGN
    size = ctypes.c_size_t()
    assert lib.cache4_attn_fwd_workspace(2, 4, 2, 3, 64, 40, None) == NULL
    assert lib.cache4_attn_fwd_workspace(2, 4, 2, 3, 65, 40, ctypes.byref(size)) == DIM
    for N in (1, 17, 512, 100000):
        assert ta.cache4_attn_fwd_workspace(4, 8, 2, N, 128, 1000) < 72 << 20


def test_wrappers_refuse():
    torch = pytest.importorskip("torch")
    cache = ta.cache4_new(3, 2, 64, device="cpu")
    assert [tuple(x.shape) for x in cache] == [(3, 2, 128, 32)] * 2 + [(3, 2, 2, 128)] * 2
    x = torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16)
    i = torch.zeros(1, 1, dtype=torch.int32)
    for call in (lambda: ta.cache4_write(x, x, *cache, i, i[0]), lambda: ta.cache4_read(*cache, i, i[0], 3),
                 lambda: ta.cache4_attn(x, *cache, i, i[0])):
        with pytest.raises(ValueError, match="GPU"):
            call()
