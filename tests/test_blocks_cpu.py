"""Host-side checks of the block attention and cache entry points that need no GPU: exports,
argument errors (found before any HIP call, so nothing is enqueued), workspace sizes, and the torch
wrappers' checks."""
import ctypes
import os
import re

import numpy as np
import pytest

import paper_2502_06155_amd as ta
from paper_2502_06155_amd._lib import lib
from tests.conftest import ROOT

NULL, SHAPE, DIM, ALIGN, SCALE, OVERLAP = 1, 2, 3, 5, 6, 7
M = 1 << 20  # addresses a MiB apart: every tensor below is smaller


def test_every_declared_symbol_is_exported_and_bound():
    src = open(os.path.join(ROOT, "include", "block_attn.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    names = sorted(set(re.findall(r"^\s*int\s+(\w+)\s*\(", src, flags=re.M)))
    assert len(names) == 9
    for name in names:
        assert hasattr(lib, name) and hasattr(ta, name), name


def _means(**kw):
    a = dict(x=M, means=2 * M, B=2, H=2, S=300, d=64, lens=None)
    a.update(kw)
    return lib.block_attn_means(*a.values(), None)


def _lists(**kw):
    a = dict(q=M, kmeans=2 * M, lists=3 * M, B=2, H=4, Hkv=2, Sq=300, Skv=300, d=64, n_list=3, sink=0, local=1,
             causal=1, lens=None)
    a.update(kw)
    return lib.block_attn_lists(*a.values(), None)


def _fwd(**kw):
    a = dict(q=M, k=2 * M, v=3 * M, lists=4 * M, out=5 * M, lse=6 * M, B=2, H=4, Hkv=2, Sq=300, Skv=300, d=64,
             n_list=3, causal=1, lens=None, scale=0.1, ws=16 * M, bytes=1 << 30)
    a.update(kw)
    return lib.block_attn_fwd(*a.values(), None)


def _bwd(**kw):
    a = dict(q=M, k=2 * M, v=3 * M, lists=4 * M, out=5 * M, dout=6 * M, lse=7 * M, dq=8 * M, dk=9 * M, dv=10 * M, B=2,
             H=4, Hkv=2, Sq=300, Skv=300, d=64, n_list=3, causal=1, lens=None, scale=0.1, ws=16 * M, bytes=1 << 30)
    a.update(kw)
    return lib.block_attn_bwd(*a.values(), None)


def _write(**kw):
    a = dict(k=M, v=2 * M, kp=3 * M, vp=4 * M, ks=5 * M, vs=6 * M, table=7 * M, lens=8 * M, n_new=None, B=2, Hkv=2,
             N=3, d=64, max_pages=4, n_pages=8)
    a.update(kw)
    return lib.cache_attn_write(*a.values(), None)


def _cache(**kw):
    a = dict(q=M, kp=2 * M, vp=3 * M, ks=4 * M, vs=5 * M, table=6 * M, lens=7 * M, per_head=0, out=8 * M, lse=9 * M, B=2,
             H=4, Hkv=2, N=3, d=64, max_pages=40, n_pages=8, scale=0.1, ws=16 * M, bytes=1 << 30)
    a.update(kw)
    return lib.cache_attn_fwd(*a.values(), None)


@pytest.mark.parametrize("call,pointers", [
    (_means, "x means"), (_lists, "q kmeans lists"), (_fwd, "q k v lists out"),
    (_bwd, "q k v lists out dout lse dq dk dv"), (_write, "k v kp vp ks vs table lens"),
    (_cache, "q kp vp ks vs table lens out")])
def test_null_pointers(call, pointers):
    for p in pointers.split():
        assert call(**{p: None}) == NULL, p


@pytest.mark.parametrize("call", [_lists, _fwd, _bwd])
def test_shapes_of_block_calls(call):
    for kw in (dict(B=0), dict(H=0), dict(Hkv=0), dict(Hkv=3), dict(Sq=0), dict(Skv=-1), dict(Sq=301), dict(n_list=0),
               dict(Skv=128 * 16384 + 1), dict(n_list=16385), dict(B=1 << 20, H=1 << 10, Hkv=1 << 10)):
        assert call(**kw) == SHAPE, kw
    for d in (0, 32, 80, 256):
        assert call(d=d) == DIM
    assert call(lens=8 * M + 2) == ALIGN


def test_lists_refuse_what_a_list_cannot_hold():
    for kw in (dict(sink=-1), dict(local=-1),
               dict(Sq=2560, Skv=2560, n_list=3, sink=2, local=2),            # 2 + 2 forced
               dict(Sq=2500, Skv=2560, n_list=2, local=2),                    # rows in two blocks, one before
               dict(Sq=2560, Skv=2560, n_list=2, local=2, causal=0)):         # one before, one behind
        assert _lists(**kw) == SHAPE, kw
    assert "forced" in lib.tile_attn_last_error().decode()
    assert _lists(q=M + 8) == ALIGN and _lists(lists=3 * M + 2) == ALIGN
    assert _lists(lists=M + 64) == OVERLAP and _lists(lists=2 * M) == OVERLAP


def test_means_errors():
    assert _means(S=0) == SHAPE and _means(d=65) == DIM and _means(means=2 * M + 2) == ALIGN
    assert _means(means=M + 1024) == OVERLAP and _means(lens=2 * M) == OVERLAP


def test_forward_errors():
    assert _fwd(scale=float("nan")) == SCALE and _fwd(scale=float("inf")) == SCALE
    assert _fwd(v=3 * M + 8) == ALIGN and _fwd(lse=6 * M + 1) == ALIGN and _fwd(lists=4 * M + 2) == ALIGN
    assert _fwd(out=M + 64) == OVERLAP and _fwd(out=4 * M) == OVERLAP and _fwd(lse=5 * M) == OVERLAP
    need = dict(Skv=128 * 64, Sq=1, n_list=32)  # few units: pieces
    n = ta.block_attn_fwd_workspace(2, 4, 2, 1, 128 * 64, 64, 32)
    assert n > 0
    assert _fwd(**need, bytes=n - 1) == SHAPE and "workspace" in lib.tile_attn_last_error().decode()
    assert _fwd(**need, ws=None) == SHAPE and _fwd(**need, ws=16 * M + 8) == ALIGN
    assert _fwd(**need, ws=2 * M) == OVERLAP and _fwd(**need, ws=5 * M - n + 64) == OVERLAP


def test_gradient_errors():
    assert _bwd(scale=float("inf")) == SCALE and _bwd(dq=8 * M + 8) == ALIGN and _bwd(lse=7 * M + 2) == ALIGN
    for kw in (dict(dq=M), dict(dk=2 * M), dict(dv=9 * M + 64), dict(dk=7 * M), dict(dv=6 * M), dict(ws=3 * M)):
        assert _bwd(**kw) == OVERLAP, kw
    n = ta.block_attn_bwd_workspace(2, 4, 2, 300, 300, 64, 3)
    assert _bwd(bytes=n - 1) == SHAPE and _bwd(ws=None) == SHAPE


def test_cache_errors():
    for call in (_write, _cache):
        for kw in (dict(B=0), dict(Hkv=0), dict(N=0), dict(max_pages=0), dict(n_pages=0), dict(max_pages=1 << 24),
                   dict(B=40000)):
            assert call(**kw) == SHAPE, kw
        assert call(d=80) == DIM and call(ks=5 * M + 2) == ALIGN and call(kp=3 * M + 8) == ALIGN
    assert _cache(Hkv=3) == SHAPE and _cache(scale=float("nan")) == SCALE and _cache(out=M) == OVERLAP
    assert _cache(ws=3 * M) == OVERLAP and _cache(lse=8 * M) == OVERLAP and _cache(bytes=16) == SHAPE
    assert _write(kp=4 * M) == OVERLAP and _write(vp=M) == OVERLAP and _write(table=5 * M) == OVERLAP
    assert _write(n_new=8 * M + 2) == ALIGN


def test_workspaces():
    assert ta.block_attn_fwd_workspace(1, 24, 24, 28800, 28800, 96, 32) == 0  # units enough: nothing is cut
    for bad in ((0, 1, 1, 1, 1, 64, 1), (1, 3, 2, 1, 1, 64, 1), (1, 1, 1, 2, 1, 64, 1)):
        for fn in (ta.block_attn_fwd_workspace, ta.block_attn_bwd_workspace):
            with pytest.raises(ta.TileAttnError):
                fn(*bad)
    with pytest.raises(ta.TileAttnError):
        ta.cache_attn_fwd_workspace(1, 3, 2, 1, 64, 1)
    for fn, n in ((lib.block_attn_fwd_workspace, 7), (lib.block_attn_bwd_workspace, 7), (lib.cache_attn_fwd_workspace, 6)):
        assert fn(*([1] * n), ctypes.POINTER(ctypes.c_size_t)()) == NULL


def _piece_bound(B, H, Hkv, Sq, Skv, n_list):
    """The gradient's cutting rule: entries per piece and the slots reserved for pieces."""
    nq, nb = -(-Sq // 128), -(-Skv // 128)
    held, cols, G = B * Hkv * nq * min(n_list, nb), B * Hkv * nb, H // Hkv
    most = max(2 * -(-held // cols), held // 4096)
    least = max((3 + G) // G, -(-held // cols) if 5 * cols >= 1024 else 0)  # at d = 64
    entries = min(most, max(min(most, least), -(-held // 512)))
    pieces = -(-nq // entries)
    return nq, nb, held, cols, entries, 0 if pieces == 1 else min(cols * pieces, 2 * held // entries)


@pytest.mark.parametrize("sizes", [(1, 4, 4, 1000, 1000, 3), (2, 8, 2, 5000, 5000, 40), (1, 1, 1, 128 * 300, 128 * 300, 2),
                                   (1, 16, 1, 40000, 40000, 24), (3, 2, 2, 777, 3000, 9)])
def test_reserved_pieces_hold_the_worst_lists(sizes):
    """No lists need more partial results than the workspace has room for: the worst ones fill as
    many columns as they can just past a multiple of the piece length."""
    nq, nb, held, cols, entries, slots = _piece_bound(*sizes)
    lists = sizes[0] * sizes[2]
    for take in [entries + 1 + m * entries for m in range(0, nq // entries + 1)] + [nq]:
        take = min(take, nq)
        if take <= entries:
            continue
        full = min(cols, held // take, lists * nb)
        assert full * -(-take // entries) <= slots, (take, full)
    n = ta.block_attn_bwd_workspace(*sizes[:5], 64, sizes[5])
    rows = sizes[0] * sizes[1] * sizes[3]
    assert n >= rows * 8 + slots * 2 * 128 * 64 * 4


def _share_items(counts, entries):
    """Items per XCD as the gradient's plan deals them out: contiguous shares of equal work, a column
    counting its query blocks and s, pieces of at most `entries` query blocks."""
    total, cols = int(counts.sum()), len(counts)
    s = max(1, -(-total // (4 * cols)))
    before = np.concatenate([[0], np.cumsum(counts + s)[:-1]])
    xcd = before * 8 // (total + s * cols)
    assert xcd.max() <= 7
    return np.bincount(xcd, np.maximum(1, -(-counts // entries)), 8).astype(int)


@pytest.mark.parametrize("sizes", [(1, 4, 4, 1000, 1000, 3), (2, 8, 2, 5000, 5000, 40), (1, 1, 1, 128 * 300, 128 * 300, 2),
                                   (1, 16, 1, 40000, 40000, 24), (3, 2, 2, 777, 3000, 9), (1, 24, 24, 28800, 28800, 32),
                                   (1, 2, 2, 100, 128 * 2000, 5)])
def test_no_share_of_the_key_side_holds_more_items_than_there_is_room_for(sizes):
    nq, nb, held, cols, entries, slots = _piece_bound(*sizes)
    pieces = -(-nq // entries)
    cap = min(cols * pieces, (5 * cols + 7) // 8 + ((5 * held + 31) // 32 + (cols + 7) // 8 + nq) // entries)
    rng = np.random.default_rng(cols)
    for trial in range(60):
        counts = np.zeros(cols, np.int64)
        left = held if trial % 3 else int(rng.integers(0, held + 1))
        order = {0: np.arange(cols), 1: np.arange(cols)[::-1], 2: rng.permutation(cols)}[trial % 3]
        for c in order:  # few full columns, or many at a piece's edge, or anything
            most = [nq, min(nq, entries + 1), int(rng.integers(0, nq + 1)), 1][trial % 4]
            counts[c] = min(left, most)
            left -= counts[c]
        assert _share_items(counts, entries).max() <= cap, (trial, cap)
        assert (np.where(counts > entries, -(-counts // entries), 0)).sum() <= max(slots, 0)


def test_wrappers_check_tensors_before_any_launch():
    torch = pytest.importorskip("torch")
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    q, k = bf(1, 4, 300, 64), bf(1, 2, 300, 64)
    lists = torch.zeros(1, 2, 3, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        ta.block_attn(q, k, k, lists)
    with pytest.raises(ValueError, match="GPU"):
        ta.block_means(k)
    with pytest.raises(ValueError, match="GPU"):
        ta.block_lists(q, k, 300, 2)
    with pytest.raises(ValueError, match=r"\[B, H, S, d\]"):
        ta.block_attn(q[0], k, k, lists)
    with pytest.raises(ValueError, match="GPU"):
        ta.cache_write(k, k, *([None] * 6))
    with pytest.raises(ValueError, match="GPU"):
        ta.cache_attn(q, *([None] * 6))


def test_header_names_the_limits():
    with open(os.path.join(ROOT, "include", "block_attn.h")) as f:
        hdr = f.read()
    assert "#define TA_BLOCK 128" in hdr and ta.BLOCK_TOKENS == 128
    assert np.log2(128 * 16384) == 21 and "#define TA_MAX_BLOCKS 16384" in hdr


@pytest.mark.parametrize("cols,nq,G,causal", [(1, 1, 1, 0), (3, 2, 4, 1), (8, 300, 1, 0), (128, 32, 4, 1), (512, 128, 4, 1),
                                              (5000, 40, 2, 0), (40, 16384, 1, 1)])
def test_the_line_of_columns_gives_every_query_block_to_one_worker(cols, nq, G, causal):
    """The cut of the gradients' key side at d = 128: even stretches of the line of all columns, pieces
    of a column numbered by their workers, partial sums within the reserved 510."""
    start, least = -(-16 // G) + 4 * causal, 4 * ((3 + G) // G)
    entry = lambda at, n: int(min(max((at - start + 3) >> 2, 0), n))  # noqa: E731
    rng = np.random.default_rng(cols + nq)
    for trial in range(20):
        counts = rng.integers(0, nq + 1, cols) * (rng.random(cols) < [1, 0.5, 0.02, 0][trial % 4])
        total = int(4 * counts.sum() + start * cols)
        workers = max(1, min(256, total // least))
        each, more = divmod(total, workers)
        begin = lambda w: w * each + min(w, more)  # noqa: E731
        worker = lambda x: x // (each + 1) if x < more * (each + 1) else more + (x - more * (each + 1)) // each  # noqa: E731
        at = np.concatenate([[0], np.cumsum(start + 4 * counts)])
        slots, pieces = 0, []
        for c, n in enumerate(counts):
            first = worker(int(at[c]) + (start if n else 0))
            last = worker(int(at[c + 1]) - 4) if n else first
            pieces.append((first, last - first + 1))
            slots += last - first + 1 if last > first else 0
        assert slots <= 510
        seen = [[] for _ in range(cols)]
        starts = [(int(np.searchsorted(at, begin(w), "right")) - 1, 0) for w in range(workers)] + [(cols, 0)]
        starts = [(c, begin(w) - int(at[c])) for w, (c, _) in enumerate(starts[:-1])] + [(cols, 0)]
        for w in range(workers):
            (c0, a0), (c1, a1) = starts[w], starts[w + 1]
            for c in range(c0, min(c1, cols - 1) + 1):
                n, a = int(counts[c]), a0 if c == c0 else 0
                e0, e1 = entry(a, n), entry(a1, n) if c == c1 else n
                if (a != 0 or (c == c1 and a1 == 0)) if n == 0 else e0 >= e1:
                    continue
                assert w - pieces[c][0] == len(seen[c])
                seen[c].append((e0, e1))
        for c, n in enumerate(counts):
            assert len(seen[c]) == pieces[c][1]
            assert seen[c][0][0] == 0 and seen[c][-1][1] == n and all(x[1] == y[0] for x, y in zip(seen[c], seen[c][1:]))


def test_the_workspace_of_cache_attention_stays_small_however_many_tokens():
    for d in (64, 128):
        for G, N in ((4, 1), (4, 5), (4, 40), (1, 300), (4, 512), (4, 2048), (8, 4095), (4, 8192), (1, 32737), (4, 65536),
                     (1, 524280)):
            for B, Hkv in ((1, 1), (1, 8), (7, 4)):
                for pages in (1, 40, 512, 16384):
                    assert ta.cache_attn_fwd_workspace(B, G * Hkv, Hkv, N, d, pages) < 70e6, (G, N, B, pages)
    assert ta.cache_attn_fwd_workspace(1, 32, 8, 1, 128, 512) == 512 * 2 * 16 * 132 * 4   # few rows: as many workgroups
    assert ta.cache_attn_fwd_workspace(1, 32, 8, 32, 128, 512) == 4 * 256 * 2 * 32 * 132 * 4  # as the device holds


def test_a_prompt_of_any_length_may_be_written():
    """Only attention has a limit on its tokens (of a key head's rows); these tensors overlap, which is
    found behind the sizes."""
    assert _write(N=600000, max_pages=5000) == OVERLAP and _write(N=2 ** 31 - 1, max_pages=1 << 23) == OVERLAP
    assert _cache(N=600000, max_pages=5000) == SHAPE and "H / Hkv * N" in lib.tile_attn_last_error().decode()
    with pytest.raises(ta.TileAttnError):
        ta.cache_attn_fwd_workspace(1, 1, 1, 8 * 65535 + 1, 64, 5000)
