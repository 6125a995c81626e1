"""The 4-bit cache: writing it and reading it back (to the bit), and attention over it, against the float64 reference.

Tolerances of attention. K and V become bf16 exactly. A logit is a sum of up to 128 products in fp32: off by at most
128 * 2^-24 of sum |q k| * scale, below 60 here: ROOM, which is also the log-sum-exp's. Weights are rounded to bf16
once (2^-8 of p |v|) and so are results (2^-8 of the value)."""
import numpy as np
import pytest

import workloads
from oracle import blocks as ob
from oracle import cache4 as o4
from oracle import heads as oh
from tests.gpu_helpers import from_dev, to_dev, widen

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2502_06155_amd as ta  # noqa: E402

HALF = 2.0 ** -8
ROOM = 5e-4


def i32(x):
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def bits(rng, *shape):
    return workloads.f32_to_bf16_bits(rng.standard_normal(shape).astype(np.float32))


def any_bytes(rng, n, Hkv, d):
    """Pages of any bytes, scales of NaN among them: what a cache holds where nobody has written."""
    return [rng.integers(0, 256, s).astype(np.uint8)
            for s in ((n, Hkv, 128, d // 2),) * 2 + ((n, Hkv, d // 32, 128),) * 2]


def to_gpu(cache):
    return [torch.from_numpy(x.copy()).cuda() for x in cache]


def same(gpu, cache):
    for name, a, b in zip(("k codes", "v codes", "k scales", "v scales"), gpu, cache):
        got = a.cpu().numpy()
        assert np.array_equal(got, b), (name, np.argwhere(got != b)[:4])


def write_both(k, v, cache, gpu, table, lens, n_new=None):
    want = o4.write(k, v, *cache, np.asarray(table), lens, n_new)
    got = ta.cache4_write(to_dev(k), to_dev(v), *gpu, i32(table), i32(lens), i32(n_new), return_held=True)
    for a, b in zip(got, want):
        assert np.array_equal(widen(from_dev(a)), b, equal_nan=True)


@pytest.mark.parametrize("B,Hkv,N,d,lens,n_new", [
    (1, 1, 1, 64, [0], None),
    (2, 2, 1, 128, [127, 128], None),
    (3, 1, 5, 96, [0, 126, 300], [5, 3, 0]),
    (2, 3, 300, 64, [100, 511], None),
    (2, 2, 129, 96, [0, 127], [129, 128]),
    (1, 2, 400, 128, [5], [1000]),
    (2, 1, 3, 64, [-4, 640], None),      # a length below 0 is 0; 640: past the table's pages
    (1, 1, 200, 64, [600], [-1]),
    (1, 1, 3, 96, [2 ** 31 - 1], None),
])
def test_write(B, Hkv, N, d, lens, n_new):
    rng = np.random.default_rng(N + d)
    cache = any_bytes(rng, 5 * B + 2, Hkv, d)
    gpu = to_gpu(cache)
    table = rng.permutation(5 * B + 2)[:5 * B].reshape(B, 5).astype(np.int32)
    k, v = bits(rng, B, Hkv, N, d), bits(rng, B, Hkv, N, d)
    write_both(k, v, cache, gpu, table, lens, n_new)
    same(gpu, cache)
    assert ta.cache4_write(to_dev(k), to_dev(v), *gpu, i32(table), i32(lens), i32(n_new)) is None
    same(gpu, cache)


def test_every_bf16_value():
    """All 2^16 bit patterns among tokens of their own magnitude and of any: codes and scales to the bit, at both
    ends of the scales' range; tokens with infinities or NaN are marked."""
    b = np.arange(1 << 16, dtype=np.uint32).astype(np.uint16)
    k = b[np.argsort(b & 0x7FFF, kind="stable")].reshape(1, 1, 1024, 64)
    v = np.random.default_rng(1).permutation(b[(b & 0x7F80) != 0x7F80]).reshape(1, 1, -1, 64)[:, :, :1016]
    v = np.concatenate([v, k[:, :, :8]], 2)
    cache = any_bytes(np.random.default_rng(0), 8, 1, 64)
    gpu = to_gpu(cache)
    write_both(k, v, cache, gpu, np.arange(8, dtype=np.int32)[None], [0])
    same(gpu, cache)
    assert cache[3].max() == 125 + 127 and cache[2].min() == 27 and (cache[2] == 255).any()


@pytest.mark.parametrize("bad", [0x7F80, 0xFF80, 0x7FC0, 0xFFFF])
@pytest.mark.parametrize("d", [64, 96, 128])
def test_a_token_that_is_no_number_is_marked_and_no_other(bad, d):
    rng = np.random.default_rng(d)
    k, v = bits(rng, 2, 2, 40, d), bits(rng, 2, 2, 40, d)
    k[0, 1, 3, 0], k[1, 0, 17, d - 1], v[0, 0, 4, 33], v[1, 1, 39, 1] = bad, bad, bad, bad
    cache = any_bytes(rng, 3, 2, d)
    gpu, table = to_gpu(cache), np.array([[2], [0]], np.int32)
    write_both(k, v, cache, gpu, table, [3, 88])
    same(gpu, cache)
    back = [widen(from_dev(x)) for x in ta.cache4_read(*gpu, i32(table), i32([43, 128]), 128)]
    nan = np.isnan(back[0]).all(-1)
    assert {tuple(int(y) for y in x) for x in np.argwhere(nan)} == {(0, 1, 6), (1, 0, 105), (0, 0, 7), (1, 1, 127)} | {
        tuple(int(y) for y in x) for x in np.argwhere(nan) if x[0] == 1 and x[2] < 88}


def test_tokens_one_by_one_are_tokens_at_once():
    rng = np.random.default_rng(2)
    k, v = bits(rng, 2, 2, 140, 96), bits(rng, 2, 2, 140, 96)
    cache = any_bytes(rng, 4, 2, 96)
    one, all_ = to_gpu(cache), to_gpu(cache)
    table = i32([[2, 0], [1, 3]])
    for t in range(140):
        ta.cache4_write(to_dev(k[:, :, t:t + 1].copy()), to_dev(v[:, :, t:t + 1].copy()), *one, table, i32([t, t]))
    ta.cache4_write(to_dev(k), to_dev(v), *all_, table, i32([0, 0]))
    for a, b in zip(one, all_):
        assert torch.equal(a, b)


def test_pages_that_are_none():
    rng = np.random.default_rng(3)
    cache = any_bytes(rng, 3, 1, 64)
    gpu, table = to_gpu(cache), np.array([[0, -1, 2], [3, 1, -2 ** 31]], np.int32)
    write_both(bits(rng, 2, 1, 384, 64), bits(rng, 2, 1, 384, 64), cache, gpu, table, [0, 0])
    same(gpu, cache)


@pytest.mark.parametrize("B,Hkv,N,d,lens,first", [
    (1, 1, 1, 64, [1], 0), (1, 1, 1, 64, [0], 0), (2, 3, 300, 96, [300, 131], 0), (2, 2, 77, 128, [400, 130], 100),
    (1, 2, 129, 64, [-3], 5), (2, 1, 700, 96, [2 ** 31 - 1, 640], 17), (1, 1, 5, 128, [640], 2 ** 31 - 6)])
def test_read(B, Hkv, N, d, lens, first):
    rng = np.random.default_rng(N + d)
    cache = any_bytes(rng, 5 * B + 2, Hkv, d)
    for s in cache[2:]:  # finite bf16 numbers, and NaN
        s[...] = np.where(s > 252, 255, s)
    table = rng.permutation(5 * B + 2)[:5 * B].reshape(B, 5).astype(np.int32)
    table[0, 3] = -1
    table[-1, 2] = 5 * B + 2
    got = ta.cache4_read(*to_gpu(cache), i32(table), i32(lens), N, first)
    want = o4.read(*cache, table, lens, N, first) if first < 10000 else np.zeros((2, B, Hkv, N, d))
    for a, b in zip(got, want):
        assert np.array_equal(widen(from_dev(a)), b, equal_nan=True)


def held(rng, B, Hkv, d, lens, width=None, spare=2):
    """A cache whose sequences hold lens tokens; everything behind them is any byte."""
    need = [-(-x // 128) for x in lens]
    width = max(1, max(need)) if width is None else width
    cache = any_bytes(rng, sum(need) + spare, Hkv, d)
    perm = rng.permutation(sum(need) + spare)
    table = np.full((B, width), -1, np.int32)
    at = 0
    for b in range(B):
        table[b, :need[b]] = perm[at:at + need[b]]
        at += need[b]
        for i in range(need[b]):
            n = min(128, lens[b] - 128 * i)
            for s in cache[2:]:
                s[table[b, i], :, :, :n] = rng.integers(124, 128, s[table[b, i], :, :, :n].shape)
    return cache, table


def check(out, lse, q, cache, table, lens, scale=None):
    ref, rlse, mag = o4.attention(q, *cache, np.asarray(table), np.asarray(lens), scale)
    got, l = widen(from_dev(out)), lse.cpu().numpy().astype(np.float64)
    nan = np.isnan(rlse)
    assert np.isnan(got[nan]).all() and np.isnan(l[nan]).all() and np.isfinite(got[~nan]).all()
    off = (np.abs(got - ref) - (HALF * np.abs(ref) + (HALF + ROOM) * mag + 1e-30))[~nan]
    assert off.max(initial=-1) <= 0, off.max()
    some = np.isfinite(rlse)
    assert np.array_equal(l[~some], rlse[~some], equal_nan=True) and not got[np.isneginf(rlse)].any()
    assert np.abs(l[some] - rlse[some]).max(initial=0) <= ROOM


@pytest.mark.parametrize("B,H,Hkv,N,d,lens", [
    (1, 1, 1, 1, 64, [1]),
    (2, 2, 1, 1, 96, [0, 63]),
    (3, 4, 2, 1, 128, [64, 65, 127]),
    (3, 8, 1, 1, 64, [128, 129, 1000]),
    (2, 3, 3, 4, 96, [2, 700]),       # fewer tokens than rows: some rows see none
    (2, 16, 2, 2, 128, [193, 3000]),
    (2, 20, 1, 1, 64, [500, 77]),     # more than 16 rows
    (1, 9, 1, 3, 96, [2900]),         # 27 rows
    (2, 8, 1, 4, 128, [1500, 66]),    # 32 rows, a last page of which the second half is empty
    (1, 16, 1, 5, 96, [900]),         # 80 rows: one pass of 128
    (2, 34, 2, 3, 128, [130, 257]),
    (20, 6, 3, 1, 64, [0, 5, 0, 0, 300, 128, 0, 1, 640, 2, 0, 256, 7, 0, 90, 0, 0, 1280, 3, 0]),
])
@pytest.mark.parametrize("scale,width", [(None, None), (None, 40), (-0.2, 40), (0.0, None)])
def test_attention(B, H, Hkv, N, d, lens, scale, width):
    """Tables as short as the sequences (a workgroup a segment, where they are short enough) and tables
    of 40 pages (work shared evenly and joined)."""
    rng = np.random.default_rng(sum(lens) + d)
    cache, table = held(rng, B, Hkv, d, lens, width)
    q = bits(rng, B, H, N, d)
    out = torch.full((B, H, N, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    got, lse = ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(table), i32(lens), scale, out, return_lse=True)
    assert got is out
    check(got, lse, q, cache, table, lens, scale)


def test_many_short_sequences_and_one_long():
    """More segments than a wave scans at once, and one that most workgroups share."""
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.integers(0, 200, 150)]
    lens[77] = 20000
    cache, table = held(rng, 150, 2, 64, lens)
    q = bits(rng, 150, 4, 1, 64)
    out, lse = ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(table), i32(lens), return_lse=True)
    check(out, lse, q, cache, table, lens)


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("B,pages,H,N", [(32, 12, 4, 2), (40, 7, 2, 1), (150, 9, 4, 1), (130, 24, 2, 1)])
def test_short_tables_of_many_sequences(B, pages, H, N, d):
    """Workgroups of eight and of four waves with a segment each; lengths of none to full tables, a marked token."""
    rng = np.random.default_rng(B + d)
    lens = [int(x) for x in rng.integers(0, 128 * pages + 1, B)]
    lens[0], lens[1], lens[2] = 128 * pages, 0, 128 * pages - 1
    cache, table = held(rng, B, 2, d, lens)
    cache[2][table[2, pages - 1], 1, 0, 126] = 255
    q = bits(rng, B, H, N, d)
    assert ta.cache4_attn_fwd_workspace(B, H, 2, N, d, pages) == 0
    out, lse = ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(table), i32(lens), return_lse=True)
    some = [0, 1, 2, 3, B // 2, B - 2, B - 1]  # (the reference is slow)
    check(out[some], lse[some], q[some], cache, table[some], [lens[b] for b in some])
    shared = np.concatenate([table, np.full((B, 60), -1, np.int32)], 1)
    other, l2 = ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(shared), i32(lens), return_lse=True)
    assert ta.cache4_attn_fwd_workspace(B, H, 2, N, d, pages + 60) > 0
    ok = ~torch.isnan(out)
    assert torch.equal(ok, ~torch.isnan(other)) and torch.allclose(out[ok].float(), other[ok].float(), rtol=0.02, atol=0.02)
    assert torch.allclose(lse.nan_to_num(7.0), l2.nan_to_num(7.0), rtol=0, atol=2 * ROOM)


def test_lengths_past_the_table_and_pages_that_are_none():
    rng = np.random.default_rng(6)
    cache, table = held(rng, 2, 2, 96, [512, 512])
    table[0, 1], table[1, 3], table[1, 0] = -1, 99, -2 ** 31
    q, lens = bits(rng, 2, 4, 1, 96), [2 ** 31 - 1, 512]
    out, lse = ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(table), i32(lens), return_lse=True)
    check(out, lse, q, cache, table, lens)
    none = np.full_like(table, -1)
    out, lse = ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(none), i32([512, 3]), return_lse=True)
    assert not from_dev(out).any() and torch.isneginf(lse).all()


@pytest.mark.parametrize("d", [64, 96, 128])
def test_scales_of_any_magnitude(d):
    """Groups of a token far apart in magnitude, at both ends of a scale's range where the row's others are 0."""
    rng = np.random.default_rng(d)
    cache, table = held(rng, 1, 2, d, [200])
    cache[2][...] = rng.integers(115, 127, cache[2].shape)
    cache[3][...] = rng.integers(60, 200, cache[3].shape)
    q = bits(rng, 1, 4, 1, d)
    out, lse = ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(table), i32([200]), return_lse=True)
    check(out, lse, q, cache, table, [200])
    cache[3][...] = rng.choice([0, 1, 252], cache[3].shape)
    cache[1][...] = rng.choice([0, 1, 0x10, 0x91], cache[1].shape)  # 0.5 at most: sums stay finite
    out, lse = ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(table), i32([200]), return_lse=True)
    check(out, lse, q, cache, table, [200])


@pytest.mark.parametrize("e", [31, 60, 122])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("B,H,Hkv,N,d,pages,width", [
    (1, 4, 2, 2, 64, 6, 6), (2, 8, 2, 1, 128, 30, 40),    # up to 16 rows: a workgroup a segment, and shared
    (1, 8, 1, 3, 96, 9, 40),                              # 24 rows: half a page at a time
    (1, 6, 1, 8, 96, 6, 6), (1, 4, 2, 45, 128, 20, 40)])  # 48 rows a workgroup a segment, 90 shared
def test_logits_far_from_zero(B, H, Hkv, N, d, pages, width, sign, e):
    """Keys of one value, times 2^e, and queries that take it as it is: every row has one largest logit (all of them may
    be far below zero), and its weight is exactly 1. The log-sum-exp is the logit in base 2 (two roundings) in base e
    (one of the factor, one of the product): 2^-22 of it."""
    rng = np.random.default_rng(e + d)
    n = 128 * pages - 3
    cache, table = held(rng, B, Hkv, d, [n] * B, width)
    cache[0][...] = 0
    cache[0][..., 0] = rng.choice([2, 3, 4, 5] if sign > 0 else [12, 13, 14, 15], cache[0].shape[:3])  # 1 to 3; -2 to -6
    cache[2][:, :, 0] = e + 127
    top = rng.integers(0, n - N, (B, Hkv))
    for b in range(B):
        for h in range(Hkv):
            page, at = table[b, top[b, h] // 128], top[b, h] % 128
            cache[0][page, h, at, 0] = 6 if sign > 0 else 10  # 4; -1
    q = np.zeros((B, H, N, d), np.uint16)
    q[..., 0] = 0x3F80
    out, lse = ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(table), i32([n] * B), 1.0, return_lse=True)
    logit = (4.0 if sign > 0 else -1.0) * 2.0 ** e
    assert (np.abs(lse.cpu().numpy().astype(np.float64) - logit) <= 2.0 ** -22 * abs(logit)).all()
    for b in range(B):
        for h in range(H):
            g = h * Hkv // H
            page, at = table[b, top[b, g] // 128], top[b, g] % 128
            v = o4.values(cache[1][page, g, at:at + 1], cache[3][page, g, :, at:at + 1])[0]
            assert np.array_equal(widen(from_dev(out[b, h])), np.broadcast_to(v, (N, d)))


@pytest.mark.parametrize("H,Hkv,N,d,pages,width", [(4, 1, 2, 64, 6, 6), (8, 1, 3, 96, 20, 40), (4, 1, 30, 128, 20, 40)])
def test_rows_far_from_zero_leave_others_as_they_were(H, Hkv, N, d, pages, width):
    """A query of large numbers, and one of infinities, beside others in the same wave: theirs keep every bit, with logits of
    some 3e5, whose products' rounding would show."""
    rng = np.random.default_rng(d)
    n = 128 * pages - 9
    cache, table = held(rng, 1, Hkv, d, [n], width)
    cache[0][..., :16] = 0
    cache[0][..., 0], cache[2][:, :, 0] = 2, 20 + 127  # every key's first value is 2^20
    q = bits(rng, 1, H, N, d)
    q[..., 0] = 0x3F80
    gpu = to_gpu(cache)
    want, l0 = ta.cache4_attn(to_dev(q), *gpu, i32(table), i32([n]), 0.3, return_lse=True)
    far = q.copy()
    far[0, 1, 0] = workloads.f32_to_bf16_bits((widen(q[0, 1, 0]) * 2.0 ** 90).astype(np.float32))
    far[0, 2, N - 1, ::2] = 0x7F80
    got, l1 = ta.cache4_attn(to_dev(far), *gpu, i32(table), i32([n]), 0.3, return_lse=True)
    same_rows = torch.ones(1, H, N, dtype=torch.bool, device="cuda")
    same_rows[0, 1, 0] = same_rows[0, 2, N - 1] = False
    assert torch.equal(got[same_rows], want[same_rows]) and torch.equal(l1[same_rows], l0[same_rows])
    assert torch.isfinite(got[0, 1, 0]).all() and not torch.equal(got[0, 1, 0], want[0, 1, 0])


@pytest.mark.parametrize("width", [3, 40])
@pytest.mark.parametrize("d", [64, 96, 128])
def test_marked_tokens_reach_the_rows_that_see_them_alone(d, width):
    rng = np.random.default_rng(d + width)
    cache, table = held(rng, 1, 2, d, [300], width)
    q = bits(rng, 1, 6, 5, d)
    clean = ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(table), i32([300]), return_lse=True)
    at = 298 - 256
    cache[2][table[0, 2], 0, :, at] = 255
    got, lse = ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(table), i32([300]), return_lse=True)
    check(got, lse, q, cache, table, [300])
    assert torch.equal(got[:, :, :3], clean[0][:, :, :3]) and torch.equal(got[:, 3:], clean[0][:, 3:])
    assert got[:, :3, 3:].isnan().all() and lse[:, :3, 3:].isnan().all()


@pytest.mark.parametrize("width", [4, 40])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("N", [7, 20, 40])  # 21 rows a key head: half a page at a time; 60 and 120: a page's tokens shared by two waves
def test_marked_tokens_among_many_rows(N, d, width):
    rng = np.random.default_rng(N + d + width)
    cache, table = held(rng, 1, 3, d, [400], width)
    cache[2][table[0, 3], 0, :, 398 - 384] = 255  # the last but one: two rows see it
    cache[2][table[0, 0], 2, :, 100] = 255        # in the second half of the first page: every row
    q = bits(rng, 1, 9, N, d)
    got, lse = ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(table), i32([400]), return_lse=True)
    check(got, lse, q, cache, table, [400])
    assert got[:, :3, N - 2:].isnan().all() and not got[:, :6, :N - 2].isnan().any() and got[:, 6:].isnan().all()


@pytest.mark.parametrize("B,H,Hkv,N,d,lens,width", [
    (1, 8, 2, 40, 128, [3000], 40),             # 160 rows: two passes, each a share of the workgroups
    (2, 8, 2, 300, 64, [900, 333], 40),         # as many tokens as one sequence holds, fewer than the other's
    (1, 4, 4, 257, 96, [257], None),            # short tables: a workgroup a segment and pass
    (3, 8, 1, 129, 128, [128, 0, 2100], 40),    # rows before a sequence's start, and none at all
    (1, 40, 1, 500, 64, [700], 20),             # two workgroups a pass
    (2, 32, 1, 1030, 64, [1030, 5], 20),        # more passes than workgroups: one a pass, no workspace
])
def test_chunks_of_a_prompt(B, H, Hkv, N, d, lens, width):
    rng = np.random.default_rng(N + d)
    cache, table = held(rng, B, Hkv, d, lens, width)
    q = bits(rng, B, H, N, d)
    out = torch.full((B, H, N, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    got, lse = ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(table), i32(lens), None, out, return_lse=True)
    check(got, lse, q, cache, table, lens)
    assert torch.equal(got, ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(table), i32(lens)))


def stretch(B, H, Hkv, N, d, width):
    """Pages on the line of all sequences (each segment with the five that its start counts as) for a workgroup, if all
    tables were full: workspaces hold two partial results of every workgroup's rows."""
    rows = H // Hkv * N
    per = 16 if rows <= 16 else 32 if rows <= 32 else 64 if rows <= 64 else 128
    workers = ta.cache4_attn_fwd_workspace(B, H, Hkv, N, d, width) // (2 * per * (d + 4) * 4 * -(-rows // per))
    return B * Hkv * (width + 5) / workers


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("N", [1, 3, 6, 12])  # 8, 24, 48 and 96 rows a key head: each of the kernels' ways through a page
def test_long_stretches_of_pages(N, d):
    """Workgroups that go through many pages of a sequence: 16 sequences of 40 to 130 pages, the last ones in part, pages that
    are none among them, and tokens that are marked in a late page, for all rows and for the last ones."""
    B, H, Hkv, width = 16, 32, 4, 130
    rng = np.random.default_rng(N + d)
    lens = [int(x) for x in rng.integers(40 * 128, width * 128, B)]
    lens[0], lens[5], lens[9] = 128 * 47 + 1, 128 * 61 - 1, 128 * 44 + 70
    cache, table = held(rng, B, Hkv, d, lens, width)
    assert stretch(B, H, Hkv, N, d, width) > 12
    cache[2][table[5, 57], 1, :, 3] = 255                # (key head 1)
    cache[2][table[9, 44], 2, :, 70 - min(N, 2)] = 255   # the last tokens'
    table[0, 9], table[0, 10], table[0, 33], table[5, 20], table[9, 0] = -1, -1, len(cache[0]), -2 ** 31, -1
    q = bits(rng, B, H, N, d)
    out, lse = ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(table), i32(lens), return_lse=True)
    some = [0, 5, 9]  # (the reference is slow)
    check(out[some], lse[some], q[some], cache, table[some], [lens[b] for b in some])
    bad = torch.isnan(lse)
    assert bad[5, 8:16].all() and bad[9, 16:24, -1].all() and bad.sum() == 8 * N + 8 * min(N, 2)


@pytest.mark.parametrize("H,Hkv,N,d", [(16, 2, 640, 128), (16, 2, 640, 96), (12, 1, 300, 64), (24, 4, 200, 128)])
def test_long_stretches_under_many_passes(H, Hkv, N, d):
    """Prompts of thousands of rows a key head, so that few workgroups share a pass and each goes through many pages, with pages
    that are none in between and a marked token that the last rows see."""
    width, n = 70, 128 * 55 + 77
    rng = np.random.default_rng(N + d)
    cache, table = held(rng, 1, Hkv, d, [n], width)
    assert stretch(1, H, Hkv, N, d, width) > 8
    table[0, 3], table[0, 17], table[0, 18], table[0, 40] = -1, len(cache[0]), -1, -2 ** 31
    cache[2][table[0, 55], 0, :, 77 - 5] = 255
    q = bits(rng, 1, H, N, d)
    out, lse = ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(table), i32([n]), return_lse=True)
    check(out, lse, q, cache, table, [n])
    assert torch.isnan(lse).sum() == 5 * H // Hkv


@pytest.mark.parametrize("B,H,Hkv,N,d,width,most", [
    (1, 4, 4, 1, 64, 40, 40),
    (3, 8, 2, 1, 128, 40, 23),
    (2, 12, 3, 4, 96, 33, 33),
    (2, 40, 2, 2, 128, 20, 20),    # 40 rows a key head
    (40, 6, 3, 1, 64, 20, 20),     # more segments than a wave scans at once
    (1, 8, 2, 70, 64, 40, 30),     # three passes that share the workgroups
    (2, 8, 2, 1, 96, 5, 5),        # short tables
])
def test_a_page_table_for_each_key_head(B, H, Hkv, N, d, width, most):
    """Lengths of every kind per key head: none, within the first page, full pages, past the table; some entries
    name no page."""
    rng = np.random.default_rng(width + H)
    n_pages = 4 * width
    cache = any_bytes(rng, n_pages, Hkv, d)
    for s in cache[2:]:
        s[...] = rng.integers(124, 128, s.shape)
    table = np.stack([rng.permutation(n_pages)[:width] for _ in range(B * Hkv)]).reshape(B, Hkv, width).astype(np.int32)
    table[rng.random(table.shape) < 0.05] = -1
    table[rng.random(table.shape) < 0.02] = n_pages
    lens = rng.integers(N, 128 * most + 1, (B, Hkv)).astype(np.int32)
    lens.flat[rng.permutation(B * Hkv)[:max(1, B * Hkv // 4)]] = rng.choice([0, 1, 128, 128 * width, 2 ** 31 - 1])
    lens.flat[0] = 128 * most
    q = bits(rng, B, H, N, d)
    out = torch.full((B, H, N, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    got, lse = ta.cache4_attn(to_dev(q), *to_gpu(cache), i32(table), i32(lens), None, out, return_lse=True)
    check(got, lse, q, cache, table, lens)


def test_a_decoding_step_captured_and_replayed():
    """Norms and rotation of a token, its key and value into the cache, attention over it: in one graph, lengths
    and positions moved on between replays by the program, every replay against the eager calls and the reference."""
    rng = np.random.default_rng(12)
    B, H, Hkv, d, start = 3, 6, 2, 128, [126, 5, 400]
    cache, table = held(rng, B, Hkv, d, start, width=5, spare=12)
    free = [p for p in range(len(cache[0])) if p not in table]
    for b in range(B):
        for i in range(5):
            if table[b, i] < 0 and free:
                table[b, i] = free.pop()
    gpu, t, lens = to_gpu(cache), i32(table), i32(start)
    freqs, w = ta.rope_freqs((d,)), 1 + 0.2 * torch.randn(d, device="cuda")
    x = torch.zeros(B, 1, H + 2 * Hkv, d, dtype=torch.bfloat16, device="cuda")

    def step():
        q, k, v = ta.head_rope(x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:], positions=lens.view(B, 1, 1),
                               freqs=freqs, layout="halves", norm="rms", q_weight=w, k_weight=w)
        ta.cache4_write(k, v, *gpu, t, lens)
        return q, k, v, *ta.cache4_attn(q, *gpu, t, lens + 1, return_lse=True)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step()
    for i in range(5):
        xb = bits(rng, B, 1, H + 2 * Hkv, d)
        x.copy_(to_dev(xb))
        at = [s + i for s in start]
        lens.copy_(i32(at))
        graph.replay()
        torch.cuda.synchronize()
        q, k, v, out, lse = got
        ref = oh.forward(widen(xb)[:, :, :H + Hkv], "rms", w.cpu().numpy(), positions=np.array(at).reshape(B, 1, 1),
                         freqs=freqs.cpu().numpy(), dims=(d,), layout="halves")
        turned = np.concatenate([widen(from_dev(q)), widen(from_dev(k))], 1)
        assert (np.abs(turned - ref) <= HALF * np.abs(ref) + 2.0 ** -12).all()
        o4.write(from_dev(k), from_dev(v), *cache, table, at)
        same(gpu, cache)
        check(out, lse, from_dev(q), cache, table, [y + 1 for y in at])
        eager = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, got))


@pytest.mark.parametrize("d", [64, 128])
def test_a_prompt_attends_to_what_the_cache_holds(d):
    """A prompt in two chunks: the first into the cache with its held values for its own attention; the second reads
    the prefix back. Attention over the cache says the same as attention over the lists of all blocks."""
    rng = np.random.default_rng(d)
    H, Hkv, S, cut = 4, 2, 300, 170
    k, v, q = (bits(rng, 1, h, S, d) for h in (Hkv, Hkv, H))
    cache = any_bytes(rng, 4, Hkv, d)
    gpu, table = to_gpu(cache), i32([[3, 0, 1]])
    part = lambda x, a, b: to_dev(x[:, :, a:b].copy())  # noqa: E731

    def attend(x, keys, values):
        n = -(-x.shape[2] // 128)
        nb = -(-keys.shape[2] // 128)
        lists = torch.arange(nb, dtype=torch.int32, device="cuda").expand(1, Hkv, n, nb).contiguous()
        return ta.block_attn(x, keys, values, lists, causal=True, return_lse=True)

    held_k, held_v = ta.cache4_write(part(k, 0, cut), part(v, 0, cut), *gpu, table, i32([0]), return_held=True)
    outs = [attend(part(q, 0, cut), held_k, held_v)]
    ta.cache4_write(part(k, cut, S), part(v, cut, S), *gpu, table, i32([cut]))
    every = ta.cache4_read(*gpu, table, i32([S]), S)
    assert torch.equal(every[0][:, :, :cut], held_k) and torch.equal(every[1][:, :, :cut], held_v)
    outs.append(attend(part(q, cut, S), *every))
    cache = [x.cpu().numpy() for x in gpu]
    for (out, lse), a, b in zip(outs, (0, cut), (cut, S)):
        check(out, lse, from_dev(part(q, a, b)), cache, np.array([[3, 0, 1]]), [b])
        got, gl = ta.cache4_attn(part(q, a, b), *gpu, table, i32([b]), return_lse=True)
        check(got, gl, from_dev(part(q, a, b)), cache, np.array([[3, 0, 1]]), [b])


def test_two_graphs_at_once_and_another_stream():
    rng = np.random.default_rng(8)
    cache, table = held(rng, 2, 2, 128, [5000, 3000])
    gpu, t, lens = to_gpu(cache), i32(table), i32([5000, 3000])
    q = [to_dev(bits(rng, 2, 8, 1, 128)) for _ in range(2)]
    want = [ta.cache4_attn(x, *gpu, t, lens, return_lse=True) for x in q]
    graphs, outs = [], []
    for x in q:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(ta.cache4_attn(x, *gpu, t, lens, return_lse=True))
        graphs.append(g)
    side = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
            mine = ta.cache4_attn(q[0], *gpu, t, lens)
        torch.cuda.synchronize()
        assert torch.equal(mine, want[0][0])
        for a, b in zip(outs, want):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_offsets_past_32_bits():
    """A cache of more than 2^32 bytes a tensor: pages at its far end."""
    d, Hkv = 128, 8
    n = 2 ** 32 // (Hkv * 128 * d // 2) + 40
    gpu = ta.cache4_new(n, Hkv, d)
    rng = np.random.default_rng(13)
    k, v, q = bits(rng, 1, Hkv, 300, d), bits(rng, 1, Hkv, 300, d), bits(rng, 1, Hkv, 1, d)
    table = np.array([[n - 1, 3, n - 7]], np.int32)
    ta.cache4_write(to_dev(k), to_dev(v), *gpu, i32(table), i32([0]))
    out, lse = ta.cache4_attn(to_dev(q), *gpu, i32(table), i32([300]), return_lse=True)
    small = any_bytes(rng, 3, Hkv, d)
    near = np.array([[0, 1, 2]], np.int32)
    want = o4.write(k, v, *small, near, [0])
    for a, b in zip(ta.cache4_read(*gpu, i32(table), i32([300]), 300), want):
        assert np.array_equal(widen(from_dev(a)), b)
    check(out, lse, q, small, near, [300])


@pytest.mark.parametrize("first", [2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 64, -2 ** 32])
def test_a_first_token_past_a_c_int_is_refused(first):
    cache, table = held(np.random.default_rng(1), 1, 1, 64, [200])
    with pytest.raises(ValueError, match="first"):
        ta.cache4_read(*to_gpu(cache), i32(table), i32([200]), 3, first=first)


def test_a_long_prompt_written_at_once():
    """Into a table a little too short for it: the same bytes as in two calls, and back."""
    N, d, pages = 540000, 64, 4200
    gen = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn((1, 1, N, d), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    table = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)[None]
    got = []
    for cuts in ((0, N), (0, 128 * 2000 + 5, N)):
        cache = ta.cache4_new(pages, 1, d)
        for a, b in zip(cuts, cuts[1:]):
            kept = ta.cache4_write(k[:, :, a:b].contiguous(), v[:, :, a:b].contiguous(), *cache, table, i32([a]), return_held=True)
        got.append(cache)
    assert all(torch.equal(a, b) for a, b in zip(*got))
    back = ta.cache4_read(*got[0], table, i32([N]), N)
    for x, y, z in zip((k, v), back, kept):
        assert not y[:, :, 128 * pages:].any() and torch.equal(y[:, :, b - z.shape[2]:], z)
        off = (x - y).float()[:, :, :128 * pages].view(-1, 32).abs()
        top = x.float()[:, :, :128 * pages].reshape(-1, 32).abs().amax(1, keepdim=True)
        assert (off <= top * (2 / 7)).all()  # at most 2^e, and the largest is above 3.5 * 2^e


def test_the_functions_of_the_c_abi():
    rng = np.random.default_rng(4)
    cache, table = held(rng, 2, 2, 96, [5000, 300], spare=3)
    gpu, t, lens = to_gpu(cache), i32(table), i32([5000, 299])
    k, v, q = (to_dev(bits(rng, 2, h, 1, 96)) for h in (2, 2, 6))
    pages, width, stream = len(cache[0]), table.shape[1], torch.cuda.current_stream()
    mine = [x.clone() for x in gpu]
    want = ta.cache4_write(k, v, *mine, t, i32([-5, 299]), return_held=True)
    got = [torch.empty_like(k), torch.empty_like(k)]
    ta.cache4_attn_write(k, v, *gpu, t, i32([-5, 299]), None, *got, 2, 2, 1, 96, width, pages, stream)
    assert all(torch.equal(a, b) for a, b in zip((*mine, *want), (*gpu, *got)))
    ta.cache4_attn_read(*gpu, t, lens + 1, None, got[1], 2, 2, 1, 96, width, pages, 299, stream)
    assert torch.equal(got[1], ta.cache4_read(*gpu, t, lens + 1, 1, first=299)[1])
    out, lse = torch.empty_like(q), torch.empty(2, 6, 1, device="cuda")
    n = ta.cache4_attn_fwd_workspace(2, 6, 2, 1, 96, width)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")  # (NaN)
    ta.cache4_attn_fwd(q, *gpu, t, lens, False, out, lse, 2, 6, 2, 1, 96, width, pages, 0.1, ws, n, stream)
    a, b = ta.cache4_attn(q, *gpu, t, lens, 0.1, return_lse=True)
    assert n > 0 and torch.equal(a, out) and torch.equal(b, lse)


def test_wrappers_refuse():
    rng = np.random.default_rng(1)
    cache, table = held(rng, 1, 2, 64, [200])
    gpu, t, lens = to_gpu(cache), i32(table), i32([200])
    q = torch.zeros(1, 4, 1, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(1, 2, 1, 64, dtype=torch.bfloat16, device="cuda")
    for match, call in (
            ("k_pages must be torch.uint8", lambda: ta.cache4_attn(q, gpu[0].view(torch.int8), *gpu[1:], t, lens)),
            ("v_pages must have", lambda: ta.cache4_attn(q, gpu[0], gpu[1][:-1], *gpu[2:], t, lens)),
            ("k_scales must have", lambda: ta.cache4_attn(q, *gpu[:2], gpu[2][:, :, :1].contiguous(), gpu[3], t, lens)),
            ("q must have", lambda: ta.cache4_attn(q[..., :32].contiguous(), *gpu, t, lens)),
            ("lens must", lambda: ta.cache4_attn(q, *gpu, t[:, None].expand(1, 2, 2).contiguous(), lens)),
            ("table must", lambda: ta.cache4_attn(q, *gpu, t.long(), lens)),
            ("k must have", lambda: ta.cache4_write(k[:, :1], k, *gpu, t, lens)),
            ("v must be", lambda: ta.cache4_write(k, k.half(), *gpu, t, lens)),
            ("n_new must", lambda: ta.cache4_write(k, k, *gpu, t, lens, n_new=t)),
            ("table must be", lambda: ta.cache4_read(*gpu, t[0], lens, 3)),
            ("lens must", lambda: ta.cache4_read(*gpu, t, lens.long(), 3)),
            ("N must", lambda: ta.cache4_read(*gpu, t, lens, 0))):
        with pytest.raises(ValueError, match=match):
            call()
    with pytest.raises(ta.TileAttnError, match="overlap"):
        ta.cache4_attn(q, *gpu, t, lens, out=q)
    with pytest.raises(ta.TileAttnError, match="first"):
        ta.cache4_read(*gpu, t, lens, 3, first=-1)
    with pytest.warns(UserWarning, match="no gradient"):
        ta.cache4_attn(q.clone().requires_grad_(), *gpu, t, lens)
