"""The 8-bit cache: writing it (codes and scales to the bit) and attention over it, against the
float64 reference. Tolerances as for attention over lists: codes are exact numbers, weights times
the page's scale are rounded to bf16 once, results once (2^-8 of the value each)."""
import numpy as np
import pytest

import workloads
from oracle import blocks as ob
from tests.gpu_helpers import from_dev, to_dev, widen

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2502_06155_amd as ta  # noqa: E402

HALF = 2.0 ** -8
FP32 = 5e-4


def i32(x):
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def bits(rng, *shape):
    return workloads.f32_to_bf16_bits(rng.standard_normal(shape).astype(np.float32))


def new_pages(rng, n, Hkv, d):
    """Pages of any codes, NaN among them, with power-of-two scales: what a cache holds where nobody
    has written."""
    k, v = (rng.integers(0, 256, s).astype(np.uint8) for s in ((n, Hkv, 128, d), (n, Hkv, d, 128)))
    return [k, v, *(2.0 ** rng.integers(-9, -5, (n, Hkv)).astype(np.float32) for _ in range(2))]


def to_gpu(cache):
    codes = [torch.from_numpy(x.copy()).cuda().view(torch.float8_e4m3fn) for x in cache[:2]]
    return codes + [torch.from_numpy(x.copy()).cuda() for x in cache[2:]]


def same(gpu, cache):
    for name, a, b in zip(("k codes", "v codes", "k scales", "v scales"), gpu, cache):
        got = a.view(torch.uint8).cpu().numpy() if a.dtype == torch.float8_e4m3fn else a.cpu().numpy()
        assert np.array_equal(got, b), (name, np.argwhere(got != b)[:4])


def write_both(k, v, cache, gpu, table, lens, n_new=None):
    ob.cache_write(k, v, *cache, np.asarray(table), lens, n_new)
    ta.cache_write(to_dev(k), to_dev(v), *gpu, i32(table), i32(lens), i32(n_new))


@pytest.mark.parametrize("B,Hkv,N,d,lens,n_new", [
    (1, 1, 1, 64, [0], None),
    (2, 2, 1, 128, [127, 128], None),
    (3, 1, 5, 96, [0, 126, 300], [5, 3, 0]),
    (2, 3, 300, 64, [100, 511], None),
    (2, 2, 129, 96, [0, 127], [129, 128]),
    (1, 2, 400, 128, [5], [1000]),
    (2, 1, 3, 64, [-4, 640], None),      # a length below 0 is 0; 640: past the table's pages
    (1, 1, 200, 64, [600], [-1]),
])
def test_write(B, Hkv, N, d, lens, n_new):
    rng = np.random.default_rng(N + d)
    cache = new_pages(rng, 5 * B + 2, Hkv, d)
    for x in cache[:2]:
        x[(x & 127) == 127] = 0  # held tokens are numbers
    gpu = to_gpu(cache)
    table = rng.permutation(5 * B + 2)[:5 * B].reshape(B, 5).astype(np.int32)
    write_both(bits(rng, B, Hkv, N, d), bits(rng, B, Hkv, N, d), cache, gpu, table, lens, n_new)
    same(gpu, cache)


def test_every_finite_bf16_value_and_the_others():
    """All 2^16 bit patterns as tokens of pages of their own magnitude: codes to the bit, scales at
    both ends of their range, infinities at the largest code, NaN kept."""
    b = np.arange(1 << 16, dtype=np.uint32).astype(np.uint16)
    order = np.argsort(b & 0x7FFF, kind="stable")
    k = b[order].reshape(1, 1, 1024, 64)
    cache = new_pages(np.random.default_rng(0), 8, 1, 64)
    gpu = to_gpu(cache)
    table = np.arange(8, dtype=np.int32)[None]
    write_both(k, k[:, :, ::-1].copy(), cache, gpu, table, [0])
    codes = gpu[0].view(torch.uint8).cpu().numpy()
    nan = (codes & 127) == 127
    assert np.array_equal(nan, (cache[0] & 127) == 127)
    assert np.array_equal(np.where(nan, 0, codes), np.where(nan, 0, cache[0]))
    assert np.array_equal(gpu[2].cpu().numpy(), cache[2]) and np.array_equal(gpu[3].cpu().numpy(), cache[3])
    assert cache[2].min() == 2.0 ** -100 and cache[2].max() == 2.0 ** 120


def test_tokens_one_by_one_raise_the_scale_of_their_page():
    """Magnitudes that grow and shrink: old codes move with the scale, down to subnormal ones."""
    rng = np.random.default_rng(2)
    cache = new_pages(rng, 4, 2, 96)
    gpu = to_gpu(cache)
    table = np.array([[2, 0, 1]], np.int32)
    for t in range(140):
        k, v = (workloads.f32_to_bf16_bits((rng.standard_normal((1, 2, 1, 96)) * 2.0 ** rng.integers(-9, 9)).astype(np.float32))
                for _ in range(2))
        write_both(k, v, cache, gpu, table, [t])
    same(gpu, cache)


def test_pages_that_are_none_and_a_written_prefix_at_once():
    rng = np.random.default_rng(3)
    cache = new_pages(rng, 3, 1, 64)
    gpu = to_gpu(cache)
    table = np.array([[0, -1, 2], [3, 1, -2 ** 31]], np.int32)
    write_both(bits(rng, 2, 1, 384, 64), bits(rng, 2, 1, 384, 64), cache, gpu, table, [0, 0])
    same(gpu, cache)


def check(out, lse, q, cache, table, lens, scale=None):
    ref, rlse, mag = ob.cache_attention(q, *cache, np.asarray(table), np.asarray(lens), scale)
    got = widen(from_dev(out))
    assert np.isfinite(got).all()
    off = np.abs(got - ref) - (HALF * np.abs(ref) + (HALF + FP32) * mag + 1e-30)
    assert off.max() <= 0, np.unravel_index(np.argmax(off), off.shape)
    some = np.isfinite(rlse)
    l = lse.cpu().numpy().astype(np.float64)
    assert np.array_equal(l[~some], rlse[~some]) and not from_dev(out)[~some].any()
    assert np.abs(l[some] - rlse[some]).max(initial=0) <= 2e-4


@pytest.mark.parametrize("e", [40, 110])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("H,N,d,pages,width", [(4, 2, 64, 4, 4), (8, 1, 128, 30, 40), (8, 5, 96, 12, 40)])
def test_logits_far_from_zero(H, N, d, pages, width, sign, e):
    """Keys of one value and a scale of 2^e, with one largest logit a row, below zero too: its weight is exactly 1. The
    log-sum-exp: the logit times two factors, rounded each (and their product), in base 2 and back: 2^-21 of it."""
    rng = np.random.default_rng(e + d)
    n = 128 * pages - 3
    k, v, k_scales, v_scales = new_pages(rng, pages, 1, d)
    v[(v & 127) == 127] = 0
    k[...] = 0
    k[..., 0] = rng.choice([0x38, 0x3C, 0x40] if sign > 0 else [0xC0, 0xC8], k.shape[:3])  # 1, 1.5, 2; -2, -4
    k_scales[...] = 2.0 ** e
    table = np.full((1, width), -1, np.int32)
    table[0, :pages] = rng.permutation(pages)
    top = int(rng.integers(0, n - N))
    page, at = table[0, top // 128], top % 128
    k[page, 0, at, 0] = 0x44 if sign > 0 else 0xB8  # 3; -1
    q = np.zeros((1, H, N, d), np.uint16)
    q[..., 0] = 0x3F80
    cache = [k, v, k_scales, v_scales]
    out, lse = ta.cache_attn(to_dev(q), *to_gpu(cache), i32(table), i32([n]), 1.0, return_lse=True)
    logit = (3.0 if sign > 0 else -1.0) * 2.0 ** e
    assert (np.abs(lse.cpu().numpy().astype(np.float64) - logit) <= 2.0 ** -21 * abs(logit)).all()
    row = torch.from_numpy(v[page, 0, :, at].copy()).view(torch.float8_e4m3fn).double().numpy() * float(v_scales[page, 0])
    assert np.array_equal(widen(from_dev(out)), np.broadcast_to(row, (1, H, N, d)))


def held(rng, B, Hkv, d, lens, width=None, spare=2):
    """A cache whose sequences hold lens tokens; everything behind them is any code."""
    need = [-(-x // 128) for x in lens]
    width = max(1, max(need)) if width is None else width
    cache = new_pages(rng, sum(need) + spare, Hkv, d)
    perm = rng.permutation(sum(need) + spare)
    table = np.full((B, width), -1, np.int32)
    at = 0
    for b in range(B):
        table[b, :need[b]] = perm[at:at + need[b]]
        at += need[b]
        for i in range(need[b]):
            n = min(128, lens[b] - 128 * i)
            p = table[b, i]
            for x in (cache[0][p, :, :n], cache[1][p, :, :, :n]):
                x[(x & 127) == 127] = 5
    return cache, table


@pytest.mark.parametrize("B,H,Hkv,N,d,lens", [
    (1, 1, 1, 1, 64, [1]),
    (2, 2, 1, 1, 96, [0, 63]),
    (3, 4, 2, 1, 128, [64, 65, 127]),
    (3, 8, 1, 1, 64, [128, 129, 1000]),
    (2, 3, 3, 4, 96, [2, 700]),       # fewer tokens than rows: some rows see none
    (2, 16, 2, 2, 128, [193, 3000]),
    (2, 20, 1, 1, 64, [500, 77]),     # more than 16 rows
    (1, 16, 1, 5, 96, [900]),         # 80 rows: three passes
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
    got, lse = ta.cache_attn(to_dev(q), *to_gpu(cache), i32(table), i32(lens), scale, out, return_lse=True)
    assert got is out
    check(got, lse, q, cache, table, lens, scale)


def test_many_short_sequences_and_one_long():
    """More segments than a wave scans at once, and one that most workgroups share."""
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.integers(0, 200, 150)]
    lens[77] = 20000
    cache, table = held(rng, 150, 2, 64, lens)
    q = bits(rng, 150, 4, 1, 64)
    out, lse = ta.cache_attn(to_dev(q), *to_gpu(cache), i32(table), i32(lens), return_lse=True)
    check(out, lse, q, cache, table, lens)


def test_lengths_past_the_table_and_pages_that_are_none():
    rng = np.random.default_rng(6)
    cache, table = held(rng, 2, 2, 96, [512, 512])
    table[0, 1], table[1, 3], table[1, 0] = -1, 99, -2 ** 31
    q, lens = bits(rng, 2, 4, 1, 96), [2 ** 31 - 1, 512]
    out, lse = ta.cache_attn(to_dev(q), *to_gpu(cache), i32(table), i32(lens), return_lse=True)
    check(out, lse, q, cache, table, lens)
    none = np.full_like(table, -1)
    out, lse = ta.cache_attn(to_dev(q), *to_gpu(cache), i32(none), i32([512, 3]), return_lse=True)
    assert not from_dev(out).any() and torch.isneginf(lse).all()


def test_scales_of_any_kind():
    rng = np.random.default_rng(7)
    cache, table = held(rng, 1, 1, 64, [400])
    cache[2] = rng.uniform(-0.01, 0.01, cache[2].shape).astype(np.float32)
    cache[3] = rng.uniform(-2, 2, cache[3].shape).astype(np.float32)
    q = bits(rng, 1, 2, 1, 64)
    out, lse = ta.cache_attn(to_dev(q), *to_gpu(cache), i32(table), i32([400]), return_lse=True)
    check(out, lse, q, cache, table, [400])


def _generate(B, H, Hkv, d, prompt, steps, seed, sink=1, local=1, n=3):
    """A program that generates: the prompt into the cache, then token after token: its keys and
    values written, the pages of the best blocks chosen for each key head, attention over those."""
    rng = np.random.default_rng(seed)
    total = max(prompt) + steps
    width = -(-total // 128)
    k, v, q = (bits(rng, B, x, total, d) for x in (Hkv, Hkv, H))
    cache = new_pages(rng, B * width, Hkv, d)
    table = rng.permutation(B * width).reshape(B, width).astype(np.int32)
    return dict(k=k, v=v, q=q, cache=cache, table=table, prompt=prompt, steps=steps, n=n, sink=sink, local=local)


def test_generating_with_chosen_pages():
    B, H, Hkv, d, prompt = 2, 4, 2, 64, [700, 513]
    g = _generate(B, H, Hkv, d, prompt, 3, 11)
    gpu, table = to_gpu(g["cache"]), i32(g["table"])
    lens = i32([0, 0])
    first = max(prompt)
    ta.cache_write(to_dev(g["k"][:, :, :first]), to_dev(g["v"][:, :, :first]), *gpu, table, lens, i32(prompt))
    ob.cache_write(g["k"][:, :, :first], g["v"][:, :, :first], *g["cache"], g["table"], [0, 0], prompt)
    same(gpu, g["cache"])
    keys = np.zeros((B, Hkv, first + 3, d), np.uint16)  # what the program keeps block means of
    for b in range(B):
        keys[b, :, :prompt[b]] = g["k"][b, :, :prompt[b]]
    for step in range(3):
        held_now = [p + step for p in prompt]
        now = [g[x][np.arange(B), :, held_now][:, :, None].copy() for x in "kvq"]
        ta.cache_write(to_dev(now[0]), to_dev(now[1]), *gpu, table, i32(held_now))
        ob.cache_write(now[0], now[1], *g["cache"], g["table"], held_now)
        same(gpu, g["cache"])
        pages = np.full((B, Hkv, 3), -1, np.int32)
        lens_h = np.zeros((B, Hkv), np.int32)
        for b in range(B):  # one sequence a call: their positions differ
            keys[b, :, held_now[b]] = now[0][b, :, 0]
            S = held_now[b] + 1
            kb = keys[b:b + 1, :, :S].copy()
            lists = ta.block_lists(to_dev(now[2][b:b + 1]), ta.block_means(to_dev(kb)), S, 3, True, 1, 1).cpu().numpy()
            assert np.array_equal(lists, ob.block_lists(now[2][b:b + 1], ob.block_means(kb), S, 3, True, 1, 1))
            for h in range(Hkv):
                chosen = [j for j in lists[0, h, 0] if j >= 0]
                pages[b, h, :len(chosen)] = g["table"][b][chosen]
                lens_h[b, h] = 128 * (len(chosen) - 1) + S - 128 * chosen[-1]
        out, lse = ta.cache_attn(to_dev(now[2]), *gpu, i32(pages), i32(lens_h), return_lse=True)
        check(out, lse, now[2], g["cache"], pages, lens_h)
        # attention over the lists on the cache's numbers says the same
        values = ob.e4m3_values()
        whole, wl = ta.cache_attn(to_dev(now[2]), *gpu, table, i32([x + 1 for x in held_now]), return_lse=True)
        check(whole, wl, now[2], g["cache"], g["table"], [x + 1 for x in held_now])
        assert not np.isnan(values[g["cache"][0][g["table"][0, 0]]]).any()


def test_captured_write_and_attention_replayed():
    """Writing and reading in one graph, lengths moved on between the replays by the program."""
    rng = np.random.default_rng(12)
    B, H, Hkv, d = 3, 6, 2, 128
    start = [126, 5, 400]
    cache, table = held(rng, B, Hkv, d, start, width=5, spare=12)
    free = [p for p in range(len(cache[0])) if p not in table]
    for b in range(B):
        for i in range(5):
            if table[b, i] < 0 and free:
                table[b, i] = free.pop()
    gpu, t = to_gpu(cache), i32(table)
    lens = i32(start)
    k, v, q = (torch.zeros(B, x, 1, d, dtype=torch.bfloat16, device="cuda") for x in (Hkv, Hkv, H))

    def step():
        ta.cache_write(k, v, *gpu, t, lens)
        after = lens + 1
        return ta.cache_attn(q, *gpu, t, after, return_lse=True)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out, lse = step()
    for i in range(5):
        x = [bits(rng, B, h, 1, d) for h in (Hkv, Hkv, H)]
        for a, b in zip((k, v, q), x):
            a.copy_(to_dev(b))
        at = [s + i for s in start]
        lens.copy_(i32(at))
        graph.replay()
        ob.cache_write(x[0], x[1], *cache, table, at)
        torch.cuda.synchronize()
        same(gpu, cache)
        check(out, lse, x[2], cache, table, [y + 1 for y in at])
        eager = ta.cache_attn(q, *gpu, t, lens + 1, return_lse=True)
        assert torch.equal(eager[0], out) and torch.equal(eager[1], lse)


def test_offsets_past_32_bits():
    """A cache of more than 2^32 bytes a tensor: pages at its far end."""
    d, Hkv = 128, 8
    n = 2 ** 32 // (Hkv * 128 * d) + 40
    kp = torch.zeros((n, Hkv, 128, d), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    vp = torch.zeros((n, Hkv, d, 128), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    ks, vs = torch.ones((n, Hkv), device="cuda"), torch.ones((n, Hkv), device="cuda")
    rng = np.random.default_rng(13)
    k, v, q = bits(rng, 1, Hkv, 300, d), bits(rng, 1, Hkv, 300, d), bits(rng, 1, Hkv, 1, d)
    table = np.array([[n - 1, 3, n - 7]], np.int32)
    ta.cache_write(to_dev(k), to_dev(v), kp, vp, ks, vs, i32(table), i32([0]))
    out, lse = ta.cache_attn(to_dev(q), kp, vp, ks, vs, i32(table), i32([300]), return_lse=True)
    small = [np.zeros((3, Hkv, 128, d), np.uint8), np.zeros((3, Hkv, d, 128), np.uint8),
             np.ones((3, Hkv), np.float32), np.ones((3, Hkv), np.float32)]
    near = np.array([[0, 1, 2]], np.int32)
    ob.cache_write(k, v, *small, near, [0])
    for i, page in enumerate(table[0]):
        assert np.array_equal(kp[page].view(torch.uint8).cpu().numpy(), small[0][i])
        assert np.array_equal(vp[page].view(torch.uint8).cpu().numpy(), small[1][i])
    check(out, lse, q, small, near, [300])


def test_wrappers_refuse():
    rng = np.random.default_rng(1)
    cache, table = held(rng, 1, 2, 64, [200])
    gpu, t, lens = to_gpu(cache), i32(table), i32([200])
    q = torch.zeros(1, 4, 1, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(1, 2, 1, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="k_pages"):
        ta.cache_attn(q, gpu[0].view(torch.uint8), *gpu[1:], t, lens)
    with pytest.raises(ValueError, match="v_pages"):
        ta.cache_attn(q, gpu[0], gpu[0], *gpu[2:], t, lens)
    with pytest.raises(ValueError, match="lens"):
        ta.cache_attn(q, *gpu, t[:, None].expand(1, 2, 2).contiguous(), lens)
    with pytest.raises(ValueError, match="table"):
        ta.cache_attn(q, *gpu, t.long(), lens)
    with pytest.raises(ValueError, match="k must"):
        ta.cache_write(k[:, :1], k, *gpu, t, lens)
    with pytest.raises(ta.TileAttnError, match="overlap"):
        ta.cache_attn(q[:, :, :, :], *gpu, t, lens, out=q)


@pytest.mark.parametrize("width", [3, 40])
@pytest.mark.parametrize("d", [64, 96, 128])
def test_a_later_token_that_is_no_number_leaves_earlier_rows(d, width):
    """NaN keys and values in the last two of five new tokens: the three rows before keep their bits,
    the others are NaN in the dims of the values."""
    rng = np.random.default_rng(d + width)
    cache, table = held(rng, 1, 2, d, [300], width)
    q = bits(rng, 1, 6, 5, d)
    p, at = table[0, 2], 298 - 256
    clean = [x.copy() for x in cache]
    clean[1][p, :, 9, at:at + 2] = 0
    cache[1][p, 0, 9, at], cache[1][p, 0, 9, at + 1] = 127, 255
    cache[1][p, 1, 9, at] = 255
    run = lambda c: ta.cache_attn(to_dev(q), *to_gpu(c), i32(table), i32([300]), return_lse=True)  # noqa: E731
    (got, lse), (ref, rlse) = run(cache), run(clean)
    assert torch.equal(lse, rlse)
    want = ref.clone()
    want[:, :, 3:, 9] = float("nan")
    assert np.array_equal(got.float().cpu().numpy(), want.float().cpu().numpy(), equal_nan=True)
    cache[0][p, :, at, 4] = 127  # now a key: the rows that see it are NaN, and so is their sum
    got, lse = run(cache)
    assert torch.equal(got[:, :, :3], ref[:, :, :3]) and torch.equal(lse[:, :, :3], rlse[:, :, :3])
    assert got[:, :, 3:].isnan().all() and lse[:, :, 3:].isnan().all()


@pytest.mark.parametrize("B,H,Hkv,N,d,lens,width", [
    (1, 8, 2, 40, 128, [3000], 40),             # five passes of 32 rows, each a share of the workgroups
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
    got, lse = ta.cache_attn(to_dev(q), *to_gpu(cache), i32(table), i32(lens), None, out, return_lse=True)
    check(got, lse, q, cache, table, lens)
    again = ta.cache_attn(to_dev(q), *to_gpu(cache), i32(table), i32(lens))
    assert torch.equal(got, again)
    assert N < 1030 or ta.cache_attn_fwd_workspace(B, H, Hkv, N, d, width) == 0


def test_a_long_prompt_written_at_once():
    """More tokens than attention takes rows, into a table a little too short for them: the same codes
    as in two calls."""
    N, d, pages = 540000, 64, 4200
    gen = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn((1, 1, N, d), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    table = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)[None]
    got = []
    for cuts in ((0, N), (0, 128 * 2000, N)):
        cache = [torch.zeros((pages, 1, *s), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for s in ((128, d), (d, 128))]
        cache += [torch.zeros((pages, 1), device="cuda") for _ in range(2)]
        for a, b in zip(cuts, cuts[1:]):
            ta.cache_write(k[:, :, a:b].contiguous(), v[:, :, a:b].contiguous(), *cache, table, i32([a]))
        got.append([x.view(torch.uint8) for x in cache])
    assert all(torch.equal(a, b) for a, b in zip(*got))
    last = int(table[0, -1])
    want = k[0, 0, 128 * (pages - 1):128 * pages].float()
    codes = got[0][0][last, 0].view(torch.float8_e4m3fn).float() * got[0][2].view(torch.float32)[last, 0]
    assert ((codes - want).abs() <= 2.0 ** -4 * want.abs() + 2.0 ** -16).all()


@pytest.mark.parametrize("B,H,Hkv,N,d,width,most", [
    (1, 4, 4, 1, 64, 40, 40),
    (3, 8, 2, 1, 128, 40, 23),
    (2, 12, 3, 4, 96, 33, 33),
    (2, 40, 2, 2, 128, 20, 20),    # 40 rows a key head: two passes
    (40, 6, 3, 1, 64, 20, 20),     # more segments than a wave scans at once
    (1, 8, 2, 70, 64, 40, 30),     # nine passes that share the workgroups
])
def test_a_page_table_for_each_key_head_on_the_shared_line(B, H, Hkv, N, d, width, most):
    """Tables longer than a workgroup takes alone, with lengths of every kind per key head: none, within
    the first page, full pages, past the table; some entries name no page."""
    rng = np.random.default_rng(width + H)
    n_pages = 4 * width
    cache = new_pages(rng, n_pages, Hkv, d)
    for x in cache[:2]:
        x[(x & 127) == 127] = 3
    table = np.stack([rng.permutation(n_pages)[:width] for _ in range(B * Hkv)]).reshape(B, Hkv, width).astype(np.int32)
    table[rng.random(table.shape) < 0.05] = -1
    table[rng.random(table.shape) < 0.02] = n_pages
    lens = rng.integers(N, 128 * most + 1, (B, Hkv)).astype(np.int32)
    lens.flat[rng.permutation(B * Hkv)[:max(1, B * Hkv // 4)]] = rng.choice([0, 1, 128, 128 * width, 2 ** 31 - 1])
    lens.flat[0] = 128 * most
    assert ta.cache_attn_fwd_workspace(B, H, Hkv, N, d, width) > 0
    q = bits(rng, B, H, N, d)
    out = torch.full((B, H, N, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    got, lse = ta.cache_attn(to_dev(q), *to_gpu(cache), i32(table), i32(lens), None, out, return_lse=True)
    check(got, lse, q, cache, table, lens)


def test_pages_chosen_for_each_key_head_of_a_long_sequence():
    """The lists of a token as page tables of more than 16 pages, made on the device and captured with
    the attention: replayed for other queries, the same as over the lists on the numbers the pages hold."""
    rng = np.random.default_rng(41)
    H, Hkv, d, S, n = 8, 2, 128, 128 * 60 - 37, 24
    nb = -(-S // 128)
    cache, table = held(rng, 1, Hkv, d, [S])
    gpu, t = to_gpu(cache), i32(table)
    values = ob.e4m3_values()
    keys = np.zeros((1, Hkv, S, d))
    for i in range(nb):
        m = min(128, S - 128 * i)
        for h in range(Hkv):
            keys[0, h, 128 * i:128 * i + m] = values[cache[0][table[0, i], h, :m]] * cache[2][table[0, i], h]
    kb = ob.to_bf16(keys)
    assert np.array_equal(ob.widen(kb), keys)
    km = ta.block_means(to_dev(kb))
    q = to_dev(bits(rng, 1, H, 1, d))

    def step():
        lists = ta.block_lists(q, km, S, n, True, 1, 2)[:, :, 0]       # ascending, the last block last
        pages = t[0][lists.clamp(min=0).long()].to(torch.int32)
        lens = (torch.full_like(pages[..., 0], n * 128 - (128 * nb - S)))
        return lists, *ta.cache_attn(q, *gpu, pages, lens, return_lse=True)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lists, out, lse = step()
    for _ in range(3):
        x = bits(rng, 1, H, 1, d)
        q.copy_(to_dev(x))
        graph.replay()
        torch.cuda.synchronize()
        want = ob.block_lists(x, ob.block_means(kb), S, n, True, 1, 2)
        assert np.array_equal(lists.cpu().numpy(), want[:, :, 0])
        check(out, lse, x, cache, table[0][want[:, :, 0]], np.full((1, Hkv), n * 128 - (128 * nb - S)))
        eager = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, (lists, out, lse)))


def test_attention_that_autograd_does_not_record_says_so():
    rng = np.random.default_rng(1)
    cache, table = held(rng, 1, 2, 64, [200])
    q = to_dev(bits(rng, 1, 4, 1, 64))
    ref = ta.cache_attn(q, *to_gpu(cache), i32(table), i32([200]))
    with pytest.warns(UserWarning, match="no gradient"):
        out = ta.cache_attn(q.clone().requires_grad_(), *to_gpu(cache), i32(table), i32([200]))
    assert torch.equal(out, ref) and not out.requires_grad
