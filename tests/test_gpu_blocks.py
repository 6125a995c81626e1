"""Block means, lists, attention over lists and its gradients against the float64 reference.

Tolerances count roundings (half a step of bf16 is 2^-8 of the value): weights and dS are rounded to
bf16 once before their second product and results once more; scores are fp32 sums of up to 128
exact products, whose error (below 128 * 2^-24 of the sum of their magnitudes, about 1e-4 in the
exponent at these sizes, twice that where the log-sum-exp enters as well) changes weights by less
than 5e-4."""
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
NAN = 0x7FC1


def bits(rng, *shape, scale=1.0):
    return workloads.f32_to_bf16_bits((scale * rng.standard_normal(shape)).astype(np.float32))


def i32(x):
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def within(got, ref, bound, what):
    off = np.abs(got - ref) - bound
    assert np.isfinite(got).all(), what
    worst = np.unravel_index(np.argmax(off), off.shape)
    print(f"[parity] {what}: error {np.abs(got - ref).max():.2e}, at the worst {got[worst]:.5g} for {ref[worst]:.5g}, "
          f"bound {bound[worst]:.2e}", flush=True)
    assert off[worst] <= 0, what


def some_lists(rng, B, Hkv, Sq, Skv, n, kind="random"):
    """Lists in any order, with gaps, repeats and entries that name no block; "near": every query
    block's own block among them; "empty": none at all for every second query block."""
    nq, nb = -(-Sq // 128), -(-Skv // 128)
    x = rng.integers(0, nb, (B, Hkv, nq, n)).astype(np.int32)
    x[rng.random(x.shape) < 0.2] = -1
    x[rng.random(x.shape) < 0.05] = nb + 3
    x[rng.random(x.shape) < 0.03] = 2 ** 31 - 1
    x[rng.random(x.shape) < 0.03] = -2 ** 31
    if kind == "near":
        x[..., n // 2] = (Skv - Sq + 128 * np.arange(nq)) // 128
    if kind == "empty":
        x[:, :, ::2] = -1
    return x


# B, H, Hkv, Sq, Skv, d, n, causal, lens, kind
CASES = [
    (1, 1, 1, 1, 1, 64, 1, True, None, "near"),
    (1, 2, 1, 127, 127, 96, 1, False, None, "near"),
    (1, 2, 2, 128, 128, 128, 2, True, None, "near"),
    (2, 2, 1, 129, 129, 64, 3, True, [129, 128], "near"),
    (2, 4, 2, 300, 300, 96, 3, True, [300, 0], "near"),
    (1, 3, 1, 333, 333, 128, 2, False, None, "empty"),
    (3, 2, 2, 257, 257, 64, 4, False, [257, 1, 200], "random"),
    (1, 4, 1, 200, 777, 128, 5, True, None, "random"),
    (2, 6, 2, 1, 700, 96, 6, True, [700, 650], "random"),
    (2, 8, 1, 3, 900, 64, 9, False, None, "random"),
    (1, 2, 2, 150, 650, 96, 4, True, [600], "near"),
    (1, 5, 1, 40, 300, 128, 3, True, None, "random"),
    (1, 1, 1, 640, 640, 64, 40, True, None, "random"),
    (1, 48, 2, 700, 700, 128, 6, True, [650], "near"),  # the key side by stretches of a line, columns cut often
    (2, 26, 1, 900, 900, 128, 8, False, [900, 300], "empty"),
    (1, 36, 1, 300, 1500, 128, 20, True, None, "random"),
    (2, 2, 1, 1000, 1000, 64, 1100, True, [1000, 555], "random"),  # long lists of repeats: a launch of its own plans
]
IDS = ["-".join(str(x) for x in c[:7]) + ("-causal" if c[7] else "") + ("-" + c[9]) for c in CASES]


def make(case, seed=0):
    B, H, Hkv, Sq, Skv, d, n, causal, lens, kind = case
    rng = np.random.default_rng(1000 + seed + sum(case[:7]))
    q, k, v, go = bits(rng, B, H, Sq, d), bits(rng, B, Hkv, Skv, d), bits(rng, B, Hkv, Skv, d), bits(rng, B, H, Sq, d)
    if lens is not None:  # what lies behind the end counts for nobody
        for b, ln in enumerate(lens):
            k[b, :, ln:] = NAN
            v[b, :, ln:] = NAN
            q[b, :, max(0, ln - (Skv - Sq)):] = NAN
            go[b, :, max(0, ln - (Skv - Sq)):] = NAN
    return q, k, v, go, some_lists(rng, B, Hkv, Sq, Skv, n, kind)


def zero_nan(x):
    return np.where(x == NAN, np.uint16(0), x)


@pytest.mark.parametrize("case", CASES, ids=IDS)
@pytest.mark.parametrize("scale", [None, -0.3, 0.0])
def test_forward_and_gradients(case, scale):
    B, H, Hkv, Sq, Skv, d, n, causal, lens, kind = case
    q, k, v, go, lists = make(case)
    qd, kd, vd, gd = (to_dev(x) for x in (q, k, v, go))
    out = torch.full_like(qd, float("nan"))
    got, lse = ta.block_attn(qd, kd, vd, i32(lists), causal, scale, i32(lens), out, return_lse=True)
    assert got is out
    plain = [zero_nan(x) for x in (q, k, v, go)]
    ref, rlse, mag = ob.attention(*plain[:3], lists, causal, lens, scale)
    within(widen(from_dev(got)), ref, HALF * np.abs(ref) + (HALF + FP32) * mag + 1e-30, "out")
    some = np.isfinite(rlse)
    lse_h = lse.cpu().numpy().astype(np.float64)
    assert np.array_equal(lse_h[~some], rlse[~some])
    assert np.abs(lse_h[some] - rlse[some]).max(initial=0) <= 2e-4
    assert not from_dev(got)[~some].any()

    grads = ta.block_attn_grad(qd, kd, vd, i32(lists), got, gd, lse, causal, scale, i32(lens))
    dq, dk, dv = ob.attention_backward(*plain, lists, causal, lens, scale)
    for name, g, r in zip(("dq", "dk"), grads, (dq, dk)):
        bound = HALF * np.abs(r[0]) + HALF * r[1] + FP32 * r[2] + r[3] + 1e-30
        within(widen(from_dev(g)), r[0], bound, name)
    within(widen(from_dev(grads[2])), dv[0], HALF * np.abs(dv[0]) + (HALF + FP32) * dv[1] + 1e-30, "dv")


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_enough_units_for_whole_lists_and_cut_columns(d, causal):
    """As many units as the device holds (lists are not cut), grouped heads, a block that every
    query block keeps and an odd length; rows of some heads against the reference, gradients of one
    group."""
    B, H, Hkv, S, n = 2, 32, 8, 1300, 5
    assert ta.block_attn_fwd_workspace(B, H, Hkv, S, S, d, n) == 0
    rng = np.random.default_rng(d + causal)
    q, k, v, go = (bits(rng, B, h, S, d) for h in (H, Hkv, Hkv, H))
    lists = some_lists(rng, B, Hkv, S, S, n, "near")
    lists[..., 0] = 0
    qd, kd, vd, gd = (to_dev(x) for x in (q, k, v, go))
    out, lse = ta.block_attn(qd, kd, vd, i32(lists), causal, return_lse=True)
    grads = ta.block_attn_grad(qd, kd, vd, i32(lists), out, gd, lse, causal)
    for b, g in ((0, 0), (1, Hkv - 1), (1, 3)):
        hs = slice(4 * g, 4 * g + 4)
        part = (q[b:b + 1, hs], k[b:b + 1, g:g + 1], v[b:b + 1, g:g + 1])
        ref, rlse, mag = ob.attention(*part, lists[b:b + 1, g:g + 1], causal)
        within(widen(from_dev(out[b:b + 1, hs])), ref, HALF * np.abs(ref) + (HALF + FP32) * mag + 1e-30, f"out {b} {g}")
        some = np.isfinite(rlse)
        got = lse[b:b + 1, hs].cpu().numpy()
        assert np.abs(got[some] - rlse[some]).max() <= 2e-4 and np.array_equal(got[~some], rlse[~some].astype(np.float32))
        dq, dk, dv = ob.attention_backward(*part, go[b:b + 1, hs], lists[b:b + 1, g:g + 1], causal)
        for name, x, r in (("dq", grads[0][b:b + 1, hs], dq), ("dk", grads[1][b:b + 1, g:g + 1], dk)):
            bound = HALF * np.abs(r[0]) + HALF * r[1] + FP32 * r[2] + r[3] + 1e-30
            within(widen(from_dev(x)), r[0], bound, f"{name} {b} {g}")
        within(widen(from_dev(grads[2][b:b + 1, g:g + 1])), dv[0], HALF * np.abs(dv[0]) + (HALF + FP32) * dv[1] + 1e-30,
               f"dv {b} {g}")


def test_order_and_repeats_of_a_list_change_no_bit():
    case = (2, 4, 2, 700, 700, 64, 6, True, [700, 555], "near")
    q, k, v, go, lists = make(case)
    q, k, v, go = (zero_nan(x) for x in (q, k, v, go))
    args = [to_dev(x) for x in (q, k, v)]
    lens = i32(case[8])
    rng = np.random.default_rng(5)
    longer = np.concatenate([lists, lists[..., ::-1], lists[..., :2]], -1)
    ref = None
    for x in (lists, rng.permuted(lists, axis=-1), longer):
        out, lse = ta.block_attn(*args, i32(x), True, lens=lens, return_lse=True)
        grads = ta.block_attn_grad(*args, i32(x), out, to_dev(go), lse, True, lens=lens)
        if x is not longer:
            got = [out, lse, *grads]
            if ref is not None:
                assert all(torch.equal(a, b) for a, b in zip(got, ref))
            ref = got
        else:  # a longer list may be cut into other pieces
            right, _, mag = ob.attention(q, k, v, lists, True, case[8])
            within(widen(from_dev(out)), right, HALF * np.abs(right) + (HALF + FP32) * mag + 1e-30, "repeats")


def test_blocks_outside_the_lists_and_later_keys_are_never_used():
    """NaN keys and values in unlisted blocks, and NaN keys behind a row, change nothing."""
    rng = np.random.default_rng(8)
    q, k, v, go = (bits(rng, 1, h, 512, 96) for h in (2, 1, 1, 2))
    lists = np.array([[[[0, -1], [1, 0], [0, 2], [3, 0]]]], np.int32)
    kn, vn = k.copy(), v.copy()
    lists[0, 0, 3] = [0, -1]  # nobody keeps block 3
    kn[:, :, 384:] = NAN
    vn[:, :, 384:] = NAN
    q2 = q.copy()
    out = [ta.block_attn(to_dev(q2), to_dev(a), to_dev(b), i32(lists), True, return_lse=True) for a, b in ((k, v), (kn, vn))]
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    grads = [ta.block_attn_grad(to_dev(q2), to_dev(a), to_dev(b), i32(lists), *o[:1], to_dev(go), o[1], True)
             for (a, b), o in zip(((k, v), (kn, vn)), out)]
    assert all(torch.equal(a, b) for a, b in zip(*grads))
    assert not from_dev(grads[0][1])[:, :, 384:].any() and not from_dev(grads[0][2])[:, :, 384:].any()
    late = k.copy()
    late[:, :, 120:] = NAN  # rows before 120 of the first block mask them
    first = ta.block_attn(to_dev(q2), to_dev(late), to_dev(v), i32(lists), True)
    assert torch.equal(first[:, :, :120], out[0][0][:, :, :120])


def test_large_logits():
    rng = np.random.default_rng(9)
    q, k, v = bits(rng, 1, 2, 300, 64, scale=8.0), bits(rng, 1, 2, 300, 64, scale=8.0), bits(rng, 1, 2, 300, 64)
    lists = np.array([[[[2, 0], [1, 2], [0, 1]]] * 2], np.int32)
    out, lse = ta.block_attn(*(to_dev(x) for x in (q, k, v)), i32(lists), return_lse=True)
    ref, rlse, mag = ob.attention(q, k, v, lists)
    # scores up to some 300: fp32 sums of 64 products and the base-2 logarithm's scaling are off by
    # at most 66 * 2^-24 of the products' magnitudes (about 400 here), 1.6e-3, in the exponent
    within(widen(from_dev(out)), ref, HALF * np.abs(ref) + (HALF + 4e-3) * mag + 1e-30, "out")
    assert np.abs(lse.cpu().numpy() - rlse).max() <= 2e-3


@pytest.mark.parametrize("B,H,S,d,lens", [(1, 1, 1, 64, None), (2, 3, 129, 96, [129, 7]), (1, 2, 1000, 128, None),
                                          (3, 1, 384, 64, [0, 384, 257])])
def test_means(B, H, S, d, lens):
    rng = np.random.default_rng(S)
    x = bits(rng, B, H, S, d)
    if lens:
        for b, ln in enumerate(lens):
            x[b, :, ln:] = NAN
    got = ta.block_means(to_dev(x), i32(lens))
    assert np.array_equal(from_dev(got), ob.block_means(zero_nan(x), lens))


@pytest.mark.parametrize("B,H,Hkv,Sq,Skv,d,n,causal,sink,local,lens", [
    (1, 1, 1, 1, 1, 64, 1, False, 0, 0, None),
    (2, 4, 2, 300, 300, 64, 2, True, 0, 1, [300, 200]),
    (1, 6, 2, 1500, 1500, 96, 4, False, 1, 1, None),
    (1, 2, 1, 1500, 1500, 128, 6, False, 1, 2, None),
    (2, 2, 2, 1, 5000, 128, 9, True, 1, 2, [5000, 4990]),
    (1, 2, 2, 700, 1000, 64, 5, True, 1, 2, None),
    (1, 2, 2, 600, 1000, 64, 50, False, 0, 0, [900]),
    (1, 1, 1, 90, 128 * 1100, 64, 33, True, 0, 1, None),
    (1, 1, 1, 130, 128 * 4500, 64, 200, False, 2, 1, None),
    (1, 1, 1, 1, 128 * 16384, 64, 64, True, 0, 0, None),
])
def test_lists(B, H, Hkv, Sq, Skv, d, n, causal, sink, local, lens):
    rng = np.random.default_rng(Sq + Skv)
    nb = -(-Skv // 128)
    q, km = bits(rng, B, H, Sq, d), bits(rng, B, Hkv, nb, d)
    if lens:
        for b, ln in enumerate(lens):
            q[b, :, max(0, ln - (Skv - Sq)):] = NAN
    out = torch.full((B, Hkv, -(-Sq // 128), n), 77, dtype=torch.int32, device="cuda")
    got = ta.block_lists(to_dev(q), to_dev(km), Skv, n, causal, sink, local, i32(lens), out)
    assert got is out
    ref = ob.block_lists(zero_nan(q), km, Skv, n, causal, sink, local, lens)
    assert np.array_equal(got.cpu().numpy(), ref)


def test_lists_with_equal_scores_take_the_lower_index_and_nan_last():
    d, nb = 64, 300
    means = np.zeros((1, 1, nb, d))
    means[..., 0] = np.arange(nb) % 7  # many equal scores
    means[0, 0, 5] = -0.0
    kb = ob.to_bf16(means)
    q = ob.to_bf16(np.eye(1, d)[None, None].repeat(1, 2))
    for n in (1, 42, 43, 44, 150, 299, 300):
        got = ta.block_lists(to_dev(q), to_dev(kb), 128 * nb, n, local=0).cpu().numpy()
        assert np.array_equal(got, ob.block_lists(q, kb, 128 * nb, n, local=0)), n
    kb[0, 0, 6, 0] = NAN  # the best score of the first seven
    got = ta.block_lists(to_dev(q), to_dev(kb), 128 * nb, 1, local=0).cpu().numpy()
    assert got.ravel().tolist() == [13]
    every = ta.block_lists(to_dev(q), to_dev(kb), 128 * nb, nb, local=0).cpu().numpy()
    assert every.ravel().tolist() == list(range(nb))
    most = ta.block_lists(to_dev(q), to_dev(kb), 128 * nb, nb - 1, local=0).cpu().numpy()
    assert 6 not in most.ravel().tolist() and most.ravel().tolist()[-1] == nb - 1


def _step(x, lens):
    """Lists from the data, forward, gradients: a sparse layer's training step."""
    q, k, v, go = x
    lists = ta.block_lists(q, ta.block_means(k, lens), k.shape[2], 3, True, 1, 1, lens)
    out, lse = ta.block_attn(q, k, v, lists, True, lens=lens, return_lse=True)
    return [lists, out, lse, *ta.block_attn_grad(q, k, v, lists, out, go, lse, True, lens=lens)]


def _inputs(seed, S=900):
    rng = np.random.default_rng(seed)
    return [to_dev(bits(rng, 2, h, S, 64)) for h in (4, 2, 2, 4)]


def test_a_training_step_of_all_operators_together():
    x, lens = _inputs(1), [900, 700]
    lists, out, lse, dq, dk, dv = _step(x, i32(lens))
    qb, kb, vb, gb = (from_dev(t) for t in x)
    chosen = ob.block_lists(qb, ob.block_means(kb, lens), 900, 3, True, 1, 1, lens)
    assert np.array_equal(lists.cpu().numpy(), chosen)
    ref, rlse, mag = ob.attention(qb, kb, vb, chosen, True, lens)
    within(widen(from_dev(out)), ref, HALF * np.abs(ref) + (HALF + FP32) * mag + 1e-30, "out")
    rq, rk, rv = ob.attention_backward(qb, kb, vb, gb, chosen, True, lens)
    for name, g, r in (("dq", dq, rq), ("dk", dk, rk)):
        within(widen(from_dev(g)), r[0], HALF * np.abs(r[0]) + HALF * r[1] + FP32 * r[2] + r[3] + 1e-30, name)
    within(widen(from_dev(dv)), rv[0], HALF * np.abs(rv[0]) + (HALF + FP32) * rv[1] + 1e-30, "dv")


def test_two_captured_steps_replayed_with_eager_work_between():
    """Two graphs of whole steps, captured one after the other on one stream, replayed in turns on
    two streams: each has its own workspaces, and the results are the eager ones' bits."""
    lens = i32([900, 700])
    sets = [_inputs(20 + i) for i in range(4)]
    eager = [[t.clone() for t in _step(x, lens)] for x in sets]
    graphs, inputs, results = [], [], []
    for g in range(2):
        static = [t.clone() for t in sets[g]]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results.append(_step(static, lens))
        graphs.append(graph)
        inputs.append(static)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(4):
        for g in range(2):
            for a, b in zip(inputs[g], sets[(turn + 2 * g) % 4]):
                a.copy_(b)
        torch.cuda.synchronize()
        for g in range(2):
            with torch.cuda.stream(streams[g]):
                graphs[g].replay()
        again = _step(sets[turn], lens)  # the program's own work meanwhile
        torch.cuda.synchronize()
        for g in range(2):
            for a, b in zip(results[g], eager[(turn + 2 * g) % 4]):
                assert torch.equal(a, b), (turn, g)
        assert all(torch.equal(a, b) for a, b in zip(again, eager[turn]))


def test_another_stream_and_repeated_calls_give_the_same_bits():
    lens = i32([900, 700])
    x = _inputs(30)
    ref = _step(x, lens)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = [_step(x, lens) for _ in range(3)]
    s.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(g, ref))


def test_workspace_contents_do_not_matter():
    B, H, Hkv, S, d, n = 1, 4, 2, 900, 96, 6
    rng = np.random.default_rng(3)
    q, k, v, go = (to_dev(bits(rng, B, h, S, d)) for h in (H, Hkv, Hkv, H))
    lists = some_lists(rng, B, Hkv, S, S, n, "near")
    lists[..., 1] = 0
    lists = i32(lists)
    got = []
    for fill in (0, 255, 127):
        out, lse = torch.empty_like(q), torch.empty((B, H, S), device="cuda")
        grads = [torch.empty_like(t) for t in (q, k, v)]
        nf, nb = (f(B, H, Hkv, S, S, d, n) for f in (ta.block_attn_fwd_workspace, ta.block_attn_bwd_workspace))
        assert nf > 0
        wf, wb = (torch.full((x + 64,), fill, dtype=torch.uint8, device="cuda") for x in (nf, nb))
        stream = torch.cuda.current_stream()
        ta.block_attn_fwd(q, k, v, lists, out, lse, B, H, Hkv, S, S, d, n, True, None, 0.1, wf, nf, stream)
        ta.block_attn_bwd(q, k, v, lists, out, go, lse, *grads, B, H, Hkv, S, S, d, n, True, None, 0.1, wb, nb, stream)
        got.append([out, lse, *grads])
        assert (wf[nf:] == fill).all() and (wb[nb:] == fill).all()
    for g in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(g, got[0]))


def test_wrappers_refuse():
    q, k = torch.zeros(1, 4, 300, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 2, 300, 64, dtype=torch.bfloat16, device="cuda")
    lists = torch.zeros(1, 2, 3, 2, dtype=torch.int32, device="cuda")
    for bad in ((q.half(), k, k, lists), (q, k, k[:, :1], lists), (q, k, k, lists.long()), (q, k, k, lists[:, :, :2]),
                (q, k.transpose(1, 2).contiguous().transpose(1, 2), k, lists), (q, k, k.cpu(), lists)):
        with pytest.raises(ValueError):
            ta.block_attn(*bad)
    with pytest.raises(ValueError, match="lens"):
        ta.block_attn(q, k, k, lists, lens=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ta.TileAttnError, match="multiple"):
        ta.block_attn(q[:, :3].contiguous(), k, k, lists)
    with pytest.raises(ta.TileAttnError, match="overlap"):
        ta.block_attn(k, k, k, lists, out=k)
    with pytest.raises(ta.TileAttnError, match="forced"):
        ta.block_lists(q, torch.zeros(1, 2, 3, 64, dtype=torch.bfloat16, device="cuda"), 300, 1, sink=1)
    with pytest.raises(ValueError, match="blocks"):
        ta.block_lists(q, torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16, device="cuda"), 300, 2)


@pytest.mark.parametrize("kind", ["zeros", "equal", "near", "huge", "infinite"])
def test_lists_where_scores_are_hard_to_tell_apart(kind):
    """Scores that 32 bits cannot order: all equal, equal but for the last bits, sums that cancel, and
    infinities: the choice is the one that 64 bits make."""
    rng = np.random.default_rng(17)
    B, H, S, d, nb, n = 1, 2, 300, 96, 700, 33
    q, km = bits(rng, B, H, S, d), bits(rng, B, H, nb, d)
    if kind == "zeros":
        km[:] = 0
    elif kind == "equal":
        km[:] = km[:, :, :1]
    elif kind == "near":  # one step of bf16 in one small value apart
        km[:] = km[:, :, :1]
        km[..., 3] = 0x2000 + rng.integers(0, 64, (B, H, nb))
    elif kind == "huge":  # pairs that cancel
        x = ob.widen(km) * 2.0 ** 30
        x[..., 1::2] = -x[..., 0::2]
        x[..., 5] += 2.0 ** 22
        km = ob.to_bf16(x)
        q[..., 1::2] = q[..., 0::2]
    else:
        km[0, 0, 5, 7], km[0, 1, 600, 2] = 0x7F80, 0xFF80
    got = ta.block_lists(to_dev(q), to_dev(km), 128 * nb, n, local=1).cpu().numpy()
    with np.errstate(invalid="ignore"):
        ref = ob.block_lists(q, km, 128 * nb, n, local=1)
    assert np.array_equal(got, ref)


def test_the_longest_sequences():
    """TA_MAX_BLOCKS key blocks: the listed ones (the last among them) give what the same blocks give
    side by side in a short sequence, gradients too, and the rest get zeros."""
    d, nb, Sq, n = 64, 16384, 130, 3
    rng = np.random.default_rng(23)
    k, v = (torch.randn(1, 1, 128 * nb - 5, d, device="cuda").to(torch.bfloat16) for _ in range(2))
    q, go = to_dev(bits(rng, 1, 2, Sq, d)), to_dev(bits(rng, 1, 2, Sq, d))
    far = np.array([[[[nb - 1, 5, 9000], [nb - 1, 12345, -1]]]], np.int32)
    blocks = [5, 9000, 12345, nb - 1]
    near = np.array([[[[3, 0, 1], [3, 2, -1]]]], np.int32)
    ks, vs = (torch.cat([x[:, :, 128 * j:128 * (j + 1)] for j in blocks], 2).contiguous() for x in (k, v))
    out, lse = ta.block_attn(q, k, v, i32(far), return_lse=True)
    ref, rlse = ta.block_attn(q, ks, vs, i32(near), return_lse=True)
    assert torch.equal(out, ref) and torch.equal(lse, rlse)
    grads = ta.block_attn_grad(q, k, v, i32(far), out, go, lse)
    refs = ta.block_attn_grad(q, ks, vs, i32(near), ref, go, rlse)
    assert torch.equal(grads[0], refs[0])
    for g, r in zip(grads[1:], refs[1:]):
        assert torch.equal(torch.cat([g[:, :, 128 * j:128 * (j + 1)] for j in blocks], 2), r)
        assert g.count_nonzero() == r.count_nonzero()


@pytest.mark.parametrize("d", [64, 128])
def test_gradients_against_differences(d):
    """Along a direction: the change of sum(out * dout) between two points, computed in float64 from the
    reference's formula, against the kernels' gradients."""
    rng = np.random.default_rng(31)
    grid = lambda *s: np.round(rng.uniform(-0.5, 0.5, s) * 64) / 64  # noqa: E731
    S, H, lists = 260, 2, np.array([[[[0, -1], [1, 0], [2, 1]]]], np.int32)
    q, k, v, go = grid(1, H, S, d), grid(1, 1, S, d), grid(1, 1, S, d), grid(1, H, S, d)
    dev = [to_dev(ob.to_bf16(x)) for x in (q, k, v, go)]
    out, lse = ta.block_attn(*dev[:3], i32(lists), True, return_lse=True)
    grads = ta.block_attn_grad(*dev[:3], i32(lists), out, dev[3], lse, True)
    for i, x in enumerate((q, k, v)):
        step = rng.integers(-1, 2, x.shape) * 2.0 ** -8
        at = [[ob.to_bf16(y + s * step if j == i else y) for j, y in enumerate((q, k, v))] for s in (1, -1)]
        plus, minus = (float((ob.attention(*z, lists, True)[0] * go).sum()) for z in at)
        got = widen(from_dev(grads[i]))
        # the kernels' own bound, and the differences' (their step is 2^-8)
        r = ob.attention_backward(*(ob.to_bf16(y) for y in (q, k, v, go)), lists, True)[i]
        slack = HALF * np.abs(r[0]) + (HALF + FP32) * r[1] + (FP32 * r[2] + r[3] if i < 2 else 0)
        bound = float((slack * np.abs(step)).sum()) + 1e-3 * float((np.abs(r[0]) * np.abs(step)).sum())
        assert abs((plus - minus) / 2 - float((got * step).sum())) <= bound, i


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("Sq,Skv,n,ends", [(300, 300, 3, 300), (300, 300, 3, 270), (40, 2000, 16, 2000)],
                         ids=["whole", "padded", "pieces"])
def test_values_that_are_no_numbers_reach_only_the_rows_that_see_them(d, Sq, Skv, n, ends):
    """NaN and infinities among the values, in causal order: earlier rows and padded ones keep their
    bits, later ones get what the sum gives, in these dims only."""
    rng = np.random.default_rng(d + Skv)
    q, k, v = (bits(rng, 1, h, s, d) for h, s in ((4, Sq), (2, Skv), (2, Skv)))
    lists = np.broadcast_to(np.arange(n, dtype=np.int32), (1, 2, -(-Sq // 128), n)).copy()
    lens = [ends]
    assert (ta.block_attn_fwd_workspace(1, 4, 2, Sq, Skv, d, n) > 0) == (n == 16)
    t0 = Skv - 100 if n < 16 else Skv - 20
    t1 = t0 + 10
    bad = v.copy()
    bad[:, :, t0, [3, 5, 40]] = [NAN, 0x7F80, 0xFF80]  # dim 5: +inf, then inf - inf; dim 40: -inf
    bad[:, :, t1, [5, 7]] = [0xFF80, 0x7F80]
    zeroed = v.copy()
    zeroed[:, :, t0, [3, 5, 40]] = 0
    zeroed[:, :, t1, [5, 7]] = 0
    run = lambda x: ta.block_attn(to_dev(q), to_dev(k), to_dev(x), i32(lists), True, None, i32(lens), return_lse=True)  # noqa: E731
    (got, lse), (ref, rlse) = run(bad), run(zeroed)
    assert torch.equal(lse, rlse)
    want, got = ref.float().cpu().numpy(), got.float().cpu().numpy()
    pos = Skv - Sq + np.arange(Sq)
    sees0, sees1 = (pos >= t0) & (pos < ends), (pos >= t1) & (pos < ends)
    assert sees0.any() and sees1.any() and not sees0.all()
    want[:, :, sees0, 3] = np.nan
    want[:, :, sees0, 5] = np.inf
    want[:, :, sees0, 40] = -np.inf
    want[:, :, sees1, 5] = np.nan
    want[:, :, sees1, 7] = np.inf
    assert np.array_equal(got, want, equal_nan=True)


@pytest.mark.parametrize("Sq,Skv,n", [(200, 400, 3), (6, 2000, 16)])
def test_a_query_that_is_no_number_shows_in_its_row_and_gradients(Sq, Skv, n):
    rng = np.random.default_rng(Skv)
    q, k, v, go = (bits(rng, 1, h, s, 64) for h, s in ((2, Sq), (1, Skv), (1, Skv), (2, Sq)))
    lists = np.broadcast_to(np.arange(n, dtype=np.int32), (1, 1, -(-Sq // 128), n)).copy()
    bad = q.copy()
    bad[0, 1, 4, 9] = NAN
    (out, lse), (ref, rlse) = (ta.block_attn(to_dev(x), to_dev(k), to_dev(v), i32(lists), return_lse=True) for x in (bad, q))
    assert out[0, 1, 4].isnan().all() and lse[0, 1, 4].isnan()
    other = torch.ones((2, Sq), dtype=torch.bool, device="cuda")
    other[1, 4] = False
    assert torch.equal(out[0, other], ref[0, other]) and torch.equal(lse[0, other], rlse[0, other])
    dq, dk, _ = ta.block_attn_grad(to_dev(bad), to_dev(k), to_dev(v), i32(lists), out, to_dev(go), lse)
    clean = ta.block_attn_grad(to_dev(q), to_dev(k), to_dev(v), i32(lists), ref, to_dev(go), rlse)
    assert dq[0, 1, 4].isnan().all() and torch.equal(dq[0, other], clean[0][0, other])
    assert dk[0, 0, : 128 * n].isnan().all()


def test_stretches_of_the_line_whatever_the_workspace_holds_and_replayed():
    """d = 128 with work enough for the key side's line: any contents of the workspace, three streams at
    once and replays of a captured call give the same bits."""
    B, H, Hkv, S, d, n = 1, 48, 2, 900, 128, 6
    rng = np.random.default_rng(31)
    q, k, v, go = (to_dev(bits(rng, B, h, S, d)) for h in (H, Hkv, Hkv, H))
    lists = some_lists(rng, B, Hkv, S, S, n, "near")
    lists[..., 1] = 0
    lists, lens = i32(lists), i32([850])
    out, lse = ta.block_attn(q, k, v, lists, True, None, lens, return_lse=True)
    ref = ta.block_attn_grad(q, k, v, lists, out, go, lse, True, None, lens)
    bytes_ = ta.block_attn_bwd_workspace(B, H, Hkv, S, S, d, n)
    streams, got, held = [torch.cuda.Stream() for _ in range(3)], [], []
    torch.cuda.synchronize()
    for fill, s in zip((0, 255, 127), streams):
        with torch.cuda.stream(s):
            ws = torch.full((bytes_ + 64,), fill, dtype=torch.uint8, device="cuda")
            grads = [torch.empty_like(t) for t in (q, k, v)]
            ta.block_attn_bwd(q, k, v, lists, out, go, lse, *grads, B, H, Hkv, S, S, d, n, True, lens, d ** -0.5, ws, bytes_, s)
        got.append(grads)
        held.append((ws, fill))
    torch.cuda.synchronize()
    for grads, (ws, fill) in zip(got, held):
        assert all(torch.equal(a, b) for a, b in zip(grads, ref)) and (ws[bytes_:] == fill).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = ta.block_attn_grad(q, k, v, lists, out, go, lse, True, None, lens)
    for _ in range(3):
        for t in again:
            t.fill_(1)
        graph.replay()
        eager = ta.block_attn_grad(q, k, v, lists, out, go, lse, True, None, lens)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, ref)) and all(torch.equal(a, b) for a, b in zip(eager, ref))


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("top", [-9, -12])
def test_lists_where_a_large_channel_lies_beside_a_small_one_of_the_other_sign(d, top):
    """Key means with 1024 beside -2^-10, twice, cancelled by the query: the sums in 32 bits keep of the
    small channels, which order the blocks, what is left of an ulp of 1024, and the bound on their
    error has to come from the 1024."""
    rng = np.random.default_rng(d - top)
    nb, n = 300, 33
    km, q = np.zeros((1, 1, nb, d)), np.zeros((1, 1, 1, d))
    km[..., [0, 32]], km[..., [1, 33]] = 1024, -2.0 ** -10
    km[..., [2, 34]] = -rng.uniform(0, 2.0 ** top, (nb, 2))
    q[..., [0, 2, 34]], q[..., 32] = 1, -1
    kb, qb = ob.to_bf16(km), ob.to_bf16(q)
    got = ta.block_lists(to_dev(qb), to_dev(kb), 128 * nb, n, local=0).cpu().numpy()
    assert np.array_equal(got, ob.block_lists(qb, kb, 128 * nb, n, local=0))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nb,infinite,n", [(80, 4, 5), (300, 8, 6), (700, 40, 30), (90, 3, 88), (60, 5, 5)])
def test_lists_with_more_infinite_scores_than_places(d, nb, infinite, n):
    """Forced blocks, then key means of +inf, of which only the first find a place: the last bin of
    the search ends with them, not with the forced blocks behind."""
    rng = np.random.default_rng(nb + n)
    q, km = bits(rng, 1, 2, 200, d), bits(rng, 1, 1, nb, d)
    q[..., 5] = 0x3F80
    where = rng.permutation(nb)[:infinite]
    km[0, 0, where, 5] = 0x7F80
    got = ta.block_lists(to_dev(q), to_dev(km), 128 * nb, n, sink=2, local=1).cpu().numpy()
    with np.errstate(invalid="ignore"):
        ref = ob.block_lists(q, km, 128 * nb, n, sink=2, local=1)
    assert np.array_equal(got, ref)


@pytest.mark.parametrize("B,H,Hkv,Sq,Skv,d,n,causal,lens", [
    (1, 2, 1, 200, 400, 64, 3, False, None),
    (1, 2, 1, 6, 2000, 64, 16, False, None),
    (2, 4, 2, 500, 500, 96, 4, True, [500, 333]),
    (1, 6, 3, 300, 555, 128, 5, True, [550]),
    (1, 48, 2, 900, 900, 128, 6, True, [850]),  # the line of columns
], ids=["rows", "token", "causal", "items", "line"])
def test_rows_that_are_no_numbers_show_in_dv_of_the_keys_they_attend_to(B, H, Hkv, Sq, Skv, d, n, causal, lens):
    """A query, and a key, that is NaN: its rows' weights are NaN, and so is dv of all keys these rows
    attend to, as in the formula; every other dv keeps its bits."""
    rng = np.random.default_rng(Skv + d)
    q, k, v, go = (bits(rng, B, h, s, d) for h, s in ((H, Sq), (Hkv, Skv), (Hkv, Skv), (H, Sq)))
    lists = some_lists(rng, B, Hkv, Sq, Skv, n, "near")
    run = lambda *x: ta.block_attn(*(to_dev(y) for y in x), i32(lists), causal, lens=i32(lens), return_lse=True)  # noqa: E731
    grad = lambda x, o: ta.block_attn_grad(*(to_dev(y) for y in x), i32(lists), o[0], to_dev(go), o[1], causal,  # noqa: E731
                                           lens=i32(lens))
    clean = grad((q, k, v), run(q, k, v))
    off, at = Skv - Sq, 4 if Sq < 100 else 70
    sees = [[ob.attends(lists[b, h], Sq, Skv, causal, Skv if lens is None else lens[b]) for h in range(Hkv)] for b in range(B)]
    for what in ("query", "key"):
        x = [y.copy() for y in (q, k, v)]
        bad = np.zeros((B, H, Sq), bool)
        if what == "query":
            x[0][0, H - 1, at, 9] = NAN
            bad[0, H - 1, at] = True
        else:
            t = off + at
            x[1][0, 0, t, 5] = NAN
            bad[0, :H // Hkv] = sees[0][0][:, t]
        out = run(*x)
        some = np.array([[sees[b][h * Hkv // H].any(1) for h in range(H)] for b in range(B)])
        assert np.array_equal(np.isnan(out[1].cpu().numpy()), bad & some)
        want = np.zeros((B, Hkv, Skv), bool)
        for b in range(B):
            for h in range(H):
                want[b, h * Hkv // H] |= sees[b][h * Hkv // H][bad[b, h]].any(0)
        assert what == "key" or want.any()
        dv = grad(x, out)[2]
        assert np.array_equal(np.isnan(widen(from_dev(dv))), np.broadcast_to(want[..., None], dv.shape))
        keep = torch.from_numpy(~want).cuda()
        assert torch.equal(dv[keep], clean[2][keep])


def test_means_are_rounded_once():
    """Means just past and just before a tie of bf16, nearer than fp32 can tell: the side they lie on."""
    x = np.zeros((1, 1, 512, 64))
    x[0, 0, [0, 128, 256, 384]], x[0, 0, [1, 129, 257, 385]] = 4 * 32, 32 * 2.0 ** -6  # means 1 + 2^-8, a tie, and
    x[0, 0, [2, 130]] = [[32 * 2.0 ** -28], [-32 * 2.0 ** -28]]                        # 2^-30 more and less
    x[0, 0, 257] = 32 * 3 * 2.0 ** -6                                                  # 1 + 3 * 2^-8, a tie,
    x[0, 0, 258] = -32 * 2.0 ** -28                                                    # 2^-30 less
    xb = ob.to_bf16(x)
    assert np.array_equal(ob.widen(xb), x)
    want = [1 + 2.0 ** -7, 1.0, 1 + 2.0 ** -7, 1.0]
    got = ta.block_means(to_dev(xb))
    assert (widen(from_dev(got)) == np.array(want)[:, None]).all()
    assert np.array_equal(from_dev(got), ob.block_means(xb))
    # the same of a query block's mean: its score beside one of 1
    km = ob.to_bf16(np.eye(2, 64)[None, None, ::-1])  # block 0 picks dim 1, block 1 dim 0
    for i, best in enumerate([1, 0, 1, 0]):
        q = x[:, :, 128 * i:128 * (i + 1)].copy()
        q[..., 1] = 1
        assert ta.block_lists(to_dev(ob.to_bf16(q)), to_dev(km), 256, 1, local=0).item() == best, i


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("size", [2.0 ** 20, 2.0 ** 28])
def test_logits_of_a_large_size(d, size):
    """Scores of few bits, exact in fp32, up to the stated limit: the rows give the mean of the values
    of their largest ones (the next are at least 2^15 below), and nothing overflows."""
    rng = np.random.default_rng(d)
    S = 300
    q, k, v = np.zeros((1, 1, S, d)), np.zeros((1, 1, S, d)), bits(rng, 1, 1, S, d)
    q[..., 3] = rng.choice([-1.0, 1.0], (1, 1, S))
    k[..., 3] = rng.integers(-32, 33, (1, 1, S)) * (size / 32)
    qb, kb = ob.to_bf16(q), ob.to_bf16(k)
    lists = np.array([[[[0, 1, 2]] * 3]], np.int32)
    for causal in (False, True):
        out, lse = ta.block_attn(to_dev(qb), to_dev(kb), to_dev(v), i32(lists), causal, 1.0, return_lse=True)
        ref, rlse, mag = ob.attention(qb, kb, v, lists, causal, None, 1.0)
        # the weights of equal scores are equal, one rounding to bf16 each
        within(widen(from_dev(out)), ref, HALF * np.abs(ref) + (HALF + FP32) * mag + 1e-30, "out")
        assert (np.abs(lse.cpu().numpy() - rlse) <= 2.0 ** -22 * np.abs(rlse) + 1e-3).all()


def test_calls_that_autograd_does_not_record_say_so(recwarn):
    q, k, v, go = _inputs(3)
    lists = ta.block_lists(q, ta.block_means(k), 900, 3)
    ref, lse = ta.block_attn(q, k, v, lists, return_lse=True)
    with torch.no_grad():
        ta.block_attn(q.clone().requires_grad_(), k, v, lists)
    assert not recwarn.list
    for i in range(3):
        x = [t.clone().requires_grad_() if j == i else t for j, t in enumerate((q, k, v))]
        with pytest.warns(UserWarning, match="block_attn_grad"):
            out = ta.block_attn(*x, lists)
        assert torch.equal(out, ref) and not out.requires_grad

    class Sparse(torch.autograd.Function):  # how a program records it
        @staticmethod
        def forward(ctx, q, k, v):
            out, lse = ta.block_attn(q, k, v, lists, return_lse=True)
            ctx.save_for_backward(q, k, v, out, lse)
            return out

        @staticmethod
        def backward(ctx, dout):
            q, k, v, out, lse = ctx.saved_tensors
            return ta.block_attn_grad(q, k, v, lists, out, dout.contiguous(), lse)

    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    Sparse.apply(*leaves).backward(go)
    assert not recwarn.list
    for t, g in zip(leaves, ta.block_attn_grad(q, k, v, lists, ref, go, lse)):
        assert torch.equal(t.grad, g)


def test_a_causal_list_is_chosen_by_all_rows_of_its_query_block():
    """What the documentation says of lists: a later row of the same block moves the choice of an
    earlier one, rows of later blocks do not; and with lens a query block of padding has none."""
    S, d = 128 * 12, 64
    q, k = np.zeros((1, 1, S, d)), np.zeros((1, 1, S, d))
    for j in range(12):
        k[0, 0, 128 * j:128 * (j + 1), j] = 1
    q[0, 0, 128 * 8, 2], q[0, 0, 128 * 8 + 100, 5], q[0, 0, 128 * 9:, 7] = 1, 2, 9
    means = ta.block_means(to_dev(ob.to_bf16(k)))
    run = lambda x, lens=None: ta.block_lists(to_dev(ob.to_bf16(x)), means, S, 2, True, 0, 1, i32(lens)).cpu().numpy()[0, 0]  # noqa: E731
    assert run(q)[8].tolist() == [5, 8]
    q[0, 0, 128 * 8 + 100] = 0
    assert run(q)[8].tolist() == [2, 8]
    assert run(q, [128 * 8])[7:].tolist() == [[0, 7]] + [[-1, -1]] * 4
    alone = ta.block_lists(to_dev(ob.to_bf16(q[:, :, 128 * 8:128 * 8 + 1])), means[:, :, :9].contiguous(), 128 * 8 + 1, 2, True)
    assert alone.flatten().tolist() == [2, 8]
