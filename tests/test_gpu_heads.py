"""Head norms and rotations and their gradients on the GPU against the float64 reference.

Tolerances. A result is rounded to bf16 once: 2^-8 of its value. Before that, in fp32 and relative to
the numbers that are added (a value and its partner, normed and weighted: mag below): the row's sum of up to 128
squares at most 128 * 2^-24 = 2^-17, half of it in the factor; sine and cosine 1.3e-7 and their argument's
rounding 2^-25 turns = 1.9e-7; a handful of products and sums at 2^-24: together below 2^-16. The mean of "layer" is
off by at most 2^-17 of the row's mean magnitude, which mag contains. Gradients have two more sums over the row
(2^-17 each) and their products: 2^-14 of their mag. Sums over rows: every term off by less than 2^-16 of its mag,
chains of fewer than 256 additions of 2^-24 (2^-16) a lane and 32 more behind: 2^-14 of the sum of mags."""
import numpy as np
import pytest

import workloads
from oracle import heads as oh
from tests.gpu_helpers import from_dev, to_dev, widen

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2502_06155_amd as ta  # noqa: E402

HALF = 2.0 ** -8
WEIGHTS = ("q_weight", "k_weight", "q_bias", "k_bias")


def bits(rng, *shape):
    return workloads.f32_to_bf16_bits(rng.standard_normal(shape, dtype=np.float32))


def params(rng, d, norm):
    f = lambda c, s: (c + s * rng.standard_normal(d)).astype(np.float32)  # noqa: E731
    p = dict.fromkeys(WEIGHTS)
    if norm:
        p.update(q_weight=f(1, 0.3), k_weight=f(1, 0.3))
    if norm == "layer":
        p.update(q_bias=f(0, 0.2), k_bias=f(0, 0.2))
    return p


def gpu(x, dtype=None):
    return None if x is None else torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


class Case:
    """One call's inputs: x bits [B, S, H + 2 Hkv, d], as a projection of everything leaves them."""

    def __init__(self, B, S, H, Hkv, d, norm, layout, dims, lens=None, far=False, eps=1e-6, seed=0, shared=True):
        rng = np.random.default_rng(seed + S + d)
        self.sizes, self.norm, self.layout, self.dims, self.lens, self.eps = (B, S, H, Hkv, d), norm, layout, dims, lens, eps
        self.x = bits(rng, B, S, H + 2 * Hkv, d)
        self.p = params(rng, d, norm)
        self.dy = [bits(rng, B, h, S, d) for h in (H, Hkv, Hkv)]
        self.positions = self.freqs = None
        if dims:
            self.positions = rng.integers(-2 ** 31 if far else 0, 2 ** 31 if far else 300,
                                          (S if shared else B * S, len(dims))).astype(np.int32)
            if not shared:
                self.positions = self.positions.reshape(B, S, len(dims))
            self.freqs = np.concatenate([10000.0 ** (-np.arange(0, n, 2) / n) for n in dims])

    def parts(self, x):
        _, _, H, Hkv, _ = self.sizes
        return x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]

    def how(self):
        """The oracle's arguments."""
        p = self.positions
        if p is not None and p.ndim == 2:
            p = np.broadcast_to(p, (self.sizes[0],) + p.shape)
        return dict(norm=self.norm, eps=self.eps, positions=p, freqs=self.freqs, dims=self.dims, layout=self.layout,
                    lens=self.lens)

    def args(self):
        """The wrappers' arguments."""
        a = dict(norm=self.norm, eps=self.eps, lens=gpu(self.lens, torch.int32), dims=self.dims,
                 **{n: gpu(w) for n, w in self.p.items()})
        if self.positions is not None:
            a.update(positions=gpu(self.positions), freqs=gpu(self.freqs), layout=self.layout)
        return a

    def magnitudes(self, x, name):
        """[B, S, heads, d]: the numbers that a result is made of, a value's and its partner's."""
        x = np.asarray(x, np.float64)
        hat, r = oh.normed(x, self.norm, self.eps)
        mag = np.abs(hat)
        if self.norm == "layer":
            mag = (np.abs(x) + np.abs(x).mean(-1, keepdims=True)) * r
        w, b = self.p[name + "_weight"], self.p[name + "_bias"]
        mag = mag * (1.0 if w is None else np.abs(w.astype(np.float64))) + (0.0 if b is None else np.abs(b))
        return self.with_partner(mag)

    def with_partner(self, mag):
        out = mag.copy()
        for i, j, _ in oh.pairs(self.dims, self.layout) if self.dims else ():
            out[..., i] = out[..., j] = mag[..., i] + mag[..., j]
        return out


def near(got, ref, room, what):
    off = np.abs(got - ref) - room
    assert np.isfinite(got).all(), what
    assert off.max() <= 0, (what, np.unravel_index(np.argmax(off), off.shape), off.max())


def check_forward(c, got):
    x = widen(c.x)
    for name, part, y in zip("qkv", c.parts(x), got):
        if name == "v":
            ref = oh.forward(part, lens=c.lens)
            assert np.array_equal(widen(from_dev(y)), ref)
            continue
        ref = oh.forward(part, weight=c.p[name + "_weight"], bias=c.p[name + "_bias"], **c.how())
        mag = c.magnitudes(part, name).transpose(0, 2, 1, 3)
        near(widen(from_dev(y)), ref, HALF * np.abs(ref) + 2.0 ** -16 * mag, name)
        if c.lens is not None:
            for b, n in enumerate(c.lens):
                assert not from_dev(y)[b, :, max(n, 0):].any()


def check_gradients(c, got):
    x = widen(c.x)
    for i, (name, part) in enumerate(zip("qkv", c.parts(x))):
        dy = widen(c.dy[i])
        if name == "v":
            ref, _, _ = oh.backward(part, dy, lens=c.lens)
            assert np.array_equal(widen(from_dev(got[2])), ref)
            continue
        how = c.how()
        ref, dw, db = oh.backward(part, dy, weight=c.p[name + "_weight"], bias=c.p[name + "_bias"], **how)
        hat, r = oh.normed(part, c.norm, c.eps)
        wide = np.abs(hat)
        if c.norm == "layer":
            wide = (np.abs(part) + np.abs(part).mean(-1, keepdims=True)) * r
        g = np.abs(dy.transpose(0, 2, 1, 3)).copy()
        for b, n in enumerate(c.lens or ()):
            g[b, max(n, 0):] = 0
        g = c.with_partner(g)
        w = c.p[name + "_weight"]
        u = g * (1.0 if w is None else np.abs(w.astype(np.float64)))
        mag = r * (u + u.mean(-1, keepdims=True) + wide * (u * wide).mean(-1, keepdims=True)) if c.norm else g
        near(widen(from_dev(got[i])), ref, HALF * np.abs(ref) + 2.0 ** -14 * mag, "d" + name)
        for n, (sum_, of) in enumerate(((dw, g * wide), (db, g))):
            t = got[3 + i + 2 * n]
            assert (t is None) == (c.p[name + ("_weight", "_bias")[n]] is None)
            if t is not None:
                near(t.cpu().numpy().astype(np.float64), sum_, 2.0 ** -14 * of.sum((0, 1, 2)), ("dw", "db")[n])


CASES = [
    # one token, one sequence, few heads: every norm and pairing
    dict(B=1, S=1, H=1, Hkv=1, d=64, norm="rms", layout="interleaved", dims=(64,)),
    dict(B=1, S=1, H=1, Hkv=1, d=128, norm=None, layout="halves", dims=(128,)),
    dict(B=37, S=1, H=5, Hkv=1, d=128, norm="rms", layout="halves", dims=(128,), far=True, shared=False),
    dict(B=5, S=1, H=32, Hkv=8, d=96, norm="layer", layout="split", dims=(96,), far=True, shared=False),
    # axes of a video, and parts that are not turned
    dict(B=2, S=123, H=6, Hkv=2, d=64, norm="layer", layout="interleaved", dims=(16, 24, 24), lens=[123, 70]),
    dict(B=1, S=301, H=3, Hkv=3, d=96, norm="rms", layout="halves", dims=(32, 32, 32)),
    dict(B=1, S=77, H=2, Hkv=1, d=128, norm="rms", layout="interleaved", dims=(44, 42, 42)),
    dict(B=2, S=50, H=2, Hkv=1, d=128, norm="rms", layout="halves", dims=(44, 42, 42)),
    dict(B=2, S=51, H=2, Hkv=2, d=128, norm="rms", layout="split", dims=(32, 48, 48), shared=False),
    dict(B=1, S=40, H=3, Hkv=1, d=96, norm="layer", layout="split", dims=(6, 10, 14, 20)),
    # a multiple of 16 in all, but eight values that follow each other turn with two axes
    dict(B=1, S=45, H=2, Hkv=1, d=128, norm="rms", layout="split", dims=(16, 56, 56)),
    dict(B=2, S=13, H=3, Hkv=1, d=64, norm=None, layout="split", dims=(10, 22), lens=[13, 6]),
    dict(B=1, S=30, H=2, Hkv=2, d=96, norm="layer", layout="split", dims=(8, 40), shared=False),
    dict(B=1, S=9, H=3, Hkv=1, d=64, norm="rms", layout="halves", dims=(2, 2)),
    dict(B=1, S=33, H=4, Hkv=2, d=128, norm="rms", layout="interleaved", dims=(32,)),
    dict(B=3, S=7, H=9, Hkv=1, d=96, norm="rms", layout="halves", dims=(16,), lens=[0, 9, -3]),
    # norms alone, rotation alone, the layout alone
    dict(B=2, S=19, H=4, Hkv=2, d=96, norm="layer", layout=None, dims=None),
    dict(B=2, S=19, H=4, Hkv=2, d=64, norm="rms", layout=None, dims=None, lens=[4, 19]),
    dict(B=2, S=19, H=4, Hkv=2, d=64, norm=None, layout="split", dims=(64,)),
    dict(B=2, S=65, H=4, Hkv=2, d=128, norm=None, layout="interleaved", dims=(64, 32)),
    dict(B=2, S=19, H=4, Hkv=2, d=128, norm=None, layout=None, dims=None, lens=[19, 1]),
    # enough tokens that waves take many heads and items
    dict(B=1, S=9001, H=3, Hkv=1, d=64, norm="layer", layout="halves", dims=(64,)),
    # nine heads a wave forward, for each pairing; three items a wave in the gradients
    dict(B=1, S=8197, H=5, Hkv=2, d=96, norm="layer", layout="interleaved", dims=(32, 32, 32)),
    dict(B=2, S=8200, H=5, Hkv=2, d=64, norm="rms", layout="split", dims=(16, 48), lens=[8200, 5001]),
    dict(B=1, S=30001, H=3, Hkv=1, d=96, norm="layer", layout="halves", dims=(28, 34, 34)),
]


def named(c):
    return "-".join(str(v).replace(" ", "") for v in c.values())


@pytest.mark.parametrize("c", CASES, ids=named)
def test_forward_and_gradients(c):
    c = Case(**c)
    x = to_dev(c.x)
    q, k, v = c.parts(x)
    check_forward(c, ta.head_rope(q, k, v, **c.args()))
    dy = [to_dev(g) for g in c.dy]
    check_gradients(c, ta.head_rope_grad(q, k, v, *dy, **c.args()))


def test_layouts_of_memory():
    """The same rows from one projection, from three tensors, transposed, with gaps, and one row for all heads
    or sequences give the same bits; gradients land in views of one tensor and leave the rest alone."""
    c = Case(3, 21, 4, 2, 96, "rms", "halves", (32, 32, 32), lens=[21, 5, 13])
    x = to_dev(c.x)
    want = ta.head_rope(*c.parts(x), **c.args())
    dy = [to_dev(g) for g in c.dy]
    grads = ta.head_rope_grad(*c.parts(x), *dy, **c.args())
    forms = [
        [p.contiguous() for p in c.parts(x)],
        [p.transpose(1, 2).contiguous().transpose(1, 2) for p in c.parts(x)],
        [p.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3) for p in c.parts(x)],
        [torch.nn.functional.pad(p, (8, 24)).narrow(3, 8, 96) for p in c.parts(x)],
    ]
    for form in forms:
        for a, b in zip(want, ta.head_rope(*form, **c.args())):
            assert torch.equal(a, b)
        out = [torch.full_like(p, 7.0) for p in form]  # (strides kept where they are dense)
        for a, b in zip(grads, ta.head_rope_grad(*form, *dy, out=out, **c.args())):
            assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
    wide = torch.full((3, 21, 12, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    views = [wide[:, :, 1:5, 16:112], wide[:, :, 6:8, 16:112], wide[:, :, 9:11, 16:112]]
    ta.head_rope_grad(*c.parts(x), *dy, out=views, **c.args())
    for a, b in zip(grads, views):
        assert torch.equal(a, b)
    for view in views:
        view.fill_(7.0)
    assert (wide == 7.0).all()
    first = torch.empty(21, 3, 8, 96, dtype=torch.bfloat16, device="cuda").transpose(0, 1)  # tokens before sequences
    first.copy_(x)
    into = torch.zeros(21, 3, 8, 96, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    ta.head_rope_grad(*c.parts(first), *dy, out=c.parts(into), **c.args())
    assert torch.equal(into, torch.cat(grads[:3], 2))
    one = x[:1, :, :1].expand(3, 21, 4, 96)
    a, b = (ta.head_rope(t, None, None, **{**c.args(), "k_weight": None})[0] for t in (one, one.contiguous()))
    assert torch.equal(a, b)


def test_parts_alone():
    c = Case(2, 30, 6, 2, 128, "layer", "interleaved", (32, 48, 48))
    x = to_dev(c.x)
    q, k, v = c.parts(x)
    dy = [to_dev(g) for g in c.dy]
    every, grads = ta.head_rope(q, k, v, **c.args()), ta.head_rope_grad(q, k, v, *dy, **c.args())
    for keep in ((0,), (1,), (2,), (0, 1), (1, 2)):
        some = [t if i in keep else None for i, t in enumerate((q, k, v))]
        g = [t if i in keep else None for i, t in enumerate(dy)]
        for i, (a, b) in enumerate(zip(ta.head_rope(*some, **c.args()), every)):
            assert (a is None) == (i not in keep) and (a is None or torch.equal(a, b))
        for i, (a, b) in enumerate(zip(ta.head_rope_grad(*some, *g, **c.args()), grads)):
            here = (i if i < 3 else (i - 3) % 2) in keep
            assert (a is not None) == here
            if i < 3 and here:
                assert torch.equal(a, b)
            elif here:  # sums over other numbers of workgroups
                assert torch.allclose(a, b, rtol=1e-4, atol=1e-3)


def test_what_padding_holds_reaches_nothing():
    c = Case(2, 40, 4, 2, 64, "layer", "halves", (64,), lens=[40, 11])
    x = to_dev(c.x)
    dy = [to_dev(g) for g in c.dy]
    want, grads = ta.head_rope(*c.parts(x), **c.args()), ta.head_rope_grad(*c.parts(x), *dy, **c.args())
    for bad in (float("nan"), float("inf"), 3e38):
        x[1, 11:] = bad
        for g in dy:
            g[1, :, 11:] = bad
        for a, b in zip((*want, *grads), (*ta.head_rope(*c.parts(x), **c.args()),
                                          *ta.head_rope_grad(*c.parts(x), *dy, **c.args()))):
            assert torch.equal(a, b)


def test_a_row_that_is_no_number_stays_alone():
    c = Case(1, 20, 4, 2, 96, "rms", "halves", (96,))
    x = to_dev(c.x)
    want = ta.head_rope(*c.parts(x), **c.args())
    x[0, 3, 1, 40] = float("nan")
    x[0, 5, 4, 0] = float("inf")
    got = ta.head_rope(*c.parts(x), **c.args())
    for h, (a, b) in enumerate(zip(want, got)):
        bad = torch.isnan(b).any(-1)
        rows = {(0, 1, 3)} if h == 0 else {(0, 0, 5)} if h == 1 else set()
        assert {tuple(i) for i in torch.nonzero(bad).tolist()} == rows
        assert torch.equal(a[~bad], b[~bad])


@pytest.mark.parametrize("norm", [None, "rms"])
@pytest.mark.parametrize("layout,dims,d", [
    ("interleaved", (32,), 64), ("interleaved", (6, 12, 12), 96), ("halves", (32,), 64), ("halves", (16, 32), 96),
    ("halves", (20,), 128), ("split", (32, 32), 128), ("split", (10, 24), 96), ("split", (8,), 64)])
def test_values_that_are_not_turned_take_nothing_from_others(layout, dims, d, norm):
    """Infinities and NaN behind the turned values: each stays at its place, or (with a norm) reaches what the
    formula says, and no neighbour; forward and gradients, in rows and in weights."""
    R = sum(dims)
    c = Case(1, 12, 2, 1, d, norm, layout, dims)
    places = (R, R + 1, d - 8, d - 1)
    for t, (bad, e) in enumerate((b, e) for b in (0x7F80, 0xFF80, 0x7FC0) for e in places):  # inf, -inf, NaN
        c.x[0, t, :2, e] = bad
    x = widen(c.x)
    got = ta.head_rope(*c.parts(to_dev(c.x)), **c.args())
    for name, part, y in zip("qk", c.parts(x), got):
        with np.errstate(invalid="ignore"):
            ref = oh.forward(part, weight=c.p[name + "_weight"], **c.how())
        y = widen(from_dev(y))
        assert np.array_equal(np.isnan(y), np.isnan(ref)) and np.array_equal(y[np.isinf(ref)], ref[np.isinf(ref)])
        some = np.isfinite(ref)
        mag = c.magnitudes(np.where(np.isfinite(part), part, 0), name).transpose(0, 2, 1, 3)
        room = HALF * np.abs(ref) + 2.0 ** -16 * mag
        assert (np.abs(y[some] - ref[some]) <= room[some]).all()
        if norm is None:
            assert np.array_equal(y[..., R:], ref[..., R:], equal_nan=True) and not np.isnan(y[..., :R]).any()
    # gradients: of the rows without a norm; with one, of a weight for each value
    c = Case(1, 12, 2, 1, d, norm, layout, dims, seed=1)
    for t, e in enumerate(places):
        c.dy[0][0, 1, t, e] = (0x7F80, 0x7FC0)[t % 2]
    dx, _, _, dw, _, _, _ = ta.head_rope_grad(*c.parts(to_dev(c.x)), *(to_dev(g) for g in c.dy), **c.args())
    if norm is None:
        ref, _, _ = oh.backward(c.parts(widen(c.x))[0], widen(c.dy[0]), **c.how())
        dx = widen(from_dev(dx))
        assert np.array_equal(dx[..., R:], ref[..., R:], equal_nan=True) and np.isfinite(dx[..., :R]).all()
    else:
        bad = ~torch.isfinite(dw).cpu().numpy()
        assert set(np.flatnonzero(bad)) == set(places)
        c = Case(1, 5, 2, 1, d, norm, layout, dims)
        c.p["q_weight"][R], c.p["q_weight"][d - 1] = np.inf, np.nan
        y = widen(from_dev(ta.head_rope(*c.parts(to_dev(c.x)), **c.args())[0]))
        assert set(np.flatnonzero(~np.isfinite(y).all((0, 1, 2)))) == {R, d - 1}


def test_rows_of_zeros_and_of_large_values():
    c = Case(1, 8, 2, 1, 64, "layer", "interleaved", (64,))
    x = to_dev(c.x)
    x[0, 0] = 0
    x[0, 1] = 5.0          # no variance
    x[0, 2] *= 2.0 ** 60
    x[0, 3] *= 2.0 ** -60
    c.x = from_dev(x)
    check_forward(c, ta.head_rope(*c.parts(x), **c.args()))


def test_far_positions_keep_their_angles():
    """The same offsets around positions a billion apart give the same products of queries and keys, for
    frequencies whose period divides the distance."""
    d, n = 64, 1 << 28
    freqs = 2 * np.pi * np.arange(32) / 4096  # whole turns after 4096 positions
    rng = np.random.default_rng(5)
    x = to_dev(bits(rng, 1, 9, 2, d))
    got = []
    for base in (0, n, 7 * n):
        p = torch.arange(base, base + 9, dtype=torch.int32, device="cuda")[:, None]
        got.append(ta.head_rope(x, None, None, positions=p, freqs=gpu(freqs), layout="halves")[0].float())
    # fp64 turns: 2^31 * 2^-53 of a turn; results rounded to bf16 may differ by one step where they are at a border
    for a in got[1:]:
        assert ((a - got[0]).abs() <= 2.0 ** -7 * got[0].abs() + 1e-6).all()
        assert (a != got[0]).float().mean() < 1e-3


@pytest.mark.parametrize("norm,layout,dims,d", [("rms", "halves", (32, 32, 32), 96), ("layer", "interleaved", (64,), 64)])
def test_captured_and_replayed(norm, layout, dims, d):
    c = Case(2, 333, 6, 2, d, norm, layout, dims, lens=[333, 200])
    other = Case(2, 333, 6, 2, d, norm, layout, dims, lens=[333, 200], seed=9)
    x, dy, args = to_dev(c.x), [to_dev(g) for g in c.dy], c.args()
    q, k, v = c.parts(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ta.head_rope(q, k, v, **args)
        ta.head_rope_grad(q, k, v, *dy, **args)
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for _ in range(2):  # two graphs, each with its own workspace
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append((*ta.head_rope(q, k, v, **args), *ta.head_rope_grad(q, k, v, *dy, **args)))
        graphs.append(g)
    for inputs in (c, other, c):
        x.copy_(to_dev(inputs.x))
        for a, b in zip(dy, inputs.dy):
            a.copy_(to_dev(b))
        want = (*ta.head_rope(q, k, v, **args), *ta.head_rope_grad(q, k, v, *dy, **args))
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for out in outs:
            for a, b in zip(want, out):
                assert (a is None) == (b is None) and (a is None or torch.equal(a, b))


def test_on_another_stream_and_under_any_workspace_contents():
    c = Case(1, 700, 5, 5, 128, "rms", "split", (128,))
    x, dy, args = to_dev(c.x), [to_dev(g) for g in c.dy], c.args()
    q, k, v = c.parts(x)
    want = (*ta.head_rope(q, k, v, **args), *ta.head_rope_grad(q, k, v, *dy, **args))
    torch.full((1 << 24,), float("nan"), device="cuda")  # what the allocator hands on
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = (*ta.head_rope(q, k, v, **args), *ta.head_rope_grad(q, k, v, *dy, **args))
    s.synchronize()
    for a, b in zip(want, got):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))


@pytest.mark.parametrize("B,S,H,Hkv,d,norm,layout,dims,lens", [
    (1, 86400, 24, 24, 96, "rms", "halves", (32, 32, 32), None),         # pieces of 8: 72 heads a wave
    (1, 33001, 31, 8, 64, "layer", "interleaved", (16, 24, 24), None),   # neighbours: 47 heads, 12 a wave
    (2, 20003, 13, 3, 96, "layer", "split", (28, 34, 34), [20003, 9999]),  # anywhere: 19 heads, 18 and 1
    (1, 20001, 40, 8, 128, "rms", "halves", (44, 42, 42), None),         # anywhere: 56 heads
    (2, 9000, 9, 9, 128, "rms", "interleaved", (64,), [8999, 9000]),     # half of a head turned
    (1, 60000, 14, 2, 64, "layer", "halves", (20, 10), None)])
def test_whole_layers(B, S, H, Hkv, d, norm, layout, dims, lens):
    """Calls whose waves go through many heads, several steps of each kind and several items: every result and
    gradient against the formulas in 64 bits, a head at a time."""
    gen = torch.Generator(device="cuda").manual_seed(S + d)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    heads = H + 2 * Hkv
    x = torch.empty(B, S, heads, d, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    dy = [torch.empty(B, h, S, d, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for h in (H, Hkv, Hkv)]
    w = {n: 1 + 0.3 * rand(d) if n.endswith("weight") else 0.2 * rand(d) if norm == "layer" else None for n in WEIGHTS}
    p = torch.randint(0, 400, (S, len(dims)), generator=gen, device="cuda").to(torch.int32)
    how = dict(positions=p, freqs=ta.rope_freqs(dims), dims=dims, layout=layout, norm=norm, lens=gpu(lens, torch.int32), **w)
    parts = x.split_with_sizes([H, Hkv, Hkv], 2)
    got, grads = ta.head_rope(*parts, **how), ta.head_rope_grad(*parts, *dy, **how)

    # every value's partner, cosine and signed sine; 1 and 0 where it is not turned
    angle = torch.cat([p[:, a:a + 1].double() * f for a, f in enumerate(how["freqs"].split_with_sizes([n // 2 for n in dims]))], 1)
    partner = torch.arange(d, device="cuda")
    cos, sin = torch.ones(S, d, dtype=torch.float64, device="cuda"), torch.zeros(S, d, dtype=torch.float64, device="cuda")
    for i, (e0, e1, _) in enumerate(oh.pairs(dims, layout)):
        partner[e0], partner[e1] = e1, e0
        cos[:, e0] = cos[:, e1] = angle[:, i].cos()
        sin[:, e1] = angle[:, i].sin()
        sin[:, e0] = -sin[:, e1]
    turned = (sin != 0).any(0)
    with_partner = lambda m: m + torch.where(turned, m[..., partner], 0)  # noqa: E731
    valid = torch.ones(B, S, 1, dtype=torch.bool, device="cuda")
    for b, n in enumerate(lens or ()):
        valid[b, n:] = False

    def near(a, ref, room, what):
        off = (a.double() - ref).abs() - room
        assert off.max().item() <= 0, (what, off.max().item())

    for i, name in enumerate("qk"):
        weight, bias = (None if t is None else t.double() for t in (w[name + "_weight"], w[name + "_bias"]))
        sums = [0.0, 0.0, 0.0, 0.0]  # dw, db, and their terms' magnitudes
        for h in range(parts[i].shape[2]):
            row = torch.where(valid, parts[i][:, :, h].double(), 0)
            mean = row.mean(-1, keepdim=True) if norm == "layer" else 0.0
            r = ((row - mean).square().mean(-1, keepdim=True) + 1e-6).rsqrt()
            hat = (row - mean) * r
            wide = (row.abs() + row.abs().mean(-1, keepdim=True)) * r if norm == "layer" else hat.abs()
            n, mag = hat * weight, wide * weight.abs()
            if bias is not None:
                n, mag = n + bias, mag + bias.abs()
            y = torch.where(valid, n * cos + n[..., partner] * sin, 0)
            near(got[i][:, h], y, HALF * y.abs() + 2.0 ** -16 * with_partner(mag), name)
            g = torch.where(valid, dy[i][:, h].double(), 0)
            gm = with_partner(g.abs())
            g = g * cos + (g * sin)[..., partner]
            for j, term in enumerate((g * hat, g, gm * wide, gm)):
                sums[j] = sums[j] + term.sum((0, 1))
            u, um = g * weight, gm * weight.abs()
            dx = u - hat * (u * hat).mean(-1, keepdim=True) - (u.mean(-1, keepdim=True) if norm == "layer" else 0)
            room = r * (um + um.mean(-1, keepdim=True) + wide * (um * wide).mean(-1, keepdim=True))
            near(grads[i][:, :, h], dx * r, HALF * (dx * r).abs() + 2.0 ** -14 * room, "d" + name)
        near(grads[3 + i], sums[0], 2.0 ** -14 * sums[2], "dw")
        if bias is not None:
            near(grads[5 + i], sums[1], 2.0 ** -14 * sums[3], "db")
    keep = valid[:, None]
    assert torch.equal(got[2], torch.where(keep, parts[2].transpose(1, 2), 0))
    assert torch.equal(grads[2], torch.where(keep, dy[2], 0).transpose(1, 2))


def test_long_sums_keep_their_small_terms():
    """Sums over 26 million rows: a large term first in every lane's part, ones behind it. With rows of 1 and -1 normed rows
    are the rows themselves, and all terms are exact. Chains: 256 rows a lane, its 4 parts, 3 additions of lanes, 4 of
    waves, 64 and 16 of workgroups: 347 additions of 2^-24."""
    S, H, d, first = 131072, 200, 64, 32768
    one = torch.tensor([1.0, -1.0] * (d // 2), dtype=torch.bfloat16, device="cuda")
    g = torch.ones(1, H, S, d, dtype=torch.bfloat16, device="cuda")
    g[0, 0, :first] = 2.0 ** 24
    w = torch.ones(d, device="cuda")
    _, _, _, dw, _, db, _ = ta.head_rope_grad(one.expand(1, S, H, d), None, None, g, None, None, norm="layer", q_weight=w,
                                              q_bias=torch.zeros_like(w), eps=1e-30)
    want = first * 2.0 ** 24 + (S * H - first)
    for got, sign in ((dw, one.double()), (db, 1.0)):
        off = (got.double() * sign - want).abs().max().item()
        assert off <= 347 * 2.0 ** -24 * want, off / want


@pytest.mark.parametrize("layout,dims", [("halves", (128,)), ("split", (10, 36, 36))])
def test_offsets_past_32_bits(layout, dims):
    """A projection of more than 2^32 bytes, and results of as many: its last tokens as in a call of their own."""
    S, H, Hkv, d, last = 165000, 96, 4, 128, 77
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(1, S, H + 2 * Hkv, d, dtype=torch.bfloat16, device="cuda")
    assert x.numel() * 2 > 2 ** 32
    x.normal_(generator=gen)
    p = torch.randint(0, 1000, (S, len(dims)), generator=gen, device="cuda").to(torch.int32)
    how = dict(freqs=ta.rope_freqs(dims), dims=dims, layout=layout, norm="rms",
               q_weight=1 + 0.2 * torch.randn(d, generator=gen, device="cuda"))
    cut = lambda t: (t[:, :, :H], t[:, :, H:H + Hkv], t[:, :, H + Hkv:])  # noqa: E731
    got = ta.head_rope(*cut(x), positions=p, **how)
    tail = cut(x[:, S - last:])
    want = ta.head_rope(*tail, positions=p[S - last:].contiguous(), **how)
    for a, b in zip(got, want):
        assert torch.equal(a[:, :, S - last:], b)
    dx = ta.head_rope_grad(*cut(x), *got, positions=p, **how)
    part = ta.head_rope_grad(*tail, *want, positions=p[S - last:].contiguous(), **how)
    for a, b in zip(dx[:3], part[:3]):
        assert torch.equal(a[:, S - last:], b)


def test_the_functions_of_the_c_abi():
    c = Case(2, 30, 4, 2, 64, "layer", "split", (32, 16), lens=[30, 8])
    x, dy, args = to_dev(c.x), [to_dev(g) for g in c.dy], c.args()
    want = (*ta.head_rope(*c.parts(x), **args), *ta.head_rope_grad(*c.parts(x), *dy, **args))
    w = {n: args[n].data_ptr() for n in WEIGHTS}
    spec = ta.HeadRopeSpec(B=2, S=30, H=4, Hkv=2, d=64, norm=2, eps=1e-6, layout=3, axes=2, dims=(32, 16, 0, 0),
                           freqs=args["freqs"].data_ptr(), positions=args["positions"].data_ptr(), positions_batch=0,
                           lens=args["lens"].data_ptr(), **w)
    row = lambda t, h: ta.Rows(t.data_ptr() + 2 * 64 * h, 30 * 8 * 64, 8 * 64, 64)  # noqa: E731
    outs = [torch.empty_like(g) for g in dy]
    stream = torch.cuda.current_stream()
    ta.head_rope_fwd(spec, row(x, 0), row(x, 4), row(x, 6), *outs, stream)
    dx, sums = torch.empty_like(x), [torch.empty(64, device="cuda") for _ in range(4)]
    n = ta.head_rope_bwd_workspace(spec)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    ta.head_rope_bwd(spec, row(x, 0), row(x, 4), *dy, row(dx, 0), row(dx, 4), row(dx, 6), *sums, ws, n, stream)
    for a, b in zip(want, (*outs, *c.parts(dx), *sums)):
        assert torch.equal(a, b)
    with pytest.raises(ta.TileAttnError, match="workspace"):
        ta.head_rope_bwd(spec, row(x, 0), row(x, 4), *dy, row(dx, 0), row(dx, 4), row(dx, 6), *sums, ws, n - 1, stream)


def test_wrappers_refuse():
    c = Case(2, 10, 4, 2, 64, "rms", "halves", (64,))
    x, dy, args = to_dev(c.x), [to_dev(g) for g in c.dy], c.args()
    q, k, v = c.parts(x)

    def refused(match, f=ta.head_rope, t=(q, k, v), exc=ValueError, **kw):
        with pytest.raises(exc, match=match):
            f(*t, **{**args, **kw})

    refused("k must have the shape", t=(q, k[:, :5], v))
    refused("v must have the shape", t=(q, k, v[:, :, :1]))
    refused("must be torch.bfloat16", t=(q.float(), k, v))
    refused("last dimension", t=(q.transpose(2, 3).contiguous().transpose(2, 3), k, v))
    refused("GPU", t=(q, k.cpu(), v))
    refused("norm must be", norm="l2")
    refused("layout must be", layout="neox")
    refused("freqs must have the shape", freqs=args["freqs"][:-1].contiguous())
    refused("freqs must be", freqs=args["freqs"].float())
    refused("positions must have the shape", positions=args["positions"][:-1].contiguous())
    refused("positions must be", positions=args["positions"].long())
    refused("need freqs", freqs=None)
    refused("dims must name", dims=(16, 16, 16, 8, 8))
    refused("q_weight must have", q_weight=args["q_weight"][:32].contiguous())
    refused("k_weight must be", k_weight=args["k_weight"].double())
    refused("lens must be", lens=torch.zeros(2, device="cuda"))
    refused("biases need", exc=ta.TileAttnError, q_bias=args["q_weight"])
    refused("strides", exc=ta.TileAttnError, t=(torch.zeros(2 * 10 * 4 * 68, dtype=torch.bfloat16, device="cuda").as_strided((2, 10, 4, 64), (2720, 272, 68, 1)), k, v))
    refused("out must have", out=(q, k, v))
    refused("dq must have", f=ta.head_rope_grad, t=(q, k, v, dy[0][:, :2], dy[1], dy[2]))
    refused("go together", f=ta.head_rope_grad, t=(q, k, v, dy[0], dy[1], None))
    refused("overlap", f=ta.head_rope_grad, t=(q, k, v, *dy), exc=ta.TileAttnError, out=(q, k, v))
    with pytest.warns(UserWarning, match="not recorded"):
        ta.head_rope(q.detach().clone().requires_grad_(), k, v, **args)


def test_what_autograd_would_have_recorded_is_said():
    """Inputs that require a gradient, gradients that do, and tangents of forward mode: a warning each, and none where
    nothing would have been recorded."""
    import warnings

    import torch.autograd.forward_ad as fw

    c = Case(1, 6, 2, 1, 64, "rms", "halves", (64,))
    q, k, v = (x.contiguous() for x in c.parts(to_dev(c.x)))
    dy, args = [to_dev(g) for g in c.dy], c.args()
    at = dict(dtype=torch.int32, device="cuda")
    held = (*ta.cache4_new(1, 1, 64), torch.zeros(1, 1, **at), torch.zeros(1, **at))
    kt, qt = (torch.zeros(1, h, 3, 64, dtype=torch.bfloat16, device="cuda") for h in (1, 2))
    lists = torch.zeros(1, 1, 1, 1, **at)

    def calls(f):
        return [
            ("head_rope ", lambda: ta.head_rope(f(q), k, v, **args)), ("head_rope ", lambda: ta.head_rope(q, k, f(v), **args)),
            ("head_rope ", lambda: ta.head_rope(q, k, v, **{**args, "k_weight": f(args["k_weight"])})),
            ("head_rope_grad ", lambda: ta.head_rope_grad(q, k, v, dy[0], f(dy[1]), dy[2], **args)),
            ("cache4_write ", lambda: ta.cache4_write(f(kt), kt, *held, return_held=True)),
            ("cache4_write ", lambda: ta.cache4_write(kt, f(kt), *held, return_held=True)),
            ("cache4_attn ", lambda: ta.cache4_attn(f(qt), *held)),
            ("block_attn ", lambda: ta.block_attn(qt, f(kt), kt, lists))]

    for name, call in calls(lambda t: t.clone().requires_grad_()):
        with pytest.warns(UserWarning, match=name + "is not recorded"):
            call()
    with fw.dual_level():
        dual = calls(lambda t: fw.make_dual(t.clone(), torch.ones_like(t)))
        dual.append(("head_rope_grad ", lambda: ta.head_rope_grad(fw.make_dual(q, q.clone()), k, v, *dy, **args)))
        for name, call in dual:
            with pytest.warns(UserWarning, match=name + "is not recorded"):
                call()
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        for _, call in calls(lambda t: t):
            call()
        with fw.dual_level():
            for _, call in calls(lambda t: t):
                call()
        with torch.no_grad():
            for _, call in calls(lambda t: t.clone().requires_grad_()):
                call()
        ta.head_rope_grad(q.clone().requires_grad_(), k, v, *dy, **args)  # a program that goes back by itself
        ta.cache4_write(kt.clone().requires_grad_(), kt, *held)           # nothing comes back


@pytest.mark.parametrize("causal", [False, True])
def test_between_a_projection_and_attention(causal):
    """A layer's attention and its gradients: from the projection's output through norms, rotation, lists and
    attention, and back; against the reference of each step on the values before it."""
    from oracle import blocks as ob

    B, S, H, Hkv, d = 1, 300, 4, 2, 64
    c = Case(B, S, H, Hkv, d, "rms", "interleaved", (16, 24, 24))
    x, args = to_dev(c.x), c.args()
    parts = c.parts(x)
    q, k, v = ta.head_rope(*parts, **args)
    check_forward(c, (q, k, v))
    lists = ta.block_lists(q, ta.block_means(k), S, 2, causal=causal)
    out, lse = ta.block_attn(q, k, v, lists, causal=causal, return_lse=True)
    ref, *_ = ob.attention(from_dev(q), from_dev(k), from_dev(v), lists.cpu().numpy(), causal)
    assert np.abs(widen(from_dev(out)) - ref).max() <= 0.02
    dout = to_dev(bits(np.random.default_rng(1), B, H, S, d))
    c.dy = [from_dev(g) for g in ta.block_attn_grad(q, k, v, lists, out, dout, lse, causal=causal)]
    check_gradients(c, ta.head_rope_grad(*parts, *(to_dev(g) for g in c.dy), **args))


@pytest.mark.parametrize("P", [0, 37])
def test_between_a_projection_and_tile_attention(P):
    """The same with the fixed frame mask, with and without text before the video (at position 0, not turned): one
    projection and norm for both, the layout that the attention takes, and back."""
    from oracle import mmdit as om
    from tests.gpu_helpers import assert_parity

    B, H, d, F, h, w = 1, 3, 96, 4, 6, 11
    T, S = h * w, P + F * h * w
    c = Case(B, S, H, H, d, "rms", "halves", (32, 32, 32))
    c.positions = ta.grid_positions(F, h, w, P).cpu().numpy()
    x, args = to_dev(c.x), c.args()
    q, k, v = ta.head_rope(*c.parts(x), **args)
    check_forward(c, (q, k, v))
    mask, scale, stream = ta.tile_attn_make_mask(F, 1, "col"), d ** -0.5, torch.cuda.current_stream()
    out, lse = torch.empty_like(q), torch.empty(B, H, S, device="cuda")
    ta.tile_attn_fwd_mmdit(q, k, v, out, B, H, F, T, P, d, mask, scale, lse, stream)
    assert_parity(from_dev(out), om.attention_mmdit(from_dev(q), from_dev(k), from_dev(v), mask, T, P, scale), f"P = {P}")
    if P == 0:
        assert torch.equal(out, ta.tile_attn(q, k, v, mask, T))
    dout = to_dev(bits(np.random.default_rng(2), B, H, S, d))
    back = [torch.empty_like(q) for _ in range(3)]
    ta.tile_attn_bwd_mmdit(q, k, v, out, dout, lse, *back, B, H, F, T, P, d, mask, scale, stream)
    c.dy = [from_dev(g) for g in back]
    check_gradients(c, ta.head_rope_grad(*c.parts(x), *back, **args))
