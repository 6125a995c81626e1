"""The float64 reference of the 4-bit cache: its numbers, roundings and scales by hand."""
import numpy as np

import workloads
from oracle import blocks as ob
from oracle import cache4 as o4


def test_the_numbers():
    x = np.concatenate([o4.GRID, -o4.GRID])
    assert np.array_equal(o4.nearest(x), np.arange(16))
    # every tie goes to the even code
    ties = (o4.GRID[1:] + o4.GRID[:-1]) / 2
    assert o4.nearest(ties).tolist() == [0, 2, 2, 4, 4, 6, 6]
    assert o4.nearest([7.0, 100.0, 5.01, 4.99, 0.2499, -0.2501]).tolist() == [7, 7, 7, 6, 0, 9]


def test_scales_are_the_least_that_hold():
    for a, e in ((7.0, 0), (7.01, 1), (3.5, -1), (3.51, 0), (1e-40, -100), (0.0, -100), (3.38e38, 125)):
        assert o4.exponent(np.array([a, -a / 2])) == e, a
    # what lies between 6 and 7 goes to 6: no further off than half the step from 4 to 6
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 32))
    for g in x:
        e = o4.exponent(g)
        got = o4.GRID[o4.nearest(g / 2.0 ** e) & 7] * 2.0 ** e
        assert np.abs(got - np.abs(g)).max() <= 2.0 ** e


def new(rng, pages, Hkv, d):
    return [rng.integers(0, 256, s).astype(np.uint8) for s in ((pages, Hkv, 128, d // 2),) * 2 + ((pages, Hkv, d // 32, 128),) * 2]


def test_written_tokens_read_back_and_leave_others_alone():
    rng = np.random.default_rng(1)
    k, v = (workloads.f32_to_bf16_bits(rng.standard_normal((2, 2, 130, 64)).astype(np.float32)) for _ in range(2))
    v[1, 0, 3, 5] = 0x7F80  # an infinity marks the token's key
    cache = new(rng, 6, 2, 64)
    before = [x.copy() for x in cache]
    table = np.array([[4, 1, -1], [0, 5, 2]], np.int32)
    held = o4.write(k, v, *cache, table, [7, 100], [130, 90])
    back = o4.read(*cache, table, [137, 190], 90, first=100)
    assert np.array_equal(back[:, 1], held[:, 1, :, :90], equal_nan=True) and not held[:, 1, :, 90:].any()
    assert np.array_equal(back[:, 0, :, :37], held[:, 0, :, 93:130]) and not back[:, 0, :, 37:].any()
    assert np.isnan(held[0, 1, 0, 3]).all() and held[1, 1, 0, 3, 5] == 0 and np.isfinite(held[1]).all()
    ok = np.isfinite(held[0])
    x = ob.widen(k)
    room = np.abs(x).reshape(2, 2, 130, 2, 32).max(-1, keepdims=True) * (2 / 7)  # 2^e at a largest value above 3.5 * 2^e
    wrote = np.zeros((2, 2, 130, 64), bool)
    wrote[0], wrote[1, :, :90] = True, True
    assert (np.abs(held[0] - x) <= np.broadcast_to(room, (2, 2, 130, 2, 32)).reshape(x.shape) + 1e-30)[ok & wrote].all()
    for a, b in zip(cache, before):
        assert np.array_equal(a[3], b[3]) and np.array_equal(a[2], b[2])
    assert np.array_equal(cache[0][4, :, :7], before[0][4, :, :7])
    assert np.array_equal(cache[2][4, :, :, :7], before[2][4, :, :, :7])
    assert np.array_equal(cache[2][1, :, :, 9:], before[2][1, :, :, 9:])


def test_attention_over_one_page_by_hand():
    rng = np.random.default_rng(2)
    cache = new(rng, 2, 1, 64)
    for s in cache[2:]:
        s[...] = rng.integers(124, 128, s.shape)
    q = workloads.f32_to_bf16_bits(rng.standard_normal((1, 2, 2, 64)).astype(np.float32))
    out, lse, _ = o4.attention(q, *cache, np.array([[1]]), [3])
    k, v = o4.values(cache[0][1, 0], cache[2][1, 0]), o4.values(cache[1][1, 0], cache[3][1, 0])
    for h in range(2):
        for t in range(2):
            s = k[:t + 2] @ ob.widen(q)[0, h, t] / 8
            p = np.exp(s - s.max())
            assert np.allclose(out[0, h, t], p @ v[:t + 2] / p.sum())
            assert np.isclose(lse[0, h, t], np.log(p.sum()) + s.max())
