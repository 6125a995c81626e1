"""The float64 reference of attention over blocks and over the cache: against differences, against
plain masked attention, and its e4m3 codes against torch's."""
import numpy as np
import pytest

import workloads
from oracle import blocks as ob


def _bits(rng, *shape):
    return workloads.f32_to_bf16_bits(rng.standard_normal(shape).astype(np.float32))


@pytest.mark.parametrize("causal", [False, True])
def test_gradients_against_differences(causal):
    """The derivative along a random direction, from the formula and from the function's values at
    two points a step of 2^-8 apart on either side (inputs on a grid of 2^-8, so the step is exact
    in bf16): the quotient's own error is the third derivative times the step squared."""
    rng = np.random.default_rng(3)
    B, H, Hkv, S, d = 1, 2, 1, 150, 64
    lists = np.array([[[[0, -1], [1, 0]]]], np.int32)
    grid = lambda *s: np.round(rng.uniform(-0.5, 0.5, s) * 64) / 64  # noqa: E731
    q, k, v, go = grid(B, H, S, d), grid(B, Hkv, S, d), grid(B, Hkv, S, d), grid(B, H, S, d)
    lens = [140]

    def value(q, k, v):
        out, _, _ = ob.attention(*(ob.to_bf16(x) for x in (q, k, v)), lists, causal, lens)
        return float((out * go).sum())

    grads = ob.attention_backward(*(ob.to_bf16(x) for x in (q, k, v, go)), lists, causal, lens)
    for i, x in enumerate((q, k, v)):
        step = rng.integers(-1, 2, x.shape) * 2.0 ** -8
        plus, minus = ([y + s * step if j == i else y for j, y in enumerate((q, k, v))] for s in (1, -1))
        assert np.array_equal(ob.widen(ob.to_bf16(plus[i])), plus[i])
        diff = (value(*plus) - value(*minus)) / 2
        along = float((grads[i][0] * step).sum())
        assert abs(diff - along) <= 1e-3 * float((np.abs(grads[i][0]) * np.abs(step)).sum()), (i, diff, along)


def test_all_blocks_is_plain_attention_and_a_repeated_block_counts_once():
    rng = np.random.default_rng(4)
    q, k, v = _bits(rng, 1, 2, 200, 64), _bits(rng, 1, 2, 200, 64), _bits(rng, 1, 2, 200, 64)
    out, lse, _ = ob.attention(q, k, v, np.array([[[[1, 0, 1]] * 2] * 2], np.int32))
    s = ob.widen(q) @ ob.widen(k).transpose(0, 1, 3, 2) / 8
    p = np.exp(s - s.max(-1, keepdims=True))
    assert np.allclose(out, (p / p.sum(-1, keepdims=True)) @ ob.widen(v), atol=1e-12)
    assert np.allclose(lse, np.log(np.exp(s).sum(-1)), atol=1e-12)


def test_lists_take_forced_blocks_then_scores_then_the_lower_index():
    d = 64
    means = np.zeros((1, 1, 5, d))
    means[0, 0, :, 0] = [1.0, 3.0, 3.0, 2.0, -1.0]
    q = np.zeros((1, 1, 1, d))
    q[..., 0] = 1.0
    args = (ob.to_bf16(q), ob.to_bf16(means), 600)
    assert ob.block_lists(*args, 1, local=0).tolist() == [[[[1]]]]
    assert ob.block_lists(*args, 2, local=1).tolist() == [[[[1, 4]]]]  # the row lies in block 4
    assert ob.block_lists(*args, 3, sink=1, local=1).tolist() == [[[[0, 1, 4]]]]
    assert ob.block_lists(*args, 7, causal=True, local=1).tolist() == [[[[0, 1, 2, 3, 4, -1, -1]]]]
    assert ob.block_lists(*args, 2, lens=[599]).tolist() == [[[[-1, -1]]]]


def test_e4m3_codes_against_torch():
    torch = pytest.importorskip("torch")
    values = ob.e4m3_values()
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(values, t, equal_nan=True)
    x = np.concatenate([values[:127], (values[:126] + values[1:127]) / 2, np.linspace(0, 448, 3001)])
    x = np.concatenate([x, -x])
    got = torch.tensor(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ob.e4m3_codes(x), got)
    assert ob.e4m3_codes(np.array([np.inf, -np.inf, np.nan])).tolist() == [126, 254, 127]


def test_cache_write_and_attention_on_whole_numbers():
    """Codes, scales and results that can be worked out by hand."""
    k = ob.to_bf16(np.full((1, 1, 2, 64), 448.0))
    kp, vp = np.zeros((2, 1, 128, 64), np.uint8), np.zeros((2, 1, 64, 128), np.uint8)
    ks, vs = np.ones((2, 1), np.float32), np.ones((2, 1), np.float32)
    table = np.array([[1, 0]], np.int32)
    ob.cache_write(k, k, kp, vp, ks, vs, table, [127])
    # token 127 is the last of page 1 (which holds tokens, so scale max(1, 1)), token 128 starts page 0
    assert ks[1, 0] == 1 and ks[0, 0] == 1 and kp[1, 0, 127, 0] == 126 and kp[0, 0, 0, 0] == 126
    assert vp[1, 0, 0, 127] == 126 and vp[0, 0, 0, 0] == 126 and kp[1, 0, 126, 0] == 0
    ob.cache_write(ob.to_bf16(np.full((1, 1, 1, 64), 450.0)), k[:, :, :1], kp, vp, ks, vs, table, [129])
    assert ks[0, 0] == 2 and kp[0, 0, 0, 0] == ob.e4m3_codes(224.0) and vs[0, 0] == 1
    out, lse, _ = ob.cache_attention(ob.to_bf16(np.zeros((1, 1, 1, 64))), kp, vp, ks, vs, table, [130])
    assert np.allclose(out, 448 * 3 / 130) and np.allclose(lse, np.log(130))


def test_to_bf16_takes_the_nearest_number():
    """Every bf16 of a few binades, the ties between neighbours, and numbers 2^-40 beside those: nearer
    to a tie than float32 can tell."""
    bits = np.concatenate([s + np.arange(0x3F00, 0x4100) for s in (0, 0x8000)]).astype(np.uint16)
    assert np.array_equal(ob.to_bf16(ob.widen(bits)), bits)
    a, b = ob.widen(bits[:-1]), ob.widen(bits[1:])
    keep = (a > 0) == (b > 0)
    a, b, low = a[keep], b[keep], bits[:-1][keep]
    tie = (a + b) / 2
    assert np.array_equal(ob.to_bf16(tie), low + (low & 1))
    up = 1 + 2.0 ** -40
    assert np.array_equal(ob.to_bf16(tie * up), low + 1) and np.array_equal(ob.to_bf16(tie / up), low)
