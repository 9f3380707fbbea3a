"""CPU pins of the plain definitions that the GPU tests of 4-bit weights and of the gated delta rule compare with."""
import numpy as np
import pytest

import delta_reference as delta
import w4_reference as w4


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("cols", [1, 31, 100, 128, 300])
def test_memory_order_goes_there_and_back(group, cols):
    rng = np.random.default_rng(cols)
    codes, z = rng.integers(0, 16, (5, cols)).astype(np.uint8), rng.integers(0, 16, (5, -(-cols // group))).astype(np.uint8)
    ld = (cols + 127) // 128 * 64
    data = w4.pack(codes, z, group, ld)
    assert data.shape == (5, ld) and (w4.unpack(data, cols) == codes).all()
    # a block's word 4 g + t: columns 32 t + 8 g and up; column 2 j + e at bit 4 j + 16 e
    one = np.zeros((1, 128), np.uint8)
    one[0, 32 * 2 + 8 * 3 + 5] = 9
    word = w4.pack(one, np.zeros((1, 4), np.uint8), 32, 64).view(np.uint32)[0]
    assert word[4 * 3 + 2] == 9 << (4 * 2 + 16) and np.count_nonzero(word) == 1


@pytest.mark.parametrize("group", [32, 64, 128])
def test_values_are_within_half_a_step(group):
    """Within half a step of every weight, and a whole one at the two ends (where the rounded zero point moves the range); zeros exact."""
    rng = np.random.default_rng(group)
    W = (rng.standard_normal((40, 300)) * np.exp(rng.standard_normal((40, 1)) * 5)).astype(np.float32)
    W[:, ::17] = 0.0
    codes, s, z = w4.quantize(W, group)
    v = w4.values(codes, s, z, group)
    step = s.astype(np.float64)[:, np.arange(300) // group]
    inside = (codes > 0) & (codes < 15)
    assert (np.abs(v - W)[inside] <= 0.5000001 * step[inside]).all() and (np.abs(v - W) <= 1.0000001 * step).all()
    assert (v[:, ::17] == 0.0).all()
    assert ((s.view(np.uint32) & 0xFFFF) == 0).all()


def test_scales_are_the_least_that_hold_the_range():
    """(hi - lo) / 15 in eight significant bits, from below and above."""
    for lo, hi, want in ((0.0, 15.0, 1.0), (-15.0, 0.0, 1.0), (-7.5, 7.5, 1.0), (0.0, 15.0 * (1 + 2.0 ** -7), 1 + 2.0 ** -7), (0.0, 15.0 * (1 + 2.0 ** -8), 1 + 2.0 ** -7),
                         (0.0, 3.75, 0.25), (0.0, 0.0, 1.0), (0.0, 2.0 ** -101, 1.0)):
        _, s, z = w4.quantize(np.array([[lo, hi]], np.float32), 32)
        assert s[0, 0] == np.float32(want), (lo, hi)
        assert z[0, 0] == (np.rint(-lo / want) if max(hi, -lo) >= 2.0 ** -100 else 0)


def test_the_rule_by_hand():
    """One head of 1 x 1: S = a S; S += k b (v - k S); o = q S."""
    one = lambda x: np.array(x, np.float32).reshape(-1, 1, 1)
    gate = lambda x: np.array(x, np.float32).reshape(-1, 1)
    o, s = delta.sequence(one([2.0, 1.0]), one([1.0, 1.0]), one([3.0, 5.0]), gate([0.0, np.log(0.5)]), gate([0.5, 1.0]), [0, 2], normalize=False)
    assert np.allclose(o[:, 0, 0], [2 * 1.5, 5.0], rtol=1e-7) and np.allclose(s, 5.0, rtol=1e-7)


def test_open_gates_store_what_a_key_is_asked_for():
    """With b = 1, no decay and orthogonal keys every value comes back for its key; the last value of a key wins."""
    d = 8
    k = np.eye(d, dtype=np.float32)[:, None, :]
    v = np.random.default_rng(0).standard_normal((d, 1, 5)).astype(np.float32)
    kk, vv = np.concatenate([k, k]), np.concatenate([v, 2 * v])
    ones, zeros = np.ones((2 * d, 1), np.float32), np.zeros((2 * d, 1), np.float32)
    o, s = delta.sequence(kk, kk, vv, zeros, ones, [0, 2 * d], normalize=False)
    assert np.allclose(o, vv, atol=1e-12) and np.allclose(s[0, 0], 2 * v[:, 0], atol=1e-12)


def test_bounds_hold_for_sums_in_32_bits():
    """The rule token by token in fp32 is within the bounds that the GPU's chunks are held to."""
    rng = np.random.default_rng(1)
    f = lambda *s: rng.standard_normal(s).astype(np.float32)
    N, hk, hv, dk, dv, off = 50, 1, 2, 16, 12, [0, 33, 50]
    x = dict(q=f(N, hk, dk), k=f(N, hk, dk), v=f(N, hv, dv), g=-np.abs(f(N, hv)), beta=1 / (1 + np.exp(-f(N, hv))))
    qn, kn = (t.astype(np.float32) for t in delta.prepared(x["q"], x["k"], 1.0, True, 2))
    out, ends = np.zeros((N, hv, dv), np.float32), []
    for s in range(2):
        S = np.zeros((hv, dk, dv), np.float32)
        for t in range(off[s], off[s + 1]):
            S, out[t] = delta.token(S, qn[t], kn[t], x["v"][t], np.exp(x["g"][t]), x["beta"][t])
        ends.append(S)
    assert S.dtype == np.float32
    want, bound = delta.sequence(**x, off=off), delta.sequence_bound(**x, off=off)
    assert (np.abs(out - want[0]) <= bound[0]).all() and (np.linalg.norm(np.stack(ends) - want[1], axis=2) <= bound[1]).all()
