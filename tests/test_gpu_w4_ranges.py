"""Products of 4-bit weights whose scales lie anywhere in fp32's range: results that fit are there, whatever a sum without the vector's power of two would be."""
import numpy as np
import pytest
import torch

import w4_reference as ref
from parity import np_
from test_gpu_w4 import _mat, _padded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q():
    import paper_1804_05038_amd as q
    return q


# rows, columns, vectors: up to 16 vectors in one launch (rows in one part and in several), then every form of the tiles (test_w4_delta_route has the rule)
FORMS = [(70, 400, 1), (70, 400, 5), (300, 1500, 16), (1500, 1100, 40), (700, 300, 150), (9000, 500, 90), (20000, 200, 50), (60000, 130, 66), (1300, 130, 1000), (12000, 300, 250), (16500, 150, 1000)]


@pytest.mark.parametrize("rows,cols,n", FORMS)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("kind", ["large", "mixed"])
def test_scales(q, rows, cols, n, group, kind):
    """large: scales of 2^96 to 2^122, vectors of 1e-27 to 1e3; mixed: each group's scale between 2^-104 and 2^122.  Judged where the magnitudes together stay
    below 2^127: no partial sum passes fp32's range there."""
    rng = np.random.default_rng(rows + cols + n + group)
    ng = -(-cols // group)
    codes, z = rng.integers(0, 16, (rows, cols)).astype(np.uint8), rng.integers(0, 16, (rows, ng)).astype(np.uint8)
    lo = 96 if kind == "large" else -104
    e = rng.integers(lo, 123, (rows, ng))
    e[::5] = rng.integers(-20, 20, (len(e[::5]), ng))                               # rows of everyday sizes between them
    s = np.ldexp(rng.integers(128, 256, (rows, ng)).astype(np.float32), e - 7)
    X = (rng.standard_normal((n, cols)) * 10.0 ** rng.uniform(-27, 3 if kind == "mixed" else -3, (n, 1))).astype(np.float32)
    X[0] = rng.standard_normal(cols).astype(np.float32) * np.float32(1e-20)
    b = rng.standard_normal(rows).astype(np.float32)
    ctx = q.Context(workspace_bytes=q.q8_gemm_w4_bytes(n, cols))
    got = np_(q.q8_gemm_w4(ctx, _mat(q, ctx, codes, s, z, group), _padded(ctx, X), ctx.f32(b))).astype(np.float64)
    wv = ref.values(codes, s, z, group)
    x = X.astype(np.float64)
    y = x @ wv.T + b
    fits = np.abs(x) @ np.abs(wv).T < 2.0 ** 127
    assert fits[0].sum() > rows // 3
    assert np.isfinite(got[fits]).all()
    assert (np.abs(got - y)[fits] <= ref.tolerance(wv, x, y, group)[fits]).all()


@pytest.mark.parametrize("rows,cols,n", FORMS)
@pytest.mark.parametrize("group", [32, 128])
def test_small_groups_beside_large_ones(q, rows, cols, n, group):
    """A vector without numbers in the columns of a row's large groups: the small ones count in full, as exactly as alone."""
    rng = np.random.default_rng(rows + n + group)
    ng = -(-cols // group)
    codes, z = rng.integers(0, 16, (rows, cols)).astype(np.uint8), rng.integers(0, 16, (rows, ng)).astype(np.uint8)
    large = np.arange(ng) % 2 == 0 if ng > 1 else np.zeros(1, bool)
    s = np.where(large, np.float32(2.0 ** 110), np.ldexp(rng.integers(128, 256, (rows, ng)).astype(np.float32), rng.integers(-104, -70, (rows, ng)) - 7)).astype(np.float32)
    X = rng.standard_normal((n, cols)).astype(np.float32) * np.float32(1e20)
    X[:, large[np.arange(cols) // group]] = 0.0
    ctx = q.Context(workspace_bytes=q.q8_gemm_w4_bytes(n, cols))
    got = np_(q.q8_gemm_w4(ctx, _mat(q, ctx, codes, s, z, group), _padded(ctx, X))).astype(np.float64)
    wv = np.where(large[np.arange(cols) // group], 0.0, ref.values(codes, s, z, group))
    x = X.astype(np.float64)
    y = x @ wv.T
    assert (np.abs(got - y) <= ref.tolerance(wv, x, y, group)).all()


@pytest.mark.parametrize("n", [4, 40])
def test_quantized_matrix_of_the_largest_weights(q, n):
    """A matrix of weights up to 3e38, quantized here."""
    rng = np.random.default_rng(n)
    W = (rng.uniform(-1, 1, (200, 300)) * 3e38).astype(np.float32)
    X = (rng.standard_normal((n, 300)) * 1e-20).astype(np.float32)
    ctx = q.Context(workspace_bytes=q.q8_gemm_w4_bytes(n, 300))
    m = q.q8_quantize_matrix_w4(ctx, ctx.f32(W), group=64)
    wv = ref.values(*ref.quantize(W, 64), 64)
    x = X.astype(np.float64)
    y = x @ wv.T
    assert (np.abs(np_(q.q8_gemm_w4(ctx, m, ctx.f32(X))) - y) <= ref.tolerance(wv, x, y, 64)).all()
