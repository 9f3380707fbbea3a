"""GPU parity of 4-bit weights with group scales: codes and words equal the definition's, products are within what sums in fp32 may be off of
the values' products in 64 bits, and equal them where every partial sum is exact."""
import numpy as np
import pytest
import torch

import w4_reference as ref
from parity import np_

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q():
    import paper_1804_05038_amd as q
    return q


@pytest.fixture(scope="module")
def ctx(q):
    return q.Context(workspace_bytes=q.q8_workspace_bytes(max_n=1024, max_l=64, max_rows=8192, max_ld=2048))


def _random(rng, rows, cols):
    return (rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)) * 2)).astype(np.float32)


def _mat(q, ctx, codes, s, z, group):
    """A MatW4 of given codes, laid out by the definition."""
    rows, cols = codes.shape
    ld, lds = (cols + 127) // 128 * 64, (s.shape[1] + 3) // 4 * 4
    return q.MatW4(torch.from_numpy(ref.pack(codes, z, group, ld)).to(ctx.device), torch.from_numpy(ref.words(s, z, lds).view(np.int32)).to(ctx.device), cols, group)


# ---- quantization ----

@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 31), (2, 33), (5, 128), (2, 129), (7, 620), (4, 2048), (1, 16384), (130, 100)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_quantize(q, ctx, rows, cols, group):
    rng = np.random.default_rng(rows * 31 + cols + group)
    W = _random(rng, rows, cols)
    W[rng.random((rows, cols)) < 0.02] = 0.0
    m = q.q8_quantize_matrix_w4(ctx, ctx.f32(W), group=group)
    codes, s, z = ref.quantize(W, group)
    assert (np_(m.data) == ref.pack(codes, z, group, m.ld)).all()
    assert (np_(m.scale).view(np.uint32) == ref.words(s, z, m.scale.shape[1])).all()


def test_quantize_edges(q, ctx):
    """One sign only, one value, the largest range, tiny groups, ties, values that are not finite, each in a group of its own."""
    big = np.float32(3.4028235e38)
    rows = [[1.0, 2.0, 15.0], [-1.0, -2.0, -15.0], [0.25], [-0.25] * 32, [big, -big, 1e38], [2.0 ** -100], [-2.0 ** -100, 2.0 ** -101], [2.0 ** -101, -1e-45], [0.0, -0.0],
            list(np.arange(16) + 0.5), list(np.arange(-8, 8) + 0.5), [15.0, 0.5, 1.5, 2.5, 7.5], [np.nan, 1.0, -3.0], [np.inf, 2.0, -1.0], [-np.inf, 2.0, -1.0], [np.inf, -np.inf, np.nan],
            [15.0 * (1 + 2.0 ** -8), 1.0], [15.0 * (1 + 2.0 ** -7), 1.0], [np.nan], [np.inf, 2.0 ** -120]]
    W = np.zeros((len(rows), 70), np.float32)
    for i, r in enumerate(rows):
        W[i, :len(r)] = r[:32]
        W[i, 32:32 + len(r)] = r[:32]
    m = q.q8_quantize_matrix_w4(ctx, ctx.f32(W), group=32)
    codes, s, z = ref.quantize(W, 32)
    assert (ref.unpack(np_(m.data), 70) == codes).all()
    assert (np_(m.scale).view(np.uint32) == ref.words(s, z, m.scale.shape[1])).all()


@pytest.mark.parametrize("off,pitch,ld,lds", [(0, 133, 128, 8), (1, 132, 192, 8), (3, 301, 128, 16), (0, 400, 8192, 12)])
def test_quantize_pitches(q, ctx, off, pitch, ld, lds):
    """Rows that begin anywhere, pitches beyond the last block and group; nothing outside is written."""
    from paper_1804_05038_amd.binding import _MatW4
    import ctypes as C
    rows, cols, group, guard = 11, 130, 32, 64
    rng = np.random.default_rng(off + pitch)
    buf = torch.from_numpy(rng.standard_normal(off + rows * pitch + 8).astype(np.float32)).to(ctx.device)
    X = buf[off:off + rows * pitch].view(rows, pitch)[:, :cols]
    codes = torch.full((rows * ld + guard,), 0xAA, dtype=torch.uint8, device=ctx.device)
    scale = torch.full((rows * lds + guard,), 0x55, dtype=torch.int32, device=ctx.device)
    m = _MatW4(codes.data_ptr(), scale.data_ptr(), rows, cols, ld, lds, group)
    ctx.check(ctx.lib.q8_quantize_matrix_w4(ctx.handle, X.data_ptr(), rows, cols, pitch, C.byref(m)))
    c, s, z = ref.quantize(np_(X), group)
    assert (np_(codes)[:rows * ld].reshape(rows, ld) == ref.pack(c, z, group, ld)).all()
    assert (np_(scale).view(np.uint32)[:rows * lds].reshape(rows, lds) == ref.words(s, z, lds)).all()
    assert (np_(codes)[rows * ld:] == 0xAA).all() and (np_(scale)[rows * lds:] == 0x55).all()


# ---- products ----

SHAPES = [(1, 1, 1), (16, 16, 1), (15, 100, 2), (17, 127, 3), (768, 256, 1), (100, 128, 5), (63, 129, 8), (64, 255, 9), (65, 256, 15), (1000, 620, 16), (130, 512, 17),
          (300, 640, 31), (257, 1024, 33), (2500, 512, 5), (96, 2048, 48), (129, 1000, 64), (511, 130, 65), (333, 620, 128), (640, 384, 129), (768, 512, 257), (200, 4100, 40),
          (37, 16384, 1), (37, 16384, 7), (33, 16384, 70), (1030, 516, 300), (3000, 1000, 4), (20001, 32, 20), (5000, 8192, 1), (70, 8192, 2), (40000, 600, 3), (9000, 256, 1000)]


@pytest.mark.parametrize("rows,cols,n", SHAPES)
@pytest.mark.parametrize("group", [32, 64, 128])
def test_product(q, ctx, rows, cols, n, group):
    rng = np.random.default_rng(rows + 7 * cols + 11 * n + group)
    ng = -(-cols // group)
    codes, z = rng.integers(0, 16, (rows, cols)).astype(np.uint8), rng.integers(0, 16, (rows, ng)).astype(np.uint8)
    s = np.ldexp(rng.integers(128, 256, (rows, ng)).astype(np.float32), rng.integers(-14, -8, (rows, ng)))
    X = (rng.standard_normal((n, cols)) * np.exp(rng.standard_normal((n, 1)))).astype(np.float32)
    b = rng.standard_normal(rows).astype(np.float32) if (rows + n) % 2 else None
    pad = (cols + 3) // 4 * 4 + 4 * (n % 3)
    buf = torch.zeros(n, pad, device=ctx.device)
    buf[:, :cols] = torch.from_numpy(X)
    Y = torch.full((n, rows + n % 5), 7.0, device=ctx.device)
    tmp = ctx if n * cols <= 1 << 21 else q.Context(workspace_bytes=q.q8_gemm_w4_bytes(n, cols))
    q.q8_gemm_w4(tmp, _mat(q, ctx, codes, s, z, group), buf[:, :cols], ctx.f32(b) if b is not None else None, Y=Y[:, :rows])
    wv = ref.values(codes, s, z, group)
    y = np.asarray(X, np.float64) @ wv.T + (b if b is not None else 0.0)
    got = np_(Y)
    assert (got[:, rows:] == 7.0).all()
    assert (np.abs(got[:, :rows] - y) <= ref.tolerance(wv, X, y, group)).all()


@pytest.mark.parametrize("rows,cols,n", [(50, 300, 1), (50, 300, 16), (200, 700, 40), (300, 1024, 130)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_exact_products(q, ctx, rows, cols, n, group):
    """Whole numbers and powers of two whose partial sums fit 24 bits: every column, group, code and zero point has its own place."""
    rng = np.random.default_rng(rows + cols + n + group)
    ng = -(-cols // group)
    codes, z = rng.integers(0, 16, (rows, cols)).astype(np.uint8), rng.integers(0, 16, (rows, ng)).astype(np.uint8)
    s = np.ldexp(np.float32(1.0), rng.integers(0, 3, (rows, ng))).astype(np.float32)
    X = rng.integers(-50, 51, (n, cols)).astype(np.float32)
    Y = q.q8_gemm_w4(ctx, _mat(q, ctx, codes, s, z, group), _padded(ctx, X))
    assert (np_(Y) == X.astype(np.float64) @ ref.values(codes, s, z, group).T).all()


def _padded(ctx, X):
    n, cols = X.shape
    buf = torch.zeros(n, (cols + 3) // 4 * 4, device=ctx.device)
    buf[:, :cols] = torch.as_tensor(X)
    return buf[:, :cols]


@pytest.mark.parametrize("n", [4, 50])
def test_values_of_any_size(q, ctx, n):
    """Vectors whose values differ by many orders, the largest and smallest scales, zeros."""
    rng = np.random.default_rng(n)
    W = (rng.standard_normal((70, 400)) * np.exp(rng.standard_normal((70, 400)) * 6)).astype(np.float32)
    X = (rng.standard_normal((n, 400)) * np.exp(rng.standard_normal((n, 400)) * 6)).astype(np.float32)
    X[0] *= np.float32(1e30)
    X[1] *= np.float32(1e-27)
    X[2] = 0.0
    m = q.q8_quantize_matrix_w4(ctx, ctx.f32(W), group=64)
    wv = ref.values(*ref.quantize(W, 64), 64)
    y = np.asarray(X, np.float64) @ wv.T
    got = np_(q.q8_gemm_w4(ctx, m, ctx.f32(X)))
    # some results of the first vector are past fp32's range: no partial sum is where the magnitudes together stay below 2^127
    fits = np.abs(X).astype(np.float64) @ np.abs(wv).T < 2.0 ** 127
    assert fits[1:].all() and fits[0].any()
    assert (np.abs(got - y) <= ref.tolerance(wv, X, y, 64))[fits].all()
    assert (got[2] == 0.0).all()


@pytest.mark.parametrize("n", [3, 16, 70])
def test_a_value_that_is_not_finite_stays_with_its_vector(q, ctx, n):
    rng = np.random.default_rng(5)
    W, X = _random(rng, 90, 300), rng.standard_normal((n, 300)).astype(np.float32)
    m = q.q8_quantize_matrix_w4(ctx, ctx.f32(W), group=32)
    clean = np_(q.q8_gemm_w4(ctx, m, ctx.f32(X)))
    X[1, 7], X[2, 299] = np.nan, np.inf
    got = np_(q.q8_gemm_w4(ctx, m, ctx.f32(X)))
    keep = [j for j in range(n) if j not in (1, 2)]
    assert (got[keep] == clean[keep]).all()
    assert np.isnan(got[1]).all() and not np.isfinite(got[2]).any()


@pytest.mark.parametrize("n", [2, 40])
def test_what_lies_past_the_columns_does_not_count(q, ctx, n):
    """Codes past the columns, words past the last group and columns between the vectors: anything."""
    rng = np.random.default_rng(n)
    rows, cols, group = 60, 150, 32
    codes, s, z = ref.quantize(_random(rng, rows, cols), group)
    m = _mat(q, ctx, codes, s, z, group)
    X = rng.standard_normal((n, cols)).astype(np.float32)
    want = np_(q.q8_gemm_w4(ctx, m, _padded(ctx, X)))
    w = np_(m.data).view(np.uint32).copy()
    for k in range(cols, 256):
        b, t, g, e = k // 128, k % 128 // 32, k % 32 // 8, k % 8
        w[:, 16 * b + 4 * g + t] |= np.uint32(15) << np.uint32(4 * (e // 2) + 16 * (e % 2))
    sc = np_(m.scale).copy()
    sc[:, 5:] = np.array(np.nan, np.float32).view(np.int32)
    other = q.MatW4(torch.from_numpy(w.view(np.uint8)).to(ctx.device), torch.from_numpy(sc).to(ctx.device), cols, group)
    buf = torch.full((n, 152), float("nan"), device=ctx.device)
    buf[:, :cols] = torch.from_numpy(X)
    assert (np_(q.q8_gemm_w4(ctx, other, buf[:, :cols])) == want).all()


@pytest.mark.parametrize("n", [1, 8, 60])
def test_results_over_the_vectors(q, ctx, n):
    rng = np.random.default_rng(n)
    m = q.q8_quantize_matrix_w4(ctx, ctx.f32(_random(rng, 256, 256)))
    X = ctx.f32(rng.standard_normal((n, 256)).astype(np.float32))
    x = np_(X).astype(np.float64)
    apart = np_(q.q8_gemm_w4(ctx, m, X))
    q.q8_gemm_w4(ctx, m, X, Y=X)
    wv = ref.values(ref.unpack(np_(m.data), 256), *_words(m), 128)
    y = x @ wv.T
    for got in (apart, np_(X)):
        assert (np.abs(got - y) <= ref.tolerance(wv, x, y, 128)).all()


def _words(m):
    w = np_(m.scale).view(np.uint32)[:, :-(-m.cols // m.group)]
    return (w & np.uint32(0xFFFF0000)).view(np.float32), (w & 15).astype(np.uint8)


@pytest.mark.parametrize("n", [5, 40])
def test_captured_and_replayed(q, n):
    """A product and a quantization in a graph on a stream of its own, replayed with other inputs and eager work between."""
    st = torch.cuda.Stream()
    ctx = q.Context(workspace_bytes=q.q8_gemm_w4_bytes(n, 640), stream=st)
    rng = np.random.default_rng(n)
    W, X = ctx.f32(_random(rng, 500, 640)), ctx.f32(rng.standard_normal((n, 640)).astype(np.float32))
    torch.cuda.synchronize()
    quant = q.q8_quantize_matrix_w4(ctx, W, group=64, bind=True)
    prod = q.q8_gemm_w4(ctx, quant.out["W"], X, bind=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        quant.launch()
        prod.launch()
    for t in range(4):
        W.copy_(torch.from_numpy(_random(rng, 500, 640)))
        X.copy_(torch.from_numpy(rng.standard_normal((n, 640)).astype(np.float32)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = np_(prod.out["Y"]).copy()
        quant.launch()
        prod.launch()
        torch.cuda.synchronize()
        assert (got == np_(prod.out["Y"])).all() and np.isfinite(got).all()
        wv = ref.values(*ref.quantize(np_(W)[:40], 64), 64)
        y = np_(X).astype(np.float64) @ wv.T
        assert (np.abs(got[:, :40] - y) <= ref.tolerance(wv, np_(X), y, 64)).all()


@pytest.mark.parametrize("n,k", [(1, 0), (5, 12), (20, 5), (100, 0)])
def test_output_layer(q, ctx, n, k):
    """From hidden vectors given: logits, their log-sum-exp and the best words."""
    rng = np.random.default_rng(n + k)
    V, R = 3001, 256
    W, b = _random(rng, V, R) * np.float32(0.05), rng.standard_normal(V).astype(np.float32)
    t = np.tanh(rng.standard_normal((n, R))).astype(np.float32)
    m = q.q8_quantize_matrix_w4(ctx, ctx.f32(W), group=64)
    r = q.output_logits_w4(ctx, None, m, ctx.f32(b), t_in=ctx.f32(t), k=k)
    wv = ref.values(*ref.quantize(W, 64), 64)
    y = np.asarray(t, np.float64) @ wv.T + b
    lg = np_(r["logits"])
    assert (np.abs(lg - y) <= ref.tolerance(wv, t, y, 64)).all()
    if k:
        lse = np.log(np.exp(lg - lg.max(1, keepdims=True)).sum(1)) + lg.max(1)
        assert np.abs(np_(r["lse"]) - lse).max() <= 1e-5 * max(1.0, np.abs(lse).max())
        order = np.lexsort((np.broadcast_to(np.arange(V), lg.shape), -lg), axis=1)[:, :k]
        assert (np_(r["topk_idx"]) == order).all()


@pytest.mark.parametrize("n", [3, 30])
def test_output_layer_with_its_first_layer(q, ctx, n):
    """With the readout's matrices the logits are those of the hidden vectors that the call returns."""
    rng = np.random.default_rng(n)
    V, R, H = 2000, 128, 64
    mat = lambda r, c: q.q8_quantize_matrix(ctx, rng.standard_normal((r, c)).astype(np.float32) * 0.1)
    ro = q.ReadoutWeights(mat(R, H), mat(R, H), mat(R, H), ctx.f32(rng.standard_normal(R).astype(np.float32)))
    m = q.q8_quantize_matrix_w4(ctx, ctx.f32(_random(rng, V, R)), group=32)
    x = [ctx.f32(rng.standard_normal((n, H)).astype(np.float32)) for _ in range(3)]
    r = q.output_logits_w4(ctx, ro, m, None, s=x[0], y_emb=x[1], ctx_vec=x[2], k=4)
    again = q.output_logits_w4(ctx, None, m, None, t_in=r["t"], k=4)
    plain = q.output_logits_q8(ctx, ro, q.q8_quantize_matrix(ctx, rng.standard_normal((V, R)).astype(np.float32)), None, s=x[0], y_emb=x[1], ctx_vec=x[2], k=4)
    assert (np_(r["t"]) == np_(plain["t"])).all()
    for f in ("logits", "lse", "topk_logp", "topk_idx"):
        assert (np_(r[f]) == np_(again[f])).all()
