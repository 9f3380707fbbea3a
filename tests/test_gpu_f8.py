"""GPU parity of the 8-bit floating point operators: codes and scales equal the definition's, products are within what sums
in fp32 may be off of the values' products in 64 bits, and equal them where every partial sum is exact."""
import numpy as np
import pytest
import torch

import f8_reference as ref
from parity import np_

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q():
    import paper_1804_05038_amd as q
    return q


@pytest.fixture(scope="module")
def ctx(q):
    return q.Context(workspace_bytes=q.q8_workspace_bytes(max_n=1024, max_l=64, max_rows=8192, max_ld=2048))


def _same_codes(got, want):
    """Equal codes, any NaN for a NaN."""
    g, w = ref.VALUES[got], ref.VALUES[want]
    assert ((g == w) | (np.isnan(g) & np.isnan(w))).all(), "%d codes differ" % (~((g == w) | (np.isnan(g) & np.isnan(w)))).sum()


# ---- quantization ----

@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 3), (3, 127), (5, 128), (2, 129), (33, 620), (7, 5), (300, 2048), (1, 16384), (4097, 256), (9, 1000)])
def test_quantize(q, ctx, rows, cols):
    rng = np.random.default_rng(rows * 31 + cols)
    X = (rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)) * 4)).astype(np.float32)
    X[rng.random((rows, cols)) < 0.02] = 0.0
    m = q.q8_quantize_matrix_f8(ctx, ctx.f32(X))
    codes, scale = ref.quantize(X)
    assert (np_(m.scale_rows) == scale).all()
    _same_codes(np_(m.data), codes)
    assert not np_(m.data)[:, cols:].any()


def test_quantize_edges(q, ctx):
    """Ties, the largest value of a scale, tiny and huge blocks, values that are not finite, each in a block of its own."""
    f = ref.VALUES[(ref.VALUES >= 0)]
    rows = [np.concatenate([(f[:-1] + f[1:]) / 2, [448.0]]), np.concatenate([-(f[:-1] + f[1:]) / 2 * 2.0 ** -90, [448 * 2.0 ** -90]]),
            [448.0, 447.9], [np.nextafter(np.float32(448), np.float32(500)), 1.0], [3.4028235e38, -1e30, 1.0], [2.0 ** -100, -2.0 ** -108], [2.0 ** -101, 1e-45],
            [0.0, -0.0], [np.nan, 1.0, -3.0], [np.inf, 2.0, -np.inf], [np.inf, np.nan], [np.inf, 2.0 ** -120, 1e-44]]
    X = np.zeros((len(rows), 300), np.float32)
    for i, r in enumerate(rows):
        X[i, :min(len(r), 128)] = r[:128]
        X[i, 128:128 + len(r)] = r[:172][:128]
    m = q.q8_quantize_matrix_f8(ctx, ctx.f32(X))
    codes, scale = ref.quantize(X)
    assert (np_(m.scale_rows) == scale).all()
    _same_codes(np_(m.data), codes)


def test_blocks_of_zeros_have_codes_of_zero(q, ctx):
    """Blocks below 2^-100 in all places, negative ones too: bytes of zero; zeros of other blocks keep their sign."""
    X = np.zeros((4, 300), np.float32)
    X[0] = -0.0
    X[1] = -2.0 ** -101
    X[2, ::2] = -1e-45
    X[3, :128] = -1e-38
    X[3, 128:] = -0.0
    X[3, 200] = 1.0
    m = q.q8_quantize_matrix_f8(ctx, ctx.f32(X))
    c = np_(m.data)
    assert not c[:3].any() and not c[3, :128].any() and not c[3, 256:].any()
    assert (np_(m.scale)[:, 0] == 127).all()
    want = np.full(128, 0x80, np.uint8)
    want[200 - 128] = ref.e4m3_round(256.0)
    assert (c[3, 128:256] == want).all()


@pytest.mark.parametrize("off,pitch,ld_out,lds", [(0, 133, 144, 4), (1, 132, 144, 4), (3, 301, 512, 8), (0, 400, 384, 12), (2, 130, 16384, 128)])
def test_quantize_pitches(q, ctx, off, pitch, ld_out, lds):
    """Rows that begin anywhere, a pitch of codes and of scales beyond the last block; nothing outside is written."""
    rows, cols = 11, 130
    rng = np.random.default_rng(off + pitch)
    buf = torch.from_numpy(rng.standard_normal(off + rows * pitch + 8).astype(np.float32)).to(ctx.device)
    X = buf[off:off + rows * pitch].view(rows, pitch)[:, :cols]
    guard = 64
    codes = torch.full((rows * ld_out + guard,), 0xAA, dtype=torch.uint8, device=ctx.device)
    scale = torch.full((rows * lds + guard,), 0xAA, dtype=torch.uint8, device=ctx.device)
    ctx.check(ctx.lib.q8_quantize_matrix_f8(ctx.handle, X.data_ptr(), rows, cols, pitch, codes.data_ptr(), ld_out, scale.data_ptr(), lds))
    c, s = ref.quantize(np_(X), ld_out, lds)
    _same_codes(np_(codes)[:rows * ld_out].reshape(rows, ld_out), c)
    assert (np_(scale)[:rows * lds].reshape(rows, lds) == s).all()
    assert (np_(codes)[rows * ld_out:] == 0xAA).all() and (np_(scale)[rows * lds:] == 0xAA).all()


# ---- products ----

def _tolerance(wv, xv, y):
    """Sums of K exact products in fp32, in an order that the matrix cores choose: at most K - 1 additions see a product, each
    off by at most 2^-23 of a partial sum (2^-24 where they round to nearest; they need not), and no partial sum exceeds the
    sum of the magnitudes; one more for the bias."""
    K = wv.shape[1]
    return (K + 1) * 2.0 ** -23 * (np.abs(xv) @ np.abs(wv).T) + 2.0 ** -23 * np.abs(y)


SHAPES = [(1, 1, 1), (16, 16, 1), (15, 100, 2), (17, 127, 3), (768, 256, 1), (100, 128, 5), (63, 129, 8), (64, 255, 9), (65, 256, 15), (1000, 620, 16),
          (130, 512, 17), (300, 640, 31), (257, 1024, 33), (2500, 512, 5), (96, 2048, 48), (129, 1000, 64), (511, 130, 65), (1024, 2048, 100), (333, 620, 128),
          (640, 384, 129), (260, 16, 200), (768, 512, 257), (200, 4100, 40), (37, 16384, 7), (37, 16384, 70), (1030, 516, 300), (2050, 900, 1000), (3000, 1000, 4), (50000, 512, 5),
          (520, 1100, 513), (20001, 32, 20), (8192, 128, 1024)]


@pytest.mark.parametrize("rows,cols,n", SHAPES)
@pytest.mark.parametrize("codes", [False, True])
def test_product(q, ctx, rows, cols, n, codes):
    rng = np.random.default_rng(rows * 7 + cols * 3 + n)
    W = (rng.standard_normal((rows, cols)) * 0.05 * np.exp(rng.standard_normal((rows, 1)))).astype(np.float32)
    X = np.tanh(rng.standard_normal((n, (cols + 3) // 4 * 4))).astype(np.float32)
    b = rng.standard_normal(rows).astype(np.float32)
    M = q.q8_quantize_matrix_f8(ctx, ctx.f32(W))
    c = ctx if codes else q.Context(workspace_bytes=q.q8_gemm_f8_bytes(n, cols))
    x = ctx.f32(X)[:, :cols]
    Y = q.q8_gemm_f8(c, M, q.q8_quantize_matrix_f8(c, x) if codes else x, ctx.f32(b))
    wv, xv = ref.values(*ref.quantize(W), cols), ref.values(*ref.quantize(X[:, :cols]), cols)
    want = xv @ wv.T + b.astype(np.float64)
    err = np.abs(np_(Y) - want)
    assert (err <= _tolerance(wv, xv, want)).all(), "worst %.3g of the tolerance" % (err / _tolerance(wv, xv, want)).max()


@pytest.mark.parametrize("rows,cols,n", [(100, 620, 3), (64, 512, 16), (70, 2048, 20), (300, 1030, 64), (260, 640, 130), (513, 512, 600), (900, 384, 2100),
                                          (3300, 2100, 4200), (2900, 1100, 2900), (16500, 300, 77), (52000, 260, 77), (16100, 260, 129), (512, 4100, 17), (500, 8200, 1), (37, 16384, 1),
                                          (2050, 2000, 3), (3000, 1000, 4), (20000, 1200, 2), (40000, 1100, 4), (33000, 130, 16)])
def test_product_of_whole_numbers_is_exact(q, ctx, rows, cols, n):
    """Codes of whole numbers up to 8 and scales of powers of two up to 4: every sum is exact in fp32, in any order."""
    rng = np.random.default_rng(rows + cols + n)
    nb = -(-cols // 128)
    Wi, Xi = rng.integers(-8, 9, (rows, cols)), rng.integers(-8, 9, (n, cols))

    def mat(v):
        c = np.zeros((len(v), -(-cols // 16) * 16), np.uint8)
        c[:, :cols] = ref.e4m3_round(v)
        s = np.full((len(v), -(-nb // 4) * 4), 127, np.uint8)
        s[:, :nb] = rng.integers(125, 130, (len(v), nb))
        return q.MatF8(torch.from_numpy(c).to(ctx.device), torch.from_numpy(s).to(ctx.device), cols), ref.values(c, s, cols)

    W, wv = mat(Wi)
    X, xv = mat(Xi)
    assert (np_(q.q8_gemm_f8(ctx, W, X)) == xv @ wv.T).all()


@pytest.mark.parametrize("rows,cols,n", [(49300, 620, 77), (65500, 513, 96), (50000, 1100, 65), (65537, 620, 77), (49152, 620, 96), (90000, 530, 70)])
def test_products_of_65_to_96_vectors(q, ctx, rows, cols, n):
    """On both sides of where they go in tiles of 128 x 96: whole numbers, every sum exact."""
    rng = np.random.default_rng(rows + n)
    Wi, Xi = rng.integers(-8, 9, (rows, cols)).astype(np.float32), rng.integers(-8, 9, (n, cols)).astype(np.float32)
    Wi[:, ::128], Xi[:, ::128] = 8.0, -8.0               # every block has the same scale, and every whole number up to 8 a code
    b = rng.integers(-99, 100, rows).astype(np.float32)
    W = q.q8_quantize_matrix_f8(ctx, ctx.f32(Wi))
    assert (np_(q.q8_gemm_f8(ctx, W, q.q8_quantize_matrix_f8(ctx, ctx.f32(Xi)), ctx.f32(b))) == Xi @ Wi.T + b).all()


@pytest.mark.parametrize("rows,cols,n", [(70, 200, 3), (70, 200, 20), (130, 300, 70), (300, 256, 300)])
@pytest.mark.parametrize("off", [0, 1])
def test_product_leaves_the_rest_of_y(q, ctx, rows, cols, n, off):
    """A pitch of Y that is no multiple of four and results that begin between 16-byte boundaries; nothing else is written."""
    rng = np.random.default_rng(rows + n)
    W = q.q8_quantize_matrix_f8(ctx, ctx.f32(rng.standard_normal((rows, cols)).astype(np.float32)))
    x = ctx.f32(rng.standard_normal((n, cols)).astype(np.float32))
    plain = np_(q.q8_gemm_f8(ctx, W, x))
    pitch = rows + 7
    buf = torch.full((n + 2, pitch), 123.0, device=ctx.device)
    flat = buf.view(-1)
    Y = flat[off:off + n * pitch].view(n, pitch)[:, :rows]
    q.q8_gemm_f8(ctx, W, x, Y=Y)
    assert (np_(Y) == plain).all()
    Y.fill_(123.0)
    assert bool((buf == 123.0).all())


def test_product_keeps_nan_where_it_is(q, ctx):
    for n in (3, 40, 300):
        rng = np.random.default_rng(n)
        W, X = rng.standard_normal((200, 256)).astype(np.float32), rng.standard_normal((n, 256)).astype(np.float32)
        X[1, 7], W[150, 130] = np.nan, np.inf
        Y = np_(q.q8_gemm_f8(ctx, q.q8_quantize_matrix_f8(ctx, ctx.f32(W)), ctx.f32(X)))
        bad = np.zeros((n, 200), bool)
        bad[1], bad[:, 150] = True, True
        assert (np.isnan(Y) == bad).all()


def test_product_of_extreme_scales(q, ctx):
    for n in (2, 50, 200):
        W, X = np.zeros((40, 256), np.float32), np.zeros((n, 256), np.float32)
        W[:, 0], X[:, 0] = 2.0 ** 100, 2.0 ** -99           # 2
        W[:, 130], X[:, 130] = 2.0 ** -100, 2.0 ** 101      # 2
        W[3, 0], X[1, 0] = 2.0 ** 120, 2.0 ** 120           # past fp32's range
        Y = np_(q.q8_gemm_f8(ctx, q.q8_quantize_matrix_f8(ctx, ctx.f32(W)), ctx.f32(X)))
        want = X.astype(np.float64) @ W.T.astype(np.float64)
        with np.errstate(over="ignore"):
            assert (Y == want.astype(np.float32)).all()


@pytest.mark.parametrize("n", [1, 3, 16, 17, 70, 300])
@pytest.mark.parametrize("cols", [100, 620, 1300])
def test_scale_bytes_past_the_last_block_do_not_count(q, ctx, n, cols):
    """1, 5 and 11 blocks of columns: what stands in the rest of a row's scales changes nothing, in either operand."""
    rng = np.random.default_rng(cols + n)
    nb = -(-cols // 128)
    W = q.q8_quantize_matrix_f8(ctx, ctx.f32(rng.standard_normal((300, cols)).astype(np.float32)))
    X = q.q8_quantize_matrix_f8(ctx, ctx.f32(rng.standard_normal((n, cols)).astype(np.float32)))
    want = np_(q.q8_gemm_f8(ctx, W, X)).copy()
    for byte in (0, 1, 254, 255):
        for m in (W, X):
            m.scale_rows[:, nb:] = byte
        assert (np_(q.q8_gemm_f8(ctx, W, X)) == want).all(), byte


@pytest.mark.parametrize("n", [2, 40, 200])
@pytest.mark.parametrize("byte,other", [(3, 230), (246, 40)])
def test_the_smallest_and_the_largest_scale_hold_every_code(q, ctx, n, byte, other):
    """Every code times every scale from 3 to 246 is a bf16 value: 2^-9 2^(3 - 127) = 2^-133, the smallest there is, and 448 2^(246 - 127) < 2^128.
    One product a result, exact in fp32."""
    codes = np.array([c for c in range(256) if c & 127 != 127], np.uint8)
    W, X = np.zeros((len(codes), 128), np.uint8), np.zeros((n, 128), np.uint8)
    W[:, 77] = codes
    X[:, 77] = ref.e4m3_round(np.where(np.arange(n) % 2, 1.0, -1.5))
    sw, sx = np.full((len(codes), 4), byte, np.uint8), np.full((n, 4), other, np.uint8)
    dev = lambda c, s: q.MatF8(torch.from_numpy(c).to(ctx.device), torch.from_numpy(s).to(ctx.device), 128)
    want = ref.values(X, sx, 128) @ ref.values(W, sw, 128).T
    assert (np_(q.q8_gemm_f8(ctx, dev(W, sw), dev(X, sx))) == want).all()


def test_product_over_its_vectors(q, ctx):
    """Results that overwrite the vectors they are made of."""
    for n in (2, 16, 90):
        rng = np.random.default_rng(n)
        W = q.q8_quantize_matrix_f8(ctx, ctx.f32(rng.standard_normal((512, 512)).astype(np.float32)))
        x = ctx.f32(rng.standard_normal((n, 512)).astype(np.float32))
        want = np_(q.q8_gemm_f8(ctx, W, x))
        q.q8_gemm_f8(ctx, W, x, Y=x)
        assert (np_(x) == want).all()


def test_product_of_a_matrix_with_itself(q, ctx):
    W = np.random.default_rng(0).standard_normal((300, 300)).astype(np.float32)
    M = q.q8_quantize_matrix_f8(ctx, ctx.f32(W))
    v = ref.values(*ref.quantize(W), 300)
    want = v @ v.T
    assert (np.abs(np_(q.q8_gemm_f8(ctx, M, M)) - want) <= _tolerance(v, v, want)).all()


def test_results_past_32_bit_offsets(q, ctx):
    rows, n, cols = 65600, 33000, 16
    rng = np.random.default_rng(1)
    W, X = rng.standard_normal((rows, cols)).astype(np.float32), rng.standard_normal((n, cols)).astype(np.float32)
    M, xc = q.q8_quantize_matrix_f8(ctx, ctx.f32(W)), q.q8_quantize_matrix_f8(ctx, ctx.f32(X))
    Y = q.q8_gemm_f8(ctx, M, xc)
    wv, xv = ref.values(*ref.quantize(W), cols), ref.values(*ref.quantize(X), cols)
    for rs, js in ((slice(0, 70), slice(0, 70)), (slice(rows - 70, rows), slice(n - 70, n)), (slice(0, 70), slice(n - 70, n)), (slice(30000, 30100), slice(32700, 32800))):
        want = xv[js] @ wv[rs].T
        assert (np.abs(np_(Y[js, rs]) - want) <= _tolerance(wv[rs], xv[js], want)).all()


def test_results_repeat_and_replay(q, ctx):
    """The same bits on every run, and from a graph replayed with the program's own work between the replays."""
    rng = np.random.default_rng(3)
    for n in (4, 60, 400):
        W = q.q8_quantize_matrix_f8(ctx, ctx.f32(rng.standard_normal((1500, 700)).astype(np.float32)))
        x = ctx.f32(rng.standard_normal((n, 700)).astype(np.float32))
        # (the matrix cores' sums need not be odd: the negated vectors have results of their own)
        want = [q.q8_gemm_f8(ctx, W, v).clone() for v in (x, -x)]
        stream = torch.cuda.Stream()
        c = q.Context(workspace_bytes=q.q8_gemm_f8_bytes(n, 700), stream=stream)
        Y = ctx.empty(n, 1500)
        xin = torch.zeros_like(x)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            q.q8_gemm_f8(c, W, xin, Y=Y)
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            q.q8_gemm_f8(c, W, xin, Y=Y)
        for k in range(3):
            xin.copy_(x if k != 1 else -x)
            Y.zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert bool((Y == want[k == 1]).all()), k
            assert bool((q.q8_gemm_f8(ctx, W, x) == want[0]).all())


def test_two_streams_at_once(q):
    rng = np.random.default_rng(9)
    base = q.Context()
    W = q.q8_quantize_matrix_f8(base, base.f32(rng.standard_normal((9000, 512)).astype(np.float32)))
    xs = [base.f32(rng.standard_normal((40, 512)).astype(np.float32)) for _ in range(2)]
    want = [q.q8_gemm_f8(q.Context(workspace_bytes=q.q8_gemm_f8_bytes(40, 512)), W, x).clone() for x in xs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    cs = [q.Context(workspace_bytes=q.q8_gemm_f8_bytes(40, 512), stream=s) for s in streams]
    Ys = [base.empty(40, 9000) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, x, y in zip(cs, xs, Ys):
            q.q8_gemm_f8(c, W, x, Y=y)
    torch.cuda.synchronize()
    assert all(bool((y == w).all()) for y, w in zip(Ys, want))


def test_refusals(q, ctx):
    """What the binding refuses (the library's own refusals: test_f8_refusals.py, on the host)."""
    W = q.q8_quantize_matrix_f8(ctx, ctx.f32(np.ones((32, 64), np.float32)))
    x = ctx.f32(np.ones((4, 64), np.float32))
    for bad in (lambda: q.q8_gemm_f8(ctx, W, x[:, :60]), lambda: q.q8_gemm_f8(ctx, W, x, Y=ctx.empty(4, 33)), lambda: q.q8_gemm_f8(ctx, W, x, Y=ctx.empty(3, 32)),
                lambda: q.q8_gemm_f8(ctx, W, x, ctx.empty(31)), lambda: q.q8_gemm_f8(ctx, W, x.double()), lambda: q.q8_gemm_f8(ctx, W, ctx.empty(64, 4).t())):
        with pytest.raises(ValueError):
            bad()
    for bad in (dict(t_in=x[:, :60].contiguous()), dict(t_in=x.double()), dict(t_in=x.cpu()), dict(t_in=ctx.empty(64, 4).t()), dict(t_in=x, logits=ctx.empty(4, 33)), dict(t_in=x, logits=ctx.empty(3, 32))):
        with pytest.raises(ValueError):
            q.output_logits_f8(ctx, None, W, None, k=4, **bad)
    small = q.Context(workspace_bytes=q.q8_gemm_f8_bytes(1, 64))
    with pytest.raises(q.Q8Error) as e:                   # 400 vectors of 64 codes, a workspace for one
        q.q8_gemm_f8(small, W, ctx.empty(400, 64))
    assert e.value.code == 4
    q.q8_gemm_f8(ctx, W, x)
    torch.cuda.synchronize()


# ---- the output layer ----

@pytest.mark.parametrize("n,V,R,k", [(1, 5000, 64, 12), (5, 3333, 620, 12), (8, 2000, 512, 16), (9, 4001, 128, 5), (70, 2050, 640, 12), (5, 70000, 64, 0), (40, 700, 512, 0)])
@pytest.mark.parametrize("readout", [False, True])
def test_output_layer(q, ctx, n, V, R, k, readout):
    """The first layer is output_logits_q8's, the logits are the product of its t, and the k best are those of the logits."""
    from parity import gpu_mat
    rng = np.random.default_rng(V + n)
    c = q.Context(workspace_bytes=q.q8_workspace_bytes(max_n=max(n, 8), max_l=64, max_rows=V, max_ld=1024))
    W = q.q8_quantize_matrix_f8(ctx, ctx.f32((rng.standard_normal((V, R)) * 0.2).astype(np.float32)))
    b = ctx.f32(rng.standard_normal(V).astype(np.float32))
    H, E, Cd = 96, 64, 192
    f = lambda *s: ctx.f32(rng.standard_normal(s).astype(np.float32))
    if readout:
        ro = q.ReadoutWeights(gpu_mat(q, ctx, rng.standard_normal((R, H)).astype(np.float32) * 0.1), gpu_mat(q, ctx, rng.standard_normal((R, E)).astype(np.float32) * 0.1),
                              gpu_mat(q, ctx, rng.standard_normal((R, Cd)).astype(np.float32) * 0.1), f(R))
        s, y, cv = f(n, H), f(n, E), f(n, Cd)
        o = q.output_logits_f8(c, ro, W, b, s, y, cv, k=k)
        some = q.q8_quantize_matrix(ctx, rng.standard_normal((64, R)).astype(np.float32))
        t = q.output_logits_q8(c, ro, some, None, s, y, cv, k=1)["t"]
        assert bool((o["t"] == t).all())
    else:
        t = torch.tanh(f(n, R))
        o = q.output_logits_f8(c, None, W, b, t_in=t, k=k)
    assert bool((o["logits"] == q.q8_gemm_f8(c, W, t, b)).all())
    if k == 0:
        assert o["lse"] is None
        return
    lg = np_(o["logits"]).astype(np.float64)
    m = lg.max(1)
    lse = m + np.log(np.exp(lg - m[:, None]).sum(1))
    order = np.argsort(-lg, axis=1, kind="stable")[:, :k]
    assert (np_(o["topk_idx"]) == order).all()
    # exponentials of 2^-22 each, sums in double, one rounding
    assert (np.abs(np_(o["lse"]) - lse) <= 2.0 ** -22 + 2.0 ** -24 * np.abs(lse)).all()
    lp = np.take_along_axis(lg, order, 1) - lse[:, None]
    assert (np.abs(np_(o["topk_logp"]) - lp) <= 2.0 ** -22 + 2.0 ** -23 * (np.abs(lse)[:, None] + np.abs(lp))).all()
    # the same without keeping the logits
    if readout:
        o2 = q.output_logits_f8(c, ro, W, b, s, y, cv, k=k, want_logits=False)
    else:
        o2 = q.output_logits_f8(c, None, W, b, t_in=t, k=k, want_logits=False)
    assert o2["logits"] is None and bool((o2["topk_idx"] == o["topk_idx"]).all()) and bool((o2["topk_logp"] == o["topk_logp"]).all())
