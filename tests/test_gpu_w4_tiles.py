"""Every kernel that the rule on sizes (csrc/q8_route.h) chooses for products of 4-bit weights, with stores past the caches and through them; that these
sizes are all of its forms is checked in test_w4_delta_route.py."""
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


# (rows, columns, vectors) by form
TILES = {
    "stream": [(70, 400, 3), (3001, 130, 16), (40000, 300, 5), (300, 4000, 4)],
    "32x32, four groups of waves": [(1500, 1100, 40), (500, 770, 260), (33, 4100, 17)],
    "64x32, four": [(700, 300, 150), (5000, 1000, 90), (250, 500, 1000)],
    "64x32, two": [(20000, 400, 20), (1030, 1300, 900), (9000, 500, 65)],
    "128x32": [(60000, 130, 20), (9000, 100, 130), (20000, 600, 50)],
    "128x64": [(12000, 500, 250), (41001, 300, 60), (50000, 100, 40)],
    "128x96": [(41001, 300, 65), (42000, 500, 77), (50000, 130, 96)],
    "256x64": [(16500, 200, 1000), (50001, 520, 330)],
}
CASES = [(form, *size) for form, sizes in TILES.items() for size in sizes]


def _inputs(rng, rows, cols, group):
    ng = -(-cols // group)
    return rng.integers(0, 16, (rows, cols)).astype(np.uint8), rng.integers(0, 16, (rows, ng)).astype(np.uint8)


def _results(ctx, n, rows, past):
    """[n x rows] with pitches of whole 64 bytes or odd ones, and numbers beside them."""
    pitch = -(-rows // 16) * 16 + 16 if past else rows + 3 | 1
    return torch.full((n, pitch), 7.0, device=ctx.device)


@pytest.mark.parametrize("form,rows,cols,n", CASES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("past", [True, False])
def test_whole_numbers(q, form, rows, cols, n, group, past):
    """Whole numbers and powers of two whose partial sums fit 24 bits (at most 15 x 4 x 8 a column): every
    column, group, code, zero point and vector has its own place, and each result is exact."""
    rng = np.random.default_rng(rows + cols + n + group)
    codes, z = _inputs(rng, rows, cols, group)
    s = np.ldexp(np.float32(1.0), rng.integers(0, 3, z.shape)).astype(np.float32)
    X = rng.integers(-8, 9, (n, cols)).astype(np.float32)
    assert 15 * 4 * 8 * cols < 2 ** 24
    b = rng.integers(-100, 101, rows).astype(np.float32)
    ctx = q.Context(workspace_bytes=q.q8_gemm_w4_bytes(n, cols))
    Y = _results(ctx, n, rows, past)
    q.q8_gemm_w4(ctx, _mat_fast(q, ctx, codes, s, z, group), _padded(ctx, X), ctx.f32(b), Y=Y[:, :rows])
    got = np_(Y)
    assert (got[:, rows:] == 7.0).all()
    want = X @ _values32(codes, s, z, group).T + b              # (exact in 32 bits, in any order)
    assert (got[:, :rows] == want).all()


@pytest.mark.parametrize("form,rows,cols,n", CASES)
@pytest.mark.parametrize("group", [32, 64, 128])
def test_any_numbers(q, form, rows, cols, n, group):
    rng = np.random.default_rng(rows + 3 * cols + n + group)
    codes, z = _inputs(rng, rows, cols, group)
    s = np.ldexp(rng.integers(128, 256, z.shape).astype(np.float32), rng.integers(-14, -8, z.shape))
    X = (rng.standard_normal((n, cols)) * np.exp(rng.standard_normal((n, 1)))).astype(np.float32)
    ctx = q.Context(workspace_bytes=q.q8_gemm_w4_bytes(n, cols))
    Y = _results(ctx, n, rows, n % 2 == 0)
    q.q8_gemm_w4(ctx, _mat_fast(q, ctx, codes, s, z, group), _padded(ctx, X), Y=Y[:, :rows])
    keep = rng.permutation(rows)[:2000]                         # (rows whose results are formed in 64 bits)
    wv = ref.values(codes[keep], s[keep], z[keep], group)
    x = X.astype(np.float64)
    y = x @ wv.T
    assert (np.abs(np_(Y)[:, keep] - y) <= ref.tolerance(wv, x, y, group)).all()


def _values32(codes, s, z, group):
    at = np.arange(codes.shape[1]) // group
    return (codes.astype(np.float32) - z[:, at]) * s[:, at]


def _mat_fast(q, ctx, codes, s, z, group):
    """_mat, of matrices that are too large to be packed column by column: 16-bit halves of a word by whole arrays."""
    rows, cols = codes.shape
    nb = -(-cols // 128)
    full = np.zeros((rows, nb, 4, 4, 4, 2), np.uint32)          # block, t, g, j, e: column 128 b + 32 t + 8 g + 2 j + e
    full.reshape(rows, -1)[:, :cols] = codes
    shift = (4 * np.arange(4)[:, None] + 16 * np.arange(2)[None, :]).astype(np.uint32)
    words = (full << shift).sum((4, 5), dtype=np.uint32).transpose(0, 1, 3, 2)          # word 4 g + t
    data = np.ascontiguousarray(words).view(np.uint8).reshape(rows, 64 * nb)
    sc = ref.words(s, z, (s.shape[1] + 3) // 4 * 4).view(np.int32)
    return q.MatW4(torch.from_numpy(data).to(ctx.device), torch.from_numpy(sc).to(ctx.device), cols, group)


@pytest.mark.parametrize("rows,cols,group", [(5, 100, 32), (7, 300, 64), (3, 129, 128)])
def test_fast_packing_is_the_definitions(q, rows, cols, group):
    rng = np.random.default_rng(cols)
    codes, z = _inputs(rng, rows, cols, group)
    s = np.ones(z.shape, np.float32)
    ctx = q.Context(workspace_bytes=1 << 20)
    a, b = _mat_fast(q, ctx, codes, s, z, group), _mat(q, ctx, codes, s, z, group)
    assert (ref.unpack(np_(a.data), cols) == codes).all() and (ref.unpack(np_(b.data), cols) == codes).all() and (np_(a.scale) == np_(b.scale)).all()
