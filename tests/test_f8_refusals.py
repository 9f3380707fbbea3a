"""CPU checks that the library's entry points for 8-bit floating point and for drawing refuse bad arguments before they
launch anything.  The context is host memory laid out as q8_internal.h has it (stream, workspace, its size, error text; all
else zero) and no pointer is ever followed: a call that got as far as a launch would return Q8_ERR_DEVICE (5) here, where
there is no device."""
import ctypes as C
import struct

import pytest
import torch

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up: only where nothing can be launched")

NULL, SHAPE, ALIGN, WORKSPACE, DEVICE = 1, 2, 3, 4, 5
P = 0x10000                                             # an aligned address


@pytest.fixture()
def lib():
    import paper_1804_05038_amd as q
    return q.load_library()


def context(ws_bytes):
    mem = C.create_string_buffer(4096)
    mem[:24] = struct.pack("QQQ", 0, 1 << 20, ws_bytes)
    return mem


def mat(**k):
    from paper_1804_05038_amd.binding import _MatF8
    d = dict(data=P, scale=P, rows=32, cols=64, ld=64, lds=4)
    d.update(k)
    return C.byref(_MatF8(*[d[f] for f in ("data", "scale", "rows", "cols", "ld", "lds")]))


BAD_MATS = [(dict(data=None), NULL), (dict(scale=None), NULL), (dict(rows=0), SHAPE), (dict(rows=-1), SHAPE), (dict(rows=(1 << 24) + 1), SHAPE), (dict(cols=0), SHAPE),
            (dict(cols=65), SHAPE), (dict(ld=63), SHAPE), (dict(ld=16400), SHAPE), (dict(lds=0), SHAPE), (dict(cols=600, ld=608), SHAPE), (dict(ld=72), ALIGN), (dict(lds=6), ALIGN),
            (dict(data=P + 8), ALIGN), (dict(scale=P + 2), ALIGN)]


def test_good_calls_reach_the_launch(lib):
    c = context(1 << 30)
    assert lib.q8_quantize_matrix_f8(c, P, 4, 64, 64, P, 64, P, 4) == DEVICE
    assert lib.q8_gemm_f8(c, mat(), P, 4, 64, None, P, 32) == DEVICE
    assert lib.q8_gemm_codes_f8(c, mat(), mat(rows=4), None, P, 32) == DEVICE
    assert lib.output_logits_f8(c, None, mat(), None, None, None, None, P, 4, 0, P, None, None, None, None) == DEVICE
    assert lib.q8_sample_logits(c, P, 4, 100, 100, None, P, P, None, None, 0, None) == DEVICE


@pytest.mark.parametrize("bad,want", BAD_MATS)
def test_matrices(lib, bad, want):
    c = context(1 << 30)
    assert lib.q8_gemm_f8(c, mat(**bad), P, 4, 64, None, P, 64) == want
    assert lib.q8_gemm_codes_f8(c, mat(**bad), mat(), None, P, 64) == want
    assert lib.q8_gemm_codes_f8(c, mat(), mat(**bad), None, P, 64) == want
    assert lib.output_logits_f8(c, None, mat(**bad), None, None, None, None, P, 4, 0, P, None, None, None, None) == want
    d = dict(data=P, scale=P, rows=32, cols=64, ld=64, lds=4)
    d.update(bad)
    assert lib.q8_quantize_matrix_f8(c, P, d["rows"], d["cols"], 16384, d["data"], d["ld"], d["scale"], d["lds"]) == want


def test_products(lib):
    c = context(lib.q8_gemm_f8_bytes(4, 64))
    call = lambda x=P, n=4, ldx=64, b=None, y=P, ldy=32: lib.q8_gemm_f8(c, mat(), x, n, ldx, b, y, ldy)
    assert lib.q8_gemm_f8(c, None, P, 4, 64, None, P, 32) == NULL and call(x=None) == NULL and call(y=None) == NULL
    assert call(n=0) == call(n=-3) == call(n=(1 << 20) + 1) == call(ldx=60) == call(ldy=31) == SHAPE
    assert call(ldx=66) == call(x=P + 4) == call(y=P + 2) == call(b=P + 1) == ALIGN
    assert call(n=1 << 20) == call(n=100) == WORKSPACE
    assert call() == call(n=1, ldx=0, ldy=0) == DEVICE
    assert lib.q8_gemm_codes_f8(c, mat(), mat(cols=60), None, P, 32) == SHAPE
    assert lib.q8_gemm_codes_f8(c, mat(rows=1 << 24), mat(rows=1 << 20), None, P, 1 << 24) == SHAPE     # 2^44 results
    assert lib.q8_gemm_codes_f8(c, mat(), mat(rows=(1 << 20) + 1), None, P, 32) == SHAPE


def test_quantization(lib):
    c = context(1 << 20)
    call = lambda x=P, rows=4, cols=64, ld=64: lib.q8_quantize_matrix_f8(c, x, rows, cols, ld, P, 64, P, 4)
    assert call(x=None) == NULL and call(ld=63) == SHAPE and call(x=P + 2) == ALIGN and call(x=P + 4) == DEVICE


def test_output_layer(lib):
    c = context(1 << 30)
    call = lambda w=None, t=P, n=4, k=0, lg=P, lp=None, idx=None, to=None, b=None: lib.output_logits_f8(c, None, w or mat(), b, None, None, None, t, n, k, lg, None, lp, idx, to)
    assert call(t=None) == call(lg=None) == call(k=3) == call(k=3, lp=P) == NULL
    assert call(n=0) == call(n=1025) == call(k=-1) == call(k=17, lp=P, idx=P) == call(w=mat(rows=8), k=9, lp=P, idx=P) == call(w=mat(rows=65537), k=4, lp=P, idx=P) == SHAPE
    assert call(w=mat(cols=62)) == call(t=P + 4) == call(lg=P + 1) == call(b=P + 2) == call(to=P + 8) == ALIGN
    small = context(300000)
    assert lib.output_logits_f8(small, None, mat(rows=60000), None, None, None, None, P, 8, 4, None, None, P, P, None) == WORKSPACE
    from paper_1804_05038_amd.binding import _Mat, _Readout
    m = lambda rows=64, cols=96, ld=96: _Mat(P, rows, cols, ld, 1.0, None)
    ro = lambda a=None, b=None, d=None: C.byref(_Readout(a or m(), b or m(), d or m(), None))
    full = lambda r, s=P, y=P, v=P, n=4: lib.output_logits_f8(c, r, mat(), None, s, y, v, None, n, 0, P, None, None, None, None)
    assert full(ro()) == full(ro(), n=40) == DEVICE
    assert full(ro(), s=None) == full(ro(), y=None) == full(ro(), v=None) == full(ro(a=_Mat(None, 64, 96, 96, 1.0, None))) == NULL
    assert full(ro(a=m(rows=63))) == full(ro(b=m(cols=97))) == full(ro(d=m(cols=8016, ld=8016)), n=8) == full(ro(a=m(cols=9000, ld=9008)), n=8) == SHAPE
    assert full(ro(a=m(cols=94))) == full(ro(), s=P + 4) == full(ro(), v=P + 8) == ALIGN


def test_draws(lib):
    from paper_1804_05038_amd.binding import _Sampling
    c = context(lib.q8_sample_bytes(4, 100))
    call = lambda lg=P, n=4, V=100, ld=100, s=None, u=P, tok=P, lp=None, e=None, E=0, y=None: lib.q8_sample_logits(c, lg, n, V, ld, s, u, tok, lp, e, E, y)
    assert call(lg=None) == call(u=None) == call(tok=None) == call(e=P, E=8) == call(y=P, E=8) == NULL
    assert call(n=0) == call(n=65537) == call(V=0) == call(V=(1 << 24) + 1, ld=1 << 25) == call(ld=99) == call(e=P, E=0, y=P) == SHAPE
    assert call(lg=P + 2) == call(u=P + 1) == call(tok=P + 2) == call(lp=P + 2) == call(e=P + 1, E=8, y=P) == ALIGN
    assert call(V=9000, ld=9000) == WORKSPACE and lib.q8_sample_bytes(4, 9000) > lib.q8_sample_bytes(4, 100)
    for k in range(4):
        assert call(s=C.byref(_Sampling(*[P + 2 if i == k else None for i in range(4)]))) == ALIGN
    assert call() == call(s=C.byref(_Sampling(P, P, P, P)), e=P, E=8, y=P, lp=P) == call(n=1, ld=0) == DEVICE


def _up(v):
    return -(-v // 256) * 256


@pytest.mark.parametrize("n,l,rows,ld", [(1, 1, 1000, 512), (8, 64, 65536, 2048), (60, 50, 50000, 1024), (1024, 64, 50000, 2048), (1024, 1, 2049, 512), (5, 1, 1 << 24, 1024)])
def test_workspace_of_callers_who_draw_nothing(lib, n, l, rows, ld):
    """Drawing and 8-bit floating point lay their room out over that of the other calls: nothing on top of it at a model's sizes."""
    nv, tiles, header = max(n, l), -(-rows // 16), 262144
    others = header + _up(nv * ld) + _up(nv * 4) + 2 * _up(l * rows * 4) + 8 * _up(n * rows * 4) + _up(n * l * 4) + _up(tiles * n * 4) + _up(tiles * n * 8) + 65536
    assert lib.q8_workspace_bytes(n, l, rows, ld) == others


@pytest.mark.parametrize("n", [1, 8, 9, 300, 1024])
@pytest.mark.parametrize("V,R,H", [(1, 16384, 16), (16, 16, 1024), (100, 64, 7000), (3000, 620, 1000), (70000, 512, 1024)])
def test_workspace_is_enough(lib, n, V, R, H):
    """q8_workspace_bytes: every call succeeds at the sizes that it was asked for."""
    from paper_1804_05038_amd.binding import _Mat, _Readout
    ld = lambda c: -(-c // 16) * 16
    ro = C.byref(_Readout(*[_Mat(P, R, H, ld(H), 1.0, None)] * 3, None))
    w = mat(rows=V, cols=R, ld=ld(R), lds=-(-R // 512) * 4)
    k = min(V, 12)
    plain = context(lib.q8_workspace_bytes(n, 1, V, ld(R)))
    whole = context(lib.q8_workspace_bytes(n, 1, max(V, R), max(ld(R), ld(H))))
    for logits in (P, None):
        for kk in (0, k) if logits else (k,):
            if kk and V > 65536:
                continue
            assert lib.output_logits_f8(plain, None, w, None, None, None, None, P, n, kk, logits, None, P, P, None) == DEVICE
            if R <= 1024 and (n > 8 or 3 * n * ld(H) <= 65536):
                assert lib.output_logits_f8(whole, ro, w, None, P, P, P, None, n, kk, logits, None, P, P, None) == DEVICE
    assert lib.q8_gemm_f8(plain, w, P, n, -(-R // 4) * 4, None, P, V) == DEVICE
    assert lib.q8_sample_logits(plain, P, n, V, V, None, P, P, None, None, 0, None) == DEVICE


def test_more_than_a_launch_holds(lib):
    """Blocks of 256 threads, 32 blocks of columns or bytes of scales each: 2^32 threads are one too many.  (Wider pitches of the scales
    had the number of blocks cut to 32 bits.)"""
    c = context(1 << 20)
    call = lambda rows, lds: lib.q8_quantize_matrix_f8(c, P, rows, 1, 1, P, 16, P, lds)
    assert call((1 << 24) - 1, 32) == call(1 << 24, 28) == call(1 << 15, 16380) == DEVICE
    assert call(1 << 24, 32) == call(1 << 24, 8196) == call(1 << 24, 16384) == call(1 << 23, 64) == SHAPE
    # products: tiles of 128 x 64 in 512 threads
    many = lambda rows, n: lib.q8_gemm_codes_f8(c, mat(rows=rows), mat(rows=n), None, P, rows)
    assert many(1 << 24, 4032) == DEVICE and many(1 << 24, 4160) == many(1 << 24, 1 << 18) == SHAPE


@pytest.mark.parametrize("V", [2049, 50000, 250001, 600000, (1 << 22) + 1, 1 << 24])
def test_lists_of_words_grow_with_the_vocabulary(lib, V):
    """A row's list holds 1/32 of its words: a longer row must not be one that a single block goes through again."""
    one, two = lib.q8_sample_bytes(1, V), lib.q8_sample_bytes(2, V)
    assert two - one >= 8 * (V // 32)
    assert lib.q8_workspace_bytes(2, 1, V, 16) >= two
