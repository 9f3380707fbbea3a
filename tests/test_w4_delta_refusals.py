"""CPU checks that the entry points for 4-bit weights and for the gated delta rule refuse bad arguments before they launch anything.  The context is
host memory laid out as q8_internal.h has it (stream, workspace, its size, error text; all else zero) and no pointer is ever followed: a
call that got as far as a launch would return Q8_ERR_DEVICE (5) here, where there is no device."""
import ctypes as C
import struct

import pytest
import torch

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up: only where nothing can be launched")

NULL, SHAPE, ALIGN, WORKSPACE, DEVICE = 1, 2, 3, 4, 5
P = 0x100000                                            # an aligned address


@pytest.fixture()
def lib():
    import paper_1804_05038_amd as q
    return q.load_library()


def context(ws_bytes):
    mem = C.create_string_buffer(4096)
    mem[:24] = struct.pack("QQQ", 0, 1 << 20, ws_bytes)
    return mem


def mat(**k):
    from paper_1804_05038_amd.binding import _MatW4
    d = dict(data=P, scale=P, rows=32, cols=64, ld=64, lds=4, group=64)
    d.update(k)
    return C.byref(_MatW4(*[d[f] for f in ("data", "scale", "rows", "cols", "ld", "lds", "group")]))


BAD_MATS = [(dict(data=None), NULL), (dict(scale=None), NULL), (dict(rows=0), SHAPE), (dict(rows=-1), SHAPE), (dict(rows=(1 << 24) + 1), SHAPE), (dict(cols=0), SHAPE),
            (dict(cols=129), SHAPE), (dict(ld=0), SHAPE), (dict(ld=8256), SHAPE), (dict(lds=0), SHAPE), (dict(cols=300, ld=192, group=32, lds=8), SHAPE), (dict(cols=16385, ld=8256, lds=260), SHAPE),
            (dict(group=0), SHAPE), (dict(group=16), SHAPE), (dict(group=96), SHAPE), (dict(group=256), SHAPE), (dict(ld=80), ALIGN), (dict(lds=6), ALIGN), (dict(data=P + 8), ALIGN),
            (dict(scale=P + 4), ALIGN)]


def test_good_calls_reach_the_launch(lib):
    c = context(1 << 30)
    assert lib.q8_quantize_matrix_w4(c, P, 32, 64, 64, mat()) == DEVICE
    for n in (1, 4, 40):
        assert lib.q8_gemm_w4(c, mat(), P, n, 64, None, P, 32) == DEVICE
        assert lib.output_logits_w4(c, None, mat(), None, None, None, None, P, n, 0, P, None, None, None, None) == DEVICE


@pytest.mark.parametrize("bad,want", BAD_MATS)
def test_matrices(lib, bad, want):
    c = context(1 << 30)
    assert lib.q8_gemm_w4(c, mat(**bad), P, 4, 1 << 15, None, P, 64) == want
    assert lib.output_logits_w4(c, None, mat(**bad), None, None, None, None, P, 4, 0, P, None, None, None, None) == want
    assert lib.q8_quantize_matrix_w4(c, P, bad.get("rows", 32), bad.get("cols", 64), 1 << 15, mat(**bad)) == want


def test_products(lib):
    c = context(lib.q8_gemm_w4_bytes(4, 64))
    call = lambda x=P, n=4, ldx=64, b=None, y=P, ldy=32: lib.q8_gemm_w4(c, mat(), x, n, ldx, b, y, ldy)
    assert lib.q8_gemm_w4(None, mat(), P, 4, 64, None, P, 32) == lib.q8_gemm_w4(c, None, P, 4, 64, None, P, 32) == NULL
    assert call(x=None) == call(y=None) == NULL
    assert call(n=0) == call(n=-3) == call(n=(1 << 20) + 1) == call(ldx=60) == call(ldy=31) == call(ldy=(1 << 25) + 4) == SHAPE
    assert call(ldx=66) == call(x=P + 4) == call(y=P + 2) == call(b=P + 1) == ALIGN
    assert call(n=1 << 20) == call(n=1000) == WORKSPACE
    assert call() == call(n=1, ldx=0, ldy=0) == DEVICE


def test_quantization(lib):
    c = context(1 << 20)
    call = lambda x=P, rows=32, cols=64, ld=64, m=None: lib.q8_quantize_matrix_w4(c, x, rows, cols, ld, m or mat())
    assert call(x=None) == lib.q8_quantize_matrix_w4(c, P, 32, 64, 64, None) == NULL and call(ld=63) == call(rows=31) == call(cols=60) == SHAPE
    assert call(x=P + 2) == ALIGN and call(x=P + 4) == call(ld=65) == DEVICE
    # blocks of 256 threads, 8 blocks of columns or words of scales each: 2^32 threads are one too many
    big = lambda rows, ld: call(rows=rows, m=mat(rows=rows, ld=ld))
    assert big((1 << 24) - 8, 512) == DEVICE and big(1 << 24, 512) == big(1 << 20, 8192) == SHAPE


def test_output_layer(lib):
    c = context(1 << 30)
    call = lambda w=None, t=P, n=4, k=0, lg=P, lp=None, idx=None, to=None, b=None: lib.output_logits_w4(c, None, w or mat(), b, None, None, None, t, n, k, lg, None, lp, idx, to)
    assert call(t=None) == call(lg=None) == call(k=3) == call(k=3, lp=P) == NULL
    assert call(n=0) == call(n=1025) == call(k=-1) == call(k=17, lp=P, idx=P) == call(w=mat(rows=8), k=9, lp=P, idx=P) == call(w=mat(rows=65537), k=4, lp=P, idx=P) == SHAPE
    assert call(w=mat(cols=62)) == call(t=P + 4) == call(lg=P + 1) == call(b=P + 2) == call(to=P + 8) == ALIGN
    assert lib.output_logits_w4(context(300000), None, mat(rows=60000), None, None, None, None, P, 8, 4, None, None, P, P, None) == WORKSPACE


@pytest.mark.parametrize("n", [1, 8, 9, 300, 1024])
@pytest.mark.parametrize("V,R", [(1, 16384), (16, 16), (100, 64), (3000, 620), (70000, 512)])
def test_workspace_is_enough(lib, n, V, R):
    c = context(lib.q8_workspace_bytes(n, 1, V, -(-R // 16) * 16))
    w = mat(rows=V, cols=R, ld=-(-R // 128) * 64, lds=-(-R // 128) * 4, group=32)
    for k in (0, min(V, 12)):
        if k and V > 65536:
            continue
        assert lib.output_logits_w4(c, None, w, None, None, None, None, P, n, k, P if k == 0 else None, None, P, P, None) == DEVICE
    assert lib.q8_gemm_w4(c, w, P, n, -(-R // 4) * 4, None, P, V) == DEVICE


def inputs(**k):
    from paper_1804_05038_amd.binding import _DeltaInputs
    d = dict(q=P, k=P, v=P, g=P, beta=P, ldq=128, ldk=128, ldv=256, ldg=4, ldb=4, hk=2, hv=4, dk=64, dv=64, scale=1.0, normalize=1)
    d.update(k)
    return C.byref(_DeltaInputs(*d.values()))


BAD_INPUTS = [(dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(g=None), NULL), (dict(beta=None), NULL), (dict(dk=0), SHAPE), (dict(dk=257, ldq=2000, ldk=2000), SHAPE),
              (dict(dv=0), SHAPE), (dict(dv=257, ldv=2000), SHAPE), (dict(hk=0), SHAPE), (dict(hv=0), SHAPE), (dict(hk=3, ldq=300, ldk=300), SHAPE), (dict(hk=4, hv=2), SHAPE),
              (dict(hk=1, hv=1025, ldv=1 << 20, ldg=2000, ldb=2000), SHAPE), (dict(ldq=127), SHAPE), (dict(ldk=127), SHAPE), (dict(ldv=255), SHAPE), (dict(ldg=3), SHAPE), (dict(ldb=3), SHAPE),
              (dict(q=P + 2), ALIGN), (dict(k=P + 1), ALIGN), (dict(v=P + 2), ALIGN), (dict(g=P + 2), ALIGN), (dict(beta=P + 3), ALIGN)]
FAR = P + (1 << 30)


@pytest.mark.parametrize("bad,want", BAD_INPUTS)
def test_delta_inputs(lib, bad, want):
    c = context(1 << 30)
    ldo = 1 << 20
    assert lib.q8_delta_step(c, inputs(**bad), 3, P, 3, None, P, P, ldo) == want
    assert lib.q8_delta_sequence(c, inputs(**bad), 30, P, 2, P, P, P, ldo) == want


def test_delta_steps(lib):
    c = context(1 << 18)
    call = lambda n=3, state=P, slots=3, parent=None, so=P, out=P, ldo=256, i=None: lib.q8_delta_step(c, i or inputs(), n, state, slots, parent, so, out, ldo)
    assert lib.q8_delta_step(None, inputs(), 3, P, 3, None, P, P, 256) == lib.q8_delta_step(c, None, 3, P, 3, None, P, P, 256) == call(so=None) == call(out=None) == NULL
    assert call(n=0) == call(n=65537) == call(slots=2) == call(slots=0) == call(slots=4) == call(ldo=255) == call(parent=P, slots=65537) == SHAPE
    assert call(so=P + 2) == call(state=P + 2) == call(out=P + 2) == call(parent=P + 2, so=FAR) == ALIGN
    # states that are written over before they are read: any overlap with parents, a shifted one without
    assert call(parent=P) == call(so=P + 4) == call(state=P + 1024) == call(parent=P, so=P + 4 * (3 * 4 * 64 * 64) - 4) == SHAPE
    assert call() == call(so=FAR) == call(parent=P, so=FAR, slots=7) == call(parent=P, so=P + 4 * (3 * 4 * 64 * 64)) == call(state=None, slots=0) == DEVICE
    assert call(n=65536, slots=65536, so=P) == DEVICE
    many = inputs(hk=1, hv=256, dv=1, dk=1, ldq=1, ldk=1, ldv=256, ldg=256, ldb=256)
    assert call(n=65535, slots=65535, i=many) == DEVICE and call(n=65536, slots=65536, i=many) == SHAPE


def test_delta_sequences(lib):
    c = context(lib.q8_delta_bytes(100, 2, 4, 64, 64))
    call = lambda L=100, off=P, S=2, state=P, so=P, out=P, ldo=256, i=None: lib.q8_delta_sequence(c, i or inputs(), L, off, S, state, so, out, ldo)
    assert lib.q8_delta_sequence(None, inputs(), 100, P, 2, P, P, P, 256) == lib.q8_delta_sequence(c, None, 100, P, 2, P, P, P, 256) == call(off=None) == call(out=None) == NULL
    assert call(L=-1) == call(L=(1 << 24) + 1) == call(S=0) == call(S=65537) == call(ldo=255) == SHAPE
    assert call(off=P + 2) == call(state=P + 1) == call(so=P + 2) == call(out=P + 2) == ALIGN
    assert call(so=P + 4) == call(so=P - 1024) == SHAPE
    assert call(L=4000) == call(S=300) == WORKSPACE
    assert call() == call(state=None) == call(so=None) == call(so=FAR) == call(L=0) == call(L=1, S=1, ldo=0) == DEVICE
    assert call(L=0, out=None, i=inputs(q=None, k=None, v=None, g=None, beta=None)) == DEVICE
    huge = inputs(hk=1, hv=64, dv=1, dk=1, ldq=1, ldk=1, ldv=64, ldg=64, ldb=64)
    assert call(L=1 << 23, S=1, i=huge, ldo=64) == SHAPE
    wide = inputs(hk=1, hv=128, dv=1, dk=1, ldq=1, ldk=1, ldv=128, ldg=128, ldb=128)
    big = context(lib.q8_delta_bytes(0, 65536, 128, 1, 1))
    wide_call = lambda S: lib.q8_delta_sequence(big, wide, 0, P, S, None, None, P, 128)
    assert wide_call(65535) == DEVICE and wide_call(65536) == SHAPE


def test_delta_bytes(lib):
    assert lib.q8_delta_bytes(0, 1, 1, 1, 1) > 262144
    assert lib.q8_delta_bytes(1 << 20, 3, 16, 128, 128) > lib.q8_delta_bytes(1 << 19, 3, 16, 128, 128) > lib.q8_delta_bytes(1 << 19, 1, 16, 128, 128)
    for bad in ((-1, 1, 1, 1, 1), (1, 0, 1, 1, 1), (1, 1, 0, 1, 1), (1, 1, 1025, 1, 1), (1, 1, 1, 0, 1), (1, 1, 1, 1, 257), ((1 << 24) + 1, 1, 1, 1, 1)):
        assert lib.q8_delta_bytes(*bad) == 262144


def test_the_binding_refuses(lib):
    """Host tensors, wrong types and shapes never reach the library."""
    import paper_1804_05038_amd as q
    from paper_1804_05038_amd import binding as b

    class Ctx:
        workspace = torch.empty(0)
    f = torch.zeros
    with pytest.raises(ValueError):
        q.MatW4(f(4, 64, dtype=torch.uint8), f(4, 4, dtype=torch.int32), 100, 64)               # on the host
    with pytest.raises(ValueError):
        q.q8_quantize_matrix_w4(Ctx(), f(4, 64), group=48)
    with pytest.raises(ValueError):
        b._heads(f(3, 2, 8), "q", (3, 2, 8))
    with pytest.raises(ValueError):
        q.q8_delta_step(Ctx(), f(3, 2, 8), f(3, 2, 8), f(3, 2, 8), f(3, 2), f(3, 2))
    with pytest.raises(ValueError):
        q.q8_delta_sequence(Ctx(), f(3, 16), f(3, 16), f(3, 16), f(3, 2), f(3, 2), f(2, dtype=torch.int32))


def test_the_binding_refuses_tensors_of_another_gpu():
    """(Tensors without memory, which torch lets be on any device.)"""
    from types import SimpleNamespace

    from torch._subclasses.fake_tensor import FakeTensorMode

    import paper_1804_05038_amd as q

    with FakeTensorMode():
        on = lambda d: lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device=d)
        here, there = on("cuda:0"), on("cuda:1")
        ctx = SimpleNamespace(workspace=here(256, dtype=torch.uint8), device=torch.device("cuda:0"), stream=None, empty=here, handle=None)
        u8, i32 = torch.uint8, torch.int32
        with pytest.raises(ValueError, match="codes on cuda:0, scales on cuda:1"):
            q.MatW4(here(32, 64, dtype=u8), there(32, 4, dtype=i32), 64, 64)

        def mat(data):                                   # (its address is not asked for: refused before)
            m = q.MatW4.__new__(q.MatW4)
            m.data, m.rows, m.cols, m.ld, m.group = data(32, 64, dtype=u8), 32, 64, 64, 64
            return m
        for W, X, bias, Y in ((mat(there), here(4, 64), None, None), (mat(here), there(4, 64), None, None), (mat(here), here(4, 64), there(32), None), (mat(here), here(4, 64), None, there(4, 32))):
            with pytest.raises(ValueError, match="the context is on cuda:0"):
                q.q8_gemm_w4(ctx, W, X, bias, Y=Y)
        with pytest.raises(ValueError, match="t_in: on cuda:1"):
            q.output_logits_w4(ctx, None, mat(here), None, t_in=there(4, 64))
        names = ("q", "k", "v", "g", "beta")
        shapes = {"q": (4, 2, 8), "k": (4, 2, 8), "v": (4, 2, 8), "g": (4, 2), "beta": (4, 2)}
        for far in names:
            x = {n: (there if n == far else here)(*shapes[n]) for n in names}
            with pytest.raises(ValueError, match=far + ": on cuda:1"):
                q.q8_delta_step(ctx, **x)
            with pytest.raises(ValueError, match=far + ": on cuda:1"):
                q.q8_delta_sequence(ctx, **x, sent_off=here(3, dtype=i32))


@pytest.mark.parametrize("hv,dk,dv", [(1, 256, 32), (4, 64, 64), (16, 128, 128), (24, 32, 128), (25, 32, 128), (96, 8, 32), (97, 8, 32), (3, 100, 72)])
def test_workspace_of_fewer_tokens_and_sequences(lib, hv, dk, dv):
    """q8_delta_bytes grows with both, and a call with less of either finds room: few long sequences take more than many."""
    i = inputs(hk=1, hv=hv, dk=dk, dv=dv, ldq=dk, ldk=dk, ldv=hv * dv, ldg=hv, ldb=hv)
    for L, S in ((800, 1), (5000, 3), (40000, 40), (200000, 7), (200001, 100)):
        c = context(lib.q8_delta_bytes(L, S, hv, dk, dv))
        for l in (0, 1, 767, 768, 769, 1000, 3000, 3100, 3500, 10000, 65536, 131071, 131072, L):
            for s in (1, 2, 3, 4, 5, 24, 32, 96, S):
                if l <= L and s <= S:
                    assert lib.q8_delta_bytes(l, s, hv, dk, dv) <= lib.q8_delta_bytes(L, S, hv, dk, dv)
                    assert lib.q8_delta_sequence(c, i, l, P, s, P, P, P, hv * dv) == DEVICE, (l, s)
