"""CPU pins of the plain definitions that the GPU tests of 8-bit floating point and of drawing compare with, and the
refusals that the binding makes before anything reaches the library."""
import numpy as np
import pytest
import torch

import f8_reference as ref


def test_codes_are_those_of_torch():
    rng = np.random.default_rng(0)
    finite = ref.VALUES[~np.isnan(ref.VALUES)]
    mid = (finite[:-1] + finite[1:]) / 2
    x = np.concatenate([finite, mid, rng.uniform(-448, 448, 4000), np.ldexp(rng.uniform(-1, 1, 4000), rng.integers(-14, 9, 4000))])
    x = x[np.abs(x) <= 448].astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn)
    assert (ref.e4m3_round(x) == want.view(torch.uint8).numpy()).all()
    assert (ref.VALUES[ref.e4m3_round(x)] == want.double().numpy()).all()


def test_scales_are_the_smallest_that_hold_the_block():
    for m, e in ((448.0, 0), (np.nextafter(np.float32(448), np.float32(449)), 1), (224.0, -1), (1.0, -8), (1.75, -8), (1.7500001, -7), (2.0 ** 127, 119),
                 (3.4e38, 120), (2.0 ** -100, -108), (2.0 ** -101, 0), (0.0, 0)):
        _, s = ref.quantize(np.array([[m, 0, 0]], np.float32))
        assert s[0, 0] == e + 127, (m, s[0, 0])


def test_draw_by_hand():
    v = np.log(np.array([0.1, 0.4, 0.2, 0.3], np.float64)).astype(np.float32)
    pick = lambda u, **k: ref.draw(v, u, **k)[0]
    assert [pick(u) for u in (0.0, 0.39, 0.41, 0.69, 0.71, 0.89, 0.91)] == [1, 1, 3, 3, 2, 2, 0]
    assert [pick(u, top_k=2) for u in (0.5, 0.58, 0.99)] == [1, 3, 3]
    assert [pick(u, top_p=0.45) for u in (0.5, 0.58, 0.99)] == [1, 3, 3]
    assert [pick(u, min_p=0.6) for u in (0.5, 0.58, 0.99)] == [1, 3, 3]
    assert pick(0.99, top_p=0.0) == pick(0.99, min_p=2.0) == pick(0.99, T=0.0) == pick(0.99, top_k=1) == 1
    assert ref.draw(np.full(5, -np.inf, np.float32), 0.5)[:2] == (-1, -np.inf)


def test_the_binding_refuses_what_the_kernels_do_not_take():
    import paper_1804_05038_amd as q
    with pytest.raises(ValueError):                      # not on the device
        q.MatF8(torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8), 16)
    for bad in (torch.zeros(4, 16), torch.zeros(4, dtype=torch.float32), torch.zeros(4, 16, dtype=torch.float16)):
        with pytest.raises(ValueError):
            q.q8_sample_logits(None, bad, torch.zeros(4))
        with pytest.raises(ValueError):
            q.q8_quantize_matrix_f8.__globals__["_rows"](bad, "X")


def test_calls_without_a_context_return_the_null_code():
    import paper_1804_05038_amd as q
    lib = q.load_library()
    assert lib.q8_quantize_matrix_f8(None, None, 1, 1, 1, None, 16, None, 4) == 1
    assert lib.q8_gemm_f8(None, None, None, 1, 16, None, None, 16) == 1
    assert lib.q8_gemm_codes_f8(None, None, None, None, None, 16) == 1
    assert lib.output_logits_f8(None, None, None, None, None, None, None, None, 1, 0, None, None, None, None, None) == 1
    assert lib.q8_sample_logits(None, None, 1, 16, 16, None, None, None, None, None, 0, None) == 1
    assert q.q8_gemm_f8_bytes(0, 0) < q.q8_gemm_f8_bytes(1, 512) < q.q8_gemm_f8_bytes(1 << 20, 16384)
    assert q.q8_sample_bytes(1, 1) > 0
    for n, cols in ((1, 16384), (1024, 16384), (1024, 16), (700, 620)):
        assert q.q8_workspace_bytes(n, 1, 1, (cols + 15) // 16 * 16) >= q.q8_gemm_f8_bytes(n, cols)
    for n, V in ((1, 8193), (1024, 9000), (1, 1 << 24)):
        assert q.q8_workspace_bytes(n, 1, V, 16) >= q.q8_sample_bytes(n, V)


def test_the_binding_refuses_tensors_of_another_gpu():
    """(Tensors without memory, which torch lets be on any device.)"""
    from types import SimpleNamespace

    from torch._subclasses.fake_tensor import FakeTensorMode

    import paper_1804_05038_amd as q

    class Converted(Exception):
        pass

    def f32(t):
        raise Converted

    with FakeTensorMode():
        here, there = (lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda:0")), (lambda *s, dtype=torch.float32: torch.empty(*s, dtype=dtype, device="cuda:1"))
        ctx = SimpleNamespace(workspace=here(256, dtype=torch.uint8), device=torch.device("cuda:0"), stream=None, empty=here, f32=f32, handle=None)
        u8 = torch.uint8

        def mat(data, scale):                            # (its address is not asked for: refused before)
            m = q.MatF8.__new__(q.MatF8)
            m.data, m.scale_rows, m.rows, m.cols, m.ld = data(32, 64, dtype=u8), scale(32, 4, dtype=u8), 32, 64, 64
            return m
        with pytest.raises(ValueError, match="codes on cuda:0, scales on cuda:1"):
            q.MatF8(here(32, 64, dtype=u8), there(32, 4, dtype=u8), 64)
        W, far = mat(here, here), mat(there, there)
        x, lg, u = here(4, 64), here(4, 100), here(4)
        for name, call in (("W", lambda: q.q8_gemm_f8(ctx, far, x)), ("X", lambda: q.q8_gemm_f8(ctx, W, there(4, 64))), ("X", lambda: q.q8_gemm_f8(ctx, W, far)),
                           ("bias", lambda: q.q8_gemm_f8(ctx, W, x, there(32))), ("Y", lambda: q.q8_gemm_f8(ctx, W, x, Y=there(4, 32))),
                           ("W_out", lambda: q.output_logits_f8(ctx, None, far, None, t_in=x)), ("t_in", lambda: q.output_logits_f8(ctx, None, W, None, t_in=there(4, 64))),
                           ("b_out", lambda: q.output_logits_f8(ctx, None, W, there(32), t_in=x)), ("logits", lambda: q.output_logits_f8(ctx, None, W, None, t_in=x, logits=there(4, 32))),
                           ("logits", lambda: q.q8_sample_logits(ctx, there(4, 100), u)), ("u", lambda: q.q8_sample_logits(ctx, lg, there(4))),
                           ("top_k", lambda: q.q8_sample_logits(ctx, lg, u, top_k=there(4, dtype=torch.int32))), ("temperature", lambda: q.q8_sample_logits(ctx, lg, u, there(4))),
                           ("tokens", lambda: q.q8_sample_logits(ctx, lg, u, tokens=there(4, dtype=torch.int32))), ("E_tgt", lambda: q.q8_sample_logits(ctx, lg, u, E_tgt=there(100, 8)))):
            with pytest.raises(ValueError, match="%s: on cuda:1, the context is on cuda:0" % name):
                call()
        with pytest.raises(Converted):                   # a matrix to be quantized comes to the context's device first, as one of the host does
            q.q8_quantize_matrix_f8(ctx, there(32, 64))
