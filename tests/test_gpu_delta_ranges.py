"""The gated delta rule over sequences with numbers next to fp32's upper end: results that fit are there, as exact as others."""
import numpy as np
import pytest
import torch

import delta_reference as ref
from parity import np_
from test_gpu_delta import _dev, _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q():
    import paper_1804_05038_amd as q
    return q


def _by_columns(got, want, dk):
    """Each column as a whole within what independent roundings leave (three sums in a row of up to dk + 2 C products, times eight)."""
    for a, b in zip(got, want):
        dv = b.shape[-1]
        assert np.isfinite(a).all()
        off_by = np.linalg.norm((a.astype(np.float64) - b).reshape(-1, dv), axis=0)
        assert (off_by <= 8 * 3 * 2.0 ** -24 * np.sqrt(dk + 2 * ref.C) * np.linalg.norm(b.reshape(-1, dv), axis=0)).all()


@pytest.mark.parametrize("L", [1, 40, 70, 1200])
@pytest.mark.parametrize("dk,dv", [(48, 36), (64, 32), (200, 20)])
def test_large_columns(q, L, dk, dv):
    """Values and states of up to 1e36 a column, keys and queries of unit length: no result passes 2e38.  (1200 tokens of 48 or 64 rows go in segments.)"""
    rng = np.random.default_rng(L + dk)
    x = _inputs(rng, L, 1, 2, dk, dv)
    size = (10.0 ** rng.integers(30, 37, dv)).astype(np.float32)
    size[0] = 1.0
    x["v"] = np.clip(x["v"], -3, 3) * size
    x["g"] *= np.float32(0.01)
    S = np.clip(rng.standard_normal((1, 2, dk, dv)), -3, 3).astype(np.float32) * size
    ctx = q.Context(workspace_bytes=q.q8_delta_bytes(L, 1, 2, dk, dv))
    got = q.q8_delta_sequence(ctx, **_dev(ctx, x), sent_off=torch.tensor([0, L], dtype=torch.int32, device=ctx.device), state=ctx.f32(S))
    want = ref.sequence(**x, off=[0, L], state=S)
    assert max(np.abs(w).max() for w in want) < 2e38
    _by_columns((np_(got["out"]), np_(got["state"])), want, dk)


@pytest.mark.parametrize("L", [1, 40, 1200])
@pytest.mark.parametrize("step", [False, True])
def test_long_keys_and_queries_of_unit_length(q, L, step):
    """Lengths from 1 to 2^50 before they become one."""
    rng = np.random.default_rng(L)
    dk, dv = 48, 36
    x = _inputs(rng, L, 1, 2, dk, dv)
    for f in ("k", "q"):
        x[f] *= (2.0 ** rng.uniform(0, 50, (L, 1, 1)) / np.linalg.norm(x[f], axis=2, keepdims=True)).astype(np.float32)
    x["g"] *= np.float32(0.01)
    ctx = q.Context(workspace_bytes=q.q8_delta_bytes(L, 1, 2, dk, dv))
    if step:
        S = rng.standard_normal((L, 2, dk, dv)).astype(np.float32)
        got, want = q.q8_delta_step(ctx, **_dev(ctx, x), state=ctx.f32(S)), ref.step(**x, state=S)
    else:
        got = q.q8_delta_sequence(ctx, **_dev(ctx, x), sent_off=torch.tensor([0, L], dtype=torch.int32, device=ctx.device))
        want = ref.sequence(**x, off=[0, L])
    _by_columns((np_(got["out"]), np_(got["state"])), want, dk)


@pytest.mark.parametrize("L", [1, 40, 1200])
@pytest.mark.parametrize("ks,qs,vs", [(1e-12, 1e-3, 1e36), (1.0, 1e34, 1e-12), (1e-15, 1e5, 1e30), (1.0, 1e-30, 1e36)])
def test_lengths_against_columns(q, L, ks, qs, vs):
    """Keys and queries as they are given, short ones with large columns and long ones with small columns.  Keys of 1e-12 leave next to nothing of a value:
    the state to start from is what is read."""
    rng = np.random.default_rng(L)
    dk, dv = 48, 36
    x = _inputs(rng, L, 1, 2, dk, dv, normalize=False)
    x["k"] *= np.float32(ks)
    x["q"] = np.clip(x["q"], -3, 3) * np.float32(qs)
    x["v"] = np.clip(x["v"], -3, 3) * np.float32(vs)
    x["g"] *= np.float32(0.01)
    S = np.clip(rng.standard_normal((1, 2, dk, dv)), -3, 3).astype(np.float32) * np.float32(vs)
    ctx = q.Context(workspace_bytes=q.q8_delta_bytes(L, 1, 2, dk, dv))
    got = q.q8_delta_sequence(ctx, **_dev(ctx, x), sent_off=torch.tensor([0, L], dtype=torch.int32, device=ctx.device), state=ctx.f32(S), normalize=False)
    want = ref.sequence(**x, off=[0, L], state=S, normalize=False)
    assert max(np.abs(w).max() for w in want) < 2e38
    _by_columns((np_(got["out"]), np_(got["state"])), want, dk)
