"""What a number that is not finite reaches in the gated delta rule: its own token and the later ones of its sequence and head, as in the rule token
by token, and nothing before or beside them."""
import numpy as np
import pytest
import torch

import delta_reference as ref
from parity import np_
from test_gpu_delta import _dev, _inputs

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def q():
    import paper_1804_05038_amd as q
    return q


# (what, value): which number of the bad token is not finite
BAD = [("v", NAN), ("v", INF), ("v", -INF), ("k", NAN), ("k", INF), ("q", NAN), ("q", -INF), ("beta", NAN), ("beta", INF), ("g", NAN), ("g", INF)]


def _planted(x, what, value, t):
    """x with one number of token t, of its second head (of values, or of keys), in place of which `value` stands."""
    y = {f: a.copy() for f, a in x.items()}
    if what in ("g", "beta"):
        y[what][t, 1] = value
    else:
        y[what][t, min(1, y[what].shape[1] - 1), 3] = value
    return y


def _judge(got, clean, want, bound, first, dk):
    """Numbers that the rule leaves finite are as near as any; the others are not finite.  Before the bad token's chunk the bits are those without it."""
    out, state = got
    fin = np.isfinite(want[0])
    assert (np.isfinite(out) == fin).all() and (np.isfinite(state) == np.isfinite(want[1])).all()
    assert (np.abs(out - want[0])[fin] <= bound[0][fin]).all()
    assert (out[:first] == clean[0][:first]).all()
    b = np.where(fin, want[0], 0.0)
    assert np.linalg.norm(np.where(fin, out, 0.0) - b) <= 8 * 3 * 2.0 ** -24 * np.sqrt(dk + 2 * ref.C) * np.linalg.norm(b)


@pytest.mark.parametrize("what,value", BAD)
@pytest.mark.parametrize("hk,hv,dk,dv", [(2, 2, 64, 64), (1, 3, 33, 20), (2, 4, 130, 40)])
@pytest.mark.parametrize("t", [0, 5, 14, 21, 31, 44])
def test_sequence(q, what, value, hk, hv, dk, dv, t):
    """Two sequences of 70 and 40 tokens, the bad token in the first one."""
    rng = np.random.default_rng(dk + t)
    off = [0, 70, 110]
    x = _inputs(rng, off[-1], hk, hv, dk, dv)
    S = rng.standard_normal((2, hv, dk, dv)).astype(np.float32)
    ctx = q.Context(workspace_bytes=q.q8_delta_bytes(off[-1], 2, hv, dk, dv))
    call = lambda x: q.q8_delta_sequence(ctx, **_dev(ctx, x), sent_off=torch.tensor(off, dtype=torch.int32, device=ctx.device), scale=0.5, state=ctx.f32(S))
    r = call(x)
    clean = np_(r["out"]).copy(), np_(r["state"]).copy()
    bad = _planted(x, what, value, t)
    r = call(bad)
    got = np_(r["out"]), np_(r["state"])
    with np.errstate(all="ignore"):
        want = ref.sequence(**bad, off=off, scale=0.5, state=S)
    bound = ref.sequence_bound(**x, off=off, scale=0.5, state=S)
    assert (~np.isfinite(want[0][t])).any() and np.isfinite(want[0][:t]).all()
    _judge(got, clean, want, bound, t // 32 * 32, dk)
    # the other sequence, and heads that the number does not belong to, keep their bits
    assert (got[0][70:] == clean[0][70:]).all() and (got[1][1] == clean[1][1]).all()
    beside = [h for h in range(hv) if np.isfinite(want[0][:, h]).all()]
    assert beside or (hk == 1 and what in "qk")
    assert (got[0][:, beside] == clean[0][:, beside]).all() and (got[1][:, beside] == clean[1][:, beside]).all()
    if what == "v":                                     # ... and the other columns of its head
        cols = [c for c in range(dv) if c != 3]
        assert (got[0][:, :, cols] == clean[0][:, :, cols]).all() and (got[1][..., cols] == clean[1][..., cols]).all()


@pytest.mark.parametrize("what,value", [("v", INF), ("k", NAN), ("q", NAN), ("beta", NAN), ("g", NAN)])
@pytest.mark.parametrize("t", [3, 1500, 2047])
def test_long_sequence(q, what, value, t):
    """In segments (test_w4_delta_route has the rule): one sequence of 2048 tokens."""
    rng = np.random.default_rng(t)
    hk, hv, dk, dv, off = 2, 2, 32, 40, [0, 2048]
    x = _inputs(rng, 2048, hk, hv, dk, dv)
    x["g"] *= np.float32(0.01)
    ctx = q.Context(workspace_bytes=q.q8_delta_bytes(2048, 1, hv, dk, dv))
    call = lambda x: q.q8_delta_sequence(ctx, **_dev(ctx, x), sent_off=torch.tensor(off, dtype=torch.int32, device=ctx.device))
    r = call(x)
    clean = np_(r["out"]).copy(), np_(r["state"]).copy()
    bad = _planted(x, what, value, t)
    r = call(bad)
    with np.errstate(all="ignore"):
        want = ref.sequence(**bad, off=off)
    bound = ref.sequence_bound(**x, off=off)
    # (a segment's matrix multiplies a state once more)
    _judge((np_(r["out"]), np_(r["state"])), clean, want, (bound[0] * (1 + np.sqrt(dk)), bound[1]), t // 32 * 32, dk)
    assert (np_(r["out"])[:, 0] == clean[0][:, 0]).all() and (np_(r["state"])[:, 0] == clean[1][:, 0]).all()


@pytest.mark.parametrize("value", [NAN, INF])
@pytest.mark.parametrize("L", [70, 2048])
def test_state_to_start_from(q, value, L):
    """A number of the state: its column, in every token; the other columns keep their bits."""
    rng = np.random.default_rng(L)
    hv, dk, dv, off = 2, 32, 40, [0, L]
    x = _inputs(rng, L, hv, hv, dk, dv)
    S = rng.standard_normal((1, hv, dk, dv)).astype(np.float32)
    ctx = q.Context(workspace_bytes=q.q8_delta_bytes(L, 1, hv, dk, dv))
    call = lambda S: q.q8_delta_sequence(ctx, **_dev(ctx, x), sent_off=torch.tensor(off, dtype=torch.int32, device=ctx.device), state=ctx.f32(S))
    r = call(S)
    clean = np_(r["out"]).copy(), np_(r["state"]).copy()
    S[0, 1, 7, 11] = value
    r = call(S)
    for a, b in ((np_(r["out"]), clean[0]), (np_(r["state"]), clean[1])):
        assert not np.isfinite(a[:, 1, ..., 11]).any()
        a, b = np.delete(a, 11, -1), np.delete(b, 11, -1)
        assert (a == b).all()
    assert (np_(r["out"])[:, 0] == clean[0][:, 0]).all()


@pytest.mark.parametrize("what,value", BAD)
def test_step(q, what, value):
    """One slot of five, and in it one head (a column of it)."""
    rng = np.random.default_rng(4)
    n, hk, hv, dk, dv = 5, 2, 4, 24, 20
    ctx = q.Context(workspace_bytes=1 << 20)
    x = _inputs(rng, n, hk, hv, dk, dv)
    S = rng.standard_normal((n, hv, dk, dv)).astype(np.float32)
    call = lambda x: q.q8_delta_step(ctx, **_dev(ctx, x), state=ctx.f32(S))
    r = call(x)
    clean = np_(r["out"]).copy(), np_(r["state"]).copy()
    bad = _planted(x, what, value, 2)
    r = call(bad)
    with np.errstate(all="ignore"):
        want = ref.step(**bad, state=S)
    for a, c, w in ((np_(r["out"]), clean[0], want[0]), (np_(r["state"]), clean[1], want[1])):
        fin = np.isfinite(w)
        assert (np.isfinite(a) == fin).all() and (a[fin] == c[fin]).all()
