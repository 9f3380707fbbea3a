"""The gated delta rule over few long sequences, whose chunks go in segments: every width of the kernels, rows in whole 16-byte pieces and not, more than one slice
of columns.  That these cases do go in segments is checked against the rule in test_w4_delta_route.py."""
import numpy as np
import pytest
import torch

import delta_reference as ref
from parity import np_
from test_gpu_delta import _close, _dev, _edges, _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q():
    import paper_1804_05038_amd as q
    return q


# lengths, heads of keys and values, dk, dv, with edge decays and gates, rows off 16 bytes
SEGMENTED = [
    ([3000], 1, 1, 64, 100, False, False),              # two slices of values in the first pass, four of 32 later
    ([1500, 0, 1499], 1, 1, 64, 100, True, False),
    ([3000], 1, 2, 128, 130, False, False),             # (rows of values not in whole pieces)
    ([3000], 1, 2, 128, 160, True, False),
    ([3000], 1, 2, 70, 33, True, False),                # keys of 65 to 128, not in whole pieces
    ([2500, 1500], 2, 2, 127, 70, False, False),
    ([3000], 1, 2, 100, 40, True, True),                # whole pieces at other places than whole ones
    ([2500, 700], 1, 2, 48, 36, True, True),
    ([8195], 1, 1, 130, 64, True, False),
    ([4700, 5, 4300], 1, 1, 130, 64, True, False),
    ([8195], 1, 1, 256, 40, True, False),
    ([4600, 4400], 1, 1, 256, 40, True, True),
    ([7000, 7000], 1, 1, 130, 100, False, False),
    ([8000, 8000], 1, 1, 256, 100, False, False),
]


@pytest.mark.parametrize("lengths,hk,hv,dk,dv,edges,off16", SEGMENTED)
def test_in_segments(q, lengths, hk, hv, dk, dv, edges, off16):
    """Against the rule in 64 bits; twice the same bits; tokens of no sequence as they were; the new state over the old one."""
    rng = np.random.default_rng(sum(lengths) + dk + dv)
    front = 5
    off = [front] + [front + int(c) for c in np.cumsum(lengths)]
    L, S = off[-1] + 3, len(lengths)
    ctx = q.Context(workspace_bytes=q.q8_delta_bytes(L, S, hv, dk, dv))
    x = _inputs(rng, L, hk, hv, dk, dv)
    x["g"] *= np.float32(0.01)                          # states that last over many segments
    if edges:
        _edges(rng, x)
        x["g"][700:1400] = 0.0
        x["beta"] = np.minimum(x["beta"], np.float32(1.0))
    dev = _dev(ctx, x)
    if off16:
        for f in ("q", "k", "v"):
            n = x[f].size
            buf = torch.empty(n + 1, device=ctx.device)[1:]
            buf.copy_(dev[f].reshape(-1))
            dev[f] = buf.view(x[f].shape)
    st = rng.standard_normal((S, hv, dk, dv)).astype(np.float32)
    out = torch.full((L, hv, dv), 5.0, device=ctx.device)
    state = ctx.f32(st)
    call = lambda **k: q.q8_delta_sequence(ctx, **dev, sent_off=torch.tensor(off, dtype=torch.int32, device=ctx.device), scale=0.3, state=state, out=out, **k)
    got = call()
    first = np_(out).copy(), np_(got["state"]).copy()
    assert (first[0][:front] == 5.0).all() and (first[0][off[-1]:] == 5.0).all() and (np_(state) == st).all()
    again = call()
    assert (np_(out) == first[0]).all() and (np_(again["state"]) == first[1]).all()
    out[:front] = 0.0
    out[off[-1]:] = 0.0
    want, bound = ref.sequence(**x, off=off, scale=0.3, state=st), ref.sequence_bound(**x, off=off, scale=0.3, state=st)
    # a segment's matrix is as far off as a state, in each of its dk columns, and multiplies a state once more
    _close(got, want, (bound[0] * (1 + np.sqrt(dk)), bound[1] * (1 + np.sqrt(dk))), dk)
    call(state_out=state)
    assert (np_(state) == first[1]).all() and (np_(out)[front:off[-1]] == first[0][front:off[-1]]).all()


@pytest.mark.parametrize("lengths,hk,hv,dk,dv,edges,off16", [SEGMENTED[1], SEGMENTED[9]])
def test_in_segments_captured(q, lengths, hk, hv, dk, dv, edges, off16):
    """The four launches in a graph, replayed with other inputs: the eager call's bits."""
    stream = torch.cuda.Stream()
    rng = np.random.default_rng(dk)
    off = np.concatenate([[0], np.cumsum(lengths)]).tolist()
    L, S = off[-1], len(lengths)
    ctx = q.Context(workspace_bytes=q.q8_delta_bytes(L, S, hv, dk, dv), stream=stream)
    d = _dev(ctx, _inputs(rng, L, hk, hv, dk, dv))
    sent = torch.tensor(off, dtype=torch.int32, device=ctx.device)
    torch.cuda.synchronize()
    call = q.q8_delta_sequence(ctx, **d, sent_off=sent, bind=True)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        call.launch()
    for _ in range(3):
        for f, v in _inputs(rng, L, hk, hv, dk, dv).items():
            d[f].copy_(torch.from_numpy(v))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = np_(call.out["out"]).copy(), np_(call.out["state"]).copy()
        call.launch()
        torch.cuda.synchronize()
        assert (got[0] == np_(call.out["out"])).all() and (got[1] == np_(call.out["state"])).all() and np.isfinite(got[0]).all()
