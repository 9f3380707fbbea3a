"""GPU parity of q8_sample_logits with the plain definition in 64 bits."""
import ctypes as C

import numpy as np
import pytest
import torch

import f8_reference as ref
from parity import np_

pytestmark = pytest.mark.gpu

TOP = 1 - 2.0 ** -24


@pytest.fixture(scope="module")
def q():
    import paper_1804_05038_amd as q
    return q


@pytest.fixture(scope="module")
def ctx(q):
    return q.Context(workspace_bytes=q.q8_sample_bytes(1024, 1 << 24) + (64 << 20))


def _check(q, ctx, lg, u, T=None, top_k=None, top_p=None, min_p=None, logits=None):
    """Every row against the definition.  Weights are whole multiples of 2^-46 of the largest (2^-38 at the largest vocabulary),
    half a unit off each, and words under half a unit or past 32 T below the best count for nothing: V units in all, and a
    row whose margin is less than that may take a neighbour."""
    n, V = lg.shape
    dev = lambda a, t: None if a is None else torch.from_numpy(np.asarray(a, t)).to(ctx.device)
    g = dev(lg, np.float32) if logits is None else logits
    r = q.q8_sample_logits(ctx, g, dev(u, np.float32), dev(T, np.float32), dev(top_k, np.int32), dev(top_p, np.float32), dev(min_p, np.float32))
    tokens, logp = np_(r["tokens"]), np_(r["logp"]).astype(np.float64)
    unit = 2.0 ** -min(46, 62 - max(0, (V - 1).bit_length()))
    at = lambda a, j, d: d if a is None else a[j]
    for j in range(n):
        tok, lp, margin = ref.draw(lg[j], u[j], at(T, j, 1.0), int(at(top_k, j, 0)), at(top_p, j, 1.0), at(min_p, j, 0.0))
        if margin > 2 * V * unit + 1e-14:
            assert tokens[j] == tok, (j, tokens[j], tok, margin)
            # the sum of exponentials: distances up to 28 count (exp(-28) V < 2^-16 of it for V <= 2^24, and what is off there is off by
            # a small share of that); each distance and its product with log2(e) are rounded once in fp32, 2^-24 of themselves
            # each, the exponential is 2^-23 off and pairs are added in fp32: 28 (2^-24 + 2^-24) + 2^-23 + 2^-24 < 2^-18; the result is
            # rounded once
            assert logp[j] == lp or abs(logp[j] - lp) <= 2.0 ** -18 + 2.0 ** -24 * abs(lp), (j, logp[j], lp)
    return tokens


def _logits(rng, n, V):
    lg = rng.standard_normal((n, V)) * 1.5 - 0.6 * np.log(np.arange(V) + 20.0)
    for j in range(n):
        lg[j, rng.integers(0, V, 24)] += 9 * rng.random(24)
    return lg.astype(np.float32)


SIZES = [(1, 1), (2, 2047), (3, 2048), (5, 2049), (300, 2050), (3, 8192), (3, 8193), (20, 9001), (3, 2), (2, 63), (4, 64), (5, 65), (3, 1000), (2, 1023), (3, 1025), (7, 4097), (40, 8001), (2, 33658), (300, 5003), (2, 65536), (2, 65537), (2, 100003), (1, 262145), (1025, 300), (1100, 2100), (130, 70000)]


@pytest.mark.parametrize("n,V", SIZES)
@pytest.mark.parametrize("filters", ["none", "T", "top_k", "top_p", "min_p", "all"])
def test_draw(q, ctx, n, V, filters):
    rng = np.random.default_rng(n * 13 + V)
    lg, u = _logits(rng, n, V), rng.random(n).astype(np.float32).clip(0, TOP)
    T = top_k = top_p = min_p = None
    if filters != "none":
        T = (0.3 + 1.5 * rng.random(n)).astype(np.float32)
    if filters in ("top_k", "all"):
        top_k = rng.integers(0, min(V + 3, 200), n).astype(np.int32)
    if filters in ("top_p", "all"):
        top_p = rng.random(n).astype(np.float32)
    if filters in ("min_p", "all"):
        min_p = (0.3 * rng.random(n)).astype(np.float32)
    _check(q, ctx, lg, u, T, top_k, top_p, min_p)


@pytest.mark.parametrize("V", [50, 3000, 50000, 90000])
def test_large_top_k(q, ctx, V):
    rng = np.random.default_rng(V)
    ks = np.array([1, 2, V // 3, V - 1, V, V + 1, 2 ** 31 - 1, -5], np.int64).astype(np.int32)
    n = len(ks)
    _check(q, ctx, _logits(rng, n, V), rng.random(n).astype(np.float32).clip(0, TOP), top_k=ks)
    _check(q, ctx, (rng.standard_normal((n, V)) * 0.01).astype(np.float32), rng.random(n).astype(np.float32).clip(0, TOP), top_k=ks, top_p=np.full(n, 0.9, np.float32))


@pytest.mark.parametrize("V", [7, 5000, 50000, 70001])
def test_rows_of_equal_logits(q, ctx, V):
    """Everything ties: the order is that of the indices."""
    rng = np.random.default_rng(V)
    n = 12
    u = rng.random(n).astype(np.float32).clip(0, TOP)
    u[:2] = 0.0, TOP
    lg = np.full((n, V), 2.5, np.float32)
    lg[3, ::2] = 0.0
    lg[4, ::2] = -0.0
    lg[4, 1::2] = 0.0                                    # the two zeros tie
    lg[5:, :V // 2] = -np.inf
    _check(q, ctx, lg, u)
    _check(q, ctx, lg, u, top_k=np.full(n, max(1, V // 4), np.int32))
    _check(q, ctx, lg, u, top_p=np.full(n, 0.37, np.float32))
    _check(q, ctx, lg, u, min_p=np.full(n, 1.0, np.float32), T=np.full(n, 0.5, np.float32))


@pytest.mark.parametrize("n,V,words,apart", [(n, V, words, apart) for n, V in [(3, 250001), (2, 600000), (900, 9001)] for words in (300, 1500, 3000, 7000)
                                             for apart in (1, 31) if words * apart <= V])
def test_many_words_of_nearly_the_same_weight(q, ctx, n, V, words, apart):
    """Borders among many words within 1/64 nat, next to each other or spread over the row."""
    rng = np.random.default_rng(words + apart)
    lg = np.full((n, V), -30.0, np.float32)
    for j in range(n):
        at = int(rng.integers(0, V - words * apart + 1))
        lg[j, at:at + words * apart:apart] = 2.0 + rng.random(words) / 64
    u = rng.random(n).astype(np.float32).clip(0, TOP)
    _check(q, ctx, lg, u)
    _check(q, ctx, lg, u, top_k=rng.integers(1, words, n).astype(np.int32), top_p=rng.random(n).astype(np.float32))
    _check(q, ctx, lg, u, T=np.full(n, 0.4, np.float32), top_p=rng.random(n).astype(np.float32), min_p=np.full(n, 0.97, np.float32))


def test_two_values_that_many_words_share(q, ctx):
    rng = np.random.default_rng(2)
    lg = rng.choice(np.array([1.0, 1.0000001, 0.9999999], np.float32), (8, 40000))
    u = rng.random(8).astype(np.float32).clip(0, TOP)
    _check(q, ctx, lg, u)
    _check(q, ctx, lg, u, top_k=rng.integers(1, 40000, 8).astype(np.int32), top_p=rng.random(8).astype(np.float32))


def test_masks(q, ctx):
    inf, low = np.inf, np.finfo(np.float32).min
    rng = np.random.default_rng(5)
    V = 3001
    lg = np.full((10, V), -inf, np.float32)              # 0: a row without words
    lg[1, 1234] = -700.0                                 # one word
    lg[2] = low                                          # every word masked by the lowest value: they share the mass
    lg[3] = low
    lg[3, [5, 17]] = 3.0
    lg[4] = np.nan
    lg[5] = np.nan
    lg[5, [9, 2000]] = 0.0, 1.0
    lg[6] = _logits(rng, 1, V)[0]
    lg[6, ::3] = -inf
    lg[6, 1::3] = np.nan
    lg[7] = _logits(rng, 1, V)[0]
    lg[7, [100, 50, 2999]] = inf                         # they share the mass
    lg[8, [0, V - 1]] = 3e38, -3e38                      # a difference past fp32's range
    lg[9, :40] = np.linspace(-80, 80, 40)
    for u in (0.0, 0.3, 0.5, 0.9, TOP):
        us = np.full(10, u, np.float32)
        t = _check(q, ctx, lg, us)
        assert t[0] == t[4] == -1 and t[1] == 1234 and t[3] in (5, 17) and t[7] in (50, 100, 2999)
        _check(q, ctx, lg, us, T=np.full(10, 0.7, np.float32), top_k=np.full(10, 2, np.int32), top_p=np.full(10, 0.8, np.float32), min_p=np.full(10, 0.1, np.float32))
        _check(q, ctx, lg, us, T=np.zeros(10, np.float32))


def test_parameters_at_and_past_their_ends(q, ctx):
    rng = np.random.default_rng(6)
    n, V = 14, 6000
    lg = _logits(rng, n, V)
    u = np.array([0.0, TOP, 1.0, 2.0, -1.0, np.nan, np.inf, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5], np.float32)
    T = np.array([1, 1, 1, 1, 1, 1, 1, 0, -1, np.nan, 1e-30, np.inf, 1e30, 1e-3], np.float32)
    _check(q, ctx, lg, u, T)
    half = np.full(n, 0.5, np.float32)
    _check(q, ctx, lg, half, top_p=np.array([0, -1, 1, 2, np.nan, 1e-30, 0.999999] * 2, np.float32))
    _check(q, ctx, lg, half, min_p=np.array([0, -1, 1, 2, np.nan, 1e-30, 1e-4] * 2, np.float32))
    # one number for all rows
    g = torch.from_numpy(lg).to(ctx.device)
    uu = torch.full((n,), 0.5, device=ctx.device)
    a = q.q8_sample_logits(ctx, g, uu, 0.7, 40, 0.9, 0.01)["tokens"]
    b = q.q8_sample_logits(ctx, g, uu, torch.full((n,), 0.7, device=ctx.device), torch.full((n,), 40, dtype=torch.int32, device=ctx.device),
                           torch.full((n,), 0.9, device=ctx.device), torch.full((n,), 0.01, device=ctx.device))["tokens"]
    assert bool((a == b).all())


def test_every_token_by_its_share(q, ctx):
    """u over a grid: each token comes as often as its probability says, to one step of the grid."""
    rng = np.random.default_rng(8)
    V, n = 37, 4096
    row = (rng.standard_normal(V) * 1.5).astype(np.float32)
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    t = np_(q.q8_sample_logits(ctx, torch.from_numpy(row).to(ctx.device).expand(n, V).contiguous(), torch.from_numpy(u).to(ctx.device))["tokens"])
    p = np.exp(row.astype(np.float64) - row.max())
    p /= p.sum()
    assert (np.abs(np.bincount(t, minlength=V) - n * p) <= 1.0 + 1e-6 * n).all()


@pytest.mark.parametrize("off,pitch", [(0, 5003), (1, 5004), (2, 5001), (0, 6000)])
def test_pitches_embeddings_and_guards(q, ctx, off, pitch):
    rng = np.random.default_rng(off + pitch)
    n, V, E = 6, 5000, 33
    lg = _logits(rng, n, V)
    lg[2] = -np.inf
    buf = torch.full((off + n * pitch,), 99.0, device=ctx.device)          # words past V would win if they were read
    view = buf[off:].view(n, pitch)[:, :V]
    view.copy_(torch.from_numpy(lg))
    u = rng.random(n).astype(np.float32).clip(0, TOP)
    tok = _check(q, ctx, lg, u, T=np.full(n, 0.9, np.float32), logits=view)
    E_tgt = ctx.f32(rng.standard_normal((V, E)).astype(np.float32))
    guard = torch.full((n + 1, E), 7.0, device=ctx.device)
    tk = torch.full((n + 2,), -9, dtype=torch.int32, device=ctx.device)
    r = q.q8_sample_logits(ctx, view, torch.from_numpy(u).to(ctx.device), 0.9, E_tgt=E_tgt, y_emb=guard[:n], tokens=tk[:n])
    assert (np_(r["tokens"]) == tok).all() and np_(tk)[n:].tolist() == [-9, -9]
    want = np.where(tok[:, None] >= 0, np_(E_tgt)[np.maximum(tok, 0)], 0.0)
    assert (np_(guard[:n]) == want).all() and bool((guard[n] == 7.0).all())


def test_logits_past_32_bit_offsets(q, ctx):
    n, V = 9000, 250000                                   # 2.25e9 logits
    lg = torch.full((n, V), -3.0, device=ctx.device)
    lg[:, 77] = 0.0
    lg[-1, V - 1] = 30.0
    lg[-2, V - 2] = 30.0
    t = np_(q.q8_sample_logits(ctx, lg, torch.full((n,), 0.5, device=ctx.device), 0.1)["tokens"])
    assert (t[:-2] == 77).all() and t[-1] == V - 1 and t[-2] == V - 2


def test_the_largest_vocabulary(q, ctx):
    rng = np.random.default_rng(11)
    V = 1 << 24
    lg = rng.standard_normal((1, V)).astype(np.float32)
    for k in (dict(), dict(top_k=np.array([5], np.int32)), dict(top_p=np.array([0.3], np.float32))):
        _check(q, ctx, lg, np.array([0.77], np.float32), **k)


def _pinned(q, ctx, lg, u, T=1.0, top_k=0, top_p=1.0):
    """The rows of a long vocabulary, each of them held to the definition.  A word's mass is half a unit off, and 4e-12 of itself
    (the place in 2^-33 of 1/32 octave, the polynomial); so the mass up to a border and the one that it is compared with are together
    V units and 1e-11 of the whole off at most, in shares of the row's whole mass, as the margin is.  The log-probability is that of
    the drawn word, its tolerance _check's."""
    n, V = lg.shape
    full = lambda v, t: torch.full((n,), v, dtype=t, device=ctx.device)
    r = q.q8_sample_logits(ctx, torch.from_numpy(lg).to(ctx.device), torch.from_numpy(u).to(ctx.device), full(T, torch.float32), full(top_k, torch.int32),
                           full(top_p, torch.float32))
    tokens, logp = np_(r["tokens"]), np_(r["logp"]).astype(np.float64)
    unit = 2.0 ** -min(46, 62 - (V - 1).bit_length())
    for j in range(n):
        gap = np.float64(lg[j].max()) - lg[j].astype(np.float64)
        tok, _, margin = ref.draw(lg[j], u[j], T, top_k, top_p)
        assert margin > V * unit / np.exp(-gap / float(np.float32(T))).sum() + 1e-11, (j, margin)     # (of the inputs: no row is left out)
        assert tokens[j] == tok, (j, tokens[j], tok, margin)
        lp = -gap[tokens[j]] - np.log(np.exp(-gap).sum())
        assert abs(logp[j] - lp) <= 2.0 ** -18 + 2.0 ** -24 * abs(lp), (j, logp[j], lp)


@pytest.mark.parametrize("k", [dict(), dict(top_k=5), dict(top_p=0.3), dict(T=0.5), dict(T=0.5, top_k=1000, top_p=0.9)])
def test_the_largest_vocabulary_to_its_last_word(q, ctx, k):
    """Three dozen likely words up to the very end, all others some 40 nat below; and Gaussian logits."""
    rng = np.random.default_rng(23)
    V, n = 1 << 24, 2
    lg = (rng.standard_normal((n, V), dtype=np.float32) - 40).astype(np.float32)
    for j in range(n):
        lg[j, np.concatenate([rng.integers(0, V, 33), [0, V - 2, V - 1]])] = (2 * rng.random(36)).astype(np.float32)
    lg[0, V - 1] = 3.0
    _pinned(q, ctx, lg, np.array([0.31, 0.93], np.float32), **k)
    if k != dict(T=0.5):                                  # (there, no word's share clears the units of 2^24 words)
        _pinned(q, ctx, rng.standard_normal((1, V), dtype=np.float32), np.array([0.77], np.float32), **k)


@pytest.mark.parametrize("V,low", [(1 << 19, -30.6), ((1 << 19) + 1, -29.9), (1 << 21, -29.2), ((1 << 22) + 1, -27.8), (1 << 24, -27.1)])
def test_log_probability_counts_words_too_light_to_be_drawn(q, ctx, V, low):
    """One likely word, every other one just under half a unit of mass: none of these is drawn, and all of them are in the sum of
    the exponentials, at every temperature.  The distances are exact in fp32; an exponential is off by 30 2^-24 + 2^-23 of itself, their
    sum (below 2^-14) by less than 2^-32; the likely word's pair is rounded to 2^-24, and the result once."""
    lg = torch.full((1, V), float(np.float32(low)), device=ctx.device)
    lg[0, V - 2] = 0.0
    want = -np.log1p((V - 1) * np.exp(np.float64(np.float32(low))))
    for T in (1.0, 0.999):
        r = q.q8_sample_logits(ctx, lg, torch.full((1,), 0.5, device=ctx.device), T)
        assert int(r["tokens"]) == V - 2
        assert abs(float(r["logp"]) - want) <= 2.0 ** -23, (T, float(r["logp"]), want)


@pytest.mark.parametrize("V", [1500, 6000, 50000, 250001])
@pytest.mark.parametrize("sigma", [1e-6, 1e-3, 0.05, 0.4])
@pytest.mark.parametrize("mask", ["none", "half", "fourths", "run", "tail"])
def test_flat_rows(q, ctx, V, sigma, mask):
    """Logits that spread over little, so that a bin of one width would hold most words, beside masks and a tail that do not."""
    n = 4
    rng = np.random.default_rng(V + int(1e6 * sigma))
    lg = (7.25 + sigma * rng.standard_normal((n, V))).astype(np.float32)
    if mask == "half":
        lg[rng.random((n, V)) < 0.5] = np.finfo(np.float32).min
    elif mask == "fourths":
        lg[:, ::4] = -1e9
    elif mask == "run":
        lg[:, V // 3:] = -1e4
    elif mask == "tail":
        t = rng.random((n, V)) < 0.02
        lg[t] -= (30 * rng.random(int(t.sum()))).astype(np.float32)
    u = rng.random(n).astype(np.float32).clip(0, TOP)
    _check(q, ctx, lg, u)
    _check(q, ctx, lg, u, T=np.array([0.5, 1.0, 2.0, 30.0], np.float32), top_p=rng.random(n).astype(np.float32))
    _check(q, ctx, lg, u, top_k=rng.integers(1, V, n).astype(np.int32), min_p=np.full(n, 0.9, np.float32))


@pytest.mark.parametrize("V", [1500, 6000, 50000])
@pytest.mark.parametrize("sigma", [1e-30, 1e-12, 1e-8, 1e-7, 1e-6, 1e-4])
def test_flat_rows_around_zero(q, ctx, V, sigma):
    """Logits whose differences are near what a word's place is rounded to, the largest of them zero."""
    n = 6
    rng = np.random.default_rng(V)
    lg = (-sigma * np.abs(rng.standard_normal((n, V)))).astype(np.float32)
    lg[np.arange(n), rng.integers(0, V, n)] = 0.0
    lg[1] *= 50.0
    lg[2, ::2] = 0.0
    u = rng.random(n).astype(np.float32).clip(0, TOP)
    _check(q, ctx, lg, u)
    _check(q, ctx, lg, u, T=np.array([0.01, 0.3, 1.0, 1.0, 2.0, 30.0], np.float32), top_p=rng.random(n).astype(np.float32))
    _check(q, ctx, lg, u, top_k=rng.integers(1, V, n).astype(np.int32))


@pytest.mark.parametrize("V", [700, 5000, 50000])
def test_without_log_probabilities(q, ctx, V):
    """logp NULL: the same tokens, whatever form draws them."""
    rng = np.random.default_rng(V)
    n = 6
    lg = ctx.f32(_logits(rng, n, V))
    u = ctx.f32(rng.random(n).astype(np.float32).clip(0, TOP))
    T, k = ctx.f32(np.array([1, 0.7, 0, 1, 2, 1], np.float32)), torch.tensor([0, 5, 0, 40, 0, 1], dtype=torch.int32, device=ctx.device)
    for top_k in (None, k):
        want = np_(q.q8_sample_logits(ctx, lg, u, T, top_k)["tokens"]).copy()
        s = q.binding._Sampling(T.data_ptr(), top_k.data_ptr() if top_k is not None else None, None, None)
        tokens = torch.full((n,), -9, dtype=torch.int32, device=ctx.device)
        ctx.check(ctx.lib.q8_sample_logits(ctx.handle, lg.data_ptr(), n, V, V, C.byref(s), u.data_ptr(), tokens.data_ptr(), None, None, 0, None))
        assert (np_(tokens) == want).all()


def test_two_streams_at_once(q):
    """Rows over several blocks, whose launches leave sums for each other, on two streams; one number for all rows."""
    rng = np.random.default_rng(17)
    n, V = 40, 50000
    base = q.Context(workspace_bytes=q.q8_sample_bytes(n, V))
    lg = [base.f32(_logits(rng, n, V)) for _ in range(2)]
    u = base.f32(rng.random(n).astype(np.float32))
    full = lambda v, t=torch.float32: torch.full((n,), v, dtype=t, device=base.device)
    want = [np_(q.q8_sample_logits(base, g, u, full(0.9), full(200, torch.int32), full(0.8), full(0.001))["tokens"]).copy() for g in lg]
    streams = [torch.cuda.Stream() for _ in range(2)]
    cs = [q.Context(workspace_bytes=q.q8_sample_bytes(n, V), stream=s) for s in streams]
    torch.cuda.synchronize()
    for _ in range(20):
        r = [q.q8_sample_logits(c, g, u, 0.9, 200, 0.8, 0.001) for c, g in zip(cs, lg)]
        torch.cuda.synchronize()
        assert all((np_(o["tokens"]) == w).all() for o, w in zip(r, want))


def test_refusals(q, ctx):
    """What the binding refuses (the library's own refusals: test_f8_refusals.py, on the host)."""
    lg, u, E, y = ctx.empty(4, 100), ctx.empty(4), ctx.empty(100, 8), ctx.empty(4, 8)
    for bad in (lambda: q.q8_sample_logits(ctx, lg, u[:3]), lambda: q.q8_sample_logits(ctx, lg.double(), u), lambda: q.q8_sample_logits(ctx, lg.t(), u),
                lambda: q.q8_sample_logits(ctx, lg, u, top_k=u), lambda: q.q8_sample_logits(ctx, lg, u, E_tgt=E[:99]), lambda: q.q8_sample_logits(ctx, lg, u, y_emb=y),
                lambda: q.q8_sample_logits(ctx, lg, u, tokens=u)):
        with pytest.raises(ValueError):
            bad()
    torch.cuda.synchronize()


def test_a_decoding_loop(q):
    """Decoder step, output layer in 8-bit floating point, drawn tokens and their embeddings, step after step, eagerly and
    from a graph: the same tokens, each the definition's draw from that step's logits."""
    from parity import gpu_gru, gpu_mat
    from workloads import synth
    V, E, H, A, R, S, steps = 3001, 64, 128, 96, 64, 11, 5
    p = synth.full_model(seed=4, V=V, E=E, H=H, A=A, R=R)
    base = q.Context(workspace_bytes=q.q8_workspace_bytes(max_n=64, max_l=64, max_rows=V, max_ld=512))
    rng = np.random.default_rng(0)
    lens = [int(v) for v in rng.integers(3, 9, S)]
    L = sum(lens)
    enc = base.f32(np.tanh(rng.standard_normal((L, 2 * H))).astype(np.float32))
    P = q.q8_gemm_narrow(base, gpu_mat(q, base, p["att.W"]), enc, base.f32(p["att.b"]))
    off = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device=base.device)
    w = q.CgruWeights(gpu_gru(q, base, p, "dec_r"), gpu_mat(q, base, p["att.U"]), base.f32(p["att.v"]), gpu_gru(q, base, p, "dec_q"))
    ro = q.ReadoutWeights(gpu_mat(q, base, p["ro.Ws"]), gpu_mat(q, base, p["ro.Wy"]), gpu_mat(q, base, p["ro.Wc"]), base.f32(p["ro.b"]))
    W_out, b_out = q.q8_quantize_matrix_f8(base, base.f32(p["out.W"])), base.f32(p["out.b"])
    E_tgt = base.f32(p["E_tgt"])
    u_all = rng.random((steps, S)).astype(np.float32).clip(0, TOP)
    s0 = np.tanh(rng.standard_normal((S, H))).astype(np.float32)

    def loop(ctx):
        y, u = E_tgt[:1].repeat(S, 1).contiguous(), base.empty(S)
        s = [base.f32(s0), base.empty(S, H)]
        calls = []
        for i in (0, 1):
            c1 = q.cgru_decoder_step_batch_q8(ctx, w, P, enc, off, 1, max(lens), y, s[i], out={"s": s[1 - i]}, bind=True)
            c2 = q.output_logits_f8(ctx, ro, W_out, b_out, s[1 - i], y, c1.out["ctx"], k=0, bind=True)
            c3 = q.q8_sample_logits(ctx, c2.out["logits"], u, 0.8, 50, 0.95, 0.01, E_tgt=E_tgt, y_emb=y, bind=True)
            calls.append((c1, c2, c3))
        return y, u, s, calls

    y, u, s, calls = loop(base)
    tokens = []
    for t in range(steps):
        u.copy_(torch.from_numpy(u_all[t]))
        for c in calls[t & 1]:
            c.launch()
        tokens.append(np_(calls[t & 1][2].out["tokens"]).copy())
        lg = np_(calls[t & 1][1].out["logits"])
        for j in range(S):
            tok, lp, margin = ref.draw(lg[j], u_all[t, j], 0.8, 50, 0.95, 0.01)
            assert margin < 1e-9 or tokens[-1][j] == tok
        assert (np_(y) == p["E_tgt"][tokens[-1]]).all()
    stream = torch.cuda.Stream()
    ctx = q.Context(workspace_bytes=q.q8_workspace_bytes(max_n=64, max_l=64, max_rows=V, max_ld=512), stream=stream)
    y, u, s, calls = loop(ctx)
    torch.cuda.synchronize()
    for c in calls[0] + calls[1]:                         # outside of capture first
        c.launch()
    stream.synchronize()
    graphs = []
    for i in (0, 1):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            for c in calls[i]:
                c.launch()
        graphs.append(g)
    for again in range(2):
        y.copy_(E_tgt[:1].expand(S, E))
        s[0].copy_(base.f32(s0))
        for t in range(steps):
            u.copy_(torch.from_numpy(u_all[t]))
            torch.cuda.synchronize()
            graphs[t & 1].replay()
            torch.cuda.synchronize()
            assert (np_(calls[t & 1][2].out["tokens"]) == tokens[t]).all(), (again, t)
