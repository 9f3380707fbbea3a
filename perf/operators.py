"""Operators of the output layer in 8-bit floating point, as cases that can be timed and checked one by one.

Three operators.  `quantize`: rows of fp32 into e4m3 codes with one power-of-two scale per block of 128 columns (weights when
a model is loaded, vectors that several products share).  `product`: the matrix product of such codes, from one vector (one
hypothesis) over panels (sentences side by side) to thousands (a table over the vocabulary).  `sample`: one token drawn per
row of logits from given random numbers, under temperature, top-k, top-p and min-p, with its log-probability and its embedding.

Where `own` is true `run` makes the library's calls; else it computes the same in elementary torch operations.  `exact` is the
definition in 64 bits.  Sizes are those of this repository's models (vocabularies of 33658 to 63644 words, 50000 most often,
inner dimensions 256 to 2048, the paper's 620) and, for the largest product and the largest vocabulary, generic ones.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
BLOCK = 128
E4M3_MAX = 448.0


def listed():
    return [
        # the gates' product of the smallest cell of the repository, one vector: a call whose time is latency
        {"name": "product_768x256_n1", "kind": "product", "rows": 768, "cols": 256, "n": 1, "x": "f32", "bias": True},
        # vocabulary matrix times the five hypotheses of a beam, inside a decoding step
        {"name": "product_50000x512_n5", "kind": "product", "rows": 50000, "cols": 512, "n": 5, "x": "f32", "bias": True},
        # the paper's largest vocabulary and inner dimension (rows that end inside a block and a tile), 77 sentences side by side
        {"name": "product_63644x620_n77", "kind": "product", "rows": 63644, "cols": 620, "n": 77, "x": "f32", "bias": True},
        # a full panel of 1024 slots against the vocabulary, vectors quantized by an earlier call
        {"name": "product_50000x512_n1024", "kind": "product", "rows": 50000, "cols": 512, "n": 1024, "x": "codes", "bias": True},
        # the largest: a table of products over thousands of vectors
        {"name": "product_8192x8192_n8192", "kind": "product", "rows": 8192, "cols": 8192, "n": 8192, "x": "codes", "bias": False},
        # vectors of a decoding step that two products share
        {"name": "quantize_8x1024", "kind": "quantize", "rows": 8, "cols": 1024},
        # the vocabulary matrix when a model is loaded
        {"name": "quantize_50000x620", "kind": "quantize", "rows": 50000, "cols": 620},
        # one sentence, plain drawing over the whole vocabulary, embedding of the next step
        {"name": "sample_50000_n1", "kind": "sample", "n": 1, "V": 50000, "filters": "none", "masked": False, "E": 512},
        # a serving batch, every row with its own temperature, top-k, top-p and min-p, some words masked
        {"name": "sample_50000_n64_mixed", "kind": "sample", "n": 64, "V": 50000, "filters": "mixed", "masked": True, "E": 512},
        # a small vocabulary, short list
        {"name": "sample_8001_n5_topk", "kind": "sample", "n": 5, "V": 8001, "filters": "top_k", "masked": False, "E": 0},
        # back-translation of a large batch under top-p, the paper's largest vocabulary
        {"name": "sample_63644_n1000_topp", "kind": "sample", "n": 1000, "V": 63644, "filters": "top_p", "masked": False, "E": 0},
        # a vocabulary of the size that multilingual models have, min-p
        {"name": "sample_250001_n12_minp", "kind": "sample", "n": 12, "V": 250001, "filters": "min_p", "masked": True, "E": 0},
    ]


def _between(rng, lo, hi):
    """A whole number in [lo, hi], even over the logarithm where the range is wide."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 1))) if hi > 10 * lo else rng.uniform(lo, hi + 1)
    return max(lo, min(hi, int(v)))


def draw(rng):
    kind = rng.choice(["product", "product", "panel", "quantize", "sample", "sample"])
    if kind == "product":                 # up to the slots of one batched call
        return {"kind": "product", "rows": _between(rng, 256, 63644), "cols": _between(rng, 64, 4096), "n": _between(rng, 1, 1024),
                "x": rng.choice(["f32", "codes"]), "bias": rng.random() < 0.7}
    if kind == "panel":                   # many vectors
        return {"kind": "product", "rows": _between(rng, 256, 8192), "cols": _between(rng, 64, 8192), "n": _between(rng, 1024, 8192),
                "x": rng.choice(["f32", "codes"]), "bias": rng.random() < 0.5}
    if kind == "quantize":
        return {"kind": "quantize", "rows": _between(rng, 1, 60000), "cols": _between(rng, 16, 2048)}
    V = _between(rng, 1000, 250000)
    return {"kind": "sample", "n": min(_between(rng, 1, 1024), 60_000_000 // V), "V": V, "masked": rng.random() < 0.5,
            "filters": rng.choice(["none", "top_k", "top_p", "min_p", "mixed"]), "E": rng.choice([0, 512, 620])}


# ---- inputs ---------------------------------------------------------------------------------------

def _up(v, m):
    return -(-v // m) * m


class _Draws:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def n(self, *shape, std=1.0):
        return torch.randn(*shape, generator=self.g, device=DEV, dtype=torch.float32) * std

    def u(self, *shape):
        """Uniform numbers of 24 bits in [0, 1)."""
        return torch.rand(*shape, generator=self.g, device=DEV, dtype=torch.float32)

    def i(self, lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=self.g, device=DEV)


def _padded(t):
    """The same rows at a pitch of whole 16 bytes, as the library's vectors have it."""
    n, cols = t.shape
    if cols % 4 == 0:
        return t
    buf = torch.zeros(n, _up(cols, 4), device=DEV)
    buf[:, :cols] = t
    return buf[:, :cols]


def _inputs(case, seed):
    """Every tensor of a case, from its seed."""
    d, kind = _Draws(seed), case["kind"]
    if kind == "quantize":
        # rows whose sizes differ, as those of a trained matrix do
        return {"X": _padded(d.n(case["rows"], case["cols"], std=0.05) * torch.exp(d.n(case["rows"], 1, std=0.7)))}
    if kind == "product":
        r, c, n = case["rows"], case["cols"], case["n"]
        p = {"W": d.n(r, c, std=0.05) * torch.exp(d.n(r, 1, std=0.5)), "X": _padded(torch.tanh(d.n(n, c)))}
        p["b"] = d.n(r, std=0.01) if case["bias"] else None
        return p
    n, V, f = case["n"], case["V"], case["filters"]
    # a model's logits: a frequency slope over the vocabulary, noise, and a few words that the context makes likely
    lg = d.n(n, V, std=1.5) - 0.6 * torch.log(torch.arange(V, device=DEV, dtype=torch.float32) + 20.0)
    lg.scatter_add_(1, d.i(0, V, n, 24), 9.0 * d.u(n, 24))
    if case["masked"]:
        lg.masked_fill_(d.u(n, V) < 0.02, -math.inf)                        # words that may not follow
        lg[:, d.i(0, V, max(1, V // 500))] = torch.finfo(torch.float32).min  # words that never may, masked by the lowest value
        if n > 8:
            lg[n // 2] = -math.inf                                          # a slot that is not in use
    p = {"logits": lg, "u": d.u(n), "T": None, "top_k": None, "top_p": None, "min_p": None}
    mixed = f == "mixed"
    if f != "none":
        p["T"] = 0.6 + 0.8 * d.u(n)
    if f == "top_k" or mixed:
        p["top_k"] = d.i(0 if mixed else 1, 100, n).to(torch.int32)         # 0: not in force
    if f == "top_p" or mixed:
        p["top_p"] = 0.5 + 0.5 * d.u(n)
    if f == "min_p" or mixed:
        p["min_p"] = 0.2 * d.u(n) * (d.u(n) < 0.7 if mixed else 1.0)        # 0: not in force
    if mixed:
        p["T"][::7] = 0.0                                                   # the best word, nothing drawn
    p["E_tgt"] = d.n(V, case["E"]) if case["E"] else None
    return p


# ---- the plain forms --------------------------------------------------------------------------------

def _blocks(X):
    """The rows as [rows, blocks, 128], filled up with zeros."""
    rows, cols = X.shape
    nb = -(-cols // BLOCK)
    if cols == nb * BLOCK:
        return X.reshape(rows, nb, BLOCK)
    return torch.nn.functional.pad(X, (0, nb * BLOCK - cols)).view(rows, nb, BLOCK)


def _quantize_plain(X):
    """(codes [rows, 16-byte pitch] as e4m3, exponents + 127 [rows, blocks] as bytes)."""
    cols, B = X.shape[1], _blocks(X)
    m = B.abs().amax(2)
    mant, ex = torch.frexp(m)                                # m = mant 2^ex, mant in [0.5, 1)
    e = ex - 9 + (mant > E4M3_MAX / 512.0).to(ex.dtype)      # smallest with m <= 448 2^e
    none = m < 2.0 ** -100
    e = torch.where(none, torch.zeros_like(e), e)
    inv = ((127 - e).to(torch.int32) << 23).view(torch.float32) * (~none).to(torch.float32)
    codes = (B * inv[:, :, None]).reshape(X.shape[0], -1).to(torch.float8_e4m3fn)
    ld = _up(cols, 16)
    if ld <= codes.shape[1]:
        codes = codes[:, :ld]
    return codes, (e + 127).to(torch.uint8)


def _values_plain(codes, scale, cols):
    v = _blocks(codes.to(torch.float32)[:, :cols])
    return (v * (scale.to(torch.int32) << 23).view(torch.float32)[:, :, None]).reshape(v.shape[0], -1)[:, :cols]


def _sample_plain(p):
    lg, u = p["logits"], p["u"].double()
    n, V = lg.shape
    inf = math.inf
    v = torch.where(torch.isnan(lg), torch.full_like(lg, -inf), lg)
    v, order = torch.sort(v, dim=1, descending=True, stable=True)
    best = v[:, :1]
    dead = v == -inf
    d = torch.where(v == best, 0.0, best.double() - v.double())
    T = torch.ones(n, device=lg.device) if p["T"] is None else p["T"]
    greedy = T <= 0
    w = torch.exp(-d / torch.where(greedy, torch.ones_like(T), T).double()[:, None])
    w = torch.where(dead, 0.0, w)
    rank = torch.arange(V, device=lg.device)[None, :]
    keep = ~dead
    if p["top_k"] is not None:
        k = p["top_k"][:, None]
        keep = keep & ((rank < k) | (k <= 0))
    if p["min_p"] is not None:
        small = w < p["min_p"].double()[:, None]
    w = torch.where(keep, w, 0.0)
    cum = torch.cumsum(w, 1)
    if p["top_p"] is not None:
        tp = p["top_p"].double()[:, None]
        before = torch.cat([torch.zeros_like(cum[:, :1]), cum[:, :-1]], 1)
        keep = keep & ((before < tp * cum[:, -1:]) | (tp >= 1))
    if p["min_p"] is not None:
        keep = keep & ~small
    keep[:, 0] = True
    Z = torch.where(keep, w, 0.0).sum(1, keepdim=True)
    hit = keep & (cum > u[:, None] * Z)
    at = torch.where(greedy, 0, torch.argmax(hit.to(torch.int8), 1))[:, None]
    empty = dead[:, 0]
    tokens = torch.where(empty, -1, torch.gather(order, 1, at)[:, 0]).to(torch.int32)
    e = torch.where(dead, 0.0, torch.exp(-d))
    logp = -torch.gather(d, 1, at)[:, 0] - torch.log(e.sum(1))
    out = {"tokens": tokens, "logp": torch.where(empty, -inf, logp).float()}
    if p["E_tgt"] is not None:
        out["y"] = p["E_tgt"][tokens.clamp(min=0).long()] * (tokens >= 0).to(torch.float32)[:, None]
    return out


# ---- states and passes --------------------------------------------------------------------------------

class _State:
    pass


def prepare(case, seed):
    st, p, kind = _State(), _inputs(case, seed), case["kind"]
    st.kind, st.case = kind, case
    if own:
        import paper_1804_05038_amd as q
    if kind == "quantize":
        st.p = p
        if own:
            ctx = q.Context(DEV, workspace_bytes=q.q8_workspace_bytes(1, 1, 16, 16))
            st.call = q.q8_quantize_matrix_f8(ctx, p["X"], bind=True)
    elif kind == "product":
        # the matrix as a program keeps it: quantized once
        r, c, n = case["rows"], case["cols"], case["n"]
        st.cols = c
        if own:
            ctx = q.Context(DEV, workspace_bytes=q.q8_gemm_f8_bytes(n, c))
            W = q.q8_quantize_matrix_f8(ctx, p["W"])
            X = p["X"] if case["x"] == "f32" else q.q8_quantize_matrix_f8(ctx, p["X"])
            Y = ctx.empty(n, _up(r, 4))[:, :r]
            st.call = q.q8_gemm_f8(ctx, W, X, p["b"], Y=Y, bind=True)
        else:
            st.W, st.b = _quantize_plain(p["W"]), p["b"]
            st.X = p["X"] if case["x"] == "f32" else _quantize_plain(p["X"])
    else:
        st.p = p
        if own:
            n, V = p["logits"].shape
            ctx = q.Context(DEV, workspace_bytes=q.q8_sample_bytes(n, V))
            y = ctx.empty(n, case["E"]) if case["E"] else None
            st.call = q.q8_sample_logits(ctx, p["logits"], p["u"], temperature=p["T"], top_k=p["top_k"], top_p=p["top_p"],
                                         min_p=p["min_p"], E_tgt=p["E_tgt"], y_emb=y, bind=True)
    return st


def run(st):
    kind = st.kind
    if own:
        st.call.launch()
        o = st.call.out
        if kind == "quantize":
            return {"codes": o["W"].data.view(torch.float8_e4m3fn), "scale": o["W"].scale}
        if kind == "product":
            return {"Y": o["Y"]}
        r = {"tokens": o["tokens"], "logp": o["logp"]}
        if st.case["E"]:
            r["y"] = o["y_emb"]
        return r
    if kind == "quantize":
        codes, scale = _quantize_plain(st.p["X"])
        return {"codes": codes, "scale": scale}
    if kind == "product":
        codes, scale = _quantize_plain(st.X) if st.case["x"] == "f32" else st.X
        y = _values_plain(codes, scale, st.cols) @ _values_plain(*st.W, st.cols).t()
        return {"Y": y if st.b is None else y + st.b}
    return _sample_plain(st.p)


# ---- what a pass cannot do without ------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "quantize":
        r, c = case["rows"], case["cols"]
        return {"bytes": 5 * r * c + r * -(-c // BLOCK), "flops": 3 * r * c}
    if kind == "product":
        r, c, n = case["rows"], case["cols"], case["n"]
        nb = -(-c // BLOCK)
        x = 4 * n * c if case["x"] == "f32" else n * (c + nb)
        return {"bytes": r * (c + nb) + x + 4 * n * r + (4 * r if case["bias"] else 0), "flops": 2 * n * r * c}
    n, V = case["n"], case["V"]
    # an exponential (taken as 10 operations), a comparison and a sum per word
    return {"bytes": 4 * n * V + 28 * n + 8 * n * case["E"], "flops": 12 * n * V}


# ---- the definition in 64 bits ------------------------------------------------------------------------

def _power(e):
    """2^e for whole e, exactly: the exponent field of a double."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _below(m):
    """The exponent of the power of two at or below m > 0."""
    return (m.view(torch.int64) >> 52) - 1023


def _e4m3(q):
    """|q| <= 448 rounded to the nearest e4m3 value, ties to even: steps of 2^-3 of the power of two below, at least 2^-9."""
    step = _power(_below(q.abs().clamp(min=2.0 ** -6)) - 3)
    return torch.round(q / step) * step


def _quantize_exact(X):
    """(values of the codes [rows, blocks, 128], exponents [rows, blocks]), in double."""
    rows, cols = X.shape
    nb = -(-cols // BLOCK)
    B = torch.zeros(rows, nb * BLOCK, device=DEV, dtype=torch.float64)
    B[:, :cols] = X
    B = B.view(rows, nb, BLOCK)
    m = B.abs().max(2).values
    none = m < 2.0 ** -100
    e = _below(m.clamp(min=2.0 ** -100)) - 8                 # 2^e 256 <= m
    e = torch.where(m > E4M3_MAX * _power(e), e + 1, e)
    e = torch.where(none, torch.zeros_like(e), e)
    return _e4m3(B / _power(e)[:, :, None]) * (~none)[:, :, None], e


def _whole(X):
    c, e = _quantize_exact(X)
    return (c * _power(e)[:, :, None]).view(X.shape[0], -1)


def _draw_exact(v, T, k, tp, mp, u):
    """One row, in numpy: (token, log-probability)."""
    live = np.flatnonzero(~np.isnan(v) & (v > -np.inf))
    if not len(live):
        return -1, -np.inf
    x = v[live].astype(np.float64)
    order = np.lexsort((live, -x))
    x, live = x[order], live[order]
    gap = np.zeros(len(x))
    np.subtract(x[0], x, out=gap, where=x != x[0])
    lse = math.log(math.fsum(np.exp(-gap)))
    if T <= 0:
        return int(live[0]), -lse
    w = np.exp(-gap / T)
    if k > 0:
        w = w[:k]
    m = len(w)
    cum = np.cumsum(w)
    if tp < 1:
        m = max(1, int(np.searchsorted(cum, tp * cum[-1], side="left")) + 1)
    m = max(1, min(m, int((w >= mp).sum())))
    at = min(int(np.searchsorted(cum[:m], u * cum[m - 1], side="right")), m - 1)
    return int(live[at]), -gap[at] - lse


def exact(case, seed):
    p, kind = _inputs(case, seed), case["kind"]
    if kind == "quantize":
        c, e = _quantize_exact(p["X"])
        rows, cols = p["X"].shape
        out = torch.zeros(rows, _up(cols, 16), device=DEV, dtype=torch.float64)
        out[:, :cols] = c.view(rows, -1)[:, :cols]
        return {"codes": out, "scale": (e + 127).to(torch.uint8)}
    if kind == "product":
        y = _whole(p["X"]) @ _whole(p["W"]).t()
        return {"Y": y if p["b"] is None else y + p["b"].double()}
    n = case["n"]
    col = lambda t, other: np.full(n, other) if t is None else t.cpu().numpy().astype(np.float64)
    lg, u = p["logits"].cpu().numpy(), p["u"].cpu().numpy().astype(np.float64)
    T, k, tp, mp = col(p["T"], 1.0), col(p["top_k"], 0), col(p["top_p"], 1.0), col(p["min_p"], 0.0)
    got = [_draw_exact(lg[i], T[i], int(k[i]), tp[i], mp[i], u[i]) for i in range(n)]
    tokens = torch.tensor([g[0] for g in got], dtype=torch.int32, device=DEV)
    out = {"tokens": tokens, "logp": torch.tensor([g[1] for g in got], dtype=torch.float64, device=DEV)}
    if p["E_tgt"] is not None:
        y = p["E_tgt"].double()[tokens.clamp(min=0).long()]
        y[tokens < 0] = 0.0
        out["y"] = y
    return out
