"""Operators of a recurrent decoder with 4-bit weights, as cases that can be timed and checked one by one.

Three operators.  `product`: the product of a matrix in 4 bits (a scale and a zero point per group of 32, 64 or 128 columns of a
row) with fp32 vectors, from one vector (one hypothesis) over a beam to the slots of a batched call.  `step`: one token of the
gated delta rule for n slots, S = a S + b k (v - k a S), o = q S with a state of dk x dv numbers per slot and head, where a beam
search may hand a slot another slot's state.  `sequence`: the same rule over whole sentences laid end to end, a source sentence
or a prompt, with the states they start from and end in.

Where `own` is true `run` makes the library's calls; else it computes the same in elementary torch operations.  `exact` is the
definition in 64 bits.  Sizes of products are those of this repository's models (vocabularies of 33658 to 63644 words, 50000 most
often, inner dimensions 256 to 2048, the paper's 620), of slots those of its beams and batches, of sentences those of its
workloads (up to 1024 words); heads and the longest sequence are generic.
"""
import itertools
import math
import random

import torch

own = False

DEV = "cuda:0"
CHUNK = 32              # of the plain sequence


def listed():
    return [
        # the gates' product of the smallest cell of the repository, one vector: a call whose time is latency
        {"name": "product_768x256_n1", "kind": "product", "rows": 768, "cols": 256, "n": 1, "group": 64, "bias": True},
        # a projection of one hypothesis, long rows
        {"name": "product_2048x8192_n1", "kind": "product", "rows": 2048, "cols": 8192, "n": 1, "group": 128, "bias": False},
        # vocabulary matrix times the five hypotheses of a beam, inside a decoding step
        {"name": "product_50000x512_n5", "kind": "product", "rows": 50000, "cols": 512, "n": 5, "group": 128, "bias": True},
        # the paper's largest vocabulary and inner dimension (rows that end inside a group), 77 sentences side by side, the finest groups
        {"name": "product_63644x620_n77", "kind": "product", "rows": 63644, "cols": 620, "n": 77, "group": 32, "bias": True},
        # a full panel of 1024 slots against the vocabulary
        {"name": "product_50000x512_n1024", "kind": "product", "rows": 50000, "cols": 512, "n": 1024, "group": 128, "bias": True},
        # the five hypotheses of a beam that take over each other's states, small heads: a call whose time is latency
        {"name": "step_n5_h4_64x64", "kind": "step", "n": 5, "hk": 4, "hv": 4, "dk": 64, "dv": 64, "parents": True, "resets": False},
        # 64 sentences side by side, every slot its own state
        {"name": "step_n64_h16_128x128", "kind": "step", "n": 64, "hk": 16, "hv": 16, "dk": 128, "dv": 128, "parents": False, "resets": False},
        # 200 sentences at beam 5, two heads of values for one of keys, odd sizes, some slots that start afresh
        {"name": "step_n1000_h6_100x72", "kind": "step", "n": 1000, "hk": 3, "hv": 6, "dk": 100, "dv": 72, "parents": True, "resets": True},
        # one source sentence
        {"name": "sequence_l50_h8_128x128", "kind": "sequence", "S": 1, "l": 50, "ragged": False, "hk": 8, "hv": 8, "dk": 128, "dv": 128,
         "start": False, "resets": False},
        # 64 source sentences of different lengths, two heads of values for one of keys, odd sizes
        {"name": "sequence_64xl120_h6_100x72", "kind": "sequence", "S": 64, "l": 120, "ragged": True, "hk": 3, "hv": 6, "dk": 100, "dv": 72,
         "start": True, "resets": True},
        # a batch of documents that go on from states
        {"name": "sequence_8xl1024_h16_128x128", "kind": "sequence", "S": 8, "l": 1024, "ragged": False, "hk": 16, "hv": 16, "dk": 128, "dv": 128,
         "start": True, "resets": False},
        # one long text
        {"name": "sequence_l16384_h16_128x128", "kind": "sequence", "S": 1, "l": 16384, "ragged": False, "hk": 16, "hv": 16, "dk": 128, "dv": 128,
         "start": False, "resets": False},
    ]


def _between(rng, lo, hi):
    """A whole number in [lo, hi], even over the logarithm where the range is wide."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 1))) if hi > 10 * lo else rng.uniform(lo, hi + 1)
    return max(lo, min(hi, int(v)))


def _heads(rng):
    hk, share = rng.choice([(1, 1), (2, 1), (4, 1), (8, 1), (16, 1), (1, 4), (3, 2), (4, 2), (8, 2)])
    d = lambda: rng.choice([32, 64, 64, 128, 128, _between(rng, 8, 128)])
    return {"hk": hk, "hv": hk * share, "dk": d(), "dv": d()}


def draw(rng):
    kind = rng.choice(["product", "product", "step", "sequence", "sequence"])
    if kind == "product":
        return {"kind": "product", "rows": _between(rng, 256, 50000), "cols": _between(rng, 64, 2048), "n": _between(rng, 1, 256),
                "group": rng.choice([32, 64, 128]), "bias": rng.random() < 0.7}
    h = _heads(rng)
    if kind == "step":
        return {"kind": "step", "n": min(_between(rng, 1, 1024), 33_000_000 // (h["hv"] * h["dk"] * h["dv"])), **h, "parents": rng.random() < 0.6,
                "resets": rng.random() < 0.4}
    l = _between(rng, 1, 4096)
    most = max(1, min(200, 100_000 // (l * h["hv"])))
    return {"kind": "sequence", "S": _between(rng, 1, most), "l": l, "ragged": rng.random() < 0.6, **h, "start": rng.random() < 0.5,
            "resets": rng.random() < 0.4}


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
    if kind == "product":
        r, c, n = case["rows"], case["cols"], case["n"]
        p = {"W": d.n(r, c, std=0.05) * torch.exp(d.n(r, 1, std=0.5)), "X": _padded(torch.tanh(d.n(n, c)))}
        p["b"] = d.n(r, std=0.01) if case["bias"] else None
        return p
    hk, hv, dk, dv = case["hk"], case["hv"], case["dk"], case["dv"]
    p = {"off": None, "parent": None, "scale": dk ** -0.5}
    if kind == "step":
        N, slots = case["n"], case["n"]
        if case["parents"]:                          # a beam's: groups of five slots take over states of their group
            at = torch.arange(N, device=DEV)
            p["parent"] = torch.minimum(at - at % 5 + d.i(0, 5, N), torch.full_like(at, N - 1)).to(torch.int32)
            if case["resets"]:
                p["parent"][d.u(N) < 0.1] = -1       # a new sentence in the slot
    else:
        S, l = case["S"], case["l"]
        lengths, rng = [l] * S, random.Random(S * 4099 + l)           # the same for every seed
        if case["ragged"]:
            lengths = [l] + [rng.randint(max(1, l // 12), l) for _ in range(S - 1)]
            if S > 4:
                lengths[S // 2] = 0                  # a slot that is not in use
        p["off"] = torch.tensor([0, *itertools.accumulate(lengths)], device=DEV, dtype=torch.int32)
        N, slots = sum(lengths), S
    # projections of one row of a layer lie side by side, as one product leaves them
    row = d.n(N, _up(2 * hk * dk + hv * dv, 4))
    row[:, hk * dk:2 * hk * dk] += 0.7 * d.n(hk * dk)                           # keys of a head resemble each other
    p["q"] = row[:, :hk * dk].view(N, hk, dk)
    p["k"] = row[:, hk * dk:2 * hk * dk].view(N, hk, dk)
    p["v"] = row[:, 2 * hk * dk:2 * hk * dk + hv * dv].view(N, hv, dv)
    rate = torch.exp(d.u(hv) * math.log(16.0)) * 0.03
    p["g"] = -rate * torch.nn.functional.softplus(d.n(N, hv))                   # the logarithm of the decay
    p["beta"] = torch.sigmoid(d.n(N, hv))
    if case["resets"]:
        p["g"][d.u(N) < 0.02] = -math.inf                                       # where a new document begins inside a sentence's place
    p["state"] = d.n(slots, hv, dk, dv, std=0.3) if kind == "step" or case["start"] else None
    return p


# ---- the plain forms --------------------------------------------------------------------------------

def _groups(X, G):
    rows, cols = X.shape
    ng = -(-cols // G)
    if cols != ng * G:
        X = torch.nn.functional.pad(X, (0, ng * G - cols))
    return X.reshape(rows, ng, G)


def _quantize_plain(W, G):
    """(codes [rows, groups, G], scales [rows, groups, 1], zero points) of finite weights."""
    B = _groups(W, G)
    lo, hi = B.amin(2, keepdim=True).clamp(max=0.0), B.amax(2, keepdim=True).clamp(min=0.0)
    # quotients rounded to 32 bits once, by way of 64: the device's own division in 32 bits may be an ulp off, which counts next to a border
    over = lambda x, y: (x.double() / y.double()).float()
    s = over(hi * 0.0625 - lo * 0.0625, torch.full_like(hi, 15.0)) * 16.0
    s = ((s.contiguous().view(torch.int32) + 0xFFFF) & -0x10000).view(torch.float32)       # up to 8 significant bits
    none = torch.maximum(hi, -lo) < 2.0 ** -100
    s = torch.where(none, torch.ones_like(s), s)
    z = torch.round(over(-lo, s))
    return (torch.round(over(B, s)) + z).clamp(0.0, 15.0).to(torch.uint8), s, z.to(torch.uint8)


def _values_plain(codes, s, z, cols):
    return ((codes.to(torch.float32) - z.to(torch.float32)) * s).reshape(codes.shape[0], -1)[:, :cols]


def _unit(x):
    return x / torch.sqrt((x * x).sum(-1, keepdim=True) + 1e-6)


def _step_plain(p):
    share = p["v"].shape[1] // p["q"].shape[1]
    q = (_unit(p["q"]) * p["scale"]).repeat_interleave(share, 1)
    k = _unit(p["k"]).repeat_interleave(share, 1)
    S = p["state"]
    if p["parent"] is not None:
        S = S[p["parent"].clamp(min=0).long()] * (p["parent"] >= 0).to(torch.float32)[:, None, None, None]
    S = S * torch.exp(p["g"])[:, :, None, None]
    u = (p["v"] - (k[..., None] * S).sum(2)) * p["beta"][..., None]
    S = S + k[..., None] * u[:, :, None, :]
    return {"out": (q[..., None] * S).sum(2), "state": S}


def _sequence_plain(p):
    """In chunks of 32 tokens: with D_ij = exp(sum of g over (j, i]) and A_ij = b_i D_ij k_i k_j below the diagonal, a chunk's
    updates are U = (I + A)^-1 b (V - exp(g_1 + .. + g_i) K S), and what it reads and leaves are products of those."""
    N, hv, dv = p["v"].shape
    hk, dk = p["q"].shape[1:]
    share, off = hv // hk, p["off"].long()
    S = off.numel() - 1
    lengths = off[1:] - off[:-1]
    nc = max(1, -(-p["l"] // CHUNK))
    # every sentence in whole chunks; what lies past its end keeps the state: no decay, nothing written
    at = torch.arange(nc * CHUNK, device=DEV)
    live = at[None, :] < lengths[:, None]
    src = torch.where(live, off[:-1, None] + at[None, :], 0)

    def laid(x, share=1):                              # [S, heads, chunks, 32, ...]
        x = torch.where(live.view(S, -1, *[1] * (x.dim() - 1)), x[src], torch.zeros((), device=DEV))
        x = x.reshape(S, nc, CHUNK, *x.shape[2:]).movedim(3, 1)
        return (x.repeat_interleave(share, 1) if share > 1 else x).contiguous()

    q, k, v = laid(_unit(p["q"]) * p["scale"], share), laid(_unit(p["k"]), share), laid(p["v"])
    g, b = laid(p["g"]), laid(p["beta"])
    run = torch.cumsum(g.double().clamp(min=-200.0), 3)       # exp(-200) is 0 here, and sums stay exact enough
    low = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=DEV).tril()
    D = torch.where(low, torch.exp(torch.where(low, run[..., :, None] - run[..., None, :], 0.0)), 0.0).float()
    kt = k.transpose(-1, -2).contiguous()
    A = (b[..., None] * D * torch.matmul(k, kt)).tril(-1)
    T = -A
    for i in range(1, CHUNK):                          # (I + A)^-1, row by row
        T[..., i, :i] += (T[..., i, :i, None] * T[..., :i, :i]).sum(-2)
    T = (T + torch.eye(CHUNK, device=DEV)) * b[..., None, :]
    M = D * torch.matmul(q, kt)
    e = torch.exp(run).float()[..., None]
    last = torch.exp(run[..., -1:] - run).float()[..., None]
    kt = (k * last).transpose(-1, -2).contiguous()
    state = torch.zeros(S, hv, dk, dv, device=DEV) if p["state"] is None else p["state"]
    out = torch.empty(S, hv, nc, CHUNK, dv, device=DEV)
    for c in range(nc):
        U = torch.matmul(T[:, :, c], v[:, :, c] - e[:, :, c] * torch.matmul(k[:, :, c], state))
        out[:, :, c] = e[:, :, c] * torch.matmul(q[:, :, c], state) + torch.matmul(M[:, :, c], U)
        state = state * e[:, :, c, -1:] + torch.matmul(kt[:, :, c], U)
    out = out.movedim(1, 3).reshape(S, nc * CHUNK, hv, dv)
    # back, sentence after sentence
    sent = torch.repeat_interleave(torch.arange(S, device=DEV), lengths, output_size=N)
    return {"out": out[sent, torch.arange(N, device=DEV) - off[sent]], "state": state}


# ---- states and passes --------------------------------------------------------------------------------

class _State:
    pass


def prepare(case, seed):
    st, p, kind = _State(), _inputs(case, seed), case["kind"]
    st.kind, st.case = kind, case
    if own:
        import paper_1804_05038_amd as q
    if kind == "product":
        # the matrix as a program keeps it: quantized once
        r, c, n = case["rows"], case["cols"], case["n"]
        st.cols = c
        if own:
            ctx = q.Context(DEV, workspace_bytes=q.q8_gemm_w4_bytes(n, c))
            W = q.q8_quantize_matrix_w4(ctx, p["W"], group=case["group"])
            Y = ctx.empty(n, _up(r, 4))[:, :r]
            st.call = q.q8_gemm_w4(ctx, W, p["X"], p["b"], Y=Y, bind=True)
        else:
            st.W, st.b, st.X = _quantize_plain(p["W"], case["group"]), p["b"], p["X"]
    elif own:
        if kind == "step":
            ctx = q.Context(DEV, workspace_bytes=q.q8_workspace_bytes(1, 1, 16, 16))
            st.call = q.q8_delta_step(ctx, p["q"], p["k"], p["v"], p["g"], p["beta"], p["state"], scale=p["scale"], normalize=True,
                                      parent=p["parent"], state_out=torch.empty_like(p["state"]), bind=True)
        else:
            ctx = q.Context(DEV, workspace_bytes=q.q8_delta_bytes(p["v"].shape[0], case["S"], case["hv"], case["dk"], case["dv"]))
            st.call = q.q8_delta_sequence(ctx, p["q"], p["k"], p["v"], p["g"], p["beta"], p["off"], scale=p["scale"], normalize=True,
                                          state=p["state"], bind=True)
    else:
        st.p = p
        if kind == "sequence":
            p["l"] = case["l"]
    return st


def run(st):
    kind = st.kind
    if own:
        st.call.launch()
        o = st.call.out
        return {"Y": o["Y"]} if kind == "product" else {"out": o["out"], "state": o["state"]}
    if kind == "product":
        y = st.X @ _values_plain(*st.W, st.cols).t()
        return {"Y": y if st.b is None else y + st.b}
    return _step_plain(st.p) if kind == "step" else _sequence_plain(st.p)


# ---- what a pass cannot do without ------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "product":
        r, c, n = case["rows"], case["cols"], case["n"]
        return {"bytes": r * (-(-c // 2) + 4 * -(-c // case["group"])) + 4 * n * c + 4 * n * r + (4 * r if case["bias"] else 0), "flops": 2 * n * r * c}
    hk, hv, dk, dv = case["hk"], case["hv"], case["dk"], case["dv"]
    slots = case["n"] if kind == "step" else case["S"]
    tokens = slots if kind == "step" else case["S"] * case["l"] * (0.55 if case["ragged"] and case["S"] > 1 else 1)
    states = 2 if kind == "step" or case["start"] else 1
    # the rule as it is written: k S, the update, q S
    return {"bytes": int(tokens * 4 * (2 * hk * dk + 2 * hv * dv + 2 * hv)) + 4 * states * slots * hv * dk * dv, "flops": int(6 * tokens * hv * dk * dv)}


# ---- the definition in 64 bits ------------------------------------------------------------------------

def _quantized_exact(W, G):
    """The values that the 4-bit codes stand for, in double.  The quotients are rounded to 32 bits, as the definition has them."""
    rows, cols = W.shape
    ng = -(-cols // G)
    B = torch.zeros(rows, ng * G, device=DEV, dtype=torch.float64)
    B[:, :cols] = W
    B = B.view(rows, ng, G)
    lo = torch.minimum(B.min(2).values, torch.zeros((), device=DEV, dtype=torch.float64))
    hi = torch.maximum(B.max(2).values, torch.zeros((), device=DEV, dtype=torch.float64))
    s = (((hi - lo).float().double() / torch.full_like(hi, 15.0)).float()).double()
    # the next number of 8 significant bits at or above
    unit = (((s.view(torch.int64) >> 52) - 7) << 52).view(torch.float64)
    s = torch.where(s > 0, torch.ceil(s / unit) * unit, torch.ones_like(s))[:, :, None]
    z = torch.round((-lo[:, :, None] / s).float()).double()
    c = torch.clamp(torch.round((B / s).float()).double() + z, 0, 15)
    return ((c - z) * s).view(rows, -1)[:, :cols]


def exact(case, seed):
    p, kind = _inputs(case, seed), case["kind"]
    if kind == "product":
        y = p["X"].double() @ _quantized_exact(p["W"], case["group"]).t()
        return {"Y": y if p["b"] is None else y + p["b"].double()}
    N, hv, dv = p["v"].shape
    hk, dk = p["q"].shape[1:]
    heads = torch.arange(hv, device=DEV) // (hv // hk)
    q, k, v, beta = (p[f].double() for f in ("q", "k", "v", "beta"))
    q = (q * (p["scale"] / torch.sqrt((q ** 2).sum(2, keepdim=True) + 1e-6)))[:, heads]
    k = (k / torch.sqrt((k ** 2).sum(2, keepdim=True) + 1e-6))[:, heads]
    a = torch.exp(p["g"].double())

    def token(S, t):
        """S [slots, heads, dk, dv] after the tokens t, and what they read."""
        S = S * a[t][:, :, None, None]
        miss = v[t] - torch.matmul(k[t][:, :, None, :], S)[:, :, 0]
        S = S + k[t][..., None] * (beta[t][..., None] * miss)[:, :, None, :]
        return S, torch.matmul(q[t][:, :, None, :], S)[:, :, 0]

    if kind == "step":
        S = p["state"].double()
        if p["parent"] is not None:
            S = torch.cat([S, torch.zeros_like(S[:1])])[torch.where(p["parent"] < 0, N, p["parent"]).long()]
        S, o = token(S, torch.arange(N, device=DEV))
        return {"out": o, "state": S}
    if case["l"] * max(1.0, case["S"] * hv * dk * dv / 1.5e7) > 40000:
        return None
    off = p["off"].tolist()
    # longest first: the sentences that still have a token are the first ones
    order = sorted(range(case["S"]), key=lambda s: off[s] - off[s + 1])
    first = torch.tensor([off[s] for s in order], device=DEV)
    S = torch.zeros(case["S"], hv, dk, dv, device=DEV, dtype=torch.float64)
    if p["state"] is not None:
        S += p["state"].double()[order]
    out = torch.zeros(N, hv, dv, device=DEV, dtype=torch.float64)
    lengths = [off[s + 1] - off[s] for s in order]
    m = case["S"]
    for t in range(lengths[0]):
        while lengths[m - 1] <= t:
            m -= 1
        at = first[:m] + t
        S[:m], out[at] = token(S[:m], at)
    back = torch.empty(case["S"], dtype=torch.int64, device=DEV)
    back[torch.tensor(order, device=DEV)] = torch.arange(case["S"], device=DEV)
    return {"out": out, "state": S[back]}
