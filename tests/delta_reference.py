"""The gated delta rule in 64 bits, token by token, and a bound of what sums in fp32 may be off."""
import numpy as np

EPS = 1e-6
C = 32


def prepared(q, k, scale, normalize, share):
    """Queries and keys per value head, in double: of unit length where asked, queries scaled."""
    q, k = np.asarray(q, np.float64), np.asarray(k, np.float64)
    if normalize:
        q = q / np.sqrt((q * q).sum(-1, keepdims=True) + EPS)
        k = k / np.sqrt((k * k).sum(-1, keepdims=True) + EPS)
    return np.repeat(q * scale, share, 1), np.repeat(k, share, 1)


def token(S, q, k, v, a, b):
    """S [hv, dk, dv] after one token, and what it reads [hv, dv]."""
    S = S * a[:, None, None]
    u = b[:, None] * (v - (k[:, None, :] @ S)[:, 0])
    S = S + k[:, :, None] * u[:, None, :]
    return S, (q[:, None, :] @ S)[:, 0]


def sequence(q, k, v, g, beta, off, scale=1.0, normalize=True, state=None):
    """(out [L, hv, dv], state [S, hv, dk, dv]); rows of no sequence are zeros."""
    hv, dk, dv = v.shape[1], q.shape[2], v.shape[2]
    q, k = prepared(q, k, scale, normalize, hv // q.shape[1])
    v, a, beta = np.asarray(v, np.float64), np.exp(np.asarray(g, np.float64)), np.asarray(beta, np.float64)
    out = np.zeros(v.shape)
    states = []
    for s in range(len(off) - 1):
        S = np.zeros((hv, dk, dv)) if state is None else np.asarray(state[s], np.float64)
        for t in range(off[s], off[s + 1]):
            S, out[t] = token(S, q[t], k[t], v[t], a[t], beta[t])
        states.append(S)
    return out, np.stack(states)


def step(q, k, v, g, beta, state, scale=1.0, normalize=True, parent=None):
    """(out [n, hv, dv], state [n, hv, dk, dv])."""
    n, hv, dv = v.shape
    dk = q.shape[2]
    S = np.zeros((n, hv, dk, dv)) if state is None else np.asarray(state, np.float64)
    if parent is not None:
        S = np.stack([S[p] if 0 <= p < len(S) else np.zeros((hv, dk, dv)) for p in parent])
    return sequence(q, k, v, g, beta, list(range(n + 1)), scale, normalize, S)


U = 2.0 ** -23        # of one operation: additions inside matrix operations need not round to nearest
TINY = 2.0 ** -100    # what may be lost besides: exp(-150) is 7e-66, below fp32's smallest number 2^-149, so that a decay is 0 in 32 bits and is not in 64;
                      # it multiplies states, keys and values of at most 2^20 here


def step_bound(q, k, v, g, beta, state, scale=1.0, normalize=True, parent=None):
    """What one token may be off, per slot, head and column: (out [n, hv, dv], state in 2-norm over dk [n, hv, dv]).  Sums of dk products and
    of the squares behind a unit length are off by at most dk U of the sum of magnitudes, at most the product of the two vectors' lengths; the
    other operations, the exponential's (two units) among them, are at most ten."""
    n, hv, dv = v.shape
    dk = q.shape[2]
    share = hv // q.shape[1]
    qn, kn = prepared(q, k, scale, normalize, share)
    S = np.zeros((n, hv, dk, dv)) if state is None else np.asarray(state, np.float64)
    if parent is not None:
        S = np.stack([S[p] if 0 <= p < len(S) else np.zeros((hv, dk, dv)) for p in parent])
    S = np.linalg.norm(S, axis=2) * np.exp(np.asarray(g, np.float64))[:, :, None]                              # length of a column
    kl, ql, b = np.linalg.norm(kn, axis=2)[..., None], np.linalg.norm(qn, axis=2)[..., None], np.abs(np.asarray(beta, np.float64))[..., None]
    u = b * (np.abs(v) + kl * S)                                                                   # at least |u|
    du = (2 * dk + 10) * U * u
    dS = kl * du + (dk + 10) * U * (S + kl * u)
    return ql * dS + (2 * dk + 10) * U * ql * (S + kl * u) + TINY, dS + TINY


def sequence_bound(q, k, v, g, beta, off, scale=1.0, normalize=True, state=None):
    """What chunks of C tokens in fp32 may be off: (out [L, hv, dv], state in 2-norm over dk [S, hv, dv]), for keys of at most unit length and
    beta in [0, 1], where the rule's own step does not lengthen an error of the state.  Per chunk, with A, T, M and K as matrices of
    magnitudes (their 2-norms), S the length of a column of the state and R >= |V| + |K S|:
      R: dk products a row;  T: substitution leaves a residual of at most C U |A| |T| in (I + A) T, so T is off by |T| C U |A| |T|, and A by
      (2 dk + 10) U |A| (its dot products, unit lengths, exponentials);  U = T R, O, and the new state: sums of C products."""
    hv, dk, dv = v.shape[1], q.shape[2], v.shape[2]
    share = hv // q.shape[1]
    qn, kn = prepared(q, k, scale, normalize, share)
    g, b = np.maximum(np.asarray(g, np.float64), -200.0), np.asarray(beta, np.float64)
    v = np.asarray(v, np.float64)
    out = np.zeros(v.shape)
    ends = []
    norm = lambda M: np.linalg.norm(M, 2, axis=(-2, -1))[:, None]                                  # [heads, 1]
    col = lambda M: np.linalg.norm(M, axis=1)                                                      # [heads, columns]
    for s in range(len(off) - 1):
        S = np.zeros((hv, dk, dv)) if state is None else np.asarray(state[s], np.float64)
        E = np.zeros((hv, dv))                                                                     # the error so far
        for t0 in range(off[s], off[s + 1], C):
            t1 = min(t0 + C, off[s + 1])
            m = t1 - t0
            K, Q, V = kn[t0:t1].transpose(1, 0, 2), qn[t0:t1].transpose(1, 0, 2), v[t0:t1].transpose(1, 0, 2)
            c, bb = np.cumsum(g[t0:t1], 0).T, b[t0:t1].T
            low = np.tril(np.ones((m, m)))
            D = np.exp(np.where(low > 0, c[:, :, None] - c[:, None, :], 0.0)) * low
            A = np.tril(bb[:, :, None] * D * (K @ K.transpose(0, 2, 1)), -1)
            T = np.linalg.inv(np.eye(m) + A) * bb[:, None, :]
            M = D * (Q @ K.transpose(0, 2, 1))
            e = np.exp(c)[:, :, None]
            R = V - e * (K @ S)
            Uu = T @ R
            # magnitudes: dot products of keys and queries are bounded by lengths, not by their values
            kl, ql = np.linalg.norm(K, axis=2), np.linalg.norm(Q, axis=2)
            Am = np.tril(bb[:, :, None] * D * kl[:, :, None] * kl[:, None, :], -1)
            Mm = D * ql[:, :, None] * kl[:, None, :]
            Ti = np.abs(np.linalg.inv(np.eye(m) + A))
            size = col(np.abs(V)) + np.linalg.norm(e[:, :, 0] * kl, axis=1)[:, None] * col(S)
            dR = (2 * dk + 10) * U * size
            dT = norm(Ti) ** 2 * (m * U * norm(np.abs(A)) + (2 * dk + 10) * U * norm(Am))
            dU = norm(T) * dR + dT * col(R) + (m + 10) * U * norm(np.abs(T)) * col(R)
            Kt = np.exp(c[:, -1:] - c)[:, :, None] * K
            after = e[:, -1] * 1.0
            dS = norm(Kt) * dU + (m + 2 * dk + 10) * U * norm(np.abs(Kt)) * col(Uu) + 6 * U * after * col(S)
            dO = np.max(e * ql[:, :, None], axis=1) * ((2 * dk + 10) * U * col(S) + E) + np.max(np.linalg.norm(M, axis=2), axis=1)[:, None] * dU + \
                (m + 2 * dk + 10) * U * np.max(np.linalg.norm(Mm, axis=2), axis=1)[:, None] * col(Uu)
            # an error of the chunk's first state reaches the results through the rule itself, whose step does not lengthen it
            out[t0:t1] = (dO + np.max(ql, axis=1)[:, None] * E)[None]
            S = after[:, :, None] * S + Kt.transpose(0, 2, 1) @ Uu
            E = after * E + dS
        ends.append(E)
    return out + TINY, np.stack(ends) + TINY
