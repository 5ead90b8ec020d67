"""CPU oracle of the operators on logits in hand and of the embedding.  TEST INFRASTRUCTURE ONLY.

Plain statements in fp64 and in whole numbers of what ``alr_top_logits``, ``alr_distill_*``,
``alr_sample_tokens``, ``alr_embed`` and ``alr_embed_grad`` compute.  Imports nothing from the
product package.  Pinned by tests/test_oracle_logits.py.
"""

from __future__ import annotations

import math

import numpy as np

NEG = -np.inf


def _f64(x):
    return np.asarray(x, dtype=np.float64)


def _lse(x):
    """log sum exp of a vector; -inf for none."""
    m = x.max() if x.size else NEG
    return NEG if m == NEG else m + math.log(np.exp(x - m).sum())


def order(z):
    """Token ids of a row's candidates (not -inf, not NaN), value descending, id ascending."""
    z = _f64(z)
    ids = np.flatnonzero(~np.isnan(z) & (z != NEG))
    return ids[np.argsort(-z[ids], kind="stable")]


def top_logits(Z, K, T=1.0):
    Z = _f64(Z)
    N, V = Z.shape
    val, idx = np.full((N, K), NEG), np.full((N, K), -1, dtype=np.int64)
    lse, rest = np.empty(N), np.empty(N)
    for r in range(N):
        o = order(Z[r])
        n = min(K, len(o))
        idx[r, :n], val[r, :n] = o[:n], Z[r, o[:n]]
        lse[r], rest[r] = _lse(Z[r, o] / T), _lse(Z[r, o[n:]] / T)
    return dict(top_val=val, top_idx=idx, lse=lse, lse_rest=rest)


def distill(Z, top_val, top_idx, rest=None, weight=None, T=1.0, lam=1.0):
    """Forward results and G, row by row; also `size`, the sum of the absolute terms of every G
    entry (what rounding errors are relative to)."""
    Z, top_val = _f64(Z), _f64(top_val)
    N, V = Z.shape
    w = np.ones(N) if weight is None else _f64(weight)
    out = {k: np.zeros(N) for k in ("loss_row", "ent_row", "lse", "lse_rest")}
    out["argmax"] = np.full(N, -1, dtype=np.int64)
    G, size = np.zeros((N, V)), np.zeros((N, V))
    for r in range(N):
        if w[r] == 0:
            continue
        s = Z[r] / T
        inside = (top_idx[r] >= 0) & (top_idx[r] < V)
        ids = np.asarray(top_idx[r])[inside].astype(np.int64)
        outside = np.ones(V, dtype=bool)
        outside[ids] = False
        lse, lse_rest = _lse(s), _lse(s[outside])
        out["lse"][r], out["lse_rest"][r] = lse, lse_rest
        if lse == NEG:
            continue
        out["argmax"][r] = int(np.argmax(s))
        a = np.append(top_val[r][inside] / T, NEG if rest is None else float(rest[r]))
        total = _lse(a)
        if total == NEG:
            continue
        p = np.exp(a - total)
        logq = np.append(s[ids] - lse, lse_rest - lse)
        on = p > 0
        out["loss_row"][r] = -(p[on] * logq[on]).sum()
        out["ent_row"][r] = -(p[on] * (a - total)[on]).sum()
        q = np.exp(s - lse)
        G[r], size[r] = q, q.copy()
        if p[-1] > 0 and lse_rest > NEG:
            share = p[-1] * np.exp(s[outside] - lse_rest)
            G[r, outside] -= share
            size[r, outside] += share
        np.subtract.at(G[r], ids, p[:-1])
        np.add.at(size[r], ids, p[:-1])
        G[r] *= w[r]
        size[r] *= w[r]
    ws = w.sum()
    out["weight_sum"] = ws
    out["wl_sum"] = float((w * out["loss_row"]).sum()) if N else 0.0
    out["loss_total"] = lam * out["wl_sum"] / ws if ws > 0 else 0.0
    f = lam / (ws * T) if ws > 0 else 0.0
    out["G"], out["size"] = G * f, size * abs(f)
    return out


def sample(Z, w32, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """The draws in whole numbers.  w32 [N, V]: exp2((z - max) log2(e) / temperature) of each row as
    fp32 values (the definition's rounding); everything after them is exact."""
    Z = _f64(Z)
    N, V = Z.shape
    token, kept_n = np.full(N, -1, dtype=np.int64), np.zeros(N, dtype=np.int64)
    prob = np.zeros(N)
    for r in range(N):
        o = [int(v) for v in order(Z[r])]
        if not o:
            continue
        if temperature is not None and not temperature[r] > 0:
            token[r], prob[r], kept_n[r] = o[0], 1.0, 1
            continue
        a = {v: int(math.floor(float(w32[r, v]) * 2.0 ** 31)) for v in o}
        o = [v for v in o if a[v] > 0]
        if top_k is not None and top_k[r] > 0:
            o = o[:int(top_k[r])]
        if top_p is not None and top_p[r] < 1:
            lim, got, n = float(np.float32(top_p[r])) * float(sum(a[v] for v in o)), 0, 0
            while n < len(o) and (n == 0 or float(got) < lim):
                got += a[o[n]]
                n += 1
            o = o[:n]
        if min_p is not None:
            least = min(float(np.float32(min_p[r])), 1.0)
            o = [v for v in o if float(w32[r, v]) >= least]
        S = sum(a[v] for v in o)
        target, run = (int(u[r]) & 0xffffffff) * S >> 32, 0
        for v in sorted(o):
            run += a[v]
            if run > target:
                token[r], prob[r] = v, a[v] / S
                break
        kept_n[r] = len(o)
    return dict(token=token, prob=prob, n_kept=kept_n)


def embed(E, tokens, scale=1.0):
    E = _f64(E)
    out = np.zeros((len(tokens), E.shape[1]))
    for i, t in enumerate(tokens):
        if 0 <= t < E.shape[0]:
            out[i] = scale * E[t]
    return out


def embed_grad(dY, tokens, V, scale=1.0):
    """(gradient, sum of the absolute terms) of the table."""
    dY = _f64(dY)
    dE, size = np.zeros((V, dY.shape[1])), np.zeros((V, dY.shape[1]))
    for i, t in enumerate(tokens):
        if 0 <= t < V:
            dE[t] += scale * dY[i]
            size[t] += abs(scale) * np.abs(dY[i])
    return dE, size
