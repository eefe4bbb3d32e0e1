"""Scoring of given tokens in float64: log-probs with entropy and alternatives, their gradient, and the 8-bit product.

Written from the definitions in include/dppo.h, row by row; no code shared with the GPU path.
"""
import numpy as np


def token_logprobs(z, target, top_k, temperature):
    """z: float64 [T, V].  Returns a dict of float64 arrays logp, entropy, lse [T], top_ids (int) and top_logp [T, top_k]."""
    T, V = z.shape
    out = dict(logp=np.zeros(T), entropy=np.zeros(T), lse=np.zeros(T),
               top_ids=np.full((T, top_k), -1, dtype=np.int64), top_logp=np.full((T, top_k), -np.inf))
    for t in range(T):
        row = z[t]
        if np.isnan(row).any() or np.isposinf(row).any():
            for n in ("logp", "entropy", "lse"):
                out[n][t] = np.nan
            out["top_logp"][t] = np.nan
            continue
        live = np.flatnonzero(row > -np.inf)
        if live.size == 0:
            out["logp"][t] = out["lse"][t] = -np.inf
            continue
        m = row[live].max()
        x = (row[live] - m) / temperature
        e = np.exp(x)
        s = e.sum()
        l = np.log(s)
        out["lse"][t] = m / temperature + l
        out["entropy"][t] = l - (e * x).sum() / s
        if target is not None:
            out["logp"][t] = (row[target[t]] - m) / temperature - l
        order = live[np.lexsort((live, -row[live]))][:top_k]
        out["top_ids"][t, :len(order)] = order
        out["top_logp"][t, :len(order)] = (row[order] - m) / temperature - l
    return out


def token_logprobs_backward(z, target, dlogp, dentropy, temperature):
    """Gradient [T, V] of sum_t dlogp[t] logp[t] + dentropy[t] entropy[t] with respect to z (either may be None)."""
    T, V = z.shape
    g = np.zeros((T, V))
    for t in range(T):
        row = z[t]
        live = row > -np.inf
        if not live.any():
            continue
        x = (row[live] - row[live].max()) / temperature
        lnp = np.full(V, -np.inf)
        lnp[live] = x - np.log(np.exp(x).sum())
        p = np.exp(lnp)
        plnp = np.where(p > 0, p * np.where(p > 0, lnp, 0.0), 0.0)
        if dlogp is not None:
            g[t] -= dlogp[t] * p
            g[t, target[t]] += dlogp[t]
        if dentropy is not None:
            g[t] -= dentropy[t] * (plnp - p * plnp.sum())
    return g / temperature


def quantize_rows_i8(x):
    """x: float32 [M, K] (exact values of the input's type).  Returns codes int8 [M, K], scales float32 [M]."""
    x = x.astype(np.float32)
    amax = np.abs(x).max(axis=1)
    with np.errstate(all="ignore"):
        s = (amax * (np.float32(1.0) / np.float32(127.0))).astype(np.float32)
        q = np.rint((x / s[:, None]).astype(np.float32))
    fine = np.isfinite(amax)
    live = fine & (s > 0)
    q = np.where(live[:, None], np.clip(np.where(np.isfinite(q), q, 0), -127, 127), 0).astype(np.int8)
    return q, np.where(fine, s, np.float32(np.nan)).astype(np.float32)


def linear_i8(q, q_scale, w, w_scale):
    """Exact integer sums times the product of the scales, in float64 [M, N]."""
    acc = q.astype(np.int64) @ w.astype(np.int64).T
    return acc.astype(np.float64) * q_scale.astype(np.float64)[:, None] * w_scale.astype(np.float64)[None, :]
