"""Verification of drafted tokens in float64, from the definitions in include/dppo.h, sequence by sequence."""
import numpy as np


def _softmax(row, tau):
    if np.isnan(row).any() or np.isposinf(row).any():
        return None
    p = np.zeros(row.size)
    live = row > -np.inf
    if live.any():
        x = (row[live] - row[live].max()) / tau
        p[live] = np.exp(x) / np.exp(x).sum()
    return p


def verify_drafts(target, draft, drafts, cu, u, noise, tau, draft_tau):
    """target float64 [T + B, V], draft [T, V] or None, drafts int [T], cu int [B + 1], u [T], noise [B, V].  Returns n_accepted [B],
    tokens [T + B], logp [T + B], and margin [B]: the smallest relative distance at which a decision of the sequence turns."""
    B, V = len(cu) - 1, target.shape[1]
    T = cu[-1]
    out = dict(n_accepted=np.zeros(B, dtype=np.int64), tokens=np.full(T + B, -1, dtype=np.int64), logp=np.zeros(T + B), margin=np.full(B, np.inf))
    for b in range(B):
        n = cu[b + 1] - cu[b]
        at = cu[b] + b
        for j in range(n + 1):
            p = _softmax(target[at + j], tau)
            q = _softmax(draft[cu[b] + j], draft_tau) if draft is not None and j < n else np.zeros(V)
            y = drafts[cu[b] + j] if j < n else -1
            if draft is None and 0 <= y < V:
                q[y] = 1.0
            if p is None or q is None or not p.any():
                out["logp"][at + j] = -np.inf if p is not None and q is not None else np.nan
                break
            if 0 <= y < V:
                uq = u[cu[b] + j] * q[y]
                if p[y] > 0:
                    out["margin"][b] = min(out["margin"][b], abs(uq - p[y]) / p[y])
                if uq < p[y]:
                    out["tokens"][at + j], out["logp"][at + j] = y, np.log(p[y])
                    out["n_accepted"][b] += 1
                    continue
            w = np.maximum(p - q, 0.0)
            if not w.any():
                w = p
            r = w / noise[b]
            v = int(np.argmax(r))
            second = np.delete(r, v).max() if V > 1 else 0.0
            out["margin"][b] = min(out["margin"][b], 1.0 - second / r[v])
            out["tokens"][at + j], out["logp"][at + j] = v, np.log(p[v])
            break
    return out
