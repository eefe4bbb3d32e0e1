"""Distillation from a teacher's top log-probs in float64, from the definitions in include/dppo.h, row by row."""
import numpy as np

GIVEN, NORMALIZED, REST = 0, 1, 2
LEAST_REST = 2.0 ** -16


def distill_topk(z, top_ids, top_logp, mode, temperature):
    """z: float64 [T, V]; top_ids int [T, K] (-1: no entry); top_logp [T, K].  Returns a dict: loss, lse [T], dz [T, V] (the gradient
    of each row's loss), and P, r, sigma [T] of the formulas."""
    T, V = z.shape
    out = dict(loss=np.zeros(T), lse=np.zeros(T), dz=np.zeros((T, V)), P=np.zeros(T), r=np.zeros(T), sigma=np.ones(T))
    for t in range(T):
        row = z[t]
        if np.isnan(row).any() or np.isposinf(row).any():
            out["loss"][t] = out["lse"][t] = np.nan
            out["dz"][t] = np.nan
            continue
        have = top_ids[t] >= 0
        ids, lp = top_ids[t][have], top_logp[t][have].astype(np.float64)
        p = np.exp(lp)
        P = p.sum()
        if mode == NORMALIZED:
            if P > 0:
                p, lp = p / P, lp - np.log(P)
            P = 1.0 if P > 0 else 0.0
        r = 1.0 - P if mode == REST and 1.0 - P > LEAST_REST else 0.0
        out["P"][t], out["r"][t] = P, r
        live = np.flatnonzero(row > -np.inf)
        if live.size == 0:
            out["lse"][t], out["loss"][t] = -np.inf, np.inf if P > 0 else 0.0
            continue
        m = row[live].max()
        x = np.full(V, -np.inf)
        x[live] = (row[live] - m) / temperature
        e = np.exp(x)
        S = e.sum()
        out["lse"][t] = m / temperature + np.log(S)
        lns = x - np.log(S)
        s = e / S
        on = p > 0
        with np.errstate(invalid="ignore"):
            loss = float((p[on] * (lp[on] - lns[ids[on]])).sum())
        listed = np.zeros(V, dtype=bool)
        listed[ids] = True
        out["sigma"][t] = e[~listed].sum() / S
        xr = x[~listed]                                              # the unlisted ones relative to their own maximum
        mr = xr.max() if xr.size else -np.inf
        er = np.exp(xr - mr) if mr > -np.inf else np.zeros(xr.size)
        dz = s * (P + r)
        np.subtract.at(dz, ids, p)
        if r > 0:
            loss += r * (np.log(r) - (np.log(er.sum()) + mr - np.log(S))) if mr > -np.inf else np.inf
            if mr > -np.inf:
                dz[~listed] -= r * er / er.sum()
        out["loss"][t] = loss
        out["dz"][t] = dz / temperature
    return out
