"""Attention over packed sequences and over a paged cache, and its gradient, in fp64 from the definition."""
from __future__ import annotations

import numpy as np


def rows(q, k, v, first, causal, scale, dout=None, u=2.0 ** -8):
    """One head of one sequence: queries q [M][d] at positions first, first + 1, ... over keys k, v [N][d]. A dict: o, lse, and with
    dout [M][d] dq, dk, dv; "tol" holds how far a computation may be off that has float32 scores and sums and rounds
    probabilities, dS and results to a type of half-step u:

      a score is off by some 130 roundings of 2^-24 of scale sum |q k|, which is below 30: 2^-12 in the exponent, so 2^-11 of a
      probability; the probability is rounded once, u; the result once more, u of it. In the gradient probabilities are
      recomputed (2^-11 again, and 2^-20 for the stored sum-exp), dP is off by 2^-17 of sum |dO V|, D = dO . O by sum |dO| times O's
      own tolerance, and dS is rounded once."""
    m, n = q.shape[0], k.shape[0]
    i, j = np.arange(m)[:, None], np.arange(n)[None, :]
    keep = (j <= first + i) if causal else np.ones((m, n), bool)
    s = np.where(keep, scale * (q @ k.T), -np.inf)
    top = s.max(-1, initial=-np.inf)
    safe = np.where(np.isneginf(top), 0.0, top)
    e = np.exp(s - safe[:, None])
    total = e.sum(-1)
    with np.errstate(divide="ignore"):
        lse = safe + np.log(total)
    p = e / np.where(total > 0, total, 1.0)[:, None]
    o, av, arith = p @ v, np.abs(v), (u + 2.0 ** -11) * (1 + u)
    # of fp16 probabilities, held 2^7 times larger, those below 2^-21 are off by 2^-32 each; its results below 2^-14 by 2^-25
    tiny = n * 2.0 ** -32 * (av.max(initial=0.0)) + 2.0 ** -25
    out = dict(o=o, lse=lse, tol=dict(o=arith * (p @ av) + u * np.abs(o) + tiny))
    if dout is None:
        return out
    ad, aq, ak = np.abs(dout), np.abs(q), np.abs(k)
    dp, d = dout @ v.T, (dout * o).sum(-1)
    err_d = (ad * out["tol"]["o"]).sum(-1) + 2.0 ** -17 * (ad * np.abs(o)).sum(-1)
    rel = 2.0 ** -11 + 2.0 ** -20
    ds = p * (dp - d[:, None]) * scale
    err_ds = scale * p * (rel * (np.abs(dp) + np.abs(d)[:, None]) + 2.0 ** -17 * (ad @ av.T) + err_d[:, None]) * (1 + rel)
    err_ds += u * (np.abs(ds) + err_ds)
    out.update(dq=ds @ k, dk=ds.T @ q, dv=p.T @ dout)
    out["tol"].update(dq=err_ds @ ak, dk=err_ds.T @ aq, dv=(rel + u * (1 + rel)) * (p.T @ ad))
    return out


def packed(q, k, v, starts, causal=True, scale=None, dout=None, u=2.0 ** -8):
    """q [T][H][d], k, v [T][Hk][d], starts a list. o, lse [H][T] (and dq, dk, dv), with "tol"; rows of no sequence are NaN."""
    t, h, d = q.shape
    grp, scale = h // k.shape[1], 1 / np.sqrt(d) if scale is None else scale
    names = ("o",) if dout is None else ("o", "dq", "dk", "dv")
    shape = dict(o=q.shape, dq=q.shape, dk=k.shape, dv=v.shape)
    out = {x: np.full(shape[x], np.nan) for x in names}
    tol = {x: np.full(shape[x], np.nan) for x in names}
    out["lse"] = np.full((h, t), np.nan)
    for a, b in zip(starts, starts[1:]):
        for x in ("dk", "dv"):
            if x in out:
                out[x][a:b], tol[x][a:b] = 0.0, 0.0
        for i in range(h):
            x = i // grp
            r = rows(q[a:b, i], k[a:b, x], v[a:b, x], 0, causal, scale, None if dout is None else dout[a:b, i], u)
            out["o"][a:b, i], tol["o"][a:b, i], out["lse"][i, a:b] = r["o"], r["tol"]["o"], r["lse"]
            if dout is not None:
                out["dq"][a:b, i], tol["dq"][a:b, i] = r["dq"], r["tol"]["dq"]
                for name in ("dk", "dv"):
                    out[name][a:b, x] += r[name]
                    tol[name][a:b, x] += r["tol"][name]
    for x in names[1:]:  # rounded once in the end
        tol[x] += u * np.abs(out[x])
    out["tol"] = tol
    return out


def paged(q, k, v, starts, causal=True, scale=None, u=2.0 ** -8):
    """k, v: lists of each sequence's keys and values [N_b][Hk][d]; its queries are the last of them."""
    t, h, d = q.shape
    scale = 1 / np.sqrt(d) if scale is None else scale
    out = dict(o=np.full(q.shape, np.nan), lse=np.full((h, t), np.nan), tol=dict(o=np.full(q.shape, np.nan)))
    for b, (a, e) in enumerate(zip(starts, starts[1:])):
        for i in range(h):
            x = i // (h // k[b].shape[1])
            r = rows(q[a:e, i], k[b][:, x], v[b][:, x], k[b].shape[0] - (e - a), causal, scale, None, u)
            out["o"][a:e, i], out["tol"]["o"][a:e, i], out["lse"][i, a:e] = r["o"], r["tol"]["o"], r["lse"]
    return out
