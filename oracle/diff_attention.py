"""Differential attention and its gradient in fp64, row by row from the definition."""
from __future__ import annotations

import numpy as np


def kept_keys(shape, b, h, mask=None, causal=False, q_start=None, kv_lens=None):
    """bool [q_len][kv_len]: the keys that the queries of head h of sequence b see. shape: (m, n, block)."""
    m, n, blk = shape
    i, j = np.arange(m)[:, None], np.arange(n)[None, :]
    keep = np.broadcast_to(j < (n if kv_lens is None else int(kv_lens[b])), (m, n)).copy()
    if causal:
        keep &= j <= i + (n - m if q_start is None else int(q_start[b]))
    if mask is not None:
        keep &= mask[b, h][i // blk, j // blk] != 0
    return keep


def softmax_map(q, k, keep, scale):
    """(P, log-sum-exp) of one map; a row that sees no key gets P = 0 and -inf."""
    s = np.where(keep, scale * (q @ k.T), -np.inf)
    top = s.max(-1, initial=-np.inf)
    safe = np.where(np.isneginf(top), 0.0, top)
    e = np.exp(s - safe[:, None])
    total = e.sum(-1)
    with np.errstate(divide="ignore"):
        lse = safe + np.log(total)
    return e / np.where(total > 0, total, 1.0)[:, None], lse


def forward_backward(q, k, v, lam, block=128, scale=None, dout=None, **kw):
    """q [B][2H][M][d], k [B][2Hk][N][d], v [B][Hk][N][dv], lam [H], fp64. A dict: o, maps (each P_m V), lse and, given dout, dq, dk, dv,
    dlam; "bound" holds the same outputs with every product and sum taken of magnitudes (for error bounds)."""
    b_, h2, m, d = q.shape
    hk, n, dv = v.shape[1:]
    h_ = h2 // 2
    scale = 1 / np.sqrt(d) if scale is None else scale
    out = dict(o=np.zeros((b_, h_, m, dv)), maps=np.zeros((b_, h2, m, dv)), lse=np.zeros((b_, h2, m)))
    names = ("dq", "dk", "dv") if dout is not None else ()
    out.update({x: np.zeros_like(y) for x, y in zip(names, (q, k, v))})
    bound = {x: np.zeros_like(y) for x, y in out.items()}
    if names:
        out["dlam"], bound["dlam"] = np.zeros(h_), np.zeros(h_)
    for b in range(b_):
        for h in range(h_):
            x = h // (h_ // hk)
            keep = kept_keys((m, n, block), b, h, **kw)
            vx = np.where(keep.any(0)[:, None], v[b, x], 0.0)     # keys no query sees do not matter, whatever they hold
            ks = [np.where(keep.any(0)[:, None], k[b, 2 * x + t], 0.0) for t in range(2)]
            maps = [softmax_map(q[b, 2 * h + t], ks[t], keep, scale) for t in range(2)]
            p = [y[0] for y in maps]
            out["lse"][b, 2 * h], out["lse"][b, 2 * h + 1] = maps[0][1], maps[1][1]
            av = np.abs(vx)
            for t in range(2):
                out["maps"][b, 2 * h + t], bound["maps"][b, 2 * h + t] = p[t] @ vx, p[t] @ av
            out["o"][b, h] = out["maps"][b, 2 * h] - lam[h] * out["maps"][b, 2 * h + 1]
            bound["o"][b, h] = bound["maps"][b, 2 * h] + abs(lam[h]) * bound["maps"][b, 2 * h + 1]
            if not names:
                continue
            do = dout[b, h]
            dp, adp = do @ vx.T, np.abs(do) @ av.T
            out["dv"][b, x] += (p[0] - lam[h] * p[1]).T @ do
            bound["dv"][b, x] += (p[0] + abs(lam[h]) * p[1]).T @ np.abs(do)
            for t, w in ((0, 1.0), (1, -lam[h])):
                mean, amean = (p[t] * dp).sum(-1), (p[t] * adp).sum(-1)
                ds, ads = w * p[t] * (dp - mean[:, None]) * scale, abs(w) * p[t] * (adp + amean[:, None]) * scale
                out["dq"][b, 2 * h + t] = ds @ ks[t]
                out["dk"][b, 2 * x + t] += ds.T @ q[b, 2 * h + t]
                bound["dq"][b, 2 * h + t] = ads @ np.abs(ks[t])
                bound["dk"][b, 2 * x + t] += ads.T @ np.abs(q[b, 2 * h + t])
                if t == 1:
                    out["dlam"][h] -= mean.sum()
                    bound["dlam"][h] += amean.sum()
    out["bound"] = bound
    return out
