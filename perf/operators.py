"""Performance cases of rotary positions and of differential attention.

A case is a dict of plain values; ``op`` names the calls it stands for:

  rotary  rotary: q and k rotated by their positions, read in one layout and written in another
          ("back": the gradient's direction)
  diff    diff_attn: q, k, v and the heads' weights in, O out
  step    diff_attn with its statistics, then diff_attn_backward: one training pass through the layer,
          O and every gradient out

``own`` false computes them in elementary torch operations in 32 bits (angles in 64), so the file also runs where
the framework lacks the calls.

Differential attention has two maps a head, P_m = softmax(Q_m K_m^T / sqrt(d)) over the kept keys, and
O = P_1 V - lam_h P_2 V. Sizes are those of the repository's video workloads (32,760 tokens of 30 x 52 latent
frames, 75,600 of 45 x 80) or generic ones of text models. Masks keep, per query block, a heavy-tailed number of
blocks, most of them near.
"""
from __future__ import annotations

import math

import torch

own = False

_CHUNK = 1 << 28  # scores that the plain form holds at once


# ---- cases -------------------------------------------------------------------------------------------------

def _rotary(batch, tokens, heads, kv_heads, d, pairs, layout="half", dtype="bf16", axes=1, scaling="none", factor=1.0,
            far=0, token_major=False, back=False):
    """``pairs``: rotated pairs of a head (2 pairs <= d); ``far``: the first position, 0 for positions that
    start at zero; ``token_major``: the side of the projections is [B][N][H][d]."""
    return dict(op="rotary", batch=batch, tokens=tokens, heads=heads, kv_heads=kv_heads, d=d, pairs=pairs, layout=layout,
                dtype=dtype, axes=axes, scaling=scaling, factor=factor, far=far, token_major=token_major, back=back)


def _diff(op, batch, heads, kv_heads, q_len, kv_len, d, dv, block=128, rho=1.0, causal=False, ragged=False):
    """``rho``: share of the blocks that the mask keeps, 1 for no mask; ``ragged``: sequences of half to the
    whole kv_len in the batch."""
    return dict(op=op, batch=batch, heads=heads, kv_heads=kv_heads, q_len=q_len, kv_len=kv_len, d=d, dv=dv, block=block,
                rho=rho, causal=causal, ragged=ragged)


def listed():
    cases = [
        # one new token of eight sequences, at positions far past the trained length (latency)
        ("rotary-token", _rotary(8, 1, 32, 8, 128, 64, scaling="yarn", factor=8.0, far=100000)),
        # a small video layer: (t, y, x) positions, from the projections' layout to the attention's
        ("rotary-480p", _rotary(1, 32760, 12, 12, 128, 64, layout="interleaved", axes=3, token_major=True)),
        # gradients in 32 bits, half of the head rotated, odd length, stretched positions
        ("rotary-back-odd", _rotary(3, 4999, 7, 7, 64, 16, dtype="fp32", scaling="linear", factor=4.0, back=True)),
        # gradients of a large video layer, back to the projections' layout
        ("rotary-back-720p", _rotary(1, 75600, 40, 40, 128, 64, layout="interleaved", axes=3, token_major=True,
                                     back=True)),
        # one new token of sixteen sequences of different lengths, four heads to a key head
        ("diff-token", _diff("diff", 16, 16, 4, 1, 8192, 64, 128, causal=True, ragged=True)),
        # one new token of one long sequence: a few rows, a long axis
        ("diff-token-long", _diff("diff", 1, 8, 8, 1, 131072, 128, 256, causal=True)),
        # a small odd layer of 64-token blocks
        ("diff-odd", _diff("diff", 2, 5, 5, 1237, 1237, 64, 64, block=64, rho=0.3)),
        # a prompt of a text model
        ("diff-causal", _diff("diff", 2, 16, 4, 4096, 4096, 64, 128, causal=True)),
        # a small video layer: 12 maps in 6 differential heads over the block mask
        ("diff-480p", _diff("diff", 1, 6, 6, 32760, 32760, 128, 256, rho=0.15)),
        # training of a small odd layer
        ("step-odd", _diff("step", 2, 3, 3, 777, 777, 128, 128, block=64, rho=0.5)),
        # training of a text layer with shared key heads and a padded batch
        ("step-causal", _diff("step", 2, 16, 4, 2048, 2048, 64, 128, causal=True, ragged=True)),
        # training of a short video layer: nine latent frames
        ("step-video", _diff("step", 1, 6, 6, 14040, 14040, 128, 256, rho=0.25)),
    ]
    return [dict(c, name=n) for n, c in cases]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "rotary", "diff", "diff", "token", "step", "step"])
    if kind == "rotary":
        d = rng.choice([64, 96, 128])
        heads = rng.choice([4, 7, 12, 16, 32, 40])
        kv = rng.choice([heads, heads, max(1, heads // 4)])
        batch = rng.choice([1, 1, 2, 5, 8])
        tokens = _log(rng, 1, max(2, 75600 * 80 * 128 // (d * batch * (heads + kv) * 2)))
        axes = rng.choice([1, 1, 3])
        scaling = "none" if axes == 3 else rng.choice(["none", "linear", "ntk", "yarn"])
        return _rotary(batch, tokens, heads, kv, d, rng.choice([d // 2, d // 2, d // 4, 11]),
                       layout=rng.choice(["half", "interleaved"]), dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                       axes=axes, scaling=scaling, factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]),
                       far=0 if axes == 3 else rng.choice([0, 0, 30000, 1000000]), token_major=rng.choice([True, False]),
                       back=rng.choice([True, False]))
    d, dv = rng.choice([(64, 64), (64, 128), (128, 128), (128, 256)])
    kv = rng.choice([1, 2, 3, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 4])
    if kind == "token":
        batch = rng.choice([1, 2, 7, 16])
        kv_len = _log(rng, 1, 131072 * 8 // (kv * batch))
        q_len = min(kv_len, rng.choice([1, 1, 1, 2, 5]))
        return _diff("diff", batch, heads, kv, q_len, kv_len, d, dv, causal=True, ragged=rng.choice([True, False]))
    batch = rng.choice([1, 1, 2, 3])
    top = 32760 if kind == "diff" else 14040
    n = _log(rng, 33, min(top, int(math.sqrt(top * top * 6 / (batch * heads)))))
    if rng.random() < 0.5:
        return _diff(kind, batch, heads, kv, n, n, d, dv, causal=True, ragged=rng.choice([True, False]))
    return _diff(kind, batch, heads, kv, n, n, d, dv, block=rng.choice([64, 128]), rho=round(rng.uniform(0.05, 0.6), 3),
                 ragged=rng.choice([True, False]))


# ---- inputs ------------------------------------------------------------------------------------------------

def _types(case):
    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[case.get("dtype", "bf16")]


def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _axis_pairs(case):
    """Pairs of each axis: for three axes the first takes what two equal thirds leave."""
    p = case["pairs"]
    return [p] if case["axes"] == 1 else [p - 2 * (p // 3), p // 3, p // 3]


def _frequencies(case):
    """(float64 frequency per pair, factor of the rotated values): base^(-i/pairs) per axis, for one axis
    stretched by ``factor`` ("linear": all frequencies; "ntk": the base so that the last one is; "yarn": from none
    at 32 turns over the trained length to all at one, and the values grow by 0.1 ln factor + 1)."""
    base, s = 10000.0, case["factor"]
    if case["scaling"] == "ntk":
        base *= s ** (case["pairs"] / max(case["pairs"] - 1, 1))
    parts = [base ** (-torch.arange(p, dtype=torch.float64) / p) for p in _axis_pairs(case)]
    f, grow = torch.cat(parts), 1.0
    if case["scaling"] == "linear":
        f = f / s
    if case["scaling"] == "yarn":
        turns = 4096 * f / (2 * math.pi)
        keep = ((turns - 1) / (32 - 1)).clamp(0, 1)
        f = f * keep + f / s * (1 - keep)
        grow = 0.1 * math.log(s) + 1
    return f.cuda(), grow


def _positions(case, g):
    """int32 [axes][B][N]: one axis counts on from a first position of each sequence; three are the frame and the
    place in a 30 x 52 or 45 x 80 latent frame."""
    b, n = case["batch"], case["tokens"]
    t = torch.arange(n, device="cuda")
    if case["axes"] == 3:
        h, w = (45, 80) if n > 40000 else (30, 52)
        return torch.stack([t // (h * w), t // w % h, t % w]).to(torch.int32)[:, None].expand(3, b, n).contiguous()
    first = torch.randint(0, 4096, (b, 1), generator=g, device="cuda") + case["far"]
    return (first + t).to(torch.int32)[None].contiguous()


def _lengths(case, g):
    """int32 [B]: evenly from half to the whole of kv_len, in an order of the seed."""
    b, n = case["batch"], case["kv_len"]
    lens = [n - (n // 2) * i // b for i in range(b)]
    order = torch.randperm(b, generator=g, device="cuda")
    return torch.tensor(lens, dtype=torch.int32, device="cuda")[order]


def _row_counts(case):
    """Kept blocks of each query block: log-normal quantiles (sigma 0.8) around rho of the blocks, one row empty."""
    mb, nb = -(-case["q_len"] // case["block"]), -(-case["kv_len"] // case["block"])
    u = (torch.arange(mb, dtype=torch.float64) + 0.5) / mb
    w = torch.exp(0.8 * math.sqrt(2.0) * torch.erfinv(2 * u - 1))
    n = (w / w.mean() * case["rho"] * nb).round().clamp(1, nb).long()
    if mb > 4:
        n[0] = 0
    return n


def _mask(case, g):
    """uint8 [B][H][M_B][N_B]: row i keeps n_i blocks, drawn the likelier the nearer they are."""
    n = _row_counts(case).cuda()
    mb, nb = n.numel(), -(-case["kv_len"] // case["block"])
    shape = (case["batch"], case["heads"], mb, nb)
    order = torch.rand(shape[:3], generator=g, device="cuda").argsort(-1)
    far = (torch.arange(mb, device="cuda")[:, None] * nb / mb - torch.arange(nb, device="cuda")).abs() + 1
    rank = (far * -torch.log(torch.rand(shape, generator=g, device="cuda") + 1e-9)).argsort(-1).argsort(-1)
    return (rank < n[order][..., None]).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=case)
    if case["op"] == "rotary":
        b, n, d, dt = case["batch"], case["tokens"], case["d"], _types(case)
        outer = case["token_major"] and not case["back"]
        for name, h in (("q", case["heads"]), ("k", case["kv_heads"])):
            s[name] = _randn(g, (b, n, h, d), dt).transpose(1, 2) if outer else _randn(g, (b, h, n, d), dt)
        s["freq"], s["grow"] = _frequencies(case)
        s["pos"] = _positions(case, g)
        return s
    b, h, hk, d, dv = (case[x] for x in ("batch", "heads", "kv_heads", "d", "dv"))
    # gains of normalised queries and keys: scores of about one and a half in standard deviation
    s["q"] = _randn(g, (b, 2 * h, case["q_len"], d), torch.bfloat16, 1.25)
    s["k"] = _randn(g, (b, 2 * hk, case["kv_len"], d), torch.bfloat16, 1.25)
    s["v"] = _randn(g, (b, hk, case["kv_len"], dv), torch.bfloat16)
    s["lam"] = 0.2 + 0.6 * torch.rand(h, generator=g, device="cuda")
    s["mask"] = _mask(case, g) if case["rho"] < 1 else None
    s["lens"] = _lengths(case, g) if case["ragged"] else None
    # single tokens are the last of their sequences; a whole sequence starts at its first key
    whole = case["q_len"] == case["kv_len"]
    s["start"] = s["lens"] - case["q_len"] if case["ragged"] and case["causal"] and not whole else None
    if case["op"] == "step":
        s["dout"] = _randn(g, (b, h, case["q_len"], dv), torch.bfloat16)
    return s


# ---- the calls ---------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        import paper_2609_34814_amd as W
        if case["op"] == "rotary":
            out = {}
            if case["token_major"] and case["back"]:
                for name, x in (("out_q", state["q"]), ("out_k", state["k"])):
                    b, h, n, d = x.shape
                    out[name] = torch.empty((b, n, h, d), dtype=x.dtype, device=x.device).transpose(1, 2)
            return W.rotary(state["q"], state["k"], inv_freq=state["freq"], positions=state["pos"], layout=case["layout"],
                            axis_pairs=_axis_pairs(case), scale=state["grow"], backward=case["back"], **out)
        how = dict(block=case["block"], causal=case["causal"], q_start=state["start"], kv_lens=state["lens"])
        args = [state[x] for x in ("q", "k", "v", "lam", "mask")]
        if case["op"] == "diff":
            return W.diff_attn(*args, **how)
        o, maps, stats = W.diff_attn(*args, return_stats=True, **how)
        return (o, *W.diff_attn_backward(state["dout"], *args, maps, stats, **how))
    if case["op"] == "rotary":
        return tuple(_plain_rotary(state, state[x]) for x in ("q", "k"))
    return _plain_diff(state)


def _plain_rotary(state, x):
    case = state["case"]
    axis = torch.repeat_interleave(torch.arange(case["axes"], device="cuda"),
                                   torch.tensor(_axis_pairs(case), device="cuda"), output_size=case["pairs"])
    angle = state["pos"][axis].permute(1, 2, 0).double() * state["freq"]  # [B][N][pairs]
    if case["back"]:
        angle = -angle
    c, s = ((f(angle) * state["grow"]).float()[:, None] for f in (torch.cos, torch.sin))
    r = 2 * case["pairs"]
    xf = x.float()
    a, b = (xf[..., :r:2], xf[..., 1:r:2]) if case["layout"] == "interleaved" else (xf[..., :r // 2], xf[..., r // 2:r])
    lo, hi = a * c - b * s, a * s + b * c
    rot = torch.stack([lo, hi], -1).flatten(-2) if case["layout"] == "interleaved" else torch.cat([lo, hi], -1)
    y = torch.cat([rot, xf[..., r:]], -1).to(x.dtype)
    return y.transpose(1, 2).contiguous().transpose(1, 2) if case["token_major"] and case["back"] else y.contiguous()


def _kept(state, b, h, r0, r1):
    """Which keys rows [r0, r1) of heads ``h`` (a slice) of sequence ``b`` see: [heads or 1][rows][kv_len]."""
    case = state["case"]
    n, blk = case["kv_len"], case["block"]
    keys = torch.arange(n, device="cuda")
    ok = torch.ones((1, r1 - r0, n), dtype=torch.bool, device="cuda")
    if state["lens"] is not None:
        ok = ok & (keys < state["lens"][b])
    if case["causal"]:
        start = n - case["q_len"] if state["start"] is None else state["start"][b]
        ok = ok & (keys <= start + torch.arange(r0, r1, device="cuda")[:, None])
    if state["mask"] is not None:
        rows = state["mask"][b, h].bool()[:, torch.arange(r0, r1, device="cuda") // blk]
        ok = ok & rows[:, :, keys // blk]
    return ok


def _plain_diff(state):
    case = state["case"]
    q, k, v, lam = (state[x].float() for x in ("q", "k", "v", "lam"))
    b_, h_, hk, m, n, d, dv = (case[x] for x in ("batch", "heads", "kv_heads", "q_len", "kv_len", "d", "dv"))
    grp, scale, step = h_ // hk, 1 / math.sqrt(d), case["op"] == "step"
    q, k = q.view(b_, hk, grp, 2, m, d), k.view(b_, hk, 2, n, d)
    o = torch.empty((b_, h_, m, dv), device="cuda")
    if step:
        dout = state["dout"].float()
        dq, dk, dv_, dlam = torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v), torch.zeros_like(lam)
    rows = max(1, min(m, _CHUNK // (grp * n)))
    for b in range(b_):
        for x in range(hk):
            heads = slice(x * grp, (x + 1) * grp)
            lm = lam[heads, None, None]
            vx = v[b, x]
            for r0 in range(0, m, rows):
                r1 = min(r0 + rows, m)
                ok = _kept(state, b, heads, r0, r1)
                p = []
                for t in range(2):
                    s = torch.matmul(q[b, x, :, t, r0:r1], k[b, x, t].t().contiguous()) * scale
                    s = torch.where(ok, s, torch.full_like(s, -math.inf))
                    top = s.amax(-1, keepdim=True)
                    e = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
                    total = e.sum(-1, keepdim=True)
                    p.append(e / torch.where(total > 0, total, torch.ones_like(total)))
                diff = p[0] - lm * p[1]
                o[b, heads, r0:r1] = torch.matmul(diff, vx)
                if not step:
                    continue
                do = dout[b, heads, r0:r1]
                dp = torch.matmul(do, vx.t().contiguous())
                dv_[b, x] += torch.matmul(diff.flatten(0, 1).t().contiguous(), do.flatten(0, 1))
                for t in range(2):
                    mean = (p[t] * dp).sum(-1, keepdim=True)
                    ds = p[t] * (dp - mean) * scale
                    if t == 1:
                        dlam[heads] -= mean.sum((1, 2))
                        ds = -lm * ds
                    dq[b, x, :, t, r0:r1] = torch.matmul(ds, k[b, x, t])
                    dk[b, x, t] += torch.matmul(ds.flatten(0, 1).t().contiguous(), q[b, x, :, t, r0:r1].flatten(0, 1))
    o = o.bfloat16()
    if not step:
        return o
    return o, dq.view(b_, 2 * h_, m, d).bfloat16(), dk.view(b_, 2 * hk, n, d).bfloat16(), dv_.bfloat16(), dlam


# ---- what a pass cannot do without -------------------------------------------------------------------------

def _scores(case):
    """Kept (query, key) pairs of one head, over the batch: exact without a mask; with one, rows of whole blocks."""
    b, m, n = case["batch"], case["q_len"], case["kv_len"]
    lens = [n - (n // 2) * i // b if case["ragged"] else n for i in range(b)]
    total = 0.0
    for length in lens:
        if case["rho"] < 1:
            total += float(_row_counts(case).sum()) * case["block"] ** 2 * length / (-(-n // case["block"]) * case["block"])
        elif case["causal"]:
            start = length - m if m < n else n - m
            first, last = min(max(start + 1, 0), length), min(max(start + m, 0), length)
            total += (first + last) * (last - first + 1) / 2 + (m - (last - first + 1)) * length
        else:
            total += float(m) * length
    return total


def work(case):
    if case["op"] == "rotary":
        size = 4 if case["dtype"] == "fp32" else 2
        rows = case["batch"] * case["tokens"] * (case["heads"] + case["kv_heads"])
        return dict(bytes=2 * rows * case["d"] * size + 4 * case["axes"] * case["batch"] * case["tokens"] + 8 * case["pairs"],
                    flops=6 * rows * case["pairs"])
    b, h, hk, m, n, d, dv = (case[x] for x in ("batch", "heads", "kv_heads", "q_len", "kv_len", "d", "dv"))
    used = sum(n - (n // 2) * i // b for i in range(b)) if case["ragged"] else b * n
    kv, qs, os_ = 2 * hk * used * (2 * d + dv), 2 * b * 2 * h * m * d, 2 * b * h * m * dv
    mask = b * h * -(-m // case["block"]) * -(-n // case["block"]) if case["rho"] < 1 else 0
    pairs = h * _scores(case)
    if case["op"] == "diff":
        return dict(bytes=kv + qs + os_ + mask, flops=pairs * (4 * d + 4 * dv))
    grads = 2 * b * hk * n * (2 * d + dv) + qs
    return dict(bytes=kv + qs + 2 * os_ + mask + grads, flops=pairs * (16 * d + 8 * dv))


# ---- from the definition, in 64 bits -----------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return tuple(_exact_rotary(s, s[x]) for x in ("q", "k"))
    b_, h_, hk, m, n = (case[x] for x in ("batch", "heads", "kv_heads", "q_len", "kv_len"))
    step, grp = case["op"] == "step", h_ // hk
    names = ("q", "k", "v", "lam")
    leaf = {x: s[x].double().requires_grad_(step) for x in names}
    out = torch.zeros((b_, h_, m, case["dv"]), dtype=torch.float64, device="cuda")
    rows = max(1, min(m, (1 << 27) // n))
    grads = {x: torch.zeros_like(leaf[x]) for x in names}
    with torch.set_grad_enabled(step):
        for b in range(b_):
            for h in range(h_):
                for r0 in range(0, m, rows):
                    r1 = min(r0 + rows, m)
                    ok = _exact_kept(s, b, h, r0, r1)
                    pick = [leaf["q"][b, 2 * h:2 * h + 2, r0:r1], leaf["k"][b, 2 * (h // grp):2 * (h // grp) + 2],
                            leaf["v"][b, h // grp], leaf["lam"][h]]
                    pick = [x.detach().requires_grad_(step) for x in pick]
                    qx, kx, vx, lm = pick
                    some = ok.any(-1, keepdim=True)
                    maps = []
                    for t in range(2):
                        sc = (qx[t] @ kx[t].T) / math.sqrt(case["d"])
                        lse = torch.logsumexp(sc.masked_fill(~ok, -math.inf).masked_fill(~some, 0.0), -1, keepdim=True)
                        maps.append(torch.exp(sc - lse).masked_fill(~ok, 0.0) @ vx)
                    y = maps[0] - lm * maps[1]
                    out[b, h, r0:r1] = y.detach()
                    if step:
                        gq, gk, gv, gl = torch.autograd.grad(y, pick, s["dout"][b, h, r0:r1].double())
                        grads["q"][b, 2 * h:2 * h + 2, r0:r1] = gq
                        grads["k"][b, 2 * (h // grp):2 * (h // grp) + 2] += gk
                        grads["v"][b, h // grp] += gv
                        grads["lam"][h] += gl
    return (out, *(grads[x].detach() for x in names)) if step else out


def _exact_kept(s, b, h, r0, r1):
    case = s["case"]
    i = torch.arange(r0, r1, device="cuda")[:, None]
    j = torch.arange(case["kv_len"], device="cuda")[None, :]
    length = case["kv_len"] if s["lens"] is None else int(s["lens"][b])
    keep = (j < length).expand(r1 - r0, -1)
    if case["causal"]:
        first = case["kv_len"] - case["q_len"] if s["start"] is None else int(s["start"][b])
        keep = keep & (i + first >= j)
    if s["mask"] is not None:
        keep = keep & (s["mask"][b, h][i // case["block"], j // case["block"]] != 0)
    return keep


def _exact_rotary(s, x):
    """The pairs as complex numbers, turned by grow * exp(i p f)."""
    case, p = s["case"], s["case"]["pairs"]
    first = 0
    turn = []
    for a, width in enumerate(_axis_pairs(case)):
        turn.append(s["pos"][a].double()[..., None] * s["freq"][first:first + width])
        first += width
    theta = torch.cat(turn, -1)[:, None]
    rot = torch.polar(torch.full_like(theta, s["grow"]), -theta if case["back"] else theta)
    xd = x.double()
    head = xd[..., :2 * p]
    pairs = head.unflatten(-1, (p, 2)) if case["layout"] == "interleaved" else head.unflatten(-1, (2, p)).transpose(-1, -2)
    z = torch.view_as_real(torch.complex(pairs[..., 0], pairs[..., 1]) * rot)
    if case["layout"] != "interleaved":
        z = z.transpose(-1, -2)
    return torch.cat([z.flatten(-2), xd[..., 2 * p:]], -1)
