"""Masked calls of many tiles in which some rows and columns of the block mask keep far more blocks than the others: those tiles are
computed in chunks that are joined."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2609_34814_amd as W                                     # noqa: E402
from tests.test_diff_attn import DIMS, make, reference               # noqa: E402


def uneven_mask(b, h, m, n, block):
    """Two or three blocks a row at random; full rows, full columns, and in some heads a row of nothing."""
    mb, nb = -(-m // block), -(-n // block)
    g = torch.Generator(device="cuda").manual_seed(3)
    mask = torch.rand((b, h, mb, nb), generator=g, device="cuda") < 2.5 / nb
    mask[..., ::9, :] = True
    mask[..., 3::7] = True
    mask[:, 1::3, -1] = False
    mask[:, 1::3, 0] &= torch.arange(nb, device="cuda") % 5 == 0
    return mask.to(torch.uint8)


def tiles_are_cut(lengths, block, waves):
    """More than 256 tiles, the longest of more blocks than its share."""
    slots = 256 if waves == 4 else 512
    share = max(-(-int(lengths.sum()) // slots), 1024 // block)
    return 256 < lengths.numel() <= 8192 and int(lengths.max()) > share


def check(args, mask, block, kw):
    """Equal calls give equal bits; the heads of the second key head, of two sequences at most, against the oracle."""
    q, k, v, lam = args
    b, h, hk, m, dv = q.shape[0], lam.numel(), v.shape[1], q.shape[2], v.shape[3]
    dout = torch.randn((b, h, m, dv), device="cuda", generator=torch.Generator(device="cuda").manual_seed(50)).to(torch.bfloat16)
    o, maps, stats = W.diff_attn(*args, mask, return_stats=True, **kw)
    assert torch.equal(W.diff_attn(*args, mask, **kw), o)
    got = W.diff_attn_backward(dout, *args, mask, maps, stats, **kw)
    assert all(torch.equal(x, y) for x, y in zip(got, W.diff_attn_backward(dout, *args, mask, maps, stats, **kw)))

    r, bs = h // hk, min(b, 2)
    hs, ks = slice(r, 2 * r), slice(1, 2)
    ms, kms = slice(2 * r, 4 * r), slice(2, 4)
    del kw["block"]
    if "kv_lens" in kw:
        kw["kv_lens"] = kw["kv_lens"][:bs]
    ref = reference([q[:bs, ms], k[:bs, kms], v[:bs, ks], lam[hs]], mask[:bs, hs], block, kw, dout[:bs, hs])
    # tolerances as for tiles that are not cut: chunks are held and joined in float32
    err = np.abs(o[:bs, hs].double().cpu().numpy() - ref["o"])
    tol = (2.0 ** -8 + 2.0 ** -11) * (1 + 2.0 ** -8) * ref["bound"]["o"] + 2.0 ** -8 * np.abs(ref["o"])
    assert np.all(err <= tol), float((err - tol).max())
    lse = stats[:bs, ms, :, 0].double().cpu().numpy()
    assert np.array_equal(np.isneginf(lse), np.isneginf(ref["lse"]))
    some = np.isfinite(ref["lse"])
    assert np.all(np.abs(lse[some] - ref["lse"][some]) <= 2.0 ** -11 + 2.0 ** -22 * np.abs(ref["lse"][some]))
    parts = dict(dq=got[0][:bs, ms], dk=got[1][:bs, kms], dv=got[2][:bs, ks])
    if bs == b:
        parts["dlam"] = got[3][hs]
    for name, y in parts.items():
        steps = {"dv": 1, "dlam": 0}.get(name, 2)
        err = np.abs(y.double().cpu().numpy() - ref[name])
        tol = (steps * 2.0 ** -8 + 2.0 ** -10) * (1 + 2.0 ** -7) * ref["bound"][name]
        tol += (2.0 ** -24 if name == "dlam" else 2.0 ** -8) * np.abs(ref[name])
        assert np.all(err <= tol), (name, float((err - tol).max()), float(err.max()))
        if np.linalg.norm(ref[name]) > 0 and name != "dlam":
            assert np.linalg.norm(err) <= 2.0 ** -6 * np.linalg.norm(ref[name]), name


@pytest.mark.gpu
@pytest.mark.parametrize("b,h,hk,m,n,block,causal,d,dv",
                         [(1, 16, 8, 2112, 2112, 64, False, *x) for x in DIMS]
                         + [(1, 16, 8, 2090, 2112, 64, True, 64, 64), (1, 16, 8, 2112, 2090, 64, True, 128, 256),
                            (1, 9, 9, 3900, 3900, 128, False, 128, 256), (1, 9, 9, 3900, 3900, 128, True, 64, 128),
                            (20, 14, 14, 5, 2300, 64, False, 128, 128), (20, 14, 14, 2300, 7, 64, False, 64, 64)])
def test_cut_tiles(b, h, hk, m, n, block, causal, d, dv):
    args, mask, kw = make(b, h, hk, m, n, d, dv), uneven_mask(b, h, m, n, block), dict(block=block, causal=causal)
    lens = torch.randint(n // 2, n + 1, (b,), generator=torch.Generator().manual_seed(4)).to("cuda", torch.int32)
    kw["kv_lens"] = lens
    rows = mask.long().sum(-1).flatten()
    cols = mask.long().view(b, hk, -1, mask.shape[-1]).sum(2).flatten()
    waves = 2 if block == 64 else 4
    assert tiles_are_cut(rows, block, waves) or tiles_are_cut(cols, block, waves)
    check(args, mask, block, kw)


@pytest.mark.gpu
@pytest.mark.parametrize("b,h,hk,m,n,block,causal,d,dv",
                         [(150, 28, 14, 2300, 7, 64, False, 64, 64), (76, 14, 14, 2300, 40, 64, False, 128, 128),
                          (76, 14, 14, 2300, 100, 128, False, 64, 128), (76, 14, 14, 2300, 100, 128, True, 128, 256)])
def test_cut_key_tiles(b, h, hk, m, n, block, causal, d, dv):
    """So many tiles of keys that none is cut by their number alone; those of one key head in every other sequence are seen by
    all queries, the others by few."""
    args = make(b, h, hk, m, n, d, dv)
    g = torch.Generator(device="cuda").manual_seed(3)
    mask = torch.rand((b, h, -(-m // block), 1), generator=g, device="cuda") < 0.03
    mask[::2, h // hk:2 * h // hk] = True
    cols = mask.long().view(b, hk, -1).sum(2).flatten()
    assert cols.numel() > (1024 if d == 64 else 512) * (2 if n <= 64 else 1) and tiles_are_cut(cols, block, 2 if n <= 64 else 4)
    check(args, mask.to(torch.uint8), block, dict(block=block, causal=causal))


@pytest.mark.gpu
def test_replays_follow_the_mask():
    """The cuts are found on the device: a captured call takes the mask that its buffer holds at each replay."""
    b, h, hk, m, n, block = 1, 18, 18, 2112, 2112, 128
    args = make(b, h, hk, m, n, 128, 128)
    dout = torch.randn((b, h, m, 128), device="cuda").to(torch.bfloat16)
    masks = [uneven_mask(b, h, m, n, block), torch.ones((b, h, 17, 17), dtype=torch.uint8, device="cuda")]
    masks += [masks[0].flip(1).contiguous(), torch.zeros_like(masks[0])]
    mask = masks[1].clone()
    shape = W.diff_shape_of(b, h, hk, m, n, 128, 128, block)
    ws = torch.empty(W.diff_attn_workspace_size(shape), dtype=torch.uint8, device="cuda")
    ws_back = torch.empty(W.diff_attn_backward_workspace_size(shape), dtype=torch.uint8, device="cuda")

    def both(**kw):
        o, maps, stats = W.diff_attn(*args, mask, block=block, return_stats=True, workspace=kw.get("ws"))
        return (o, *W.diff_attn_backward(dout, *args, mask, maps, stats, block=block, workspace=kw.get("back")))

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(ws=ws, back=ws_back)
    for x in masks + masks[:1]:
        mask.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        want = both()
        assert all(torch.equal(y, z) for y, z in zip(got, want))
        if not x.any():
            assert not any(y.any() for y in got)
