"""One layer's path as a model runs it: projections' layout -> rotary -> produced mask -> differential attention ->
its gradient -> the rotary gradient back in the projections' layout, against float64 autograd of the same chain."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def _layer(x, f, pos, lam, dout, axis, block, keep):
    """x: q, k, v as [B][N][heads][d] bf16. (o, mask, dq, dk, dv, dlam), gradients laid out as x."""
    import paper_2609_34814_amd as W
    q, k, v = x
    kw = dict(inv_freq=f, positions=pos, layout="interleaved", axis_pairs=axis)
    qr, kr = W.rotary(q.transpose(1, 2), k.transpose(1, 2), **kw)
    vh = v.transpose(1, 2).contiguous()
    mask = W.produce_block_mask(qr[:, ::2].contiguous(), kr[:, ::2].contiguous(), block=block, keep=keep)
    o, maps, stats = W.diff_attn(qr, kr, vh, lam, mask, block=block, return_stats=True)
    dqr, dkr, dvh, dlam = W.diff_attn_backward(dout, qr, kr, vh, lam, mask, maps, stats, block=block)
    dq, dk = torch.empty_like(q), torch.empty_like(k)
    W.rotary(dqr, dkr, backward=True, out_q=dq.transpose(1, 2), out_k=dk.transpose(1, 2), **kw)
    return o, mask, dq, dk, dvh.transpose(1, 2).contiguous(), dlam


def _exact(x, f, pos, lam, dout, axis, block, mask):
    leaf = [y.double().requires_grad_() for y in (*x, lam)]
    q, k, v, lm = leaf
    which = torch.repeat_interleave(torch.arange(3), torch.tensor(axis)).to(q.device)
    angle = pos.double()[which].permute(1, 2, 0) * f            # [B][N][P]
    turn = torch.polar(torch.ones_like(angle), angle)[:, :, None]

    def rot(y):
        z = torch.view_as_complex(y.unflatten(-1, (-1, 2)).contiguous())
        return torch.view_as_real(z * turn).flatten(-2).transpose(1, 2)
    q, k, v = rot(q), rot(k), v.transpose(1, 2)
    n = torch.arange(q.shape[2], device=q.device) // block
    keep = mask.bool()[:, :, n][:, :, :, n]
    p = []
    for t in range(2):
        s = (q[:, t::2] @ k[:, t::2].transpose(-1, -2).contiguous()) / math.sqrt(q.shape[-1])
        p.append(torch.softmax(s.masked_fill(~keep, -math.inf), -1))
    o = (p[0] - lm[None, :, None, None] * p[1]) @ v
    return (o.detach(), *torch.autograd.grad(o, leaf, dout.double()))


@pytest.mark.parametrize("d,dv,block", [(64, 128, 64), (128, 256, 128)])
def test_layer(d, dv, block):
    from paper_2609_34814_amd import rotary_frequencies
    b, h, grid = 2, 3, (5, 9, 11)
    n = grid[0] * grid[1] * grid[2] - 3
    g = torch.Generator(device="cuda").manual_seed(1)

    def r(*s):
        return torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)
    x = [r(b, n, 2 * h, d), r(b, n, 2 * h, d), r(b, n, h, dv)]
    lam = torch.rand(h, generator=g, device="cuda")
    dout = r(b, h, n, dv)
    third = d // 6
    axis = [d // 2 - 2 * third, third, third]
    f = torch.cat([rotary_frequencies(p)[0] for p in axis])
    t = torch.arange(n, device="cuda")
    pos = torch.stack([t // 99, t // 11 % 9, t % 11]).to(torch.int32)[:, None].expand(3, b, n).contiguous()
    got = _layer(x, f, pos, lam, dout, axis, block, 3)
    mask = got[1]
    ref = _exact(x, f, pos, lam, dout, axis, block, mask)
    # in the 2-norm: the rotated q and k are rounded (2^-8), which moves scores, and so P, by as much; then the
    # gradient's own 2^-6; the rotary gradient rounds once more
    for name, y, z in zip(("o", "dq", "dk", "dv", "dlam"), (got[0], *got[2:]), ref):
        assert (y.double() - z).norm() <= 2.0 ** -5 * z.norm(), name

    # captured while the eager results live, and replayed on other inputs between eager runs
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = _layer(x, f, pos, lam, dout, axis, block, 3)
    for _ in range(3):
        for y in (*x, dout):
            y.copy_(r(*y.shape))
        want = _layer(x, f, pos, lam, dout, axis, block, 3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, z) for y, z in zip(held, want))
