"""The gradient of differential attention: refusals on the CPU, the kernels against the fp64 oracle on the GPU."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2609_34814_amd as W                                     # noqa: E402
from paper_2609_34814_amd import _lib as L                           # noqa: E402
from tests.test_abi import FAKE, _lib                                # noqa: E402
from tests.test_diff_attn import (DIMS, INVALID, ALIGN, WORK, UNSUP, _host, _shape, block_mask, check_forward,  # noqa: E402
                                  make, reference)


def test_argument_refusals():
    lib = _lib()
    n, shape = ctypes.c_size_t(0), _shape()
    assert lib.wa_diff_attn_backward_workspace_size(ctypes.byref(shape), ctypes.byref(n)) == 0
    assert n.value >= 4 * 2 * 2 * 4 * 300
    assert lib.wa_diff_attn_backward_workspace_size(ctypes.byref(shape), None) == INVALID
    assert lib.wa_diff_attn_backward_workspace_size(None, ctypes.byref(n)) == INVALID
    odd, opts = ctypes.c_void_p((1 << 20) + 2), L.WaDiffOptions(0.0, 1)
    names = ["dout", "q", "k", "v", "lam", "maps", "stats", "mask", "start", "lens", "dq", "dk", "dv", "dlam"]

    def call(shape=shape, opts=opts, ws=FAKE, size=n.value, **kw):
        a = dict.fromkeys(names, FAKE)
        a.update(kw)
        a = [a[x] for x in names]
        return lib.wa_diff_attn_backward(*a[:10], ctypes.byref(shape), ctypes.byref(opts) if opts else None, *a[10:], ws,
                                         size, None)

    for name in names:
        if name not in ("mask", "start", "lens"):
            assert call(**{name: None}) == INVALID, name
        if name != "mask":
            assert call(**{name: odd}) == ALIGN, name
    assert call(opts=None) == INVALID and call(opts=L.WaDiffOptions(0.0, 0)) == INVALID     # start without causal
    assert call(ws=None) == INVALID and call(size=n.value - 1) == WORK
    assert call(ws=ctypes.c_void_p((1 << 20) + 64)) == ALIGN
    assert call(shape=_shape(head_dim=80)) == UNSUP


@pytest.mark.parametrize("kw", [dict(dout=torch.zeros(1, 2, 70, 64)), dict(maps=torch.zeros(1, 4, 70, 32, dtype=torch.int16)),
                                dict(maps=torch.zeros(1, 4, 70, 64)), dict(stats=torch.zeros(1, 4, 70)), dict()])
def test_binding_refusals(kw):
    args = dict(_host(), mask=None, dout=torch.zeros(1, 2, 70, 64, dtype=torch.bfloat16),
                maps=torch.zeros(1, 4, 70, 64, dtype=torch.int16), stats=torch.zeros(1, 4, 70, 3))
    args.update(kw)
    with pytest.raises(ValueError):
        W.diff_attn_backward(**args)


# ---- GPU ---------------------------------------------------------------------------------------------------

def check_gradient(args, mask=None, block=128, seed=50, **kw):
    """Roundings to bf16, each at most 2^-8 of what it rounds: P (dV) or dS (dQ, dK) once before the product, the result
    once. dO . O_m is off by what the forward's probabilities were rounded, 2^-8 of P (|dO| |V|), the bound's mean, and by
    2^-16 of the row's largest, which P dominates. float32 arithmetic adds 2^-10 (scores: 2^-11 of P, see the forward's
    check, and the log-sum-exp as much). dlam: sums of P_2 dP within 2^-10 as before."""
    dout = torch.randn((args[0].shape[0], args[0].shape[1] // 2, args[0].shape[2], args[2].shape[3]), device="cuda",
                       generator=torch.Generator(device="cuda").manual_seed(seed)).to(torch.bfloat16)
    _, maps, stats = W.diff_attn(*args, mask, block=block, return_stats=True, **kw)
    got = W.diff_attn_backward(dout, *args, mask, maps, stats, block=block, **kw)
    again = W.diff_attn_backward(dout, *args, mask, maps, stats, block=block, **kw)
    assert all(torch.equal(x, y) for x, y in zip(got, again))
    ref = reference(args, mask, block, kw, dout)
    for name, y in zip(("dq", "dk", "dv", "dlam"), got):
        steps = {"dv": 1, "dlam": 0}.get(name, 2)
        err = np.abs(y.double().cpu().numpy() - ref[name])
        tol = (steps * 2.0 ** -8 + 2.0 ** -10) * (1 + 2.0 ** -7) * ref["bound"][name]
        tol += (2.0 ** -24 if name == "dlam" else 2.0 ** -8) * np.abs(ref[name])
        assert np.all(err <= tol), (name, float((err - tol).max()), float(err.max()))
        # the worst case above is far off what independent roundings do: in the 2-norm, 2^-8 of each of three
        if np.linalg.norm(ref[name]) > 0 and name != "dlam":
            assert np.linalg.norm(err) <= 2.0 ** -6 * np.linalg.norm(ref[name]), name
    return got


@pytest.mark.gpu
@pytest.mark.parametrize("d,dv", DIMS)
@pytest.mark.parametrize("b,h,hk,m,n", [(1, 1, 1, 2, 3), (1, 2, 1, 200, 200), (1, 3, 3, 33, 500), (2, 2, 1, 65, 31),
                                        (2, 4, 2, 130, 257)])
@pytest.mark.parametrize("causal", [False, True])
def test_dense(b, h, hk, m, n, d, dv, causal):
    check_gradient(make(b, h, hk, m, n, d, dv), causal=causal)


@pytest.mark.gpu
@pytest.mark.parametrize("d,dv", DIMS)
@pytest.mark.parametrize("block", [64, 128])
@pytest.mark.parametrize("b,h,hk,m,n,causal", [(1, 2, 2, 300, 300, False), (2, 2, 1, 321, 321, True), (1, 2, 1, 20, 900, False),
                                               (1, 1, 1, 4300, 100, False)])
def test_block_masks(b, h, hk, m, n, d, dv, block, causal):
    """The last shape's columns are longer than one word of 64 blocks (of 64)."""
    args = make(b, h, hk, m, n, d, dv)
    check_gradient(args, block_mask(b, h, m, n, block, 0.4), block, causal=causal)


@pytest.mark.gpu
@pytest.mark.parametrize("b,h,hk,block", [(4, 8, 8, 64), (8, 10, 10, 128), (6, 16, 8, 64)])
def test_masked_tiles_in_order_of_length(b, h, hk, block):
    """More than 256 tiles of queries and of keys run longest first."""
    m = 5 * block - 9 if block == 128 else 9 * block
    check_gradient(make(b, h, hk, m, m, 64, 64), block_mask(b, h, m, m, block, 0.4), block)


@pytest.mark.gpu
@pytest.mark.parametrize("d,dv", DIMS)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("h,hk,m,n", [(1, 1, 1100, 1100), (4, 1, 70, 1500), (3, 1, 1300, 60)])
def test_tiles_in_parts(d, dv, causal, h, hk, m, n):
    """Few tiles, so that each is computed in parts; of grouped heads they begin and end inside a head's queries."""
    check_gradient(make(1, h, hk, m, n, d, dv), causal=causal)


@pytest.mark.gpu
@pytest.mark.parametrize("h,m", [(86, 300), (101, 300), (128, 470), (129, 470)])
def test_causal_tiles_that_run_at_once(h, m):
    """257 to 512 tiles, of which the second ones of a compute unit run in the other order, and more."""
    check_gradient(make(1, h, h, m, m, 64, 64), causal=True)
    check_forward(make(1, h, h, m, m, 64, 64), causal=True)


@pytest.mark.gpu
@pytest.mark.parametrize("d,dv", DIMS)
def test_one_key_or_none(d, dv):
    """One key takes all: dS is 0 but for roundings, and dV is (1 - lam) dO; a mask that keeps nothing gives zeros."""
    args = make(1, 2, 2, 1, 1, d, dv)
    o, maps, stats = W.diff_attn(*args, return_stats=True)
    dout = torch.randn(o.shape, device="cuda").to(torch.bfloat16)
    dq, dk, dval, _ = W.diff_attn_backward(dout, *args, None, maps, stats)
    # |dP - D| <= 2^-12 sum |dO| |V| <= 2^-12 * 2000 (a value off by 2^-16 of the row's largest, and float32 sums)
    assert dq.float().abs().max() <= 0.5 and dk.float().abs().max() <= 0.5
    want = ((1 - args[3]) * 1.0)[None, :, None, None] * dout.float()
    assert ((dval.float() - want).abs() <= (2.0 ** -7 + 2.0 ** -12) * (1 + args[3].abs())[None, :, None, None] * dout.float().abs()).all()
    args = make(2, 2, 1, 200, 300, d, dv)
    none = torch.zeros((2, 2, 2, 3), dtype=torch.uint8, device="cuda")
    o, maps, stats = W.diff_attn(*args, none, return_stats=True)
    dout = torch.randn(o.shape, device="cuda").to(torch.bfloat16)
    assert all(not x.any() for x in W.diff_attn_backward(dout, *args, none, maps, stats))


@pytest.mark.gpu
@pytest.mark.parametrize("d,dv", DIMS)
@pytest.mark.parametrize("m,hk", [(70, 4), (260, 1)])
def test_ragged_batches(d, dv, m, hk):
    n, lens = 300, [0, 1, 63, 64, 65, 299, 300]
    args = make(len(lens), 4, hk, m, n, d, dv)
    for b, x in enumerate(lens):
        args[1][b, :, x:] = float("nan")
        args[2][b, :, x:] = float("nan")
    kv = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for kw in (dict(kv_lens=kv), dict(kv_lens=kv, causal=True, q_start=kv - m)):
        _, dk, dval, _ = check_gradient(args, **kw)
        for b, x in enumerate(lens):
            assert not dk[b, :, x:].any() and not dval[b, :, x:].any()


@pytest.mark.gpu
@pytest.mark.parametrize("m,n", [(40, 300), (300, 300), (130, 40)])
def test_query_positions(m, n):
    start = torch.tensor([-m, -7, 0, n // 2, n], dtype=torch.int32, device="cuda")
    check_gradient(make(5, 2, 1, m, n, 64, 128), causal=True, q_start=start)


@pytest.mark.gpu
def test_scale_and_dropped_blocks():
    args = make(1, 1, 1, 256, 512, 128, 128)
    mask = torch.tensor([[1, 0, 1, 0], [0, 0, 1, 0]], dtype=torch.uint8, device="cuda").view(1, 1, 2, 4)
    for x in (1, 2):
        args[x][:, :, 128:256] = args[x][:, :, 384:] = float("nan")
    check_gradient(args, mask, scale=0.2)


@pytest.mark.gpu
def test_gradient_by_differences():
    """dO . O moves by gradient . step: the forward in float64 (the oracle) at q + e, k + e', ... against the kernel's
    gradients. The kernels' gradients are within 2^-6 of exact in the 2-norm (check_gradient), and the central difference
    of step 2^-10 of the inputs is within 2^-16 of the derivative here."""
    from oracle import diff_attention as D
    args = make(1, 2, 1, 40, 40, 64, 64)
    dout = torch.randn((1, 2, 40, 64), device="cuda").to(torch.bfloat16)
    o, maps, stats = W.diff_attn(*args, causal=True, return_stats=True)
    got = [x.double().cpu().numpy() for x in W.diff_attn_backward(dout, *args, None, maps, stats, causal=True)]
    host, g = [x.double().cpu().numpy() for x in args], dout.double().cpu().numpy()
    rng = np.random.default_rng(8)
    for i in range(4):
        e = rng.standard_normal(host[i].shape)
        e = e / np.linalg.norm(e) + got[i] / np.linalg.norm(got[i])       # along the gradient, so nothing cancels
        moved = []
        for sign in (1, -1):
            x = list(host)
            x[i] = host[i] + sign * 2.0 ** -10 * e
            moved.append((D.forward_backward(*x, causal=True)["o"] * g).sum())
        slope = (moved[0] - moved[1]) / 2.0 ** -9
        assert abs(slope - (got[i] * e).sum()) <= (2.0 ** -6 + 2.0 ** -10) * 2 * np.linalg.norm(got[i])


@pytest.mark.gpu
def test_streams_and_replays():
    """A captured forward and backward, replayed on new inputs between eager calls, with a workspace of its own."""
    args = make(2, 4, 2, 300, 300, 64, 128)
    mask = block_mask(2, 4, 300, 300, 128, 0.6)
    dout = torch.randn((2, 4, 300, 128), device="cuda").to(torch.bfloat16)

    def step():
        o, maps, stats = W.diff_attn(*args, mask, return_stats=True)
        return (o, *W.diff_attn_backward(dout, *args, mask, maps, stats))
    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(other, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in (7, 8, 9):
        for x, y in zip(args, make(2, 4, 2, 300, 300, 64, 128, seed=seed)):
            x.copy_(y)
        for x in held:
            x.zero_()
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, want))
