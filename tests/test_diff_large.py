"""Differential attention with scores of hundreds, where few keys share a row, in both directions; and one map alone."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2609_34814_amd as W                                            # noqa: E402
from tests.test_diff_attn import DIMS, block_mask, make, reference          # noqa: E402

pytestmark = pytest.mark.gpu


def exponent_error(args):
    """Most that the float32 exponents of two keys of a row differ from exact, in natural units: products of bf16 are exact, the d sums
    of a score and its product with the scale round by 2^-24 of at most scale sum |q k|, and so do the reference that is taken off (the
    running maximum, or the log-sum-exp) and its own start value: d + 8 roundings each."""
    q, k = args[0].double(), args[1].double()
    h, hk, d = q.shape[1] // 2, k.shape[1] // 2, q.shape[3]
    most = 0.0
    for x in range(2 * h):
        y = 2 * (x // 2 // (h // hk)) + x % 2
        most = max(most, (q[:, x].abs() @ k[:, y].abs().transpose(-1, -2).contiguous()).max().item() / d ** 0.5)
    return 2 * (d + 8) * 2.0 ** -24 * most


@pytest.mark.parametrize("d,dv", DIMS)
@pytest.mark.parametrize("b,h,hk,m,n,masked,gain", [(1, 2, 1, 1, 700, False, 100.0), (1, 2, 2, 200, 333, False, 100.0),
                                                    (2, 2, 1, 130, 130, True, 100.0), (1, 4, 2, 65, 300, True, 30.0)])
@pytest.mark.parametrize("causal", [False, True])
def test_scores_of_hundreds(b, h, hk, m, n, masked, gain, causal, d, dv):
    args = make(b, h, hk, m, n, d, dv, gain=gain)
    mask = block_mask(b, h, m, n, 64, 0.6) if masked else None
    off = exponent_error(args)      # 0.002 to 0.01
    kw = dict(block=64, causal=causal)
    o, maps, stats = W.diff_attn(*args, mask, return_stats=True, **kw)
    dout = torch.randn(o.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).to(torch.bfloat16)
    got = W.diff_attn_backward(dout, *args, mask, maps, stats, **kw)
    ref = reference(args, mask, 64, dict(causal=causal), dout)
    assert off < 0.02 and np.abs(ref["lse"][np.isfinite(ref["lse"])]).max() > 3 * gain
    # float32 holds no probability below 2^-126: each such one is taken as 0, and 2^10 keys (queries of all heads) at most add up to it
    # times dP, scale and q or k, which are below 2^20 together here
    tiny = 2.0 ** (-126 + 10 + 20)
    # probabilities: rounded once (2^-8), and off by the exponents of the numerator and of the sum
    arith = (2.0 ** -8 + 2 * off) * (1 + 2.0 ** -6)
    err = np.abs(o.double().cpu().numpy() - ref["o"])
    tol = arith * ref["bound"]["o"] + 2.0 ** -8 * np.abs(ref["o"]) + tiny
    assert np.all(err <= tol), float((err - tol).max())
    lse = stats[..., 0].double().cpu().numpy()
    assert np.array_equal(np.isneginf(lse), np.isneginf(ref["lse"]))
    some = np.isfinite(ref["lse"])
    assert np.all(np.abs(lse[some] - ref["lse"][some]) <= off)
    # the gradient's: P and dS rounded once each and off by their own exponents, and by those of the forward's that D is taken from
    for name, y in zip(("dq", "dk", "dv", "dlam"), got):
        steps = {"dv": 1, "dlam": 0}.get(name, 2)
        err = np.abs(y.double().cpu().numpy() - ref[name])
        tol = (steps * 2.0 ** -8 + 2.0 ** -10 + 4 * off) * (1 + 2.0 ** -6) * ref["bound"][name]
        tol += (2.0 ** -24 if name == "dlam" else 2.0 ** -8) * np.abs(ref[name]) + tiny
        assert np.all(err <= tol), (name, float((err - tol).max()), float(err.max()))


@pytest.mark.parametrize("d", [64, 128])
def test_first_map_alone(d):
    """lam 0 leaves the first map, which sparse_attn computes too: each within its own roundings, probabilities once (2^-8, and 2^-11
    of float32 scores) and the result once."""
    q, k, v, lam = make(1, 2, 2, 512, 512, d, d)
    lam.zero_()
    mask = block_mask(1, 2, 512, 512, 128, 0.6)
    ref = reference((q, k, v, lam), mask, 128, {})
    tol = (2.0 ** -8 + 2.0 ** -11) * (1 + 2.0 ** -8) * ref["bound"]["o"] + 2.0 ** -8 * np.abs(ref["o"])
    first = W.sparse_attn(q[:, ::2].contiguous(), k[:, ::2].contiguous(), v, mask, block=128)
    for o in (W.diff_attn(q, k, v, lam, mask), first):
        err = np.abs(o.double().cpu().numpy() - ref["o"])
        assert np.all(err <= tol), float((err - tol).max())
