"""Rotary positions: frequencies and refusals on the CPU, the kernel against the fp64 oracle on the GPU."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2609_34814_amd as W                     # noqa: E402
from oracle import rotary as R                       # noqa: E402
from paper_2609_34814_amd import _lib as L           # noqa: E402
from tests.test_abi import FAKE, _lib                # noqa: E402

FAR = ctypes.c_void_p(1 << 21)


# ---- CPU ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kw", [dict(), dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0),
                                dict(scaling="yarn", factor=16.0, original_len=8192.0),
                                dict(scaling="yarn", factor=1.0), dict(base=5e5, scaling="yarn", factor=2.5,
                                                                       beta_fast=20.0, beta_slow=0.0)])
@pytest.mark.parametrize("pairs", [1, 2, 11, 64])
def test_frequencies(pairs, kw):
    _lib()
    if kw.get("scaling") == "ntk" and pairs == 1:
        with pytest.raises(W.WaError):
            W.rotary_frequencies(pairs, device="cpu", **kw)
        return
    f, s = W.rotary_frequencies(pairs, device="cpu", **kw)
    ref, ref_s = R.frequencies(pairs, **kw)
    # a handful of fp64 operations: 2^-53 each; log(base) in the oracle's exponent costs |exponent| <= 14 more
    np.testing.assert_allclose(f.numpy(), ref, rtol=64 * 2.0 ** -53, atol=0)
    assert abs(s - ref_s) <= 4 * 2.0 ** -53 * ref_s


def test_ntk_divides_the_last_frequency_by_the_factor():
    _lib()
    plain, _ = W.rotary_frequencies(64, device="cpu")
    ntk, _ = W.rotary_frequencies(64, scaling="ntk", factor=8.0, device="cpu")
    assert ntk[0] == plain[0] == 1.0
    assert abs(ntk[-1] / plain[-1] - 1 / 8) <= 1e-13


@pytest.mark.parametrize("kw", [dict(scaling="other"), dict(scaling="linear", factor=0.5), dict(base=0.0),
                                dict(scaling="yarn", factor=2.0, original_len=0.0),
                                dict(scaling="yarn", factor=2.0, beta_fast=1.0, beta_slow=1.0),
                                dict(scaling="linear", factor=float("nan"))])
def test_frequency_refusals(kw):
    _lib()
    with pytest.raises((ValueError, W.WaError)):
        W.rotary_frequencies(8, device="cpu", **kw)


def _params(**kw):
    d = dict(batch=2, tokens=100, head_dim=64, dtype=L.WA_BF16, layout=L.WA_ROTARY_HALF, pairs=32, axes=1,
             axis_pairs=(32, 0, 0), position_batch=1, backward=0, scale=1.0)
    d.update(kw)
    d["axis_pairs"] = (ctypes.c_int32 * 3)(*d["axis_pairs"])
    return L.WaRotaryParams(*[d[n] for n, _ in L.WaRotaryParams._fields_])


def _tensor(**kw):
    d = dict(inp=FAKE, out=FAR, heads=4, in_stride=(25600, 6400, 64), out_stride=(25600, 6400, 64))
    d.update(kw)
    t = L.WaRotaryTensor()
    t.inp, t.out, t.heads = d["inp"], d["out"], d["heads"]
    t.in_stride[:], t.out_stride[:] = d["in_stride"], d["out_stride"]
    return t


def test_packed_structures_are_the_declared_ones():
    p, t = _params(scale=2.5, axes=2, axis_pairs=(20, 12, 0)), _tensor()
    assert bytes(p) == L.ROTARY_PARAMS.pack(2, 100, 64, L.WA_BF16, L.WA_ROTARY_HALF, 32, 2, 20, 12, 0, 1, 0, 2.5)
    assert bytes(t) == L.ROTARY_TENSOR.pack(1 << 20, 1 << 21, 4, 25600, 6400, 64, 25600, 6400, 64)


INVALID, ALIGN, UNSUP = L.WA_ERR_INVALID_ARG, L.WA_ERR_ALIGNMENT, L.WA_ERR_UNSUPPORTED


@pytest.mark.parametrize("params,tensor,code", [
    (dict(batch=0), {}, INVALID), (dict(tokens=0), {}, INVALID), (dict(dtype=3), {}, INVALID),
    (dict(layout=2), {}, INVALID), (dict(pairs=33, axis_pairs=(33, 0, 0)), {}, INVALID),
    (dict(pairs=0, axis_pairs=(0, 0, 0)), {}, INVALID), (dict(axes=0), {}, INVALID), (dict(axes=4), {}, INVALID),
    (dict(axes=2, axis_pairs=(33, -1, 0)), {}, INVALID), (dict(axis_pairs=(31, 0, 0)), {}, INVALID),
    (dict(scale=float("inf")), {}, INVALID), (dict(scale=1e300), {}, INVALID),
    (dict(head_dim=65538), {}, UNSUP), (dict(batch=1 << 20, tokens=1 << 20), {}, None),
    ({}, dict(inp=None), INVALID), ({}, dict(out=None), INVALID), ({}, dict(heads=0), INVALID),
    ({}, dict(inp=ctypes.c_void_p((1 << 20) + 1)), ALIGN), ({}, dict(in_stride=(25600, -64, 64)), INVALID),
    ({}, dict(out_stride=(25600, 0, 64)), INVALID), ({}, dict(out_stride=(25600, 6400, 63)), INVALID),
    ({}, dict(out_stride=(6400, 6400, 64)), INVALID), ({}, dict(in_stride=(1 << 41, 6400, 64)), UNSUP),
    ({}, dict(out=FAKE, in_stride=(25600, 64, 256)), INVALID),
])
def test_refusals(params, tensor, code):
    lib = _lib()
    t = (L.WaRotaryTensor * 2)(_tensor(**tensor))
    got = lib.wa_rotary(ctypes.byref(_params(**params)), t, 1, FAKE, None, None)
    assert got == code if code is not None else got in (INVALID, UNSUP)
    assert lib.wa_last_error()


def test_refusals_of_pointers_and_counts():
    lib = _lib()
    p, t = _params(), (L.WaRotaryTensor * 2)(_tensor(), _tensor())
    assert lib.wa_rotary(None, t, 1, FAKE, None, None) == INVALID
    assert lib.wa_rotary(ctypes.byref(p), None, 1, FAKE, None, None) == INVALID
    assert lib.wa_rotary(ctypes.byref(p), t, 1, None, None, None) == INVALID
    assert lib.wa_rotary(ctypes.byref(p), t, 0, FAKE, None, None) == INVALID
    assert lib.wa_rotary(ctypes.byref(p), t, 3, FAKE, None, None) == INVALID
    assert lib.wa_rotary(ctypes.byref(p), t, 2, FAKE, None, None) == INVALID        # one output for both
    assert lib.wa_rotary(ctypes.byref(p), t, 1, ctypes.c_void_p((1 << 20) + 4), None, None) == ALIGN
    assert lib.wa_rotary(ctypes.byref(p), t, 1, FAKE, ctypes.c_void_p((1 << 20) + 2), None) == ALIGN
    three = _params(axes=3, axis_pairs=(12, 10, 10))
    assert lib.wa_rotary(ctypes.byref(three), t, 1, FAKE, None, None) == INVALID    # no positions
    some = _params(position_batch=3)
    assert lib.wa_rotary(ctypes.byref(some), t, 1, FAKE, FAKE, None) == INVALID


@pytest.mark.parametrize("kw,says", [
    (dict(inv_freq=torch.ones(8)), "inv_freq"), (dict(layout="other"), "layout"),
    (dict(q=torch.zeros(2, 3, 5, 16, dtype=torch.float64)), "q must be"), (dict(k=torch.zeros(2, 3, 6, 16)), "k must be"),
    (dict(k=torch.zeros(2, 3, 5, 16, dtype=torch.bfloat16)), "k must be"), (dict(k=torch.zeros(3, 5, 16)), "k must be"),
    (dict(positions=torch.zeros(5)), "positions"), (dict(positions=torch.zeros(3, 5, dtype=torch.int32)), "positions"),
    (dict(positions=torch.zeros(2, 5, dtype=torch.int32), axis_pairs=[4, 4]), "positions"),
    (dict(positions=torch.zeros(2, 3, 5, dtype=torch.int32), axis_pairs=[4, 4]), "positions"),
    (dict(axis_pairs=[2, 2, 2, 2]), "axis_pairs"), (dict(out_q=torch.zeros(2, 3, 5, 8)), "out_q"),
    (dict(out_k=torch.zeros(2, 3, 5, 16)), "out_k without k"),
    (dict(q=torch.zeros(2, 3, 16, 5).transpose(2, 3)), "contiguous rows"), (dict(), "device tensor"),
])
def test_binding_refusals(kw, says):
    args = dict(q=torch.zeros(2, 3, 5, 16), inv_freq=torch.ones(8, dtype=torch.float64))
    args.update(kw)
    with pytest.raises(ValueError, match=says):
        W.rotary(args.pop("q"), args.pop("k", None), **args)


def test_oracle_turns_by_relative_positions():
    """The product of a rotated query and a rotated key depends on the distance of their positions only."""
    rng = np.random.default_rng(3)
    f, _ = R.frequencies(8)
    q, k = rng.standard_normal((2, 1, 1, 1, 16))
    dots = []
    for a, b in ((5, 2), (105, 102)):
        dots.append((R.rotate(q, f, np.array([[[a]]])) * R.rotate(k, f, np.array([[[b]]]))).sum())
    assert abs(dots[0] - dots[1]) < 1e-12


# ---- GPU ---------------------------------------------------------------------------------------------------

def _tolerance(x, scale, dtype, out, pairs, layout):
    """Rounding of the result, half a step, plus the float32 arithmetic: the rest of the angle is at most half a turn,
    rounded to 2^-24 of it (2 pi 2^-25 < 2^-22 radians; positions below 2^21 add less than 2^-30 in float64), its sine within
    2^-22, scale, two products and a sum 2^-24 each: below 2^-20.5 of |x| + |y| in all."""
    lo = np.abs(x[..., 0:2 * pairs:2] if layout == "interleaved" else x[..., :pairs])
    hi = np.abs(x[..., 1:2 * pairs:2] if layout == "interleaved" else x[..., pairs:2 * pairs])
    both = (lo + hi) * abs(scale)
    tol = np.zeros_like(x)
    if layout == "interleaved":
        tol[..., 0:2 * pairs:2] = tol[..., 1:2 * pairs:2] = both
    else:
        tol[..., :pairs] = tol[..., pairs:2 * pairs] = both
    arith = tol * 2.0 ** -20.5
    half_step = torch.finfo(dtype).eps / 2
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0     # half of float16's smallest number
    return arith + half_step * (np.abs(out) + arith) + tiny


def _check(y, x, f, pos, layout, axis, scale, backward):
    ref = R.rotate(x.double().cpu().numpy(), f.cpu().numpy(), None if pos is None else pos.cpu().numpy(), layout, axis,
                   scale, backward)
    err = np.abs(y.double().cpu().numpy() - ref)
    tol = _tolerance(x.double().cpu().numpy(), scale, x.dtype, ref, len(f), layout)
    assert np.all(err <= tol), float((err - tol).max())
    assert torch.equal(y[..., 2 * len(f):], x[..., 2 * len(f):])


def _randn(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("b,hq,hk,n,d,pairs", [
    (1, 1, 1, 1, 2, 1), (8, 32, 8, 1, 128, 64), (2, 3, 3, 257, 64, 16), (1, 5, 2, 33, 96, 11), (3, 2, 1, 70, 130, 65),
    (2, 19, 4, 61, 72, 32), (1, 40, 40, 1000, 128, 64), (1, 3, 1, 20, 65, 32), (1, 4, 2, 50, 40, 16)])
def test_matches_oracle(b, hq, hk, n, d, pairs, dtype, layout):
    q, k = _randn((b, hq, n, d), dtype, 1), _randn((b, hk, n, d), dtype, 2)
    f, s = W.rotary_frequencies(pairs, scaling="yarn", factor=4.0)
    pos = torch.randint(-5000, 2 ** 20, (1, b, n), dtype=torch.int32, device="cuda")
    for backward in (False, True):
        yq, yk = W.rotary(q, k, inv_freq=f, positions=pos, layout=layout, scale=s, backward=backward)
        _check(yq, q, f, pos, layout, None, s, backward)
        _check(yk, k, f, pos, layout, None, s, backward)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", ["none", "n", "bn", "1bn", "11n"])
def test_position_shapes(shape):
    q = _randn((3, 2, 40, 32), torch.float32, 4)
    f, _ = W.rotary_frequencies(16)
    full = torch.randint(0, 5000, (1, 3, 40), dtype=torch.int32, device="cuda")
    one = full[:, :1].contiguous()
    pos, ref = {"none": (None, None), "n": (one[0, 0], one.expand(1, 3, 40)), "bn": (full[0], full), "1bn": (full, full),
                "11n": (one, one.expand(1, 3, 40))}[shape]
    _check(W.rotary(q, inv_freq=f, positions=pos), q, f, ref, "half", None, 1.0, False)


@pytest.mark.gpu
@pytest.mark.parametrize("axis", [[22, 21, 21], [3, 60, 1], [64, 0], [0, 32, 32]])
def test_axes(axis):
    pairs = sum(axis)
    q = _randn((2, 3, 77, 2 * pairs), torch.bfloat16, 5)
    f = torch.cat([W.rotary_frequencies(max(p, 1))[0][:p] for p in axis])
    pos = torch.randint(0, 100, (len(axis), 2, 77), dtype=torch.int32, device="cuda")
    y = W.rotary(q, inv_freq=f, positions=pos, layout="interleaved", axis_pairs=axis)
    _check(y, q, f, pos, "interleaved", axis, 1.0, False)


@pytest.mark.gpu
def test_far_positions():
    """Near the largest position, 3.4e8 turns: the float64 product keeps 2^-53 of them, 2^-24.6 turns; the oracle too."""
    q = _randn((1, 1, 4, 64), torch.float32, 6)
    f, _ = W.rotary_frequencies(32)
    pos = torch.tensor([2 ** 31 - 1, 2 ** 31 - 2, -2 ** 31, 12345678], dtype=torch.int32, device="cuda").view(1, 1, 4)
    y = W.rotary(q, inv_freq=f, positions=pos)
    ref = R.rotate(q.double().cpu().numpy(), f.cpu().numpy(), pos.cpu().numpy())
    assert np.abs(y.double().cpu().numpy() - ref).max() <= 2 * 5 * (2.0 ** -20.5 + 2 * 2 * np.pi * 2.0 ** -24.6)


@pytest.mark.gpu
@pytest.mark.parametrize("d,pairs", [(64, 32), (64, 12), (33, 16)])
def test_strides_and_in_place(d, pairs):
    """Parts of a fused projection in, any layout out, bytes between the rows left alone."""
    b, n, h = 2, 50, 3
    f, _ = W.rotary_frequencies(pairs)
    fused = _randn((b, n, 3 * h * d), torch.bfloat16, 7)
    q, k = (fused[..., i * h * d:(i + 1) * h * d].unflatten(-1, (h, d)).transpose(1, 2) for i in range(2))
    want = W.rotary(q.contiguous(), k.contiguous(), inv_freq=f)
    got = W.rotary(q, k, inv_freq=f)
    assert all(torch.equal(a, c) and a.is_contiguous() for a, c in zip(got, want))
    wide = torch.full((b, n, h, d + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    out = wide[..., :d].transpose(1, 2)
    assert W.rotary(q, inv_freq=f, out_q=out) is out
    assert torch.equal(out, want[0]) and torch.all(wide[..., d:] == 7.0)
    v = fused[..., 2 * h * d:].clone()
    W.rotary(q, k, inv_freq=f, out_q=q, out_k=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(fused[..., 2 * h * d:], v)
    # an input repeated over the heads
    one = _randn((b, 1, n, d), torch.bfloat16, 8)
    assert torch.equal(W.rotary(one.expand(b, h, n, d), inv_freq=f), W.rotary(one.expand(b, h, n, d).contiguous(), inv_freq=f))


@pytest.mark.gpu
def test_unaligned_rows():
    f, _ = W.rotary_frequencies(32)
    flat = _randn((1 + 2 * 30 * 64,), torch.bfloat16, 9)
    q = flat[1:].view(1, 2, 30, 64)
    assert torch.equal(W.rotary(q, inv_freq=f), W.rotary(q.clone(), inv_freq=f))


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """2.2e9 elements: the last tokens of the last head are what they are alone."""
    f, _ = W.rotary_frequencies(64)
    q = torch.randn((1, 40, 430000, 128), device="cuda", dtype=torch.bfloat16)
    assert q.numel() > 2 ** 31
    tail = q[:, -1:, -50:].contiguous()
    pos = torch.arange(430000, dtype=torch.int32, device="cuda")
    want = W.rotary(tail, inv_freq=f, positions=pos[-50:].contiguous())
    W.rotary(q, inv_freq=f, positions=pos, out_q=q)
    assert torch.equal(q[:, -1:, -50:], want)


@pytest.mark.gpu
def test_gradient_is_the_transposed_map():
    """For a linear map the difference quotient is exact: <g, R(x + e) - R(x)> = <R^T g, e> up to float32 roundings
    (2^-20.5 of at most 2 |x| |g| a product, over 2 x 3 x 40 x 32 of them)."""
    f, _ = W.rotary_frequencies(12)
    x, e, g = (_randn((2, 3, 40, 32), torch.float32, s) for s in (10, 11, 12))
    pos = torch.randint(0, 9000, (2, 40), dtype=torch.int32, device="cuda")
    kw = dict(inv_freq=f, positions=pos, layout="interleaved", scale=1.25)
    left = (g.double() * (W.rotary(x + e, **kw).double() - W.rotary(x, **kw).double())).sum()
    right = (W.rotary(g, backward=True, **kw).double() * e.double()).sum()
    bound = 2.0 ** -20.5 * 1.25 * 2 * (g.abs() * (x.abs() + (x + e).abs() + e.abs())).double().sum() * 2
    assert abs(left - right) <= bound


@pytest.mark.gpu
def test_two_streams_and_replays():
    f, s = W.rotary_frequencies(32, scaling="linear", factor=2.0)
    q, k = _randn((2, 4, 600, 64), torch.bfloat16, 13), _randn((2, 2, 600, 64), torch.bfloat16, 14)
    want = W.rotary(q, k, inv_freq=f, scale=s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = W.rotary(q, k, inv_freq=f, scale=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(other, want))
    oq, ok = torch.empty_like(q), torch.empty_like(k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        W.rotary(q, k, inv_freq=f, scale=s, out_q=oq, out_k=ok)
    for seed in range(3):
        q.copy_(_randn(q.shape, q.dtype, 20 + seed))
        oq.zero_()
        want = W.rotary(q, k, inv_freq=f, scale=s)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(oq, want[0]) and torch.equal(ok, want[1])
