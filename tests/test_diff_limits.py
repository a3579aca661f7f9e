"""Calls that differential attention refuses on the host, by their whole size, arguments or memory."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

import paper_2609_34814_amd as W                     # noqa: E402
from paper_2609_34814_amd import _lib as L           # noqa: E402
from tests.test_abi import FAKE, _lib                # noqa: E402
from tests.test_diff_attn import _host, _shape       # noqa: E402

INVALID, UNSUP = L.WA_ERR_INVALID_ARG, L.WA_ERR_UNSUPPORTED


def _sizes(**kw):
    """(status of the forward's workspace query, of the gradient's)."""
    lib, n, s = _lib(), ctypes.c_size_t(0), _shape(**kw)
    return tuple(f(ctypes.byref(s), ctypes.byref(n)) for f in (lib.wa_diff_attn_workspace_size, lib.wa_diff_attn_backward_workspace_size))


@pytest.mark.parametrize("kw,want", [
    # 2^25 workgroups of 128 threads (at most 32 queries forward; 64 queries or keys in the gradient), or 2^24 of 256, are 2^32 threads,
    # more than a dimension of a launch holds
    (dict(batch=1 << 20, heads=31, kv_heads=31, q_len=1, kv_len=1), (0, 0)),
    (dict(batch=1 << 20, heads=32, kv_heads=32, q_len=1, kv_len=1), (UNSUP, UNSUP)),
    (dict(batch=1 << 20, heads=15, kv_heads=15, q_len=33, kv_len=33), (0, 0)),
    (dict(batch=1 << 20, heads=16, kv_heads=16, q_len=33, kv_len=33), (UNSUP, 0)),
    (dict(batch=1 << 20, heads=16, kv_heads=16, q_len=1, kv_len=65), (0, UNSUP)),
    (dict(batch=1 << 20, heads=16, kv_heads=1, q_len=1, kv_len=65), (0, 0)),
])
def test_workgroups_fit_a_launch(kw, want):
    assert _sizes(**kw) == want


@pytest.mark.parametrize("scale", [float("nan"), float("inf")])
def test_scales_that_are_no_numbers(scale):
    lib, shape, opts = _lib(), _shape(), L.WaDiffOptions(scale, 0)
    size = 1 << 40
    assert lib.wa_diff_attn(*[FAKE] * 4, None, None, None, ctypes.byref(shape), ctypes.byref(opts), FAKE, None, None, FAKE, size,
                            None) == INVALID
    assert b"softmax_scale" in lib.wa_last_error()
    assert lib.wa_diff_attn_backward(*[FAKE] * 7, None, None, None, ctypes.byref(shape), ctypes.byref(opts), *[FAKE] * 5, size,
                                     None) == INVALID
    assert b"softmax_scale" in lib.wa_last_error()
    opts.softmax_scale = 2e30
    assert lib.wa_diff_attn(*[FAKE] * 4, None, None, None, ctypes.byref(shape), ctypes.byref(opts), FAKE, None, None, FAKE, size,
                            None) == UNSUP


@pytest.mark.parametrize("scale", [0.0, -0.125, 1e-50, float("nan"), float("inf"), 1e39])
def test_scales_of_the_binding(scale):
    """None is the default; another value that the kernels cannot take is not replaced by it."""
    with pytest.raises(ValueError, match="scale"):
        W.diff_attn(**_host(), scale=scale)
    with pytest.raises(ValueError, match="scale"):
        W.diff_attn_backward(torch.zeros(1, 2, 70, 64, dtype=torch.bfloat16), **_host(), mask=None,
                             maps=torch.zeros(1, 4, 70, 64, dtype=torch.int16), stats=torch.zeros(1, 4, 70, 3), scale=scale)


def _span_call(backward, **at):
    """A call whose tensors lie 1 GiB apart, but for those that `at` places."""
    lib, shape = _lib(), _shape(batch=1, heads=2, kv_heads=2, q_len=1, kv_len=8192, head_dim=64, value_dim=64)
    ins = ["dout", "q", "k", "v", "lam", "maps", "stats", "mask", "start", "lens"] if backward else \
        ["q", "k", "v", "lam", "mask", "start", "lens"]
    outs = ["dq", "dk", "dv", "dlam", "ws"] if backward else ["o", "maps", "stats", "ws"]
    a = {x: (i + 1) << 30 for i, x in enumerate(ins + outs)}
    for x, (other, bytes_on) in at.items():
        a[x] = a[other] + bytes_on
    opts, p = L.WaDiffOptions(0.0, 1), [ctypes.c_void_p(a[x]) for x in ins + outs]
    call = lib.wa_diff_attn_backward if backward else lib.wa_diff_attn
    return call(*p[:len(ins)], ctypes.byref(shape), ctypes.byref(opts), *p[len(ins):], 1 << 28, None)


@pytest.mark.parametrize("backward,at,says", [
    # 2 x 8192 values of 64 columns are 2 MiB, keys twice that
    (False, dict(o=("v", 0)), "o overlaps v"), (False, dict(o=("k", (4 << 20) - 256)), "o overlaps k"),
    (False, dict(maps=("o", 16)), "o overlaps maps"), (False, dict(stats=("lens", 0)), "stats overlaps kv_lens"),
    (False, dict(ws=("q", 256)), "workspace overlaps q"), (False, dict(v=("ws", 512)), "workspace overlaps v"),
    (True, dict(dq=("q", 0)), "dq overlaps q"), (True, dict(dv=("v", 0)), "dv overlaps v"), (True, dict(dk=("dv", 16)), "dk overlaps dv"),
    (True, dict(dlam=("lam", 4)), "dlam overlaps lam"), (True, dict(ws=("maps", 256)), "workspace overlaps maps"),
])
def test_overlapping_memory(backward, at, says):
    assert _span_call(backward, **at) == INVALID
    assert _lib().wa_last_error().decode() == says
