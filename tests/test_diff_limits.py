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
