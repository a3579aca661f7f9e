"""Keys that no query of a sequence sees, by `causal` and q_start: room of a cache that is not written yet. What lies there does not
matter, and its gradient is 0."""
import pytest

torch = pytest.importorskip("torch")

from tests.test_diff_attn import DIMS, block_mask, check_forward, make      # noqa: E402
from tests.test_diff_attn_grad import check_gradient                        # noqa: E402

pytestmark = pytest.mark.gpu


def _unwritten(h, hk, m, n, d, dv):
    """Sequences of which the last query is at -1 (sees nothing) to n - 1; the keys behind it are not numbers."""
    last = [-1, 0, 30, 63, 64, n - 2, n - 1]
    args = make(len(last), h, hk, m, n, d, dv)
    for b, x in enumerate(last):
        args[1][b, :, x + 1:] = float("nan")
        args[2][b, :, x + 1:] = float("nan")
    return args, torch.tensor([x - m + 1 for x in last], dtype=torch.int32, device="cuda"), last


@pytest.mark.parametrize("d,dv", DIMS)
@pytest.mark.parametrize("m,hk", [(1, 1), (3, 2), (33, 1), (70, 4), (260, 1)])
def test_forward(d, dv, m, hk):
    args, start, _ = _unwritten(4, hk, m, 600, d, dv)
    check_forward(args, causal=True, q_start=start)
    check_forward(args, block_mask(7, 4, m, 600, 64, 0.5), 64, causal=True, q_start=start)


@pytest.mark.parametrize("d,dv", DIMS)
@pytest.mark.parametrize("m,hk", [(3, 2), (70, 4), (260, 1)])
def test_gradient(d, dv, m, hk):
    args, start, last = _unwritten(4, hk, m, 300, d, dv)
    for mask, block in ((None, 128), (block_mask(7, 4, m, 300, 64, 0.5), 64)):
        _, dk, dval, _ = check_gradient(args, mask, block, causal=True, q_start=start)
        for b, x in enumerate(last):
            assert not dk[b, :, x + 1:].any() and not dval[b, :, x + 1:].any()


def test_prompt_without_a_start():
    """More queries than keys: the first see nothing."""
    args = make(1, 2, 1, 130, 40, 64, 128)
    check_forward(args, causal=True)
    check_gradient(args, causal=True)
