"""Rotary positions of more elements than one dimension of a launch holds threads (a pair a thread): 2^31 threads count in 64 bits, 2^32
need a second dimension."""
import pytest

torch = pytest.importorskip("torch")

import paper_2609_34814_amd as W                     # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("copies", [65, 129])
def test_more_threads_than_32_bits(copies):
    """One head of one pair, 1024 sequences of 32,771 tokens so many times over: every copy is what one is alone, the last too."""
    n = 32771
    assert copies * 1024 * n > 2 ** (31 if copies == 65 else 32)
    f, _ = W.rotary_frequencies(1, base=7.0)
    one = torch.randn((1024, 1, n, 2), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).to(torch.bfloat16)
    want = W.rotary(one, inv_freq=f)
    small = W.rotary(one[:2].contiguous(), inv_freq=f)
    assert torch.equal(want[:2], small)
    q = one.repeat(copies, 1, 1, 1)
    W.rotary(q, inv_freq=f, out_q=q)
    for x in q.split(1024):
        assert torch.equal(x, want)
