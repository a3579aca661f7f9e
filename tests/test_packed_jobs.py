"""How the gradient over packed sequences cuts its tiles into jobs: its whole-number arithmetic, compiled for the host, against Python's."""
import random
import shutil
import subprocess

import pytest

from paper_2609_34814_amd import build

PROGRAM = r"""
#include <cstdio>
#define __host__
#define __device__
#include "packed_jobs.h"
int main() {
  long long sum;
  int share, longest;
  while (std::scanf("%lld %d %d", &sum, &share, &longest) == 3) {
    const int most = wa::longest_whole(sum, share, longest);
    std::printf("%d %d %d\n", most, most > 0 ? wa::parts_of(longest, most) : -1, most > 0 ? wa::jobs_upto(longest, most) : -1);
  }
}
"""
KEYS, QUERIES = 4, 3          # of the seven products of a pair


def accepted(tokens, heads, kv_heads):
    """What the call takes, of one sequence."""
    tiles = -(-tokens // 128)
    return tokens < 1 << 26 and tokens * heads < 1 << 31 and tiles * (heads + kv_heads) < (1 << 24) - 2048 \
        and -(-tokens // 16) * heads < 1 << 25


def shapes():
    out = [((1 << 26) - 1, 2, 1), ((1 << 26) - 1, 7, 1), ((1 << 26) - 1, 1, 1), (1, 1, 1), (129, 64, 8), (2 ** 24, 31, 31)]
    rng = random.Random(3)
    while len(out) < 400:
        kv = rng.choice([1, 2, 3, 8, 32])
        x = (int(2 ** rng.uniform(0, 26)), kv * rng.choice([1, 2, 4, 7]), kv)
        if accepted(*x):
            out.append(x)
    return out


@pytest.mark.skipif(shutil.which("g++") is None, reason="no compiler")
def test_jobs_of_one_sequence(tmp_path):
    source, program = tmp_path / "jobs.cpp", tmp_path / "jobs"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", build.CSRC, str(source), "-o", str(program)], check=True, capture_output=True)
    asked = []
    for tokens, heads, kv_heads in shapes():
        assert accepted(tokens, heads, kv_heads)
        t = -(-tokens // 128)
        for causal in (True, False):
            for share, cols in ((KEYS, kv_heads), (QUERIES, heads)):
                asked.append(((t * (t + 1) // 2 if causal else t * t) * cols, share, t, cols, causal))
    run = subprocess.run([str(program)], input="\n".join(f"{s} {a} {t}" for s, a, t, _, _ in asked), capture_output=True, text=True,
                         check=True)
    got = [[int(x) for x in line.split()] for line in run.stdout.splitlines()]
    assert len(got) == len(asked)
    for (total, share, t, cols, causal), (most, parts, jobs) in zip(asked, got):
        want = min(-(-7 * total // (share * 512)), t)
        assert most == want >= 1 and parts == -(-t // most)
        # lengths 1 to t once each, causal; cut tiles and their parts have room in the tables
        q, r = divmod(t, most)
        assert jobs == q * (q + 1) // 2 * most + r * (q + 1) and (t > 5000 or jobs == sum(-(-x // most) for x in range(1, t + 1)))
        cut = max(t - most, 0) if causal else (t if t > most else 0)
        extra = jobs - t if causal else t * (parts - 1)
        assert cut * cols < 512 and (cut + extra) * cols < 1024 and extra * cols <= 512
