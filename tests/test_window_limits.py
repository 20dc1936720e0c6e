"""The last token that a query row sees, on the CPU: csrc/mla_kernels.h compiled here
with g++ (which stops at a signed sum that wraps) against Python's integers, up to
the longest sequences and prefixes that tables hold."""
import os
import random
import subprocess

import pytest

from paper_2606_01502_amd import build as B

_MAIN = r"""
#include "mla_kernels.h"
#include <cstdio>
int main() {
  int pos0, i, n_tok;
  while (std::scanf("%d %d %d", &pos0, &i, &n_tok) == 3) std::printf("%d\n", mla::last_token(pos0, i, n_tok));
}
"""
MOST = 64 * (2 ** 25 - 1)  # tokens of the widest table


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    tmp = str(tmp_path_factory.mktemp("last"))
    src, out = os.path.join(tmp, "last.cc"), os.path.join(tmp, "last")
    with open(src, "w") as f:
        f.write(_MAIN)
    rocm = os.path.dirname(os.path.dirname(B.HIPCC))
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=signed-integer-overflow", "-fno-sanitize-recover=all",
                    "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"), "-I", B.CSRC, "-o", out, src],
                   check=True)
    return out


def answers(exe, calls):
    out = subprocess.run([exe], input="".join("%d %d %d\n" % c for c in calls), capture_output=True, text=True)
    assert out.returncode == 0, out.stderr[-500:]
    return [int(v) for v in out.stdout.split()]


def test_rows_of_a_group_behind_the_longest_prefixes(exe):
    """A prefix's rows begin at its last token and see all of it, whatever their
    number in the group (B Mq of up to 2^26 / H)."""
    calls = [(n - 1, i, n) for n in (MOST, MOST - 1, MOST - 63, MOST - 2 ** 20, 2 ** 30, 64, 1, 0)
             for i in (0, 1, 63, 64, 65, 66, 1000, 2 ** 20, 2 ** 26 - 1)]
    assert answers(exe, calls) == [n - 1 for _, _, n in calls]


def test_rows_of_windows(exe):
    """len tokens, qn of them query rows, a table that holds as many, fewer or none."""
    rng, calls = random.Random(1), []
    for _ in range(20000):
        n = rng.choice([0, 1, 63, 64, rng.randint(0, 5000), rng.randint(0, 2 ** 31 - 1), 2 ** 31 - 1])
        Mq = rng.choice([1, 2, rng.randint(1, 4000), 2 ** 24])
        qn = rng.choice([1, Mq, rng.randint(1, Mq)])
        held = min(n, rng.choice([0, 64, rng.randint(0, MOST), MOST, n]))
        calls.append((n - qn, rng.choice([0, qn - 1, rng.randint(0, qn - 1)]), held))
    assert answers(exe, calls) == [min(p + i, n - 1) for p, i, n in calls]
