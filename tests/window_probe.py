"""The plans of windows and 4-bit caches on the CPU: csrc/mla_plan.h compiled here
with g++ into a small program that reads calls and prints their plans."""
import os
import subprocess
from dataclasses import dataclass

from paper_2606_01502_amd import build as B

CUS = 256
LIST_HALVES = 512       # half blocks that one split lists
SHARE_REQUESTS = 256    # requests that splits are shared out between

_MAIN = r"""
#include "mla_plan.h"
#include <cstdio>
static void show(const mla::Planner& p, const mla::Plan& q) {
  std::printf(" %d %lld %lld %lld %.17g %llu %llu %d %d", q.row_groups, (long long)q.row_tiles, (long long)q.S,
              (long long)q.sps, q.us, (unsigned long long)(q.S > 1 ? p.ws_rows_bytes(q.S) : 0),
              (unsigned long long)(q.S > 1 ? p.ws_size(q.S) : 0), (int)p.ws_half(q.S), (int)p.shares(q.S));
}
int main() {
  std::printf("%d %d\n", mla::kWindowList, mla::kShareRequests);
  long long R, Mq, H, NB, K, tok, fp8, mx4, win, ns, rt;
  while (std::scanf("%lld %lld %lld %lld %lld %lld %lld %lld %lld %lld %lld", &R, &Mq, &H, &NB, &K, &tok, &fp8, &mx4,
                    &win, &ns, &rt) == 11) {
    const mla::Planner p({R, Mq, H, NB, K, tok != 0, false, fp8 != 0, (int)ns, (int)rt, 256, mx4 != 0, win != 0});
    if (p.refused) { std::printf("refused\n"); continue; }
    show(p, p.choose());
    show(p, p.cover);
    std::printf("\n");
  }
}
"""


@dataclass
class Call:
    R: int
    Mq: int
    H: int
    NB: int
    K: int  # blocks that a tile's rows may see (windows), or slots of a selection
    kv: str = "bf16"
    window: bool = True
    tokens: bool = False
    n_splits: int = 0
    row_tile: int = 0

    @property
    def rows(self):
        return self.Mq * self.H


@dataclass
class Plan:
    row_groups: int
    row_tiles: int
    S: int
    sps: int
    us: float
    rows_bytes: int
    ws: int
    half: bool
    shares: bool


def build(tmp):
    src, exe = os.path.join(tmp, "plan.cc"), os.path.join(tmp, "plan")
    with open(src, "w") as f:
        f.write(_MAIN)
    rocm = os.path.dirname(os.path.dirname(B.HIPCC))
    subprocess.run(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"), "-I",
                    B.CSRC, "-o", exe, src], check=True)
    return exe


def _parse(v):
    return Plan(int(v[0]), int(v[1]), int(v[2]), int(v[3]), float(v[4]), int(v[5]), int(v[6]), v[7] == "1", v[8] == "1")


def plans(exe, calls):
    """[(plan, covering plan)] of the calls, as the library plans them: 4-bit caches
    in 64-row tiles."""
    lines = [f"{c.R} {c.Mq} {c.H} {c.NB} {c.K} {int(c.tokens)} {int(c.kv == 'fp8')} {int(c.kv == 'mx4')} "
             f"{int(c.window)} {c.n_splits} {64 if c.kv == 'mx4' else c.row_tile}" for c in calls]
    out = subprocess.run([exe], input="\n".join(lines) + "\n", check=True, capture_output=True, text=True)
    rows = out.stdout.splitlines()
    assert rows[0] == f"{LIST_HALVES} {SHARE_REQUESTS}" and len(rows) == len(calls) + 1
    return [(_parse(v[:9]), _parse(v[9:])) for v in (ln.split() for ln in rows[1:])]


def window_halves(Mq, H, NB, window, n_sink):
    """The most half blocks that the rows of a tile may see, as the library bounds
    them: a tile of 128 rows meets at most 127 // H + 2 query rows."""
    if window == 0:
        return 2 * NB
    n_i = min(Mq, 127 // H + 2)
    return min(2 * NB, (n_sink + 31) // 32 + (window + n_i - 2) // 32 + 2)


def window_blocks(Mq, H, NB, window, n_sink):
    return (window_halves(Mq, H, NB, window, n_sink) + 1) // 2


def draw(rng):
    def log(lo, hi):
        return int(round(2 ** rng.uniform(lo, hi)))
    kv = rng.choice(["bf16", "fp8", "mx4"])
    R, Mq, H = log(0, 10), log(0, 9), rng.choice([1, 3, 8, 16, 24, 40, 64, 65, 128, 200])
    if Mq * H * R > 1 << 20:
        Mq = 1
    NB = log(0, 13)
    if rng.random() < 0.15:  # a selection over a 4-bit cache
        tokens = rng.random() < 0.5
        return Call(R, Mq, H, NB, log(0, 12), "mx4", window=False, tokens=tokens, n_splits=rng.choice([0, 0, 0, 1, 3, 40]))
    window = rng.choice([0, 0, log(0, 18)])
    K = window_blocks(Mq, H, NB, window, rng.choice([0, 4, log(0, 12)]))
    return Call(R, Mq, H, NB, K, kv, n_splits=rng.choice([0, 0, 0, 0, 1, 2, 7, 300, 100000]),
                row_tile=rng.choice([0, 0, 64, 128]))
