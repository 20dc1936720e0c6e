"""Shared prefixes of as many tokens as a table may name, 2^31 - 64, of which a few
blocks are held: every row of a group sees them, also the rows whose number in the
group and the prefix's last token add up to 2^31 and more."""
import numpy as np
import pytest
import torch

from oracle import choose as C
from paper_2606_01502_amd import mla
from tests import step_helpers as T

pytestmark = pytest.mark.gpu
SCALE = 0.0721688
NBP = 2 ** 25 - 1


@pytest.mark.parametrize("row_tile,plen", [(64, 2 ** 31 - 64), (128, 2 ** 31 - 1), (64, 2 ** 31 - 64 - 40)])
def test_every_row_sees_the_longest_prefix(row_tile, plen):
    """70 requests of one row and one head in one group: from the 66th on the sum
    passes 2^31."""
    print(f"case: far prefix {row_tile} {plen}", flush=True)
    B = 70
    c = T.Cache(3, 6, "bf16")
    at, blocks = np.array([0, 12345678, NBP - 1]), [4, 1, 2]
    ptable = torch.full((1, NBP), -1, dtype=torch.int32, device="cuda")
    ptable[0, torch.from_numpy(at).cuda()] = T.i32(blocks)
    ql, qp = T.randn(1, B, 1, 1, 512), T.randn(2, B, 1, 1, 64)
    lens = np.arange(B) % 9
    out, lse = mla.prefix_attn(ql, qp, c.ckv, c.kpe, ptable, T.i32([plen]), T.i32([0, B]), T.i32([[3]] * B),
                               T.i32(lens), SCALE, row_tile=row_tile)
    torch.cuda.synchronize()
    q, o, st = np.concatenate([T.host(ql), T.host(qp)], -1), T.host(out), T.host(lse)
    pk, pv = c.tokens(blocks)
    held = np.repeat(64 * at, 64) + np.tile(np.arange(64), 3) < plen
    k, v = c.tokens([3])
    for b in range(B):
        ref = C.prefix_row(q[b, 0], (pk[held], pv[held]), (k, v), int(lens[b]), int(lens[b]) - 1, float(np.float32(SCALE)))
        T.check_row(ref, o[b, 0], st[b, 0], False, f"request {b}")
