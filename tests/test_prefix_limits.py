"""The most work items of one call of mla_prefix_attn, refused past that on the host
(CPU only)."""
import pytest
import torch

from paper_2606_01502_amd import mla
from tests.test_choose_abi import opts, prefix_args, prefix_call
from tests.test_step_abi import F32, I32, UNSUPPORTED, z

MOST = 1 << 22


def args(B, Mq, H, NBP, NB, **o):
    a = prefix_args()
    # (rows given once and repeated: what a call of this size reads is not the point)
    a.update(q_lat=z(1, 1, 1, 512).expand(B, Mq, H, 512), q_pe=z(1, 1, 1, 64).expand(B, Mq, H, 64),
             ptable=torch.empty((1, NBP), dtype=I32), plens=z(1, dt=I32), starts=z(2, dt=I32),
             table=torch.empty((B, NB), dtype=I32), lens=z(B, dt=I32), q_lens=None,
             out=torch.empty((B, Mq, H, 512), dtype=F32), lse=torch.empty((B, Mq, H), dtype=F32),
             opts=opts(mla.PrefixOpts, **o))
    return a


@pytest.mark.parametrize("B,Mq,H,NBP,NB,o", [
    (1, 33, 128, 2 ** 25 - 1, 1, {}),                  # 33 tiles of 128 rows in 131,072 splits of 256 blocks
    (1, 17, 128, 2 ** 25 - 1, 1, dict(row_tile=64)),   # 34 of 64 rows
    (MOST + 1, 1, 1, 1, 1, {}),                        # a work item for each request's own token
    (65, 1, 1, 1, 1 << 16, dict(own_splits=1 << 16)),  # 65 requests in 65,536 splits each
    (2049, 1, 64, 2048, 1, dict(n_splits=2048)),
])
def test_more_work_items_than_a_call_holds(B, Mq, H, NBP, NB, o):
    st, msg = prefix_call(args(B, Mq, H, NBP, NB, **o))
    assert st == UNSUPPORTED and "grid" in msg, (st, msg)


def test_the_declaration_names_the_limit():
    import os
    from paper_2606_01502_amd import build
    with open(os.path.join(build.ROOT, "include", "mla_sparse.h")) as f:
        text = f.read()
    at = text.index("Attention for a batch that shares long prefixes")
    assert "2^22 work items" in text[at:text.index("mla_status_t mla_prefix_attn")]
