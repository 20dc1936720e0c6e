"""Every exponent byte of a 4-bit row on the GPU: read back as the value it stands
for, and in attention from the smallest to the largest that scores hold."""
import numpy as np
import pytest
import torch

from oracle import step as S
from paper_2606_01502_amd import mla
from tests import test_gpu_mx4 as M
from tests import step_helpers as T

pytestmark = pytest.mark.gpu


def test_gather_of_every_byte_and_code():
    """Exact, subnormal numbers among them; past bf16's largest number (255 x 2^120)
    an infinity; byte 255 a NaN."""
    print("case: gather of every exponent", flush=True)
    rs = np.random.default_rng(6)
    pool = np.stack([rs.permutation(np.tile(np.arange(16), 32)) for _ in range(256 * 4)]).reshape(1, 16, 64, 512)
    pool = np.concatenate([pool[..., 0::2] | (pool[..., 1::2] << 4),
                           np.repeat(np.arange(256), 64).reshape(1, 16, 64, 16)], -1).astype(np.uint8)
    out, _ = mla.fetch_gather(torch.from_numpy(pool).cuda(), torch.zeros(1, 16, 64, 64).bfloat16().cuda(),
                              T.i32(np.arange(16)), T.i32(np.arange(1024)))
    torch.cuda.synchronize()
    want = S.mx4_decode(pool.reshape(1, 1024, 272))
    want = np.where(np.abs(want) > 255 * 2.0 ** 120, np.copysign(np.inf, want), want)
    got = T.host(out)
    assert np.array_equal(got, want, equal_nan=True)
    assert np.array_equal(np.signbit(got), np.signbit(want) & ~np.isnan(want) | np.signbit(got) & np.isnan(want))


@pytest.mark.parametrize("lo,hi,sigma", [(0, 4, 1.0), (0, 128, 1.0), (128, 201, 2.0 ** -73), (220, 246, 2.0 ** -118)])
@pytest.mark.parametrize("H,n_splits", [(16, 0), (64, 2), (128, 3)])
def test_attention_over_small_and_large_exponents(lo, hi, sigma, H, n_splits):
    """Groups of bytes lo .. hi - 1 side by side, the query as much smaller as keeps
    scores near 1 (in 3 splits of 128 rows the split rows are scaled fp16)."""
    print(f"case: exponents {lo} {hi} {H} {n_splits}", flush=True)
    R = 3
    c, ql, qp, table, sel = M.inputs(21, R, 1, H, 8, 7)
    rows = c.ckv.cpu().numpy()
    rows[..., 256:] = np.random.default_rng(lo).integers(lo, hi, rows[..., 256:].shape)
    c.ckv, c.lat = torch.from_numpy(rows).cuda(), S.mx4_decode(rows)
    ql, qp = T.randn(5, *ql.shape, sigma=sigma), T.randn(6, *qp.shape, sigma=sigma)
    M.check(c, ql, qp, table, sel, n_splits=n_splits)
    M.check(c, ql, qp, table, sel, n_splits=n_splits, wire=True)
