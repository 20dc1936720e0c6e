"""The turned write against the formula, each value held to its own pair."""
import numpy as np
import pytest
import torch

from oracle import step as S
from paper_2606_01502_amd import mla
from tests import step_helpers as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pairing", [0, 1])
@pytest.mark.parametrize("far", [1, 1 << 20, 1 << 31])
def test_rope_append_pairs(pairing, far):
    """x' = x c - y s, y' = x s + y c in fp32: cosine and sine off by 2^-20 (the angle
    reduced in double, where 2^31 positions of a turn at most leave 2^-22 of one, 2 pi
    2^-22 < 2^-19 of an angle), products and sum by 2^-23 of |x| + |y|, one rounding to
    bf16 (2^-8).  Both signs of positions."""
    print(f"case: pairs {pairing} {far}", flush=True)
    n, P = 300, 6
    rs = np.random.default_rng(far % 1000 + pairing)
    pos = rs.integers(-far, far, n)
    at = rs.permutation(P * 64)[:n]
    new = T.randn(9, n, 576)
    ckv = torch.zeros((P, 64, 512), dtype=torch.bfloat16, device="cuda")
    kpe = torch.zeros((P, 64, 64), dtype=torch.bfloat16, device="cuda")
    mla.rope_append(new[:, :512], new[:, 512:], T.i32(pos), T.i32(at), ckv, kpe, pairing=pairing)
    torch.cuda.synchronize()
    got, x = T.host(kpe).reshape(-1, 64)[at], T.host(new)[:, None, 512:]
    want = S.rope(x, pos, 0, 64, pairing, 10000.0)[:, 0]
    a = np.abs(x[:, 0])
    pair = a.reshape(n, 32, 2).sum(-1).repeat(2, -1) if pairing == 0 else np.tile(a[:, :32] + a[:, 32:], (1, 2))
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -18 + 2.0 ** -22) * pair
    assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()
    assert np.array_equal(T.host(ckv).reshape(-1, 512)[at], T.host(new)[:, :512])
