"""The fastest rotation that mla_rope takes: a pair may turn once a position, of
which a position of 2^31 leaves a double about 2^-20 of a turn.  Refusals on the
CPU; the fastest accepted ones on the GPU against 64 bits of mantissa."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2606_01502_amd import mla


def call(x, pos, out, **o):
    opts = dict(rot_offset=0, rot_dim=x.shape[2], base=1e4, factor=1.0, beta_fast=32.0, beta_slow=1.0, mscale=1.0,
                orig_len=4096)
    opts.update(o)
    lib = mla.load()
    d = [mla.describe(t) for t in (x, pos, out)]
    st = lib.mla_rope(*[ctypes.byref(t) for t in d], ctypes.byref(mla.RopeOpts(**opts)), None)
    return st, lib.mla_last_error().decode()


@pytest.mark.parametrize("o", [dict(base=0.1), dict(base=1e-3), dict(base=1.0, scaling=1, factor=0.159),
                               dict(scaling=1, factor=1e-4), dict(scaling=2, factor=1e-4),
                               dict(base=1e-9), dict(scaling=1, factor=1e-6)])
def test_pairs_that_turn_more_than_once_a_position_are_refused(o):
    z = torch.zeros(2, 1, 64, dtype=torch.bfloat16)
    st, msg = call(z, torch.zeros(2, dtype=torch.int32), torch.zeros_like(z), **o)
    assert st == mla.MLA_ERR_INVALID_ARGUMENT and "turns more than once a position" in msg, (st, msg)


@pytest.mark.gpu
@pytest.mark.parametrize("pairing", [0, 1])
@pytest.mark.parametrize("inverse", [False, True])
def test_the_fastest_accepted(pairing, inverse):
    """All 16 pairs turn 1 / (2 pi factor) = 0.9947 times a position.  That number is
    off by 3 roundings of a double (the power, the factor's and 2 pi's division), its
    product with the position by one more: 4 x 2^-53 x 2^31 = 2^-20 turns, 2 pi times
    as much in radians, and as much again of |x| + |y| in the result; fp32 arithmetic
    adds 2^-20 of it, as for near positions."""
    print(f"case: rope fastest {pairing} {inverse}", flush=True)
    pos = np.array([2 ** 31 - 1, -(2 ** 31), 2 ** 31 - 12345, -(10 ** 9) - 7, 1, 0])
    g = torch.Generator().manual_seed(3)
    x = torch.randn((6, 2, 32), generator=g).cuda()
    factor = 0.16
    got = mla.rope(x, torch.from_numpy(pos.astype(np.int32)).cuda(), pairing=pairing, base=1.0, scaling="linear",
                   factor=factor, inverse=inverse)
    torch.cuda.synchronize()
    ld = np.longdouble
    assert np.finfo(ld).nmant >= 63
    turns = pos.astype(ld) / (ld(factor) * 8 * np.arctan(ld(1)))
    a = ((turns - np.rint(turns)) * 8 * np.arctan(ld(1))).astype(np.float64)[:, None, None] * (-1 if inverse else 1)
    h = x.double().cpu().numpy()
    u, v = (h[..., 0::2], h[..., 1::2]) if pairing == 0 else (h[..., :16], h[..., 16:])
    ref = np.empty_like(h)
    i, j = (np.arange(0, 32, 2), np.arange(1, 32, 2)) if pairing == 0 else (np.arange(16), np.arange(16, 32))
    ref[..., i], ref[..., j] = u * np.cos(a) - v * np.sin(a), u * np.sin(a) + v * np.cos(a)
    tol = np.empty_like(h)
    tol[..., i] = tol[..., j] = (np.abs(u) + np.abs(v)) * (2 * np.pi + 1) * 2.0 ** -20
    err = np.abs(got.double().cpu().numpy() - ref)
    assert (err <= tol).all(), (err / tol).max()
