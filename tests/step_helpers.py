"""Shared by the tests of windows and 4-bit caches: caches with their exact
values, and the comparison of partials with the float64 reference."""
import numpy as np
import torch

from oracle import step as S

KVS = ("bf16", "fp8", "fp8split", "mx4")


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def host(t):
    return t.detach().double().cpu().numpy()


def randn(seed, *shape, sigma=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * sigma).bfloat16().cuda()


class Cache:
    """A pool of P blocks of a kind, with its values in float64."""

    def __init__(self, seed, P, kv, sigma=0.5):
        rs = np.random.default_rng([seed, 5])
        self.kv, self.scales = kv, {}
        lat, pe = rs.standard_normal((P, 64, 512)) * sigma, rs.standard_normal((P, 64, 64)) * sigma
        if kv in ("bf16", "mx4"):
            self.kpe = torch.from_numpy(pe).bfloat16().cuda()
            self.pe = host(self.kpe)
        if kv == "bf16":
            self.ckv = torch.from_numpy(lat).bfloat16().cuda()
            self.lat = host(self.ckv)
        elif kv == "mx4":
            # group magnitudes over a wide range, as outlier channels have them
            lat *= np.exp2(rs.integers(-3, 3, (P, 64, 16))).repeat(32, -1)
            rows = S.mx4_encode(lat)
            self.ckv, self.lat = torch.from_numpy(rows).cuda(), S.mx4_decode(rows)
        else:
            # (block scales differ, so that a wrong block's would show)
            f = np.exp2(rs.integers(-2, 3, P))[:, None, None]
            vals, scales = [], []
            for x, g in ((lat * f, 1.0), (pe * f, 1.0 if kv == "fp8" else 0.37)):
                s = (np.abs(x).max((1, 2)) if kv != "fp8" else
                     np.maximum(np.abs(lat * f).max((1, 2)), np.abs(pe * f).max((1, 2)))) / 448.0 * g
                s = s.astype(np.float32)
                c = torch.from_numpy(np.clip(x / s[:, None, None], -448, 448)).to(torch.float8_e4m3fn)
                vals.append((c, c.double().numpy() * s.astype(np.float64)[:, None, None]))
                scales.append(torch.from_numpy(s).cuda())
            (c0, self.lat), (c1, self.pe) = vals
            self.ckv, self.kpe = c0.view(torch.uint8).cuda(), c1.view(torch.uint8).cuda()
            self.scales = dict(ckv_scale=scales[0], kpe_scale=scales[0] if kv == "fp8" else scales[1])

    def tokens(self, blocks):
        """(keys [n, 576], values [n, 512]) of the pool blocks, in order."""
        blocks = np.asarray(blocks, np.int64)
        lat, pe = self.lat[blocks].reshape(-1, 512), self.pe[blocks].reshape(-1, 64)
        return np.concatenate([lat, pe], 1), lat


def check_row(ref, out, stat, wire, what):
    """One query row [h] of a partial against attend()'s.

    Scores are bf16 products summed in fp32 (18 products of 32 dims a score,
    inside which the order is the hardware's): off by ds <= 2^-18 of the sum of
    magnitudes.  Weights carry that twice (their own and the denominator's) and
    one rounding to bf16, 2^-8 of each, which the normaliser shares: out is off
    by (2 ds + 2^-7) mag; split rows may be held in fp16 scaled by the row's
    largest value, 2^-11 of it; the wire form adds half a bf16 step."""
    ds = 2.0 ** -18 * ref["smag"] + 2.0 ** -20
    dead = ref["l"] == 0
    if wire:
        m, ell = stat[..., 0], stat[..., 1]
        assert np.array_equal(np.isneginf(m), dead), f"{what}: empty rows"
        assert (ell[dead] == 0).all(), what
        live = ~dead
        m, ref = np.where(dead, 0, m), dict(ref, m=np.where(dead, 0, ref["m"]))
        assert (np.abs(m - ref["m"])[live] <= ds[live] + 2.0 ** -22 * np.abs(ref["m"][live])).all(), f"{what}: m"
        assert (np.abs(ell - ref["l"])[live] <= ref["l"][live] * (4 * ds[live] + 2.0 ** -18)).all(), f"{what}: l"
    else:
        assert np.array_equal(np.isneginf(stat), dead), f"{what}: empty rows"
        err = np.abs(stat[~dead] - ref["lse"][~dead])
        assert (err <= 2 * ds[~dead] + 2.0 ** -20 * (1 + np.abs(ref["lse"][~dead]))).all(), f"{what}: lse {err.max()}"
    assert np.isfinite(out).all(), f"{what}: not finite"
    assert (out[dead] == 0).all(), f"{what}: empty rows are 0"
    tol = (4 * ds[:, None] + 2.0 ** -7) * ref["mag"] + 2.0 ** -11 * np.abs(ref["out"]).max(1, keepdims=True)
    if wire:
        tol = tol + 2.0 ** -8 * np.abs(ref["out"])
    bad = np.abs(out - ref["out"]) > tol + 1e-30
    assert not bad.any(), f"{what}: out off by {(np.abs(out - ref['out']) / (tol + 1e-30)).max():.3g} x tolerance"
