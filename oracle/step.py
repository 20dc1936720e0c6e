"""fp64 / integer references of a serving step's way into the paged cache.

TEST INFRASTRUCTURE ONLY, in numpy, written from the definitions: the tables
and slots of a batch, rotary positions, the 4-bit latent rows, the tokens a
window leaves visible.  Shares nothing with the HIP path.
"""
import math

import numpy as np

BLOCK = 64
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def batch_slots(cached, new, free, table, T):
    """(slots, positions, seq_lens, starts, info, table): request by request,
    block by block, token by token."""
    cached = [max(int(c), 0) for c in cached]
    new = [max(int(n), 0) for n in new]
    table = np.array(table, dtype=np.int64)
    NB = table.shape[1]
    free = [int(f) for f in free]
    slots, pos, starts = [], [], [0]
    taken = 0
    for b, (c, n) in enumerate(zip(cached, new)):
        for j in range(min(-(-c // BLOCK), NB), min(-(-(c + n) // BLOCK), NB)):
            table[b, j] = free[taken] if taken < len(free) else -1
            taken += 1
        for p in range(c, c + n):
            blk = table[b, p // BLOCK] if p // BLOCK < NB else -1
            slots.append(blk * BLOCK + p % BLOCK if 0 <= blk < 2 ** 25 else -1)
            pos.append(p)
        starts.append(starts[-1] + n)
    total = starts[-1]
    slots, pos = (slots + [-1] * T)[:T], (pos + [-1] * T)[:T]
    info = [total, min(taken, len(free)), max(taken - len(free), 0), max(total - T, 0)]
    return (np.array(slots, np.int64), np.array(pos, np.int64),
            np.array([c + n for c, n in zip(cached, new)], np.int64), np.array(starts, np.int64),
            np.array(info, np.int64), table)


def rope_freqs(d, base, scaling="none", factor=1.0, orig_len=0, beta_fast=32.0, beta_slow=1.0):
    """Radians a position of pairs 0 .. d/2 - 1."""
    out = []
    if scaling == "yarn":
        def pair(turns):
            return d / 2 * math.log(orig_len / (2 * math.pi * turns), base)
        lo, hi = max(math.floor(pair(beta_fast)), 0), min(math.ceil(pair(beta_slow)), d - 1)
    for i in range(d // 2):
        w = base ** (-2.0 * i / d)
        if scaling == "linear":
            w /= factor
        if scaling == "yarn":
            r = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            w = w * (1 - r) + w / factor * r
        out.append(w)
    return np.array(out)


def rope(x, positions, at, d, pairing, base, mscale=1.0, inverse=False, **scaling):
    """float64 [T, H, D] with dims at .. at + d - 1 turned."""
    x = np.array(x, dtype=np.float64)
    a = np.asarray(positions, np.float64)[:, None] * rope_freqs(d, base, **scaling)[None]
    if inverse:
        a = -a
    c, s = np.cos(a)[:, None] * mscale, np.sin(a)[:, None] * mscale
    if pairing == 0:
        i, j = np.arange(at, at + d, 2), np.arange(at + 1, at + d, 2)
    else:
        i, j = np.arange(at, at + d // 2), np.arange(at + d // 2, at + d)
    u, v = x[..., i].copy(), x[..., j].copy()
    x[..., i], x[..., j] = u * c - v * s, u * s + v * c
    return x


def mx4_encode(x):
    """float64 [..., 512] -> rows uint8 [..., 272], by the nearest of E2M1's
    magnitudes (halfway: the even code)."""
    x = np.asarray(x, np.float64)
    v = x.reshape(x.shape[:-1] + (16, 32))
    bad = ~np.isfinite(v).all(-1)
    a = np.where(np.isfinite(v), np.abs(v), 0.0)
    amax = a.max(-1)
    e = np.where(amax > 0, np.frexp(np.where(amax > 0, amax, 1.0))[1] - 1 - 2, -125)
    e = np.clip(e, -125, 125)
    u = a / np.exp2(e)[..., None]
    dist = np.abs(u[..., None] - E2M1)
    best = dist.min(-1, keepdims=True)
    hit = dist == best  # one, or two neighbours of which one is even
    odd_first = np.where(hit & (np.arange(8) % 2 == 0), 2, np.where(hit, 1, 0))
    code = odd_first.argmax(-1).astype(np.uint8) | (np.signbit(v).astype(np.uint8) << 3)
    code = code.reshape(x.shape[:-1] + (512,))
    byte = np.where(bad, 255, e + 127).astype(np.uint8)
    return np.concatenate([code[..., 0::2] | (code[..., 1::2] << 4), byte], -1)


def mx4_decode(rows):
    """rows uint8 [..., 272] -> float64 [..., 512]."""
    rows = np.asarray(rows, np.uint8)
    code = np.stack([rows[..., :256] & 15, rows[..., :256] >> 4], -1).reshape(rows.shape[:-1] + (512,))
    v = E2M1[code & 7] * np.where(code & 8, -1.0, 1.0)
    byte = rows[..., 256:].astype(np.int64)
    s = np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127))
    return v * np.repeat(s, 32, axis=-1)


def visible(n, pos, window, n_sink):
    """Which of tokens 0 .. n - 1 a row at position pos sees."""
    t = np.arange(n)
    see = t <= pos
    return see & ((t > pos - window) | (t < n_sink)) if window else see


def attend(q, keys, values, see, scale):
    """Attention of rows q [h, 576] over the tokens `see` of keys [n, 576] /
    values [n, 512], all float64, in two passes.  Returns a dict of out [h,
    512], lse, m, l [h]; sum_t p_t |v_t| (mag) and the largest sum |q| |k|
    |scale| of a row's tokens (smag), which tolerances are made of."""
    h = q.shape[0]
    if not see.any():
        return dict(out=np.zeros((h, values.shape[1])), lse=np.full(h, -np.inf), m=np.full(h, -np.inf),
                    l=np.zeros(h), mag=np.zeros((h, values.shape[1])), smag=np.zeros(h))
    k, v = keys[see], values[see]
    s = scale * (q @ k.T)
    m = s.max(1)
    e = np.exp(s - m[:, None])
    ell = e.sum(1)
    p = e / ell[:, None]
    return dict(out=p @ v, lse=m + np.log(ell), m=m, l=ell, mag=p @ np.abs(v),
                smag=abs(scale) * (np.abs(q) @ np.abs(k).T).max(1))
