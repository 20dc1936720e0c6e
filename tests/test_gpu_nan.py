"""A NaN in the cache on the GPU: every row that attends its token is NaN, in its
output and in its statistics, whatever the form, the tile and the number of
splits, and stays so through a merge; no other row changes."""
import numpy as np
import pytest
import torch

from paper_2606_01502_amd import mla
from tests import step_helpers as T

pytestmark = pytest.mark.gpu
SCALE = 0.0721688
# what a latent row is filled with to hold a NaN (4 bits: the exponent of group 7)
NAN = {"bf16": torch.nan, "fp8": 0x7F, "fp8split": 0xFF, "mx4": 255}


def poison(c, block, t):
    if c.kv == "mx4":
        c.ckv[block, t, 256 + 7] = 255
    else:
        c.ckv[block, t, 200:210] = NAN[c.kv]


def inputs(seed, R, Mq, H, NB, kv):
    c = T.Cache(seed, R * NB + 2, kv)
    table = np.random.default_rng(seed).permutation(R * NB + 2)[:R * NB].reshape(R, NB)
    return c, T.randn(seed, R, Mq, H, 512), T.randn(seed + 1, R, Mq, H, 64), table


def check(call, c, place):
    """call() before and after the NaN at `place`: job 0 is NaN, job 1 unchanged."""
    want = [t.clone() for t in call()]
    poison(c, *place)
    got = call()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.isfinite(b).all()
        assert torch.isnan(a[0]).all(), "rows that attend the NaN"
        assert torch.equal(a[1], b[1]), "rows that do not"


@pytest.mark.parametrize("wire", [False, True])
@pytest.mark.parametrize("n_splits", [1, 2, 17, 40])  # (40: split rows of 128 rows in fp16)
@pytest.mark.parametrize("H,row_tile", [(16, 64), (64, 64), (128, 64), (128, 128)])
@pytest.mark.parametrize("kv", T.KVS)
def test_blocks(kv, H, row_tile, n_splits, wire):
    print(f"case: nan blocks {kv} {H} {row_tile} {n_splits} {wire}", flush=True)
    if kv == "mx4" and row_tile == 128:
        return  # refused
    c, ql, qp, table = inputs(3, 2, 1, H, 48, kv)
    sel = np.tile(np.arange(44), (2, 1))
    check(lambda: mla.sparse_partial_attn(ql, qp, c.ckv, c.kpe, T.i32(table), T.i32(sel), SCALE, wire=wire,
                                          n_splits=n_splits, row_tile=row_tile, **c.scales), c, (table[0, 21], 40))


@pytest.mark.parametrize("n_splits", [1, 20])
@pytest.mark.parametrize("kv", T.KVS)
def test_tokens_and_rows_of_their_own(kv, n_splits):
    print(f"case: nan tokens {kv} {n_splits}", flush=True)
    c, ql, qp, table = inputs(5, 2, 2, 24, 30, kv)
    sel = np.tile(np.random.default_rng(1).permutation(30 * 64)[:1300], (2, 1))
    b, t = divmod(int(sel[0, 700]), 64)
    check(lambda: mla.sparse_partial_attn(ql, qp, c.ckv, c.kpe, T.i32(table), T.i32(sel), SCALE, tokens=True,
                                          n_splits=n_splits, **c.scales), c, (table[0, b], t))
    if kv == "mx4":
        return  # one selection per job
    c, ql, qp, table = inputs(5, 2, 2, 24, 30, kv)
    sel = np.stack([np.stack([np.arange(20), np.arange(8, 28)])] * 2)
    check(lambda: mla.sparse_partial_attn(ql, qp, c.ckv, c.kpe, T.i32(table), T.i32(sel), SCALE,
                                          n_splits=n_splits, **c.scales), c, (table[0, 15], 7))


@pytest.mark.parametrize("wire", [False, True])
@pytest.mark.parametrize("n_splits", [0, 1, 2, 17, 40])
@pytest.mark.parametrize("H,row_tile", [(16, 64), (64, 64), (128, 128)])
@pytest.mark.parametrize("kv", T.KVS)
def test_windows(kv, H, row_tile, n_splits, wire):
    print(f"case: nan window {kv} {H} {row_tile} {n_splits} {wire}", flush=True)
    if kv == "mx4" and row_tile == 128:
        return  # refused
    c, ql, qp, table = inputs(7, 2, 2, H, 48, kv)
    lens = T.i32([48 * 64 - 9, 2000])
    check(lambda: mla.window_attn(ql, qp, c.ckv, c.kpe, T.i32(table), lens, SCALE, wire=wire, n_splits=n_splits,
                                  row_tile=row_tile, **c.scales), c, (table[0, 21], 40))


@pytest.mark.parametrize("kv,row_tile", [("bf16", 64), ("bf16", 128), ("fp8", 64), ("mx4", 64)])
def test_scores_that_are_all_nan(kv, row_tile):
    """A split, or a whole call, without a score that is a number."""
    print(f"case: all nan {kv} {row_tile}", flush=True)
    for n_splits in (1, 3, 18):
        for wire in (False, True):
            c, ql, qp, table = inputs(9, 2, 1, 64, 20, kv)
            for b in table[0]:
                c.ckv[b] = NAN[kv]
            got = mla.sparse_partial_attn(ql, qp, c.ckv, c.kpe, T.i32(table), T.i32(np.tile(np.arange(20), (2, 1))),
                                          SCALE, wire=wire, n_splits=n_splits, row_tile=row_tile, **c.scales)
            torch.cuda.synchronize()
            assert all(torch.isnan(t[0]).all() and torch.isfinite(t[1]).all() for t in got)


@pytest.mark.parametrize("wire", [False, True])
@pytest.mark.parametrize("n", [1, 2, 4, 8, 16, 17, 40, 64])
def test_merge(n, wire):
    """A part whose log-sum-exp is NaN takes part: its rows are NaN, alone or among
    others; empty parts are skipped as ever, whatever they hold."""
    print(f"case: nan merge {n} {wire}", flush=True)
    g = torch.Generator().manual_seed(n)
    lat = torch.randn((n, 2, 1, 4, 512), generator=g)
    lse = torch.randn((n, 2, 1, 4), generator=g)
    lat[n // 2, 0, 0, 1], lse[n // 2, 0, 0, 1] = torch.nan, torch.nan  # one part of a row
    lat[:, 0, 0, 2], lse[:, 0, 0, 2] = torch.nan, -torch.inf           # empty in every part
    lat[:, 0, 0, 3], lse[:, 0, 0, 3] = torch.nan, -torch.inf           # in every part but one
    lse[n - 1, 0, 0, 3] = torch.nan
    if wire:
        pair = torch.stack([lse, torch.ones_like(lse)], -1)
        pair[torch.isneginf(lse)] = torch.tensor([-torch.inf, 0.0])
        pair[torch.isnan(lse)] = torch.tensor([0.5, torch.nan])  # (a largest score that is a number)
        lat, stat = lat.bfloat16(), pair
    else:
        stat = lse
    out, got = mla.merge_partials([x.cuda() for x in lat], [x.cuda() for x in stat], out_lse=True)
    torch.cuda.synchronize()
    out, got = out.cpu(), got.cpu()
    for h, state in enumerate(["live", "nan", "empty", "nan"]):
        if state == "nan":
            assert torch.isnan(out[0, 0, h]).all() and torch.isnan(got[0, 0, h]), h
        elif state == "empty":
            assert (out[0, 0, h] == 0).all() and torch.isneginf(got[0, 0, h]), h
        else:
            assert torch.isfinite(out[0, 0, h]).all() and torch.isfinite(got[0, 0, h]), h
    assert torch.isfinite(out[1]).all() and torch.isfinite(got[1]).all()


def test_a_partial_and_its_merge():
    """The way of a NaN from the cache through a partial in splits to the merged row."""
    print("case: nan, partial and merge", flush=True)
    for kv in ("bf16", "mx4"):
        for wire in (False, True):
            c, ql, qp, table = inputs(11, 2, 1, 16, 40, kv)
            poison(c, table[0, 3], 9)
            kw = dict(wire=wire, **c.scales)
            a = mla.sparse_partial_attn(ql, qp, c.ckv, c.kpe, T.i32(table), T.i32([list(range(20))] * 2), SCALE,
                                        n_splits=18, **kw)
            b = mla.window_attn(ql, qp, c.ckv, c.kpe, T.i32(table), T.i32([2560] * 2), SCALE, window=1000, **kw)
            out, lse = mla.merge_partials([a[0], b[0]], [a[1], b[1]], out_lse=True)
            torch.cuda.synchronize()
            assert torch.isnan(out[0]).all() and torch.isnan(lse[0]).all()
            assert torch.isfinite(out[1]).all() and torch.isfinite(lse[1]).all()


# ---------------------------------------------------------------- rows without a token
@pytest.mark.parametrize("wire", [False, True])
@pytest.mark.parametrize("n_splits", [0, 1, 2, 20])
@pytest.mark.parametrize("H,row_tile", [(5, 64), (12, 64), (12, 128)])
@pytest.mark.parametrize("kv", T.KVS)
def test_rows_without_a_token_are_empty(kv, H, row_tile, n_splits, wire):
    """Padding rows and rows at negative positions, in one tile with rows that
    attend a NaN: 0, and the statistics of an empty row."""
    print(f"case: nan beside empty rows {kv} {H} {row_tile} {n_splits} {wire}", flush=True)
    if kv == "mx4" and row_tile == 128:
        return  # refused
    c, ql, qp, table = inputs(13, 2, 6, H, 24, kv)
    lens, q_lens = [24 * 64 - 3, 2], [4, 6]  # of the second: rows 0 to 3 lie ahead of its start
    poison(c, table[0, 2], 5)
    poison(c, table[1, 0], 0)
    for window, sinks in ((0, 0), (3, 200)):
        out, stat = mla.window_attn(ql, qp, c.ckv, c.kpe, T.i32(table), T.i32(lens), SCALE, window=window,
                                    n_sink=sinks, q_lens=T.i32(q_lens), n_splits=n_splits, row_tile=row_tile,
                                    wire=wire, **c.scales)
        torch.cuda.synchronize()
        empty = np.zeros((2, 6), bool)
        empty[0, 4:] = empty[1, :4] = True
        o, st = T.host(out), T.host(stat)
        assert (o[empty] == 0).all() and np.isnan(o[~empty]).all() and np.isnan(st[~empty]).all()
        assert np.isneginf(st[empty][..., 0] if wire else st[empty]).all() and (not wire or (st[empty][..., 1] == 0).all())


@pytest.mark.parametrize("wire", [False, True])
@pytest.mark.parametrize("n_splits", [30, 60])
@pytest.mark.parametrize("sinks", [2, 1900])  # (few splits a row; more than a wave reads in one trip)
@pytest.mark.parametrize("kv,H,row_tile", [("bf16", 1, 64), ("bf16", 2, 64), ("bf16", 1, 128), ("fp8", 1, 64), ("fp8", 1, 128),
                                           ("fp8split", 1, 64), ("mx4", 1, 64), ("mx4", 2, 64)])
def test_splits_without_a_token(kv, H, row_tile, sinks, n_splits, wire):
    """Splits of a stage or two: rows that see none of the tokens of a NaN's split
    are what they were, however many splits they have; rows that see it are NaN."""
    print(f"case: nan in other rows' split {kv} {H} {row_tile} {sinks} {n_splits} {wire}", flush=True)
    Mq, n, window = 128 // H, 2570, 8
    c, ql, qp, table = inputs(15, 1, Mq, H, 41, kv)
    n_splits += 24 if sinks > 1000 else 0

    def call():
        return mla.window_attn(ql, qp, c.ckv, c.kpe, T.i32(table), T.i32([n]), SCALE, window=window, n_sink=sinks,
                               n_splits=n_splits, row_tile=row_tile, wire=wire, **c.scales)
    want = [t.clone() for t in call()]
    t = n - 2
    poison(c, table[0, t // 64], t % 64)
    got = call()
    torch.cuda.synchronize()
    pos = n - Mq + np.arange(Mq)
    sees = pos >= t
    # The NaN is in the last split.  A call takes at most K splits, K the blocks that a
    # tile may see: with 2 sinks 3 or 4 for as many stages, one a split; with 1900
    # sinks 32 or 33, for 33 stages of 64 tokens, or 62 or 63 of 32, two in the last.
    first = t // 64 * 64 if row_tile == 128 else t // 32 * 32 - (32 if sinks > 1000 else 0)
    apart = pos < first
    assert sees.sum() == 2 and apart.sum() > 20
    for a, b in zip(got, want):
        assert torch.isnan(a[0][T.host(torch.from_numpy(sees)).astype(bool)]).all()
        keep = torch.from_numpy(apart).cuda()
        assert torch.equal(a[0][keep], b[0][keep])


def test_rows_with_an_empty_selection_of_their_own():
    """Rows that select nothing beside rows that attend a NaN."""
    for kv in ("bf16", "fp8", "fp8split"):
        for H, row_tile in ((5, 64), (12, 64), (12, 128)):
            for n_splits in (0, 1, 3):
                for wire in (False, True):
                    print(f"case: nan beside empty selections {kv} {H} {row_tile} {n_splits} {wire}", flush=True)
                    c, ql, qp, table = inputs(17, 2, 3, H, 12, kv)
                    sel = np.tile(np.arange(9), (2, 3, 1))
                    sel[:, 1] = -1
                    poison(c, table[0, 4], 9)
                    out, stat = mla.sparse_partial_attn(ql, qp, c.ckv, c.kpe, T.i32(table), T.i32(sel), SCALE,
                                                        wire=wire, n_splits=n_splits, row_tile=row_tile, **c.scales)
                    torch.cuda.synchronize()
                    assert (out[:, 1] == 0).all() and torch.isneginf(stat[:, 1, :, 0] if wire else stat[:, 1]).all()
                    assert torch.isnan(out[0, 0]).all() and torch.isnan(stat[0, 2]).all()
                    assert torch.isfinite(out[1]).all()
