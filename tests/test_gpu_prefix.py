"""Attention behind shared prefixes on the GPU against the float64 reference
(oracle/choose.py): every cache type, groups of any size, prefixes and own tokens
that end inside a block or are none, ragged and padded batches, splits, strides,
graphs."""
import numpy as np
import pytest
import torch

from oracle import choose as C
from paper_2606_01502_amd import mla
from tests import step_helpers as T

pytestmark = pytest.mark.gpu
SCALE = 0.0721688


class Case:
    def __init__(self, seed, B, Mq, H, starts, NBP, NB, kv="bf16", extra=3):
        G = len(starts) - 1
        P = G * NBP + B * NB + extra
        self.c = T.Cache(seed, P, kv)
        blocks = np.random.default_rng(seed).permutation(P)
        self.ptable, self.table = blocks[:G * NBP].reshape(G, NBP), blocks[G * NBP:G * NBP + B * NB].reshape(B, NB)
        self.q = T.randn(seed, B, Mq, H, 512), T.randn(seed + 1, B, Mq, H, 64)
        self.starts = starts

    def run(self, plens, lens, q_lens=None, q=None, wire=False, **kw):
        return mla.prefix_attn(*(q or self.q), self.c.ckv, self.c.kpe, T.i32(self.ptable), T.i32(plens),
                               T.i32(self.starts), T.i32(self.table), T.i32(lens), SCALE,
                               q_lens=None if q_lens is None else T.i32(q_lens), wire=wire, **self.c.scales, **kw)

    def check(self, plens, lens, q_lens=None, wire=False, got=None, **kw):
        out, stat = got or self.run(plens, lens, q_lens, wire=wire, **kw)
        torch.cuda.synchronize()
        o, st = T.host(out), T.host(stat)
        q = np.concatenate([T.host(self.q[0]), T.host(self.q[1])], -1)
        B, Mq, _, _ = q.shape
        G, P = len(self.starts) - 1, self.c.lat.shape[0]
        starts = [0, *[min(max(s, 0), B) for s in self.starts[1:-1]], B]

        def held(table, n):
            n = min(max(int(n), 0), 64 * len(table))
            e = np.asarray(table)
            ok = (e >= 0) & (e < P)
            k, v = self.c.tokens(np.where(ok, e, 0))
            return k[:n], v[:n], np.repeat(ok, 64)[:n]
        for g in range(G):
            pk, pv, pok = held(self.ptable[g], plens[g])
            for b in range(starts[g], starts[g + 1]):
                n = int(max(lens[b], 0))
                qn = Mq if q_lens is None else min(max(int(q_lens[b]), 0), Mq)
                k, v, ok = held(self.table[b], n)
                for i in range(Mq):
                    if i < qn:
                        t = np.arange(len(k))
                        keep = ok & (t <= n - qn + i)
                        ref = C.prefix_row(q[b, i], (pk[pok], pv[pok]), (k[keep], v[keep]), int(keep.sum()),
                                           len(t), float(np.float32(SCALE)))
                    else:
                        ref = C.prefix_row(q[b, i], (pk[:0], pv[:0]), (k[:0], v[:0]), 0, 0, 1.0)
                    T.check_row(ref, o[b, i], st[b, i], wire, f"group {g} request {b} row {i}")
        return out, stat


@pytest.mark.parametrize("kv", T.KVS)
@pytest.mark.parametrize("H", [1, 16, 40, 128])
def test_one_group(kv, H):
    print(f"case: one group {kv} {H}", flush=True)
    Case(H, 3, 1, H, [0, 3], 9, 2, kv).check([550], [1, 64, 100])


@pytest.mark.parametrize("kv", T.KVS)
@pytest.mark.parametrize("wire", [False, True])
@pytest.mark.parametrize("row_tile", [64, 128])
def test_groups_of_any_size(kv, wire, row_tile):
    """Groups of none, one and several requests, whose rows end inside tiles; rows
    that see nothing but the prefix, nothing but their own, nothing at all."""
    print(f"case: groups {kv} {wire} {row_tile}", flush=True)
    a = Case(7, 9, 3, 11, [0, 0, 4, 5, 5, 9, 9], 4, 3, kv)
    args = [256, 100, 0, 7, 64, 1], [3, 192, 0, 77, 1, 0, 2, 130, 64], [3, 2, 0, 1, 3, 3, 1, 0, 2]
    if kv == "mx4" and row_tile == 128:
        with pytest.raises(mla.MlaError, match="64-row"):
            a.run(*args, wire=wire, row_tile=128)
        return
    a.check(*args, wire=wire, row_tile=row_tile)


@pytest.mark.parametrize("kv", ["bf16", "fp8", "fp8split"])
@pytest.mark.parametrize("B,Mq,H,starts", [(4, 1, 128, [0, 1, 4]), (3, 2, 128, [0, 0, 3]), (5, 1, 100, [0, 2, 5]),
                                           (2, 3, 64, [0, 1, 2]), (9, 1, 300, [0, 4, 9])])
def test_tiles_of_128_rows(kv, B, Mq, H, starts):
    print(f"case: 128 rows {kv} {B} {Mq} {H} {starts}", flush=True)
    a = Case(B + H, B, Mq, H, starts, 6, 3, kv)
    lens = np.random.default_rng(H).integers(0, 193, B)
    for n_splits, own_splits in ((0, 0), (1, 1), (5, 3)):
        a.check([384, 200], lens, row_tile=128, n_splits=n_splits, own_splits=own_splits)


@pytest.mark.parametrize("n_splits,own_splits", [(1, 1), (2, 1), (7, 3), (30, 30), (0, 2), (5, 0)])
@pytest.mark.parametrize("kv", ["bf16", "fp8", "mx4"])
def test_splits(kv, n_splits, own_splits):
    print(f"case: splits {kv} {n_splits} {own_splits}", flush=True)
    a = Case(3, 4, 2, 20, [0, 1, 4], 11, 5, kv)
    for row_tile in (64, 64 if kv == "mx4" else 128):
        a.check([700, 390], [320, 33, 200, 2], n_splits=n_splits, own_splits=own_splits, row_tile=row_tile)


@pytest.mark.parametrize("plen", [0, 1, 31, 32, 33, 63, 64, 65, 128])
def test_prefix_lengths(plen):
    a = Case(4, 2, 1, 16, [0, 2], 2, 1)
    a.check([plen], [1, 64])


@pytest.mark.parametrize("row_tile", [64, 128])
def test_tables_of_no_blocks(row_tile):
    """No prefix, or nothing of the requests' own: neither is read."""
    a = Case(17, 3, 2, 16, [0, 1, 3], 2, 2)
    a.table = a.table[:, :0]
    a.check([100, 128], [70, 2, 0], row_tile=row_tile)
    a = Case(18, 3, 2, 16, [0, 1, 3], 2, 2)
    a.ptable = a.ptable[:, :0]
    a.check([100, 128], [70, 2, 0], row_tile=row_tile)


def test_lengths_past_the_tables_and_below_zero():
    a = Case(5, 3, 2, 8, [0, 2, 3], 2, 1)
    a.check([1000, -7], [100, -3, 64], [2, 2, 5])


def test_starts_outside_the_batch():
    """The first group begins with the first request and the last ends with the
    last; starts in between are kept within the batch."""
    a = Case(6, 5, 1, 24, [3, 2, 99, -8], 3, 1)
    a.check([190, 100, 64], [1, 2, 3, 4, 64])


def test_table_entries_that_name_no_block():
    a = Case(8, 3, 1, 40, [0, 2, 3], 5, 3)
    a.ptable = a.ptable.copy()
    a.ptable[0, 2], a.ptable[1] = -1, 10 ** 6
    a.table = a.table.copy()
    a.table[1, 0], a.table[2] = 1 << 30, -1
    a.check([320, 300], [150, 192, 70])


def test_nothing_behind_the_sequences_is_read():
    a = Case(9, 2, 1, 16, [0, 2], 2, 2)
    a.c.ckv[a.ptable[0, 1], 20:] = float("nan")
    a.c.kpe[a.ptable[0, 1], 20:] = float("nan")
    a.c.ckv[a.table[0, 0], 5:] = float("inf")
    a.c.kpe[a.table[1, 1], 40:] = float("nan")
    out, _ = a.check([84], [5, 104])
    assert torch.isfinite(out).all()


def test_a_nan_in_the_prefix_reaches_its_group_only():
    a = Case(10, 4, 1, 16, [0, 2, 4], 2, 1)
    a.c.ckv[a.ptable[0, 0], 3, 7] = float("nan")
    out, lse = a.run([128, 128], [4, 4, 4, 4])
    torch.cuda.synchronize()
    assert torch.isnan(lse[:2]).all() and torch.isfinite(lse[2:]).all() and torch.isfinite(out[2:]).all()


def test_many_groups():
    """More groups than a wave has lanes, each of one request or none."""
    B = 150
    starts = np.sort(np.random.default_rng(0).integers(0, B + 1, 200)).tolist()
    starts[0], starts[-1] = 0, B
    a = Case(11, B, 1, 3, starts, 1, 1)
    a.check(np.random.default_rng(1).integers(0, 65, 199), np.random.default_rng(2).integers(0, 65, B))


def test_a_large_batch_and_long_prefix():
    a = Case(12, 33, 2, 64, [0, 20, 33], 40, 3)
    a.check([2560, 2222], np.random.default_rng(3).integers(2, 193, 33))


def test_merged_with_the_calls_that_it_joins():
    """The same sequences, prefix and own tokens in one table, by window_attn."""
    a = Case(13, 6, 1, 128, [0, 6], 8, 2)
    out, lse = a.run([512], [100, 3, 128, 64, 65, 1])
    table = np.concatenate([np.tile(a.ptable, (6, 1)), a.table], 1)
    ref, rl = mla.window_attn(*a.q, a.c.ckv, a.c.kpe, T.i32(table), T.i32(512 + np.array([100, 3, 128, 64, 65, 1])), SCALE)
    torch.cuda.synchronize()
    assert (lse - rl).abs().max() <= 1e-5 * (1 + rl.abs().max())
    # weights of either are rounded to bf16 against other maxima: 2^-8 each
    assert ((out - ref).abs().amax(-1) <= 2.0 ** -6 * ref.abs().amax(-1)).all()


def test_strides_and_given_outputs():
    a = Case(14, 4, 3, 16, [0, 1, 4], 3, 1)
    wide = torch.zeros((12, 20, 600), dtype=torch.bfloat16, device="cuda")
    wide = torch.zeros((4, 3, 20, 640), dtype=torch.bfloat16, device="cuda")
    wide[..., :16, :512], wide[..., :16, 512:576] = a.q
    out = torch.full((4, 3, 18, 512), 5.0, device="cuda")
    lse = torch.full((4, 3, 17), 5.0, device="cuda")
    got = a.run([190, 64], [9, 64, 3, 30], q=(wide[..., :16, :512], wide[..., :16, 512:576]), out_lat=out[:, :, :16],
                out_lse=lse[..., :16])
    a.check([190, 64], [9, 64, 3, 30], got=got)
    assert (out[:, :, 16:] == 5.0).all() and (lse[..., 16:] == 5.0).all()


def test_captured_and_replayed():
    a = Case(15, 5, 1, 32, [0, 2, 5], 6, 2)
    plens, lens = T.i32([384, 300]), T.i32([1, 2, 3, 4, 5])
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call = mla.prepare_prefix(*a.q, a.c.ckv, a.c.kpe, T.i32(a.ptable), plens, T.i32(a.starts), T.i32(a.table),
                                  lens, SCALE)
        call()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call()
        for k in range(4):
            rs = np.random.default_rng(k)
            n, m = rs.integers(0, 385, 2), rs.integers(1, 129, 5)
            plens.copy_(T.i32(n))
            lens.copy_(T.i32(m))
            g.replay()
            s.synchronize()
            a.check(n, m, got=call.result)
            s.synchronize()


def test_capture_without_a_workspace_is_refused():
    a = Case(16, 2, 1, 16, [0, 2], 2, 1)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        call = mla.prepare_prefix(*a.q, a.c.ckv, a.c.kpe, T.i32(a.ptable), T.i32([128]), T.i32(a.starts),
                                  T.i32(a.table), T.i32([1, 2]), SCALE)
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            torch.zeros(1, device="cuda")
            with pytest.raises(mla.MlaError, match="capture"):
                call()


def test_random_calls():
    rs = np.random.default_rng(99)
    for k in range(24):
        kv = T.KVS[k % 4]
        B, Mq, H = int(rs.integers(1, 9)), int(rs.integers(1, 4)), int(rs.choice([1, 5, 16, 33, 64]))
        G, NBP, NB = int(rs.integers(1, 5)), int(rs.integers(1, 9)), int(rs.integers(1, 4))
        starts = [0, *np.sort(rs.integers(0, B + 1, G - 1)).tolist(), B]
        print(f"case: random {k} {kv} {B} {Mq} {H} {starts} {NBP} {NB}", flush=True)
        a = Case(1000 + k, B, Mq, H, starts, NBP, NB, kv)
        a.check(rs.integers(0, 64 * NBP + 1, G), rs.integers(0, 64 * NB + 1, B),
                rs.integers(0, Mq + 1, B) if k % 2 else None, wire=bool(k % 3))
