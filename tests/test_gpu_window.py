"""Window attention on the GPU against the float64 reference (oracle/step.py):
every cache type, both tile forms, windows and sinks around block and half
block borders, ragged and padded batches, empty rows, what lies behind a
sequence, invalid table entries, splits, strides, graphs."""
import numpy as np
import pytest
import torch

from oracle import step as S
from paper_2606_01502_amd import mla
from tests import step_helpers as T

pytestmark = pytest.mark.gpu
SCALE = 0.0721688


def run(c, q_lat, q_pe, table, lens, q_lens=None, window=0, n_sink=0, wire=False, scale=SCALE, **kw):
    out, stat = mla.window_attn(q_lat, q_pe, c.ckv, c.kpe, T.i32(table), T.i32(lens), scale,
                                window=window, n_sink=n_sink,
                                q_lens=None if q_lens is None else T.i32(q_lens), wire=wire,
                                **c.scales, **kw)
    torch.cuda.synchronize()
    return out, stat


def check(c, q_lat, q_pe, table, lens, q_lens=None, window=0, n_sink=0, wire=False, scale=SCALE, rows=None, **kw):
    out, stat = run(c, q_lat, q_pe, table, lens, q_lens, window, n_sink, wire, scale, **kw)
    B, Mq, H, _ = q_lat.shape
    o, st = T.host(out), T.host(stat)
    ql = np.concatenate([T.host(q_lat), T.host(q_pe)], -1)
    P = c.lat.shape[0]
    s32 = float(np.float32(scale))
    for b in range(B):
        n, qn = int(lens[b]), Mq if q_lens is None else min(max(int(q_lens[b]), 0), Mq)
        nb = min(-(-max(n, 0) // 64), len(table[b]))
        entries = np.asarray(table[b][:nb])
        ok = (entries >= 0) & (entries < P)
        keys, values = c.tokens(np.where(ok, entries, 0))
        held = np.repeat(ok, 64)
        for i in (range(Mq) if rows is None else rows):
            see = S.visible(nb * 64, n - qn + i if i < qn else -1, window, n_sink) & held
            T.check_row(S.attend(ql[b, i], keys, values, see, s32), o[b, i], st[b, i], wire, f"b {b} row {i}")
    return out, stat


def inputs(seed, B, Mq, H, NB, kv, extra=3):
    c = T.Cache(seed, B * NB + extra, kv)
    table = np.random.default_rng(seed).permutation(B * NB + extra)[:B * NB].reshape(B, NB)
    return c, T.randn(seed, B, Mq, H, 512), T.randn(seed + 1, B, Mq, H, 64), table


@pytest.mark.parametrize("kv", T.KVS)
@pytest.mark.parametrize("H", [1, 16, 40, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 4)])
def test_decode(kv, H, window, sinks):
    print(f"case: decode {kv} {H} {window} {sinks}", flush=True)
    c, ql, qp, table = inputs(H, 3, 1, H, 7, kv)
    check(c, ql, qp, table, [1, 200, 448], window=window, n_sink=sinks)


@pytest.mark.parametrize("kv", T.KVS)
@pytest.mark.parametrize("wire", [False, True])
def test_rows_of_a_prompt(kv, wire):
    print(f"case: prompt {kv} {wire}", flush=True)
    c, ql, qp, table = inputs(11, 2, 37, 5, 6, kv)
    check(c, ql, qp, table, [37, 300], window=50, n_sink=3, wire=wire)
    check(c, ql, qp, table, [37, 300], wire=wire)


@pytest.mark.parametrize("kv", ["bf16", "mx4"])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 95, 96, 97, 128, 129, 160, 255])
def test_lengths(kv, n):
    """Every number of stages, and ends inside them."""
    print(f"case: length {kv} {n}", flush=True)
    c, ql, qp, table = inputs(n, 1, 2, 20, 4, kv)
    check(c, ql, qp, table, [n])
    check(c, ql, qp, table, [n], n_splits=3)


@pytest.mark.parametrize("kv", T.KVS)
@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 64, 65, 127, 250, 400, 2 ** 31 - 1])
@pytest.mark.parametrize("sinks", [0, 1, 32, 33, 64, 100, 2 ** 31 - 1])
def test_windows_and_sinks(kv, window, sinks):
    print(f"case: window {kv} {window} {sinks}", flush=True)
    c, ql, qp, table = inputs(3, 2, 3, 8, 6, kv)
    check(c, ql, qp, table, [70, 383], window=window, n_sink=sinks)


@pytest.mark.parametrize("kv", T.KVS)
def test_ragged_batch(kv):
    """Padding rows, no rows at all, lengths of 0, more rows than tokens,
    lengths past the table, negative ones."""
    print(f"case: ragged {kv}", flush=True)
    lens = [100, 5, 0, 64, 256, 400, -3, 130, 9]
    q_lens = [9, 7, 3, 0, 1, 9, 4, 20, -1]
    c, ql, qp, table = inputs(8, len(lens), 9, 12, 4, kv)
    for window, sinks in ((0, 0), (40, 5), (200, 70)):
        check(c, ql, qp, table, lens, q_lens, window=window, n_sink=sinks)
    check(c, ql, qp, table, lens, q_lens, window=40, n_sink=5, wire=True, n_splits=2)
    out, lse = run(c, ql, qp, table, [0] * 9, window=4)
    assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("kv", T.KVS)
def test_behind_the_sequence_and_padding_hold_anything(kv):
    """NaN and infinities behind the last token, in blocks a window has let go
    of and in padding rows' queries change nothing."""
    print(f"case: garbage {kv}", flush=True)
    c, ql, qp, table = inputs(21, 3, 6, 11, 4, kv)
    lens, q_lens = [71, 256, 130], [6, 2, 4]
    kw = dict(window=60, n_sink=2)
    want = run(c, ql, qp, table, lens, q_lens, **kw)
    nan_rows = {"bf16": torch.nan, "mx4": 255, "fp8": 0x7F, "fp8split": 0xFF}[kv]
    for b in range(3):
        for t in range(lens[b], 256):
            c.ckv[table[b, t // 64], t % 64] = nan_rows
            c.kpe[table[b, t // 64], t % 64] = torch.inf if c.kpe.dtype == torch.bfloat16 else 0x7F
        ql[b, q_lens[b]:] = torch.nan
        qp[b, q_lens[b]:] = torch.inf
    got = run(c, ql, qp, table, lens, q_lens, **kw)
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    # the blocks between the sinks and the window may be gone from the table, or
    # be another's
    t2 = table.copy()
    t2[1, 1], t2[1, 2] = -1, 10 ** 6
    got = run(c, ql, qp, t2, lens, q_lens, **kw)
    for a, b in zip(want, got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("kv", ["bf16", "fp8split", "mx4"])
def test_table_entries_that_name_no_block_are_left_out(kv):
    print(f"case: bad entries {kv}", flush=True)
    c, ql, qp, table = inputs(31, 2, 2, 24, 8, kv)
    table = table.copy()
    table[0, 2], table[0, 7], table[1, 0], table[1, 5] = -1, c.lat.shape[0], -(2 ** 31), 2 ** 31 - 1
    check(c, ql, qp, table, [512, 480])
    check(c, ql, qp, table, [512, 480], window=150, n_sink=70, n_splits=2)
    none = np.full_like(table, -1)
    out, lse = run(c, ql, qp, none, [512, 480])
    assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("kv", T.KVS)
@pytest.mark.parametrize("splits", [1, 2, 3, 7, 50])
def test_splits(kv, splits):
    print(f"case: splits {kv} {splits}", flush=True)
    c, ql, qp, table = inputs(41, 2, 2, 70, 12, kv)
    check(c, ql, qp, table, [700, 129], window=500, n_sink=10, n_splits=splits)
    check(c, ql, qp, table, [700, 129], n_splits=splits, wire=True)


@pytest.mark.parametrize("kv", ["bf16", "mx4"])
def test_long_sequences_over_several_lists(kv):
    """More half blocks than one split's list holds, in one split asked for."""
    print(f"case: long {kv}", flush=True)
    c, ql, qp, table = inputs(51, 1, 2, 3, 600, kv)
    check(c, ql, qp, table, [600 * 64 - 13], n_splits=1)
    check(c, ql, qp, table, [600 * 64 - 13], window=20000, n_sink=9000, n_splits=1)


@pytest.mark.parametrize("kv", T.KVS)
def test_many_tiles(kv):
    """A prompt of many tiles whose windows overlap, checked at rows throughout."""
    print(f"case: many tiles {kv}", flush=True)
    c, ql, qp, table = inputs(61, 1, 400, 16, 12, kv)
    check(c, ql, qp, table, [700], window=129, n_sink=4, rows=range(0, 400, 23))
    check(c, ql, qp, table, [400], rows=range(0, 400, 37))


@pytest.mark.parametrize("scale", [0.0, -0.5, 30.0])
@pytest.mark.parametrize("kv", ["bf16", "mx4"])
def test_scales(kv, scale):
    print(f"case: scale {kv} {scale}", flush=True)
    c, ql, qp, table = inputs(71, 2, 2, 16, 5, kv)
    check(c, ql, qp, table, [300, 77], window=100, n_sink=4, scale=scale)


def test_strided_rows_and_views():
    """Query and output rows inside larger tensors, a table view of a wider one."""
    print("case: strides", flush=True)
    c, ql, qp, table = inputs(81, 2, 3, 10, 5, "bf16")
    joined = torch.cat([ql, qp], -1)
    wide = T.i32(np.concatenate([table, table[:, :3]], 1))
    big = torch.full((2, 3, 12, 520), 7.0, device="cuda")
    lse = torch.full((3, 2, 10), 7.0, device="cuda").transpose(0, 1)
    want = run(c, ql, qp, table, [300, 64], window=70)
    mla.window_attn(joined[..., :512], joined[..., 512:], c.ckv, c.kpe, wide[:, :5], T.i32([300, 64]), SCALE,
                    window=70, out_lat=big[:, :, 1:11, :512], out_lse=lse)
    torch.cuda.synchronize()
    assert torch.equal(big[:, :, 1:11, :512], want[0]) and torch.equal(lse, want[1])
    assert (big[:, :, 0] == 7).all() and (big[:, :, 11] == 7).all() and (big[..., 512:] == 7).all()


def test_merges_with_selected_blocks():
    """A window's partial and the partial of blocks before it merge to attention
    over both (the window's part beside a sparse selection)."""
    print("case: merge", flush=True)
    for kv in ("bf16", "mx4"):
        c, ql, qp, table = inputs(91, 2, 1, 16, 10, kv)
        lens, window = [640, 640], 128  # the last two blocks
        sel = np.array([[0, 3, 7], [1, 2, -1]])
        a = run(c, ql, qp, table, lens, window=window)
        b = mla.sparse_partial_attn(ql, qp, c.ckv, c.kpe, T.i32(table), T.i32(sel), SCALE)
        out, lse = mla.merge_partials([a[0], b[0]], [a[1], b[1]], out_lse=True)
        torch.cuda.synchronize()
        q = np.concatenate([T.host(ql), T.host(qp)], -1)
        for r in range(2):
            blocks = [s for s in sel[r] if s >= 0] + [8, 9]
            keys, values = c.tokens(table[r, blocks])
            ref = S.attend(q[r, 0], keys, values, np.ones(len(keys), bool), float(np.float32(SCALE)))
            T.check_row(ref, T.host(out)[r, 0], T.host(lse)[r, 0], False, f"{kv} {r}")


def test_captured_and_replayed():
    """Lengths, tables and tokens change between replays; eager work between them."""
    print("case: graph", flush=True)
    for kv in ("bf16", "mx4"):
        c, ql, qp, table = inputs(101, 4, 2, 24, 20, kv)
        d_table, lens, q_lens = T.i32(table), T.i32([1280] * 4), T.i32([2] * 4)
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            call = mla.prepare_window(ql, qp, c.ckv, c.kpe, d_table, lens, SCALE, window=300, n_sink=4,
                                      q_lens=q_lens, **c.scales)
            call()
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            got = call()
        for seed in range(4):
            rs = np.random.default_rng(seed)
            lens.copy_(T.i32(rs.integers(0, 1281, 4)))
            q_lens.copy_(T.i32(rs.integers(0, 3, 4)))
            d_table.copy_(T.i32(rs.permutation(80).reshape(4, 20)))
            ql.copy_(T.randn(seed, *ql.shape))
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                g.replay()
            side.synchronize()
            want = mla.window_attn(ql, qp, c.ckv, c.kpe, d_table, lens, SCALE, window=300, n_sink=4,
                                   q_lens=q_lens, **c.scales)
            torch.cuda.synchronize()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            del want


def test_no_rows():
    c, ql, qp, table = inputs(111, 2, 3, 4, 2, "bf16")
    out, _ = run(c, ql[:0], qp[:0], table[:0], [])
    assert out.shape == (0, 3, 4, 512)
    out, _ = run(c, ql[:, :0], qp[:, :0], table, [5, 6])
    assert out.shape == (2, 0, 4, 512)
    out, lse = run(c, ql, qp, table[:, :0], [5, 6])  # a table of no blocks
    assert (out == 0).all() and torch.isneginf(lse).all()


# ---------------------------------------------------------------- both tiles
@pytest.mark.parametrize("tile", [64, 128])
@pytest.mark.parametrize("kv", ["bf16", "fp8", "fp8split"])
def test_both_tiles(kv, tile):
    """128-row tiles take whole blocks, 64-row tiles half blocks: windows, sinks
    and ends around both, ragged rows, splits."""
    print(f"case: tiles {kv} {tile}", flush=True)
    c, ql, qp, table = inputs(121, 3, 9, 40, 7, kv)
    lens, q_lens = [440, 60, 129], [9, 3, 7]
    for window, sinks in ((0, 0), (1, 0), (33, 1), (64, 64), (65, 33), (300, 70), (2 ** 31 - 1, 2 ** 31 - 1)):
        check(c, ql, qp, table, lens, q_lens, window=window, n_sink=sinks, row_tile=tile)
    check(c, ql, qp, table, lens, q_lens, window=200, n_sink=4, row_tile=tile, n_splits=3, wire=True)
    check(c, ql, qp, table, lens, row_tile=tile, wire=True)


@pytest.mark.parametrize("n", [1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 193, 256])
@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_lengths_in_128_row_tiles(kv, n):
    print(f"case: length 128 {kv} {n}", flush=True)
    c, ql, qp, table = inputs(n, 1, 2, 70, 4, kv)
    check(c, ql, qp, table, [n], row_tile=128)
    check(c, ql, qp, table, [n], row_tile=128, n_splits=3)


@pytest.mark.parametrize("kv", ["bf16", "fp8", "fp8split"])
def test_garbage_in_128_row_tiles(kv):
    """What lies behind a sequence, in padding rows and in blocks a window has let
    go of, in 128-row tiles."""
    print(f"case: garbage 128 {kv}", flush=True)
    c, ql, qp, table = inputs(131, 3, 6, 30, 4, kv)
    lens, q_lens = [71, 256, 130], [6, 2, 4]
    kw = dict(window=60, n_sink=2, row_tile=128)
    want = run(c, ql, qp, table, lens, q_lens, **kw)
    check(c, ql, qp, table, lens, q_lens, **kw)
    for b in range(3):
        for t in range(lens[b], 256):
            c.ckv[table[b, t // 64], t % 64] = {"bf16": torch.nan, "fp8": 0x7F, "fp8split": 0xFF}[kv]
            c.kpe[table[b, t // 64], t % 64] = torch.inf if kv == "bf16" else 0x7F
        ql[b, q_lens[b]:] = torch.nan
        qp[b, q_lens[b]:] = torch.inf
    t2 = table.copy()
    t2[1, 1], t2[1, 2] = -1, 10 ** 6
    for tab in (table, t2):
        got = run(c, ql, qp, tab, lens, q_lens, **kw)
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    bad = table.copy()
    bad[0, 1], bad[2, 0] = -1, c.lat.shape[0]
    got = run(c, ql, qp, bad, lens, q_lens, row_tile=128)
    assert torch.isfinite(got[0]).all()


@pytest.mark.parametrize("kv", ["bf16", "fp8split"])
def test_long_and_many_tiles_of_128_rows(kv):
    print(f"case: long 128 {kv}", flush=True)
    c, ql, qp, table = inputs(141, 1, 2, 65, 600, kv)
    check(c, ql, qp, table, [600 * 64 - 13], n_splits=1, row_tile=128)
    c, ql, qp, table = inputs(142, 1, 300, 16, 10, kv)
    check(c, ql, qp, table, [600], window=129, n_sink=4, rows=range(0, 300, 17), row_tile=128)
    check(c, ql, qp, table, [300], rows=range(0, 300, 29), row_tile=128)


def pooled(seed, B, Mq, H, NB, P, kv):
    """Requests whose tables draw on one small pool."""
    c = T.Cache(seed, P, kv)
    table = np.random.default_rng(seed).integers(0, P, (B, NB))
    return c, T.randn(seed, B, Mq, H, 512), T.randn(seed + 1, B, Mq, H, 64), table


@pytest.mark.parametrize("kv", T.KVS)
@pytest.mark.parametrize("B,Mq,H,NB,longest", [(40, 1, 16, 48, 48 * 64), (64, 1, 128, 16, 1024), (2, 1, 16, 600, 600 * 64),
                                               (64, 2, 64, 300, 300 * 64), (63, 3, 24, 64, 64 * 64), (17, 1, 130, 90, 90 * 64)])
@pytest.mark.parametrize("spread", ["one long", "any", "alike"])
def test_splits_shared_by_length(kv, B, Mq, H, NB, longest, spread):
    """Automatic plans over requests of unlike lengths: none, one token, the whole table."""
    print(f"case: shares {kv} {B} {Mq} {H} {NB} {spread}", flush=True)
    rs = np.random.default_rng([B, NB])
    lens = {"one long": rs.integers(0, 200, B), "any": rs.integers(0, min(longest, 3000), B),
            "alike": np.full(B, min(longest, 1000))}[spread]
    if spread != "alike":
        lens[B // 2] = longest
        lens[0], lens[-1] = (0, 1) if B > 2 else (70, longest)
    q_lens = rs.integers(0, Mq + 1, B) if Mq > 1 else None
    if q_lens is not None:
        q_lens[B // 2] = Mq
    c, ql, qp, table = pooled(B, B, Mq, H, NB, 37, kv)
    table[1, :2] = -1
    check(c, ql, qp, table, lens, q_lens, rows=[0, Mq - 1], wire=spread == "any")
    if spread == "one long":  # (a window of more than half the table, with sinks)
        check(c, ql, qp, table, lens, q_lens, rows=[0, Mq - 1], window=40 * NB + 7, n_sink=33)


@pytest.mark.parametrize("kv", ["bf16", "mx4"])
def test_shared_splits_follow_the_lengths_of_a_replay(kv):
    print(f"case: shares replayed {kv}", flush=True)
    B, H, NB = 40, 16, 48
    c, ql, qp, table = pooled(4, B, 1, H, NB, 37, kv)
    tab, lens = T.i32(table), T.i32(np.full(B, 900))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        f = mla.prepare_window(ql, qp, c.ckv, c.kpe, tab, lens, SCALE, **c.scales)
        f()  # (the workspace grows outside of the capture)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        out, lse = f()
    for seed in range(4):
        new = np.random.default_rng(seed).integers(0, NB * 64 + 1, B) // (1 if seed & 1 else np.arange(1, B + 1))
        lens.copy_(T.i32(new))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        side.synchronize()
        got, got_lse = out.clone(), lse.clone()
        eager, eager_lse = check(c, ql, qp, table, new)
        assert torch.equal(got, eager) and torch.equal(got_lse, eager_lse)


@pytest.mark.parametrize("kv", ["bf16", "fp8", "mx4"])
@pytest.mark.parametrize("B,H,NB", [(65, 16, 130), (128, 128, 130), (129, 24, 140), (193, 8, 128), (256, 5, 256), (257, 8, 130)])
def test_splits_shared_in_large_batches(kv, B, H, NB):
    """Several requests a lane, the last lanes without any; more than are shared between."""
    print(f"case: shares, large batch {kv} {B} {H} {NB}", flush=True)
    rs = np.random.default_rng([B, NB])
    lens = rs.integers(0, 150, B)
    lens[rs.integers(0, B, 3)] = NB * 64 - 5
    lens[rs.integers(0, B, 9)] = rs.integers(0, 3000, 9)
    lens[-1] = 777
    c, ql, qp, table = pooled(B, B, 1, H, NB, 37, kv)
    check(c, ql, qp, table, lens, wire=B % 2 == 0)
