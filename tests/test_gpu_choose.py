"""The choice of blocks on the GPU against the float64 references
(oracle/choose.py): the turned write into the cache, mean keys, scores, the K best,
and a run of them with the attention that reads the choice."""
import numpy as np
import pytest
import torch

from oracle import choose as C
from oracle import step as S
from paper_2606_01502_amd import mla
from tests import step_helpers as T

pytestmark = pytest.mark.gpu
SCALE = 0.0721688
F = float(np.float32(SCALE))


def sync():
    torch.cuda.synchronize()


# ---- rope_append: what rope and cache_append write
def pools(P, mx4, fill=7):
    ckv = torch.full((P, 64, 272), fill, dtype=torch.uint8, device="cuda") if mx4 else \
        torch.full((P, 64, 512), float(fill), dtype=torch.bfloat16, device="cuda")
    return ckv, torch.full((P, 64, 64), float(fill), dtype=torch.bfloat16, device="cuda")


YARN = dict(scaling="yarn", factor=40.0, orig_len=4096, mscale=1.2)


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("T_,rot", [(1, dict(pairing=0)), (2, dict(pairing=1)), (5, dict(pairing=0, **YARN)),
                                    (130, dict(pairing=1, scaling="linear", factor=8.0)),
                                    (67, dict(pairing=1, rot_offset=3, rot_dim=30)),
                                    (67, dict(pairing=0, rot_offset=1, rot_dim=2)),
                                    (4097, dict(pairing=0)), (5001, dict(pairing=1, **YARN))])
def test_rope_append_is_rope_and_append(mx4, T_, rot):
    print(f"case: rope_append {mx4} {T_} {rot}", flush=True)
    rs = np.random.default_rng(T_)
    P = T_ // 64 + 3
    new = T.randn(T_, T_, 576)
    pos = T.i32(rs.integers(-5, 163840, T_))
    at = rs.permutation(P * 64)[:T_]
    if T_ > 3:
        at[2], at[3] = -1, P * 64  # no place, and past the pool
    got = mla.rope_append(new[:, :512], new[:, 512:], pos, T.i32(at), *pools(P, mx4), **rot)
    turned = mla.rope(new[:, None, 512:], pos, **rot)[:, 0]
    want = mla.cache_append(new[:, :512], turned, T.i32(at), *pools(P, mx4))
    sync()
    assert torch.equal(got[0].view(torch.uint8), want[0].view(torch.uint8))
    # either kernel may fuse one of the two products with the sum: fp32 values 2^-23
    # (|x| + |y|) m apart, and where that crosses a border two neighbouring bf16 values
    g, w = got[1].float(), want[1].float()
    size = float(2 * new[:, 512:].abs().max()) * 1.2
    assert ((g - w).abs() <= 2.0 ** -7 * w.abs() + 2.0 ** -22 * size).all()
    assert (g != w).sum() <= 1 + T_ // 8  # (a border is met once in 2^14 values or so)


@pytest.mark.parametrize("pairing", [0, 1])
def test_rope_append_values(pairing):
    """Against the formula: products and their sum off by 2^-23 of |x| + |y|, cosines
    by 2^-20 at these positions, one rounding to bf16."""
    rs = np.random.default_rng(3)
    new, pos, at = T.randn(3, 300, 576), rs.integers(0, 1 << 20, 300), rs.permutation(6 * 64)[:300]
    _, kpe = mla.rope_append(new[:, :512], new[:, 512:], T.i32(pos), T.i32(at), *pools(6, False), pairing=pairing)
    got = T.host(kpe).reshape(-1, 64)[at]
    x = T.host(new)[:, None, 512:]
    want = S.rope(x, pos, 0, 64, pairing, 10000.0)[:, 0]
    size = np.sqrt(want ** 2 + S.rope(x, pos + 0, 0, 64, pairing, 10000.0)[:, 0] ** 2) + np.abs(x).max(-1)
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * size).all()


def test_rope_append_no_tokens():
    ckv, kpe = pools(1, False)
    mla.rope_append(torch.empty((0, 512), dtype=torch.bfloat16, device="cuda"),
                    torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), T.i32([]), T.i32([]), ckv, kpe)
    sync()
    assert (ckv == 7).all() and (kpe == 7).all()


# ---- block_means
def check_means(c, slots, extra=None):
    P = c.lat.shape[0]
    means = torch.full((P, 576), 5.0, dtype=torch.bfloat16, device="cuda")
    mla.block_means(c.ckv, c.kpe, T.i32(slots), means, **c.scales)
    sync()
    got = T.host(means)
    slots = np.asarray(slots, np.int64)
    ends = set((slots[(slots >= 0) & (slots < 64 * P) & (slots % 64 == 63)] // 64).tolist())
    keys = np.concatenate([c.lat, c.pe], -1)
    want, mag = C.means(keys), np.abs(keys).mean(1)
    for b in range(P):
        if b not in ends:
            assert (got[b] == 5.0).all(), f"block {b} was written"
            continue
        # 64 values and a scale in fp32, one rounding to bf16
        tol = 2.0 ** -8 * np.abs(want[b]) + 2.0 ** -17 * mag[b]
        assert (np.abs(got[b] - want[b]) <= tol).all(), f"block {b}"
    return means


@pytest.mark.parametrize("kv", T.KVS)
@pytest.mark.parametrize("what", ["one", "none", "list", "run", "twice"])
def test_means(kv, what):
    print(f"case: means {kv} {what}", flush=True)
    c = T.Cache(11, 9, kv)
    slots = {"one": [5 * 64 + 63], "none": [0, 62, 64, -1, 9 * 64 + 63, -63], "list": [b * 64 + 63 for b in range(9)],
             "run": np.arange(100, 400), "twice": [127, 127, 63, 127]}[what]
    check_means(c, slots)


def test_means_of_many_tokens():
    """More tokens than workgroups, in runs whose block ends lie 64 apart."""
    c = T.Cache(12, 130, "bf16")
    check_means(c, np.arange(130 * 64))
    check_means(c, np.tile(np.arange(130 * 64), 70))  # over 256 slots a workgroup


def test_means_keep_nan_and_infinity():
    c = T.Cache(13, 3, "bf16")
    c.ckv[1, 5, 7], c.kpe[1, 63, 0] = float("nan"), float("inf")
    means = torch.zeros((3, 576), dtype=torch.bfloat16, device="cuda")
    mla.block_means(c.ckv, c.kpe, T.i32([63, 127, 191]), means)
    sync()
    m = T.host(means)
    assert np.isnan(m[1, 7]) and np.isposinf(m[1, 512]) and np.isfinite(np.delete(m, [576 + 7, 576 + 512])).all()


# ---- block_scores
def scores_case(seed, B, Mq, H, NB, extra=3, sigma=0.5):
    P = B * NB + extra
    rs = np.random.default_rng(seed)
    return (T.randn(seed, B, Mq, H, 512), T.randn(seed + 1, B, Mq, H, 64), T.randn(seed + 2, P, 576, sigma=sigma),
            rs.permutation(P)[:B * NB].reshape(B, NB))


def check_scores(ql, qp, means, table, lens, window=0, n_sink=0, q_lens=None, scale=SCALE, **kw):
    got = mla.block_scores(ql, qp, means, T.i32(table), T.i32(lens), scale, window=window, n_sink=n_sink,
                           q_lens=None if q_lens is None else T.i32(q_lens), **kw)
    sync()
    g, m = T.host(got), T.host(means)
    q = np.concatenate([T.host(ql), T.host(qp)], -1)
    B, Mq, H, _ = q.shape
    for b in range(B):
        e = np.asarray(table[b])
        ok = (e >= 0) & (e < len(m))
        qn = Mq if q_lens is None else min(max(int(q_lens[b]), 0), Mq)
        want, mag = C.scores(q[b], m[np.where(ok, e, 0)], ok, int(lens[b]), qn, window, n_sink, float(np.float32(scale)))
        assert np.array_equal(np.isneginf(g[b]), np.isneginf(want)), f"b {b}: blocks that may be chosen"
        # logits off by 2^-18 of the sum of magnitudes (18 products of 32 in fp32, and
        # the scale), twice in a weight and its denominator; exponentials, the sums
        # over blocks and heads
        live = np.isfinite(want)
        tol = (4 * 2.0 ** -18 * mag[:, None] + 2.0 ** -18 + 2.0 ** -23 * (want.shape[1] + H)) * np.where(live, want, 0)
        err = np.abs(np.where(live, g[b], 0) - np.where(live, want, 0))
        assert (err <= tol + 1e-37).all(), f"b {b}: off by {(err / (tol + 1e-37)).max():.3g} x tolerance"
    return got


@pytest.mark.parametrize("H", [1, 5, 16, 33, 64, 128, 200])
@pytest.mark.parametrize("Mq,NB", [(1, 1), (1, 70), (3, 130), (17, 9)])
def test_scores(H, Mq, NB):
    print(f"case: scores {H} {Mq} {NB}", flush=True)
    a = scores_case(H + NB, 3, Mq, H, NB)
    check_scores(*a, [NB * 64, max(1, NB * 40), Mq])


@pytest.mark.parametrize("window,n_sink", [(1, 0), (64, 64), (65, 1), (300, 128), (4000, 0), (0, 5000)])
@pytest.mark.parametrize("n_splits", [0, 1, 2, 3])
def test_scores_windows_and_splits(window, n_sink, n_splits):
    print(f"case: scores {window} {n_sink} {n_splits}", flush=True)
    a = scores_case(5, 4, 2, 40, 150)
    check_scores(*a, [0, 64, 5001, 150 * 64], window=window, n_sink=n_sink, n_splits=n_splits)


def test_scores_padded_rows_and_odd_lengths():
    a = scores_case(6, 6, 5, 16, 20)
    check_scores(*a, [1280, 700, 3, -4, 1281, 5000], q_lens=[5, 3, 9, 2, 0, -1])
    # a table one entry of which names no block, and one none at all
    table = a[3].copy()
    table[0, 3], table[1], table[2, ::2] = -1, 10 ** 6, -5
    check_scores(*a[:3], table, [1280] * 6, n_splits=1)


def test_scores_strides_and_given_output():
    ql, qp, means, table = scores_case(7, 2, 3, 24, 40)
    wide = torch.zeros((2, 3, 24, 640), dtype=torch.bfloat16, device="cuda")
    wide[..., :512], wide[..., 512:576] = ql, qp
    tab = torch.full((2, 64), 99999, dtype=torch.int32, device="cuda")
    tab[:, :40] = T.i32(table)
    buf = torch.full((2, 3, 50), 3.0, device="cuda")
    mla.block_scores(wide[..., :512], wide[..., 512:576], means, tab[:, :40], T.i32([2560, 2000]), SCALE,
                     scores=buf[..., :40])
    want = check_scores(ql, qp, means, table, [2560, 2000])
    assert torch.equal(buf[..., :40], want) and (buf[..., 40:] == 3.0).all()


def test_scores_of_nan_and_infinity():
    ql, qp, means, table = scores_case(8, 3, 1, 20, 10)
    means[table[0, 4], 3] = float("nan")
    means[table[1, 9]] = float("nan")  # not whole yet: not looked at
    ql[2, 0, 3, 100] = float("nan")
    got = mla.block_scores(ql, qp, means, T.i32(table), T.i32([640, 639, 640]), SCALE)
    sync()
    g = T.host(got)
    assert np.isnan(g[0]).all() and np.isnan(g[2]).all() and np.isfinite(g[1, 0, :9]).all() and np.isneginf(g[1, 0, 9])


def test_scores_of_large_logits():
    """One block takes all of a head's weight, others none."""
    ql, qp, means, table = scores_case(9, 2, 1, 16, 70, sigma=40.0)
    check_scores(ql, qp, means, table, [70 * 64] * 2, scale=1.0)


def test_scores_of_no_pool_and_no_blocks():
    ql, qp, _, _ = scores_case(10, 2, 1, 16, 3)
    empty = torch.empty((0, 576), dtype=torch.bfloat16, device="cuda")
    got = mla.block_scores(ql, qp, empty, T.i32([[0, 1, 2], [3, 4, 5]]), T.i32([192, 192]), SCALE)
    assert torch.isneginf(got).all()
    none = torch.empty((2, 0), dtype=torch.int32, device="cuda")
    assert mla.block_scores(ql, qp, empty, none, T.i32([192, 192]), SCALE).shape == (2, 1, 0)


# ---- select_topk
def check_topk(x, K, **kw):
    got = mla.select_topk(x, K, **kw).cpu().numpy().reshape(-1, K)
    rows = x.cpu().numpy().reshape(-1, x.shape[-1])
    for r in range(len(rows)):
        assert got[r].tolist() == C.topk(rows[r], K), f"row {r}"


@pytest.mark.parametrize("N", [1, 2, 63, 64, 65, 255, 256, 257, 1000, 1024, 1025, 2048, 2049, 5000, 16384, 16385])
@pytest.mark.parametrize("how", ["random", "ties", "holes"])
def test_topk(N, how):
    print(f"case: topk {N} {how}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(N)
    x = torch.randn((3, 2, N), generator=g, device="cuda")
    if how == "ties":
        x = torch.round(x * 2) / 2  # (-0 and 0 among them)
    if how == "holes":
        x[torch.rand(x.shape, generator=g, device="cuda") < 0.6] = -float("inf")
        x[0, 0] = -float("inf")
    for K in sorted({1, 2, max(1, N // 3), N, N + 5}):
        if K <= 6000:
            check_topk(x, K)


@pytest.mark.parametrize("N", [200, 1500, 20000])
def test_topk_of_extremes(N):
    rs = np.random.default_rng(N)
    pool = np.array([np.nan, -np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-45, -1e-45, 3.4e38, -3.4028235e38, 1.0], np.float32)
    x = torch.from_numpy(pool[rs.integers(0, len(pool), (4, N))]).cuda()
    for K in (1, N // 4, N // 2, N):
        check_topk(x, K)


@pytest.mark.parametrize("N", [100, 3000, 40000])
def test_topk_all_equal_and_sorted(N):
    up = torch.arange(N, device="cuda", dtype=torch.float32)
    for x in (torch.zeros((2, N), device="cuda"), up[None], up.flip(0)[None], -up[None]):
        check_topk(x, 7)
        check_topk(x, N // 2)


@pytest.mark.parametrize("N,K", [(16385, 100), (30000, 1), (65536, 2048), (65537, 5), (70001, 2048), (100003, 3000),
                                 (100003, 40000), (300000, 500), (1 << 20, 2048)])
@pytest.mark.parametrize("how", ["random", "ties", "holes"])
def test_topk_of_long_rows(N, K, how):
    """Rows that go in pieces, once and twice, and those that do not."""
    print(f"case: topk {N} {K} {how}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(N + K)
    x = torch.rand((2, 2, N), generator=g, device="cuda")
    if how == "ties":
        x = torch.round(x * 30)
    if how == "holes":
        x[0, 0, 9000:] = -float("inf")
        x[0, 1] = -float("inf")
        x[1, 0, :17000] = -float("inf")
    got = mla.select_topk(x, K)
    v, at = torch.sort(x, dim=-1, descending=True, stable=True)
    at = torch.where(v[..., :K] == -float("inf"), N, at[..., :K])
    want = torch.sort(at, dim=-1).values
    assert torch.equal(got.long(), torch.where(want == N, -1, want))


def test_topk_of_long_rows_captured_without_a_workspace():
    x = torch.rand((3, 70000), device="cuda")
    s = torch.cuda.Stream()
    sync()
    with torch.cuda.stream(s):
        call = mla.prepare_select_topk(x, 64)
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call()
        for _ in range(3):
            x.uniform_()
            g.replay()
            s.synchronize()
            ids = call.result.clone()
            assert torch.equal(ids, mla.select_topk(x, 64))
            s.synchronize()


def test_topk_of_more_rows_than_a_launch_holds():
    """2^21 rows a launch: the rows on either side of the border and the last ones."""
    n = (1 << 21) + 1000
    x = torch.rand((n, 6), device="cuda")
    got = mla.select_topk(x, 2)
    want = torch.sort(torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :2], dim=-1).values
    assert torch.equal(got.long(), want)


def test_topk_strided_rows_and_given_ids():
    x = torch.randn((3, 5, 90), device="cuda")
    ids = torch.full((3, 5, 20), 9, dtype=torch.int32, device="cuda")
    mla.select_topk(x[:, ::2, 10:80], ids=ids[:, ::2, 4:12])
    want = mla.select_topk(x[:, ::2, 10:80].contiguous(), 8)
    sync()
    assert torch.equal(ids[:, ::2, 4:12], want)
    assert (ids[:, 1::2] == 9).all() and (ids[..., :4] == 9).all() and (ids[..., 12:] == 9).all()
    one = torch.randn(300, device="cuda").expand(4, 300)  # a row given four times
    check_topk(one, 11)


def test_topk_empty():
    assert mla.select_topk(torch.empty((0, 5), device="cuda"), 3).shape == (0, 3)
    assert mla.select_topk(torch.randn((2, 5), device="cuda"), 0).shape == (2, 0)
    assert (mla.select_topk(torch.empty((2, 0), device="cuda"), 3) == -1).all()


def test_topk_more_rows_than_a_wave_of_workgroups():
    x = torch.randn((9000, 70), device="cuda")
    got = mla.select_topk(x, 5)
    want = torch.sort(torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :5], -1).values
    assert torch.equal(got.long(), want)


# ---- a run of them, as a step uses them
@pytest.mark.parametrize("kv", ["bf16", "mx4"])
def test_step_over_chosen_blocks(kv):
    """Prompt tokens into the cache, mean keys, scores and choice of a decode step's
    rows, attention over the choice and the rest, joined: with every block chosen
    that is attention over all of the sequence, with fewer that over the choice."""
    B, H, NB, W = 3, 32, 12, 100
    lens = np.array([700, 64, 331])
    c, table, ql, qp, means = step_inputs(kv, B, H, NB, lens)
    for k in (NB, 3):
        sc = mla.block_scores(ql, qp, means, T.i32(table), T.i32(lens), SCALE, window=W, n_sink=64)
        ids = mla.select_topk(sc, k)
        part = mla.sparse_partial_attn(ql, qp, c[0], c[1], T.i32(table), ids[:, 0].contiguous(), SCALE)
        near = mla.window_attn(ql, qp, c[0], c[1], T.i32(table), T.i32(lens), SCALE, window=W, n_sink=64,
                               whole_blocks=True)
        out, lse = mla.merge_partials([part[0], near[0]], [part[1], near[1]], out_lse=True)
        sync()
        check_chosen(kv, c, table, lens, ql, qp, ids.cpu().numpy(), W, 64, out, lse)
    full = mla.window_attn(ql, qp, c[0], c[1], T.i32(table), T.i32(lens), SCALE)
    sc = mla.block_scores(ql, qp, means, T.i32(table), T.i32(lens), SCALE, window=W, n_sink=64)
    n = np.isfinite(T.host(sc)).sum(-1)[:, 0]
    assert n.tolist() == [8, 0, 2]
    assert full[0].shape == out.shape


def step_inputs(kv, B, H, NB, lens):
    P = B * NB
    table = np.random.default_rng(4).permutation(P).reshape(B, NB)
    ckv, kpe = pools(P, kv == "mx4", fill=0)
    slots = np.concatenate([table[b, np.arange(n) // 64] * 64 + np.arange(n) % 64 for b, n in enumerate(lens)])
    pos = np.concatenate([np.arange(n) for n in lens])
    new = T.randn(40, len(slots), 576, sigma=0.7)
    mla.rope_append(new[:, :512], new[:, 512:], T.i32(pos), T.i32(slots), ckv, kpe, pairing=1)
    means = torch.zeros((P, 576), dtype=torch.bfloat16, device="cuda")
    mla.block_means(ckv, kpe, T.i32(slots), means)
    return (ckv, kpe), table, T.randn(41, B, 1, H, 512), T.randn(42, B, 1, H, 64), means


def check_chosen(kv, c, table, lens, ql, qp, ids, window, n_sink, out, lse):
    lat = S.mx4_decode(c[0].cpu().numpy()) if kv == "mx4" else T.host(c[0])
    pe = T.host(c[1])
    q = np.concatenate([T.host(ql), T.host(qp)], -1)
    o, st = T.host(out), T.host(lse)
    for b, n in enumerate(lens):
        e = table[b]
        keys = np.concatenate([lat[e].reshape(-1, 512), pe[e].reshape(-1, 64)], 1)
        t = np.arange(len(keys))
        p = n - 1
        see = (t <= p) & ((t >= 64 * C.end_block(p, window)) | (t < n_sink))
        for j in ids[b, 0]:
            if j >= 0:
                assert not see[64 * j:64 * j + 64].any(), "chosen and attended anyway"
                see[64 * j:64 * j + 64] = True
        T.check_row(S.attend(q[b, 0], keys, keys[:, :512], see, F), o[b, 0], st[b, 0], False, f"b {b}")


def test_windows_of_whole_blocks():
    c = T.Cache(21, 30, "bf16")
    table = np.random.default_rng(2).permutation(30).reshape(2, 15)
    for Mq, window, n_sink in ((1, 1, 0), (1, 64, 0), (3, 65, 10), (9, 130, 64), (2, 2000, 3), (40, 7, 0)):
        ql, qp = T.randn(Mq, 2, Mq, 16, 512), T.randn(Mq + 1, 2, Mq, 16, 64)
        lens = [960, 517]
        out, lse = mla.window_attn(ql, qp, c.ckv, c.kpe, T.i32(table), T.i32(lens), SCALE, window=window,
                                   n_sink=n_sink, whole_blocks=True)
        sync()
        q, o, st = np.concatenate([T.host(ql), T.host(qp)], -1), T.host(out), T.host(lse)
        for b in range(2):
            keys, values = c.tokens(table[b])
            t = np.arange(len(keys))
            for i in range(Mq):
                p = lens[b] - Mq + i
                see = (t <= p) & ((t >= 64 * C.end_block(p, window)) | (t < n_sink))
                T.check_row(S.attend(q[b, i], keys, values, see, F), o[b, i], st[b, i], False, f"{window} {b} {i}")


def test_step_captured_and_replayed():
    """The choice captured into a graph, replayed over new queries and lengths."""
    B, H, NB = 4, 64, 140
    ql, qp, means, table = scores_case(50, B, 1, H, NB)
    tab, lens = T.i32(table), T.i32([NB * 64] * B)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call = mla.prepare_block_scores(ql, qp, means, tab, lens, SCALE, window=64)
        pick = mla.prepare_select_topk(call(), 9)
        pick()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call()
            pick()
        for k in range(4):
            ql.copy_(T.randn(60 + k, B, 1, H, 512))
            lens.copy_(T.i32(np.random.default_rng(k).integers(1, NB * 64, B)))
            g.replay()
            s.synchronize()
            ids, sc = pick.result.clone(), call.result.clone()
            assert torch.equal(mla.block_scores(ql, qp, means, tab, lens, SCALE, window=64), sc)
            assert torch.equal(mla.select_topk(sc, 9), ids)
            s.synchronize()


def test_scores_captured_without_a_workspace():
    """On a stream whose workspace cannot grow the call takes one split."""
    ql, qp, means, table = scores_case(51, 1, 1, 16, 300)
    s = torch.cuda.Stream()
    sync()
    with torch.cuda.stream(s):
        out = torch.empty((1, 1, 300), device="cuda")
        call = mla.prepare_block_scores(ql, qp, means, T.i32(table), T.i32([300 * 64]), SCALE, scores=out)
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call()
        for _ in range(3):
            out.zero_()
            g.replay()
            s.synchronize()
            want = mla.block_scores(ql, qp, means, T.i32(table), T.i32([300 * 64]), SCALE, n_splits=1)
            s.synchronize()
            assert torch.equal(out, want)


def test_two_streams_at_once():
    cases = [scores_case(70 + k, 2, 1, 128, 200) for k in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    lens = T.i32([200 * 64, 9000])
    want = [mla.block_scores(a[0], a[1], a[2], T.i32(a[3]), lens, SCALE) for a in cases]
    tabs = [T.i32(a[3]) for a in cases]
    sync()
    got = [[], []]
    for _ in range(10):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(mla.block_scores(*cases[k][:3], tabs[k], lens, SCALE))
    sync()
    for k in range(2):
        assert all(torch.equal(x, want[k]) for x in got[k])
