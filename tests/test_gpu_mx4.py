"""Partial attention over 4-bit caches (MXFP4 latents, bf16 RoPE rows) on the
GPU: against the float64 reference on the values that the codes stand for, and
as one piece of a serving step with the calls that fill the cache."""
import numpy as np
import pytest
import torch

from oracle import step as S
from paper_2606_01502_amd import mla
from tests import step_helpers as T

pytestmark = pytest.mark.gpu
SCALE = 0.0721688


def check(c, q_lat, q_pe, table, sel, wire=False, scale=SCALE, **kw):
    out, stat = mla.sparse_partial_attn(q_lat, q_pe, c.ckv, c.kpe, T.i32(table), T.i32(sel), scale, wire=wire, **kw)
    torch.cuda.synchronize()
    o, st = T.host(out), T.host(stat)
    q = np.concatenate([T.host(q_lat), T.host(q_pe)], -1)
    P = c.lat.shape[0]
    for r in range(len(table)):
        ids = [int(s) for s in sel[r] if 0 <= s < len(table[r])]
        blocks = [int(table[r][s]) for s in ids if 0 <= table[r][s] < P]
        keys, values = c.tokens(blocks)
        rq = r % q_lat.shape[0]
        for i in range(q_lat.shape[1]):
            ref = S.attend(q[rq, i], keys, values, np.ones(len(keys), bool), float(np.float32(scale)))
            T.check_row(ref, o[r, i], st[r, i], wire, f"job {r} row {i}")
    return out, stat


def inputs(seed, R, Mq, H, NB, K, Rq=None):
    c = T.Cache(seed, R * NB + 2, "mx4")
    rs = np.random.default_rng(seed)
    table = rs.permutation(R * NB + 2)[:R * NB].reshape(R, NB)
    sel = np.stack([rs.permutation(NB)[:K] for _ in range(R)])
    sel[rs.random(sel.shape) < 0.15] = -1
    Rq = Rq or R
    return c, T.randn(seed, Rq, Mq, H, 512), T.randn(seed + 1, Rq, Mq, H, 64), table, sel


@pytest.mark.parametrize("wire", [False, True])
@pytest.mark.parametrize("R,Mq,H,NB,K", [(1, 1, 16, 4, 2), (1, 1, 128, 20, 12), (3, 2, 16, 9, 5), (2, 3, 40, 30, 17),
                                         (1, 1, 1, 3, 1), (2, 1, 33, 40, 40), (40, 1, 8, 5, 3)])
def test_matches(R, Mq, H, NB, K, wire):
    print(f"case: mx4 {R} {Mq} {H} {NB} {K} {wire}", flush=True)
    check(*inputs(R + H, R, Mq, H, NB, K), wire=wire)


@pytest.mark.parametrize("splits", [1, 2, 5])
@pytest.mark.parametrize("H", [16, 64])
def test_splits_and_slots(splits, H):
    """Empty, repeated and invalid slots, entries past the pool, q shared by jobs."""
    print(f"case: mx4 slots {splits} {H}", flush=True)
    c, ql, qp, table, sel = inputs(5, 4, 2, H, 12, 9, Rq=2)
    sel[0] = -1
    sel[1] = [3, 3, 3, 12, -7, 2 ** 30, 0, 1, 2]
    table = table.copy()
    table[2, 4] = c.lat.shape[0]
    table[3, :] = -1
    check(c, ql, qp, table, sel, n_splits=splits)


def test_agrees_with_a_bf16_cache_of_the_same_values():
    """The values are exact in bf16: a bf16 pool that holds them gives the same
    partials but for the order of the scores' sums (columns are summed in another
    order) and what the roundings of the weights make of it."""
    print("case: mx4 as bf16", flush=True)
    for H, Mq in ((16, 1), (64, 2)):
        c, ql, qp, table, sel = inputs(7, 3, Mq, H, 20, 14)
        check(c, ql, qp, table, sel, n_splits=2)
        c.ckv = torch.from_numpy(c.lat).bfloat16().cuda()
        assert np.array_equal(T.host(c.ckv), c.lat)
        check(c, ql, qp, table, sel, n_splits=2, row_tile=64)


def test_every_exponent_the_writer_uses():
    """Scores and values far from 1: rows of small exponents beside a large one."""
    print("case: mx4 exponents", flush=True)
    c, ql, qp, table, sel = inputs(9, 1, 1, 16, 4, 4)
    rs = np.random.default_rng(1)
    rows = c.ckv.cpu().numpy()
    rows[..., 256:] = rs.integers(2, 127, rows[..., 256:].shape)
    c.ckv, c.lat = torch.from_numpy(rows).cuda(), S.mx4_decode(rows)
    check(c, ql, qp, table, sel)


def test_a_group_that_is_nan():
    """Exponent byte 255: every row that attends the token is NaN, whatever the
    codes and the scores; jobs without it are not touched."""
    print("case: mx4 nan", flush=True)
    for H in (16, 64):
        c, ql, qp, table, sel = inputs(17, 2, 1, H, 6, 4)
        sel[:] = [[0, 1, 2, 3], [2, 3, 4, 5]]
        want, _ = mla.sparse_partial_attn(ql, qp, c.ckv, c.kpe, T.i32(table), T.i32(sel), SCALE)
        c.ckv[table[0, 2], 40, 256 + 7] = 255
        c.ckv[table[0, 2], 40, :256] = 0
        out, _ = mla.sparse_partial_attn(ql, qp, c.ckv, c.kpe, T.i32(table), T.i32(sel), SCALE)
        torch.cuda.synchronize()
        assert torch.isnan(out[0, ..., 224:256]).all() and torch.equal(out[1], want[1])


@pytest.mark.parametrize("no_alloc", [False, True])
def test_entry_points(no_alloc):
    print(f"case: mx4 entry {no_alloc}", flush=True)
    check(*inputs(13, 2, 1, 128, 30, 25), no_alloc=no_alloc)


@pytest.mark.parametrize("wire", [False, True])
@pytest.mark.parametrize("R,Mq,H,NB,K", [(1, 1, 16, 4, 1), (2, 1, 128, 9, 200), (3, 2, 16, 9, 33), (2, 3, 40, 30, 97),
                                         (1, 1, 1, 3, 64), (2, 1, 33, 60, 1500), (9, 1, 8, 5, 31), (1, 2, 32, 40, 2048)])
def test_token_selections(R, Mq, H, NB, K, wire):
    print(f"case: mx4 tokens {R} {Mq} {H} {NB} {K} {wire}", flush=True)
    c = T.Cache(R + H, R * NB + 2, "mx4")
    rs = np.random.default_rng(K)
    table = rs.permutation(R * NB + 2)[:R * NB].reshape(R, NB)
    sel = rs.integers(0, NB * 64, (R, K))  # (repeats among them)
    sel[rs.random(sel.shape) < 0.1] = -1
    if K > 3:
        sel[0, :2] = NB * 64, -9
        table = table.copy()
        table[-1, 0] = c.lat.shape[0] + 5
    ql, qp = T.randn(K, R, Mq, H, 512), T.randn(K + 1, R, Mq, H, 64)
    for kw in (dict(), dict(n_splits=3)):
        out, stat = mla.sparse_partial_attn(ql, qp, c.ckv, c.kpe, T.i32(table), T.i32(sel), SCALE, wire=wire,
                                            tokens=True, **kw)
        torch.cuda.synchronize()
        q = np.concatenate([T.host(ql), T.host(qp)], -1)
        for r in range(R):
            ids = sel[r][(sel[r] >= 0) & (sel[r] < NB * 64)]
            ids = ids[table[r][ids // 64] < c.lat.shape[0]]
            b, t = table[r][ids // 64], ids % 64
            keys = np.concatenate([c.lat[b, t], c.pe[b, t]], -1)
            for i in range(Mq):
                ref = S.attend(q[r, i], keys, c.lat[b, t], np.ones(len(ids), bool), float(np.float32(SCALE)))
                T.check_row(ref, T.host(out)[r, i], T.host(stat)[r, i], wire, f"job {r} row {i}")


def test_refused_forms():
    c, ql, qp, table, sel = inputs(15, 2, 2, 16, 6, 4)
    args = (ql, qp, c.ckv, c.kpe, T.i32(table))
    for kw, s in ((dict(row_tile=128), sel), (dict(row_tile=128, tokens=True), sel), (dict(), np.stack([sel, sel], 1))):
        with pytest.raises(mla.MlaError) as e:
            mla.sparse_partial_attn(*args, T.i32(s), SCALE, **kw)
        assert e.value.status == mla.MLA_ERR_UNSUPPORTED
    with pytest.raises(mla.MlaError) as e:
        mla.sparse_partial_attn(ql, qp, c.ckv, c.kpe.view(torch.uint8)[..., :64].contiguous(), T.i32(table),
                                T.i32(sel), SCALE)
    assert e.value.status == mla.MLA_ERR_INVALID_ARGUMENT


@pytest.mark.parametrize("kv", ["bf16", "mx4"])
def test_a_serving_step(kv):
    """Prompts, then decode steps, of a batch: tables and slots, rotation of
    queries and keys, the write into the cache, window attention with sinks; every
    step against float64 attention over the tokens written so far (as the cache
    holds them: the keys' rotation rounded to bf16, latents in the cache's type)."""
    print(f"case: step {kv}", flush=True)
    B, H, NB, P, window, sinks = 3, 6, 5, 17, 70, 5
    rs = np.random.default_rng(2)
    pool = torch.zeros((P, 64, 272), dtype=torch.uint8, device="cuda") if kv == "mx4" else \
        torch.full((P, 64, 512), torch.nan, dtype=torch.bfloat16, device="cuda")
    if kv == "mx4":
        pool.fill_(255)
    kpool = torch.full((P, 64, 64), torch.nan, dtype=torch.bfloat16, device="cuda")
    table = torch.full((B, NB), -1, dtype=torch.int32, device="cuda")
    free = T.i32(rs.permutation(P))
    cached = np.zeros(B, int)
    past = [np.zeros((0, 576)) for _ in range(B)]
    for step, new in enumerate([[100, 1, 64], [1, 1, 1], [3, 2, 1], [1, 0, 1], [40, 64, 2]]):
        new = np.array(new)
        total, most = int(new.sum()), int(new.max())
        ckv, kpe = T.randn(10 * step, total, 512, sigma=0.5), T.randn(10 * step + 1, total, 64)
        q = T.randn(10 * step + 2, total, H, 576)
        plan = mla.batch_slots(T.i32(cached), T.i32(new), free, table, n_tokens=total + 5)
        pos = plan.positions[:total]
        kr = mla.rope(kpe[:, None], pos)[:, 0]
        qr = mla.rope(q, pos, rot_offset=512)
        mla.cache_append(ckv, kr, plan.slots[:total], pool, kpool)
        starts = plan.starts.cpu().numpy()
        padded = torch.full((B, most, H, 576), torch.nan, dtype=torch.bfloat16, device="cuda")
        for b in range(B):
            padded[b, :new[b]] = qr[starts[b]:starts[b] + new[b]]
        out, lse = mla.window_attn(padded[..., :512], padded[..., 512:], pool, kpool, table, plan.seq_lens,
                                   SCALE, window=window, n_sink=sinks, q_lens=T.i32(new))
        torch.cuda.synchronize()
        assert plan.info.cpu().tolist()[2:] == [0, 0]
        free = free[int(plan.info[1]):].contiguous()
        lat = T.host(ckv) if kv == "bf16" else S.mx4_decode(S.mx4_encode(T.host(ckv)))
        for b in range(B):
            mine = slice(starts[b], starts[b] + new[b])
            past[b] = np.concatenate([past[b], np.concatenate([lat[mine], T.host(kr)[mine]], 1)])
            n = len(past[b])
            assert n == cached[b] + new[b]
            for i in range(most):
                see = S.visible(n, n - new[b] + i if i < new[b] else -1, window, sinks)
                row = T.host(padded)[b, i] if i < new[b] else np.zeros((H, 576))
                ref = S.attend(row, past[b], past[b][:, :512], see, float(np.float32(SCALE)))
                T.check_row(ref, T.host(out)[b, i], T.host(lse)[b, i], False, f"step {step} b {b} row {i}")
        cached += new
