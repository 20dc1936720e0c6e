"""A serving step's way into the paged cache on the GPU against the references
of oracle/step.py: tables and slots (integers, equal), rotary positions, the
write of new tokens into bf16 and 4-bit pools and the 4-bit read-back (equal
bit for bit: the quantisation is exact arithmetic on bf16 values)."""
import numpy as np
import pytest
import torch

from oracle import step as S
from paper_2606_01502_amd import mla

pytestmark = pytest.mark.gpu


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def randn(seed, *shape, dtype=torch.bfloat16, sigma=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * sigma).to(dtype).cuda()


# ---------------------------------------------------------------- slots
def _slots_case(seed, B, NB, F, T, most=200):
    rs = np.random.default_rng(seed)
    cached = rs.integers(0, most, B)
    new = rs.integers(0, most, B) * (rs.random(B) < 0.8)
    perm = rs.permutation(B * NB + F + 1)
    table = np.full((B, NB), -7, np.int64)
    for b in range(B):
        h = min(-(-int(cached[b]) // 64), NB)
        table[b, :h] = perm[b * NB:b * NB + h]
    return cached, new, perm[B * NB:B * NB + F], table


def _check_slots(cached, new, free, table, T, strided=False):
    d_table = i32(table)
    if strided:
        wide = torch.full((table.shape[0], table.shape[1] + 5), -9, dtype=torch.int32, device="cuda")
        wide[:, :table.shape[1]] = d_table
        d_table = wide[:, :table.shape[1]]
    got = mla.batch_slots(i32(cached), i32(new), i32(free), d_table, n_tokens=T)
    torch.cuda.synchronize()
    want = S.batch_slots(cached, new, free, table, T)
    for name, g, w in zip((*mla.SlotPlan._fields, "table"), (*got, d_table), want):
        assert np.array_equal(g.cpu().numpy(), w), name
    if strided:
        assert (wide[:, table.shape[1]:] == -9).all()


@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 511, 513, 1500])
def test_slots_match(B):
    print(f"case: slots B={B}", flush=True)
    c, n, f, t = _slots_case(B, B, 7, 4 * B, 0)
    _check_slots(c, n, f, t, int(n.sum()))


@pytest.mark.parametrize("what", ["few free", "no free", "table full", "T short", "T long", "T zero", "strided",
                                  "negative lengths", "no new", "bad entries", "block borders"])
def test_slots_edges(what):
    print(f"case: slots {what}", flush=True)
    c, n, f, t = _slots_case(7, 40, 5, 100, 0)
    T = int(n.sum())
    if what == "few free":
        f = f[:13]
    if what == "no free":
        f = f[:0]
    if what == "table full":
        n = n + 200
        T = int(n.sum())
    if what == "T short":
        T -= 77
    if what == "T long":
        T += 3000
    if what == "T zero":
        T = 0
    if what == "negative lengths":
        n[3], n[9], c[5] = -4, -(2 ** 31), -1
        t[5] = -7
        T = int(np.maximum(n, 0).sum())
    if what == "no new":
        n[:] = 0
        T = 5
    if what == "bad entries":
        t[t >= 0] = np.where(np.arange((t >= 0).sum()) % 3 == 0, 2 ** 25, t[t >= 0])
    if what == "block borders":
        c = np.arange(40) % 3 * 64
        n = np.arange(40) // 3 % 3 * 64
        t[:, :2] = np.arange(80).reshape(40, 2)
        T = int(n.sum())
    _check_slots(c, n, f, t, T, strided=what == "strided")


def test_slots_most_requests():
    print("case: slots 8192", flush=True)
    rs = np.random.default_rng(3)
    c, n = rs.integers(0, 70, 8192), rs.integers(0, 3, 8192)
    t = np.full((8192, 3), -1)
    t[:, 0], t[:, 1] = np.arange(8192), np.where(c > 64, 8192 + np.arange(8192), -1)
    t[c == 0, 0] = -1
    _check_slots(c, n, np.arange(20000, 30000), t, int(n.sum()))


def test_slots_no_requests():
    _check_slots(np.zeros(0, int), np.zeros(0, int), np.arange(3), np.zeros((0, 4), int), 10)


def test_slots_many_tokens_over_workgroups():
    """One request of most tokens and many of none, over several workgroups."""
    print("case: slots 50000 tokens", flush=True)
    c, n = np.full(300, 130), np.zeros(300, int)
    n[5], n[200], n[299] = 40001, 3, 9999
    t = np.full((300, 700), -1)
    t[:, :3] = np.arange(900).reshape(300, 3)
    _check_slots(c, n, np.arange(900, 1900), t, int(n.sum()))


def test_slots_huge_lengths_are_cut_at_the_table():
    """Lengths whose sums pass 2^31: offsets saturate, and nothing past the
    table or the outputs is touched."""
    print("case: slots huge", flush=True)
    big = 2 ** 31 - 1
    cached, new = i32([5, big, 7]), i32([big, big, big])
    table, free = i32([[3, -1], [4, 5], [6, -1]]), i32([10, 11, 12])
    got = mla.batch_slots(cached, new, free, table, n_tokens=200)
    torch.cuda.synchronize()
    pos = 5 + np.arange(200)
    blk = np.where(pos < 64, 3, 10)
    assert np.array_equal(got.slots.cpu(), np.where(pos < 128, blk * 64 + pos % 64, -1))
    assert np.array_equal(got.positions.cpu(), pos)
    assert table.cpu().tolist() == [[3, 10], [4, 5], [6, 11]]
    assert got.seq_lens.cpu().tolist() == [big, big, big]
    assert got.starts.cpu().tolist() == [0, big, big, big]
    assert got.info.cpu().tolist() == [big, 2, 0, big - 200]


# ---------------------------------------------------------------- rope
SCALINGS = [dict(), dict(scaling="linear", factor=4.0),
            dict(scaling="yarn", factor=40.0, orig_len=4096, mscale=1.25)]


def _check_rope(x, pos, at, rot, pairing, inverse=False, out=None, base=1e4, **kw):
    got = mla.rope(x, i32(pos), out=out, rot_offset=at, rot_dim=rot, pairing=pairing, base=base,
                   inverse=inverse, **kw)
    torch.cuda.synchronize()
    ref = S.rope(x_host(x), pos, at, rot, pairing, base, inverse=inverse, **kw)
    _close(got, ref, x_host(x), at, rot, pairing, kw.get("mscale", 1.0))
    return got


def x_host(x):
    return x.detach().double().cpu().numpy()


def _close(got, ref, x, at, rot, pairing, m):
    """Copied values equal; rotated ones within half a step of the type and the
    fp32 arithmetic: angle (2^-25 of a turn's reduced part), sine and cosine,
    two products and a sum, together under 2^-20 (|x| + |y|) m."""
    g = x_host(got)
    keep = np.r_[0:at, at + rot:x.shape[-1]]
    assert np.array_equal(g[..., keep], x[..., keep])
    h = rot // 2
    i = np.arange(at, at + rot, 2) if pairing == 0 else np.arange(at, at + h)
    j = i + 1 if pairing == 0 else i + h
    mag = (np.abs(x[..., i]) + np.abs(x[..., j])) * abs(m)
    half = torch.finfo(got.dtype).eps / 2
    for k in (i, j):
        tol = half * np.abs(ref[..., k]) * 1.01 + 2.0 ** -20 * mag + 1e-37
        assert (np.abs(g[..., k] - ref[..., k]) <= tol).all(), np.max(np.abs(g[..., k] - ref[..., k]) / tol)


@pytest.mark.parametrize("scaling", range(3))
@pytest.mark.parametrize("pairing", [0, 1])
@pytest.mark.parametrize("T,H,D,at,rot", [(1, 1, 64, 0, 64), (5, 128, 192, 128, 64), (67, 3, 80, 16, 32),
                                          (700, 1, 64, 0, 64), (33, 16, 256, 0, 256), (9, 7, 40, 8, 16)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rope_matches(T, H, D, at, rot, pairing, scaling, dtype):
    print(f"case: rope {T} {H} {D} {at} {rot} {pairing} {scaling} {dtype}", flush=True)
    rs = np.random.default_rng(T + H)
    _check_rope(randn(T * 3 + H, T, H, D, dtype=dtype), rs.integers(0, 200000, T), at, rot, pairing,
                **SCALINGS[scaling])


@pytest.mark.parametrize("pairing", [0, 1])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rope_odd_layouts(pairing, dtype):
    """Sizes and strides that no 16-byte access fits."""
    print(f"case: rope odd {pairing} {dtype}", flush=True)
    _check_rope(randn(1, 13, 5, 37, dtype=dtype), np.arange(13) * 999, 3, 22, pairing)
    _check_rope(randn(2, 6, 2, 2, dtype=dtype), np.arange(6), 0, 2, pairing)
    base = randn(3, 11, 6, 70, dtype=dtype)
    _check_rope(base[1:, 1::2, 3:67], np.arange(10) * 7, 0, 64, pairing)          # unaligned base
    wide = randn(4, 11, 6, 72, dtype=dtype)
    _check_rope(wide[::2, :, 8:], np.arange(6) * 7, 0, 64, pairing)               # aligned, strided
    _check_rope(wide.transpose(0, 1), np.arange(6) * 31, 8, 64, pairing)
    _check_rope(wide[:1].expand(4, 6, 72), np.arange(4) * 31, 8, 64, pairing)     # one row under all positions


@pytest.mark.parametrize("pairing", [0, 1])
def test_rope_far_and_negative_positions(pairing):
    print(f"case: rope far {pairing}", flush=True)
    pos = np.array([2 ** 31 - 1, -(2 ** 31), -1, 0, 2 ** 24 + 1, 10 ** 9 + 7])
    _check_rope(randn(5, 6, 2, 64, dtype=torch.float32), pos, 0, 64, pairing)
    _check_rope(randn(5, 6, 2, 64, dtype=torch.float32), pos, 0, 64, pairing, base=5e5,
                scaling="linear", factor=3.0)


@pytest.mark.parametrize("pairing,aligned", [(0, True), (1, True), (0, False), (1, False)])
def test_rope_in_place_and_into_a_view(pairing, aligned):
    print(f"case: rope in place {pairing} {aligned}", flush=True)
    w = 72 if aligned else 71
    base = randn(6, 9, 4, w)
    x = base[..., :w - 8]
    before, edge = x.clone(), base[..., w - 8:].clone()
    pos = np.arange(9) * 100
    want = mla.rope(before, i32(pos), pairing=pairing, rot_offset=w - 8 - 32, rot_dim=32)
    got = mla.rope(x, i32(pos), out=x, pairing=pairing, rot_offset=w - 8 - 32, rot_dim=32)
    torch.cuda.synchronize()
    assert got.data_ptr() == x.data_ptr() and torch.equal(x, want) and torch.equal(base[..., w - 8:], edge)


@pytest.mark.parametrize("pairing", [0, 1])
def test_rope_inverse_is_the_gradient(pairing):
    """inverse is the map's transpose: against the reference, against <y, g> =
    <x, rope^T g>, and against differences of the map itself."""
    print(f"case: rope inverse {pairing}", flush=True)
    kw = dict(scaling="yarn", factor=40.0, orig_len=4096, mscale=1.25)
    T, H, D = 17, 3, 96
    x, g = randn(7, T, H, D, dtype=torch.float32), randn(8, T, H, D, dtype=torch.float32)
    pos = np.random.default_rng(1).integers(0, 10 ** 6, T)
    gx = _check_rope(g, pos, 32, 64, pairing, inverse=True, **kw)
    y = mla.rope(x, i32(pos), rot_offset=32, rot_dim=64, pairing=pairing, **kw)
    a, b = (y.double() * g.double()).sum(), (x.double() * gx.double()).sum()
    scale = (y.double().abs() * g.double().abs()).sum()
    assert abs(a - b) <= 2.0 ** -19 * scale
    # the map is linear: a difference over any step is its gradient
    for t, h, d in ((0, 0, 32), (3, 1, 95), (16, 2, 64), (5, 0, 7)):
        dx = torch.zeros_like(x)
        dx[t, h, d] = 1.0
        up = mla.rope(x + dx, i32(pos), rot_offset=32, rot_dim=64, pairing=pairing, **kw)
        dn = mla.rope(x - dx, i32(pos), rot_offset=32, rot_dim=64, pairing=pairing, **kw)
        num = ((up.double() - dn.double()) / 2 * g.double()).sum()
        tol = 2.0 ** -19 * float((up.double().abs()[t, h] * g.double().abs()[t, h]).sum())
        assert abs(num - gx[t, h, d].double()) <= tol


def test_rope_no_rows():
    for T, H in ((0, 4), (4, 0)):
        assert mla.rope(randn(9, T, H, 64), i32(np.zeros(T))).shape == (T, H, 64)


# ---------------------------------------------------------------- append, gather
def _bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def _append_case(seed, T, P, mx4, skip=0.2):
    rs = np.random.default_rng(seed)
    slots = rs.permutation(P * 64)[:T].astype(np.int64)
    slots[rs.random(T) < skip] = -1
    if T > 3:
        slots[1], slots[2] = P * 64, -5
    ckv, kpe = randn(seed, T, 512, sigma=0.5), randn(seed + 1, T, 64)
    pool = torch.from_numpy(rs.integers(0, 250, (P, 64, 272)).astype(np.uint8)).cuda() if mx4 else \
        randn(seed + 2, P, 64, 512)
    return slots, ckv, kpe, pool, randn(seed + 3, P, 64, 64)


def _check_append(slots, ckv, kpe, pool, kpool):
    mx4 = pool.dtype == torch.uint8
    want, kwant = pool.cpu().clone(), kpool.cpu().clone()
    ok = (slots >= 0) & (slots < pool.shape[0] * 64)
    rows = torch.from_numpy(S.mx4_encode(x_host(ckv))) if mx4 else ckv.cpu()
    want.view(-1, want.shape[-1])[torch.from_numpy(slots[ok])] = rows[torch.from_numpy(ok)]
    kwant.view(-1, 64)[torch.from_numpy(slots[ok])] = kpe.cpu()[torch.from_numpy(ok)]
    got = mla.cache_append(ckv, kpe, i32(slots), pool, kpool)
    torch.cuda.synchronize()
    assert got[0] is pool and got[1] is kpool
    assert np.array_equal(_bits(kpool), _bits(kwant))
    if not mx4:
        assert np.array_equal(_bits(pool), _bits(want))
        return
    g, w = pool.cpu().numpy().reshape(-1, 272), want.numpy().reshape(-1, 272)
    nan = np.repeat(w[:, 256:] == 255, 16, axis=1)  # whose codes mean nothing
    assert np.array_equal(g[:, 256:], w[:, 256:])
    assert np.array_equal(np.where(nan, 0, g[:, :256]), np.where(nan, 0, w[:, :256]))


@pytest.mark.parametrize("mx4", [False, True])
@pytest.mark.parametrize("T,P", [(1, 1), (3, 2), (64, 3), (333, 8), (4096, 70), (4097, 70), (4102, 70)])
def test_append_matches_bit_for_bit(T, P, mx4):
    print(f"case: append {T} {P} {mx4}", flush=True)
    _check_append(*_append_case(T, T, P, mx4))


def test_append_strided_rows_and_no_tokens():
    print("case: append strided", flush=True)
    slots, ckv, kpe, pool, kpool = _append_case(5, 50, 4, True)
    joined = torch.cat([ckv, kpe], -1)  # a projection's joint output
    _check_append(slots, joined[:, :512], joined[:, 512:], pool, kpool)
    _check_append(slots, ckv[:1].expand(50, 512), kpe, pool, kpool)
    _check_append(slots[:0], ckv[:0], kpe[:0], pool, kpool)


def test_append_every_bf16_value():
    """Every finite bf16 bit pattern, beside others of its own magnitude and
    beside the largest of a group at random, subnormal numbers and signed zeros
    among them; then groups with an infinity or a NaN."""
    print("case: append all bf16", flush=True)
    bits = np.arange(65536, dtype=np.uint32).astype(np.uint16)
    bits = bits[(bits & 0x7F80) != 0x7F80]
    rs = np.random.default_rng(3)
    a = np.sort(bits & 0x7FFF)[:len(bits) // 512 * 512] | (rs.integers(0, 2, len(bits) // 512 * 512) << 15).astype(np.uint16)
    b = rs.permutation(bits)[:len(bits) // 512 * 512]
    near = rs.integers(0, 0x7F80 - 0x400, (600, 1)) + rs.integers(0, 0x400, (600, 512))
    near = near.astype(np.uint16) | (rs.integers(0, 2, (600, 512)) << 15).astype(np.uint16)
    x = np.concatenate([a.reshape(-1, 512), b.reshape(-1, 512), near])
    extra = x[:40].copy()
    extra[np.arange(40), rs.integers(0, 512, 40)] = np.resize([0x7F80, 0xFF80, 0x7FC0, 0xFFFF], 40)
    x = np.concatenate([x, extra])
    T = len(x)
    ckv = torch.from_numpy(x.view(np.int16)).view(torch.bfloat16).cuda()
    pool = torch.zeros((T // 64 + 1, 64, 272), dtype=torch.uint8, device="cuda")
    kpool = torch.zeros((T // 64 + 1, 64, 64), dtype=torch.bfloat16, device="cuda")
    with np.errstate(invalid="ignore"):
        _check_append(np.arange(T), ckv, randn(1, T, 64), pool, kpool)


def test_gather_of_4bit_rows_is_exact():
    """Every code under every exponent the writer uses, in every column: codes
    times a power of two, equal to the reference in bf16 bit for bit."""
    print("case: gather 4 bits", flush=True)
    rs = np.random.default_rng(4)
    L, P, NB = 2, 9, 7
    pool = rs.integers(0, 256, (L, P, 64, 272)).astype(np.uint8)
    pool[..., 256:] = rs.integers(2, 253, (L, P, 64, 16))
    pool[0, 0, :, 256:] = 255  # NaN
    kpe = randn(5, L, P, 64, 64)
    table = rs.permutation(P)[:NB]
    table[3] = P + 4
    sel = rs.integers(0, NB * 64, 333)
    sel[[4, 7, 9]] = [-1, NB * 64, -9]
    oc, ok = mla.fetch_gather(torch.from_numpy(pool).cuda(), kpe, i32(table), i32(sel))
    torch.cuda.synchronize()
    live = (sel >= 0) & (sel < NB * 64)
    blk = table[np.where(live, sel, 0) // 64]
    live &= blk < P
    at = (np.where(live, blk, 0), np.where(live, sel, 0) % 64)
    want = S.mx4_decode(pool[:, at[0], at[1]]) * live[None, :, None]
    want = np.where(live[None, :, None], want, 0.0)
    got = oc.float().cpu().numpy().astype(np.float64)
    assert np.array_equal(got, want, equal_nan=True)
    assert np.array_equal(_bits(ok), np.where(live[None, :, None], _bits(kpe)[:, at[0], at[1]], 0))


def test_pools_past_4_gib():
    """The last blocks of pools of more than 4 GiB, written, read back and attended."""
    print("case: large pools", flush=True)
    P, n = 262000, 150
    far = np.array([P - 1, P - 70000, P - 2])
    slots = (far[:, None] * 64 + np.arange(64)).reshape(-1)[:n]
    ckv, kpe = randn(1, n, 512, sigma=0.5), randn(2, n, 64)
    q = randn(3, 1, 2, 24, 576)
    for kv in ("mx4", "bf16"):
        row, dt = (272, torch.uint8) if kv == "mx4" else (512, torch.bfloat16)
        got = []
        for blocks, at in ((P, slots), (3, np.arange(n))):
            pool = torch.empty((blocks, 64, row), dtype=dt, device="cuda")
            kpool = torch.empty((blocks, 64, 64), dtype=torch.bfloat16, device="cuda")
            mla.cache_append(ckv, kpe, i32(at), pool, kpool)
            table = far if blocks == P else np.arange(3)
            back = mla.fetch_gather(pool[None], kpool[None], i32(table), i32(np.arange(n)))
            args = (q[..., :512], q[..., 512:], pool, kpool, i32(table[None]))
            outs = [mla.window_attn(*args, i32([n]), 0.07, window=100, n_sink=2)]
            outs += [mla.sparse_partial_attn(*args, i32([[0, 1]]), 0.07, row_tile=64)]
            outs += [mla.sparse_partial_attn(*args, i32(np.arange(n)[None]), 0.07, tokens=True, row_tile=64)]
            if kv == "bf16":
                outs += [mla.window_attn(*args, i32([n]), 0.07, window=100, n_sink=2, row_tile=128)]
            got.append([x.clone() for o in [back, *outs] for x in o])
            del pool, kpool
            torch.cuda.empty_cache()
        for a, b in zip(*got):
            assert torch.equal(a, b)
        assert torch.isfinite(got[0][2]).all()


# ---------------------------------------------------------------- streams, graphs
def test_step_captured_and_replayed():
    """Slots, rotation and append of a step in one graph, replayed with new
    lengths and tokens between eager work; every replay against eager calls."""
    print("case: step graph", flush=True)
    B, NB, P, H = 6, 4, 40, 3
    cached, new = i32(np.zeros(B)), i32(np.zeros(B))
    table, free = i32(np.zeros((B, NB))), i32(np.arange(P))
    T = 200
    q, k = randn(1, T, H, 64), randn(2, T, 1, 64)
    ckv = randn(3, T, 512)
    pool = torch.zeros((P, 64, 272), dtype=torch.uint8, device="cuda")
    kpool = torch.zeros((P, 64, 64), dtype=torch.bfloat16, device="cuda")

    def step(pool, kpool, table):
        plan = mla.batch_slots(cached, new, free, table, n_tokens=T)
        qr, kr = mla.rope(q, plan.positions), mla.rope(k, plan.positions)
        mla.cache_append(ckv, kr[:, 0], plan.slots, pool, kpool)
        return plan, qr

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(pool, kpool, table)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        plan, qr = step(pool, kpool, table)
    for seed in range(4):
        rs = np.random.default_rng(seed)
        c, n = rs.integers(0, 90, B), rs.integers(0, 33, B)
        t0 = np.full((B, NB), -1)
        t0[:, :2] = rs.permutation(B * 2).reshape(B, 2)
        cached.copy_(i32(c))
        new.copy_(i32(n))
        free.copy_(i32(rs.permutation(np.arange(12, 12 + P))[:P] % P))
        table.copy_(i32(t0))
        q.copy_(randn(10 + seed, T, H, 64))
        ckv.copy_(randn(20 + seed, T, 512))
        pool.zero_()
        kpool.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        side.synchronize()
        e_pool, e_kpool, e_table = torch.zeros_like(pool), torch.zeros_like(kpool), i32(t0)
        e_plan, e_qr = step(e_pool, e_kpool, e_table)
        torch.cuda.synchronize()
        for a, b in zip((*plan, qr, table, pool, kpool), (*e_plan, e_qr, e_table, e_pool, e_kpool)):
            assert torch.equal(a, b)


def test_step_on_a_stream_of_its_own():
    """Calls take the current stream: work queued there first is seen."""
    print("case: step stream", flush=True)
    s = torch.cuda.Stream()
    x = torch.zeros((4096, 16, 64), dtype=torch.bfloat16, device="cuda")
    fill = randn(1, 4096, 16, 64)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(20):
            x.copy_(fill)
        y = mla.rope(x, i32(np.arange(4096)))
    s.synchronize()
    assert torch.equal(y, mla.rope(fill, i32(np.arange(4096))))
