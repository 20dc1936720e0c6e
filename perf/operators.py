"""Performance cases of a serving step over the paged latent cache: the block
tables and slot maps of a batch, rotary positions, the write of new tokens
into the cache (in bf16 or in 4 bits) and its read-back, attention over a
4-bit cache, and attention through a sliding window with sinks.

`own` false computes each operator in plain torch operations, true calls the
framework's kernels through the Python binding.  Attention and the small
calls of a step are prepared once, as a serving loop over static buffers
holds them.

Fields of a case (those that its kind uses):
  kind    slots   batch_slots: tables and slots of a batch from its lengths
          rope    rope: rotated query or key heads
          append  cache_append of T tokens, then fetch_gather of the whole pool
          window  window_attn: each query row attends the last `window` tokens
                  of its sequence (0: all of them) and the first n_sink
          blocks  sparse_partial_attn over one block selection per job
  B, Mq, H        requests (or jobs), query rows of a request, heads
  NB, K           blocks of a request's table, selected blocks of a job
  T               slots, rope, append: tokens; slots: the new tokens all told
  kv              bf16 | fp8 (one scale per block) | fp8split (separate latent
                  and RoPE scales) | mx4 (E2M1 codes, a scale per 32 columns)
  window, sinks   window: the masks
  ragged          window: requests with fewer than Mq query rows
  D, at, rot, pairing, scaling, dtype   rope: head width, first rotated dim,
                  rotated dims, pairing, long-context scaling, type
"""
import math

import numpy as np
import torch

own = False

DLAT, DPE, BLOCK, GROUP = 512, 64, 64, 32
SCALE = 1.0 / math.sqrt(192.0)
BASE = 10000.0
FACTOR, ORIG_LEN, FAST, SLOW, MSCALE = 40.0, 4096, 32.0, 1.0, 1.2
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # one new token for each request of a decode batch: launch and latency
        dict(name="slots-decode", kind="slots", B=64, T=64, NB=128),
        # prompts of very different lengths admitted together
        dict(name="slots-prefill", kind="slots", B=300, T=100003, NB=1024),
        # the RoPE part of a decode batch's queries, pairs of neighbours
        dict(name="rope-decode", kind="rope", T=64, H=128, D=64, at=0, rot=64, pairing=0,
             scaling="none", dtype="bf16"),
        # a prefill's whole query heads, of which the last 64 of 192 dims
        # turn, under long-context scaling
        dict(name="rope-prefill", kind="rope", T=4096, H=128, D=192, at=128, rot=64, pairing=1,
             scaling="yarn", dtype="bf16"),
        # a decode batch's new tokens into a 4-bit cache
        dict(name="append-decode", kind="append", T=64, P=64, kv="mx4"),
        # a prefill's tokens into a 4-bit cache
        dict(name="append-prefill", kind="append", T=30001, P=512, kv="mx4"),
        # the smallest attention call: a 16-head share of one request
        dict(name="window-one", kind="window", B=1, Mq=1, H=16, NB=32, kv="bf16", window=512,
             sinks=4, ragged=False),
        # a decode batch at full width over a window of an fp8 cache
        dict(name="window-batch", kind="window", B=64, Mq=1, H=128, NB=128, kv="fp8",
             window=1024, sinks=64, ragged=False),
        # two prompts' chunks of up to 512 query rows, an odd window
        dict(name="window-prefill", kind="window", B=2, Mq=512, H=128, NB=64, kv="bf16",
             window=1000, sinks=4, ragged=True),
        # four speculative rows a request over all of a long 4-bit cache
        dict(name="causal-mx4", kind="window", B=16, Mq=4, H=32, NB=512, kv="mx4", window=0,
             sinks=0, ragged=True),
        # one routed request over the top-2048 budget of a 4-bit chunk
        dict(name="mx4-one-request", kind="blocks", B=1, Mq=1, H=128, NB=64, K=32, kv="mx4"),
        # dense decode of 16-head shares over long 4-bit contexts: memory
        dict(name="mx4-dense", kind="blocks", B=32, Mq=1, H=16, NB=1024, K=1024, kv="mx4"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["slots", "rope", "append", "window", "window", "blocks"])
    if kind == "slots":
        B = _log(rng, 1, 600)
        return dict(kind="slots", B=B, T=max(B, _log(rng, B, 100000)), NB=1024)
    if kind == "rope":
        rot = rng.choice([32, 64, 64, 64, 128])
        extra = rng.choice([0, 0, 64, 128])
        return dict(kind="rope", T=_log(rng, 1, 4096), H=rng.choice([1, 8, 16, 40, 128]),
                    D=rot + extra, at=rng.choice([0, extra]), rot=rot, pairing=rng.randint(0, 1),
                    scaling=rng.choice(["none", "linear", "yarn"]),
                    dtype=rng.choice(["bf16", "bf16", "fp32"]))
    if kind == "append":
        T = _log(rng, 1, 30000)
        return dict(kind="append", T=T, P=(T + BLOCK - 1) // BLOCK + rng.randint(0, 40),
                    kv=rng.choice(["bf16", "mx4", "mx4"]))
    kv = rng.choice(["bf16", "fp8", "fp8split", "mx4", "mx4"])
    if kind == "blocks":
        B, K = _log(rng, 1, 40), _log(rng, 2, 128)
        return dict(kind="blocks", B=B, Mq=rng.randint(1, 3), H=rng.choice([8, 16, 24, 40, 64, 128]),
                    NB=min(512, _log(rng, K, 4 * K)), K=K, kv="mx4")
    if rng.random() < 0.4:  # a prefill's chunk
        return dict(kind="window", B=rng.randint(1, 2), Mq=_log(rng, 20, 300),
                    H=rng.choice([5, 16, 32, 64]), NB=rng.randint(8, 64), kv=kv,
                    window=rng.choice([0, _log(rng, 30, 2000)]), sinks=rng.choice([0, 4, 70]),
                    ragged=rng.random() < 0.7)
    return dict(kind="window", B=_log(rng, 1, 40), Mq=rng.randint(1, 3),
                H=rng.choice([1, 8, 16, 24, 64, 128]), NB=_log(rng, 4, 128), kv=kv,
                window=rng.choice([0, _log(rng, 30, 4000), _log(rng, 30, 4000)]),
                sinks=rng.choice([0, 1, 4, 64, 130]), ragged=rng.random() < 0.5)


# ---------------------------------------------------------------- inputs
def _normal(g, shape, sigma, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype).mul_(sigma)


def _gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _to_mx4(x):
    """fp32 [..., 512] -> bytes [..., 272]: 512 E2M1 codes, the even column in
    the low half of a byte, then 16 scale exponents (plus 127)."""
    v = x.reshape(x.shape[:-1] + (DLAT // GROUP, GROUP))
    e = (torch.frexp(v.abs().amax(-1)).exponent - 3).clamp(-125, 125)
    a = torch.ldexp(v.abs(), -e[..., None])
    q = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5)
         + (a >= 3.5) + (a > 5.0)) | (torch.signbit(v).to(torch.uint8) << 3)
    q = q.reshape(x.shape[:-1] + (DLAT,))
    return torch.cat([q[..., 0::2] | (q[..., 1::2] << 4), (e + 127).to(torch.uint8)], -1)


def _from_mx4(rows):
    """Bytes [..., 272] -> the fp32 values they stand for, [..., 512]."""
    lut = torch.tensor(E2M1 + [-v for v in E2M1], device=rows.device)
    c = rows[..., :DLAT // 2]
    v = lut[torch.stack([c & 15, c >> 4], -1).flatten(-2).int()]
    e = rows[..., DLAT // 2:].to(torch.int32) - 127
    v = v.view(v.shape[:-1] + (DLAT // GROUP, GROUP))
    return torch.ldexp(v, e[..., None].expand(v.shape)).reshape(rows.shape[:-1] + (DLAT,))


def _pools(g, P, kv, sigma=0.5):
    """(ckv, kpe, ckv_scale, kpe_scale): a pool of P blocks ~ N(0, sigma)."""
    if kv == "bf16":
        return (_normal(g, (P, BLOCK, DLAT), sigma), _normal(g, (P, BLOCK, DPE), sigma), None, None)
    if kv == "mx4":
        ckv = torch.empty((P, BLOCK, DLAT // 2 + DLAT // GROUP), dtype=torch.uint8, device="cuda")
        for lo in range(0, P, 2048):
            n = min(P - lo, 2048)
            ckv[lo:lo + n] = _to_mx4(_normal(g, (n, BLOCK, DLAT), sigma, torch.float32))
        return ckv, _normal(g, (P, BLOCK, DPE), sigma), None, None
    ckv = torch.empty((P, BLOCK, DLAT), dtype=torch.uint8, device="cuda")
    kpe = torch.empty((P, BLOCK, DPE), dtype=torch.uint8, device="cuda")
    cs = torch.empty(P, dtype=torch.float32, device="cuda")
    ks = cs if kv == "fp8" else torch.empty_like(cs)
    for lo in range(0, P, 2048):
        hi = min(P, lo + 2048)
        x = _normal(g, (hi - lo, BLOCK, DLAT + DPE), sigma, torch.float32)
        for v, codes, s in ((x[..., :DLAT], ckv, cs), (x[..., DLAT:], kpe, ks)):
            s[lo:hi] = (x if kv == "fp8" else v).abs().amax(dim=(1, 2)) / 448.0
            q = (v / s[lo:hi, None, None]).clamp_(-448.0, 448.0)
            codes[lo:hi] = q.to(torch.float8_e4m3fn).view(torch.uint8)
    return ckv, kpe, cs, ks


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rs = np.random.default_rng([seed, 41])
    kind = case["kind"]
    if kind == "slots":
        B, T, NB = case["B"], case["T"], case["NB"]
        # T new tokens over the requests, most of them in a few; then tokens
        # already cached, as far as the table holds both
        share = rs.exponential(size=B) ** 2
        new = 1 + np.floor((T - B) * share / share.sum()).astype(np.int64)
        new[rs.integers(B)] += T - new.sum()
        over = np.maximum(new - NB * BLOCK, 0)
        new -= over
        cached = np.floor(rs.random(B) * np.minimum(NB * BLOCK - new, 8192)).astype(np.int64)
        have, all_ = (cached + 63) // 64, (cached + new + 63) // 64
        perm = rs.permutation(int(all_.sum()) + 64).astype(np.int32)
        table = np.full((B, NB), -1, np.int32)
        col = np.arange(NB)[None] < have[:, None]
        table[col] = perm[:int(have.sum())]
        return dict(cached=_gpu(cached.astype(np.int32)), new=_gpu(new.astype(np.int32)),
                    free=_gpu(perm[int(have.sum()):]), table=_gpu(table))
    if kind == "rope":
        dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
        return dict(x=_normal(g, (case["T"], case["H"], case["D"]), 1.0, dt),
                    pos=_gpu(rs.integers(0, 163840, case["T"]).astype(np.int32)))
    if kind == "append":
        T, P = case["T"], case["P"]
        ckv, kpe, _, _ = _pools(g, P, case["kv"])
        return dict(new_ckv=_normal(g, (T, DLAT), 0.5), new_kpe=_normal(g, (T, DPE), 0.5), ckv=ckv,
                    kpe=kpe, slots=_gpu(rs.permutation(P * BLOCK)[:T].astype(np.int32)),
                    table=_gpu(np.arange(P, dtype=np.int32)),
                    every=_gpu(np.arange(P * BLOCK, dtype=np.int32)))
    B, Mq, H, NB = case["B"], case["Mq"], case["H"], case["NB"]
    ckv, kpe, cs, ks = _pools(g, B * NB, case["kv"])
    t = dict(q_lat=_normal(g, (B, Mq, H, DLAT), 1.0), q_pe=_normal(g, (B, Mq, H, DPE), 1.0), ckv=ckv,
             kpe=kpe, cs=cs, ks=ks, table=_gpu(rs.permutation(B * NB).astype(np.int32).reshape(B, NB)))
    if kind == "blocks":
        key = rs.random((B, NB))
        t["sel"] = _gpu(np.sort(np.argsort(key, axis=1)[:, :case["K"]], axis=1).astype(np.int32))
        return t
    lens = rs.integers(max(1, NB * BLOCK * 2 // 3), NB * BLOCK + 1, B)
    q_lens = rs.integers((Mq + 1) // 2, Mq + 1, B) if case["ragged"] else np.full(B, Mq)
    t["lens"] = _gpu(lens.astype(np.int32))
    t["q_lens"] = _gpu(q_lens.astype(np.int32))
    return t


def _outputs(case):
    """The outputs' buffers, kept by the program from pass to pass."""
    def i32(*s):
        return torch.empty(s, dtype=torch.int32, device="cuda")
    kind = case["kind"]
    if kind == "slots":
        B, T = case["B"], case["T"]
        return dict(slots=i32(T), positions=i32(T), seq_lens=i32(B), starts=i32(B + 1), info=i32(4))
    if kind == "append":
        n = case["P"] * BLOCK
        return dict(out_ckv=torch.empty((1, n, DLAT), dtype=torch.bfloat16, device="cuda"),
                    out_kpe=torch.empty((1, n, DPE), dtype=torch.bfloat16, device="cuda"))
    return {}


def prepare(case, seed):
    s = dict(case=case, **_inputs(case, seed))
    if not own:
        return s
    from paper_2606_01502_amd import mla
    kind, o = case["kind"], _outputs(case)
    # the calls of a step over static buffers, their arguments fixed
    if kind == "slots":
        s["call"] = mla.prepare_batch_slots(s["cached"], s["new"], s["free"], s["table"], **o)
    elif kind == "rope":
        s["call"] = mla.prepare_rope(s["x"], s["pos"], rot_offset=case["at"], rot_dim=case["rot"],
                                     pairing=case["pairing"], base=BASE, **_scaling(case))
    elif kind == "append":
        s["call"] = mla.prepare_cache_append(s["new_ckv"], s["new_kpe"], s["slots"], s["ckv"], s["kpe"])
        s["mla"], s["out"] = mla, o
    elif kind == "window":
        s["call"] = mla.prepare_window(s["q_lat"], s["q_pe"], s["ckv"], s["kpe"], s["table"],
                                       s["lens"], SCALE, window=case["window"],
                                       n_sink=case["sinks"], q_lens=s["q_lens"],
                                       ckv_scale=s["cs"], kpe_scale=s["ks"], wire=True)
    else:
        s["call"] = mla.prepare_partial(s["q_lat"], s["q_pe"], s["ckv"], s["kpe"], s["table"],
                                        s["sel"], SCALE, ckv_scale=s["cs"], kpe_scale=s["ks"],
                                        wire=True)
    return s


def _scaling(case):
    if case["scaling"] == "none":
        return {}
    if case["scaling"] == "linear":
        return dict(scaling="linear", factor=FACTOR)
    return dict(scaling="yarn", factor=FACTOR, orig_len=ORIG_LEN, beta_fast=FAST, beta_slow=SLOW,
                mscale=MSCALE)


# ---------------------------------------------------------------- a pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        got = state["call"]()
        if kind == "slots":
            return (*got, state["table"])
        if kind == "append":
            return state["mla"].fetch_gather(state["ckv"][None], state["kpe"][None], state["table"],
                                             state["every"], **state["out"])
        return got
    if kind == "slots":
        return _plain_slots(state)
    if kind == "rope":
        return _plain_rope(state)
    if kind == "append":
        return _plain_append(state)
    return _plain_window(state) if kind == "window" else _plain_blocks(state)


def _plain_slots(s):
    T = s["case"]["T"]
    cached, new, free, table = s["cached"].long(), s["new"].long(), s["free"].long(), s["table"].long()
    NB, F = table.shape[1], free.shape[0]
    have = (cached + 63) // 64
    need = (cached + new + 63) // 64 - have
    ends = torch.cumsum(new, 0)
    starts = ends - new
    first = torch.cumsum(need, 0) - need
    t = torch.arange(T, device=table.device)
    b = torch.searchsorted(ends, t, right=True).clamp(max=ends.shape[0] - 1)
    live = t < ends[-1]
    pos = cached[b] + t - starts[b]
    at = pos // 64
    j = first[b] + at - have[b]
    blk = torch.where(at < have[b], table[b, at.clamp(max=NB - 1)], free[j.clamp(0, F - 1)])
    ok = live & (at < NB) & ((at < have[b]) | (j < F)) & (blk >= 0)
    slots = torch.where(ok, blk * 64 + pos % 64, -1)
    col = torch.arange(NB, device=table.device)[None]
    k = first[:, None] + col - have[:, None]
    taken = torch.where(k < F, free[k.clamp(0, F - 1)], -1)
    table = torch.where((col >= have[:, None]) & (col < (have + need)[:, None]), taken, table)
    total, blocks = ends[-1], need.sum()
    info = torch.stack([total, blocks.clamp(max=F), (blocks - F).clamp(min=0), (total - T).clamp(min=0)])
    return (slots.int(), torch.where(live, pos, -1).int(), (cached + new).int(),
            torch.cat([starts, ends[-1:]]).int(), info.int(), table.int())


def _freqs(case, device):
    """Angles a position, of each pair, in 64 bits."""
    d = case["rot"]
    i = torch.arange(d // 2, device=device, dtype=torch.float64)
    f = BASE ** (-2.0 * i / d)
    if case["scaling"] == "linear":
        return f / FACTOR
    if case["scaling"] == "yarn":
        lo = math.floor(d / 2 * math.log(ORIG_LEN / (2 * math.pi * FAST)) / math.log(BASE))
        hi = math.ceil(d / 2 * math.log(ORIG_LEN / (2 * math.pi * SLOW)) / math.log(BASE))
        lo, hi = max(lo, 0), min(hi, d - 1)
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * (1 - ramp) + f / FACTOR * ramp
    return f


def _plain_rope(s):
    case, x = s["case"], s["x"]
    at, d = case["at"], case["rot"]
    ang = s["pos"].double()[:, None] * _freqs(case, x.device)
    m = MSCALE if case["scaling"] == "yarn" else 1.0
    c, sn = (torch.cos(ang) * m).float()[:, None], (torch.sin(ang) * m).float()[:, None]
    v = x[..., at:at + d].float()
    if case["pairing"] == 0:
        a, b = v[..., 0::2], v[..., 1::2]
        y = torch.stack([a * c - b * sn, a * sn + b * c], -1).flatten(-2)
    else:
        a, b = v[..., :d // 2], v[..., d // 2:]
        y = torch.cat([a * c - b * sn, a * sn + b * c], -1)
    return torch.cat([x[..., :at], y.to(x.dtype), x[..., at + d:]], -1)


def _plain_append(s):
    ckv, kpe, at = s["ckv"], s["kpe"], s["slots"].long()
    rows = s["new_ckv"] if s["case"]["kv"] == "bf16" else _to_mx4(s["new_ckv"].float())
    ckv.view(-1, ckv.shape[-1])[at] = rows
    kpe.view(-1, DPE)[at] = s["new_kpe"]
    values = ckv if s["case"]["kv"] == "bf16" else _from_mx4(ckv).bfloat16()
    return values.view(1, -1, DLAT), kpe.view(1, -1, DPE)


def _tokens32(s, blocks):
    """Keys [J, n, 576] in 32 bits of the pool blocks [J, n / 64]."""
    J, kv = blocks.shape[0], s["case"]["kv"]
    lat, pe = s["ckv"][blocks], s["kpe"][blocks]
    if kv == "mx4":
        lat = _from_mx4(lat)
    elif kv != "bf16":
        lat = lat.view(torch.float8_e4m3fn).float() * s["cs"][blocks][..., None, None]
        pe = pe.view(torch.float8_e4m3fn).float() * s["ks"][blocks][..., None, None]
    return torch.cat([lat.float(), pe.float()], -1).view(J, -1, DLAT + DPE)


def _softmax_rows(s, scores, keys):
    """(out bf16, (m, l) fp32) of masked scores [J, rows, n]."""
    q = s["q_lat"]
    m = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - m.clamp(min=-3e38))
    ell = p.sum(-1, keepdim=True)
    out = torch.bmm(p, keys[..., :DLAT].contiguous()) / ell.clamp(min=1e-38)
    return out.bfloat16().view(q.shape), torch.cat([m, ell], -1).view(q.shape[:3] + (2,))


def _scores32(s, keys):
    J, _, H, _ = s["q_lat"].shape
    q = torch.cat([s["q_lat"], s["q_pe"]], -1).float().view(J, -1, DLAT + DPE)
    return torch.bmm(q, keys.transpose(1, 2).contiguous()) * SCALE


def _plain_window(s):
    case, q = s["case"], s["q_lat"]
    B, Mq, H, _ = q.shape
    keys = _tokens32(s, s["table"].long())
    i = torch.arange(Mq, device=q.device)[None, :, None, None]
    t = torch.arange(keys.shape[1], device=q.device)
    qn, n = s["q_lens"].long().view(B, 1, 1, 1), s["lens"].long().view(B, 1, 1, 1)
    p = n - qn + i
    see = (t <= p) & (i < qn)
    if case["window"]:
        see &= (t > p - case["window"]) | (t < case["sinks"])
    scores = _scores32(s, keys).view(B, Mq, H, -1).masked_fill_(~see, -math.inf)
    return _softmax_rows(s, scores.view(B, Mq * H, -1), keys)


def _plain_blocks(s):
    keys = _tokens32(s, torch.gather(s["table"].long(), 1, s["sel"].long()))
    return _softmax_rows(s, _scores32(s, keys), keys)


# ---------------------------------------------------------------- bounds
def work(case):
    kind = case["kind"]
    if kind == "slots":
        B, T = case["B"], case["T"]
        return dict(bytes=8 * B + 4 * (T // BLOCK + B) * 2 + 8 * T + 8 * B, flops=0)
    if kind == "rope":
        n = case["T"] * case["H"] * case["D"]
        return dict(bytes=2 * n * (4 if case["dtype"] == "fp32" else 2) + 4 * case["T"],
                    flops=3 * case["T"] * case["H"] * case["rot"])
    token = {"bf16": 2 * (DLAT + DPE), "mx4": DLAT // 2 + DLAT // GROUP + 2 * DPE}.get(case["kv"], DLAT + DPE)
    if kind == "append":
        n = case["P"] * BLOCK
        return dict(bytes=case["T"] * (2 * (DLAT + DPE) + token + 4) + n * (token + 2 * (DLAT + DPE)), flops=0)
    B, Mq, H = case["B"], case["Mq"], case["H"]
    # lengths are spread over the last third of the table, ragged rows over
    # the upper half of Mq
    mean = case["NB"] * BLOCK * 5 / 6
    rows = Mq * (0.75 if kind == "window" and case["ragged"] and Mq > 1 else 1.0)
    if kind == "blocks":
        pairs, read = B * rows * case["K"] * BLOCK, B * case["K"] * BLOCK
    elif case["window"] == 0 or case["window"] + case["sinks"] >= mean:
        pairs, read = B * rows * max(mean - rows / 2, mean / 2), B * mean
    else:
        pairs = B * rows * (case["window"] + case["sinks"])
        read = B * min(mean, case["window"] + case["sinks"] + rows)
    return dict(bytes=read * token + B * Mq * H * (2 * (DLAT + DPE) + 2 * DLAT + 8),
                flops=pairs * H * 2 * (2 * DLAT + DPE))


# ---------------------------------------------------------------- 64-bit values
def _turn(case, i):
    """The angle a position of pair i."""
    d, kind = case["rot"], case["scaling"]
    w = math.exp(-2.0 * i / d * math.log(BASE))
    if kind == "none":
        return w
    if kind == "linear":
        return w / FACTOR
    # pairs that turn FAST times and more in ORIG_LEN keep their angle, those
    # that turn SLOW times and less are slowed FACTOR times
    at = [0.5 * d * math.log(ORIG_LEN / (2 * math.pi * turns), BASE) for turns in (FAST, SLOW)]
    lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), d - 1)
    share = min(max((i - lo) / (hi - lo if hi > lo else 0.001), 0.0), 1.0)
    return w * (1 - share + share / FACTOR)


def _values64(rows):
    """Bytes [..., 272] -> float64 [..., 512], a code's bits taken apart."""
    codes = torch.repeat_interleave(rows[..., :DLAT // 2], 2, -1)
    codes[..., 1::2] >>= 4
    e, m = ((codes >> 1) & 3).double(), (codes & 1).double()
    mag = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * torch.exp2(e - 1))
    unit = torch.exp2(rows[..., DLAT // 2:].double() - 127).repeat_interleave(GROUP, -1)
    return torch.where((codes & 8) != 0, -mag, mag) * unit


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "slots":
        return None
    if kind == "rope":
        at, d = case["at"], case["rot"]
        x = s["x"].double()
        v = x[..., at:at + d].clone()
        z = torch.complex(v[..., 0::2], v[..., 1::2]) if case["pairing"] == 0 else \
            torch.complex(v[..., :d // 2], v[..., d // 2:])
        turn = torch.tensor([_turn(case, i) for i in range(d // 2)], device="cuda", dtype=torch.float64)
        z = z * torch.polar(torch.full_like(z.real, MSCALE if case["scaling"] == "yarn" else 1.0),
                            (s["pos"].double()[:, None, None] * turn).expand(z.shape))
        if case["pairing"] == 0:
            x[..., at:at + d:2], x[..., at + 1:at + d:2] = z.real, z.imag
        else:
            x[..., at:at + d // 2], x[..., at + d // 2:at + d] = z.real, z.imag
        return x
    if kind == "append":
        # the nearest of the eight magnitudes under the group's power of two
        pool = s["ckv"].double() if case["kv"] == "bf16" else _values64(s["ckv"])
        new = s["new_ckv"].double()
        if case["kv"] == "mx4":
            v = new.view(-1, DLAT // GROUP, GROUP)
            unit = torch.exp2(torch.floor(torch.log2(v.abs().amax(-1, keepdim=True))) - 2)
            grid = torch.tensor(E2M1, device=v.device, dtype=torch.float64)
            # halfway goes to the even code: the magnitudes at even places are
            # taken as a hair nearer
            hair = torch.tensor([0.0, 1e-9] * 4, device=v.device, dtype=torch.float64)
            near = torch.cat([((c.abs() / u).unsqueeze(-1) - grid).abs().add_(hair).argmin(-1)
                              for c, u in zip(v.split(2048), unit.split(2048))])
            new = (torch.copysign(grid[near], v) * unit).view(-1, DLAT)
        pool.view(-1, DLAT)[s["slots"].long()] = new
        kpe = s["kpe"].double()
        kpe.view(-1, DPE)[s["slots"].long()] = s["new_kpe"].double()
        return pool.view(1, -1, DLAT), kpe.view(1, -1, DPE)
    B, Mq, H = case["B"], case["Mq"], case["H"]
    out = torch.zeros((B, Mq, H, DLAT), dtype=torch.float64, device="cuda")
    stat = torch.zeros((B, Mq, H, 2), dtype=torch.float64, device="cuda")
    stat[..., 0] = -math.inf
    table = s["table"].cpu().numpy()

    def tokens(blocks):
        at = _gpu(blocks).long()
        k, kp = s["ckv"][at], s["kpe"][at]
        if case["kv"] == "mx4":
            k = _values64(k)
        elif case["kv"] != "bf16":
            k = k.view(torch.float8_e4m3fn).double() * s["cs"][at].double()[:, None, None]
            kp = kp.view(torch.float8_e4m3fn).double() * s["ks"][at].double()[:, None, None]
        return k.double().reshape(-1, DLAT), kp.double().reshape(-1, DPE)

    def attend(b, i0, i1, k, kp, see):
        sc = s["q_lat"][b, i0:i1].double() @ k.T + s["q_pe"][b, i0:i1].double() @ kp.T
        sc = sc * float(np.float32(SCALE))
        if see is not None:
            sc = torch.where(see[:, None], sc, torch.full_like(sc, -math.inf))
        m = sc.amax(-1)
        p = torch.exp(sc - m[..., None])
        ell = p.sum(-1)
        out[b, i0:i1] = (p @ k) / ell[..., None]
        stat[b, i0:i1] = torch.stack([m, ell], -1)

    if kind == "blocks":
        sel = s["sel"].cpu().numpy()
        for b in range(B):
            attend(b, 0, Mq, *tokens(table[b, sel[b]]), None)
        return out, stat
    lens, q_lens = s["lens"].cpu().numpy(), s["q_lens"].cpu().numpy()
    for b in range(B):
        n, qn = int(lens[b]), int(q_lens[b])
        k, kp = tokens(table[b, :(n + BLOCK - 1) // BLOCK])
        k, kp = k[:n], kp[:n]
        for i0 in range(0, qn, 64):
            i1 = min(qn, i0 + 64)
            p = torch.arange(n - qn + i0, n - qn + i1, device="cuda")[:, None]
            t = torch.arange(n, device="cuda")[None]
            see = t <= p
            if case["window"]:
                see = see & ((t > p - case["window"]) | (t < case["sinks"]))
            attend(b, i0, i1, k, kp, see)
    return out, stat
