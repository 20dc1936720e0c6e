"""Performance cases of the operators that choose what a step attends, and of a
batch that shares its prefix, over the paged latent cache: the write of new
tokens with their rotary positions turned on the way, the mean keys of the blocks
that became whole, the cheap scores of those blocks for each query row, the choice
of the best ones, and attention over a prefix that a group of requests shares
beside what each has of its own.

`own` false computes each operator in plain torch operations, true calls the
framework's kernels through the Python binding, prepared once, as a serving loop
over static buffers holds them.

Fields of a case (those that its kind uses):
  kind    append  rope_append of T tokens (a 4-bit pool is then read back)
          means   block_means: the mean keys of the blocks that T slots complete
          scores  block_scores: how much of its attention a query row's heads
                  would give each block, by the blocks' mean keys
          topk    select_topk: the K best of N scores of each row
          prefix  prefix_attn: each request's rows over the prefix of its group
                  and over its own tokens
  B, Mq, H        requests, query rows of a request, heads
  NB              blocks of a request's table
  T, P            new tokens, blocks of the pool
  kv              bf16 | fp8 (one scale per block) | fp8split (separate latent
                  and RoPE scales) | mx4 (E2M1 codes, a scale per 32 columns)
  ragged          requests with fewer than Mq query rows
  pairing, scaling   append: of the rotation
  every           means: the slots are those of a list of whole blocks, not of
                  sequences' new tokens
  window, sinks   scores: the last tokens and the first ones, which a window
                  attends and no block chosen here may hold
  N, K, ties, holes   topk: scores and picks of a row; scores of a few values
                  only; shares of scores that may not be picked
  G, NBP          prefix: groups, and blocks of a group's table
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
        # a decode batch's new tokens: launch and latency
        dict(name="append-decode", kind="append", T=64, P=64, kv="bf16", pairing=0, scaling="none"),
        # a prefill's tokens, under long-context scaling
        dict(name="append-prefill", kind="append", T=30001, P=512, kv="bf16", pairing=1, scaling="yarn"),
        # a decode step in which two of 128 requests complete a block
        dict(name="means-decode", kind="means", T=128, P=1024, kv="bf16", every=False),
        # the blocks that a prefill completes, in an fp8 cache
        dict(name="means-prefill", kind="means", T=100003, P=2048, kv="fp8", every=False),
        # one request's 16-head share, 4096 tokens of context
        dict(name="scores-one", kind="scores", B=1, Mq=1, H=16, NB=64, window=128, sinks=0, ragged=False),
        # a decode batch at full width, 65,536 tokens of context each
        dict(name="scores-batch", kind="scores", B=64, Mq=1, H=128, NB=1024, window=512, sinks=64, ragged=False),
        # two prompts' chunks of up to 300 query rows, an odd window
        dict(name="scores-prefill", kind="scores", B=2, Mq=300, H=64, NB=500, window=1000, sinks=4, ragged=True),
        # the budget of 32 blocks out of a decode batch's 1024
        dict(name="topk-blocks", kind="topk", B=64, Mq=1, N=1024, K=32, ties=False, holes=True),
        # a budget of 2048 tokens, an indexer's, out of contexts of 65,536
        dict(name="topk-tokens", kind="topk", B=32, Mq=1, N=65536, K=2048, ties=False, holes=False),
        # four requests' 16-head share behind one instruction of 2000 tokens
        dict(name="prefix-small", kind="prefix", B=4, Mq=1, H=16, G=1, NBP=32, NB=4, kv="bf16", ragged=False),
        # a decode batch at full width behind one document
        dict(name="prefix-batch", kind="prefix", B=64, Mq=1, H=128, G=1, NBP=256, NB=8, kv="bf16", ragged=False),
        # speculative rows of requests that share five documents, fp8 cache
        dict(name="prefix-groups", kind="prefix", B=40, Mq=3, H=32, G=5, NBP=200, NB=13, kv="fp8", ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "means", "scores", "scores", "topk", "topk", "prefix", "prefix"])
    kv = rng.choice(["bf16", "fp8", "fp8split", "mx4"])
    heads = [1, 8, 16, 24, 40, 64, 128]
    if kind == "append":
        T = _log(rng, 1, 30000)
        return dict(kind="append", T=T, P=(T + BLOCK - 1) // BLOCK + rng.randint(0, 40),
                    kv=rng.choice(["bf16", "mx4"]), pairing=rng.randint(0, 1),
                    scaling=rng.choice(["none", "linear", "yarn"]))
    if kind == "means":
        every = rng.random() < 0.4
        T = _log(rng, 1, 1000) if every else _log(rng, 1, 60000)
        return dict(kind="means", T=T, P=(T if every else T // BLOCK + 300) + rng.randint(0, 40), kv=kv, every=every)
    if kind == "scores":
        if rng.random() < 0.4:  # a prefill's chunk
            return dict(kind="scores", B=rng.randint(1, 2), Mq=_log(rng, 20, 250), H=rng.choice([5, 16, 32, 64]),
                        NB=rng.randint(6, 500), window=rng.choice([0, 64, _log(rng, 30, 2000)]),
                        sinks=rng.choice([0, 4, 70]), ragged=rng.random() < 0.7)
        return dict(kind="scores", B=_log(rng, 1, 60), Mq=rng.randint(1, 3), H=rng.choice(heads),
                    NB=_log(rng, 1, 1000), window=rng.choice([0, 64, _log(rng, 30, 4000)]),
                    sinks=rng.choice([0, 1, 64, 130]), ragged=rng.random() < 0.5)
    if kind == "topk":
        N = _log(rng, 1, 65536)
        rows = _log(rng, 1, max(1, min(1000, 2000000 // N)))
        Mq = rng.choice([1, 1, 2, 7])
        return dict(kind="topk", B=max(1, rows // Mq), Mq=Mq, N=N, K=_log(rng, 1, min(N, 2048)),
                    ties=rng.random() < 0.4, holes=rng.random() < 0.5)
    B, Mq, H, NBP = _log(rng, 1, 60), rng.randint(1, 3), rng.choice(heads), _log(rng, 1, 256)
    NBP = max(1, min(NBP, 64 * 128 * 256 // (B * Mq * H * 2)))
    return dict(kind="prefix", B=B, Mq=Mq, H=H, G=rng.randint(1, min(B, 8)), NBP=NBP, NB=_log(rng, 1, 16), kv=kv,
                ragged=rng.random() < 0.5)


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
    rs = np.random.default_rng([seed, 43])
    kind = case["kind"]
    if kind == "append":
        T, P = case["T"], case["P"]
        ckv, kpe, _, _ = _pools(g, P, case["kv"])
        # the projection's rows, latent and RoPE part beside each other
        new = _normal(g, (T, DLAT + DPE), 0.5)
        return dict(new_ckv=new[:, :DLAT], new_kpe=new[:, DLAT:], ckv=ckv, kpe=kpe,
                    pos=_gpu(rs.integers(0, 163840, T).astype(np.int32)),
                    slots=_gpu(rs.permutation(P * BLOCK)[:T].astype(np.int32)),
                    table=_gpu(np.arange(P, dtype=np.int32)),
                    every=_gpu(np.arange(P * BLOCK, dtype=np.int32)))
    if kind == "means":
        T, P = case["T"], case["P"]
        ckv, kpe, cs, ks = _pools(g, P, case["kv"])
        blocks = rs.permutation(P)
        if case["every"]:
            slots = blocks[:T] * BLOCK + BLOCK - 1
        else:
            # requests that begin anywhere in a block, their tokens one after
            # another (a decode batch: one token each); rows of a block that
            # no request holds are not written, so a mean may cover old rows
            n = 1 if T <= P else max(1, T // 200)
            cut = np.sort(rs.integers(0, T + 1, n - 1)) if T > P else np.arange(1, T)
            lens = np.diff(np.concatenate([[0], cut, [T]])).astype(np.int64)
            first = rs.integers(0, BLOCK, len(lens))
            if T <= P:
                first[:2] = BLOCK - 1
            held = (first + lens + BLOCK - 1) // BLOCK
            base = np.concatenate([[0], np.cumsum(held)[:-1]])
            b = np.repeat(np.arange(len(lens)), lens)
            i = np.arange(T) - np.repeat(np.cumsum(lens) - lens, lens) + first[b]
            slots = blocks[(base[b] + i // BLOCK) % P] * BLOCK + i % BLOCK
        return dict(ckv=ckv, kpe=kpe, cs=cs, ks=ks, slots=_gpu(slots.astype(np.int32)),
                    means=_normal(g, (P, DLAT + DPE), 0.1))
    if kind == "topk":
        shape = (case["B"], case["Mq"], case["N"])
        x = torch.rand(shape, generator=g, device="cuda").square_()
        if case["ties"]:
            x = torch.round(x * 16.0) / 16.0
        if case["holes"]:
            # each row's first picks are held by its sinks, the last ones by its window
            n = torch.rand(shape[:2], generator=g, device="cuda")[..., None] * (case["N"] + 1)
            at = torch.arange(case["N"], device="cuda")
            x = torch.where((at < 1) | (at >= n), -math.inf, x)
        return dict(scores=x)
    B, Mq, H, NB = case["B"], case["Mq"], case["H"], case["NB"]
    q = dict(q_lat=_normal(g, (B, Mq, H, DLAT), 1.0), q_pe=_normal(g, (B, Mq, H, DPE), 1.0))
    q_lens = rs.integers((Mq + 1) // 2, Mq + 1, B) if case["ragged"] else np.full(B, Mq)
    if kind == "scores":
        table = rs.permutation(B * NB).astype(np.int32).reshape(B, NB)
        lens = rs.integers(max(1, NB * BLOCK * 2 // 3), NB * BLOCK + 1, B)
        return dict(**q, means=_normal(g, (B * NB, DLAT + DPE), 0.5), table=_gpu(table),
                    lens=_gpu(lens.astype(np.int32)), q_lens=_gpu(q_lens.astype(np.int32)))
    G, NBP = case["G"], case["NBP"]
    ckv, kpe, cs, ks = _pools(g, G * NBP + B * NB, case["kv"])
    blocks = rs.permutation(G * NBP + B * NB).astype(np.int32)
    starts = np.concatenate([[0], np.sort(rs.integers(0, B + 1, G - 1)), [B]])
    plens = rs.integers(max(1, NBP * BLOCK * 9 // 10), NBP * BLOCK + 1, G)
    lens = np.maximum(q_lens, rs.integers(1, NB * BLOCK + 1, B))
    return dict(**q, ckv=ckv, kpe=kpe, cs=cs, ks=ks, ptable=_gpu(blocks[:G * NBP].reshape(G, NBP)),
                table=_gpu(blocks[G * NBP:].reshape(B, NB)), starts=_gpu(starts.astype(np.int32)),
                plens=_gpu(plens.astype(np.int32)), lens=_gpu(lens.astype(np.int32)),
                q_lens=_gpu(q_lens.astype(np.int32)), most=int(np.diff(starts).max()))


def _scaling(case):
    if case["scaling"] == "none":
        return {}
    if case["scaling"] == "linear":
        return dict(scaling="linear", factor=FACTOR)
    return dict(scaling="yarn", factor=FACTOR, orig_len=ORIG_LEN, beta_fast=FAST, beta_slow=SLOW,
                mscale=MSCALE)


def prepare(case, seed):
    s = dict(case=case, **_inputs(case, seed))
    if not own:
        return s
    from paper_2606_01502_amd import mla
    kind = case["kind"]
    # the calls of a step over static buffers, their arguments fixed
    if kind == "append":
        s["call"] = mla.prepare_rope_append(s["new_ckv"], s["new_kpe"], s["pos"], s["slots"], s["ckv"], s["kpe"],
                                            pairing=case["pairing"], base=BASE, **_scaling(case))
        s["mla"] = mla
    elif kind == "means":
        s["call"] = mla.prepare_block_means(s["ckv"], s["kpe"], s["slots"], s["means"], ckv_scale=s["cs"],
                                            kpe_scale=s["ks"])
    elif kind == "scores":
        s["call"] = mla.prepare_block_scores(s["q_lat"], s["q_pe"], s["means"], s["table"], s["lens"], SCALE,
                                             window=case["window"], n_sink=case["sinks"], q_lens=s["q_lens"])
    elif kind == "topk":
        s["call"] = mla.prepare_select_topk(s["scores"], case["K"])
    else:
        s["call"] = mla.prepare_prefix(s["q_lat"], s["q_pe"], s["ckv"], s["kpe"], s["ptable"], s["plens"],
                                       s["starts"], s["table"], s["lens"], SCALE, q_lens=s["q_lens"],
                                       ckv_scale=s["cs"], kpe_scale=s["ks"], wire=True)
    return s


# ---------------------------------------------------------------- a pass
def run(state):
    kind = state["case"]["kind"]
    if own:
        got = state["call"]()
        if kind == "append" and state["case"]["kv"] == "mx4":
            return state["mla"].fetch_gather(state["ckv"][None], state["kpe"][None], state["table"], state["every"])
        return got
    if kind == "append":
        return _plain_append(state)
    if kind == "means":
        return _plain_means(state)
    if kind == "scores":
        return _plain_scores(state)
    return _plain_topk(state) if kind == "topk" else _plain_prefix(state)


def _freqs(case, device):
    """Angles a position, of each pair, in 64 bits."""
    d = DPE
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


def _plain_append(s):
    case, ckv, kpe, at = s["case"], s["ckv"], s["kpe"], s["slots"].long()
    ang = s["pos"].double()[:, None] * _freqs(case, ckv.device)
    m = MSCALE if case["scaling"] == "yarn" else 1.0
    c, sn = (torch.cos(ang) * m).float(), (torch.sin(ang) * m).float()
    v = s["new_kpe"].float()
    if case["pairing"] == 0:
        a, b = v[:, 0::2], v[:, 1::2]
        y = torch.stack([a * c - b * sn, a * sn + b * c], -1).flatten(-2)
    else:
        a, b = v[:, :DPE // 2], v[:, DPE // 2:]
        y = torch.cat([a * c - b * sn, a * sn + b * c], -1)
    ckv.view(-1, ckv.shape[-1])[at] = s["new_ckv"] if case["kv"] == "bf16" else _to_mx4(s["new_ckv"].float())
    kpe.view(-1, DPE)[at] = y.bfloat16()
    if case["kv"] == "bf16":
        return ckv, kpe
    return _from_mx4(ckv).bfloat16().view(1, -1, DLAT), kpe.view(1, -1, DPE)


def _blocks32(s, blocks):
    """Entries [..., 64, 576] in 32 bits of the pool blocks."""
    kv = s["case"]["kv"]
    lat, pe = s["ckv"][blocks], s["kpe"][blocks]
    if kv == "mx4":
        lat = _from_mx4(lat)
    elif kv != "bf16":
        lat = lat.view(torch.float8_e4m3fn).float() * s["cs"][blocks][..., None, None]
        pe = pe.view(torch.float8_e4m3fn).float() * s["ks"][blocks][..., None, None]
    return torch.cat([lat.float(), pe.float()], -1)


def _plain_means(s):
    slots, means = s["slots"].long(), s["means"]
    blocks = slots[slots % BLOCK == BLOCK - 1] // BLOCK
    means[blocks] = (_blocks32(s, blocks).sum(-2) / BLOCK).bfloat16()
    return means


def _plain_scores(s):
    case, q = s["case"], s["q_lat"]
    B, Mq, H, _ = q.shape
    keys = s["means"][s["table"].long()].float()
    rows = torch.cat([q, s["q_pe"]], -1).float().view(B, Mq * H, -1)
    x = torch.bmm(rows, keys.transpose(1, 2).contiguous()).view(B, Mq, H, -1) * SCALE
    i = torch.arange(Mq, device=q.device)[None, :, None]
    j = torch.arange(keys.shape[1], device=q.device)
    qn, n = s["q_lens"].long().view(B, 1, 1), s["lens"].long().view(B, 1, 1)
    p = n - qn + i
    # the last whole block before what the window holds
    lo = (p + 1 - case["window"]).clamp(min=0) // BLOCK
    may = (i < qn) & (j < lo) & (j * BLOCK >= case["sinks"])
    x = x.masked_fill_(~may[:, :, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp(min=-3e38)
    w = torch.exp(x - m)
    w = (w / w.sum(-1, keepdim=True).clamp(min=1e-38)).sum(2)
    return torch.where(may, w, -math.inf)


def _plain_topk(s):
    x, K = s["scores"], s["case"]["K"]
    v, at = torch.sort(x, dim=-1, descending=True, stable=True)
    none = x.shape[-1]
    at = torch.sort(torch.where(v[..., :K] == -math.inf, none, at[..., :K]), dim=-1).values
    return torch.where(at == none, -1, at).int()


def _part(q, keys, see):
    """(m, l, sum of weighted values) of q [J, r, 576] over keys [J, n, 576],
    where see [J, r, n] allows."""
    x = torch.bmm(q, keys.transpose(1, 2).contiguous()) * SCALE
    x = x.masked_fill_(~see, -math.inf)
    m = x.amax(-1, keepdim=True)
    w = torch.exp(x - m.clamp(min=-3e38))
    return m, w.sum(-1, keepdim=True), torch.bmm(w, keys[..., :DLAT].contiguous())


def _plain_prefix(s):
    q = s["q_lat"]
    B, Mq, H, _ = q.shape
    rows, n = torch.cat([q, s["q_pe"]], -1).float().view(B, Mq * H, -1), s["most"]
    dev = q.device
    i = torch.arange(Mq, device=dev).repeat_interleave(H)[None]
    live = i < s["q_lens"].long()[:, None]
    # the shared part: every group's rows over its prefix, read once
    starts = s["starts"].long()
    at = (starts[:-1, None] + torch.arange(n, device=dev)).clamp(max=B - 1)
    G = at.shape[0]
    pkeys = _blocks32(s, s["ptable"].long()).view(G, -1, DLAT + DPE)
    in_prefix = torch.arange(pkeys.shape[1], device=dev) < s["plens"].long()[:, None]
    see = live[at].view(G, -1, 1) & in_prefix[:, None]
    pm, pl, po = _part(rows[at].view(G, n * Mq * H, -1), pkeys, see)
    b = torch.arange(B, device=dev)
    g = torch.searchsorted(starts[1:].contiguous(), b, right=True)
    k = b - starts[g]
    pm, pl, po = (t.view(G, n, Mq * H, -1)[g, k] for t in (pm, pl, po))
    # each request's own tokens
    keys = _blocks32(s, s["table"].long()).view(B, -1, DLAT + DPE)
    t = torch.arange(keys.shape[1], device=dev)
    last = s["lens"].long()[:, None] - s["q_lens"].long()[:, None] + i
    om, ol, oo = _part(rows, keys, live[..., None] & (t <= last[..., None]))
    m = torch.maximum(pm, om)
    wp, wo = torch.exp(pm - m.clamp(min=-3e38)), torch.exp(om - m.clamp(min=-3e38))
    ell = wp * pl + wo * ol
    out = (wp * po + wo * oo) / ell.clamp(min=1e-38)
    return out.bfloat16().view(q.shape), torch.cat([m, ell], -1).view(B, Mq, H, 2)


# ---------------------------------------------------------------- bounds
def work(case):
    kind = case["kind"]
    token = {"bf16": 2 * (DLAT + DPE), "mx4": DLAT // 2 + DLAT // GROUP + 2 * DPE}.get(case.get("kv"), DLAT + DPE)
    if kind == "append":
        back = case["P"] * BLOCK * (token + 2 * (DLAT + DPE)) if case["kv"] == "mx4" else 0
        return dict(bytes=case["T"] * (2 * (DLAT + DPE) + token + 8) + back, flops=3 * case["T"] * DPE)
    if kind == "means":
        n = case["T"] if case["every"] else 2 + case["T"] // BLOCK
        return dict(bytes=4 * case["T"] + n * (BLOCK * token + 2 * (DLAT + DPE)), flops=n * BLOCK * (DLAT + DPE))
    if kind == "topk":
        rows = case["B"] * case["Mq"]
        return dict(bytes=4 * rows * (case["N"] + case["K"]), flops=0)
    B, Mq, H, NB = case["B"], case["Mq"], case["H"], case["NB"]
    rows = Mq * (0.75 if case["ragged"] and Mq > 1 else 1.0)
    q = B * Mq * H * 2 * (DLAT + DPE)
    if kind == "scores":
        # lengths are spread over the last third of the table
        n = max(1.0, NB * 5 / 6 - case["window"] / BLOCK - case["sinks"] / BLOCK)
        return dict(bytes=q + B * n * 2 * (DLAT + DPE) + 4 * B * Mq * NB, flops=B * rows * H * n * 2 * (DLAT + DPE))
    # a prefix is 95 % of its table, what a request has of its own half of its
    shared, mine = case["NBP"] * BLOCK * 0.95, NB * BLOCK / 2
    return dict(bytes=(case["G"] * shared + B * mine) * token + q + B * Mq * H * (2 * DLAT + 8),
                flops=B * rows * H * (shared + mine) * 2 * (2 * DLAT + DPE))


# ---------------------------------------------------------------- 64-bit values
def _turn(case, i):
    """The angle a position of pair i."""
    d, kind = DPE, case["scaling"]
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


def _latents64(new, kv):
    """What the cache holds of new latent rows [T, 512]."""
    new = new.double()
    if kv == "bf16":
        return new
    # the nearest of the eight magnitudes under the group's power of two,
    # halfway to the even code: those at even places are taken as a hair nearer
    v = new.view(-1, DLAT // GROUP, GROUP)
    unit = torch.exp2(torch.floor(torch.log2(v.abs().amax(-1, keepdim=True))) - 2)
    grid = torch.tensor(E2M1, device=v.device, dtype=torch.float64)
    hair = torch.tensor([0.0, 1e-9] * 4, device=v.device, dtype=torch.float64)
    near = torch.cat([((c.abs() / u).unsqueeze(-1) - grid).abs().add_(hair).argmin(-1)
                      for c, u in zip(v.split(2048), unit.split(2048))])
    return (torch.copysign(grid[near], v) * unit).view(-1, DLAT)


def _entries64(s, blocks):
    """(latent [n, 512], RoPE [n, 64]) in float64 of pool blocks, a host array."""
    at, kv = _gpu(blocks).long(), s["case_kv"]
    k, kp = s["ckv"][at], s["kpe"][at]
    if kv == "mx4":
        k = _values64(k)
    elif kv != "bf16":
        k = k.view(torch.float8_e4m3fn).double() * s["cs"][at].double()[:, None, None]
        kp = kp.view(torch.float8_e4m3fn).double() * s["ks"][at].double()[:, None, None]
    return k.double().reshape(-1, DLAT), kp.double().reshape(-1, DPE)


def exact(case, seed):
    kind = case["kind"]
    if kind == "topk":
        return None
    s = _inputs(case, seed)
    s["case_kv"] = case.get("kv")
    if kind == "append":
        v = s["new_kpe"].double()
        z = torch.complex(v[:, 0::2], v[:, 1::2]) if case["pairing"] == 0 else \
            torch.complex(v[:, :DPE // 2], v[:, DPE // 2:])
        turn = torch.tensor([_turn(case, i) for i in range(DPE // 2)], device="cuda", dtype=torch.float64)
        z = z * torch.polar(torch.full_like(z.real, MSCALE if case["scaling"] == "yarn" else 1.0),
                            s["pos"].double()[:, None] * turn)
        y = torch.empty_like(v)
        if case["pairing"] == 0:
            y[:, 0::2], y[:, 1::2] = z.real, z.imag
        else:
            y[:, :DPE // 2], y[:, DPE // 2:] = z.real, z.imag
        pool = s["ckv"].double() if case["kv"] == "bf16" else _values64(s["ckv"])
        pool.view(-1, DLAT)[s["slots"].long()] = _latents64(s["new_ckv"], case["kv"])
        kpe = s["kpe"].double()
        kpe.view(-1, DPE)[s["slots"].long()] = y
        return (pool, kpe) if case["kv"] == "bf16" else (pool.view(1, -1, DLAT), kpe.view(1, -1, DPE))
    if kind == "means":
        out = s["means"].double()
        slots = s["slots"].cpu().numpy()
        for part in np.array_split(slots[slots % BLOCK == BLOCK - 1] // BLOCK, 8):
            if len(part):
                k, kp = _entries64(s, part)
                out[_gpu(part).long()] = torch.cat([k.view(-1, BLOCK, DLAT).mean(1), kp.view(-1, BLOCK, DPE).mean(1)], -1)
        return out
    B, Mq, H = case["B"], case["Mq"], case["H"]
    lens, q_lens = s["lens"].cpu().numpy(), s["q_lens"].cpu().numpy()
    scale = float(np.float32(SCALE))
    if kind == "scores":
        out = torch.full((B, Mq, case["NB"]), -math.inf, dtype=torch.float64, device="cuda")
        table = s["table"].cpu().numpy()
        lowest = (case["sinks"] + BLOCK - 1) // BLOCK
        for b in range(B):
            keys = s["means"][_gpu(table[b]).long()].double()
            x = torch.cat([s["q_lat"][b], s["q_pe"][b]], -1).double() @ keys.T * scale  # [Mq, H, NB]
            for i in range(int(q_lens[b])):
                p = int(lens[b]) - int(q_lens[b]) + i
                end = min(max(p + 1 - case["window"], 0) // BLOCK, case["NB"])
                if end > lowest:
                    out[b, i, lowest:end] = torch.softmax(x[i, :, lowest:end], -1).sum(0)
        return out
    out = torch.zeros((B, Mq, H, DLAT), dtype=torch.float64, device="cuda")
    stat = torch.zeros((B, Mq, H, 2), dtype=torch.float64, device="cuda")
    stat[..., 0] = -math.inf
    table, ptable = s["table"].cpu().numpy(), s["ptable"].cpu().numpy()
    starts, plens = s["starts"].cpu().numpy(), s["plens"].cpu().numpy()
    for g in range(case["G"]):
        if starts[g] == starts[g + 1]:
            continue
        n = int(plens[g])
        pk, pp = (t[:n] for t in _entries64(s, ptable[g]))
        for b in range(int(starts[g]), int(starts[g + 1])):
            qn, m = int(q_lens[b]), int(lens[b])
            mk, mp = (t[:m] for t in _entries64(s, table[b]))
            k, kp = torch.cat([pk, mk]), torch.cat([pp, mp])
            sc = (s["q_lat"][b, :qn].double() @ k.T + s["q_pe"][b, :qn].double() @ kp.T) * scale
            t = torch.arange(n + m, device="cuda")
            last = n + m - qn + torch.arange(qn, device="cuda")
            sc = torch.where(t <= last[:, None, None], sc, torch.full_like(sc, -math.inf))
            top = sc.amax(-1)
            w = torch.exp(sc - top[..., None])
            ell = w.sum(-1)
            out[b, :qn] = (w @ k) / ell[..., None]
            stat[b, :qn] = torch.stack([top, ell], -1)
    return out, stat
