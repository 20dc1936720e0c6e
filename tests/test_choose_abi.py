"""What the entry points of the choice of blocks, of the turned write and of shared
prefixes refuse on the host, and the references' own checks (CPU only)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import choose as C
from oracle import step as S
from paper_2606_01502_amd import mla
from tests.test_step_abi import BF16, F32, I32, INVALID, U8, UNSUPPORTED, off, rope_args, z


def d(t, scale=None):
    if t is None:
        return None
    return ctypes.byref(mla._describe_latent(t, scale) if t.dtype == U8 else mla.describe(t))


def opts(cls, **kw):
    o = cls()
    for k, v in kw.items():
        if k == "reserved":
            o.reserved[3] = v
        else:
            setattr(o, k, v)
    return o


def answer(fn, *args):
    lib = mla.load()
    st = getattr(lib, fn)(*args)
    return st, lib.mla_last_error().decode()


# ---- rope_append
def append_args(mx4=False):
    return dict(ckv=z(5, 512), kpe=z(5, 64), pos=z(5, dt=I32), slots=z(5, dt=I32),
                pool=z(2, 64, 272, dt=U8) if mx4 else z(2, 64, 512), kpe_pool=z(2, 64, 64),
                opts=mla.RopeOpts(rot_offset=0, rot_dim=64, base=1e4, mscale=1.0))


def append_call(a):
    return answer("mla_rope_append", *[d(a[k]) for k in ("ckv", "kpe", "pos", "slots", "pool", "kpe_pool")],
                  ctypes.byref(a["opts"]) if a["opts"] is not None else None, None)


APPEND = [
    ("ckv null", dict(ckv=None), INVALID, "ckv"),
    ("kpe fp32", dict(kpe=z(5, 64, dt=F32)), INVALID, "kpe: wrong dtype"),
    ("positions null", dict(pos=None), INVALID, "positions"),
    ("positions int64", dict(pos=z(5, dt=torch.int64)), INVALID, "positions: wrong dtype"),
    ("positions length", dict(pos=z(4, dt=I32)), INVALID, "positions"),
    ("slots length", dict(slots=z(6, dt=I32)), INVALID, "slots"),
    ("fp8 pool", dict(pool=z(2, 64, 512, dt=U8)), UNSUPPORTED, "fp8"),
    ("pool strided", dict(pool=z(4, 64, 512)[::2]), INVALID, "contiguous"),
    ("ckv unaligned", dict(ckv=off(z(5, 512), 1)), INVALID, "aligned"),
    ("opts null", dict(opts=None), INVALID, "opts"),
    ("rot past the part", dict(opts=rope_args(rot_offset=2, rot_dim=64)["opts"]), INVALID, "within the head"),
    ("fast pair", dict(opts=rope_args(rot_offset=0, base=1e-9)["opts"]), INVALID, "2^20"),
]


@pytest.mark.parametrize("name,change,status,text", APPEND, ids=[c[0] for c in APPEND])
def test_rope_append_refused(name, change, status, text):
    a = append_args()
    a.update(change)
    st, msg = append_call(a)
    assert st == status and text in msg, (st, msg)


def test_rope_append_overlaps_refused():
    a = append_args()
    a["pos"] = a["kpe_pool"].view(I32).view(-1)[:5]
    st, msg = append_call(a)
    assert st == INVALID and "overlaps" in msg
    a = append_args()
    a["kpe"] = a["kpe_pool"].view(-1, 64)[:5]
    st, msg = append_call(a)
    assert st == INVALID and "overlaps" in msg


# ---- block_means
def means_args():
    return dict(ckv=z(4, 64, 512), kpe=z(4, 64, 64), slots=z(7, dt=I32), means=z(4, 576), s=None)


def means_call(a):
    return answer("mla_block_means", d(a["ckv"], a["s"]), d(a["kpe"], a["s"]), d(a["slots"]), d(a["means"]), None)


MEANS = [
    ("pool null", dict(ckv=None), INVALID, "null"),
    ("fp8 without scales", dict(ckv=z(4, 64, 512, dt=U8), kpe=z(4, 64, 64, dt=U8)), INVALID, "block_scale"),
    ("mx4 beside 8 bits", dict(ckv=z(4, 64, 272, dt=U8), kpe=z(4, 64, 64, dt=U8)), INVALID, "kpe_pool: wrong dtype"),
    ("P of kpe", dict(kpe=z(3, 64, 64)), INVALID, "kpe_pool: shape"),
    ("pool unaligned", dict(ckv=off(z(4, 64, 512), 1)), INVALID, "aligned"),
    ("slots int64", dict(slots=z(7, dt=torch.int64)), INVALID, "slots: wrong dtype"),
    ("slots strided", dict(slots=z(14, dt=I32)[::2]), INVALID, "innermost stride"),
    ("means fp32", dict(means=z(4, 576, dt=F32)), INVALID, "means: wrong dtype"),
    ("means P", dict(means=z(5, 576)), INVALID, "means"),
    ("means width", dict(means=z(4, 512)), INVALID, "means"),
    ("means strided", dict(means=z(4, 640)[:, :576]), INVALID, "contiguous"),
    ("means unaligned", dict(means=off(z(4, 576), 1)), INVALID, "aligned"),
]


@pytest.mark.parametrize("name,change,status,text", MEANS, ids=[c[0] for c in MEANS])
def test_means_refused(name, change, status, text):
    a = means_args()
    a.update(change)
    st, msg = means_call(a)
    assert st == status and text in msg, (st, msg)


def test_means_overlaps_refused():
    a = means_args()
    a["means"] = a["ckv"].view(-1)[:4 * 576].view(4, 576)
    st, msg = means_call(a)
    assert st == INVALID and "overlaps" in msg


# ---- block_scores
def scores_args():
    return dict(q_lat=z(2, 3, 16, 512), q_pe=z(2, 3, 16, 64), means=z(9, 576), table=z(2, 5, dt=I32),
                lens=z(2, dt=I32), q_lens=z(2, dt=I32), scale=0.1, out=z(2, 3, 5, dt=F32),
                opts=opts(mla.ScoresOpts))


def scores_call(a):
    return answer("mla_block_scores", *[d(a[k]) for k in ("q_lat", "q_pe", "means", "table", "lens", "q_lens")],
                  ctypes.c_float(a["scale"]), d(a["out"]),
                  ctypes.byref(a["opts"]) if a["opts"] is not None else None, None)


SCORES = [
    ("q null", dict(q_lat=None), INVALID, "q_lat"),
    ("q fp32", dict(q_lat=z(2, 3, 16, 512, dt=F32)), INVALID, "q_lat: wrong dtype"),
    ("q_pe shape", dict(q_pe=z(2, 3, 16, 32)), INVALID, "q_pe: shape"),
    ("B of q", dict(q_lat=z(1, 3, 16, 512)), INVALID, "q_lat: shape"),
    ("no heads", dict(q_lat=z(2, 3, 0, 512), q_pe=z(2, 3, 0, 64)), INVALID, "no heads"),
    ("q unaligned", dict(q_lat=off(z(2, 3, 16, 512), 1)), INVALID, "aligned"),
    ("means width", dict(means=z(9, 512)), INVALID, "means"),
    ("means fp32", dict(means=z(9, 576, dt=F32)), INVALID, "means: wrong dtype"),
    ("means unaligned", dict(means=off(z(9, 576), 4)), INVALID, "aligned"),
    ("lens length", dict(lens=z(3, dt=I32)), INVALID, "seq_lens"),
    ("q_lens int64", dict(q_lens=z(2, dt=torch.int64)), INVALID, "q_lens: wrong dtype"),
    ("scores bf16", dict(out=z(2, 3, 5)), INVALID, "scores: wrong dtype"),
    ("scores shape", dict(out=z(2, 3, 6, dt=F32)), INVALID, "scores: shape"),
    ("scores rows", dict(out=z(1, 3, 5, dt=F32).expand(2, 3, 5)), INVALID, "rows overlap"),
    ("scale inf", dict(scale=float("inf")), INVALID, "scale"),
    ("opts null", dict(opts=None), INVALID, "opts"),
    ("window", dict(opts=opts(mla.ScoresOpts, window=-1)), INVALID, "window"),
    ("n_sink", dict(opts=opts(mla.ScoresOpts, n_sink=-1)), INVALID, "n_sink"),
    ("n_splits", dict(opts=opts(mla.ScoresOpts, n_splits=-1)), INVALID, "n_splits"),
    ("reserved", dict(opts=opts(mla.ScoresOpts, reserved=1)), INVALID, "reserved"),
    ("too many rows", dict(q_lat=z(2, 1, 1, 512).expand(2, 1 << 20, 17, 512),
                           q_pe=z(2, 1, 1, 64).expand(2, 1 << 20, 17, 64),
                           out=z(2, 1 << 20, 5, dt=F32)), UNSUPPORTED, "index range"),
]


@pytest.mark.parametrize("name,change,status,text", SCORES, ids=[c[0] for c in SCORES])
def test_scores_refused(name, change, status, text):
    a = scores_args()
    a.update(change)
    st, msg = scores_call(a)
    assert st == status and text in msg, (st, msg)


def test_scores_overlaps_refused():
    a = scores_args()
    a["out"] = a["means"].view(-1).view(F32)[:30].view(2, 3, 5)
    st, msg = scores_call(a)
    assert st == INVALID and "overlaps" in msg


# ---- select_topk
TOPK = [
    ("scores null", None, z(2, 3, 4, dt=I32), "scores"),
    ("scores bf16", z(2, 3, 9), z(2, 3, 4, dt=I32), "scores: wrong dtype"),
    ("ids int64", z(2, 3, 9, dt=F32), z(2, 3, 4, dt=torch.int64), "ids: wrong dtype"),
    ("dims", z(2, 3, 9, dt=F32), z(6, 4, dt=I32), "ids: expected 3"),
    ("dims", z(6, 9, dt=F32), z(2, 3, 4, dt=I32), "ids: expected 2"),
    ("rows", z(2, 3, 9, dt=F32), z(2, 4, 4, dt=I32), "ids: shape"),
    ("rows overlap", z(2, 3, 9, dt=F32), z(1, 3, 4, dt=I32).expand(2, 3, 4), "rows overlap"),
    ("strided", z(2, 3, 18, dt=F32)[..., ::2], z(2, 3, 4, dt=I32), "innermost"),
]


@pytest.mark.parametrize("name,x,ids,text", TOPK, ids=[f"{c[0]}-{i}" for i, c in enumerate(TOPK)])
def test_topk_refused(name, x, ids, text):
    st, msg = answer("mla_select_topk", d(x), d(ids), None)
    assert st == INVALID and text in msg, (st, msg)


def test_topk_overlap_and_size_refused():
    x = z(4, 9, dt=F32)
    st, msg = answer("mla_select_topk", d(x), d(x.view(I32)[:, :4]), None)
    assert st == INVALID and "overlaps" in msg
    x, ids = mla.describe(z(1, 1, dt=F32)), mla.describe(z(1, 1, dt=I32))
    for t in (x, ids):
        t.shape[0], t.stride[0] = 1 << 30, 1
    ids.data += 1 << 40
    st, msg = answer("mla_select_topk", ctypes.byref(x), ctypes.byref(ids), None)
    assert st == UNSUPPORTED and "index range" in msg


def test_topk_more_places_than_an_index_refused():
    """Places past a row's values are filled 1024 at a time: K within that of 2^31 would wrap."""
    x, ids = mla.describe(z(1, 4, dt=F32)), mla.describe(z(1, 1, dt=I32))
    ids.shape[1] = ids.stride[0] = (1 << 31) - 1
    ids.data += 1 << 40
    st, msg = answer("mla_select_topk", ctypes.byref(x), ctypes.byref(ids), None)
    assert st == UNSUPPORTED and "index range" in msg


# ---- prefix_attn
def prefix_args(kv="bf16", wire=False):
    row, dt = (272 if kv == "mx4" else 512), (BF16 if kv == "bf16" else U8)
    return dict(q_lat=z(4, 3, 16, 512), q_pe=z(4, 3, 16, 64), ckv=z(8, 64, row, dt=dt),
                kpe=z(8, 64, 64, dt=U8 if kv == "fp8" else BF16), ptable=z(2, 6, dt=I32), plens=z(2, dt=I32),
                starts=z(3, dt=I32), table=z(4, 5, dt=I32), lens=z(4, dt=I32), q_lens=z(4, dt=I32),
                out=z(4, 3, 16, 512, dt=BF16 if wire else F32),
                lse=z(*((4, 3, 16, 2) if wire else (4, 3, 16)), dt=F32), scale=0.1,
                s=torch.ones(8) if kv == "fp8" else None,
                opts=opts(mla.PrefixOpts, out_format=1 if wire else 0))


def prefix_call(a):
    return answer("mla_prefix_attn", d(a["q_lat"]), d(a["q_pe"]), d(a["ckv"], a["s"]), d(a["kpe"], a["s"]),
                  *[d(a[k]) for k in ("ptable", "plens", "starts", "table", "lens", "q_lens")],
                  ctypes.c_float(a["scale"]), d(a["out"]), d(a["lse"]),
                  ctypes.byref(a["opts"]) if a["opts"] is not None else None, None)


PREFIX = [
    ("q null", dict(q_lat=None), INVALID, "q_lat"),
    ("pool null", dict(kpe=None), INVALID, "null"),
    ("ckv fp32", dict(ckv=z(8, 64, 512, dt=F32)), INVALID, "bf16 or fp8"),
    ("prefix table int64", dict(ptable=z(2, 6, dt=torch.int64)), INVALID, "prefix_table: wrong dtype"),
    ("no groups", dict(ptable=z(0, 6, dt=I32), plens=z(0, dt=I32), starts=z(1, dt=I32)), INVALID, "one group"),
    ("prefix lens", dict(plens=z(3, dt=I32)), INVALID, "prefix_lens"),
    ("starts", dict(starts=z(2, dt=I32)), INVALID, "group_starts"),
    ("lens", dict(lens=z(3, dt=I32)), INVALID, "seq_lens"),
    ("q_lens", dict(q_lens=z(5, dt=I32)), INVALID, "q_lens"),
    ("B of q", dict(q_lat=z(3, 3, 16, 512)), INVALID, "q_lat: shape"),
    ("q_pe", dict(q_pe=z(4, 3, 16, 32)), INVALID, "q_pe: shape"),
    ("out dtype", dict(out=z(4, 3, 16, 512)), INVALID, "out_lat: wrong dtype"),
    ("out shape", dict(out=z(4, 3, 15, 512, dt=F32)), INVALID, "out_lat: shape"),
    ("lse shape", dict(lse=z(4, 3, 15, dt=F32)), INVALID, "out_lse: shape"),
    ("out rows overlap", dict(out=z(1, 3, 16, 512, dt=F32).expand(4, 3, 16, 512)), INVALID, "rows overlap"),
    ("q unaligned", dict(q_lat=off(z(4, 3, 16, 512), 1)), INVALID, "aligned"),
    ("q rows in two dims", dict(q_lat=z(4, 6, 16, 512)[:, :3]), UNSUPPORTED, "one dim"),
    ("out rows in two dims", dict(out=z(3, 4, 16, 512, dt=F32).transpose(0, 1)), UNSUPPORTED, "one dim"),
    ("scale nan", dict(scale=float("nan")), INVALID, "scale"),
    ("opts null", dict(opts=None), INVALID, "opts"),
    ("n_splits", dict(opts=opts(mla.PrefixOpts, n_splits=-1)), INVALID, "n_splits"),
    ("own_splits", dict(opts=opts(mla.PrefixOpts, own_splits=-1)), INVALID, "own_splits"),
    ("out_format", dict(opts=opts(mla.PrefixOpts, out_format=2)), INVALID, "out_format"),
    ("row_tile", dict(opts=opts(mla.PrefixOpts, row_tile=96)), INVALID, "row_tile"),
    ("128 rows of a 4-bit cache", dict(ckv=z(8, 64, 272, dt=U8), opts=opts(mla.PrefixOpts, row_tile=128)), UNSUPPORTED,
     "64-row"),
    ("reserved", dict(opts=opts(mla.PrefixOpts, reserved=1)), INVALID, "reserved"),
    ("groups", dict(ptable=z(4097, 6, dt=I32), plens=z(4097, dt=I32), starts=z(4098, dt=I32)), UNSUPPORTED, "4096"),
]


@pytest.mark.parametrize("name,change,status,text", PREFIX, ids=[c[0] for c in PREFIX])
def test_prefix_refused(name, change, status, text):
    a = prefix_args()
    a.update(change)
    st, msg = prefix_call(a)
    assert st == status and text in msg, (st, msg)


def test_prefix_overlaps_refused():
    a = prefix_args()
    a["lse"] = a["out"].view(-1)[:4 * 3 * 16].view(4, 3, 16)
    st, msg = prefix_call(a)
    assert st == INVALID and "overlap" in msg
    a = prefix_args()
    a["out"] = torch.zeros(4 * 3 * 16 * 512)[:].view(4, 3, 16, 512)
    a["plens"] = a["out"].view(-1).view(I32)[:2]
    st, msg = prefix_call(a)
    assert st == INVALID and "overlaps an input" in msg


@pytest.mark.parametrize("value", [-1, 2])
def test_window_of_whole_blocks_refused(value):
    from tests.test_step_abi import window_args, window_call, wopts
    a = window_args()
    a["opts"] = wopts(whole_blocks=value)
    st, msg = window_call(a)
    assert st == INVALID and "whole_blocks" in msg


def test_binding_refuses_host_tensors():
    a = prefix_args()
    calls = [
        lambda: mla.rope_append(z(5, 512), z(5, 64), z(5, dt=I32), z(5, dt=I32), z(2, 64, 512), z(2, 64, 64)),
        lambda: mla.block_means(z(4, 64, 512), z(4, 64, 64), z(7, dt=I32), z(4, 576)),
        lambda: mla.block_scores(a["q_lat"], a["q_pe"], z(9, 576), a["table"], a["lens"], 0.1),
        lambda: mla.select_topk(z(2, 9, dt=F32), 4),
        lambda: mla.prefix_attn(a["q_lat"], a["q_pe"], a["ckv"], a["kpe"], a["ptable"], a["plens"], a["starts"],
                                a["table"], a["lens"], 0.1)]
    for call in calls:
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(ValueError, match="give k"):
        mla.select_topk(z(2, 9, dt=F32))


@pytest.mark.parametrize("k", range(6))
def test_tensors_and_streams_of_another_device(monkeypatch, k):
    from tests.test_devices import Fake, Stream

    def calls(on, stream=None):
        def t(*shape):
            return Fake(*shape, on=on)
        q, qp, pool, kpool, table, lens = t(1, 1, 1, 512), t(1, 1, 1, 64), t(1, 64, 512), t(1, 64, 64), t(1, 1), t(1)
        out, lse = t(1, 1, 1, 512), t(1, 1, 1)
        return [
            lambda: mla.rope_append(t(1, 512), t(1, 64), lens, lens, pool, kpool, stream=stream),
            lambda: mla.block_means(pool, kpool, lens, t(1, 576), stream=stream),
            lambda: mla.block_scores(q, qp, t(1, 576), table, lens, 1.0, scores=t(1, 1, 1), stream=stream),
            lambda: mla.select_topk(t(1, 5), ids=t(1, 3), stream=stream),
            lambda: mla.prefix_attn(q, qp, pool, kpool, table, lens, t(2), table, lens, 1.0, out_lat=out, out_lse=lse,
                                    stream=stream),
            lambda: mla.prepare_prefix(q, qp, pool, kpool, table, lens, t(2), table, lens, 1.0, out_lat=out,
                                       out_lse=lse, stream=stream)]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="cuda:1, which is not the current device"):
        calls(1)[k]()
    with pytest.raises(ValueError, match="the stream is on cuda:1"):
        calls(0, Stream(1))[k]()


# ---- the references
def test_scores_reference_is_the_shares_of_attention():
    """Scores of a row sum to the number of heads; blocks of one key repeated
    64 times get exactly the attention that their tokens get."""
    rs = np.random.default_rng(0)
    q, keys = rs.standard_normal((1, 5, 576)), rs.standard_normal((6, 576))
    got, _ = C.scores(q, keys, np.ones(6, bool), 6 * 64, 1, 0, 0, 0.05)
    assert abs(got.sum() - 5) < 1e-12
    tokens = np.repeat(keys, 64, 0)
    want = 0
    for h in range(5):
        w = np.exp(tokens @ q[0, h] * 0.05)
        want = want + (w / w.sum()).reshape(6, 64).sum(1)
    assert np.allclose(got[0], want, rtol=1e-12)


@pytest.mark.parametrize("window,n_sink", [(0, 0), (1, 0), (64, 64), (100, 1), (1000, 0)])
def test_scores_reference_leaves_what_windows_attend(window, n_sink):
    """Blocks that may be chosen and tokens that a window of whole blocks sees
    are apart, and with sinks of whole blocks they are all of the sequence."""
    q, keys = np.ones((1, 1, 576)), np.zeros((8, 576))
    for n in (1, 63, 64, 65, 128, 300, 512):
        got, _ = C.scores(q, keys, np.ones(8, bool), n, 1, window, n_sink, 1.0)
        chosen = np.repeat(np.isfinite(got[0]), 64)
        p = n - 1
        lo = 64 * C.end_block(p, window)
        t = np.arange(512)
        seen = (t <= p) & ((t >= lo) | (t < n_sink))
        assert not (chosen & seen).any() and not (chosen & (t > p)).any()
        if n_sink % 64 == 0:
            assert ((chosen | seen) == (t <= p)).all()


def test_topk_reference():
    x = np.array([1.0, -np.inf, np.nan, 3.0, 3.0, -0.0, 0.0, np.inf])
    assert C.topk(x, 3) == [2, 3, 7] and C.topk(x, 4) == [2, 3, 4, 7]
    assert C.topk(x, 6) == [0, 2, 3, 4, 5, 7] and C.topk(x, 9) == [0, 2, 3, 4, 5, 6, 7, -1, -1]


def test_prefix_reference_is_the_whole_sequence():
    rs = np.random.default_rng(1)
    q, k = rs.standard_normal((3, 576)), rs.standard_normal((90, 576))
    got = C.prefix_row(q, (k[:70], k[:70, :512]), (k[70:], k[70:, :512]), 20, 12, 0.05)
    want = S.attend(q, k, k[:, :512], np.arange(90) <= 82, 0.05)
    assert all(np.allclose(got[key], want[key]) for key in ("out", "lse", "m", "l"))
