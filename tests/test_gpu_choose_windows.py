"""What a row may choose and what mla_window_attn with whole_blocks attends, by the
calls themselves: with a window of 1 or more in both they share no token and leave
none out; with window 0 the one offers all whole blocks and the other attends all."""
import numpy as np
import pytest
import torch

from oracle import step as S
from paper_2606_01502_amd import mla
from tests import step_helpers as T

pytestmark = pytest.mark.gpu
SCALE = 0.0721688
F = float(np.float32(SCALE))
LENS = [1, 63, 64, 65, 128, 700, 768]
B, H, NB = len(LENS), 16, 12


class Step:
    def __init__(self, Mq):
        self.c = T.Cache(Mq, B * NB, "bf16")
        self.Mq, self.table = Mq, np.random.default_rng(Mq).permutation(B * NB).reshape(B, NB)
        self.q = T.randn(Mq, B, Mq, H, 512), T.randn(Mq + 1, B, Mq, H, 64)
        self.means = torch.zeros((B * NB, 576), dtype=torch.bfloat16, device="cuda")
        mla.block_means(self.c.ckv, self.c.kpe, T.i32(np.arange(B * NB) * 64 + 63), self.means)
        self.tab, self.lens = T.i32(self.table), T.i32(LENS)

    def scores(self, **kw):
        return mla.block_scores(*self.q, self.means, self.tab, self.lens, SCALE, **kw)

    def chosen(self, ids):
        if self.Mq == 1:
            ids = ids[:, 0].contiguous()
        return mla.sparse_partial_attn(*self.q, self.c.ckv, self.c.kpe, self.tab, ids, SCALE)

    def near(self, **kw):
        return mla.window_attn(*self.q, self.c.ckv, self.c.kpe, self.tab, self.lens, SCALE, **kw)


@pytest.mark.parametrize("Mq", [1, 3])
@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 130, 5000])
@pytest.mark.parametrize("n_sink", [0, 64, 128, 6400])
def test_every_block_chosen_is_all_of_the_sequence(Mq, window, n_sink):
    print(f"case: all chosen {Mq} {window} {n_sink}", flush=True)
    s = Step(Mq)
    sc = s.scores(window=window, n_sink=n_sink)
    ids = mla.select_topk(sc, NB)
    a, b = s.chosen(ids), s.near(window=window, n_sink=n_sink, whole_blocks=True)
    out, lse = mla.merge_partials([a[0], b[0]], [a[1], b[1]], out_lse=True)
    torch.cuda.synchronize()
    o, st, picks = T.host(out), T.host(lse), ids.cpu().numpy()
    q = np.concatenate([T.host(s.q[0]), T.host(s.q[1])], -1)
    for r, n in enumerate(LENS):
        keys, values = s.c.tokens(s.table[r])
        t = np.arange(len(keys))
        for i in range(Mq):
            p = n - Mq + i
            # what the window attends, as its declaration says, and the choice beside it
            see = (t <= p) & ((t >= 64 * ((p - window + 1) // 64)) | (t < n_sink))
            for j in picks[r, i][picks[r, i] >= 0]:
                assert not see[64 * j:64 * j + 64].any(), "chosen and attended anyway"
                see[64 * j:64 * j + 64] = True
            assert np.array_equal(see, t <= p), "neither chosen nor attended, or behind the row"
            # (either part is within its own bound, and their shares of a row add up to 1)
            T.check_row(S.attend(q[r, i], keys, values, t <= p, F), o[r, i], st[r, i], False, f"request {r} row {i}")


@pytest.mark.parametrize("Mq", [1, 3])
def test_window_0_says_all_in_the_one_and_none_in_the_other(Mq):
    s = Step(Mq)
    sc = T.host(s.scores())
    full, whole = s.near(), s.near(whole_blocks=True)
    a = s.chosen(mla.select_topk(s.scores(), NB))
    _, lse = mla.merge_partials([a[0], whole[0]], [a[1], whole[1]], out_lse=True)
    torch.cuda.synchronize()
    assert torch.equal(full[0], whole[0]) and torch.equal(full[1], whole[1])
    for r, n in enumerate(LENS):
        for i in range(Mq):
            assert np.isfinite(sc[r, i]).sum() == max(n - Mq + i + 1, 0) // 64
    # so that joined they count those blocks twice
    la, lf, got = T.host(a[1]), T.host(full[1]), T.host(lse)
    live = np.isfinite(la)
    assert live.any() and (got[live] > lf[live] + 1e-3).all()
    assert np.allclose(got[live], np.logaddexp(la, lf)[live], rtol=0, atol=1e-4)


def test_scores_of_given_splits_are_refused_without_a_workspace():
    """A stream that is being captured cannot grow its workspace: the call takes one
    split where the number is left to it (see test_gpu_choose.py) and is refused
    where several are asked for; the capture goes on."""
    s = Step(1)
    # 256 query rows of 128 heads in 4096 splits: a gigabyte of statistics
    q = torch.zeros((1, 256, 128, 512), dtype=torch.bfloat16, device="cuda")
    wide = torch.zeros((1, 1 << 18), dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        many = mla.prepare_block_scores(q, q[..., :64].contiguous(), s.means, wide, T.i32([1]), SCALE, n_splits=4096)
        many.result.fill_(7.0)
        out = torch.zeros((B, 1, NB), device="cuda")
        one = mla.prepare_block_scores(*s.q, s.means, s.tab, s.lens, SCALE, scores=out, n_splits=1)
        # (a table of one tile holds one split, which needs no workspace)
        two = mla.prepare_block_scores(*s.q, s.means, s.tab, s.lens, SCALE, n_splits=2)
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            with pytest.raises(mla.MlaError, match="capture"):
                many()
            one()
            two()
        for _ in range(3):
            out.zero_()
            g.replay()
            stream.synchronize()
            want = s.scores(n_splits=1)
            stream.synchronize()
            assert torch.equal(out, want) and torch.equal(two.result, want)
        assert (many.result == 7.0).all()
