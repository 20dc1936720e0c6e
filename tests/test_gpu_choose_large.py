"""The choice of blocks and shared prefixes over pools past 4 GiB, from several host
threads on one stream, and on streams of their own beside each other."""
import threading

import numpy as np
import pytest
import torch

from paper_2606_01502_amd import mla
from tests import step_helpers as T

pytestmark = pytest.mark.gpu
SCALE = 0.0721688


def blocks_of(seed, n):
    return T.randn(seed, n, 64, 512, sigma=0.5), T.randn(seed + 1, n, 64, 64, sigma=0.5)


@pytest.fixture(scope="module")
def pools():
    """A pool of 70,000 blocks (4.6 GB of latents), eight of them filled, and the same
    eight in a pool of their own."""
    P, at = 70000, np.array([69999, 3, 65537, 40000, 69998, 0, 58255, 66000])
    ckv = torch.empty((P, 64, 512), dtype=torch.bfloat16, device="cuda")
    kpe = torch.empty((P, 64, 64), dtype=torch.bfloat16, device="cuda")
    small = blocks_of(1, 8)
    ckv[torch.from_numpy(at).cuda()], kpe[torch.from_numpy(at).cuda()] = small
    return (ckv, kpe), small, at


def test_means_and_prefixes_past_4_gib(pools):
    big, small, at = pools
    means = torch.zeros((len(big[0]), 576), dtype=torch.bfloat16, device="cuda")
    mla.block_means(*big, T.i32(at * 64 + 63), means)
    want = torch.zeros((8, 576), dtype=torch.bfloat16, device="cuda")
    mla.block_means(*small, T.i32(np.arange(8) * 64 + 63), want)
    assert torch.equal(means[torch.from_numpy(at).cuda()], want)
    q = T.randn(5, 4, 1, 128, 512), T.randn(6, 4, 1, 128, 64)
    local = np.arange(8)
    for row_tile in (64, 128):
        got, ref = (mla.prefix_attn(*q, *p, T.i32(t[None, :4]), T.i32([250]), T.i32([0, 4]), T.i32(t[4:, None]),
                                    T.i32([64, 1, 7, 40]), SCALE, row_tile=row_tile)
                    for p, t in ((big, at), (small, local)))
        torch.cuda.synchronize()
        assert all(torch.equal(g, r) for g, r in zip(got, ref))


def test_appended_past_4_gib(pools):
    big, small, at = pools
    new = T.randn(9, 3, 576)
    ckv, kpe = big[0].clone(), big[1].clone()
    slots = T.i32(at[[0, 2, 7]] * 64 + [63, 0, 5])
    mla.rope_append(new[:, :512], new[:, 512:], T.i32([5, 6, 7]), slots, ckv, kpe)
    s_ckv, s_kpe = small[0].clone(), small[1].clone()
    mla.rope_append(new[:, :512], new[:, 512:], T.i32([5, 6, 7]), T.i32(np.array([0, 2, 7]) * 64 + [63, 0, 5]), s_ckv, s_kpe)
    i = torch.from_numpy(at).cuda()
    assert torch.equal(ckv[i], s_ckv) and torch.equal(kpe[i], s_kpe)


def test_scores_by_means_past_4_gib():
    P = 4_000_000
    means = torch.empty((P, 576), dtype=torch.bfloat16, device="cuda")
    at = np.array([P - 1, 0, 3_728_271, 3_728_270, 1_864_136, P - 2])
    rows = T.randn(3, 6, 576, sigma=0.5)
    means[torch.from_numpy(at).cuda()] = rows
    q = T.randn(4, 1, 2, 33, 512), T.randn(5, 1, 2, 33, 64)
    got = mla.block_scores(*q, means, T.i32(at[None]), T.i32([384]), SCALE)
    want = mla.block_scores(*q, rows, T.i32([[0, 1, 2, 3, 4, 5]]), T.i32([384]), SCALE)
    assert torch.equal(got, want)


def calls(seed):
    """Calls that split, of sizes that go by the seed, as functions of no arguments."""
    B, NB, H = 1 + seed, 100 + 40 * seed, 16 * (1 + seed)
    table = T.i32(np.random.default_rng(seed).permutation(B * NB).reshape(B, NB))
    q = T.randn(seed, B, 1, H, 512), T.randn(seed + 1, B, 1, H, 64)
    means, lens = T.randn(seed + 2, B * NB, 576, sigma=0.5), T.i32([64 * NB - seed] * B)
    x = T.randn(seed + 3, 2, 20000 + 9000 * seed).float()
    ckv, kpe = blocks_of(seed + 10, 12)
    ptable, own = T.i32(np.arange(8)[None]), T.i32(np.resize([8, 9, 10, 11], (B, 1)))
    plens, starts, mine = T.i32([512 - seed]), T.i32([0, B]), T.i32([3 + seed] * B)
    return [lambda: (mla.block_scores(*q, means, table, lens, SCALE),),
            lambda: (mla.select_topk(x, 300),),
            lambda: mla.prefix_attn(*q, ckv, kpe, ptable, plens, starts, own, mine, SCALE, n_splits=3)]


@pytest.mark.parametrize("streams", [1, 4])
def test_threads(streams):
    jobs = [calls(k) for k in range(4)]
    torch.cuda.synchronize()
    own = [torch.cuda.Stream() for _ in range(streams)]
    want = [[f() for f in fs] for fs in jobs]
    torch.cuda.synchronize()
    got, wrong = [[] for _ in jobs], []

    def work(k):
        try:
            with torch.cuda.stream(own[k % streams]):
                for _ in range(12):
                    got[k].append([f() for f in jobs[k]])
        except Exception as e:  # noqa: BLE001 (shown by the main thread)
            wrong.append(e)
    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong, wrong
    for k in range(4):
        for one in got[k]:
            for a, b in zip(one, want[k]):
                assert all(torch.equal(x, y) for x, y in zip(a, b)), f"thread {k}"
