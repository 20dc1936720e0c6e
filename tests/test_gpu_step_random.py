"""Random calls of a serving step's operators on the GPU, each against its
float64 or exact reference: windows over every cache type, block selections of
4-bit caches, rotations, tables and slots, writes.  And calls from several
threads and streams at once."""
import threading

import numpy as np
import pytest
import torch

from paper_2606_01502_amd import mla
from tests import step_helpers as T
from tests import test_gpu_mx4 as mx4
from tests import test_gpu_step as step
from tests import test_gpu_window as win

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", range(40))
def test_windows(seed):
    rs = np.random.default_rng([seed, 77])
    kv = T.KVS[seed % 4]
    B, NB = int(rs.integers(1, 7)), int(rs.integers(1, 14))
    Mq, H = int(rs.choice([1, 1, 2, 5, 33])), int(rs.choice([1, 2, 7, 8, 16, 24, 65, 128]))
    if Mq * H > 600:
        Mq = 1
    c, ql, qp, table = win.inputs(seed, B, Mq, H, NB, kv)
    lens = rs.integers(0, NB * 64 + 40, B)
    q_lens = rs.integers(0, Mq + 2, B) if rs.random() < 0.5 else None
    table = np.where(rs.random(table.shape) < 0.1, rs.choice([-1, len(c.lat), 2 ** 31 - 1]), table)
    kw = dict(window=int(rs.choice([0, rs.integers(1, 40), rs.integers(1, NB * 64 + 1)])),
              n_sink=int(rs.choice([0, 1, rs.integers(0, 140)])), wire=bool(rs.random() < 0.5),
              n_splits=int(rs.choice([0, 0, 1, 3, 40])), row_tile=int(rs.choice([0, 0, 64, 64 if kv == "mx4" else 128])),
              scale=float(rs.choice([0.0721688, 0.3, -0.05])))
    print(f"case: random window {seed} {kv} {B} {Mq} {H} {NB} {lens} {q_lens} {kw}", flush=True)
    win.check(c, ql, qp, table, lens, q_lens, **kw)


@pytest.mark.parametrize("seed", range(16))
def test_blocks_of_4_bits(seed):
    rs = np.random.default_rng([seed, 78])
    R, NB = int(rs.integers(1, 6)), int(rs.integers(1, 40))
    Mq, H = int(rs.integers(1, 4)), int(rs.choice([1, 5, 8, 16, 33, 64, 128]))
    K = int(rs.integers(1, NB + 1))
    kw = dict(wire=bool(rs.random() < 0.5), n_splits=int(rs.choice([0, 0, 1, 4])), no_alloc=bool(rs.random() < 0.3))
    print(f"case: random 4-bit blocks {seed} {R} {Mq} {H} {NB} {K} {kw}", flush=True)
    mx4.check(*mx4.inputs(seed, R, Mq, H, NB, K), **kw)


@pytest.mark.parametrize("seed", range(24))
def test_rope(seed):
    rs = np.random.default_rng([seed, 79])
    rot = 2 * int(rs.integers(1, 129))
    at, tail = int(rs.integers(0, 40)), int(rs.integers(0, 40))
    n, H = int(rs.integers(1, 90)), int(rs.choice([1, 2, 3, 16, 40, 128]))
    x = step.randn(seed, n, H, at + rot + tail, dtype=torch.float32 if seed % 3 == 0 else torch.bfloat16)
    if seed % 4 == 1:  # (heads outermost in memory)
        x = x.transpose(0, 1).contiguous().transpose(0, 1)
    print(f"case: random rope {seed} {tuple(x.shape)} {at} {rot}", flush=True)
    step._check_rope(x, rs.integers(-2 ** 20, 2 ** 20, n), at, rot, seed % 2, inverse=bool(seed & 2),
                     **step.SCALINGS[int(rs.integers(0, 3))])


@pytest.mark.parametrize("seed", range(12))
def test_slots_and_writes(seed):
    rs = np.random.default_rng([seed, 80])
    B, NB = int(rs.integers(1, 900)), int(rs.integers(1, 9))
    cached, new, free, table = step._slots_case(seed, B, NB, int(rs.integers(0, 3 * B + 1)), 0, most=int(rs.integers(2, 300)))
    print(f"case: random slots {seed} {B} {NB} {len(free)}", flush=True)
    step._check_slots(cached, new, free, table, int(rs.integers(0, new.sum() + 50)), strided=bool(seed & 1))
    n, P = int(rs.integers(0, 6000)), int(rs.integers(94, 120))
    print(f"case: random append {seed} {n} {P}", flush=True)
    step._check_append(*step._append_case(seed, n, P, bool(seed & 1)))


def test_threads_and_streams_at_once():
    """Four threads with a stream and sizes of their own, whole steps at once:
    each result is that of the lone call."""
    def make(k):
        kv = T.KVS[k]
        c, ql, qp, table = win.inputs(50 + k, 3 + k, 2, 16 * (k + 1), 9, kv)
        tab, lens = T.i32(table), T.i32([100 + 90 * k + 30 * b for b in range(3 + k)])
        x, pos = step.randn(k, 40 + k, 8, 64), T.i32(np.arange(40 + k))
        pool, kpool = torch.zeros(4, 64, 272, dtype=torch.uint8, device="cuda"), torch.zeros(4, 64, 64, device="cuda").bfloat16()
        src, slots = step.randn(k + 9, 40 + k, 512), T.i32(np.random.default_rng(k).permutation(256)[:40 + k])

        def run():
            out, lse = mla.window_attn(ql, qp, c.ckv, c.kpe, tab, lens, 0.07, window=130, n_sink=3, n_splits=3, **c.scales)
            y = mla.rope(x, pos, rot_offset=0, rot_dim=64, pairing=0, base=1e4)
            mla.cache_append(src, y[:, 0], slots, pool, kpool)
            return out, lse, y, pool, kpool
        return run

    runs = [make(k) for k in range(4)]
    want = [[t.clone() for t in run()] for run in runs]
    torch.cuda.synchronize()
    failed = []

    def work(k):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(20):
                    got = runs[k]()
                    s.synchronize()
                    if not all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want[k])):
                        failed.append(k)
        except Exception as e:  # shown by the assertion below
            failed.append((k, repr(e)))

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
