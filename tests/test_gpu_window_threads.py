"""Windows whose splits are shared out by length, from several threads: the shares
lie in the stream's workspace, written by one kernel and read by the next."""
import threading

import numpy as np
import pytest
import torch

from paper_2606_01502_amd import mla
from tests import step_helpers as T
from tests import test_gpu_window as win
from tests import window_probe as P

pytestmark = pytest.mark.gpu
SIZES = [(20, 1, 16, 66), (40, 1, 16, 48), (9, 2, 64, 120), (12, 2, 32, 200)]  # requests, rows, heads, blocks


def test_these_calls_share_their_splits(tmp_path):
    exe = P.build(str(tmp_path))
    for k, kv in enumerate(T.KVS):
        B, Mq, H, NB = SIZES[k]
        (p, _), = P.plans(exe, [P.Call(B, Mq, H, NB, NB, "fp8" if kv == "fp8split" else kv)])
        assert p.shares and p.S > 1, (kv, p)


def _make(k):
    B, Mq, H, NB = SIZES[k]
    c, ql, qp, table = win.pooled(70 + k, B, Mq, H, NB, 37, T.KVS[k])
    tab = T.i32(table)
    rs = np.random.default_rng(k)
    spreads = []
    for s in range(3):  # one long among short ones, any, alike
        lens = [rs.integers(0, 200, B), rs.integers(0, NB * 64 + 1, B), np.full(B, NB * 64 - 70)][s]
        if s == 0:
            lens[rs.integers(B)] = NB * 64
        spreads.append(T.i32(lens))

    def run(i):
        return mla.window_attn(ql, qp, c.ckv, c.kpe, tab, spreads[i % 3], win.SCALE, wire=bool(k & 1), **c.scales)
    return run


@pytest.mark.parametrize("own_streams", [True, False])
def test_threads_at_once(own_streams):
    """Four threads, each on a stream of its own or all on one; every call's lengths
    are others than the last one's.  Each result is that of the lone call."""
    print(f"case: shares from threads {own_streams}", flush=True)
    runs = [_make(k) for k in range(4)]
    want = [[[t.clone() for t in run(i)] for i in range(3)] for run in runs]
    torch.cuda.synchronize()
    one = torch.cuda.Stream()
    failed = []

    def work(k):
        try:
            s = torch.cuda.Stream() if own_streams else one
            with torch.cuda.stream(s):
                for i in range(24):
                    got = runs[k](i)
                    s.synchronize()
                    if not all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want[k][i % 3])):
                        failed.append((k, i))
        except Exception as e:  # shown by the assertion below
            failed.append((k, repr(e)))

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(timeout=100)
    assert not any(t.is_alive() for t in threads) and not failed, failed
