"""Tensors, streams and prepared calls of another device than the current one are
refused before anything is launched (two devices played on the CPU)."""
import pytest
import torch

from paper_2606_01502_amd import mla


class Fake:
    """A tensor as far as the binding looks at it before it describes it."""
    is_cuda = True
    requires_grad = False
    dtype = torch.bfloat16

    def __init__(self, *shape, on=1):
        self.shape, self.on, self.device = shape, on, f"cuda:{on}"

    def get_device(self):
        return self.on

    def dim(self):
        return len(self.shape)


class Stream:
    cuda_stream = 0

    def __init__(self, on):
        self.device_index = on


def calls(on, stream=None):
    def t(*shape):
        return Fake(*shape, on=on)
    q, qp, pool, kpool, out, lse = t(1, 1, 1, 512), t(1, 1, 1, 64), t(1, 64, 512), t(1, 64, 64), t(1, 1, 1, 512), t(1, 1, 1)
    table, ids, lens = t(1, 1), t(1, 1), t(1)
    attn = dict(out_lat=out, out_lse=lse, stream=stream)
    slots = dict(slots=t(1), positions=t(1), seq_lens=t(1), starts=t(2), info=t(4), stream=stream)
    return [
        lambda: mla.sparse_partial_attn(q, qp, pool, kpool, table, ids, 1.0, **attn),
        lambda: mla.prepare_partial(q, qp, pool, kpool, table, ids, 1.0, **attn),
        lambda: mla.window_attn(q, qp, pool, kpool, table, lens, 1.0, **attn),
        lambda: mla.merge_partials([out], [lse], out=out, out_lse=lse, stream=stream),
        lambda: mla.prepare_merge([out], [lse], out=out, stream=stream),
        lambda: mla.fetch_gather(pool, kpool, lens, ids, out_ckv=out, out_kpe=out, stream=stream),
        lambda: mla.fetch_splice(out, out, pool, kpool, lens, 0, 0, stream=stream),
        lambda: mla.batch_slots(lens, lens, lens, table, **slots),
        lambda: mla.rope(t(1, 1, 64), lens, out=t(1, 1, 64), stream=stream),
        lambda: mla.cache_append(q, qp, lens, pool, kpool, stream=stream)]


@pytest.mark.parametrize("k", range(10))
def test_tensors_of_another_device(monkeypatch, k):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="cuda:1, which is not the current device"):
        calls(1)[k]()


@pytest.mark.parametrize("k", range(10))
def test_a_stream_of_another_device(monkeypatch, k):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="cuda:0, the stream is on cuda:1"):
        calls(0, Stream(1))[k]()


def test_a_prepared_call_under_another_device(monkeypatch):
    monkeypatch.setattr(mla, "_several_gpus", lambda: True)
    current, made = [0], []
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])

    def fn(x):
        made.append(x)
        return mla.MLA_OK
    call = mla._Prepared(fn, (7,), None, "result", 0)
    assert call() == "result" and made == [7]
    current[0] = 1
    with pytest.raises(ValueError, match="prepared on cuda:0"):
        call()
    assert made == [7]
