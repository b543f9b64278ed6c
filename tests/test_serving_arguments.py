"""What the serving entry points refuse, before any CUDA call: runs without a GPU."""
import ctypes

import numpy as np
import pytest

from paper_2605_13319_b200 import binding

P = 4096          # stands for an aligned device address: nothing here is launched
INVALID = binding.E_INVALID


def sample(logits=P, dtype=binding.F32, stride=1024, rows=2, vocab=1024, shaping=P, u=P, tokens=P, probs=None, probs_stride=0):
    return binding.lib().pipesd_sample(logits, dtype, stride, rows, vocab, shaping, u, tokens, probs, probs_stride, None)


@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(shaping=None), dict(u=None), dict(tokens=None), dict(dtype=2), dict(dtype=-1), dict(rows=0), dict(rows=-3),
    dict(vocab=0), dict(vocab=(1 << 18) + 1, stride=1 << 19), dict(stride=1023), dict(stride=-1024), dict(logits=P + 2),
    dict(dtype=binding.BF16, logits=P + 1), dict(probs=P, probs_stride=1023), dict(probs=P, probs_stride=1024),
])
def test_sample_refuses(bad):
    assert sample(**bad) == INVALID


def accept(logits=P, dtype=binding.F32, stride=1024, n_req=2, rows=6, vocab=1024, row0=P, shaping=P, q=P, q_stride=1024, drafts=P, u=P, n=P,
           token=P, scratch=P):
    return binding.lib().pipesd_accept(logits, dtype, stride, n_req, rows, vocab, row0, shaping, q, q_stride, drafts, u, n, token, scratch, None)


@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(row0=None), dict(shaping=None), dict(q=None), dict(drafts=None), dict(u=None), dict(n=None), dict(token=None),
    dict(scratch=None), dict(scratch=P + 4), dict(n_req=0), dict(n_req=7), dict(rows=0), dict(dtype=5), dict(stride=1000), dict(q_stride=1000),
    dict(vocab=1 << 19, stride=1 << 19), dict(n_req=65536, rows=70000),
])
def test_accept_refuses(bad):
    assert accept(**bad) == INVALID
    assert binding.lib().pipesd_accept_scratch_bytes(0) == 0 and binding.lib().pipesd_accept_scratch_bytes(3) > 0


GOOD = dict(n_kv_heads=8, head_dim=128, page_size=16, n_pages=10, max_pages=4, reserved=0)
BAD_CFG = [dict(n_kv_heads=0), dict(head_dim=96), dict(head_dim=256), dict(page_size=8), dict(page_size=24), dict(page_size=8192), dict(n_pages=0),
           dict(max_pages=0), dict(max_pages=1 << 28), dict(reserved=1)]


def cfg(**change):
    return binding.Kv4Cfg(*(GOOD | change).values())


@pytest.mark.parametrize("bad", BAD_CFG)
def test_kv4_refuses_configurations(bad):
    L, c = binding.lib(), ctypes.byref(cfg(**bad))
    assert L.pipesd_kv4_pool_bytes(c) == 0 and L.pipesd_kv4_attend_scratch_bytes(c) == 0
    assert L.pipesd_kv4_append(c, P, P, P, 0, 1024, 1024, 1, 1, P, P, P, None) == INVALID
    assert L.pipesd_kv4_read(c, P, P, P, 1, 1, P, P, P, None) == INVALID
    assert L.pipesd_kv4_attend(c, P, P, P, 0, 1024, 1024, 8, 0.1, 1, 1, P, P, P, P, None) == INVALID


def test_kv4_sizes():
    assert binding.lib().pipesd_kv4_pool_bytes(ctypes.byref(cfg())) == 10 * 8 * 20 * 128
    assert binding.lib().pipesd_kv4_pool_bytes(ctypes.byref(cfg(head_dim=64, page_size=48))) == 10 * 8 * 3 * 20 * 64
    assert binding.lib().pipesd_kv4_pool_bytes(None) == 0


def call(name, **change):
    args = dict(append=dict(pool=P, k=P, v=P, dtype=0, ks=1024, vs=1024, n_req=2, rows=5, row0=P, base=P, table=P),
                read=dict(pool=P, k=P, v=P, n_req=2, rows=5, row0=P, base=P, table=P),
                attend=dict(pool=P, q=P, out=P, dtype=0, qs=4096, os=4096, heads=32, scale=0.1, n_req=2, rows=5, row0=P, base=P, table=P, scratch=P))[name]
    return getattr(binding.lib(), "pipesd_kv4_" + name)(ctypes.byref(cfg()), *(args | change).values(), None)


@pytest.mark.parametrize("name,bad", [(n, {a: None}) for n, names in (
    ("append", "pool k v row0 base table"), ("read", "pool k v row0 base table"), ("attend", "pool q out row0 base table scratch"))
    for a in names.split()] + [(n, b) for n in ("append", "read", "attend") for b in (dict(pool=P + 8), dict(n_req=0), dict(rows=0))] + [
    ("append", dict(dtype=3)), ("append", dict(ks=1023)), ("append", dict(vs=0)), ("append", dict(k=P + 2)), ("append", dict(dtype=1, v=P + 1)),
    ("read", dict(k=P + 4)), ("read", dict(v=P + 8)), ("attend", dict(dtype=-1)), ("attend", dict(qs=4095)), ("attend", dict(os=4000)),
    ("attend", dict(heads=0)), ("attend", dict(heads=12)), ("attend", dict(scale=0.0)), ("attend", dict(scale=-1.0)), ("attend", dict(scale=float("nan"))),
    ("attend", dict(scale=float("inf"))), ("attend", dict(scratch=P + 4)), ("attend", dict(q=P + 1)), ("attend", dict(out=P + 2))])
def test_kv4_refuses_arguments(name, bad):
    assert call(name, **bad) == INVALID


def test_settings_are_checked_on_the_host():
    s = binding.shaping(3, temperature=[0.0, 1.0, 0.5], top_k=[0, 5, -1], top_p=0.9, min_p=0.1, device="cpu").numpy()
    assert s.shape == (3, 4) and s.dtype == np.int32
    assert s[:, 0].view(np.float32).tolist() == [0.0, 1.0, 0.5] and s[:, 1].tolist() == [0, 5, -1]
    for bad in (dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(top_p=0.0), dict(top_p=float("nan")),
                dict(min_p=-0.1), dict(min_p=1.5), dict(min_p=float("nan"))):
        with pytest.raises(ValueError):
            binding.shaping(2, device="cpu", **bad)


class _Tensor:
    def __init__(self, cuda=True):
        self.is_cuda, self.on = cuda, []

    def record_stream(self, stream):
        self.on.append(stream)


def test_streams_belong_to_the_tensors_device():
    import torch
    other = type("Stream", (), {"device": torch.device("cuda", 1)})()
    with pytest.raises(AssertionError, match="stream"):
        binding._on(torch.device("cuda", 0), other)
    binding._on(torch.device("cuda", 1), other)


def test_memory_is_kept_for_a_stream_of_its_own(monkeypatch):
    import contextlib
    import torch
    monkeypatch.setattr(torch.cuda, "device", lambda i: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    home = type("Stream", (), {"cuda_stream": 7})()
    monkeypatch.setattr(torch.cuda, "current_stream", lambda i: home)
    side = type("Stream", (), {"device": torch.device("cuda", 0)})()
    given, on_host, made = _Tensor(), _Tensor(False), _Tensor()
    on = binding._on(torch.device("cuda", 0), side, given, None, on_host)
    with on as st:
        on.made(made)
    assert st == 7 and given.on == [side] and on_host.on == [] and made.on == [home]
