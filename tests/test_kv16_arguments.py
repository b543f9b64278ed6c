"""What the entry points of trees, prompts and the bf16 cache refuse, before any CUDA call: runs without a GPU."""
import ctypes

import numpy as np
import pytest

from oracle import trees
from paper_2605_13319_b200 import binding

P = 4096          # stands for an aligned device address: nothing here is launched
INVALID = binding.E_INVALID
GOOD = dict(n_layers=2, n_kv_heads=8, head_dim=128, page_size=16, n_pages=10, max_pages=4, reserved=0)
BAD_CFG = [dict(n_layers=0), dict(n_layers=65536), dict(n_kv_heads=0), dict(n_kv_heads=65536), dict(head_dim=96), dict(head_dim=256), dict(page_size=4), dict(page_size=12),
           dict(page_size=8192), dict(n_pages=0), dict(n_pages=1 << 28), dict(max_pages=0), dict(max_pages=1 << 28), dict(reserved=1)]


def cfg(**change):
    return binding.Kv16Cfg(*(GOOD | change).values())


ARGS = dict(
    append=dict(pool=P, layer=1, k=P, v=P, dtype=0, ks=1024, vs=1024, n_req=2, rows=5, row0=P, base=P, table=P),
    read=dict(pool=P, layer=0, k=P, v=P, n_req=2, rows=5, row0=P, base=P, table=P),
    attend=dict(pool=P, layer=0, q=P, out=P, dtype=0, qs=4096, os=4096, heads=32, scale=0.1, n_req=2, rows=5, row0=P, base=P, table=P, mask=P, words=1, scratch=P),
    reserve=dict(n_req=2, length=P, table=P, refs=P, pages=P, scratch=P),
    fork=dict(pool=P, n=2, src=P, dst=P, length=P, own=P, n_slots=4, table=P, refs=P, pages=P, scratch=P),
    compact=dict(pool=P, n_req=2, keep=P, words=1, base=P, table=P, kept=P),
    release=dict(n_req=2, length=P, table=P, refs=P))
POINTERS = "pool k v q out row0 base table length refs pages src dst own keep kept scratch".split()


def call(name, config=None, **change):
    return getattr(binding.lib(), "pipesd_kv16_" + name)(ctypes.byref(config or cfg()), *(ARGS[name] | change).values(), None)


@pytest.mark.parametrize("bad", BAD_CFG)
def test_configurations(bad):
    L, c = binding.lib(), cfg(**bad)
    assert L.pipesd_kv16_pool_bytes(ctypes.byref(c)) == 0 and L.pipesd_kv16_plan_scratch_bytes(ctypes.byref(c), 2) == 0
    assert L.pipesd_kv16_attend_scratch_bytes(ctypes.byref(c), 5, 32) == 0
    for name in ARGS:
        assert call(name, c) == INVALID


def test_sizes():
    L = binding.lib()
    assert L.pipesd_kv16_pool_bytes(ctypes.byref(cfg())) == 2 * 10 * 2 * 8 * 16 * 128 * 2
    assert L.pipesd_kv16_pool_bytes(ctypes.byref(cfg(head_dim=64, page_size=24))) == 2 * 10 * 2 * 8 * 24 * 64 * 2
    assert L.pipesd_kv16_pool_bytes(None) == 0
    for rows, heads in ((0, 32), (5, 0), (5, 12), (5, 8 * 129)):
        assert L.pipesd_kv16_attend_scratch_bytes(ctypes.byref(cfg()), rows, heads) == 0
    assert L.pipesd_kv16_attend_scratch_bytes(ctypes.byref(cfg()), 5, 32) > 0 and L.pipesd_kv16_plan_scratch_bytes(ctypes.byref(cfg()), 0) == 0


@pytest.mark.parametrize("name,bad", [(n, {a: None}) for n, args in ARGS.items() for a in args if a in POINTERS] + [
    (n, {a: 0}) for n, args in ARGS.items() for a in ("n_req", "rows", "n", "n_slots") if a in args] + [
    (n, {"layer": x}) for n in ("append", "read", "attend") for x in (-1, 2)] + [
    (n, {"pool": P + 8}) for n in ("append", "read", "attend", "fork", "compact")] + [
    ("append", dict(dtype=2)), ("append", dict(ks=1023)), ("append", dict(vs=0)), ("append", dict(k=P + 2)), ("append", dict(dtype=1, v=P + 1)),
    ("read", dict(k=P + 8)), ("read", dict(v=P + 2)), ("attend", dict(dtype=-1)), ("attend", dict(qs=4095)), ("attend", dict(os=4000)),
    ("attend", dict(heads=0)), ("attend", dict(heads=12)), ("attend", dict(heads=8 * 129, qs=1 << 20, os=1 << 20)), ("attend", dict(scale=0.0)),
    ("attend", dict(scale=-1.0)), ("attend", dict(scale=float("nan"))), ("attend", dict(scale=float("inf"))), ("attend", dict(scratch=P + 4)),
    ("attend", dict(q=P + 1)), ("attend", dict(out=P + 2)), ("attend", dict(words=0)), ("attend", dict(words=257)), ("compact", dict(words=0)),
    ("compact", dict(words=1 << 26)), ("reserve", dict(scratch=P + 2)), ("fork", dict(scratch=P + 1))])
def test_arguments(name, bad):
    assert call(name, **bad) == INVALID


TREE = dict(n_req=2, rows=5, row0=P, parent=P, words=1, mask=P, depth=P)
PACKED = dict(q=P, k=P, v=P, out=P, qs=4096, ks=1024, vs=1024, os=4096, heads=32, kv_heads=8, hd=128, scale=0.1, n_req=1, rows=9, row0=P)


@pytest.mark.parametrize("bad", [dict(n_req=0), dict(rows=0), dict(row0=None), dict(parent=None), dict(words=0), dict(words=257), dict(mask=None), dict(depth=None)])
def test_trees(bad):
    assert binding.lib().pipesd_tree_mask(*(TREE | bad).values(), None) == INVALID


@pytest.mark.parametrize("bad", [{a: None} for a in ("q", "k", "v", "out", "row0")] + [{a: P + 8} for a in ("q", "k", "v", "out")] + [
    dict(qs=4095), dict(ks=1000), dict(vs=1020), dict(os=4088 - 4096), dict(qs=4100), dict(heads=0), dict(heads=12), dict(heads=8 * 129, qs=1 << 20, os=1 << 20),
    dict(kv_heads=0), dict(hd=96), dict(hd=32), dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(n_req=0), dict(rows=0)])
def test_packed(bad):
    assert binding.lib().pipesd_attend_packed(*(PACKED | bad).values(), None) == INVALID


def test_binding_checks_shapes():
    import torch
    q, kv, row0 = torch.zeros((4, 4, 64), dtype=torch.bfloat16), torch.zeros((4, 2, 64), dtype=torch.bfloat16), torch.tensor([0, 4], dtype=torch.int32)
    for bad in ((q.float(), kv, kv), (q, kv[:3], kv[:3]), (q, kv, kv[:, :1]), (q[0], kv, kv), (q, kv[..., :32], kv[..., :32])):
        with pytest.raises(AssertionError):
            binding.attend_packed(*bad, row0)
    with pytest.raises(binding.PipesdError):
        binding.Kv16Cache(8, 96, n_pages=4)
    with pytest.raises(binding.PipesdError):
        binding.Kv16Cache(8, 64, n_pages=4, page_size=12)
    with pytest.raises(AssertionError):
        binding.Kv16Cache(8, 64, pool=torch.zeros((1, 4, 2, 8, 2, 8, 8, 8), dtype=torch.bfloat16))      # not on a CUDA device


def test_plain_forms_agree_with_themselves():
    """What the GPU tests compare with: pages handed out and taken back leave the references as they were."""
    rng = np.random.default_rng(0)
    page, table, refs = 16, np.full((6, 5), -1, np.int32), np.zeros(20, np.int32)
    assert trees.reserve([40, 16, 0], table[:3], refs, page) == [3, 1, 0]
    assert table[0, :3].tolist() == [0, 1, 2] and table[1, 0] == 3
    assert trees.fork([0, 0, 1], [3, 4, 5], [40, 40, 10], [32, 20, 16], table, refs, page) == [3, 3, 1]
    assert table[3].tolist() == [0, 1, 4, -1, -1] and table[4].tolist() == [0, 5, 6, -1, -1] and table[5, 0] == 3
    assert refs[:8].tolist() == [3, 2, 1, 2, 1, 1, 1, 0]
    trees.release([0] * 6, table, refs, page)
    assert (refs == 0).all() and (table == -1).all()
    mask, depth = trees.ancestors([-1, 0, 0, 2, 5, -1], 1)
    assert mask[:, 0].tolist() == [1, 3, 5, 13, 16, 32] and depth.tolist() == [0, 1, 1, 2, 0, 0]
    assert trees.bits_of(mask, 40)[3].nonzero()[0].tolist() == [0, 2, 3]
    rows = rng.integers(0, 100, (2, 64)).astype(np.uint16)
    pool = trees.Pool(np.zeros((1, 3, 2, 2, 8 * 64), np.uint16), 64, 8)
    pool.put([2, 0], 9, 0, 1, rows)
    assert np.array_equal(pool.get([2, 0], 9, 0, 1), rows) and pool.get([2, 0], 16, 0, 1) is None
    assert pool.compact([2, 0], 7, [0, 2, 50]) == 2 and np.array_equal(pool.get([2, 0], 8, 0, 1), rows)
