"""The bf16 cache and its attention, further: rows in turn over rings, pages as long as tiles, long contexts, what sees only infinities."""
import numpy as np
import pytest

from oracle import trees
from test_gpu_kv16 import Case, _ints, _row0

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,hd", [(128, 128), (80, 128), (128, 64)])
@pytest.mark.parametrize("lengths", [[128, 256, 384], [128], [384], [640, 128, 129, 127]])
def test_single_tokens_of_wide_groups(heads, hd, lengths):
    """65 to 128 query rows a request: both streams take its tiles in turn, odd numbers of them among requests that end with a tile; many requests a CTA."""
    import torch
    total = [lengths[i % len(lengths)] for i in range(900)]
    c = Case(heads + len(lengths), [1] * len(total), [n - 1 for n in total], heads, 1, hd)
    c.fill()
    for dtype in (torch.bfloat16, torch.float32):
        q = c.queries(dtype)
        out = c.attend(q, None)
        c.check(q, None, out)
        assert all(torch.equal(out, c.attend(q, None)) for _ in range(20))


def test_more_pages_wanted_than_32_bits_count():
    """Sixteen requests of 2^27 pages each, 2^31 together: none is served, the small ones behind them are; nothing else changes."""
    import torch
    from paper_2605_13319_b200 import binding
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GB")
    width, page, n_pages = 1 << 27, 8, 64
    cache = binding.Kv16Cache(1, 64, n_pages=n_pages, page_size=page)
    before = cache.pool.normal_().clone()
    table, refs = torch.full((18, width), -1, dtype=torch.int32, device="cuda"), _ints(np.zeros(n_pages))
    refs[[0, 3, 5]] = 1
    assert cache.reserve(_ints([width * page] * 16 + [24, 8 * 59]), table, refs).tolist() == [-1] * 16 + [3, -1]
    assert (table[:16] == -1).all() and table[16, :4].tolist() == [1, 2, 4, -1] and (table[17] == -1).all()
    # a source that has every one of its pages, sixteen targets, and a small one behind them
    table[0] = 5
    got = cache.fork(_ints([0] * 17), _ints(range(1, 18)), _ints([width * page] * 16 + [20]), _ints([0] * 17), table, refs)
    assert got.tolist() == [-1] * 16 + [3]
    assert (table[1:16] == -1).all() and table[16, :4].tolist() == [1, 2, 4, -1] and table[17, :4].tolist() == [6, 7, 8, -1]
    want = np.zeros(n_pages)
    want[:9] = 1
    assert refs.tolist() == want.tolist()
    copied = torch.zeros(n_pages, dtype=torch.bool, device="cuda")
    copied[6:9] = True
    assert torch.equal(cache.pool[:, ~copied], before[:, ~copied]) and torch.equal(cache.pool[:, copied], before[:, 5:6].expand(-1, 3, *before.shape[2:]))
