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
