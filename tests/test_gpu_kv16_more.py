"""The bf16 cache and its attention, further: rows in turn over rings, pages as long as tiles, long contexts, what sees only infinities."""
import numpy as np
import pytest

from oracle import trees
from test_gpu_kv16 import Case, Packed, _close, _ints
from test_kv16_bounds import marked, marked_queries, marked_result, marked_tolerance, norm_bound, norm_error

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


def _blind(k, keys):
    """Keys whose score is minus infinity for a query with a positive first column."""
    k[keys, :, 0] = -float("inf")


@pytest.mark.parametrize("heads,kvh,hd", [(4, 2, 128), (8, 2, 64), (64, 2, 128)])
@pytest.mark.parametrize("new,base", [([9], [40]), ([1], [0]), ([5], [0]), ([1], [9000]), ([40], [20000]), ([3] * 60, [300] * 60), ([1] * 300, [100] * 300)])
def test_rows_that_see_nothing_but_minus_infinity(new, base, heads, kvh, hd):
    """A softmax of minus infinities alone has no value: NaN.  One finite score among them takes all the weight, and a row that sees nothing gives 0."""
    import torch
    nan = float("nan")
    c = Case(heads + sum(new), new, base, heads, kvh, hd)
    for r, (n, b) in enumerate(zip(new, base)):
        _blind(c.k[r], slice(0, b + n))
    c.fill()
    words = 2
    some = c.trees(words)
    some[c.rng.random(c.rows) < 0.3] = 0
    for dtype in (torch.bfloat16, torch.float32):
        q = c.queries(dtype)
        q[:, :, 0] = q[:, :, 0].abs() + 0.25
        for mask in (None, some):
            out = c.attend(q, mask)
            for r in range(len(new)):
                rows = slice(int(c.row0[r]), int(c.row0[r + 1]))
                sees = c.seen(r, mask).any(1)
                assert torch.isnan(out[rows][sees]).all() and (out[rows][~sees] == 0).all()
    # every third request has one key with a score of its own, early, in the middle or the last one
    for r, (n, b) in enumerate(zip(new, base)):
        if r % 3 == 0:
            c.k[r][[0, (b + n) // 2, b + n - 1][r // 3 % 3], :, 0] = 1.0
    c.fill()
    q = c.queries(torch.bfloat16)
    q[:, :, 0] = q[:, :, 0].abs() + 0.25
    for mask in (None, some):
        out = c.attend(q, mask)
        for r in range(len(new)):
            rows, seen = slice(int(c.row0[r]), int(c.row0[r + 1])), c.seen(r, mask)
            want, size, mag = trees.attend(q[rows], c.k[r], c.v[r], seen, hd ** -0.5)
            finite = torch.isfinite(c.k[r][:, 0, 0])
            want[seen.any(1) & ~(seen & finite).any(1)] = nan
            _close(out[rows], (want, size, mag), q.dtype, base[r] + new[r])


@pytest.mark.parametrize("heads,kvh,hd", [(4, 2, 128), (8, 1, 64)])
def test_prompts_that_begin_with_minus_infinity(heads, kvh, hd):
    import torch
    from paper_2605_13319_b200 import binding
    c = Packed(5, [300, 1, 40, 7], heads, kvh, hd)
    c.q[:, :, 0] = c.q[:, :, 0].abs() + 0.25
    for (rows, _), blind in zip(c.spans(), (200, 1, 0, 7)):
        _blind(c.k, slice(rows.start, rows.start + blind))
    out = binding.attend_packed(c.q, c.k, c.v, c.row0)
    for (rows, n), blind in zip(c.spans(), (200, 1, 0, 7)):
        seen = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
        want, size, mag = trees.attend(c.q[rows], c.k[rows], c.v[rows], seen, c.scale)
        want[:blind] = float("nan")
        _close(out[rows], (want, size, mag), out.dtype, n)


def _blocks_that_give_up(call, clean):
    """call() with each block having given up in turn: what it had is NaN, all of a row's head or nothing, the rest what it is without.  Returns
    how many blocks had a part of each [row, head]."""
    import torch
    from paper_2605_13319_b200 import binding
    parts = torch.zeros(clean.shape[:2], dtype=torch.int32, device="cuda")
    try:
        for block in range(148):
            assert binding.lib().pipesd_debug_attend_gives_up(block) == 0
            out = call()
            gone = torch.isnan(out)
            assert torch.equal(gone.all(2), gone.any(2))
            assert torch.equal(torch.where(gone, clean, out), clean)
            parts += gone.all(2)
    finally:
        assert binding.lib().pipesd_debug_attend_gives_up(-1) == 0
    assert torch.equal(call(), clean)
    return parts


@pytest.mark.parametrize("heads,kvh,hd", [(8, 2, 128), (4, 4, 64), (40, 1, 128)])
@pytest.mark.parametrize("new,base", [([1], [40000]), ([40, 3, 0, 7], [2000, 100, 4, 0]), ([1] * 200, [300] * 200), ([100], [5000])])
def test_a_block_that_gives_up_leaves_nan(new, base, heads, kvh, hd):
    import torch
    c = Case(heads + sum(new), new, base, heads, kvh, hd)
    c.fill()
    mask = c.trees(-(-max(new) // 32))
    bits = _ints(mask.view(np.int32))
    for dtype in (torch.bfloat16, torch.float32):
        q = c.queries(dtype)
        clean = c.attend(q, mask)
        c.check(q, mask, clean)
        parts = _blocks_that_give_up(lambda: c.cache.attend(q, *c.where, mask=bits, out=torch.full_like(q, 5.0)), clean)
        assert (parts > 0).all()


@pytest.mark.parametrize("lengths,heads,kvh,hd", [([37], 8, 2, 128), ([3000, 1, 200], 8, 2, 128), ([64] * 100, 4, 4, 64)])
def test_a_block_that_gives_up_leaves_nan_in_prompts(lengths, heads, kvh, hd):
    import torch
    from paper_2605_13319_b200 import binding
    c = Packed(8, lengths, heads, kvh, hd, pad=3)
    n = sum(lengths)
    clean = binding.attend_packed(c.q, c.k, c.v, c.row0, out=torch.full(c.q.shape, 5.0, dtype=torch.bfloat16, device="cuda"))
    c.check(clean)
    parts = _blocks_that_give_up(lambda: binding.attend_packed(c.q, c.k, c.v, c.row0, out=torch.full_like(clean, 5.0)), clean)
    assert (parts[:n] == 1).all() and (parts[n:] == 0).all() and (clean[n:] == 5).all()


# --------------------------------------------------------------------------- long contexts
LONG = [([1], [40000]), ([9], [20055]), ([1], [131071]), ([17, 3, 60], [8000, 100, 30500]), ([64] * 3, [20000, 4000, 9990]), ([1] * 40, [int(x) for x in np.linspace(100, 9000, 40)]),
        ([512], [3000])]


@pytest.mark.parametrize("heads,kvh,hd", [(8, 2, 128), (8, 2, 64), (48, 1, 128)])
@pytest.mark.parametrize("new,base", LONG)
def test_long_contexts_in_norm(new, base, heads, kvh, hd):
    import torch
    c = Case(heads + sum(new) + hd, new, base, heads, kvh, hd)
    c.fill()
    for dtype in (torch.bfloat16, torch.float32):
        for mask in (None, c.trees(-(-max(new) // 32))):
            q = c.queries(dtype)
            out = c.attend(q, mask)
            want = torch.cat([trees.attend(q[a:b], c.k[r], c.v[r], c.seen(r, mask), hd ** -0.5)[0] for r, (a, b) in enumerate(zip(c.row0[:-1].tolist(), c.row0[1:].tolist()))])
            assert norm_error(out, want) < norm_bound(dtype)
            for a, b in zip(c.row0[:-1].tolist(), c.row0[1:].tolist()):      # a request's alone: few values, whose roundings may all be near half a step
                assert norm_error(out[a:b], want[a:b]) < 2 * norm_bound(dtype)


@pytest.mark.parametrize("heads,kvh,hd", [(8, 2, 128), (8, 2, 64), (48, 1, 128)])
@pytest.mark.parametrize("new,base", LONG)
@pytest.mark.parametrize("every", [1, 16])
def test_long_contexts_key_by_key(new, base, heads, kvh, hd, every):
    """Every key, or one of each page, counts alike: a lost or a doubled one shows."""
    import torch
    c = Case(heads + sum(new) + hd, new, base, heads, kvh, hd)
    for r, (n, b) in enumerate(zip(new, base)):
        c.k[r], c.v[r] = marked(b + n, np.arange(5 % every, b + n, every), hd, kvh, "cuda")
    c.fill()
    for dtype in (torch.bfloat16, torch.float32):
        if dtype is torch.bfloat16 and every == 1 and max(base) > 20000:
            continue                               # (one key is less than half a step)
        q = marked_queries(c.rows, heads, hd, dtype, "cuda")
        out = c.attend(q, None)
        for r, (n, b) in enumerate(zip(new, base)):
            rows = slice(int(c.row0[r]), int(c.row0[r + 1]))
            seen = b + 1 + np.arange(n)            # positions of each row
            want = marked_result((seen - 1 - 5 % every) // every + 1, hd, heads, kvh).cuda()
            assert ((out[rows].double() - want).abs() <= marked_tolerance(dtype) * want).all()


@pytest.mark.parametrize("lengths,heads,kvh,hd", [([5000], 8, 2, 128), ([3000, 1, 2049, 700], 4, 4, 64), ([4100], 6, 2, 128)])
def test_long_prompts_in_norm_and_key_by_key(lengths, heads, kvh, hd):
    import torch
    from paper_2605_13319_b200 import binding
    c = Packed(sum(lengths), lengths, heads, kvh, hd)
    out = binding.attend_packed(c.q, c.k, c.v, c.row0)
    for rows, n in c.spans():
        seen = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
        want = trees.attend(c.q[rows], c.k[rows], c.v[rows], seen, c.scale)[0]
        assert norm_error(out[rows], want) < norm_bound(out.dtype)
        if n > 2000:                               # (the last rows alone, which see most)
            assert norm_error(out[rows][-512:], want[-512:]) < norm_bound(out.dtype)
    for every in (1, 16):
        for rows, n in c.spans():
            c.k[rows], c.v[rows] = marked(n, np.arange(0, n, every), hd, kvh, "cuda")
        c.q[:] = marked_queries(c.rows, heads, hd, torch.bfloat16, "cuda")
        out = binding.attend_packed(c.q, c.k, c.v, c.row0)
        for rows, n in c.spans():
            want = marked_result(np.arange(n) // every + 1, hd, heads, kvh).cuda()
            assert ((out[rows].double() - want).abs() <= marked_tolerance(out.dtype) * want).all()


# --------------------------------------------------------------------------- long pages
def _ends(page):
    """Numbers of positions in front of, at and behind a page's end, a tile's, and both."""
    return [page - 1, page, page + 1, 2 * page + 127, 3 * page, 127, 128, 129]


@pytest.mark.parametrize("heads,kvh,hd", [(4, 2, 128), (4, 2, 64), (40, 1, 128)])
@pytest.mark.parametrize("page", [72, 128, 136, 256, 4096])
def test_pages_as_long_as_tiles(page, heads, kvh, hd):
    import torch
    new = [1, 2, 5, 1, 9, 3, 1, 4]
    base = [max(0, e - n) for e, n in zip(_ends(page), new)]
    many = ([1] * 24 + [20], [_ends(page)[i % 8] - 1 for i in range(24)] + [page + 60])
    for new, base in ((new, base), many, ([30], [2 * page + 20])):
        c = Case(page + heads + len(new), new, base, heads, kvh, hd, page)
        c.fill()
        for dtype in (torch.bfloat16, torch.float32):
            for mask in (None, c.trees(1)):
                q = c.queries(dtype)
                out = c.attend(q, mask)
                c.check(q, mask, out)
                assert torch.equal(out, c.attend(q, mask))
    hidden = Case(page, [3, 40], [3 * page - 3, page + 7], heads, kvh, hd, page, hide=[(0, 1, -1), (1, 0, 10 ** 9)])
    hidden.fill()
    for dtype in (torch.bfloat16, torch.float32):
        q = hidden.queries(dtype)
        hidden.check(q, None, hidden.attend(q, None))


def test_a_long_way_between_values_that_are_not_finite():
    """Two tiles with a border, each with a NaN, two million positions apart: rows see the NaN in its column, and the search for it takes no
    block so long that its waits run out."""
    import torch
    from paper_2605_13319_b200 import binding
    page, hd, n_req = 4088, 128, 450
    n_pages = (1 << 21) // page
    total = n_pages * page - 50
    g = torch.Generator("cuda").manual_seed(0)
    cache = binding.Kv16Cache(1, hd, n_pages=n_pages, page_size=page)
    k, v = (torch.randn((total, 1, hd), generator=g, device="cuda").bfloat16() for _ in range(2))
    v[page + 2, 0, 3] = float("nan")               # beside the page that is not there, and near the last position
    v[total - 3, 0, 40] = float("nan")
    table = torch.arange(n_pages, dtype=torch.int32, device="cuda")[None]
    cache.append(k, v, _ints([0, total]), _ints([0]), table)
    table = table.expand(n_req, -1).contiguous()   # read by all
    table[:, 0] = -1
    q = torch.randn((n_req, 1, hd), generator=g, device="cuda").bfloat16()
    out = cache.attend(q, _ints(range(n_req + 1)), _ints([total - 1] * n_req), table)
    assert torch.isnan(out[..., [3, 40]]).all() and torch.isfinite(out[:, 0, [i for i in range(hd) if i not in (3, 40)]]).all()
    clean = v.clone()
    clean[page + 2, 0, 3] = clean[total - 3, 0, 40] = 0.0
    rows = [0, 1, n_req // 2, n_req - 1]
    want = trees.attend(q[rows], k[page:], clean[page:], torch.ones((4, total - page), dtype=torch.bool, device="cuda"), hd ** -0.5)[0]
    keep = [i for i in range(hd) if i not in (3, 40)]
    assert norm_error(out[rows][..., keep], want[..., keep]) < 2 * norm_bound(q.dtype)


@pytest.mark.parametrize("scale", [2.0 ** 127, 2.0 ** -100])
def test_largest_and_smallest_scales(scale):
    import torch
    from paper_2605_13319_b200 import binding
    c = Case(3, [9, 1], [200, 30], 4, 2, 64)
    c.fill()
    for dtype in (torch.bfloat16, torch.float32):
        q = c.queries(torch.float32) * (2.0 ** -64 if scale > 1 else 2.0 ** 50)
        if scale > 1:                              # (keys' part of it, so that a score's products are normal numbers)
            for k in c.k:
                k *= 2.0 ** -62
            c.fill()
        q = q.to(dtype)
        out = c.attend(q, None, scale=scale)
        c.check(q, None, out, scale)
        if scale > 1:
            for k in c.k:
                k *= 2.0 ** 62
    p = Packed(4, [100, 5], 4, 2, 128)
    p.q *= 2.0 ** -64 if scale > 1 else 2.0 ** 50
    p.k *= 2.0 ** -62 if scale > 1 else 1.0
    p.scale = scale
    p.check(binding.attend_packed(p.q, p.k, p.v, p.row0, scale=scale))


@pytest.mark.parametrize("heads,new", [(4, [7, 1, 30]), (32, [20, 40, 3])])
def test_padded_batches(heads, new):
    """Rows in front of the first request and behind the last: not read into anything, left as they were, in every call that takes rows."""
    import torch
    from paper_2605_13319_b200 import binding
    c = Case(heads, new, [300, 0, 77], heads, 2, 128)
    c.fill()
    mask = c.trees(2)
    lead, pad = 3, 60
    inside = slice(lead, lead + c.rows)
    where = [c.where[0] + lead, *c.where[1:]]
    for dtype in (torch.bfloat16, torch.float32):
        q = c.queries(dtype)
        wide = torch.full((lead + c.rows + pad, heads, 128), float("nan"), dtype=dtype, device="cuda")
        wide[inside] = q
        bits = torch.full((len(wide), 2), -1, dtype=torch.int32, device="cuda")
        bits[inside] = _ints(mask.view(np.int32))
        for m, b in ((None, None), (mask, bits)):
            out = c.cache.attend(wide, *where, mask=b, out=torch.full_like(wide, 5.0))
            c.check(q, m, out[inside])
            assert (out[:lead] == 5).all() and (out[inside.stop:] == 5).all()
    k, v = (torch.randn((len(wide), 2, 128), device="cuda").bfloat16() for _ in range(2))
    before = c.cache.pool.clone()
    c.cache.append(k, v, *where)
    got = c.cache.read(len(wide), *where)
    for x, y in zip((k, v), got):
        assert torch.equal(y[inside], x[inside]) and (y[:lead] == 0).all() and (y[inside.stop:] == 0).all()
    new_pages = {int(c.table[r, p // c.page]) for r, (n, b) in enumerate(zip(c.new, c.base)) for p in range(b, b + n)}
    rest = [p for p in range(c.cache.n_pages) if p not in new_pages]
    assert torch.equal(c.cache.pool[:, rest].view(torch.int16), before[:, rest].view(torch.int16))
    parent = _ints([-1, 0] * ((len(wide) + 1) // 2))[:len(wide)].contiguous()
    trees_mask, depth = binding.tree_mask(parent, where[0], 2)
    assert (trees_mask[:lead] == 0).all() and (trees_mask[inside.stop:] == 0).all() and (depth[:lead] == 0).all() and (depth[inside.stop:] == 0).all()
