"""Pages of the bf16 cache: reserve, fork, compact, release against plain forms; a round of drafted trees served with all of it."""
import numpy as np
import pytest

from oracle import trees

pytestmark = pytest.mark.gpu


def _ints(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Pages:
    """A pool, a table of slots and references, on the device and in plain form."""

    def __init__(self, seed, n_slots, max_pages, n_pages, page=16, layers=2, kvh=2, hd=64):
        import torch
        from paper_2605_13319_b200 import binding
        g = torch.Generator("cuda").manual_seed(seed)
        pool = torch.randint(-2 ** 15, 2 ** 15, (layers, n_pages, 2, kvh, page // 8, hd // 8, 8, 8), generator=g, device="cuda", dtype=torch.int16)
        self.ref = trees.Pool(pool.cpu().numpy().view(np.uint16).reshape(layers, n_pages, 2, kvh, -1).copy(), hd, page)
        self.cache = binding.Kv16Cache(kvh, hd, pool=pool.view(torch.bfloat16), page_size=page)
        self.page, self.table, self.refs = page, np.full((n_slots, max_pages), -1, np.int32), np.zeros(n_pages, np.int32)
        self.d_table, self.d_refs = _ints(self.table), _ints(self.refs)

    def reserve(self, length):
        n = len(length)
        got = self.cache.reserve(_ints(length), self.d_table[:n], self.d_refs).tolist()
        assert got == trees.reserve(length, self.table[:n], self.refs, self.page)
        return self.same()

    def fork(self, src, dst, length, own):
        got = self.cache.fork(*map(_ints, (src, dst, length, own)), self.d_table, self.d_refs).tolist()
        want = trees.fork(src, dst, length, own, self.table, self.refs, self.page, self.ref)
        assert got == want
        self.same()
        return got

    def release(self, length, first=0):
        self.cache.release(_ints(length), self.d_table[first:first + len(length)], self.d_refs)
        trees.release(length, self.table[first:first + len(length)], self.refs, self.page)
        return self.same()

    def compact(self, keep, base, rows):
        bits = _ints(keep.view(np.int32))
        got = self.cache.compact(bits, _ints(base), self.d_table[rows].contiguous()).tolist()
        want = [self.ref.compact(self.table[r], b, trees.bits_of(k[None], 32 * len(k))[0].nonzero()[0].tolist()) for r, b, k in zip(rows, base, keep)]
        assert got == want
        self.same()
        return got

    def same(self):
        import torch
        assert np.array_equal(self.d_table.cpu().numpy(), self.table)
        assert np.array_equal(self.d_refs.cpu().numpy(), self.refs)
        assert np.array_equal(self.cache.pool.view(torch.int16).cpu().numpy().view(np.uint16).reshape(self.ref.bits.shape), self.ref.bits)


def test_reserve_and_release():
    p = Pages(0, 5, 6, 17)
    p.reserve([40, 0, 16, 96, 1])
    p.reserve([49, 0, 10, 96, 1])                                            # grows one, leaves the rest
    p.reserve([97, 16, -1, 200, 17])                                         # lengths behind the table and below 0: refused
    p.release([16, 0, -1, 95, 0])
    p.reserve([96, 96, 96, 96, 96])                                          # not enough for all: the first that fit
    p.release([0, 17, 96, 2 ** 31 - 1, 33])
    p.reserve([0, 32, 96, 96, 96])
    p.release([0] * 5)
    assert (p.refs == 0).all()


def test_fork_shares_and_copies():
    p = Pages(1, 8, 5, 30)
    p.reserve([50, 16, 80, 0])
    assert p.fork([0, 0, 1, 2, 3], [3, 4, 5, 6, 7], [50, 50, 16, 70, 0], [40, 48, 16, 0, 5]) == [4, 4, 1, 5, 0]
    p.release([0, 0], first=3)
    # numbers that make no sense, a slot to itself; those behind are served
    assert p.fork([0, -1, 0, 9, 0, 0, 0, 1], [3, 4, 8, 4, 0, 4, 4, 4], [50, 5, 5, 5, 5, 81, 5, 7], [3, 0, 0, 0, 0, 0, -1, 0]) == [4, -1, -1, -1, -1, -1, -1, 1]
    p.release([0] * 8)
    assert (p.refs == 0).all()


def test_fork_without_enough_pages():
    p = Pages(2, 6, 4, 12)
    p.reserve([64, 30])
    assert p.fork([0, 0, 1], [2, 3, 4], [64, 64, 30], [0, 10, 16]) == [4, -1, 2]      # 6 free: 4, then none for 4, then 1
    p.release([0], first=2)
    assert p.fork([0, 0], [2, 3], [64, 64], [0, 63]) == [4, 4]
    # entries that are no page are no page of the fork either
    p.d_table[0, 1], p.table[0, 1] = -1, -1
    p.d_table[0, 2], p.table[0, 2] = 10 ** 9, 10 ** 9
    p.release([0, 0], first=2)
    p.fork([0, 0], [2, 3], [64, 40], [0, 32])


def test_fork_of_slots_that_are_targets_too():
    """Not served in any set way (no dst is a src within a call), but pages of other slots stay what they were."""
    import torch
    p = Pages(8, 9, 6, 60)
    p.reserve([96, 96, 80, 0, 0, 0, 0, 0, 50])
    before = p.cache.pool.clone()
    for src, dst in (([0, 1, 2, 3, 4], [1, 2, 3, 4, 5]), ([3, 2, 1], [2, 1, 0]), ([0, 0], [3, 3])):
        pages = p.cache.fork(_ints(src), _ints(dst), _ints([90] * len(src)), _ints([20] * len(src)), p.d_table, p.d_refs)
        assert ((pages == -1) | (pages == 6)).all()
    table = p.d_table.cpu().numpy()
    assert ((table >= -1) & (table < 60)).all() and np.array_equal(table[8], p.table[8])
    for page in table[8][:4]:
        assert torch.equal(p.cache.pool[:, page].view(torch.int16), before[:, page].view(torch.int16))


def test_fork_of_many_and_large_pools():
    import torch
    p = Pages(3, 300, 3, 3000, page=8, layers=1, kvh=1)
    p.reserve([24] * 100)
    p.fork([i % 100 for i in range(200)], list(range(100, 300)), [24 - i % 3 for i in range(200)], [i % 25 for i in range(200)])
    p.release([int(x) for x in np.arange(300) % 20])
    p.reserve([24] * 300)
    # lowest free ids of half a million references
    from paper_2605_13319_b200 import binding
    refs = torch.randint(0, 5, (500000,), device="cuda", dtype=torch.int32)
    refs[:100000] = 1
    free = torch.nonzero(refs == 0)[:40, 0]
    cache = binding.Kv16Cache(1, 64, n_pages=500000, page_size=8)
    table = torch.full((2, 20), -1, dtype=torch.int32, device="cuda")
    assert cache.reserve(_ints([160, 153]), table, refs).tolist() == [20, 20]
    assert torch.equal(table.flatten().long(), free) and (refs[free] == 1).all()


def test_pages_over_many_calls():
    rng = np.random.default_rng(4)
    p = Pages(5, 10, 6, 24)
    for step in range(60):
        kind = rng.integers(4)
        if kind == 0:
            p.reserve([int(x) for x in rng.integers(0, 97, 5)])
        elif kind == 1:
            dst = [int(r) for r in range(5, 10) if (p.table[r] < 0).all()][:int(rng.integers(1, 4))]
            if dst:
                src = [int(x) for x in rng.integers(0, 5, len(dst))]
                length = [int(x) for x in rng.integers(0, 97, len(dst))]
                p.fork(src, dst, length, [int(rng.integers(0, n + 1)) for n in length])
        else:
            lengths = [int(x) if rng.random() < 0.5 else -1 for x in rng.integers(0, 97, 10)]
            p.release(lengths)
        held = np.bincount(p.table[p.table >= 0], minlength=24)
        assert np.array_equal(held, p.refs)


@pytest.mark.parametrize("hd,page,kvh,layers", [(64, 16, 2, 2), (128, 8, 1, 3), (64, 24, 5, 1), (128, 16, 8, 5)])
def test_compact(hd, page, kvh, layers):
    rng = np.random.default_rng(hd + page)
    width = -(-200 // page)
    p = Pages(hd, 5, width, 5 * width + 2, page=page, layers=layers, kvh=kvh, hd=hd)
    p.reserve([200] * 5)
    keep = rng.integers(0, 2 ** 32, (5, 4), dtype=np.uint32)
    keep[0] = 0
    keep[1] = [0xffffffff, 0xffffffff, 7, 0]                                 # nothing has to move
    keep[2] = [0, 0, 0, 0x80000000]                                          # the last one to the front
    assert p.compact(keep, [0, 30, 5, 17, 190], [0, 1, 2, 3, 4])[:3] == [0, 67, 1]      # the last one's bits reach behind the table
    p.table[3, 1] = -1
    p.d_table[3, 1] = -1
    p.compact(keep, [0, 30, 5, 17, -1], [0, 1, 2, 3, 4])                     # rows and new positions without a page; a base below 0


def test_compact_long_sets():
    rng = np.random.default_rng(8)
    p = Pages(6, 2, 400, 800, page=16, layers=1, kvh=1)
    p.reserve([6400, 6400])
    for share in (0.5, 0.02, 0.98):
        keep = np.packbits(rng.random((2, 6400)) < share, axis=1, bitorder="little").view(np.uint32)
        p.compact(keep, [0, 3], [0, 1])


def test_pages_in_graphs_and_on_streams():
    import torch
    p = Pages(7, 4, 4, 20)
    p.reserve([64, 40])
    src, dst, length, own, none = map(_ints, ([0, 1], [2, 3], [64, 40], [20, 33], [0, 0]))
    keep, base = _ints([[0x5555], [0x700]]), _ints([20, 33])
    before = [t.clone() for t in (p.d_table, p.d_refs)]
    side = torch.cuda.Stream()

    def branch(stream=None):
        pages = p.cache.fork(src, dst, length, own, p.d_table, p.d_refs, stream=stream)
        kept = p.cache.compact(keep, base, p.d_table[2:], stream=stream)
        out = p.cache.read(30, _ints_30, _ints_base, p.d_table[2:], stream=stream)
        p.cache.release(none, p.d_table[2:], p.d_refs, stream=stream)
        return [pages, kept, *(x.view(torch.int16) for x in out)]            # (patterns: NaN among them)

    _ints_30, _ints_base = _ints([0, 20, 30]), _ints([16, 32])
    want = branch()
    assert want[0].tolist() == [4, 3] and want[1].tolist() == [8, 3]
    torch.cuda.synchronize()
    got = branch(side)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = branch()
    for _ in range(3):
        for t in held:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, want))
        assert all(torch.equal(x, y) for x, y in zip((p.d_table, p.d_refs), before))


def test_a_round_of_trees_together():
    """Prompts attended and appended; trees drafted, appended and attended; an accepted path each, and a fork with another one; compacted; then
    a token behind it.  The token's attention is that over the prompt and the path alone, in 64 bits, and rows of the tree saw their path."""
    import torch
    from paper_2605_13319_b200 import binding
    for dtype, hd, heads, kvh, page in ((torch.bfloat16, 128, 8, 2, 16), (torch.float32, 64, 4, 4, 24)):
        g = torch.Generator("cuda").manual_seed(hd)
        rng = np.random.default_rng(hd)
        lengths, sizes = [50, 130, 7], [20, 1, 40]
        n, layers, scale = len(lengths), 2, hd ** -0.5
        tol = 3 * 2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -17       # of the norm: the roundings of one attention, see test_gpu_kv16

        def rows(count, h):
            return torch.randn((count, h, hd), generator=g, device="cuda").bfloat16()

        cache = binding.Kv16Cache(kvh, hd, n_layers=layers, n_pages=40, page_size=page)
        table, refs = _ints(np.full((2 * n, 12), -1)), _ints(np.zeros(40))
        row0 = _ints(np.concatenate([[0], np.cumsum(lengths)]))
        base0, base = _ints([0] * n), _ints(lengths)
        pk, pv = ([rows(sum(lengths), kvh) for _ in range(layers)] for _ in range(2))
        pages = cache.reserve(_ints([a + b for a, b in zip(lengths, sizes)]), table[:n], refs)
        assert pages.tolist() == [-(-(a + b) // page) for a, b in zip(lengths, sizes)]
        for l in range(layers):
            q = rows(sum(lengths), heads)
            out = binding.attend_packed(q, pk[l], pv[l], row0)
            cache.append(pk[l], pv[l], row0, base0, table[:n], layer=l)
            over = cache.attend(q, row0, base0, table[:n], layer=l)          # the same rows over the cache
            assert (out.double() - over.double()).norm() < 2 * 2.0 ** -8 * over.double().norm()
        parents = [[max(-1, i - 1 - int(rng.exponential(2))) for i in range(s)] for s in sizes]
        tree0 = _ints(np.concatenate([[0], np.cumsum(sizes)]))
        mask, depth = binding.tree_mask(_ints(sum(parents, [])), tree0, 2)
        tk, tv = ([rows(sum(sizes), kvh).to(dtype) for _ in range(layers)] for _ in range(2))
        start = np.concatenate([[0], np.cumsum(sizes)])

        def path(r, node):
            out = []
            while node >= 0:
                out.insert(0, node)
                node = parents[r][node]
            return out

        def plain(q, r, l, nodes, k, v):
            at = slice(int(row0[r]), int(row0[r + 1]))
            keys, values = (torch.cat([a[l][at].double(), b[l][[int(start[r]) + i for i in nodes]].bfloat16().double()]) for a, b in ((pk, k), (pv, v)))
            return trees.attend(q[None], keys, values, torch.ones((1, len(keys)), dtype=torch.bool, device="cuda"), scale)[0][0]

        for l in range(layers):
            cache.append(tk[l], tv[l], tree0, base, table[:n], layer=l)
            q = rows(sum(sizes), heads).to(dtype)
            out = cache.attend(q, tree0, base, table[:n], mask=mask, layer=l)
            for r in range(n):
                for i in (0, sizes[r] - 1):
                    want = plain(q[start[r] + i], r, l, path(r, i), tk, tv)
                    assert (out[start[r] + i].double() - want).norm() < tol * want.norm()
        first, second = [sizes[r] - 1 for r in range(n)], [sizes[r] // 2 for r in range(n)]
        whole = base + (tree0[1:] - tree0[:-1])
        assert (cache.fork(_ints(range(n)), _ints(range(n, 2 * n)), whole, base, table, refs) > 0).all()
        leaves = torch.tensor([int(start[r]) + x for nodes in (first, second) for r, x in enumerate(nodes)], device="cuda")
        base2 = torch.cat([base, base])
        kept = cache.compact(mask[leaves], base2, table)
        assert kept.tolist() == [len(path(r, x)) for nodes in (first, second) for r, x in enumerate(nodes)] and torch.equal(kept, depth[leaves] + 1)
        length = base2 + kept
        cache.release(length, table, refs)
        assert (cache.reserve(length + 1, table, refs) > 0).all()
        for l in range(layers):
            q, k, v = rows(2 * n, heads).to(dtype), rows(2 * n, kvh), rows(2 * n, kvh)
            cache.append(k, v, _ints(range(2 * n + 1)), length, table, layer=l)
            out = cache.attend(q, _ints(range(2 * n + 1)), length, table, layer=l)
            for i, (r, x) in enumerate([(r, x) for nodes in (first, second) for r, x in enumerate(nodes)]):
                keys, values = [], []
                at = slice(int(row0[r]), int(row0[r + 1]))
                nodes = [int(start[r]) + j for j in path(r, x)]
                ks, vs = (torch.cat([a[l][at].double(), b[l][nodes].bfloat16().double(), c[i:i + 1].double()]) for a, b, c in ((pk, tk, k), (pv, tv, v)))
                want = trees.attend(q[i:i + 1], ks, vs, torch.ones((1, len(ks)), dtype=torch.bool, device="cuda"), scale)[0][0]
                assert (out[i].double() - want).norm() < tol * want.norm()
        cache.release(_ints([0] * 2 * n), table, refs)
        assert (refs == 0).all() and (table == -1).all()
