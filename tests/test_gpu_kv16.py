"""Packed prompts, the bf16 cache and attention of trees over it (pipesd_attend_packed, pipesd_tree_mask, pipesd_kv16_*) against 64-bit forms."""
import numpy as np
import pytest

from oracle import trees

pytestmark = pytest.mark.gpu


def _ints(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _row0(new):
    return np.concatenate([[0], np.cumsum(new)]).astype(np.int32)


def _close(got, ref, dtype, keys):
    """Elementwise, counted from the roundings.  With S = sum of p |v| and A = a score's sum of magnitudes: fp32 sums of 128 products on the
    tensor cores, eight steps of 16 that may truncate, 2^-22 of A each: 2^-19 A, which both the numerator and the denominator take; p is rounded to bf16
    (2^-8) for the numerator, the output to its type.  fp32: three terms of q and of p (2^-24), 24 steps a score, and three additions per 16 keys to
    the running sums, 2^-23 of S each, sixteen more where shares are merged."""
    import torch
    want, size, mag = ref
    if dtype is torch.bfloat16:
        tol = 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2 * 2.0 ** -19 * mag) * size
    else:
        tol = 2.0 ** -24 * want.abs() + (3 * 2.0 ** -24 + 2 * 2.0 ** -18 * mag + (3 * keys / 16 + 16) * 2.0 ** -23) * size
    got = got.double()
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), "not finite elsewhere"
    ok = torch.isfinite(want)
    err = (got - want).abs()
    bad = ok & (err > tol + 1e-30)
    assert not bad.any(), (bad.nonzero()[:4].tolist(), err[bad].max().item(), tol[bad].min().item())


# --------------------------------------------------------------------------- prompts
class Packed:
    def __init__(self, seed, lengths, heads, kvh, hd, pad=0, lead=0):
        import torch
        g = torch.Generator("cuda").manual_seed(seed)
        self.lengths, self.lead, self.rows = lengths, lead, lead + sum(lengths) + pad
        self.row0 = _ints(lead + _row0(lengths))
        qkv = torch.randn((self.rows, heads + 2 * kvh, hd), generator=g, device="cuda").bfloat16()
        qkv[:, :heads] *= 1.5
        self.q, self.k, self.v = qkv[:, :heads], qkv[:, heads:heads + kvh], qkv[:, heads + kvh:]
        self.scale = hd ** -0.5

    def spans(self):
        at = self.lead
        for n in self.lengths:
            yield slice(at, at + n), n
            at += n

    def check(self, out):
        import torch
        for rows, n in self.spans():
            if n:
                seen = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
                _close(out[rows], trees.attend(self.q[rows], self.k[rows], self.v[rows], seen, self.scale), out.dtype, n)


@pytest.mark.parametrize("heads,kvh,hd", [(4, 4, 128), (8, 2, 128), (4, 1, 64), (6, 2, 64), (5, 1, 128), (32, 1, 64), (71, 1, 64), (128, 1, 128), (65, 1, 128)])
@pytest.mark.parametrize("lengths", [[1], [2], [31], [128], [129], [257, 1, 0, 40], [513], [127, 128, 385]])
def test_prompts_match(heads, kvh, hd, lengths):
    from paper_2605_13319_b200 import binding
    c = Packed(heads + sum(lengths), lengths, heads, kvh, hd)
    c.check(binding.attend_packed(c.q, c.k, c.v, c.row0))


@pytest.mark.parametrize("lengths,heads,kvh,hd", [([3000], 8, 8, 128), ([2500, 1, 700, 1300], 8, 2, 128), ([1999, 2001], 16, 4, 64), ([1] * 300, 8, 2, 128),
                                                   (list(range(0, 180)), 4, 2, 64), ([64] * 100, 8, 1, 128), ([5000], 2, 1, 64)])
def test_prompts_large(lengths, heads, kvh, hd):
    import torch
    from paper_2605_13319_b200 import binding
    c = Packed(7, lengths, heads, kvh, hd, pad=13, lead=5)
    out = torch.full(c.q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    assert binding.attend_packed(c.q, c.k, c.v, c.row0, out=out) is out
    c.check(out)
    assert (out[:5] == 7).all() and (out[c.rows - 13:] == 7).all()
    again = torch.full_like(out, 7.0)
    binding.attend_packed(c.q, c.k, c.v, c.row0, out=again)
    assert torch.equal(out, again)                                           # the same bits every time


@pytest.mark.parametrize("heads,kvh,hd", [(8, 2, 128), (2, 2, 64)])
def test_prompts_keep_to_themselves(heads, kvh, hd):
    """What is not finite in rows of no prompt, of another prompt, or behind a row, does not reach it; what it sees does."""
    import torch
    from paper_2605_13319_b200 import binding
    nan, inf = float("nan"), float("inf")
    c = Packed(3, [100, 77, 300, 5], heads, kvh, hd, pad=60, lead=9)
    clean = binding.attend_packed(c.q, c.k, c.v, c.row0)
    for t in (c.k, c.v, c.q):
        t[:9], t[c.rows - 60:] = nan, inf
    first = 9 + 100 + 77
    c.v[first + 150, 0, 3] = nan
    c.v[first + 151, kvh - 1, 7] = -inf
    c.v[first + 299] = nan
    c.k[9 + 60] = nan
    c.q[9 + 30, 1] = nan
    out = binding.attend_packed(c.q, c.k, c.v, c.row0)
    c.check(torch.where(torch.isinf(out), nan, out))
    same = torch.ones(c.rows, dtype=torch.bool, device="cuda")
    same[:9], same[c.rows - 60:] = False, False
    same[9 + 60:9 + 100], same[9 + 30], same[first + 150:first + 300] = False, False, False
    assert torch.equal(out[same], clean[same])


def test_prompts_scores_that_grow():
    """Every row's maximum moves far, tile after tile, in both directions; scores of one size; a scale of its own."""
    import torch
    from paper_2605_13319_b200 import binding
    for sign in (1, -1):
        c = Packed(4, [700], 4, 2, 128)
        c.k *= (torch.arange(700, device="cuda") * 0.05 * sign + (0 if sign > 0 else 40))[:, None, None]
        c.check(binding.attend_packed(c.q, c.k, c.v, c.row0))
    c.k[:] = 0.5
    c.check(binding.attend_packed(c.q, c.k, c.v, c.row0))
    c = Packed(5, [300], 4, 2, 64)
    c.scale = 0.9
    c.check(binding.attend_packed(c.q, c.k, c.v, c.row0, scale=0.9))


def test_prompts_strides_streams_and_graphs():
    import torch
    from paper_2605_13319_b200 import binding
    c = Packed(6, [200, 33, 1], 8, 2, 128, pad=4)
    out = binding.attend_packed(c.q, c.k, c.v, c.row0)
    apart = [t.contiguous() for t in (c.q, c.k, c.v)]
    wide = torch.full((c.rows, 24, 128), 3.0, device="cuda", dtype=torch.bfloat16)
    got = binding.attend_packed(*apart, c.row0, out=wide[:, 8:16])
    n = sum(c.lengths)
    assert torch.equal(got[:n], out[:n])
    assert (wide[:, :8] == 3).all() and (wide[:, 16:] == 3).all() and (wide[n:] == 3).all()
    with pytest.raises(binding.PipesdError):                                 # rows that do not begin at a multiple of 16 bytes
        odd = torch.zeros((c.rows, 8 * 128 + 4), device="cuda", dtype=torch.bfloat16)[:, :1024].unflatten(1, (8, 128))
        binding.attend_packed(odd, c.k, c.v, c.row0)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    many = [binding.attend_packed(c.q, c.k, c.v, c.row0, stream=s) for _ in range(4) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(x[:n], out[:n]) for x in many)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = binding.attend_packed(c.q, c.k, c.v, c.row0)
    c.q[:] = c.q.flip(0)
    c.row0.copy_(_ints([0, 100, 200, 234]))                                  # lengths are read when it runs
    c.lengths = [100, 100, 34]
    g.replay()
    torch.cuda.synchronize()
    c.check(held)


# --------------------------------------------------------------------------- masks
@pytest.mark.parametrize("sizes,words", [([1], 1), ([5, 0, 64, 33], 2), ([100], 4), ([40], 1), ([300, 7], 10), ([8192], 256), ([9000, 3], 256)])
def test_tree_masks(sizes, words):
    import torch
    from paper_2605_13319_b200 import binding
    rng = np.random.default_rng(sum(sizes))
    parents = []
    for n in sizes:
        p = [max(-1, i - 1 - int(rng.exponential(3))) for i in range(n)]
        for i in rng.integers(0, max(n, 1), n // 10):
            p[i] = int(rng.choice([-7, n + 3, i, i + 1, 2 ** 31 - 1, -2 ** 31]))      # no parent of i: a child of the prefix
        parents.append(p)
    row0 = _row0(sizes)
    mask, depth = binding.tree_mask(_ints([x for p in parents for x in p] + [-1, 0]), _ints(row0), words)
    assert mask.shape == (row0[-1] + 2, words)
    for r, p in enumerate(parents):
        if len(p):
            want, deep = trees.ancestors(p, words)
            rows = slice(row0[r], row0[r + 1])
            assert np.array_equal(mask[rows].cpu().numpy().view(np.uint32), want)
            assert np.array_equal(depth[rows].cpu().numpy(), deep)
    assert (mask[-2:] == 0).all() and (depth[-2:] == 0).all()                # rows of no request
    chain, deep = binding.tree_mask(_ints(np.arange(-1, 39)), _ints([0, 40]), 2)
    assert deep.tolist() == list(range(40)) and chain[39].tolist() == [-1, 255]


# --------------------------------------------------------------------------- the cache
class Case:
    """Requests with pages in no order, in a pool of noise with NaN and infinities in it; K and V of every position are known."""

    def __init__(self, seed, new, base, heads, kvh, hd, page=16, layers=1, layer=0, hide=(), extra=1):
        import torch
        from paper_2605_13319_b200 import binding
        rng = np.random.default_rng(seed)
        g = torch.Generator("cuda").manual_seed(seed)
        self.new, self.base, self.heads, self.kvh, self.hd, self.page, self.layer = list(new), list(base), heads, kvh, hd, page, layer
        self.row0 = _row0(new)
        self.rows = int(self.row0[-1])
        used = [-(-(b + n) // page) for b, n in zip(base, new)]
        n_pages = sum(used) + 2
        order = rng.permutation(n_pages)
        self.table = np.full((len(new), max(max(used), 1) + extra), -1, np.int32)
        at = 0
        for r, n in enumerate(used):
            self.table[r, :n] = order[at:at + n]
            at += n
        pool = torch.randn((layers, n_pages, 2, kvh, page // 8, hd // 8, 8, 8), generator=g, device="cuda").bfloat16()
        noise = torch.rand(pool.shape, generator=g, device="cuda")
        pool[noise < 0.01], pool[noise > 0.99] = float("nan"), float("-inf")
        self.cache = binding.Kv16Cache(kvh, hd, pool=pool, page_size=page)
        total = [b + n for b, n in zip(base, new)]
        self.k, self.v = ([torch.randn((t, kvh, hd), generator=g, device="cuda").bfloat16() for t in total] for _ in range(2))
        self.whole = [_ints(_row0(total)), _ints([0] * len(new)), _ints(self.table)]
        for r, c, v in hide:
            self.table[r, c] = v
        self.where = [_ints(self.row0), _ints(base), _ints(self.table)]
        self.gen, self.rng = g, rng

    def fill(self):
        import torch
        self.cache.append(torch.cat(self.k), torch.cat(self.v), *self.whole, layer=self.layer)

    def queries(self, dtype, std=1.5):
        import torch
        return (torch.randn((self.rows, self.heads, self.hd), generator=self.gen, device="cuda") * std).to(dtype)

    def trees(self, words):
        masks = []
        for n in self.new:
            p = [max(-1, i - 1 - int(self.rng.exponential(2))) for i in range(n)]
            masks.append(trees.ancestors(p, words)[0] if n else np.zeros((0, words), np.uint32))
        return np.concatenate(masks)

    def seen(self, r, mask):
        """[rows, positions] of a request."""
        import torch
        n, b = self.new[r], self.base[r]
        there = np.array([0 <= self.table[r, p // self.page] < self.cache.n_pages for p in range(b + n)])
        if mask is None:
            new = np.tril(np.ones((n, n), bool))
        else:
            new = trees.bits_of(mask[self.row0[r]:self.row0[r + 1]], n)
        return torch.from_numpy(np.concatenate([np.ones((n, b), bool), new], 1) & there).cuda()

    def check(self, q, mask, out, scale=None):
        for r, n in enumerate(self.new):
            if n:
                rows = slice(int(self.row0[r]), int(self.row0[r + 1]))
                ref = trees.attend(q[rows], self.k[r], self.v[r], self.seen(r, mask), scale or self.hd ** -0.5)
                _close(out[rows], ref, q.dtype, self.base[r] + n)

    def attend(self, q, mask, **kw):
        return self.cache.attend(q, *self.where, mask=None if mask is None else _ints(mask.view(np.int32)), layer=self.layer, **kw)


@pytest.mark.parametrize("hd,kvh", [(64, 1), (64, 3), (128, 2)])
@pytest.mark.parametrize("new,base,page", [([1], [0], 16), ([1], [15], 8), ([2], [15], 16), ([17], [7], 24), ([5, 0, 40, 1], [9, 4, 30, 0], 16), ([100], [3], 64)])
def test_append_and_read(new, base, page, hd, kvh):
    import torch
    c = Case(sum(new) + hd, new, base, kvh, kvh, hd, page, layers=3, layer=1)
    ref = trees.Pool(c.cache.pool.view(torch.int16).cpu().numpy().view(np.uint16).reshape(3, c.cache.n_pages, 2, kvh, -1).copy(), hd, page)
    for dtype in (torch.float32, torch.bfloat16):
        k, v = (torch.randn((c.rows, kvh, hd), generator=c.gen, device="cuda").to(dtype) for _ in range(2))
        k[0, 0, :3] = torch.tensor([float("nan"), float("inf"), 1e-40])
        c.cache.append(k, v, *c.where, layer=1)
        bits = [x.bfloat16().view(torch.int16).cpu().numpy().view(np.uint16) for x in (k, v)]
        for r, n in enumerate(new):
            for i in range(n):
                for kv in range(2):
                    ref.put(c.table[r], base[r] + i, 1, kv, bits[kv][c.row0[r] + i])
        assert np.array_equal(c.cache.pool.view(torch.int16).cpu().numpy().view(np.uint16).reshape(ref.bits.shape), ref.bits)      # every byte
        got = c.cache.read(c.rows, *c.where, layer=1)
        assert all(np.array_equal(x.view(torch.int16).cpu().numpy().view(np.uint16), y) for x, y in zip(got, bits))


def test_append_from_a_fused_projection_and_rows_that_have_no_page():
    import torch
    c = Case(2, [20, 3, 4], [10, 60, 0], 2, 2, 128, hide=[(0, 1, -1), (2, 0, 10 ** 6)], extra=0)      # 16..31 of request 0; all of request 2
    fused = torch.randn((c.rows, 6, 128), generator=c.gen, device="cuda")
    odd = torch.randn((c.rows, 2 * 128 + 3), generator=c.gen, device="cuda", dtype=torch.bfloat16)[:, 3:].unflatten(1, (2, 128))
    for k, v in ((fused[:, 2:4], fused[:, 4:]), (odd, odd)):
        c.cache.append(k, v, *c.where)
        got = c.cache.read(c.rows, *c.where)
        for x, y in zip((k, v), got):
            want = x.bfloat16().clone()
            want[6:20], want[23:] = 0, 0
            assert torch.equal(y, want)
    before = c.cache.pool.view(torch.int16).clone()
    w = [_ints([0, 20, 19, 27]), _ints([80, 5, -1]), c.where[2]]             # behind the table, row0 that makes no sense, a negative base
    c.cache.append(fused[:, 2:4], fused[:, 4:], *w)
    assert torch.equal(c.cache.pool.view(torch.int16), before)
    q = c.queries(torch.bfloat16)
    out = torch.full_like(q, 5.0)
    c.cache.attend(q, *w, out=out)
    assert (out[:19] == 0).all()


TREES = [([1], [0], 16), ([1], [1], 16), ([1], [127], 16), ([1], [128], 8), ([9], [40], 24), ([33], [0], 16), ([64], [100], 48), ([65], [190], 16),
         ([1, 1, 1, 1], [3, 200, 64, 0], 16), ([5, 0, 2, 16], [130, 4, 16, 700], 48), ([40, 3], [383, 1000], 64), ([200], [5], 16)]


@pytest.mark.parametrize("heads,kvh,hd", [(2, 2, 64), (4, 1, 128), (6, 2, 128), (16, 2, 64), (5, 1, 64), (32, 1, 128), (100, 1, 64)])
@pytest.mark.parametrize("new,base,page", TREES)
def test_attend_matches(heads, kvh, hd, new, base, page):
    import torch
    c = Case(hd + heads + sum(new) + sum(base), new, base, heads, kvh, hd, page, layers=2, layer=1)
    c.fill()
    words = -(-max(new) // 32) + heads % 2
    any_bits = c.rng.integers(0, 2 ** 32, (c.rows, words), dtype=np.uint32)
    any_bits[c.rng.random(c.rows) < 0.3] = 0                                 # rows that see nothing of the tree
    for dtype in (torch.bfloat16, torch.float32):
        for mask in (None, c.trees(words), any_bits):
            q = c.queries(dtype)
            out = c.attend(q, mask)
            c.check(q, mask, out)
            for r, (n, b) in enumerate(zip(new, base)):
                if mask is any_bits and b == 0:
                    empty = ~c.seen(r, mask).any(1)
                    assert (out[c.row0[r]:c.row0[r + 1]][empty] == 0).all()


@pytest.mark.parametrize("new,base,heads,kvh,hd", [
    ([1], [40000], 8, 2, 128), ([9], [2048], 32, 32, 128), ([17, 3, 60], [8000, 100, 2500], 32, 8, 128), ([600], [0], 8, 4, 64), ([130], [1000], 8, 2, 128),
    ([1] * 64, [int(x) for x in np.linspace(0, 2900, 64)], 16, 4, 64), ([1] * 300, [31] * 300, 4, 4, 128), ([64] * 3, [20000, 1, 4000], 8, 2, 128),
    ([3] * 40, [int(x) for x in np.linspace(1, 900, 40)], 8, 2, 64)])
def test_attend_large(new, base, heads, kvh, hd):
    import torch
    c = Case(sum(new), new, base, heads, kvh, hd)
    c.fill()
    for dtype in (torch.bfloat16, torch.float32):
        for mask in (None, c.trees(-(-max(new) // 32))):
            q = c.queries(dtype)
            out = c.attend(q, mask)
            c.check(q, mask, out)
            assert torch.equal(out, c.attend(q, mask))                       # the same bits every time


def test_fp32_keeps_what_fp32_has():
    """Scores of up to 8 in magnitude lose 24 truncations of 2^-23 of their sums of magnitudes, of up to 16, at random: 2^-18 in the norm."""
    import torch
    for new, base, heads, kvh, hd in (([1], [16000], 32, 8, 128), ([20, 9, 5], [4000, 500, 1], 32, 8, 128), ([17, 3], [700, 2900], 8, 8, 64)):
        c = Case(9, new, base, heads, kvh, hd)
        c.fill()
        q = c.queries(torch.float32)
        mask = c.trees(1)
        out = c.attend(q, mask)
        for r, n in enumerate(new):
            rows = slice(int(c.row0[r]), int(c.row0[r + 1]))
            want = trees.attend(q[rows], c.k[r], c.v[r], c.seen(r, mask), hd ** -0.5)[0]
            assert (out[rows].double() - want).norm() < 2.0 ** -18 * want.norm()


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_attend_keeps_to_what_is_seen(dtype):
    """NaN and infinities in nodes that are not ancestors, in stale positions and on pages that are not there reach nobody; what is seen does."""
    import torch
    nan, inf = float("nan"), float("inf")
    dtype = getattr(torch, dtype)
    for heads, new, base in ((4, [40, 7], [150, 300]), (8, [64, 40], [300, 20])):
        c = Case(11, new, base, heads, 2, 128, hide=[(0, 2, -1), (1, 0, 10 ** 9)])
        mask = c.trees(2)
        c.fill()
        q = c.queries(dtype)
        clean = c.attend(q, mask)
        c.check(q, mask, clean)
        bad = 5                                                              # of request 0: K and V of this node, V of one of the prefix, of request 1
        c.k[0][base[0] + bad], c.v[0][base[0] + bad] = nan, inf
        c.v[0][base[0] + bad, 1] = nan
        c.v[0][base[0] + 9, 0, 17] = -inf
        c.v[1][base[1] + 3, 1, 100] = nan
        c.fill()
        out = c.attend(q, mask)
        c.check(q, mask, torch.where(torch.isinf(out), nan, out))
        sees = trees.bits_of(mask, 64)
        same = np.ones(c.rows, bool)
        same[:new[0]] = ~(sees[:new[0], bad] | sees[:new[0], 9])
        same[new[0]:] = ~sees[new[0]:, 3]
        assert same.any() and not same.all()
        same = torch.from_numpy(same).cuda()
        assert torch.equal(out[same], clean[same])
        # a prefix that holds a NaN reaches every row of its request and no other
        c.v[1][17, 0, 5] = nan
        c.fill()
        got = c.attend(q, mask)
        assert torch.isnan(got[new[0]:, :heads // 2, 5]).all() and torch.equal(got[:new[0]].nan_to_num(), out[:new[0]].nan_to_num())
        # queries
        q[3, 1] = nan
        got = c.attend(q, mask)
        assert torch.isnan(got[3, 1]).all() and torch.equal(got[4:new[0]].nan_to_num(), out[4:new[0]].nan_to_num())


def test_attend_scores_that_grow():
    import torch
    for sign in (1, -1):
        c = Case(13, [40], [700], 4, 2, 128)
        c.k[0] *= (torch.arange(740, device="cuda") * 0.05 * sign + (0 if sign > 0 else 40))[:, None, None]
        c.fill()
        for dtype in (torch.bfloat16, torch.float32):
            q, mask = c.queries(dtype), c.trees(2)
            c.check(q, mask, c.attend(q, mask))
            c.check(q, mask, c.attend(q, mask, scale=0.3), 0.3)


def test_attend_strides_streams_and_graphs():
    import torch
    c = Case(14, [20, 1, 40], [700, 30, 1990], 16, 4, 128)
    c.fill()
    for dtype in (torch.bfloat16, torch.float32):
        q, mask = c.queries(dtype), c.trees(2)
        bits = _ints(mask.view(np.int32))
        out = c.attend(q, mask)
        wide = torch.full((c.rows, 48, 128), float("nan"), device="cuda", dtype=dtype)
        wide[:, 8:24] = q
        odd = torch.full((c.rows, 16 * 128 + 1), 3.0, device="cuda", dtype=dtype)
        target = odd[:, 1:].unflatten(1, (16, 128))                          # rows at odd addresses
        assert torch.equal(c.attend(wide[:, 8:24], mask, out=target), out) and (odd[:, 0] == 3).all()
        assert torch.equal(c.cache.attend(target.copy_(q), *c.where, mask=bits), out)
        streams = [torch.cuda.Stream() for _ in range(3)]
        torch.cuda.synchronize()
        many = [c.cache.attend(q, *c.where, mask=bits, stream=s) for _ in range(5) for s in streams]
        torch.cuda.synchronize()
        assert all(torch.equal(x, out) for x in many)
        graphs, outs = [], []
        k = torch.randn((c.rows, 4, 128), device="cuda", dtype=torch.bfloat16)
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                c.cache.append(k, k, *c.where)
                outs.append(c.cache.attend(q, *c.where, mask=bits))
            graphs.append(g)
        for shift in (0, -25):
            c.where[1].copy_(_ints([700 + shift, 30 + shift, 1990 + shift]))
            for g in (graphs[1], graphs[0], graphs[1]):
                g.replay()
            torch.cuda.synchronize()
            want = c.cache.attend(q, *c.where, mask=bits)
            assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
        c.where[1].copy_(_ints([700, 30, 1990]))
        c.fill()


@pytest.mark.parametrize("new,base,heads,kvh,hd,page", [
    ([1] * 400, [int(x) for x in np.linspace(0, 800, 400)], 8, 2, 64, 16), ([100] + [1] * 40, [300] + [129] * 40, 8, 2, 128, 16),
    ([0] * 70 + [3] * 70, [50] * 70 + [int(x) for x in np.linspace(0, 500, 70)], 6, 2, 128, 24), ([16] * 9, [200] * 9, 4, 1, 128, 8),
    ([17] * 9, [200] * 9, 4, 1, 128, 8), ([2] * 1500, [30] * 1500, 2, 1, 64, 16), ([0, 0, 1, 0], [5, 6000, 5000, 0], 32, 8, 128, 64),
    ([64], [1000], 8, 8, 128, 16), ([65], [1000], 8, 8, 128, 16), ([1], [0], 64, 1, 64, 16)])
def test_many_requests_with_few_rows(new, base, heads, kvh, hd, page):
    """Up to 64 query rows by KV head a request on average, and just beyond; groups of more than 128 rows among them; requests without rows."""
    import torch
    c = Case(len(new), new, base, heads, kvh, hd, page)
    c.fill()
    for mask in (None, c.trees(-(-max(new) // 32))):
        q = c.queries(torch.bfloat16)
        out = c.attend(q, mask)
        c.check(q, mask, out)
        assert all(torch.equal(out, c.attend(q, mask)) for _ in range(5))
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        both = [c.attend(q, mask, stream=st) for _ in range(4) for st in (None, side)]
        torch.cuda.synchronize()
        assert all(torch.equal(out, x) for x in both)


def test_few_rows_scores_that_grow_and_graphs():
    import torch
    c = Case(17, [20, 1, 0, 5], [700, 30, 0, 256], 4, 2, 128)
    c.k[0] *= (torch.arange(720, device="cuda") * 0.05)[:, None, None]
    c.fill()
    q, mask = c.queries(torch.bfloat16), c.trees(1)
    bits = _ints(mask.view(np.int32))
    c.check(q, mask, c.attend(q, mask))
    odd = torch.full((c.rows, 4 * 128 + 1), 3.0, device="cuda", dtype=q.dtype)[:, 1:].unflatten(1, (4, 128))       # rows at odd addresses
    want = c.attend(q, mask)
    assert torch.equal(c.attend(q, mask, out=odd), want) and torch.equal(c.attend(odd.copy_(q), mask), want)
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(c.cache.attend(q, *c.where, mask=bits))
        graphs.append(g)
    for shift in (0, -25, -30):
        c.where[1].copy_(_ints([700 + shift, 30 + shift, 0, 256 + shift]))
        for g in (graphs[1], graphs[0], graphs[1]):
            g.replay()
        torch.cuda.synchronize()
        want = c.cache.attend(q, *c.where, mask=bits)
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


def test_rows_of_requests_without_positions():
    """A base below 0 or behind the table: zeros, however many rows; the other requests' rows are theirs."""
    import torch
    for heads in (4, 8):                           # few rows and many
        c = Case(19, [7] * 40 + [30], [100] * 41, heads, 2, 64)
        c.fill()
        q = c.queries(torch.bfloat16)
        want = c.attend(q, None)
        c.where[1][[3, 20, 40]] = _ints([-1, 10 ** 6, -2 ** 31])
        out = c.attend(q, None, out=torch.full_like(q, 5.0))
        gone = [*range(21, 28), *range(140, 147), *range(280, 310)]
        assert (out[gone] == 0).all()
        want[gone] = 0
        c.where[1][[3, 20, 40]] = 100
        assert torch.equal(out == 0, want == 0) and ((out.double() - want.double()).norm() < 2.0 ** -7 * want.double().norm())


def test_pools_of_another_shape_are_refused():
    import torch
    from paper_2605_13319_b200 import binding
    pool = torch.zeros((1, 4, 2, 2, 2, 8, 8, 8), dtype=torch.bfloat16, device="cuda")       # two heads of 64, 16 positions a page
    assert binding.Kv16Cache(2, 64, pool=pool).n_pages == 4
    for kvh, hd, page in ((4, 64, 8), (1, 64, 32), (1, 128, 16), (2, 64, 8)):
        with pytest.raises(AssertionError):
            binding.Kv16Cache(kvh, hd, pool=pool, page_size=page)
    with pytest.raises(AssertionError):
        binding.Kv16Cache(2, 64, pool=pool.flatten(), n_pages=3)
    assert binding.Kv16Cache(2, 64, pool=pool.flatten(), n_pages=4).n_layers == 1


def test_offsets_beyond_32_bits():
    """A pool of 10 GB, 5 * 10^9 values: a request whose pages lie at its end."""
    import torch
    from paper_2605_13319_b200 import binding
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GB")
    kvh, hd, page, layers = 8, 128, 64, 2
    n_pages = (5 << 30) // (layers * 2 * kvh * page * hd * 2)
    pool = torch.empty((layers, 2 * n_pages, 2, kvh, page // 8, hd // 8, 8, 8), dtype=torch.bfloat16, device="cuda")
    cache = binding.Kv16Cache(kvh, hd, pool=pool, page_size=page)
    far = torch.arange(2 * n_pages - 1, 2 * n_pages - 6, -1, dtype=torch.int32, device="cuda")[None].contiguous()
    near = torch.arange(5, dtype=torch.int32, device="cuda")[None].contiguous()
    k, v = (torch.randn((300, kvh, hd), device="cuda") for _ in range(2))
    q = torch.randn((40, 16, hd), device="cuda", dtype=torch.bfloat16)
    got = []
    for table in (far, near):
        cache.append(k, v, _ints([0, 300]), _ints([0]), table, layer=1)
        cache.append(v, k, _ints([0, 300]), _ints([0]), table, layer=0)
        kept = cache.compact(_ints([[0x0ff0f0f0, 0x7]]), _ints([200]), table)
        got.append([cache.attend(q, _ints([0, 40]), _ints([260]), table, layer=1), kept, *cache.read(300, _ints([0, 300]), _ints([0]), table, layer=1)])
    assert all(torch.equal(x, y) for x, y in zip(*got))


def test_the_pass_has_the_same_layout():
    """A context's own K/V memory, taken as a pool: what the pass wrote is read, attended and forked by these calls."""
    import torch
    from paper_2605_13319_b200 import binding, synth
    shape = synth.TINY
    ctx = binding.Context(shape, synth.make_weights(shape, 0), n_pages=16, max_seq=128)
    req = ctx.req_open()
    ctx.prefill(req, synth.make_prefix(shape, 50, 0))
    cache = binding.Kv16Cache(shape.n_kv_heads, shape.head_dim, n_layers=shape.n_layers, n_pages=16, page_size=16,
                              pool=ctx._kvbuf[:shape.n_layers * 16 * 2 * shape.n_kv_heads * 16 * shape.head_dim * 2].view(torch.bfloat16))
    want = {l: ctx.debug_read_kv(req, l, 0, 50) for l in range(shape.n_layers)}
    hits = 0
    for first in range(16):                                                  # the context's pages of one request: four in a row, up or down
        for step in (1, -1):
            table = [first + step * i for i in range(4)]
            if min(table) < 0 or max(table) > 15:
                continue
            got = cache.read(50, _ints([0, 50]), _ints([0]), _ints([table]), layer=1)
            same = all(np.array_equal(x.view(torch.int16).cpu().numpy().view(np.uint16).reshape(50, -1), y) for x, y in zip(got, want[1]))
            hits += same
    assert hits == 1
    ctx.close()
