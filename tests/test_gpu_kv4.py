"""The 4-bit K/V cache (pipesd_kv4_*) against 64-bit numpy: bytes after an append, values, attention."""
import numpy as np
import pytest

from oracle import serving

pytestmark = pytest.mark.gpu


class Case:
    """Requests with pages in no order; the pool starts as noise, NaN scales among it."""

    def __init__(self, rng, new, base, kv_heads, hd, page=16, spare=2, hide=()):
        import torch
        from paper_2605_13319_b200 import binding
        self.new, self.base, self.kvh, self.hd, self.page = list(new), list(base), kv_heads, hd, page
        self.row0 = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.rows = int(self.row0[-1])
        used = [-(-(b + n) // page) for b, n in zip(base, new)]
        self.n_pages = sum(used) + spare
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(new), max(max(used), 1) + 1), -1, np.int32)
        at = 0
        for r, n in enumerate(used):
            self.table[r, :n] = order[at:at + n]
            at += n
        for r, c, v in hide:
            self.table[r, c] = v
        pool = rng.integers(0, 256, (self.n_pages, kv_heads, page // 16, 20 * hd)).astype(np.uint8)
        pool[rng.random(pool.shape) < 0.2] = 255
        self.ref = serving.Cache(pool.copy(), hd, page)
        self.pool = torch.from_numpy(pool).cuda()
        self.cache = binding.Kv4Cache(kv_heads, hd, pool=self.pool, page_size=page)
        self.where = [torch.from_numpy(a).cuda() for a in (self.row0, np.array(base, np.int32), self.table)]

    def row(self, r, i):
        return int(self.row0[r]) + i

    def write_ref(self, k, v, base=None):
        for r, n in enumerate(self.new):
            for i in range(n):
                for h in range(self.kvh):
                    for kv, x in enumerate((k, v)):
                        self.ref.write(self.table[r], h, (base or self.base)[r] + i, kv, x[self.row(r, i), h])

    def fill(self, rng, spread=None):
        """Values in every position before the new rows too (written by the 64-bit form, bytes sent over)."""
        import torch
        for r, b in enumerate(self.base):
            for pos in range(b):
                for h in range(self.kvh):
                    for kv in range(2):
                        x = rng.standard_normal(self.hd) if spread is None else spread(rng, r, pos, h, kv)
                        self.ref.write(self.table[r], h, pos, kv, x)
        self.pool.copy_(torch.from_numpy(self.ref.pool))


def _rows(rng, rows, heads, hd, dtype, std=1.0):
    import torch
    return torch.from_numpy((rng.standard_normal((rows, heads, hd)) * std).astype(np.float32)).cuda().to(dtype)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new,base,page", [
    ([1], [0], 16), ([1], [15], 16), ([1], [16], 16), ([2], [15], 16), ([16], [0], 16), ([17], [7], 48), ([1, 1, 1], [3, 31, 64], 32),
    ([5, 0, 40, 1], [9, 4, 30, 0], 16), ([100], [3], 64)])
def test_append_bytes_and_values(new, base, page, hd):
    import torch
    rng = np.random.default_rng(sum(new) + hd)
    for heads, dtype in ((1, torch.float32), (3, torch.bfloat16)):
        c = Case(rng, new, base, heads, hd, page)
        k, v = (_rows(rng, c.rows, heads, hd, dtype, s) for s in (2.0, 0.01))
        c.cache.append(k, v, *c.where)
        c.write_ref(k.double().cpu().numpy(), v.double().cpu().numpy())
        assert np.array_equal(c.pool.cpu().numpy(), c.ref.pool)              # codes, scales, and every byte that is no row's
        got = c.cache.read(c.rows, *c.where)
        for x, y in zip((k, v), got):
            codes, s, z = serving.quantise(x.double().cpu().numpy())
            want = serving.values(codes, s, z)
            assert (np.abs(y.cpu().numpy() - want) <= np.abs(want) * 2.0 ** -24).all()      # one rounding to fp32
            err = np.abs(y.double().cpu().numpy() - x.double().cpu().numpy()).reshape(*s.shape, 32)
            # half a step, and what the roundings of the zero and of the scale (2^-8 each, the scale 15 times) push over the ends
            span = 15 * s[..., None]
            assert (err <= 0.5 * s[..., None] + 2.0 ** -8 * (np.abs(z[..., None]) + span) + 1e-30).all()


def test_append_special_values():
    import torch
    rng = np.random.default_rng(1)
    c = Case(rng, [8], [5], 2, 64)
    k, v = (_rows(rng, 8, 2, 64, torch.float32) for _ in range(2))
    k[0] = 1.003                                                             # constant groups
    k[1, 0, :32] = 0.0
    k[2, 0, 3], k[2, 1, 5], k[2, 1, 40] = float("nan"), float("inf"), float("-inf")
    k[3] = float("nan")
    k[4, 0] *= 1e30                                                          # beyond the limit
    k[5, 0] = 1e-40
    v[6] = v[6] * 1e-42
    v[7, 0, :31], v[7, 0, 31] = -1.0, 1e6
    c.cache.append(k, v, *c.where)
    c.write_ref(k.double().cpu().numpy(), v.double().cpu().numpy())
    assert np.array_equal(c.pool.cpu().numpy(), c.ref.pool)
    assert all(torch.isfinite(x).all() for x in c.cache.read(8, *c.where))


def test_append_from_a_fused_projection_and_rows_that_have_no_page():
    import torch
    rng = np.random.default_rng(2)
    hd, heads = 128, 2
    c = Case(rng, [20, 3, 4], [10, 60, 0], heads, hd, hide=[(0, 1, -1), (2, 0, 10 ** 6)])      # 16..31 of request 0; all of request 2
    c.table = c.table[:, :5].copy()
    c.where[2] = torch.from_numpy(c.table).cuda()
    c.new[1] = 3
    qkv = _rows(rng, c.rows, 3 * heads, hd, torch.bfloat16)
    k, v = qkv[:, heads:2 * heads], qkv[:, 2 * heads:]
    before = c.pool.clone()
    c.cache.append(k, v, *c.where)
    c.write_ref(k.double().cpu().numpy(), v.double().cpu().numpy())
    assert np.array_equal(c.pool.cpu().numpy(), c.ref.pool)
    read_k, _ = c.cache.read(c.rows, *c.where)
    assert (read_k[6:20] == 0).all() and (read_k[23:] == 0).all()            # positions 16..29 of request 0, request 2
    # rows behind the table's last position, negative bases, row0 that makes no sense: dropped
    c.pool.copy_(before)
    w = [torch.tensor([0, 20, 19, 27], dtype=torch.int32, device="cuda"), torch.tensor([80, 5, -1], dtype=torch.int32, device="cuda"), c.where[2]]
    c.cache.append(k, v, *w)
    assert torch.equal(c.pool, before)
    q = _rows(rng, c.rows, 4, hd, torch.bfloat16)
    out = c.cache.attend(q, *w)
    assert (out[:19] == 0).all()


def _attend_check(c, q, scale, out):
    """Elementwise bounds, counted from the kernel's roundings.  With S = sum over the positions of p (s |c - 8| + |z + 8 s|):
    fp16 P, P s and middles, 2^-11 each, one for the scores' error times two; bf16 output 2^-8 of the result.
    fp32: two fp16 terms, 2^-22 each (and 2^-22 of the exponential, 2^-23 per unit's addition on the tensor cores, which truncate,
    over at most 32 additions per warp here); scores lose 2^-21 of their sum of magnitudes."""
    import torch
    half = q.dtype == torch.bfloat16
    x, got = q.double().cpu().numpy(), out.double().cpu().numpy()
    G = x.shape[1] // c.kvh
    for r, n in enumerate(c.new):
        for h in range(c.kvh):
            for i in range(n):
                row, heads = c.row(r, i), slice(h * G, (h + 1) * G)
                want, size, mag = c.ref.attend(x[row, heads], c.table[r], h, c.base[r] + i, scale)
                score = mag[:, None] * 2.0 ** -21
                tol = 2.0 ** -8 * np.abs(want) + (4 * 2.0 ** -11 + 2 * score) * size if half else \
                    2.0 ** -24 * np.abs(want) + (5 * 2.0 ** -22 + 32 * 2.0 ** -23 + 2 * score) * size
                bad = np.abs(got[row, heads] - want) > tol + 1e-30
                assert not bad.any(), (r, h, i, np.abs(got[row, heads] - want).max(), tol.min())


@pytest.mark.parametrize("hd,heads,kvh", [(64, 2, 2), (128, 4, 1), (128, 6, 2), (64, 16, 2), (128, 2, 2), (64, 5, 1)])
@pytest.mark.parametrize("new,base,page", [
    ([1], [0], 16), ([1], [1], 16), ([1], [15], 16), ([1], [127], 16), ([9], [40], 32), ([17], [0], 16), ([1, 1, 1, 1], [3, 200, 64, 0], 16),
    ([5, 0, 2, 16], [130, 4, 16, 300], 48), ([33], [5], 16)])
def test_attend_matches(hd, heads, kvh, new, base, page):
    import torch
    rng = np.random.default_rng(hd + heads + sum(new) + sum(base))
    c = Case(rng, new, base, kvh, hd, page)
    c.fill(rng)
    k, v = (_rows(rng, c.rows, kvh, hd, torch.float32) for _ in range(2))
    c.cache.append(k, v, *c.where)
    c.write_ref(k.double().cpu().numpy(), v.double().cpu().numpy())
    for dtype in (torch.bfloat16, torch.float32):
        q = _rows(rng, c.rows, heads, hd, dtype, 1.5)
        _attend_check(c, q, hd ** -0.5, c.cache.attend(q, *c.where))


def _by_position(f):
    return lambda rng, r, pos, h, kv: rng.standard_normal(128) * f(pos, kv)


@pytest.mark.parametrize("name,spread", [
    ("growing scores", _by_position(lambda pos, kv: 1 + 0.03 * pos if kv == 0 else 1.0)),
    ("growing values", _by_position(lambda pos, kv: 1.0 if kv == 0 else 2.0 ** (pos // 16 * 3 - 30))),
    ("shrinking values", _by_position(lambda pos, kv: 1.0 if kv == 0 else 2.0 ** (20 - pos // 16 * 3))),
    ("offset values", lambda rng, r, pos, h, kv: rng.standard_normal(128) * (1.0 if kv == 0 else 0.1) + (0.0 if kv == 0 else 7.0)),
    ("offset keys", lambda rng, r, pos, h, kv: rng.standard_normal(128) + (3.0 * (np.arange(128) % 7 == 0) if kv == 0 else 0.0)),
    ("zero values", lambda rng, r, pos, h, kv: rng.standard_normal(128) * (1 - kv)),
    ("equal keys", lambda rng, r, pos, h, kv: np.full(128, 0.5) if kv == 0 else rng.standard_normal(128)),
])
def test_attend_ranges(name, spread):
    """Scores and scales that leave what the first unit of a warp set, in both directions; large middles; all-zero values."""
    import torch
    rng = np.random.default_rng(len(name))
    c = Case(rng, [3], [300], 1, 128)
    c.fill(rng, spread)
    k, v = (torch.from_numpy(np.stack([spread(rng, 0, 300 + i, 0, kv) for i in range(3)]).astype(np.float32)[:, None]).cuda() for kv in range(2))
    c.cache.append(k, v, *c.where)
    c.write_ref(k.double().cpu().numpy(), v.double().cpu().numpy())
    for dtype in (torch.bfloat16, torch.float32):
        for std in (0.01, 2.0, 20.0):
            q = _rows(rng, 3, 2, 128, dtype, std)
            _attend_check(c, q, 128 ** -0.5, c.cache.attend(q, *c.where))


def test_attend_pages_that_are_not_there():
    import torch
    rng = np.random.default_rng(3)
    c = Case(rng, [4, 2, 3], [100, 40, 0], 2, 64, hide=[(0, 2, -1), (0, 5, 10 ** 9), (2, 0, -5)])
    c.fill(rng)
    k, v = (_rows(rng, c.rows, 2, 64, torch.bfloat16) for _ in range(2))
    c.cache.append(k, v, *c.where)
    c.write_ref(k.double().cpu().numpy(), v.double().cpu().numpy())
    for dtype in (torch.bfloat16, torch.float32):
        q = _rows(rng, c.rows, 4, 64, dtype)
        out = c.cache.attend(q, *c.where)
        _attend_check(c, q, 0.125, out)
        assert (out[6:] == 0).all()


def _big(seed, new, base, heads, kvh, hd, dtype, page=16):
    """A case too large for the 64-bit loops, with a plain 64-bit form on the device."""
    import torch
    from paper_2605_13319_b200 import binding
    g = torch.Generator("cuda").manual_seed(seed)
    row0 = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")
    rows, used = sum(new), [-(-(b + n) // page) for b, n in zip(base, new)]
    order = torch.randperm(sum(used), generator=g, device="cuda").int()
    table = torch.full((len(new), max(used)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for r, n in enumerate(used):
        table[r, :n] = order[at:at + n]
        at += n
    cache = binding.Kv4Cache(kvh, hd, n_pages=sum(used), page_size=page)
    cache.pool.fill_(255)
    outs, wants = [], []
    full_k = [torch.randn((b + n, kvh, hd), generator=g, device="cuda") for b, n in zip(base, new)]
    full_v = [torch.randn((b + n, kvh, hd), generator=g, device="cuda") for b, n in zip(base, new)]
    zero = torch.zeros(len(new), dtype=torch.int32, device="cuda")
    whole0 = torch.tensor([0] + list(np.cumsum([b + n for b, n in zip(base, new)])), dtype=torch.int32, device="cuda")
    cache.append(torch.cat(full_k), torch.cat(full_v), whole0, zero, table)
    rk, rv = (t.double() for t in cache.read(int(whole0[-1]), whole0, zero, table))
    q = torch.randn((rows, heads, hd), generator=g, device="cuda").to(dtype)
    b = torch.tensor(base, dtype=torch.int32, device="cuda")
    out = cache.attend(q, row0, b, table)
    want = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    for r in range(len(new)):
        kk, vv = (t[int(whole0[r]):int(whole0[r + 1])].repeat_interleave(heads // kvh, 1) for t in (rk, rv))
        qq = q[int(row0[r]):int(row0[r + 1])].double()
        s = torch.einsum("rhc,lhc->hrl", qq, kk) * hd ** -0.5
        hidden = torch.arange(kk.shape[0], device="cuda")[None] > base[r] + torch.arange(new[r], device="cuda")[:, None]
        want[int(row0[r]):int(row0[r + 1])] = torch.einsum("hrl,lhc->rhc", torch.softmax(s.masked_fill(hidden, -float("inf")), -1), vv)
    return cache, (row0, b, table), q, out, want


@pytest.mark.parametrize("new,base,heads,kvh,hd", [
    ([1], [40000], 8, 2, 128), ([9], [2048], 32, 32, 128), ([17, 3, 9], [8000, 100, 3000], 32, 8, 128), ([600], [0], 8, 4, 64), ([130], [1000], 8, 2, 128),
    ([1] * 64, [int(x) for x in np.linspace(0, 3000, 64)], 16, 4, 64), ([1] * 100, [31] * 100, 4, 4, 128)])
def test_attend_large(new, base, heads, kvh, hd):
    import torch
    for dtype, tol in ((torch.bfloat16, 2.0 ** -8), (torch.float32, 2.0 ** -17)):
        cache, where, q, out, want = _big(sum(new), new, base, heads, kvh, hd, dtype)
        # relative to the outputs' norm: the roundings of _attend_check are independent from position to position, and a result's size
        # is that of the mean it is of; 2^-8 covers the output's own rounding, fp32 2^-22 times the score sums (below 2^5)
        rel = ((out.double() - want).norm() / want.norm()).item()
        assert rel < tol, rel
        assert torch.equal(out, cache.attend(q, *where))                     # the same bits every time


@pytest.mark.parametrize("new,base,heads,kvh,hd", [([1], [15], 8, 8, 128), ([1], [16000], 32, 8, 128), ([2, 9, 5], [4000, 500, 1], 32, 8, 128), ([17, 3], [700, 3000], 8, 8, 64)])
def test_attend_fp32_keeps_what_fp32_has(new, base, heads, kvh, hd):
    """Half steps of 22 bits (2^-23) for P, P s and the middles, twice that for Q's in scores of up to 2, an exponential off by 2^-22 at an
    argument of up to 16 (half a step 2^-21, times ln 2): 2^-20 together, in the norm."""
    import torch
    cache, where, q, out, want = _big(sum(new), new, base, heads, kvh, hd, torch.float32)
    rel = ((out.double() - want).norm() / want.norm()).item()
    assert rel < 2.0 ** -20, rel


def test_attend_strides_streams_and_graphs():
    import torch
    cache, where, q, out, _ = _big(3, [9, 1, 4], [700, 30, 2000], 16, 4, 128, torch.bfloat16)
    wide = torch.full((14, 48, 128), float("nan"), device="cuda", dtype=torch.bfloat16)
    wide[:, 8:24] = q
    target = torch.full((14, 48, 128), 3.0, device="cuda", dtype=torch.bfloat16)
    got = cache.attend(wide[:, 8:24], *where, out=target[:, 16:32])
    assert torch.equal(got, out)
    target[:, 16:32] = 3.0
    assert (target == 3.0).all()
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    many = [cache.attend(q, *where, stream=s) for _ in range(5) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(x, out) for x in many)
    # two graphs, replayed in any order, and one with the append before it: lengths are read when they run
    graphs, outs = [], []
    k = torch.randn((14, 4, 128), device="cuda", dtype=torch.bfloat16)
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            cache.append(k, k, *where)
            outs.append(cache.attend(q, *where))
        graphs.append(g)
    for shift in (0, -25):
        where[1].copy_(torch.tensor([700 + shift, 30 + shift, 2000 + shift], dtype=torch.int32))
        for g in (graphs[1], graphs[0], graphs[1]):
            g.replay()
        torch.cuda.synchronize()
        want = cache.attend(q, *where)
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


def test_attend_offsets_beyond_32_bits():
    """A pool of 4.3 GB: a request whose pages lie at its end."""
    import torch
    from paper_2605_13319_b200 import binding
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GB")
    kvh, hd, page = 8, 128, 64
    n_pages = (1 << 32) // (kvh * 4 * 20 * hd) + 40
    cache = binding.Kv4Cache(kvh, hd, n_pages=n_pages, page_size=page)
    far = torch.arange(n_pages - 1, n_pages - 6, -1, dtype=torch.int32, device="cuda")[None]
    near = torch.arange(5, dtype=torch.int32, device="cuda")[None]
    k, v = (torch.randn((300, kvh, hd), device="cuda") for _ in range(2))
    row0, base = torch.tensor([0, 300], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.randn((300, 16, hd), device="cuda", dtype=torch.bfloat16)
    got = []
    for table in (far, near):
        cache.append(k, v, row0, base, table.contiguous())
        got.append(cache.attend(q, row0, base, table.contiguous()))
    assert torch.equal(*got)


def test_serving_round_together():
    """A model of one layer, served as these operators are meant to be: the prompt's K and V appended and attended, the output
    projected by the library's GEMM, the pending token sampled; then draft steps (sampled with their distributions), one
    verification of all of them, and the cache rolled back to what was accepted.  Every step against the 64-bit forms on the
    step's own inputs; the verification's outputs are those of single steps."""
    import torch
    from paper_2605_13319_b200 import binding
    rng = np.random.default_rng(11)
    V, kvh, heads, hd, prompt, k = 1024, 2, 4, 64, 37, 4
    d = heads * hd
    g = torch.Generator("cuda").manual_seed(6)
    emb = torch.randn((V, d), generator=g, device="cuda")
    wq, wk, wv, wo = (torch.randn((n, d), generator=g, device="cuda").mul_(d ** -0.5).bfloat16() for n in (d, kvh * hd, kvh * hd, V))
    packed = [(binding.gemm_pack(w), w.shape[0]) for w in (wq, wk, wv, wo)]

    def project(x, which):
        w, n = packed[which]
        y = torch.empty((x.shape[0], n), device="cuda")
        binding.gemm_run(w, x.contiguous(), y, binding.gemm_scratch(x.shape[0], n, d, "cuda"), n, d)
        return y

    cache = binding.Kv4Cache(kvh, hd, n_pages=8)
    table = torch.tensor([[3, 1, 6, 0, 7, -1]], dtype=torch.int32, device="cuda")

    def step(tokens, base):
        x = emb[tokens.long()]
        n = x.shape[0]
        where = (torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.tensor([base], dtype=torch.int32, device="cuda"), table)
        cache.append(project(x, 1).view(n, kvh, hd), project(x, 2).view(n, kvh, hd), *where)
        q = project(x, 0).view(n, heads, hd)
        out = cache.attend(q, *where)
        ref = serving.Cache(cache.pool.cpu().numpy().reshape(8, kvh, 1, -1), hd, 16)
        for i in (0, n - 1):
            for h in range(kvh):
                want, size, mag = ref.attend(q[i, 2 * h:2 * h + 2].double().cpu().numpy(), table[0].tolist(), h, base + i, hd ** -0.5)
                assert (np.abs(out[i, 2 * h:2 * h + 2].double().cpu().numpy() - want) <= 2.0 ** -24 * abs(want) + (40 * 2.0 ** -23 + 2.0 ** -20 * mag[:, None]) * size).all()
        return project(out.reshape(n, d) * 3.0, 3)

    def uniforms(n):
        return torch.from_numpy((rng.integers(0, 1 << 24, n) * 2.0 ** -24).astype(np.float32)).cuda()

    tokens = torch.randint(V, (prompt,), generator=g, device="cuda").int()
    draft_set, target_set = dict(temperature=0.9, top_k=50), dict(temperature=0.7, top_p=0.95, min_p=0.01)
    length = prompt
    logits = step(tokens, 0)
    pending = binding.sample(logits[-1:], binding.shaping(1, **target_set), uniforms(1))
    for _ in range(3):
        chunk, rows, q = [pending], [], torch.empty((k, V), device="cuda")
        for i in range(k):
            rows.append(step(chunk[-1], length + i))
            noisy = rows[-1] + torch.randn((1, V), generator=g, device="cuda") * 0.3
            u = uniforms(1)
            chunk.append(binding.sample(noisy, binding.shaping(1, **draft_set), u, probs=q[i:i + 1]))
            assert chunk[-1].item() == serving.draw(serving.shaped(noisy[0].cpu().numpy(), 0.9, 50), u.item())[0]
        logits = step(torch.cat(chunk), length)
        single = torch.cat(rows)
        assert (logits[:k] - single).norm() <= 1e-4 * single.norm()          # the same positions, another order of sums
        u = uniforms(k + 1)
        drafts = torch.cat(chunk[1:])
        n, token = binding.accept(logits, torch.tensor([0, k + 1], dtype=torch.int32, device="cuda"), binding.shaping(1, **target_set), q, drafts, u)
        want = serving.accept(logits.cpu().numpy(), (0.7, 0, 0.95, 0.01), q.cpu().numpy(), drafts.cpu().numpy(), u.cpu().numpy())
        assert (n.item(), token.item()) == want[:2] or want[2] < 1e-9
        length += 1 + n.item()
        pending = token.clone()


def test_rows_of_no_request():
    """Rows behind the last request's: attention leaves them, reads give 0, appends drop them."""
    import torch
    rng = np.random.default_rng(4)
    c = Case(rng, [3, 2], [20, 0], 2, 128)
    c.fill(rng)                                                              # (positions 0..19 of request 0 are part of its cache)
    k, v = (_rows(rng, 8, 2, 128, torch.float32) for _ in range(2))
    c.cache.append(k, v, *c.where)
    c.write_ref(k.double().cpu().numpy(), v.double().cpu().numpy())
    assert np.array_equal(c.pool.cpu().numpy(), c.ref.pool)
    got = c.cache.read(8, *c.where)
    assert all((x[5:] == 0).all() and (x[3:5] != 0).any() for x in got)
    for dtype in (torch.bfloat16, torch.float32):
        q = _rows(rng, 8, 4, 128, dtype)
        out = torch.full_like(q, 9.0)
        c.cache.attend(q, *c.where, out=out)
        assert (out[5:] == 9.0).all() and torch.isfinite(out).all() and (out[:5] != 9.0).any()


def test_exact_ties_of_codes():
    """bf16 rows put quotients exactly on borders every few hundred values: to even, as in exact arithmetic."""
    import torch
    from paper_2605_13319_b200 import binding
    n = 4096
    g = torch.Generator("cuda").manual_seed(0)
    where = (torch.tensor([0, n], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"),
             torch.arange(n // 16, dtype=torch.int32, device="cuda")[None])
    for dtype in (torch.bfloat16, torch.float32):
        ties = 0
        for std, off in ((1.0, 0.0), (0.01, 3.0), (100.0, 1.0), (1e-20, 0.0)):
            k = (torch.randn((n, 2, 128), generator=g, device="cuda") * std + off).to(dtype)
            cache = binding.Kv4Cache(2, 128, n_pages=n // 16)
            cache.append(k, k, *where)
            x = k.double().unflatten(-1, (-1, 32))
            z = x.amin(-1, keepdim=True).bfloat16().double()
            s = ((x.amax(-1, keepdim=True) - z) / 15).bfloat16().double()
            q = (x - z) / torch.where(s > 0, s, 1.0)
            ties += int(((q - q.floor()) == 0.5).sum())
            want = (torch.round(q).clamp(0, 15) * (s > 0) * s + z).flatten(-2).float()
            assert all(torch.equal(y, want) for y in cache.read(n, *where))
        assert ties > 100 or dtype == torch.float32


@pytest.mark.parametrize("hd,heads,kvh", [(64, 4, 1), (128, 2, 2), (128, 8, 2)])
def test_attend_queries_that_are_no_numbers(hd, heads, kvh):
    """A NaN or an infinity in a query makes its row of its head a NaN, and nothing else."""
    import torch
    rng = np.random.default_rng(hd + heads)
    c = Case(rng, [5, 2], [90, 33], kvh, hd)
    c.fill(rng)
    k, v = (_rows(rng, c.rows, kvh, hd, torch.float32) for _ in range(2))
    c.cache.append(k, v, *c.where)
    c.write_ref(k.double().cpu().numpy(), v.double().cpu().numpy())
    for dtype in (torch.bfloat16, torch.float32):
        q = _rows(rng, c.rows, heads, hd, dtype)
        clean = c.cache.attend(q, *c.where)
        _attend_check(c, q, hd ** -0.5, clean)
        bad = {(0, 0): float("nan"), (2, 1): float("inf"), (4, heads - 1): float("-inf"), (6, 0): float("nan")}
        x = q.clone()
        for (row, head), value in bad.items():
            x[row, head, rng.integers(hd)] = value
        x[4, heads - 1, :2] = float("inf")
        out = c.cache.attend(x, *c.where)
        for (row, head) in bad:
            assert out[row, head].isnan().all()
            out[row, head] = clean[row, head]
        _attend_check(c, q, hd ** -0.5, out)


def _widen(c, units):
    """The same requests with a page table wide enough for `units` units of all of them."""
    import torch
    per = c.page // 16 * c.kvh * len(c.new)
    wide = np.full((len(c.new), -(-units // per)), -1, np.int32)
    wide[:, :c.table.shape[1]] = c.table
    c.table = wide
    c.where[2] = torch.from_numpy(wide).cuda()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("heads,kvh,new,base,page", [
    (2, 2, [9, 16, 11], [130, 0, 300], 16), (4, 1, [4, 3, 2, 3], [60, 250, 15, 1], 32), (8, 2, [9, 10, 8], [33, 200, 5], 48),
    (7, 1, [5, 0, 7, 7], [16, 40, 100, 31], 16), (16, 2, [1, 3, 2], [90, 17, 400], 16), (3, 1, [16, 1, 11], [2, 500, 64], 64)])
def test_attend_two_row_tiles(hd, heads, kvh, new, base, page):
    """9 to 16, 33 to 48 or many query rows of a KV head in the mean and work for all CTAs, going by the page table: CTAs of two row tiles.
    Ragged requests, of which one may have fewer rows than a tile, row groups that end inside a tile, units shared by several CTAs."""
    import torch
    rng = np.random.default_rng(hd + heads + sum(new) + sum(base))
    mean = -(-sum(new) // len(new)) * heads // kvh
    assert -(-mean // 16) * 16 * 5 <= -(-mean // 8) * 8 * 6
    c = Case(rng, new, base, kvh, hd, page)
    c.fill(rng)
    _widen(c, 50000)
    k, v = (_rows(rng, c.rows, kvh, hd, torch.float32) for _ in range(2))
    c.cache.append(k, v, *c.where)
    c.write_ref(k.double().cpu().numpy(), v.double().cpu().numpy())
    for dtype in (torch.bfloat16, torch.float32):
        q = _rows(rng, c.rows, heads, hd, dtype, 1.5)
        out = torch.full_like(q, 7.0)
        _attend_check(c, q, hd ** -0.5, c.cache.attend(q, *c.where, out=out))
        x = q.clone()
        x[1, 0, 3] = float("nan")
        again = c.cache.attend(x, *c.where)
        assert again[1, 0].isnan().all()
        again[1, 0] = out[1, 0]
        _attend_check(c, q, hd ** -0.5, again)


@pytest.mark.parametrize("name,spread", [
    ("growing scores", _by_position(lambda pos, kv: 1 + 0.03 * pos if kv == 0 else 1.0)),
    ("growing values", _by_position(lambda pos, kv: 1.0 if kv == 0 else 2.0 ** (pos // 16 * 3 - 30))),
    ("shrinking values", _by_position(lambda pos, kv: 1.0 if kv == 0 else 2.0 ** (20 - pos // 16 * 3))),
    ("offset values", lambda rng, r, pos, h, kv: rng.standard_normal(128) * (1.0 if kv == 0 else 0.1) + (0.0 if kv == 0 else 7.0)),
    ("zero values", lambda rng, r, pos, h, kv: rng.standard_normal(128) * (1 - kv))])
def test_attend_ranges_of_two_row_tiles(name, spread):
    import torch
    rng = np.random.default_rng(len(name))
    c = Case(rng, [6], [300], 1, 128)
    c.fill(rng, spread)
    _widen(c, 50000)
    k, v = (torch.from_numpy(np.stack([spread(rng, 0, 300 + i, 0, kv) for i in range(6)]).astype(np.float32)[:, None]).cuda() for kv in range(2))
    c.cache.append(k, v, *c.where)
    c.write_ref(k.double().cpu().numpy(), v.double().cpu().numpy())
    for dtype in (torch.bfloat16, torch.float32):
        for std in (0.01, 2.0, 20.0):
            q = _rows(rng, 6, 2, 128, dtype, std)                            # 12 query rows
            _attend_check(c, q, 128 ** -0.5, c.cache.attend(q, *c.where))


@pytest.mark.parametrize("new,base,heads,kvh,hd", [
    ([150, 50], [1200, 3000], 35, 5, 64), ([170], [4000], 33, 11, 128), ([9] * 8, [int(x) for x in np.linspace(500, 4000, 8)], 32, 32, 128), ([700], [0], 32, 8, 128)])
def test_attend_large_with_two_row_tiles(new, base, heads, kvh, hd):
    """Also merges whose warps take several heads of a row, and a number of heads that those do not divide.  Bounds as for one row tile."""
    import torch
    for dtype, tol in ((torch.bfloat16, 2.0 ** -8), (torch.float32, 2.0 ** -20)):
        cache, where, q, out, want = _big(sum(new), new, base, heads, kvh, hd, dtype)
        rel = ((out.double() - want).norm() / want.norm()).item()
        assert rel < tol, rel
        assert torch.equal(out, cache.attend(q, *where))


def test_a_prompt_does_not_go_by_the_width_of_the_page_table():
    """2000 rows are work for all CTAs however narrow their table is: the same kernel and the same bits as with a wide one."""
    import torch
    cache, where, q, out, _ = _big(1, [2000], [0], 8, 8, 128, torch.bfloat16)
    wide = torch.full((1, 4000), -1, dtype=torch.int32, device="cuda")
    wide[:, :where[2].shape[1]] = where[2]
    assert torch.equal(out, cache.attend(q, where[0], where[1], wide))


@pytest.mark.parametrize("hd", [64, 128])
def test_groups_of_one_value(hd):
    """Their zero, rounded to bf16, may lie above the value (a scale below 0) or on it (a scale of 0): code 0, which stands for the zero."""
    import torch
    rng = np.random.default_rng(hd)
    c = Case(rng, [20], [0], 2, hd)
    k, v = (_rows(rng, 20, 2, hd, torch.float32) for _ in range(2))
    for x, i in ((k, 0), (v, 3)):
        x[i] = 1.0059                                                        # (bf16: 1.0078)
        x[i + 1] = -1.0059                                                   # (bf16: -1.0078, below it)
        x[i + 2] = 1.5
        x[i + 3, 0] = 77.77
        x[i + 4, 1, 32:64] = 2.0 ** -20 * 1.0059
    c.cache.append(k, v, *c.where)
    c.write_ref(k.double().cpu().numpy(), v.double().cpu().numpy())
    assert np.array_equal(c.pool.cpu().numpy(), c.ref.pool)
    rk, rv = c.cache.read(20, *c.where)
    assert (rk[0] == 1.0078125).all() and (rv[3] == 1.0078125).all() and (rk[2] == 1.5).all() and (rv[5] == 1.5).all()
    scales = [float(serving.quantise(x[i, 0, :32].double().cpu().numpy())[1][0]) for x, i in ((k, 0), (k, 1), (k, 2))]
    assert scales[0] < 0 < scales[1] and scales[2] == 0
    for dtype in (torch.bfloat16, torch.float32):
        q = _rows(rng, 20, 4, hd, dtype)
        _attend_check(c, q, hd ** -0.5, c.cache.attend(q, *c.where))


@pytest.mark.parametrize("units", [0, 50000])
@pytest.mark.parametrize("hd", [64, 128])
def test_attend_scores_far_below_zero(hd, units):
    """scale * |q| just below 2^96 and keys that make every score -2^97 times their number of columns and less: still the softmax of
    them, which is the value of the one key that is smallest.  Few positions (most warps see none) and many."""
    import torch
    rng = np.random.default_rng(hd)
    for n in (12, 600):
        c = Case(rng, [n], [0], 1, hd)
        _widen(c, units or c.table.size)
        k = torch.ones((n, 1, hd), device="cuda") * (2.0 + torch.arange(n, device="cuda") % 8)[:, None, None]
        k[n // 2] = 1.0
        v = _rows(rng, n, 1, hd, torch.float32)
        c.cache.append(k, v, *c.where)
        _, held = c.cache.read(n, *c.where)
        for dtype in (torch.bfloat16, torch.float32):
            q = torch.full((n, 2, hd), -7.5e28, device="cuda").to(dtype)
            out = c.cache.attend(q, *c.where, scale=1.0)[n // 2:]
            want = held[n // 2].expand(n - n // 2, 2, hd)
            size = held[n // 2].abs().max() * 2.2                            # s |c - 8| + |z + 8 s|: 16 / 15 and 1 times the largest, and the roundings of s and z
            assert torch.isfinite(out).all()
            assert ((out.float() - want).abs() <= 2.0 ** -8 * want.abs() + 4 * 2.0 ** -11 * size).all()
