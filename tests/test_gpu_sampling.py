"""Shaped sampling and acceptance (pipesd_sample, pipesd_accept) against 64-bit numpy."""
import numpy as np
import pytest

from oracle import serving

pytestmark = pytest.mark.gpu

NEAR = 1e-9     # masses are rounded to 2^-46 of the most likely id's weight: over 2^18 ids a border moves by less than this


def _cuda(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def _rng_rows(rng, rows, vocab, kind):
    if kind == "peaked":
        x = rng.standard_normal((rows, vocab)) * 2
        for r in range(rows):
            x[r, rng.integers(0, vocab, 20)] += rng.uniform(2, 9, 20)
    elif kind == "flat":
        x = rng.standard_normal((rows, vocab)) * 0.01
    elif kind == "ties":
        x = rng.integers(-2, 3, (rows, vocab)).astype(np.float64)
    elif kind == "equal":
        x = np.full((rows, vocab), -0.0)
        x[:, ::2] = 0.0
    elif kind == "banned":      # most of the row masked: -inf and the type's lowest value
        x = rng.standard_normal((rows, vocab)) * 3
        x[rng.random((rows, vocab)) < 0.9] = -np.inf
        x[rng.random((rows, vocab)) < 0.5] = -3.3e38
        x[:, rng.integers(0, vocab)] = 0.25
    else:                       # a huge range
        x = rng.standard_normal((rows, vocab)) * 1e4
    return x.astype(np.float32)


def _settings(rng, rows, vocab):
    t = rng.choice([0.0, 1.0, 0.7, 0.3, 1.7, 1e-6, 50.0], rows)
    k = rng.choice([0, 0, 1, 2, 40, vocab - 1, vocab, vocab + 5, -3], rows)
    p = rng.choice([1.0, 1.0, 2.0, 0.9, 0.5, 0.999, 1 - 2.0 ** -24, 1e-6], rows)
    m = rng.choice([0.0, 0.0, 0.05, 0.5, 1.0, 1e-6], rows)
    return t.astype(np.float32), k.astype(np.int32), p.astype(np.float32), m.astype(np.float32)


def _check(logits, settings, u, tokens, probs=None):
    for r in range(len(logits)):
        s = [v[r] for v in settings]
        w = serving.shaped(logits[r], *s)
        if w is None or not 0 <= u[r] < 1:
            assert tokens[r] == -1
            if probs is not None:
                assert (probs[r] == 0).all()
            continue
        token, margin = serving.draw(w, u[r])
        assert tokens[r] == token or margin < NEAR, f"row {r}: {tokens[r]} for {token}, settings {s}, margin {margin}"
        if probs is not None:
            want = w / w.sum()
            # one rounding to fp32 (2^-24) and the sum's 2^-46 per id; below fp32's range the values are its subnormals
            assert (np.abs(probs[r] - want) <= want * (2.0 ** -24 + len(w) * 2.0 ** -46) + 2.0 ** -149).all(), f"row {r}: settings {s}"


@pytest.mark.parametrize("kind", ["peaked", "flat", "ties", "equal", "banned", "range"])
@pytest.mark.parametrize("rows,vocab", [(7, 1), (7, 2), (9, 31), (40, 33), (33, 1000), (6, 4099), (17, 8192), (5, 32000), (40, 32001), (3, 50257)])
def test_sample_matches(rows, vocab, kind):
    import torch
    from paper_2605_13319_b200 import binding
    rng = np.random.default_rng(vocab * 7 + rows)
    x, settings = _rng_rows(rng, rows, vocab, kind), _settings(rng, rows, vocab)
    u = (rng.integers(0, 1 << 24, rows) * 2.0 ** -24).astype(np.float32)
    u[0], u[-1] = 0.0, 1 - 2.0 ** -24
    t, k, p, m = settings
    shaping = binding.shaping(rows, temperature=t, top_k=k, top_p=p, min_p=m)
    for dtype in (torch.float32, torch.bfloat16):
        logits = _cuda(x, dtype)
        probs = torch.full((rows, vocab), float("nan"), device="cuda")
        tokens = binding.sample(logits, shaping, _cuda(u), probs=probs)
        again = binding.sample(logits, shaping, _cuda(u))
        assert torch.equal(tokens, again)
        _check(logits.float().cpu().numpy(), settings, u, tokens.cpu().numpy(), probs.cpu().numpy())


@pytest.mark.parametrize("rows", [1, 2, 30, 60, 130, 320])
def test_sample_large_vocabulary_every_cluster_size(rows):
    """The number of CTAs per row follows the number of rows; results do not."""
    import torch
    from paper_2605_13319_b200 import binding
    rng = np.random.default_rng(rows)
    vocab = 128256
    x = torch.randn((rows, vocab), generator=torch.Generator("cuda").manual_seed(rows), device="cuda") * 2
    settings = _settings(rng, rows, vocab)
    u = (rng.integers(0, 1 << 24, rows) * 2.0 ** -24).astype(np.float32)
    t, k, p, m = settings
    shaping = binding.shaping(rows, temperature=t, top_k=k, top_p=p, min_p=m)
    tokens = binding.sample(x, shaping, _cuda(u))
    some = rng.permutation(rows)[:12]
    _check(x[some].cpu().numpy(), [v[some] for v in settings], u[some], tokens.cpu().numpy()[some])
    for r in some[:3]:     # a row alone
        assert binding.sample(x[r:r + 1], shaping[r:r + 1].contiguous(), _cuda(u[r:r + 1])).item() == tokens[r].item()


def test_sample_most_ids_there_can_be():
    import torch
    from paper_2605_13319_b200 import binding
    x = torch.randn((2, 1 << 18), generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    x[1] = 1.5                                                       # all alike: the sum is 2^63
    u = np.array([0.37, 0.75], np.float32)
    tokens = binding.sample(x, binding.shaping(2, top_p=[0.9, 1.0]), _cuda(u)).cpu().numpy()
    _check(x.cpu().numpy(), [np.float32([1, 1]), np.int32([0, 0]), np.float32([0.9, 1]), np.float32([0, 0])], u, tokens)
    assert tokens[1] == 3 << 16


def test_sample_rows_without_a_distribution():
    import torch
    from paper_2605_13319_b200 import binding
    V, rows = 5000, 14
    x = np.random.default_rng(0).standard_normal((rows, V)).astype(np.float32)
    x[0] = -np.inf
    x[1, 4999] = np.nan
    x[2, 17] = np.inf
    x[3, 0] = -np.nan
    u = np.full(rows, 0.5, np.float32)
    u[4], u[5], u[6] = 1.0, -0.1, np.nan
    shaping = binding.shaping(rows)
    bits = shaping.cpu().numpy().copy()
    for r, (col, v) in {7: (0, -1.0), 8: (0, np.nan), 9: (0, np.inf), 10: (2, 0.0), 11: (2, np.nan), 12: (3, 1.01)}.items():
        bits[r, col] = np.float32(v).view(np.int32)
    probs = torch.full((rows, V), 7.0, device="cuda")
    tokens = binding.sample(_cuda(x), _cuda(bits), _cuda(u), probs=probs).cpu().numpy()
    assert (tokens[:13] == -1).all() and 0 <= tokens[13] < V
    assert (probs[:13] == 0).all() and abs(probs[13].sum().item() - 1) < 1e-5


@pytest.mark.parametrize("offset,ld", [(0, 1024), (1, 1031), (3, 1001), (4, 1004)])
def test_sample_strides_and_what_lies_between_rows(offset, ld):
    import torch
    from paper_2605_13319_b200 import binding
    rows, V = 9, 1000
    rng = np.random.default_rng(ld)
    settings = _settings(rng, rows, V)
    u = (rng.integers(0, 1 << 24, rows) * 2.0 ** -24).astype(np.float32)
    t, k, p, m = settings
    shaping = binding.shaping(rows, temperature=t, top_k=k, top_p=p, min_p=m)
    for dtype in (torch.float32, torch.bfloat16):
        flat = torch.full((rows * ld + offset + 8,), float("nan"), device="cuda", dtype=dtype)          # NaN wherever there is no logit
        logits = flat[offset:].as_strided((rows, V), (ld, 1))
        logits.copy_(_cuda(_rng_rows(rng, rows, V, "peaked")))
        out = torch.full((rows * ld + offset + 8,), 5.0, device="cuda")
        probs = out[offset:].as_strided((rows, V), (ld, 1))
        tokens = binding.sample(logits, shaping, _cuda(u), probs=probs)
        _check(logits.float().cpu().numpy(), settings, u, tokens.cpu().numpy(), probs.cpu().numpy())
        probs.fill_(5.0)
        assert (out == 5.0).all()


def test_sample_in_a_graph_and_on_other_streams():
    import torch
    from paper_2605_13319_b200 import binding
    rows, V = 20, 32000
    g = torch.Generator("cuda").manual_seed(1)
    logits, u = torch.randn((rows, V), generator=g, device="cuda") * 2, torch.rand(rows, generator=g, device="cuda")
    shaping, tokens = binding.shaping(rows, top_p=0.8, top_k=1000), torch.zeros(rows, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.sample(logits, shaping, u, tokens=tokens)
    for seed in (2, 3):
        logits.copy_(torch.randn((rows, V), generator=g, device="cuda") * 2)
        graph.replay()
        want = binding.sample(logits, shaping, u)
        assert torch.equal(tokens, want)
        streams = [torch.cuda.Stream() for _ in range(3)]
        torch.cuda.synchronize()
        got = [binding.sample(logits, shaping, u, stream=s) for s in streams for _ in range(4)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, want) for x in got)


def test_inputs_that_are_let_go_while_another_stream_waits():
    import torch
    from paper_2605_13319_b200 import binding
    rows, V = 20, 32000
    g = torch.Generator("cuda").manual_seed(1)
    logits, u = torch.randn((rows, V), generator=g, device="cuda") * 2, torch.rand(rows, generator=g, device="cuda")
    shaping, side = binding.shaping(rows, top_p=0.8), torch.cuda.Stream()
    want = binding.sample(logits, shaping, u)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    got = binding.sample(logits, shaping, u, stream=side)
    place = logits.data_ptr()
    del logits
    others = [torch.zeros((rows, V), device="cuda") for _ in range(2)]
    assert place not in [x.data_ptr() for x in others]
    torch.cuda.synchronize()
    assert torch.equal(got, want)


# --------------------------------------------------------------------------- acceptance
def _rounds(rng, ks, vocab, sharp):
    """Logits of all rows, q and drafts (from q) of all drafts, uniforms."""
    rows = sum(ks) + len(ks)
    logits = (rng.standard_normal((rows, vocab)) * 2).astype(np.float32)
    q, drafts, at = [], [], 0
    for k in ks:
        for i in range(k):
            e = logits[at + i].astype(np.float64) + sharp * rng.standard_normal(vocab)
            e = np.exp(e - e.max())
            e[e < np.sort(e)[-min(vocab, 50)]] = 0
            q.append((e / e.sum()).astype(np.float32))
            drafts.append(rng.choice(vocab, p=e / e.sum()))
        at += k + 1
    u = (rng.integers(0, 1 << 24, rows) * 2.0 ** -24).astype(np.float32)
    return logits, np.array(q, np.float32).reshape(-1, vocab), np.array(drafts, np.int32), u


@pytest.mark.parametrize("vocab", [16, 1000, 1024, 32000, 50257])
@pytest.mark.parametrize("ks", [[1], [8], [0, 3, 16, 1, 0, 5, 2], [31, 40]])
def test_accept_matches(vocab, ks):
    import torch
    from paper_2605_13319_b200 import binding
    rng = np.random.default_rng(vocab + len(ks))
    for trial, sharp in enumerate([0.1, 0.7, 2.0]):
        logits, q, drafts, u = _rounds(rng, ks, vocab, sharp)
        row0 = np.concatenate([[0], np.cumsum(np.array(ks) + 1)]).astype(np.int32)
        t, k, p, m = _settings(rng, len(ks), vocab)
        if trial == 0:
            t, k, p, m = (np.full(len(ks), v) for v in (np.float32(1), np.int32(0), np.float32(1), np.float32(0)))
        shaping = binding.shaping(len(ks), temperature=t, top_k=k, top_p=p, min_p=m)
        for dtype in (torch.float32, torch.bfloat16):
            dev = _cuda(logits, dtype)
            n, token = binding.accept(dev, _cuda(row0), shaping, _cuda(q), _cuda(drafts), _cuda(u))
            n2, token2 = binding.accept(dev, _cuda(row0), shaping, _cuda(q), _cuda(drafts), _cuda(u))
            assert torch.equal(n, n2) and torch.equal(token, token2)
            x = dev.float().cpu().numpy()
            for r in range(len(ks)):
                a, b, first = row0[r], row0[r + 1], row0[r] - r
                want = serving.accept(x[a:b], (t[r], k[r], p[r], m[r]), q[first:first + ks[r]], drafts[first:first + ks[r]], u[a:b])
                assert (n[r].item(), token[r].item()) == want[:2] or want[2] < NEAR, (r, want)


def test_accept_without_drafts_and_odd_requests():
    import torch
    from paper_2605_13319_b200 import binding
    rng = np.random.default_rng(5)
    V, n = 3001, 6
    x = rng.standard_normal((n, V)).astype(np.float32)
    u = rng.random(n).astype(np.float32)
    s = binding.shaping(n, top_k=20)
    got, token = binding.accept(_cuda(x), torch.arange(n + 1, dtype=torch.int32, device="cuda"), s, None, None, _cuda(u))
    assert (got == 0).all() and torch.equal(token, binding.sample(_cuda(x), s, _cuda(u)))
    # P = q wherever q is: nothing is left to correct with, a rejected draft (outside of the vocabulary) falls back to P
    row = rng.standard_normal((2, V)).astype(np.float32)
    P = serving.shaped(row[0], 1.0, 20)
    q = np.where(P > 0, 1.0, 0.0).astype(np.float32)[None]
    for draft in (-1, V, 1 << 30):
        u2 = np.array([0.0, 0.6], np.float32)
        got, token = binding.accept(_cuda(row), _cuda(np.int32([0, 2])), binding.shaping(1, top_k=20), _cuda(q), _cuda(np.int32([draft])), _cuda(u2))
        assert got.item() == 0 and token.item() == serving.draw(P, u2[1])[0]
    # a row without a distribution ends the round there; a bad final uniform gives no token; entries of row0 that make no sense: no round
    rows = rng.standard_normal((9, V)).astype(np.float32)
    rows[1] = -np.inf
    qq = np.full((6, V), 1e-9, np.float32)                          # accepts any draft of the support
    drafts = rows[[0, 1, 3, 4, 6, 7]].argmax(1).astype(np.int32)
    u3 = np.full(9, 0.5, np.float32)
    u3[5] = np.nan
    s3 = binding.shaping(3)
    got, token = binding.accept(_cuda(rows), _cuda(np.int32([0, 3, 6, 9])), s3, _cuda(qq), _cuda(drafts), _cuda(u3))
    assert got.tolist() == [1, 2, 2] and token[0].item() == -1 and token[1].item() == -1 and token[2].item() >= 0
    for bad in ([0, 3, 2, 9], [-1, 3, 6, 9], [0, 3, 6, 12], [0, 0, 6, 9], [5, -2 ** 31 + 3, 6, 9], [2 ** 31 - 1, -2 ** 31, 6, 9]):
        got, token = binding.accept(_cuda(rows), _cuda(np.int32(bad)), s3, _cuda(qq), _cuda(drafts), _cuda(u3))
        for r in range(3):
            if bad[r] < 0 or bad[r + 1] > 9 or bad[r + 1] <= bad[r]:
                assert got[r].item() == 0 and token[r].item() == -1


def test_greedy_settings_are_the_greedy_rule():
    import torch
    from paper_2605_13319_b200 import binding
    rng = np.random.default_rng(8)
    V, k = 1024, 6
    for cut in range(k + 1):
        x = rng.standard_normal((k + 1, V)).astype(np.float32)
        drafts = x.argmax(1)[:k].astype(np.int32)
        if cut < k:
            drafts[cut] = (drafts[cut] + 5) % V
        q = np.zeros((k, V), np.float32)
        q[np.arange(k), drafts] = 1
        u = rng.random(k + 1).astype(np.float32)
        n, token = binding.accept(_cuda(x), _cuda(np.int32([0, k + 1])), binding.shaping(1, temperature=0.0), _cuda(q), _cuda(drafts), _cuda(u))
        assert (n.item(), token.item()) == (cut, x[cut].argmax())


def test_draft_and_accept_leave_the_target_distribution():
    """One draft per request, sampled by pipesd_sample with its settings, verified by pipesd_accept with the target's: the first
    emitted token follows the target's shaped distribution whatever the draft's is."""
    import torch
    from paper_2605_13319_b200 import binding
    V, n = 24, 40000
    g = torch.Generator("cuda").manual_seed(4)
    edge, target, bonus = (torch.randn(V, generator=g, device="cuda") * 1.5 for _ in range(3))
    q = torch.empty((n, V), device="cuda")
    drafts = binding.sample(edge.expand(n, V).contiguous(), binding.shaping(n, temperature=0.8, top_k=12), torch.rand(n, generator=g, device="cuda"), probs=q)
    logits = torch.stack([target, bonus]).repeat(n, 1)
    row0 = torch.arange(0, 2 * n + 1, 2, dtype=torch.int32, device="cuda")
    acc, token = binding.accept(logits, row0, binding.shaping(n, temperature=1.2, top_p=0.9), q, drafts, torch.rand(2 * n, generator=g, device="cuda"))
    first = torch.where(acc == 1, drafts, token).cpu().numpy()
    w = serving.shaped(target.cpu().numpy(), 1.2, 0, 0.9)
    P = w / w.sum()
    share = np.bincount(first, minlength=V) / n
    assert (share[P == 0] == 0).all()
    assert (np.abs(share - P) <= 5 * np.sqrt(P * (1 - P) / n) + 1e-12).all()      # five standard deviations of a frequency
    assert 0 < acc.float().mean().item() < 1


def test_accept_in_a_graph_and_on_other_streams():
    import torch
    from paper_2605_13319_b200 import binding
    rng = np.random.default_rng(12)
    ks, V = [4, 0, 7], 8000
    logits, q, drafts, u = (_cuda(a) for a in _rounds(rng, ks, V, 0.7))
    row0 = _cuda(np.concatenate([[0], np.cumsum(np.array(ks) + 1)]).astype(np.int32))
    shaping = binding.shaping(3, temperature=[1.0, 0.8, 0.0], top_k=[0, 50, 0], top_p=[0.9, 1.0, 1.0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = binding.accept(logits, row0, shaping, q, drafts, u)
    for _ in range(3):
        u.copy_(torch.rand(u.shape, device="cuda"))
        graph.replay()
        want = binding.accept(logits, row0, shaping, q, drafts, u)
        torch.cuda.synchronize()
        got = [binding.accept(logits, row0, shaping, q, drafts, u, stream=s) for s in [torch.cuda.Stream() for _ in range(3)]]
        torch.cuda.synchronize()
        for a in [captured] + got:
            assert torch.equal(a[0], want[0]) and torch.equal(a[1], want[1])


@pytest.mark.parametrize("vocab", [40000, 128256])
def test_sample_windows_that_overflow_their_lists(vocab):
    """More ids than a list holds near a cut: dense flat tails (a third pass), thousands of equal logits at the cut (digit by digit)
    and a maximum far above the row's first ids (bins anew)."""
    import torch
    from paper_2605_13319_b200 import binding
    g = torch.Generator("cuda").manual_seed(vocab)
    rows = []
    for std in (0.05, 0.3):
        rows.append(torch.randn(vocab, generator=g, device="cuda") * std)
    rows.append(torch.randint(0, 3, (vocab,), generator=g, device="cuda").float())
    x = torch.randn(vocab, generator=g, device="cuda")
    x[-1] = 200.0
    rows.append(x)
    x = torch.randn(vocab, generator=g, device="cuda") * 2 - 500.0
    x[:4000] = -900.0
    rows.append(x)
    logits = torch.stack(rows)
    n = len(rows)
    rng = np.random.default_rng(7)
    for t, k, p, m in ((1.0, 0, 0.9, 0.0), (1.0, 0, 0.31, 0.0), (1.3, 5000, 1.0, 0.0), (0.9, 30000, 0.95, 0.0), (1.0, 1100, 0.5, 0.2), (60.0, 0, 0.999, 0.0), (0.02, 0, 0.99, 0.0)):
        u = (rng.integers(0, 1 << 24, n) * 2.0 ** -24).astype(np.float32)
        s = [np.full(n, v, d) for v, d in ((t, np.float32), (k, np.int32), (p, np.float32), (m, np.float32))]
        probs = torch.empty_like(logits)
        for dtype in (torch.float32, torch.bfloat16):
            y = logits.to(dtype)
            tokens = binding.sample(y, binding.shaping(n, temperature=t, top_k=k, top_p=p, min_p=m), _cuda(u), probs=probs)
            _check(y.float().cpu().numpy(), s, u, tokens.cpu().numpy(), probs.cpu().numpy())


@pytest.mark.parametrize("n", [20, 60, 300])          # clusters of eight, four and two CTAs per request
def test_accept_of_tiny_vocabularies_beside_other_work(n):
    """Most warps have no ids, so that totals cross the cluster at once, while another stream keeps the SMs busy."""
    import torch
    from paper_2605_13319_b200 import binding
    rng = np.random.default_rng(n)
    ks, V = [int(k) for k in rng.integers(0, 4, n)], 16
    logits, q, drafts, u = _rounds(rng, ks, V, 0.7)
    row0 = np.concatenate([[0], np.cumsum(np.array(ks) + 1)]).astype(np.int32)
    shaping = binding.shaping(n, temperature=0.9)
    args = [_cuda(logits), _cuda(row0), shaping, _cuda(q), _cuda(drafts), _cuda(u)]
    busy, busy_u, side = torch.randn((200, 32000), device="cuda"), torch.rand(200, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        binding.sample(busy, binding.shaping(200, top_p=0.9), busy_u, stream=side)
        got.append(binding.accept(*args))
    torch.cuda.synchronize()
    for a, b in got:
        assert torch.equal(a, got[0][0]) and torch.equal(b, got[0][1])
    for r in range(n):
        a, b, first = row0[r], row0[r + 1], row0[r] - r
        want = serving.accept(logits[a:b], (0.9, 0, 1.0, 0.0), q[first:first + ks[r]], drafts[first:first + ks[r]], u[a:b])
        assert (got[0][0][r].item(), got[0][1][r].item()) == want[:2] or want[2] < NEAR, (r, want)


@pytest.mark.parametrize("n", [3, 20, 45, 120])
def test_accept_where_entries_of_row0_make_no_sense(n):
    """Every request with settings of its own: those whose entries make sense get what they would get alone, the others (0, -1), however
    many of them claim a row.  Rows go by clusters and by single CTAs, requests by clusters of eight, four and two."""
    import torch
    from paper_2605_13319_b200 import binding
    rng = np.random.default_rng(n)
    V, rows = 17000, 4 * n
    logits = (rng.standard_normal((rows, V)) * 2).astype(np.float32)
    q = np.full((rows - n, V), 2e-5, np.float32)
    drafts = rng.integers(0, V, rows - n).astype(np.int32)
    u = (rng.integers(0, 1 << 24, rows) * 2.0 ** -24).astype(np.float32)
    t, k, p, m = (rng.choice(v, n) for v in ([0.0, 1.0, 0.7], [0, 0, 1, 40, 3000], [1.0, 0.9, 0.3], [0.0, 0.1]))
    settings = [v.astype(d) for v, d in ((t, np.float32), (k, np.int32), (p, np.float32), (m, np.float32))]
    shaping = binding.shaping(n, temperature=settings[0], top_k=settings[1], top_p=settings[2], min_p=settings[3])
    good = np.arange(0, rows + 1, 4).astype(np.int32)
    for trial in range(6):
        row0 = good.copy()
        if trial == 1:                                   # many requests claim the rows of others
            row0[2::2] = 0
        elif trial == 2:
            row0[1:n:3] = rows
        elif trial == 3:
            row0[n // 2] = -7
        elif trial == 4:
            row0 = rng.integers(0, rows + 1, n + 1).astype(np.int32)
        elif trial == 5:
            row0 = rng.permutation(good)
        got, token = (x.tolist() for x in binding.accept(_cuda(logits), _cuda(row0), shaping, _cuda(q), _cuda(drafts), _cuda(u)))
        for r in range(n):
            a, b, first = int(row0[r]), int(row0[r + 1]), int(row0[r]) - r
            if not (0 <= first and a < b <= rows and b - r - 1 <= rows - n and (row0[:r] <= a).all()):
                assert (got[r], token[r]) == (0, -1), (trial, r)
            elif rng.random() < 30 / n:
                want = serving.accept(logits[a:b], [v[r] for v in settings], q[first:first + b - a - 1], drafts[first:first + b - a - 1], u[a:b])
                assert (got[r], token[r]) == want[:2] or want[2] < NEAR, (trial, r, want)


@pytest.mark.parametrize("vocab", [40, 32000])
def test_accept_where_q_or_u_are_no_probabilities(vocab):
    """Every request has a result: NaN, infinities and numbers below 0 at the draft's q, elsewhere in its row, and among the uniforms."""
    import torch
    from paper_2605_13319_b200 import binding
    rng = np.random.default_rng(vocab)
    n = 24
    logits, q, drafts, u = _rounds(rng, [2] * n, vocab, 0.3)
    at_draft = [np.nan, -1.0, -np.inf, np.inf, -0.0, 0.0]
    for r, v in enumerate(at_draft):                                 # the first draft's own
        q[2 * r, drafts[2 * r]] = v
    for r, v in enumerate([np.nan, -0.25, -np.inf, np.inf]):         # the whole row of a draft that is not accepted
        q[2 * (6 + r)] = v
        drafts[2 * (6 + r)] = -1
    for r, v in enumerate([np.nan, -np.inf]):                        # one entry that top-k cuts, and one that it keeps
        worst, best = logits[3 * (10 + r)].argmin(), logits[3 * (10 + r)].argmax()
        q[2 * (10 + r), worst if r == 0 else best] = v
        drafts[2 * (10 + r)] = vocab
    for r, v in enumerate([np.nan, -0.5, -np.inf, 1.0, 2.0, np.inf]):        # a test's uniform
        u[3 * (12 + r)] = v
    for r, v in enumerate([np.nan, -0.5, 1.0, np.inf]):              # the last one
        u[3 * (18 + r) + 2] = v
    row0 = np.arange(0, 3 * n + 1, 3).astype(np.int32)
    for k in (0, 10):
        got, token = (x.tolist() for x in binding.accept(_cuda(logits), _cuda(row0), binding.shaping(n, top_k=k), _cuda(q), _cuda(drafts), _cuda(u)))
        for r in range(n):
            want = serving.accept(logits[3 * r:3 * r + 3], (1.0, k, 1.0, 0.0), q[2 * r:2 * r + 2], drafts[2 * r:2 * r + 2], u[3 * r:3 * r + 3])
            assert (got[r], token[r]) == want[:2] or want[2] < NEAR, (k, r, want)
            if r in (0, 1, 2, 3, 6, 7, 8, 9, 10, 11) or 12 <= r < 18:
                assert got[r] == 0
            if r in (6, 7, 8, 11) or 18 <= r < 22:
                assert token[r] == -1
        assert token[10] == -1 if k == 0 else token[10] >= 0


@pytest.mark.parametrize("n,vocab", [(20, 128256), (60, 32000), (60, 128256), (200, 32000), (200, 128256), (80, 1 << 18)])
def test_accept_of_many_requests_over_whole_vocabularies(n, vocab):
    """Clusters of eight, four and two CTAs per request, up to 32 batches of ids for a warp."""
    import torch
    from paper_2605_13319_b200 import binding
    rng = np.random.default_rng(n + vocab)
    g = torch.Generator("cuda").manual_seed(n)
    ks = rng.integers(0, 4, n) if vocab < 1 << 18 else np.ones(n, int)
    row0 = np.concatenate([[0], np.cumsum(ks + 1)]).astype(np.int32)
    rows = int(row0[-1])
    settings = _settings(rng, n, vocab)
    settings[0][settings[0] == np.float32(1e-6)] = 1.0
    shaping = binding.shaping(n, temperature=settings[0], top_k=settings[1], top_p=settings[2], min_p=settings[3])
    u = (rng.integers(0, 1 << 24, rows) * 2.0 ** -24).astype(np.float32)
    scored = np.setdiff1d(np.arange(rows), row0[1:] - 1)
    for dtype in (torch.float32, torch.bfloat16):
        logits = (torch.randn((rows, vocab), generator=g, device="cuda") * 2).to(dtype)
        q = torch.softmax(logits[torch.from_numpy(scored).cuda()].float() + torch.randn((rows - n, vocab), generator=g, device="cuda"), 1)
        drafts = torch.multinomial(q, 1, generator=g)[:, 0].int()
        got, token = binding.accept(logits, _cuda(row0), shaping, q, drafts, _cuda(u))
        for r in rng.permutation(n)[:8]:
            a, b, first = int(row0[r]), int(row0[r + 1]), int(row0[r] - r)
            mine = slice(first, first + int(ks[r]))
            want = serving.accept(logits[a:b].float().cpu().numpy(), [v[r] for v in settings], q[mine].cpu().numpy(), drafts[mine].cpu().numpy(), u[a:b])
            assert (got[r].item(), token[r].item()) == want[:2] or want[2] < NEAR, (r, want)
