"""Measured calls of the serving operators: shaped sampling and acceptance, and the 4-bit key/value cache.

Four operators, as a server of speculative decoding calls them around its passes:

  sample   tokens (and, for drafts, the distributions they came from) out of logits by temperature, top-k, top-p and min-p
  accept   the acceptance rule of speculative sampling for a target that is sampled with such settings
  append   K and V rows of a pass quantised to 4 bits into the pages of their requests, and read back
  attend   attention of every request's new rows over its 4-bit pages

Shapes are the repository's (synth: vocabularies of 1024, 32000 and 128256, heads of 64 and 128, 32 query heads over 8 or 32 KV
heads), prefix and draft lengths those of its benchmark.  Every token of a row's order is "higher logit first, lower id first".
"""
import math
import random

import torch

own = False

GROUP = 32          # columns that share a scale and a zero
UNIT = 16           # positions that are laid out together
LIMIT = 2.0 ** 48   # K and V values beyond are stored as this


# --------------------------------------------------------------------------- cases
def _sample(name, rows, vocab, filters, *, dtype="fp32", probs=False):
    return dict(name=name, op="sample", rows=rows, vocab=vocab, filters=filters, dtype=dtype, probs=probs)


def _accept(name, n_req, k_lo, k_hi, vocab, filters, *, dtype="fp32"):
    return dict(name=name, op="accept", n_req=n_req, k_lo=k_lo, k_hi=k_hi, vocab=vocab, filters=filters, dtype=dtype)


def _cache(name, op, n_req, n_lo, n_hi, p_lo, p_hi, heads, kv_heads, head_dim, *, dtype="bf16", page=16):
    return dict(name=name, op=op, n_req=n_req, n_lo=n_lo, n_hi=n_hi, p_lo=p_lo, p_hi=p_hi, heads=heads, kv_heads=kv_heads,
                head_dim=head_dim, dtype=dtype, page=page)


def listed():
    return [
        # the pending token of one request after its prompt: latency
        _sample("sample-1x32000", 1, 32000, "top_p"),
        # a draft model's step for 16 edges, with the q rows that the verification needs
        _sample("sample-16x32000-q", 16, 32000, "mixed", probs=True),
        # the requests of a large batch, every one with settings of its own, logits in 16 bits
        _sample("sample-256x128256", 256, 128256, "mixed", dtype="bf16"),
        # one edge's round of 8 drafts
        _accept("accept-1x8-32000", 1, 8, 8, 32000, "top_p"),
        # a ragged batch of rounds on the large vocabulary
        _accept("accept-32-128256", 32, 1, 16, 128256, "mixed"),
        # one token each for a batch of requests
        _cache("append-32x1", "append", 32, 1, 1, 256, 4096, 32, 8, 128),
        # a prompt of the headline's length on the 32-head shape
        _cache("append-2048", "append", 1, 2048, 2048, 0, 0, 32, 32, 128),
        # prompt chunks of several requests behind odd prefixes, activations in fp32, heads of 64
        _cache("append-5-ragged-fp32", "append", 5, 100, 700, 1, 1500, 32, 8, 64, dtype="fp32"),
        # one request, 8 drafts, 32 KV heads: the headline's attention
        _cache("attend-1x9-2048", "attend", 1, 9, 9, 2048, 2048, 32, 32, 128),
        # a single token over a very long context
        _cache("attend-1x1-131072", "attend", 1, 1, 1, 131071, 131071, 32, 8, 128),
        # single tokens of a batch of requests
        _cache("attend-32x1-4096", "attend", 32, 1, 1, 256, 4096, 32, 8, 128),
        # ragged rounds of a batch: up to 17 rows, four query heads per KV head, activations in fp32
        _cache("attend-16-ragged-fp32", "attend", 16, 2, 17, 256, 8192, 32, 8, 128, dtype="fp32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sample", "accept", "append", "attend", "attend"])
    if op in ("sample", "accept"):
        vocab = rng.choice([1024, 32000, 128256, _log_int(rng, 1000, 130000)])
        filters = rng.choice(["none", "top_k", "top_p", "min_p", "mixed", "mixed"])
        dtype = rng.choice(["fp32", "fp32", "bf16"])
        if op == "sample":
            c = _sample("", _log_int(rng, 1, 128), vocab, filters, dtype=dtype, probs=rng.random() < 0.4)
        else:
            k = rng.randint(1, 16)
            c = _accept("", _log_int(rng, 1, 24), rng.randint(1, k), k, vocab, filters, dtype=dtype)
    else:
        kv_heads, head_dim = rng.choice([(8, 128), (32, 128), (8, 64), (4, 64)])
        heads = kv_heads * rng.choice([1, 2, 4] if kv_heads < 32 else [1])
        dtype, page = rng.choice(["bf16", "bf16", "fp32"]), rng.choice([16, 16, 32, 64])
        n_req = _log_int(rng, 1, 24)
        if op == "append":
            n = _log_int(rng, 1, 2048 // n_req)
            c = _cache("", op, n_req, max(1, n // 3), n, 0, 1 + _log_int(rng, 1, 2000), heads, kv_heads, head_dim, dtype=dtype, page=page)
        else:
            n, p = rng.choice([1, 1, rng.randint(2, 17)]), _log_int(rng, 16, min(65536, 262144 // (n_req * kv_heads) * 4))
            c = _cache("", op, n_req, max(1, n // 2), n, max(1, p // 8), p, heads, kv_heads, head_dim, dtype=dtype, page=page)
    del c["name"]
    return c


# --------------------------------------------------------------------------- inputs, from the seed alone
_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _between(n, lo, hi):
    """n whole numbers of [lo, hi], the largest among them: lengths belong to the case, not to the seed."""
    rng = random.Random(1000003 * n + 1009 * lo + hi)
    v = [rng.randint(lo, hi) for _ in range(n)]
    v[n // 2] = hi
    return v


def _whole(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _spread_ids(gen, rows, n, vocab):
    """n different ids per row."""
    at = torch.arange(n, device="cuda") + torch.rand((rows, n), generator=gen, device="cuda", dtype=torch.float64) * 0.999
    return (at * (vocab / n)).long()


def _settings(gen, n, filters):
    """Rows of (temperature, top-k, top-p, min-p)."""
    def unit():
        return torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)

    def some(share):
        return unit() < share

    mixed = filters == "mixed"
    t = 0.5 + 0.8 * unit()
    k, p, mp = torch.floor(torch.exp(unit() * math.log(300.0))), 0.6 + 0.38 * unit(), 0.01 + 0.15 * unit()
    on = [some(0.5) if mixed else torch.full((n,), filters == f, device="cuda") for f in ("top_k", "top_p", "min_p")]
    if mixed:
        t = torch.where(some(0.1), 0.0, t)      # greedy requests among the others
    k, p, mp = torch.where(on[0], k, 0.0), torch.where(on[1], p, 1.0), torch.where(on[2], mp, 0.0)
    return dict(temperature=t.float(), top_k=k.int(), top_p=p.float(), min_p=mp.float())


def _pack_settings(s):
    """The settings as the library's rows of 16 bytes."""
    return torch.stack([s["temperature"].view(torch.int32), s["top_k"], s["top_p"].view(torch.int32), s["min_p"].view(torch.int32)], 1).contiguous()


def _logits(gen, rows, vocab, dtype):
    """About as peaked as a trained model's: a broad bulk, some tens of likely tokens, and some banned ones."""
    x = torch.randn((rows, vocab), generator=gen, device="cuda") * 1.8
    likely = _spread_ids(gen, rows, 40, vocab)
    x.scatter_(1, likely, 3.0 + 7.0 * torch.rand((rows, 40), generator=gen, device="cuda"))
    banned = _spread_ids(gen, rows, 8, vocab)
    x.scatter_(1, banned, float("-inf"))
    return x.to(_TYPES[dtype])


def _uniforms(gen, n):
    return torch.randint(1 << 24, (n,), generator=gen, device="cuda").float() * 2.0 ** -24


def _row0(counts):
    return torch.cat([counts.new_zeros(1), counts.cumsum(0, dtype=torch.int32)])


def _unit_bytes(hd):
    return 20 * hd


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    if op == "sample":
        rows, vocab = case["rows"], case["vocab"]
        s = _settings(gen, rows, case["filters"])
        return dict(op=op, settings=s, packed=_pack_settings(s), logits=_logits(gen, rows, vocab, case["dtype"]),
                    u=_uniforms(gen, rows), probs=torch.empty((rows, vocab), device="cuda") if case["probs"] else None)
    if op == "accept":
        n, vocab = case["n_req"], case["vocab"]
        ks = _whole(_between(n, case["k_lo"], case["k_hi"]))
        row0 = _row0(ks + 1)
        rows = int(row0[-1])
        s = _settings(gen, n, case["filters"])
        logits = _logits(gen, rows, vocab, case["dtype"])
        of = torch.repeat_interleave(torch.arange(n, device="cuda"), (ks + 1).long())       # request of a row
        scored = torch.ones(rows, dtype=torch.bool, device="cuda")
        scored[(row0[1:] - 1).long()] = False                                               # the last row scores no draft
        # the edge's distributions: the same logits with some noise, cut to their likely part
        edge = logits[scored].float() + 0.5 * torch.randn((rows - n, vocab), generator=gen, device="cuda")
        edge = edge.masked_fill_(edge < edge.amax(1, keepdim=True) - 6.0, float("-inf"))
        q = torch.softmax(edge, 1)
        drafts = torch.multinomial(q, 1, generator=gen)[:, 0].int()
        return dict(op=op, n_req=n, rows=rows, of=of, row0=row0, settings=s, packed=_pack_settings(s), logits=logits, q=q,
                    drafts=drafts, u=_uniforms(gen, rows))
    n, hd, kvh, page = case["n_req"], case["head_dim"], case["kv_heads"], case["page"]
    new = _whole(_between(n, case["n_lo"], case["n_hi"]))
    base = _whole(_between(n, case["p_lo"], case["p_hi"]))
    row0 = _row0(new)
    rows, longest = int(row0[-1]), int((base + new).max())
    max_pages = -(-longest // page)
    used = (base + new + page - 1) // page
    n_pages = int(used.sum()) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").int()                      # pages in no order
    col = torch.arange(max_pages, device="cuda")[None]
    table = order[(_row0(used)[:-1].long()[:, None] + col).clamp_(max=n_pages - 1)]
    table = torch.where(col < used[:, None], table, torch.full_like(table, -1)).contiguous()
    groups, units = hd // GROUP, page // UNIT
    # a cache of values with a spread of about 1: codes of all 16 levels, scales and zeros that fit
    pool = torch.randint(0, 256, (n_pages, kvh, units, _unit_bytes(hd)), dtype=torch.uint8, generator=gen, device="cuda")
    shape = (n_pages, kvh, units, 2, UNIT * groups)
    scale = ((0.15 + 0.15 * torch.rand(shape, generator=gen, device="cuda"))).bfloat16()
    zero = (-scale.float() * (6.5 + 2.0 * torch.rand(shape, generator=gen, device="cuda"))).bfloat16()
    pool[..., 8 * hd:10 * hd] = torch.stack([scale[..., 0, :], zero[..., 0, :]], -1).flatten(-2).view(torch.uint8)
    pool[..., 18 * hd:19 * hd] = scale[..., 1, :].contiguous().view(torch.uint8)
    pool[..., 19 * hd:20 * hd] = zero[..., 1, :].contiguous().view(torch.uint8)
    state = dict(op=op, n_req=n, rows=rows, longest=longest, most=int(new.max()), heads=case["heads"], kv_heads=kvh, head_dim=hd, page=page, pool=pool,
                 row0=row0, base=base, table=table, cache=None)
    if op == "append":
        k, v = (torch.randn((rows, kvh, hd), generator=gen, device="cuda") * std for std in (1.5, 0.8))
        k[:, :, 5] += 6.0                                                                    # keys have columns that stand out
        state |= dict(k=k.to(_TYPES[case["dtype"]]), v=v.to(_TYPES[case["dtype"]]))
    else:
        q = torch.randn((rows, case["heads"], hd), generator=gen, device="cuda") * 1.2
        state |= dict(q=q.to(_TYPES[case["dtype"]]), scale=hd ** -0.5)
    return state


# --------------------------------------------------------------------------- plain forms
def _shaped(logits, s):
    """Weights in id order (0 where a token is cut), in 64 bits: a threshold or a draw falls next to a border otherwise."""
    x = logits.double()
    top, first = x.max(1, keepdim=True)
    first = (x == top).int().argmax(1, keepdim=True)
    t = s["temperature"].double()[:, None]
    w = torch.exp((x - top) / torch.where(t > 0, t, 1.0))
    ids = torch.arange(x.shape[1], device=x.device)[None]
    w = torch.where(t > 0, w, (ids == first).double())
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    k = s["top_k"][:, None]
    ws = ws * ((k <= 0) | (ids < k))
    run_ = ws.cumsum(1)
    p = s["top_p"].double()[:, None]
    ws = ws * ((p >= 1) | (run_ - ws < p * run_[:, -1:]))
    ws = ws * (ws >= s["min_p"].double()[:, None])
    return torch.zeros_like(w).scatter_(1, order, ws)


def _drawn(w, u):
    """First id whose running weight exceeds u times the whole."""
    run_ = w.cumsum(1)
    return (run_ > u.double()[:, None] * run_[:, -1:]).int().argmax(1).int()


def _plain_sample(st):
    w = _shaped(st["logits"], st["settings"])
    token = _drawn(w, st["u"])
    return [token] if st["probs"] is None else [token, (w / w.sum(1, keepdim=True)).float()]


def _plain_accept(st):
    of, row0, n, rows = st["of"], st["row0"].long(), st["n_req"], st["rows"]
    w = _shaped(st["logits"], {key: v[of] for key, v in st["settings"].items()})
    p = w / w.sum(1, keepdim=True)
    at = torch.arange(rows, device="cuda")
    place = at - row0[of]                                             # 0..k inside its request
    last = at == row0[of + 1] - 1
    slot = (at - of).clamp_(max=rows - n - 1)                         # its row of q and its draft
    x = st["drafts"].long()[slot]
    px, qx = p[at, x], st["q"][slot, x].double()
    ratio = torch.where(qx > 0, px / qx, torch.where(px > 0, float("inf"), 0.0))
    stops = last | ~(st["u"].double() < ratio.clamp(max=1.0))
    accepted = torch.full((n,), rows, device="cuda").scatter_reduce_(0, of, torch.where(stops, place, rows), "amin")
    row = row0[:-1] + accepted
    target = p[row]
    rest = (target - st["q"][slot[row]].double()).clamp_(min=0.0)
    use = ~last[row][:, None] & (rest.sum(1, keepdim=True) > 0)
    token = _drawn(torch.where(use, rest, target), st["u"][row0[1:] - 1])
    return [accepted.int(), token]


def _positions(st):
    """Request and position of every new row."""
    at = torch.arange(st["rows"], device="cuda")
    of = torch.searchsorted(st["row0"][1:].contiguous(), at.int(), right=True)
    return of, st["base"][of].long() + at - st["row0"][of]


def _plain_quantised(x):
    """What 4 bits, a scale and a zero per 32 columns hold of x.  In 64 bits: codes are decided next to borders."""
    x = torch.nan_to_num(x.double(), nan=0.0).clamp_(-LIMIT, LIMIT).unflatten(-1, (-1, GROUP))
    zero = x.amin(-1, keepdim=True).bfloat16().double()
    scale = ((x.amax(-1, keepdim=True) - zero) / 15).bfloat16().double()
    code = torch.round((x - zero) / torch.where(scale > 0, scale, 1.0)).clamp_(0, 15) * (scale > 0)
    return (code * scale + zero).flatten(-2).float()


def _plain_cache(st):
    """K and V of every request, [request, position, KV head, column], out of its pages."""
    hd, groups = st["head_dim"], st["head_dim"] // GROUP
    block = st["pool"][st["table"].clamp(min=0).long()]               # request, page, head, unit, bytes

    def nibbles(b):
        return torch.stack([b & 15, b >> 4], -1).flatten(-2).float()

    # K: a position's 32-bit words are ordered [8 columns of a group][group]
    k = nibbles(block[..., :8 * hd].contiguous()).unflatten(-1, (UNIT, 4, groups, 8)).transpose(-2, -3).flatten(-3)
    sz = block[..., 8 * hd:10 * hd].contiguous().view(torch.bfloat16).float().unflatten(-1, (UNIT, groups, 2)).repeat_interleave(GROUP, -2)
    k = k * sz[..., 0] + sz[..., 1]
    # V: words [four column tiles][column % 8][position pair][tile], nibbles [position % 2][position / 8][column / 8 % 2]
    v = nibbles(block[..., 10 * hd:18 * hd].contiguous()).unflatten(-1, (hd // 64, 8, 4, 4, 2, 2, 2))
    lead = v.dim() - 7
    v = v.permute(*range(lead), lead + 5, lead + 2, lead + 4, lead, lead + 3, lead + 6, lead + 1).flatten(lead + 3).flatten(lead, lead + 2)
    s, z = (block[..., o * hd:(o + 1) * hd].contiguous().view(torch.bfloat16).float().unflatten(-1, (groups, UNIT)).transpose(-1, -2)
            .repeat_interleave(GROUP, -1) for o in (18, 19))
    v = v * s + z
    return [t.permute(0, 1, 3, 4, 2, 5).flatten(1, 3) for t in (k, v)]


def _plain_attend(st):
    k, v = (t[:, :st["longest"]] for t in _plain_cache(st))
    of, pos = _positions(st)
    at = torch.arange(st["rows"], device="cuda")
    per = st["heads"] // st["kv_heads"]
    q = torch.zeros((st["n_req"], st["most"], st["heads"], st["head_dim"]), device="cuda")
    place = at - st["row0"][of]
    q[of, place] = st["q"].float()
    horizon = torch.zeros((st["n_req"], st["most"]), dtype=torch.int64, device="cuda")
    horizon[of, place] = pos
    scores = torch.einsum("nrhgc,nlhc->nhgrl", q.unflatten(2, (-1, per)), k) * st["scale"]
    hidden = torch.arange(k.shape[1], device="cuda")[None, None] > horizon[:, :, None]
    scores.masked_fill_(hidden[:, None, None], float("-inf"))
    e = torch.exp(scores - scores.amax(-1, keepdim=True))
    v = torch.where((torch.arange(k.shape[1], device="cuda")[None] <= horizon.amax(1, keepdim=True))[:, :, None, None], v, 0.0)
    out = torch.einsum("nhgrl,nlhc->nrhgc", e / e.sum(-1, keepdim=True), v).flatten(2, 3)
    return out[of, place].to(st["q"].dtype)


def run(state):
    op = state["op"]
    if own:
        from paper_2605_13319_b200 import binding
        if op == "sample":
            token = binding.sample(state["logits"], state["packed"], state["u"], probs=state["probs"])
            return [token] if state["probs"] is None else [token, state["probs"]]
        if op == "accept":
            return list(binding.accept(state["logits"], state["row0"], state["packed"], state["q"], state["drafts"], state["u"]))
        if state["cache"] is None:
            state["cache"] = binding.Kv4Cache(state["kv_heads"], state["head_dim"], pool=state["pool"], page_size=state["page"])
        cache, where = state["cache"], (state["row0"], state["base"], state["table"])
        if op == "append":
            cache.append(state["k"], state["v"], *where)
            return list(cache.read(state["rows"], *where))
        return [cache.attend(state["q"], *where, scale=state["scale"])]
    if op == "sample":
        return _plain_sample(state)
    if op == "accept":
        return _plain_accept(state)
    if op == "append":
        return [_plain_quantised(state["k"]), _plain_quantised(state["v"])]
    return [_plain_attend(state)]


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    op = case["op"]
    size = 4 if case["dtype"] == "fp32" else 2
    if op == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * size + (4 * n if case["probs"] else 0) + 24 * case["rows"], "flops": 2 * n}
    if op == "accept":
        rows = sum(_between(case["n_req"], case["k_lo"], case["k_hi"])) + case["n_req"]
        return {"bytes": rows * case["vocab"] * size + case["n_req"] * case["vocab"] * 4, "flops": 2 * rows * case["vocab"]}
    hd = case["head_dim"]
    new, base = _between(case["n_req"], case["n_lo"], case["n_hi"]), _between(case["n_req"], case["p_lo"], case["p_hi"])
    rows, keys = sum(new), sum(new) + sum(base)
    if op == "append":     # the rows in, the cache's bytes out and back, their values out
        return {"bytes": rows * case["kv_heads"] * hd * (2 * size + 2 * 1.25 + 8), "flops": 8 * rows * case["kv_heads"] * hd}
    pairs = sum(n * (b + (n + 1) / 2) for n, b in zip(new, base))
    return {"bytes": keys * case["kv_heads"] * 1.25 * hd + 2 * rows * case["heads"] * hd * size, "flops": 4 * case["heads"] * hd * pairs}


# --------------------------------------------------------------------------- the definitions in 64 bits, one row or request at a time
def _exact_weights(x, t, k, p, mp):
    x = x.double()
    by_id = torch.arange(x.numel(), device=x.device)
    order = by_id[torch.argsort(-x, stable=True)]
    keep = x.numel() if k <= 0 else min(k, x.numel())
    w = torch.zeros_like(x)
    if t == 0:
        w[order[0]] = 1.0
        return w
    e = torch.exp(x / t - x[order[0]] / t)[order[:keep]]
    if p < 1:
        before = torch.nn.functional.pad(e.cumsum(0), (1, 0))
        e = e[:int((before[:-1] < p * before[-1]).sum())]
    e = e[e >= mp]
    w[order[:e.numel()]] = e
    return w


def _exact_settings(st):
    s = st["settings"]
    return list(zip(s["temperature"].tolist(), s["top_k"].tolist(), s["top_p"].tolist(), s["min_p"].tolist()))


def _exact_draw(w, u):
    run_ = w.cumsum(0)
    return int(torch.searchsorted(run_, run_[-1] * u, right=True))


def _exact_rows(st, which, hd):
    """Dequantised (position, head, column) values of one request, by the layout's formulas."""
    table = [p for p in st["table"][which].tolist() if p >= 0]
    b = st["pool"][table].transpose(1, 2).flatten(0, 1).long()                   # unit, head, bytes
    c, g = torch.arange(hd, device="cuda"), hd // GROUP
    slot = torch.arange(UNIT, device="cuda")[:, None]
    word = c % GROUP // 8 * g + c // GROUP
    at = slot * (hd // 2) + word * 4 + c % 8 // 2
    codes_k = b[:, :, at] >> (4 * (c % 2)) & 15
    tile, low = c // 16, c % 8
    nib = c // 8 % 2 + 2 * (slot // 8) + 4 * (slot % 2)
    lane = low * 4 + slot % 8 // 2
    at = 10 * hd + ((tile // 4 * 32 + lane) * 4 + tile % 4) * 4 + nib // 2
    codes_v = b[:, :, at] >> (4 * (nib % 2)) & 15

    def bf16(o):
        return ((b[:, :, o + 1] << 8 | b[:, :, o]) << 16).int().view(torch.float32).double()

    sk = 8 * hd + (slot * g + c // GROUP) * 4
    sv = 18 * hd + (c // GROUP * UNIT + slot) * 2
    k = codes_k * bf16(sk) + bf16(sk + 2)
    v = codes_v * bf16(sv) + bf16(sv + hd)
    return k.transpose(1, 2).flatten(0, 1), v.transpose(1, 2).flatten(0, 1)


def exact(case, seed):
    st = prepare(case, seed)
    if st["op"] == "sample":
        ws = [_exact_weights(x, *s) for x, s in zip(st["logits"], _exact_settings(st))]
        token = torch.tensor([_exact_draw(w, u) for w, u in zip(ws, st["u"].double().tolist())], dtype=torch.int32)
        return [token] if st["probs"] is None else [token, torch.stack([w / w.sum() for w in ws])]
    if st["op"] == "accept":
        u, first, drafts = st["u"].double().tolist(), st["row0"].tolist(), st["drafts"].tolist()
        accepted, tokens = [], []
        for r, s in enumerate(_exact_settings(st)):
            k, a = first[r + 1] - first[r] - 1, 0
            while True:
                p = _exact_weights(st["logits"][first[r] + a], *s)
                p = p / p.sum()
                if a == k:
                    break
                q = st["q"][first[r] - r + a].double()
                x = drafts[first[r] - r + a]
                if not u[first[r] + a] * float(q[x]) < float(p[x]):
                    rest = (p - q).clamp(min=0)
                    p = rest if float(rest.sum()) > 0 else p
                    break
                a += 1
            accepted.append(a)
            tokens.append(_exact_draw(p, u[first[r] + k]))
        return [torch.tensor(v, dtype=torch.int32) for v in (accepted, tokens)]
    hd = st["head_dim"]
    if st["op"] == "append":
        out = []
        for x in (st["k"], st["v"]):
            x = x.double().clamp(-LIMIT, LIMIT).reshape(-1, GROUP)
            lo = x.min(1).values.to(torch.bfloat16).double()
            step = ((x.max(1).values - lo) / 15.0).to(torch.bfloat16).double()
            held = torch.round((x - lo[:, None]) / step[:, None]).clamp(0, 15) * step[:, None] + lo[:, None]
            out.append(held.reshape(st["rows"], st["kv_heads"], hd))
        return out
    q, first, base = st["q"].double(), st["row0"].tolist(), st["base"].tolist()
    out, per = torch.empty_like(q), st["heads"] // st["kv_heads"]
    for r in range(st["n_req"]):
        k, v = _exact_rows(st, r, hd)
        for i in range(first[r], first[r + 1]):
            n = base[r] + i - first[r] + 1
            for h in range(st["kv_heads"]):
                a = torch.softmax(q[i, h * per:(h + 1) * per] @ k[:n, h].T * st["scale"], 1)
                out[i, h * per:(h + 1) * per] = a @ v[:n, h]
    return [out]
