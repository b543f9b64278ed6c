"""Bounds on the bf16 attention that a lost page, or a rounding that should not be there, does not pass; and that they reject these.

Elementwise bounds add up magnitudes, so that over a long context they are as large as what they bound.  Norms are not: with values of both signs
the roundings of many weights add up as their squares.  A weight's rounding to bf16 is uniform within half a step, 2^-8 of the value at most and 2^-8 /
sqrt(6) in the mean square (a mantissa between 1 and 2), relative to the result's norm, which is the same sum of squares; the output's rounding is as much
again, together 0.58 * 2^-8: 2^-8 for bf16.  fp32: scores of up to 8 lose 24 truncations of 2^-23 of their sums of magnitudes, of up to 16, at
random: 2^-18 in all.  A page of 16 out of n positions is sqrt(16 / n) of the norm: 2^-8 up to a million positions.

Values that are one column's alone count what was seen exactly: where every marked key has the same score and all others none, column c of the result is
the share of marked keys whose value is column c, without any rounding of weights (they are 1), sums of whole numbers, one division and the output's
rounding."""
import numpy as np
import pytest


def norm_bound(dtype):
    import torch
    return 2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -18


def norm_error(got, want):
    """Of whole numbers of rows: |got - want| / |want|."""
    return ((got.double() - want.double()).norm() / want.double().norm()).item()


def marked(n, marks, hd, kvh, device):
    """(k, v) [n, kvh, hd] in bf16 with marks (positions) whose score for queries that are 32 in column 0 is 0, and far less elsewhere; value i of the marks is
    column (i + head) % hd alone."""
    import torch
    g = torch.Generator(device).manual_seed(n)
    k, v = (torch.randn((n, kvh, hd), generator=g, device=device) for _ in range(2))
    at = torch.as_tensor(marks, device=device)
    k[..., 0] = -64.0
    k[at] = 0.0
    v[at] = 0.0
    i = torch.arange(len(at), device=device)
    for h in range(kvh):
        v[at, h, (i + h) % hd] = 1.0
    return k.bfloat16(), v.bfloat16()


def marked_queries(rows, heads, hd, dtype, device):
    import torch
    q = torch.zeros((rows, heads, hd), dtype=dtype, device=device)
    q[..., 0] = 32.0
    return q


def marked_result(counts, hd, heads, kvh):
    """What a row gives that has seen the first `counts` [rows] marks: [rows, heads, hd]."""
    import torch
    n = torch.as_tensor(counts, dtype=torch.int64)[:, None, None]
    column = (torch.arange(hd)[None] - (torch.arange(heads) // (heads // kvh))[:, None])[None] % hd      # the mark that is this column's first
    per = torch.where(n > column, (n - 1 - column) // hd + 1, 0)
    return per.double() / n


def marked_tolerance(dtype):
    """Of the value: the output's rounding, and a division and a product in fp32."""
    import torch
    return 2.0 ** -8 + 2.0 ** -21 if dtype is torch.bfloat16 else 2.0 ** -21


# --------------------------------------------------------------------------- what they reject
def _case(n, rows=4, heads=8, hd=128):
    import torch
    g = torch.Generator().manual_seed(n)
    q = torch.randn((rows, heads, hd), generator=g).double() * 1.5
    k, v = (torch.randn((n, 2, hd), generator=g).bfloat16().double() for _ in range(2))
    return q, k, v


def _attention(q, k, v, weights=lambda p: p, leave=None):
    import torch
    G = q.shape[1] // k.shape[1]
    s = torch.einsum("rhd,nhd->hrn", q, k.repeat_interleave(G, 1)) * q.shape[2] ** -0.5
    if leave is not None:
        s[..., leave] = -float("inf")
    e = torch.exp(s - s.amax(-1, keepdim=True))
    return torch.einsum("hrn,nhd->rhd", weights(e), v.repeat_interleave(G, 1)) / e.sum(-1).T[..., None]


@pytest.mark.parametrize("n", [5000, 20064, 40001])
def test_norms_reject_lost_pages_and_short_weights(n):
    import torch
    q, k, v = _case(n)
    want = _attention(q, k, v)
    short = _attention(q, k, v, lambda e: e.bfloat16().double())
    assert 0.3 * 2.0 ** -8 < norm_error(short.bfloat16(), want) < norm_bound(torch.bfloat16)       # what the kernels do
    assert norm_error(want.float(), want) < norm_bound(torch.float32)
    assert norm_error(short, want) > 100 * norm_bound(torch.float32)
    for lost in (slice(n // 2, n // 2 + 16), slice(n - 16, n), slice(0, 128)):
        less = _attention(q, k, v, lambda e: e.bfloat16().double(), lost).bfloat16()
        assert norm_error(less, want) > norm_bound(torch.bfloat16)


@pytest.mark.parametrize("n,every", [(20064, 16), (40001, 16), (40001, 1)])
def test_marks_reject_lost_and_doubled_keys(n, every):
    import torch
    hd, heads, kvh = 64, 4, 2
    marks = np.arange(every // 2, n, every)
    k, v = marked(n, marks, hd, kvh, "cpu")
    q = marked_queries(1, heads, hd, torch.float32, "cpu")
    want = marked_result([len(marks)], hd, heads, kvh)
    for dtype in (torch.bfloat16, torch.float32) if every > 1 else (torch.float32,):
        out = _attention(q.double(), k.double(), v.double()).to(dtype)
        assert ((out.double() - want).abs() <= marked_tolerance(dtype) * want).all()
        for lost in (marks[7], marks[len(marks) // 2], marks[-1]):
            less = _attention(q.double(), k.double(), v.double(), leave=slice(int(lost), int(lost) + 1)).to(dtype)
            assert ((less.double() - want).abs() > marked_tolerance(dtype) * want).any()
            twice = _attention(q.double(), torch.cat([k, k[lost:lost + 1]]).double(), torch.cat([v, v[lost:lost + 1]]).double()).to(dtype)
            assert ((twice.double() - want).abs() > marked_tolerance(dtype) * want).any()
