"""Attention of many rows over values far apart from token to token: a weight counts by what its value makes of it."""
import math

import pytest
import torch

from kv_helpers import Cache, attention, parts, queries, score_size, scores
from operator_helpers import DEV

pytestmark = pytest.mark.gpu


def check_products(c, Q, out, lse, large, **options):
    """As check_attention, but for what a weight is off by as a float16.  It is held times the largest scale of its 128 tokens, E, with the largest such product at
    2^10 at least: off by 2^-25, 2^-35 of the largest product.  `large` [tokens] of each sequence: the largest scale of the 128 that a token is among (where
    these begin at a multiple of 128), or within 127 tokens of it.  A value is at most eight of those."""
    ref, ref_lse, mag = attention(c, Q, **options)
    dx = 2.0 ** -19 * score_size(c, Q) + 2.0 ** -20
    assert ((lse.double() - ref_lse).abs() <= dx + 2.0 ** -22 * ref_lse.abs() + 2.0 ** -20).all()
    assert torch.isfinite(out).all()
    tol = (2 * dx + 2.0 ** -11) * mag + 2.0 ** -8 * ref.abs()
    for b, n in enumerate(c.new):
        start, _ = c.rows(b)
        x = scores(c, Q, b, **options)
        w = torch.exp(x - torch.logsumexp(x, -1, keepdim=True))
        seen = (x > -math.inf).sum(-1)
        off = 2.0 ** -35 * 8 * seen * (w * large[b]).amax(-1)              # [heads, group, new]
        tol[start:start + n] += off.permute(2, 0, 1).reshape(n, -1, 1)
    worst = ((out.double() - ref).abs() / tol).max().item()
    assert worst <= 1.0, worst
    return tol, ref


def with_large_values(fmt, dim, gap, tokens, push, lens, new, aligned=True):
    """Values of `tokens` (of each sequence) 2^gap larger than the others; their scores are lower by what `push` makes of 32 features."""
    c = Cache(fmt, lens, 8, 4, dim, 32, new=new, spread=1, low=110)
    large = []
    for b, n in enumerate(lens):
        at = torch.arange(n, device=DEV)
        there = (at >= tokens[0]) & (at < tokens[1])
        page, slot = c.at(b, at)
        k_codes, k_scales, _, v_scales = parts(c.pages, fmt, dim)
        k_codes[page, :, slot, :16] = torch.where(there, 0x22, 0).to(torch.uint8).view(-1, 1, 1)
        k_scales[page, :, slot, 0] = 110
        c.K[b][..., :32] = torch.where(there, (1.0 if fmt == "mxfp4" else 2.0) * 2.0 ** -17, 0.0).view(-1, 1, 1)
        v_scales[page, :, slot] = torch.where(there, 110 + gap, 110).to(torch.uint8).view(-1, 1, 1)
        c.V[b] *= torch.where(there, 2.0 ** gap, 1.0).view(-1, 1, 1)
        s = torch.where(there, 2.0 ** gap, 1.0) * 2.0 ** -17
        if aligned:
            large.append(torch.nn.functional.max_pool1d(s.view(1, 1, -1), 128, ceil_mode=True).view(-1).repeat_interleave(128)[:n])
        else:
            large.append(torch.nn.functional.max_pool1d(s.view(1, 1, -1), 255, 1, 127).view(-1))
    Q = queries(c, size=0.5).double() * 2.0 ** 17
    Q[..., :32] = -push * 2.0 ** 17
    return c, Q.to(torch.bfloat16), large


@pytest.mark.parametrize("tokens", [(0, 128), (256, 384)], ids=["first", "middle"])
@pytest.mark.parametrize("push", [16.0, 2.0])
@pytest.mark.parametrize("gap", [20, 30, 34, 45, 60, 100])
@pytest.mark.parametrize("fmt,dim", [("mxfp4", 128), ("mxint4", 64), ("mxint4", 256)])
def test_large_values_of_tokens_with_small_weights(fmt, dim, gap, push, tokens):
    c, Q, large = with_large_values(fmt, dim, gap, tokens, push, [640, 500], [256, 100])
    assert c.tokens // len(c.lens) * c.G >= 64           # the kernel of many rows
    out, lse = c.call("attention", Q, return_lse=True)
    check_products(c, Q, out, lse, large)


@pytest.mark.parametrize("lens,new,heads", [([5000, 5001], [65, 700], 3)])
@pytest.mark.parametrize("fmt,dim", [("mxfp4", 128), ("mxint4", 256)])
def test_parts_with_values_far_apart(fmt, dim, lens, new, heads):
    """Items that CTAs share: a part with the large values, others without."""
    c, Q, large = with_large_values(fmt, dim, 50, (1024, 2048), 16.0, lens, new)
    out, lse = c.call("attention", Q, return_lse=True)
    check_products(c, Q, out, lse, large)


@pytest.mark.parametrize("fmt,dim", [("mxfp4", 128), ("mxint4", 64), ("mxint4", 256)])
def test_large_values_that_some_rows_do_not_see(fmt, dim):
    """A window, and documents: rows that see the large values share their tiles with rows that do not."""
    c, Q, large = with_large_values(fmt, dim, 60, (0, 128), 0.0, [640, 500], [500, 400], aligned=False)
    first = []
    for b in range(2):
        _, p = c.rows(b)
        first.append(torch.where((p % 2 == 0) & (p >= 310), 300, 0))
    for options in (dict(window=100), dict(first=torch.cat(first).to(torch.int32))):
        seen = []
        for b, n in enumerate(c.new):
            start, p = c.rows(b)
            lo = p - 99 if "window" in options else options["first"][start:start + n]
            seen.append(lo >= 256)                       # no large value within 128 tokens of what it sees
        out, lse = c.call("attention", Q, return_lse=True, **options)
        tol, ref = check_products(c, Q, out, lse, large, **options)
        apart = torch.cat(seen)
        assert apart.any() and not apart.all()
        small = 8 * 2.0 ** -17
        assert (tol[apart] <= 0.02 * small).all() and (ref[apart].abs() <= small).all()    # the bound says something of them
