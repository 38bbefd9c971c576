"""Keys at both ends of E8M0: what attention gives does not depend on where the powers of two stand, in the keys or in the queries."""
import pytest
import torch

from kv_helpers import Cache, check_attention, parts, queries
from operator_helpers import DEV
from test_gpu_kv_weights import check_weights

pytestmark = pytest.mark.gpu

E8M0 = ("mxfp4", "mxint4")
NEW = [None, [5, 1, 3], [60, 290, 64]]
IDS = ["one", "few", "many"]


def move_scales(c, part, by, sequences=None):
    """Scale bytes of the keys (part 1) or of the values (part 3) up by `by`."""
    for b in range(len(c.lens)) if sequences is None else sequences:
        page, slot = c.at(b, torch.arange(c.lens[b], device=DEV))
        p = parts(c.pages, c.fmt, c.D)[part]
        moved = p[page, :, slot].int() + by
        assert moved.min() >= 1 and moved.max() <= 253   # those that the quantizer gives to finite numbers that are not nearly zero
        p[page, :, slot] = moved.to(torch.uint8)


def short_queries(c, **kw):
    """Of so few bits that any power of two times them is a bfloat16."""
    return (queries(c, **kw).double() * 16).round() / 16


@pytest.mark.parametrize("by", [-121, -60, 60, 100, 118, 126])
@pytest.mark.parametrize("new", NEW, ids=IDS)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("fmt", E8M0)
def test_keys_far_from_one(fmt, dim, new, by):
    c = Cache(fmt, [129, 500, 64], 4, 3, dim, 32, new=new)
    move_scales(c, 1, by)
    c.K = [k * 2.0 ** by for k in c.K]
    Q = (short_queries(c) * 2.0 ** -by).to(torch.bfloat16)
    out, lse = c.call("attention", Q, return_lse=True)
    check_attention(c, Q, out, lse)
    check_weights(c, Q)


@pytest.mark.parametrize("new", NEW, ids=IDS)
@pytest.mark.parametrize("fmt", E8M0)
def test_sequences_whose_keys_are_far_apart(fmt, new):
    c = Cache(fmt, [129, 500, 64], 4, 3, 128, 32, new=new)
    Q = short_queries(c)
    for b, by in enumerate((110, -110, 0)):
        move_scales(c, 1, by, [b])
        c.K[b] = c.K[b] * 2.0 ** by
        start, _ = c.rows(b)
        Q[start:start + c.new[b]] *= 2.0 ** -by
    Q = Q.to(torch.bfloat16)
    out, lse = c.call("attention", Q, return_lse=True)
    check_attention(c, Q, out, lse)
    check_weights(c, Q)


def few_and_far(c, Q):
    """Blocks of tokens whose keys are far larger than others of the same 32 tokens, 2^120, but meet zeros of the queries."""
    for b, n in enumerate(c.lens):
        page, slot = c.at(b, torch.arange(1, n, 4, device=DEV))
        p = parts(c.pages, c.fmt, c.D)[1]
        p[page, :, slot, 0] = 240
        codes = parts(c.pages, c.fmt, c.D)[0]
        codes[page, :, slot, :16] = 0x11
        c.K[b][1::4, :, :32] = (0.5 if c.fmt == "mxfp4" else 1.0) * 2.0 ** 113
    Q[..., :32] = 0
    return Q


@pytest.mark.parametrize("new", NEW[:2], ids=IDS[:2])
@pytest.mark.parametrize("fmt", E8M0)
def test_large_keys_that_meet_zeros(fmt, new):
    """Few rows: a key's scale of 2^-126 of the largest of the 32 tokens still counts."""
    c = Cache(fmt, [129, 500, 64], 4, 2, 128, 32, new=new)
    Q = few_and_far(c, queries(c))
    out, lse = c.call("attention", Q, return_lse=True)
    check_attention(c, Q, out, lse)
    check_weights(c, Q)
