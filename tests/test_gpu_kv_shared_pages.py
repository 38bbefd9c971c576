"""Sequences with pages in common: a prompt that they share is read by all of them; the account of a batch that shares is made sequence after sequence."""
import pytest
import torch

from kv_helpers import FMTS, Cache, attention, check_attention, queries, score_size, scores
from operator_helpers import DEV, gen

pytestmark = pytest.mark.gpu

SHARED = 5                                               # pages


def sharing(fmt, new):
    c = Cache(fmt, [700, 333, 400], 8, 4, 128, 32, new=new)
    for b in (1, 2):
        c.table_rows[b][:SHARED] = c.table_rows[0][:SHARED]
        c.K[b][:SHARED * c.P], c.V[b][:SHARED * c.P] = c.K[0][:SHARED * c.P], c.V[0][:SHARED * c.P]
    c.table[:, :SHARED] = c.table[:1, :SHARED]
    return c


NEW = [None, [3, 1, 2], [150, 100, 120]]


@pytest.mark.parametrize("new", NEW, ids=["one", "few", "many"])
@pytest.mark.parametrize("fmt", FMTS)
def test_attention_and_read(fmt, new):
    c = sharing(fmt, new)
    Q = queries(c)
    out, lse = c.call("attention", Q, *c.scales, return_lse=True)
    check_attention(c, Q, out, lse)
    starts, c.starts = c.starts, torch.tensor([0, 700, 1033, 1433], dtype=torch.int32, device=DEV)
    K, V = c.call("read", c.D, sum(c.lens), *c.scales, out_dtype=torch.float32)
    for got, want in ((K, c.K), (V, c.V)):
        want = torch.cat(want)
        assert ((got.double() - want).abs() <= 2.0 ** -23 * want.abs()).all()          # two products, NVFP4's are rounded
    c.starts = starts


@pytest.mark.parametrize("new", NEW, ids=["one", "few", "many"])
@pytest.mark.parametrize("fmt", FMTS)
def test_the_account_sequence_after_sequence(fmt, new):
    """One call for each sequence, in place: the slots that they share have the sum of all."""
    from paper_2605_19561_b200 import torq
    c = sharing(fmt, new)
    Q = queries(c)
    lse = attention(c, Q)[1].float()
    w = torch.rand(c.pages.shape[0], c.H, c.P, generator=gen(3), device=DEV)
    want = w.double()
    f = getattr(torq, f"torq_{fmt}_kv_weights")
    tol = torch.zeros_like(want)
    off = 2.0 ** -19 * score_size(c, Q) + 2.0 ** -22 * lse.abs().max().item() + 2.0 ** -20 + (max(c.new) * c.G + 8) * 2.0 ** -24
    for b, n in enumerate(c.new):
        start, _ = c.rows(b)
        slots = torch.arange(c.lens[b], device=DEV)
        page, slot = c.at(b, slots)
        x = torch.exp(scores(c, Q, b) - lse[start:start + n].double().view(n, c.H, c.G).permute(1, 2, 0).unsqueeze(-1)).sum((1, 2)).t()
        want[page, :, slot] = torch.where((slots < c.lens[b] - n).unsqueeze(1), want[page, :, slot], 0.0) + x
        tol[page, :, slot] += off * x + 2.0 ** -23 * want[page, :, slot]
        rows = slice(start, start + n)
        one = None if new is None else torch.tensor([0, n], dtype=torch.int32, device=DEV)
        f(c.pages, c.table[b:b + 1], c.lengths[b:b + 1], Q[rows], lse[rows].contiguous(), w, *c.scales[:1], starts=one)
    assert ((w.double() - want).abs() <= tol).all()
