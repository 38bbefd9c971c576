"""A bias by distance so steep that a row is left with the token at its own place: float32's largest slopes among them."""
import pytest
import torch

from kv_helpers import FMTS, Cache, check_attention, queries, score_size
from operator_helpers import DEV, gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("slope", [1e4, 1e30, 2e38, 3.4e38])
@pytest.mark.parametrize("new", [None, [5, 1, 3], [60, 290, 64]], ids=["one", "few", "many"])
@pytest.mark.parametrize("fmt", FMTS)
def test_only_its_own_place(fmt, new, slope):
    c = Cache(fmt, [129, 500, 64], 4, 3, 128, 32, new=new)
    Q = queries(c)
    slopes = torch.full((c.H * c.G,), slope, device=DEV)
    out, lse = c.call("attention", Q, *c.scales, slopes=slopes, return_lse=True)
    # the others weigh nothing, as without a bias but for a window of one token
    check_attention(c, Q, out, lse, window=1)
    first = torch.cat([c.rows(b)[1] for b in range(3)]).to(torch.int32)
    w = torch.rand(c.pages.shape[0], c.H, c.P, generator=gen(6), device=DEV)
    steep = c.call("weights", Q, lse, w.clone(), *c.scales[:1], slopes=slopes)
    alone = c.call("weights", Q, lse, w.clone(), *c.scales[:1], first=first, window=1)
    owned = torch.zeros(w.shape, dtype=torch.bool, device=DEV)
    for b in range(3):
        page, slot = c.at(b, torch.arange(c.lens[b], device=DEV))
        owned[page, :, slot] = True
    # each is off by what check_weights allows: an exponent by dx, the sum of n by n 2^-24.  (Not equal: a score with a bias is rounded once more.)
    dx = 2.0 ** -19 * score_size(c, Q) + 2.0 ** -22 * lse.abs().max().item() + 2.0 ** -20
    off = 2 * (dx + (max(c.new) * c.G + 8) * 2.0 ** -24)
    a, b = steep[owned].double(), alone[owned].double()
    assert ((a - b).abs() <= off * b.abs()).all()
