"""Eviction: weights of zero, of either sign."""
import pytest
import torch

from kv_helpers import Cache
from operator_helpers import DEV, gen
from test_gpu_kv_weights import check_evict, with_evict

pytestmark = pytest.mark.gpu


def test_zeros_of_either_sign_are_equal():
    lens = [500, 4099]
    c = with_evict(Cache("mxfp4", lens, 2, 1, 64, 16))
    g = gen(21)
    shape = (c.pages.shape[0], 2, 16)
    w = torch.where(torch.rand(shape, generator=g, device=DEV) < 0.5, -0.0, 0.0)
    w = torch.where(torch.rand(shape, generator=g, device=DEV) < 0.1, torch.randn(shape, generator=g, device=DEV), w)
    assert (torch.signbit(w) & (w == 0)).any()
    check_evict(c, w, 300, 10)
