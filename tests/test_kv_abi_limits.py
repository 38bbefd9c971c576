"""Sizes of the 4-bit key/value cache just behind what the header allows, where a product of them would pass 64 or 31 bits: refused, without a device."""
import pytest

from test_kv_abi import CALLS, FMTS, SHAPE, append, cache, evict, read


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("fmt", FMTS)
def test_tables_whose_tokens_pass_64_bits(fmt, call):
    for page, width in ((16, 1 << 60), (1024, 1 << 54), (1024, (1 << 54) + 1), (16, (1 << 63) - 1), (16, (1 << 26) + 1), (1024, (1 << 20) + 1)):
        assert call(fmt, cache(page_tokens=page, table_width=width)) == SHAPE, (page, width)


@pytest.mark.parametrize("fmt", FMTS)
def test_elements_of_new_tokens(fmt):
    """tokens kv_heads head_dim / 4 is a 31-bit number."""
    c = cache(kv_heads=16, head_dim=256)
    assert append(fmt, c, ks=4096, vs=4096, tokens=1 << 21) == SHAPE and read(fmt, c, tokens=1 << 21) == SHAPE
    assert evict(fmt, cache(batch=65536, kv_heads=1), keep=32) == SHAPE
