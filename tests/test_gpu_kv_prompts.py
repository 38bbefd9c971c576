"""Attention of many new tokens, and of the batches at the border to few, over the 4-bit cache against the definition in 64 bits."""
import pytest
import torch

from helpers import captured_launches
from kv_helpers import FMTS, Cache, check_attention, parts, queries
from operator_helpers import DEV, gen
from test_gpu_kv_attention import OPTIONS, options_of, run

pytestmark = pytest.mark.gpu


def kernel(c, Q, **options):
    """Name of the first kernel that the call launches."""
    c.call("attention", Q, *c.scales, **options)
    return captured_launches(lambda: c.call("attention", Q, *c.scales, **options))[0][0]


@pytest.mark.parametrize("page", [16, 64, 1024])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("fmt", FMTS)
def test_prompts(fmt, dim, page):
    c = Cache(fmt, [200, 401, 1300], 8, 4, dim, page, new=[150, 401, 300])
    Q = queries(c)
    assert "prefill" in kernel(c, Q)
    run(c, Q)


@pytest.mark.parametrize("o", OPTIONS, ids=lambda o: "-".join(o))
@pytest.mark.parametrize("dim", [128, 256])
@pytest.mark.parametrize("fmt", FMTS)
def test_scoring(fmt, dim, o):
    c = Cache(fmt, [129, 500, 64], 16, 3, dim, 32, new=[60, 290, 64])
    Q = queries(c)
    assert "prefill" in kernel(c, Q)
    run(c, Q, **options_of(c, o))


@pytest.mark.parametrize("fmt", FMTS)
def test_uneven_batch(fmt):
    # empty, without new rows, one row, shorter than its rows, a whole tile, one more, one less
    c = Cache(fmt, [0, 300, 700, 90, 64, 65, 63, 128, 129, 1, 600], 32, 1, 64, 16, new=[3, 0, 1, 100, 64, 65, 63, 128, 129, 1, 600])
    Q = queries(c)
    assert "prefill" in kernel(c, Q)
    run(c, Q, window=100)
    run(c, Q)


@pytest.mark.parametrize("new", [7, 8, 9, 16, 17, 37, 38, 39, 40, 75, 148])
@pytest.mark.parametrize("dim", [64, 256])
def test_either_side_of_the_borders(dim, new):
    """The other kernel is taken from 64 rows of a head on."""
    c = Cache("mxfp4", [333], 64, 4, dim, 16, new=[new])
    Q = queries(c)
    assert ("prefill" in kernel(c, Q)) == (new * 4 >= 64)
    run(c, Q)


@pytest.mark.parametrize("new", [None, [5, 2, 9], [300, 310, 305]], ids=["one", "few", "many"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("fmt", FMTS)
def test_scales_of_every_size(fmt, dim, new):
    """Scales far apart, blocks of zeros, queries of zero and large ones; the largest values in the first tokens and in the last ones."""
    lens = [700, 333, 1000]
    c = Cache(fmt, lens, 8, 4, dim, 32, new=new, spread=10 if fmt == "nvfp4" else 14, low=118, seed=3)
    for b, n in enumerate(lens):
        g = gen(b)
        for part in (1, 3):
            sf = torch.randint(8, 110, (n, c.H, dim // 16), generator=g, device=DEV) if fmt == "nvfp4" else \
                torch.randint(118, 132, (n, c.H, dim // 32), generator=g, device=DEV)
            ramp = torch.arange(n, device=DEV).view(n, 1, 1) * 8 // n
            sf = sf + (ramp if b == 0 else -ramp if b == 1 else 0)
            if fmt == "nvfp4":
                sf = torch.where(torch.rand(sf.shape, generator=g, device=DEV) < 0.2, 0, sf)
            sf = sf.to(torch.uint8)
            codes = torch.randint(0, 256, (n, c.H, dim // 2), generator=g, device=DEV, dtype=torch.uint8) & 0x77
            codes = torch.where(torch.rand((n, c.H, 1), generator=g, device=DEV) < 0.1, 0, codes)
            c.put(b, part - 1, codes)
            c.put(b, part, sf)
            (c.K if part == 1 else c.V)[b] = c.values(codes, sf, part // 2)
    Q = queries(c, size=0.02)
    Q[::3, ::2] = 0
    Q[1::3, 1::2] *= 30
    run(c, Q)


@pytest.mark.parametrize("new", [[2, 0, 1], [250, 200, 0]], ids=["few", "many"])
def test_rows_that_no_sequence_has(new):
    """Rows before the first sequence and behind the last: zeros and -inf; the others as without them."""
    c = Cache("nvfp4", [300, 200, 40], 32, 2, 128, 16, new=new)
    Q = queries(c)
    out, lse = run(c, Q)
    before, behind = 3, 5
    padded = torch.full((before + c.tokens + behind, *Q.shape[1:]), float("nan"), dtype=torch.bfloat16, device=DEV)
    padded[before:before + c.tokens] = Q
    c.starts += before
    y, z = c.call("attention", padded, *c.scales, return_lse=True)
    none = torch.ones(len(padded), dtype=torch.bool, device=DEV)
    none[before:before + c.tokens] = False
    assert (y[none] == 0).all() and torch.isneginf(z[none]).all()
    c.starts -= before
    check_attention(c, Q, y[before:before + c.tokens], z[before:before + c.tokens])


@pytest.mark.parametrize("batch", [33, 200, 1000])
def test_many_sequences(batch):
    g = torch.Generator().manual_seed(batch)
    lens = [int(x) for x in torch.randint(0, 90, (batch,), generator=g)]
    c = Cache("mxfp4", lens, 1, 3, 64, 16)
    run(c, queries(c))
    c = Cache("nvfp4", lens, 1, 3, 64, 16, new=[min(n, i % 3) for i, n in enumerate(lens)])
    run(c, queries(c))


@pytest.mark.parametrize("new", [None, [250, 200]], ids=["one", "many"])
@pytest.mark.parametrize("fmt", FMTS)
def test_what_lies_behind_a_sequence_is_not_read_into_it(fmt, new):
    """Slots behind the length within the last page, and whole pages that no sequence has: any bytes give the same bits."""
    c = Cache(fmt, [301, 205], 32, 2, 128, 64, new=new)
    Q = queries(c)
    out, lse = run(c, Q)
    free = torch.tensor(c.free, device=DEV)
    for byte in (0, 0x7F, 0x7E, 0x80):
        c.pages[free] = byte
        for b in range(2):
            n = c.lens[b]
            page, slot = c.at(b, torch.arange(n, -(-n // c.P) * c.P, device=DEV))
            for part in parts(c.pages, fmt, c.D):
                part[page, :, slot] = byte
        y, z = c.call("attention", Q, *c.scales, return_lse=True)
        assert torch.equal(y, out) and torch.equal(z, lse)


@pytest.mark.parametrize("new", [[1, 1], [3, 2], [250, 200]], ids=["one", "few", "many"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("fmt", FMTS)
def test_what_no_row_sees_may_hold_anything(fmt, dim, new):
    """Tokens in front of every row's document, of all scales up to no number: the same bits as with ordinary ones."""
    c = Cache(fmt, [777, 540], 32, 2, dim, 32, new=new)
    begins = [77, 301]
    first = torch.cat([torch.full((n,), begins[b], dtype=torch.int32, device=DEV) for b, n in enumerate(new)])
    Q = queries(c)
    options = dict(first=first)
    out, lse = run(c, Q, **options)
    w = torch.rand(c.pages.shape[0], c.H, c.P, generator=gen(4), device=DEV)
    account = c.call("weights", Q, lse, w.clone(), *c.scales[:1], **options)
    for byte in (0x7E, 0x7F, 0xFD, 0xFE, 0xFF):
        for b in range(2):
            page, slot = c.at(b, torch.arange(begins[b], device=DEV))
            for part in parts(c.pages, fmt, c.D):
                part[page, :, slot] = byte
        y, z = c.call("attention", Q, *c.scales, return_lse=True, **options)
        assert torch.equal(y, out) and torch.equal(z, lse)
        assert torch.equal(c.call("weights", Q, lse, w.clone(), *c.scales[:1], **options), account)


@pytest.mark.parametrize("o", [dict(), dict(window=700), dict(first=True), dict(prefix=True, slopes=True)], ids=lambda o: "-".join(o) or "plain")
@pytest.mark.parametrize("fmt,dim", [("mxfp4", 128), ("nvfp4", 64), ("mxint4", 256)])
@pytest.mark.parametrize("lens,new,heads", [([20000], [300], 1), ([3000, 17, 9000], [300, 3, 150], 2), ([6000], [6000], 1), ([5000, 5001], [65, 700], 3)])
def test_items_that_ranges_cut(lens, new, heads, fmt, dim, o):
    """Few items with many tokens: CTAs share them, their parts are joined."""
    c = Cache(fmt, lens, heads, 2, dim, 64, new=new)
    run(c, queries(c), **options_of(c, o))
