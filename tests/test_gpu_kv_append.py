"""New keys and values in the pages of the 4-bit cache: codes and scale bytes are those of the library's quantizers, everything else stays."""
import pytest
import torch

from kv_helpers import FMTS, Cache, parts
from operator_helpers import DEV, gen, heavy, untile
from paper_2605_19561_b200 import torq

pytestmark = pytest.mark.gpu


def quantized(x, fmt, ts):
    """x [tokens, heads, dim] through the library's quantizer: codes and scale bytes of each row."""
    n, h, d = x.shape
    z = torch.zeros(n * h, max(d, 128), dtype=x.dtype, device=DEV)
    z[:, :d] = x.reshape(n * h, d)
    if fmt == "nvfp4":
        codes, sf = torq.torq_quantize_nvfp4(z, ts)
    elif fmt == "mxint4":
        codes, sf = torq.torq_quantize_mxint4(z, packed=True)
    else:
        codes, sf = torq.torq_quantize_mxfp4(z)
    blocks = d // (16 if fmt == "nvfp4" else 32)
    return codes[:, :d // 2].view(n, h, -1), untile(sf, n * h, blocks).reshape(n, h, blocks)


def expected(c, K, V):
    pages = c.pages.clone()
    p = parts(pages, c.fmt, c.D)
    for b, n in enumerate(c.new):
        first, place = c.rows(b)
        at = place >= 0
        if not n or not at.any():
            continue
        page, slot = c.at(b, place[at])
        for i, x in enumerate((K, V)):
            codes, sf = quantized(x[first:first + n][at].contiguous(), c.fmt, c.scales[i] if c.scales else 1.0)
            p[2 * i][page, :, slot], p[2 * i + 1][page, :, slot] = codes, sf
    return pages


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("fmt", FMTS)
def test_append(fmt, dim, dtype):
    for lens, new, heads, page in (([1, 17, 64, 0, 5], None, 3, 16), ([40, 100, 7], [40, 33, 0], 2, 32), ([3, 9], [5, 9], 1, 1024), ([1], None, 1, 16)):
        c = Cache(fmt, lens, heads, 1, dim, page, new=new)
        g = gen(3)
        K, V = (heavy(g, c.tokens, heads, dim).to(dtype) for _ in range(2))
        K[0, 0, :32] = 0                                 # a block of zeros, and one that is very small
        V[-1, -1, :32] *= 1e-30
        want = expected(c, K, V)
        assert c.call("append", K, V, *c.scales) is None
        assert torch.equal(c.pages, want)
        k, v = c.call("read", dim, c.tokens, *c.scales, out_dtype=torch.float32)
        for b, n in enumerate(c.new):
            first, place = c.rows(b)
            there = place >= 0
            assert not k[first:first + n][~there].any() and not v[first:first + n][~there].any()
            if there.any():
                page, slot = c.at(b, place[there])
                p = parts(c.pages, fmt, dim)
                for i, x in enumerate((k, v)):
                    ref = c.values(p[2 * i][page, :, slot], p[2 * i + 1][page, :, slot], i)
                    assert ((x[first:first + n][there].double() - ref).abs() <= 2.0 ** -24 * ref.abs()).all()
        bk, bv = c.call("read", dim, c.tokens, *c.scales)
        assert torch.equal(bk, k.to(torch.bfloat16)) and torch.equal(bv, v.to(torch.bfloat16))


@pytest.mark.parametrize("fmt", FMTS)
def test_columns_of_a_fused_projection(fmt):
    c = Cache(fmt, [5, 33], 2, 4, 128, 16, new=[5, 20])
    rows = heavy(gen(4), 25, 12, 128).to(torch.bfloat16)
    K, V = rows[:, 8:10], rows[:, 10:]
    want = expected(c, K.contiguous(), V.contiguous())
    c.call("append", K, V, *c.scales)
    assert torch.equal(c.pages, want)


def test_a_bad_page_or_length_is_an_error_and_nothing_is_written():
    torq.torq_last_device_error()
    c = Cache("mxfp4", [20, 5], 1, 1, 64, 16)
    K = V = heavy(gen(5), 2, 1, 64).to(torch.bfloat16)
    for bad in (-1, c.pages.shape[0], 1 << 30):
        table = c.table.clone()
        table[0, 1] = bad
        before = c.pages.clone()
        before_1 = c.pages.clone()
        p, slot = c.at(1, torch.tensor([4], device=DEV))
        torq.torq_mxfp4_kv_append(c.pages, table, c.lengths, K, V)
        assert torq.torq_last_device_error() == 8 and torq.torq_last_device_error() == 0
        q = torq.torq_mxfp4_kv_read(c.pages, table, c.lengths, 64, 2)
        assert torq.torq_last_device_error() == 8 and not q[0][0].any()
        before[p], before_1[p] = 0, c.pages[p]
        assert torch.equal(torch.where(torch.arange(c.pages.shape[0], device=DEV).view(-1, 1, 1) == p, 0, c.pages), before)
    long = torch.tensor([100, 5], dtype=torch.int32, device=DEV)
    torq.torq_mxfp4_kv_append(c.pages, c.table, long, K, V)
    assert torq.torq_last_device_error() == 8


def test_starts_that_make_no_sense_do_no_harm():
    c = Cache("mxfp4", [20, 30], 1, 1, 64, 16, new=[3, 4])
    K = V = heavy(gen(6), 7, 1, 64).to(torch.bfloat16)
    for s in ([-5, 3, 7], [0, 9, 2], [5, 5, 100], [8, 9, 10], [3, 2, 1]):
        c.starts = torch.tensor(s, dtype=torch.int32, device=DEV)
        c.call("append", K, V)
        c.call("read", 64, 7)
        c.call("attention", heavy(gen(7), 7, 1, 64).to(torch.bfloat16))
    torch.cuda.synchronize()
    torq.torq_last_device_error()
