"""The account of attention weight and the eviction by it."""
import math

import pytest
import torch

from kv_helpers import FMTS, Cache, attention, parts, queries, score_size, scores
from operator_helpers import DEV, gen
from paper_2605_19561_b200 import torq
from test_gpu_kv_attention import OPTIONS, options_of

pytestmark = pytest.mark.gpu


def check_weights(c, Q, **options):
    """A weight is off by its score's error and that of lse, which is rounded to float32 here, its exp by 2^-21, the sum of n by n 2^-24."""
    lse = attention(c, Q, **options)[1].float()
    old = torch.rand(c.pages.shape[0], c.H, c.P, generator=gen(9), device=DEV)
    out = torch.full_like(old, -7.0)
    want = out.double()
    assert c.call("weights", Q, lse, old, *c.scales[:1], weights_out=out, **options) is out
    for b, n in enumerate(c.new):
        if not c.lens[b]:
            continue
        start, _ = c.rows(b)
        slots = torch.arange(c.lens[b], device=DEV)
        page, slot = c.at(b, slots)
        base = torch.where((slots < c.lens[b] - n).unsqueeze(1), old[page, :, slot].double(), 0.0)
        if n:
            y = lse[start:start + n].double().view(n, c.H, c.G).permute(1, 2, 0).unsqueeze(-1)
            x = scores(c, Q, b, **options)
            base = base + torch.where(torch.isinf(y), 0.0, torch.exp(x - y)).sum((1, 2)).t()
        want[page, :, slot] = base
    top = lse[~torch.isinf(lse)].abs().max().item() if (~torch.isinf(lse)).any() else 0.0
    extra = 0.0
    if options.get("slopes") is not None:
        extra = float(options["slopes"].abs().max()) * max(c.lens) * 2.0 ** -22
    dx = 2.0 ** -19 * score_size(c, Q, options.get("scale")) + 2.0 ** -22 * top + extra + 2.0 ** -20
    tol = (dx + (max(c.new) * c.G + 8) * 2.0 ** -24) * want.abs() + 1e-30
    worst = ((out.double() - want).abs() / tol).max().item()
    assert worst <= 1.0, worst
    again = old.clone()
    c.call("weights", Q, lse, again, *c.scales[:1], **options)             # in place, and the same bits
    seen = out != -7.0
    assert torch.equal(again[seen], out[seen]) and torch.equal(again[~seen], old[~seen])


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 32), (256, 64)])
@pytest.mark.parametrize("fmt", FMTS)
def test_one_token_of_each_sequence(fmt, dim, page):
    c = Cache(fmt, [1, 77, 300, 0, 16, 129, 1000], 2, 4, dim, page)
    check_weights(c, queries(c))


@pytest.mark.parametrize("heads,group,new", [(1, 1, [3, 0]), (3, 5, [2, 2]), (1, 16, [9, 1]), (2, 4, [70, 31]), (1, 40, None)])
@pytest.mark.parametrize("fmt", FMTS)
def test_heads_and_new_tokens(fmt, heads, group, new):
    c = Cache(fmt, [150, 31], heads, group, 128, 16, new=new)
    check_weights(c, queries(c))


@pytest.mark.parametrize("o", OPTIONS, ids=lambda o: "-".join(o))
@pytest.mark.parametrize("fmt,new", [("mxfp4", None), ("nvfp4", [5, 1, 3]), ("mxint4", [60, 290, 64])])
def test_scoring(fmt, new, o):
    c = Cache(fmt, [129, 500, 64], 2, 3, 128, 32, new=new)
    check_weights(c, queries(c), **options_of(c, o))


def check_evict(c, w, keep, recent, width=None):
    """Places, lengths, codes, scale bytes and weights, to the bit."""
    P = c.P
    more = [-(-min(n, keep) // P) for n in c.lens]
    width = width or max(1, max(more))
    pool = torch.full((sum(more) + 1, *c.pages.shape[1:]), 0xEE, dtype=torch.uint8, device=DEV)
    c.pages = torch.cat([c.pages, pool])
    w = torch.cat([w, torch.full((pool.shape[0], *w.shape[1:]), -3.0, device=DEV)])
    at, rows = c.pages.shape[0] - pool.shape[0], []
    for n in more:
        rows.append(list(range(at, at + n)) + [-9] * (width - n))
        at += n
    new_table = torch.tensor(rows, dtype=torch.int32, device=DEV)
    want_pages, want_w = c.pages.clone(), w.clone()
    src, dst = parts(c.pages, c.fmt, c.D), parts(want_pages, c.fmt, c.D)
    lengths, kept = c.call_evict(w, new_table, keep, recent)
    assert lengths.tolist() == [min(n, keep) for n in c.lens]
    for b, n in enumerate(c.lens):
        stay = min(n, keep)
        late = min(recent, stay)
        for h in range(c.H):
            page, slot = c.at(b, torch.arange(n, device=DEV))
            v = want_w[page, h, slot][:n - late].tolist()
            best = sorted(range(n - late), key=lambda j: (-v[j], j))[:stay - late]
            places = sorted(best) + list(range(n - late, n))
            assert kept[b, h].tolist() == places + [-1] * (keep - stay), (b, h)
            if stay:
                s = torch.tensor(places, device=DEV)
                to = torch.arange(stay, device=DEV)
                tp, ts = torch.tensor(rows[b], device=DEV)[to // P], to % P
                fp, fs = c.at(b, s)
                for a, d in zip(src, dst):
                    d[tp, h, ts] = a[fp, h, fs]
                want_w[tp, h, ts] = want_w[fp, h, fs]
    assert torch.equal(c.pages, want_pages) and torch.equal(w, want_w)


def with_evict(c):
    c.call_evict = lambda *a: getattr(torq, f"torq_{c.fmt}_kv_evict")(c.pages, c.table, c.lengths, c.D, *a)
    return c


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (256, 32)])
@pytest.mark.parametrize("fmt", FMTS)
def test_evict(fmt, dim, page):
    for lens, keep, recent in (([100, 1, 0, 33, 64], 32, 8), ([70, 500], 1, 1), ([70, 500], 1, 0), ([40, 40], 40, 3), ([40, 39], 64, 64), ([300], 299, 0),
                               ([300, 20], 30, 30)):
        c = with_evict(Cache(fmt, lens, 2, 1, dim, page))
        w = torch.rand(c.pages.shape[0], 2, page, generator=gen(11), device=DEV)
        check_evict(c, w, keep, recent)


@pytest.mark.parametrize("kind", ["equal", "few values", "signs", "wide"])
def test_evict_equal_and_unequal_weights(kind):
    c = with_evict(Cache("mxfp4", [5000, 4099, 10], 2, 1, 64, 16))
    g = gen(12)
    shape = (c.pages.shape[0], 2, 16)
    w = {"equal": torch.zeros(shape, device=DEV), "few values": torch.randint(0, 3, shape, generator=g, device=DEV).float(),
         "signs": torch.randn(shape, generator=g, device=DEV) * (torch.rand(shape, generator=g, device=DEV) < 0.5),
         "wide": torch.exp(30 * torch.randn(shape, generator=g, device=DEV)).clamp(max=3e38)}[kind]
    w = w + 0.0                                          # -0 and 0 are different keys
    for keep, recent in ((4097, 100), (1000, 0), (7, 3)):
        check_evict(with_evict(Cache("mxfp4", [5000, 4099, 10], 2, 1, 64, 16)), w, keep, recent)


def test_account_and_eviction_over_a_few_steps():
    """Append, attend, account, evict and go on in the new pages, as a serving loop does."""
    fmt, H, G, D, P, keep = "nvfp4", 2, 4, 128, 16, 48
    g = gen(13)
    pages = torch.zeros(20, H, torq.torq_kv_page_bytes(fmt, P, D), dtype=torch.uint8, device=DEV)
    w = torch.zeros(20, H, P, device=DEV)
    table = torch.tensor([[0, 1, 2, 3], [4, 5, 6, 7]], dtype=torch.int32, device=DEV)
    other = torch.tensor([[8, 9, 10, 11], [12, 13, 14, 15]], dtype=torch.int32, device=DEV)
    lengths = torch.zeros(2, dtype=torch.int32, device=DEV)
    ts = (0.0125, 0.0031)
    plain = [[[], []], [[], []]]                         # of each sequence and head the keys and values, in 64 bits
    account = [[[], []], [[], []]]
    for step in range(70):
        n = 20 if step == 0 else 1
        starts = torch.tensor([0, n, 2 * n], dtype=torch.int32, device=DEV)
        lengths = lengths + n
        K, V = (torch.randn(2 * n, H, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
        Q = (2 * torch.randn(2 * n, H * G, D, generator=g, device=DEV)).to(torch.bfloat16)
        torq.torq_nvfp4_kv_append(pages, table, lengths, K, V, *ts, starts=starts)
        k, v = torq.torq_nvfp4_kv_read(pages, table, lengths, D, 2 * n, *ts, starts=starts, out_dtype=torch.float32)
        out, lse = torq.torq_nvfp4_kv_attention(pages, table, lengths, Q, *ts, starts=starts, return_lse=True)
        torq.torq_nvfp4_kv_weights(pages, table, lengths, Q, lse, w, ts[0], starts=starts)
        for b in (0, 1):
            for h in (0, 1):
                for i in range(n):
                    plain[b][h].append((k[b * n + i, h].double(), v[b * n + i, h].double()))
                    account[b][h].append(0.0)
                kk, vv = (torch.stack([x[i] for x in plain[b][h]]) for i in (0, 1))
                L = kk.shape[0]
                assert L == int(lengths[b])
                place = torch.arange(L - n, L, device=DEV).unsqueeze(1)
                for q in range(h * G, h * G + G):
                    x = Q[b * n:b * n + n, q].double() @ kk.t() * D ** -0.5
                    p = torch.where(torch.arange(L, device=DEV) <= place, x, -math.inf).softmax(-1)
                    ref = p @ vv
                    assert (out[b * n:b * n + n, q].double() - ref).abs().max() <= 0.02 * ref.abs().max()
                    account[b][h] = [a + t for a, t in zip(account[b][h], p.sum(0).tolist())]
        if int(lengths.max()) > 60:
            lengths, kept = torq.torq_nvfp4_kv_evict(pages, table, lengths, D, w, other, keep, 16)
            for b in (0, 1):
                for h in (0, 1):
                    places = kept[b, h].tolist()
                    sums = sorted(account[b][h][:-16], reverse=True)
                    assert all(account[b][h][j] >= sums[keep - 17] - 1e-3 for j in places[:keep - 16])     # of those near the edge either may stay
                    plain[b][h], account[b][h] = [plain[b][h][j] for j in places], [account[b][h][j] for j in places]
            table, other = other, table
    assert torq.torq_last_device_error() == 0
