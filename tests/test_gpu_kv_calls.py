"""How the operators of the 4-bit cache may be called: streams, graphs, strides, workspaces, pages far into a large cache, bad pages."""
import pytest
import torch

from kv_helpers import FMTS, Cache, attention, check_attention, queries, score_size
from operator_helpers import DEV, gen
from paper_2605_19561_b200 import torq

pytestmark = pytest.mark.gpu

# few and many new tokens
NEW = [None, [120, 200]]


def cache(fmt, new, dim=128, **kw):
    return Cache(fmt, [700, 333], 32, 2, dim, 32, new=new, **kw)


@pytest.mark.parametrize("new", NEW, ids=["one", "many"])
@pytest.mark.parametrize("fmt", FMTS)
def test_the_same_call_gives_the_same_bits(fmt, new):
    c = cache(fmt, new)
    Q = queries(c)
    first = c.call("attention", Q, *c.scales, return_lse=True)
    w = torch.zeros(c.pages.shape[0], c.H, c.P, device=DEV)
    args = (c.scales[0],) if c.scales else ()
    account = c.call("weights", Q, first[1], w.clone(), *args)
    for _ in range(5):
        again = c.call("attention", Q, *c.scales, return_lse=True)
        assert all(torch.equal(a, b) for a, b in zip(first, again))
        assert torch.equal(account, c.call("weights", Q, first[1], w.clone(), *args))


@pytest.mark.parametrize("new", NEW, ids=["one", "many"])
def test_queries_that_are_columns_of_a_projection(new):
    c = cache("mxfp4", new)
    Q = queries(c)
    wide = torch.full((c.tokens, c.H * c.G * c.D + 2 * c.H * c.D), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, :c.H * c.G * c.D] = Q.flatten(1)
    view = wide[:, :c.H * c.G * c.D].unflatten(1, (c.H * c.G, c.D))
    a, b = c.call("attention", Q, return_lse=True), c.call("attention", view, return_lse=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    w = torch.zeros(c.pages.shape[0], c.H, c.P, device=DEV)
    assert torch.equal(c.call("weights", Q, a[1], w.clone()), c.call("weights", view, a[1], w.clone()))


@pytest.mark.parametrize("new", NEW, ids=["one", "many"])
def test_two_streams_at_once_with_their_own_workspaces(new):
    cs = [cache("nvfp4", new, seed=i) for i in range(2)]
    Qs = [queries(c, seed=7 + i) for i, c in enumerate(cs)]
    want = [c.call("attention", Q, *c.scales, return_lse=True) for c, Q in zip(cs, Qs)]
    size = torq.torq_kv_attention_workspace_bytes(cs[0].tokens, 2, 64, 32, 128)
    work = [torch.full((size,), 255, dtype=torch.uint8, device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(cs[i].call("attention", Qs[i], *cs[i].scales, return_lse=True, workspace=work[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i][0]) and torch.equal(z, want[i][1]) for y, z in got[i])


def test_a_named_stream():
    """stream=: the launches go there; memory that the call takes itself belongs to it."""
    c = cache("mxfp4", None)
    Q = queries(c)
    want = c.call("attention", Q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = [c.call("attention", Q, stream=s) for _ in range(20)]
    s.synchronize()
    assert all(torch.equal(g, want) for g in got)


@pytest.mark.parametrize("fmt", FMTS)
def test_a_captured_step_replayed_over_a_growing_cache(fmt):
    """A decoding step - append, attention, account - captured once: the lengths on the device grow from replay to replay."""
    H, G, D, P = 4, 4, 128, 16
    c = Cache(fmt, [1, 30, 95], H, G, D, P, width=10)
    n = c.pages.shape[0]
    pages = torch.cat([c.pages, torch.full((30, *c.pages.shape[1:]), 255, dtype=torch.uint8, device=DEV)])
    table = torch.tensor([(r + [n + 10 * b + i for i in range(10)])[:10] for b, r in enumerate(c.table_rows)], dtype=torch.int32, device=DEV)
    lengths = c.lengths.clone()
    K, V = (torch.zeros(3, H, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    Q = torch.zeros(3, H * G, D, dtype=torch.bfloat16, device=DEV)
    weights = torch.zeros(pages.shape[0], H, P, device=DEV)
    out, work = torch.zeros_like(Q), torch.zeros(torq.torq_kv_attention_workspace_bytes(3, 3, H * G, H, D), dtype=torch.uint8, device=DEV)
    f = {name: getattr(torq, f"torq_{fmt}_kv_{name}") for name in ("append", "attention", "weights")}

    def step(p, n, w, **kw):
        f["append"](p, table, n, K, V, *c.scales)
        y, lse = f["attention"](p, table, n, Q, *c.scales, return_lse=True, **kw)
        f["weights"](p, table, n, Q, lse, w, *c.scales[:1], weights_out=w)
        return y, lse

    step(pages.clone(), lengths.clone(), weights.clone())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        _, lse = step(pages, lengths, weights, out=out, workspace=work)
    eager = [pages.clone(), lengths.clone(), weights.clone()]
    g = gen(9)
    for i in range(40):
        K.copy_(torch.randn(K.shape, generator=g, device=DEV))
        V.copy_(torch.randn(V.shape, generator=g, device=DEV))
        Q.copy_(torch.randn(Q.shape, generator=g, device=DEV))
        lengths += 1
        eager[1] += 1
        work.fill_(255)                                  # nothing is kept in it
        graph.replay()
        y, z = step(*eager)
        assert torch.equal(out, y) and torch.equal(lse, z)
        assert torch.equal(pages, eager[0]) and torch.equal(weights, eager[2])
    assert torq.torq_last_device_error() == 0


@pytest.mark.parametrize("new", NEW, ids=["one", "many"])
@pytest.mark.parametrize("fmt", FMTS)
def test_pages_behind_2_to_31_bytes(fmt, new):
    c = cache(fmt, new)
    Q = queries(c)
    w = torch.rand(c.pages.shape[0], c.H, c.P, generator=gen(2), device=DEV)
    args = (c.scales[0],) if c.scales else ()
    out, lse = c.call("attention", Q, *c.scales, return_lse=True)
    check_attention(c, Q, out, lse)
    account = c.call("weights", Q, lse, w.clone(), *args)
    read = c.call("read", c.D, c.tokens, *c.scales)
    far = (1 << 32) // c.pages[0].numel() + 1
    used = c.pages.shape[0]
    big = torch.empty(far + used, *c.pages.shape[1:], dtype=torch.uint8, device=DEV)
    big[far:] = c.pages
    table, owned = c.table, (c.table >= 0) & (c.table < used)
    c.pages, c.table = big, torch.where(owned, table + far, table)
    got = c.call("attention", Q, *c.scales, return_lse=True)
    assert torch.equal(got[0], out) and torch.equal(got[1], lse)
    assert all(torch.equal(a, b) for a, b in zip(c.call("read", c.D, c.tokens, *c.scales), read))
    wide = torch.zeros(far + used, c.H, c.P, device=DEV)
    wide[far:] = w
    assert torch.equal(c.call("weights", Q, lse, wide, *args, weights_out=wide)[far:], account)
    assert not wide[:far].any()


@pytest.mark.parametrize("new", NEW, ids=["one", "many"])
@pytest.mark.parametrize("fmt", FMTS)
def test_a_bad_page_is_an_error_and_the_other_sequences_stay_right(fmt, new):
    c = cache(fmt, new)
    Q = queries(c)
    out, lse = c.call("attention", Q, *c.scales, return_lse=True)
    w = torch.rand(c.pages.shape[0], c.H, c.P, generator=gen(2), device=DEV)
    args = (c.scales[0],) if c.scales else ()
    account = c.call("weights", Q, lse, w.clone(), *args)
    torq.torq_last_device_error()
    rows = slice(1, 2) if new is None else slice(new[0], None)
    keep = torch.tensor(c.table_rows[1], device=DEV)
    for page in (-1, c.pages.shape[0], 2 ** 31 - 1, -2 ** 31):
        c.table[0, 3] = page
        y, z = c.call("attention", Q, *c.scales, return_lse=True)
        assert torq.torq_last_device_error() == 8
        assert torch.equal(y[rows], out[rows]) and torch.equal(z[rows], lse[rows])
        a = c.call("weights", Q, lse, w.clone(), *args)
        assert torq.torq_last_device_error() == 8
        assert torch.equal(a[keep], account[keep])


def test_a_bad_page_of_an_eviction_is_an_error():
    c = cache("mxfp4", None)
    w = torch.rand(c.pages.shape[0], c.H, c.P, generator=gen(2), device=DEV)
    n = c.pages.shape[0]
    c.pages = torch.cat([c.pages, torch.zeros(20, *c.pages.shape[1:], dtype=torch.uint8, device=DEV)])
    w = torch.cat([w, torch.zeros(20, c.H, c.P, device=DEV)])
    target = torch.arange(n, n + 20, dtype=torch.int32, device=DEV).view(2, 10)
    good, good_w = c.pages.clone(), w.clone()
    f = torq.torq_mxfp4_kv_evict
    f(good, c.table, c.lengths, c.D, good_w, target, keep=300, recent=10)
    torq.torq_last_device_error()
    for which in ("source", "target"):
        for page in (-1, n + 20, 2 ** 31 - 1, -2 ** 31):
            pages, weights, t, nt = c.pages.clone(), w.clone(), c.table.clone(), target.clone()
            (t if which == "source" else nt)[0, 3] = page
            f(pages, t, c.lengths, c.D, weights, nt, keep=300, recent=10)
            assert torq.torq_last_device_error() == 8
            assert torch.equal(pages[n + 10:], good[n + 10:]) and torch.equal(weights[n + 10:], good_w[n + 10:])
            assert torch.equal(pages[:n], c.pages[:n])
            if which == "target":                        # what has a page to go to is there
                other = torch.arange(n, n + 10, device=DEV) != n + 3
                assert torch.equal(pages[n:n + 10][other], good[n:n + 10][other])


def test_lengths_that_the_table_has_no_room_for():
    """A length above the table's room is an error, one below zero counts as none; no page outside is touched.  (The other sequence's result may be
    summed in another order, so it is held to the definition: the bounds of check_attention with scores of the size that they have here.)"""
    c = cache("mxint4", None)
    Q = queries(c)
    ref, _, mag = attention(c, Q)
    tol = (2.0 ** -18 * score_size(c, Q) + 2.0 ** -18 + 2.0 ** -11) * mag + 2.0 ** -8 * ref.abs() + 2.0 ** -35 * c.V[1].abs().sum(0).repeat_interleave(c.G, 0)
    torq.torq_last_device_error()
    for bad in (c.width * c.P + 1, 2 ** 31 - 1, -1, -2 ** 31):
        c.lengths[0] = bad
        y = c.call("attention", Q)
        assert torq.torq_last_device_error() == (8 if bad > 0 else 0)
        assert ((y[1].double() - ref[1]).abs() <= tol[1]).all()
        if bad < 0:
            assert not y[0].any()


def test_refusals_on_the_device():
    """The checks that need tensors on the GPU: what is wrong is named, nothing runs."""
    c = cache("mxfp4", None)
    Q = queries(c)
    for bad in (dict(Q=Q.float()), dict(Q=Q[:1]), dict(Q=Q[:, :63]), dict(Q=Q[..., ::2]), dict(Q=Q[..., :96]), dict(Q=Q.cpu())):
        with pytest.raises((ValueError, torq.TorqError)):
            c.call("attention", bad["Q"])
    for kw in (dict(slopes=torch.zeros(3, device=DEV)), dict(slopes=torch.zeros(64, device=DEV, dtype=torch.bfloat16)), dict(window=-1), dict(softcap=-1.0),
               dict(prefix=torch.zeros(3, dtype=torch.int32, device=DEV)), dict(first=torch.zeros(2, dtype=torch.int64, device=DEV)),
               dict(out=torch.zeros(2, 64, 64, dtype=torch.bfloat16, device=DEV)), dict(workspace=torch.zeros(16, dtype=torch.uint8, device=DEV)),
               dict(scale=float("nan")), dict(softcap=float("inf"))):
        with pytest.raises((ValueError, torq.TorqError)):
            c.call("attention", Q, **kw)
    with pytest.raises((ValueError, torq.TorqError)):
        torq.torq_mxfp4_kv_attention(c.pages, c.table.long(), c.lengths, Q)
    with pytest.raises((ValueError, torq.TorqError)):
        torq.torq_mxfp4_kv_attention(c.pages[:, :, ::2], c.table, c.lengths, Q)
    with pytest.raises((ValueError, torq.TorqError)):
        torq.torq_mxfp4_kv_attention(c.pages, c.table, c.lengths[:1], Q)
    lse, w = torch.zeros(2, 64, device=DEV), torch.zeros(c.pages.shape[0], c.H, c.P, device=DEV)
    for a in ((lse.double(), w), (lse[:1], w), (lse, w[:-1]), (lse, w.double())):
        with pytest.raises((ValueError, torq.TorqError)):
            c.call("weights", Q, *a)
    for kw in (dict(keep=0, recent=0), dict(keep=4, recent=5), dict(keep=64, recent=-1)):
        with pytest.raises((ValueError, torq.TorqError)):
            torq.torq_mxfp4_kv_evict(c.pages, c.table, c.lengths, c.D, w, c.table.clone(), **kw)
    torch.cuda.synchronize()
    assert torq.torq_last_device_error() == 0
