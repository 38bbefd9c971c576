"""The 4-bit key/value cache, what needs no GPU: argument errors of the C entry points are status codes before anything touches a device, and the
Python calls refuse tensors that are not what a call takes."""
import ctypes

import pytest
import torch

from paper_2605_19561_b200 import torq

FMTS = ["mxfp4", "nvfp4", "mxint4"]
ONE, ODD, TWO = 256, 264, 258                            # never dereferenced on these paths
NULL, SHAPE, ALIGN, WORKSPACE = 1, 2, 3, 7


def cache(**k):
    d = dict(pages=ONE, table=ONE, lengths=ONE, num_pages=4, page_tokens=16, kv_heads=2, head_dim=128, batch=3, table_width=2, k_tensor_scale=1.0,
             v_tensor_scale=1.0)
    d.update(k)
    return torq._KvCache(*(d[n] for n, _ in torq._KvCache._fields_))


def scoring(**k):
    d = dict(scale=0.1, softcap=0.0, slopes=None, window=0, prefix=None, first=None)
    d.update(k)
    return torq._KvScoring(*(d[n] for n, _ in torq._KvScoring._fields_))


def append(fmt, c=None, K=ONE, V=ONE, t=1, ks=256, vs=256, starts=ONE, tokens=5):
    return getattr(torq.lib(), f"torq_{fmt}_kv_append")(c or cache(), K, V, t, ks, vs, starts, tokens, None)


def read(fmt, c=None, starts=ONE, tokens=5, K=ONE, V=ONE, t=1):
    return getattr(torq.lib(), f"torq_{fmt}_kv_read")(c or cache(), starts, tokens, K, V, t, None)


def attention(fmt, c=None, s=None, Q=ONE, qs=1024, heads=8, starts=ONE, tokens=5, out=ONE, lse=ONE, ws=ONE, n=1 << 40):
    return getattr(torq.lib(), f"torq_{fmt}_kv_attention")(c or cache(), s or scoring(), Q, qs, heads, starts, tokens, out, lse, ws, n, None)


def weights(fmt, c=None, s=None, Q=ONE, qs=1024, heads=8, starts=ONE, tokens=5, lse=ONE, w=ONE, o=ONE):
    return getattr(torq.lib(), f"torq_{fmt}_kv_weights")(c or cache(), s or scoring(), Q, qs, heads, starts, tokens, lse, w, o, None)


def evict(fmt, c=None, w=ONE, table=ONE, width=2, keep=32, recent=4, lengths=ONE, kept=ONE):
    return getattr(torq.lib(), f"torq_{fmt}_kv_evict")(c or cache(), w, table, width, keep, recent, lengths, kept, None)


CALLS = [append, read, attention, weights, evict]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("fmt", FMTS)
def test_the_cache(fmt, call):
    for k in ("pages", "table", "lengths"):
        assert call(fmt, cache(**{k: None})) == NULL
        assert call(fmt, cache(**{k: TWO})) == ALIGN
    assert call(fmt, cache(pages=ODD)) == ALIGN
    for k, values in (("head_dim", (0, 32, 96, 512)), ("page_tokens", (0, 8, 24, 2048, -16)), ("kv_heads", (0, -1, 1025)),
                      ("num_pages", (0, 1 << 31)), ("batch", (0, -1, 65537)), ("table_width", (0, -1, 1 << 27))):
        for v in values:
            assert call(fmt, cache(**{k: v})) == SHAPE, (k, v)
    for ts in (0.0, -1.0, float("nan"), float("inf")):
        for k in ("k_tensor_scale", "v_tensor_scale"):
            if fmt == "nvfp4":
                assert call(fmt, cache(**{k: ts})) == SHAPE


@pytest.mark.parametrize("fmt", FMTS)
def test_append_and_read(fmt):
    for k in ("K", "V"):
        assert append(fmt, **{k: None}) == NULL and append(fmt, **{k: ODD}) == ALIGN
        assert read(fmt, **{k: None}) == NULL and read(fmt, **{k: ODD}) == ALIGN
    for call in (append, read):
        assert call(fmt, tokens=0) == SHAPE and call(fmt, tokens=(1 << 24) + 1) == SHAPE and call(fmt, t=2) == SHAPE
        assert call(fmt, starts=None) == SHAPE and call(fmt, starts=TWO) == ALIGN          # 5 tokens of 3 sequences
        assert call(fmt, cache(kv_heads=1024, head_dim=256), tokens=1 << 24, **({"ks": 1 << 20, "vs": 1 << 20} if call is append else {})) == SHAPE
    assert append(fmt, ks=255) == SHAPE and append(fmt, vs=0) == SHAPE
    assert append(fmt, ks=260) == ALIGN and append(fmt, t=0, vs=258) == ALIGN


@pytest.mark.parametrize("call", [attention, weights])
@pytest.mark.parametrize("fmt", FMTS)
def test_queries_and_scoring(fmt, call):
    assert call(fmt, Q=None) == NULL and call(fmt, Q=ODD) == ALIGN
    assert call(fmt, heads=0) == SHAPE and call(fmt, heads=7, qs=896) == SHAPE and call(fmt, qs=1016) == SHAPE and call(fmt, qs=1028) == ALIGN
    assert call(fmt, starts=None) == SHAPE and call(fmt, starts=TWO) == ALIGN and call(fmt, tokens=0) == SHAPE
    for k, values in (("scale", (0.0, -1.0, float("nan"), float("inf"))), ("softcap", (-1.0, float("nan"), float("inf"))), ("window", (-1,))):
        for v in values:
            assert call(fmt, s=scoring(**{k: v})) == SHAPE, (k, v)
    for k in ("slopes", "prefix", "first"):
        assert call(fmt, s=scoring(**{k: TWO})) == ALIGN
    assert call(fmt, lse=TWO) == ALIGN


@pytest.mark.parametrize("fmt", FMTS)
def test_attention_weights_evict(fmt):
    assert attention(fmt, out=None) == NULL and attention(fmt, out=ODD) == ALIGN and attention(fmt, ws=ODD) == ALIGN
    need = torq.torq_kv_attention_workspace_bytes(5, 3, 8, 2, 128)
    if need:
        assert attention(fmt, ws=None) == WORKSPACE and attention(fmt, n=need - 1) == WORKSPACE
    for k in ("lse", "w", "o"):
        assert weights(fmt, **{k: None}) == NULL
    assert weights(fmt, w=ODD) == ALIGN and weights(fmt, o=ODD) == ALIGN
    for k in ("w", "table", "lengths", "kept"):
        assert evict(fmt, **{k: None}) == NULL and evict(fmt, **{k: TWO}) == ALIGN
    assert evict(fmt, keep=0) == SHAPE and evict(fmt, recent=-1) == SHAPE and evict(fmt, recent=33) == SHAPE
    assert evict(fmt, width=0) == SHAPE and evict(fmt, width=1) == SHAPE                  # no room for 32 tokens
    assert evict(fmt, cache(batch=65536)) == SHAPE


def test_page_bytes():
    assert torq.torq_kv_page_bytes("mxfp4", 64, 128) == 2 * 64 * (64 + 4) and torq.torq_kv_page_bytes("nvfp4", 16, 64) == 2 * 16 * (32 + 4)
    L = torq.lib()
    assert L.torq_kv_page_bytes(8, 16, 64) == 0 and L.torq_kv_page_bytes(32, 0, 64) == 0 and L.torq_kv_page_bytes(32, 16, -64) == 0
    assert L.torq_status_string(8) not in (b"", b"unknown")


def test_python_refuses_host_tensors():
    pages, table, lengths = torch.zeros(4, 2, 2 * 16 * 68, dtype=torch.uint8), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    x, w = torch.zeros(3, 2, 128, dtype=torch.bfloat16), torch.zeros(4, 2, 16)
    for f in (lambda: torq.torq_mxfp4_kv_append(pages, table, lengths, x, x), lambda: torq.torq_nvfp4_kv_append(pages, table, lengths, x, None, 1.0, 1.0),
              lambda: torq.torq_mxint4_kv_read(pages, table, lengths, 128, 3), lambda: torq.torq_mxfp4_kv_attention(pages, table, lengths, x),
              lambda: torq.torq_mxfp4_kv_attention(pages, table, lengths, None), lambda: torq.torq_mxfp4_kv_weights(pages, table, lengths, x, w, w),
              lambda: torq.torq_mxfp4_kv_evict(pages, table, lengths, 128, w, table, 4), lambda: torq.torq_mxfp4_kv_evict(pages, None, lengths, 128, w, table, 4)):
        with pytest.raises(ValueError):
            f()
