"""The gated pair of projections on quantized activations, and a feed-forward block of the operators around the layer, on a GPU
against their definitions in 64 bits."""
import pytest
import torch

from operator_helpers import (DEV, NORM_REL, check_gated, check_mxfp8, check_sums, gemm_steps, gen, matvec_error, norm_inputs, norm_ref,
                              quantized, untile, values)
from paper_2605_19561_b200 import torq

pytestmark = pytest.mark.gpu


def gated_gemm(fmt, A, W, **kw):
    if fmt == "nvfp4":
        return torq.torq_nvfp4_gated_gemm(A[0], A[1], A[2], W[0], W[1], W[2], **kw)
    return getattr(torq, f"torq_{'mxfp4' if fmt == 'mxfp4' else 'mxint4'}_gated_gemm")(A[0], A[1], W[0], W[1], **kw)


def operands(g, M, N, K, fmt):
    """Activations and weights; MXINT4 and w4a8 weights (and MXINT4 activations) in the operand form."""
    A = quantized(g, M, K, fmt, spread=8 if fmt == "w4a8" else 6, low=112 if fmt == "w4a8" else 118)
    W = quantized(g, 2 * N, K, "mxint4" if fmt == "w4a8" else fmt, spread=3, low=114, ts=0.0123 / 16)
    if fmt == "mxint4":
        A = (torq.torq_mxint4_expand(A[0]), *A[1:])
    if fmt in ("mxint4", "w4a8"):
        W = (torq.torq_mxint4_expand(W[0]), *W[1:])
    return A, W


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4", "mxint4", "w4a8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K", [(1, 128, 128), (3, 256, 384), (8, 25600, 640), (17, 384, 2304), (24, 5632, 1024), (25, 256, 896), (32, 1024, 512), (33, 128, 256), (128, 128, 256), (129, 384, 640), (256, 1024, 2048), (300, 2176, 1152),
                                   (777, 5504, 1024), (2600, 5632, 512)])
def test_gated_gemm(fmt, dtype, M, N, K):
    A, W = operands(gen(M + N), M, N, K, fmt)
    buf = torch.full((M * N + 64,), 7.0, dtype=dtype, device=DEV)
    before = torq.torq_launch_count()
    Y = gated_gemm(fmt, A, W, Y=buf[:M * N].view(M, N))
    assert torq.torq_launch_count() == before + 1
    check_gated(Y, A[3], W[3], gemm_steps(K))
    assert (buf[M * N:] == 7).all()
    assert torch.equal(gated_gemm(fmt, A, W, out_dtype=dtype), Y)
    assert torq.torq_last_device_error() == 0


@pytest.mark.parametrize("M", [1, 100, 300])
def test_mxfp8_activations_through_the_integer_gemm(M):
    g, N, K = gen(M), 520, 896
    W, A = quantized(g, N, K, "mxint4"), quantized(g, M, K, "w4a8", low=112, spread=8)
    Y = torq.torq_mxint4_gemm(A[0], A[1], torq.torq_mxint4_expand(W[0]), W[1], out_dtype=torch.float32)
    check_sums(Y, A[3], W[3], gemm_steps(K))


def test_refusals():
    A, W = operands(gen(1), 4, 128, 256, "mxfp4")
    f = torq.torq_mxfp4_gated_gemm
    bad = [lambda: f(A[0].to(torch.bfloat16), A[1], W[0], W[1]), lambda: f(A[0], None, W[0], W[1]), lambda: f(A[0], A[1][:-16], W[0], W[1]),
           lambda: f(A[0], A[1], W[0], W[1][:-16]), lambda: f(A[0][:, :64].contiguous(), A[1], W[0], W[1]), lambda: f(A[0], A[1], W[0][:255], W[1]),
           lambda: f(A[0], A[1], W[0], W[1], Y=torch.empty(4, 256, dtype=torch.bfloat16, device=DEV)), lambda: f(A[0].cpu(), A[1], W[0], W[1])]
    before = torq.torq_launch_count()
    for call in bad:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(torq.TorqError) as e:
        f(A[0], A[1], W[0][:128], W[1])                  # 64 features: no whole scale tiles
    assert e.value.code == 2
    assert torq.torq_launch_count() == before


# ---- together ----------------------------------------------------------------------------------------------------------
def ffn_weights(g, d, F):
    """Gate and up [2F, d], down [d, F] by the library's quantizer in MXINT4: (stored form, operand form, scales, values)."""
    out = []
    for w in (torch.randn(2 * F, d, generator=g, device=DEV) * d ** -0.5, torch.randn(d, F, generator=g, device=DEV) * F ** -0.5):
        packed, s = torq.torq_quantize_mxint4(w, packed=True)
        out.append((packed, torq.torq_mxint4_expand(packed), s, values(packed, untile(s, w.shape[0], w.shape[1] // 32), "mxint4")))
    return out


def ffn_decode(x, r, w, up, down):
    y, h = torq.torq_add_rmsnorm(x, w, r)
    z = torq.torq_mxint4_gated_matvec(y, up[0], up[2])
    return y, h, z, torq.torq_mxint4_matvec(z, down[0], down[2])


def ffn_prefill(x, r, w, up, down):
    a, s, h = torq.torq_add_rmsnorm_mxfp8(x, w, r)
    z = torq.torq_mxint4_gated_gemm(a, s, up[1], up[2])
    q, qs = torq.torq_quantize_mxint4(z)
    return a, s, h, z, q, qs, torq.torq_mxint4_gemm(q, qs, down[1], down[2])


@pytest.mark.parametrize("M", [1, 6, 23])
def test_feed_forward_block_decoding(M):
    d, F = 512, 1408
    up, down = ffn_weights(gen(M), d, F)
    x, r, w = norm_inputs(M, d, torch.bfloat16, torch.bfloat16)
    y, _, z, out = ffn_decode(x, r, w, up, down)
    ref = norm_ref(x, r, w, 1e-6)
    assert ((y.double() - ref).abs() <= (2.0 ** -8 + NORM_REL) * ref.abs()).all()
    check_gated(z, y.double(), up[3], *matvec_error("mxint4", y.double()))
    check_sums(out, z.double(), down[3], *matvec_error("mxint4", z.double()))


@pytest.mark.parametrize("M", [1, 130, 555])
def test_feed_forward_block_prefill(M):
    d, F = 512, 1408
    up, down = ffn_weights(gen(M), d, F)
    x, r, w = norm_inputs(M, d, torch.float32, torch.float32)
    a, s, _, z, q, qs, out = ffn_prefill(x, r, w, up, down)
    check_mxfp8(a, s, norm_ref(x, r, w, 1e-6))
    check_gated(z, values(a, untile(s, M, d // 32), "w4a8"), up[3], gemm_steps(d))
    check_sums(out, values(q, untile(qs, M, F // 32), "w4a8"), down[3], gemm_steps(F))


@pytest.mark.parametrize("M", [4, 6, 40])
def test_feed_forward_block_captured_and_on_another_stream(M):
    d, F = 512, 1408
    up, down = ffn_weights(gen(0), d, F)
    x, r, w = norm_inputs(M, d, torch.bfloat16, torch.bfloat16)

    def both():
        return (*ffn_decode(x, r, w, up, down), *ffn_prefill(x, r, w, up, down))

    want = [t.clone() for t in both()]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):                           # the current stream is the one that is used
        got = both()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = both()
    other = norm_inputs(M, d, torch.bfloat16, torch.bfloat16, seed=9)
    keep = x.clone(), r.clone()
    for xs in (other[:2], keep):
        x.copy_(xs[0])
        r.copy_(xs[1])
        for t in captured:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, both()))
    assert torq.torq_last_device_error() == 0


def test_calls_through_ctypes_are_the_same(monkeypatch):
    """The native marshalling and the one that stands in for it where it cannot be had."""
    d, F, M = 512, 1408, 4
    up, down = ffn_weights(gen(0), d, F)
    x, r, w = norm_inputs(M, d, torch.bfloat16, torch.bfloat16)

    def both():
        return (*ffn_decode(x, r, w, up, down), *ffn_prefill(x, r, w, up, down), torq.torq_add_rmsnorm(x, w), *torq.torq_add_rmsnorm_mxfp8(x, w))

    want = both()
    monkeypatch.setattr(torq, "_product_native", lambda *a: -1)
    monkeypatch.setattr(torq, "_norm_native", lambda *a: -1)
    assert all(torch.equal(a, b) and a.dtype is b.dtype for a, b in zip(both(), want, strict=True))


def test_two_graphs_replayed_in_turn():
    """Each has its own workspace and results, whatever the other does in between."""
    d, F = 512, 1408
    up, down = ffn_weights(gen(0), d, F)
    graphs = []
    for M in (6, 9):
        x, r, w = norm_inputs(M, d, torch.bfloat16, torch.bfloat16, seed=M)
        want = [t.clone() for t in ffn_decode(x, r, w, up, down)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = ffn_decode(x, r, w, up, down)
        graphs.append((graph, got, want, x, r, w))
    for _ in range(3):
        for graph, *_ in graphs:
            graph.replay()
    torch.cuda.synchronize()
    for _, got, want, *_ in graphs:
        assert all(torch.equal(a, b) for a, b in zip(got, want))
