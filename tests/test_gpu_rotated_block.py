"""The operators with the layer's own rotations and weights: norm -> rotation and quantizer -> gated pair of projections -> rotated layer,
all of it by the library, against 64 bits at every step, and captured."""
import pytest
import torch

from operator_helpers import DEV, NORM_REL, check_gated, check_sums, gemm_steps, gen, norm_inputs, norm_ref, silu, untile, values
from paper_2605_19561_b200 import torq

pytestmark = pytest.mark.gpu
D, F = 512, 1408
BLOCK = {"mxfp4": 32, "nvfp4": 16, "mxint4": 32}


def rotation(g, d, fmt):
    """Inter [d, d] and intra rotation in the form that the kernels take."""
    q = lambda *s: torch.linalg.qr(torch.randn(*s, generator=g, device=DEV, dtype=torch.float64))[0].to(torch.bfloat16).contiguous()
    R, b = q(d, d), BLOCK[fmt]
    Ri = q(d // b, b, b)
    return R, torq.torq_expand_intra16(Ri) if fmt == "nvfp4" else Ri


def prepared(fmt, R, Ri, W):
    """Operands of the GEMM and the values they stand for."""
    p = getattr(torq, "torq_prepare_weights" + ("" if fmt == "mxfp4" else "_" + fmt))(R, Ri, W)
    codes, Ws, ts = (p[1], p[2], 1.0) if fmt == "mxint4" else (*p, 1.0)[:3]
    return codes, Ws, ts, values(codes, untile(Ws, W.shape[1], W.shape[0] // BLOCK[fmt]), "w4a8" if fmt == "mxint4" else fmt, ts)


def run(fmt, x, r, w, first, second):
    R, Ri, W, ts = first
    y, h = torq.torq_add_rmsnorm(x, w, r)
    if fmt == "nvfp4":
        a, s = torq.torq_rotate_quantize_nvfp4(y, R, Ri, ts)
        z = torq.torq_nvfp4_gated_gemm(a, s, ts, W[0], W[1], W[2])
        R, Ri, W, ts = second
        return y, h, a, s, z, torq.torq_rotated_linear_nvfp4(z, R, Ri, ts, W[0], W[1], W[2], out_dtype=torch.float32)
    tail = "" if fmt == "mxfp4" else "_mxint4"
    a, s = getattr(torq, "torq_rotate_quantize" + tail)(y, R, Ri)
    z = getattr(torq, f"torq_{fmt}_gated_gemm")(a, s, W[0], W[1])
    R, Ri, W, ts = second
    return y, h, a, s, z, getattr(torq, "torq_rotated_linear" + tail)(z, R, Ri, W[0], W[1], out_dtype=torch.float32)


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4", "mxint4"])
@pytest.mark.parametrize("M", [1, 24, 130, 700])
def test_block(fmt, M):
    g = gen(M)
    x, r, w = norm_inputs(M, D, torch.bfloat16, torch.bfloat16)
    (R, Ri), (R2, Ri2) = rotation(g, D, fmt), rotation(g, F, fmt)
    up, down = torch.randn(D, 2 * F, generator=g, device=DEV) * D ** -0.5, torch.randn(F, D, generator=g, device=DEV) * F ** -0.5
    W, W2 = prepared(fmt, R, Ri, up), prepared(fmt, R2, Ri2, down)
    first, second = (R, Ri, W, 8.0 / 2688), (R2, Ri2, W2, 4.0 / 2688)          # tensor scales as calibration leaves them
    y, h, a, s, z, out = want = run(fmt, x, r, w, first, second)
    ref = norm_ref(x, r, w, 1e-6)
    assert ((y.double() - ref).abs() <= (2.0 ** -8 + NORM_REL) * ref.abs()).all()
    v = values(a, untile(s, M, D // BLOCK[fmt]), "w4a8" if fmt == "mxint4" else fmt, first[3] if fmt == "nvfp4" else 1.0)
    check_gated(z, v, W[3], gemm_steps(D))
    # The layer takes the same z through the library's rotation and quantizer, whose tests stand elsewhere
    if fmt == "nvfp4":
        q = torq.torq_rotate_quantize_nvfp4(z, R2, Ri2, second[3])
    else:
        q = getattr(torq, "torq_rotate_quantize" + ("" if fmt == "mxfp4" else "_mxint4"))(z, R2, Ri2)
    check_sums(out, values(q[0], untile(q[1], M, F // BLOCK[fmt]), "w4a8" if fmt == "mxint4" else fmt, second[3] if fmt == "nvfp4" else 1.0), W2[3], gemm_steps(F))
    # The rotation of the activations meets the inverse one in the weights: without it the cosine with the unquantized product is a random one
    # (below 0.1 in thousands of elements); four bits leave a noise of a seventh per operand, so of a third at most in the product of both sums
    g64, u64 = y.double() @ up.double()[:, :F], y.double() @ up.double()[:, F:]
    assert torch.cosine_similarity(z.double().flatten(), (silu(g64) * u64).flatten(), dim=0) > 0.85
    # captured, and replayed with other tokens
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run(fmt, x, r, w, first, second)
    keep = x.clone(), r.clone()
    for xs in (norm_inputs(M, D, torch.bfloat16, torch.bfloat16, seed=7)[:2], keep):
        x.copy_(xs[0])
        r.copy_(xs[1])
        for t in captured:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, e) for p, e in zip(captured, run(fmt, x, r, w, first, second)))
    assert all(torch.equal(p, e) for p, e in zip(captured, want))
    assert torq.torq_last_device_error() == 0
