"""The activation of the gated projections at its ends, through every kernel that has it: gates of every size up to float32's largest."""
import pytest
import torch

from operator_helpers import DEV, E2M1, silu, tile
from paper_2605_19561_b200 import torq

pytestmark = pytest.mark.gpu
FMTS = ("mxfp4", "nvfp4", "mxint4")
# 1.390625 2^127 is above float32's largest over log2(e), and its digits are all positive: no partial sum passes the largest
LARGEST = 1.390625 * 2.0 ** 127
GATES = [0.0, 2.0 ** -90, 1.5, 17.25, 80.0, 86.5, 87.0, 87.5, 88.0, 88.5, 89.0, 90.0, 92.0, 97.0, 101.0, 110.0, 2.0 ** 100, LARGEST]
GATES = GATES + [-g for g in GATES]


def check(Y, g, u):
    """Against silu(g) u in 64 bits.  Relative: 2^t 2^-22 (the instruction's), its correction with the addition of 1/2, the constant and the
    product 2^-22, the quotient 2^-23, the sum and two products 2^-24 each, so below 2^-20 together.  Below -87.3 the result may be zero:
    silu(-87.3) = -87.3 exp(-87.3) > -2^-119.  A product below 2^-126 is held to a multiple of 2^-149."""
    ref = silu(g) * u
    limit = torch.finfo(torch.float32).max
    far = ref.abs() > limit
    assert (Y.double()[far] == torch.sign(ref[far]) * torch.inf).all()
    tol = 2.0 ** -20 * ref.abs() + (g < -87.3) * 2.0 ** -119 * u.abs() + 2.0 ** -149
    bad = ~((Y.double() - ref).abs() <= tol) & ~far
    assert not bad.any(), [(a.item(), b.item(), y.item()) for a, b, y in zip(g.expand_as(Y)[bad][:8], u.expand_as(Y)[bad][:8], Y[bad][:8])]


def weights(fmt, N, K, gate_at, power):
    """Gate rows with 1 at `gate_at` times 2^power, up rows with 1 at 64: features below 64; above, the up row is the gate row."""
    v = torch.zeros(2 * N, K, dtype=torch.long, device=DEV)
    one = 1 if fmt == "mxint4" else 2                    # its code
    for k in gate_at:
        v[:, k] = one
    low = (torch.arange(2 * N, device=DEV) >= N) & (torch.arange(2 * N, device=DEV) % 128 < 64)
    v[low] = 0
    v[low, 64] = one
    codes = (v[:, 0::2] | v[:, 1::2] << 4).to(torch.uint8)
    block = 16 if fmt == "nvfp4" else 32
    lin = torch.full((2 * N, K // block), 0x38 if fmt == "nvfp4" else 127, dtype=torch.uint8, device=DEV)
    if power:
        lin[:, gate_at[0] // block] += power
    return codes, tile(lin)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("N,at_once", [(128, 3), (128, 8), (128, len(GATES)), (4096, len(GATES))])
def test_gated_matvec(fmt, N, at_once):
    K, power = 128, 7 if fmt == "mxint4" else 0          # MXINT4 takes magnitudes below 2^126
    codes, Ws = weights(fmt, N, K, (0,), power)
    g = torch.tensor(GATES, dtype=torch.float64, device=DEV)
    X = torch.zeros(len(GATES), K, dtype=torch.bfloat16, device=DEV)
    X[:, 0] = (g * 2.0 ** -power).to(torch.bfloat16)
    assert torch.equal(X[:, 0].double() * 2.0 ** power, g)
    X[:, 64] = 1
    f, ts = getattr(torq, f"torq_{fmt}_gated_matvec"), (1.0,) if fmt == "nvfp4" else ()
    Y = torch.cat([f(x.contiguous(), codes, Ws, *ts, out_dtype=torch.float32) for x in X.split(at_once)])
    n = torch.arange(N, device=DEV) % 128
    u = torch.where(n < 64, 1.0, g[:, None])
    fine = torch.ones(len(GATES), dtype=torch.bool, device=DEV)
    if fmt == "nvfp4":                                   # x is off by 2^-38 of its token's largest there: 1 beside 2^100, 2^-90 beside 1
        fine = (g == 0) | (g.abs() < 2.0 ** 32) & (g.abs() > 2.0 ** -32)
        check(Y[g.abs() > 1][:, n >= 64], g[g.abs() > 1][:, None], u[g.abs() > 1][:, n >= 64])
    check(Y[fine], g[fine][:, None], u[fine])
    assert torq.torq_last_device_error() == 0


def activations(fmt, parts, K):
    """Quantized rows with parts[m] = (mantissa, power) of the elements at 0 and 32, and 1 at 64."""
    M = len(parts)
    v = torch.zeros(M, K, dtype=torch.float64)
    lin = torch.full((M, K // (16 if fmt == "nvfp4" else 32)), 0x38 if fmt == "nvfp4" else 127, dtype=torch.uint8)
    g = torch.zeros(M, dtype=torch.float64)
    for m, row in enumerate(parts):
        for j, (mantissa, power) in enumerate(row):
            v[m, 32 * j] = mantissa
            lin[m, (2 if fmt == "nvfp4" else 1) * j] = 0x38 + 8 * power if fmt == "nvfp4" else 127 + power
            g[m] += mantissa * 2.0 ** power
    v[:, 64] = 1
    if fmt == "w4a8":
        q = v.to(torch.float32).to(torch.float8_e4m3fn)
        assert torch.equal(q.to(torch.float64), v)
        codes = q.view(torch.uint8)
    else:
        n = (v.abs()[..., None] == E2M1).long().argmax(-1) + 8 * (v < 0)
        codes = (n[:, 0::2] | n[:, 1::2] << 4).to(torch.uint8)
    return codes.contiguous().to(DEV), tile(lin.to(DEV)), g.to(DEV)


@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4", "w4a8"])
@pytest.mark.parametrize("few", [True, False])
def test_gated_gemm(fmt, few):
    N, K = 256, 128
    far = 7 if fmt == "nvfp4" else 127                   # 1.5 2^127, there with a tensor scale
    rows = []
    for s in (1.0, -1.0):
        rows += [((s, 6), (s, 4)), ((s, 6), (s * 1.5, 4)), ((s * 1.5, 6), (s, 1)), ((s * 1.5, 6), (s, 3)), ((s, 0), (s, 0)), ((s * 1.5, far), (s, 0))]
    rows = rows * (2 if few else 4)                      # 24 tokens; 48
    W = weights("mxint4" if fmt == "w4a8" else fmt, N, K, (0, 32), 0)
    if fmt == "w4a8":
        W = (torq.torq_mxint4_expand(W[0]), W[1])
    codes, As, g = activations(fmt, rows, K)
    n = torch.arange(N, device=DEV) % 128
    for ts in (1.0, 2.0 ** 120) if fmt == "nvfp4" else (None,):
        if ts is None:
            Y, scale = getattr(torq, f"torq_{'mxint4' if fmt == 'w4a8' else fmt}_gated_gemm")(codes, As, *W, out_dtype=torch.float32), 1.0
        else:                                            # 1.5 2^7 2^120 and the like: every gate is far from zero
            Y, scale = torq.torq_nvfp4_gated_gemm(codes, As, ts, *W, 1.0, out_dtype=torch.float32), ts
        check(Y, g[:, None] * scale, torch.where(n < 64, scale, g[:, None] * scale))
    assert torq.torq_last_device_error() == 0
