"""Products of few tokens whose every partial sum is a float32: equal to the 64-bit ones bit for bit, at every kernel's sizes."""
import pytest
import torch

from operator_helpers import DEV, code_values, gen, silu, tile
from paper_2605_19561_b200 import torq

pytestmark = pytest.mark.gpu
FMTS = ("mxfp4", "nvfp4", "mxint4")
BLOCK = {"mxfp4": 32, "nvfp4": 16, "mxint4": 32}


def product(fmt, X, codes, power, gated):
    """Block scales of 2^power everywhere."""
    lin = torch.full((codes.shape[0], X.shape[1] // BLOCK[fmt]), 0x38 + 8 * power if fmt == "nvfp4" else 127 + power, dtype=torch.uint8, device=DEV)
    f, ts = getattr(torq, f"torq_{fmt}_{'gated_' if gated else ''}matvec"), (1.0,) if fmt == "nvfp4" else ()
    return f(X, codes, tile(lin, 0xFF), *ts, out_dtype=torch.float32)


def check(Y, x, v, gated):
    if not gated:
        assert torch.equal(Y.double(), x @ v.t())
        return
    N = v.shape[0] // 2
    g, u = x @ v[:N].t(), x @ v[N:].t()
    ref = silu(g) * u
    # exp 2^-22, its correction with the addition of 1/2, the constant and the product 2^-22, the quotient 2^-23, the sum and two products
    # 2^-24 each; gates below -87.3 count as zero
    tol = 2.0 ** -20 * ref.abs() + (g < -87.3) * 2.0 ** -119 * u.abs() + 2.0 ** -149
    assert ((Y.double() - ref).abs() <= tol).all()
    assert (silu(g).abs() > 2.0 ** -10).double().mean() > 0.3      # most are not at the flat end


SIZES = [(1, 128, 128), (2, 64, 65536), (3, 136, 65408), (4, 1000, 5120), (7, 128, 40832), (12, 256, 40960), (16, 200, 14336), (20, 128, 28672), (40, 256, 57344),
         (17, 13320, 1408), (33, 6920, 2432), (100, 4096, 5120), (257, 2048, 14464)]
GATED = [(1, 128, 128), (2, 128, 65536), (3, 128, 65408), (5, 256, 40832), (8, 384, 14336), (12, 128, 40960), (40, 128, 57344), (9, 19072, 1408), (17, 3840, 5120),
         (100, 1024, 14464)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M,N,K,gated", [(*s, False) for s in SIZES] + [(*s, True) for s in GATED])
def test_integers(fmt, M, N, K, gated):
    """x of whole numbers up to 8, every code: a stage of K that is left out, taken twice or read elsewhere shows in every sum.  Every block
    has an 8, so the first digit counts 8 and the second 1, up to 4 of them: sums below 65536 * 8 * 8 = 2^22 in units of 4 (codes come in
    halves) and below 65536 * 4 * 8 = 2^21 in units of 1/2, together below 2^23 in units of 1/2."""
    g = gen(M + N + K)
    codes = torch.randint(0, 256, (2 * N if gated else N, K // 2), generator=g, device=DEV, dtype=torch.uint8)
    X = torch.randint(-8, 9, (M, K), generator=g, device=DEV).to(torch.bfloat16)
    X[:, ::32], X[:, 16::32] = 8, -8
    power = -max(0, (K // 64).bit_length() // 2 + 5) if gated and fmt != "nvfp4" else (-5 if gated else 0)
    if fmt == "nvfp4" and gated:                         # scales reach no further down: fewer codes
        codes &= 0x99
    Y = product(fmt, X, codes, power, gated)
    check(Y, X.double(), code_values(codes, fmt) * 2.0 ** power, gated)
    assert torq.torq_last_device_error() == 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M,N,gated", [(1, 64, False), (3, 128, False), (8, 1000, False), (40, 64, False), (17, 13320, False), (100, 4096, False),
                                       (2, 128, True), (6, 256, True), (40, 128, True), (9, 19072, True), (17, 3840, True), (100, 1024, True)])
def test_the_last_digits(fmt, M, N, gated):
    """Every block has an element of 2^12 that meets codes of zero, beside elements of all 8 bits from 2^-2 to 2^4: their bits lie in the digits
    that count 2^6 ... 2^-9, down to 2^-21 of the largest.  Eight such elements a token: sums of digits below 3 * 8 * 16 * 8 < 2^12 in units of
    2^-10."""
    g, K, block = gen(M + N), 256, BLOCK[fmt]
    codes = torch.randint(0, 256, (2 * N if gated else N, K // 2), generator=g, device=DEV, dtype=torch.uint8)
    codes[:, ::block // 2] &= 0xF0                       # the first of each block
    X = torch.zeros(M, K, device=DEV)
    for m in range(M):
        at = torch.randperm(K, generator=g, device=DEV)[:8]
        X[m, at] = (torch.randint(128, 256, (8,), generator=g, device=DEV) * torch.exp2(torch.randint(-9, -3, (8,), generator=g, device=DEV).float())
                    * (1 - 2 * torch.randint(0, 2, (8,), generator=g, device=DEV)))
    X[:, ::block] = 2.0 ** 12
    X = X.to(torch.bfloat16)
    power = -3 if gated else 0
    Y = product(fmt, X, codes, power, gated)
    v = code_values(codes, fmt) * 2.0 ** power
    assert not v[:, ::block].any()
    check(Y, X.double(), v, gated)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("gated", [False, True])
def test_every_code_and_position_in_the_pair_gemm(fmt, gated):
    """One element of x at a time, 256 tokens: enough tiles for the GEMM on CTA pairs."""
    K, N = 256, 2048
    codes = (torch.arange(2 * N if gated else N, device=DEV) % 16 * 0x11).to(torch.uint8)
    if gated:
        codes[N:] = torch.randint(0, 16, (N,), generator=gen(0), device=DEV).to(torch.uint8) * 0x11
    codes = codes[:, None].expand(-1, K // 2).contiguous()
    X = torch.eye(K, dtype=torch.bfloat16, device=DEV)
    check(product(fmt, X, codes, 0, gated), X.double(), code_values(codes, fmt), gated)


@pytest.mark.parametrize("M", [1, 3, 8, 20])
def test_mxint4_takes_magnitudes_below_two_to_the_126(M):
    N, K = 128, 256
    codes = (torch.arange(N, device=DEV) % 16 * 0x11).to(torch.uint8)[:, None].expand(-1, K // 2).contiguous()
    X = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
    X[:, 5] = 1.9921875 * 2.0 ** 125
    X[:, 40] = -1.5
    v = code_values(codes, "mxint4") * 2.0 ** -60
    Y = product("mxint4", X, codes, -60, False)
    assert torch.equal(Y, (X.double() @ v.t()).float())
    X[M - 1, 5] = 2.0 ** 126                             # its scale for the upper halves has no byte
    Z = product("mxint4", X, codes, -60, False)
    assert Z[M - 1].isnan().all() and torch.equal(Z[:M - 1], Y[:M - 1])
