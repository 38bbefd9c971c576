"""What the tests of the operators around the layer share: random quantized operands with the values they stand for, in 64 bits."""
import torch

DEV = "cuda"
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # of a rounding, relative to the value
E2M1 = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def heavy(g, *shape):
    """Student t with 3 degrees of freedom."""
    x = torch.randn(*shape, generator=g, device=DEV, dtype=torch.float64)
    return x / torch.randn(3, *shape, generator=g, device=DEV, dtype=torch.float64).square().mean(0).sqrt()


def tile(lin, fill=0):
    """[rows, blocks] bytes -> the tiled layout; `fill` in the rows and blocks of the padding."""
    rows, nb = lin.shape
    rt, bt = -(-rows // 128), -(-nb // 4)
    p = torch.full((rt * 128, bt * 4), fill, dtype=torch.uint8, device=lin.device)
    p[:rows, :nb] = lin
    return p.view(rt, 4, 32, bt, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def untile(t, rows, nb):
    bt = -(-nb // 4)
    return t.view(-1, bt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, bt * 4)[:rows, :nb]


def e4m3(b):
    return b.view(torch.float8_e4m3fn).to(torch.float64)


def scale_values(lin, fmt):
    return e4m3(lin) if fmt == "nvfp4" else torch.exp2(lin.to(torch.float64) - 127)


def code_values(codes, fmt):
    """The elements without their scales: two codes to a byte, the even one in the low nibble; w4a8: E4M3 bytes."""
    if fmt == "w4a8":
        return e4m3(codes)
    n = torch.stack((codes & 15, codes >> 4), -1).view(codes.shape[0], -1).long()
    if fmt == "mxint4":
        return torch.where(n > 7, n - 16, n).to(torch.float64)
    return E2M1.to(codes.device)[n & 7] * torch.where(n > 7, -1.0, 1.0).to(torch.float64)


def values(codes, lin, fmt, ts=1.0):
    ts = float(torch.tensor(ts, dtype=torch.float32))
    return code_values(codes, fmt) * scale_values(lin, fmt).repeat_interleave(16 if fmt == "nvfp4" else 32, 1) * ts


def quantized(g, rows, K, fmt, spread=6, pad=0, low=118, ts=0.0123):
    """(codes, tiled scales, tensor scale, values): every code; E8M0 scales from `low` on over `spread` powers of two, or every
    E4M3 scale from zero and the subnormals to 448."""
    codes = torch.randint(0, 256, (rows, K if fmt == "w4a8" else K // 2), generator=g, device=DEV, dtype=torch.uint8)
    if fmt == "w4a8":
        codes[(codes & 0x7F) == 0x7F] = 0x3C             # not a number
    if fmt == "nvfp4":
        lin = torch.randint(0, 127, (rows, K // 16), generator=g, device=DEV, dtype=torch.uint8)
    else:
        lin, ts = (low + torch.randint(0, spread, (rows, K // 32), generator=g, device=DEV)).to(torch.uint8), 1.0
    return codes, tile(lin, pad), ts, values(codes, lin, fmt, ts)


# ---- the norm -----------------------------------------------------------------------------------------------------
# h is off by 2^-24 of itself, the sum of its squares by at most 42 roundings of 2^-24 (32 elements of a lane one after the
# other, then trees of 5 and 5), half of which comes into the root; mean, sum with eps, root, quotient and two products by one
# rounding each
NORM_REL = 40 * 2.0 ** -24


def norm_inputs(M, d, x_dtype, r_dtype, seed=0):
    g = gen(seed)
    x = heavy(g, M, d)
    x[:, 3::97] *= 50
    r = None if r_dtype is None else (3 * heavy(g, M, d)).to(r_dtype)
    return x.to(x_dtype), r, (1 + 0.4 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16)


def norm_ref(x, r, w, eps):
    h = x.double() + (0 if r is None else r.double())
    return h * torch.rsqrt(h.square().mean(-1, keepdim=True) + eps) * w.double()


def check_mxfp8(codes, scales, ref):
    """Scale bytes by the rule (one apart only where the largest magnitude lies at a power of two), codes within half a step,
    zeros in the padding."""
    M, d = ref.shape
    b = untile(scales, M, d // 32).double()
    blocks = ref.view(M, -1, 32)
    amax = blocks.abs().amax(-1)
    lo, hi = (torch.floor(torch.log2(amax * f)).clamp(min=-119) for f in (1 - NORM_REL, 1 + NORM_REL))
    zero = amax == 0
    assert ((b >= torch.where(zero, 0, lo + 119)) & (b <= torch.where(zero, 0, hi + 119))).all()
    v, q = blocks / torch.exp2(b - 127).unsqueeze(-1), e4m3(codes).view(M, -1, 32)
    half = torch.maximum(v.abs() * 2.0 ** -4, torch.tensor(2.0 ** -10, device=DEV, dtype=torch.float64))
    fine = (q - v).abs() <= half + NORM_REL * v.abs()
    assert (fine | ((v.abs() > 448) & (q == 448 * v.sign()))).all()
    p = untile(scales, -(-M // 128) * 128, -(-(d // 32) // 4) * 4).clone()
    p[:M, :d // 32] = 0
    assert not p.any()


# ---- products -----------------------------------------------------------------------------------------------------
def silu(v):
    return v * torch.sigmoid(v)


def check_sums(Y, x, w, steps, dx=None):
    """|Y - x w^T| <= steps 2^-22 sum |x| |w| + the rounding of the result.  Products are exact; `steps` additions in float32
    follow one another on the way of a product into the result, each off by at most 2^-23 of the largest partial sum if it
    truncates; the factor of two leaves room for the power of two that the largest partial sum may exceed the final one by.
    dx: what x itself is off by."""
    ref, mag = x @ w.t(), x.abs() @ w.abs().t()
    tol = steps * 2.0 ** -22 * mag + HALF_STEP[Y.dtype] * ref.abs() + 1e-40
    if dx is not None:
        tol += dx @ w.abs().t()
    assert torch.isfinite(Y).all()
    worst = ((Y.double() - ref).abs() / tol).max().item()
    assert worst <= 1.0, worst


def check_gated(Y, x, w, steps, dx=None):
    """The error of both sums as above, through silu(g) u (the derivative of silu is at most 1.1), exp and the quotient at 2^-21."""
    N = w.shape[0] // 2
    g, u = x @ w[:N].t(), x @ w[N:].t()
    e = steps * 2.0 ** -22
    dx = e * x.abs() + (0 if dx is None else dx)
    dg, du = dx @ w[:N].abs().t(), dx @ w[N:].abs().t()
    ref = silu(g) * u
    tol = 1.1 * dg * (u.abs() + du) + silu(g).abs() * du + ref.abs() * (HALF_STEP[Y.dtype] + 2.0 ** -21) + 1e-40
    assert torch.isfinite(Y).all()
    worst = ((Y.double() - ref).abs() / tol).max().item()
    assert worst <= 1.0, worst


def matvec_error(fmt, x):
    """(steps, dx) of the few-token products.  x is rounded to a multiple of 2^-21 of the power of two at or below its block's largest
    magnitude (NVFP4: a block's counts as 2^-17 of its token's at least); the magnitudes of a number's digits add up to at most
    three times its own (MXINT4: those of the two halves of a weight to three times its own as well); one instruction per 64 of K
    (MXINT4: two), what it adds aligned before it is added, then 8 digits and 8 CTAs."""
    M, K = x.shape
    block = 16 if fmt == "nvfp4" else 32
    top = x.abs().view(M, -1, block).amax(-1)
    if fmt == "nvfp4":
        top = torch.maximum(top, x.abs().amax(-1, keepdim=True) * 2.0 ** -16)
    dx = (top * 2.0 ** -22 + 2.0 ** -128).repeat_interleave(block, 1)
    return (9 * 2 * (K // 32 + 16) if fmt == "mxint4" else 3 * 2 * (K // 64 + 16)), dx


def gemm_steps(K):
    """Of the GEMMs: at most one instruction per 32 of K, twice because what is added inside one is aligned before it is added."""
    return 2 * (K // 32 + 8)
