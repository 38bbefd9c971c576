"""Workloads of the operators around the 4-bit linear layer of a transformer block: the norm before it with its 8-bit
output, products of few tokens with 4-bit weights, and the gated pair of projections.

One case is one call as a serving program makes it.  The weights are laid out once per layer (packed 4-bit codes, or the
MXINT4 operand bytes, with their block scales in the library's tiled layout); the activations change from call to call.

  norm           h = x + r;  y = h / sqrt(mean(h^2) + eps) * w;  h and y out, y in bfloat16 or as MXFP8 (E4M3 bytes with one
                 E8M0 scale per 32 elements, the form the MXINT4 product takes on its activation side)
  matvec         y = x W^T with W in MXFP4, NVFP4 or MXINT4 and x in bfloat16
  gated_matvec   silu(x Wg^T) * (x Wu^T), both projections stacked in one W [2 N, K], x in bfloat16
  gated_gemm     the same with x quantized: MXFP4, NVFP4, or MXFP8 against MXINT4 weights ("w4a8")
"""
import math

import torch

own = False

_EPS = 1e-6
_MAX_COST = 8192 * 5120 * 51200                  # multiply-adds of the largest listed case
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _norm(M, d, x, residual, out):
    return {"op": "norm", "M": M, "d": d, "x": x, "residual": residual, "out": out}


def _product(op, fmt, M, K, N, out="bf16"):
    return {"op": op, "fmt": fmt, "M": M, "K": K, "N": N, "out": out}


def listed():
    return [
        # the norm in front of the projections of one token: latency only
        dict(_norm(1, 5120, "bf16", "bf16", "bf16"), name="norm_decode_1"),
        # a ragged prompt with a float32 residual stream, 8-bit output for the quantized projections
        dict(_norm(777, 4096, "f32", "f32", "mxfp8"), name="norm_prompt_777_mxfp8"),
        # long prefill, everything in bfloat16, 8-bit output: memory bandwidth
        dict(_norm(8192, 5120, "bf16", "bf16", "mxfp8"), name="norm_prefill_mxfp8"),
        # the smallest layer of the test suite: launch and latency
        dict(_product("matvec", "mxfp4", 1, 256, 256, "f32"), name="matvec_tiny"),
        # one sequence being decoded: the weights are streamed once for a single token
        dict(_product("matvec", "mxfp4", 1, 5120, 5120), name="matvec_1_mxfp4"),
        # a small decode batch through the longest contraction
        dict(_product("matvec", "nvfp4", 8, 14336, 4096), name="matvec_8_nvfp4_down"),
        # an odd batch, integer weights in their stored form, float32 result
        dict(_product("matvec", "mxint4", 13, 4096, 6144, "f32"), name="matvec_13_mxint4"),
        # gate and up projections of one token on the largest layer
        dict(_product("gated_matvec", "mxfp4", 1, 5120, 25600), name="gated_1_mxfp4"),
        # the same for a few sequences in NVFP4
        dict(_product("gated_matvec", "nvfp4", 5, 4096, 14336), name="gated_5_nvfp4"),
        # a ragged prompt: 8-bit activations against integer weights
        dict(_product("gated_gemm", "w4a8", 777, 4096, 14336), name="gated_prompt_777_w4a8"),
        # ragged prefill in NVFP4
        dict(_product("gated_gemm", "nvfp4", 1900, 4096, 14336), name="gated_prefill_nvfp4"),
        # long prefill through the largest gate and up projections
        dict(_product("gated_gemm", "mxfp4", 8192, 5120, 25600), name="gated_prefill_mxfp4"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more call: any sizes between the smallest and the largest ones, 1 to 8192 tokens (products of few tokens: 64)."""
    op = rng.choice(["norm", "matvec", "matvec", "gated_matvec", "gated_gemm"])
    out = "f32" if rng.random() < 0.3 else "bf16"
    if op == "norm":
        d = 32 * max(1, _log_int(rng, 32, 16384) // 32)
        M = _log_int(rng, 1, min(8192, 8192 * 8192 // d))
        return _norm(M, d, rng.choice(["bf16", "f32"]), rng.choice(["none", "bf16", "f32"]), rng.choice(["bf16", "mxfp8", "mxfp8"]))
    K = 128 * max(1, _log_int(rng, 128, 14336) // 128)
    if op == "matvec":
        return _product(op, rng.choice(["mxfp4", "nvfp4", "mxint4"]), _log_int(rng, 1, 64), K, 8 * _log_int(rng, 1, 6400), out)
    N = 128 * max(1, _log_int(rng, 128, 25600) // 128)
    if op == "gated_matvec":
        return _product(op, rng.choice(["mxfp4", "nvfp4", "mxint4"]), _log_int(rng, 1, 64), K, N, out)
    M = _log_int(rng, 1, min(8192, max(1, _MAX_COST // (2 * N * K))))
    return _product(op, rng.choice(["mxfp4", "nvfp4", "w4a8"]), M, K, N, out)


# ---- inputs ---------------------------------------------------------------------------------------------------
def _gaussian(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _activations(g, M, d):
    """Heavy tails (Student t, 3 degrees of freedom) and a few channels that are far larger than the others."""
    x = _gaussian(g, M, d) / _gaussian(g, 3, M, d).square_().mean(0).sqrt_()
    x[:, torch.randperm(d, generator=g, device="cuda")[:max(1, d // 1024)]] *= 50.0
    return x


def _tile_scales(s):
    """[rows, blocks] bytes -> 512-byte tiles of 128 rows x 4 blocks, padding zero."""
    rows, blocks = s.shape
    rt, bt = -(-rows // 128), -(-blocks // 4)
    p = torch.zeros(rt * 128, bt * 4, dtype=torch.uint8, device=s.device)
    p[:rows, :blocks] = s
    return p.view(rt, 4, 32, bt, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _e8m0_of(amax, below):
    """floor(log2 amax) - below as a byte with bias 127, read from the float32 exponent."""
    return (((amax.view(torch.int32) >> 23) & 255) - below).clamp_(min=0)


def _quantize(v, fmt, tensor_scale):
    """v [rows, k] float32 -> (codes, plain scale bytes) of one format."""
    rows, k = v.shape
    b = v.view(rows, -1, 16 if fmt == "nvfp4" else 32)
    amax = b.abs().amax(-1)
    if fmt == "nvfp4":
        sf = (amax / (6.0 * tensor_scale)).clamp_(max=448.0).to(torch.float8_e4m3fn)
        q = (b / (sf.float() * tensor_scale).clamp_(min=1e-30).unsqueeze(-1)).reshape(rows, k)
        sf = sf.view(torch.uint8)
    else:
        e = _e8m0_of(amax, 8 if fmt == "mxfp8" else 2)
        q = torch.ldexp(b, (127 - e).unsqueeze(-1)).reshape(rows, k)
        sf = e.to(torch.uint8)
    if fmt == "mxfp8":
        return q.clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8), sf
    if fmt == "mxint4":
        n = q.round().clamp_(-7.0, 7.0).to(torch.int32)
        n = n & 15
    else:
        edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=v.device)
        n = torch.bucketize(q.abs(), edges, out_int32=True) + (q < 0).to(torch.int32) * 8
    return (n[:, ::2] | (n[:, 1::2] << 4)).to(torch.uint8), sf


def _int4_operand(packed):
    """Stored nibbles -> the E4M3 bytes of the same integers."""
    return _decode(packed, "mxint4").to(torch.float8_e4m3fn).view(torch.uint8)


def _weights(g, rows, k, fmt):
    """Gaussian weights of rows x k, quantized: (codes, tiled scales, tensor scale)."""
    tensor_scale = 0.02 * 5.5 / (6 * 448) if fmt == "nvfp4" else 1.0
    codes, scales = _quantize(_gaussian(g, rows, k) * 0.02, fmt, tensor_scale)
    return codes, _tile_scales(scales), tensor_scale


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    if case["op"] == "norm":
        types = {"bf16": torch.bfloat16, "f32": torch.float32}
        s["X"] = _activations(g, case["M"], case["d"]).to(types[case["x"]])
        s["R"] = None if case["residual"] == "none" else (4 * _activations(g, case["M"], case["d"])).to(types[case["residual"]])
        s["weight"] = (1 + 0.3 * _gaussian(g, case["d"])).to(torch.bfloat16)
        return s
    M, K, N = case["M"], case["K"], case["N"]
    s["out_dtype"] = torch.float32 if case["out"] == "f32" else torch.bfloat16
    rows = N if case["op"] == "matvec" else 2 * N
    w_fmt = "mxint4" if case["fmt"] == "w4a8" else case["fmt"]
    s["Wq"], s["Ws"], s["w_scale"] = _weights(g, rows, K, w_fmt)
    x = _activations(g, M, K)
    if case["op"] != "gated_gemm":
        s["X"] = x.to(torch.bfloat16)
        return s
    if case["fmt"] == "w4a8":
        s["Wq"] = _int4_operand(s["Wq"])
    s["x_scale"] = 400.0 / (6 * 448) if case["fmt"] == "nvfp4" else 1.0       # calibrated ahead of time
    s["Aq"], sa = _quantize(x, "mxfp8" if case["fmt"] == "w4a8" else case["fmt"], s["x_scale"])
    s["As"] = _tile_scales(sa)
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------
def _decode(codes, fmt):
    """Packed codes -> float32 values without their scales."""
    if fmt in ("mxfp8", "e4m3"):
        return codes.view(torch.float8_e4m3fn).float()
    n = torch.stack((codes & 15, codes >> 4), dim=-1).view(codes.shape[0], -1)
    if fmt == "mxint4":
        return ((n ^ 8).to(torch.int8) - 8).float()
    table = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=codes.device)
    return table[n.int()]


def _dequantize(codes, tiled, fmt, tensor_scale):
    v = _decode(codes, fmt)
    rows, k = v.shape
    block = 16 if fmt == "nvfp4" else 32
    bt = -(-(k // block) // 4)
    s = tiled.view(-1, bt, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, bt * 4)[:rows, :k // block]
    if fmt == "nvfp4":
        s = s.view(torch.uint8).contiguous().view(torch.float8_e4m3fn).float() * tensor_scale
        return (v.view(rows, -1, block) * s.unsqueeze(-1)).view(rows, k)
    return torch.ldexp(v.view(rows, -1, block), s.int().unsqueeze(-1) - 127).view(rows, k)


def _plain_norm(s):
    h = s["X"].float()
    if s["R"] is not None:
        h = h + s["R"].float()
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + _EPS) * s["weight"].float()
    if s["out"] == "bf16":
        out = (y.to(torch.bfloat16),)
    else:
        codes, sf = _quantize(y, "mxfp8", 1.0)
        out = (codes.view(torch.float8_e4m3fn), _tile_scales(sf).view(torch.float8_e8m0fnu))
    return out if s["R"] is None else out + (h.to(s["R"].dtype),)


def _silu_product(gate, up):
    return gate / (1 + torch.exp(-gate)) * up


def _plain_product(s):
    w_fmt = {"w4a8": "e4m3"}.get(s["fmt"], s["fmt"])
    W = _dequantize(s["Wq"], s["Ws"], w_fmt, s["w_scale"])
    if s["op"] == "gated_gemm":
        x = _dequantize(s["Aq"], s["As"], w_fmt, s["x_scale"])
    else:
        x = s["X"].float()
    y = x @ W.t()
    if s["op"] != "matvec":
        y = _silu_product(y[:, :s["N"]], y[:, s["N"]:])
    return y.to(s["out_dtype"])


def run(s):
    if not own:
        return _plain_norm(s) if s["op"] == "norm" else _plain_product(s)
    from paper_2605_19561_b200 import torq
    if s["op"] == "norm":
        if s["out"] == "bf16":
            out = torq.torq_add_rmsnorm(s["X"], s["weight"], s["R"], _EPS)
            return (out,) if s["R"] is None else out
        codes, scales, *h = torq.torq_add_rmsnorm_mxfp8(s["X"], s["weight"], s["R"], _EPS)
        return (codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu), *h)
    if s["op"] == "matvec":
        if s["fmt"] == "mxfp4":
            return torq.torq_mxfp4_matvec(s["X"], s["Wq"], s["Ws"], s["out_dtype"])
        if s["fmt"] == "nvfp4":
            return torq.torq_nvfp4_matvec(s["X"], s["Wq"], s["Ws"], s["w_scale"], s["out_dtype"])
        return torq.torq_mxint4_matvec(s["X"], s["Wq"], s["Ws"], s["out_dtype"])
    if s["op"] == "gated_matvec":
        if s["fmt"] == "mxfp4":
            return torq.torq_mxfp4_gated_matvec(s["X"], s["Wq"], s["Ws"], s["out_dtype"])
        if s["fmt"] == "nvfp4":
            return torq.torq_nvfp4_gated_matvec(s["X"], s["Wq"], s["Ws"], s["w_scale"], s["out_dtype"])
        return torq.torq_mxint4_gated_matvec(s["X"], s["Wq"], s["Ws"], s["out_dtype"])
    if s["fmt"] == "mxfp4":
        return torq.torq_mxfp4_gated_gemm(s["Aq"], s["As"], s["Wq"], s["Ws"], s["out_dtype"])
    if s["fmt"] == "nvfp4":
        return torq.torq_nvfp4_gated_gemm(s["Aq"], s["As"], s["x_scale"], s["Wq"], s["Ws"], s["w_scale"], s["out_dtype"])
    return torq.torq_mxint4_gated_gemm(s["Aq"], s["As"], s["Wq"], s["Ws"], s["out_dtype"])


def work(case):
    size = {"none": 0, "bf16": 2, "f32": 4}
    if case["op"] == "norm":
        M, d = case["M"], case["d"]
        out = 2 * M * d if case["out"] == "bf16" else M * d + M * d // 32
        return {"bytes": M * d * (size[case["x"]] + 2 * size[case["residual"]]) + 2 * d + out, "flops": 5 * M * d}
    M, K, N = case["M"], case["K"], case["N"]
    rows = N if case["op"] == "matvec" else 2 * N
    block = 16 if case["fmt"] == "nvfp4" else 32
    w_bytes = rows * K // (1 if case["fmt"] == "w4a8" else 2) + rows * K // block
    if case["op"] == "gated_gemm":
        x_bytes = M * K // (1 if case["fmt"] == "w4a8" else 2) + M * K // block
    else:
        x_bytes = 2 * M * K
    return {"bytes": w_bytes + x_bytes + M * N * size[case["out"]], "flops": 2 * M * rows * K}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------
def _e2m1_number(n):
    """sign, two exponent bits (bias 1), one mantissa bit."""
    e, m = (n >> 1) & 3, (n & 1).double()
    v = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * torch.exp2((e - 1).double()))
    return torch.where(n >= 8, -v, v)


def _e4m3_number(b):
    """sign, four exponent bits (bias 7), three mantissa bits."""
    b = b.long()
    e, m = (b >> 3) & 15, (b & 7).double()
    v = torch.where(e == 0, m / 512, (1 + m / 8) * torch.exp2((e - 7).double()))
    return torch.where(b >= 128, -v, v)


def _numbers(codes, tiled, fmt, tensor_scale, first, rows):
    """Rows first .. first + rows of a quantized matrix in float64; scale bytes found by their address."""
    c = codes[first:first + rows].long()
    if fmt in ("mxfp8", "e4m3"):
        v = _e4m3_number(c)
    else:
        n = torch.empty(c.shape[0], 2 * c.shape[1], dtype=torch.long, device=c.device)
        n[:, 0::2], n[:, 1::2] = c % 16, c // 16
        v = torch.where(n > 7, n - 16, n).double() if fmt == "mxint4" else _e2m1_number(n)
    k = v.shape[1]
    block = 16 if fmt == "nvfp4" else 32
    row = torch.arange(first, first + v.shape[0], device=c.device).unsqueeze(1)
    blk = torch.arange(k // block, device=c.device).unsqueeze(0)
    per_row = -(-(k // block) // 4)
    byte = tiled[(row // 128 * per_row + blk // 4) * 512 + row % 32 * 16 + row % 128 // 32 * 4 + blk % 4].long()
    scale = _e4m3_number(byte) * tensor_scale if fmt == "nvfp4" else torch.exp2((byte - 127).double())
    return v * scale.repeat_interleave(block, dim=1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        h = s["X"].double() + (0 if s["R"] is None else s["R"].double())
        y = h / torch.sqrt((h * h).sum(-1, keepdim=True) / case["d"] + _EPS) * s["weight"].double()
        out = (y,)
        if case["out"] == "mxfp8":
            b = y.view(case["M"], -1, 32)
            top = b.abs().amax(-1)
            e = torch.where(top > 0, torch.frexp(top)[1].double() - 9, -127.0).clamp_(min=-127.0)
            q = b * torch.exp2(-e).unsqueeze(-1)
            unit = torch.exp2((torch.frexp(q.abs())[1].double() - 1).clamp_(min=-6.0) - 3)
            q = (torch.round(q / unit) * unit).clamp_(-448.0, 448.0)
            blocks = case["d"] // 32
            scales = torch.full((-(-case["M"] // 128) * -(-blocks // 4) * 512,), 2.0 ** -127, dtype=torch.float64, device="cuda")
            row = torch.arange(case["M"], device="cuda").unsqueeze(1)
            blk = torch.arange(blocks, device="cuda").unsqueeze(0)
            scales[(row // 128 * -(-blocks // 4) + blk // 4) * 512 + row % 32 * 16 + row % 128 // 32 * 4 + blk % 4] = torch.exp2(e)
            out = (q.view_as(y), scales)
        return out if s["R"] is None else out + (h,)
    w_fmt = {"w4a8": "e4m3"}.get(case["fmt"], case["fmt"])
    if case["op"] == "gated_gemm":
        x = _numbers(s["Aq"], s["As"], w_fmt, s["x_scale"], 0, case["M"])
    else:
        x = s["X"].double()
    N, parts = case["N"], []
    for r in range(0, N, 4096):
        n = min(4096, N - r)
        y = x @ _numbers(s["Wq"], s["Ws"], w_fmt, s["w_scale"], r, n).t()
        if case["op"] != "matvec":
            up = x @ _numbers(s["Wq"], s["Ws"], w_fmt, s["w_scale"], N + r, n).t()
            y = y * torch.sigmoid(y) * up
        parts.append(y)
    return torch.cat(parts, dim=1)
