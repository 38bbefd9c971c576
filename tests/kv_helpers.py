"""What the tests of the 4-bit key/value cache share: a cache with random contents and the definition of its operators in 64 bits, one sequence
and head after the other."""
import math

import torch

from operator_helpers import DEV, code_values, gen, scale_values
from paper_2605_19561_b200 import torq

FMTS = ("mxfp4", "nvfp4", "mxint4")
TS = {"mxfp4": (), "nvfp4": (0.0125, 0.0031), "mxint4": ()}


def block(fmt):
    return 16 if fmt == "nvfp4" else 32


def parts(pages, fmt, dim):
    """key codes, key scale bytes, value codes, value scale bytes: views [pages, heads, page, bytes]."""
    code, sf = dim // 2, dim // block(fmt)
    page = pages.shape[2] // (2 * (code + sf))
    out, at = [], 0
    for n in (code, sf, code, sf):
        out.append(pages[:, :, at:at + page * n].unflatten(2, (page, n)))
        at += page * n
    return out


class Cache:
    """lens: tokens of each sequence; new: how many of them are new rows (None: starts is None).  What no sequence owns holds 0xFF (no numbers
    as scales), table entries behind a length are no pages."""

    def __init__(self, fmt, lens, heads, group, dim, page=16, new=None, seed=0, spread=4, width=0, low=124):
        g = gen(seed)
        self.fmt, self.lens, self.H, self.G, self.D, self.P = fmt, list(lens), heads, group, dim, page
        self.scales = TS[fmt]
        self.new = list(new) if new is not None else [1] * len(lens)
        counts = [-(-n // page) for n in lens]
        total = sum(counts) + 2
        order = torch.randperm(total, generator=g, device=DEV).tolist()
        self.table_rows, at = [], 0
        for n in counts:
            self.table_rows.append(order[at:at + n])
            at += n
        self.free = order[at:]
        self.width = max(1, width, max(counts))
        pad = [-1, 1 << 30, total, -(1 << 31)]
        self.table = torch.tensor([r + [pad[i % 4] for i in range(self.width - len(r))] for r in self.table_rows], dtype=torch.int32, device=DEV)
        self.lengths = torch.tensor(self.lens, dtype=torch.int32, device=DEV)
        self.starts = None if new is None else torch.tensor([sum(self.new[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=DEV)
        self.tokens = sum(self.new)
        self.pages = torch.full((total, heads, torq.torq_kv_page_bytes(fmt, page, dim)), 255, dtype=torch.uint8, device=DEV)
        self.K, self.V = [], []
        for b, n in enumerate(self.lens):
            kv = []
            for i in (0, 1):
                codes = torch.randint(0, 256, (n, heads, dim // 2), generator=g, device=DEV, dtype=torch.uint8)
                if fmt == "mxint4":                      # the quantizer gives no -8
                    codes = torch.where((codes & 15) == 8, codes ^ 8, codes)
                    codes = torch.where((codes >> 4) == 8, codes ^ 128, codes)
                if fmt == "nvfp4":
                    sf = torch.randint(48, 48 + 8 * spread, (n, heads, dim // 16), generator=g, device=DEV)
                else:
                    sf = low + torch.randint(0, spread, (n, heads, dim // 32), generator=g, device=DEV)
                sf = sf.to(torch.uint8)
                self.put(b, 2 * i, codes)
                self.put(b, 2 * i + 1, sf)
                kv.append(self.values(codes, sf, i))
            self.K.append(kv[0])
            self.V.append(kv[1])

    def values(self, codes, sf, i):
        """[n, heads, dim] in 64 bits."""
        n, heads = codes.shape[:2]
        if n == 0:
            return torch.zeros(0, heads, self.D, dtype=torch.float64, device=DEV)
        v = code_values(codes.reshape(n * heads, codes.shape[2]), self.fmt) * scale_values(sf.reshape(n * heads, sf.shape[2]), self.fmt).repeat_interleave(block(self.fmt), 1)
        ts = float(torch.tensor(self.scales[i], dtype=torch.float32)) if self.scales else 1.0
        return (v * ts).view(n, heads, self.D)

    def at(self, b, slots):
        return torch.tensor(self.table_rows[b], device=DEV, dtype=torch.long)[slots // self.P], slots % self.P

    def put(self, b, part, x):
        page, slot = self.at(b, torch.arange(x.shape[0], device=DEV))
        parts(self.pages, self.fmt, self.D)[part][page, :, slot] = x

    def rows(self, b):
        """Rows of sequence b in the batch and their places."""
        first = sum(self.new[:b])
        return first, torch.arange(self.new[b], device=DEV) + self.lens[b] - self.new[b]

    def call(self, name, *args, **kw):
        return getattr(torq, f"torq_{self.fmt}_kv_{name}")(self.pages, self.table, self.lengths, *args, starts=self.starts, **kw)


def queries(c, seed=1, size=1.0, spread=None):
    q = torch.randn(c.tokens, c.H * c.G, c.D, generator=gen(seed), device=DEV, dtype=torch.float64) * size
    return q.to(torch.bfloat16)


def scores(c, Q, b, scale=None, softcap=0.0, slopes=None, window=0, prefix=None, first=None):
    """x [heads, group, new, length] in 64 bits, -inf where a row does not see."""
    start, p = c.rows(b)
    q = Q[start:start + c.new[b]].double().view(c.new[b], c.H, c.G, c.D)
    x = torch.einsum("nhgd,lhd->hgnl", q, c.K[b]) * (c.D ** -0.5 if scale is None else float(torch.tensor(scale, dtype=torch.float32)))
    if softcap:
        x = softcap * torch.tanh(x / softcap)
    j, p = torch.arange(c.lens[b], device=DEV), p.unsqueeze(1)
    if slopes is not None:
        x = x - slopes.double().view(c.H, c.G, 1, 1) * (p - j).abs()
    high = p if prefix is None else torch.clamp(p, min=int(prefix[b]) - 1)
    seen = j <= high
    if window:
        seen = seen & (j > p - window)
    if first is not None:
        seen = seen & (j >= first[start:start + c.new[b]].unsqueeze(1))
    return torch.where(seen, x, -math.inf)


def attention(c, Q, **options):
    """(out, lse, sum of weight times |v|) in 64 bits."""
    heads = c.H * c.G
    out = torch.zeros(c.tokens, heads, c.D, dtype=torch.float64, device=DEV)
    mag, lse = torch.zeros_like(out), torch.full((c.tokens, heads), -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(c.new):
        if not n or not c.lens[b]:
            continue
        x = scores(c, Q, b, **options)
        y = torch.logsumexp(x, -1)
        w = torch.where(torch.isinf(y).unsqueeze(-1), 0.0, torch.exp(x - torch.where(torch.isinf(y), 0.0, y).unsqueeze(-1)))
        start, _ = c.rows(b)
        lse[start:start + n] = y.permute(2, 0, 1).reshape(n, heads)
        out[start:start + n] = torch.einsum("hgnl,lhd->nhgd", w, c.V[b]).reshape(n, heads, c.D)
        mag[start:start + n] = torch.einsum("hgnl,lhd->nhgd", w, c.V[b].abs()).reshape(n, heads, c.D)
    return out, lse, mag


def score_size(c, Q, scale=None):
    """The largest sum of magnitudes of the products of a score."""
    worst = 0.0
    for b, n in enumerate(c.new):
        if n and c.lens[b]:
            start, _ = c.rows(b)
            q = Q[start:start + n].double().abs().view(n, c.H, c.G, c.D)
            worst = max(worst, torch.einsum("nhgd,lhd->hgnl", q, c.K[b].abs()).max().item() * (c.D ** -0.5 if scale is None else scale))
    return worst


def check_attention(c, Q, out, lse, **options):
    """A score is a sum of up to 256 exact products in float32 (steps of at most 16 on the tensor cores, what is added in one aligned first, then
    one addition per block): off by at most 2^-20 of the magnitudes that it adds, its factors and the cap by 2^-21 more.  exp and the sums
    carry that over to every weight, 2 dx of it, and to the result; a weight is rounded to 11 bits (2^-11 with what exp2 is off by); the result
    to bfloat16.  A weight is held as a float16 in which the largest is 2^10 at least: its half step is 2^-25 at least, 2^-35 of the largest weight,
    which is at most 1.  (So where the large weights meet values of zero, the small ones, which alone make the result, are off by that.)"""
    ref, ref_lse, mag = attention(c, Q, **options)
    extra = 0.0
    if options.get("slopes") is not None:
        extra = float(options["slopes"].abs().max()) * max(c.lens) * 2.0 ** -22
    dx = 2.0 ** -19 * score_size(c, Q, options.get("scale")) + extra + 2.0 ** -20
    none = torch.isinf(ref_lse)
    assert torch.equal(torch.isinf(lse), none) and not torch.isnan(lse).any()
    assert (lse[none] < 0).all() and (out[none] == 0).all()
    err = torch.where(none, 0.0, (lse.double() - ref_lse).abs())
    tol = dx + 2.0 ** -22 * torch.where(none, 0.0, ref_lse.abs()) + 2.0 ** -20
    assert (err <= tol).all(), ((err / tol).max().item(), err.max().item())
    assert torch.isfinite(out).all()
    tol = (2 * dx + 2.0 ** -11) * mag + 2.0 ** -8 * ref.abs() + 1e-30
    for b, n in enumerate(c.new):
        start, _ = c.rows(b)
        tol[start:start + n] += 2.0 ** -35 * c.V[b].abs().sum(0).repeat_interleave(c.G, 0)
    worst = ((out.double() - ref).abs() / tol).max().item()
    assert worst <= 1.0, worst
