"""Workloads of the 4-bit key/value cache: keys and values quantized into its pages, attention that reads them, the weight
that attention gives to every cached token, and the eviction of the tokens that got the least.

One case is one call as a serving program makes it.  The cache lies in pages of some tokens that the sequences share through
a table; every sequence has a length of its own.  A call's query tokens are the last of their sequences, `starts` says
where each sequence's begin in the batch (absent: one token each).

A page of one head holds, for its tokens, the codes of the keys, their scale bytes, the codes of the values, their scale bytes.

  append      new keys and values (columns of the rows of a fused projection) quantized into their slots, and read back
  attention   softmax(cap(scale q k) + bias) v over the cached tokens that a query may see, and the logarithm of the sum:
              causal, optionally a window, a prefix seen by all, a first token of each query's document, scores capped by a
              tanh, a bias by distance
  weights     what each cached token got, summed over queries and the heads that share it, added to the account of the cache
  evict       the tokens with the largest accounts and the newest ones moved to other pages, in their order
"""
import math
import random

import torch

own = False

_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_MAX_CACHED = 8 * 131072 * 128                   # elements of the keys of the largest cache
_MAX_PRODUCTS = 2048 * 8192 * 32 * 128           # multiply-adds of the scores of the largest prompt, all of its pairs counted


def _case(op, fmt, batch, longest, kv_heads, group, dim, page, **more):
    c = {"op": op, "fmt": fmt, "batch": batch, "longest": longest, "kv_heads": kv_heads, "group": group, "dim": dim, "page": page,
         "new": 1, "ragged": batch > 1, "padded": False, "softcap": 0.0, "window": 0, "bias": False, "prefix": False,
         "documents": False, "keep": 0, "recent": 0}
    c.update(more)
    return c


def listed():
    return [
        # a decoding step writes the keys and values of one token of each sequence: latency only
        dict(_case("append", "mxfp4", 64, 4096, 8, 4, 128, 64), name="append_decode_64"),
        # the prompts of a few requests, ragged
        dict(_case("append", "nvfp4", 5, 4000, 8, 4, 128, 64, new=4000), name="append_prompts_nvfp4"),
        # one short sequence: launch and latency
        dict(_case("attention", "mxfp4", 1, 77, 2, 4, 64, 16), name="attention_decode_tiny"),
        # an ordinary decoding batch, ragged, one padded row
        dict(_case("attention", "mxfp4", 32, 8192, 8, 4, 128, 64, padded=True), name="attention_decode_32"),
        # one long document being read, all of the card on eight heads
        dict(_case("attention", "nvfp4", 1, 131072, 8, 8, 128, 128), name="attention_decode_long_nvfp4"),
        # wide heads with capped scores and a window, integers in the cache
        dict(_case("attention", "mxint4", 48, 6000, 4, 2, 256, 32, softcap=50.0, window=4096), name="attention_decode_capped_mxint4"),
        # five drafted tokens verified at once, bias by distance
        dict(_case("attention", "nvfp4", 16, 5000, 8, 4, 128, 64, new=5, bias=True), name="attention_drafts_nvfp4"),
        # a piece of a long prompt behind what is cached already
        dict(_case("attention", "mxfp4", 1, 8192, 8, 4, 128, 64, new=2048), name="attention_prompt_2048"),
        # the account of a decoding batch
        dict(_case("weights", "mxfp4", 32, 8192, 8, 4, 128, 64), name="weights_decode_32"),
        # the account that a prompt starts with: its last tokens look at all of it
        dict(_case("weights", "nvfp4", 3, 3000, 8, 4, 128, 64, new=48), name="weights_prompt_nvfp4"),
        # a batch over its budget by some hundred tokens
        dict(_case("evict", "mxfp4", 8, 4500, 8, 4, 128, 64, keep=4096, recent=256), name="evict_8_to_4096"),
        # half of one long document is dropped
        dict(_case("evict", "nvfp4", 1, 65000, 8, 8, 128, 128, keep=32768, recent=1024), name="evict_long_nvfp4"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """One more call: one to 64 sequences of one to 131072 tokens, one to 16 heads with one to 16 queries each."""
    op = rng.choice(["append", "attention", "attention", "attention", "weights", "evict"])
    fmt, dim, page = rng.choice(["mxfp4", "nvfp4", "mxint4"]), rng.choice([64, 128, 128, 256]), rng.choice([16, 32, 64, 128])
    kv_heads, group, batch = _log_int(rng, 1, 16), rng.choice([1, 2, 3, 4, 5, 7, 8, 16]), _log_int(rng, 1, 64)
    longest = _log_int(rng, 1, min(131072, _MAX_CACHED // (batch * kv_heads * dim)))
    c = _case(op, fmt, batch, longest, kv_heads, group, dim, page)
    if op == "append":
        c["new"] = rng.choice([1, 1, _log_int(rng, 1, longest)])
    elif op == "evict":
        c["keep"] = _log_int(rng, 1, longest)
        c["recent"] = rng.randint(0, c["keep"])
    else:
        most = min(longest, _MAX_PRODUCTS // (batch * longest * kv_heads * group * dim))
        c["new"] = rng.choice([1, 1, rng.randint(1, max(1, min(8, most))), _log_int(rng, 1, max(1, min(4096, most)))])
        c["padded"] = batch > 1 and rng.random() < 0.2
        c["softcap"] = rng.choice([0.0, 0.0, 30.0])
        c["window"] = rng.choice([0, 0, _log_int(rng, 1, longest)])
        c["bias"], c["prefix"] = rng.random() < 0.2, c["new"] > 1 and rng.random() < 0.3
        c["documents"] = c["new"] > 1 and rng.random() < 0.2
    return c


# ---- inputs ---------------------------------------------------------------------------------------------------
def _gaussian(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _lengths(case):
    """Lengths with the new tokens, and how many of them are new, the same for every seed: the first sequence is the longest, a
    padded one is empty."""
    r = random.Random(f"{case['batch']} {case['longest']} {case['new']}")
    r = [r.random() for _ in range(case["batch"])]
    lengths = [case["longest"] if i == 0 or not case["ragged"] else max(1, int(case["longest"] * (0.15 + 0.85 * x))) for i, x in enumerate(r)]
    if case["padded"]:
        lengths[-1] = 0
    new = [case["new"] if i == 0 or case["new"] < 9 else max(1, int(case["new"] * (0.3 + 0.7 * x))) for i, x in enumerate(r)]
    return lengths, new if case["new"] == 1 else [min(n, length) for n, length in zip(new, lengths)]


def _e4m3(b):
    return b.view(torch.float8_e4m3fn).float()


def _quantize(x, fmt, tensor_scale):
    """x [..., dim] -> (codes, two to a byte with the even one in the low nibble, and scale bytes), in 32 bits."""
    b = x.float().view(*x.shape[:-1], -1, 16 if fmt == "nvfp4" else 32)
    amax = b.abs().amax(-1)
    if fmt == "nvfp4":
        c = 1.0 / (6.0 * torch.tensor(tensor_scale, device=x.device))
        sf = (amax * c).clamp(max=448.0).to(torch.float8_e4m3fn).view(torch.uint8)
        q = b * torch.where(sf == 0, 0.0, 1.0 / (_e4m3(sf) * tensor_scale)).unsqueeze(-1)
    else:
        e = (((amax.view(torch.int32) >> 23) & 255) - 2).clamp_(min=0)
        sf, q = e.to(torch.uint8), torch.ldexp(b, (127 - e).unsqueeze(-1))
    q = q.reshape(x.shape)
    if fmt == "mxint4":
        n = q.round().clamp_(-7.0, 7.0).to(torch.int32) & 15
    else:
        a = q.abs()
        n = (a > 0.25).to(torch.int32)                     # a value in the middle goes to the even code
        for edge, even_above in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
            n += (a >= edge) if even_above else (a > edge)
        n += torch.signbit(q).to(torch.int32) * 8
    return (n[..., ::2] | (n[..., 1::2] << 4)).to(torch.uint8), sf


def _dequantize(codes, sf, fmt, tensor_scale):
    n = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2)
    if fmt == "mxint4":
        v = ((n ^ 8).to(torch.int8) - 8).float()
    else:
        v = torch.tensor(_E2M1 + tuple(-a for a in _E2M1), device=codes.device)[n.int()]
    v = v.view(*sf.shape, -1)
    if fmt == "nvfp4":
        return (v * (_e4m3(sf) * tensor_scale).unsqueeze(-1)).flatten(-2)
    return torch.ldexp(v, sf.int().unsqueeze(-1) - 127).flatten(-2)


def _page_parts(pages, fmt, dim):
    """The parts of pages [pages, kv_heads, bytes]: of the keys and of the values, codes [.., page, dim / 2] and scale bytes [.., page, blocks]."""
    code, sf = dim // 2, dim // (16 if fmt == "nvfp4" else 32)
    page = pages.shape[2] // (2 * (code + sf))
    parts, at = [], 0
    for n in (code, sf, code, sf):
        parts.append(pages[:, :, at:at + page * n].unflatten(2, (page, n)))
        at += page * n
    return parts


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    H, D, P, B, fmt = case["kv_heads"], case["dim"], case["page"], case["batch"], case["fmt"]
    s["lens"], s["news"] = _lengths(case)
    s["kept"] = [min(n, case["keep"]) for n in s["lens"]]
    counts, more = [-(-n // P) for n in s["lens"]], [-(-n // P) for n in s["kept"]]
    total = sum(counts) + sum(more) + 3
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    s["table"], s["new_table"] = _table(counts, order), _table(more, order[sum(counts):])
    s["lengths"] = torch.tensor(s["lens"], dtype=torch.int32, device="cuda")
    s["tokens"] = T = sum(s["news"])
    s["starts"] = None if case["new"] == 1 else _starts(s["news"])
    s["scales"] = (80.0 / (6 * 448), 5.0 / (6 * 448)) if fmt == "nvfp4" else ()              # calibrated ahead of time
    loud = torch.where(torch.rand(H, D, generator=g, device="cuda") < 0.02, 8.0, 1.0)        # a few channels of the keys
    heads = H * case["group"]
    if case["op"] == "append":
        rows = _gaussian(g, T, heads + 2 * H, D)
        rows[:, heads:heads + H] *= loud
        s["K"], s["V"] = rows.to(torch.bfloat16).split([heads, H, H], dim=1)[1:]
        s["pages"] = torch.zeros(total, H, 2 * P * (D // 2 + D // (16 if fmt == "nvfp4" else 32)), dtype=torch.uint8, device="cuda")
        return s
    K, V = (_gaussian(g, total, H, P, D) * loud.unsqueeze(1)).to(torch.bfloat16), _gaussian(g, total, H, P, D).to(torch.bfloat16)
    s["pages"] = torch.cat([x.flatten(2) for x in (*_quantize(K, fmt, _scale(s, 0)), *_quantize(V, fmt, _scale(s, 1)))], dim=2)
    if case["op"] == "evict":
        w = _gaussian(g, total, H, P).mul_(2.0).exp_()
        s["weights"] = torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.1, 0.0, w)    # and some that nobody looked at
        s["new_starts"], s["new_tokens"] = _starts(s["kept"]), sum(s["kept"])
        return s
    s["Q"] = (1.5 * _gaussian(g, T, heads, D) / (1.0 + 0.4 * loud.repeat_interleave(case["group"], 0))).to(torch.bfloat16)
    s["factor"] = D ** -0.5
    s["slopes"] = torch.exp2(-8.0 * torch.arange(1, heads + 1, device="cuda") / heads) if case["bias"] else None
    s["prefixes"] = (s["lengths"] // 3).to(torch.int32) if case["prefix"] else None
    s["first"] = None
    if case["documents"]:                                  # two documents: the later half of the new tokens starts another one
        seq, slot = _places(s)
        middle = s["lengths"][seq] - torch.tensor([n - n // 2 for n in s["news"]], device="cuda")[seq]
        s["first"] = torch.where(slot < middle, 0, middle).to(torch.int32)
    if case["op"] == "weights":
        s["weights"] = _gaussian(g, total, H, P).abs_()
        s["out"] = torch.zeros_like(s["weights"])
        s["lse"] = _unpadded(s, _scores(s).double().logsumexp(-1).float().permute(0, 3, 1, 2)).flatten(1)
    return s


def _table(counts, order):
    """A row of page numbers for each sequence, taken one after the other from `order`; zeros behind them."""
    c = torch.tensor(counts, device="cuda").unsqueeze(1)
    at = c.cumsum(0) - c + torch.arange(max(1, max(counts)), device="cuda")
    return torch.where(at < c.cumsum(0), order[at.clamp(max=order.numel() - 1)], 0).to(torch.int32)


def _starts(counts):
    return torch.tensor([0] + counts, device="cuda").cumsum(0).to(torch.int32)


def _scale(s, i):
    return s["scales"][i] if s["scales"] else 1.0


# ---- plain forms ----------------------------------------------------------------------------------------------
def _places(s, lengths=None, starts=None, tokens=None):
    """Of each new token its sequence and its place in that, in the order of the batch."""
    lengths = s["lengths"] if lengths is None else lengths
    starts = s["starts"] if starts is None else starts
    if starts is None:
        starts = torch.arange(s["batch"] + 1, device="cuda")
    i = torch.arange(s["tokens"] if tokens is None else tokens, device="cuda")
    seq = torch.bucketize(i, starts[1:], right=True)
    return seq, lengths[seq] - starts[seq + 1] + i


def _padded(s, x):
    """[tokens, ...] -> [batch, most new tokens of a sequence, ...], what is not there repeats some token."""
    starts = torch.arange(s["batch"] + 1, device="cuda") if s["starts"] is None else s["starts"]
    i = starts[:-1].unsqueeze(1) + torch.arange(max(s["news"]), device="cuda")
    return x[i.clamp(max=s["tokens"] - 1)]


def _unpadded(s, x):
    seq, slot = _places(s)
    first = s["lengths"] - (1 if s["starts"] is None else s["starts"].diff())
    return x[seq, slot - first[seq]]


def _cached(s, i):
    """The keys (0) or values (1) of all sequences, [batch, kv_heads, longest, dim] in 32 bits."""
    codes, sf = _page_parts(s["pages"], s["fmt"], s["dim"])[2 * i:2 * i + 2]
    codes, sf = (x[s["table"].long()].transpose(1, 2).flatten(2, 3)[:, :, :s["longest"]] for x in (codes, sf))
    return _dequantize(codes, sf, s["fmt"], _scale(s, i))


def _scores(s):
    """Scores of all queries with the tokens of their sequence, [batch, kv_heads, group, new, longest], -inf where a query may not look."""
    B, H, n = s["batch"], s["kv_heads"], max(s["news"])
    q = _padded(s, s["Q"]).float().view(B, n, H, s["group"], s["dim"]).permute(0, 2, 3, 1, 4)
    x = (q.flatten(2, 3) @ _cached(s, 0).transpose(2, 3)).view(B, H, s["group"], n, -1).mul_(s["factor"])
    if s["softcap"]:
        x = x.div_(s["softcap"]).tanh_().mul_(s["softcap"])
    j = torch.arange(s["longest"], device="cuda")
    p = _padded(s, _places(s)[1]).unsqueeze(2)
    if s["slopes"] is not None:
        x -= s["slopes"].view(H, -1, 1, 1) * (p - j).abs().view(B, 1, 1, n, -1)
    seen = j <= p if s["prefixes"] is None else (j <= p) | (j < s["prefixes"].view(B, 1, 1))
    if s["window"]:
        seen = seen & (j > p - s["window"])
    if s["first"] is not None:
        seen = seen & (j >= _padded(s, s["first"]).unsqueeze(2))
    seen = seen & (j < s["lengths"].view(B, 1, 1))
    return x.masked_fill_(~seen.view(B, 1, 1, n, -1), -math.inf)


def _plain_read(s, table, lengths, starts, tokens):
    seq, slot = _places(s, lengths, starts, tokens)
    page = table[seq, slot // s["page"]].long()
    parts = [x[page, :, slot % s["page"]] for x in _page_parts(s["pages"], s["fmt"], s["dim"])]
    return tuple(_dequantize(*parts[2 * i:2 * i + 2], s["fmt"], _scale(s, i)).to(torch.bfloat16) for i in (0, 1))


def _plain_append(s):
    seq, slot = _places(s)
    page = s["table"][seq, slot // s["page"]].long()
    new = (*_quantize(s["K"], s["fmt"], _scale(s, 0)), *_quantize(s["V"], s["fmt"], _scale(s, 1)))
    for part, x in zip(_page_parts(s["pages"], s["fmt"], s["dim"]), new):
        part[page, :, slot % s["page"]] = x
    return _plain_read(s, s["table"], s["lengths"], s["starts"], s["tokens"])


def _plain_attention(s):
    x = _scores(s)
    m = x.amax(-1, keepdim=True).clamp_(min=-1e30)
    x = x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x.flatten(2, 3) @ _cached(s, 1)).view(*x.shape[:4], -1) / total.clamp(min=1e-30)
    lse = (m + total.log()).squeeze(-1)
    return _unpadded(s, o.permute(0, 3, 1, 2, 4)).flatten(1, 2).to(torch.bfloat16), _unpadded(s, lse.permute(0, 3, 1, 2)).flatten(1)


def _plain_weights(s):
    B, j = s["batch"], torch.arange(s["longest"], device="cuda")
    new = 1 if s["starts"] is None else s["starts"].diff().view(B, 1, 1)
    lse = _padded(s, s["lse"]).view(B, -1, s["kv_heads"], s["group"]).permute(0, 2, 3, 1).unsqueeze(-1)
    there = (lse > -math.inf) & (torch.arange(max(s["news"]), device="cuda").unsqueeze(1) < torch.as_tensor(new, device="cuda").view(-1, 1, 1, 1, 1))
    w = torch.where(there, (_scores(s) - lse).exp_(), 0.0).sum((2, 3))
    lengths = s["lengths"].view(B, 1, 1)
    old = s["weights"][s["table"].long()].transpose(1, 2).flatten(2, 3)[:, :, :s["longest"]]
    w += torch.where(j < lengths - new, old, 0.0)
    out = torch.zeros_like(s["weights"])
    seq, slot = (j < lengths.squeeze(1)).nonzero(as_tuple=True)
    out[s["table"][seq, slot // s["page"]].long(), :, slot % s["page"]] = w[seq, :, slot]
    return out


def _plain_evict(s):
    B, H, P, keep = s["batch"], s["kv_heads"], s["page"], s["keep"]
    lengths = s["lengths"].clamp(max=keep)
    n, old, j = lengths.view(B, 1, 1), s["lengths"].view(B, 1, 1), torch.arange(s["longest"], device="cuda")
    w = s["weights"][s["table"].long()].transpose(1, 2).flatten(2, 3)[:, :, :s["longest"]]
    w = torch.where(j >= old - n.clamp(max=s["recent"]), math.inf, w).masked_fill_(j >= old, -math.inf)
    order = torch.sort(w, dim=2, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(2, order, j.expand_as(order))
    src = torch.where(rank < n, j, s["longest"]).sort(dim=2).values[:, :, :keep]
    to = torch.arange(src.shape[2], device="cuda")
    kept = torch.full((B, H, keep), -1, dtype=torch.int32, device="cuda")
    kept[:, :, :src.shape[2]] = torch.where(to < n, src, -1)
    b, h, to = (to < n).expand_as(src).nonzero(as_tuple=True)
    src = src[b, h, to]
    from_page, to_page = s["table"][b, src // P].long(), s["new_table"][b, to // P].long()
    for part in (*_page_parts(s["pages"], s["fmt"], s["dim"]), s["weights"]):
        part[to_page, h, to % P] = part[from_page, h, src % P]
    return (lengths, kept, s["weights"]) + _plain_read(s, s["new_table"], lengths, s["new_starts"], s["new_tokens"])


def run(s):
    if not own:
        return {"append": _plain_append, "attention": _plain_attention, "weights": _plain_weights, "evict": _plain_evict}[s["op"]](s)
    from paper_2605_19561_b200 import torq
    call = lambda name: getattr(torq, f"torq_{s['fmt']}_kv_{name}")
    if s["op"] == "append":
        call("append")(s["pages"], s["table"], s["lengths"], s["K"], s["V"], *s["scales"], starts=s["starts"])
        return call("read")(s["pages"], s["table"], s["lengths"], s["dim"], s["tokens"], *s["scales"], starts=s["starts"])
    if s["op"] == "evict":
        lengths, kept = call("evict")(s["pages"], s["table"], s["lengths"], s["dim"], s["weights"], s["new_table"], s["keep"], s["recent"])
        return (lengths, kept, s["weights"]) + call("read")(
            s["pages"], s["new_table"], lengths, s["dim"], s["new_tokens"], *s["scales"], starts=s["new_starts"])
    options = {"starts": s["starts"], "scale": s["factor"], "softcap": s["softcap"], "slopes": s["slopes"], "window": s["window"],
               "prefix": s["prefixes"], "first": s["first"]}
    if s["op"] == "attention":
        return call("attention")(s["pages"], s["table"], s["lengths"], s["Q"], *s["scales"], return_lse=True, **options)
    return call("weights")(s["pages"], s["table"], s["lengths"], s["Q"], s["lse"], s["weights"], *s["scales"][:1], weights_out=s["out"], **options)


def work(case):
    H, D = case["kv_heads"], case["dim"]
    lens, new = _lengths(case)
    token = D // 2 + D // (16 if case["fmt"] == "nvfp4" else 32)         # bytes of a key or of a value in the cache
    queries, heads = sum(new), H * case["group"]
    if case["op"] == "append":
        return {"bytes": queries * H * (4 * D + 2 * token + 4 * D), "flops": 8 * queries * H * D}
    if case["op"] == "evict":
        moved = sum(min(n, case["keep"]) for n in lens)
        return {"bytes": H * (4 * sum(lens) + moved * (4 * token + 8 + 4 + 4 * D)), "flops": H * sum(lens)}
    pairs, cached = 0, 0                                   # of queries and tokens that they see; tokens that any query sees
    for n, length in zip(new, lens):
        window = case["window"] or length
        pairs += sum(min(window, length - n + i + 1) for i in range(n)) if length else 0
        cached += min(length, window + n - 1)
    if case["op"] == "attention":
        return {"bytes": 2 * cached * H * token + queries * heads * (4 * D + 4), "flops": 4 * pairs * heads * D}
    return {"bytes": cached * H * token + 2 * 4 * H * sum(lens) + queries * heads * (2 * D + 4), "flops": 2 * pairs * heads * D}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------
def _number(codes, sf, fmt, tensor_scale):
    """The values of codes [n, dim / 2] with scale bytes [n, blocks], from the bits."""
    n = torch.empty(codes.shape[0], 2 * codes.shape[1], dtype=torch.long, device=codes.device)
    n[:, 0::2], n[:, 1::2] = codes.long() % 16, codes.long() // 16
    if fmt == "mxint4":
        v = torch.where(n > 7, n - 16, n).double()
    else:
        e, m = (n >> 1) & 3, (n & 1).double()
        v = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * torch.exp2((e - 1).double()))
        v = torch.where(n > 7, -v, v)
    b = sf.long()
    if fmt == "nvfp4":
        e, m = (b >> 3) & 15, (b & 7).double()
        scale = torch.where(e == 0, m / 512, (1 + m / 8) * torch.exp2((e - 7).double())) * float(torch.tensor(tensor_scale))
    else:
        scale = torch.exp2((b - 127).double())
    return v * scale.repeat_interleave(v.shape[1] // b.shape[1], dim=1)


def _rounded(x, fmt, tensor_scale):
    """x [n, dim] in 64 bits to the nearest numbers of the format, halves to the even code."""
    b = x.view(x.shape[0], -1, 16 if fmt == "nvfp4" else 32)
    top = b.abs().amax(-1, keepdim=True)
    if fmt == "nvfp4":                                     # the format's definition rounds every step to 32 bits
        ts = float(torch.tensor(tensor_scale))
        f32 = lambda v: v.to(torch.float32).double()
        c = f32(1.0 / f32(torch.tensor(6.0 * ts, dtype=torch.float64, device=x.device)))
        t = f32(top * c).clamp(max=448.0)
        unit = torch.exp2((torch.frexp(t)[1].double() - 1).clamp(min=-6.0) - 3)
        e4m3 = torch.round(t / unit) * unit
        scale = e4m3 * ts
        q = f32(b * torch.where(e4m3 > 0, f32(1.0 / f32(scale)), 0.0))
    else:
        scale = torch.exp2(torch.where(top > 0, torch.frexp(top)[1].double() - 3, -127.0).clamp(min=-127.0))
        q = b / scale
    if fmt == "mxint4":
        q = torch.round(q).clamp(-7.0, 7.0)
    else:
        unit = torch.exp2((torch.frexp(q.abs())[1].double() - 1).clamp(0.0, 2.0) - 1)
        q = (torch.round(q / unit) * unit).clamp(-6.0, 6.0)
    return (q * scale).view_as(x)


def _gathered(s, part, b, h, slots, table="table"):
    return part[s[table][b].long()[slots // s["page"]], h, slots % s["page"]]


def _read_exact(s, b, h, slots):
    p = [_gathered(s, x, b, h, slots) for x in _page_parts(s["pages"], s["fmt"], s["dim"])]
    return _number(p[0], p[1], s["fmt"], _scale(s, 0)), _number(p[2], p[3], s["fmt"], _scale(s, 1))


def exact(case, seed):
    s = prepare(case, seed)
    H, G, D, fmt = case["kv_heads"], case["group"], case["dim"], case["fmt"]
    if case["op"] == "append":
        return tuple(_rounded(s[n].double().reshape(-1, D), fmt, _scale(s, i)).view(s[n].shape) for i, n in enumerate(("K", "V")))
    if case["op"] == "evict":
        kept = torch.full((case["batch"], H, case["keep"]), -1, dtype=torch.int64, device="cuda")
        weights, parts = s["weights"].double().clone(), ([], [])
        for b, (length, n) in enumerate(zip(s["lens"], s["kept"])):
            slots, rows = torch.arange(length, device="cuda"), ([], [])
            recent = min(case["recent"], n)
            for h in range(H):
                w = _gathered(s, s["weights"], b, h, slots).double()
                w[length - recent:] = math.inf
                # kept: how many come before a token, by weight and then by place, is less than the room
                rank = torch.empty_like(slots)
                rank[torch.sort(-w, stable=True).indices] = slots
                src = slots[rank < n]
                kept[b, h, :n] = src
                to = slots[:n]
                weights[s["new_table"][b].long()[to // s["page"]], h, to % s["page"]] = _gathered(s, s["weights"], b, h, src).double()
                for r, x in zip(rows, _read_exact(s, b, h, src)):
                    r.append(x)
            for p, r in zip(parts, rows):
                p.append(torch.stack(r, dim=1))
        return (torch.tensor(s["kept"], device="cuda"), kept, weights, torch.cat(parts[0]), torch.cat(parts[1]))
    if sum(n * length for n, length in zip(s["news"], s["lens"])) * H * G * D > _MAX_PRODUCTS:
        return None
    T = sum(s["news"])
    out = torch.zeros(T, H * G, D, dtype=torch.float64, device="cuda")
    lse = torch.full((T, H * G), -math.inf, dtype=torch.float64, device="cuda")
    account, at = torch.zeros(s["weights"].shape if case["op"] == "weights" else 0, dtype=torch.float64, device="cuda"), 0
    for b, (n, length) in enumerate(zip(s["news"], s["lens"])):
        slots = torch.arange(length, device="cuda")
        place = torch.arange(n, device="cuda").unsqueeze(1) + (length - n)
        low, high = torch.zeros_like(place), place.clone()
        if case["window"]:
            low = torch.maximum(low, place - case["window"] + 1)
        if s["first"] is not None:
            low = torch.maximum(low, s["first"][at:at + n].long().unsqueeze(1))
        if s["prefixes"] is not None:
            high = torch.maximum(high, s["prefixes"][b].long() - 1)
        hidden = (slots < low) | (slots > high)
        for h in range(H if n and length else 0):
            k, v = _read_exact(s, b, h, slots)
            total = torch.zeros(length, dtype=torch.float64, device="cuda")
            for q in range(h * G, h * G + G):
                x = s["Q"][at:at + n, q].double() @ k.t() * s["factor"]
                if case["softcap"]:
                    x = case["softcap"] * torch.tanh(x / case["softcap"])
                if s["slopes"] is not None:
                    x = x - float(s["slopes"][q]) * (place - slots).abs()
                x[hidden] = -math.inf
                if case["op"] == "weights":
                    y = s["lse"][at:at + n, q].double().unsqueeze(1)
                    total += torch.where(torch.isinf(y), 0.0, torch.exp(x - y)).sum(0)
                    continue
                y = torch.logsumexp(x, -1)
                lse[at:at + n, q] = y
                out[at:at + n, q] = torch.where(torch.isinf(y).unsqueeze(1), 0.0, torch.exp(x - y.unsqueeze(1))) @ v
            if case["op"] == "weights":
                old = _gathered(s, s["weights"], b, h, slots).double()
                account[s["table"][b].long()[slots // case["page"]], h, slots % case["page"]] = total + torch.where(slots < length - n, old, 0.0)
        at += n
    return account if case["op"] == "weights" else (out, lse)
