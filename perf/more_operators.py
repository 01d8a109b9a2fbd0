"""Operators of a model's attention over paged 4-bit caches, as measurable
cases, each in a plain form of elementary torch operations (own = False) and
through the public calls of paper_2606_22768_amd (own = True):

  heads    queries and keys normed head by head and rotated by their
           positions (rotate_heads)
  grads    the same operator's gradients (rotate_heads_grads)
  cache    keys and values into a paged cache in microscaled 4-bit floating
           point, and their values back (mx4_cache_write, mx4_cache_read)
  attend   attention over such a cache (mx4_attend): one query per sequence,
           or several, causal, in a window or not
  pages    the cache's block tables and slot maps from the requests' lengths
           (extend_pages), and what was not kept given back (truncate_pages)

Heads: y = R(x / sqrt(mean(x^2) + eps) * w), R turning the pairs (i, i + n/2),
or (2 i, 2 i + 1) where they are interleaved, of the first n elements by
position * freqs[i]; without w there is no norm.

The 4-bit format: blocks of 32 consecutive elements of a head share the scale
2^e, e = floor(log2(largest magnitude)) - 2 held in [-127, 127]; an element
is x / 2^e rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the
even code, saturating at 6) with its sign.

Attention: query i of a sequence of L keys and n queries stands at position
L - n + i and sees the keys up to its own position (the last `window` of them
where window > 0); o = sum_j softmax_j(scale q.k_j) v_j, zero where it sees
none.

Pages: request after request takes the pages that its new tokens need from
the top of a stack of free ones, all or none of them; token at position p of
request b has slot table[b][p / page] * page + p % page.

Sizes: 1 to 8192 tokens, 1 to 64 heads of 32 to 256, caches of up to 65 536
keys a sequence, 1 to 1024 requests, up to four workers; powers of two as
layers have them, and odd ones.
"""

import math

import torch

own = False

BLOCK = 32
CODES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


def listed():
    return [
        # 64 sequences' next tokens in one layer: latency.
        dict(name="heads_t64_h32_8_d128_bf16", op="heads", M=1, T=64, HQ=32, HK=8, D=128, rot=128, interleaved=False,
             norm=True, dtype="bf16", far=32_768),
        # Four workers' training step, each with weights of its own.
        dict(name="heads_m4_t2048_h32_8_d128_bf16", op="heads", M=4, T=2048, HQ=32, HK=8, D=128, rot=128,
             interleaved=False, norm=True, dtype="bf16", far=2048),
        # The same step's gradients.
        dict(name="grads_m4_t2048_h32_8_d128_bf16", op="grads", M=4, T=2048, HQ=32, HK=8, D=128, rot=128,
             interleaved=False, norm=True, dtype="bf16", far=2048),
        # A ragged batch of a model that rotates part of a head, in float32.
        dict(name="grads_t777_h7_1_d96_f32_part", op="grads", M=1, T=777, HQ=7, HK=1, D=96, rot=64, interleaved=True,
             norm=True, dtype="f32", far=1_000_000),
        # 64 sequences' new keys and values, a token each, all over the cache.
        dict(name="cache_t64_h8_d128_bf16", op="cache", T=64, H=8, D=128, page=64, prompts=64, dtype="bf16"),
        # Five prompts' keys and values.
        dict(name="cache_t8191_h8_d128_bf16", op="cache", T=8191, H=8, D=128, page=64, prompts=5, dtype="bf16"),
        # One long sequence's next token: latency, and one pass over its cache.
        dict(name="attend_b1_len65536_h32_8_d128_bf16", op="attend", B=1, n=1, least=65_536, most=65_536, HQ=32, HK=8,
             D=128, page=64, window=0, dtype="bf16"),
        # 64 sequences of different lengths decoded together.
        dict(name="attend_b64_len8192_h32_8_d128_bf16", op="attend", B=64, n=1, least=500, most=8192, HQ=32, HK=8,
             D=128, page=64, window=0, dtype="bf16"),
        # Five drafted tokens verified for each of 17 sequences, one key head, a window.
        dict(name="attend_b17_n5_len3001_h8_1_d96_f32", op="attend", B=17, n=5, least=1, most=3001, HQ=8, HK=1, D=96,
             page=16, window=1000, dtype="f32"),
        # The largest: chunks of four long prompts.
        dict(name="attend_b4_n512_len8192_h32_8_d128_bf16", op="attend", B=4, n=512, least=4096, most=8192, HQ=32,
             HK=8, D=128, page=64, window=0, dtype="bf16"),
        # A decoding turn of 64 requests, one token each.
        dict(name="pages_b64_n1", op="pages", B=64, least=1, most=1, held=8192, page=64, short=0.0),
        # 513 requests with prompts and decoded tokens mixed, in a pool that cannot serve them all.
        dict(name="pages_b513_n256_short", op="pages", B=513, least=0, most=256, held=4096, page=16, short=0.2),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choices(("heads", "grads", "cache", "attend", "pages"), (3, 3, 2, 7, 2))[0]
    dtype = rng.choice(("f32", "bf16", "bf16"))
    D = rng.choice((32, 64, 64, 96, 128, 128, 128, 160, 192, 256))
    HK = rng.choice((1, 1, 2, 3, 4, 8, 8))
    HQ = HK * rng.choice((1, 2, 3, 4, 4, 7, 8))
    page = rng.choice((16, 32, 64, 128, 256))
    if op in ("heads", "grads"):
        M = rng.choice((1, 1, 2, 4))
        D = rng.choice((D, D, 40, 80, 512))
        T = _log_uniform(rng, 1, max(2, min(8192, 40_000_000 // ((HQ + HK) * D * M))))
        return dict(op=op, M=M, T=T, HQ=HQ, HK=HK, D=D, rot=rng.choice((D, D, D // 2, D // 4 // 2 * 2)),
                    interleaved=rng.random() < 0.3, norm=rng.random() < 0.8, dtype=dtype,
                    far=_log_uniform(rng, 64, 1_000_000))
    if op == "cache":
        T = _log_uniform(rng, 1, min(8192, 8_000_000 // (HK * D)))
        return dict(op=op, T=T, H=HK, D=D, page=page, prompts=_log_uniform(rng, 1, T), dtype=dtype)
    if op == "pages":
        most = _log_uniform(rng, 1, 512)
        B = _log_uniform(rng, 1, min(1024, 60_000 // most))
        return dict(op=op, B=B, least=rng.choice((0, 1)), most=most, held=_log_uniform(rng, 16, 16_384), page=page,
                    short=rng.choice((0.0, 0.0, 0.3)))
    n = rng.choice((1, 1, 1, 1, 2, 5, 8, _log_uniform(rng, 10, 600)))
    most = _log_uniform(rng, max(n, 16), 65_536)
    n = max(1, min(n, 35_000_000_000 // (most * HQ * D)))
    B = _log_uniform(rng, 1, max(1, min(128, 300_000_000 // (most * HK * D), 35_000_000_000 // (most * n * HQ * D))))
    return dict(op=op, B=B, n=n, least=rng.choice((0, 1, most // 2)), most=most, HQ=HQ, HK=HK, D=D, page=page,
                window=rng.choice((0, 0, 0, _log_uniform(rng, 1, most))), dtype=dtype)


# ---------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _heads(shape, dtype, g, spread=1.0):
    """Projected heads: channels of different size, a few of them far larger."""
    gain = torch.exp(0.5 * torch.randn(shape[-2:], generator=g, device="cuda"))
    gain[torch.rand(shape[-2:], generator=g, device="cuda") < 0.01] *= 8.0
    return (torch.randn(shape, generator=g, device="cuda") * gain * spread).to(DTYPES[dtype])


def _heads_inputs(case, g):
    """Queries and keys as views of one projection that holds the values too;
    positions, frequencies and weights."""
    M, T, HQ, HK, D, rot = (case[k] for k in ("M", "T", "HQ", "HK", "D", "rot"))
    lead = (T,) if M == 1 else (M, T)
    qkv = _heads((*lead, HQ + 2 * HK, D), case["dtype"], g)
    start = torch.randint(0, max(1, case["far"] - T), (1,), generator=g, device="cuda")
    s = dict(case, q=qkv[..., :HQ, :], k=qkv[..., HQ:HQ + HK, :],
             positions=(start + torch.arange(T, device="cuda")).to(torch.int32),
             freqs=10_000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) * 2 / max(rot, 1)),
             q_weight=None, k_weight=None)
    if case["far"] > 10_000 and T > 1:  # tokens of several sequences
        s["positions"] = torch.randint(0, case["far"], (T,), generator=g, device="cuda", dtype=torch.int32)
    if case["norm"]:
        for n in ("q_weight", "k_weight"):
            s[n] = 1.0 + 0.3 * torch.randn((D,) if M == 1 else (M, D), generator=g, device="cuda")
    if case["op"] == "grads":
        s["dq"] = (torch.randn((*lead, HQ, D), generator=g, device="cuda") * 1e-3).to(DTYPES[case["dtype"]])
        s["dk"] = (torch.randn((*lead, HK, D), generator=g, device="cuda") * 1e-3).to(DTYPES[case["dtype"]])
    return s


def _cache_inputs(case, g):
    T, H, D, page, prompts = (case[k] for k in ("T", "H", "D", "page", "prompts"))
    kv = _heads((T, 2 * H, D), case["dtype"], g)
    bounds = [T * i // prompts for i in range(prompts + 1)]
    room = [-(-(b - a + 37) // page) for a, b in zip(bounds, bounds[1:])]  # a prompt starts within its first page
    pages = sum(room) + 3
    order = torch.randperm(pages, generator=g, device="cuda")
    at = torch.empty(T, dtype=torch.int64)
    first = 0
    for i, (a, b) in enumerate(zip(bounds, bounds[1:])):
        at[a:b] = first * page + (11 * i) % min(page, 37) + torch.arange(b - a)
        first += room[i]
    at = at.to("cuda")
    return dict(case, k=kv[:, :H], v=kv[:, H:], slots=order[at // page] * page + at % page, pages=pages)


def _requests(case, g):
    """(lengths, queries) of a ragged batch's sequences, the longest among
    them: spread over their range, in the seed's order."""
    B, n, least, most = (case[k] for k in ("B", "n", "least", "most"))
    i = torch.randperm(B, generator=g, device="cuda").cpu()
    lengths = most - i * (most - least) // max(1, B - 1)
    counts = n - i * 7 % (n // 2 + 1)
    return lengths, torch.minimum(counts, lengths) if n > 1 else counts  # no more queries than keys


def _attend_inputs(case, g):
    """Queries, every sequence's keys and values by slot, and where they lie."""
    B, n, HQ, HK, D, page = (case[k] for k in ("B", "n", "HQ", "HK", "D", "page"))
    lengths, counts = _requests(case, g)
    starts = torch.zeros(B + 1, dtype=torch.int64)
    starts[1:] = counts.cumsum(0)
    held = (lengths + page - 1) // page
    width = -(-case["most"] // page) + 1
    pages = int(held.sum()) + 1
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    tables = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    slots, first = [], 0
    for b in range(B):
        own_pages = order[first:first + int(held[b])]
        tables[b, :own_pages.numel()] = own_pages
        at = torch.arange(int(lengths[b]), device="cuda")
        slots.append(own_pages.long()[at // page] * page + at % page)
        first += int(held[b])
    slots = torch.cat(slots)
    k = _heads((slots.numel(), HK, D), case["dtype"], g)
    v = _heads((slots.numel(), HK, D), case["dtype"], g)
    q = _heads((int(starts[-1]), HQ, D), case["dtype"], g, 1.5)
    return dict(case, q=q, k=k, v=v, slots=slots, tables=tables, lengths=lengths.to("cuda", torch.int32),
                starts=starts.to("cuda", torch.int32), counts=counts.tolist(), held=lengths.tolist(), pages=pages)


def _pages_inputs(case, g):
    B, page = case["B"], case["page"]
    least, most = case["least"], case["most"]
    i = torch.randperm(B, generator=g, device="cuda").to(torch.int32)  # the requests' order
    lengths = case["held"] - i * case["held"] // max(1, B - 1)
    counts = most - i * 37 % (most - least + 1)
    width = -(-(case["held"] + case["most"]) // page)
    used = (lengths.long() + page - 1) // page
    need = (lengths.long() + counts + page - 1) // page - used
    spare = int(int(need.sum()) * (1.0 - case["short"])) + (0 if case["short"] else 5)
    total = int(used.sum()) + spare
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    before = used.cumsum(0) - used
    j = torch.arange(width, device="cuda")
    tables = torch.where(j < used.unsqueeze(1), order[(before.unsqueeze(1) + j).clamp(max=max(0, total - 1))]
                         if total else -1, -1).to(torch.int32)
    free = torch.full((total,), -1, dtype=torch.int32, device="cuda")
    free[:spare] = order[total - spare:]
    return dict(case, tables=tables, lengths=lengths, counts=counts, keep=lengths.clone(), free=free,
                free_count=torch.tensor([spare], dtype=torch.int32, device="cuda"), tokens=B * case["most"])


def prepare(case, seed):
    g, op = _generator(seed), case["op"]
    if op in ("heads", "grads"):
        return _heads_inputs(case, g)
    if op == "pages":
        return _pages_inputs(case, g)
    s = _cache_inputs(case, g) if op == "cache" else _attend_inputs(case, g)
    if own:
        import paper_2606_22768_amd as fgd

        s["cache"] = fgd.Mx4Cache(s["pages"], case["page"], s["k"].shape[1], case["D"], device="cuda")
    else:
        size = (s["pages"] * case["page"], s["k"].shape[1], case["D"])
        codes = lambda: torch.zeros((*size[:2], size[2] // 2), dtype=torch.uint8, device="cuda")  # noqa: E731
        scales = lambda: torch.zeros((*size[:2], size[2] // BLOCK), dtype=torch.uint8, device="cuda")  # noqa: E731
        s["cache"] = (codes(), scales(), codes(), scales())
    if op == "attend":  # filled by the steps before this one
        _write(s["cache"], s["k"], s["v"], s["slots"])
        del s["k"], s["v"], s["slots"]
    return s


def _write(cache, k, v, slots):
    if own:
        import paper_2606_22768_amd as fgd

        fgd.mx4_cache_write(cache, k, v, slots)
        return
    for codes, scales, x in ((cache[0], cache[1], k), (cache[2], cache[3], v)):
        c, s = _quantise(x)
        codes[slots] = c[..., 0::2] | c[..., 1::2] << 4
        scales[slots] = s


# ---------------------------------------------------------------- plain forms

def _angles(s):
    """cos and sin, [T][1][n / 2], of angles in 64 bits."""
    a = s["positions"].double().unsqueeze(-1) * s["freqs"]
    return torch.cos(a).float().unsqueeze(-2), torch.sin(a).float().unsqueeze(-2)


def _turn(x, cos, sin, rot, interleaved):
    """The first `rot` elements of x in pairs, turned."""
    if rot == 0:
        return x
    y = x.clone()
    one, two = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., one], x[..., two]
    y[..., one] = a * cos - b * sin
    y[..., two] = a * sin + b * cos
    return y


def _per_head(w):
    """Weights [D] or [M][D] against [T][H][D] or [M][T][H][D]."""
    return w if w.dim() == 1 else w[:, None, None, :]


def _rotate(x, w, s, cos, sin):
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * _per_head(w)
    return _turn(y, cos, sin, s["rot"], s["interleaved"]).to(x.dtype)


def _rotate_grads(dy, x, w, s, cos, sin):
    g = _turn(dy.float(), cos, -sin, s["rot"], s["interleaved"])
    if w is None:
        return g.to(x.dtype), None
    xf = x.float()
    r = torch.rsqrt((xf * xf).mean(-1, keepdim=True) + EPS)
    xn = xf * r
    dw = (g * xn).flatten(-3, -2).sum(-2)
    gw = g * _per_head(w)
    dx = r * (gw - xn * (gw * xn).mean(-1, keepdim=True))
    return dx.to(x.dtype), dw


def _quantise(x):
    """(codes uint8 [..., D], scale bytes uint8 [..., D / 32])."""
    x = x.float().unflatten(-1, (-1, BLOCK))
    top = x.abs().amax(-1).contiguous().view(torch.int32) >> 23  # the exponent field: floor(log2) + 127
    scale = torch.where(top == 255, 255, (top - 2).clamp(min=0))
    a = x.abs() * ((254 - scale.clamp(max=253)) << 23).view(torch.float32).unsqueeze(-1)
    code = (a > 0.25).to(torch.uint8)
    code += a >= 0.75
    code += a > 1.25
    code += a >= 1.75
    code += a > 2.5
    code += a >= 3.5
    code += a > 5.0
    code += torch.signbit(x).to(torch.uint8) << 3
    return code.flatten(-2), scale.to(torch.uint8)


def _values(packed, scales):
    """The float32 values that packed codes and scale bytes stand for."""
    table = torch.tensor(CODES + tuple(-c for c in CODES), device=packed.device)
    v = table[torch.stack((packed & 15, packed >> 4), -1).flatten(-2).int()].unflatten(-1, (-1, BLOCK))
    bits = torch.where(scales == 0, 1 << 22, scales.int() << 23)  # of 2^(byte - 127); the smallest is denormal
    scale = torch.where(scales == 255, math.nan, bits.view(torch.float32))
    return (v * scale.unsqueeze(-1)).flatten(-2)


def _attend(s):
    q, page, HK, D, window = s["q"], s["page"], s["HK"], s["D"], s["window"]
    out = torch.zeros_like(q)
    first = 0
    for b, (n, L) in enumerate(zip(s["counts"], s["held"])):
        if n == 0:
            continue
        rows, first = slice(first, first + n), first + n
        if L == 0:
            continue
        at = torch.arange(L, device=q.device)
        slots = s["tables"][b].long()[at // page] * page + at % page
        k, v = (_values(s["cache"][i][slots], s["cache"][i + 1][slots]).transpose(0, 1).contiguous() for i in (0, 2))
        x = q[rows].float().unflatten(1, (HK, -1)).permute(1, 0, 2, 3).reshape(HK, -1, D)  # rows: query, then head
        z = torch.matmul(x, k.transpose(1, 2).contiguous()) * D ** -0.5
        position = (L - n + torch.arange(n, device=q.device)).repeat_interleave(x.shape[1] // n).unsqueeze(1)
        seen = at <= position
        if window > 0:
            seen &= at > position - window
        z.masked_fill_(~seen, -math.inf)
        p = torch.exp(z - z.amax(-1, keepdim=True))
        o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
        out[rows] = o.unflatten(1, (n, -1)).permute(1, 0, 2, 3).flatten(1, 2).to(out.dtype)
    return out


def _extend(tables, lengths, counts, free, free_count, page, tokens):
    B, width = tables.shape
    held, asked = lengths.long(), counts.long()
    have, want = (held + page - 1) // page, (held + asked + page - 1) // page
    asked = torch.where(want <= width, asked, 0)
    need = torch.where(want <= width, want - have, 0)
    upto = need.cumsum(0)
    total = asked.cumsum(0)
    granted = ((need == 0) | (upto <= free_count)) & (asked > 0) & (total <= tokens)
    need, asked = torch.where(granted, need, 0), torch.where(granted, asked, 0)
    taken = need.cumsum(0) - need
    j = torch.arange(width, device=tables.device) - have.unsqueeze(1)
    source = (free_count - 1 - taken.unsqueeze(1) - j).clamp(0, max(0, free.numel() - 1))
    fresh = (j >= 0) & (j < need.unsqueeze(1))
    if free.numel():
        tables.copy_(torch.where(fresh, free[source], tables))
    free_count -= need.sum().to(torch.int32)
    starts = torch.zeros(B + 1, dtype=torch.int64, device=tables.device)
    starts[1:] = asked.cumsum(0)
    t = torch.arange(tokens, device=tables.device)
    b = torch.searchsorted(starts[1:].contiguous(), t, right=True)
    real = b < B
    b = b.clamp(max=B - 1)
    position = torch.where(real, held[b] + t - starts[b], 0)
    slot = tables[b, (position // page).clamp(max=max(0, width - 1))].long() * page + position % page
    lengths += asked.to(torch.int32)
    return starts.to(torch.int32), position.to(torch.int32), torch.where(real, slot, -1)


def _truncate(tables, lengths, keep, free, free_count, page):
    width = tables.shape[1]
    held = lengths.long()
    left = torch.minimum(held, keep.long())
    have, stay = (held + page - 1) // page, (left + page - 1) // page
    back = have - stay
    before = back.cumsum(0) - back
    j = torch.arange(width, device=tables.device)
    given = (j >= stay.unsqueeze(1)) & (j < have.unsqueeze(1))
    at = free_count + back.sum() - 1 - before.unsqueeze(1) - (j - stay.unsqueeze(1))
    free[at[given]] = tables[given]
    tables.masked_fill_(given, -1)
    free_count += back.sum().to(torch.int32)
    lengths.copy_(left)


def run(state):
    op, s = state["op"], state
    if own:
        import paper_2606_22768_amd as fgd

        if op == "heads":
            return fgd.rotate_heads(s["q"], s["k"], s["positions"], s["freqs"], s["q_weight"], s["k_weight"], eps=EPS,
                                    interleaved=s["interleaved"])
        if op == "grads":
            return _present(fgd.rotate_heads_grads(s["dq"], s["dk"], s["q"], s["k"], s["positions"], s["freqs"],
                                                   s["q_weight"], s["k_weight"], eps=EPS,
                                                   interleaved=s["interleaved"]))
        if op == "cache":
            fgd.mx4_cache_write(s["cache"], s["k"], s["v"], s["slots"])
            return fgd.mx4_cache_read(s["cache"], s["slots"], s["dtype"])
        if op == "attend":
            if s["n"] == 1:
                return fgd.mx4_attend(s["q"], s["cache"], s["tables"], s["lengths"], window=s["window"])
            return fgd.mx4_attend(s["q"], s["cache"], s["tables"], s["lengths"], starts=s["starts"], max_q=s["n"],
                                  window=s["window"])
        made = fgd.extend_pages(s["tables"], s["lengths"], s["counts"], s["free"], s["free_count"], s["page"],
                                s["tokens"])
        fgd.truncate_pages(s["tables"], s["lengths"], s["keep"], s["free"], s["free_count"], s["page"])
        return (*made, s["tables"], s["lengths"], s["free"], s["free_count"])
    if op in ("heads", "grads"):
        cos, sin = _angles(s)
        if op == "heads":
            return tuple(_rotate(s[n], s[n + "_weight"], s, cos, sin) for n in "qk")
        dq, dq_weight = _rotate_grads(s["dq"], s["q"], s["q_weight"], s, cos, sin)
        dk, dk_weight = _rotate_grads(s["dk"], s["k"], s["k_weight"], s, cos, sin)
        return _present((dq, dk, dq_weight, dk_weight))
    if op == "cache":
        _write(s["cache"], s["k"], s["v"], s["slots"])
        return tuple(_values(s["cache"][i][s["slots"]], s["cache"][i + 1][s["slots"]]).to(DTYPES[s["dtype"]])
                     for i in (0, 2))
    if op == "attend":
        return _attend(s)
    made = _extend(s["tables"], s["lengths"], s["counts"], s["free"], s["free_count"], s["page"], s["tokens"])
    _truncate(s["tables"], s["lengths"], s["keep"], s["free"], s["free_count"], s["page"])
    return (*made, s["tables"], s["lengths"], s["free"], s["free_count"])


def _present(outputs):
    return tuple(t for t in outputs if t is not None)


def work(case):
    op, es = case["op"], 4 if case.get("dtype") == "f32" else 2
    if op in ("heads", "grads"):
        tokens = case["M"] * case["T"]
        n = tokens * (case["HQ"] + case["HK"]) * case["D"]
        weights = 2 * case["M"] * case["D"] * 4 if case["norm"] else 0
        if op == "heads":
            return {"bytes": 2 * n * es + case["T"] * 4 + weights, "flops": 7 * n}
        return {"bytes": (3 if case["norm"] else 2) * n * es + case["T"] * 4 + 2 * weights, "flops": 14 * n}
    if op == "cache":
        n = case["T"] * case["H"] * case["D"]
        return {"bytes": 4 * n * es + 2 * 2 * n * 17 // 32 + 8 * case["T"], "flops": 6 * n}
    if op == "pages":
        tokens = case["B"] * (case["least"] + case["most"]) // 2
        pages = tokens // case["page"] + 1
        return {"bytes": 12 * case["B"] * case["most"] + 16 * case["B"] + 16 * pages, "flops": 4 * tokens}
    rows = keys = seen = 0
    for i in range(case["B"]):
        length = case["most"] - i * (case["most"] - case["least"]) // max(1, case["B"] - 1)
        n = case["n"] - i * 7 % (case["n"] // 2 + 1)
        n = min(n, length) if case["n"] > 1 else n
        window = case["window"] or length
        rows += n
        keys += min(length, window + n - 1)
        seen += sum(min(length - n + 1 + j, window) for j in range(n))
    return {"bytes": int(keys * case["HK"] * case["D"] * 2 * 17 / 32 + 2 * rows * case["HQ"] * case["D"] * es),
            "flops": int(4 * seen * case["HQ"] * case["D"])}


# ---------------------------------------------------------------- in 64 bits

def _power(e):
    """2^e in 64 bits, from its bits (pow is not exact)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_values(x):
    """x in the 4-bit format, by its definition: the grid's step at a is
    2^(max(floor(log2 a), 0) - 1), and rounding is to the nearest multiple,
    the even one of two."""
    b = x.double().unflatten(-1, (-1, BLOCK))
    top = b.abs().amax(-1, keepdim=True)
    e = (torch.frexp(top).exponent - 3).clamp(-127, 127)
    a = b.abs() * _power(-e)
    step = _power((torch.frexp(a).exponent - 1).clamp(min=0) - 1)
    v = (torch.round(a / step) * step).clamp(max=6) * _power(e)
    return torch.where(torch.isfinite(top), v * torch.sign(b), math.nan).flatten(-2)


def _exact_matrix(s):
    """Every position's rotation as complex numbers."""
    a = s["positions"].double()[:, None, None] * s["freqs"]
    return torch.polar(torch.ones_like(a), a)


def _exact_turn(x, turn, s):
    n = s["rot"]
    if n == 0:
        return x
    pairs = x[..., :n].unflatten(-1, (-1, 2)) if s["interleaved"] else x[..., :n].unflatten(-1, (2, -1)).mT
    pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    head = pairs.flatten(-2) if s["interleaved"] else pairs.mT.flatten(-2)
    return torch.cat((head, x[..., n:]), -1)


def _exact_heads(s):
    turn = _exact_matrix(s)
    out, weights = [], []
    for name in "qk":
        x, w = s[name].double(), s[name + "_weight"]
        norm = torch.sqrt((x ** 2).mean(-1, keepdim=True) + EPS)
        if w is not None:
            w = w.double().reshape(*w.shape[:-1], *(1, 1) * (w.dim() - 1), -1)
        if s["op"] == "heads":
            out.append(_exact_turn(x if w is None else x / norm * w, turn, s))
            continue
        g = _exact_turn(s["d" + name].double(), turn.conj(), s)
        if w is not None:
            weights.append((g * x / norm).sum((-3, -2)))
            g = g * w
            g = g / norm - x * (g * x).mean(-1, keepdim=True) / norm ** 3
        out.append(g)
    return (*out, *weights)


def _exact_attend(s):
    k, v = _exact_values(s["k"]), _exact_values(s["v"])
    group = s["HQ"] // s["HK"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    row = key = 0
    for n, L in zip(s["counts"], s["held"]):
        if n and L:
            for h in range(s["HK"]):
                heads = slice(h * group, (h + 1) * group)
                x = s["q"][row:row + n, heads].double()
                z = (x.reshape(n * group, -1) @ k[key:key + L, h].T.contiguous() / math.sqrt(s["D"])).view(n, group, L)
                back = torch.arange(L - n, L, device="cuda")[:, None, None] - torch.arange(L, device="cuda")
                hidden = (back < 0) | (back >= (s["window"] or L))
                p = torch.softmax(z.masked_fill(hidden, -math.inf), -1)
                out[row:row + n, heads] = (p.view(n * group, L) @ v[key:key + L, h].contiguous()).view(n, group, -1)
        row, key = row + n, key + L
    return out


def exact(case, seed):
    op, g = case["op"], _generator(seed)
    if op in ("heads", "grads"):
        return _exact_heads(_heads_inputs(case, g))
    if op == "cache":
        s = _cache_inputs(case, g)
        return _exact_values(s["k"]), _exact_values(s["v"])
    if op == "attend":
        return _exact_attend(_attend_inputs(case, g))
    return None  # whole numbers throughout
