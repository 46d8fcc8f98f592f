"""Timed cases of the operators around a quantized key/value cache: rotary positions,
writing and reading the cache, and attention over it; each with its plain form and its
definition in 64 bits.

* ``rotary``: the rotation of queries and keys by their positions, on the whole-sequence
  layout [B, H, N, d] of the forwards or on the heads of a fused projection [n, heads, d];
* ``cache``: new tokens quantized into a paged cache, and the sequence read back (a
  chunk of a prompt joins its cached prefix, and the dense forwards take both);
* ``attention``: single tokens, ragged chunks or trees of drafted tokens over the cache.

Inputs are seeded and synthetic.  Keys have a few large channels, as models' keys have;
pages are dealt in random order, as an allocator leaves them after some time.
"""
import math
import random

import torch

own = False   # True: the framework's operators; False: their plain forms

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---------------------------------------------------------------- cases

def _rotary(name, layout, B, H, N, d, r, src="bf16", extra=0, interleaved=False, inverse=False, yarn=False,
            far=32768):
    c = dict(kind="rotary", layout=layout, B=B, H=H, N=N, d=d, r=r, src=src, extra=extra, interleaved=interleaved,
             inverse=inverse, yarn=yarn, far=far)
    return dict(name=name, **c) if name else c


def _cache(name, n, prefix, H, d, page, fp8=False, src="bf16", pad=0, q_heads=0):
    c = dict(kind="cache", n=n, prefix=prefix, H=H, d=d, page=page, fp8=fp8, src=src, pad=pad, q_heads=q_heads)
    return dict(name=name, **c) if name else c


def _attention(name, B, H, G, d, length, page, fp8=False, T=1, spread=1, empty=0, tree=False, lse=False):
    c = dict(kind="attention", B=B, H=H, G=G, d=d, length=length, page=page, fp8=fp8, T=T, spread=spread, empty=empty,
             tree=tree, lse=lse)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # one decode step of 16 requests: query and key heads side by side in the fused projection's output
        _rotary("rotary_step", "nhd", 1, 40, 16, 128, 128, extra=8),
        # queries of a long prompt in the forward's layout, angles stretched for a long context
        _rotary("rotary_prompt", "bhnd", 1, 32, 16384, 128, 128, yarn=True, far=131072),
        # the gradient with part of the head rotated, interleaved pairs, fp32, odd lengths
        _rotary("rotary_gradient", "bhnd", 3, 10, 1921, 64, 32, src="fp32", interleaved=True, inverse=True),
        # a short chunk appended to a cached prefix
        _cache("cache_chunk", 16, 1031, 8, 128, 64, q_heads=32),
        # a long prompt, written and read back whole
        _cache("cache_prompt", 16384, 0, 8, 128, 64),
        # FP8 cache with small pages, fp32 projections, a padded batch
        _cache("cache_fp8_padded", 2501, 4987, 5, 64, 16, fp8=True, src="fp32", pad=249),
        # one request, one token, a short conversation: latency
        _attention("decode_one", 1, 8, 4, 128, 517, 64),
        # a serving batch, conversations of very different lengths, two idle places
        _attention("decode_batch", 64, 8, 4, 128, 16384, 64, spread=128, empty=2),
        # long documents, FP8 cache
        _attention("decode_long_fp8", 4, 8, 8, 128, 131072, 128, fp8=True, spread=2),
        # small heads, seven queries to a key head, small pages
        _attention("decode_d64_fp8", 40, 2, 7, 64, 4099, 16, fp8=True, spread=8),
        # verification of a few drafted tokens, with the normaliser for merging
        _attention("tree_small", 8, 8, 4, 128, 2047, 64, T=16, spread=2, tree=True, lse=True),
        # verification of large trees in a full batch
        _attention("tree_large", 32, 8, 8, 128, 8192, 64, T=64, spread=4, tree=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rotary", "cache", "attention", "attention"))
    d = rng.choice((64, 128, 128))
    if kind == "rotary":
        while True:
            layout = rng.choice(("nhd", "bhnd"))
            c = _rotary(None, layout, 1 if layout == "nhd" else rng.choice((1, 2, 3)), _log_int(rng, 1, 64),
                        _log_int(rng, 1, 16384), d, rng.choice((d, d, d // 2, d // 4)), rng.choice(("bf16", "bf16", "fp32")),
                        rng.choice((0, 2, 8)) if layout == "nhd" else 0, rng.random() < 0.4, rng.random() < 0.3,
                        rng.random() < 0.4, _log_int(rng, 16384, 1 << 20))
            if c["B"] * c["H"] * c["N"] * d <= 32 * 16384 * 128:
                return c
    if kind == "cache":
        while True:
            n = _log_int(rng, 1, 16384)
            c = _cache(None, n, rng.choice((0, _log_int(rng, 1, 16384))), _log_int(rng, 1, 16), d,
                       rng.choice((16, 32, 64, 128)), rng.random() < 0.5, rng.choice(("bf16", "bf16", "fp32")),
                       rng.choice((0, n // 10)), rng.choice((0, 4, 32)))
            if (c["n"] + c["prefix"]) * c["H"] * d <= 16384 * 8 * 128:
                return c
    while True:
        T = rng.choice((1, 1, _log_int(rng, 2, 64)))
        c = _attention(None, _log_int(rng, 1, 64), _log_int(rng, 1, 8), _log_int(rng, 1, 8), d,
                       max(T, _log_int(rng, 1, 131072)), rng.choice((16, 32, 64, 128, 256)), rng.random() < 0.5, T,
                       rng.choice((1, 2, 16, 64)), rng.choice((0, 0, 1)), T > 1 and rng.random() < 0.6,
                       rng.random() < 0.3)
        w = work(c)
        if w["bytes"] < 8.7e8 and w["flops"] < 2.6e11:
            return c


def _lengths(c):
    """Tokens and keys (new tokens included) of each sequence, from the case alone."""
    rng = random.Random(repr(sorted((k, v) for k, v in c.items() if k != "name")))
    new, keys = [], []
    for b in range(c["B"]):
        t = c["T"] if c["T"] == 1 or b == 0 else rng.randint(max(1, c["T"] // 2), c["T"])
        n = c["length"] if b == 0 else _log_int(rng, max(1, c["length"] // c["spread"]), c["length"])
        idle = b > 0 and b >= c["B"] - c["empty"]
        new.append(0 if idle and c["T"] > 1 else t)
        keys.append(0 if idle else max(n, t))
    return new, keys


def work(c):
    if c["kind"] == "rotary":
        n = c["B"] * c["H"] * c["N"] * c["d"]
        size = 2 if c["src"] == "bf16" else 4
        return {"bytes": 2 * n * size + 8 * c["N"], "flops": 3 * c["B"] * c["H"] * c["N"] * c["r"]}
    bits = 8 if c["fp8"] else 4
    token = 2 * c["H"] * (c["d"] * bits // 8 + c["d"] // 32)   # K and V of one token in the cache
    if c["kind"] == "cache":
        size = 2 if c["src"] == "bf16" else 4
        values = 2 * c["H"] * c["d"]
        m = c["n"] - c["pad"] + c["prefix"]   # read back, the new tokens included
        return {"bytes": (c["n"] - c["pad"]) * (values * size + token + 8) + m * (token + 2 * values + 8),
                "flops": (c["n"] - c["pad"]) * values * 4 + m * values}
    new, keys = _lengths(c)
    rows = sum(new) * c["H"] * c["G"]
    flops = sum(4 * t * c["H"] * c["G"] * n * c["d"] for t, n in zip(new, keys))
    return {"bytes": sum(n for t, n in zip(new, keys) if t) * token + rows * c["d"] * 4 + (4 * rows if c["lse"] else 0),
            "flops": flops}


def _two_to(e):
    """2^e in fp64, exact, of integers e in [-1022, 1023] (pow and exp2 may be an ulp off)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


# ---------------------------------------------------------------- inputs

def _normal(shape, dtype, g):
    return torch.randn(shape, dtype=dtype, device="cuda", generator=g)


def _keys(shape, g):
    """Values of keys: unit variance, one channel in 32 eight times as large."""
    gain = torch.ones(shape[-1], device="cuda")
    gain[torch.randperm(shape[-1], device="cuda", generator=g)[: shape[-1] // 32]] = 8.0
    return _normal(shape, torch.float32, g).mul_(gain)


def _pack_k(codes, fp8):
    """Codes [..., d] (uint8, one a value) as the cache holds keys."""
    return codes if fp8 else codes[..., 0::2] | (codes[..., 1::2] << 4)


def _fill_cache(values, fp8):
    """A cache [pages, H, page] filled with ``values`` [pages, H, page, d]: a fast rounding for inputs, not the quantizer.
    Returns codes [..., d] (one a value) and scale bytes [..., d / 32]."""
    x = values.unflatten(-1, (-1, 32))
    amax = x.abs().amax(-1, keepdim=True)
    if fp8:
        e = torch.frexp(amax).exponent - 8        # amax / 2^e in [128, 256)
        codes = (x * _two_to(-e).float()).to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        e = torch.frexp(amax).exponent            # amax / 2^e in [1/2, 1)
        r = (x * _two_to(-e).float()).abs_().mul_(6.0)
        codes = torch.bucketize(r, torch.tensor((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0), device="cuda"), out_int32=True)
        codes = codes.to(torch.uint8) | ((x < 0).to(torch.uint8) << 3)
    return codes.flatten(-2), (e.squeeze(-1) + 127).to(torch.uint8)


def _cache_tensors(pages, H, page, d, fp8, g, empty=False):
    """k_codes, k_scales, v_codes, v_scales in the cache's layout."""
    width = d if fp8 else d // 2
    k_codes = torch.zeros((pages, H, page, width), dtype=torch.uint8, device="cuda")
    k_scales = torch.zeros((pages, H, page, d // 32), dtype=torch.uint8, device="cuda")
    v_codes = torch.zeros((pages, H, page // 8, 16, 8, width // 16), dtype=torch.uint8, device="cuda")
    v_scales = torch.zeros((pages, H, page // 8, d // 32, 8), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (H * page * d))
    for p in range(0, 0 if empty else pages, step):
        n = min(step, pages - p)
        c, s = _fill_cache(_keys((n, H, page, d), g), fp8)
        k_codes[p:p + n], k_scales[p:p + n] = _pack_k(c, fp8), s
        c, s = _fill_cache(_normal((n, H, page, d), torch.float32, g), fp8)
        c = _pack_k(c, fp8).view(n, H, page // 8, 8, 16, width // 16)
        v_codes[p:p + n] = c.transpose(3, 4)
        v_scales[p:p + n] = s.view(n, H, page // 8, 8, d // 32).transpose(3, 4)
    return k_codes, k_scales, v_codes, v_scales


def _frequencies(r, yarn):
    """Radians a position of each pair in fp64, and the magnitude.  ``yarn``: a context stretched by 4 from 32768:
    fast pairs (over 32 turns in the old context) keep their angle, slow ones (under 1) turn 4 times slower."""
    j = torch.arange(r // 2, dtype=torch.float64)
    f = 10000.0 ** (-2.0 * j / r)
    if not yarn:
        return f.cuda(), 1.0
    low, high = (r * math.log(32768 / (turns * 2 * math.pi)) / (2 * math.log(10000.0)) for turns in (32, 1))
    low, high = max(math.floor(low), 0), min(math.ceil(high), r - 1)
    keep = 1.0 - ((j - low) / max(high - low, 1e-3)).clamp(0, 1)
    return (f * keep + f / 4.0 * (1.0 - keep)).cuda(), 0.1 * math.log(4.0) + 1.0


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"c": c}
    if c["kind"] == "rotary":
        B, H, N, d = c["B"], c["H"], c["N"], c["d"]
        if c["layout"] == "nhd":   # the first H heads of a fused projection, a position a token
            x = _normal((N, H + c["extra"], d), torch.float32, g).to(DTYPES[c["src"]])
            s["x"] = x[:, :H]
            s["positions"] = torch.randint(0, c["far"], (N,), device="cuda", generator=g)
        else:                      # sequences that begin at different positions
            s["x"] = _normal((B, H, N, d), torch.float32, g).to(DTYPES[c["src"]])
            start = torch.randint(0, max(1, c["far"] - N), (B, 1), device="cuda", generator=g)
            s["positions"] = start + torch.arange(N, device="cuda")
        s["inv_freq"], s["magnitude"] = _frequencies(c["r"], c["yarn"])
        return s
    H, d, page = c["H"], c["d"], c["page"]
    if c["kind"] == "cache":
        n, prefix = c["n"], c["prefix"]
        fresh = n - c["pad"]
        own_pages = -(-(prefix + fresh) // page)
        pages = own_pages + own_pages // 4 + 1
        s["cache"] = _cache_tensors(pages, H, page, d, c["fp8"], g, empty=prefix == 0)
        table = torch.randperm(pages, device="cuda", generator=g)[:own_pages]
        at = torch.arange(prefix + fresh, device="cuda")
        s["read"] = table[at // page] * page + at % page
        s["slots"] = torch.full((n,), -1, dtype=torch.int64, device="cuda")
        s["slots"][:fresh] = s["read"][prefix:]
        fused = torch.cat((_normal((n, c["q_heads"], d), torch.float32, g), _keys((n, H, d), g),
                           _normal((n, H, d), torch.float32, g)), 1).to(DTYPES[c["src"]])
        s["k"], s["v"] = fused[:, c["q_heads"]:-H], fused[:, -H:]
        return s
    new, keys = _lengths(c)
    need = [-(-n // page) for n in keys]
    pages = sum(need) + 1
    s["cache"] = _cache_tensors(pages, H, page, d, c["fp8"], g)
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).int()
    table = torch.zeros((c["B"], max(need) + 1), dtype=torch.int32)   # places past a sequence's pages are never read
    at = 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    s["table"] = table.cuda()
    s["lengths"] = torch.tensor(keys, dtype=torch.int32, device="cuda")
    s["new"], s["keys"] = new, keys
    n = sum(new)
    s["q"] = _normal((n, c["G"] * H, d), torch.bfloat16, g)
    s["q_starts"] = None
    if c["T"] > 1:
        s["q_starts"] = torch.tensor([sum(new[:b]) for b in range(c["B"] + 1)], dtype=torch.int32, device="cuda")
    s["tree"] = None
    if c["tree"]:   # each drafted token's parent is an earlier one (or the prefix): its ancestors and itself are seen
        rng, bits = random.Random(seed), []
        for t in new:
            seen = []
            for i in range(t):
                up = rng.randint(-1, i - 1)
                seen.append((1 << i) | (seen[up] if up >= 0 else 0))
            bits += seen
        s["tree"] = torch.tensor([x - (1 << 64) if x >> 63 else x for x in bits], dtype=torch.int64, device="cuda")
    return s


# ---------------------------------------------------------------- plain forms

def _rotary_plain(s):
    c, x = s["c"], s["x"]
    r, half = c["r"], c["r"] // 2
    angle = s["positions"].double()[..., None] * s["inv_freq"]
    cos, sin = (f(angle).float() * s["magnitude"] for f in (torch.cos, torch.sin))
    cos, sin = (cos[:, None], sin[:, None])                       # over the heads: [n, 1, r/2] or [B, 1, N, r/2]
    if c["inverse"]:
        sin = -sin
    y = x.float()
    if c["interleaved"]:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    else:
        a, b = y[..., :half], y[..., half:r]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    return torch.cat((turned, y[..., r:]), -1).to(x.dtype)


def _quantize_plain(x, fp8):
    """Codes [..., d] (one a value) and scale bytes [..., d / 32] of the library's MXFP4 and MXFP8, decided in fp64."""
    x = x.double().unflatten(-1, (-1, 32))
    amax = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(amax)
    zero = amax == 0
    if fp8:   # the smallest amplitude that leaves no payload above 448
        e = (e - 9 + (amax * _two_to(9 - e) > 448)).clamp(-127, 127)
        codes = (x * _two_to(-e)).float().to(torch.float8_e4m3fn).view(torch.uint8)
    else:     # the floor amplitude if its squared error is the smaller, else the ceiling
        edges = ((0.25, 0), (0.75, 1), (1.25, 0), (1.75, 1), (2.5, 0), (3.5, 1), (5.0, 0))   # 1: a tie goes up
        grid = torch.tensor(E2M1, dtype=torch.float64, device=x.device)

        def encode(e):
            r = 6.0 * x.abs() * _two_to(-e)
            k = sum((r >= edge if up else r > edge).to(torch.int64) for edge, up in edges)
            return k, (grid[k] * _two_to(e) - 6.0 * x.abs()).square().sum(-1, keepdim=True)

        e_ceil, e_floor = torch.where(m == 0.5, e - 1, e), e - 1
        k_ceil, err_ceil = encode(e_ceil)
        k_floor, err_floor = encode(e_floor)
        low = err_floor < err_ceil
        e = torch.where(low, e_floor, e_ceil).clamp(-127, 127)
        codes = torch.where(low, k_floor, k_ceil).to(torch.uint8) | (torch.signbit(x).to(torch.uint8) << 3)
    scales = torch.where(zero, torch.zeros_like(e), e + 127).squeeze(-1).to(torch.uint8)
    return codes.flatten(-2), scales


def _decode(codes, scales, fp8):
    """Values of cache bytes [..., d bytes or d / 2] with scales [..., d / 32]."""
    if fp8:
        v = codes.view(torch.float8_e4m3fn).float()
    else:
        grid = torch.tensor(E2M1 + tuple(-x for x in E2M1), device=codes.device) / 6.0
        v = grid[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return (v.unflatten(-1, (-1, 32)) * _two_to(scales.int()[..., None] - 127).float()).flatten(-2)


def _v_rows(v_codes, v_scales, page, off):
    """V bytes and scales [m, H, ...] of offset ``off`` of page ``page``, in order of d."""
    return v_codes[page, :, off // 8, :, off % 8].flatten(-2), v_scales[page, :, off // 8, :, off % 8]


def _cache_plain(s):
    c = s["c"]
    k_codes, k_scales, v_codes, v_scales = s["cache"]
    page = c["page"]
    valid = s["slots"] >= 0
    slots = s["slots"][valid]
    p, off = slots // page, slots % page
    codes, scales = _quantize_plain(s["k"][valid], c["fp8"])
    k_codes[p, :, off], k_scales[p, :, off] = _pack_k(codes, c["fp8"]), scales
    codes, scales = _quantize_plain(s["v"][valid], c["fp8"])
    v_codes[p, :, off // 8, :, off % 8] = _pack_k(codes, c["fp8"]).unflatten(-1, (16, -1))
    v_scales[p, :, off // 8, :, off % 8] = scales
    p, off = s["read"] // page, s["read"] % page
    k = _decode(k_codes[p, :, off], k_scales[p, :, off], c["fp8"]).bfloat16()
    return k, _decode(*_v_rows(v_codes, v_scales, p, off), c["fp8"]).bfloat16()


def _visible(s, b, n, device):
    """[T, n] truth values: which keys each new token of sequence b sees."""
    t = s["new"][b]
    prefix = n - t
    key = torch.arange(n, device=device)
    if s["tree"] is None:
        return key <= prefix + torch.arange(t, device=device)[:, None]
    first = sum(s["new"][:b])
    word = s["tree"][first:first + t, None]
    return (key < prefix) | ((key >= prefix) & ((word >> (key - prefix).clamp(0, 63)) & 1).bool())


def _attention_plain(s):
    c = s["c"]
    k_codes, k_scales, v_codes, v_scales = s["cache"]
    H, G, d, page = c["H"], c["G"], c["d"], c["page"]
    outs, norms, at = [], [], 0
    for b in range(c["B"]):
        t, n = s["new"][b], s["keys"][b]
        q = s["q"][at:at + t].float()
        at += t
        if t == 0 or n == 0:
            outs.append(torch.zeros_like(q))
            norms.append(q.new_full(q.shape[:2], -math.inf))
            continue
        p = s["table"][b, : -(-n // page)].long()
        k = _decode(k_codes[p], k_scales[p], c["fp8"]).transpose(0, 1).flatten(1, 2)[:, :n]            # [H, n, d]
        v = v_codes[p].transpose(-3, -2).flatten(-2)                                                   # [p, H, page/8, 8, .]
        v = _decode(v, v_scales[p].transpose(-2, -1), c["fp8"]).flatten(2, 3).transpose(0, 1).flatten(1, 2)[:, :n]
        x = q.unflatten(1, (H, G)).permute(1, 0, 2, 3).flatten(1, 2)                                   # [H, t G, d]
        z = torch.matmul(x, k.transpose(1, 2).contiguous()) / math.sqrt(d)
        seen = _visible(s, b, n, z.device).repeat_interleave(G, 0)
        z = z.masked_fill(~seen, -math.inf)
        top = z.amax(-1, keepdim=True)
        w = torch.exp(z - top)
        total = w.sum(-1, keepdim=True)
        o = torch.matmul(w, v) / total
        outs.append(o.unflatten(1, (t, G)).permute(1, 0, 2, 3).flatten(1, 2))
        norms.append((top + torch.log(total)).squeeze(-1).unflatten(1, (t, G)).permute(1, 0, 2).flatten(1, 2))
    out = torch.cat(outs).bfloat16()
    return (out, torch.cat(norms)) if c["lse"] else out


# ---------------------------------------------------------------- the framework's operators

def _run_own(s):
    import paper_2609_04105_amd as fa

    c = s["c"]
    if c["kind"] == "rotary":
        return fa.rotary(s["x"], s["positions"], s["inv_freq"], interleaved=c["interleaved"], magnitude=s["magnitude"],
                         inverse=c["inverse"])
    cache = fa.KVCache(*s["cache"])
    if c["kind"] == "cache":
        fa.cache_write(s["k"], s["v"], cache, s["slots"])
        return fa.cache_read(cache, s["read"], out_dtype=torch.bfloat16)
    lse = torch.empty(s["q"].shape[:2], device=s["q"].device) if c["lse"] else None
    out = fa.cache_attention(s["q"], cache, s["table"], s["lengths"], q_starts=s["q_starts"], max_q=c["T"],
                             tree=s["tree"], lse=lse, out_dtype=torch.bfloat16)
    return (out, lse) if c["lse"] else out


def run(state):
    if own:
        return _run_own(state)
    return {"rotary": _rotary_plain, "cache": _cache_plain, "attention": _attention_plain}[state["c"]["kind"]](state)


# ---------------------------------------------------------------- definitions in 64 bits

def _exact_rotary(s):
    """Pairs as complex numbers times m exp(+- i angle)."""
    c, x = s["c"], s["x"].double()
    r = c["r"]
    angle = s["positions"].double().unsqueeze(-1) * s["inv_freq"]
    turn = torch.polar(torch.full_like(angle, s["magnitude"]), -angle if c["inverse"] else angle).unsqueeze(1)
    head = x[..., :r]
    pairs = head.unflatten(-1, (r // 2, 2)) if c["interleaved"] else head.unflatten(-1, (2, r // 2)).transpose(-1, -2)
    y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    y = y.flatten(-2) if c["interleaved"] else y.transpose(-1, -2).flatten(-2)
    return torch.cat((y, x[..., r:]), -1)


def _nearest(x, grid):
    """The nearest of the ascending values ``grid`` >= 0 to |x| with x's sign; ties to the even place."""
    a = x.abs()
    hi = torch.searchsorted(grid, a.contiguous()).clamp(1, grid.numel() - 1)
    lo = hi - 1
    up, down = grid[hi] - a, a - grid[lo]
    pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return torch.copysign(grid[pick], x)


def _exact_quantized(x, fp8):
    """What the quantized values of x stand for, from their definition."""
    x = x.double().unflatten(-1, (-1, 32))
    amax = x.abs().amax(-1, keepdim=True)
    safe = torch.where(amax == 0, torch.ones_like(amax), amax)
    low = torch.floor(torch.log2(safe))                      # may be one off next to a power of two
    low = low - (_two_to(low) > safe).double()
    low = low + (_two_to(low + 1) <= safe).double()
    high = low + (_two_to(low) < safe).double()
    if fp8:
        grid = torch.tensor([m * 2.0 ** -9 for m in range(8)] +
                            [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1],
                            dtype=torch.float64, device=x.device)
        amp = _two_to(low - 8)
        amp = torch.where(safe / amp > 448, 2 * amp, amp)
        return torch.where(amax == 0, x, amp * _nearest(x / amp, grid)).flatten(-2)
    grid = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
    best, cost = None, None
    for exponent in (high, low):                             # the ceiling keeps a tie
        amp = _two_to(exponent)
        k = amp * _nearest(6 * x / amp, grid)                # 6 times the value
        e = (k - 6 * x).square().sum(-1, keepdim=True)
        best, cost = (k, e) if best is None else (torch.where(e < cost, k, best), torch.minimum(e, cost))
    return torch.where(amax == 0, x, best / 6).flatten(-2)


def _exact_bytes(codes, scales, fp8):
    """fp64 values of code bytes, from the formats' bit fields."""
    if fp8:
        e, m = (codes >> 3) & 15, (codes & 7).double()
        v = torch.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * _two_to(e.int() - 7))
        v = torch.where(codes > 127, -v, v)
    else:
        n = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
        e, m = (n >> 1) & 3, (n & 1).double()
        v = torch.where(e == 0, m / 2, (1 + m / 2) * _two_to(e.int() - 1)) / 6
        v = torch.where(n > 7, -v, v)
    return v * _two_to(scales.int() - 127).repeat_interleave(32, -1)


def _exact_cache(s):
    """The read slots hold the prefix as it was and the new tokens' quantized values."""
    c = s["c"]
    k_codes, k_scales, v_codes, v_scales = s["cache"]
    old = s["read"][: c["prefix"]]
    p, off = old // c["page"], old % c["page"]
    fresh = s["slots"] >= 0
    k = _exact_bytes(k_codes[p, :, off], k_scales[p, :, off], c["fp8"])
    v = _exact_bytes(*_v_rows(v_codes, v_scales, p, off), c["fp8"])
    return (torch.cat((k, _exact_quantized(s["k"][fresh], c["fp8"]))),
            torch.cat((v, _exact_quantized(s["v"][fresh], c["fp8"]))))


def _exact_attention(s):
    """Head by head, the softmax written out over the visible keys."""
    c = s["c"]
    k_codes, k_scales, v_codes, v_scales = s["cache"]
    G, page = c["G"], c["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=s["q"].device)
    first = 0
    for b, (t, n) in enumerate(zip(s["new"], s["keys"])):
        rows = slice(first, first + t)
        first += t
        if t == 0 or n == 0:
            continue
        at = torch.arange(n, device=out.device)
        p, off = s["table"][b].long()[at // page], at % page
        hide = torch.zeros((t, 1, n), dtype=torch.float64, device=out.device)
        hide[~_visible(s, b, n, out.device)[:, None]] = -math.inf
        for h in range(c["H"]):
            k = _exact_bytes(k_codes[p, h, off], k_scales[p, h, off], c["fp8"])
            v = _exact_bytes(v_codes[p, h, off // 8, :, off % 8].flatten(-2), v_scales[p, h, off // 8, :, off % 8],
                             c["fp8"])
            heads = slice(h * G, (h + 1) * G)
            z = (s["q"][rows, heads].double().flatten(0, 1) @ k.T).unflatten(0, (t, G)) / math.sqrt(c["d"]) + hide
            lse[rows, heads] = torch.logsumexp(z, -1)
            out[rows, heads] = (torch.exp(z - lse[rows, heads, None]).flatten(0, 1) @ v).unflatten(0, (t, G))
    return (out, lse) if c["lse"] else out


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "cache": _exact_cache, "attention": _exact_attention}[case["kind"]](s)
