"""More serving operators around the paged cache whose speed counts: the norm of each head of queries and keys in the
pass that rotates them and writes the cache, a cache held in 8 bits (written from the projection, read back into pages
that prefill attention takes), decode attention over that cache, and decode attention for requests that share a prefix.

A case is one call (or, for the 8-bit cache, the write and the read-back) on the tokens of one iteration, formed as an
engine forms it: decodes first, then prefill chunks.  `listed()` holds the cases that are always measured, `draw()` gives
others of the same ranges.  `run` computes the operators in plain torch operations, or, where `own` is set, by the
library's own calls.

A key or value of the 8-bit cache is e4m3 times a power of two that the d values of its token and head share: the smallest
that brings the largest of them to at most 448, at least 2^-126 and held as a byte, the exponent plus 127.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
DECODE, PREFILL = 1, 0
HEADS_8B = (32, 8, 128)    # Llama-3-8B
HEADS_70B = (64, 8, 128)   # Llama-3-70B
HEADS_RANK = (8, 1, 128)   # one of eight tensor-parallel ranks of Llama-3-70B
HEADS_SMALL = (8, 2, 64)
EPS = 1e-6


def _split(op, name, heads, decodes=0, ctx=(1, 1), chunks=0, chunk=0, prefix=0, lens=1, dtype="bf16", rot=-1,
           adjacent=False, norm=True):
    """`decodes` requests with contexts drawn from ctx, and `chunks` prefill chunks: the first of `chunk` tokens after
    `prefix` cached ones, the others shorter.  rot: rotated dimensions of a head (-1: all, 0: no rotation).  norm: queries
    and keys are normalised.  `lens` seeds the lengths."""
    c = dict(op=op, hq=heads[0], hkv=heads[1], d=heads[2], decodes=decodes, ctx_lo=ctx[0], ctx_hi=ctx[1], chunks=chunks,
             chunk=chunk, prefix=prefix, lens=lens, dtype=dtype, rot=heads[2] if rot < 0 else rot, adjacent=adjacent, norm=norm)
    return dict(c, name=name) if name else c


def _attn(name, cache, heads, reqs, ctx, groups=0, prefix=(0, 0), alone=0.0, lens=1):
    """`reqs` decode requests with ctx tokens of their own.  Where groups is above 0 all but a share of `alone` belong to
    one of the groups, whose members begin with the same tokens (a length drawn from `prefix`)."""
    c = dict(op="shared" if groups else "attn8", cache=cache, hq=heads[0], hkv=heads[1], d=heads[2], reqs=reqs, ctx_lo=ctx[0],
             ctx_hi=ctx[1], groups=groups, prefix_lo=prefix[0], prefix_hi=prefix[1], alone=alone, lens=lens)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The next token of one request on an idle server: a single row, bound by the launch.
        _split("norm", "norm-decode-1", HEADS_8B, 1, (4096, 4096)),
        # A small model in float32, half of each head rotated in neighbouring pairs, ragged chunks beside decodes.
        _split("norm", "norm-f32-ragged", HEADS_SMALL, 9, (1, 3000), 3, 777, 333, lens=3, dtype="f32", rot=32, adjacent=True),
        # A late chunk of a long prompt beside running requests: the most tokens of one call.
        _split("norm", "norm-chunk-70b", HEADS_70B, 32, (2048, 2048), 1, 8192, 24576),
        # A short prompt into the 8-bit cache, read back for its attention: latency counts.
        _split("cache8", "cache8-prompt-100", HEADS_8B, 0, (1, 1), 1, 100, 0, norm=False),
        # Ragged chunks of several prompts on one tensor-parallel rank, with and without cached tokens.
        _split("cache8", "cache8-ragged-rank", HEADS_RANK, 0, (1, 1), 5, 2049, 4001, lens=5),
        # A chunk of a long prompt: written, and its whole context read back.
        _split("cache8", "cache8-chunk-8b", HEADS_8B, 0, (1, 1), 1, 8192, 24576, norm=False),
        # One running request.
        _attn("attn8-1", "e4m3", HEADS_8B, 1, (4096, 4096)),
        # Two long documents on one tensor-parallel rank: few rows, a long axis.
        _attn("attn8-long-rank", "e4m3", HEADS_RANK, 2, (65537, 131072), lens=2),
        # A loaded server.
        _attn("attn8-256-8b", "e4m3", HEADS_8B, 256, (512, 8192), lens=3),
        # A few requests that begin with the same instructions.
        _attn("shared-8", "bf16", HEADS_8B, 8, (1, 300), 1, (1000, 1000), lens=4),
        # Several products' requests, a few without a prefix, over the 8-bit cache.
        _attn("shared8-256-8b", "e4m3", HEADS_8B, 256, (16, 1500), 5, (500, 8000), 0.1, lens=5),
        # Questions about one long document, a bf16 cache.
        _attn("shared-64-70b", "bf16", HEADS_70B, 64, (200, 1000), 1, (32768, 32768), lens=6),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _cost(c):
    """About what a pass of the plain form costs, in seconds."""
    w = work(c)
    if c["op"] in ("norm", "cache8"):
        return w["bytes"] / 1e12
    longest = max(n for _, n in _contexts(c)[1])
    return w["flops"] / 1e14 + 64 * c["reqs"] * longest * c["hkv"] * c["d"] / 2e12


def draw(rng):
    op = rng.choice(["norm", "cache8", "attn8", "shared"])
    limit = max(_cost(c) for c in listed() if c["op"] == op)
    while True:
        lens = rng.randrange(1 << 20)
        heads = rng.choice([HEADS_8B, HEADS_70B, HEADS_RANK, HEADS_SMALL, (16, 2, 64), (8, 2, 128), (12, 4, 128), (6, 6, 64)])
        if op in ("norm", "cache8"):
            kinds = "prefill" if op == "cache8" and rng.random() < 0.7 else rng.choice(["decode", "prefill", "both"])
            decodes = 0 if kinds == "prefill" else _log(rng, 1, 256 if op == "norm" else 32)
            chunks = 0 if kinds == "decode" else rng.choice([1, 1, 2, 3, 5])
            chunk = _log(rng, 1, 8192) if chunks else 0
            lo = _log(rng, 1, 2000)
            prefix = _log(rng, 1, 24576) if chunks and rng.random() < 0.6 else 0
            rot = rng.choice([heads[2], heads[2], heads[2] // 2, 48, 0])
            c = _split(op, "", heads, decodes, (lo, _log(rng, lo, 4096)), chunks, chunk, prefix, lens,
                       rng.choice(["bf16", "bf16", "bf16", "f32"]) if op == "norm" else "bf16", rot, rng.random() < 0.3,
                       op == "norm" or rng.random() < 0.5)
        else:
            reqs = _log(rng, 1, 256)
            lo = _log(rng, 1, 4000)
            ctx = (lo, _log(rng, lo, 131072 if reqs < 8 else 8192))
            if op == "attn8":
                c = _attn("", "e4m3", heads, reqs, ctx, lens=lens)
            else:
                p = _log(rng, 16, 32768)
                c = _attn("", rng.choice(["bf16", "e4m3"]), heads, reqs, ctx, min(reqs, rng.choice([1, 1, 2, 5, 16])),
                          (p, _log(rng, p, 32768)), rng.choice([0.0, 0.0, 0.3]), lens)
        if _cost(c) <= limit:
            return c


# ---- the requests of a case -------------------------------------------------------------------


def _log_lengths(rng, lo, hi):
    return int(min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _requests(c):
    """(kind, new tokens, cached tokens) of each request, decodes first."""
    rng = np.random.Generator(np.random.PCG64(c["lens"]))
    reqs = [(DECODE, 1, _log_lengths(rng, c["ctx_lo"], c["ctx_hi"]) - 1) for _ in range(c["decodes"])]
    for i in range(c["chunks"]):
        q = c["chunk"] if i == 0 else _log_lengths(rng, 1, c["chunk"])
        reqs.append((PREFILL, q, c["prefix"] if i == 0 or not c["prefix"] else _log_lengths(rng, 1, c["prefix"])))
    return reqs


def _contexts(c):
    """Lengths of the groups' prefixes (whole pages), and (group or -1, all tokens) of each decode request."""
    rng = np.random.Generator(np.random.PCG64(c["lens"]))
    prefix = [PAGE * max(1, _log_lengths(rng, c["prefix_lo"], c["prefix_hi"]) // PAGE) for _ in range(c["groups"])]
    reqs = []
    for r in range(c["reqs"]):
        g = -1 if not prefix or (r >= len(prefix) and rng.random() < c["alone"]) else r % len(prefix)
        reqs.append((g, (prefix[g] if g >= 0 else 0) + _log_lengths(rng, c["ctx_lo"], c["ctx_hi"])))
    return prefix, reqs


def _meta(reqs):
    starts = np.concatenate([[0], np.cumsum([q for _, q, _ in reqs])])
    return np.array([(k, s, q, p) for (k, q, p), s in zip(reqs, starts)], dtype=np.int32)


def _table(rows, columns, lists):
    table = np.full((rows, columns), -1, dtype=np.int32)
    for r, ids in enumerate(lists):
        table[r, :len(ids)] = ids
    return torch.from_numpy(table).cuda()


def _frequencies(c):
    return [500000.0 ** (-2.0 * i / c["rot"]) for i in range(c["rot"] // 2)]


# ---- inputs -----------------------------------------------------------------------------------


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _eight_bits(x, dim):
    """x as e4m3 (bytes) and the exponents' bytes along `dim`, the head's dimensions: 448 is 1.75 times 2^8."""
    bits = x.abs().amax(dim, keepdim=True).view(torch.int32)
    e = ((bits + 0x1FFFFF) >> 23).sub_(8).clamp_(min=1)
    return (x * _power(254 - e)).to(torch.float8_e4m3fn).view(torch.uint8), e.to(torch.uint8).squeeze(dim)


def _power(e):
    """2^(e - 127) for e of 1 .. 254."""
    return (e.to(torch.int32) << 23).view(torch.float32)


def prepare(case, seed):
    """The inputs, drawn on the GPU from the seed alone, and the buffers that a serving program keeps."""
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    hkv, d = c["hkv"], c["d"]

    def normal(*shape, dtype=torch.bfloat16):
        return torch.empty(*shape, dtype=dtype, device="cuda").normal_(0.0, 1.0, generator=g)

    def pages(pool, dtype):
        """Pages of keys and of values whose tokens differ in magnitude."""
        k, v = normal(pool, hkv, PAGE, d, dtype=dtype), normal(pool, hkv, d, PAGE, dtype=dtype)
        k *= torch.exp(0.3 * normal(pool, hkv, PAGE, 1, dtype=dtype))
        v *= torch.exp(0.3 * normal(pool, hkv, 1, PAGE, dtype=dtype))
        return k, v

    def pages8(pool):
        """The same in 8 bits, some thousand pages at a time: keys' and values' bytes, exponents [pool, hkv, 2, 16]."""
        k, v = (torch.empty(pool, hkv, *s, dtype=torch.uint8, device="cuda") for s in ((PAGE, d), (d, PAGE)))
        scales = torch.empty(pool, hkv, 2, PAGE, dtype=torch.uint8, device="cuda")
        for a in range(0, pool, 8192):
            b = min(pool, a + 8192)
            x, y = pages(b - a, torch.float32)
            k[a:b], scales[a:b, :, 0] = _eight_bits(x, 3)
            v[a:b], scales[a:b, :, 1] = _eight_bits(y, 2)
        return dict(k8=k, v8=v, scales=scales)

    def order(pool):
        return torch.randperm(pool, generator=g, device="cuda", dtype=torch.int64).to(torch.int32).cpu().numpy()

    if c["op"] in ("attn8", "shared"):
        prefix, reqs = _contexts(c)
        need = [p // PAGE for p in prefix] + [-(-n // PAGE) - (prefix[i] // PAGE if i >= 0 else 0) for i, n in reqs]
        pool = int(sum(need) * 1.05) + 1
        ids, ends = order(pool), np.concatenate([[0], np.cumsum(need)])
        runs = [ids[a:b] for a, b in zip(ends[:-1], ends[1:])]
        lists = [np.concatenate([runs[i] if i >= 0 else ids[:0], runs[len(prefix) + r]]) for r, (i, _) in enumerate(reqs)]
        s = dict(case=c, meta=_meta([(DECODE, 1, n - 1) for _, n in reqs]), table=_table(len(reqs), max(map(len, lists)), lists),
                 q=normal(len(reqs), c["hq"], d), prefix_len=np.array(prefix, dtype=np.int32),
                 prefix_of=np.array([i for i, _ in reqs], dtype=np.int32))
        s["out"] = torch.empty_like(s["q"])
        if c["cache"] == "e4m3":
            s.update(pages8(pool))
        else:
            s["k"], s["v"] = pages(pool, torch.bfloat16)
        return s
    reqs = _requests(c)
    t = sum(q for _, q, _ in reqs)
    need = [-(-(cached + q) // PAGE) for _, q, cached in reqs]
    pool = int(sum(need) * 1.1) + 1
    ids, ends = order(pool), np.concatenate([[0], np.cumsum(need)])
    dt, hq = _dtype(c), c["hq"]
    x = normal(t, hq + 2 * hkv, d, dtype=dt)
    x *= torch.exp(0.5 * normal(t, hq + 2 * hkv, 1, dtype=dt))
    s = dict(case=c, meta=_meta(reqs), table=_table(len(reqs), max(need), [ids[a:b] for a, b in zip(ends[:-1], ends[1:])]),
             qkv=x.view(t, -1), q=torch.empty(t, hq, d, dtype=dt, device="cuda"), freq=_frequencies(c))
    if c["norm"]:
        s["wq"], s["wk"] = 1.0 + 0.1 * normal(d, dtype=dt), 1.0 + 0.1 * normal(d, dtype=dt)
    if c["op"] == "norm":
        s["k"], s["v"] = pages(pool, dt)
        return s
    # The pages that the requests are read back into: in order, after each other.
    s.update(pages8(pool))
    lists = [np.arange(a, b) for a, b in zip(ends[:-1], ends[1:])]
    s["out_table"] = _table(len(reqs), max(need), lists)
    s["k"] = torch.zeros(sum(need), hkv, PAGE, d, dtype=dt, device="cuda")
    s["v"] = torch.zeros(sum(need), hkv, d, PAGE, dtype=dt, device="cuda")
    return s


# ---- one pass -----------------------------------------------------------------------------------


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _run_norm, "cache8": _run_cache8, "attn8": _run_attn, "shared": _run_attn}[state["case"]["op"]](state)


def _run_own(s):
    import paper_2511_04791_amd as duet
    ctx, c = duet.default_context(), s["case"]
    if "shape" not in s:
        s["shape"] = duet.AttnShape(c["hq"], c["hkv"], c["d"], c.get("dtype", "bf16"))
        if "k8" in s:
            s["cache"] = duet.Cache8(s["k8"], s["v8"], s["scales"])
        if s.get("freq"):
            s["rope"] = duet.Rope(s["freq"], adjacent=c["adjacent"])
        if "wq" in s:
            s["norm"] = duet.HeadNorm(s["wq"], s["wk"], EPS)
    if c["op"] in ("attn8", "shared"):
        prefixes = dict(prefix_of=s["prefix_of"], prefix_len=s["prefix_len"]) if c["groups"] else {}
        cache = s["cache"] if c["cache"] == "e4m3" else (s["k"], s["v"])
        return ctx.attn_decode_shared(s["q"], cache, s["table"], s["meta"], out=s["out"], **prefixes)
    norm, rope = s.get("norm"), s.get("rope")
    if c["op"] == "norm":
        ctx.qkv_norm_rope_split(s["qkv"], s["k"], s["v"], s["table"], s["meta"], s["shape"], norm, rope, q=s["q"])
    else:
        ctx.qkv_split8(s["qkv"], s["cache"], s["table"], s["meta"], s["shape"], norm=norm, rope=rope, q=s["q"])
        ctx.cache8_read(s["cache"], s["table"], s["meta"], s["k"], s["v"], s["out_table"])
    return dict(q=s["q"], k=s["k"], v=s["v"])


def _tokens(lengths, first):
    """Request and cache position of every token first .. first + length - 1 of each request, on the GPU."""
    req = np.repeat(np.arange(len(lengths)), lengths)
    starts = np.concatenate([[0], np.cumsum(lengths)])[:-1]
    both = torch.from_numpy(np.stack([req, np.arange(len(req)) - starts[req] + first[req]])).cuda()
    return both[0], both[1]


def _turned(s):
    """Queries and keys [T, hq + hkv, d] after the norm and the rotation, in 32 bits."""
    c = s["case"]
    hq, hkv, d, rot = c["hq"], c["hkv"], c["d"], c["rot"]
    qk = s["qkv"].view(-1, hq + 2 * hkv, d)[:, :hq + hkv].float()
    if c["norm"]:
        weight = torch.cat([s["wq"].float().expand(hq, d), s["wk"].float().expand(hkv, d)])
        qk = qk * torch.rsqrt(qk.square().mean(-1, keepdim=True) + EPS) * weight
    if not rot:
        return qk
    _, pos = _tokens(s["meta"][:, 2], s["meta"][:, 3])
    angle = pos[:, None].double() * torch.tensor(s["freq"], dtype=torch.float64, device="cuda")
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    a, b = (qk[..., 0:rot:2], qk[..., 1:rot:2]) if c["adjacent"] else (qk[..., :rot // 2], qk[..., rot // 2:rot])
    ra, rb = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([ra, rb], -1).flatten(-2) if c["adjacent"] else torch.cat([ra, rb], -1)
    return torch.cat([turned, qk[..., rot:]], -1)


def _run_norm(s):
    c = s["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    req, pos = _tokens(s["meta"][:, 2], s["meta"][:, 3])
    page, slot = s["table"][req, pos // PAGE].long(), pos % PAGE
    out = _turned(s).to(s["qkv"].dtype)
    s["k"][page, :, slot] = out[:, hq:]
    s["v"][page, :, :, slot] = s["qkv"].view(-1, hq + 2 * hkv, d)[:, hq + hkv:]
    return dict(q=out[:, :hq].contiguous(), k=s["k"], v=s["v"])


def _run_cache8(s):
    c = s["case"]
    hq, hkv, d, dt = c["hq"], c["hkv"], c["d"], s["qkv"].dtype
    new, cached = s["meta"][:, 2], s["meta"][:, 3]
    req, pos = _tokens(new, cached)
    page, slot = s["table"][req, pos // PAGE].long(), pos % PAGE
    qk, v = _turned(s), s["qkv"].view(-1, hq + 2 * hkv, d)[:, hq + hkv:].float()
    s["k8"][page, :, slot], s["scales"][page, :, 0, slot] = _eight_bits(qk[:, hq:], 2)
    s["v8"][page, :, :, slot], s["scales"][page, :, 1, slot] = _eight_bits(v, 2)
    req, pos = _tokens(new + cached, 0 * cached)
    page, to, slot = s["table"][req, pos // PAGE].long(), s["out_table"][req, pos // PAGE].long(), pos % PAGE
    back = s["k8"][page, :, slot].view(torch.float8_e4m3fn).float() * _power(s["scales"][page, :, 0, slot])[..., None]
    s["k"][to, :, slot] = back.to(dt)
    back = s["v8"][page, :, :, slot].view(torch.float8_e4m3fn).float() * _power(s["scales"][page, :, 1, slot])[..., None]
    s["v"][to, :, :, slot] = back.to(dt)
    return dict(q=qk[:, :hq].to(dt).contiguous(), k=s["k"], v=s["v"])


def _run_attn(s):
    """Every request's whole context gathered and padded to the longest."""
    c = s["case"]
    hkv, d, group = c["hkv"], c["d"], c["hq"] // c["hkv"]
    at = s["table"].clamp(min=0).long()
    n, longest = at.shape[0], at.shape[1] * PAGE
    if c["cache"] == "e4m3":
        scales = s["scales"][at]
        k = s["k8"][at].view(torch.float8_e4m3fn).float() * _power(scales[:, :, :, 0])[..., None]
        v = s["v8"][at].view(torch.float8_e4m3fn).float() * _power(scales[:, :, :, 1])[:, :, :, None]
    else:
        k, v = s["k"][at].float(), s["v"][at].float()
    k = k.permute(0, 2, 1, 3, 4).reshape(n * hkv, longest, d)
    v = v.permute(0, 2, 1, 4, 3).reshape(n * hkv, longest, d)
    scores = torch.bmm(s["q"].float().view(n * hkv, group, d), k.transpose(1, 2)) / math.sqrt(d)
    tokens = torch.from_numpy(s["meta"][:, 3] + 1).cuda().repeat_interleave(hkv)
    scores.masked_fill_(torch.arange(longest, device="cuda") >= tokens[:, None, None], -math.inf)
    w = torch.exp(scores - scores.amax(-1, keepdim=True))
    return (torch.bmm(w, v) / w.sum(-1, keepdim=True)).view(n, c["hq"], d).to(torch.bfloat16)


# ---- what a pass cannot do without --------------------------------------------------------------


def work(case):
    c = case
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    if c["op"] in ("attn8", "shared"):
        prefix, reqs = _contexts(c)
        tokens = sum(n for _, n in reqs)
        held = sum(prefix) + tokens - sum(prefix[g] for g, _ in reqs if g >= 0)  # a shared token once
        return {"bytes": 2 * held * hkv * (d + 1 if c["cache"] == "e4m3" else 2 * d) + 4 * len(reqs) * hq * d,
                "flops": 4 * tokens * hq * d}
    reqs = _requests(c)
    t = sum(q for _, q, _ in reqs)
    b = 2 if c["dtype"] == "bf16" else 4
    flops = t * (hq + hkv) * (3 * c["rot"] + (4 * d if c["norm"] else 0))
    if c["op"] == "norm":
        return {"bytes": 2 * t * (hq + 2 * hkv) * d * b, "flops": flops}
    tokens = t + sum(p for _, _, p in reqs)
    return {"bytes": t * (2 * hq + 2 * hkv) * d * b + 2 * tokens * hkv * (d + 1 + d * b),
            "flops": flops + 2 * (t + tokens) * hkv * d}


# ---- the same results in 64 bits ----------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    return (_exact_attn if case["op"] in ("attn8", "shared") else _exact_split)(case, s)


def _value_of_byte(scale_bits):
    return torch.pow(2.0, scale_bits.double() - 127.0)


def _e4m3_values():
    """The value of each byte: sign, four bits of exponent with bias 7, three of fraction; 127 is no number."""
    b = torch.arange(256, device="cuda")
    e, m = (b >> 3) & 15, (b & 7).double()
    x = torch.where(e > 0, torch.pow(2.0, e.double() - 7.0) * (1.0 + m / 8), m * 2.0 ** -9)
    x[127], x[255] = math.nan, math.nan
    return torch.where(b >= 128, -x, x)


def _in_8_bits(x):
    """The values that x [..., d] is held as: multiples of an eighth of their power of two, ties to even."""
    most = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(most > 0, most, torch.ones_like(most)) / 448.0))
    e = torch.where(most > 0, e, torch.full_like(e, -126.0)).clamp(min=-126.0)
    y = x / torch.pow(2.0, e)
    own_power = torch.floor(torch.log2(torch.where(y == 0, torch.ones_like(y), y.abs()))).clamp(min=-6.0)
    step = torch.pow(2.0, own_power - 3.0)
    return torch.round(y / step) * step * torch.pow(2.0, e)


def _exact_split(c, s):
    """Request by request: each row normalised, then turned as complex numbers by exp(i angle)."""
    hq, hkv, d, half = c["hq"], c["hkv"], c["d"], c["rot"] // 2
    q = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    kc, vc, values = s["k"].double(), s["v"].double(), _e4m3_values()
    freq = torch.tensor([500000.0 ** (-i / half) for i in range(half)], dtype=torch.float64, device="cuda")
    for r, (kind, start, n, cached) in enumerate(s["meta"].tolist()):
        x = s["qkv"][start:start + n].double().view(n, hq + 2 * hkv, d)
        y = x[:, :hq + hkv].clone()
        if c["norm"]:
            y /= torch.sqrt((y * y).sum(-1, keepdim=True) / d + EPS)
            y[:, :hq] *= s["wq"].double()
            y[:, hq:] *= s["wk"].double()
        if half:
            p = cached + torch.arange(n, device="cuda", dtype=torch.float64)
            turn = torch.polar(torch.ones(n, half, dtype=torch.float64, device="cuda"), p[:, None] * freq)
            even, odd = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if c["adjacent"] else \
                (slice(0, half), slice(half, 2 * half))
            z = torch.complex(y[..., even].contiguous(), y[..., odd].contiguous()) * turn[:, None]
            y[..., even], y[..., odd] = z.real, z.imag
        q[start:start + n] = y[:, :hq]
        at = torch.arange(cached + n, device="cuda")
        page, slot = s["table"][r].long()[at // PAGE], at % PAGE
        if c["op"] == "norm":
            page, slot = page[cached:], slot[cached:]
            kc[page, :, slot], vc[page, :, :, slot] = y[:, hq:], x[:, hq + hkv:]
            continue
        to = s["out_table"][r].long()[at // PAGE]
        kc[to, :, slot] = values[s["k8"][page, :, slot].long()] * _value_of_byte(s["scales"][page, :, 0, slot])[..., None]
        vc[to, :, :, slot] = values[s["v8"][page, :, :, slot].long()] * _value_of_byte(s["scales"][page, :, 1, slot])[..., None]
        to, slot = to[cached:], slot[cached:]
        kc[to, :, slot], vc[to, :, :, slot] = _in_8_bits(y[:, hq:]), _in_8_bits(x[:, hq + hkv:])
    return dict(q=q, k=kc, v=vc)


def _exact_attn(c, s):
    """Request by request and head by head of the cache, over the context as it lies in the pages."""
    group = c["hq"] // c["hkv"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    values = _e4m3_values()
    for r, (_, _, _, cached) in enumerate(s["meta"].tolist()):
        page = s["table"][r, :cached // PAGE + 1].long()
        for h in range(c["hkv"]):
            if c["cache"] == "e4m3":
                k = values[s["k8"][page, h].long()] * _value_of_byte(s["scales"][page, h, 0])[..., None]
                v = values[s["v8"][page, h].long()] * _value_of_byte(s["scales"][page, h, 1])[:, None]
            else:
                k, v = s["k"][page, h].double(), s["v"][page, h].double()
            k = k.reshape(-1, c["d"])[:cached + 1]
            v = v.transpose(1, 2).reshape(-1, c["d"])[:cached + 1]
            q = s["q"][r, h * group:(h + 1) * group].double()
            p = torch.softmax(q @ k.t().contiguous() / math.sqrt(c["d"]), -1)
            out[r, h * group:(h + 1) * group] = p @ v
    return out
