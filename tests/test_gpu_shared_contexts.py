"""Decode attention with shared prefixes over contexts in which every page is seen on its own: counted tokens, and keys that one row each
finds.  With random keys and values a long context's result is so small beside its bound that a lost page would stay within it."""
import numpy as np
import pytest

from _helpers import to64
from test_gpu_cache_ops import BATCHES, E, U, WIDE, _bytes, _shared_batch, ctx  # noqa: F401 (the fixture)
from test_gpu_shared_prefixes import _plan

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# (heads, prefixes, requests; whether many rows go to workgroups, over bf16 and over 8-bit pages)
CONTEXTS = {
    **{name: (*WIDE[name], many) for name, many in (("few_waves", (True, False)), ("long", (False, False)), ("group3_long", (True, True)),
                                                    ("one_long", (True, True)), ("group16_long", (True, True)),
                                                    ("uploaded_long", (True, True)))},
    "document": ((64, 8, 64), [32768], [(0, 1 + 97 * i % 700) for i in range(40)], (True, True)),
    "joined": ((8, 2, 128), *BATCHES["long"], (False, False)),
    "full": ((8, 2, 128), *BATCHES["full"], (False, False)),
    "alone": ((8, 1, 128), [], [(-1, 98309), (-1, 65537), (-1, 33)], (False, False)),
}


def _context(name, cache, seed):
    import paper_2511_04791_amd as duet
    heads, prefixes, reqs, many = CONTEXTS[name]
    sh = duet.AttnShape(*heads, "bf16")
    table, meta, pool, used = _shared_batch(sh, seed, prefixes, reqs)
    of = [i for i, _ in reqs]
    assert (_plan(sh, meta, of, prefixes, cache == "e4m3")[0].many_rows > 0) == many[cache == "e4m3"]
    return sh, table, meta, pool, used, dict(prefix_of=of, prefix_len=prefixes) if prefixes else {}


def _power_bytes(x, p):
    """x [...] of 0, 1 and -1 times 2^p as bytes, p of -6 .. 8."""
    return (((p + 7) << 3) * (x != 0) + 128 * (x < 0)).astype(np.uint8)


def _spread(values, table, meta, empty):
    """values [positions, ...] at every request's tokens of a pool of `empty`."""
    for r, m in enumerate(meta):
        t = np.arange(m[3] + 1)
        empty[table[r, t // 16], :, t % 16] = values[t][:, None]
    return empty


@pytest.mark.parametrize("name", list(CONTEXTS))
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_every_token_counts_once(ctx, name, cache):  # noqa: F811
    """Queries of 0 weigh all tokens alike.  A value is 1 at the dimension of its page, and at that of its place in the row, so the result
    is how many of the tokens are of that page or place."""
    import paper_2511_04791_amd as duet
    sh, table, meta, pool, used, pre = _context(name, cache, 9800)
    hq, hkv, d = sh.num_q_heads, sh.num_kv_heads, sh.head_dim
    n = int(meta[:, 3].max()) + 1
    t = np.arange(n)
    hot = np.zeros((n, d), np.int8)
    hot[t, t // 16 % (d // 2)] = 1
    hot[t, d // 2 + t % (d // 2)] = 1
    q = torch.zeros(len(meta), hq, d, dtype=torch.bfloat16, device="cuda")
    free = torch.from_numpy(~used)[:, None]
    if cache == "bf16":
        v = torch.from_numpy(_spread(hot, table, meta, np.zeros((pool, hkv, 16, d), np.int8))).bfloat16()
        v.masked_fill_(free[..., None], float("nan"))
        k = torch.randn(pool, hkv, 16, d, device="cuda", dtype=torch.bfloat16)
        c = (k, v.transpose(2, 3).contiguous().cuda())
    else:
        p = t * 7 % 14 - 6  # the byte's power; the token's is the other way
        v = torch.from_numpy(_spread(_power_bytes(hot, p[:, None]), table, meta, np.full((pool, hkv, 16, d), 127, np.uint8)))
        s = _bytes(9801, pool, hkv, 2, 16, hi=20) + 110
        s[:, :, 1] = torch.from_numpy(_spread((127 - p).astype(np.uint8), table, meta, np.full((pool, hkv, 16), 255, np.uint8)))
        k = _bytes(9802, pool, hkv, 16, d, hi=120)
        c = duet.Cache8(k.cuda(), v.transpose(2, 3).contiguous().cuda(), s.cuda())
    out = to64(ctx.attn_decode_shared(q, c, torch.as_tensor(table, device="cuda"), meta, check_errors=True, **pre))
    # Weights are one power of two, so sums are exact: one quotient, by way of an inverse, and one rounding.
    counts = np.concatenate([np.zeros((1, d)), np.cumsum(hot, 0)])[meta[:, 3] + 1]
    want = (counts / (meta[:, 3:] + 1))[:, None]
    # A page that is lost, or taken twice, moves its dimension by more than twice the bound.
    pages, tokens = counts[:, :d // 2].max(-1), meta[:, 3] + 1.0
    assert (16 / pages - 16 / tokens > 2.5 * U)[tokens > 16].all()
    assert (np.abs(out - want) <= (U + 4 * E) * want).all(), np.argwhere(np.abs(out - want) > (U + 4 * E) * want)[:4]


@pytest.mark.parametrize("name", list(CONTEXTS))
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_every_row_finds_its_keys(ctx, name, cache):  # noqa: F811
    """Queries are rows of a Hadamard matrix, and so are a few keys, four times as large, on the borders of pages, tiles and parts; the other
    keys are 0.  A row's result is the mean of the values of its own keys."""
    import paper_2511_04791_amd as duet
    from oracle import cache8 as oc
    from scipy.linalg import hadamard
    sh, table, meta, pool, used, pre = _context(name, cache, 9900)
    hq, hkv, d = sh.num_q_heads, sh.num_kv_heads, sh.head_dim
    g, h, lens = hq // hkv, hadamard(d), meta[:, 3] + 1
    rows = (np.arange(len(meta))[:, None] * g + np.arange(hq) % g) % d  # of the matrix
    q = torch.from_numpy(h[rows]).bfloat16()

    def places(n, many, seed):
        """Up to `many` places of n tokens: the ends, then first and last tokens of pages and of tiles all along."""
        page = np.random.default_rng(seed).permutation(-(-n // 16))
        at = [0, n - 1, *np.stack([16 * page, 16 * page + 15], 1).reshape(-1)]
        return list(dict.fromkeys(int(x) for x in at if 0 <= x < n))[:many]
    keys = np.zeros((pool, hkv, 16, d), np.int8)
    found = [[[] for _ in range(hq)] for _ in meta]
    of = np.array(pre["prefix_of"]) if pre else np.full(len(meta), -1)
    for i, L in enumerate(pre.get("prefix_len", [])):
        members = np.flatnonzero(of == i)
        if not len(members) or not L:
            continue
        for x, t in enumerate(places(L, d, 9901 + i)):
            keys[table[members[0], t // 16], :, t % 16] = h[x]
            for r in members:
                for head in np.flatnonzero(rows[r] == x):
                    found[r][head].append(t)
    for r in range(len(meta)):
        before = pre["prefix_len"][of[r]] if of[r] >= 0 else 0
        if of[r] >= 0 and r % 2:
            continue
        for x, t in zip(dict.fromkeys(rows[r].tolist()), places(int(lens[r] - before), g, 9950 + r)):
            keys[table[r, (before + t) // 16], :, (before + t) % 16] = h[x]
            for head in np.flatnonzero(rows[r] == x):
                found[r][head].append(before + t)
    free = torch.from_numpy(~used)[:, None]
    if cache == "bf16":
        k, v = torch.from_numpy(keys).bfloat16() * 4, torch.randn(pool, hkv, d, 16, generator=torch.Generator().manual_seed(9902)).bfloat16()
        v = torch.where(v == 0, 1, v).masked_fill_(free[:, :, None], float("nan"))
        k.masked_fill_(free[..., None], float("nan"))
        c, values = (k.cuda(), v.cuda()), v
    else:
        s = _bytes(9903, pool, hkv, 2, 16, hi=12) + 122
        k = torch.from_numpy(_power_bytes(keys, 129 - s[:, :, 0].numpy().astype(np.int64)[..., None]))
        v = _bytes(9904, pool, hkv, d, 16, hi=80) | _bytes(9905, pool, hkv, d, 16, hi=2) << 7
        k[free[..., None].expand_as(k)], v[free[:, :, None].expand_as(v)], s[free[:, :, None].expand_as(s)] = 127, 255, 255
        c = duet.Cache8(k.cuda(), v.cuda(), s.cuda())
        values = torch.from_numpy(oc.e4m3_values())[v.int()] * torch.exp2(s[:, :, 1].double() - 127)[:, :, None]
    out = to64(ctx.attn_decode_shared(q.cuda(), c, torch.as_tensor(table, device="cuda"), meta, check_errors=True, **pre))
    # Scores are 4 sqrt(d), 32 at least: the others' weights are e^-32 each, 2^17 of them 2e-9 of the largest value.
    most = float(values[torch.isfinite(values)].abs().max())
    checked = 0
    for r in range(len(meta)):
        for head in range(hq):
            t = np.array(found[r][head])
            if not len(t):
                continue
            x = values[torch.from_numpy(table[r, t // 16].astype(np.int64)), head // g, :, torch.from_numpy(t % 16)].double().numpy()
            want, mag = x.mean(0), np.abs(x).mean(0)
            assert (np.abs(out[r, head] - want) <= U * np.abs(want) + 8 * E * mag + 4e-9 * most).all(), (r, head, t)
            checked += 1
    assert checked >= len(meta) * hq // 4
