"""Decode attention with shared prefixes where its arithmetic, its cuts and its kernels' variants end: far magnitudes and powers, and every
variant of the kernel for many rows."""
import ctypes

import numpy as np
import pytest

from _helpers import to64
from test_gpu_cache_ops import E, U, _attn_inputs, _bytes, _shared_batch, ctx  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

LOST = 2.0 ** -80  # a weight over its row's largest, or a weight times a value, under which a token may count as nothing


def _check(got, q, values, table, meta, lost=0.0):
    """As `_check_attn` derives it, and what weights and products that count as nothing take from the result: of n tokens n times LOST of
    the largest value, and n times LOST itself."""
    from oracle import cache8 as oc
    want, mag, most = oc.decode_attention(to64(q), *values, table, meta)
    n = np.asarray(meta)[:, 3][:, None, None] + 80
    near = (1.02 * U + 2 * ((q.shape[2] + 4) * most[..., None] + n + 8) * E) * (mag + np.abs(want)) + n * lost
    err = np.abs(to64(got) - want)
    bound = U * np.abs(want) + (1 + U) * near
    assert np.isfinite(to64(got)).all() and (err <= bound).all(), (np.nanmax(err / bound), np.argwhere(~(err <= bound))[:4])


# ---- far magnitudes -------------------------------------------------------------------------------

FAR = {
    # a wave alone, a team, both straight to the result; runs that are joined; a prefix for few rows and one for many
    "lone": ((4, 2, 128), [], [(-1, n) for n in (1, 16, 33, 64)]),
    "team": ((8, 1, 64), [], [(-1, n) for n in (65, 200, 256)]),
    "joined": ((4, 2, 128), [], [(-1, 9000), (-1, 3), (-1, 2600)]),
    "few_rows": ((16, 2, 64), [1040], [(0, 1), (0, 300), (-1, 40)]),
    "many_rows": ((32, 8, 128), [4016], [(0, 1 + i % 40) for i in range(60)]),
}


@pytest.mark.parametrize("name", list(FAR))
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_values_next_to_the_largest(ctx, name, cache):  # noqa: F811
    """Their weighted mean is finite, so the result is: also where scores rise by less than moves the reference maximum, so that weights
    are above 1 before they are divided."""
    import paper_2511_04791_amd as duet
    from oracle import cache8 as oc
    heads, prefixes, reqs = FAR[name]
    hq, hkv, d = heads
    table, meta, pool, used = _shared_batch(duet.AttnShape(*heads, "bf16"), 9500, prefixes, reqs)
    # scores of 0 for 256 tokens and 7.5 powers of two for 256
    q = torch.full((len(reqs), hq, d), 7.5 * np.log(2.0) / np.sqrt(d)).bfloat16()
    k = torch.zeros(pool, hkv, 16, d, dtype=torch.uint8)
    for r, m in enumerate(meta):
        t = np.arange(m[3] + 1)
        t = t[t % 512 >= 256]
        k[table[r, t // 16], :, t % 16] = 0x38  # 1
    # 2^7 to 1.75 2^8 of either sign, half of the dimensions above 0, times 2^119
    v = _bytes(9501, pool, hkv, d, 16, hi=15) + 0x70
    v[:, :, d // 2:] |= _bytes(9502, pool, hkv, d // 2, 16, hi=2) << 7
    free = torch.from_numpy(~used)
    k[free[:, None, :, None].expand_as(k)], v[free[:, None, None].expand_as(v)] = 127, 127
    scales = torch.full((pool, hkv, 2, 16), 127, dtype=torch.uint8)
    scales[:, :, 1] = 246
    values = oc.decode(k.numpy(), v.numpy(), scales.numpy())
    if cache == "e4m3":
        c = duet.Cache8(k.cuda(), v.cuda(), scales.cuda())
    else:
        c = tuple(torch.from_numpy(x).bfloat16().cuda() for x in values)
    pre = dict(prefix_of=[i for i, _ in reqs], prefix_len=prefixes) if prefixes else {}
    out = ctx.attn_decode_shared(q.cuda(), c, torch.as_tensor(table, device="cuda"), meta, check_errors=True, **pre)
    _check(out, q, values, table, meta, LOST * 2.0 ** 128)
    if prefixes:
        assert (_plan(duet.AttnShape(*heads, "bf16"), meta, pre["prefix_of"], prefixes, cache == "e4m3")[0].many_rows > 0) == (name == "many_rows")


@pytest.mark.parametrize("name", list(FAR))
@pytest.mark.parametrize("powers", ["values", "small_values", "small_keys", "large_keys"])
def test_powers_of_the_whole_range(ctx, name, powers):  # noqa: F811
    """Tokens' powers from the smallest to the largest that the split stores, next to each other; keys' ones beside queries of the other
    end."""
    import paper_2511_04791_amd as duet
    from oracle import cache8 as oc
    heads, prefixes, reqs = FAR[name]
    sh = duet.AttnShape(*heads, "bf16")
    table, meta, pool, used = _shared_batch(sh, 9600, prefixes, reqs)
    q, c, _ = _attn_inputs(sh, "e4m3", 9601, pool, used, len(reqs))
    scales = c.scales.cpu()
    held = torch.from_numpy(used)[:, None].expand(pool, heads[1], 16)
    e = {"values": _bytes(9602, *held.shape, hi=246) + 1, "small_values": _bytes(9602, *held.shape, hi=16) + 1,
         "small_keys": scales[:, :, 0] - 100, "large_keys": scales[:, :, 0] + 100}[powers]
    side = int(powers.endswith("values"))
    scales[:, :, side] = torch.where(held, e, scales[:, :, side])
    if powers.endswith("keys"):
        q = q * (2.0 ** 100 if powers == "small_keys" else 2.0 ** -100)
    c = duet.Cache8(c.k, c.v, scales.cuda())
    values = oc.decode(c.k.cpu().numpy(), c.v.cpu().numpy(), scales.numpy())
    pre = dict(prefix_of=[i for i, _ in reqs], prefix_len=prefixes) if prefixes else {}
    out = ctx.attn_decode_shared(q.cuda(), c, torch.as_tensor(table, device="cuda"), meta, check_errors=True, **pre)
    most = max(1.0, np.abs(np.where(np.isfinite(values[1]), values[1], 0)).max())
    _check(out, q, values, table, meta, LOST * most)


# ---- how a batch is cut ---------------------------------------------------------------------------


def _plan(sh, meta, prefix_of, prefix_len, eight):
    """(what the library says of the call, rows that each prefix is taken with)"""
    import paper_2511_04791_amd as duet
    from paper_2511_04791_amd import _native as N
    b, cut, rows = duet._BatchC(meta), N.SharedCut(), (ctypes.c_int32 * max(1, len(prefix_len)))()
    p = N.Prefixes(len(prefix_len), *[(ctypes.c_int32 * max(1, len(x)))(*x) for x in (prefix_len, prefix_of)])
    N.check(N.lib().duet_shared_plan(ctypes.byref(duet._shape_c(sh)), ctypes.byref(b.c), ctypes.byref(p), int(eight), ctypes.byref(cut), rows),
            "duet_shared_plan")
    return cut, list(rows)


def _meta(prefixes, reqs):
    return np.array([(1, r, 1, (prefixes[i] if i >= 0 else 0) + n - 1) for r, (i, n) in enumerate(reqs)], np.int32)


# Rows of a kv head by the tables that their batch needs: (query heads a kv head, members of the prefix looked at, of another one long enough
# that both go to workgroups of many rows, requests alone).  One to eight waves, and two blocks of rows, none of them full.
ROWS = {32: [(15, m, min(30 - m, 17), 1) for m in (2, 4, 6, 8, 10, 12, 14, 16)] + [(15, 18, 12, 1)],
        256: [(3, 10, 160, 9), (3, 50, 160, 9), (3, 75, 160, 9), (5, 53, 160, 9)],
        0: [(3, 10, 170, 90), (3, 32, 170, 60), (3, 64, 170, 30), (5, 60, 100, 100)]}
KINDS = [(cache, d, tables, *r) for cache in ("bf16", "e4m3") for d in (64, 128) for tables in (32, 256, 0) for r in ROWS[tables]
         if r[0] * r[1] > (48 if cache == "e4m3" else 32 if d == 64 else 16)]  # fewer rows always go to teams


def _many_rows(cache, d, tables, group, members, others, alone, hkv=4):
    """A batch whose first prefix goes to workgroups of many rows: the first such lengths of both, no whole tiles."""
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(group * hkv, hkv, d, "bf16")
    for first in (1008, 208):
        for second in (1040, 2000, 4016, 8048, 16016, 32048, 64080):
            prefixes = [first, second]
            reqs = [(0, i * 7 % 40) for i in range(members)] + [(1, i * 5 % 30) for i in range(others)] + [(-1, 1 + i % 70) for i in range(alone)]
            reqs = [reqs[i] for i in np.random.default_rng(9700).permutation(len(reqs))]
            cut, rows = _plan(sh, _meta(prefixes, reqs), [i for i, _ in reqs], prefixes, cache == "e4m3")
            if rows[0] > 16:
                blocks = -(-group * members // 256)
                assert rows[0] == 32 * -(-(-(-group * members // 32)) // blocks)
                assert cut.tables == tables and cut.many_rows > 0 and not cut.direct
                return sh, prefixes, reqs
    raise AssertionError("no length sends these rows to workgroups of many")


@pytest.mark.parametrize("cache,d,tables,group,members,others,alone", KINDS)
def test_every_kind_of_many_rows(ctx, cache, d, tables, group, members, others, alone):  # noqa: F811
    """Also with pages outside the pool in both prefixes, which do not count and are reported."""
    import paper_2511_04791_amd as duet
    sh, prefixes, reqs = _many_rows(cache, d, tables, group, members, others, alone)
    table, meta, pool, used = _shared_batch(sh, 9701, prefixes, reqs)
    q, c, values = _attn_inputs(sh, cache, 9702, pool, used, len(reqs))
    pre = dict(prefix_of=[i for i, _ in reqs], prefix_len=prefixes)
    first, second, rest = ([r for r, (i, _) in enumerate(reqs) if i == x] for x in (0, 1, -1))
    # rows of every wave of both blocks, both ends, and some of the other requests
    some = sorted({*first[::7], first[-1], second[0], second[-1], rest[0]})
    bad = table.copy()
    for x, n in ((first, prefixes[0] // 16), (second, prefixes[1] // 16)):
        for j, page in ((0, -1), (5, pool), (n - 2, 2 ** 31 - 1), (n - 1, -7)):
            bad[x, j] = page
    out = torch.empty_like(q, device="cuda")
    for t in (table, bad):
        out.fill_(float("nan"))
        args = (q.cuda(), c, torch.as_tensor(t, device="cuda"), meta)
        if t is bad:
            with pytest.raises(duet.DuetError) as e:
                ctx.attn_decode_shared(*args, out=out, check_errors=True, **pre)
            assert e.value.code == -6
        else:
            ctx.attn_decode_shared(*args, out=out, check_errors=True, **pre)
        assert torch.isfinite(out).all()
        _check(out[some], q[some], values, t[some], meta[some])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tables", [32, 256, 0])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_infinite_and_nan_scores_of_many_rows(ctx, cache, d, tables):  # noqa: F811
    """Of many rows' prefix: a NaN key makes all its rows NaN and no others, keys of -inf weigh nothing."""
    sh, prefixes, reqs = _many_rows(cache, d, tables, *ROWS[tables][3])
    table, meta, pool, used = _shared_batch(sh, 9711, prefixes, reqs)
    q, c, values = _attn_inputs(sh, cache, 9712, pool, used, len(reqs))
    q = q.abs() + 0.1
    first = [r for r, (i, _) in enumerate(reqs) if i == 0]
    some, others = [first[0], first[len(first) // 2], first[-1]], [r for r, (i, _) in enumerate(reqs) if i != 0]
    pre = dict(prefix_of=[i for i, _ in reqs], prefix_len=prefixes)
    pt, q_gpu = torch.as_tensor(table, device="cuda"), q.cuda()
    if cache == "bf16":
        k = c[0].cpu()
        for page in (0, 1, 2, 3, 4, prefixes[0] // 16 - 1):  # a whole tile and more, and the last page
            k[table[first[0], page]] = float("-inf")
        c = (k.cuda(), c[1])
        out = ctx.attn_decode_shared(q_gpu, c, pt, meta, **pre)
        gone = table.copy()
        gone[np.ix_(first, [0, 1, 2, 3, 4, prefixes[0] // 16 - 1])] = -1  # as if these were outside the pool
        _check(out[some], q[some], (np.where(np.isfinite(to64(k)), to64(k), 0), values[1]), gone[some], meta[some])
        k[table[first[0], prefixes[0] // 16 - 2], :, 15] = float("nan")
        c = (k.cuda(), c[1])
    else:
        c.k[int(table[first[0], prefixes[0] // 16 - 2]), :, 15, 3] = 127
    out = ctx.attn_decode_shared(q_gpu, c, pt, meta, **pre)
    assert torch.isnan(out[first]).all() and torch.isfinite(out[others]).all()


@pytest.mark.parametrize("d,tables", [(64, 32), (128, 32), (64, 256), (64, 0)])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_many_rows_in_a_graph(ctx, cache, d, tables):  # noqa: F811
    sh, prefixes, reqs = _many_rows(cache, d, tables, *ROWS[tables][3])
    table, meta, pool, used = _shared_batch(sh, 9721, prefixes, reqs)
    q, c, values = _attn_inputs(sh, cache, 9722, pool, used, len(reqs))
    pre = dict(prefix_of=[i for i, _ in reqs], prefix_len=prefixes)
    pt, x, g = torch.as_tensor(table, device="cuda"), q.cuda(), torch.cuda.CUDAGraph()
    out = torch.empty_like(x)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        ctx.attn_decode_shared(x, c, pt, meta, out=out, **pre)
    for i in range(3):
        x.copy_(q * (1 - 0.25 * i))
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ctx.attn_decode_shared(x, c, pt, meta, **pre))
        ctx.attn_decode_shared(x[:1], c, pt[:1], meta[:1])
    some = slice(0, len(reqs), 29)
    _check(out[some], x.cpu()[some], values, table[some], meta[some])
