"""Decode attention with shared prefixes where its arithmetic, its cuts and its kernels' variants end: far magnitudes and powers, against the
fp64 definition."""
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
