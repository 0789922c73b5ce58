"""Prompt attention over an 8-bit cache: chunks written by the split, the contexts read back, attended by the mixed batch, against the fp64
definition over what the cache holds."""
import numpy as np
import pytest

from _helpers import to64
from test_gpu_cache_ops import E, U, _freq, _randn, _table, ctx  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("heads", [(8, 2, 64), (12, 4, 128), (5, 5, 128)])
@pytest.mark.parametrize("rot,with_norm", [(64, True), (0, False)])
def test_chunks_of_prompts_beside_decodes(ctx, heads, rot, with_norm):  # noqa: F811
    """Three iterations: first chunks, the rest of the prompts beside the first's next token, and a token each."""
    import paper_2511_04791_amd as duet
    from oracle import cache8 as oc
    from paper_2511_04791_amd import workloads as wl
    hq, hkv, d = heads
    sh = duet.AttnShape(*heads, "bf16")
    rope, norm = duet.Rope(_freq(rot)) if rot else None, duet.HeadNorm(eps=1e-6) if with_norm else None
    lens = [33, 70, 200, 17]
    b = wl.make_batch(sh, [(0, n + 2, 0) for n in lens], page_seed=8450)
    pt, cache = _table(b), duet.Cache8.empty(b.num_phys_pages, hkv, d)
    ko, vo = (torch.full((b.num_phys_pages, hkv, *s), float("nan"), dtype=torch.bfloat16, device="cuda") for s in ((16, d), (d, 16)))
    steps = [[(0, 33, 0), (0, 20, 0), (0, 90, 0), (0, 1, 0)], [(1, 1, 33), (0, 50, 20), (0, 110, 90), (0, 16, 1)],
             [(1, 1, 34), (1, 1, 70), (1, 1, 200), (1, 1, 17)]]
    for i, step in enumerate(steps):
        meta = duet._meta_rows(step)
        x = _randn(8451 + i, int(meta[:, 2].sum()), (hq + 2 * hkv) * d).cuda()
        q = ctx.qkv_split8(x, cache, pt, meta, sh, norm=norm, rope=rope, check_errors=True)
        ctx.cache8_read(cache, pt, meta, ko, vo, pt, check_errors=True)
        out = to64(ctx.attn_mixed_batch(q, ko, vo, pt, meta, check_errors=True))
        # Every row as a decode request over what the cache holds: its own request's pages up to its place.
        values = oc.decode(*[y.cpu().numpy() for y in (cache.k, cache.v, cache.scales)])
        rows = np.array([(1, 0, 1, cached + j) for _, _, n, cached in meta.tolist() for j in range(n)])
        want, mag, most = oc.decode_attention(to64(q), *values, np.repeat(b.page_table, meta[:, 2], 0), rows)
        # Probabilities are rounded to bf16; scores are off by d half steps of their products' sum, sums by one a term; one rounding.
        n = rows[:, 3][:, None, None] + 80
        near = (1.02 * U + 2 * ((d + 4) * most[..., None] + n + 8) * E) * (mag + np.abs(want))
        bound = U * np.abs(want) + (1 + U) * near
        assert (np.abs(out - want) <= bound).all(), (i, np.argwhere(~(np.abs(out - want) <= bound))[:4])
