"""GPU parity of the head norms in the rotating split, of the 8-bit cache and of decode attention with shared prefixes with
their fp64 definitions, at the sizes, layouts and masks where they can go wrong."""
import numpy as np
import pytest

from _helpers import to64

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -8   # half a step of bf16, relative
E = 2.0 ** -24  # of fp32
Q = 2.0 ** -4   # of e4m3


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2511_04791_amd as duet
    c = duet.Context(0)
    yield c
    c.close()


def _randn(seed, *shape, scale=1.0, dtype=torch.bfloat16):
    gen = torch.Generator(device="cpu")
    gen.manual_seed(seed)
    return (torch.randn(*shape, generator=gen) * scale).to(dtype)


def _bytes(seed, *shape, hi=256):
    gen = torch.Generator(device="cpu")
    gen.manual_seed(seed)
    return torch.randint(0, hi, shape, generator=gen, dtype=torch.int32).to(torch.uint8)


def _table(b):
    return torch.as_tensor(b.page_table, device="cuda")


# ---- the split with a norm ------------------------------------------------------------------------

REQUESTS = {
    # whole pages, pages covered in part at either end or both, one row, every start in a page
    "pages": [(0, 16, 0), (0, 48, 32), (0, 17, 15), (0, 31, 1), (0, 15, 0), (0, 2, 15), (1, 1, 16)],
    "starts": [(0, 40 + s, s) for s in range(16)],
    "one": [(1, 1, 5000)],
    # more requests than travel with one launch's arguments, and than one round of the search takes
    "many": [(1, 1, 7 * i % 90) for i in range(300)] + [(0, 33, 20), (1, 1, 3), (0, 1, 0)],
}


def _inputs(sh, reqs, seed):
    from paper_2511_04791_amd import workloads as wl
    b = wl.make_batch(sh, reqs, page_seed=seed)
    dt = torch.bfloat16 if sh.dtype == "bf16" else torch.float32
    qkv = _randn(seed + 3, b.num_tokens, (sh.num_q_heads + 2 * sh.num_kv_heads) * sh.head_dim, dtype=dt)
    qkv *= torch.exp2(torch.arange(b.num_tokens) % 7 - 3).to(dt)[:, None]
    w = [_randn(seed + 4 + i, sh.head_dim, scale=0.3, dtype=dt) + 1 for i in range(2)]
    return b, qkv, w


def _freq(rot, theta=10000.0):
    return [theta ** (-2.0 * i / rot) for i in range(rot // 2)]


def _near(sh, qkv, norm, rope, b, table):
    """How far the kernel's fp32 queries and keys may be from the exact ones, as (q, k cache): the norm is off by at most 20 half
    steps (sums of squares over 16 of a lane's values and 4 lanes' moves, halved by the root; mean, eps, root, quotient, two products), sine
    and cosine by 3, the two products and their sum by one each."""
    from oracle import cache8 as oc, serving as so
    hq, hkv, d = sh.num_q_heads, sh.num_kv_heads, sh.head_dim
    x = np.abs(to64(qkv) if norm is None else oc.normalised(to64(qkv), hq, hkv, d, *norm)).reshape(len(qkv), -1, d)
    mag = x.copy()
    if rope is not None:
        n = len(rope[0])
        i = np.arange(n)
        p, q = (2 * i, 2 * i + 1) if rope[1] else (i, i + n)
        mag[..., p] = mag[..., q] = x[..., p] + x[..., q]
    zeros = np.zeros((b.num_phys_pages, hkv, 16, d))
    mq, mk, _ = so.rope_split(mag.reshape(len(qkv), -1), zeros, zeros.transpose(0, 1, 3, 2), table, b.seq_meta, hq, hkv, d, [0.0], False)
    f = ((20 if norm is not None else 0) + (6 if rope is not None else 0)) * E
    return f * mq, f * mk


SHAPES = [((4, 2, 128), "bf16", 128, False), ((6, 3, 64), "bf16", 64, True), ((20, 4, 128), "bf16", 48, False),
          ((8, 1, 128), "bf16", 80, True), ((2, 1, 64), "bf16", 16, False), ((5, 5, 64), "bf16", 0, False)]
F32_SHAPES = [((2, 2, 64), "f32", 64, False), ((5, 1, 64), "f32", 16, True), ((4, 2, 128), "f32", 112, True), ((3, 1, 128), "f32", 0, False)]


@pytest.mark.parametrize("name", list(REQUESTS))
@pytest.mark.parametrize("heads,dtype,rot,adjacent", SHAPES + F32_SHAPES)
def test_norm_split(ctx, name, heads, dtype, rot, adjacent):
    import paper_2511_04791_amd as duet
    from oracle import cache8 as oc
    sh = duet.AttnShape(*heads, dtype)
    b, qkv, w = _inputs(sh, REQUESTS[name], 7000)
    hq, hkv, d, P = *heads, b.num_phys_pages
    kc, vc = _randn(7001, P, hkv, 16, d, dtype=qkv.dtype), _randn(7002, P, hkv, d, 16, dtype=qkv.dtype)
    kg, vg = kc.cuda(), vc.cuda()
    weights = (w[0], None) if name == "starts" else (None, w[1]) if name == "one" else tuple(w)
    norm = duet.HeadNorm(*[x.cuda() if x is not None else None for x in weights], eps=1e-5)
    rope = duet.Rope(_freq(rot), adjacent=adjacent) if rot else None
    q = ctx.qkv_norm_rope_split(qkv.cuda(), kg, vg, _table(b), b.seq_meta, sh, norm, rope, check_errors=True)
    n64 = (*[to64(x) if x is not None else None for x in weights], np.float64(np.float32(1e-5)))
    r64 = (_freq(rot), adjacent) if rot else None
    want = oc.norm_split(to64(qkv), to64(kc), to64(vc), b.page_table, b.seq_meta, hq, hkv, d, n64, r64)
    near = _near(sh, qkv, n64, r64, b, b.page_table)
    rel = U if dtype == "bf16" else E
    for what, g, x, m in zip(("q", "k"), (q, kg), want, near):
        err, touched = np.abs(to64(g) - x), m > 0
        bound = np.where(touched | (what == "q"), rel * np.abs(x) + (1 + rel) * m, 0.0)
        assert (err <= bound).all(), (what, err.max(), np.argwhere(err > bound)[:5])
    assert np.array_equal(to64(vg), want[2])


def test_norm_split_positions_and_streams(ctx):
    """Given positions on three axes, on another stream, the same bits with and without a workspace."""
    import paper_2511_04791_amd as duet
    from oracle import cache8 as oc
    sh = duet.AttnShape(4, 2, 128, "bf16")
    b, qkv, w = _inputs(sh, REQUESTS["pages"], 7100)
    pos = np.random.default_rng(7101).integers(-50, 70000, size=(3, b.num_tokens)).astype(np.int32)
    axis = [i % 3 for i in range(32)]
    kc, vc = torch.zeros(b.num_phys_pages, 2, 16, 128, dtype=torch.bfloat16), torch.zeros(b.num_phys_pages, 2, 128, 16, dtype=torch.bfloat16)
    norm, rope = duet.HeadNorm(w[0].cuda(), w[1].cuda(), 1e-6), duet.Rope(_freq(64), pair_axis=axis, axes=3)
    x, p = qkv.cuda(), torch.as_tensor(pos, device="cuda")
    got, st = [], torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(2):
        kg, vg = kc.cuda(), vc.cuda()
        torch.cuda.synchronize()
        q = ctx.qkv_norm_rope_split(x, kg, vg, _table(b), b.seq_meta, sh, norm, rope, positions=p, stream=st.cuda_stream,
                                    check_errors=bool(i))
        torch.cuda.synchronize()
        got.append((q, kg, vg))
    assert all(torch.equal(a, c) for a, c in zip(*got))
    n64, r64 = (to64(w[0]), to64(w[1]), np.float64(np.float32(1e-6))), (_freq(64), False, axis, pos)
    want = oc.norm_split(to64(qkv), to64(kc), to64(vc), b.page_table, b.seq_meta, 4, 2, 128, n64, r64)
    near = _near(sh, qkv, n64, r64, b, b.page_table)
    for g, y, m in zip(got[0][:2], want, near):
        assert (np.abs(to64(g) - y) <= U * np.abs(y) + (1 + U) * m).all()


def test_norm_of_zeros_and_of_far_magnitudes(ctx):
    """Rows of zeros stay zero, tiny rows are carried by eps, rows near fp32's root stay finite."""
    import paper_2511_04791_amd as duet
    from oracle import cache8 as oc
    sh = duet.AttnShape(2, 1, 64, "f32")
    b, qkv, _ = _inputs(sh, [(0, 5, 0)], 7150)
    qkv *= torch.tensor([0.0, 1e-20, 1e-3, 1e15, 1.0])[:, None]
    kc, vc = torch.zeros(b.num_phys_pages, 1, 16, 64), torch.zeros(b.num_phys_pages, 1, 64, 16)
    kg, vg = kc.cuda(), vc.cuda()
    q = ctx.qkv_norm_rope_split(qkv.cuda(), kg, vg, _table(b), b.seq_meta, sh, duet.HeadNorm(eps=1e-6))
    n64 = (None, None, np.float64(np.float32(1e-6)))
    want = oc.norm_split(to64(qkv), to64(kc), to64(vc), b.page_table, b.seq_meta, 2, 1, 64, n64, None)
    # squares below fp32's smallest are lost, of rows that eps carries alone
    assert np.isfinite(to64(q)).all() and (np.abs(to64(q) - want[0]) <= 21 * E * np.abs(want[0]) + 1e-30).all()
    assert (to64(q)[0] == 0).all()


# ---- the 8-bit cache ------------------------------------------------------------------------------


def _cache8(seed, P, hkv, d):
    """Any bytes, the not-a-number ones among them."""
    return _bytes(seed, P, hkv, 16, d), _bytes(seed + 1, P, hkv, d, 16), _bytes(seed + 2, P, hkv, 2, 16)


def _written(b, table, hkv):
    """[P, h_kv, 16]: the slots that the batch's new tokens take."""
    from oracle import serving as so
    w = np.zeros((b.num_phys_pages, hkv, 16), bool)
    req, pos = so.token_places(b.seq_meta)
    page = np.asarray(table)[req, pos // 16]
    ok = (page >= 0) & (page < b.num_phys_pages)
    w[page[ok], :, pos[ok] % 16] = True
    return w


def _check_split8(sh, b, qkv, norm, rope, before, after, q, table=None):
    from oracle import cache8 as oc
    hq, hkv, d = sh.num_q_heads, sh.num_kv_heads, sh.head_dim
    table = b.page_table if table is None else table
    zeros = np.zeros((b.num_phys_pages, hkv, 16, d))
    want = oc.norm_split(to64(qkv), zeros, zeros.transpose(0, 1, 3, 2), table, b.seq_meta, hq, hkv, d, norm, rope)
    nq, nk = _near(sh, qkv, norm, rope, b, table)
    assert (np.abs(to64(q) - want[0]) <= U * np.abs(want[0]) + (1 + U) * nq).all()
    k0, v0, s0 = (x.numpy() for x in before)
    k1, v1, s1 = (x.cpu().numpy() for x in after)
    w = _written(b, table, hkv)
    # what is not written stays
    assert np.array_equal(k1[~w], k0[~w]) and np.array_equal(v1.transpose(0, 1, 3, 2)[~w], v0.transpose(0, 1, 3, 2)[~w])
    assert np.array_equal(s1[:, :, 0][~w], s0[:, :, 0][~w]) and np.array_equal(s1[:, :, 1][~w], s0[:, :, 1][~w])
    # values: a copy, so the very bytes
    val = oc.e4m3_values()
    x, e = oc.encode(want[2].transpose(0, 1, 3, 2)[w])
    assert np.array_equal(s1[:, :, 1][w], e)
    assert np.array_equal(val[v1.transpose(0, 1, 3, 2)[w]], x, equal_nan=True)
    # keys: the very bytes without norm and rotation, else within half a step of what is near the exact ones
    y, got = want[1][w], val[k1[w]]
    if norm is None and rope is None:
        x, e = oc.encode(y)
        assert np.array_equal(s1[:, :, 0][w], e) and np.array_equal(got, x, equal_nan=True)
        return
    s, most = 2.0 ** (s1[:, :, 0][w].astype(np.float64) - 127), np.abs(y).max(-1)
    slack = 1 + nk[w].max(-1) / np.where(most > 0, most, 1)
    assert (most <= 448 * s * slack).all() and ((most * slack >= 224 * s) | (s1[:, :, 0][w] == 1)).all()
    err = np.abs(got * s[:, None] - y)
    assert (err <= np.maximum(Q * np.abs(y), 2.0 ** -10 * s[:, None]) + (1 + Q) * nk[w]).all(), err.max()


@pytest.mark.parametrize("name", list(REQUESTS))
@pytest.mark.parametrize("heads,dtype,rot,adjacent", SHAPES)
@pytest.mark.parametrize("with_norm", [False, True])
def test_split8(ctx, name, heads, dtype, rot, adjacent, with_norm):
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(*heads, dtype)
    b, qkv, w = _inputs(sh, REQUESTS[name], 7200)
    before = _cache8(7201, b.num_phys_pages, heads[1], heads[2])
    cache = duet.Cache8(*[x.cuda() for x in before])
    norm = duet.HeadNorm(w[0].cuda(), w[1].cuda(), 1e-6) if with_norm else None
    rope = duet.Rope(_freq(rot), adjacent=adjacent) if rot else None
    q = ctx.qkv_split8(qkv.cuda(), cache, _table(b), b.seq_meta, sh, norm=norm, rope=rope, check_errors=True)
    n64 = (to64(w[0]), to64(w[1]), np.float64(np.float32(1e-6))) if with_norm else None
    _check_split8(sh, b, qkv, n64, (_freq(rot), adjacent) if rot else None, before, (cache.k, cache.v, cache.scales), q)


def test_split_of_many_requests(ctx):
    """More groups of workgroups than one dimension of the grid takes, of one row each and of more."""
    import paper_2511_04791_amd as duet
    from oracle import cache8 as oc
    sh = duet.AttnShape(1, 1, 64, "bf16")
    for rows, R in ((1, 33000), (2, 16500)):
        meta = duet._meta_rows([(1 if rows == 1 else 0, rows, 3)] * R)
        pt = torch.arange(R, dtype=torch.int32, device="cuda").view(R, 1)
        qkv = _randn(7260, R * rows, 3 * 64)
        cache = duet.Cache8.empty(R, 1, 64)
        q = ctx.qkv_split8(qkv.cuda(), cache, pt, meta, sh, check_errors=True)
        assert torch.equal(q.cpu()[:, 0], qkv[:, :64])
        val = oc.e4m3_values()
        want, e = oc.encode(to64(qkv)[:, 64:].reshape(-1, 2, 64))
        k, v, s = cache.k.cpu().numpy()[:, 0, 3:3 + rows], cache.v.cpu().numpy()[:, 0, :, 3:3 + rows], cache.scales.cpu().numpy()[:, 0, :, 3:3 + rows]
        assert np.array_equal(val[k].reshape(-1, 64), want[:, 0]) and np.array_equal(val[v.transpose(0, 2, 1)].reshape(-1, 64), want[:, 1])
        assert np.array_equal(s.transpose(0, 2, 1).reshape(-1, 2), e)
        assert int((cache.k != 0).sum()) <= R * rows * 64


def test_split8_of_special_values(ctx):
    """Zeros, what is not finite, the smallest and largest magnitudes, the largest value on and next to a power's border."""
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(1, 1, 64, "bf16")
    b, qkv, _ = _inputs(sh, [(0, 40, 3)], 7300)
    x = qkv.view(40, 3, 64)
    inf, nan, big, tiny = float("inf"), float("nan"), torch.finfo(torch.bfloat16).max, 2.0 ** -133
    x[0] = 0.0
    x[1] = -0.0
    x[2, :, 5], x[3, :, 6], x[4, :, 7] = inf, -inf, nan
    x[5] = inf
    x[6] = nan
    x[7, :, 9], x[8, :, 63] = big, -big
    x[9] *= 2.0 ** -130
    x[10] = tiny
    x[11] *= 2.0 ** 120
    for i, v in enumerate([448.0, 450.0, 1.75, 1.7578125, 1.7421875, 2.0 ** -118, 1.75 * 2.0 ** -118, 1.7578125 * 2.0 ** -118]):
        x[12 + i].clamp_(-abs(v), abs(v))
        x[12 + i, :, i] = -v
    # every tie of the grid, in rows whose largest value is 448
    ties = torch.tensor([a * 2.0 ** p for p in range(-8, 8) for a in (1.0625, 1.1875, 1.9375)])[:40]
    x[30, :, 0], x[30, :, 1:41] = 448.0, ties
    x[31, :, 0], x[31, :, 1:17] = -448.0, -(torch.arange(16) + 0.5) * 2.0 ** -9
    before = _cache8(7301, b.num_phys_pages, 1, 64)
    cache = duet.Cache8(*[t.cuda() for t in before])
    q = ctx.qkv_split8(qkv.cuda(), cache, _table(b), b.seq_meta, sh)
    assert torch.equal(q.cpu().view(torch.int16), x[:, :1].contiguous().view(torch.int16))
    from oracle import cache8 as oc
    req, val = to64(x), oc.e4m3_values()
    k1, v1, s1 = (t.cpu().numpy() for t in (cache.k, cache.v, cache.scales))
    for t in range(40):
        page, slot = b.page_table[0, (3 + t) // 16], (3 + t) % 16
        for got, e, y in ((k1[page, 0, slot], s1[page, 0, 0, slot], req[t, 1]), (v1[page, 0, :, slot], s1[page, 0, 1, slot], req[t, 2])):
            want, we = oc.encode(y)
            assert e == we, t
            assert np.array_equal(val[got], want, equal_nan=True), t


@pytest.mark.parametrize("name", ["pages", "many"])
def test_split8_pages_outside_the_pool(ctx, name):
    """Skipped and reported; everything else is written."""
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(4, 2, 64, "bf16")
    b, qkv, w = _inputs(sh, REQUESTS[name], 7350)
    table = b.page_table.copy()
    table[0, 0], table[1, 3 if name == "pages" else 0], table[len(table) - 1, 0] = -1, b.num_phys_pages, 2 ** 31 - 1
    before = _cache8(7351, b.num_phys_pages, 2, 64)
    ws = torch.full((1 << 16,), 255, dtype=torch.uint8, device="cuda")
    norm = duet.HeadNorm(w[0].cuda(), w[1].cuda(), 1e-6)
    n64 = (to64(w[0]), to64(w[1]), np.float64(np.float32(1e-6)))
    q = torch.empty(b.num_tokens, 4, 64, dtype=torch.bfloat16, device="cuda")
    cache = duet.Cache8(*[x.cuda() for x in before])
    with pytest.raises(duet.DuetError) as e:
        ctx.qkv_split8(qkv.cuda(), cache, torch.as_tensor(table, device="cuda"), b.seq_meta, sh, norm=norm, q=q, workspace=ws,
                       check_errors=True)
    assert e.value.code == -6
    _check_split8(sh, b, qkv, n64, None, before, (cache.k, cache.v, cache.scales), q, table)
    ctx.qkv_split8(qkv.cuda(), cache, _table(b), b.seq_meta, sh, norm=norm, workspace=ws, check_errors=True)


READS = {
    "lengths": [(1, 1, n - 1) for n in (1, 2, 15, 16, 17, 31, 32, 33, 100)] + [(0, 30, 40), (0, 16, 0)],
    "one": [(0, 1, 0)],
    "many": [(1, 1, 7 * i % 90) for i in range(300)],
    "long": [(0, 100, 4000)],
}


@pytest.mark.parametrize("name", list(READS))
@pytest.mark.parametrize("hkv,d", [(1, 128), (3, 64), (8, 128)])
@pytest.mark.parametrize("with_errors", [False, True])
def test_cache8_read(ctx, name, hkv, d, with_errors):
    """Every byte and every power; slots past the last token stay."""
    import paper_2511_04791_amd as duet
    from oracle import cache8 as oc
    from paper_2511_04791_amd import workloads as wl
    sh = duet.AttnShape(hkv, hkv, d, "bf16")
    b = wl.make_batch(sh, READS[name], page_seed=7400)
    k, v, s = _cache8(7401, b.num_phys_pages, hkv, d)
    s[s == 255] = 254
    out = wl.make_batch(sh, READS[name], page_seed=7500)
    k0, v0 = _randn(7402, out.num_phys_pages, hkv, 16, d), _randn(7403, out.num_phys_pages, hkv, d, 16)
    ko, vo = k0.cuda(), v0.cuda()
    ctx.cache8_read(duet.Cache8(k.cuda(), v.cuda(), s.cuda()), _table(b), b.seq_meta, ko, vo, _table(out), check_errors=with_errors)
    kd, vd = oc.decode(k.numpy(), v.numpy(), s.numpy())
    kw, vw = to64(k0), to64(v0)
    for r, m in enumerate(b.seq_meta):
        t = np.arange(m[2] + m[3])
        src, dst, slot = b.page_table[r, t // 16], out.page_table[r, t // 16], t % 16
        kw[dst, :, slot], vw[dst, :, :, slot] = kd[src, :, slot], vd[src, :, :, slot]
    # Four significant bits at 2^(e - 127): exact in bf16 but above 1.9375 2^127, its largest with those, where infinities follow, and
    # below 2^-126, where e4m3's smallest step, 2^-9, times a power of 2^-126 or 2^-125 falls under bf16's smallest, 2^-133: rounded there.
    for got, want in ((ko, kw), (vo, vw)):
        want = torch.from_numpy(want).float().bfloat16()
        assert np.array_equal(to64(got), to64(want), equal_nan=True)


def test_cache8_read_pages_outside_the_pools(ctx):
    """Neither read nor written, and reported; the next call with the workspace starts clean."""
    import paper_2511_04791_amd as duet
    from paper_2511_04791_amd import workloads as wl
    sh = duet.AttnShape(2, 2, 64, "bf16")
    b = wl.make_batch(sh, [(0, 40, 0), (1, 1, 50), (1, 1, 20)], page_seed=7600)
    k, v, s = _cache8(7601, b.num_phys_pages, 2, 64)
    s.clamp_(100, 130)
    cache = duet.Cache8(k.cuda(), v.cuda(), s.cuda())
    table, to = b.page_table.copy(), b.page_table.copy()
    table[0, 1], table[1, 0], to[2, 1] = -1, b.num_phys_pages, 2 ** 31 - 1
    good = [torch.zeros(b.num_phys_pages, 2, 16, 64, dtype=torch.bfloat16, device="cuda"),
            torch.zeros(b.num_phys_pages, 2, 64, 16, dtype=torch.bfloat16, device="cuda")]
    got = [x.clone() for x in good]
    ctx.cache8_read(cache, _table(b), b.seq_meta, *good, _table(b))
    for r, j in ((0, 1), (1, 0), (2, 1)):
        for x in good:
            x[b.page_table[r, j]] = 0
    ws = torch.full((4096,), 255, dtype=torch.uint8, device="cuda")
    with pytest.raises(duet.DuetError) as e:
        ctx.cache8_read(cache, torch.as_tensor(table, device="cuda"), b.seq_meta, *got, torch.as_tensor(to, device="cuda"),
                        workspace=ws, check_errors=True)
    assert e.value.code == -6
    assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(got, good))
    ctx.cache8_read(cache, _table(b), b.seq_meta, *got, _table(b), workspace=ws, check_errors=True)


# ---- decode attention -----------------------------------------------------------------------------


def _shared_batch(sh, seed, prefixes, reqs):
    """prefixes: tokens of each; reqs: (prefix or -1, tokens of its own).  A pool with pages to spare."""
    rng = np.random.default_rng(seed)
    need = [p // 16 for p in prefixes] + [-(-n // 16) for _, n in reqs]
    pool = sum(need) + 3
    ids = rng.permutation(pool).astype(np.int32)
    ends = np.concatenate([[0], np.cumsum(need)])
    runs = [ids[a:z] for a, z in zip(ends[:-1], ends[1:])]
    rows = [np.concatenate([runs[i] if i >= 0 else ids[:0], runs[len(prefixes) + r]]) for r, (i, _) in enumerate(reqs)]
    table = np.full((len(reqs), max(map(len, rows)) + 1), -1, np.int32)
    for r, x in enumerate(rows):
        table[r, :len(x)] = x
    meta = np.array([(1, r, 1, (prefixes[i] if i >= 0 else 0) + n - 1) for r, (i, n) in enumerate(reqs)], np.int32)
    used = np.zeros((pool, 16), bool)
    for r, m in enumerate(meta):
        t = np.arange(m[3] + 1)
        used[table[r, t // 16], t % 16] = True
    return table, meta, pool, used


def _attn_inputs(sh, cache, seed, pool, used, R):
    """(q, what the call takes, the cache's values in float64); slots that no request holds are NaN."""
    import paper_2511_04791_amd as duet
    hkv, d = sh.num_kv_heads, sh.head_dim
    q = _randn(seed, R, sh.num_q_heads, d, scale=1.5)
    free = torch.from_numpy(~used)[:, None]
    if cache == "bf16":
        k, v = _randn(seed + 1, pool, hkv, 16, d), _randn(seed + 2, pool, hkv, d, 16)
        k.masked_fill_(free[..., None], float("nan"))
        v.masked_fill_(free[:, :, None], float("nan"))
        return q, (k.cuda(), v.cuda()), (to64(k), to64(v))
    from oracle import cache8 as oc
    # bytes of up to 1.875 2^3 in magnitude, a power around 2^-2 for each token
    k, v = ((_bytes(seed + i, pool, hkv, *s, hi=80) | (_bytes(seed + 9 + i, pool, hkv, *s, hi=2) << 7)) for i, s in ((1, (16, d)), (2, (d, 16))))
    s = _bytes(seed + 3, pool, hkv, 2, 16, hi=6) + 122
    k[free[..., None].expand_as(k)] = 127
    v[free[:, :, None].expand_as(v)] = 255
    s[free[:, :, None].expand_as(s)] = 255
    kd, vd = oc.decode(k.numpy(), v.numpy(), s.numpy())
    return q, duet.Cache8(k.cuda(), v.cuda(), s.cuda()), (kd, vd)


def _check_attn(got, q, values, table, meta):
    """Probabilities are rounded to bf16 in numerator and denominator alike: off by at most U of sum p |v - out|.  A score is off by
    d half steps of its products' sum (and 4 more for the scale and the exponent), a probability by that relative; the second
    sum by a half step a term and run; one rounding of the result."""
    from oracle import cache8 as oc
    want, mag, most = oc.decode_attention(to64(q), *values, table, meta)
    d, n = q.shape[2], np.asarray(meta)[:, 3][:, None, None] + 80
    near = (1.02 * U + 2 * ((d + 4) * most[..., None] + n + 8) * E) * (mag + np.abs(want))
    err = np.abs(to64(got) - want)
    bound = U * np.abs(want) + (1 + U) * near + 1e-30
    assert (np.isnan(want) == np.isnan(to64(got))).all()
    fine = ~np.isnan(want)
    if not fine.any():
        return
    assert (err <= bound)[fine].all(), (np.nanmax(err / bound), np.argwhere(err > bound)[:4])
    # on average roundings do not add up: far within the bound
    assert np.mean(err[fine]) <= 0.5 * np.mean(bound[fine])


LENGTHS = [1, 2, 15, 16, 17, 31, 48, 63, 64, 65, 66, 127, 128, 129, 500, 1025]
BATCHES = {
    "alone": ([], [(-1, n) for n in LENGTHS]),
    "one": ([], [(-1, 1)]),
    "group": ([160], [(0, n) for n in LENGTHS]),
    "two": ([16, 1040], [(i % 3 - 1, 1 + 37 * i % 200) for i in range(33)]),
    # a prefix of one request, one of nobody, one of no token, one that is a request's whole context
    "odd": ([48, 64, 0, 96], [(0, 5), (2, 7), (2, 30), (3, 0), (3, 17), (3, 0), (-1, 40)]),
    "many": ([32, 80], [(i % 4 - 1 if i % 4 < 3 else -1, 1 + i % 50) for i in range(300)]),
    "long": ([4096], [(0, 3), (0, 5000), (-1, 9001)]),
    # results that need no joining: few requests, more than travel with a launch, and prefixes that are whole contexts
    "short": ([], [(-1, n) for n in (1, 16, 17, 64, 65, 100, 128, 200, 255, 256)]),
    "lone": ([], [(-1, n) for n in (1, 2, 15, 16, 33, 64)]),
    "many_alone": ([], [(-1, 1 + 13 * i % 250) for i in range(300)]),
    "whole": ([64, 16], [(0, 0), (1, 0), (0, 0), (1, 0)]),
    # up to 256 requests that share nothing, of several runs
    "plain": ([], [(-1, 1 + 97 * i % 900) for i in range(120)] + [(-1, 9000)]),
    # many prefixes, requests past one round of the search
    "groups": ([32 * (i + 1) for i in range(30)], [(i % 31 - 1, 1 + 41 * i % 300) for i in range(150)]),
    # more prefixes than travel with a launch, and as many requests and prefixes as do
    "prefixes": ([16 * (1 + 7 * i % 25) for i in range(40)], [(i % 41 - 1, 1 + 29 * i % 400) for i in range(130)]),
    "full": ([16 * (1 + 5 * i % 30) for i in range(32)], [(i % 33 - 1, (1 + 31 * i % 180) * (i % 5 > 0 or i % 33 == 0)) for i in range(256)]),
}


@pytest.mark.parametrize("name", list(BATCHES))
@pytest.mark.parametrize("heads", [(4, 2, 128), (8, 1, 64), (16, 1, 128), (5, 5, 64), (6, 2, 128), (3, 1, 64)])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_attn_decode_shared(ctx, name, heads, cache):
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(*heads, "bf16")
    prefixes, reqs = BATCHES[name]
    table, meta, pool, used = _shared_batch(sh, 7700, prefixes, reqs)
    q, c, values = _attn_inputs(sh, cache, 7701, pool, used, len(reqs))
    pre = dict(prefix_of=[i for i, _ in reqs], prefix_len=prefixes) if prefixes else {}
    n = _space(sh, meta, pre)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    args = (q.cuda(), c, torch.as_tensor(table, device="cuda"), meta)
    out = torch.full_like(args[0], float("nan"))
    ctx.attn_decode_shared(*args, out=out, workspace=ws, check_errors=True, **pre)
    _check_attn(out, q, values, table, meta)
    assert torch.equal(out, ctx.attn_decode_shared(*args, **pre))  # a workspace of its own, nobody reads the error word


# Prefixes long enough for workgroups of many rows: one, two and no whole tile of 64 keys at the end, one block of 256 rows and two, of
# which the last is not full, tables in device memory and with the launches.
WIDE = {
    "one": ((32, 8, 128), [1008], [(0, 1 + i % 40) for i in range(60)]),
    "two": ((32, 8, 128), [976, 1280], [(i % 3 - 1, 3 + 7 * i % 90) for i in range(80)]),
    "blocks": ((64, 8, 64), [2000], [(0, i % 20) for i in range(37)]),
    "group16": ((32, 2, 128), [4096, 3008], [(i % 2, 1 + i % 17) for i in range(43)]),
    "group3": ((24, 8, 64), [2064], [(0, 5 + i) for i in range(31)]),
    "uploaded": ((16, 4, 64), [3008, 2000, 1600], [(i % 4 - 1, (1 + 11 * i % 60) * (i % 3 > 0 or i % 4 == 0)) for i in range(290)]),
    "full": ((8, 2, 128), [2400 + 16 * i for i in range(5)], [(i % 6 - 1, (1 + 11 * i % 130) * (i % 3 > 0 or i % 6 == 0)) for i in range(256)]),
    # long enough that 8-bit pages go that way too: one block and two, tiles of part pages at the end, one to eight waves
    "one_long": ((32, 8, 128), [4016], [(0, 1 + i % 40) for i in range(60)]),
    "two_long": ((32, 8, 128), [3984, 4112], [(i % 3 - 1, 3 + 7 * i % 90) for i in range(130)]),
    "blocks_long": ((64, 8, 64), [10032], [(0, i % 20) for i in range(37)]),
    "group16_long": ((32, 2, 128), [8192, 6000], [(i % 2, 1 + i % 17) for i in range(43)]),
    "group3_long": ((24, 8, 64), [20064], [(0, 5 + i) for i in range(40)]),
    "uploaded_long": ((32, 8, 128), [2000, 1600, 1200], [(i % 4 - 1, (1 + 11 * i % 60) * (i % 3 > 0 or i % 4 == 0)) for i in range(290)]),
    "few_waves": ((8, 1, 128), [65552, 33008], [(i % 2, 1 + 30 * i) for i in range(14)]),
    "long": ((8, 1, 128), [66000], [(0, 2), (0, 300), (0, 17), (0, 1), (0, 64), (-1, 5)]),
}


def _wide_case(name, seed, cache):
    import paper_2511_04791_amd as duet
    heads, prefixes, reqs = WIDE[name]
    sh = duet.AttnShape(*heads, "bf16")
    table, meta, pool, used = _shared_batch(sh, seed, prefixes, reqs)
    q, c, values = _attn_inputs(sh, cache, seed + 1, pool, used, len(reqs))
    return sh, table, meta, pool, q, c, values, dict(prefix_of=[i for i, _ in reqs], prefix_len=prefixes)


@pytest.mark.parametrize("name", list(WIDE))
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_attn_of_many_rows(ctx, name, cache):
    """Also with pages outside the pool in the prefix and behind it, then clean again.  Of long prefixes some requests' results."""
    import paper_2511_04791_amd as duet
    sh, table, meta, pool, q, c, values, pre = _wide_case(name, 9000, cache)
    ws = torch.full((_space(sh, meta, pre),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    q_gpu = q.cuda()
    members = [r for r, i in enumerate(pre["prefix_of"]) if i == 0]
    some = sorted({*range(0, len(meta), 13), members[-1], len(meta) - 1}) if name.endswith("_long") else list(range(len(meta)))

    def check(table):
        assert torch.isfinite(out).all()
        _check_attn(out[some], q[some], values, table[some], meta[some])
    for again in range(2):
        ctx.attn_decode_shared(q_gpu, c, torch.as_tensor(table, device="cuda"), meta, out=out, workspace=ws, check_errors=True, **pre)
        check(table)
        if again:
            break
        bad = table.copy()
        for j, page in ((0, -1), (5, pool), (14, 2 ** 31 - 1), (15, -7), (pre["prefix_len"][0] // 16 - 1, pool + 3)):
            bad[members, j] = page
        bad[members[-1], meta[members[-1], 3] // 16] = -2
        with pytest.raises(duet.DuetError) as e:
            ctx.attn_decode_shared(q_gpu, c, torch.as_tensor(bad, device="cuda"), meta, out=out, workspace=ws, check_errors=True, **pre)
        assert e.value.code == -6
        check(bad)


@pytest.mark.parametrize("name", ["two", "two_long", "uploaded_long"])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_attn_of_many_rows_in_a_graph(ctx, cache, name):
    sh, table, meta, pool, q, c, values, pre = _wide_case(name, 9100, cache)
    pt, x, g = torch.as_tensor(table, device="cuda"), q.cuda(), torch.cuda.CUDAGraph()
    out = torch.empty_like(x)
    ctx.attn_decode_shared(x, c, pt, meta, out=out, **pre)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        ctx.attn_decode_shared(x, c, pt, meta, out=out, **pre)
    for i in range(3):
        x.copy_(_randn(9110 + i, *q.shape))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ctx.attn_decode_shared(x, c, pt, meta, **pre))
        ctx.attn_decode_shared(x[:1], c, pt[:1], meta[:1])
    _check_attn(out[::13], x.cpu()[::13], values, table[::13], meta[::13])


@pytest.mark.parametrize("name", ["two", "group16"])
def test_attn_of_many_rows_of_infinite_scores(ctx, name):
    """Runs of keys whose scores are all -inf, for some rows and for all; a NaN reaches the rows that see it alone."""
    from oracle import cache8 as oc
    sh, table, meta, pool, q, c, _, pre = _wide_case(name, 9200, "bf16")
    q = q.abs() + 0.1
    q[5, 3] = -q[5, 3]  # sees +inf where the others see -inf
    k, v = c[0].cpu(), c[1].cpu()
    first = [r for r, i in enumerate(pre["prefix_of"]) if i == 0]
    for t in range(200, 800):
        k[table[first[0], t // 16], :, t % 16] = float("-inf")
    k[table[first[2], meta[first[2], 3] // 16], :, meta[first[2], 3] % 16] = float("nan")
    out = ctx.attn_decode_shared(q.cuda(), (k.cuda(), c[1]), torch.as_tensor(table, device="cuda"), meta, **pre).cpu()
    in_first = 5 in first
    want, mag, most = oc.decode_attention(to64(q), np.where(np.isinf(to64(k)), -1e6, to64(k)), to64(v), table, meta)
    bad = np.isnan(to64(out))
    assert bad[first[2]].all() and (bad[5, 3].all() if in_first else not bad[5].any())
    rows = [r for r in range(len(meta)) if r not in (5, first[2])]
    assert not bad[rows].any()
    finite = np.abs(np.where(np.isfinite(to64(k)), to64(k), 0)).max() * np.abs(to64(q)).sum(-1).max() / np.sqrt(128)
    err = np.abs(to64(out) - want)[rows]
    bound = (U * np.abs(want) + (1.1 * U + 2 * (132 * finite + 2000) * E) * (mag + np.abs(want)))[rows]
    assert (err <= bound).all()


def _space(sh, meta, pre):
    import ctypes
    import paper_2511_04791_amd as duet
    from paper_2511_04791_amd import _native as N
    b, n = duet._BatchC(meta), ctypes.c_size_t()
    p = None
    if pre:
        of, length = (np.ascontiguousarray(pre[k], dtype=np.int32) for k in ("prefix_of", "prefix_len"))
        ints = ctypes.POINTER(ctypes.c_int32)
        p = ctypes.byref(N.Prefixes(len(length), length.ctypes.data_as(ints), of.ctypes.data_as(ints)))
    N.check(N.lib().duet_shared_workspace_bytes(ctypes.byref(duet._shape_c(sh)), ctypes.byref(b.c), p, ctypes.byref(n)), "bytes")
    return n.value


def test_attn_of_an_empty_batch(ctx):
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(4, 2, 64, "bf16")
    cache = duet.Cache8.empty(1, 2, 64)
    q = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    table, meta = torch.zeros(0, 1, dtype=torch.int32, device="cuda"), np.zeros((0, 4), np.int32)
    assert ctx.attn_decode_shared(q, cache, table, meta, prefix_of=[], prefix_len=[16]).shape == (0, 4, 64)
    x = torch.zeros(0, 8 * 64, dtype=torch.bfloat16, device="cuda")
    assert ctx.qkv_split8(x, cache, table, meta, sh).shape == (0, 4, 64)
    k, v = torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 2, 64, 16, dtype=torch.bfloat16, device="cuda")
    ctx.cache8_read(cache, table, meta, k, v, table)


def test_attn_of_an_empty_batch_clears_the_error_word(ctx):
    import ctypes
    import paper_2511_04791_amd as duet
    from paper_2511_04791_amd import _native as N
    cache, b = duet.Cache8.empty(1, 2, 64), duet._BatchC(np.zeros((0, 4), np.int32))
    ws, x = (torch.full((4096,), 255, dtype=torch.uint8, device="cuda") for _ in range(2))
    st, shape = torch.cuda.current_stream().cuda_stream, N.Shape(4, 2, 64, 16, N.BF16, 1)
    n = ctypes.c_size_t()
    N.check(N.lib().duet_shared_workspace_bytes(ctypes.byref(shape), ctypes.byref(b.c), None, ctypes.byref(n)), "bytes")
    assert n.value <= ws.nbytes
    for _ in range(2):
        ws.fill_(255)
        N.check(N.lib().duet_attn_decode_shared(ctx.handle, ctypes.byref(shape), x.data_ptr(), ctypes.byref(cache.c), x.data_ptr(), 1,
                                                ctypes.byref(b.c), None, ws.data_ptr(), ws.nbytes, x.data_ptr() + 2048, st), "attn")
        N.check(N.lib().duet_check_device_error(ctx.handle, ws.data_ptr(), st), "error word")
    assert (x == 255).all()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_attn_placement_and_neighbours(ctx, cache):
    """The same bits wherever the pages lie."""
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(8, 2, 128, "bf16")
    prefixes, reqs = BATCHES["two"]
    table, meta, pool, used = _shared_batch(sh, 7800, prefixes, reqs)
    q, c, _ = _attn_inputs(sh, cache, 7801, pool, used, len(reqs))
    pre = dict(prefix_of=[i for i, _ in reqs], prefix_len=prefixes)
    one = ctx.attn_decode_shared(q.cuda(), c, torch.as_tensor(table, device="cuda"), meta, **pre)
    perm = np.random.default_rng(7802).permutation(pool).astype(np.int32)
    to = torch.as_tensor(np.argsort(perm), device="cuda")  # page perm[i] of the new pool is page i of the old one
    moved = np.where(table >= 0, perm[np.maximum(table, 0)], -1).astype(np.int32)
    c2 = duet.Cache8(c.k[to], c.v[to], c.scales[to]) if cache == "e4m3" else (c[0][to], c[1][to])
    two = ctx.attn_decode_shared(q.cuda(), c2, torch.as_tensor(moved, device="cuda"), meta, **pre)
    assert torch.equal(one, two)


@pytest.mark.parametrize("name", ["prefix", "one", "short", "lone", "many_alone", "plain", "many", "groups", "whole", "long", "prefixes", "full"])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_attn_pages_outside_the_pool(ctx, cache, name):
    """Their tokens do not count, in a prefix and in a request's own pages; reported; the next call starts clean."""
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(8, 2, 128, "bf16")
    prefixes, reqs = ([160], [(0, 40), (0, 100), (-1, 200), (-1, 30), (0, 33)]) if name == "prefix" else BATCHES[name]
    table, meta, pool, used = _shared_batch(sh, 7900, prefixes, reqs)
    q, c, values = _attn_inputs(sh, cache, 7901, pool, used, len(reqs))
    pre = dict(prefix_of=[i for i, _ in reqs], prefix_len=prefixes) if prefixes else {}
    bad = table.copy()
    ids = (-5, pool, 2 ** 31 - 1, -1, pool + 7)
    if name == "prefix":
        bad[[0, 1, 4], 3] = -5
        bad[1, 12], bad[2, 0], bad[2, 12], bad[3, :2] = pool, 2 ** 31 - 1, -1, pool + 7
    else:
        # the last page of some requests (never a shared one, but where all are), and a whole one
        for n, r in enumerate(range(0, len(reqs), max(1, len(reqs) // 7))):
            last = meta[r, 3] // 16
            if reqs[r][1] or name == "whole":
                bad[bad == bad[r, last]] = ids[n % 5]
    ws = torch.full((_space(sh, meta, pre),), 255, dtype=torch.uint8, device="cuda")
    out = torch.zeros(len(reqs), 8, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(duet.DuetError) as e:
        ctx.attn_decode_shared(q.cuda(), c, torch.as_tensor(bad, device="cuda"), meta, out=out, workspace=ws, check_errors=True, **pre)
    assert e.value.code == -6
    if name == "prefix":
        assert torch.isnan(out[3]).all()  # a request none of whose tokens count
    _check_attn(out, q, values, bad, meta)
    ctx.attn_decode_shared(q.cuda(), c, torch.as_tensor(table, device="cuda"), meta, out=out, workspace=ws, check_errors=True, **pre)
    _check_attn(out, q, values, table, meta)


def test_attn_of_infinite_scores(ctx):
    """Scores of -inf weigh nothing, in whole runs too; one of +inf or NaN makes the row NaN; far scores are no overflow."""
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(2, 1, 64, "bf16")
    prefixes, reqs = [1024], [(0, 70), (0, 700), (-1, 900), (-1, 40), (-1, 40), (-1, 300)]
    table, meta, pool, used = _shared_batch(sh, 8000, prefixes, reqs)
    q, c, _ = _attn_inputs(sh, "bf16", 8001, pool, used, len(reqs))
    q = q.abs() + 0.1
    k, v = c[0].cpu(), c[1].cpu()

    def put(r, tokens, value):
        for t in tokens:
            k[table[r, t // 16], :, t % 16] = value
    put(0, range(0, 1024), float("-inf"))       # the whole shared prefix
    put(2, range(128, 600), float("-inf"))
    put(3, [7], float("inf"))
    put(4, [39], float("nan"))
    put(5, range(0, 300, 3), 200.0)
    put(5, range(1, 300, 3), -200.0)
    out = ctx.attn_decode_shared(q.cuda(), (k.cuda(), c[1]), torch.as_tensor(table, device="cuda"), meta,
                                 prefix_of=[i for i, _ in reqs], prefix_len=prefixes).cpu()
    assert torch.isnan(out[3]).all() and torch.isnan(out[4]).all() and torch.isfinite(out[[0, 1, 2, 5]]).all()
    keep = [0, 1, 2, 5]
    k64 = np.where(np.isinf(to64(k)), -1e6, to64(k))  # far enough below for a weight of 0
    from oracle import cache8 as oc
    want, mag, _ = oc.decode_attention(to64(q), k64, to64(v), table, meta)
    most = 200.0 * np.abs(to64(q)).sum(-1).max() / 8  # the finite scores' largest sum of magnitudes
    err = np.abs(to64(out) - want)[keep]
    bound = (U * np.abs(want) + (1.1 * U + 2 * (68 * most + 2000) * E) * (mag + np.abs(want)))[keep]
    assert (err <= bound).all()


@pytest.mark.parametrize("prefix", [0, 2048])
def test_attn_of_nan_among_scores_of_minus_infinity(ctx, prefix):
    """A NaN score in a run whose others are -inf reaches the result, over many runs of -inf before the finite ones."""
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(16, 1, 64, "bf16")
    prefixes, reqs = ([prefix], [(0, 8192), (0, 40)]) if prefix else ([], [(-1, 10240)])
    table, meta, pool, used = _shared_batch(sh, 8050, prefixes, reqs)
    q, c, _ = _attn_inputs(sh, "bf16", 8051, pool, used, len(reqs))
    q, k = q.abs() + 0.1, c[0].cpu()
    for t in range(0, 8192):
        k[table[0, t // 16], :, t % 16] = float("-inf")
    pt, q = torch.as_tensor(table, device="cuda"), q.cuda()
    pre = dict(prefix_of=[0, 0], prefix_len=prefixes) if prefix else {}
    assert torch.isfinite(ctx.attn_decode_shared(q, (k.cuda(), c[1]), pt, meta, **pre)).all()
    k[table[0, 3], :, 5] = float("nan")
    out = ctx.attn_decode_shared(q, (k.cuda(), c[1]), pt, meta, **pre)
    assert torch.isnan(out).all()


def test_attn_far_powers(ctx):
    """Powers far from 1: tiny and huge values and keys; a value's power never leaves what fp32 and bf16 hold."""
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(4, 2, 64, "bf16")
    table, meta, pool, used = _shared_batch(sh, 8100, [], [(-1, 100), (-1, 33)])
    q, c, _ = _attn_inputs(sh, "e4m3", 8101, pool, used, 2)
    from oracle import cache8 as oc
    s = c.scales.cpu()
    s[:, :, 1] = torch.where(s[:, :, 1] == 255, s[:, :, 1], _bytes(8102, pool, 2, 16, hi=30) + 60)
    s[:, 0, 1] = torch.where(s[:, 0, 1] == 255, s[:, 0, 1], s[:, 0, 1] + 110)
    c = duet.Cache8(c.k, c.v, s.cuda())
    values = oc.decode(c.k.cpu().numpy(), c.v.cpu().numpy(), s.numpy())
    out = ctx.attn_decode_shared(q.cuda(), c, torch.as_tensor(table, device="cuda"), meta)
    _check_attn(out, q, values, table, meta)


def test_far_pages(ctx):
    """Pages whose bytes lie past 2^32: written, read back and attended, alone and as a shared prefix."""
    import paper_2511_04791_amd as duet
    from oracle import cache8 as oc
    sh = duet.AttnShape(32, 8, 128, "bf16")
    P = (1 << 32) // (8 * 16 * 128) + 40  # 4.3 GB of keys, as much of values
    cache = duet.Cache8(*[torch.empty(P, 8, *s, dtype=torch.uint8, device="cuda") for s in ((16, 128), (128, 16), (2, 16))])
    table = np.full((2, 6), -1, np.int32)
    table[:, :4], table[0, 4:], table[1, 4:] = [P - 1, 3, P - 9, P - 2], [P - 30, P - 3], [P - 4, 0]
    meta = duet._meta_rows([(0, 90, 0), (0, 90, 0)])
    qkv = _randn(8600, 180, 48 * 128)
    qkv[90:154] = qkv[:64]  # the shared pages' tokens
    pt = torch.as_tensor(table, device="cuda")
    ctx.qkv_split8(qkv.cuda(), cache, pt, meta, sh, check_errors=True)
    ko, vo = (torch.zeros(12, 8, *s, dtype=torch.bfloat16, device="cuda") for s in ((16, 128), (128, 16)))
    to = torch.arange(12, dtype=torch.int32, device="cuda").view(2, 6)
    ctx.cache8_read(cache, pt, meta, ko, vo, to, check_errors=True)
    x = to64(qkv).reshape(2, 90, 48, 128)
    for r in range(2):
        t = np.arange(90)
        for got, part in ((to64(ko)[6 * r + t // 16, :, t % 16], x[r, :, 32:40]), (to64(vo)[6 * r + t // 16, :, :, t % 16], x[r, :, 40:])):
            want, e = oc.encode(part)
            assert np.array_equal(got, want * 2.0 ** (e.astype(np.float64) - 127)[..., None])
    decode = duet._meta_rows([(1, 1, 89), (1, 1, 89)])
    q = _randn(8601, 2, 32, 128)
    values = to64(ko), to64(vo)
    for pre in ({}, dict(prefix_of=[0, 0], prefix_len=[64])):
        out = ctx.attn_decode_shared(q.cuda(), cache, pt, decode, check_errors=True, **pre)
        _check_attn(out, q, values, to.cpu().numpy(), decode)


def test_attn_on_two_streams(ctx):
    """The same call twice gives the same bits, whatever the workspace held, on two streams at once."""
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(8, 2, 128, "bf16")
    prefixes, reqs = BATCHES["groups"]
    table, meta, pool, used = _shared_batch(sh, 8700, prefixes, reqs)
    q, c, _ = _attn_inputs(sh, "e4m3", 8701, pool, used, len(reqs))
    pre = dict(prefix_of=[i for i, _ in reqs], prefix_len=prefixes)
    q, pt = q.cuda(), torch.as_tensor(table, device="cuda")
    want = ctx.attn_decode_shared(q, c, pt, meta, **pre)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for i in range(8):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(ctx.attn_decode_shared(q, c, pt, meta, **pre))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_calls_of_two_threads(ctx):
    """A step each, on a stream of its own, with the same context."""
    import threading
    import paper_2511_04791_amd as duet
    sh, norm, rope = duet.AttnShape(8, 2, 128, "bf16"), duet.HeadNorm(eps=1e-6), duet.Rope(_freq(128))
    work, got, errors = [], [[], []], []
    for i, name in enumerate(("groups", "plain")):
        prefixes, reqs = BATCHES[name]
        table, meta, pool, used = _shared_batch(sh, 8750 + i, prefixes, reqs)
        _, c, _ = _attn_inputs(sh, "e4m3", 8760 + i, pool, used, len(reqs))
        pre = dict(prefix_of=[i for i, _ in reqs], prefix_len=prefixes) if prefixes else {}
        qkv, pt = _randn(8770 + i, len(reqs), 12 * 128).cuda(), torch.as_tensor(table, device="cuda")

        def step(qkv=qkv, c=c, pt=pt, meta=meta, pre=pre):
            q = ctx.qkv_split8(qkv, c, pt, meta, sh, norm=norm, rope=rope)
            return ctx.attn_decode_shared(q, c, pt, meta, **pre)
        work.append((step, step()))
    torch.cuda.synchronize()

    def run(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    got[i].append(work[i][0]())
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001 - shown by the main thread
            errors.append(e)
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for th in threads:
        th.start()
    for th in threads:
        th.join(60)
    assert not errors and all(len(g) == 20 for g in got)
    for g, (_, want) in zip(got, work):
        assert all(torch.equal(o, want) for o in g)


@pytest.mark.parametrize("name", ["short", "plain", "groups", "many_alone"])
def test_attention_in_a_graph(ctx, name):
    """Every way that the requests reach the kernels, captured and replayed after other calls."""
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(8, 2, 64, "bf16")
    prefixes, reqs = BATCHES[name]
    table, meta, pool, used = _shared_batch(sh, 8800, prefixes, reqs)
    _, c, _ = _attn_inputs(sh, "e4m3", 8801, pool, used, len(reqs))
    pre = dict(prefix_of=[i for i, _ in reqs], prefix_len=prefixes) if prefixes else {}
    pt, q = torch.as_tensor(table, device="cuda"), torch.zeros(len(reqs), 8, 64, dtype=torch.bfloat16, device="cuda")
    out, g = torch.empty_like(q), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        ctx.attn_decode_shared(q, c, pt, meta, out=out, **pre)
    for i in range(3):
        q.copy_(_randn(8810 + i, len(reqs), 8, 64))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ctx.attn_decode_shared(q, c, pt, meta, **pre))
        ctx.attn_decode_shared(q[:1], c, pt[:1], meta[:1])


def test_graphs_that_share_a_workspace(ctx):
    """Calls after each other in one workspace, captured ones among them: none finds what another left."""
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(8, 2, 64, "bf16")
    calls = []
    for i, name in enumerate(("plain", "groups", "two", "short", "many")):
        prefixes, reqs = BATCHES[name]
        table, meta, pool, used = _shared_batch(sh, 8900 + i, prefixes, reqs)
        q, c, _ = _attn_inputs(sh, "e4m3", 8910 + i, pool, used, len(reqs))
        pre = dict(prefix_of=[i for i, _ in reqs], prefix_len=prefixes) if prefixes else {}
        args = (q.cuda(), c, torch.as_tensor(table, device="cuda"), meta)
        calls.append((args, pre, ctx.attn_decode_shared(*args, **pre), _space(sh, meta, pre)))
    ws = torch.full((max(n for *_, n in calls),), 255, dtype=torch.uint8, device="cuda")
    graphs = []
    torch.cuda.synchronize()
    for args, pre, _, _ in calls:
        g = torch.cuda.CUDAGraph()
        out = torch.empty_like(args[0])
        with torch.cuda.graph(g):
            ctx.attn_decode_shared(*args, out=out, workspace=ws, **pre)
        graphs.append((g, out))
    for order in ((0, 1, 2, 3, 4), (4, 2, 0, 3, 1), (1, 1, 3, 0, 4, 2)):
        for i in order:
            graphs[i][1].zero_()
            graphs[i][0].replay()
            args, pre, want, _ = calls[(i + 1) % 5]
            assert torch.equal(ctx.attn_decode_shared(*args, workspace=ws, **pre), want)
        torch.cuda.synchronize()
        assert all(torch.equal(graphs[i][1], calls[i][2]) for i in order)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_a_step_in_a_graph(ctx, cache):
    """Split, attention and read-back captured with buffers and workspaces of their own, replayed with eager work between."""
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(8, 2, 128, "bf16")
    prefixes, reqs = BATCHES["two"]
    table, meta, pool, used = _shared_batch(sh, 8200, prefixes, reqs)
    _, c, _ = _attn_inputs(sh, cache, 8201, pool, used, len(reqs))
    pre = dict(prefix_of=[i for i, _ in reqs], prefix_len=prefixes)
    pt = torch.as_tensor(table, device="cuda")
    norm, rope = duet.HeadNorm(eps=1e-6), duet.Rope(_freq(128))
    qkv = _randn(8202, len(reqs), 12 * 128).cuda()
    ko, vo = (torch.zeros(len(reqs) * table.shape[1], 2, *s, dtype=torch.bfloat16, device="cuda") for s in ((16, 128), (128, 16)))
    to = torch.arange(len(reqs) * table.shape[1], dtype=torch.int32, device="cuda").view(len(reqs), -1)

    def step():
        if cache == "e4m3":
            q = ctx.qkv_split8(qkv, c, pt, meta, sh, norm=norm, rope=rope)
            ctx.cache8_read(c, pt, meta, ko, vo, to)
        else:
            q = ctx.qkv_norm_rope_split(qkv, *c, pt, meta, sh, norm, rope)
        return ctx.attn_decode_shared(q, c, pt, meta, **pre)
    graphs = []
    st = torch.cuda.Stream()
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=st):
            o = step()
        graphs.append((g, o))
    for i in range(4):
        qkv.copy_(_randn(8300 + i, len(reqs), 12 * 128))
        g, o = graphs[i % 2]
        g.replay()
        torch.cuda.synchronize()
        got, pages = o.clone(), (ko.clone(), vo.clone())
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(pages[0], ko) and torch.equal(pages[1], vo)


def test_a_chunk_and_a_decode_over_an_8_bit_cache(ctx):
    """As a server uses it: a prompt is written in two chunks whose attention runs on the pages read back, then tokens are decoded.  The
    decode attention over the 8-bit cache is that over the pages that it stands for."""
    import paper_2511_04791_amd as duet
    from oracle import cache8 as oc
    from paper_2511_04791_amd import workloads as wl
    sh = duet.AttnShape(8, 2, 64, "bf16")
    rope, norm = duet.Rope(_freq(64)), duet.HeadNorm(eps=1e-6)
    lens = [70, 33, 200]
    b = wl.make_batch(sh, [(0, n + 2, 0) for n in lens], page_seed=8400)
    pt, cache = _table(b), duet.Cache8.empty(b.num_phys_pages, 2, 64)
    ko = torch.zeros(b.num_phys_pages, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    vo = torch.zeros(b.num_phys_pages, 2, 64, 16, dtype=torch.bfloat16, device="cuda")
    for first, last in ((0, 20), (20, None)):
        meta = duet._meta_rows([(0, (last or n) - first, first) for n in lens])
        T = int(meta[:, 2].sum())
        q = ctx.qkv_split8(_randn(8401 + first, T, 12 * 64).cuda(), cache, pt, meta, sh, norm=norm, rope=rope)
        ctx.cache8_read(cache, pt, meta, ko, vo, pt)
        out = ctx.attn_mixed_batch(q, ko, vo, pt, meta)
        assert torch.isfinite(out).all()
    for step in range(2):
        meta = duet._meta_rows([(1, 1, n + step) for n in lens])
        q = ctx.qkv_split8(_randn(8500 + step, 3, 12 * 64).cuda(), cache, pt, meta, sh, norm=norm, rope=rope)
        out = ctx.attn_decode_shared(q, cache, pt, meta)
        values = oc.decode(*[x.cpu().numpy() for x in (cache.k, cache.v, cache.scales)])
        _check_attn(out, q.cpu(), values, b.page_table, meta)
        ctx.cache8_read(cache, pt, meta, ko, vo, pt)
        again = ctx.attn_decode_shared(q, (ko, vo), pt, meta)
        _check_attn(again, q.cpu(), values, b.page_table, meta)
