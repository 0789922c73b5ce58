"""GPU parity of the rotating QKV split, the adapters and sampling with their fp64 definitions, at the sizes, layouts
and masks where they can go wrong."""
import numpy as np
import pytest

from _helpers import to64

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -8   # half a step of bf16, relative
E = 2.0 ** -24  # of fp32


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


# ---- the rotating split -------------------------------------------------------------------------

REQUESTS = {
    # whole pages, pages covered in part at either end or both, one row, every start in a page
    "pages": [(0, 16, 0), (0, 48, 32), (0, 17, 15), (0, 31, 1), (0, 15, 0), (0, 2, 15), (1, 1, 16)],
    "starts": [(0, 40 + s, s) for s in range(16)],
    "one": [(1, 1, 5000)],
    # more requests than travel with one launch's arguments, and than one round of the search takes
    "many": [(1, 1, 7 * i % 90) for i in range(300)] + [(0, 33, 20), (1, 1, 3), (0, 1, 0)],
    "long": [(0, 1500, 70000), (1, 1, 100000)],
}


def _rope_inputs(sh, reqs, seed):
    from paper_2511_04791_amd import workloads as wl
    b = wl.make_batch(sh, reqs, page_seed=seed)
    dt = torch.bfloat16 if sh.dtype == "bf16" else torch.float32
    P = b.num_phys_pages
    kc = _randn(seed + 1, P, sh.num_kv_heads, 16, sh.head_dim, dtype=dt)
    vc = _randn(seed + 2, P, sh.num_kv_heads, sh.head_dim, 16, dtype=dt)
    qkv = _randn(seed + 3, b.num_tokens, (sh.num_q_heads + 2 * sh.num_kv_heads) * sh.head_dim, dtype=dt)
    return b, qkv, kc, vc


def _check_rope(sh, b, qkv, kc, vc, got, rope_args, table=None):
    """rope_args: freq, adjacent, pair_axis, positions (numpy)."""
    from oracle import serving as so
    freq, adjacent, pair_axis, positions = rope_args
    hq, hkv, d, n = sh.num_q_heads, sh.num_kv_heads, sh.head_dim, len(freq)
    table = b.page_table if table is None else table
    args = (table, b.seq_meta, hq, hkv, d, freq, adjacent, pair_axis, positions)
    want = so.rope_split(to64(qkv), to64(kc), to64(vc), *args)
    # |a| + |b| of each element's pair: |x| and |x turned a quarter|, through the same slots
    x = np.abs(to64(qkv)).reshape(len(qkv), -1, d)
    i = np.arange(n)
    p, q = (2 * i, 2 * i + 1) if adjacent else (i, i + n)
    mag = x.copy()
    mag[..., p] = mag[..., q] = x[..., p] + x[..., q]
    mag = so.rope_split(mag.reshape(len(qkv), -1), np.zeros(kc.shape), np.zeros(vc.shape), table, b.seq_meta, hq, hkv, d,
                        np.zeros(n), adjacent)
    # sine and cosine are within 3 half steps (angle, series, evaluation) and the two products and their sum within
    # one each; one rounding to the stored type
    rel = U if sh.dtype == "bf16" else E
    for name, g, w, m in zip(("q", "k"), got, want, mag):
        err = np.abs(to64(g) - w)
        turned = m > 0 if name == "k" else np.ones(w.shape, bool)
        bound = np.where(turned, rel * np.abs(w) + 6 * E * (1 + rel) * m, 0.0)
        assert (err <= bound).all(), (name, err.max(), np.argwhere(err > bound)[:5])
    assert np.array_equal(to64(got[2]), want[2])


def _freq(rot, theta=10000.0):
    return [theta ** (-2.0 * i / rot) for i in range(rot // 2)]


@pytest.mark.parametrize("name", list(REQUESTS))
@pytest.mark.parametrize("heads,dtype,rot,adjacent", [((4, 2, 128), "bf16", 128, False), ((6, 3, 64), "bf16", 64, True),
                                                      ((20, 4, 128), "bf16", 48, False), ((2, 2, 64), "f32", 64, False),
                                                      ((5, 1, 64), "f32", 16, True), ((4, 2, 128), "f32", 112, True),
                                                      ((8, 1, 128), "bf16", 80, True), ((4, 4, 64), "f32", 48, False),
                                                      ((2, 1, 64), "bf16", 16, False)])
def test_rope_split(ctx, name, heads, dtype, rot, adjacent):
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(*heads, dtype)
    b, qkv, kc, vc = _rope_inputs(sh, REQUESTS[name], 6000)
    kg, vg = kc.cuda(), vc.cuda()
    q = ctx.qkv_rope_split(qkv.cuda(), kg, vg, torch.as_tensor(b.page_table, device="cuda"), b.seq_meta, sh,
                           duet.Rope(_freq(rot), adjacent=adjacent), check_errors=True)
    _check_rope(sh, b, qkv, kc, vc, (q, kg, vg), (_freq(rot), adjacent, None, None))


@pytest.mark.parametrize("axes,cyclic", [(1, False), (2, True), (3, False), (3, True), (4, True)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rope_positions_of_axes(ctx, axes, cyclic, dtype):
    """Given positions, negative and far ones among them."""
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(3, 3, 64, dtype)
    b, qkv, kc, vc = _rope_inputs(sh, REQUESTS["pages"], 6100)
    rng = np.random.default_rng(6101)
    pos = rng.integers(-50, 3000, size=(axes, b.num_tokens)).astype(np.int32)
    pos[:, ::7] = rng.integers(-2 ** 24, 2 ** 24, size=pos[:, ::7].shape)
    n = 24
    axis = [i % axes for i in range(n)] if cyclic else sorted(i % axes for i in range(n))
    kg, vg = kc.cuda(), vc.cuda()
    rope = duet.Rope.base(500000.0, 2 * n, pair_axis=axis, axes=axes)
    q = ctx.qkv_rope_split(qkv.cuda(), kg, vg, torch.as_tensor(b.page_table, device="cuda"), b.seq_meta, sh, rope,
                           positions=torch.as_tensor(pos, device="cuda"), check_errors=True)
    _check_rope(sh, b, qkv, kc, vc, (q, kg, vg), (_freq(2 * n, 500000.0), False, axis, pos))


def test_rope_of_frequency_zero_is_the_copy(ctx):
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(4, 2, 128, "bf16")
    b, qkv, kc, vc = _rope_inputs(sh, REQUESTS["starts"], 6200)
    table, x = torch.as_tensor(b.page_table, device="cuda"), qkv.cuda()
    k1, v1, k2, v2 = kc.cuda(), vc.cuda(), kc.cuda(), vc.cuda()
    q1 = ctx.qkv_split(x, k1, v1, table, b.seq_meta, sh)
    q2 = ctx.qkv_rope_split(x, k2, v2, table, b.seq_meta, sh, duet.Rope([0.0] * 64))
    assert torch.equal(q1, q2) and torch.equal(k1, k2) and torch.equal(v1, v2)


@pytest.mark.parametrize("name", ["pages", "many"])
def test_rope_pages_outside_the_pool(ctx, name):
    """Skipped and reported; the rows' queries and every other page are written.  The next call starts clean."""
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(4, 2, 64, "bf16")
    b, qkv, kc, vc = _rope_inputs(sh, REQUESTS[name], 6300)
    table = b.page_table.copy()
    table[0, 0], table[1, 3 if name == "pages" else 0], table[len(table) - 1, 0] = -1, b.num_phys_pages, 2 ** 31 - 1
    kg, vg = kc.cuda(), vc.cuda()
    ws = torch.full((1 << 16,), 255, dtype=torch.uint8, device="cuda")
    args = (b.seq_meta, sh, duet.Rope(_freq(64)))
    q = torch.empty(b.num_tokens, 4, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(duet.DuetError) as e:
        ctx.qkv_rope_split(qkv.cuda(), kg, vg, torch.as_tensor(table, device="cuda"), *args, q=q, workspace=ws, check_errors=True)
    assert e.value.code == -6
    _check_rope(sh, b, qkv, kc, vc, (q, kg, vg), (_freq(64), False, None, None), table)
    ctx.qkv_rope_split(qkv.cuda(), kg, vg, torch.as_tensor(b.page_table, device="cuda"), *args, workspace=ws, check_errors=True)


def test_rope_pages_outside_the_pool_without_a_workspace(ctx):
    """Skipped all the same; nobody is told."""
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(4, 2, 64, "f32")
    b, qkv, kc, vc = _rope_inputs(sh, REQUESTS["pages"], 6350)
    table = b.page_table.copy()
    table[0, 0], table[1, 3], table[len(table) - 1, 0] = -1, b.num_phys_pages, 2 ** 31 - 1
    kg, vg = kc.cuda(), vc.cuda()
    q = ctx.qkv_rope_split(qkv.cuda(), kg, vg, torch.as_tensor(table, device="cuda"), b.seq_meta, sh, duet.Rope(_freq(64)))
    _check_rope(sh, b, qkv, kc, vc, (q, kg, vg), (_freq(64), False, None, None), table)


# ---- adapters -------------------------------------------------------------------------------------


def _lora_case(seed, d_in, d_out, rank, n, reqs, ids=None):
    from paper_2511_04791_amd import _meta_rows
    meta = _meta_rows(reqs)
    T = int(meta[:, 2].sum())
    rng = np.random.default_rng(seed)
    ids = rng.integers(-1, n, size=len(meta)).astype(np.int32) if ids is None else np.asarray(ids, np.int32)
    x, base = _randn(seed, T, d_in), _randn(seed + 1, T, d_out)
    a, b = _randn(seed + 2, n, rank, d_in, scale=d_in ** -0.5), _randn(seed + 3, n, d_out, rank, scale=rank ** -0.5)
    scale = torch.linspace(-0.5, 2.0, n)
    return meta, ids, x, base, a, b, scale


def _check_lora(got, meta, ids, x, base, a, b, scale):
    from oracle import serving as so
    want, mag = so.lora_add(to64(x), to64(base), to64(a), to64(b), None if scale is None else to64(scale), meta, ids)
    # one rounding to bf16; before it fp32 sums over d_in and the rank (each term's error at most the count of
    # additions times half a step) and h carried with at least 16 bits
    near = (2.0 ** -16 + (x.shape[1] + a.shape[1] + 4) * E) * mag + 2 * E * np.abs(to64(base))
    err = np.abs(to64(got) - want)
    assert (err <= U * np.abs(want) + (1 + U) * near + 1e-30).all(), (err / (U * np.abs(want) + near + 1e-30)).max()


LORA_REQS = {
    "decode": [(1, 1, 9)] * 37,
    "one": [(1, 1, 0)],
    "mixed": [(1, 1, 5)] * 5 + [(0, 70, 3), (0, 16, 0), (0, 1, 0), (0, 129, 7)],
    "chunk": [(0, 517, 0)],
}


@pytest.mark.parametrize("reqs", list(LORA_REQS))
@pytest.mark.parametrize("d_in,d_out,rank,n", [(64, 64, 16, 3), (8, 8, 8, 2), (520, 136, 24, 40), (256, 1032, 64, 2),
                                               (1000, 264, 128, 5), (4096, 512, 8, 1), (264, 4104, 32, 4), (40, 72, 88, 3)])
def test_lora_add(ctx, reqs, d_in, d_out, rank, n):
    import paper_2511_04791_amd as duet
    meta, ids, x, base, a, b, scale = _lora_case(6500 + rank, d_in, d_out, rank, n, LORA_REQS[reqs])
    if len(ids) == 1:
        ids[0] = n - 1
    got = ctx.lora_add(x.cuda(), base.cuda(), duet.Lora(a.cuda(), b.cuda(), scale.cuda()), meta, ids)
    _check_lora(got, meta, ids, x, base, a, b, scale)


def test_lora_without_adapters_or_scale(ctx):
    import paper_2511_04791_amd as duet
    meta, ids, x, base, a, b, _ = _lora_case(6600, 128, 200, 16, 2, LORA_REQS["mixed"])
    lora = duet.Lora(a.cuda(), b.cuda())
    ids[:] = -1
    assert torch.equal(ctx.lora_add(x.cuda(), base.cuda(), lora, meta, ids).cpu(), base)
    ids[1::2] = 1
    _check_lora(ctx.lora_add(x.cuda(), base.cuda(), lora, meta, ids), meta, ids, x, base, a, b, None)


def test_lora_in_place_on_columns_of_a_wider_projection(ctx):
    """The columns beside the adapter's stay as they were; so do the rows of requests without one."""
    import paper_2511_04791_amd as duet
    meta, ids, x, base, a, b, scale = _lora_case(6700, 320, 328, 16, 3, LORA_REQS["mixed"])
    wide, xs = _randn(6701, len(x), 1000).cuda(), torch.zeros(len(x), 400, dtype=torch.bfloat16, device="cuda")
    before = wide.clone()
    wide[:, 64:64 + 328], xs[:, 8:328] = base.cuda(), x.cuda()
    view = wide[:, 64:64 + 328]
    out = ctx.lora_add(xs[:, 8:328], view, duet.Lora(a.cuda(), b.cuda(), scale.cuda()), meta, ids, out=view)
    assert out.data_ptr() == view.data_ptr()
    _check_lora(view, meta, ids, x, base, a, b, scale)
    assert torch.equal(wide[:, :64], before[:, :64]) and torch.equal(wide[:, 392:], before[:, 392:])


def test_lora_keeps_what_is_not_finite_to_its_own_rows(ctx):
    """A row with an infinity spoils no row of another request, nor an unused adapter's NaN any."""
    import paper_2511_04791_amd as duet
    meta, ids, x, base, a, b, scale = _lora_case(6800, 72, 80, 16, 4, LORA_REQS["mixed"], [0, 1, -1, 1, 0, 1, 0, 1, 0])
    a[3], b[2] = float("nan"), float("inf")
    x[0], base[2, 5] = float("inf"), float("nan")
    got = ctx.lora_add(x.cuda(), base.cuda(), duet.Lora(a.cuda(), b.cuda(), scale.cuda()), meta, ids).cpu()
    assert torch.isnan(got[2, 5]) and torch.equal(got[2, :5], base[2, :5])
    x[0], base[2, 5], got[2, 5] = 0, 0, 0
    clean = ctx.lora_add(x.cuda(), base.cuda(), duet.Lora(a.cuda(), b.cuda(), scale.cuda()), meta, ids).cpu()
    assert torch.equal(got[1:], clean[1:])


def test_lora_beyond_the_largest_bf16(ctx):
    """A hidden value between bf16's largest and fp32's gives infinities, not NaN."""
    import paper_2511_04791_amd as duet
    x, base = torch.ones(2, 8, dtype=torch.bfloat16), torch.ones(2, 16, dtype=torch.bfloat16)
    x[0, 0], x[0, 1], x[0, 2:] = torch.finfo(torch.bfloat16).max, 1.5 * 2.0 ** 119, 0
    a, b = torch.ones(1, 8, 8, dtype=torch.bfloat16), torch.ones(1, 16, 8, dtype=torch.bfloat16)
    h = x[0].float().sum()
    assert torch.isfinite(h) and torch.isinf(h.to(torch.bfloat16))
    got = ctx.lora_add(x.cuda(), base.cuda(), duet.Lora(a.cuda(), b.cuda()), [(0, 2, 0)], [0]).cpu()
    assert (got[0] == float("inf")).all() and (got[1] == 65).all()


# ---- sampling ---------------------------------------------------------------------------------------


def _check_sample(ctx, logits, u, **params):
    from oracle import serving as so
    num = {k: v.numpy() for k, v in params.items()}
    ids, probs = ctx.sample(logits.cuda(), u.cuda(), **{k: v.cuda() for k, v in params.items()})
    want_ids, want_probs = so.sample(to64(logits), u.numpy(), **num)
    assert np.array_equal(ids.cpu().numpy(), want_ids), np.argwhere(ids.cpu().numpy() != want_ids)[:8]
    # the sum of weights is within 2^-34 of each term; one rounding to fp32
    assert (np.abs(to64(probs) - want_probs) <= (E + 2.0 ** -33) * want_probs + 1e-38).all()


def _mixed_params(seed, rows):
    rng = np.random.default_rng(seed)
    f = lambda x: torch.from_numpy(np.asarray(x, np.float32))  # noqa: E731
    return dict(temperature=f(np.where(rng.random(rows) < 0.1, 0.0, rng.uniform(0.05, 2.0, rows))),
                top_k=torch.from_numpy(rng.choice([-1, 0, 1, 2, 5, 40, 700, 5000, 300000], rows).astype(np.int32)),
                top_p=f(rng.choice([1.0, 0.3, 0.8, 0.95, 0.999, 0.0, 2.0], rows)),
                min_p=f(rng.choice([0.0, 0.0, 0.01, 0.3, 1.0], rows)))


@pytest.mark.parametrize("vocab", [1, 2, 7, 63, 64, 65, 1000, 1024, 1025, 4099, 32000, 128256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sample_sizes(ctx, vocab, dtype):
    rows = 24
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = (_randn(7000 + vocab, rows, vocab, dtype=torch.float32) * torch.linspace(0.1, 6, rows)[:, None]).to(dt)
    u = torch.rand(rows, generator=torch.Generator().manual_seed(7001))
    _check_sample(ctx, x, u, **_mixed_params(7002 + vocab, rows))
    _check_sample(ctx, x, u)


def test_sample_the_largest_vocabulary(ctx):
    x = _randn(7100, 2, 1 << 18, scale=3.0, dtype=torch.float32)
    x[1] = 4.0  # one bin, one value, 2^18 tokens
    _check_sample(ctx, x, torch.tensor([0.7, 0.9]), top_p=torch.tensor([0.9, 0.75]))
    _check_sample(ctx, x, torch.tensor([0.3, 0.99999]), top_k=torch.tensor([100000, 0], dtype=torch.int32))


@pytest.mark.parametrize("rows", [1, 3, 40])
@pytest.mark.parametrize("vocab", [65535, 65536, 70001])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sample_few_rows(ctx, rows, vocab, dtype):
    """One workgroup a row, and several."""
    x = (_randn(7150 + vocab, rows, vocab, dtype=torch.float32) * torch.linspace(0.4, 4, rows)[:, None])
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    u = torch.rand(rows, generator=torch.Generator().manual_seed(7151))
    _check_sample(ctx, x, u, **_mixed_params(7155, rows))
    _check_sample(ctx, x, u, top_p=torch.full((rows,), 0.9))
    _check_sample(ctx, x, u)
    _check_sample(ctx, x, u, temperature=torch.zeros(rows))


ROWS = {
    "all equal": lambda v: torch.full((v,), -3.25),
    "two values": lambda v: torch.where(torch.arange(v) % 3 == 0, 2.0, 1.5),
    "few values": lambda v: (torch.arange(v) % 5).float() * 0.25,
    "one finite": lambda v: torch.full((v,), -float("inf")).index_fill(0, torch.tensor([v // 2]), -1e30),
    "masked": lambda v: _randn(1, v, dtype=torch.float32).masked_fill(torch.arange(v) % 7 != 3, -float("inf")),
    "masked with the lowest": lambda v: _randn(2, v, dtype=torch.float32).masked_fill(torch.arange(v) % 7 != 3,
                                                                                      torch.finfo(torch.float32).min),
    "all the lowest": lambda v: torch.full((v,), torch.finfo(torch.float32).min),
    "nothing": lambda v: torch.full((v,), -float("inf")),
    "NaN": lambda v: torch.full((v,), float("nan")),
    "some NaN": lambda v: _randn(3, v, dtype=torch.float32).masked_fill(torch.arange(v) % 2 == 0, float("nan")),
    "some infinite": lambda v: _randn(4, v, dtype=torch.float32).masked_fill(torch.arange(v) % 9 == 4, float("inf")),
    "zeros of both signs": lambda v: torch.where(torch.arange(v) % 2 == 0, 0.0, -0.0),
    "huge": lambda v: _randn(5, v, dtype=torch.float32) * 1e38,
    "tiny": lambda v: _randn(6, v, dtype=torch.float32) * 1e-42,
    "dense": lambda v: 1.0 + torch.arange(v) * 2.0 ** -23,
    "a far tail": lambda v: torch.where(torch.arange(v) == 11, 60.0, _randn(7, v, dtype=torch.float32)),
}


@pytest.mark.parametrize("name", list(ROWS))
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [400, 9001, 70001])
def test_sample_rows(ctx, name, dtype, vocab):
    """One row under many settings; the largest vocabulary goes to several workgroups a row."""
    rows = 40
    x = ROWS[name](vocab).to(torch.bfloat16 if dtype == "bf16" else torch.float32).repeat(rows, 1)
    u = torch.rand(rows, generator=torch.Generator().manual_seed(7200))
    u[:6] = torch.tensor([0.0, 1.0, float("nan"), -1.0, 1 - 2.0 ** -24, 7.0])
    _check_sample(ctx, x, u, **_mixed_params(7201, rows))
    _check_sample(ctx, x, u, top_p=torch.full((rows,), 0.5))
    _check_sample(ctx, x, u)


@pytest.mark.parametrize("name", list(ROWS))
def test_sample_rows_in_more_slices(ctx, name):
    """Fewer rows go to more workgroups each."""
    rows = 9
    x = ROWS[name](70001).repeat(rows, 1)
    u = torch.linspace(0, 1, rows)
    _check_sample(ctx, x, u, **_mixed_params(7221, rows))
    _check_sample(ctx, x, u, top_p=torch.full((rows,), 0.7), top_k=torch.full((rows,), 3000, dtype=torch.int32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [9001, 70001])
@pytest.mark.parametrize("ties", ["scattered", "in blocks", "at one end"])
def test_sample_places_among_many_ties(ctx, dtype, vocab, ties):
    """Hundreds of tokens of one logit, spread over the row, one behind the other, or crowded beside a few far ones: their order is
    that of the index whatever way they are listed."""
    rows, i = 24, torch.arange(vocab)
    x = {"scattered": torch.round(_randn(7250, vocab, dtype=torch.float32) * 16) / 16,
         "in blocks": -(i // 150 % 60) * 0.0625,
         "at one end": torch.where(i % 1500 == 7, 2.0, torch.where(i < 900, 1.0, -0.5 - (i % 64) * 0.0625))}[ties]
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32).repeat(rows, 1)
    u = (torch.arange(rows) + 0.37) / rows
    for params in (dict(top_p=torch.linspace(0.05, 0.95, rows)), dict(top_k=torch.arange(rows, dtype=torch.int32) * 67 + 3),
                   dict(top_p=torch.full((rows,), 0.9), min_p=torch.linspace(0.01, 0.9, rows)),
                   dict(temperature=torch.linspace(0.1, 1.5, rows), top_k=torch.full((rows,), 1000, dtype=torch.int32))):
        _check_sample(ctx, x, u, **params)


def test_sample_odd_parameters(ctx):
    """NaN and infinities among the parameters."""
    rows, nan, inf = 12, float("nan"), float("inf")
    x = _randn(7300, 1, 777, scale=2.0, dtype=torch.float32).repeat(rows, 1)
    u = torch.linspace(0.02, 0.98, rows)
    _check_sample(ctx, x, u, temperature=torch.tensor([nan, -1.0, -0.0, inf, 1e-30, 1e30] * 2),
                  top_p=torch.tensor([nan, -1.0, 0.5, nan, inf, 0.9] * 2), min_p=torch.tensor([nan, -1.0, 0.5, 5.0] * 3),
                  top_k=torch.tensor([0, -5, 2 ** 31 - 1] * 4, dtype=torch.int32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("first,vocab,width", [(0, 1000, 1000), (1, 999, 1003), (3, 50257, 50300), (5, 8, 17)])
def test_sample_rows_off_every_alignment(ctx, dtype, first, vocab, width):
    rows = 9
    wide = _randn(7400, rows, width, scale=2.0, dtype=torch.float32).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    u = torch.linspace(0.05, 0.95, rows)
    params = dict(top_p=torch.full((rows,), 0.9))
    from oracle import serving as so
    part = wide.cuda()[:, first:first + vocab]
    ids, _ = ctx.sample(part, u.cuda(), top_p=params["top_p"].cuda())
    want, _ = so.sample(to64(wide[:, first:first + vocab]), u.numpy(), top_p=params["top_p"].numpy())
    assert np.array_equal(ids.cpu().numpy(), want)


@pytest.mark.parametrize("rows", [1, 255, 256, 257, 1000])
def test_sample_a_row_is_the_same_in_any_batch(ctx, rows):
    x = _randn(7500, 1000, 2000, scale=2.0, dtype=torch.float32).cuda()
    u = torch.rand(1000, generator=torch.Generator().manual_seed(7501)).cuda()
    p = torch.full((1000,), 0.95, device="cuda")
    ids, probs = ctx.sample(x[:rows], u[:rows].clone(), top_p=p[:rows].clone())
    for _ in range(3):
        again = ctx.sample(x[:rows], u[:rows].clone(), top_p=p[:rows].clone())
        assert torch.equal(again[0], ids) and torch.equal(again[1], probs)
    i = rows - 1
    one = ctx.sample(x[i:i + 1], u[i:i + 1].clone(), top_p=p[i:i + 1].clone())
    assert int(one[0]) == int(ids[i]) and float(one[1]) == float(probs[i])


# ---- together ---------------------------------------------------------------------------------------


def _step(ctx, duet, x, w, head, lora, ids, table, meta, sh, rope, pos, kc, vc, u, params):
    """One layer of a served step: projection and adapters, rotation into the cache, attention, classifier, tokens."""
    qkv = x @ w
    ctx.lora_add(x, qkv, lora, meta, ids, out=qkv)
    q = ctx.qkv_rope_split(qkv, kc, vc, table, meta, sh, rope, positions=pos)
    a = ctx.attn_mixed_batch(q, kc, vc, table, meta)
    last = torch.as_tensor(meta[:, 1] + meta[:, 2] - 1, device="cuda").long()
    logits = (a.view(len(x), -1)[last] @ head).float()
    return qkv, q, a, logits, ctx.sample(logits, u, **params)


@pytest.mark.parametrize("side_stream", [False, True])
def test_a_served_step(ctx, side_stream):
    """The operators as a serving step runs them, each checked against its fp64 definition on what it was given."""
    import paper_2511_04791_amd as duet
    from oracle import attention as oa, serving as so
    sh = duet.AttnShape(8, 2, 64, "bf16")
    reqs = [(1, 1, 40), (1, 1, 700), (1, 1, 0), (0, 90, 33), (0, 7, 0)]
    b, _, kc, vc = _rope_inputs(sh, reqs, 8000)
    meta, T, dm, vocab = b.seq_meta, b.num_tokens, 512, 3001
    _, ids, x, _, la, lb, scale = _lora_case(8001, dm, 12 * 64, 16, 3, reqs, [0, -1, 2, 1, 2])
    w, head = _randn(8005, dm, 12 * 64, scale=dm ** -0.5), _randn(8006, dm, vocab, scale=1.0)
    axis = [i % 3 for i in range(32)]
    pos = np.random.default_rng(8007).integers(0, 900, size=(3, T)).astype(np.int32)
    u = torch.rand(len(reqs), generator=torch.Generator().manual_seed(8008))
    params = _mixed_params(8009, len(reqs))
    rope = duet.Rope.base(10000.0, 64, pair_axis=axis, axes=3)
    kg, vg, table = kc.cuda(), vc.cuda(), torch.as_tensor(b.page_table, device="cuda")
    args = (x.cuda(), w.cuda(), head.cuda(), duet.Lora(la.cuda(), lb.cuda(), scale.cuda()), ids, table, meta, sh, rope,
            torch.as_tensor(pos, device="cuda"), kg, vg, u.cuda(), {k: v.cuda() for k, v in params.items()})
    stream = torch.cuda.Stream() if side_stream else torch.cuda.current_stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        qkv, q, a, logits, (tokens, probs) = _step(ctx, duet, *args)
    torch.cuda.synchronize()
    base = (args[0] @ args[1]).cpu()
    _check_lora(qkv, meta, ids, x, base, la, lb, scale)
    _check_rope(sh, b, qkv.cpu(), kc, vc, (q, kg, vg), (_freq(64), False, axis, pos))
    want = oa.mixed_batch(to64(q), to64(kg), to64(vg), b.page_table, meta, 16)
    err = np.abs(to64(a) - want)
    assert err.max() <= 2e-2 * max(1.0, np.abs(want).max()) and err.mean() <= 4e-3
    ids64, probs64 = so.sample(to64(logits), u.numpy(), **{k: v.numpy() for k, v in params.items()})
    assert np.array_equal(tokens.cpu().numpy(), ids64)
    assert (np.abs(to64(probs) - probs64) <= (E + 2.0 ** -33) * probs64).all()


def test_graphs_of_the_operators(ctx):
    """Two captured graphs, replayed in turn between eager calls: each keeps its own batch and takes new inputs."""
    import paper_2511_04791_amd as duet
    sh = duet.AttnShape(8, 2, 64, "bf16")
    rope = duet.Rope.base(10000.0, 64)

    def make(reqs, seed):
        b, qkv, kc, vc = _rope_inputs(sh, reqs, seed)
        meta, ids, x, base, la, lb, scale = _lora_case(seed + 10, 256, 136, 16, 3, reqs)
        s = dict(meta=meta, ids=ids, qkv=qkv.cuda(), kc=kc.cuda(), vc=vc.cuda(), x=x.cuda(), base=base.cuda(),
                 table=torch.as_tensor(b.page_table, device="cuda"), lora=duet.Lora(la.cuda(), lb.cuda(), scale.cuda()),
                 logits=_randn(seed + 20, len(reqs), 70000, scale=2.0, dtype=torch.float32).cuda(),
                 u=torch.rand(len(reqs), device="cuda"), top_p=torch.full((len(reqs),), 0.9, device="cuda"))
        return s

    def call(s):
        q = ctx.qkv_rope_split(s["qkv"], s["kc"], s["vc"], s["table"], s["meta"], sh, rope)
        out = ctx.lora_add(s["x"], s["base"], s["lora"], s["meta"], s["ids"])
        return (q, out) + ctx.sample(s["logits"], s["u"], top_p=s["top_p"])

    sets = [make([(1, 1, 30 * i) for i in range(9)], 8100), make([(0, 200, 17)] + [(1, 1, i) for i in range(400)], 8200)]
    graphs, outs = [], []
    for s in sets:
        call(s)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call(s))
        graphs.append(g)
    for turn in range(4):
        for s in sets:
            s["qkv"].add_(0.25)
            s["x"].mul_(1.125)
            s["u"].copy_(torch.rand_like(s["u"]))
            s["kc"].zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        got = [[t.clone() for t in o] + [s["kc"].clone()] for o, s in zip(outs, sets)]
        for s, g in zip(sets, got):
            s["kc"].zero_()
            want = list(call(s)) + [s["kc"]]
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(g, want)), turn


def test_calls_on_two_streams_at_once(ctx):
    """Without a workspace of the caller's, calls on two streams have their own."""
    import paper_2511_04791_amd as duet
    cases = []
    for seed in (8300, 8400):
        meta, ids, x, base, a, b, scale = _lora_case(seed, 1024, 512, 32, 4, [(1, 1, 3)] * 50 + [(0, 300, 0)])
        cases.append((x.cuda(), base.cuda(), duet.Lora(a.cuda(), b.cuda(), scale.cuda()), meta, ids))
    want = [ctx.lora_add(*c).clone() for c in cases]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i in (0, 1):
            got[i].append(ctx.lora_add(*cases[i], stream=streams[i].cuda_stream))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(g, want[i]) for g in got[i])


def test_one_workspace_for_all(ctx):
    """A workspace of the caller's that holds anything, for every operator in turn and in two graphs."""
    import paper_2511_04791_amd as duet
    sh, rope = duet.AttnShape(8, 2, 64, "bf16"), duet.Rope.base(10000.0, 64)

    def make(reqs, seed):
        b, qkv, kc, vc = _rope_inputs(sh, reqs, seed)
        meta, ids, x, base, la, lb, scale = _lora_case(seed + 1, 256, 136, 16, 3, reqs)
        table, lora = torch.as_tensor(b.page_table, device="cuda"), duet.Lora(la.cuda(), lb.cuda(), scale.cuda())
        qkv, kc, vc, x, base = (t.cuda() for t in (qkv, kc, vc, x, base))
        logits = _randn(seed + 2, len(reqs), 70000, scale=2.0, dtype=torch.float32).cuda()
        u = torch.rand(len(reqs), generator=torch.Generator().manual_seed(seed)).cuda()

        def call(workspace=None):
            q = ctx.qkv_rope_split(qkv, kc, vc, table, meta, sh, rope, workspace=workspace)
            out = ctx.lora_add(x, base, lora, meta, ids, workspace=workspace)
            return (q, out) + ctx.sample(logits, u, workspace=workspace)
        return call

    # Requests past and within those that travel with the arguments; adapters whose rows lie in one run and in none.
    calls = [make([(0, 40, 7)] + [(1, 1, i) for i in range(300)], 8500), make([(1, 1, 9 * i) for i in range(30)], 8600)]
    want = [c() for c in calls]
    ws = torch.full((1 << 24,), 255, dtype=torch.uint8, device="cuda")
    for turn in range(2):
        got = [c(ws) for c in calls]
        assert all(torch.equal(g, w) for a, b in zip(got, want) for g, w in zip(a, b)), turn
    graphs, outs = [], []
    for c in calls:
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(c(ws))
        graphs.append(g)
    for turn in range(3):
        ws.fill_(255 - turn)
        for o in outs:
            for t in o:
                t.zero_()
        for g in graphs:
            g.replay()
        calls[turn % 2](ws)
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for a, b in zip(outs, want) for g, w in zip(a, b)), turn


def test_offsets_past_32_bits(ctx):
    """Pages, rows and logits more than 2^31 elements from the start."""
    import paper_2511_04791_amd as duet
    far = 1 << 30
    # The last pages of a large pool.
    sh = duet.AttnShape(8, 8, 128, "bf16")
    b, qkv, kc, vc = _rope_inputs(sh, [(0, 33, 5), (1, 1, 40)], 8700)
    P, pages = kc.shape[0], far * 2 // (8 * 16 * 128) + 64
    big = [torch.empty(pages, *c.shape[1:], dtype=torch.bfloat16, device="cuda") for c in (kc, vc)]
    for c, at in zip((kc, vc), big):
        at[pages - P:] = c.cuda()
    table = torch.as_tensor(np.where(b.page_table >= 0, b.page_table + pages - P, -1).astype(np.int32), device="cuda")
    q = ctx.qkv_rope_split(qkv.cuda(), big[0], big[1], table, b.seq_meta, sh, duet.Rope(_freq(128)), check_errors=True)
    _check_rope(sh, b, qkv, kc, vc, (q, big[0][pages - P:], big[1][pages - P:]), (_freq(128), False, None, None))
    del big
    # Rows far apart.
    meta, ids, x, base, la, lb, scale = _lora_case(8710, 72, 80, 16, 2, [(1, 1, 0)] * 3, [1, 0, 1])
    room = torch.empty(2 * far + 1024, dtype=torch.bfloat16, device="cuda")
    rows = lambda at, n: torch.as_strided(room, (3, n), (far, 1), at)  # noqa: E731
    xs, bases, out = rows(0, 72), rows(128, 80), rows(256, 80)
    xs.copy_(x), bases.copy_(base)
    ctx.lora_add(xs, bases, duet.Lora(la.cuda(), lb.cuda(), scale.cuda()), meta, ids, out=out)
    _check_lora(out, meta, ids, x, base, la, lb, scale)
    logits = _randn(8720, 3, 900, scale=2.0)
    rows(0, 900).copy_(logits)
    u = torch.tensor([0.1, 0.5, 0.9])
    ids, probs = ctx.sample(rows(0, 900), u.cuda())
    want = ctx.sample(logits.cuda(), u.cuda())
    assert torch.equal(ids, want[0]) and torch.equal(probs, want[1])
