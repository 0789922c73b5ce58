"""GPU tests of the rotating QKV split, the adapters and sampling at values and batches where ordinary inputs do not reach:
hidden values past bf16's largest, infinite weights, batches of no requests, masked slices,
results in the place of inputs, broken batches, adapters whose lists are
uploaded."""
import numpy as np
import pytest

from _helpers import to64
from test_gpu_serving_ops import E, U, _check_lora, _lora_case, _randn

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ctx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2511_04791_amd as duet
    c = duet.Context(0)
    yield c
    c.close()


# Of the adapters' second product: ranks of each of its kernels, padded ones among them, and tiles of few rows and of many.
UP = [(rank, rows) for rank in (8, 16, 24, 64, 128) for rows in (3, 40)]


@pytest.mark.parametrize("rank,rows", UP)
def test_lora_hidden_values_past_the_largest_bf16(ctx, rank, rows):
    """h between bf16's largest and fp32's, of both signs, times weights that bring the result back: finite in fp32, so here too."""
    import paper_2511_04791_amd as duet
    x = torch.zeros(rows, 16, dtype=torch.bfloat16)
    x[:, 0] = torch.finfo(torch.bfloat16).max
    x[:, 1] = torch.linspace(1.0, 1.75, rows) * 2.0 ** 119
    x[1::2] = -x[1::2]
    a = torch.zeros(1, rank, 16, dtype=torch.bfloat16)
    a[:, :, :2] = 1
    b = (_randn(9000 + rank, 1, 72, rank) * 2.0 ** -20).to(torch.bfloat16)
    h = x.float() @ a[0].float().t()
    assert torch.isfinite(h).all() and torch.isinf(h.to(torch.bfloat16)).all()
    base = _randn(9001, rows, 72)
    got = ctx.lora_add(x.cuda(), base.cuda(), duet.Lora(a.cuda(), b.cuda()), [(0, rows, 0)], [0])
    _check_lora(got, np.array([[0, 0, rows, 0]]), [0], x, base, a, b, None)


@pytest.mark.parametrize("rank,rows", UP)
def test_lora_infinite_weights(ctx, rank, rows):
    """An infinity of B gives one of h's sign (NaN beside another of the other sign, or where h is zero), whatever h's own
    rounding to bf16 leaves out; the other columns are as without it."""
    import paper_2511_04791_amd as duet
    meta, ids, x, base, a, b, _ = _lora_case(9100 + rank, 40, 136, rank, 2, [(0, rows, 0)], [1])
    inf = float("inf")
    a[1, 1] = 0  # a hidden value of zero
    a[1, 2], a[1, 2, 0] = 0, 1
    x[1, 0] = 3.0  # one that bf16 holds
    b[1, 5, 0], b[1, 6, 2], b[1, 70, 2], b[1, 71, 0], b[1, 71, 2] = inf, inf, -inf, inf, -inf
    b[1, 130, 1], b[1, 131, 3] = inf, float("nan")
    lora = duet.Lora(a.cuda(), b.cuda())
    got = to64(ctx.lora_add(x.cuda(), base.cuda(), lora, meta, ids))
    with np.errstate(invalid="ignore"):
        h = to64(x) @ to64(a)[1].T
        want = to64(base) + (h[:, None] * to64(b)[1]).sum(-1)
    special = [5, 6, 70, 71, 130, 131]
    assert np.array_equal(got[:, special], want[:, special], equal_nan=True) and not np.isfinite(want[:, special]).any()
    rest = [i for i in range(136) if i not in special]
    _check_lora(torch.from_numpy(got[:, rest]), meta, ids, x, base[:, rest], a, b[:, rest], None)


@pytest.mark.parametrize("workspace", [False, True])
def test_empty_batches(ctx, workspace):
    """A batch of no requests does nothing; a workspace's error word is cleared."""
    import ctypes

    import paper_2511_04791_amd as duet
    from paper_2511_04791_amd import _native as N
    lib, B = N.lib(), ctypes.byref
    buf = torch.full((1 << 16,), 255, dtype=torch.uint8, device="cuda")
    p = [buf.data_ptr() + 4096 * i for i in range(8)]
    ws, st = p[6] if workspace else None, torch.cuda.current_stream().cuda_stream
    none = N.Batch((N.SeqMeta * 1)(), 0)
    rope = duet.Rope.base(10000.0, 64)
    n = ctypes.c_size_t()
    assert lib.duet_rope_workspace_bytes(B(none), B(n)) == 0 and n.value <= 4096
    assert lib.duet_qkv_rope_split(ctx.handle, B(N.Shape(8, 2, 64, 16, N.BF16, 1)), B(rope.c), p[0], None, p[1], p[2], p[3], 1, p[4],
                                   1, B(none), ws, 4096 if workspace else 0, st) == 0, lib.duet_last_error()
    if workspace:
        assert lib.duet_check_device_error(ctx.handle, ws, st) == 0
    lora = N.Lora(p[0], p[1], None, 1, 8, 8, 8)
    assert lib.duet_lora_workspace_bytes(B(lora), B(none), B(n)) == 0 and n.value <= 4096
    assert lib.duet_lora_add(ctx.handle, B(lora), p[2], 8, p[3], 8, p[4], 8, B(none), None, p[6], 4096, st) == 0
    assert lib.duet_sample(ctx.handle, p[0], N.BF16, 0, 8, 8, None, p[1], p[2], p[3], None, 0, st) == 0
    torch.cuda.synchronize()
    kept = buf.cpu().numpy()
    kept[4096 * 6:4096 * 6 + 4] = 255
    assert (kept == 255).all()
    kc, vc = torch.zeros(1, 2, 16, 64, device="cuda"), torch.zeros(1, 2, 64, 16, device="cuda")
    q = ctx.qkv_rope_split(torch.zeros(0, 768, device="cuda"), kc, vc, torch.zeros(0, 1, dtype=torch.int32, device="cuda"),
                           np.zeros((0, 4), np.int32), duet.AttnShape(8, 2, 64, "f32"), rope)
    assert q.shape == (0, 8, 64)


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sample_greedy_rows_with_masked_slices(ctx, rows, dtype):
    """Rows that several workgroups share, where the mask leaves some of them no token: the lowest index of the largest logit."""
    vocab = 70001
    for kept in ([vocab - 1], [vocab - 3, vocab - 1], [0], [0, vocab - 1], [35000, 35001, vocab - 1], []):
        x = torch.full((rows, vocab), -float("inf"))
        for i in kept:
            x[:, i] = -7.5
        x = x.to(dtype)
        want = kept[0] if kept else -1
        u = torch.full((rows,), 0.5, device="cuda")
        for params in (dict(temperature=torch.zeros(rows)), dict(top_k=torch.ones(rows, dtype=torch.int32)),
                       dict(top_p=torch.zeros(rows))):
            ids, probs = ctx.sample(x.cuda(), u, **{k: v.cuda() for k, v in params.items()})
            assert (ids == want).all() and (probs == (1.0 if kept else 0.0)).all(), (kept, params)


def test_sample_results_in_the_place_of_others(ctx):
    """ids and probs are refused where they are each other or an input; nothing is written then."""
    import paper_2511_04791_amd as duet
    rows = 4
    x = _randn(9200, rows, 100, dtype=torch.float32).cuda()
    f = lambda v: torch.full((rows,), v, device="cuda")  # noqa: E731
    u, p, t, m = f(0.5), f(0.9), f(0.7), f(0.1)
    k, ids = torch.full((rows,), 7, dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    as_int = lambda v: v.view(torch.int32)  # noqa: E731
    params = dict(temperature=t, top_k=k, top_p=p, min_p=m)
    inputs = [v.clone() for v in (x, u, t, k, p, m, ids)]
    for kw in (dict(out=ids, probs=ids.view(torch.float32)), dict(out=k), dict(out=as_int(u)), dict(probs=u), dict(probs=t),
               dict(probs=p), dict(out=as_int(m)), dict(probs=x.view(-1)[:rows])):
        with pytest.raises(duet.DuetError) as e:
            ctx.sample(x, u, **params, **kw)
        assert e.value.code == -1
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(inputs, (x, u, t, k, p, m, ids)))
    ctx.sample(x, u, **params, out=ids)


@pytest.mark.parametrize("meta", [[[1, 0, 1, 5], [1, -1, 1, 5]], [[0, 0, 0, 5]], [[1, 0, 2, 0], [0, 5, -5, 0]]])
def test_broken_batches_that_end_at_row_zero(ctx, meta):
    """Requests whose rows are not packed, or are none, are refused also where the last of them ends at row 0."""
    import paper_2511_04791_amd as duet
    meta = np.array(meta, np.int32)
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    with pytest.raises(duet.DuetError) as e:
        ctx.qkv_rope_split(z(0, 768), z(3, 2, 16, 64), z(3, 2, 64, 16), z(2, 4, dt=torch.int32), meta,
                           duet.AttnShape(8, 2, 64, "bf16"), duet.Rope.base(10000.0, 64))
    assert e.value.code == -1 and "request" in str(e.value)
    with pytest.raises(duet.DuetError) as e:
        ctx.lora_add(z(0, 16), z(0, 24), duet.Lora(z(2, 8, 16), z(2, 24, 8)), meta, [0] * len(meta))
    assert e.value.code == -1 and "request" in str(e.value)


# ---- adapters whose lists do not travel with the launch ---------------------------------------------


def _lora_lists(reqs, ids):
    """(tiles, listed rows) of the rows by adapter: tiles of up to 64 rows, listed where they do not follow each other."""
    starts = np.concatenate([[0], np.cumsum([q for _, q, _ in reqs])])
    tiles = listed = 0
    for a in np.unique(ids):
        rows = np.concatenate([np.arange(starts[r], starts[r + 1]) for r in range(len(reqs)) if ids[r] == a])
        for i in range(0, len(rows), 64):
            tile = rows[i:i + 64]
            tiles += 1
            listed += len(tile) if tile[-1] - tile[0] != len(tile) - 1 else 0
    return tiles, listed


def _interleaved(counts):
    """Single rows of adapters 0, 1, ..., counts[a] of each, none beside its like as far as that goes."""
    order = sorted((((i + 0.5) / n, a) for a, n in enumerate(counts) for i in range(n)))
    return [(1, 1, 0)] * len(order), [a for _, a in order]


LISTS = {
    # Up to 128 tiles and 256 listed rows travel with the launch; both sides of each limit.
    "256 listed": (_interleaved([128, 128]), (4, 256)),
    "257 listed": (_interleaved([128, 126, 3]), (5, 257)),
    "128 tiles": (([(1, 1, 0)] * 128, list(range(128))), (128, 0)),
    "129 tiles": (([(1, 1, 0)] * 129, list(range(129))), (129, 0)),
    # A running batch, rows without an adapter among them; long and short tiles, in runs and not; more tiles than 512.
    "decode": (([(1, 1, 0)] * 431, [(i * 7) % 5 - 1 for i in range(431)]), None),
    "mixed": (([(1, 1, 0)] * 300 + [(0, 130, 0), (0, 17, 3), (0, 64, 0), (0, 70, 1)],
               [i % 3 for i in range(300)] + [0, 3, 2, 3]), None),
    "many adapters": (([(1, 1, 0), (0, 2, 0)] * 300, list(range(600))), (600, 0)),
}


@pytest.mark.parametrize("rank", [8, 16, 24, 32, 64, 88, 128])
@pytest.mark.parametrize("name", list(LISTS))
def test_lora_lists(ctx, name, rank):
    import paper_2511_04791_amd as duet
    (reqs, ids), counts = LISTS[name]
    tiles, listed = _lora_lists(reqs, np.asarray(ids))
    assert (counts is None and (tiles > 128 or listed > 256)) or (tiles, listed) == counts
    meta, ids, x, base, a, b, scale = _lora_case(9300 + rank, 72, 136, rank, max(ids) + 1, reqs, ids)
    none = np.repeat(np.asarray(ids) < 0, meta[:, 2])
    for in_place in (False, True):
        given = base.cuda()
        got = ctx.lora_add(x.cuda(), given, duet.Lora(a.cuda(), b.cuda(), scale.cuda()), meta, ids, out=given if in_place else None)
        _check_lora(got, meta, ids, x, base, a, b, scale)
        assert torch.equal(got.cpu()[none], base[none]) and (in_place or torch.equal(given.cpu(), base))


@pytest.mark.parametrize("rank", [16, 64, 128])
def test_lora_lists_of_wide_projections(ctx, rank):
    """Uploaded lists with several parts of the input and several workgroups a tile."""
    import paper_2511_04791_amd as duet
    reqs = [(1, 1, 0)] * 290 + [(0, 200, 0)]
    meta, ids, x, base, a, b, scale = _lora_case(9400 + rank, 4104, 1544, rank, 4, reqs, [i % 4 for i in range(290)] + [2])
    got = ctx.lora_add(x.cuda(), base.cuda(), duet.Lora(a.cuda(), b.cuda(), scale.cuda()), meta, ids)
    _check_lora(got, meta, ids, x, base, a, b, scale)
