"""Refusals of the rotating QKV split, the adapters and sampling: documented codes, before any GPU work; and the fp64
oracles against direct definitions."""
import ctypes

import numpy as np
import pytest

from paper_2511_04791_amd import _native as N

B = ctypes.byref


def _batch(rows):
    arr = (N.SeqMeta * max(1, len(rows)))(*[N.SeqMeta(*r) for r in rows])
    return arr, N.Batch(arr, len(rows))


def _rope(n=32, axes=1, axis=None, adjacent=0, freq=1.0, rot=None):
    f = (ctypes.c_double * n)(*([freq] * n))
    a = (ctypes.c_uint8 * n)(*axis) if axis is not None else None
    r = N.Rope(2 * n if rot is None else rot, adjacent, axes, f, a)
    r._keep = (f, a)
    return r


SHAPE = N.Shape(8, 2, 64, 16, N.BF16, 1)


@pytest.mark.parametrize("rope,code", [(_rope(n=36), -1), (_rope(n=4), -1), (_rope(rot=0), -1), (_rope(n=20), -1),
                                       (_rope(adjacent=2), -1), (_rope(axes=0), -1), (_rope(axes=5), -1),
                                       (_rope(axes=2, axis=[0] * 31 + [2]), -1), (_rope(freq=float("nan")), -1),
                                       (_rope(freq=float("inf")), -1), (_rope(freq=65.0), -1), (None, -1)])
def test_rope_descriptions(native, rope, code):
    arr, b = _batch([(1, 0, 1, 10)])
    rc = native.duet_qkv_rope_split(None, B(SHAPE), B(rope) if rope else None, 16, None, 32, 48, 64, 10, 80, 4, B(b), 96,
                                    1 << 20, None)
    assert rc == code and b"ctx" not in native.duet_last_error()


def test_rope_needs_a_context_and_a_shape(native):
    arr, b = _batch([(1, 0, 1, 10)])
    args = (16, None, 32, 48, 64, 10, 80, 4, B(b), 96, 1 << 20, None)
    assert native.duet_qkv_rope_split(None, B(SHAPE), B(_rope()), *args) == -1 and b"ctx" in native.duet_last_error()
    assert native.duet_qkv_rope_split(None, None, B(_rope()), *args) == -1 and b"shape" in native.duet_last_error()


def test_workspace_sizes(native):
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    arr, b = _batch([(1, 0, 1, 10), (0, 0, 99, 0)])
    none_arr, none = _batch([])
    assert native.duet_rope_workspace_bytes(B(b), B(n)) == 0 and n.value >= 4 + 2 * 16
    assert native.duet_rope_workspace_bytes(B(none), B(n)) == 0
    assert native.duet_rope_workspace_bytes(None, B(n)) == -1
    assert native.duet_rope_workspace_bytes(B(b), None) == -1
    lora = N.Lora(None, None, None, 3, 16, 64, 128)
    assert native.duet_lora_workspace_bytes(B(lora), B(b), B(m)) == 0 and m.value >= 100 * 16 * 4
    assert native.duet_lora_workspace_bytes(B(lora), B(none), B(m)) == 0
    assert native.duet_lora_workspace_bytes(None, B(b), B(m)) == -1
    big_arr, big = _batch([(0, 0, (1 << 22) + 1, 0)])
    assert native.duet_lora_workspace_bytes(B(lora), B(big), B(m)) == -2


def test_sample_workspace(native):
    n = ctypes.c_size_t()
    for rows, vocab in ((0, 100), (1, 1000), (1, 65535), (65, 1 << 18)):
        assert native.duet_sample_workspace_bytes(rows, vocab, B(n)) == 0
    for rows, vocab in ((1, 65536), (64, 128256)):
        assert native.duet_sample_workspace_bytes(rows, vocab, B(n)) == 0 and n.value >= rows * 4096 * 8
    for rows, vocab, code in ((-1, 10, -1), (1, 0, -1), (1, (1 << 18) + 1, -2), ((1 << 20) + 1, 10, -1)):
        assert native.duet_sample_workspace_bytes(rows, vocab, B(n)) == code
    assert native.duet_sample_workspace_bytes(1, 10, None) == -1


@pytest.mark.parametrize("kw,code", [(dict(rank=4), -2), (dict(rank=136), -2), (dict(rank=20), -2), (dict(num_adapters=0), -1),
                                     (dict(d_in=12), -1), (dict(d_out=0), -1), (dict(d_out=(1 << 20) + 8), -1)])
def test_lora_descriptions(native, kw, code):
    arr, b = _batch([(1, 0, 1, 10)])
    m = ctypes.c_size_t()
    lora = N.Lora(None, None, None, *[kw.get(k, v) for k, v in dict(num_adapters=3, rank=16, d_in=64, d_out=128).items()])
    assert native.duet_lora_workspace_bytes(B(lora), B(b), B(m)) == code


def test_lora_needs_a_context(native):
    arr, b = _batch([(1, 0, 1, 10)])
    lora = N.Lora(16, 32, None, 3, 16, 64, 128)
    ids = (ctypes.c_int32 * 1)(0)
    assert native.duet_lora_add(None, B(lora), 48, 64, 64, 128, 80, 128, B(b), ids, 96, 1 << 20, None) == -1
    assert b"ctx" in native.duet_last_error()


def test_sample_needs_a_context(native):
    assert native.duet_sample(None, 16, 0, 1, 10, 10, None, 16, 16, None, None, 0, None) == -1
    assert b"ctx" in native.duet_last_error()


def test_python_descriptions():
    import paper_2511_04791_amd as duet
    assert duet.Rope.base(10000.0, 64).c.rot_dim == 64
    for axis in ([0] * 31, [0] * 31 + [3], [0] * 31 + [-1]):
        with pytest.raises(ValueError):
            duet.Rope([1.0] * 32, pair_axis=axis, axes=3)
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        duet.Lora(torch.zeros(2, 8, 16, dtype=torch.bfloat16), torch.zeros(2, 16, 8, dtype=torch.bfloat16))  # on the host


# ---- refusals that need a context -------------------------------------------------------------------


@pytest.mark.gpu
class TestWithContext:
    @pytest.fixture(scope="class")
    def ctx(self):
        import paper_2511_04791_amd as duet
        c = duet.Context(0)
        yield c
        c.close()

    def test_rope(self, native, ctx):
        arr, b = _batch([(1, 0, 1, 10)])

        def call(qkv=16, q=32, kc=48, vc=64, pages=10, table=80, max_pages=4, ws=96, nbytes=1 << 20, batch=b, shape=SHAPE):
            return native.duet_qkv_rope_split(ctx.handle, B(shape), B(_rope()), qkv, None, q, kc, vc, pages, table, max_pages,
                                              B(batch), ws, nbytes, None)
        for kw, code in ((dict(qkv=None), -1), (dict(q=None), -1), (dict(kc=None), -1), (dict(vc=None), -1),
                         (dict(ws=None, batch=_batch([(1, r, 1, 10) for r in range(257)])[1]), -1),
                         (dict(table=None), -1), (dict(q=16), -1), (dict(q=40), -1), (dict(kc=52), -1), (dict(ws=100), -1),
                         (dict(pages=0), -1), (dict(max_pages=0), -1), (dict(nbytes=256), -3),
                         (dict(shape=N.Shape(8, 2, 96, 16, N.BF16, 1)), -2), (dict(shape=N.Shape(8, 3, 64, 16, N.BF16, 1)), -2),
                         (dict(batch=_batch([(1, 0, 2, 5)])[1]), -1), (dict(batch=_batch([(0, 3, 2, 5)])[1]), -1)):
            assert call(**kw) == code, kw
            assert native.duet_last_error()

    def test_lora(self, native, ctx):
        arr, b = _batch([(1, 0, 1, 10), (0, 1, 3, 0)])

        def call(a=16, bb=32, x=48, ldx=64, base=64, ldb=128, out=80, ldo=128, ids=(0, 2), ws=96, nbytes=1 << 20):
            lora = N.Lora(a, bb, None, 3, 16, 64, 128)
            c_ids = (ctypes.c_int32 * 2)(*ids) if ids else None
            return native.duet_lora_add(ctx.handle, B(lora), x, ldx, base, ldb, out, ldo, B(b), c_ids, ws, nbytes, None)
        for kw, code in ((dict(a=None), -1), (dict(bb=None), -1), (dict(x=None), -1), (dict(base=None), -1), (dict(out=None), -1),
                         (dict(ids=None), -1), (dict(ids=(0, 3)), -1), (dict(ids=(-2, 0)), -1), (dict(ldx=56), -1),
                         (dict(ldx=68), -1), (dict(ldb=120), -1), (dict(ldo=132), -1), (dict(x=50), -1), (dict(ws=104), -1),
                         (dict(out=48), -1), (dict(out=64, ldo=136), -1), (dict(ws=None), -1), (dict(nbytes=256), -3)):
            assert call(**kw) == code, kw
            assert native.duet_last_error()

    def test_sample(self, native, ctx):
        def call(logits=16, dtype=0, rows=1, vocab=10, stride=10, u=16, ids=16, ws=None, nbytes=0):
            return native.duet_sample(ctx.handle, logits, dtype, rows, vocab, stride, None, u, ids, None, ws, nbytes, None)
        big = dict(vocab=100000, stride=100000)
        for kw, code in ((dict(logits=None), -1), (dict(u=None), -1), (dict(ids=None), -1), (dict(dtype=2), -2), (dict(rows=-1), -1),
                         (dict(rows=(1 << 20) + 1), -1), (dict(vocab=0), -1), (dict(vocab=(1 << 18) + 1, stride=1 << 19), -2),
                         (dict(stride=9), -1), (dict(logits=17), -1), (dict(logits=18, dtype=1), -1), (dict(big), -1),
                         (dict(big, ws=16, nbytes=4096), -3), (dict(big, ws=24, nbytes=1 << 20), -1)):
            assert call(**kw) == code, kw
            assert native.duet_last_error()
        assert call(rows=0) == 0

    def test_python(self, ctx):
        import paper_2511_04791_amd as duet
        import torch
        z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
        sh = duet.AttnShape(8, 2, 64, "bf16")
        meta, rope = [(1, 1, 10)], duet.Rope.base(10000.0, 64)
        qkv, kc, vc, table = z(1, 768), z(3, 2, 16, 64), z(3, 2, 64, 16), z(1, 4, dt=torch.int32)
        for bad in (dict(qkv=z(2, 768)), dict(qkv=z(1, 768, dt=torch.float32)), dict(kc=z(3, 2, 64, 16)), dict(vc=vc.cpu()),
                    dict(table=z(1, 4, dt=torch.int64)), dict(table=z(0, 4, dt=torch.int32)),
                    dict(positions=z(3, 1, dt=torch.int32)), dict(positions=z(1, 1, dt=torch.int64)), dict(q=z(1, 8, 128))):
            kw = dict(dict(qkv=qkv, kc=kc, vc=vc, table=table), **bad)
            with pytest.raises(ValueError):
                ctx.qkv_rope_split(kw["qkv"], kw["kc"], kw["vc"], kw["table"], meta, sh, rope, q=kw.get("q"),
                                   positions=kw.get("positions"))
        far = torch.zeros(1 << 20, dtype=torch.uint8)
        with pytest.raises(ValueError):
            ctx.qkv_rope_split(qkv, kc, vc, table, meta, sh, rope, workspace=far)
        lora = duet.Lora(z(2, 8, 16), z(2, 24, 8))
        for ws in (far, z(1 << 20)[::2]):
            with pytest.raises(ValueError):
                ctx.lora_add(z(1, 16), z(1, 24), lora, meta, [0], workspace=ws)
        with pytest.raises(duet.DuetError):
            ctx.lora_add(z(1, 16), z(1, 24), lora, meta, [0], workspace=z(8))
        with pytest.raises(ValueError):
            ctx.sample(z(4, 100), z(4, dt=torch.float32), workspace=far)
        for x, base, ids, out in ((z(1, 24), z(1, 24), [0], None), (z(1, 16), z(2, 24), [0], None), (z(1, 16), z(1, 24), [0, 1], None),
                                  (z(1, 16), z(1, 24), [0], z(1, 24, dt=torch.float32)), (z(1, 16).cpu(), z(1, 24), [0], None)):
            with pytest.raises(ValueError):
                ctx.lora_add(x, base, lora, meta, ids, out=out)
        x, u = z(4, 100, dt=torch.float32), z(4, dt=torch.float32)
        for args, kw in (((x.half(), u), {}), ((x, u[:3]), {}), ((x.t(), u), {}), ((x, u), dict(top_k=u)), ((x, u), dict(top_p=u[:2])),
                         ((x, u), dict(out=u)), ((x, u), dict(temperature=u.double()))):
            with pytest.raises(ValueError):
                ctx.sample(*args, **kw)


# ---- the oracles --------------------------------------------------------------------------------------


def test_oracle_sample_draws_by_rank():
    from oracle.serving import sample_row
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    assert [sample_row(x, u=u)[0] for u in (0.0, 0.39, 0.41, 0.69, 0.71, 0.89, 0.91, 0.999)] == [1, 1, 3, 3, 2, 2, 0, 0]
    assert [sample_row(x, top_p=0.6, u=u)[0] for u in (0.0, 0.57, 0.58, 0.99)] == [1, 1, 3, 3]
    assert [sample_row(x, top_k=3, top_p=0.4, u=u)[0] for u in (0.0, 0.99)] == [1, 1]
    assert [sample_row(x, min_p=0.6, u=u)[0] for u in (0.0, 0.99)] == [1, 3]
    assert sample_row(x, top_k=2, u=0.0)[1] == pytest.approx(4 / 7)
    assert sample_row(np.array([1.0, 2.0, 2.0]), temperature=0.0) == (1, 1.0)
    assert sample_row(np.array([-np.inf, np.nan])) == (-1, 0.0)


def test_oracle_sample_frequencies():
    from oracle.serving import sample_row
    x = np.array([0.3, -1.0, 2.0, 0.5, 0.5])
    got = np.bincount([sample_row(x, temperature=0.7, u=(i + 0.5) / 4000)[0] for i in range(4000)], minlength=5) / 4000
    want = np.exp(x / 0.7) / np.exp(x / 0.7).sum()
    assert np.abs(got - want).max() <= 2 / 4000


def test_oracle_rotation_keeps_lengths_and_differences():
    """A rotated query and key depend on the difference of their positions only."""
    from oracle.serving import rotate
    rng = np.random.default_rng(1)
    q, k, f = rng.standard_normal(64), rng.standard_normal(64), 10000.0 ** (-np.arange(24) / 24)
    for adjacent in (False, True):
        a = rotate(q, 7 * f, adjacent) @ rotate(k, 3 * f, adjacent)
        b = rotate(q, 1007 * f, adjacent) @ rotate(k, 1003 * f, adjacent)
        assert a == pytest.approx(b, abs=1e-9)
        assert np.linalg.norm(rotate(q, 5 * f, adjacent)) == pytest.approx(np.linalg.norm(q))
        assert np.array_equal(rotate(q, 5 * f, adjacent)[48:], q[48:])
