"""Refusals of the split with a norm, the 8-bit cache and decode attention with shared prefixes: documented codes, before any GPU
work; and the fp64 oracles against direct definitions."""
import ctypes

import numpy as np
import pytest

from paper_2511_04791_amd import _native as N

B = ctypes.byref
SHAPE = N.Shape(8, 2, 64, 16, N.BF16, 1)


def _batch(rows):
    arr = (N.SeqMeta * max(1, len(rows)))(*[N.SeqMeta(*r) for r in rows])
    return arr, N.Batch(arr, len(rows))


def _prefixes(length, of):
    p = N.Prefixes(len(length), (ctypes.c_int32 * max(1, len(length)))(*length), (ctypes.c_int32 * max(1, len(of)))(*of))
    return p


DECODES = [(1, 0, 1, 99), (1, 1, 1, 31), (1, 2, 1, 200)]


def test_shared_workspace(native):
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    arr, b = _batch(DECODES)
    assert native.duet_shared_workspace_bytes(B(SHAPE), B(b), None, B(n)) == 0 and n.value >= 3 * 8 * (64 + 2) * 4
    p = _prefixes([32, 16], [0, 0, -1])
    assert native.duet_shared_workspace_bytes(B(SHAPE), B(b), B(p), B(m)) == 0 and m.value > 0
    none_arr, none = _batch([])
    assert native.duet_shared_workspace_bytes(B(SHAPE), B(none), None, B(n)) == 0
    assert native.duet_shared_workspace_bytes(B(SHAPE), B(b), None, None) == -1
    assert native.duet_shared_workspace_bytes(B(SHAPE), None, None, B(n)) == -1
    assert native.duet_shared_workspace_bytes(None, B(b), None, B(n)) == -1


@pytest.mark.parametrize("length,of,code", [([20], [0, 0, -1], -1), ([-16], [0, 0, -1], -1), ([32], [0, 1, -1], -1),
                                            ([32], [0, -2, -1], -1), ([48], [0, 0, -1], -1), ([112], [0, -1, 0], -1),
                                            ([32], [0, 0, 0], 0), ([96], [0, -1, 0], 0), ([], [-1, -1, -1], 0), ([0], [0, 0, 0], 0)])
def test_prefixes(native, length, of, code):
    n = ctypes.c_size_t()
    arr, b = _batch(DECODES)
    p = _prefixes(length, of)
    assert native.duet_shared_workspace_bytes(B(SHAPE), B(b), B(p), B(n)) == code
    cache = N.KvCache(16, 32, 48, 100)
    rc = native.duet_attn_decode_shared(None, B(SHAPE), 64, B(cache), 80, 20, B(b), B(p), 96, 1 << 30, 112, None)
    assert rc == -1 and (b"ctx" in native.duet_last_error()) == (code == 0)


def test_shared_takes_decodes_of_bf16(native):
    n = ctypes.c_size_t()
    arr, b = _batch([(1, 0, 1, 9), (0, 1, 4, 0)])
    assert native.duet_shared_workspace_bytes(B(SHAPE), B(b), None, B(n)) == -2
    arr, b = _batch(DECODES)
    assert native.duet_shared_workspace_bytes(B(N.Shape(8, 2, 64, 16, N.F32, 1)), B(b), None, B(n)) == -2
    assert native.duet_shared_workspace_bytes(B(N.Shape(8, 2, 96, 16, N.BF16, 1)), B(b), None, B(n)) == -2
    assert native.duet_shared_workspace_bytes(B(N.Shape(34, 2, 64, 16, N.BF16, 1)), B(b), None, B(n)) == -2


def test_shared_refuses_too_many_keys(native):
    """Before their parts are listed: of 2000 requests of 2^30 - 16 tokens these would take 33 GB."""
    n = ctypes.c_size_t()
    for requests, code in ((1, 0), (5, -2), (2000, -2), (3000, -2)):
        arr, b = _batch([(1, r, 1, (1 << 30) - 17) for r in range(requests)])
        assert native.duet_shared_workspace_bytes(B(SHAPE), B(b), None, B(n)) == code


def test_prefix_lists_are_needed(native):
    n = ctypes.c_size_t()
    arr, b = _batch(DECODES)
    for p in (N.Prefixes(1, None, (ctypes.c_int32 * 3)(0, 0, 0)), N.Prefixes(0, None, None), N.Prefixes(-1, None, (ctypes.c_int32 * 3)()),
              N.Prefixes(65537, (ctypes.c_int32 * 1)(), (ctypes.c_int32 * 3)())):
        assert native.duet_shared_workspace_bytes(B(SHAPE), B(b), B(p), B(n)) == -1


@pytest.mark.parametrize("eps", [0.0, -1.0, float("nan"), float("inf")])
def test_norm_eps(native, eps):
    arr, b = _batch([(1, 0, 1, 10)])
    norm = N.HeadNorm(None, None, eps)
    rc = native.duet_qkv_norm_rope_split(None, B(SHAPE), B(norm), None, 16, None, 32, 48, 64, 10, 80, 4, B(b), None, 0, None)
    assert rc == -1 and b"eps" in native.duet_last_error()


def test_split8_needs_a_cache(native):
    arr, b = _batch([(1, 0, 1, 10)])

    def call(cache, shape=SHAPE):
        return native.duet_qkv_split8(None, B(shape), None, None, 16, None, 32, B(cache) if cache else None, 80, 4, B(b), None, 0, None)
    for cache in (None, N.KvCache(None, 64, 96, 10), N.KvCache(48, None, 96, 10), N.KvCache(48, 64, None, 10), N.KvCache(40, 64, 96, 10),
                  N.KvCache(48, 64, 100, 10), N.KvCache(48, 48, 96, 10)):
        assert call(cache) == -1 and b"ctx" not in native.duet_last_error()
    assert call(N.KvCache(48, 64, 96, 10), N.Shape(8, 2, 64, 16, N.F32, 1)) == -2
    assert call(N.KvCache(48, 64, 96, 10)) == -1 and b"ctx" in native.duet_last_error()


def test_python_descriptions():
    import paper_2511_04791_amd as duet
    torch = pytest.importorskip("torch")
    u8 = dict(dtype=torch.uint8)
    with pytest.raises(ValueError):
        duet.Cache8(torch.zeros(3, 2, 16, 64, **u8), torch.zeros(3, 2, 64, 16, **u8), torch.zeros(3, 2, 2, 16, **u8))  # on the host
    with pytest.raises(ValueError):
        duet.Cache8(torch.zeros(3, 2, 16, 64, **u8), torch.zeros(3, 2, 16, 64, **u8), torch.zeros(3, 2, 2, 16, **u8))
    with pytest.raises(ValueError):
        duet.Cache8(torch.zeros(3, 2, 16, 64, **u8), torch.zeros(3, 2, 64, 16, **u8), torch.zeros(3, 2, 16, 2, **u8))
    with pytest.raises(ValueError):
        duet.HeadNorm(torch.zeros(64))


# ---- the oracles ----------------------------------------------------------------------------------


def test_e4m3_is_torchs():
    torch = pytest.importorskip("torch")
    from oracle import cache8 as oc
    want = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oc.e4m3_values(), want, equal_nan=True)


def test_encode_is_the_nearest():
    torch = pytest.importorskip("torch")
    from oracle import cache8 as oc
    rng = np.random.default_rng(1)
    x = (rng.normal(size=(300, 32)) * np.exp2(rng.integers(-60, 60, size=(300, 1)))).astype(np.float32).astype(np.float64)
    x[0], x[1, 0] = 0.0, 448.0
    x[2, 3], x[3, 4] = np.inf, np.nan
    q, e = oc.encode(x)
    s = 2.0 ** (e.astype(np.float64) - 127)
    fin = np.where(np.isfinite(x), np.abs(x), 0).max(-1)
    assert (fin <= 448 * s).all() and ((fin > 224 * s) | (e == 1)).all()
    want = torch.from_numpy(x / s[:, None]).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(q, np.where(np.isfinite(x), want, np.nan), equal_nan=True)


def test_decode_attention_is_the_mixed_batchs():
    from oracle import attention as oa, cache8 as oc
    rng = np.random.default_rng(2)
    k, v, q = rng.normal(size=(9, 2, 16, 8)), rng.normal(size=(9, 2, 8, 16)), rng.normal(size=(2, 4, 8))
    table, meta = np.array([[3, 1, 7, -1], [0, 5, 2, 8]]), np.array([(1, 0, 1, 40), (1, 1, 1, 63)])
    out, mag, _ = oc.decode_attention(q, k, v, table, meta)
    assert np.allclose(out, oa.mixed_batch(q, k, v, table, meta), rtol=1e-12) and (mag >= np.abs(out) - 1e-12).all()


def test_normalised_rows():
    from oracle import cache8 as oc
    rng = np.random.default_rng(3)
    x = rng.normal(size=(5, 4 * 8))
    y = oc.normalised(x, 2, 1, 8, None, np.full(8, 2.0), 0.0).reshape(5, 4, 8)
    assert np.allclose((y[:, :2] ** 2).mean(-1), 1) and np.allclose((y[:, 2] ** 2).mean(-1), 4)
    assert np.array_equal(y[:, 3], x.reshape(5, 4, 8)[:, 3])
