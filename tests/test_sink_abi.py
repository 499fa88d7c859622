"""kvd_sink_attn, kvd_mx_attn, kvd_mx_store, kvd_mx_load and budget.SinkCache on the CPU: refusals before any HIP call,
workspace sizes, the binding's checks, the cache's bookkeeping, and the oracle's own properties."""
import copy
import ctypes
import dataclasses
import pickle

import numpy as np
import pytest
import torch

import oracle as O

kvd = pytest.importorskip("paper_2603_19664_amd.kvd")
lib = kvd.lib
FAKE, MISALIGNED, ODD = 0x10000, 0x10008, 0x10002
BIG = 1 << 40
INT_MAX = 2 ** 31 - 1


def shape(**kw):
    base = dict(d_model=2560, n_q_heads=8, n_kv_heads=4, head_dim=256, rms_eps=1e-6, rope_theta=1e4,
                dtype=kvd.KVD_BF16)
    base.update(kw)
    return kvd.AttnShape(**base)


def ref(x):
    return ctypes.byref(x) if x is not None else None


def view(t_cap=64, t_off=0, k=FAKE, v=FAKE):
    return kvd.KvView(k, v, t_cap, t_off)


def mxv(t_cap=64, t_off=0, k=FAKE, v=FAKE, ks=FAKE, vs=FAKE):
    return kvd.MxView(k, v, ks, vs, t_cap, t_off)


def sink_attn(s=None, q=FAKE, N=1, kv=view(), lens=None, news=None, B=2, T=16, window=8, sink=4, out=FAKE, ws=FAKE, n=BIG):
    return lib.kvd_sink_attn(ref(s or shape()), q, N, ref(kv), lens, news, B, T, window, sink, out, ws, n, None)


def mx_attn(s=None, q=FAKE, N=1, kv=mxv(), lens=None, news=None, B=2, T=16, window=8, sink=4, out=FAKE, ws=FAKE, n=BIG):
    return lib.kvd_mx_attn(ref(s or shape()), q, N, ref(kv), lens, news, B, T, window, sink, out, ws, n, None)


def store(s=None, rows=view(), N=1, kv=mxv(), lens=None, news=None, B=2, T=16, sink=4):
    return lib.kvd_mx_store(ref(s or shape()), ref(rows), N, ref(kv), lens, news, B, T, sink, None)


def load(s=None, rows=view(), N=1, kv=mxv(), lens=None, news=None, B=2, T=16, sink=4):
    return lib.kvd_mx_load(ref(s or shape()), ref(kv), N, lens, news, B, T, sink, ref(rows), None)


COMMON = [
    (kvd.KVD_ERR_UNSUPPORTED, dict(s=shape(head_dim=96))),
    (kvd.KVD_ERR_UNSUPPORTED, dict(s=shape(dtype=5))),
    (kvd.KVD_ERR_SHAPE, dict(s=shape(n_q_heads=6))),
    (kvd.KVD_ERR_SHAPE, dict(N=-1)),
    (kvd.KVD_ERR_SHAPE, dict(B=-1)),
    (kvd.KVD_ERR_SHAPE, dict(B=65536)),
    (kvd.KVD_ERR_SHAPE, dict(T=0)),
    (kvd.KVD_ERR_SHAPE, dict(T=-3)),
    (kvd.KVD_ERR_SHAPE, dict(sink=-1)),
    (kvd.KVD_ERR_NULL, dict(kv=None)),
    (kvd.KVD_ERR_ALIGN, dict(lens=ODD)),
    (kvd.KVD_ERR_ALIGN, dict(news=ODD)),
]


def views(make):
    return [
        (kvd.KVD_ERR_NULL, dict(kv=make(k=0))),
        (kvd.KVD_ERR_NULL, dict(kv=make(v=0))),
        (kvd.KVD_ERR_ALIGN, dict(kv=make(k=MISALIGNED))),
        (kvd.KVD_ERR_ALIGN, dict(kv=make(v=MISALIGNED))),
        (kvd.KVD_ERR_SHAPE, dict(kv=make(t_cap=0))),
        (kvd.KVD_ERR_SHAPE, dict(kv=make(t_off=-1))),
        (kvd.KVD_ERR_SHAPE, dict(kv=make(t_off=64))),
        (kvd.KVD_ERR_SHAPE, dict(T=65, sink=64)),
        (kvd.KVD_ERR_SHAPE, dict(T=65, sink=INT_MAX)),
    ]


ATTN = [
    (kvd.KVD_ERR_SHAPE, dict(window=0)),
    (kvd.KVD_ERR_SHAPE, dict(window=-5)),
    (kvd.KVD_ERR_NULL, dict(q=None)),
    (kvd.KVD_ERR_NULL, dict(out=None)),
    (kvd.KVD_ERR_ALIGN, dict(q=MISALIGNED)),
    (kvd.KVD_ERR_ALIGN, dict(out=MISALIGNED)),
    # a ring that the windows of all new tokens do not fit
    (kvd.KVD_ERR_SHAPE, dict(T=65, window=61, sink=4)),
    (kvd.KVD_ERR_SHAPE, dict(T=65, window=60, sink=4, N=2)),
    (kvd.KVD_ERR_SHAPE, dict(T=INT_MAX, window=INT_MAX, sink=0)),
    (kvd.KVD_ERR_WORKSPACE, dict(ws=None)),
    (kvd.KVD_ERR_WORKSPACE, dict(n=0)),
    (kvd.KVD_ERR_ALIGN, dict(ws=FAKE + 16)),
    (kvd.KVD_ERR_SHAPE, dict(N=1 << 28, B=2, T=1, window=1)),
    (kvd.KVD_ERR_SHAPE, dict(B=65535, N=65535, T=1, window=1)),
]


@pytest.mark.parametrize("status,kw", COMMON + ATTN + views(view))
def test_sink_refusals(status, kw):
    assert sink_attn(**kw) == status
    assert kvd.last_error()


@pytest.mark.parametrize("status,kw", COMMON + ATTN + views(mxv) + [
    (kvd.KVD_ERR_NULL, dict(kv=mxv(ks=0))), (kvd.KVD_ERR_NULL, dict(kv=mxv(vs=0))),
    (kvd.KVD_ERR_ALIGN, dict(kv=mxv(ks=ODD))), (kvd.KVD_ERR_ALIGN, dict(kv=mxv(vs=MISALIGNED)))])
def test_mx_refusals(status, kw):
    assert mx_attn(**kw) == status
    assert kvd.last_error()


ROWS = COMMON + views(mxv) + [
    (kvd.KVD_ERR_NULL, dict(rows=None)),
    (kvd.KVD_ERR_NULL, dict(rows=view(k=0))),
    (kvd.KVD_ERR_ALIGN, dict(rows=view(v=MISALIGNED))),
    (kvd.KVD_ERR_SHAPE, dict(rows=view(t_cap=4), N=5)),
    (kvd.KVD_ERR_SHAPE, dict(rows=view(t_cap=8, t_off=4), N=5)),
    (kvd.KVD_ERR_SHAPE, dict(T=65, N=61)),            # two of the tokens in one row of the ring
    (kvd.KVD_ERR_NULL, dict(kv=mxv(ks=0))), (kvd.KVD_ERR_ALIGN, dict(kv=mxv(vs=MISALIGNED))),
    (kvd.KVD_ERR_SHAPE, dict(B=65535, N=1 << 14, T=1, rows=view(t_cap=1 << 14))),
]


@pytest.mark.parametrize("status,kw", ROWS)
def test_store_and_load_refusals(status, kw):
    assert store(**kw) == status
    assert load(**kw) == status
    assert kvd.last_error()


def test_empty_calls():
    for f in (sink_attn, mx_attn):
        assert f(B=0, q=None, kv=None) == kvd.KVD_OK
        assert f(N=0, q=None, kv=None) == kvd.KVD_OK
    for f in (store, load):
        assert f(B=0, rows=None, kv=None) == kvd.KVD_OK
        assert f(N=0, rows=None, kv=None) == kvd.KVD_OK
    assert lib.kvd_mx_attn(None, FAKE, 1, None, None, None, 1, 1, 1, 0, FAKE, FAKE, BIG, None) == kvd.KVD_ERR_NULL


@pytest.mark.parametrize("dtype", [kvd.KVD_BF16, kvd.KVD_F32])
@pytest.mark.parametrize("heads", [(8, 4, 256), (12, 2, 128), (9, 3, 64), (16, 1, 64)])
def test_workspace_does_not_fall_as_tokens_grow(dtype, heads):
    s = shape(dtype=dtype, n_q_heads=heads[0], n_kv_heads=heads[1], head_dim=heads[2])
    grid = sorted({1, 2, 16, 17, 100, 127, 128, 129, 255, 256, 257, 400, 511, 513, 1000, 2048, 2049, 5000, 16384, 40000,
                   1 << 20, INT_MAX - 8192, *range(1, 6000, 13)})
    for B, N in ((1, 1), (3, 1), (64, 1), (1, 33), (2, 300), (7, 9), (1, 3000)):
        for window, sink in ((INT_MAX, 0), (1024, 4), (64, 0), (1, 100), (4096, INT_MAX)):
            sizes = [lib.kvd_sink_workspace_bytes(ref(s), B, N, t, window, sink) for t in grid]
            assert sizes[0] >= 256 and sizes == sorted(sizes)
    f = lib.kvd_sink_workspace_bytes
    assert f(ref(s), 2, 1, INT_MAX, 1024, 4) == f(ref(s), 2, 1, 5000, 1024, 4)  # a stream without end
    assert f(ref(s), 2, 1, INT_MAX, INT_MAX, 0) == 0
    n = f(ref(s), 2, 1, 16, 8, 4)
    assert sink_attn(s, n=n - 1) == mx_attn(s, n=n - 1) == kvd.KVD_ERR_WORKSPACE


def test_workspace_of_invalid_arguments():
    s, f = shape(), lib.kvd_sink_workspace_bytes
    assert f(None, 1, 1, 1, 1, 0) == 0
    assert f(ref(s), 0, 1, 1, 1, 0) == 0
    assert f(ref(s), 1, 0, 1, 1, 0) == 0
    assert f(ref(s), 1, 1, 0, 1, 0) == 0
    assert f(ref(s), 1, 1, 1, 0, 0) == 0
    assert f(ref(s), 1, 1, 1, 1, -1) == 0
    assert f(ref(s), 65535, 65535, 1, 1, 0) == 0
    assert "too large" in kvd.last_error()


# ------------------------------------------------------------------ the binding

SH = kvd.Shape(512, 8, 4, 64, 1e-6, 1e4, kvd.KVD_BF16)


def _t(*dims, dt=torch.bfloat16):
    return torch.zeros(*dims, dtype=dt)


def test_binding_checks_extents_and_devices():
    q, k, ws = _t(2, 3, 8, 64), _t(2, 4, 20, 64), _t(512, dt=torch.uint8)
    c = kvd.mx_cache(SH, 2, 20, device="cpu")
    assert c.k.shape == (2, 4, 20, 32) and c.v_scale.shape == (2, 4, 20, 2) and c.t_off == 0
    three = torch.zeros(3, dtype=torch.int32)

    def no(match, fn, *a, **kw):
        with pytest.raises(ValueError, match=match):
            fn(SH, *a, **kw)

    f = kvd.kvd_sink_attn
    no("q must be", f, _t(2, 64), k, k, 20, 8, q, ws)
    no("q has shape", f, _t(2, 3, 4, 64), k, k, 20, 8, q, ws)
    no("out has shape", f, q, k, k, 20, 8, _t(2, 8, 64), ws)
    no("out is required", f, q, k, k, 20, 8, None, ws)
    no("ws must be", f, q, k, k, 20, 8, q, None)
    no("kv_len has shape", f, q, k, k, 20, 8, q, ws, kv_len=three)
    no("n_new has shape", f, q, k, k, 20, 8, q, ws, n_new=three)
    no("on the GPU", f, q, k, k, 20, 8, q, ws)
    no("on the GPU", kvd.kvd_mx_attn, q, c, 20, q, ws)
    r = kvd.kvd_mx_store
    no("k and v must both", r, k[0], k, 20, c, 20)
    no("rows_v has shape", r, k, _t(2, 4, 19, 64), 20, c, 20)
    no("rows: rows", r, k, k, 21, c, 30)
    no("rows: rows", r, k, k, 20, c, 30, t_off=1)
    no("kv_len has shape", r, k, k, 20, c, 20, kv_len=three)
    no("n_new has shape", r, k, k, 20, c, 20, n_new=three)
    no("on the GPU", r, k, k, 20, c, 20)
    no("on the GPU", kvd.kvd_mx_load, c, 20, 20, k, k)
    # the cache's own extents
    with pytest.raises(ValueError, match="MxCache"):
        kvd._mx_view(tuple(c), SH, 2, 0)
    for name, bad in (("k", c.k[..., :31]), ("v", c.v[:, :, :19]), ("k_scale", c.k_scale[..., :1]),
                      ("v_scale", c.v_scale[:1])):
        with pytest.raises(ValueError, match="has shape|must be"):
            kvd._mx_view(c._replace(**{name: bad}), SH, 2, 0)
    with pytest.raises(ValueError, match="on the GPU"):
        kvd._mx_view(c, SH, 2, 0)


def test_a_shape_in_use_is_copied_and_pickled_as_its_fields():
    s = kvd.Shape(512, 8, 4, 64, 1e-6, 1e4, kvd.KVD_BF16)
    assert s._ref is s._ref
    for t in (pickle.loads(pickle.dumps(s)), copy.deepcopy(s), copy.copy(s), dataclasses.replace(s)):
        assert t == s and hash(t) == hash(s) and t._ref is not s._ref
    assert s.packed().w_layout == kvd.KVD_W_PACKED and s.packed()._ref is not s._ref


# ------------------------------------------------------------------ the cache's bookkeeping

def sink_cache(**kw):
    from paper_2603_19664_amd.budget import SinkCache
    return SinkCache(SH, device="cpu", **kw)


@pytest.mark.parametrize("kw", [dict(window=0), dict(window=4, room=0), dict(window=4, sink=-1)])
def test_cache_refusals(kw):
    with pytest.raises(ValueError):
        sink_cache(batch=1, **kw)


@pytest.mark.parametrize("window,sink,room", [(1, 0, 1), (5, 2, 1), (4, 0, 6), (3, 7, 4), (8, 1, 3)])
def test_cache_rows_are_the_library_s(window, sink, room):
    c = sink_cache(batch=1, window=window, sink=sink, room=room)
    slots = sink + c.ring
    assert c.k.shape[2] == slots
    want = O.sink_rows(200, slots, sink)
    assert [c.row(t) for t in range(200)] == want.tolist()
    # parts of neighbouring rows that cover the tokens, and no row twice in one call
    for T in range(60):
        for N in range(1, room + 1):
            c.T = T
            parts = list(c._pieces(N))
            assert [t + i for t, n in parts for i in range(n)] == list(range(T, T + N))
            rows = [c.row(t) + i for t, n in parts for i in range(n)]
            assert rows == [c.row(t) for t in range(T, T + N)] and len(set(rows)) == N
            assert max(rows) < slots and len(parts) <= 2


def test_cache_in_4_bits_keeps_no_plain_rows():
    c = sink_cache(batch=2, window=100, sink=4, room=8, mx=True)
    assert c.k.shape == (2, 4, 8, 64) and c.mx.k.shape == (2, 4, 111, 32)


def test_a_refused_call_leaves_the_cache_as_it_was():
    c = sink_cache(batch=1, window=4)
    with pytest.raises(ValueError):
        c.step(_t(1, 512), None, None, None, None, None)
    with pytest.raises(ValueError):
        c.prompt(_t(1, 3, 500), None, None, None, None, _t(1, 3, 8, 64))
    with pytest.raises(ValueError):
        c.prompt(_t(1, 3, 512), None, None, None, None, _t(1, 2, 8, 64))
    assert c.T == 0


# ------------------------------------------------------------------ the oracle itself

def _np(*dims, seed=0):
    return np.random.default_rng(seed).standard_normal(dims)


def test_oracle_window_of_the_whole_past_is_causal_attention():
    T, n_q, n_kv, hd = 9, 4, 2, 8
    q, k, v = _np(2, T, n_q, hd), _np(2, n_kv, T, hd, seed=1), _np(2, n_kv, T, hd, seed=2)
    want, size, _ = O.rows_attention(q, None, None, k, v, [T, 4], [T, 3])
    for window, sink in ((T, 0), (1, T), (3, T), (5, 4)):
        out, sz = O.sink_attention(q, k, v, [T, 4], [T, 3], window, sink)
        assert np.abs(out - want).max() < 1e-13 and np.abs(sz - size).max() < 1e-13


def test_oracle_window_and_sinks_by_their_definition():
    T, hd = 12, 4
    q, k = _np(1, T, 1, hd), _np(1, 1, T, hd, seed=1)
    v = np.eye(T)[None, None]                       # the output is the weights
    k = np.concatenate([k, np.zeros((1, 1, T, T - hd))], -1)
    q = np.concatenate([q, np.zeros((1, T, 1, T - hd))], -1)
    for window in (1, 3, 20):
        for sink in (0, 2, 12):
            out, _ = O.sink_attention(q, k, v, [T], [T], window, sink)
            for p in range(T):
                seen = {t for t in range(p + 1) if t < sink or t > p - window}
                assert {t for t in range(T) if out[0, p, 0, t] > 0} == seen
                assert abs(out[0, p, 0].sum() - 1) < 1e-12


def test_oracle_rows_of_a_ring_hold_the_newest_tokens():
    for slots, sink in ((5, 0), (7, 3), (6, 5)):
        rows, at = O.sink_rows(50, slots, sink), {}
        for t in range(50):
            at[int(rows[t])] = t
            ring = slots - sink
            newest = list(range(min(sink, t + 1))) + list(range(max(sink, t + 1 - ring), t + 1))
            assert sorted(at.values()) == sorted(set(newest)) and max(at) < slots
    assert O.sink_rows(5, 5, 3).tolist() == [0, 1, 2, 3, 4]


def test_oracle_4_bit_numbers():
    x = np.zeros((3, 32))
    x[0, :12] = [0, -0.0, 0.24, 0.25, 0.26, 0.75, 1.25, 2.5, 3.5, 5.0, 7.0, -6.9]
    x[1, :3] = [7.01, -1.0, 0.5]                    # one power of two more
    x[2, 5] = np.inf
    codes, scales = O.mx_round(x)
    assert scales[:, 0].tolist() == [127, 128, 255]
    got = O.mx_values(codes, scales)
    assert got[0, :12].tolist() == [0, 0, 0, 0, 0.5, 1, 1, 2, 4, 4, 6, -6]
    assert got[1, :3].tolist() == [8, -1, 0]
    assert np.isnan(got[2]).all() and not codes[2].any()
    # element 0 in the low half of byte 0
    c, _ = O.mx_round(np.where(np.arange(32) == 0, 6.0, 0.0)[None])
    assert c[0, 0] == 7 and not c[0, 1:].any()
    # what stands for itself stays, and nothing is further off than half a step of the largest
    y = _np(50, 64, seed=3) * 2.0 ** np.random.default_rng(4).integers(-90, 90, (50, 1))
    v = O.mx_values(*O.mx_round(y))
    assert (O.mx_values(*O.mx_round(v)) == v).all()
    top = np.abs(y.reshape(50, 2, 32)).max(-1)
    assert (np.abs(v - y).reshape(50, 2, 32).max(-1) <= top / 3.5).all()
    assert O.mx_round(np.full((1, 32), 1e-40))[1][0, 0] == 27 and O.mx_round(np.full((1, 32), 3e38))[1][0, 0] == 252
