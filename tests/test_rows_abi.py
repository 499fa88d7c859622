"""kvd_prefix_attn, kvd_weighted_attn and kvd_evict on the CPU: refusals before any HIP call, workspace sizes, the
binding's checks, and the oracle's own properties."""
import ctypes

import numpy as np
import pytest
import torch

import oracle as O

kvd = pytest.importorskip("paper_2603_19664_amd.kvd")
lib = kvd.lib
FAKE, MISALIGNED, ODD = 0x10000, 0x10008, 0x10002
BIG = 1 << 40


def shape(**kw):
    base = dict(d_model=2560, n_q_heads=8, n_kv_heads=4, head_dim=256, rms_eps=1e-6, rope_theta=1e4,
                dtype=kvd.KVD_BF16)
    base.update(kw)
    return kvd.AttnShape(**base)


def ref(x):
    return ctypes.byref(x) if x is not None else None


def view(t_cap=64, t_off=0, k=FAKE, v=FAKE):
    return kvd.KvView(k, v, t_cap, t_off)


def prefix(s=None, q=FAKE, N=1, p=view(), Tp=16, own=view(), B=2, T=16, out=FAKE, weight=None, decay=0.0, ws=FAKE,
           n=BIG):
    return lib.kvd_prefix_attn(ref(s or shape()), q, N, ref(p), Tp, ref(own), None, None, B, T, out, weight, decay, ws,
                               n, None)


def weighted(s=None, q=FAKE, N=1, kv=view(), B=2, T=16, out=FAKE, weight=FAKE, decay=1.0, ws=FAKE, n=BIG):
    return lib.kvd_weighted_attn(ref(s or shape()), q, N, ref(kv), None, None, B, T, out, weight, decay, ws, n, None)


def evict(s=None, kv=view(), B=2, T=16, keep=8, weight=FAKE, pos=None, last=None, sink=0, recent=0, ws=FAKE, n=BIG):
    return lib.kvd_evict(ref(s or shape()), ref(kv), None, B, T, keep, weight, pos, last, sink, recent, ws, n, None)


@pytest.mark.parametrize("status,kw", [
    (kvd.KVD_ERR_UNSUPPORTED, dict(s=shape(head_dim=96))),
    (kvd.KVD_ERR_SHAPE, dict(s=shape(n_q_heads=6))),
    (kvd.KVD_ERR_SHAPE, dict(N=-1)),
    (kvd.KVD_ERR_SHAPE, dict(B=-1)),
    (kvd.KVD_ERR_SHAPE, dict(B=65536)),
    (kvd.KVD_ERR_SHAPE, dict(Tp=-1)),
    (kvd.KVD_ERR_SHAPE, dict(T=-1)),
    (kvd.KVD_ERR_SHAPE, dict(Tp=0, T=0)),
    (kvd.KVD_ERR_SHAPE, dict(T=0, weight=FAKE)),
    (kvd.KVD_ERR_SHAPE, dict(decay=float("nan"))),
    (kvd.KVD_ERR_SHAPE, dict(decay=float("inf"))),
    (kvd.KVD_ERR_NULL, dict(q=None)),
    (kvd.KVD_ERR_NULL, dict(out=None)),
    (kvd.KVD_ERR_NULL, dict(p=None)),
    (kvd.KVD_ERR_NULL, dict(own=None)),
    (kvd.KVD_ERR_NULL, dict(own=view(v=0))),
    (kvd.KVD_ERR_ALIGN, dict(q=MISALIGNED)),
    (kvd.KVD_ERR_ALIGN, dict(out=MISALIGNED)),
    (kvd.KVD_ERR_ALIGN, dict(weight=ODD)),
    (kvd.KVD_ERR_ALIGN, dict(p=view(k=MISALIGNED))),
    (kvd.KVD_ERR_SHAPE, dict(p=view(t_cap=15))),
    (kvd.KVD_ERR_SHAPE, dict(own=view(t_cap=20, t_off=5))),
    (kvd.KVD_ERR_SHAPE, dict(own=view(t_off=-1))),
    (kvd.KVD_ERR_WORKSPACE, dict(ws=None)),
    (kvd.KVD_ERR_WORKSPACE, dict(n=0)),
    (kvd.KVD_ERR_ALIGN, dict(ws=FAKE + 16)),
    (kvd.KVD_ERR_SHAPE, dict(N=1 << 28, B=2)),
    (kvd.KVD_ERR_SHAPE, dict(B=65535, N=65535)),
    # 65535 x 62 x 32 rows to merge, 4 per workgroup of 256 threads: 2^32 threads and more
    (kvd.KVD_ERR_SHAPE, dict(s=shape(n_q_heads=64, n_kv_heads=32), B=65535, N=31)),
])
def test_prefix_refusals(status, kw):
    assert prefix(**kw) == status
    assert kvd.last_error()


def test_prefix_empty_calls():
    assert prefix(B=0, q=None) == kvd.KVD_OK
    assert prefix(N=0, q=None) == kvd.KVD_OK
    assert weighted(B=0, weight=None) == kvd.KVD_OK
    assert lib.kvd_prefix_attn(None, FAKE, 1, None, 0, None, None, None, 1, 1, FAKE, None, 0.0, FAKE, BIG, None) == \
        kvd.KVD_ERR_NULL


@pytest.mark.parametrize("status,kw", [
    (kvd.KVD_ERR_NULL, dict(weight=None)),
    (kvd.KVD_ERR_NULL, dict(kv=None)),
    (kvd.KVD_ERR_SHAPE, dict(T=0)),
    (kvd.KVD_ERR_SHAPE, dict(kv=view(t_cap=15))),
    (kvd.KVD_ERR_WORKSPACE, dict(n=255)),
    (kvd.KVD_ERR_UNSUPPORTED, dict(s=shape(dtype=9))),
])
def test_weighted_refusals(status, kw):
    assert weighted(**kw) == status


@pytest.mark.parametrize("status,kw", [
    (kvd.KVD_ERR_SHAPE, dict(T=0)),
    (kvd.KVD_ERR_SHAPE, dict(keep=0)),
    (kvd.KVD_ERR_SHAPE, dict(B=-2)),
    (kvd.KVD_ERR_SHAPE, dict(sink=-1)),
    (kvd.KVD_ERR_SHAPE, dict(recent=-1)),
    (kvd.KVD_ERR_SHAPE, dict(T=65)),
    (kvd.KVD_ERR_NULL, dict(kv=None)),
    (kvd.KVD_ERR_NULL, dict(weight=None)),
    (kvd.KVD_ERR_NULL, dict(sink=1)),
    (kvd.KVD_ERR_NULL, dict(recent=1)),
    (kvd.KVD_ERR_NULL, dict(recent=1, pos=FAKE)),
    (kvd.KVD_ERR_ALIGN, dict(pos=ODD)),
    (kvd.KVD_ERR_ALIGN, dict(weight=ODD)),
    (kvd.KVD_ERR_WORKSPACE, dict(ws=None)),
    (kvd.KVD_ERR_WORKSPACE, dict(n=100)),
    (kvd.KVD_ERR_ALIGN, dict(ws=FAKE + 128)),
    # a workgroup of 1024 threads per (sequence, KV head): 2^32 threads
    (kvd.KVD_ERR_SHAPE, dict(s=shape(n_q_heads=256, n_kv_heads=256), B=1 << 14)),
])
def test_evict_refusals(status, kw):
    assert evict(**kw) == status
    assert kvd.last_error()


def test_evict_with_nothing_to_do():
    assert evict(keep=16) == kvd.KVD_OK      # nothing is launched
    assert evict(keep=1000) == kvd.KVD_OK
    assert evict(B=0, weight=None) == kvd.KVD_OK


@pytest.mark.parametrize("dtype", [kvd.KVD_BF16, kvd.KVD_F32])
@pytest.mark.parametrize("heads", [(8, 4, 256), (12, 2, 128), (9, 3, 64), (16, 1, 64)])
def test_workspace_does_not_fall_as_keys_grow(dtype, heads):
    s = shape(dtype=dtype, n_q_heads=heads[0], n_kv_heads=heads[1], head_dim=heads[2])
    for B, N in ((1, 1), (3, 1), (64, 1), (1, 33), (2, 300), (7, 9)):
        for w in (0, 1):
            def size(tp, t):
                n = lib.kvd_prefix_workspace_bytes(ref(s), B, N, tp, t, w)
                assert n >= 256
                return n
            grid = [1, 2, 16, 17, 100, 128, 129, 255, 256, 257, 400, 511, 513, 1000, 2048, 2049, 5000, 16384, 40000]
            for fixed in (1, 700):
                a = [size(t, fixed) for t in grid]
                b = [size(fixed, t) for t in grid]
                assert a == sorted(a) and b == sorted(b)
            c = [size(0, t) for t in range(1, 3000, 7)]
            assert c == sorted(c)
            # too small by a byte is refused
            assert lib.kvd_prefix_attn(ref(s), FAKE, N, ref(view()), 16, ref(view()), None, None, B, 16, FAKE,
                                       FAKE if w else None, 0.0, FAKE, size(16, 16) - 1, None) == kvd.KVD_ERR_WORKSPACE


def test_workspace_of_invalid_arguments():
    s = shape()
    f = lib.kvd_prefix_workspace_bytes
    assert f(None, 1, 1, 1, 1, 0) == 0
    assert f(ref(s), 0, 1, 1, 1, 0) == 0
    assert f(ref(s), 1, 0, 1, 1, 0) == 0
    assert f(ref(s), 1, 1, 0, 0, 0) == 0
    assert f(ref(s), 1, 1, 5, 0, 1) == 0
    assert f(ref(s), 1, 1, -1, 5, 0) == 0
    assert f(ref(s), 65535, 65535, 1, 1, 0) == 0
    assert "too large" in kvd.last_error()
    assert lib.kvd_evict_workspace_bytes(ref(s), 1, 0) == 0
    assert lib.kvd_evict_workspace_bytes(ref(s), 0, 1) == 0
    sizes = [lib.kvd_evict_workspace_bytes(ref(s), 4, t) for t in range(1, 5000, 11)]
    assert sizes == sorted(sizes) and sizes[0] > 0


# ------------------------------------------------------------------ the binding

SH = kvd.Shape(512, 8, 4, 64, 1e-6, 1e4, kvd.KVD_BF16)


def _t(*dims, dt=torch.bfloat16):
    return torch.zeros(*dims, dtype=dt)


def test_binding_checks_extents_and_devices():
    q, k, pk, w = _t(2, 3, 8, 64), _t(2, 4, 20, 64), _t(4, 30, 64), _t(2, 4, 20, dt=torch.float32)
    i = torch.zeros(2, dtype=torch.int32)

    def no(match, fn, *a, **kw):
        with pytest.raises(ValueError, match=match):
            fn(SH, *a, **kw)

    f = kvd.kvd_prefix_attn
    no("q must be", f, _t(2, 64), pk, pk, 30, k, k, 20, q, w)
    no("q has shape", f, _t(2, 3, 4, 64), pk, pk, 30, k, k, 20, q, w)
    no("out has shape", f, q, pk, pk, 30, k, k, 20, _t(2, 8, 64), w)
    no("out is required", f, q, pk, pk, 30, k, k, 20, None, w)
    no("prefix_k must be", f, q, _t(1, 4, 30, 64), pk, 30, k, k, 20, q, w)
    no("prefix_v has shape", f, q, pk, _t(4, 29, 64), 30, k, k, 20, q, w)
    no("prefix: rows", f, q, pk, pk, 31, k, k, 20, q, w)
    no("prefix: rows", f, q, pk, pk, 30, k, k, 20, q, w, prefix_t_off=1)
    no("own: rows", f, q, pk, pk, 30, k, k, 21, q, w)
    no("own_k has shape", f, q, pk, pk, 30, _t(2, 3, 20, 64), k, 20, q, w)
    no("k and v are required", f, q, pk, pk, 30, None, None, 20, q, w)
    no("weight has shape", f, q, pk, pk, 30, k, k, 20, q, w, weight=_t(2, 4, 19, dt=torch.float32))
    no("weights need own rows", f, q, pk, pk, 30, None, None, 0, q, w, weight=w)
    no("own_len has shape", f, q, pk, pk, 30, k, k, 20, q, w, own_len=torch.zeros(3, dtype=torch.int32))
    no("n_new has shape", f, q, pk, pk, 30, k, k, 20, q, w, n_new=torch.zeros(1, dtype=torch.int32))
    no("on the GPU", f, q, pk, pk, 30, k, k, 20, q, w)
    no("weight is required", kvd.kvd_weighted_attn, q, k, k, 20, None, q, w)
    no("on the GPU", kvd.kvd_weighted_attn, q, k, k, 20, w, q, w)
    e = kvd.kvd_evict
    no("k and v must both", e, q[0], k, 20, 10, w, w)
    no("kv: rows", e, k, k, 21, 10, w, w)
    no("weight is required", e, k, k, 20, 10, None, w)
    no("weight has shape", e, k, k, 20, 10, w[:, :, :9], w)
    no("pos is required", e, k, k, 20, 10, w, w, sink=1)
    no("last_pos is required", e, k, k, 20, 10, w, w, pos=w.to(torch.int32), recent=1)
    no("kv_len has shape", e, k, k, 20, 10, w, w, kv_len=torch.zeros(3, dtype=torch.int32))
    no("on the GPU", e, k, k, 20, 10, w, w, kv_len=i)


# ------------------------------------------------------------------ the oracle itself

def _np(*dims, seed=0):
    return np.random.default_rng(seed).standard_normal(dims)


def test_oracle_rows_is_decode_attention_over_the_concatenation():
    B, n_q, n_kv, hd, Tp, T = 2, 6, 2, 16, 9, 5
    q, pk, pv = _np(B, 1, n_q, hd), _np(n_kv, Tp, hd, seed=1), _np(n_kv, Tp, hd, seed=2)
    k, v = _np(B, n_kv, T, hd, seed=3), _np(B, n_kv, T, hd, seed=4)
    out, size, w = O.rows_attention(q, pk, pv, k, v, [T] * B, [1] * B)
    K, V = (np.concatenate([np.broadcast_to(p, (B, *p.shape)), o], 2) for p, o in ((pk, k), (pv, v)))
    want = O.decode_attention(q[:, 0], K, V)
    assert np.abs(out[:, 0] - want).max() < 1e-13
    assert (size >= np.abs(out)).all()
    # a value of one where a row is own gives the weights back
    one = O.rows_attention(q, pk, np.zeros_like(pv), k, np.ones_like(v), [T] * B, [1] * B)[0][..., 0]
    assert np.abs(w.sum(-1) - one[:, 0].reshape(B, n_kv, -1).sum(-1)).max() < 1e-13


def test_oracle_rows_is_causal_attention_over_a_prompt():
    T, n_q, n_kv, hd = 7, 4, 2, 8
    q, k, v = _np(1, T, n_q, hd), _np(1, n_kv, T, hd, seed=1), _np(1, n_kv, T, hd, seed=2)
    out, _, w = O.rows_attention(q, None, None, k, v, [T], [T])
    for i in range(T):
        want = O.decode_attention(q[:, i], k[:, :, :i + 1], v[:, :, :i + 1])
        assert np.abs(out[:, i] - want).max() < 1e-13
    assert abs(w.sum() - T * n_q) < 1e-12


def test_oracle_rows_without_keys():
    q = _np(2, 2, 2, 8)
    out, _, w = O.rows_attention(q, None, None, _np(2, 1, 3, 8), _np(2, 1, 3, 8, seed=1), [0, 1], [2, 2])
    assert not out[0].any() and not out[1, 0].any() and out[1, 1].any()
    assert w[1, 0].tolist() == [2.0, 0.0, 0.0]


def test_oracle_evict_keeps_the_heaviest_in_fewest_moves():
    rng = np.random.default_rng(5)
    for _ in range(200):
        T, keep = int(rng.integers(1, 12)), int(rng.integers(1, 12))
        n = int(rng.integers(0, T + 1))
        k = np.arange(T, dtype=float).reshape(1, 1, T, 1)
        w = rng.integers(0, 4, (1, 1, T)).astype(float)
        pos = rng.permutation(T).reshape(1, 1, T)
        sink, recent = int(rng.integers(0, 3)), int(rng.integers(0, 3))
        k2, v2, w2, p2, l2 = O.evict(k, k * 2, w, pos, [n], [T - 1], keep, sink, recent)
        left = min(n, keep)
        assert l2[0] == left and (v2[0, 0, :left] == 2 * k2[0, 0, :left]).all()
        stay = set(k2[0, 0, :left, 0].astype(int))
        assert len(stay) == left

        def order(t):
            fixed = pos[0, 0, t] < sink or pos[0, 0, t] > T - 1 - recent
            return (not fixed, 0 if fixed else -w[0, 0, t], t)
        assert stay == set(sorted(range(n), key=order)[:left])
        assert all(k2[0, 0, t, 0] == t for t in range(left) if t in stay)  # who could stay put did
        assert (w2[0, 0, left:n] == 0).all() and (w2[0, 0, n:] == w[0, 0, n:]).all()
        assert [w[0, 0, int(t)] for t in k2[0, 0, :left, 0]] == w2[0, 0, :left].tolist()
        assert [pos[0, 0, int(t)] for t in k2[0, 0, :left, 0]] == p2[0, 0, :left].tolist()
