"""Shared helpers of the tests of kvd_prefix_attn, kvd_weighted_attn and kvd_evict: seeded inputs, the calls, and
element-wise error bounds against the 64-bit oracle."""
from __future__ import annotations

import numpy as np
import torch

import oracle as O
from paper_2603_19664_amd import inputs
from paper_2603_19664_amd import kvd

DT = {"bf16": (kvd.KVD_BF16, torch.bfloat16), "f32": (kvd.KVD_F32, torch.float32)}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def shape(dtype, n_q, n_kv, hd):
    return kvd.Shape(512, n_q, n_kv, hd, 1e-6, 1e4, DT[dtype][0])


def make(dtype, n_q, n_kv, hd, B, N, T_prefix, T, seed=0, p_cap=None, t_cap=None, q_std=1.0):
    """q, prefix and own K/V in stores of p_cap / t_cap rows, weights; every value seeded."""
    dt = DT[dtype][1]

    def normal(shp, std, i):
        return inputs.normal(shp, std, "cuda", seed, 95, i).to(dt)

    p_cap, t_cap = p_cap or max(T_prefix, 1), t_cap or max(T, 1)
    return dict(q=normal((B, N, n_q, hd), q_std, 0), pk=normal((n_kv, p_cap, hd), 1.0, 1),
                pv=normal((n_kv, p_cap, hd), 1.0, 2), k=normal((B, n_kv, t_cap, hd), 1.0, 3),
                v=normal((B, n_kv, t_cap, hd), 1.0, 4),
                weight=torch.abs(inputs.normal((B, n_kv, t_cap), 1.0, "cuda", seed, 95, 5)))


def i32(x):
    return None if x is None else torch.as_tensor(x, dtype=torch.int32, device="cuda")


def bound(x, s, T_prefix, T, p_off, t_off, lens, news, tile):
    """(out, its element-wise bound, weights, their bound) of a call on inputs x.

    With u = 2^-24: a score of hd products added in fp32 is off by at most hd u sum|q k| / sqrt(hd) (S below, with 4
    more for the scaling and the exponential's argument), so a softmax weight by a factor of 1 +- 2 (S + 4 u |s|) and
    its exponential's last place; sums over n keys add n u.  The output is a weighted mean of V, so those factors
    act on sum p |V|; then come one rounding to the output type and, where rows are taken in tiles of bf16 weights,
    one rounding of every weight."""
    q = inputs.to_f64(x["q"])
    pk = pv = k = v = None
    if T_prefix > 0:
        pk, pv = (inputs.to_f64(x[n][:, p_off:p_off + T_prefix]) for n in ("pk", "pv"))
    if T > 0:
        k, v = (inputs.to_f64(x[n][:, :, t_off:t_off + T]) for n in ("k", "v"))
    out, size, w = O.rows_attention(q, pk, pv, k, v, lens, news)
    u, hd = 2.0 ** -24, q.shape[-1]
    top = np.linalg.norm(q, axis=-1).max() * max(
        [np.linalg.norm(a, axis=-1).max() for a in (pk, None if k is None else _seen(k, lens)) if a is not None and a.size] + [0.0])
    S = (hd + 4) * u * top / np.sqrt(hd)      # sum |q k| <= |q| |k|
    c = 2 * S + (T_prefix + T + 64) * u + 8 * u
    half = HALF_STEP[x["q"].dtype]
    tol = half * np.abs(out) + (c + (half if tile else 0.0)) * size * (1 + half) + 1e-30
    return out, tol, w, c * w + 1e-30


def _seen(k, lens):
    return np.concatenate([k[b, :, :max(int(n), 0)].reshape(-1, k.shape[-1]) for b, n in enumerate(lens)])


def call(s, x, T_prefix, T, lens=None, news=None, weight=None, decay=0.0, p_off=0, t_off=0, out=None, ws=None):
    B, N = x["q"].shape[:2]
    out = torch.full_like(x["q"], 7.0) if out is None else out
    if ws is None:
        n = kvd.kvd_prefix_workspace_bytes(s, B, N, T_prefix, T, weight is not None)
        ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")  # NaN everywhere: nothing may rely on it
    kvd.kvd_prefix_attn(s, x["q"], x["pk"] if T_prefix else None, x["pv"] if T_prefix else None, T_prefix,
                        x["k"] if T else None, x["v"] if T else None, T, out, ws, own_len=i32(lens), n_new=i32(news),
                        weight=weight, decay=decay, prefix_t_off=p_off, own_t_off=t_off)
    return out


def is_tile(dtype, N, g, B, T_prefix, T):
    """Whether some rows of the call are taken in tiles (bf16, more than 16 rows to a key range)."""
    return dtype == "bf16" and (N * g > 16 or (T_prefix > 0 and B * N * g > 16))


def within(name, got, ref, tol):
    got = inputs.to_f64(got)
    bad = ~(np.abs(got - ref) <= tol)
    worst = float(np.max(np.abs(got - ref) / tol)) if got.size else 0.0
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.size} outside the bound, worst {worst:.2f} of it"
    return worst
