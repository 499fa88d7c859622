"""How exact fp32 attention over a 4-bit cache is: a limit on the 2-norm error, and a model of the kernels' arithmetic in
which parts of the queries or the softmax weights can be left out."""
import numpy as np

U = 2.0 ** -24
# Relative 2-norm error of an output of N(0, 1) queries, keys and values.  Every step's error is independent of the
# others, so they add as squares.  A score's hd products (unit variance) added one by one: the sum after j of them is
# rounded by u sqrt(j / 3), together u hd / sqrt(6), over sqrt(hd): 6.5 u at head_dim 256.  The exponential's argument,
# up to some 10 below the maximum: 4 u, times ln 2; its last place: 1.2 u.  Sums over 3000 keys, 32 at a time: 4 u.
# 8.5 u, and nearly as much again for the order of sums that a kernel takes.
LIMIT = 16 * U
# What a part less costs: queries cut to 16 bits lose 2^-16 of an element at most, 2^-17 in the mean, all of it in one
# direction: 2^-17 / sqrt(3) and more in the weights, 74 u; weights rounded to 16 bits lose up to 2^-17 in a binade's
# lower end, uniformly: 2^-18 / sqrt(3) = 37 u, less where a weight's second part is short: above 20 u.


def error(out, ref):
    out, ref = np.asarray(out, dtype=np.float64), np.asarray(ref, dtype=np.float64)
    return np.linalg.norm(out - ref) / np.linalg.norm(ref)


def _cut(x):
    return (x.view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)


def _round(x):
    b = x.view(np.uint32)
    return ((b + ((b >> 16) & 1) + 0x7fff) & np.uint32(0xffff0000)).view(np.float32)


def parts(x, n, to_bf16):
    x, made = np.asarray(x, dtype=np.float32), []
    for _ in range(n):
        made.append(to_bf16(x))
        x = x - made[-1]
    return made


def modelled(q, k, v, query_parts, weight_parts):
    """q [M, hd] fp32 over k, v [T, hd] (numbers that bf16 holds): products of bf16 parts, sums of 32 kept in fp32."""
    f, hd, T = np.float32, q.shape[1], len(k)
    s = np.zeros((len(q), T), f)
    for c in range(0, hd, 32):
        for p in parts(q[:, c:c + 32], query_parts, _cut):
            s = (s + p.astype(np.float64) @ k[:, c:c + 32].T).astype(f)
    scale = f(np.log2(np.e) / np.sqrt(hd))
    w = np.exp2((s.astype(np.float64) * scale - s.max(1, keepdims=True) * scale).astype(f).astype(np.float64)).astype(f)
    total, o = np.zeros((len(q), 1), f), np.zeros((len(q), hd), f)
    for t in range(0, T, 32):
        total = total + w[:, t:t + 32].sum(1, keepdims=True)
        for p in parts(w[:, t:t + 32], weight_parts, _round):
            o = (o + p.astype(np.float64) @ v[t:t + 32]).astype(f)
    return o / total
