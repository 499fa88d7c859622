"""Softmax weights of row tiles (bf16, more than 16 rows to a key range) in the value product: as precise as
those of few rows, whoever shares a token's batch."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2603_19664_amd import inputs

from gpu_cases import note
from rows_cases import bound, call, make, shape, within

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    note(f"[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


def exact_weights_bound(x, s, T_prefix, T):
    """(out, its bound) where no weight is rounded to one bf16: bound() without that rounding, and 2^-17 of every
    weight for its two bf16 parts (p = hi + lo + rest: |p - hi| <= 2^-8 p, and |lo| < 2^-8 2^e of a p in [2^e, 2^(e + 1))
    has steps of 2^-16 2^e at most, half of one is lost)."""
    B, N = x["q"].shape[:2]
    lens, news = [T] * B, [N] * B
    ref, tol, _, _ = bound(x, s, T_prefix, T, 0, 0, lens, news, False)
    f = {n: inputs.to_f64(t) for n, t in x.items() if n != "weight"}
    _, size, _ = O.rows_attention(f["q"], f["pk"] if T_prefix else None, f["pv"] if T_prefix else None,
                                  f["k"] if T else None, f["v"] if T else None, lens, news)
    return ref, tol + 2.0 ** -17 * size * (1 + 2.0 ** -8)


@pytest.mark.parametrize("hd,n_q,n_kv", [(64, 9, 3), (128, 12, 2), (256, 8, 4)])
@pytest.mark.parametrize("B,N,T_prefix,T", [(20, 1, 300, 50), (1, 90, 0, 90), (2, 75, 300, 111), (3, 32, 0, 700),
                                            (2, 130, 64, 130), (1, 17, 45, 0)])
def test_tiles_keep_their_weights(hd, n_q, n_kv, B, N, T_prefix, T):
    s = shape("bf16", n_q, n_kv, hd)
    x = make("bf16", n_q, n_kv, hd, B, N, T_prefix, T, 21)
    ref, tol = exact_weights_bound(x, s, T_prefix, T)
    within("out", call(s, x, T_prefix, T), ref, tol)


@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("p", [64.25, 96.25, 127.75, 128.5, 200.5])
def test_one_key_behind_the_first_maximum(hd, p):
    # a key of the second tile has p times the first maximum's weight, which is not moved for it; p lies midway between
    # two bf16
    N, T = 64, 200
    s = shape("bf16", 2, 2, hd)
    x = make("bf16", 2, 2, hd, 1, N, T, 0, 23)
    x["q"].fill_(1.0)
    x["pk"].fill_(-40.0)                    # score -40 sqrt(hd): no weight
    x["pk"][:, 3] = 0.0
    want = np.log(p) * hd ** 0.5            # sum of the key's elements: one of them takes what bf16 leaves of the mean
    x["pk"][:, 150] = want / hd
    x["pk"][:, 150, 0] = want - float(x["pk"][0, 150, 1]) * (hd - 1)
    ref, tol = exact_weights_bound(x, s, T, 0)
    within("out", call(s, x, T, 0), ref, tol)


def test_a_token_does_not_depend_on_its_batch():
    # the same sequence alone (few rows) and among 19 others (tiles over the prefix): one rounding apart
    s = shape("bf16", 8, 4, 128)
    x = make("bf16", 8, 4, 128, 20, 1, 500, 60, 25)
    one = {n: (t if n in ("pk", "pv") else t[:1].contiguous()) for n, t in x.items()}
    ref, tol = exact_weights_bound(one, s, 500, 60)
    within("alone", call(s, one, 500, 60), ref, tol)
    within("in a batch", call(s, x, 500, 60)[:1], ref, tol)
