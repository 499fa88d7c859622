"""kvd_sink_attn and kvd_mx_attn over finite values near the largest that the type holds: a weighted mean of them is
finite, whatever the sums on the way to it.  Element by element against the 64-bit oracle, with sink_cases.bound.

The sums: without care a running maximum that lags by 8 gives weights of up to 2^8, and n weights of 1 add up to n.
Values v with n |v| >= 2^128 overflow then."""
import math

import pytest
import torch

from paper_2603_19664_amd import inputs

from gpu_cases import note
from sink_cases import bound, cache, call, held, shape, tokens, within

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    note(f"[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


HEADS = [(64, 9, 3), (128, 12, 2), (256, 8, 4)]
TOP = 3.0e38          # below the largest bf16, 3.39e38


def rising(x, step):
    """Keys whose scores rise by `step` (in powers of two) from token to token, for all queries: q = e_0, k = rising."""
    hd, T = x["k"].shape[-1], x["k"].shape[2]
    x["q"].zero_()
    x["q"][..., 0] = 1.0
    x["k"].mul_(0.01)
    t = torch.arange(T, device="cuda", dtype=torch.float32)
    x["k"][..., 0] = (t * step * math.log(2.0) * math.sqrt(hd)).to(x["k"].dtype)


def checked(dtype, n_q, n_kv, hd, x, T, window, sink, mx):
    B, N = x["q"].shape[:2]
    s = shape(dtype, n_q, n_kv, hd)
    out = call(s, x["q"], cache(x, [T] * B, T, T, sink, mx), T, window, sink)
    k, v = (held(x[n]) if mx else inputs.to_f64(x[n]) for n in ("k", "v"))
    ref, tol = bound(x["q"], k, v, [T] * B, [N] * B, window, sink)
    assert torch.isfinite(out).all()
    within("out", out, ref, tol)
    return out


ALL = pytest.mark.parametrize("dtype,mx", [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)])
# one launch, several slots, tiles of one slot and of several
SIZES = pytest.mark.parametrize("N,T,window,sink", [(1, 200, 200, 0), (1, 3000, 3000, 0), (1, 2500, 1111, 4), (4, 150, 60, 3),
                                                    (70, 190, 190, 0), (90, 1300, 1300, 0), (150, 1300, 700, 4)])


@ALL
@SIZES
@pytest.mark.parametrize("hd,n_q,n_kv", HEADS)
def test_the_mean_of_the_largest_values(dtype, mx, hd, n_q, n_kv, N, T, window, sink):
    x = tokens(dtype, n_q, n_kv, hd, 1, N, T, 41)
    x["v"] = (x["v"].float().sign() * TOP * (0.5 + 0.5 * x["v"].float().abs().clamp(max=1.0))).to(x["v"].dtype)
    x["v"][..., 0] = TOP * 0.99      # one sign: the sum is n times a value
    checked(dtype, n_q, n_kv, hd, x, T, window, sink, mx)


@ALL
@SIZES
@pytest.mark.parametrize("hd,n_q,n_kv", HEADS)
def test_scores_that_rise(dtype, mx, hd, n_q, n_kv, N, T, window, sink):
    # the maximum moves on in every block, and most of it lies below the threshold at which weights are scaled anew
    x = tokens(dtype, n_q, n_kv, hd, 1, N, T, 42)
    rising(x, 0.05)
    x["v"] = (x["v"].float() * 2e37).clamp(-TOP, TOP).to(x["v"].dtype)
    x["v"][..., 0] = 1e37
    checked(dtype, n_q, n_kv, hd, x, T, window, sink, mx)


@ALL
@pytest.mark.parametrize("N", [1, 70])
@pytest.mark.parametrize("at", [0, 700, 1499])
def test_large_values_in_one_place_alone(dtype, mx, N, at):
    # states of ordinary sums beside ones that have been scaled, and columns of ordinary values beside large ones
    hd, T = 128, 1500
    x = tokens(dtype, 6, 2, hd, 2, N, T, 43)
    x["v"][:, :, at:at + 40, :64] = TOP
    checked(dtype, 6, 2, hd, x, T, T, 0, mx)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 70])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_beside_infinities_seen_and_not_seen(dtype, N, bad):
    hd, T, window = 64, 900, 300
    s = shape(dtype, 6, 2, hd)
    x = tokens(dtype, 6, 2, hd, 1, N, T, 44)
    x["v"] = (x["v"].float().sign() * TOP).to(x["v"].dtype)
    a = checked(dtype, 6, 2, hd, x, T, window, 0, False)
    x["v"][:, :, T - N - window + 1, :32] = bad      # the oldest token of the first new token's window
    d = call(s, x["q"], (x["k"], x["v"]), T, window, 0)
    assert torch.isnan(d[:, 0, :, :32]).all() if bad != bad else (d[:, 0, :, :32] == bad).all()
    assert torch.isfinite(d[:, 0, :, 32:]).all() and torch.isfinite(d[:, 1:]).all()
    assert torch.equal(a[:, 1:], d[:, 1:])
