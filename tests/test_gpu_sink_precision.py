"""kvd_sink_attn and kvd_mx_attn in fp32: the 2-norm error against the 64-bit oracle, held to what fp32 arithmetic gives
(sink_precision.LIMIT; two bf16 parts of a query or a weight instead of three are above it)."""
import pytest
import torch

import oracle as O
from paper_2603_19664_amd import inputs

from gpu_cases import note
from sink_cases import cache, call, held, shape, tokens
from sink_precision import LIMIT, error

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    note(f"[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("mx", [False, True], ids=["plain", "mx"])
@pytest.mark.parametrize("hd,n_q,n_kv", [(64, 9, 3), (128, 12, 2), (256, 8, 4)])
@pytest.mark.parametrize("N,T,window,sink", [
    (1, 200, 200, 0), (1, 500, 500, 0), (1, 3000, 3000, 0), (1, 2600, 1100, 4), (5, 240, 240, 0), (5, 2000, 2000, 0),
    (60, 200, 200, 0), (90, 1300, 1300, 0), (90, 1300, 600, 4)])
def test_the_error_is_that_of_fp32(mx, hd, n_q, n_kv, N, T, window, sink):
    x = tokens("f32", n_q, n_kv, hd, 2, N, T, 51)
    out = call(shape("f32", n_q, n_kv, hd), x["q"], cache(x, [T] * 2, T, T, sink, mx), T, window, sink)
    k, v = (held(x[n]) if mx else inputs.to_f64(x[n]) for n in ("k", "v"))
    ref, _ = O.sink_attention(inputs.to_f64(x["q"]), k, v, [T] * 2, [N] * 2, window, sink)
    e = error(inputs.to_f64(out), ref)
    note(f"error {e:.2e}")
    assert e < LIMIT
