"""kvd_evict on both sides of the lengths at which its selection changes (8192, 16384 and 32768 rows), bit for bit."""
import pytest
import torch

from gpu_cases import note
from test_gpu_evict import cache, evict

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    note(f"[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("T", [4096, 4097, 8191, 8192, 8193, 16384, 16385, 17408, 17409, 32767, 32768, 32769])
def test_sides_of_the_limits(T):
    k, v, w, pos = cache("bf16", 3, 1, 64, T + 3, T)
    lens = [T, T // 2 + 1, 1500]
    for keep in (T - 2, T // 2, 1024, 5):
        evict("bf16", k, v, w, pos, T, keep, lens, [T - 1] * 3, 4, 64 if keep > 64 else 0, t_off=2)


@pytest.mark.parametrize("T", [8192, 8193, 16384, 16385, 32768, 32769])
def test_ties_and_odd_weights_of_long_caches(T):
    # few different weights, so that the last rank kept is shared by thousands of rows; NaN and infinities among them
    k, v, w, pos = cache("f32", 2, 2, 64, T, T + 1)
    g = torch.Generator().manual_seed(T)
    w[:, 0] = torch.randint(0, 4, (2, T), generator=g).float().cuda()
    w[0, 1, ::3] = float("nan")
    w[0, 1, 1::5] = float("inf")
    w[1, 1] = 0.0
    for keep in (T - 2, T // 3, 1):
        evict("f32", k, v, w, None, T, keep, [T, T - 700])
        evict("f32", k, v, w, pos, T, keep, None, [T - 1, 9], 1, 7)
