"""One workspace for calls of several lengths, as a decode loop keeps it: sized for the longest, each shorter call lays
it out for itself and leaves what lies behind its own size alone."""
import pytest
import torch

from paper_2603_19664_amd import kvd

from gpu_cases import note
from rows_cases import call, i32, make, shape
from test_gpu_evict import cache

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    note(f"[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


# (T_prefix, T): one slot, joint, side by side, many slots; the longest last
LENGTHS = [(1, 1), (100, 90), (0, 200), (257, 0), (300, 257), (1500, 40), (7, 2000), (2500, 2200)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_kv,hd", [(6, 2, 64), (8, 4, 256)])
@pytest.mark.parametrize("B,N", [(1, 1), (9, 1), (3, 4), (2, 40), (1, 150)])
@pytest.mark.parametrize("weights", [False, True])
def test_calls_of_other_lengths_share_it(dtype, n_q, n_kv, hd, B, N, weights):
    s = shape(dtype, n_q, n_kv, hd)
    Tp, T = LENGTHS[-1]
    x = make(dtype, n_q, n_kv, hd, B, N, Tp, T, 51)
    n = kvd.kvd_prefix_workspace_bytes(s, B, N, Tp, T, weights)
    shared = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")
    wants = {}
    for tp, t in LENGTHS + LENGTHS[::-1]:
        w = weights and t > 0
        if (tp, t) not in wants:
            size = kvd.kvd_prefix_workspace_bytes(s, B, N, tp, t, w)
            assert size <= n
            own = torch.full((size + 4096,), 0xff, dtype=torch.uint8, device="cuda")
            weight = x["weight"].clone() if w else None
            wants[tp, t] = call(s, x, tp, t, None, None, weight, 0.5, ws=own[:size]), weight
            assert (own[size:] == 0xff).all(), "bytes behind the workspace"
        weight = x["weight"].clone() if w else None
        out = call(s, x, tp, t, None, None, weight, 0.5, ws=shared)
        assert torch.equal(out, wants[tp, t][0]), (tp, t)
        assert weight is None or torch.equal(weight, wants[tp, t][1]), (tp, t)


@pytest.mark.parametrize("T,keep", [(3, 1), (100, 99), (1000, 400), (9000, 100), (33000, 20000)])
def test_eviction_keeps_to_its_workspace(T, keep):
    B, n_kv, hd = 3, 2, 64
    s = shape("bf16", 4, n_kv, hd)
    k, v, w, pos = cache("bf16", B, n_kv, hd, T, T)
    size = kvd.kvd_evict_workspace_bytes(s, B, T)
    longest = kvd.kvd_evict_workspace_bytes(s, B, 40000)
    shared = torch.full((longest,), 0xff, dtype=torch.uint8, device="cuda")
    own = torch.full((size + 4096,), 0xff, dtype=torch.uint8, device="cuda")
    got = []
    for ws in (own[:size], shared):
        a = [t.clone() for t in (k, v, w, pos)]
        lens = i32([T, T - 1, T // 2])
        kvd.kvd_evict(s, a[0], a[1], T, keep, a[2], ws, pos=a[3], last_pos=i32([T] * B), kv_len=lens, sink=1, recent=2)
        got.append((*a, lens))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert (own[size:] == 0xff).all(), "bytes behind the workspace"
