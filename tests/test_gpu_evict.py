"""kvd_evict against the oracle, bit for bit: which rows stay, where they lie, what is left as it was."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2603_19664_amd import inputs
from paper_2603_19664_amd import kvd

from gpu_cases import note
from rows_cases import DT, i32, shape

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    note(f"[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


def cache(dtype, B, n_kv, hd, t_cap, seed):
    dt = DT[dtype][1]
    k, v = (inputs.normal((B, n_kv, t_cap, hd), 1.0, "cuda", seed, 97, i).to(dt) for i in range(2))
    w = torch.exp(2.0 * inputs.normal((B, n_kv, t_cap), 1.0, "cuda", seed, 97, 2))
    order = torch.rand((B, n_kv, t_cap), generator=torch.Generator().manual_seed(seed)).argsort(-1)
    return k, v, w, order.to(torch.int32).cuda()


def evict(dtype, k, v, w, pos, T, keep, lens=None, last=None, sink=0, recent=0, t_off=0, g=2):
    """One call on copies; checks against the oracle and returns the results."""
    B, n_kv, _, hd = k.shape
    s = shape(dtype, g * n_kv, n_kv, hd)
    got = [t.clone() for t in (k, v, w)] + [None if pos is None else pos.clone()]
    n = i32(lens)
    ws = torch.full((kvd.kvd_evict_workspace_bytes(s, B, T),), 0xff, dtype=torch.uint8, device="cuda")
    kvd.kvd_evict(s, got[0], got[1], T, keep, got[2], ws, pos=got[3], last_pos=i32(last), kv_len=n, sink=sink,
                  recent=recent, t_off=t_off)
    rows = slice(t_off, t_off + T)
    L = [T] * B if lens is None else [min(max(x, 0), T) for x in lens]

    def host(t):
        return None if t is None else (t.float() if t.dtype == torch.bfloat16 else t)[:, :, rows].cpu().numpy()

    want = O.evict(host(k), host(v), host(w), host(pos), L, last, keep, sink, recent)
    for name, a, c, before in zip(("k", "v", "weight", "pos"), got, want, (k, v, w, pos)):
        if a is None:
            continue
        assert np.array_equal(host(a), c, equal_nan=True), name
        outside = torch.ones(a.shape[2], dtype=torch.bool, device="cuda")
        outside[rows] = False
        same = a[:, :, outside], before[:, :, outside]
        assert torch.equal(*(t.view(torch.int16) if t.dtype == torch.bfloat16 else t.view(torch.int32) for t in same))
    if lens is not None:
        assert n.tolist() == [int(x) for x in want[4]]
    return got


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 64), ("f32", 256)])
@pytest.mark.parametrize("T,keep", [(2, 1), (5, 4), (65, 64), (100, 99), (300, 17), (1000, 1), (1025, 1024),
                                    (2049, 2048), (3000, 1500), (4100, 2999)])
def test_sizes(dtype, hd, T, keep):
    k, v, w, pos = cache(dtype, 2, 3, hd, T + 5, T + hd)
    evict(dtype, k, v, w, pos, T, keep, t_off=2)
    evict(dtype, k, v, w, None, T, keep, t_off=5)


@pytest.mark.parametrize("sink,recent", [(0, 5), (4, 0), (4, 60), (1, 1), (0, 0)])
@pytest.mark.parametrize("keep", [64, 65, 199, 200])
def test_protected_rows(sink, recent, keep):
    k, v, w, pos = cache("bf16", 3, 2, 64, 200, keep + sink)
    evict("bf16", k, v, w, pos, 200, keep, None, [199, 190, 5], sink, recent)
    evict("bf16", k, v, w, pos, 200, keep, [200, keep, keep + 1], [199, 199, 2 ** 31 - 1], sink, recent)


@pytest.mark.parametrize("keep", [1, 30, 99])
def test_more_protected_rows_than_stay(keep):
    # every row protected: the lowest slots stay
    k, v, w, pos = cache("bf16", 2, 2, 64, 100, 3)
    out = evict("bf16", k, v, w, pos, 100, keep, None, [0, 0], 1000, 0)
    assert torch.equal(out[0][:, :, :keep], k[:, :, :keep])


@pytest.mark.parametrize("keep", [1, 7, 40, 98, 99])
def test_equal_and_odd_weights(keep):
    # ties stay by slot; NaN goes first, -0 equals +0, infinities keep their places
    k, v, w, pos = cache("bf16", 4, 2, 64, 100, 5)
    w[0] = 1.0
    w[1] = torch.randint(0, 3, (2, 100), generator=torch.Generator().manual_seed(1)).float().cuda()
    w[2] = torch.where(torch.arange(100, device="cuda") % 2 == 0, 0.0, -0.0)
    w[3, :, ::3] = float("nan")
    w[3, :, 1::9] = float("inf")
    w[3, :, 2::9] = float("-inf")
    w[3, 1, 4::9] = -3.0
    w[3, 1, 7::9] = 1e-42
    evict("bf16", k, v, w, None, 100, keep)
    evict("bf16", k, v, w, pos, 100, keep, None, None, 2, 0)


def test_lengths_of_their_own():
    lens = [0, 1, 49, 50, 51, 100, 77, 500, -3]
    k, v, w, pos = cache("f32", len(lens), 3, 64, 100, 9)
    evict("f32", k, v, w, pos, 100, 50, lens, [x for x in range(len(lens))], 1, 4)
    evict("f32", k, v, w, pos, 100, 99, lens, [99] * len(lens), 1, 4)
    evict("f32", k, v, w, None, 100, 1, lens)


@pytest.mark.parametrize("T,keep", [(70001, 70000), (70001, 33), (40000, 39000)])
def test_long_caches(T, keep):
    k, v, w, pos = cache("bf16", 1, 1, 64, T, 11)
    evict("bf16", k, v, w, pos, T, keep, None, [T - 1], 4, 100)


def test_many_sequences():
    k, v, w, pos = cache("bf16", 300, 4, 64, 40, 13)
    evict("bf16", k, v, w, pos, 40, 31, [i % 41 for i in range(300)], [39] * 300, 0, 3)


def test_again_changes_nothing():
    k, v, w, pos = cache("bf16", 2, 2, 128, 300, 15)
    a = evict("bf16", k, v, w, pos, 300, 200, [300, 250], [299, 299], 2, 20)
    b = evict("bf16", a[0], a[1], a[2], a[3], 300, 200, [200, 200], [299, 299], 2, 20)
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])


def test_captured_and_replayed():
    B, n_kv, hd, T, keep = 2, 4, 64, 500, 499
    s = shape("bf16", 8, n_kv, hd)
    k, v, w, pos = cache("bf16", B, n_kv, hd, T, 17)
    lens, last = i32([T, T]), i32([T, T])
    for keep in (499, 100):
        mine = [t.clone() for t in (k, v, w, pos)]
        ws = torch.empty(kvd.kvd_evict_workspace_bytes(s, B, T), dtype=torch.uint8, device="cuda")
        st = torch.cuda.Stream()
        lens.fill_(0)

        def go():
            kvd.kvd_evict(s, mine[0], mine[1], T, keep, mine[2], ws, pos=mine[3], last_pos=last, kv_len=lens, sink=1,
                          recent=9)
        with torch.cuda.stream(st):
            go()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            go()
        for i in range(4):
            w2 = torch.exp(inputs.normal(w.shape, 1.0, "cuda", i, 98))
            want = evict("bf16", k, v, w2, pos, T, keep, [T, T - i], [T, T], 1, 9)
            for a, c in zip(mine, (k, v, w2, pos)):
                a.copy_(c)
            lens.copy_(torch.tensor([T, T - i], dtype=torch.int32))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, c) for a, c in zip(mine, want))
            assert lens.tolist() == [keep, min(keep, T - i)]


def test_arrays_at_4_byte_alignment():
    k, v, w, pos = cache("bf16", 2, 3, 64, 77, 21)
    flat = torch.empty(2 * w.numel() + 9, dtype=torch.int32, device="cuda")
    for off in (1, 2, 3):
        w2 = flat[off:off + w.numel()].view(torch.float32).view(w.shape)
        p2 = flat[off + w.numel():off + 2 * w.numel()].view(pos.shape)
        for T, keep in ((77, 76), (70, 33)):
            w2.copy_(w)
            p2.copy_(pos)
            s = shape("bf16", 6, 3, 64)
            mine = [k.clone(), v.clone()]
            ws = torch.empty(kvd.kvd_evict_workspace_bytes(s, 2, T), dtype=torch.uint8, device="cuda")
            kvd.kvd_evict(s, *mine, T, keep, w2, ws, pos=p2, last_pos=i32([76, 76]), sink=2, recent=7)
            want = evict("bf16", k, v, w, pos, T, keep, None, [76, 76], 2, 7)
            assert all(torch.equal(a, b) for a, b in zip((*mine, w2, p2), want))
