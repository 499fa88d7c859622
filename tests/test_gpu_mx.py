"""kvd_mx_store and kvd_mx_load: bit for bit what the format says."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2603_19664_amd import inputs
from paper_2603_19664_amd import kvd

from gpu_cases import note
from sink_cases import DT, call, held, i32, shape

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    note(f"[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


def same(got, want):
    return np.array_equal(inputs.to_f64(got), want, equal_nan=True)


def filled(s, B, cap, byte=0x5a):
    return kvd.MxCache(*(t.fill_(byte) for t in kvd.mx_cache(s, B, cap)[:4]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,n_kv", [(64, 3), (128, 2), (256, 4)])
@pytest.mark.parametrize("B,N,T,sink,slots,pad", [
    (1, 1, 1, 0, 1, 0), (2, 1, 40, 4, 20, 2), (3, 17, 17, 0, 30, 1), (2, 33, 500, 3, 40, 0), (1, 300, 1000, 0, 300, 5),
    (4, 5, 9, 7, 9, 0), (2, 8, 10, 9, 17, 0)])
def test_rows_in_order_and_in_rings(dtype, hd, n_kv, B, N, T, sink, slots, pad):
    s = shape(dtype, n_kv, n_kv, hd)
    k, v = (inputs.normal((B, n_kv, N + 2 * pad, hd), 2.0, "cuda", 4, i).to(DT[dtype][1]) for i in range(2))
    c = filled(s, B, slots + pad)._replace(t_off=pad)
    kvd.kvd_mx_store(s, k, v, N, c, T, sink=sink, t_off=pad)
    rows = pad + O.sink_rows(T, slots, sink)[T - N:]
    for plain, codes, scales in ((k, c.k, c.k_scale), (v, c.v, c.v_scale)):
        wc, ws = O.mx_round(inputs.to_f64(plain[:, :, pad:pad + N]))
        assert np.array_equal(codes[:, :, rows].cpu().numpy(), wc)
        assert np.array_equal(scales[:, :, rows].cpu().numpy(), ws)
        other = torch.ones(codes.shape[2], dtype=torch.bool, device="cuda")
        other[torch.as_tensor(rows, device="cuda")] = False
        assert (codes[:, :, other] == 0x5a).all() and (scales[:, :, other] == 0x5a).all()
    back = [torch.full_like(k, 7.0) for _ in range(2)]
    kvd.kvd_mx_load(s, c, T, N, *back, sink=sink, t_off=pad)
    for plain, b in zip((k, v), back):
        assert same(b[:, :, pad:pad + N], held(plain[:, :, pad:pad + N]))
        assert (b[:, :, :pad] == 7.0).all() and (b[:, :, pad + N:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_of_their_own(dtype):
    lens, news, T, N, sink, cap = [0, 1, 5, 60, 77, 999, -4, 3], [1, 1, 2, 9, 0, 99, 3, 7], 77, 9, 4, 40
    B, n_kv, hd = len(lens), 2, 64
    s = shape(dtype, 2, n_kv, hd)
    k, v = (inputs.normal((B, n_kv, N, hd), 1.0, "cuda", 5, i).to(DT[dtype][1]) for i in range(2))
    c = filled(s, B, cap)
    kvd.kvd_mx_store(s, k, v, N, c, T, sink=sink, kv_len=i32(lens), n_new=i32(news))
    back = [torch.full_like(k, 7.0) for _ in range(2)]
    kvd.kvd_mx_load(s, c, T, N, *back, sink=sink, kv_len=i32(lens), n_new=i32(news))
    rows = O.sink_rows(T, cap, sink)
    hk, hv = held(k), held(v)
    for b in range(B):
        n, m = min(max(lens[b], 0), T), min(max(news[b], 0), N)
        touched = torch.zeros(cap, dtype=torch.bool, device="cuda")
        for i in range(N):
            t = n - m + i
            if i < m and t >= 0:
                touched[int(rows[t])] = True
                assert same(back[0][b, :, i], hk[b, :, i]) and same(back[1][b, :, i], hv[b, :, i])
            else:
                assert (back[0][b, :, i] == 7.0).all() and (back[1][b, :, i] == 7.0).all()
        assert (c.k[b][:, ~touched] == 0x5a).all() and (c.v_scale[b][:, ~touched] == 0x5a).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_size_of_number(dtype):
    # zeros of both signs, numbers below the smallest scale and above the largest, exact ties, groups of one large one
    dt = DT[dtype][1]
    s = shape(dtype, 1, 1, 64)
    rng = np.random.default_rng(1)
    rows = [np.zeros(64), -np.zeros(64), np.full(64, 3.3e38), np.full(64, -2.0 ** 127), np.full(64, 1e-38)]
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 6.5, 7.0, -0.25, -0.75, -1.25, -1.75, -2.5, -5.0])
    for e in range(-126, 126):
        r = np.resize(ties, 64) * 2.0 ** e
        r[32:] = rng.standard_normal(32) * 2.0 ** e
        rows.append(r)
    for e in range(-100, 120, 7):
        rows.append(np.where(np.arange(64) % 32 == 5, 2.0 ** e, 2.0 ** e * rng.standard_normal(64) * 0.02))
    x = torch.tensor(np.asarray(rows)).to(torch.float32).to(dt).cuda().view(1, 1, -1, 64)
    N = x.shape[2]
    c, back = kvd.mx_cache(s, 1, N), [torch.empty_like(x) for _ in range(2)]
    kvd.kvd_mx_store(s, x, -x, N, c, N)
    kvd.kvd_mx_load(s, c, N, N, *back)
    for plain, codes, scales, b in ((x, c.k, c.k_scale, back[0]), (-x, c.v, c.v_scale, back[1])):
        wc, ws = O.mx_round(inputs.to_f64(plain))
        assert np.array_equal(codes.cpu().numpy(), wc) and np.array_equal(scales.cpu().numpy(), ws)
        assert same(b, O.mx_values(wc, ws))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_group_with_an_infinity_or_nan_is_nan(dtype, bad):
    s = shape(dtype, 2, 2, 128)
    x = inputs.normal((1, 2, 8, 128), 1.0, "cuda", 3, 3).to(DT[dtype][1])
    want = held(x)
    for r in range(8):
        x[0, 0, r, 37 + 3 * r] = bad
        want[0, 0, r, 32:64] = np.nan
    c, back = kvd.mx_cache(s, 1, 8), [torch.empty_like(x) for _ in range(2)]
    kvd.kvd_mx_store(s, x, x, 8, c, 8)
    kvd.kvd_mx_load(s, c, 8, 8, *back)
    assert same(back[0], want) and same(back[1], want)


def test_numbers_of_the_format_stay_as_they_are():
    # stored, read back and stored again: the same bits
    s = shape("f32", 2, 2, 256)
    x = inputs.normal((2, 2, 50, 256), 1.0, "cuda", 6, 6)
    c, d = kvd.mx_cache(s, 2, 50), kvd.mx_cache(s, 2, 50)
    k, v = torch.empty_like(x), torch.empty_like(x)
    kvd.kvd_mx_store(s, x, 3 * x, 50, c, 50)
    kvd.kvd_mx_load(s, c, 50, 50, k, v)
    kvd.kvd_mx_store(s, k, v, 50, d, 50)
    a, b = torch.empty_like(x), torch.empty_like(x)
    kvd.kvd_mx_load(s, d, 50, 50, a, b)
    assert torch.equal(a, k) and torch.equal(b, v)


@pytest.mark.parametrize("N", [1, 3, 40])
def test_store_then_attend_in_a_captured_step(N):
    # the two calls of a decode step, replayed with other rows, lengths and queries
    s = shape("bf16", 8, 4, 256)
    B, window, sink = 3, 50, 4
    cap, T = sink + window + N - 1, 1 << 20
    c, d = kvd.mx_cache(s, B, cap), kvd.mx_cache(s, B, cap)
    k, v = (torch.zeros((B, 4, N, 256), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros((B, N, 8, 256), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros_like(q)
    lens = i32([N, N, N])
    n = kvd.kvd_sink_workspace_bytes(s, B, N, T, window, sink)
    ws, ws2 = (torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2))

    def step(cc, o, w):
        kvd.kvd_mx_store(s, k, v, N, cc, T, sink=sink, kv_len=lens)
        call(s, q, cc, T, window, sink, lens, None, out=o, ws=w)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        step(c, out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        step(c, out, ws)
    for t in (c, d):
        for part in t[:4]:
            part.zero_()
    for i in range(30):
        for j, t in enumerate((k, v, q)):
            t.copy_(inputs.normal(t.shape, 1.0, "cuda", i, 98, j).to(torch.bfloat16))
        lens.copy_(torch.tensor([N * (i + 1)] * 3, dtype=torch.int32))
        want = torch.zeros_like(out)
        step(d, want, ws2)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert all(torch.equal(a, b) for a, b in zip(c[:4], d[:4]))


def test_rows_beyond_32_bits():
    s = shape("bf16", 1, 1, 256)
    t_cap = (1 << 25) + 64   # 2^32 bytes of codes
    c = kvd.mx_cache(s, 1, t_cap)
    x = inputs.normal((1, 1, 40, 256), 1.0, "cuda", 3, 7).to(torch.bfloat16)
    kvd.kvd_mx_store(s, x, 2 * x, 40, c, t_cap)
    k, v = torch.empty_like(x), torch.empty_like(x)
    kvd.kvd_mx_load(s, c, t_cap, 40, k, v)
    assert same(k, held(x)) and same(v, held(2 * x))
    assert not c.k[:, :, :t_cap - 40].any() and not c.k_scale[:, :, :t_cap - 40].any()
