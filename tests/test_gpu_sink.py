"""kvd_sink_attn and kvd_mx_attn against the 64-bit oracle, element by element, on caches whose unused rows are NaN.

Bounds come from the arithmetic (sink_cases.bound) before any run."""
import random

import pytest
import torch

from paper_2603_19664_amd import inputs
from paper_2603_19664_amd import kvd

from gpu_cases import note
from sink_cases import bound, cache, call, held, i32, run, shape, tokens, within

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    note(f"[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


HEADS = [(64, 9, 3), (128, 12, 2), (256, 8, 4)]
BOTH = pytest.mark.parametrize("mx", [False, True], ids=["plain", "mx"])
DTYPES = pytest.mark.parametrize("dtype", ["bf16", "f32"])


@BOTH
@DTYPES
@pytest.mark.parametrize("hd,n_q,n_kv", HEADS)
@pytest.mark.parametrize("B,N,T,window,sink", [
    (1, 1, 1, 1, 0), (2, 1, 17, 5, 2), (3, 1, 65, 64, 4), (2, 1, 130, 1000, 0), (1, 1, 257, 257, 0), (2, 1, 300, 1, 1),
    (2, 4, 33, 16, 0), (1, 7, 90, 33, 40), (2, 33, 70, 20, 3), (1, 90, 90, 1, 0), (1, 90, 90, 90, 0),
    (2, 75, 211, 64, 4), (1, 150, 150, 31, 33), (5, 2, 2, 2, 0)])
def test_single_tokens_and_prompts(mx, dtype, hd, n_q, n_kv, B, N, T, window, sink):
    run(dtype, n_q, n_kv, hd, B, N, T, window, sink, mx, pad=3)


@BOTH
@DTYPES
@pytest.mark.parametrize("hd,n_q,n_kv", HEADS)
@pytest.mark.parametrize("B,N,T,window,sink,extra", [
    (1, 1, 100, 16, 4, 0), (2, 1, 500, 64, 0, 0), (3, 1, 77, 33, 1, 5), (1, 5, 333, 40, 7, 0), (2, 40, 260, 50, 4, 0),
    (1, 40, 1000, 21, 16, 3), (2, 1, 2000, 1, 0, 0), (1, 130, 700, 64, 2, 0)])
def test_rings(mx, dtype, hd, n_q, n_kv, B, N, T, window, sink, extra):
    run(dtype, n_q, n_kv, hd, B, N, T, window, sink, mx, slots=sink + window + N - 1 + extra, pad=1)


@BOTH
@pytest.mark.parametrize("N", [1, 20])
def test_every_place_of_the_rings_end(mx, N):
    # the stream's end at every row of the ring, and before the ring is full
    window, sink = 18, 3
    slots = sink + window + N - 1
    lens = list(range(0, slots + 25))
    run("bf16", 4, 2, 64, len(lens), N, 200, window, sink, mx, lens=lens, slots=slots)


@BOTH
@DTYPES
@pytest.mark.parametrize("g", [1, 2, 3, 5, 7, 8, 11, 16])
def test_group_sizes(mx, dtype, g):
    run(dtype, 2 * g, 2, 64, 3, 1, 77, 40, 2, mx)
    run(dtype, 2 * g, 2, 128, 1, 2, 35, 35, 0, mx)
    run(dtype, g, 1, 256, 2, 3, 41, 20, 4, mx)


@BOTH
@DTYPES
@pytest.mark.parametrize("N", [1, 5, 40])
def test_lengths_of_their_own(mx, dtype, N):
    # empty sequences, one token, fewer tokens than new ones, no new token, values beyond the range
    lens = [0, 1, 5, 60, 3, 77, 999, -4, 64, 40]
    news = [1, 1, 2, N, 0, N, N, 1, 99, max(N // 2, 1)]
    run(dtype, 6, 2, 128, len(lens), N, 77, 30, 4, mx, lens, news, pad=1)
    run(dtype, 6, 2, 64, len(lens), N, 77, 77, 0, mx, lens, None)
    run(dtype, 2, 1, 256, len(lens), N, 77, 9, 1, mx, None, news, slots=1 + 9 + N - 1)


@BOTH
@DTYPES
@pytest.mark.parametrize("hd,n_q,n_kv", HEADS)
def test_many_slots(mx, dtype, hd, n_q, n_kv):
    # ranges long enough to be cut many times, and rows of unequal numbers of them
    run(dtype, n_q, n_kv, hd, 2, 1, 4001, 4001, 0, mx, [4001, 700])
    run(dtype, n_q, n_kv, hd, 1, 1, 5000, 2222, 5, mx, slots=5 + 2222)
    run(dtype, n_q, n_kv, hd, 2, 50, 1200, 1200, 0, mx, [1200, 400])
    run(dtype, n_q, n_kv, hd, 1, 200, 1500, 900, 4, mx)


@BOTH
@DTYPES
@pytest.mark.parametrize("hd,n_q,n_kv", HEADS)
def test_long_prompts(mx, dtype, hd, n_q, n_kv):
    run(dtype, n_q, n_kv, hd, 2, 400, 400, 400, 0, mx, [400, 123], [400, 123])
    run(dtype, n_q, n_kv, hd, 1, 500, 500, 100, 4, mx)


@BOTH
@DTYPES
@pytest.mark.parametrize("N", [1, 4, 80])
def test_sharp_and_far_scores(mx, dtype, N):
    # scores of standard deviation 30: the running maximum moves often and most weights vanish
    run(dtype, 6, 2, 128, 2, N, 250, 150, 8, mx, q_std=30.0)


def test_the_largest_window_and_sink_are_the_whole_past():
    for mx in (False, True):
        for N in (1, 30):
            a = run("bf16", 4, 2, 64, 2, N, 90, 2 ** 31 - 1, 0, mx)
            b = run("bf16", 4, 2, 64, 2, N, 90, 1, 2 ** 31 - 1, mx)
            c = run("bf16", 4, 2, 64, 2, N, 90, 90, 0, mx)
            assert torch.equal(a, c) and torch.equal(b, c)


@DTYPES
@pytest.mark.parametrize("N", [1, 6, 60])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_is_not_seen_has_no_part(dtype, N, bad):
    # tokens between the sinks and the windows, and tokens that only the last one sees
    B, T, window, sink, hd = 2, 230, 40, 3, 64
    s = shape(dtype, 6, 2, hd)
    x = tokens(dtype, 6, 2, hd, B, N, T, 3)
    clean = {n: t.clone() for n, t in x.items()}
    a = call(s, x["q"], (x["k"], x["v"]), T, window, sink)
    for t in ("k", "v"):
        x[t][:, :, sink:T - N - window + 1] = bad
    assert torch.equal(call(s, x["q"], (x["k"], x["v"]), T, window, sink), a)
    x = clean
    hit = torch.zeros(hd, dtype=torch.bool, device="cuda")
    hit[::3] = True
    x["v"][:, :, T - 1, ::3] = bad
    d = call(s, x["q"], (x["k"], x["v"]), T, window, sink)
    assert torch.equal(d[:, :-1], a[:, :-1]) and torch.equal(d[:, -1][..., ~hit], a[:, -1][..., ~hit])
    last = d[:, -1][..., hit]
    assert torch.isnan(last).all() if bad != bad else (last == bad).all()
    # the oldest token of the first new token's window: the others have moved on
    y = tokens(dtype, 6, 2, hd, B, N, T, 3)
    y["v"][:, :, T - N - window + 1, ::3] = bad
    d = call(s, y["q"], (y["k"], y["v"]), T, window, sink)
    assert torch.equal(d[:, 1:], a[:, 1:]) and torch.equal(d[:, 0][..., ~hit], a[:, 0][..., ~hit])
    first = d[:, 0][..., hit]
    assert torch.isnan(first).all() if bad != bad else (first == bad).all()
    y["v"].copy_(tokens(dtype, 6, 2, hd, B, N, T, 3)["v"])
    y["k"][:, :, T - N - window + 1] = float("nan")
    d = call(s, y["q"], (y["k"], y["v"]), T, window, sink)
    assert torch.equal(d[:, 1:], a[:, 1:]) and torch.isnan(d[:, 0]).all()


@DTYPES
@pytest.mark.parametrize("N", [1, 6, 60])
@pytest.mark.parametrize("where", ["k", "v"])
def test_nan_groups_of_a_4_bit_cache(dtype, N, where):
    # a group of 32 that is NaN: as a value in its columns, as a key everywhere, for the tokens that see it
    B, T, window, sink, hd = 2, 150, 40, 3, 128
    s = shape(dtype, 6, 2, hd)
    x = tokens(dtype, 6, 2, hd, B, N, T, 5)
    c = cache(x, [T] * B, T, T, sink, True)
    a = call(s, x["q"], c, T, window, sink)
    scale = c.k_scale if where == "k" else c.v_scale
    keep = scale.clone()
    scale[:, :, sink:T - N - window + 1] = 255
    assert torch.equal(call(s, x["q"], c, T, window, sink), a)
    scale.copy_(keep)
    scale[:, :, T - 1, 2] = 255
    d = call(s, x["q"], c, T, window, sink)
    hit = torch.ones(hd, dtype=torch.bool, device="cuda")
    if where == "v":
        hit[:64] = hit[96:] = False
    assert torch.equal(d[:, :-1], a[:, :-1]) and torch.equal(d[:, -1][..., ~hit], a[:, -1][..., ~hit])
    assert torch.isnan(d[:, -1][..., hit]).all()


@DTYPES
@pytest.mark.parametrize("N", [1, 6, 60])
def test_a_seen_infinity_stays_one_however_small_its_weight(dtype, N):
    # sharp scores take most weights to 0 in 32 bits
    B, T, hd = 2, 600, 64
    s = shape(dtype, 4, 2, hd)
    x = tokens(dtype, 4, 2, hd, B, N, T, 6, q_std=60.0)
    x["v"][:, :, 5, 0] = float("inf")
    x["v"][:, :, 300, 1] = float("-inf")
    out = call(s, x["q"], (x["k"], x["v"]), T, T, 0)
    assert (out[..., 0] == float("inf")).all() and (out[..., 1] == float("-inf")).all()
    assert torch.isfinite(out[..., 2:]).all()


@BOTH
@DTYPES
@pytest.mark.parametrize("N,T", [(3, 90), (3, 900), (40, 90), (90, 700)])
def test_queries_of_no_token_have_no_part(mx, dtype, N, T):
    # a padded batch: the queries behind a sequence's new tokens are NaN
    news, lens = [N, 1, 0, N - 1], [T, T - 5, 7, 2]
    s = shape(dtype, 6, 2, 64)
    x = tokens(dtype, 6, 2, 64, 4, N, T, 7)
    c = cache(x, lens, T, T, 4, mx)
    a = call(s, x["q"], c, T, 200, 4, lens, news)
    for b, n in enumerate(news):
        x["q"][b, n:] = float("nan")
    d = call(s, x["q"], c, T, 200, 4, lens, news)
    assert torch.isfinite(d).all() and torch.equal(a, d)


@BOTH
@DTYPES
@pytest.mark.parametrize("N,T,window", [(1, 900, 900), (4, 300, 77), (40, 600, 600), (100, 400, 50)])
def test_repeats_and_shared_workspace(mx, dtype, N, T, window):
    # bit for bit on a workspace that other calls have written, sized for the longest
    s = shape(dtype, 6, 2, 128)
    x = tokens(dtype, 6, 2, 128, 3, N, T, 7)
    c = cache(x, [T] * 3, T, T, 0, mx)
    n = kvd.kvd_sink_workspace_bytes(s, 3, N, T + 5000, window, 0)
    ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")
    outs = [call(s, x["q"], c, T, window, 0, [t] * 3, ws=ws).clone() for t in (T, T // 2 + N, T)]
    assert torch.equal(outs[0], outs[2])
    assert torch.equal(outs[1], call(s, x["q"], c, T, window, 0, [T // 2 + N] * 3))


@BOTH
def test_nothing_is_written_behind_the_workspace(mx):
    for dtype, N, T in (("bf16", 1, 3000), ("bf16", 3, 500), ("bf16", 60, 900), ("f32", 1, 700), ("f32", 40, 300)):
        s = shape(dtype, 6, 2, 64)
        x = tokens(dtype, 6, 2, 64, 2, N, T, 8)
        c = cache(x, [T, T // 3], T, T, 4, mx)
        n = kvd.kvd_sink_workspace_bytes(s, 2, N, T, T, 4)
        ws = torch.full((n + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
        call(s, x["q"], c, T, T, 4, [T, T // 3], ws=ws[:n])
        assert (ws[n:] == 0xa5).all()


def test_plain_windows_match_weighted_attention():
    # a window of the whole past is what kvd_weighted_attn computes, up to the order of the sums
    for dtype in ("bf16", "f32"):
        for N in (1, 9, 70):
            s = shape(dtype, 8, 4, 256)
            x = tokens(dtype, 8, 4, 256, 2, N, 500, 11)
            a = call(s, x["q"], (x["k"], x["v"]), 500, 500, 0)
            out, w = torch.empty_like(a), torch.zeros((2, 4, 500), device="cuda")
            ws = torch.empty(kvd.kvd_prefix_workspace_bytes(s, 2, N, 0, 500, True), dtype=torch.uint8, device="cuda")
            kvd.kvd_weighted_attn(s, x["q"], x["k"], x["v"], 500, w, out, ws)
            lim = 2.0 ** -7 if dtype == "bf16" else 2e-6
            assert (a.float() - out.float()).abs().max() <= lim * out.float().abs().max()


@BOTH
@pytest.mark.parametrize("N", [1, 4, 50])
def test_captured_and_replayed_beside_eager_calls(mx, N):
    s = shape("bf16", 12, 2, 128)
    B, T = 4, 700
    x = tokens("bf16", 12, 2, 128, B, N, T, 13)
    c = cache(x, [T] * B, T, T, 4, mx)
    lens = i32([700, 60, 50, 350])
    out = torch.zeros_like(x["q"])
    n = kvd.kvd_sink_workspace_bytes(s, B, N, T, 600, 4)
    ws, ws2 = (torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    go = lambda o, work: call(s, x["q"], c, T, 600, 4, lens, None, out=o, ws=work)  # noqa: E731
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        go(out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        go(out, ws)
    for i in range(4):
        x["q"].copy_(inputs.normal(x["q"].shape, 1.0, "cuda", i, 96).to(torch.bfloat16))
        lens.copy_(torch.tensor([700 - i, 60 + i, 50 + i, 350], dtype=torch.int32))
        want = torch.zeros_like(out)
        go(want, ws2)
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@BOTH
def test_two_calls_at_once_on_two_streams(mx):
    s = shape("bf16", 12, 2, 128)
    xs = [tokens("bf16", 12, 2, 128, 4, 2, 1500, 20 + i) for i in range(2)]
    cs = [cache(x, [1500] * 4, 1500, 1500, 0, mx) for x in xs]
    want = [call(s, x["q"], c, 1500, 1500, 0) for x, c in zip(xs, cs)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in xs], []
    for _ in range(3):
        for x, c, st in zip(xs, cs, streams):
            with torch.cuda.stream(st):
                got.append(call(s, x["q"], c, 1500, 1500, 0))
    torch.cuda.synchronize()
    for i, o in enumerate(got):
        assert torch.equal(o, want[i % 2])


@BOTH
@pytest.mark.parametrize("ring", [False, True])
def test_offsets_beyond_32_bits(mx, ring):
    # rows that start past 2^32 bytes in the store, of one sequence and of the call
    n_kv, hd = 1, 256
    t_cap = (1 << 25) + 1000 if mx else (1 << 23) + 1000
    s = shape("bf16", 2, n_kv, hd)
    for N in (1, 40):
        T = t_cap if not ring else 3 * t_cap + 17
        window, sink = 300, 4
        x = tokens("bf16", 2, n_kv, hd, 1, N, 400, 31)
        c = cache(x, [400], 400, 400, sink, mx)
        parts = list(c[:4]) if mx else list(c)
        big = []
        for p in parts:
            st = torch.zeros((1, n_kv, t_cap, p.shape[-1]), dtype=p.dtype, device="cuda")
            t = torch.arange(T - 396, T, device="cuda")
            row = t if not ring else sink + (t - sink) % (t_cap - sink)
            st[:, :, :sink] = p[:, :, :sink]
            st[:, :, row] = p[:, :, 4:]
            big.append(st)
        kv = kvd.MxCache(*big) if mx else tuple(big)
        # (a ring's end cuts the keys into other blocks: sums of another order)
        a = call(s, x["q"], kv, T, window, sink)
        k, v = (held(x[n]) if mx else inputs.to_f64(x[n]) for n in ("k", "v"))
        ref, tol = bound(x["q"], k, v, [400], [N], window, sink)
        within("out", a, ref, tol)
        if not ring:
            assert torch.equal(a, call(s, x["q"], c, 400, window, sink))
        del big, kv


@pytest.mark.parametrize("seed", range(48))
def test_calls_of_many_shapes(seed):
    # single tokens, drafts and prompts of both formats: whole caches, windows and rings, ragged or not
    rng = random.Random(seed)
    hd, n_q, n_kv = rng.choice(HEADS)
    B, N = rng.choice([(1, 1), (3, 1), (7, 1), (2, 2), (1, 5), (2, 17), (1, 64), (1, 129)])
    window, sink = rng.choice([1, 7, 32, 64, 100, 513]), rng.choice([0, 1, 4, 31, 33, 64])
    T = N + rng.choice([0, 1, 31, 200, 777])
    slots = None
    if rng.random() < 0.4:
        slots = sink + window + N - 1 + rng.choice([0, 1, 32])
        T = slots + rng.randint(1, 600)
    lens = news = None
    if rng.random() < 0.6:
        lens = [rng.randint(0, T) for _ in range(B)]
        news = [rng.randint(0, N) for _ in range(B)]
    run(rng.choice(["bf16", "f32"]), n_q, n_kv, hd, B, N, T, window, sink, rng.random() < 0.5, lens, news, slots, seed,
        rng.choice([0, 2]))


def test_the_binding_refuses_what_the_kernels_would_misread():
    s = shape("bf16", 4, 2, 64)
    x = tokens("bf16", 4, 2, 64, 2, 3, 20, 1)
    q, k, v = x["q"], x["k"], x["v"]
    c = kvd.mx_cache(s, 2, 20)
    out, ws = torch.empty_like(q), torch.empty(4096, dtype=torch.uint8, device="cuda")
    lens = i32([20, 20])

    def no(match, fn, *a, **kw):
        with pytest.raises(ValueError, match=match):
            fn(s, *a, **kw)
    f = kvd.kvd_sink_attn
    no("q has dtype", f, q.float(), k, v, 20, 8, out, ws)
    no("out must be contiguous", f, q, k, v, 20, 8, torch.empty((2, 3, 64, 4), dtype=q.dtype, device="cuda").transpose(2, 3), ws)
    no("out is on|on the GPU", f, q, k, v, 20, 8, out.cpu(), ws)
    no("kv_k has dtype", f, q, k.float(), v.float(), 20, 8, out, ws)
    no("kv_v has shape", f, q, k, v[:, :, :19], 20, 8, out, ws)
    no("kv_k must be contiguous", f, q, k.transpose(2, 3).contiguous().transpose(2, 3), v, 20, 8, out, ws)
    no("k and v are required", f, q, k, None, 20, 8, out, ws)
    no("kv_len has dtype", f, q, k, v, 20, 8, out, ws, kv_len=lens.long())
    no("n_new has shape", f, q, k, v, 20, 8, out, ws, n_new=i32([1]))
    no("ws must be|on the GPU", f, q, k, v, 20, 8, out, ws.cpu())
    g = kvd.kvd_mx_attn
    no("cache.k has dtype", g, q, c._replace(k=c.k.char()), 20, out, ws)
    no("cache.v_scale has shape", g, q, c._replace(v_scale=c.k_scale[..., :1]), 20, out, ws)
    no("cache.k_scale is on|on the GPU", g, q, c._replace(k_scale=c.k_scale.cpu()), 20, out, ws)
    no("cache.k must be a", g, q, c._replace(k=None), 20, out, ws)
    no("cache.v must be a", g, q, c._replace(v=None), 20, out, ws)
    r = kvd.kvd_mx_store
    no("rows_k has dtype", r, k.float(), v.float(), 20, c, 20)
    no("rows: rows", r, k, v, 21, c, 20)
    no("k and v are required", r, k, None, 20, c, 20)
    for bad in (dict(T=21, window=18, N=3), dict(T=21, window=20, N=1)):
        with pytest.raises(kvd.KvdError) as e:   # a ring that is too short
            f(s, q[:, :bad["N"]].contiguous(), k, v, bad["T"], bad["window"], out[:, :bad["N"]].contiguous(), ws, sink=1)
        assert e.value.status == kvd.KVD_ERR_SHAPE
    with pytest.raises(kvd.KvdError) as e:
        f(s, q, k, v, 20, 8, out, ws[:0])
    assert e.value.status == kvd.KVD_ERR_WORKSPACE
