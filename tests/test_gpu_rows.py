"""kvd_prefix_attn and kvd_weighted_attn against the 64-bit oracle, element by element.

Bounds come from the arithmetic (rows_cases.bound) before any run: scores and sums in fp32, one rounding of the
output, and one of every softmax weight where more than 16 bf16 rows share a key range."""
import numpy as np
import pytest
import torch

from paper_2603_19664_amd import inputs
from paper_2603_19664_amd import kvd

from gpu_cases import note
from rows_cases import bound, call, i32, is_tile, make, shape, within

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    note(f"[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


def run(dtype, n_q, n_kv, hd, B, N, T_prefix, T, lens=None, news=None, weights=False, decay=0.0, seed=1, pad=0,
        q_std=1.0):
    """One call at row offsets `pad` inside longer stores, checked in full."""
    x = make(dtype, n_q, n_kv, hd, B, N, T_prefix, T, seed, T_prefix + 2 * pad or None, T + 2 * pad or None, q_std)
    s = shape(dtype, n_q, n_kv, hd)
    L = [T] * B if lens is None else [min(max(n, 0), T) for n in lens]
    M = [N] * B if news is None else [min(max(n, 0), N) for n in news]
    w0 = x["weight"].clone()
    w = x["weight"] if weights else None
    out = call(s, x, T_prefix, T, lens, news, w, decay, pad, pad)
    ref, tol, wr, wt = bound(x, s, T_prefix, T, pad, pad, L, M, is_tile(dtype, N, n_q // n_kv, B, T_prefix, T))
    for b in range(B):
        within(f"out[{b}]", out[b, :M[b]], ref[b, :M[b]], tol[b, :M[b]])
        assert (out[b, M[b]:] == 7.0).all(), "rows behind the new tokens are left as they were"
    if weights:
        base = inputs.to_f64(w0)
        for b in range(B):
            rows = slice(pad, pad + L[b])
            want = decay * base[b, :, rows] + wr[b, :, :L[b]]
            within(f"weight[{b}]", w[b, :, rows], want, wt[b, :, :L[b]] + 2.0 ** -22 * np.abs(want) + 1e-30)
            keep = torch.ones_like(w[b], dtype=torch.bool)
            keep[:, rows] = False
            assert torch.equal(w[b][keep], w0[b][keep]), "weights of other rows are left as they were"
    return out, w


HEADS = [(64, 9, 3), (128, 12, 2), (256, 8, 4)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,n_q,n_kv", HEADS)
@pytest.mark.parametrize("B,N,T_prefix,T", [
    (1, 1, 1, 1), (2, 1, 100, 17), (3, 1, 63, 65), (5, 1, 257, 130), (1, 1, 0, 33), (2, 1, 31, 0), (7, 3, 129, 16),
    (2, 33, 70, 40), (1, 90, 0, 90), (2, 75, 300, 111), (20, 2, 1, 2)])
def test_single_tokens_and_prompts(dtype, hd, n_q, n_kv, B, N, T_prefix, T):
    run(dtype, n_q, n_kv, hd, B, N, T_prefix, T, weights=T > 0, pad=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("g", [1, 2, 3, 4, 5, 7, 8, 11, 16])
def test_group_sizes(dtype, g):
    run(dtype, 2 * g, 2, 64, 3, 1, 50, 77, weights=True, decay=0.5)
    run(dtype, 2 * g, 2, 128, 1, 2, 20, 35, weights=True, decay=1.0)
    run(dtype, g, 1, 256, 2, 1, 0, 41, weights=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T_prefix", [0, 37])
@pytest.mark.parametrize("N", [1, 5, 40])
def test_lengths_of_their_own(dtype, T_prefix, N):
    # empty sequences, one row, fewer rows than new tokens, no new token, values beyond the range
    lens = [0, 1, 5, 60, 3, 77, 999, -4, 64, 40]
    news = [1, 1, 2, N, 0, N, N, 1, 99, max(N // 2, 1)]
    run(dtype, 6, 2, 128, len(lens), N, T_prefix, 77, lens, news, weights=True, decay=0.9, pad=1)
    run(dtype, 6, 2, 64, len(lens), N, T_prefix, 77, lens, None, weights=True, pad=1)
    run(dtype, 2, 1, 256, len(lens), N, T_prefix, 77, None, news, weights=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,n_q,n_kv", HEADS)
def test_many_slots(dtype, hd, n_q, n_kv):
    # ranges long enough to be cut many times, prefix and own, merged over every slot
    run(dtype, n_q, n_kv, hd, 2, 1, 3001, 1999, [1999, 700], weights=True)
    run(dtype, n_q, n_kv, hd, 6, 2, 2100, 515, [515, 2, 64, 65, 300, 514], weights=True, decay=1.0)
    run(dtype, n_q, n_kv, hd, 1, 50, 1030, 1200, weights=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,n_q,n_kv", HEADS)
def test_weights_of_long_prompts(dtype, hd, n_q, n_kv):
    # a key's rows in several parts, of other numbers for early and late keys and for each sequence
    run(dtype, n_q, n_kv, hd, 2, 300, 0, 700, [700, 350], [300, 123], weights=True, decay=0.5, pad=2)
    run(dtype, n_q, n_kv, hd, 1, 400, 130, 400, weights=True)
    run(dtype, n_q, n_kv, hd, 3, 260, 0, 260, [260, 1, 200], [260, 1, 0], weights=True, decay=1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 4, 80])
def test_sharp_and_far_scores(dtype, N):
    # scores of standard deviation 30: the running maximum moves often and most weights vanish
    run(dtype, 6, 2, 128, 2, N, 200, 150, weights=True, q_std=30.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 6, 50])
@pytest.mark.parametrize("T_prefix", [0, 45])
def test_what_is_not_seen_has_no_part(dtype, N, T_prefix):
    # rows behind the lengths, rows outside the views and rows of later tokens hold NaN and infinities
    B, T, hd = 3, 90, 64
    lens, news = [90, 70, N + 3], [N, max(N - 1, 1), N]
    s = shape(dtype, 6, 2, hd)
    x = make(dtype, 6, 2, hd, B, N, T_prefix, T, 3, T_prefix + 8, T + 8)
    w = x["weight"]
    clean = {n: t.clone() for n, t in x.items()}
    for t in ("k", "v"):
        x[t][:, :, :4] = float("nan")
        x[t][:, :, 4 + T:] = float("inf")
        for b, n in enumerate(lens):
            x[t][b, :, 4 + n:] = float("-inf") if b % 2 else float("nan")
        x["p" + t][:, :4] = float("nan")
        x["p" + t][:, 4 + T_prefix:] = float("inf")
    w[:] = float("nan")  # decay 0: not read
    a = call(s, x, T_prefix, T, lens, news, w, 0.0, 4, 4)
    w2 = clean["weight"]
    c = call(s, clean, T_prefix, T, lens, news, w2, 0.0, 4, 4)
    assert torch.equal(a, c)
    for b, n in enumerate(lens):
        assert torch.equal(w[b, :, 4:4 + n], w2[b, :, 4:4 + n])
    if N == 1:
        return
    # the last token's own row: only that token may notice
    for bad in (float("nan"), float("inf"), float("-inf")):
        y = {n: t.clone() for n, t in clean.items()}
        for b, n in enumerate(lens):
            y["k"][b, :, 4 + n - 1] = float("nan")
            y["v"][b, :, 4 + n - 1, ::3] = bad
        d = call(s, y, T_prefix, T, lens, news, None, 0.0, 4, 4)
        for b, m in enumerate(news):
            assert torch.equal(d[b, :m - 1], c[b, :m - 1])
            assert torch.isnan(d[b, m - 1]).all()
        # an infinite value of a row that is seen: its columns alone
        y["k"].copy_(clean["k"])
        d = call(s, y, T_prefix, T, lens, news, None, 0.0, 4, 4)
        for b, m in enumerate(news):
            assert torch.equal(d[b, :m - 1], c[b, :m - 1])
            hit = torch.zeros(hd, dtype=torch.bool, device="cuda")
            hit[::3] = True
            assert torch.equal(d[b, m - 1][:, ~hit], c[b, m - 1][:, ~hit])
            last = d[b, m - 1][:, hit]
            assert torch.isnan(last).all() if bad != bad else (last == bad).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,T_prefix,T", [(3, 40, 90), (3, 700, 900), (40, 40, 90), (90, 0, 700), (90, 600, 300)])
def test_queries_of_no_token_have_no_part(dtype, N, T_prefix, T):
    # a padded batch: the queries behind a sequence's new tokens are NaN, in blocks with others and in ones of their own
    B, news = 4, [N, 1, 0, N - 1]
    lens = [T, T - 5, 7, 2]
    s = shape(dtype, 6, 2, 64)
    x = make(dtype, 6, 2, 64, B, N, T_prefix, T, 7)
    w, w0 = x["weight"].clone(), x["weight"].clone()
    a = call(s, x, T_prefix, T, lens, news, w0, 0.5)
    for b, n in enumerate(news):
        x["q"][b, n:] = float("nan")
    c = call(s, x, T_prefix, T, lens, news, w, 0.5)
    assert torch.isfinite(c).all() and torch.equal(a, c) and torch.equal(w, w0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_values_at_a_range_end(dtype):
    # a seen infinity in the last, ragged block is an infinity, not 0 * inf
    for T_prefix, T, N in ((0, 37, 1), (37, 5, 1), (37, 70, 40), (333, 0, 60)):
        s = shape(dtype, 4, 2, 128)
        x = make(dtype, 4, 2, 128, 2, N, T_prefix, T, 5)
        (x["v"][:, :, T - 1 - (N - 1)] if T else x["pv"][:, T_prefix - 1])[..., 0] = float("inf")
        out = call(s, x, T_prefix, T)
        assert (out[:, -1, :, 0] == float("inf")).all()
        assert torch.isfinite(out[..., 1:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,T_prefix,T", [(1, 500, 300), (4, 77, 90), (40, 300, 400), (100, 0, 100)])
def test_repeats_and_shared_workspace(dtype, N, T_prefix, T):
    # bit for bit on a workspace that other calls have written, sized for the longest
    s = shape(dtype, 6, 2, 128)
    x = make(dtype, 6, 2, 128, 3, N, T_prefix, T, 7)
    n = kvd.kvd_prefix_workspace_bytes(s, 3, N, max(T_prefix, 1) + 500, T + 500, True)
    ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")
    outs = []
    for t in (T, T // 2 + N, T):
        w = torch.zeros_like(x["weight"])
        outs.append((call(s, x, T_prefix, T, [t] * 3, None, w, 0.0, ws=ws).clone(), w))
    assert torch.equal(outs[0][0], outs[2][0]) and torch.equal(outs[0][1], outs[2][1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,N,T_prefix,T", [(2, 1, 0, 100), (3, 1, 60, 500), (2, 4, 0, 900), (2, 2, 1000, 90),
                                            (2, 50, 0, 400), (2, 30, 300, 200), (1, 150, 40, 500)])
def test_out_is_the_same_with_weights_and_without(dtype, B, N, T_prefix, T):
    s = shape(dtype, 6, 2, 64)
    x = make(dtype, 6, 2, 64, B, N, T_prefix, T, 13)
    lens = [T, T // 3][:B] + [1] * (B - 2)
    assert torch.equal(call(s, x, T_prefix, T, lens), call(s, x, T_prefix, T, lens, None, x["weight"], 1.0))



def test_weighted_is_prefix_without_a_prefix():
    s = shape("bf16", 6, 2, 128)
    x = make("bf16", 6, 2, 128, 2, 3, 0, 200, 9)
    w1, w2 = x["weight"].clone(), x["weight"].clone()
    a = call(s, x, 0, 200, [200, 150], [3, 2], w1, 1.0)
    b = torch.full_like(x["q"], 7.0)
    ws = torch.empty(kvd.kvd_prefix_workspace_bytes(s, 2, 3, 0, 200, True), dtype=torch.uint8, device="cuda")
    kvd.kvd_weighted_attn(s, x["q"], x["k"], x["v"], 200, w2, b, ws, kv_len=i32([200, 150]), n_new=i32([3, 2]))
    assert torch.equal(a, b) and torch.equal(w1, w2)


def test_matches_decode_attention():
    # one token over one cache: what kvd_decode_attn gives, up to the order of the sums
    for dtype in ("bf16", "f32"):
        s = shape(dtype, 8, 4, 256)
        x = make(dtype, 8, 4, 256, 3, 1, 0, 777, 11)
        a = call(s, x, 0, 777)[:, 0]
        out = torch.empty_like(a)
        kvd.kvd_decode_attn(s, x["q"][:, 0].contiguous(), x["k"], x["v"], 777, out,
                            kvd.workspace(s, kvd.KVD_OP_DECODE_ATTN, 3, 777))
        lim = 2.0 ** -7 if dtype == "bf16" else 2e-6
        assert (a.float() - out.float()).abs().max() <= lim * out.float().abs().max()


def test_captured_and_replayed_beside_eager_calls():
    s = shape("bf16", 12, 2, 128)
    B, N, Tp, T = 4, 3, 900, 300
    x = make("bf16", 12, 2, 128, B, N, Tp, T, 13)
    lens = i32([300, 20, 0, 150])
    w = torch.zeros_like(x["weight"])
    out = torch.zeros_like(x["q"])
    n = kvd.kvd_prefix_workspace_bytes(s, B, N, Tp, T, True)
    ws, ws2 = (torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2))

    def go(o, weight, work, q):
        kvd.kvd_prefix_attn(s, q, x["pk"], x["pv"], Tp, x["k"], x["v"], T, o, work, own_len=lens, weight=weight)

    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        go(out, w, ws, x["q"])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        go(out, w, ws, x["q"])
    for i in range(4):
        x["q"].copy_(inputs.normal(x["q"].shape, 1.0, "cuda", i, 96).to(torch.bfloat16))
        lens.copy_(torch.tensor([300 - i, 20 + i, i, 150], dtype=torch.int32))
        want, ww = torch.zeros_like(out), torch.zeros_like(w)
        go(want, ww, ws2, x["q"])
        out.zero_()
        w.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(w, ww)


def test_two_calls_at_once_on_two_streams():
    s = shape("bf16", 12, 2, 128)
    xs = [make("bf16", 12, 2, 128, 4, 2, 1500, 400, 20 + i) for i in range(2)]
    want = [call(s, x, 1500, 400) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = []
    for _ in range(3):
        for x, st in zip(xs, streams):
            with torch.cuda.stream(st):
                got.append(call(s, x, 1500, 400))
    torch.cuda.synchronize()
    for i, o in enumerate(got):
        assert torch.equal(o, want[i % 2])


def test_offsets_beyond_32_bits():
    # rows of the last sequence start past 2^32 bytes (and 2^31 elements) in the store
    B, n_kv, hd, t_cap = 3, 2, 256, 1 << 21
    s = shape("bf16", 4, n_kv, hd)
    k = torch.zeros((B, n_kv, t_cap, hd), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    t_off, T = t_cap - 600, 600
    x = make("bf16", 4, n_kv, hd, B, 1, 0, T, 31)
    k[:, :, t_off:] = x["k"]
    v[:, :, t_off:] = x["v"]
    for N in (1, 12):
        y = make("bf16", 4, n_kv, hd, B, N, 0, T, 31)
        w, w2 = (torch.zeros((B, n_kv, c), device="cuda") for c in (t_cap, T))
        a = call(s, {**y, "k": k, "v": v}, 0, T, None, None, w, 0.0, 0, t_off)
        c = call(s, {**y, "k": x["k"], "v": x["v"]}, 0, T, None, None, w2, 0.0)
        assert torch.equal(a, c) and torch.equal(w[:, :, t_off:], w2)


@pytest.mark.parametrize("N", [1, 30])
def test_weights_at_4_byte_alignment(N):
    for dtype in ("bf16", "f32"):
        s = shape(dtype, 6, 2, 64)
        x = make(dtype, 6, 2, 64, 2, N, 50, 45, 33)
        flat = torch.zeros(x["weight"].numel() + 3, device="cuda")
        w = flat[3:].view(x["weight"].shape)
        w.copy_(x["weight"])
        a = call(s, x, 50, 45, None, None, w, 0.5)
        b = call(s, x, 50, 45, None, None, x["weight"], 0.5)
        assert torch.equal(a, b) and torch.equal(w, x["weight"])
