"""budget.SinkCache on the GPU: prompts and decode steps of projection, store and attention together, against the oracle
on the keys and values of every token so far."""
import pytest
import torch

from paper_2603_19664_amd import configs as C
from paper_2603_19664_amd import inputs
from paper_2603_19664_amd import kvd
from paper_2603_19664_amd.budget import SinkCache

from gpu_cases import make_layer, note
from sink_cases import bound, held, within

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    note(f"[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


CASES = [
    # workload, batch, window, sink, room, prompt, steps
    (C.SMOLLM_FP32, 2, 20, 2, 1, 9, 40),
    (C.SMOLLM_FP32, 1, 33, 0, 16, 70, 9),
    (C.QWEN_1_5B, 2, 64, 4, 32, 150, 20),
    (C.GEMMA3_4B, 1, 48, 5, 7, 30, 50),
    (C.GEMMA3_4B, 2, 16, 40, 80, 230, 12),
    (C.QWEN_1_5B, 1, 1, 0, 1, 3, 5),
]


@pytest.mark.parametrize("mx", [False, True], ids=["plain", "mx"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0].name.split('-')[0]}-b{c[1]}-{c[2]}+{c[3]}-r{c[4]}")
def test_prompt_and_steps(case, mx):
    wl, B, window, sink, room, T, steps = case
    L = make_layer(wl, B, T + steps, seed=5, w_q_std=0.05)
    s, args = L.shape, (L.gamma, L.lw_q, L.lw_k, L.lw_v)
    c = SinkCache(s, B, window, sink, room, mx, pos0=3)
    n = T + steps
    out = torch.empty((B, n, s.n_q_heads, s.head_dim), dtype=s.torch_dtype, device="cuda")
    q = torch.empty_like(out)
    o = torch.empty_like(out[:, :T])
    q[:, :T] = c.prompt(L.h[:, :T], *args, o)
    out[:, :T] = o
    for t in range(T, n):
        o = torch.empty_like(out[:, 0])
        q[:, t] = c.step(L.h[:, t].contiguous(), *args, o)
        out[:, t] = o
    assert c.T == n
    # every token's K and V, as the cache had them
    k = torch.empty((B, s.n_kv_heads, n, s.head_dim), dtype=s.torch_dtype, device="cuda")
    v = torch.empty_like(k)
    kvd.kvd_recompute_kv(s, L.h, L.gamma, L.lw_k, L.lw_v, torch.full((B,), 3, dtype=torch.int32, device="cuda"), n, k, v)
    kh, vh = (held(a) if mx else inputs.to_f64(a) for a in (k, v))
    ref, tol = bound(q, kh, vh, [n] * B, [n] * B, window, sink)
    within("out", out, ref, tol)
    # and what the cache holds now
    held_tokens = list(range(min(sink, n))) + list(range(max(sink, n - c.ring), n))
    rows = [c.row(t) for t in held_tokens]
    assert len(set(rows)) == len(rows)
    if mx:
        N = min(n, c.ring)
        a, b = (torch.empty((B, s.n_kv_heads, N, s.head_dim), dtype=s.torch_dtype, device="cuda") for _ in range(2))
        kvd.kvd_mx_load(s, c.mx, n, N, a, b, sink=sink)
        assert (inputs.to_f64(a) == kh[:, :, n - N:]).all() and (inputs.to_f64(b) == vh[:, :, n - N:]).all()
    else:
        assert torch.equal(c.k[:, :, rows], k[:, :, held_tokens]) and torch.equal(c.v[:, :, rows], v[:, :, held_tokens])


def test_another_stream_than_the_current_default():
    L = make_layer(C.QWEN_1_5B, 2, 40, seed=6, w_q_std=0.05)
    s, args = L.shape, (L.gamma, L.lw_q, L.lw_k, L.lw_v)
    outs = []
    for st in (torch.cuda.current_stream(), torch.cuda.Stream()):
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            c = SinkCache(s, 2, 10, 2, 8, True)
            out = torch.empty((2, 40, s.n_q_heads, s.head_dim), dtype=s.torch_dtype, device="cuda")
            c.prompt(L.h, *args, out)
            o = torch.empty_like(out[:, 0])
            c.step(L.h_new, *args, o)
        torch.cuda.synchronize()
        outs.append((out, o))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
