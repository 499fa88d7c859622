"""budget.WeightedCache on the GPU: prompts and decode steps of the three new operators together, every call checked
against the oracle on the cache that the GPU held before it (attention and weights within the arithmetic's bound,
evictions bit for bit), and what the cache finally holds against the rows it claims to hold."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2603_19664_amd import configs as C
from paper_2603_19664_amd import inputs
from paper_2603_19664_amd import kvd
from paper_2603_19664_amd.budget import WeightedCache

from gpu_cases import make_layer, note
from rows_cases import bound, is_tile, within

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    note(f"[gpu] {request.node.nodeid}")
    yield
    torch.cuda.synchronize()


class Checked(WeightedCache):
    """Checks every attention and every eviction as it happens."""

    def _attend(self, q, N, out):
        before = self.weight.clone()
        super()._attend(q, N, out)
        s, n = self.shape, self.n
        q4, o4 = (t.view(self.B, N, s.n_q_heads, s.head_dim) for t in (q, out))
        x = dict(q=q4, pk=self.prefix_k, pv=self.prefix_v, k=self.k, v=self.v)
        dtype = "bf16" if s.dtype == kvd.KVD_BF16 else "f32"
        tile = is_tile(dtype, N, s.n_q_heads // s.n_kv_heads, self.B, self.T_prefix, n)
        ref, tol, w, wt = bound(x, s, self.T_prefix, n, 0, 0, [n] * self.B, [N] * self.B, tile)
        within("out", o4, ref, tol)
        want = self.decay * inputs.to_f64(before[:, :, :n]) + w
        within("weight", self.weight[:, :, :n], want, wt + 2.0 ** -22 * np.abs(want))
        assert torch.equal(self.weight[:, :, n:], before[:, :, n:])

    def evict(self):
        if self.n <= self.budget:
            return
        f = [t.float().cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy()
             for t in (self.k, self.v, self.weight, self.pos)]
        want = O.evict(*f, [self.n] * self.B, self.last_pos.tolist(), self.budget, self.sink, self.recent)
        super().evict()
        for got, w in zip((self.k, self.v, self.weight, self.pos), want):
            assert np.array_equal(got.float().cpu().numpy() if got.dtype == torch.bfloat16 else got.cpu().numpy(), w)
        self.evictions = getattr(self, "evictions", 0) + 1


CASES = [
    # workload, batch, budget, room, prefix, sink, recent, decay, prompt, steps
    (C.SMOLLM_FP32, 2, 24, 1, 0, 2, 6, 1.0, 30, 20),
    (C.SMOLLM_FP32, 3, 40, 16, 50, 0, 8, 0.9, 70, 30),
    (C.QWEN_1_5B, 2, 64, 32, 100, 4, 16, 1.0, 90, 40),
    (C.GEMMA3_4B, 2, 48, 1, 33, 1, 1, 0.0, 7, 60),
    (C.GEMMA3_4B, 1, 100, 80, 0, 4, 20, 1.0, 230, 12),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0].name.split('-')[0]}-b{c[1]}-{c[2]}+{c[3]}-p{c[4]}")
def test_prompt_and_steps(case):
    wl, B, budget, room, T_prefix, sink, recent, decay, T, steps = case
    L = make_layer(wl, B, T, seed=5, w_q_std=0.05)
    s, args = L.shape, (L.gamma, L.lw_q, L.lw_k, L.lw_v)
    prefix = None
    if T_prefix:
        hp = inputs.normal((1, T_prefix, s.d_model), 1.0, "cuda", 5, 99).to(s.torch_dtype)
        pk = torch.empty((1, s.n_kv_heads, T_prefix, s.head_dim), dtype=s.torch_dtype, device="cuda")
        pv = torch.empty_like(pk)
        kvd.kvd_recompute_kv(s, hp, L.gamma, L.lw_k, L.lw_v, torch.full((1,), 3, dtype=torch.int32, device="cuda"),
                             T_prefix, pk, pv)
        prefix = (pk[0], pv[0])
    c = Checked(s, B, budget, room, prefix, sink, recent, decay, pos0=3)
    out = torch.empty((B, T, s.n_q_heads, s.head_dim), dtype=s.torch_dtype, device="cuda")
    c.prompt(L.h, *args, out)
    assert c.T == T and c.n == min(T, budget)
    hs = [L.h]
    for i in range(steps):
        h_new = inputs.normal((B, s.d_model), 1.0, "cuda", 6, i).to(s.torch_dtype)
        hs.append(h_new[:, None])
        o = torch.empty((B, s.n_q_heads, s.head_dim), dtype=s.torch_dtype, device="cuda")
        c.step(h_new, *args, o)
        assert torch.isfinite(o.float()).all()
    assert c.T == T + steps and c.n <= budget + room and c.evictions > 0
    # every row is the K/V of the token it names, at that token's position
    h = torch.cat(hs, 1).contiguous()
    K = torch.empty((B, s.n_kv_heads, c.T, s.head_dim), dtype=s.torch_dtype, device="cuda")
    V = torch.empty_like(K)
    p0 = torch.full((B,), 3 + T_prefix, dtype=torch.int32, device="cuda")
    kvd.kvd_recompute_kv(s, h, L.gamma, L.lw_k, L.lw_v, p0, c.T, K, V)
    idx = c.pos[:, :, :c.n].long()
    assert (idx.sort(-1).values.diff(dim=-1) > 0).all() and int(idx.max()) == c.T - 1
    rows = idx[..., None].expand(-1, -1, -1, s.head_dim)
    assert torch.equal(K.gather(2, rows), c.k[:, :, :c.n]) and torch.equal(V.gather(2, rows), c.v[:, :, :c.n])
    if sink:
        assert (idx < sink).sum(-1).eq(sink).all()
    if recent:
        assert (idx >= c.T - recent).sum(-1).eq(min(recent, c.T)).all()


def test_before_the_budget_it_is_plain_attention():
    # nothing evicted: the cache answers as kvd_decode_attn over the same rows
    L = make_layer(C.GEMMA3_4B, 2, 20, seed=9)
    s, args = L.shape, (L.gamma, L.lw_q, L.lw_k, L.lw_v)
    c = WeightedCache(s, 2, 64)
    out = torch.empty((2, 20, s.n_q_heads, s.head_dim), dtype=s.torch_dtype, device="cuda")
    c.prompt(L.h, *args, out)
    o = torch.empty((2, s.n_q_heads, s.head_dim), dtype=s.torch_dtype, device="cuda")
    q = c.step(L.h_new, *args, o)
    want = torch.empty_like(o)
    kvd.kvd_decode_attn(s, q, c.k, c.v, 21, want, kvd.workspace(s, kvd.KVD_OP_DECODE_ATTN, 2, 21))
    assert (o.float() - want.float()).abs().max() <= 2.0 ** -7 * want.float().abs().max()
    # weights: 21 tokens gave one unit per head each
    g = s.n_q_heads // s.n_kv_heads
    assert (c.weight.sum(-1) - 21 * g).abs().max() < 1e-3
