"""Algorithm 1's bounded cache (Sec. 3.4): the host bookkeeping of a decode loop
with cache budget B > 0 around libkvd's C-ABI calls.

Per layer, for a batch of sequences decoded in lockstep:

  ckpt   [batch][t_max][d]            residual checkpoints.  Row t is token t's
                                      residual h^(l) (position pos0[b] + t).  Rows
                                      0 .. T_rec-1 are the evicted tokens, which
                                      every step recomputes (RECOMPUTE_KV); rows
                                      T_rec .. T-1 belong to tokens still in the
                                      cache and wait there for their eviction.
  ring   K, V [batch][n_kv][B+1][hd]  the KV cache K[l] of B slots plus one slot
                                      for the token being decoded, used as a ring:
                                      the cached tokens sit in slots head,
                                      head + 1, ... (mod B + 1), oldest first.

One decode step (BoundedCache.step) issues, in Algorithm 1's order:
  1. kvd_store_residual: the current token's residual into ckpt row T (its
     h^(l) exists only now; STORE_RESIDUAL moves it into the recomputed range
     when it is evicted later);
  2. kvd_project_qkv: Q, K_t, V_t (Eqs. q_proj, k_proj, v_proj), K_t / V_t into
     the ring's free slot;
  3. kvd_fused_recompute_attn: RECOMPUTE_KV of ckpt rows 0 .. T_rec-1, CONCAT
     with the ring read from its oldest slot (the cache, then K_t / V_t), and
     ATTENTION, in one kernel;
  4. EVICT_OLDEST (host only): the current token has joined the cache; past
     the budget the oldest cached token leaves the ring (head advances) and its
     residual, already in ckpt row T_rec, joins the recomputed rows.

Memory per layer and sequence: (T - B) evicted residuals plus B cached K/V
entries (Eq. total_mem per layer), plus what Algorithm 1 holds beside them and
the equation leaves out: the current token's K_t / V_t (the ring's extra slot)
and the residuals of the B cached tokens, kept for their eviction.

WeightedCache bounds the cache by attention weight instead of age: it keeps the rows
that received the most (the paper's comparison systems that score cached tokens by
accumulated attention, Sec. 4), drops the others for good and recomputes nothing.  The
batch may share a prefix, whose keys and values are stored once and never evicted.

SinkCache bounds it by age as a sliding-window layer does, but keeps a few first tokens visible: sink + window rows
serve an endless stream, in the shape's dtype or in 4 bits.
"""
from __future__ import annotations

import contextlib
import dataclasses

from . import accounting


@dataclasses.dataclass
class RingState:
    """Indexes of Algorithm 1's cache for one layer (no device state).

    budget: cache slots B.  T: tokens decoded so far.  T_rec: evicted tokens
    (recomputed from checkpoints).  head: ring slot of the oldest cached token.
    n_cached: tokens in the cache (<= budget).  Invariant: T = T_rec + n_cached.
    """
    budget: int
    T: int = 0
    T_rec: int = 0
    head: int = 0
    n_cached: int = 0

    def __post_init__(self):
        if self.budget < 0:
            raise ValueError("budget must be >= 0")

    @property
    def slots(self) -> int:
        return self.budget + 1

    def free_slot(self) -> int:
        """Ring slot that receives the current token's K_t / V_t."""
        return (self.head + self.n_cached) % self.slots

    def tail_rows(self) -> int:
        """Rows the step attends from the ring: the cache, then the current token."""
        return self.n_cached + 1

    def slot_of(self, t: int) -> int:
        """Ring slot of cached token t (T_rec <= t < T_rec + n_cached), or of the current token t = T."""
        if not self.T_rec <= t <= self.T:
            raise ValueError(f"token {t} is not in the cache")
        return (self.head + (t - self.T_rec)) % self.slots

    def keys_in_order(self) -> list:
        """Tokens the step attends, in CONCAT order: recomputed, cached (oldest first), current."""
        return list(range(self.T_rec)) + [self.T_rec + i for i in range(self.n_cached)] + [self.T]

    def advance(self):
        """After the step's attention: the current token joins the cache; past the budget
        EVICT_OLDEST drops the oldest cached token, whose residual joins the recomputed rows."""
        self.T += 1
        self.n_cached += 1
        if self.n_cached > self.budget:
            self.head = (self.head + 1) % self.slots
            self.n_cached -= 1
            self.T_rec += 1

    def memory_bytes(self, d: int, n_kv: int, hd: int, b: int) -> dict:
        """Per layer and sequence: Eq. total_mem at the current T and budget, and what this
        cache holds (evicted residuals, retained residuals of cached tokens, ring slots)."""
        eq = accounting.total_memory(self.T, min(self.budget, self.T), 1, n_kv, hd, d, b)
        held = {"evicted_residuals": self.T_rec * d * b, "retained_residuals": self.n_cached * d * b,
                "ring_kv": self.slots * 2 * n_kv * hd * b}
        held["total"] = sum(held.values())
        return {"eq_total_mem": eq, "held": held}


class BoundedCache:
    """One layer's Algorithm 1 state on the GPU for `batch` sequences, `budget` cache slots and
    room for t_max tokens; step() runs one decode step through the C ABI (see module doc)."""

    def __init__(self, shape, batch: int, budget: int, t_max: int, pos0, device="cuda"):
        import torch

        from . import kvd
        self.kvd, self.torch = kvd, torch
        self.shape, self.B = shape, batch
        self.state = RingState(budget)
        dt = shape.torch_dtype
        self.t_max = t_max
        self.ckpt = torch.zeros((batch, t_max, shape.d_model), dtype=dt, device=device)
        self.ring_k = torch.zeros((batch, shape.n_kv_heads, budget + 1, shape.head_dim), dtype=dt, device=device)
        self.ring_v = torch.zeros_like(self.ring_k)
        self.pos0 = pos0
        self.q = torch.empty((batch, shape.n_q_heads, shape.head_dim), dtype=dt, device=device)
        # one workspace for every step: sized for the largest call (all t_max tokens recomputed or cached)
        ws_bytes = max(kvd.kvd_workspace_bytes(shape, kvd.KVD_OP_FUSED, batch, t_rec, budget + 1)
                       for t_rec in (0, max(t_max - 1, 0), max(t_max - budget - 1, 0)))
        ws_bytes = max(ws_bytes, kvd.kvd_workspace_bytes(shape, kvd.KVD_OP_FUSED, batch, t_max, 1))
        self.ws = torch.zeros(max(ws_bytes, 256), dtype=torch.uint8, device=device)

    def step(self, h_new, gamma, w_q, w_k, w_v, out):
        """Decode one token per sequence: h_new [batch, d] is its residual h^(l); out [batch, n_q, hd]."""
        kvd, st = self.kvd, self.state
        if st.T >= self.t_max:
            raise ValueError(f"the checkpoint store holds {self.t_max} tokens")
        pos = (self.pos0 + st.T).to(self.torch.int32)
        kvd.kvd_store_residual(self.shape, h_new, self.ckpt, st.T)                              # STORE_RESIDUAL
        kvd.kvd_project_qkv(self.shape, h_new, gamma, w_q, w_k, w_v, pos, self.q, self.ring_k, self.ring_v,
                            st.free_slot())                                                      # Q, K_t, V_t
        kvd.kvd_fused_recompute_attn(self.shape, self.q, self.ckpt, st.T_rec, gamma, w_k, w_v, self.pos0, out,
                                     self.ws, self.ring_k, self.ring_v, st.tail_rows(), st.head)  # RECOMPUTE+ATTN
        st.advance()                                                                             # EVICT_OLDEST
        return self.q


class WeightedCache:
    """One layer's stored K/V for `batch` sequences decoded in lockstep, held at `budget` rows per (sequence, KV
    head) by accumulated attention weight.

    Rows past the budget collect in `room` further slots (the tokens of one call at most); then kvd_evict keeps the
    `budget` heaviest: the first `sink` positions and the newest `recent` ones always, the others by the weight
    that kvd_prefix_attn has added up, `decay` times the earlier weight at every call (1: over the whole past, 0: the
    last call's alone).  Slots are reused, so row order says nothing about age; pos holds every row's token, counted
    from 0 behind the prefix (sink and recent count these tokens).

    prefix: (K, V) of [n_kv, T_prefix, head_dim], shared by the batch: its tokens sit at positions pos0 ..
    pos0 + T_prefix - 1 of every sequence, the sequences' own from pos0 + T_prefix on.
    """

    def __init__(self, shape, batch: int, budget: int, room: int = 1, prefix=None, sink: int = 0, recent: int = 0,
                 decay: float = 1.0, pos0: int = 0, device="cuda"):
        import torch

        from . import kvd
        if budget < 1 or room < 1:
            raise ValueError("budget and room must be >= 1")
        if sink < 0 or recent < 0 or sink + recent > budget:
            raise ValueError(f"sink={sink} and recent={recent} rows do not fit a budget of {budget}")
        self.kvd, self.torch = kvd, torch
        self.shape, self.B, self.budget, self.room = shape, batch, budget, room
        self.sink, self.recent, self.decay, self.pos0 = sink, recent, decay, pos0
        self.prefix_k, self.prefix_v = prefix if prefix is not None else (None, None)
        self.T_prefix = 0 if prefix is None else self.prefix_k.shape[1]
        dt, dev, cap = shape.torch_dtype, device, budget + room
        self.k = torch.zeros((batch, shape.n_kv_heads, cap, shape.head_dim), dtype=dt, device=dev)
        self.v = torch.zeros_like(self.k)
        self.weight = torch.zeros((batch, shape.n_kv_heads, cap), dtype=torch.float32, device=dev)
        self.pos = torch.zeros((batch, shape.n_kv_heads, cap), dtype=torch.int32, device=dev)
        self.last_pos = torch.zeros((batch,), dtype=torch.int32, device=dev)
        self.n = 0   # rows held
        self.T = 0   # tokens seen
        sizes = [kvd.kvd_evict_workspace_bytes(shape, batch, cap)] if batch else []
        sizes += [kvd.kvd_prefix_workspace_bytes(shape, batch, n, self.T_prefix, cap, True)
                  for n in sorted({1, room}) if batch]
        self.ws = torch.empty(max(sizes, default=256), dtype=torch.uint8, device=dev)
        self._ws_tokens = {1, room}

    def _here(self):
        """A context in which the cache's device is the current one: the projections launch there."""
        dev = self.k.device
        if dev.type != "cuda" or self.torch.cuda.current_device() == dev.index:
            return contextlib.nullcontext()
        return self.torch.cuda.device(dev)

    def _positions(self, N):
        """Positions of the N tokens being added, [B, N] int32."""
        t = self.torch.arange(self.T, self.T + N, dtype=self.torch.int32, device=self.k.device)
        return (t + (self.pos0 + self.T_prefix)).expand(self.B, N).contiguous()

    def _attend(self, q, N, out):
        kvd = self.kvd
        if N not in self._ws_tokens:
            need = kvd.kvd_prefix_workspace_bytes(self.shape, self.B, N, self.T_prefix, self.budget + self.room, True)
            if need > self.ws.numel():
                self.ws = self.torch.empty(need, dtype=self.torch.uint8, device=self.k.device)
            self._ws_tokens.add(N)
        self.pos[:, :, self.n:self.n + N] = self.torch.arange(self.T, self.T + N, device=self.k.device)
        kvd.kvd_prefix_attn(self.shape, q, self.prefix_k, self.prefix_v, self.T_prefix, self.k, self.v, self.n + N,
                            out, self.ws, weight=self.weight, decay=self.decay)
        # the tokens are in once the call is: a refused one leaves the cache as it was
        self.last_pos.fill_(self.T + N - 1)
        self.n += N
        self.T += N

    def evict(self):
        """Back to the budget, if there is more."""
        if self.n > self.budget:
            self.kvd.kvd_evict(self.shape, self.k, self.v, self.n, self.budget, self.weight, self.ws, pos=self.pos,
                               last_pos=self.last_pos, sink=self.sink, recent=self.recent)
            self.n = self.budget

    def step(self, h_new, gamma, w_q, w_k, w_v, out):
        """Decode one token per sequence: h_new [batch, d] is its residual h^(l); out [batch, n_q, hd].  Returns q."""
        s = self.shape
        with self._here():
            if self.n + 1 > self.budget + self.room:
                self.evict()
            q = self.torch.empty((self.B, s.n_q_heads, s.head_dim), dtype=s.torch_dtype, device=self.k.device)
            self.kvd.kvd_project_qkv(s, h_new, gamma, w_q, w_k, w_v, self._positions(1).view(self.B), q, self.k, self.v,
                                     self.n)
            self._attend(q, 1, out)
            if self.n == self.budget + self.room:
                self.evict()
        return q

    def prompt(self, h, gamma, w_q, w_k, w_v, out):
        """Take in the tokens of h [batch, T, d], at most `room` at a time, each chunk attended (causally) to what
        the cache holds and evicted down to the budget; out [batch, T, n_q, hd].  Returns q."""
        s, torch, kvd = self.shape, self.torch, self.kvd
        B, T = self.B, h.shape[1]
        if tuple(h.shape) != (B, T, s.d_model):
            raise ValueError(f"h has shape {tuple(h.shape)}, expected {(B, T, s.d_model)}")
        if tuple(out.shape) != (B, T, s.n_q_heads, s.head_dim):
            raise ValueError(f"out has shape {tuple(out.shape)}, expected {(B, T, s.n_q_heads, s.head_dim)}")
        q = torch.empty((B, T, s.n_q_heads, s.head_dim), dtype=s.torch_dtype, device=self.k.device)
        with self._here():
            for t in range(0, T, self.room):
                self.evict()
                N = min(self.room, T - t)
                x, pos = h[:, t:t + N].contiguous(), self._positions(N)
                qc = torch.empty((B, N, s.n_q_heads, s.head_dim), dtype=s.torch_dtype, device=self.k.device)
                kvd.kvd_project_q(s, x.view(B * N, s.d_model), gamma, w_q, pos.view(B * N),
                                  qc.view(B * N, s.n_q_heads, s.head_dim))
                kvd.kvd_recompute_kv(s, x, gamma, w_k, w_v, pos[:, 0].contiguous(), N, self.k, self.v, self.n)
                oc = torch.empty_like(qc)
                self._attend(qc, N, oc)
                q[:, t:t + N], out[:, t:t + N] = qc, oc
            self.evict()
        return q


class SinkCache:
    """One layer's stored K/V for `batch` sequences decoded in lockstep: the first `sink` tokens and a ring of the
    newest `window` ones (and `room` - 1 more, so that up to `room` tokens come in one call), in the shape's dtype or,
    with mx, in 4 bits.  Every new token sees the first `sink` tokens and the newest `window`, itself among them.

    A prompt is taken in parts of `room` tokens: the default of 1 is for decoding and runs a prompt token by token, as
    many launches each as a step; prompts run at full speed in parts of some hundreds, for as many more rows.

    Tokens sit at positions pos0, pos0 + 1, ..; a token's K keeps the rotation of its position.
    """

    def __init__(self, shape, batch: int, window: int, sink: int = 0, room: int = 1, mx: bool = False, pos0: int = 0,
                 device="cuda"):
        import torch

        from . import kvd
        if window < 1 or room < 1:
            raise ValueError("window and room must be >= 1")
        if sink < 0:
            raise ValueError("sink must be >= 0")
        self.kvd, self.torch = kvd, torch
        self.shape, self.B, self.window, self.sink, self.room, self.pos0 = shape, batch, window, sink, room, pos0
        self.ring = window + room - 1
        dt, cap = shape.torch_dtype, sink + self.ring
        rows = (batch, shape.n_kv_heads, room if mx else cap, shape.head_dim)
        self.mx = kvd.mx_cache(shape, batch, cap, device) if mx else None
        # in 4 bits: the rows of one call on their way into the cache
        self.k = torch.zeros(rows, dtype=dt, device=device)
        self.v = torch.zeros_like(self.k)
        self.T = 0  # tokens seen
        sizes = [kvd.kvd_sink_workspace_bytes(shape, batch, n, 2 ** 31 - 1, window, sink)
                 for n in range(1, room + 1) if batch]
        self.ws = torch.empty(max(sizes, default=256), dtype=torch.uint8, device=device)

    def _here(self):
        """A context in which the cache's device is the current one: the projections launch there."""
        dev = self.k.device
        if dev.type != "cuda" or self.torch.cuda.current_device() == dev.index:
            return contextlib.nullcontext()
        return self.torch.cuda.device(dev)

    def row(self, t: int) -> int:
        """The cache row of token t."""
        return t if t < self.sink else self.sink + (t - self.sink) % self.ring

    def _pieces(self, N):
        """(first of the N tokens being added, how many) of the parts that lie in neighbouring rows."""
        t, end = self.T, self.T + N
        while t < end:
            n = end - t if t < self.sink else min(end - t, self.ring - (t - self.sink) % self.ring)
            if t < self.sink:
                n = min(n, self.sink + self.ring - t)
            yield t, n
            t += n

    def _attend(self, q, N, out):
        kvd, s, T = self.kvd, self.shape, self.T + N
        if self.mx is not None:
            kvd.kvd_mx_store(s, self.k, self.v, N, self.mx, T, sink=self.sink)
            kvd.kvd_mx_attn(s, q, self.mx, T, out, self.ws, window=self.window, sink=self.sink)
        else:
            kvd.kvd_sink_attn(s, q, self.k, self.v, T, self.window, out, self.ws, sink=self.sink)
        self.T = T

    def step(self, h_new, gamma, w_q, w_k, w_v, out):
        """Decode one token per sequence: h_new [batch, d] is its residual h^(l); out [batch, n_q, hd].  Returns q."""
        s, torch, dev = self.shape, self.torch, self.k.device
        with self._here():
            q = torch.empty((self.B, s.n_q_heads, s.head_dim), dtype=s.torch_dtype, device=dev)
            pos = torch.full((self.B,), self.pos0 + self.T, dtype=torch.int32, device=dev)
            self.kvd.kvd_project_qkv(s, h_new, gamma, w_q, w_k, w_v, pos, q, self.k, self.v,
                                     0 if self.mx is not None else self.row(self.T))
            self._attend(q, 1, out)
        return q

    def prompt(self, h, gamma, w_q, w_k, w_v, out):
        """Take in the tokens of h [batch, T, d], at most `room` at a time; out [batch, T, n_q, hd].  Returns q."""
        s, torch, kvd, dev = self.shape, self.torch, self.kvd, self.k.device
        B, T = self.B, h.shape[1]
        if tuple(h.shape) != (B, T, s.d_model):
            raise ValueError(f"h has shape {tuple(h.shape)}, expected {(B, T, s.d_model)}")
        if tuple(out.shape) != (B, T, s.n_q_heads, s.head_dim):
            raise ValueError(f"out has shape {tuple(out.shape)}, expected {(B, T, s.n_q_heads, s.head_dim)}")
        q = torch.empty((B, T, s.n_q_heads, s.head_dim), dtype=s.torch_dtype, device=dev)
        with self._here():
            for t in range(0, T, self.room):
                N = min(self.room, T - t)
                x = h[:, t:t + N].contiguous()
                pos = torch.arange(self.pos0 + self.T, self.pos0 + self.T + N, dtype=torch.int32, device=dev)
                qc = torch.empty((B, N, s.n_q_heads, s.head_dim), dtype=s.torch_dtype, device=dev)
                kvd.kvd_project_q(s, x.view(B * N, s.d_model), gamma, w_q, pos.repeat(B),
                                  qc.view(B * N, s.n_q_heads, s.head_dim))
                for t0, n in [(self.T, N)] if self.mx is not None else list(self._pieces(N)):
                    i = t0 - self.T
                    first = torch.full((B,), self.pos0 + t0, dtype=torch.int32, device=dev)
                    kvd.kvd_recompute_kv(s, x if n == N else x[:, i:i + n].contiguous(), gamma, w_k, w_v, first, n,
                                         self.k, self.v, 0 if self.mx is not None else self.row(t0))
                oc = torch.empty_like(qc)
                self._attend(qc, N, oc)
                q[:, t:t + N], out[:, t:t + N] = qc, oc
        return q
