"""Attention over shared prefixes and weighted, evicting caches, as timed cases.

Each case is one layer's call, at the shapes of this repository's three model configurations:

  op "prefix"    N new tokens of every sequence attend a prefix of `prefix` keys that the whole batch shares and then the
                 sequence's own rows (kvd_prefix_attn), optionally adding up the weight each own row receives.
  op "weighted"  N new tokens of every sequence attend its own cache, and every cached key's attention weight is
                 added up (kvd_weighted_attn): the decode step and the prompt of a cache that evicts by weight.
  op "evict"     every (sequence, KV head) keeps its `keep` heaviest rows (kvd_evict).

Fields: model; B sequences; N new tokens a sequence, the last ones of its own rows; prefix shared keys; T own rows at
most; ragged: sequences have lengths of their own, up to T, and as many new tokens, up to N, as fit; weights: the own
rows' weights are wanted; decay: what is left of the earlier weights (0: none, they are not read).  Evict: keep, sink
(first positions that stay), recent (newest positions that stay).
"""
import math

import torch

own = False  # False: the operators' plain forms; True: the library's calls

# name: query heads, KV heads, head_dim, d_model, dtype
MODELS = {"smollm": (9, 3, 64, 576, torch.float32), "gemma": (8, 4, 256, 2560, torch.bfloat16),
          "qwen": (12, 2, 128, 1536, torch.bfloat16)}


def _prefix(model, B, N, prefix, T, ragged=True, weights=False, decay=0.0, name=None):
    c = {"op": "prefix", "model": model, "B": B, "N": N, "prefix": prefix, "T": T, "ragged": ragged,
         "weights": weights, "decay": decay}
    return c if name is None else {"name": name, **c}


def _weighted(model, B, N, T, ragged=False, decay=0.0, name=None):
    c = {"op": "weighted", "model": model, "B": B, "N": N, "prefix": 0, "T": T, "ragged": ragged, "weights": True,
         "decay": decay}
    return c if name is None else {"name": name, **c}


def _evict(model, B, T, keep, sink=4, recent=64, ragged=False, name=None):
    c = {"op": "evict", "model": model, "B": B, "T": T, "keep": keep, "sink": sink, "recent": recent,
         "ragged": ragged}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # two requests of the small fp32 model behind a short common instruction: the smallest call
        _prefix("smollm", 2, 1, 100, 17, name="smollm_prefix_step_fp32"),
        # a decode step of a serving batch with a common system prompt and conversations of different lengths
        _prefix("qwen", 32, 1, 4096, 512, name="qwen_prefix_step_b32"),
        # a decode step of many sampled continuations of one long document
        _prefix("gemma", 64, 1, 16384, 1024, name="gemma_prefix_step_b64"),
        # a drafted continuation of a few tokens checked in one call, the own rows' weights kept up
        _prefix("gemma", 16, 5, 2001, 333, weights=True, decay=1.0, name="gemma_prefix_draft_b16"),
        # the users' questions (prompts of up to 256 tokens) against a cached document
        _prefix("qwen", 8, 256, 8192, 256, name="qwen_prefix_prompts_b8"),
        # one token of the small fp32 model over its weighted cache
        _weighted("smollm", 1, 1, 257, decay=1.0, name="smollm_weighted_step_fp32"),
        # a decode step over caches held at a budget by eviction
        _weighted("gemma", 8, 1, 2049, decay=1.0, name="gemma_weighted_step_b8"),
        # the last token's weights over long contexts, before they are cut down
        _weighted("qwen", 8, 1, 16385, ragged=True, name="qwen_weighted_step_b8_16k"),
        # the last 32 tokens of long prompts as an observation window
        _weighted("qwen", 4, 32, 8209, name="qwen_weighted_window_b4"),
        # a whole prompt, causal, with the weights it leaves
        _weighted("gemma", 1, 3001, 3001, name="gemma_weighted_prompt"),
        # a decode step's eviction: one row a head leaves
        _evict("gemma", 8, 2049, 2048, name="gemma_evict_one_b8"),
        # long prompts cut down to a budget
        _evict("qwen", 8, 16385, 2048, ragged=True, name="qwen_evict_prompts_b8"),
    ]


def draw(rng):
    """One more call of the same ranges: single tokens, drafts, windows and prompts, each up to the largest listed."""
    def logint(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    op = rng.choice(["prefix", "prefix", "weighted", "weighted", "evict"])
    model = rng.choice(["smollm", "gemma", "gemma", "qwen", "qwen"])
    small = model == "smollm"
    ragged = rng.random() < 0.6
    if op == "evict":
        B = logint(1, 4 if small else 8)
        T = logint(16, 16385 // (4 if small else 1))
        keep = T - 1 if rng.random() < 0.5 else logint(8, T)
        sink, recent = rng.choice([0, 4]), rng.choice([0, 1, 32, 128])
        return _evict(model, B, T, max(keep, 1), min(sink, keep), max(0, min(recent, keep - sink)), ragged)
    kind = rng.choice(["step", "step", "draft", "prompt"])
    decay = rng.choice([0.0, 1.0, 0.9])
    if kind == "prompt":
        N = logint(33, 512)
        B = logint(1, 4 if small else 1024 // N)
        T = N if rng.random() < 0.5 else N + logint(1, 1024)
        prefix = logint(16, 1024 if small else 8192)
    else:
        N = 1 if kind == "step" else rng.randint(2, 32)
        B = logint(1, 4 if small else max(1, 64 // N))
        T = logint(N, (2048 if small else 32768) // B) if op == "weighted" else logint(N, 1024)
        prefix = logint(16, 1024 if small else 16384)
    T = max(T, N)
    if op == "weighted":
        return _weighted(model, B, N, T, ragged, decay)
    weights = rng.random() < 0.3
    return _prefix(model, B, N, prefix, T, ragged, weights, decay if weights else 0.0)


# ---------------------------------------------------------------- inputs

def _lengths(case, seed):
    """Own rows and new tokens of every sequence, host numbers: ragged lengths lie between half of T and T."""
    B, T, N = case["B"], case["T"], case.get("N", 1)
    if not case["ragged"]:
        return [T] * B, [N] * B
    gen = torch.Generator()
    gen.manual_seed(seed * 2 + 1)
    lens = torch.randint(max(1, T // 2), T + 1, (B,), generator=gen).tolist()
    lens[-1] = T
    return lens, [min(N, n) for n in lens]


def _tensors(case, seed):
    """The call's data: queries and keys N(0, 1) (scores of standard deviation 1), values N(0, 1); weights as a cache has
    them after some use (log-normal); positions as arrived, shuffled once a cache has reused its slots."""
    n_q, n_kv, hd, _, dt = MODELS[case["model"]]
    B, T = case["B"], case["T"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dt)

    lens, news = _lengths(case, seed)
    x = {"k": normal((B, n_kv, T, hd)), "v": normal((B, n_kv, T, hd)),
         "len": torch.tensor(lens, dtype=torch.int32, device="cuda"),
         "weight": torch.randn((B, n_kv, T), generator=gen, device="cuda").mul_(1.5).exp_()}
    if case["op"] == "evict":
        # a prompt's rows lie in order; a cache at its budget has its slots reused
        pos = torch.arange(T, device="cuda", dtype=torch.int32).expand(B, n_kv, T).contiguous()
        if case["keep"] == T - 1:
            order = torch.rand((B, n_kv, T - 1), generator=gen, device="cuda").argsort(-1).to(torch.int32)
            pos[:, :, :T - 1] = order
        x["pos"] = pos
        x["last"] = x["len"] - 1
        return x
    # rows that hold no token yet have gathered nothing; neither has any before the first look at the keys
    x["weight"] *= (torch.arange(T, device="cuda") < x["len"][:, None, None]) & (case["decay"] != 0.0)
    x["q"] = normal((B, case["N"], n_q, hd))
    x["new"] = torch.tensor(news, dtype=torch.int32, device="cuda")
    if case["op"] == "prefix":
        x["pk"], x["pv"] = normal((n_kv, case["prefix"], hd)), normal((n_kv, case["prefix"], hd))
    return x


def prepare(case, seed):
    st = {"case": case, **_tensors(case, seed)}
    # what the call updates in place starts from these in every pass
    if case["op"] == "evict":
        st["state0"] = torch.cat((st["weight"].view(torch.int32).flatten(), st["pos"].flatten(), st["len"]))
        st["state"] = st["state0"].clone()
        n, B = st["weight"].numel(), case["B"]
        st["weight_now"] = st["state"][:n].view(torch.float32).view(st["weight"].shape)
        st["pos_now"] = st["state"][n:2 * n].view(st["pos"].shape)
        st["len_now"] = st["state"][2 * n:2 * n + B]
    else:
        st["out"] = torch.zeros_like(st["q"])
        st["weight_now"] = st["weight"].clone()
    if own:
        from paper_2603_19664_amd import kvd
        n_q, n_kv, hd, d, dt = MODELS[case["model"]]
        s = kvd.Shape(d, n_q, n_kv, hd, 1e-6, 1e4, kvd.KVD_BF16 if dt == torch.bfloat16 else kvd.KVD_F32)
        B, T = case["B"], case["T"]
        st["kvd"], st["s"] = kvd, s
        if case["op"] == "evict":
            size = kvd.kvd_evict_workspace_bytes(s, B, T)
        else:
            size = kvd.kvd_prefix_workspace_bytes(s, B, case["N"], case["prefix"], T, case["weights"])
        st["ws"] = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
    return st


# ---------------------------------------------------------------- one pass

def run(st):
    case = st["case"]
    op, T = case["op"], case["T"]
    if op == "evict":
        st["state"].copy_(st["state0"])
        if own:
            st["kvd"].kvd_evict(st["s"], st["k"], st["v"], T, case["keep"], st["weight_now"], st["ws"],
                                pos=st["pos_now"], last_pos=st["last"], kv_len=st["len_now"], sink=case["sink"],
                                recent=case["recent"])
            return st["k"], st["v"], st["weight_now"], st["pos_now"], st["len_now"]
        return _plain_evict(st["k"], st["v"], st["weight_now"], st["pos_now"], st["len_now"], st["last"], case["keep"],
                            case["sink"], case["recent"])
    if case["decay"] != 0.0:
        st["weight_now"].copy_(st["weight"])
    lens, new = (st["len"], st["new"]) if case["ragged"] else (None, None)
    if own:
        if op == "prefix":
            st["kvd"].kvd_prefix_attn(st["s"], st["q"], st["pk"], st["pv"], case["prefix"], st["k"], st["v"], T,
                                      st["out"], st["ws"], own_len=lens, n_new=new,
                                      weight=st["weight_now"] if case["weights"] else None, decay=case["decay"])
        else:
            st["kvd"].kvd_weighted_attn(st["s"], st["q"], st["k"], st["v"], T, st["weight_now"], st["out"], st["ws"],
                                        kv_len=lens, n_new=new, decay=case["decay"])
        return (st["out"], st["weight_now"]) if case["weights"] else st["out"]
    out, w = _plain_attention(st["q"], st.get("pk"), st.get("pv"), st["k"], st["v"], st["len"], st["new"])
    out = torch.where(_valid(st["q"], st["new"])[:, :, None, None], out, 0.0).to(st["q"].dtype)
    if not case["weights"]:
        return out
    w0 = st["weight_now"]
    rows = torch.arange(T, device=w0.device) < st["len"][:, None, None]
    return out, torch.where(rows, w0 * case["decay"] + w, w0)


def _valid(q, new):
    return torch.arange(q.shape[1], device=q.device) < new[:, None]


def _plain_attention(q, pk, pv, k, v, lens, new):
    """In fp32: out [B, N, n_q, hd] and the own keys' weights [B, n_kv, T] of the valid tokens."""
    B, N, n_q, hd = q.shape
    n_kv, T = k.shape[1], k.shape[2]
    g = n_q // n_kv
    scale = 1.0 / math.sqrt(hd)
    rows = q.float().view(B, N, n_kv, g, hd).permute(2, 0, 1, 3, 4).contiguous()  # [n_kv, B, N, g, hd]
    own_rows = rows.transpose(0, 1).reshape(B, n_kv, N * g, hd)
    s = torch.matmul(own_rows, k.float().transpose(2, 3).contiguous()).mul_(scale).view(B, n_kv, N, g, T)
    t, i = torch.arange(T, device=q.device), torch.arange(N, device=q.device)
    keep = t <= (lens - new)[:, None, None] + i[None, :, None]               # [B, N, T]
    keep &= (t < lens[:, None, None]) & _valid(q, new)[:, :, None]
    s.masked_fill_(~keep[:, None, :, None, :], -math.inf)
    top = s.amax(-1, keepdim=True)
    if pk is not None:
        sp = torch.matmul(rows.view(n_kv, -1, hd), pk.float().transpose(1, 2).contiguous()).mul_(scale)
        sp = sp.view(n_kv, B, N, g, -1)
        top = torch.maximum(top, sp.amax(-1, keepdim=True).transpose(0, 1))
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, n_kv, N * g, T), v.float()).view(B, n_kv, N, g, hd)
    if pk is not None:
        pp = sp.sub_(top.transpose(0, 1)).exp_()
        total = total + pp.sum(-1, keepdim=True).transpose(0, 1)
        o = o + torch.matmul(pp.view(n_kv, B * N * g, -1), pv.float()).view(n_kv, B, N, g, hd).transpose(0, 1)
    inv = torch.where(total > 0, 1.0 / total, torch.zeros_like(total))
    w = (p * inv).sum((2, 3))
    return (o * inv).permute(0, 2, 1, 3, 4).reshape(B, N, n_q, hd), w


def _plain_evict(k, v, weight, pos, lens, last, keep, sink, recent):
    B, n_kv, T, hd = k.shape
    slot = torch.arange(T, device=k.device).expand(B, n_kv, T)
    n = lens.long()[:, None, None]
    left = n.clamp(max=keep)
    rank_by = torch.where(torch.isnan(weight), -math.inf, weight.double())
    fixed = (pos < sink) | (pos > last[:, None, None] - recent)
    rank_by = torch.where(fixed, math.inf, rank_by)
    rank_by = torch.where(slot < n, rank_by, -math.inf)
    order = rank_by.sort(dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(2, order, slot)
    kept = (rank < left) & (slot < n)
    hole, mover = ~kept & (slot < left), kept & (slot >= left)
    movers = torch.where(mover, slot, T).sort(-1).values                     # the moving rows' slots in order
    nth = (hole.long().cumsum(-1) - 1).clamp(min=0)
    src = torch.where(hole, movers.gather(2, nth), slot)
    rows = src[..., None].expand(B, n_kv, T, hd)
    w2 = torch.where((slot >= left) & (slot < n), torch.zeros_like(weight), weight.gather(2, src))
    return k.gather(2, rows), v.gather(2, rows), w2, pos.gather(2, src), left.view(B).to(lens.dtype)


# ---------------------------------------------------------------- cost and accuracy

def work(case):
    """Bytes: keys, values, queries and weights that take part read once, what changes written once.  Flops of
    attention: one multiply-add for every element of a query and a key, one for every element of a weighted value."""
    n_q, n_kv, hd, _, dt = MODELS[case["model"]]
    e = 2 if dt == torch.bfloat16 else 4
    lens, news = _lengths(case, 0)  # another seed's lengths have the same mean
    if case["ragged"]:
        mean = (max(1, case["T"] // 2) + case["T"]) / 2
        lens = [mean] * (case["B"] - 1) + [case["T"]]
        news = [min(case.get("N", 1), n) for n in lens]
    rows = sum(lens)
    if case["op"] == "evict":
        gone = sum(max(0, n - case["keep"]) for n in lens)
        # rows that move: as many as are kept beyond the kept count, a share keep / n of those
        moved = sum(max(0, n - case["keep"]) * min(n, case["keep"]) / n for n in lens)
        return {"bytes": round(n_kv * (8 * rows + 4 * gone + moved * (4 * hd * e + 16)) + 8 * case["B"]), "flops": 0}
    pairs = sum(m * (case["prefix"] + n) - m * (m - 1) / 2 for n, m in zip(lens, news))
    byts = e * (2 * (rows + case["prefix"]) * n_kv * hd + 2 * sum(news) * n_q * hd)
    if case["weights"]:
        byts += 4 * n_kv * rows * (1 if case["decay"] == 0.0 else 2)
    return {"bytes": round(byts), "flops": round(4 * hd * n_q * pairs)}


def exact(case, seed):
    x = _tensors(case, seed)
    if case["op"] == "evict":
        return _exact_evict(case, x)
    n_q, n_kv, hd, _, _ = MODELS[case["model"]]
    B, N, T = case["B"], case["N"], case["T"]
    lens, news = _lengths(case, seed)
    out = torch.zeros((B, N, n_q, hd), dtype=torch.float64, device="cuda")
    weight = x["weight"].double().clone()
    for b in range(B):
        n, m = lens[b], news[b]
        if case["weights"]:
            weight[b, :, :n] *= case["decay"]
        for h in range(n_q):
            j = h * n_kv // n_q
            keys, vals = x["k"][b, j, :n].double(), x["v"][b, j, :n].double()
            if case["op"] == "prefix":
                keys, vals = torch.cat((x["pk"][j].double(), keys)), torch.cat((x["pv"][j].double(), vals))
            s = x["q"][b, :m, h].double() @ keys.t() / hd ** 0.5
            if m > 1:  # token i of m does not see the m - 1 - i tokens behind it
                behind = torch.ones((m, m), dtype=torch.bool, device="cuda").triu(1)
                s[:, s.shape[1] - m:][behind] = -math.inf
            p = torch.softmax(s, -1)
            out[b, :m, h] = p @ vals
            if case["weights"]:
                weight[b, j, :n] += p[:, p.shape[1] - n:].sum(0)
    return (out, weight) if case["weights"] else out


def _exact_evict(case, x):
    """Row by row from the definition: who stays, then who moves where."""
    lens, _ = _lengths(case, 0)
    k, v, w, pos = x["k"].clone(), x["v"].clone(), x["weight"].clone(), x["pos"].clone()
    lens, last = x["len"].tolist(), x["last"].tolist()
    weights, positions = x["weight"].cpu().tolist(), x["pos"].cpu().tolist()
    for b, n in enumerate(lens):
        left = min(n, case["keep"])
        for j in range(k.shape[1]):
            def place(t):
                p, a = positions[b][j][t], weights[b][j][t]
                stays = p < case["sink"] or p > last[b] - case["recent"]
                return (0 if stays else 1, 0.0 if stays else -a, t)
            kept = set(sorted(range(n), key=place)[:left])
            to = [t for t in range(left) if t not in kept]
            at = sorted(t for t in kept if t >= left)
            if to:
                d, s = torch.tensor(to, device="cuda"), torch.tensor(at, device="cuda")
                for a in (k, v, w, pos):
                    a[b, j, d] = a[b, j, s]
            w[b, j, left:n] = 0.0
    return (k.double(), v.double(), w.double(), pos, x["len"].clamp(max=case["keep"]))
