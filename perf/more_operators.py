"""Caches held in 4 bits, and attention with a sliding window and sinks, as timed cases.

Each case is one layer's call, at the shapes of this repository's three model configurations:

  op "store"   N new tokens' keys and values of every sequence are put into a cache of 4-bit numbers (kvd_mx_store)
               and read back (kvd_mx_load): as the values that their bits stand for.
  op "mx"      N new tokens of every sequence attend its 4-bit cache (kvd_mx_attn).
  op "sink"    N new tokens attend stored keys and values in the model's type: the first `sink` tokens and the newest
               `window` of each (kvd_sink_attn).

Fields: model; B sequences; N new tokens a sequence, its last ones; T tokens a sequence at most; slots: rows of a
sequence's cache (T if 0).  A cache of fewer rows than tokens holds token t in row t below `sink` and behind that in a
ring, row sink + (t - sink) mod (slots - sink).  window: newest tokens that each new one sees (0: all), sink: first
tokens that stay visible beside them; ragged: sequences have lengths of their own, up to T, and as many new tokens, up
to N, as fit.

The 4-bit format: 32 neighbouring elements of a row share a power of two 2^E, the smallest with every |x| <= 7 2^E
(E from -100 to 125), held as E + 127 in a byte; each is held as the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 times 2^E
(ties to the even code) and a sign, two to a byte.
"""
import math

import torch

own = False  # False: the operators' plain forms; True: the library's calls

# name: query heads, KV heads, head_dim, d_model, dtype
MODELS = {"smollm": (9, 3, 64, 576, torch.float32), "gemma": (8, 4, 256, 2560, torch.bfloat16),
          "qwen": (12, 2, 128, 1536, torch.bfloat16)}
GROUP = 32
LEAST_E, MOST_E, BIAS = -100, 125, 127


def _case(op, model, B, N, T, window=0, sink=0, slots=0, ragged=False, name=None):
    c = {"op": op, "model": model, "B": B, "N": N, "T": T, "window": window, "sink": sink, "slots": slots,
         "ragged": ragged}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # a decode step's new rows of a serving batch, into the ring of a windowed cache
        _case("store", "qwen", 32, 1, 50001, sink=4, slots=2052, name="qwen_mx_store_step_b32"),
        # prompts of different lengths
        _case("store", "gemma", 4, 2001, 2001, ragged=True, name="gemma_mx_store_prompts_b4"),
        # two tokens of the small fp32 model: the smallest attention call
        _case("mx", "smollm", 2, 1, 257, name="smollm_mx_step_fp32"),
        # a decode step over long contexts, which the 4 bits are for
        _case("mx", "gemma", 8, 1, 32768, name="gemma_mx_step_b8_32k"),
        # a decode step of a large serving batch, conversations of different lengths
        _case("mx", "qwen", 64, 1, 8192, ragged=True, name="qwen_mx_step_b64"),
        # drafted continuations checked in one call, with a window and sinks
        _case("mx", "gemma", 16, 5, 4099, window=2048, sink=4, ragged=True, name="gemma_mx_draft_b16"),
        # questions of up to 256 tokens behind long cached documents
        _case("mx", "qwen", 8, 256, 8448, ragged=True, name="qwen_mx_prompts_b8"),
        # one token of the small fp32 model in an endless stream
        _case("sink", "smollm", 1, 1, 1001, window=128, sink=4, slots=132, name="smollm_sink_step_fp32"),
        # a decode step of a large batch of endless streams
        _case("sink", "gemma", 64, 1, 100003, window=1024, sink=4, slots=1028, name="gemma_sink_step_b64"),
        # a whole long prompt of a sliding-window layer
        _case("sink", "gemma", 1, 8192, 8192, window=1024, sink=4, name="gemma_sink_prompt_8k"),
        # prompts of different lengths
        _case("sink", "qwen", 4, 2501, 2501, window=512, sink=16, ragged=True, name="qwen_sink_prompts_b4"),
        # the next part of two long prompts, into rings that it passes the end of
        _case("sink", "qwen", 2, 512, 20011, window=4096, sink=4, slots=4611, name="qwen_sink_part_b2"),
    ]


def draw(rng):
    """One more call of the same ranges: single tokens, drafts and prompts, whole caches and rings."""
    def logint(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    op = rng.choice(["store", "mx", "mx", "sink", "sink"])
    model = rng.choice(["smollm", "gemma", "gemma", "qwen", "qwen"])
    small = model == "smollm"
    ragged = rng.random() < 0.5
    kind = rng.choice(["step", "step", "draft", "prompt"])
    sink = rng.choice([0, 1, 4, 16, 40])
    if op == "store":
        N = 1 if kind == "step" else rng.randint(2, 32) if kind == "draft" else logint(33, 2001)
        B = logint(1, max(1, min(64, (2001 if small else 8004) // N)))
        if rng.random() < 0.5:
            return _case(op, model, B, N, N + logint(1, 2000), ragged=ragged)
        slots = sink + N + logint(1, 4096)
        return _case(op, model, B, N, slots + logint(1, 100000), sink=sink, slots=slots, ragged=ragged)
    if kind == "prompt":
        N = logint(33, 1024 if small else 2501)
        B = logint(1, max(1, (1024 if small else 2501) // N))
        window = logint(16, 1024 if small else 4096)
        whole = N + (0 if rng.random() < 0.5 else logint(1, 4000))
    else:
        N = 1 if kind == "step" else rng.randint(2, 32)
        B = logint(1, 4 if small else max(1, 64 // N))
        window = logint(16, 2048 if small else 4096)
        whole = N + logint(1, (8192 if small else 65536) // B)
    window = min(window, 65536 // B)
    layout = rng.choice(["whole", "window", "ring"])
    if layout == "whole" and op == "mx":
        return _case(op, model, B, N, whole, ragged=ragged)
    if layout != "ring":
        return _case(op, model, B, N, whole, window, sink, ragged=ragged)
    slots = sink + window + N - 1 + rng.choice([0, 0, 1, 64])
    return _case(op, model, B, N, slots + logint(1, 100000), window, sink, slots, ragged)


# ---------------------------------------------------------------- inputs

def _slots(case):
    return case["slots"] or case["T"]


def _window(case):
    return case["window"] or case["T"]


def _lengths(case, seed):
    """Tokens and new tokens of every sequence, host numbers: ragged lengths lie between half of T and T."""
    B, T, N = case["B"], case["T"], case["N"]
    if not case["ragged"]:
        return [T] * B, [N] * B
    gen = torch.Generator()
    gen.manual_seed(seed * 2 + 1)
    lens = torch.randint(max(1, T // 2), T + 1, (B,), generator=gen).tolist()
    lens[-1] = T
    return lens, [min(N, n) for n in lens]


def _tensors(case, seed):
    """Queries and values N(0, 1); keys too, with channels of different sizes (log-normal), as projections leave them."""
    n_q, n_kv, hd, _, dt = MODELS[case["model"]]
    B, N = case["B"], case["N"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)

    lens, news = _lengths(case, seed)
    x = {"len": torch.tensor(lens, dtype=torch.int32, device="cuda"),
         "new": torch.tensor(news, dtype=torch.int32, device="cuda")}
    channel = torch.exp(0.4 * normal((n_kv, 1, hd)))
    channel /= channel.square().mean(-1, keepdim=True).sqrt()
    if case["op"] == "store":
        x["k"], x["v"] = (normal((B, n_kv, N, hd)) * channel).to(dt), normal((B, n_kv, N, hd)).to(dt)
        return x
    x["q"] = normal((B, N, n_q, hd)).to(dt)
    C = _slots(case)
    if case["op"] == "sink":
        x["k"], x["v"] = (normal((B, n_kv, C, hd)) * channel).to(dt), normal((B, n_kv, C, hd)).to(dt)
        return x
    for name in ("k", "v"):
        codes = torch.empty((B, n_kv, C, hd // 2), dtype=torch.uint8, device="cuda")
        scale = torch.empty((B, n_kv, C, hd // GROUP), dtype=torch.uint8, device="cuda")
        for b in range(B):
            rows = normal((n_kv, C, hd))
            codes[b], scale[b] = _pack((rows * channel if name == "k" else rows).to(dt))
        x[name], x[name + "_scale"] = codes, scale
    return x


def prepare(case, seed):
    st = {"case": case, **_tensors(case, seed)}
    n_q, n_kv, hd, d, dt = MODELS[case["model"]]
    B, N, T, C = case["B"], case["N"], case["T"], _slots(case)
    if case["op"] == "store":
        for name in ("k", "v"):
            st[name + "_codes"] = torch.zeros((B, n_kv, C, hd // 2), dtype=torch.uint8, device="cuda")
            st[name + "_scale"] = torch.zeros((B, n_kv, C, hd // GROUP), dtype=torch.uint8, device="cuda")
            st[name + "_read"] = torch.zeros((B, n_kv, N, hd), dtype=dt, device="cuda")
    else:
        st["out"] = torch.zeros_like(st["q"])
    if own:
        from paper_2603_19664_amd import kvd
        s = kvd.Shape(d, n_q, n_kv, hd, 1e-6, 1e4, kvd.KVD_BF16 if dt == torch.bfloat16 else kvd.KVD_F32)
        st["kvd"], st["s"] = kvd, s
        if case["op"] == "store":
            st["cache"] = kvd.MxCache(st["k_codes"], st["v_codes"], st["k_scale"], st["v_scale"])
        else:
            if case["op"] == "mx":
                st["cache"] = kvd.MxCache(st["k"], st["v"], st["k_scale"], st["v_scale"])
            size = kvd.kvd_sink_workspace_bytes(s, B, N, T, _window(case), case["sink"])
            st["ws"] = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
    return st


# ---------------------------------------------------------------- one pass

def run(st):
    case = st["case"]
    op, N, T, sink = case["op"], case["N"], case["T"], case["sink"]
    if own:
        kvd, s = st["kvd"], st["s"]
        lens, new = (st["len"], st["new"]) if case["ragged"] else (None, None)
        if op == "store":
            kvd.kvd_mx_store(s, st["k"], st["v"], N, st["cache"], T, sink=sink, kv_len=lens, n_new=new)
            kvd.kvd_mx_load(s, st["cache"], T, N, st["k_read"], st["v_read"], sink=sink, kv_len=lens, n_new=new)
            return st["k_read"], st["v_read"]
        if op == "mx":
            kvd.kvd_mx_attn(s, st["q"], st["cache"], T, st["out"], st["ws"], window=_window(case), sink=sink, kv_len=lens,
                            n_new=new)
        else:
            kvd.kvd_sink_attn(s, st["q"], st["k"], st["v"], T, _window(case), st["out"], st["ws"], sink=sink,
                              kv_len=lens, n_new=new)
        return st["out"]
    if op == "store":
        return _plain_store(st)
    k, v = st["k"], st["v"]
    if op == "mx":
        k, v = _unpack(k, st["k_scale"]), _unpack(v, st["v_scale"])
    return _plain_attention(st["q"], k.float(), v.float(), st["len"].long(), st["new"].long(), T, _window(case), sink)


def _pack(x):
    """Codes and scales of rows x [.., hd]: every step exact in 32 bits, powers of two and sums of few bits."""
    g = x.float().unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)                                  # top = m 2^e, 1/2 <= m < 1: 7 2^E = 7/8 2^(E + 3)
    e = torch.where(top > 0, e - 3 + (m > 0.875), LEAST_E).clamp(LEAST_E, MOST_E)
    y = torch.ldexp(g, -e).abs().clamp_max(6.0)
    step = torch.where(y < 2.0, 0.5, torch.where(y < 4.0, 1.0, 2.0))
    r = torch.round(y / step) * step                         # ties to even multiples are ties to even codes
    code = torch.where(r <= 2.0, 2.0 * r, torch.where(r <= 4.0, r + 2.0, 7.0)).to(torch.uint8)
    code |= torch.signbit(g).to(torch.uint8) << 3
    code = code.flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + BIAS).squeeze(-1).to(torch.uint8)


def _unpack(codes, scale):
    both = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    size = (both & 7).float()
    size = torch.where(size < 4.0, 0.5 * size, torch.where(size < 6.0, size - 2.0, 2.0 * size - 8.0))
    size = torch.where(both >= 8, -size, size)
    return (size.unflatten(-1, (-1, GROUP)) * torch.exp2(scale.float() - BIAS)[..., None]).flatten(-2)


def _rows_of(case, lens, news):
    """The new tokens' cache rows [B, N], and which of them are there."""
    N, C, sink = case["N"], _slots(case), case["sink"]
    i = torch.arange(N, device=lens.device)
    t = lens[:, None] - news[:, None] + i
    there = (i < news[:, None]) & (t >= 0)
    row = t if case["T"] <= C else torch.where(t < sink, t, sink + (t - sink) % max(C - sink, 1))
    return row.clamp(min=0), there


def _plain_store(st):
    row, there = _rows_of(st["case"], st["len"].long(), st["new"].long())
    b, i = there.nonzero(as_tuple=True)
    row = row[b, i]
    read = []
    for name in ("k", "v"):
        codes, scale = _pack(st[name][b, :, i])
        st[name + "_codes"][b, :, row], st[name + "_scale"][b, :, row] = codes, scale
        back = torch.zeros_like(st[name])
        back[b, :, i] = _unpack(st[name + "_codes"][b, :, row], st[name + "_scale"][b, :, row]).to(back.dtype)
        read.append(back)
    return tuple(read)


def _plain_attention(q, k, v, lens, news, T, window, sink):
    B, N, n_q, hd = q.shape
    n_kv, C = k.shape[1], k.shape[2]
    g = n_q // n_kv
    slot, i = torch.arange(C, device=q.device), torch.arange(N, device=q.device)
    last = lens[:, None] - 1
    tok = slot.expand(B, C)                                  # the token in every row, -1 in a row that holds none
    if T > C:
        tok = torch.where((slot >= sink) & (slot <= last), slot + (last - slot) // (C - sink) * (C - sink), tok)
    tok = torch.where(tok <= last, tok, -1)[:, None]
    at = (lens - news)[:, None, None] + i[:, None]           # the new tokens' positions [B, N, 1]
    seen = (tok >= 0) & (tok <= at) & ((tok < sink) | (tok > at - window))
    rows = q.float().view(B, N, n_kv, g, hd).transpose(1, 2).reshape(B, n_kv, N * g, hd)
    s = torch.matmul(rows, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(hd)).view(B, n_kv, N, g, C)
    s.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, n_kv, N * g, C), v).view(B, n_kv, N, g, hd)
    o = torch.where(total > 0, o / total, 0.0).transpose(1, 2).reshape(B, N, n_q, hd)
    return torch.where((i < news[:, None])[:, :, None, None], o, 0.0).to(q.dtype)


# ---------------------------------------------------------------- cost and accuracy

def work(case):
    """Bytes: keys, values and queries that take part read once, what changes written once; a stored row is written
    in 4 bits and read back.  Flops of attention: one multiply-add for every element of a query and a key that it
    sees, one for every element of a weighted value."""
    n_q, n_kv, hd, _, dt = MODELS[case["model"]]
    e = 2 if dt == torch.bfloat16 else 4
    B, T, N, window, sink = case["B"], case["T"], case["N"], _window(case), case["sink"]
    lens = [T] * B
    if case["ragged"]:  # another seed's lengths have the same mean
        lens = [(max(1, T // 2) + T) // 2] * (B - 1) + [T]
    held = hd // 2 + hd // GROUP
    byts = flops = 0
    for n in lens:
        m = min(N, n)
        if case["op"] == "store":
            byts += 2 * n_kv * m * (2 * hd * e + 2 * held)
            continue
        first = max(n - m - window + 1, 0)                   # the window of the first new token
        rows = n - first + min(sink, first)
        byts += 2 * n_kv * rows * (held if case["op"] == "mx" else hd * e) + 2 * m * n_q * hd * e
        flops += 4 * hd * n_q * sum(min(p + 1, window + min(sink, max(p + 1 - window, 0))) for p in range(n - m, n))
    return {"bytes": byts, "flops": flops}


def exact(case, seed):
    x = _tensors(case, seed)
    n_q, n_kv, hd, _, _ = MODELS[case["model"]]
    B, N, T, C, window, sink = case["B"], case["N"], case["T"], _slots(case), _window(case), case["sink"]
    lens, news = _lengths(case, seed)
    if case["op"] == "store":
        read = []
        for name in ("k", "v"):
            back = torch.zeros(x[name].shape, dtype=torch.float64, device="cuda")
            for b in range(B):
                back[b, :, :news[b]] = _exact_held(x[name][b, :, :news[b]])
            read.append(back)
        return tuple(read)
    out = torch.zeros((B, N, n_q, hd), dtype=torch.float64, device="cuda")
    sizes = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64,
                         device="cuda")
    for b in range(B):
        n, m = lens[b], news[b]
        # the tokens that some new one sees, and their rows
        t = torch.tensor([u for u in range(max(n - m - window + 1, 0), n)], device="cuda")
        t = torch.cat((torch.arange(min(sink, int(t[0])), device="cuda"), t))
        row = t if T <= C else torch.where(t < sink, t, (t - sink) % max(C - sink, 1) + sink)
        at = torch.arange(n - m, n, device="cuda")[:, None]
        hidden = (t > at) | ((t <= at - window) & (t >= sink))
        for j in range(n_kv):
            kv = []
            for name in ("k", "v"):
                rows = x[name][b, j, row]
                if case["op"] == "mx":
                    codes = rows.long()
                    rows = torch.stack((sizes[codes % 16], sizes[codes // 16]), -1).view(len(row), hd)
                    scale = 2.0 ** (x[name + "_scale"][b, j, row].double() - BIAS)
                    rows = rows * scale.repeat_interleave(GROUP, 1)
                kv.append(rows.double())
            for h in range(j * n_q // n_kv, (j + 1) * n_q // n_kv):
                s = x["q"][b, :m, h].double() @ kv[0].t() / hd ** 0.5
                s[hidden] = -math.inf
                out[b, :m, h] = torch.softmax(s, -1) @ kv[1]
    return out


def _exact_held(x):
    """The values that rows x are held as: every element against each of the eight sizes."""
    g = x.double().reshape(-1, GROUP)
    top = g.abs().amax(1)
    E = torch.full_like(top, LEAST_E)
    for e in range(LEAST_E, MOST_E):
        E += (top > 7.0 * 2.0 ** e).double()
    y = g / 2.0 ** E[:, None]
    best, held = torch.full_like(y, math.inf), torch.zeros_like(y)
    for size in (0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0):    # even codes first: they win ties
        away = (y.abs() - size).abs()
        held = torch.where(away < best, size, held)
        best = torch.minimum(best, away)
    return (held * torch.sign(y) * 2.0 ** E[:, None]).view(x.shape)
