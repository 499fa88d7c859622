"""budget.WeightedCache on the CPU, its calls replaced by ones that record or refuse: what the cache claims to hold."""
import contextlib
import types

import pytest
import torch

pytest.importorskip("paper_2603_19664_amd.kvd")
from paper_2603_19664_amd import kvd
from paper_2603_19664_amd.budget import WeightedCache

S = kvd.Shape(512, 8, 4, 64, 1e-6, 1e4, kvd.KVD_BF16)


class Calls:
    """Stands in for the binding: records the calls' names; those in `refuse` raise."""

    def __init__(self, refuse=()):
        self.refuse, self.names, self.seen = set(refuse), [], []

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return getattr(kvd, name)

        def call(*args, **kw):
            self.names.append(name)
            self.seen.append((name, args, kw))
            if name in self.refuse:
                raise ValueError(name)
        return call


def cache(budget=6, room=3, refuse=(), **kw):
    c = WeightedCache(S, 2, budget, room=room, device="cpu", **kw)
    c.kvd = Calls(refuse)
    return c


def x(*dims):
    return torch.zeros(dims, dtype=torch.bfloat16)


def step(c):
    c.step(x(2, 512), None, None, None, None, x(2, 8, 64))


def held(c):
    return c.n, c.T, c.last_pos.tolist()


def test_steps_advance():
    c = cache()
    for i in range(9):
        step(c)
        assert held(c)[1:] == (i + 1, [i, i])
    assert c.n == 6 and c.kvd.names.count("kvd_evict") == 1
    last = [a for n, a, _ in c.kvd.seen if n == "kvd_prefix_attn"][-1]
    assert last[7] == 9  # rows attended: the new token's among them


@pytest.mark.parametrize("refuse", ["kvd_project_qkv", "kvd_prefix_attn"])
def test_a_refused_step_leaves_the_cache_as_it_was(refuse):
    c = cache()
    for _ in range(2):
        step(c)
    before = held(c)
    c.kvd.refuse = {refuse}
    for _ in range(20):  # more than there is room
        with pytest.raises(ValueError, match=refuse):
            step(c)
        assert held(c) == before
    c.kvd.refuse = set()
    step(c)
    assert held(c) == (3, 3, [2, 2])


@pytest.mark.parametrize("refuse", ["kvd_project_q", "kvd_recompute_kv", "kvd_prefix_attn"])
def test_a_refused_chunk_leaves_the_cache_as_it_was(refuse):
    c = cache()
    c.prompt(x(2, 3, 512), None, None, None, None, x(2, 3, 8, 64))
    before = held(c)
    c.kvd.refuse = {refuse}
    with pytest.raises(ValueError, match=refuse):
        c.prompt(x(2, 3, 512), None, None, None, None, x(2, 3, 8, 64))
    assert held(c) == before == (3, 3, [2, 2])


@pytest.mark.parametrize("h,out", [((2, 7, 512), (2, 6, 8, 64)), ((2, 7, 512), (2, 7, 8, 1)), ((1, 7, 512), (1, 7, 8, 64)),
                                   ((2, 7, 511), (2, 7, 8, 64)), ((2, 7, 512), (1, 7, 8, 64))])
def test_prompts_of_other_sizes_are_refused_before_any_call(h, out):
    c = cache()
    with pytest.raises(ValueError, match="has shape"):
        c.prompt(x(*h), None, None, None, None, x(*out))
    assert held(c) == (0, 0, [0, 0]) and c.kvd.names == []


def test_calls_are_made_on_the_cache_s_device():
    # the current device is 0, the cache's 1: every call is made while its own is current
    c = cache()
    current = []

    @contextlib.contextmanager
    def device(dev):
        current.append(dev.index)
        yield
        current.pop()

    there = torch.device("cuda", 1)
    cuda = types.SimpleNamespace(current_device=lambda: 0, device=device)
    here = WeightedCache._here
    c._here = lambda: here(types.SimpleNamespace(k=types.SimpleNamespace(device=there),
                                                 torch=types.SimpleNamespace(cuda=cuda)))
    calls = []
    make = c.kvd.__getattr__
    c.kvd = types.SimpleNamespace(**{n: (lambda n: lambda *a, **kw: (calls.append((n, list(current))), make(n)(*a, **kw)))(n)
                                     for n in ("kvd_project_qkv", "kvd_project_q", "kvd_recompute_kv", "kvd_prefix_attn",
                                               "kvd_evict")},
                                  kvd_prefix_workspace_bytes=kvd.kvd_prefix_workspace_bytes)
    c.prompt(x(2, 7, 512), None, None, None, None, x(2, 7, 8, 64))
    for _ in range(4):
        step(c)
    assert {n for n, _ in calls} == {"kvd_project_qkv", "kvd_project_q", "kvd_recompute_kv", "kvd_prefix_attn", "kvd_evict"}
    assert all(at == [1] for _, at in calls) and current == []
    cuda.current_device = lambda: 1
    with c._here():
        assert current == []
