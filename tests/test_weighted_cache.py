"""budget.WeightedCache on the CPU: its refusals and the sizes of its state."""
import pytest


def test_weighted_cache_refuses_what_cannot_fit():
    pytest.importorskip("paper_2603_19664_amd.kvd")
    from paper_2603_19664_amd import kvd
    from paper_2603_19664_amd.budget import WeightedCache
    s = kvd.Shape(512, 8, 4, 64, 1e-6, 1e4, kvd.KVD_BF16)
    for kw in (dict(budget=0), dict(budget=4, room=0), dict(budget=4, sink=3, recent=2), dict(budget=4, sink=-1),
               dict(budget=4, recent=-1)):
        with pytest.raises(ValueError):
            WeightedCache(s, 2, device="cpu", **kw)
    c = WeightedCache(s, 2, 10, room=3, device="cpu")
    assert c.k.shape == (2, 4, 13, 64) and c.n == 0 and c.T_prefix == 0
    assert c.ws.numel() >= kvd.kvd_prefix_workspace_bytes(s, 2, 3, 0, 13, True)
    assert c.ws.numel() >= kvd.kvd_evict_workspace_bytes(s, 2, 13)
