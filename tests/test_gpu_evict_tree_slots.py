"""What slots weigh that a tree has committed: no call writes their entries, the caller does before they are ranked."""
import pytest
import torch

from test_gpu_evict import DEV, Setup

pytestmark = pytest.mark.gpu


def commit_tree(s, seq, B, path):
    """A tree of B nodes of which `path` is accepted."""
    assert s.sim.reserve([seq], [B]) == 0
    P = int(s.sim.len[seq])
    s.ctx.goose_pages_reserve(s.cache, [seq], [B])
    s.sim.commit([seq], [path])
    i32 = dict(dtype=torch.int32, device=DEV)
    s.ctx.goose_pages_commit(s.cache, [{"seq": seq, "B": B, "P_max": P, "path": torch.tensor(path + [0] * (B - len(path)), **i32),
                                        "accept_len": torch.tensor([len(path) - 1], **i32)}])
    assert s.ctx.goose_device_flags() == 0


@pytest.mark.parametrize("value", [0.0, float("inf")])
def test_a_second_cut_after_trees_goes_by_what_the_caller_wrote(value):
    s = Setup([300, 90], seed=41, spare=8)
    ev = [{"seq": 0, "keep": 200, "sink": 4, "recent": 10}]
    s.evict(ev, reposition=False)
    # behind the kept slots the entries are still those of slots that have moved or gone, and a commit leaves them so
    left = s.weight[:, 0, :, 200:206].clone()
    assert (left > 0).all()
    commit_tree(s, 0, 8, [0, 2, 3])
    commit_tree(s, 0, 8, [0, 1, 7])
    s.check()
    assert int(s.cache.len[0]) == 206 and torch.equal(s.weight[:, 0, :, 200:206], left)
    # written by the caller: lightest or heaviest of all
    for w in (s.weight, s.w):
        w[:, 0, :, 200:206] = value
    words = s.evict([{"seq": 0, "keep": 202, "sink": 4}], reposition=False)
    bits = (words[0].unsqueeze(-1) >> torch.arange(64)) & 1
    new = bits.reshape(s.layers, s.nkv, -1)[..., 200:206]
    assert (new == torch.tensor([1, 1, 0, 0, 0, 0] if value == 0.0 else [1] * 6)).all()
