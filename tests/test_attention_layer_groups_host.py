"""Groups of requests that are given, added to and taken away while requests run, without a GPU: every request keeps the blocks that it began behind, whatever the groups say."""
import pytest
import torch

import paper_2206_07446_amd as nnv
from paper_2206_07446_amd.attention_layer import AttentionLayer


def running():
    """Six requests, blocks of 16 tokens: the first holds 40 tokens, the fourth 20."""
    layer = AttentionLayer(256, 4, 2, 64, 6, 20, 100, block_tokens=16, device="cpu", groups=2)
    layer.held[:] = torch.tensor([40, 0, 0, 20, 0, 0], dtype=torch.int32)
    layer.table[0, :3], layer.table[3, :2] = (torch.tensor(blocks, dtype=torch.int32) for blocks in ([5, 9, 2], [7, 11]))
    return layer


def test_requests_keep_the_prefix_that_they_began_behind():
    layer = running()
    layer.share([0, 3], [32])
    assert layer.held.tolist() == [40, 32, 32, 20, 0, 0]
    layer.share([3, 6], [16])                                # the requests before these run on behind theirs
    assert layer.held.tolist() == [40, 32, 32, 20, 16, 16]
    for groups in ([[0], []], [[0, 3, 6], [32, 16]], [[0, 3], [16]], [[1, 3, 6], [32, 16]], [[4, 6], [16]]):
        layer.share(*groups)
        assert layer.held.tolist() == [40, 32, 32, 20, 16, 16]
        assert layer.table[:, :4].tolist() == [[5, 9, 2, -1], [5, 9, -1, -1], [5, 9, -1, -1], [7, 11, -1, -1], [7, -1, -1, -1], [7, -1, -1, -1]]


def test_groups_that_a_captured_step_reads():
    """As many groups as there were when it was captured: what lies behind the present ones is of no request."""
    layer = running()
    assert layer.group_ends.tolist() == [0, 0, 0] and layer.shared.tolist() == [0, 0]
    for ends, tokens, all_ends, all_tokens in (([0, 3, 6], [32, 16], [0, 3, 6], [32, 16]), ([0, 3], [32], [0, 3, 3], [32, 0]), ([0], [], [0, 0, 0], [0, 0])):
        layer.share(ends, tokens)
        assert layer.group_ends.tolist() == all_ends and layer.shared.tolist() == all_tokens and layer.n_groups == len(tokens)


def test_requests_that_are_behind_something_else():
    layer = running()
    layer.share([0, 3], [32])
    before = layer.held.tolist(), layer.table.tolist(), layer.group_ends.tolist()
    for ends, tokens in (([0, 4], [32]), ([0, 4], [16]), ([2, 4], [16])):                                    # the fourth holds blocks of its own
        with pytest.raises(ValueError):
            layer.share(ends, tokens)
    assert (layer.held.tolist(), layer.table.tolist(), layer.group_ends.tolist()) == before
    layer.held[0], layer.table[0, 3] = 60, 3
    with pytest.raises(ValueError):
        layer.share([0, 2], [48])                            # the second holds 32
    layer.held[1], layer.table[1, 2] = 50, 8
    with pytest.raises(ValueError):
        layer.share([0, 2], [48])                            # and then another third block
    layer.share([0, 2], [32])
    layer.held[4:], layer.table[3] = 16, -1                  # entries that are no block are nobody's prefix
    with pytest.raises(ValueError):
        layer.share([3, 5], [16])


def test_layers_without_groups_share_nothing(monkeypatch):
    layer = AttentionLayer(256, 4, 2, 64, 6, 20, 100, block_tokens=16, device="cpu")
    layer.share([0], [])
    names = []
    for name in ("nnv_kv_attention", "nnv_kv_attention_shared"):
        monkeypatch.setattr(nnv.binding, name, lambda *a, name=name: names.append(name))
    layer.attend(3)
    assert names == ["nnv_kv_attention"]


def test_the_first_request_of_a_group_may_end():
    """Its place is used again: the group is refused as it was, and given with another that runs behind the same blocks."""
    layer = running()
    layer.share([0, 3], [32])
    layer.held[0] = 0
    with pytest.raises(ValueError):
        layer.share([0, 3], [32])
    layer.held[0], layer.table[0, :3] = 40, torch.tensor([1, 4, 6], dtype=torch.int32)
    with pytest.raises(ValueError):
        layer.share([0, 3], [32])
    layer.share([1, 3], [32])
    assert layer.group_ends.tolist() == [1, 3, 3] and layer.held.tolist() == [40, 32, 32, 20, 0, 0]
    assert layer.table[:3, :3].tolist() == [[1, 4, 6], [5, 9, -1], [5, 9, -1]]
