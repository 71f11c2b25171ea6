"""The attention layer with selected blocks, shared prefixes and the residual stream, without a GPU: workspaces, and what is refused before anything runs."""
import pytest
import torch

import paper_2206_07446_amd as nnv
from paper_2206_07446_amd.attention_layer import AttentionLayer


def make(requests=3, rows=20, tokens=100, **kw):
    return AttentionLayer(256, 4, 2, 64, requests, rows, tokens, block_tokens=16, device="cpu", **kw)


@pytest.fixture
def calls(monkeypatch):
    """What a layer would have launched."""
    names = []
    for name in ("nnv_kv_plan", "nnv_linear_forward", "nnv_qk_norm_rope", "nnv_kv_attention", "nnv_kv_bounds", "nnv_kv_select", "nnv_kv_attention_blocks",
                 "nnv_kv_attention_shared", "nnv_residual_norm"):
        monkeypatch.setattr(nnv.binding, name, lambda *a, name=name, **kw: names.append(name))
    return names


@pytest.mark.parametrize("requests,rows,tokens", [(1, 700, 9000), (4, 300, 30000), (50, 60, 200)])
def test_the_workspace_holds_a_step_of_any_size(requests, rows, tokens):
    layer = make(requests, rows, tokens, keep=9)
    for m in range(1, rows + 1):
        assert max(nnv.nnv_kv_select_workspace_bytes(layer.desc, requests, m), nnv.nnv_kv_attention_blocks_workspace_bytes(layer.desc, requests, m, 9)) <= layer.workspace.numel()
    layer = make(requests, rows, tokens, groups=3)
    for m in range(1, rows + 1):
        for g in range(1, 4):
            assert nnv.nnv_kv_attention_shared_workspace_bytes(layer.desc, requests, m, g) <= layer.workspace.numel()


def test_the_attention_that_is_asked_for_runs(calls):
    x = torch.zeros(20, 256, dtype=torch.bfloat16)
    make().attend(3)
    make(keep=4).attend(3)
    layer = make(groups=2)
    layer.attend(3)
    layer.held[:] = torch.tensor([40, 0, 0], dtype=torch.int32)
    layer.share([0, 2, 3], [32, 0])
    layer.attend(3)
    assert layer.held.tolist() == [40, 32, 0] and layer.group_ends.tolist() == [0, 2, 3] and layer.shared.tolist() == [32, 0]
    layer.share([0], [])
    layer.attend(3)
    assert calls == ["nnv_kv_attention", "nnv_kv_bounds", "nnv_kv_select", "nnv_kv_attention_blocks", "nnv_kv_attention", "nnv_kv_attention_shared", "nnv_kv_attention"]
    del calls[:]
    make().step_stream(x.float(), x, 5, begin=True)
    assert calls[0] == calls[-1] == "nnv_residual_norm" and len(calls) == 7
    del calls[:]
    make().step_stream(x.float(), x, 5, gate=x.clone(), index=torch.zeros(5, dtype=torch.int32))
    assert calls[-1] == "nnv_residual_norm" and len(calls) == 6


def test_layers_that_cannot_be(calls):
    for kw in (dict(keep=4, window=9), dict(keep=4, groups=1), dict(keep=2), dict(keep=4, first=-1), dict(keep=4, first=2, last=3)):
        with pytest.raises(ValueError):
            make(**kw)


def test_groups_that_cannot_be():
    layer = make(groups=2)
    layer.held[:] = torch.tensor([40, 0, 5], dtype=torch.int32)
    for ends, tokens in (([0, 2], []), ([0, 1, 2, 3], [0, 0, 0]), ([0, 4], [16]), ([-1, 2], [16]), ([2, 0], [16]), ([0, 2], [17]), ([0, 2], [48]), ([0, 3], [16]),
                         ([0, 2], [-16]), ([1, 2], [16])):
        with pytest.raises(ValueError):
            layer.share(ends, tokens)
    assert layer.held.tolist() == [40, 0, 5] and layer.n_groups == 0
    with pytest.raises(ValueError):
        make().share([0, 2], [0])


def test_a_stream_that_does_not_fit_is_refused_before_any_call(calls):
    layer = make()
    new = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype)  # noqa: E731
    x, h = new(20, 256, dtype=torch.float32), new(20, 256)
    for bad in (new(4, 256), new(5, 255), new(5, 256, dtype=torch.float64), new(256, 5).t(), new(1280), new(1, 256).expand(5, 256), new(1281)[1:].view(5, 256), None,
                torch.zeros(5, 256, device="meta")):
        with pytest.raises(ValueError):
            layer.step_stream(bad, h, 5)
    for bad in (new(4, 256), new(5, 256, dtype=torch.float32), None):
        with pytest.raises(ValueError):
            layer.step_stream(x, bad, 5)
    for gate in (new(5, 255), new(5, 256, dtype=torch.float32), new(1280), new(256, 5).t()):
        with pytest.raises(ValueError):
            layer.step_stream(x, h, 5, gate=gate)
    for index in (new(5), torch.zeros(4, dtype=torch.int32), torch.zeros(10, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            layer.step_stream(x, h, 5, gate=new(3, 256), index=index)
    for gate in (new(4, 256), new(0, 256), new(1, 256).expand(5, 256), new(1281)[1:].view(5, 256)):                # too few, none, no rows of their own, off by two bytes
        with pytest.raises(ValueError):
            layer.step_stream(x, h, 5, gate=gate)
    with pytest.raises(ValueError):
        layer.step_stream(x, h, 5, scale=float("nan"))
    both = new(20, 512)
    for a, b, gate in ((both[:, :256], both[:, 256:], None), (h, h, None), (x, h, h)):                               # in each other's memory
        with pytest.raises(ValueError):
            layer.step_stream(a, b, 5, gate=gate)
    with pytest.raises(ValueError):
        layer.step_stream(x, h, 21)
    assert not calls
