"""The attention layer of attention_layer.py without a GPU: what it allocates holds every step that it may be asked for."""
import pytest
import torch

import paper_2206_07446_amd as nnv
from paper_2206_07446_amd.attention_layer import AttentionLayer

# hidden, query heads, key heads, head size, requests, rows, tokens
SHAPES = [(4096, 32, 8, 128, 1, 1024, 8192), (4096, 32, 8, 128, 2, 1024, 2048), (4096, 32, 8, 128, 4, 2048, 8192), (512, 8, 8, 64, 1, 1024, 16384),
          (6144, 2, 1, 64, 3, 800, 300), (256, 4, 2, 64, 50, 20, 100), (512, 4, 1, 256, 7, 1500, 70000)]


def make(hidden, q, kv, dim, requests, rows, tokens, **kw):
    return AttentionLayer(hidden, q, kv, dim, requests, rows, tokens, device="cpu", **kw)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_the_workspace_holds_a_step_of_any_size(shape):
    layer = make(*shape)
    have, requests, rows = layer.workspace.numel(), *shape[4:6]
    short = [m for m in range(1, rows + 1) if max(nnv.nnv_kv_attention_workspace_bytes(layer.desc, requests, m), nnv.nnv_linear_workspace_bytes(layer.qkv_desc, m),
                                                  nnv.nnv_linear_workspace_bytes(layer.out_desc, m)) > have]
    assert not short, f"{len(short)} sizes, {short[0]} to {short[-1]}"


@pytest.mark.parametrize("tokens,block", [(100, 64), (120, 16), (128, 64), (1, 256)])
def test_every_position_that_the_plan_admits_has_its_angles(tokens, block):
    """A request is held in whole blocks, and so is what the plan lets in; a position behind the rotation table would be counted but not held."""
    layer = make(256, 4, 2, 64, 3, 20, tokens, block_tokens=block)
    capacity = layer.desc.table_blocks * layer.desc.block_tokens
    assert capacity >= tokens and layer.desc.positions >= capacity and layer.rope.shape == (layer.desc.positions, 64)
    last = torch.arange(32, dtype=torch.float64) / 32
    want = (capacity - 1) * 10000.0 ** -last
    assert torch.equal(layer.rope[capacity - 1], torch.cat((want.cos(), want.sin())).float())


@pytest.fixture
def calls(monkeypatch):
    """What a layer would have launched."""
    names = []
    for name in ("nnv_kv_plan", "nnv_linear_forward", "nnv_qk_norm_rope", "nnv_kv_attention", "nnv_linear_transform_weights"):
        monkeypatch.setattr(nnv.binding, name, lambda *a, name=name, **kw: names.append(name))
    return names


def test_a_step_within_the_layers_buffers_runs(calls):
    layer, x = make(256, 4, 2, 64, 3, 20, 100), torch.zeros(20, 256, dtype=torch.bfloat16)
    for rows in (0, 1, 20):
        layer.step(x, torch.zeros(rows, 300, dtype=torch.bfloat16)[:, :256], rows)
    layer.step(x, x, 5)
    assert len(calls) == 20
    layer.transform_weights(torch.zeros(512, 256), torch.zeros(256, 256))
    assert len(calls) == 22


def test_a_step_outside_the_layers_buffers_is_refused_before_any_call(calls):
    layer = make(256, 4, 2, 64, 3, 20, 100)
    new = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype)  # noqa: E731
    x = new(30, 256)
    for rows in (21, 30, -1, 1 << 33):
        for f in (lambda: layer.step(x, x, rows), lambda: layer.plan(rows), lambda: layer.project(x, rows), lambda: layer.append(rows), lambda: layer.attend(rows),
                  lambda: layer.finish(x, rows)):
            with pytest.raises(ValueError):
                f()
    for bad in (new(4, 256), new(5, 255), new(5, 257), new(5, 256, dtype=torch.float16), new(256, 5).t(), new(1280), new(5, 256, 1), new(1, 256).expand(5, 256),
                torch.zeros(5, 256, dtype=torch.bfloat16, device="meta"), new(1281)[1:].view(5, 256), None):
        for a, b in ((bad, x), (x, bad)):
            with pytest.raises(ValueError):
                layer.step(a, b, 5)
        with pytest.raises(ValueError):
            layer.finish(bad, 5)
    good = torch.zeros(512, 256), torch.zeros(256, 256)
    for bad in (torch.zeros(256, 512).t(), torch.zeros(512, 255), torch.zeros(511, 256), torch.zeros(512, 256, dtype=torch.float16), torch.zeros(512, 256, device="meta")):
        with pytest.raises(ValueError):
            layer.transform_weights(bad, good[1])
    with pytest.raises(ValueError):
        layer.transform_weights(good[0], torch.zeros(255, 256))
    assert not calls
