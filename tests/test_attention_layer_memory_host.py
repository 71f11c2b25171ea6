"""Where the stream, the norms, gates and indices of a step may lie, without a GPU: parts of one allocation as well as tensors of their own, but not in each other."""
import pytest
import torch

import paper_2206_07446_amd as nnv
from paper_2206_07446_amd.attention_layer import AttentionLayer

ROWS, HIDDEN = 5, 256


@pytest.fixture
def calls(monkeypatch):
    names = []
    for name in ("nnv_kv_plan", "nnv_linear_forward", "nnv_qk_norm_rope", "nnv_kv_attention", "nnv_residual_norm"):
        monkeypatch.setattr(nnv.binding, name, lambda *a, name=name, **kw: names.append(name))
    return names


def make():
    return AttentionLayer(HIDDEN, 4, 2, 64, 3, 20, 100, block_tokens=16, device="cpu")


def test_parts_of_one_allocation(calls):
    layer, size = make(), ROWS * HIDDEN
    pool = torch.zeros(4 * size + 64, dtype=torch.bfloat16)
    x, h, gate = (pool[i * size:(i + 1) * size].view(ROWS, HIDDEN) for i in range(3))
    index = pool[3 * size:3 * size + 2 * ROWS].view(torch.int32)
    layer.step_stream(x, h, ROWS, gate=gate, index=index)
    layer.step_stream(h, x, ROWS, gate=gate[:1])
    layer.step_stream(pool[:2 * size].view(2 * ROWS, HIDDEN)[:ROWS], pool[size:3 * size].view(2 * ROWS, HIDDEN), ROWS)     # rows behind the step's are not looked at
    layer.step_stream(x, x, 0)
    assert calls.count("nnv_residual_norm") == 4


def test_parts_that_meet_are_refused_before_any_call(calls):
    layer, size = make(), ROWS * HIDDEN
    pool = torch.zeros(4 * size + 64, dtype=torch.bfloat16)
    at = lambda first, rows=ROWS: pool[first:first + rows * HIDDEN].view(rows, HIDDEN)  # noqa: E731
    index = pool[:2 * ROWS].view(torch.int32)
    far = torch.zeros(ROWS, HIDDEN, dtype=torch.bfloat16)
    for x, h, gate, i in ((at(0), at(0), None, None), (at(0), at(size - 8), None, None), (at(size - 8), at(0), None, None), (at(0), at(2 * size), at(size - 8), None),
                          (at(2 * size), at(0), at(size - 8), None), (at(0), at(size), far, index), (at(size), at(0), far[:1], index), (layer.out, far, None, None),
                          (far, layer.out[4:], None, None)):
        with pytest.raises(ValueError):
            layer.step_stream(x, h, ROWS, gate=gate, index=i)
    assert not calls
