"""Layers of sizes that one of a step's calls would refuse are refused themselves, before a step has run in part; no GPU."""
import pytest
import torch

import paper_2206_07446_amd as nnv
from paper_2206_07446_amd.attention_layer import AttentionLayer


def make(q_heads=4, kv_heads=2, head_dim=64, requests=3, rows=20, tokens=100, hidden=256, **kw):
    return AttentionLayer(hidden, q_heads, kv_heads, head_dim, requests, rows, tokens, block_tokens=16, device="cpu", **kw)


def test_more_blocks_than_a_selection_takes():
    with pytest.raises(ValueError, match="nnv_kv_select"):
        make(requests=1, rows=2, tokens=16 * 32769, keep=4)
    assert make(requests=1, rows=2, tokens=16 * 32769).desc.table_blocks == 32769        # attention over the whole cache does


@pytest.mark.parametrize("kw,call", [(dict(q_heads=1024, kv_heads=1024, rows=4094, keep=4), "nnv_kv_select"), (dict(rows=1 << 20), "nnv_linear_forward"),
                                     (dict(q_heads=1024, kv_heads=1024, rows=90000), "nnv_qk_norm_rope"), (dict(q_heads=1024, kv_heads=64, requests=1 << 16, rows=1 << 16, groups=1), "nnv_kv_attention_shared"),
                                     (dict(q_heads=64, kv_heads=64, requests=1 << 18), "nnv_kv_attention"), (dict(keep=(1 << 20) + 1), "nnv_kv_select"), (dict(tokens=1 << 30), "nnv_kv_plan"),
                                     (dict(head_dim=96), "nnv_kv_plan"), (dict(q_heads=5), "nnv_kv_plan")], ids=str)
def test_sizes_that_a_call_refuses(kw, call):
    with pytest.raises(ValueError, match=call):
        make(**kw)


def test_counts_beyond_32_bits():
    for kw in (dict(rows=1 << 33), dict(requests=1 << 20, tokens=1 << 20), dict(tokens=1 << 36)):
        with pytest.raises((ValueError, OverflowError)):
            make(**kw)


def test_rows_wider_than_a_stream(monkeypatch):
    names = []
    for name in ("nnv_kv_plan", "nnv_linear_forward", "nnv_qk_norm_rope", "nnv_kv_attention", "nnv_residual_norm"):
        monkeypatch.setattr(nnv.binding, name, lambda *a, name=name, **kw: names.append(name))
    layer = make(hidden=32776)
    x, h = torch.zeros(2, 32776), torch.zeros(2, 32776, dtype=torch.bfloat16)
    for begin in (False, True):
        with pytest.raises(ValueError):
            layer.step_stream(x, h, 2, begin=begin)
    assert not names
    layer.step(h, h.clone(), 2)
    make(hidden=32768).step_stream(x[:, :32768].contiguous(), h[:, :32768].contiguous(), 2)
    assert len(names) == 11
