"""Attention over shared prefixes and selected blocks, and the residual step, without a GPU: sizes and every refusal, through the compiled module and through
ctypes.  Pointers here are no memory: a call that is not refused must do nothing."""
import numpy as np
import pytest
import torch

import paper_2206_07446_amd as nnv
from oracle import serving as OS
from paper_2206_07446_amd import binding

NULL, BAD_DESC, UNSUPPORTED, WORKSPACE, ALIGN, ARG = -1, -2, -3, -4, -5, -7
BIG = 1 << 40


@pytest.fixture(params=["module", "ctypes"])
def calls(request, monkeypatch):
    nnv.load()
    if request.param == "module":
        assert binding._native.__name__ == "_nnvpy"
    else:
        monkeypatch.setattr(binding, "_native", binding._CtypesCalls)


def status(fn, *args):
    with pytest.raises(nnv.NnvError) as e:
        fn(*args, stream=0)
    return e.value.status


def layer(**kw):
    return nnv.AttentionDesc(**{**dict(q_heads=8, kv_heads=2, head_dim=128, block_tokens=64, blocks=10, table_blocks=4, dtype=nnv.BF16, scale=0.1, eps=1e-6), **kw})


def apart(n):
    """Addresses far from one another."""
    return [(i + 1) << 44 for i in range(n)]


# of each call: how many leading counts there are, and how many addresses follow (the workspace last)
CALLS = {"bounds": (nnv.nnv_kv_bounds, (1, 1), 5, False), "select": (nnv.nnv_kv_select, (1, 1, 4, 1, 2), 8, True),
         "blocks": (nnv.nnv_kv_attention_blocks, (1, 1, 400), 9, True), "shared": (nnv.nnv_kv_attention_shared, (1, 1, 1), 10, True)}


def args_of(name, counts=None):
    fn, base, n, ws = CALLS[name]
    return fn, list(counts or base) + apart(n) + ([BIG] if ws else []), len(base), n


@pytest.mark.parametrize("name", list(CALLS))
@pytest.mark.parametrize("bad,want", [(dict(q_heads=0), BAD_DESC), (dict(q_heads=9), BAD_DESC), (dict(dtype=7), BAD_DESC), (dict(dtype=nnv.F32), UNSUPPORTED),
                                      (dict(head_dim=96), UNSUPPORTED), (dict(block_tokens=48), UNSUPPORTED), (dict(window=-1), BAD_DESC)])
def test_descriptors(calls, name, bad, want):
    fn, args, _, _ = args_of(name)
    assert status(fn, layer(**bad), *args) == want


def test_descriptors_of_selection_have_no_window(calls):
    d = layer(window=64)
    for name in ("bounds", "select", "blocks"):
        fn, args, _, _ = args_of(name)
        assert status(fn, d, *args) == UNSUPPORTED
    assert nnv.nnv_kv_bounds_bytes(d) == nnv.nnv_kv_select_workspace_bytes(d, 1, 1) == nnv.nnv_kv_attention_blocks_workspace_bytes(d, 1, 1, 4) == 0
    assert nnv.nnv_kv_attention_shared_workspace_bytes(d, 1, 1, 1) > 0
    d = layer(table_blocks=32769)
    fn, args, _, _ = args_of("select")
    assert status(fn, d, *args) == UNSUPPORTED and nnv.nnv_kv_select_workspace_bytes(d, 1, 1) == 0


@pytest.mark.parametrize("name", list(CALLS))
def test_counts(calls, name):
    d = layer()
    fn, args, n_counts, _ = args_of(name)
    for at, value in ((0, -1), (1, -1), (0, 1 << 21), (1, 1 << 25)):
        args = args_of(name)[1]
        args[at] = value
        assert status(fn, d, *args) == ARG
    for rest in {"bounds": [], "select": [(0, 0, 0), (-1, 0, 0), (4, -1, 2), (4, 1, -1), (4, 3, 2), ((1 << 20) + 1, 0, 0), (4, 2 ** 31 - 1, 2 ** 31 - 1)],
                 "blocks": [(0,), (-3,), ((1 << 20) + 1,)], "shared": [(-1,), (1 << 21,)]}[name]:
        args = args_of(name)[1]
        args[2:2 + len(rest)] = rest
        assert status(fn, d, *args) == ARG


@pytest.mark.parametrize("name", list(CALLS))
def test_addresses(calls, name):
    d = layer()
    fn, good, n_counts, n = args_of(name)
    for i in range(n_counts, n_counts + n):
        args = list(good)
        args[i] = None
        assert status(fn, d, *args) == NULL
        args[i] = good[i] + 2
        assert status(fn, d, *args) == ALIGN
    # outputs in the place of inputs, and of each other
    outs = {"bounds": [4], "select": [6, 7], "blocks": [7, 8], "shared": [8, 9]}[name]
    for out in outs:
        for i in range(n):
            if i == out:
                continue
            args = list(good)
            args[n_counts + out] = good[n_counts + i]
            assert status(fn, d, *args) == ARG


def test_nothing_to_do(calls):
    d = layer()
    nnv.nnv_kv_bounds(d, 0, 5, None, None, None, None, None, stream=0)
    nnv.nnv_kv_bounds(d, 5, 0, None, None, None, None, None, stream=0)
    nnv.nnv_kv_select(d, 5, 0, 4, 1, 1, *[None] * 8, 0, stream=0)
    nnv.nnv_kv_attention_blocks(d, 5, 0, 4, *[None] * 9, 0, stream=0)
    nnv.nnv_kv_attention_shared(d, 5, 0, 2, *[None] * 10, 0, stream=0)


def test_workspaces(calls):
    d = layer(table_blocks=1000)
    for name, size, counts in (("select", nnv.nnv_kv_select_workspace_bytes, (1, 1)), ("blocks", nnv.nnv_kv_attention_blocks_workspace_bytes, (1, 1, 400)),
                               ("shared", nnv.nnv_kv_attention_shared_workspace_bytes, (1, 1, 1))):
        need = size(d, *counts)
        assert need > 0
        fn, args, n_counts, n = args_of(name)
        args[-1] = need - 1
        assert status(fn, d, *args) == WORKSPACE
        args[-2], args[-1] = torch.empty(16, dtype=torch.uint8), None
        assert status(fn, d, *args) == WORKSPACE
    assert nnv.nnv_kv_bounds_bytes(layer()) == 10 * 2 * 2 * 128 * 2
    assert nnv.nnv_kv_bounds_bytes(layer(blocks=1 << 30, kv_heads=8)) == (1 << 30) * 8 * 512         # no 32-bit product
    assert nnv.nnv_kv_select_workspace_bytes(layer(), 3, 7) == 7 * 2 * 4 * 8
    # scores of many rows are kept for some of them at a time
    assert nnv.nnv_kv_select_workspace_bytes(layer(table_blocks=32768), 3, 1 << 20) <= 256 << 20
    assert nnv.nnv_kv_select_workspace_bytes(layer(), 3, 1 << 22) == 0
    assert nnv.nnv_kv_select_workspace_bytes(layer(), 0, 1 << 21) == 0                           # 2^32 threads of 1024 a row and head
    # a wavefront joins each row and query head: no more of these than a launch has
    wide = layer(q_heads=1024, kv_heads=64)
    assert nnv.nnv_kv_attention_shared_workspace_bytes(wide, 1 << 16, 1 << 16, 1) == 0
    assert status(nnv.nnv_kv_attention_shared, wide, 1 << 16, 1 << 16, 1, *apart(10), BIG) == ARG
    fn, args, _, _ = args_of("select", (1, 1 << 22, 4, 1, 2))
    assert status(fn, layer(), *args) == ARG
    many = layer(q_heads=1024, kv_heads=1)
    for name, size, counts in (("blocks", nnv.nnv_kv_attention_blocks_workspace_bytes, (1, 1 << 20, 4)), ("shared", nnv.nnv_kv_attention_shared_workspace_bytes, (1, 1 << 20, 1))):
        fn, args, _, _ = args_of(name, counts)
        assert size(many, *counts) == 0 and status(fn, many, *args) == ARG


def residual(**kw):
    return nnv.ResidualDesc(**{**dict(n=96, x_dtype=nnv.F32, y_dtype=nnv.BF16, h_dtype=nnv.BF16, scale=1.0, eps=1e-6), **kw})


# m, x, ldx, y, ldy, post, gates, gate, ldg, index, pre, x_out, ldo, h, ldh
def residual_args(**kw):
    a = apart(9)
    names = dict(m=3, x=a[0], ldx=96, y=a[1], ldy=96, post=a[2], gates=3, gate=a[3], ldg=96, index=a[4], pre=a[5], x_out=a[6], ldo=96, h=a[7], ldh=96)
    assert set(kw) <= set(names)
    return list({**names, **kw}.values())


@pytest.mark.parametrize("bad", [dict(n=0), dict(n=-8), dict(n=32769), dict(x_dtype=3), dict(y_dtype=-1), dict(h_dtype=9), dict(scale=float("nan")),
                                 dict(scale=float("inf")), dict(eps=-1.0), dict(eps=float("nan"))])
def test_residual_descriptors(calls, bad):
    assert status(nnv.nnv_residual_norm, residual(**bad), *residual_args()) == BAD_DESC


def test_residual_refusals(calls):
    d, f = residual(), nnv.nnv_residual_norm
    for kw in (dict(m=-1), dict(m=1 << 22), dict(ldx=95), dict(ldy=95), dict(ldo=95), dict(ldh=95), dict(ldg=95), dict(gates=0), dict(gates=2, index=None),
               dict(ldx=(1 << 40) + 1)):
        assert status(f, d, *residual_args(**kw)) == ARG, kw
    for name in ("x", "x_out", "h"):
        assert status(f, d, *residual_args(**{name: None})) == NULL
    a = apart(9)
    for name, at in (("x", 0), ("y", 1), ("post", 2), ("gate", 3), ("pre", 5), ("x_out", 6), ("h", 7)):
        assert status(f, d, *residual_args(**{name: a[at] + 8})) == ALIGN
    assert status(f, d, *residual_args(index=a[4] + 2)) == ALIGN
    # outputs in inputs and in each other
    for out in ("x_out", "h"):
        for at in (0, 1, 2, 3, 4, 5):
            if (out, at) != ("x_out", 0):
                assert status(f, d, *residual_args(**{out: a[at]})) == ARG, (out, at)
    assert status(f, d, *residual_args(h=a[6])) == ARG
    assert status(f, d, *residual_args(x_out=a[0], ldo=100)) == ARG                       # in place with another distance
    assert status(f, d, *residual_args(x_out=a[0] + 2 * 96 * 4)) == ARG                   # a later row of x
    assert status(f, residual(h_dtype=nnv.F32), *residual_args(x=a[0], ldx=192, h=a[0] + 95 * 4 + 4, ldh=191)) == ARG      # columns that run into the next row
    # nothing to do
    f(d, *residual_args(m=0), stream=0)
    f(d, *residual_args(m=0, x=None, y=None, pre=None), stream=0)
    f(d, *residual_args(x=None, y=None, pre=None), stream=0)


def test_selection_of_the_oracle():
    b = np.zeros((4, 1, 2, 3))
    b[1, 0] = [[1, 2, 0], [-1, -2, 0]]
    b[2, 0] = [[1, 2, 0], [1, 2, 0]]
    q = np.array([[1.0, -1, 5], [-2, 0, 1]])
    s = OS.block_scores(q, b)
    assert s.tolist() == [[0, 3, -1, 0]]                    # heads: 1 + 2 = 3 and 2; 1 - 2 = -1 and -2
    s[0, 2] = 0
    assert OS.select(s, 4, 2, 0, 0, [True] * 4).tolist() == [[0, 1]]
    assert OS.select(s, 4, 3, 0, 1, [True] * 4).tolist() == [[0, 1, 3]]
    assert OS.select(s, 3, 5, 1, 1, [True, False, True, True]).tolist() == [[0, 2, -1, -1, -1]]
    assert OS.block_scores(q, b, negative=True).tolist() == [[0, 3, 2, 0]]
