"""The serving operators together, as attention_layer.py runs them: prompts in, then tokens from a replayed graph; at every step the plan is the
oracle's, products and attention are within the bounds of their own tests of what the oracle makes of the buffers before them, and the
replayed steps give the bytes of the same steps run eagerly."""
import numpy as np
import pytest
import torch

import paper_2206_07446_amd as nnv
from oracle import serving as OS
from paper_2206_07446_amd.attention_layer import AttentionLayer, main

pytestmark = pytest.mark.gpu
HIDDEN, Q, KV, DIM, BLOCK, TOKENS = 384, 8, 2, 64, 16, 120


def weights(seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((Q + 2 * KV) * DIM, HIDDEN, generator=g) * HIDDEN ** -0.5, torch.randn(HIDDEN, Q * DIM, generator=g) * (Q * DIM) ** -0.5


def make(rows, requests, **kw):
    layer = AttentionLayer(HIDDEN, Q, KV, DIM, requests, rows, TOKENS, BLOCK, **kw)
    layer.transform_weights(*(w.cuda() for w in weights(1)))
    layer.cache.zero_()                                  # so that what no step writes compares too
    return layer


def numpy_of(t):
    return t.double().cpu().numpy()


def check_step(layer, x, y, rows, before):
    held, fresh, table, count = before
    torch.cuda.synchronize()
    want = OS.plan(held, fresh, layer.free.tolist(), count, table, BLOCK, layer.desc.blocks, rows)
    assert layer.table.tolist() == want[0] and layer.starts.tolist() == want[1] and layer.held.tolist() == want[2]
    assert layer.positions[:rows].tolist() == want[3] and layer.slots[:rows].tolist() == want[4] and int(layer.count) == want[5]
    u = torch.finfo(layer.dtype).eps / 2
    w_qkv, w_out = (numpy_of(w) for w in weights(1))
    for got, a, w in ((layer.qkv[:rows], x[:rows], w_qkv), (y[:rows], layer.attended[:rows].flatten(1), w_out)):
        ref, size = OS.linear(numpy_of(a), w)
        bound = ((w.shape[1] + 2) * 2.0 ** -23 + 2.0 ** -16) * size + u * np.abs(ref) * (1 + 2.0 ** -8)
        assert (np.abs(numpy_of(got) - ref) <= bound).all()
    half = layer.dtype == torch.float16
    for i, n in enumerate(want[2]):
        a, b = want[1][i], want[1][i + 1]
        if b == a:
            continue
        slots = [want[0][i][j // BLOCK] * BLOCK + j % BLOCK for j in range(n)]
        k, v = (torch.empty(n, KV, DIM, dtype=layer.dtype, device="cuda") for _ in range(2))
        nnv.nnv_kv_read(layer.desc, n, torch.tensor(slots, device="cuda"), layer.cache, k, v)
        # the newest tokens' values are the projection's, rounded to 4 bits
        new = numpy_of(layer.qkv[a:b, (Q + KV) * DIM:]).reshape(b - a, KV, DIM)
        assert np.array_equal(numpy_of(v)[n - (b - a):], OS.round_head(new, half))
        ref, size, most = OS.attention(numpy_of(layer.q[a:b]), numpy_of(k), numpy_of(v), want[3][a:b], layer.desc.scale, layer.desc.window, layer.desc.sinks)
        bound = (u + 2 * OS.score_bound(DIM, most) + (n + 64) * 2.0 ** -23) * size * (1 + 2.0 ** -6) + u * (1 + 2.0 ** -6) * np.abs(ref) + 1e-30
        assert (np.abs(numpy_of(layer.attended[a:b]) - ref) <= bound).all()


@pytest.mark.parametrize("dtype,window,sinks", [(nnv.BF16, 0, 0), (nnv.F16, 20, 3)])
def test_prompts_then_tokens(dtype, window, sinks):
    prompts = [5, 70, 33, 1]
    rows, n = sum(prompts), len(prompts)
    layer, twin = (make(rows, n, dtype=dtype, window=window, sinks=sinks) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(rows, HIDDEN, device="cuda", generator=g).to(layer.dtype)
    y, y_twin = torch.zeros_like(x), torch.zeros_like(x)

    def state():
        return layer.held.tolist(), layer.fresh.tolist(), layer.table.tolist(), int(layer.count)

    for l, out in ((layer, y), (twin, y_twin)):
        l.fresh.copy_(torch.tensor(prompts, dtype=torch.int32))
        before = state() if l is layer else None
        l.step(x, out, rows)
        if l is layer:
            check_step(layer, x, y, rows, before)
        l.fresh.fill_(1)
        l.step(x, out, n)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step(x, y, n)
    for i in range(18):                                  # past the end of a block, and of several
        x[:n].copy_(torch.randn(n, HIDDEN, device="cuda", generator=g))
        before = state()
        graph.replay()
        twin.step(x, y_twin, n)
        check_step(layer, x, y, n, before)
        assert torch.equal(y[:n], y_twin[:n]) and torch.equal(layer.cache, twin.cache)
    assert layer.held.tolist() == [p + 19 for p in prompts]


def test_the_command(capsys):
    main("--hidden 256 --q-heads 4 --kv-heads 2 --head-dim 64 --requests 3 --prompt 20 --steps 5".split())
    assert "a replayed step" in capsys.readouterr().out
