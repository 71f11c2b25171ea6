"""The attention layer over selected blocks, over shared prefixes and on the residual stream: each step's attention against the definition over what its cache
holds, within the bounds of that operator's own tests; replayed steps give the bytes of the same steps run eagerly."""
import numpy as np
import pytest
import torch

import paper_2206_07446_amd as nnv
from oracle import serving as OS
from paper_2206_07446_amd.attention_layer import AttentionLayer, main

pytestmark = pytest.mark.gpu
HIDDEN, Q, KV, DIM, BLOCK = 384, 8, 2, 64, 16


def make(rows, requests, tokens, **kw):
    g = torch.Generator().manual_seed(1)
    layer = AttentionLayer(HIDDEN, Q, KV, DIM, requests, rows, tokens, BLOCK, **kw)
    layer.transform_weights((torch.randn((Q + 2 * KV) * DIM, HIDDEN, generator=g) * 3 * HIDDEN ** -0.5).cuda(), (torch.randn(HIDDEN, Q * DIM, generator=g) * (Q * DIM) ** -0.5).cuda())
    layer.cache.zero_()
    return layer


def numpy_of(t):
    return t.double().cpu().numpy()


def held(layer, request, n):
    """Keys and values of a request's tokens, from the cache."""
    slots = [layer.table[request, j // BLOCK].item() * BLOCK + j % BLOCK for j in range(n)]
    k, v = (torch.empty(n, KV, DIM, dtype=layer.dtype, device="cuda") for _ in range(2))
    nnv.nnv_kv_read(layer.desc, n, torch.tensor(slots, device="cuda"), layer.cache, k, v)
    return numpy_of(k), numpy_of(v)


def check_attention(layer, row, q, k, v, position, seen=None):
    u, n = torch.finfo(layer.dtype).eps / 2, len(k)
    ref, size, most = OS.attention(q, k, v, [position], layer.desc.scale, seen=seen)
    bound = (u + 2 * OS.score_bound(DIM, most) + (n + 64) * 2.0 ** -23) * size * (1 + 2.0 ** -6) + u * (1 + 2.0 ** -6) * np.abs(ref) + 1e-30
    assert (np.abs(numpy_of(layer.attended[row:row + 1])[:, : ref.shape[1]] - ref) <= bound).all()


def check_selected(layer, rows):
    torch.cuda.synchronize()
    starts, lengths, positions = layer.starts.tolist(), layer.held.tolist(), layer.positions[:rows].tolist()
    bounds = numpy_of(layer.bounds).reshape(-1, KV, 2, DIM)
    for i, n in enumerate(lengths):
        if starts[i] == starts[i + 1]:
            continue
        k, v = held(layer, i, n)
        blocks = layer.table[i, : -(-n // BLOCK)].tolist()
        for b, block in enumerate(blocks):
            assert np.array_equal(bounds[block], OS.bounds(k[b * BLOCK:(b + 1) * BLOCK]))
        for r in range(starts[i], starts[i + 1]):
            q, visible = numpy_of(layer.q[r:r + 1]), positions[r] // BLOCK + 1
            want = OS.select(OS.block_scores(q[0], bounds[blocks[:visible]]), visible, layer.keep, layer.first, layer.last, [True] * visible)
            assert np.array_equal(layer.selected[r].cpu().numpy(), want)
            for h in range(KV):
                seen = np.isin(np.arange(n) // BLOCK, want[h])
                group = Q // KV
                u = torch.finfo(layer.dtype).eps / 2
                ref, size, most = OS.attention(q[:, h * group:(h + 1) * group], k[:, h:h + 1], v[:, h:h + 1], [positions[r]], layer.desc.scale, seen=seen)
                bound = (u + 2 * OS.score_bound(DIM, most) + (n + 64) * 2.0 ** -23) * size * (1 + 2.0 ** -6) + u * (1 + 2.0 ** -6) * np.abs(ref) + 1e-30
                assert (np.abs(numpy_of(layer.attended[r, h * group:(h + 1) * group])[None] - ref) <= bound).all()


def test_selected_blocks_from_prompts_on():
    prompts = [5, 150, 33, 1]
    rows, n = sum(prompts), len(prompts)
    layer, twin = (make(rows, n, 220, keep=5, first=1, last=2) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(rows, HIDDEN, device="cuda", generator=g).to(layer.dtype)
    y, y_twin = torch.zeros_like(x), torch.zeros_like(x)
    for l, out in ((layer, y), (twin, y_twin)):
        l.fresh.copy_(torch.tensor(prompts, dtype=torch.int32))
        l.step(x, out, rows)
        if l is layer:
            check_selected(layer, rows)
        l.fresh.fill_(1)
        l.step(x, out, n)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step(x, y, n)
    for i in range(20):                                  # past the end of a block
        x[:n].copy_(torch.randn(n, HIDDEN, device="cuda", generator=g))
        graph.replay()
        twin.step(x, y_twin, n)
        check_selected(layer, n)
        assert torch.equal(y[:n], y_twin[:n]) and torch.equal(layer.cache, twin.cache) and torch.equal(layer.bounds, twin.bounds)


def check_shared(layer, rows, prefix, leader_of):
    torch.cuda.synchronize()
    starts, lengths, positions = layer.starts.tolist(), layer.held.tolist(), layer.positions[:rows].tolist()
    for i, n in enumerate(lengths):
        p, lead = prefix[i], leader_of[i]
        if starts[i] == starts[i + 1]:
            continue
        own_k, own_v = held(layer, i, n) if lead == i else (None, None)
        if lead != i:
            k0, v0 = held(layer, lead, p)
            slots = [layer.table[i, j // BLOCK].item() * BLOCK + j % BLOCK for j in range(p, n)]
            k1, v1 = (torch.empty(n - p, KV, DIM, dtype=layer.dtype, device="cuda") for _ in range(2))
            nnv.nnv_kv_read(layer.desc, n - p, torch.tensor(slots, device="cuda"), layer.cache, k1, v1)
            own_k, own_v = np.concatenate((k0, numpy_of(k1))), np.concatenate((v0, numpy_of(v1)))
        for r in range(starts[i], starts[i + 1]):
            check_attention(layer, r, numpy_of(layer.q[r:r + 1]), own_k, own_v, positions[r])


def test_requests_that_share_a_prefix():
    """Two groups and a request of none; first the prefixes, then prompts behind them, then tokens from a replayed graph."""
    n, rows = 6, 120
    layer, twin = (make(rows, n, 160, groups=2) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(rows, HIDDEN, device="cuda", generator=g).to(layer.dtype)
    y, y_twin = torch.zeros_like(x), torch.zeros_like(x)
    prefix, leader = [64, 64, 64, 16, 16, 0], [0, 0, 0, 3, 3, 5]
    for l, out in ((layer, y), (twin, y_twin)):
        l.fresh.copy_(torch.tensor([70, 0, 0, 20, 0, 0], dtype=torch.int32))
        l.step(x, out, 90)
        free = int(l.count)
        l.share([0, 3, 5], [64, 16])
        assert l.held.tolist() == [70, 64, 64, 20, 16, 0]
        l.fresh.copy_(torch.tensor([1, 40, 3, 1, 17, 9], dtype=torch.int32))
        l.step(x, out, 71)
        assert free - int(l.count) == 3 + 1 + 2 + 1      # blocks of 40, 3, 17 and 9 tokens; the first requests' fit what they have
        if l is layer:
            check_shared(layer, 71, prefix, leader)
        l.fresh.fill_(1)
        l.step(x, out, n)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step(x, y, n)
    for i in range(18):
        x[:n].copy_(torch.randn(n, HIDDEN, device="cuda", generator=g))
        graph.replay()
        twin.step(x, y_twin, n)
        check_shared(layer, n, prefix, leader)
        assert torch.equal(y[:n], y_twin[:n]) and torch.equal(layer.cache, twin.cache)


@pytest.mark.parametrize("stream,post,gated", [(torch.float32, False, False), (torch.bfloat16, True, True)])
def test_the_residual_stream(stream, post, gated):
    """Two layers one after the other; the step's own part is that of `step` on the same rows, byte by byte."""
    n = 5
    layers, twins = ([make(40, n, 100) for _ in range(2)] for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(n, HIDDEN, device="cuda", generator=g).to(stream)
    gate = torch.randn(3, HIDDEN, device="cuda", generator=g).to(torch.bfloat16) if gated else None
    index = torch.tensor([2, 0, 1, 1, 2], dtype=torch.int32, device="cuda") if gated else None
    h = torch.zeros(n, HIDDEN, dtype=torch.bfloat16, device="cuda")
    for l in layers + twins:
        l.fresh.fill_(1)
    for l in layers:
        for w in (l.norm_in, l.norm_next, l.norm_out):
            w.copy_(1 + 0.2 * torch.randn(HIDDEN, device="cuda", generator=g))
    for i, (layer, twin) in enumerate(zip(layers, twins)):
        before = x.double().cpu().numpy()
        came = h.clone()
        if i == 0:                                           # the first layer's input is the norm of the stream
            desc = nnv.ResidualDesc(n=HIDDEN, x_dtype=nnv.F32 if stream == torch.float32 else nnv.BF16, y_dtype=nnv.BF16, h_dtype=nnv.BF16, scale=0.5, eps=1e-6)
            nnv.nnv_residual_norm(desc, n, x, HIDDEN, None, 0, None, 0, None, 0, None, layer.norm_in, None, 0, came, HIDDEN)
        layer.step_stream(x, h, n, begin=i == 0, post=post, gate=gate, index=index, scale=0.5)
        y = torch.zeros_like(h)
        twin.step(came, y, n)
        torch.cuda.synchronize()
        assert torch.equal(y, layer.out[:n])
        gates = numpy_of(gate)[index.tolist()] if gated else None
        r, want, size = OS.residual_norm(before, numpy_of(layer.out[:n]), numpy_of(layer.norm_out) if post else None, gates, 0.5, 1e-6, numpy_of(layer.norm_next))
        u, half = 2.0 ** -24, torch.finfo(torch.bfloat16).eps / 2
        assert (np.abs(x.double().cpu().numpy() - r) <= 42 * u * size + (np.abs(r) * half * (1 + 2.0 ** -6) if stream == torch.bfloat16 else 2 * u * np.abs(r))).all()
        rms = np.sqrt((r * r).mean(-1, keepdims=True))
        factor = np.abs(numpy_of(layer.norm_next)) / rms
        slack = 42 * u * (factor * size + factor * np.sqrt((size * size).mean(-1, keepdims=True)) * np.abs(r) / rms + np.abs(want))
        assert (np.abs(numpy_of(h) - want) <= slack + half * (1 + 2.0 ** -6) * np.abs(want) + 1e-30).all()


@pytest.mark.parametrize("more", ["--keep 3", "--shared 128"])
def test_the_command(capsys, more):
    main(f"--hidden 256 --q-heads 4 --kv-heads 2 --head-dim 64 --requests 3 --prompt 20 --steps 5 {more}".split())
    assert "a replayed step" in capsys.readouterr().out
