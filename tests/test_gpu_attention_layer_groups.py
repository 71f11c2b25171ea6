"""Groups that come and go while their requests run, in steps run eagerly and in steps replayed from graphs that were captured under other groups: every row against
the definition over the tokens that its request began behind and its own, within the bound of attention over a shared prefix."""
import numpy as np
import pytest
import torch

import paper_2206_07446_amd as nnv
from oracle import serving as OS
from paper_2206_07446_amd.attention_layer import AttentionLayer

pytestmark = pytest.mark.gpu
HIDDEN, Q, KV, DIM, BLOCK = 384, 8, 2, 64, 16


def read(layer, blocks, n):
    """Keys and values of the first n tokens of these blocks."""
    k, v = (torch.empty(n, KV, DIM, dtype=layer.dtype, device="cuda") for _ in range(2))
    if n:
        nnv.nnv_kv_read(layer.desc, n, torch.tensor([blocks[j // BLOCK] * BLOCK + j % BLOCK for j in range(n)], device="cuda"), layer.cache, k, v)
    return k.double().cpu().numpy(), v.double().cpu().numpy()


def check(layer, behind):
    """behind: of each request, the blocks of the prefix that it began behind."""
    torch.cuda.synchronize()
    starts, lengths, positions, table = layer.starts.tolist(), layer.held.tolist(), layer.positions.tolist(), layer.table.tolist()
    for i, n in enumerate(lengths):
        if starts[i] == starts[i + 1]:
            continue
        k, v = read(layer, behind[i] + table[i][len(behind[i]):], n)
        rows = slice(starts[i], starts[i + 1])
        u = torch.finfo(layer.dtype).eps / 2
        ref, size, most = OS.attention(layer.q[rows].double().cpu().numpy(), k, v, positions[rows], layer.desc.scale)
        bound = (u + 2 * OS.score_bound(DIM, most) + (n + 64) * 2.0 ** -23) * size * (1 + 2.0 ** -6) + u * (1 + 2.0 ** -6) * np.abs(ref) + 1e-30
        assert (np.abs(layer.attended[rows].double().cpu().numpy() - ref) <= bound).all(), f"request {i} of {n}"


def test_groups_come_and_go_while_requests_run():
    n, rows = 6, 120
    g = torch.Generator().manual_seed(1)
    layer = AttentionLayer(HIDDEN, Q, KV, DIM, n, rows, 160, BLOCK, groups=2)
    layer.transform_weights((torch.randn((Q + 2 * KV) * DIM, HIDDEN, generator=g) * 3 * HIDDEN ** -0.5).cuda(), (torch.randn(HIDDEN, Q * DIM, generator=g) * (Q * DIM) ** -0.5).cuda())
    layer.cache.zero_()
    x = torch.randn(rows, HIDDEN, generator=g).to(layer.dtype).cuda()
    y = torch.zeros_like(x)
    behind = [[] for _ in range(n)]

    def step(fresh):
        layer.fresh.copy_(torch.tensor(fresh, dtype=torch.int32))
        layer.step(x, y, sum(fresh))
        check(layer, behind)

    def capture():
        layer.fresh.copy_(running)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer.step(x, y, n)
        return graph

    running = torch.tensor([1, 1, 1, 1, 0, 0], dtype=torch.int32)
    step([70, 0, 0, 20, 0, 0])
    plain = capture()                                        # no groups yet
    layer.share([0, 3], [64])
    behind[1] = behind[2] = layer.table[0, :4].tolist()
    step([1, 20, 3, 1, 0, 0])
    one = capture()
    layer.share([3, 6], [16])                                # a second document; the first one's requests are in no group now
    behind[4] = behind[5] = layer.table[3, :1].tolist()
    step([1, 1, 2, 1, 9, 30])
    running = torch.ones(n, dtype=torch.int32)
    layer.share([0, 3, 6], [64, 16])                         # both
    step([1, 1, 1, 1, 1, 1])
    two = capture()
    for ends, tokens in (([0, 3, 6], [64, 16]), ([3, 6], [16]), ([1, 3], [48]), ([0], []), ([1, 3, 6], [64, 16])):
        layer.share(ends, tokens)
        for graph in (plain, one, two, None):
            x.copy_(torch.randn(x.shape, generator=g))
            layer.step(x, y, n) if graph is None else graph.replay()
            check(layer, behind)
    assert max(layer.held.tolist()) > 90                     # past the end of a block
