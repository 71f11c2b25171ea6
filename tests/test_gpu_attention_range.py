"""Attention over the 4-bit cache where the scores lie far apart: one token far above thousands of others that together still count.

Tolerances: those of test_gpu_serving.py for scores, sums and the store, and half a step of the 16-bit type for each weight.  A weight may lie below float16's
normal range, where it is off by up to 2^-25; the largest of a wavefront's weights is held as 2^10 at least, so that this is 2^-35 of the largest weight for each
of the n tokens (bfloat16 has the exponents of float32)."""
import numpy as np
import pytest
import torch

import paper_2206_07446_amd as nnv
from oracle import serving as OS
from test_gpu_serving import DEV, Scene, T, ints, layer

pytestmark = pytest.mark.gpu
DIM = 64


def scene(dtype, n, fresh, keys, values, query, window=0, sinks=0):
    """One request: tokens' keys along the first value of a head, values the same for all of a head, and one query for all rows and heads."""
    s = Scene(layer(q_heads=16, kv_heads=1, head_dim=DIM, block_tokens=64, dtype=dtype, scale=1.0, window=window, sinks=sinks), [n], [fresh])
    s.k.zero_()
    s.k[:, 0, 0] = keys
    s.v[:] = values[:, None, None]
    s.q.zero_()
    s.q[:, :, 0] = query
    slots = [s.table[0][j // 64] * 64 + j % 64 for j in range(n)]
    k, v = s.k.to(DEV).contiguous(), s.v.to(DEV).contiguous()
    nnv.nnv_qk_norm_rope(s.d, n, None, 0, k, DIM, v, DIM, None, None, None, ints([0] * n), ints(slots, torch.int64), None, None, s.cache)
    return s


def check(s, n, fresh):
    d, half = s.d, s.d.dtype == nnv.F16
    k, v = OS.round_head(s.k.double().numpy(), half), OS.round_head(s.v.double().numpy(), half)
    assert np.array_equal(k, s.k.double().numpy()) and np.array_equal(v, s.v.double().numpy())       # 4 bits hold these inputs
    ref, size, most = OS.attention(s.q.double().numpy(), k, v, s.positions, d.scale, d.window, d.sinks)
    u = torch.finfo(T[d.dtype]).eps / 2
    bound = (u + 2 * OS.score_bound(DIM, most) + (n + 64) * 2.0 ** -23) * size * (1 + 2.0 ** -6) + u * (1 + 2.0 ** -6) * np.abs(ref) + float(torch.finfo(T[d.dtype]).tiny)
    bound = bound + (n * 2.0 ** -35 * np.abs(v).max() if half else 0)
    worst = (np.abs(s.run() - ref) / bound).max()
    assert worst <= 1, f"{worst:.3f} of the bound"


# rows x 16 heads of one request: the kernel for few rows, and the one for many
@pytest.mark.parametrize("n,fresh,window", [(500, 1, 0), (3000, 1, 0), (3000, 2, 1500), (500, 40, 0), (3000, 40, 0), (3000, 40, 1500)])
@pytest.mark.parametrize("gap", [9, 12, 15, 18])
@pytest.mark.parametrize("dtype", [nnv.F16, nnv.BF16])
def test_a_token_far_above_the_others(n, fresh, window, gap, dtype):
    """The first token's score lies `gap` above all others', and its value is 0."""
    keys, values = torch.zeros(n), torch.full((n,), 96.0)
    keys[0], values[0] = 6, 0
    check(scene(dtype, n, fresh, keys, values, gap / 6, window, 4 if window else 0), n, fresh)


@pytest.mark.parametrize("n,fresh", [(900, 1), (900, 40)])
@pytest.mark.parametrize("query", [0.5, 3, -3])
@pytest.mark.parametrize("dtype", [nnv.F16, nnv.BF16])
def test_scores_that_rise_or_fall(n, fresh, query, dtype):
    """From 0 to 18 in eight steps over the tokens, or down from there."""
    level = torch.arange(n) * 8 // n
    keys = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6])[level]
    values = torch.tensor([1., -2, 3, 4, -6, 1.5, 2, 0.5])[torch.arange(n) % 8]
    check(scene(dtype, n, fresh, keys, values, query), n, fresh)


@pytest.mark.parametrize("n,fresh", [(700, 1), (5000, 1), (700, 40)])
@pytest.mark.parametrize("exponent", [4, 8, 13, 30])
@pytest.mark.parametrize("dtype", [nnv.F16, nnv.BF16])
def test_scores_beyond_what_float32_counts_in_ones(n, fresh, exponent, dtype):
    """One score is the largest by so much that nothing else weighs anything: the output is that token's value, however large the scores are."""
    if dtype == nnv.F16 and exponent > 13:
        exponent = 12                                        # (what float16 holds)
    for query in (997.0, 1234.5, -3.0, 31000.0, 60000.0):
        for order in (torch.arange(n), torch.arange(n).flip(0), (torch.arange(n) * 7919) % n):
            levels = torch.tensor([0, .5, 1, 1.5, 2, 3, 4])[order * 7 // n]
            at = int(order.argmax()) if fresh == 1 else int(order[: n - fresh].argmax())      # a token that all rows see
            levels[at] = 6
            if query < 0:
                levels = -levels
            values = torch.full((n,), -2.0)
            values[at] = 3
            s = scene(dtype, n, fresh, levels * 2.0 ** exponent, values, query)
            assert (s.run() == 3).all()
