"""Products with 8-bit weights within the bounds that nnv.h states, over every way that a product is run, in both 16-bit types, where the sums cancel and where
products of one sum lie far apart.

Tolerances.  Sums of k products in float32: k * 2^-23 of the sum of their magnitudes (see test_gpu_linear.py).  16-bit results of more than 16 rows go through the
8-bit instructions, which line the products of eight neighbouring inputs up to the largest and hold them to 2^-13 of that: each other one is off by so much at
most, and by no more than itself.  The bias adds a step, the store half a step of the result's type."""
import numpy as np
import pytest
import torch

import paper_2206_07446_amd as nnv
from oracle import serving as OS
from test_gpu_linear import T, run

pytestmark = pytest.mark.gpu

# few rows; wavefronts that split the reduction, in one part and several; tiles of 128 in several parts and one; tiles of 256
WAYS = [(16, 300, 1024), (17, 300, 1024), (40, 300, 4352), (33, 250, 8448), (130, 6200, 2304), (260, 5001, 1024), (140, 20500, 256), (2500, 4900, 256), (4200, 3000, 512)]


def check(y, x, w, bias, dtype, m):
    """Of up to 48 rows and outputs, spread over all."""
    rows, outputs = (np.unique(np.linspace(0, n - 1, 48).astype(int)) for n in (y.shape[0], y.shape[1]))
    xq, wq = OS.round_rows(x.double().numpy()[rows]), OS.round_weights(w.double().numpy())[outputs]
    bias, k = bias.double().numpy()[outputs], x.shape[1]
    ref, size, lost = xq @ wq.T + bias, np.abs(xq) @ np.abs(wq).T + np.abs(bias), np.zeros((len(rows), len(outputs)))
    if m > 16 and dtype != nnv.F32:
        for i in range(len(rows)):
            p = np.abs(xq[i] * wq).reshape(len(outputs), k // 8, 8)
            lost[i] = np.minimum(p, 2.0 ** -13 * p.max(-1, keepdims=True)).sum((1, 2))
        assert (lost <= 2.0 ** -10 * size).all()
    u = torch.finfo(T[dtype]).eps / 2
    bound = (k + 2) * 2.0 ** -23 * size + lost + u * (1 + 2.0 ** -8) * np.abs(ref) + float(torch.finfo(T[dtype]).smallest_normal)
    got = y.double().cpu().numpy()
    assert np.isfinite(got).all()
    worst = (np.abs(got[np.ix_(rows, outputs)] - ref) / bound).max()
    assert worst <= 1, f"{worst:.3f} of the bound"


@pytest.mark.parametrize("m,n,k", WAYS)
@pytest.mark.parametrize("dtype", [nnv.F16, nnv.BF16, nnv.F32])
@pytest.mark.parametrize("kind", ["normal", "cancelling", "far apart"])
def test_bounds(m, n, k, dtype, kind):
    x_dtype = nnv.BF16 if dtype == nnv.F32 else dtype
    g = torch.Generator().manual_seed(m + n)
    x, w = torch.randn(m, k, generator=g), torch.randn(n, k, generator=g) * 0.1
    if kind == "cancelling":                                 # the second half takes most of the first away
        half = k // 2
        x[:, half:] = x[:, :half]
        w[:, half:] = torch.where(torch.rand(n, half, generator=g) < 0.02, w[:, half:], -w[:, :half])
    elif kind == "far apart":                                # magnitudes over 2^8 and 2^6, one input of every eight far above the others
        x = x.sign() * torch.exp2(-8 * torch.rand(m, k, generator=g))
        w = w.sign() * torch.exp2(-6 * torch.rand(n, k, generator=g) - 3)
        x[:, 3::8] = 30 * x[:, 3::8].sign()
    y, x, w, b = run(m, n, k, x_dtype, dtype, x_dtype, True, x=x, w=w)
    check(y, x, w, b, dtype, m)
