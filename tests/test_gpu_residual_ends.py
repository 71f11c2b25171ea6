"""The residual step's norms of rows at the ends of float32's range, subnormal numbers among them, without eps.

Tolerance, u = 2^-24: the root mean square is taken in 64 bits, scaling by powers of two is exact, the factor is rounded once (u), and two products follow (u each); 8 u covers them and the
products of these.  Below 2^-126 float32 has a grid of 2^-149, where both of these products round by up to half a step, the first before the weight multiplies it:
(|weight| + 1) / 2 steps, with weights below 3 two of them (1.07 with a weight of 1.39 and eps 1e30).  Every store adds half a step of its type."""
import numpy as np
import pytest
import torch

import paper_2206_07446_amd as nnv
from oracle import serving as OS
from test_gpu_residual_norm import T, Step

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = [(nnv.F32, nnv.F32, nnv.F32), (nnv.BF16, nnv.BF16, nnv.F32), (nnv.F32, nnv.BF16, nnv.BF16)]
FACTORS = (1e-37, 1e-39, 1e-40, 3e-44, 2e37, 5e37, 1e25, 1e-25)


def near(got, want, dtype, slack=8 * U):
    eps = torch.finfo(T[dtype]).eps if dtype != nnv.F32 else 0
    return np.abs(got - want) <= (slack + eps / 2 * (1 + 2.0 ** -6)) * np.abs(want) + 2.0 ** -148


@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("n", [64, 96, 3001, 5120, 16384])
def test_norms_of_the_stream(n, types):
    s = Step(len(FACTORS), n, types=types, y=False, eps=0.0)
    x = s.x.double() * torch.tensor(FACTORS, dtype=torch.float64)[:, None]
    x[:, 1::7] = 0                                           # of a row that is scaled, zeros stay zeros
    s.x = x.to(s.x.dtype)
    assert torch.isfinite(s.x).all()                         # (bfloat16 has no number as small as the smallest of these: a row of zeros there)
    _, h = s.run()
    _, want, _ = OS.residual_norm(s.x.double().numpy(), None, None, None, 1.0, 0.0, s.pre.double().numpy())
    assert near(h, want, types[2]).all()


@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("n", [64, 3001, 5120])
def test_norms_of_the_output(n, types):
    """Of what is added, where the stream holds zeros: r is the norm, of ordinary size."""
    s = Step(len(FACTORS), n, types=types, eps=0.0, scale=1.0)
    y = s.y.double() * torch.tensor(FACTORS, dtype=torch.float64)[:, None]
    y[:, 1::7] = 0
    s.y, s.x = y.to(s.y.dtype), torch.zeros_like(s.x)
    r, h = s.run()
    want, want_h, _ = OS.residual_norm(s.x.double().numpy(), s.y.double().numpy(), s.post.double().numpy(), None, 1.0, 0.0, s.pre.double().numpy())
    assert near(r, want, types[0]).all()
    # of the norm of r: its sum of squares in float32, 64 / 2 + 6 roundings
    assert near(h, want_h, types[2], 56 * U).all()


def test_eps_beside_rows_that_are_scaled():
    for eps in (1e-6, 1e-38, 1e6, 1e30):
        s = Step(len(FACTORS), 96, types=TYPES[0], y=False, eps=eps)
        s.x = (s.x.double() * torch.tensor(FACTORS, dtype=torch.float64)[:, None]).float()
        _, h = s.run()
        _, want, _ = OS.residual_norm(s.x.double().numpy(), None, None, None, 1.0, float(np.float32(eps)), s.pre.double().numpy())
        assert near(h, want, nnv.F32).all()
