"""Products with weights held in 8 bits, against the definition in float64.

Tolerances.  The rounded operands are a definition (powers of two and round to nearest), so the products are those of the oracle
and exact in float32; a sum of k of them in float32, in any order, is within k * 2^-23 of the sum of their magnitudes (2^-24 a step where
the matrix cores round to nearest, twice that where they cut off), the bias adds a step, and the store half a step of y's type."""
import numpy as np
import pytest
import torch

import paper_2206_07446_amd as nnv
from oracle import serving as OS

pytestmark = pytest.mark.gpu
T = {nnv.F32: torch.float32, nnv.F16: torch.float16, nnv.BF16: torch.bfloat16}
DEV = "cuda:0"


def check(y, ref, size, k, dtype):
    y = y.double().cpu().numpy()
    bound = (k + 2) * 2.0 ** -23 * size + torch.finfo(T[dtype]).eps / 2 * np.abs(ref) * (1 + 2.0 ** -10) + torch.finfo(T[dtype]).smallest_normal
    assert np.isfinite(y).all()
    worst = (np.abs(y - ref) / bound).max()
    assert worst <= 1, f"{worst:.3f} of the bound"


def run(m, n, k, x_dtype=nnv.BF16, y_dtype=nnv.F32, raw_dtype=nnv.F32, bias=False, pad_x=0, pad_y=0, seed=1, x=None, w=None, stream=None):
    print(f"case m={m} n={n} k={k} x={x_dtype} y={y_dtype} raw={raw_dtype} bias={bias} pads {pad_x} {pad_y}", flush=True)
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(m, k, generator=g) if x is None else x
    w = torch.randn(n, k, generator=g) * 0.1 if w is None else w
    x, w = x.to(T[x_dtype]), w.to(T[raw_dtype])
    b = torch.randn(n, generator=g) if bias else None
    d = nnv.LinearDesc(n=n, k=k, x_dtype=x_dtype, y_dtype=y_dtype, raw_dtype=raw_dtype)
    xs = torch.full((m, k + pad_x), float("nan"), dtype=T[x_dtype])
    xs[:, :k] = x
    xs, wd, bd = xs.to(DEV), w.to(DEV).contiguous(), None if b is None else b.to(DEV)
    tx = torch.full((nnv.nnv_linear_transformed_bytes(d),), 0x5A, dtype=torch.uint8, device=DEV)
    need = nnv.nnv_linear_workspace_bytes(d, m)
    ws = torch.full((need + 64,), 0x7F, dtype=torch.uint8, device=DEV)          # codes of NaN behind what the call writes
    y = torch.full((m + 2, n + pad_y), 77.0, dtype=T[y_dtype], device=DEV)
    torch.cuda.synchronize()
    nnv.nnv_linear_transform_weights(d, wd, tx, stream=stream)
    nnv.nnv_linear_forward(d, m, xs, k + pad_x, tx, bd, y, n + pad_y, ws, need, stream=stream)
    torch.cuda.synchronize()
    assert (y[m:] == 77).all() and (y[:, n:] == 77).all(), "written outside the rows and columns asked for"
    assert (ws[need:] == 0x7F).all(), "written behind the workspace"
    return y[:m, :n], x, w, b


SIZES = [(1, 1, 1), (1, 128, 128), (1, 100, 1000), (2, 16, 4096), (3, 17, 129), (15, 33, 640), (16, 16, 16), (17, 130, 257), (31, 250, 300), (33, 1000, 77), (64, 144, 512),
         (65, 65, 300), (100, 128, 2048), (128, 256, 384), (129, 257, 1100), (200, 400, 128), (257, 300, 1000), (300, 513, 130), (520, 136, 1536)]


@pytest.mark.parametrize("m,n,k", SIZES)
def test_sizes(m, n, k):
    y, x, w, _ = run(m, n, k)
    check(y, *OS.linear(x.double().numpy(), w.double().numpy()), k, nnv.F32)


# one of each way a product is run: few rows with 32 and 64 outputs to a workgroup, a reduction split among workgroups (evenly and not),
# tiles of 128 in one part and several, tiles of 256
WAYS = [(2, 6201, 260), (16, 12301, 130), (40, 300, 4300), (33, 250, 8300), (130, 6200, 2300), (260, 5001, 1030), (140, 20500, 140), (2500, 4900, 200), (4200, 3000, 384)]


@pytest.mark.parametrize("m,n,k", WAYS)
@pytest.mark.parametrize("y_dtype", [nnv.F32, nnv.BF16])
def test_ways(m, n, k, y_dtype):
    y, x, w, b = run(m, n, k, nnv.BF16, y_dtype, nnv.BF16, True, seed=11)
    ref, size = OS.linear(x.double().numpy(), w.double().numpy(), b.double().numpy())
    size += np.abs(b.double().numpy())
    if y_dtype == nnv.F32:
        return check(y, ref, size, k, y_dtype)
    # 8-bit instructions line the products of eight inputs up to the largest and drop what is 2^17 below it: at most 2^-16 of the sum of magnitudes
    got = y.double().cpu().numpy()
    bound = ((k + 2) * 2.0 ** -23 + 2.0 ** -16) * size + 2.0 ** -8 * np.abs(ref) * (1 + 2.0 ** -8)
    assert np.isfinite(got).all() and (np.abs(got - ref) <= bound).all(), (np.abs(got - ref) / bound).max()


@pytest.mark.parametrize("x_dtype", [nnv.F32, nnv.F16, nnv.BF16])
@pytest.mark.parametrize("y_dtype", [nnv.F32, nnv.F16, nnv.BF16])
@pytest.mark.parametrize("m", [5, 150])
def test_types_strides_bias(x_dtype, y_dtype, m):
    for raw, pad_x, pad_y in ((nnv.F32, 0, 0), (nnv.F16, 1, 3), (nnv.BF16, 8, 8)):
        y, x, w, b = run(m, 200, 264, x_dtype, y_dtype, raw, True, pad_x, pad_y)
        ref, size = OS.linear(x.double().numpy(), w.double().numpy(), b.double().numpy())
        check(y, ref, size + np.abs(b.double().numpy()), 264, y_dtype)


@pytest.mark.parametrize("k", [128, 100, 513])
def test_codes_of_the_weights(k):
    """Rows of the identity read the held weights back, exactly: zeros, ties, subnormal codes, the largest code, blocks of very different sizes."""
    g = torch.Generator().manual_seed(5)
    n = 300
    w = torch.randn(n, k, generator=g)
    grid = torch.tensor(np.r_[OS.E4M3, (OS.E4M3[1:] + OS.E4M3[:-1]) / 2], dtype=torch.float32)
    flat = w[:128, : min(k, 128)].reshape(-1)
    flat[: grid.numel()] = grid
    w[:128, : min(k, 128)] = flat.reshape(128, -1)
    w[128:256] *= 1e-30
    w[256:] *= 1e30
    w[129:140] = 0
    y, _, w, _ = run(k, n, k, nnv.F32, nnv.F32, w=w, x=torch.eye(k))
    assert np.array_equal(y.double().cpu().numpy(), OS.round_weights(w.double().numpy()).T)


def test_codes_of_the_rows():
    """The same for the rows of x, with the identity as weights; rows of zeros, tiny and huge ones."""
    g = torch.Generator().manual_seed(6)
    k = 256
    x = torch.randn(40, k, generator=g)
    x[1] = 0
    x[2] *= 1e-37
    x[3] *= 1e37
    x[4, :128] *= 1e-20
    x[5] = 448.0
    x[6] = torch.tensor(np.r_[OS.E4M3, (OS.E4M3[1:] + OS.E4M3[:-1]) / 2], dtype=torch.float32)[:k].repeat(2)[:k]
    y, x, _, _ = run(40, k, k, nnv.F32, nnv.F32, w=torch.eye(k), x=x)
    assert np.array_equal(y.double().cpu().numpy(), OS.round_rows(x.double().numpy()))


@pytest.mark.parametrize("m", [3, 70, 300])
def test_not_finite(m):
    """A NaN or an infinity spoils its own row of x, and nothing else; in the weights, the outputs that read it."""
    g = torch.Generator().manual_seed(7)
    x, w = torch.randn(m, 300, generator=g), torch.randn(140, 300, generator=g)
    x[1, 5], x[2, 299] = float("inf"), float("nan")
    y, _, _, _ = run(m, 140, 300, nnv.BF16, nnv.F32, x=x, w=w)
    bad = torch.zeros(m, dtype=torch.bool)
    bad[1:3] = True
    assert torch.isnan(y[bad]).all() and torch.isfinite(y[~bad]).all()
    clean = run(m, 140, 300, nnv.BF16, nnv.F32, x=torch.where(torch.isfinite(x), x, 0.), w=w)[0]
    assert torch.equal(y[~bad], clean[~bad])
    w[139, 0] = float("-inf")
    y = run(m, 140, 300, nnv.BF16, nnv.F32, x=torch.where(torch.isfinite(x), x, 0.), w=w)[0]
    assert torch.isnan(y[:, 139]).all() and torch.isfinite(y[:, :128]).all()


def test_same_bits_whatever_the_workspace_holds_and_on_another_stream():
    first = run(33, 300, 2048)[0].clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = run(33, 300, 2048)[0].clone()
    explicit = run(33, 300, 2048, stream=side)[0].clone()
    assert torch.equal(first, again) and torch.equal(first, explicit)


@pytest.mark.parametrize("m", [1, 40, 300])
def test_graph(m):
    """A captured call reads what its buffers hold at each replay."""
    d = nnv.LinearDesc(n=260, k=1100, x_dtype=nnv.F16, y_dtype=nnv.F16, raw_dtype=nnv.F32)
    g = torch.Generator(device=DEV).manual_seed(3)
    w = torch.randn(260, 1100, device=DEV, generator=g)
    tx = torch.empty(nnv.nnv_linear_transformed_bytes(d), dtype=torch.uint8, device=DEV)
    nnv.nnv_linear_transform_weights(d, w, tx)
    x, y = torch.randn(m, 1100, device=DEV, generator=g).half(), torch.zeros(m, 260, dtype=torch.float16, device=DEV)
    ws = torch.empty(nnv.nnv_linear_workspace_bytes(d, m), dtype=torch.uint8, device=DEV)
    nnv.nnv_linear_forward(d, m, x, 1100, tx, None, y, 260, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nnv.nnv_linear_forward(d, m, x, 1100, tx, None, y, 260, ws)
    for _ in range(4):
        x.copy_(torch.randn(m, 1100, device=DEV, generator=g))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got, other = y.clone(), torch.empty_like(y)
        ws.random_(0, 256, generator=g)
        nnv.nnv_linear_forward(d, m, x, 1100, tx, None, other, 260, ws)
        torch.cuda.synchronize()
        assert torch.equal(got, other) and got.any()
