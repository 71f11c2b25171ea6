"""Products that read and write columns of one buffer side by side."""
import pytest
import torch

import paper_2206_07446_amd as nnv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("m", [1, 5, 16, 40, 300])
@pytest.mark.parametrize("y_dtype", [nnv.BF16, nnv.F32])
def test_columns_beside_the_inputs(m, y_dtype):
    k, n, size = 264, 200, 2 if y_dtype == nnv.BF16 else 4
    d = nnv.LinearDesc(n=n, k=k, x_dtype=nnv.BF16, y_dtype=y_dtype, raw_dtype=nnv.F32)
    g = torch.Generator(device=DEV).manual_seed(m)
    w, x = torch.randn(n, k, device=DEV, generator=g), torch.randn(m, k, device=DEV, generator=g).bfloat16()
    tx = torch.empty(nnv.nnv_linear_transformed_bytes(d), dtype=torch.uint8, device=DEV)
    nnv.nnv_linear_transform_weights(d, w, tx)
    ws = torch.empty(max(16, nnv.nnv_linear_workspace_bytes(d, m)), dtype=torch.uint8, device=DEV)
    apart = torch.empty(m, n, dtype=torch.bfloat16 if y_dtype == nnv.BF16 else torch.float32, device=DEV)
    nnv.nnv_linear_forward(d, m, x, k, tx, None, apart, n, ws)
    row = 2 * k + size * n                                    # bytes
    buf = torch.zeros(m * row, dtype=torch.uint8, device=DEV)
    rows = buf.view(m, row)
    rows[:, : 2 * k] = x.view(torch.uint8)
    nnv.nnv_linear_forward(d, m, buf, row // 2, tx, None, buf.data_ptr() + 2 * k, row // size, ws)
    torch.cuda.synchronize()
    assert torch.equal(rows[:, 2 * k:], apart.view(torch.uint8)) and torch.equal(rows[:, : 2 * k], x.view(torch.uint8))
