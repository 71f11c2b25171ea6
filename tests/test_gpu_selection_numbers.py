"""Selection by queries some of whose values are no numbers: a head that holds one counts as -infinity, and the group's other heads decide.  Selections are exact."""
import pytest
import torch

import paper_2206_07446_amd as nnv
from test_gpu_selected_blocks import DEV, Scene, layer

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.mark.parametrize("scale", [0.1, -0.1])
@pytest.mark.parametrize("lengths,fresh", [([300, 200, 470, 90], [1, 1, 1, 1]), ([300, 470], [3, 17])], ids=["single rows", "prompts"])
@pytest.mark.parametrize("heads,dim,dtype", [((8, 2), 128, nnv.BF16), ((4, 2), 64, nnv.F16), ((10, 2), 64, nnv.BF16), ((40, 2), 256, nnv.F16)], ids=str)
def test_heads_that_hold_a_nan(heads, dim, dtype, lengths, fresh, scale):
    s = Scene(layer(head_dim=dim, q_heads=heads[0], kv_heads=heads[1], block_tokens=16, dtype=dtype, scale=scale), lengths, fresh)
    group = heads[0] // heads[1]
    # bounds above 0, and queries that make every score of theirs negative
    g = torch.Generator().manual_seed(1)
    bounds = 1 + torch.randint(0, 4, (s.d.blocks, s.d.kv_heads, 2, dim), generator=g).sort(2, descending=True).values.to(torch.bfloat16) / 4
    for r in range(s.rows):
        s.q[r] = -s.q[r].abs() if scale > 0 else s.q[r].abs()
        s.q[r, r % group] = NAN                              # a head of the first group
        s.q[r, group + (r + 1) % group, r % dim] = NAN       # a value of one of the second
    for keep, first, last in ((1, 0, 0), (4, 1, 1), (9, 0, 2)):
        s.check_select(keep, first, last, bounds.to(DEV))
    s.q[:, :group] = NAN                                     # all of the group: the lowest blocks
    s.q[0, group:] = NAN
    s.check_select(5, 0, 1, bounds.to(DEV))
    s.q[:] = NAN
    s.check_select(3, 0, 0)
