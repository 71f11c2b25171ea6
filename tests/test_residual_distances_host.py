"""Distances between rows that the residual step does not look at may be any; those that it does look at are refused outside their range.  No GPU: a misaligned weight ends each call
behind the check of distances."""
import pytest

import paper_2206_07446_amd as nnv
from paper_2206_07446_amd import binding

ALIGN, ARG = -5, -7
FAR = (1 << 40) + 1


@pytest.fixture(params=["module", "ctypes"], autouse=True)
def calls(request, monkeypatch):
    nnv.load()
    if request.param == "ctypes":
        monkeypatch.setattr(binding, "_native", binding._CtypesCalls)


def status(**kw):
    a = [(i + 1) << 44 for i in range(8)]
    names = dict(m=3, x=a[0], ldx=96, y=a[1], ldy=96, post=a[2] + 4, gates=3, gate=a[3], ldg=96, index=a[4], pre=a[5] + 4, x_out=a[6], ldo=96, h=a[7], ldh=96)
    assert set(kw) <= set(names)
    d = nnv.ResidualDesc(n=96, x_dtype=nnv.F32, y_dtype=nnv.BF16, h_dtype=nnv.BF16, scale=1.0, eps=1e-6)
    with pytest.raises(nnv.NnvError) as e:
        nnv.nnv_residual_norm(d, *{**names, **kw}.values(), stream=0)
    return e.value.status


@pytest.mark.parametrize("any_", [FAR, 2 ** 63 - 1, -2 ** 63, -1, 0])
def test_distances_that_are_not_looked_at(any_):
    for kw in (dict(m=1, ldx=any_), dict(m=1, ldx=any_, ldy=any_, ldo=any_, ldh=any_), dict(gates=1, index=None, ldg=any_), dict(gate=None, ldg=any_, gates=any_ % 5),
               dict(y=None, ldy=any_, ldg=any_, ldo=any_), dict(pre=None, h=None, ldh=any_)):
        assert status(**kw) == ALIGN, kw


@pytest.mark.parametrize("bad", [FAR, 2 ** 63 - 1, -2 ** 63, -1, 95])
def test_distances_that_are(bad):
    for name in ("ldx", "ldy", "ldg", "ldo", "ldh"):
        assert status(**{name: bad}) == ARG
    assert status(m=1, ldg=bad) == ARG                       # of several gates
    assert status(y=None, ldx=bad) == ARG
