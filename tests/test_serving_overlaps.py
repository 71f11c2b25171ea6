"""Buffers of the serving operators that overlap where one workgroup would write what another still reads: refused on the host.  Pointers here are no memory."""
import itertools

import pytest

import paper_2206_07446_amd as nnv
from test_serving_host import ARG, A, calls, layer, linear, status  # noqa: F401

N, ROWS, WIDTH = 5, 2000, 4
NAMES = ("held", "fresh", "free_blocks", "free_count", "block_table", "starts", "lengths", "positions", "slots", "free_left")
SIZES = (4 * N, 4 * N, 40, 4, 4 * N * WIDTH, 4 * (N + 1), 4 * N, 4 * ROWS, 8 * ROWS, 4)
OUTPUTS = NAMES[4:]


def apart():
    """Buffers one behind the other, with nothing between them but what alignment asks for."""
    at, places = A, []
    for size in SIZES:
        places.append(at)
        at += -(-size // 8) * 8
    return places


@pytest.mark.parametrize("a,b", [p for p in itertools.combinations(range(10), 2) if NAMES[p[1]] in OUTPUTS], ids=lambda i: NAMES[i])
def test_plan(calls, a, b):  # noqa: F811
    places = apart()
    for moved, place in ((b, places[a]), (a, places[b])):
        args = list(places)
        args[moved] = place
        assert status(nnv.nnv_kv_plan, layer(), N, ROWS, *args) == ARG
    # the last entry of one in the place of the other's first, where that may be and is known to be read
    if NAMES[a] != "free_blocks":
        args = list(places)
        args[b] = places[a] + (SIZES[a] - 4) // 8 * 8
        assert status(nnv.nnv_kv_plan, layer(), N, ROWS, *args) == ARG


def product(x, y, m=3, k=64, n=64, ldx=64, ldy=64, x_dtype=nnv.BF16, y_dtype=nnv.BF16):
    nnv.nnv_linear_forward(linear(n=n, k=k, x_dtype=x_dtype, y_dtype=y_dtype), m, x, ldx, 1 << 30, None, y, ldy, 1 << 31, 1 << 28, stream=0)


@pytest.mark.parametrize("m", [1, 16, 40])
@pytest.mark.parametrize("where", [dict(), dict(ldx=128, ldy=128), dict(y=A + 16), dict(y=A - 112), dict(ldx=128, ldy=128, y=A + 96), dict(ldx=128, ldy=128, y=A + 160),
                                   dict(y_dtype=nnv.F32), dict(y_dtype=nnv.F32, ldx=128, y=A + 112), dict(ldx=100, ldy=128)], ids=str)
def test_product_in_the_place_of_its_inputs(calls, m, where):  # noqa: F811
    args = {**dict(x=A, y=A, m=m), **where}
    if m == 1 and args["y"] == A + 160:
        return                                                    # (the next row of x is none of one row's)
    with pytest.raises(nnv.NnvError) as e:
        product(**args)
    assert e.value.status == ARG
