"""Buffers of the serving operators that overlap where one workgroup would write what another still reads: refused on the host.  Pointers here are no memory."""
import itertools

import pytest

import paper_2206_07446_amd as nnv
from test_serving_host import ALIGN, ARG, A, calls, layer, status  # noqa: F401

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
