"""The step between two blocks, against its definition in 64 bits.

Tolerances, u = 2^-24.  A norm's sum of n squares is a chain of at most 32 sums, 6 within a wavefront and 16 across; with root, quotient and two
products a norm is within (64 / 2 + 6) u of its value, relative.  r adds a product with the gate, one with scale and the sum, each of the terms' magnitudes: 42 u of those.
The norm of r takes r's error over and that of the root mean square, at most the same in the 2-norm: 42 u of the terms' magnitudes times the row's factor, and
42 u of the row's rms times the factor.  Every store adds half a step of its type."""
import numpy as np
import pytest
import torch

import paper_2206_07446_amd as nnv
from oracle import serving as OS

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
T = {nnv.F32: torch.float32, nnv.F16: torch.float16, nnv.BF16: torch.bfloat16}
U = 2.0 ** -24
TYPES = [(nnv.F32, nnv.BF16, nnv.BF16), (nnv.BF16, nnv.BF16, nnv.BF16), (nnv.F16, nnv.F16, nnv.F16), (nnv.F32, nnv.F32, nnv.F32), (nnv.BF16, nnv.F32, nnv.F16),
         (nnv.F16, nnv.BF16, nnv.F32), (nnv.F32, nnv.F16, nnv.BF16), (nnv.F16, nnv.F32, nnv.BF16), (nnv.BF16, nnv.F16, nnv.F32)]


def rounding(values, dtype):
    info = torch.finfo(T[dtype])
    return np.abs(values) * info.eps / 2 * (1 + 2.0 ** -6) + float(info.tiny) * info.eps


class Step:
    def __init__(self, m, n, types=TYPES[0], gate=None, post=True, pre=True, y=True, scale=0.7, eps=1e-6, pad=0, seed=1, gates=None):
        g = torch.Generator().manual_seed(seed)
        self.m, self.n, self.gate_kind = m, n, gate
        self.types, self.desc = types, nnv.ResidualDesc(n=n, x_dtype=types[0], y_dtype=types[1], h_dtype=types[2], scale=scale, eps=eps)
        new = lambda rows, t, std=1.0: torch.randn(max(rows, 1), n + pad, generator=g).mul(std).to(T[t])  # noqa: E731
        self.x, self.y = new(m, types[0]), new(m, types[1], 0.5) if y else None
        self.gates = gates or {None: 0, "row": m, "one": 1, "index": 5}[gate]
        self.gate = new(self.gates, types[1]) if gate else None
        self.index = torch.randint(self.gates, (m,), generator=g, dtype=torch.int32) if gate == "index" else None
        self.post, self.pre = (1 + 0.2 * torch.randn(n, generator=g) if on else None for on in (post, pre))

    def run(self, in_place=False, stream=None):
        on = lambda t: None if t is None else t.to(DEV)  # noqa: E731
        x, y, gate, index, post, pre = (on(t) for t in (self.x, self.y, self.gate, self.index, self.post, self.pre))
        rows, width = max(self.m, 1) + 1, self.x.shape[1]
        out = torch.full((rows, width), 7.0, dtype=T[self.types[0]], device=DEV)
        if in_place:
            out[:-1] = x
            x = out
        h = torch.full((rows, width), 7.0, dtype=T[self.types[2]], device=DEV)
        print(f"case residual m={self.m} n={self.n} stride={width} types={self.types} gate={self.gate_kind} post={post is not None} pre={pre is not None}", flush=True)
        nnv.nnv_residual_norm(self.desc, self.m, x, width, y, width, post, self.gates, gate, width, index, pre, out, width, h, width, stream=stream)
        torch.cuda.synchronize()
        for t in (out, h):
            assert (t[self.m:] == 7).all(), "rows behind the last"
            if not (in_place and t is out):
                assert (t[:, self.n:] == 7).all(), "columns behind the last"
        return out[:self.m, :self.n].double().cpu().numpy(), h[:self.m, :self.n].double().cpu().numpy()

    def check(self, **kw):
        got, got_h = self.run(**kw)
        of = lambda t: None if t is None else t[..., :self.n].double().numpy()  # noqa: E731
        gate = of(self.gate)
        adds = np.ones(self.m, bool)
        if gate is not None:
            which = np.arange(self.m) if self.gate_kind == "row" else np.zeros(self.m, int) if self.gate_kind == "one" else self.index.numpy()
            adds = (which >= 0) & (which < self.gates)
            gate = gate[np.where(adds, which, 0)]
        x, y = of(self.x)[:self.m], of(self.y)
        y = None if y is None else y[:self.m] * 1.0
        scale, eps = float(np.float32(self.desc.scale)), float(np.float32(self.desc.eps))
        r, h, size = OS.residual_norm(x, y, of(self.post), gate, scale, eps, of(self.pre))
        skip, h_skip, _ = OS.residual_norm(x, None, None, None, scale, eps, of(self.pre))
        r[~adds], size[~adds] = skip[~adds], np.abs(skip[~adds])
        if self.pre is not None:
            h[~adds] = h_skip[~adds]
        error = 42 * U * size
        if self.y is None:
            assert (got == 7).all()
        else:
            assert (np.abs(got - r) <= error + rounding(r, self.types[0])).all()
        if self.pre is None:
            assert (got_h == 7).all()
            return
        factor = np.abs(of(self.pre)) / np.sqrt((r * r).mean(-1, keepdims=True) + eps)
        rms = np.sqrt((size * size).mean(-1, keepdims=True))
        relative = np.abs(r) / np.sqrt((r * r).mean(-1, keepdims=True) + eps)
        bound = factor * error + factor * 42 * U * rms * relative + 42 * U * np.abs(h) + rounding(h, self.types[2])
        assert (np.abs(got_h - h) <= bound * (1 + 2.0 ** -6)).all()


SIZES = [1, 7, 8, 64, 65, 511, 512, 520, 1000, 1024, 4096, 5120, 8191, 8192, 8200, 16384, 16391, 32768]


@pytest.mark.parametrize("n", SIZES)
def test_sizes(n):
    for m in (1, 5):
        Step(m, n, gate="index").check()
        Step(m, n, types=TYPES[1], gate="row", post=False).check()


@pytest.mark.parametrize("types", TYPES, ids=str)
def test_types(types):
    for n, pad in ((96, 0), (1001, 0), (2048, 8), (2048, 3), (9000, 0)):
        Step(37, n, types=types, gate="index", pad=pad).check()


@pytest.mark.parametrize("gate", [None, "row", "one", "index"])
@pytest.mark.parametrize("post,pre,y", [(True, True, True), (False, True, True), (True, False, True), (False, False, True), (True, True, False)])
def test_parts(gate, post, pre, y):
    for n in (200, 4099):
        Step(9, n, gate=gate, post=post, pre=pre, y=y).check()
        Step(9, n, gate=gate, post=post, pre=pre, y=y).check(in_place=True) if y else None


def test_indices_that_are_no_gate():
    for n in (64, 2051):
        s = Step(7, n, gate="index")
        s.index[:4] = torch.tensor([-1, 5, 2 ** 31 - 1, -2 ** 31])
        s.y[0] = float("nan")                                # of what is not added
        got, got_h = s.run()
        assert np.array_equal(got[:4], s.x[:4, :n].double().numpy()) and np.isfinite(got_h).all()
        s.y[0] = 0
        s.check()


def test_numbers_at_the_ends_of_float32():
    """Squares that float32 does not hold; rows of zeros; rows without eps."""
    for n in (96, 3001):
        s = Step(6, n, types=TYPES[3], post=True, eps=0.0, scale=1.0)
        for row, factor in enumerate((1e25, 1e-25, 1e30, 0.0)):
            s.x[row] *= factor
            s.y[row] *= factor
        s.post.fill_(0.0)
        s.post[: n // 2] = 1.0
        s.y[:] = 0                                          # r is x; the norm of y's zeros is zeros
        got, got_h = s.run()
        x = s.x.double().numpy()
        assert np.array_equal(got, x) and np.isfinite(got_h).all() and (got_h[3] == 0).all()
        _, want, _ = OS.residual_norm(x, None, None, None, 1.0, 0.0, s.pre.double().numpy())
        assert (np.abs(got_h - want) <= 84 * U * np.abs(want)).all()


def test_values_that_are_not_numbers():
    for n in (64, 3000):
        s = Step(5, n, types=TYPES[3], post=True, scale=1.0)
        s.x[1, 3] = float("nan")
        s.y[2, 0] = float("nan")
        s.x[3, 5] = float("inf")
        got, got_h = s.run()
        ok = Step(5, n, types=TYPES[3], post=True, scale=1.0).run()
        for a, b in ((got, ok[0]), (got_h, ok[1])):
            assert np.array_equal(a[[0, 4]], b[[0, 4]])
        assert np.isnan(got[1, 3]) and np.isnan(got_h[1]).all() and np.isnan(got[2]).all() and np.isnan(got_h[2]).all()
        assert np.isinf(got[3, 5]) and np.isnan(got_h[3, 5]) and (np.delete(got_h[3], 5) == 0).all()


def test_columns_of_one_buffer():
    """Stream, output of the block and norm side by side in one buffer."""
    n, m = 128, 11
    s = Step(m, n, types=TYPES[1], post=True)
    both = torch.zeros(m, 4 * n, dtype=torch.bfloat16, device=DEV)
    both[:, :n], both[:, n:2 * n] = s.x.to(DEV), s.y.to(DEV)
    nnv.nnv_residual_norm(s.desc, m, both, 4 * n, both[:, n:], 4 * n, s.post.to(DEV), 0, None, 0, None, s.pre.to(DEV), both[:, 2 * n:], 4 * n, both[:, 3 * n:], 4 * n)
    torch.cuda.synchronize()
    got, got_h = s.run()
    assert np.array_equal(both[:, 2 * n:3 * n].double().cpu().numpy(), got) and np.array_equal(both[:, 3 * n:].double().cpu().numpy(), got_h)


def test_many_rows():
    Step(70001, 64, types=TYPES[1], gate="index").check()
    Step(3000, 1600, gate="index").check()


def test_another_stream_and_graph():
    s = Step(33, 1000, gate="index")
    on = [t.to(DEV) for t in (s.x, s.y, s.post, s.gate, s.index, s.pre)]
    x, y, post, gate, index, pre = on
    out, h = torch.empty_like(x), torch.empty(33, 1000, dtype=torch.bfloat16, device=DEV)
    call = lambda: nnv.nnv_residual_norm(s.desc, 33, x, 1000, y, 1000, post, 5, gate, 1000, index, pre, out, 1000, h, 1000)  # noqa: E731
    want, want_h = s.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert np.array_equal(out.double().cpu().numpy(), want) and np.array_equal(h.double().cpu().numpy(), want_h)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (2, 3, 4):
        other = Step(33, 1000, gate="index", seed=seed)
        for a, b in zip(on, (other.x, other.y, other.post, other.gate, other.index, other.pre)):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.double().cpu().numpy() for t in (out, h)]
        assert all(np.array_equal(a, b) for a, b in zip(got, other.run()))
