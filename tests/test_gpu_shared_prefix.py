"""Attention of requests that share a prefix, against the definition over each request's tokens.  The tolerance is that of attention over the whole cache: a float32
score is off by at most score_bound(), its weight by that factor, twice where numerator and denominator differ; weights are rounded to the 16-bit type (half a
step each), sums over n tokens and the joins are float32 (n + 64 roundings, at most 2^-23 each on the matrix cores), the store adds half a step."""
import numpy as np
import pytest
import torch

import paper_2206_07446_amd as nnv
from oracle import serving as OS

pytestmark = pytest.mark.gpu
T = {nnv.F16: torch.float16, nnv.BF16: torch.bfloat16}
DEV = "cuda:0"


def layer(**kw):
    return nnv.AttentionDesc(**{**dict(q_heads=8, kv_heads=2, head_dim=128, block_tokens=64, blocks=10, table_blocks=4, dtype=nnv.BF16, scale=0.088, eps=1e-6), **kw})


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEV)


class Shared:
    """members: of each group, what its requests hold behind the prefix; a request has its last `fresh` tokens (of prefix and own) as queries.  Only the first of a
    group has table entries for whole blocks of the prefix, others a number that is no block; 0xFF wherever nothing is held."""

    def __init__(self, d, prefixes, members, fresh, loose=(), seed=1, padding=0, before=()):
        self.d = d
        g = torch.Generator().manual_seed(seed)
        block, kv, dim, t = d.block_tokens, d.kv_heads, d.head_dim, T[d.dtype]
        self.groups, self.shared = [len(before)], list(prefixes)
        plan = [(0, n, True) for n in before]              # (tokens of the prefix, own ones, whether the first of its group)
        for p, own in zip(prefixes, members):
            plan += [(p, n, i == 0) for i, n in enumerate(own)]
            self.groups.append(len(plan))
        plan += [(0, n, True) for n in loose]
        self.lengths = [p + n for p, n, _ in plan]
        need = [(-(-(p + n) // block) if lead else -(-(p + n) // block) - p // block) for p, n, lead in plan]
        d.blocks, d.table_blocks = sum(need) + 2, max([-(-n // block) for n in self.lengths] + [1])
        order = torch.randperm(d.blocks, generator=g).tolist()
        self.table, keys, values, slots, self.k, self.v = [], [], [], [], [], []
        common = None
        for p, n, lead in plan:
            own = torch.randn(n + (p if lead else 0), 2, kv, dim, generator=g).to(t)
            skip = 0 if lead else p // block
            row = [10 ** 8] * skip + [order.pop() for _ in range(-(-(p + n) // block) - skip)]
            row += [10 ** 8] * (d.table_blocks - len(row))
            common = own[:p] if lead else common
            first = 0 if lead else p
            slots += [row[j // block] * block + j % block for j in range(first, p + n)]
            keys.append(own[:, 0])
            values.append(own[:, 1])
            whole = own if lead else torch.cat((common, own))
            self.k.append(whole[:, 0])
            self.v.append(whole[:, 1])
            self.table.append(row)
        self.cache = torch.full((nnv.nnv_kv_cache_bytes(d),), 0xFF, dtype=torch.uint8, device=DEV)
        if slots:
            kd, vd = torch.cat(keys).to(DEV).contiguous(), torch.cat(values).to(DEV).contiguous()
            nnv.nnv_qk_norm_rope(d, len(slots), None, 0, kd, kv * dim, vd, kv * dim, None, None, None, ints([0] * len(slots)), ints(slots, torch.int64), None, None, self.cache)
        self.fresh = [min(f, n) for f, n in zip(fresh if isinstance(fresh, (list, tuple)) else [fresh] * len(plan), self.lengths)]
        self.starts = [0]
        for f in self.fresh:
            self.starts.append(self.starts[-1] + f)
        self.rows = self.starts[-1] + padding
        self.q = torch.randn(self.rows, d.q_heads, dim, generator=g).mul(1.5).to(t)
        self.positions = [n - f + r for n, f in zip(self.lengths, self.fresh) for r in range(f)] + [-1] * padding

    def run(self, n_groups=None):
        d, n = self.d, len(self.lengths)
        n_groups = len(self.shared) if n_groups is None else n_groups
        need = nnv.nnv_kv_attention_shared_workspace_bytes(d, n, self.rows, n_groups)
        ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device=DEV)
        out = torch.full((self.rows + 1, d.q_heads, d.head_dim), 7.0, dtype=T[d.dtype], device=DEV)
        print(f"case shared groups={self.groups[:6]} prefixes={self.shared[:6]} lengths={self.lengths[:6]} fresh={self.fresh[:6]} heads={d.q_heads}/{d.kv_heads} "
              f"dim={d.head_dim} block={d.block_tokens} window={d.window} sinks={d.sinks} type={d.dtype} workspace={need}", flush=True)
        nnv.nnv_kv_attention_shared(d, n, self.rows, n_groups, self.q.to(DEV), ints(self.table), ints(self.starts), ints(self.lengths), ints(self.positions),
                                    ints(self.groups), ints(self.shared or [0]), self.cache, out, ws, need)
        torch.cuda.synchronize()
        assert (out[-1] == 7).all() and (ws[need:] == 0xFF).all(), "written behind the buffers"
        return out[:-1].double().cpu().numpy()

    def check(self, got=None, hidden=None):
        d = self.d
        got = self.run() if got is None else got
        half = d.dtype == nnv.F16
        u, used = torch.finfo(T[d.dtype]).eps / 2, 0
        for i, (n, f) in enumerate(zip(self.lengths, self.fresh)):
            rows = slice(self.starts[i], self.starts[i + 1])
            k, v = OS.round_head(self.k[i].double().numpy(), half), OS.round_head(self.v[i].double().numpy(), half)
            seen = None if hidden is None else ~np.isin(np.arange(n), hidden[i])
            ref, size, most = OS.attention(self.q[rows].double().numpy(), k[:n], v[:n], self.positions[rows], d.scale, d.window, d.sinks, seen)
            bound = (u + 2 * OS.score_bound(d.head_dim, most) + (n + 64) * 2.0 ** -23) * size * (1 + 2.0 ** -6) + u * (1 + 2.0 ** -6) * np.abs(ref) + float(torch.finfo(T[d.dtype]).tiny)
            worst = (np.abs(got[rows] - ref) / bound).max() if f else 0
            assert worst <= 1, f"request {i} of {n}: {worst:.3f} of the bound"
            used += f
        assert (got[used:] == 0).all()
        return got


    def check_rows(self, got, rows):
        """Some rows only."""
        d, half = self.d, self.d.dtype == nnv.F16
        u = torch.finfo(T[d.dtype]).eps / 2
        for r in rows:
            i = int(np.searchsorted(self.starts, r, "right")) - 1
            if i >= len(self.lengths):
                assert (got[r] == 0).all()
                continue
            k, v = OS.round_head(self.k[i].double().numpy(), half), OS.round_head(self.v[i].double().numpy(), half)
            ref, size, most = OS.attention(self.q[r:r + 1].double().numpy(), k, v, self.positions[r:r + 1], d.scale, d.window, d.sinks)
            bound = (u + 2 * OS.score_bound(d.head_dim, most) + (len(k) + 64) * 2.0 ** -23) * size * (1 + 2.0 ** -6) + u * (1 + 2.0 ** -6) * np.abs(ref) + float(torch.finfo(T[d.dtype]).tiny)
            assert (np.abs(got[r] - ref[0]) <= bound[0]).all(), f"row {r} of request {i}"


SCENES = [([1], [[1]], 1), ([16], [[1, 5, 40]], 1), ([100], [[3, 3, 50, 16]], 1), ([65, 33], [[2, 80], [1, 1, 1]], 1), ([200, 7, 64], [[1], [30, 2], [64, 65, 1, 1]], 2)]


@pytest.mark.parametrize("prefixes,members,fresh", SCENES, ids=str)
@pytest.mark.parametrize("block", [16, 64, 256])
def test_single_rows(prefixes, members, fresh, block):
    for dim, heads, dtype in ((64, (6, 6), nnv.F16), (128, (8, 2), nnv.BF16), (256, (5, 1), nnv.BF16)):
        Shared(layer(head_dim=dim, q_heads=heads[0], kv_heads=heads[1], block_tokens=block, dtype=dtype, scale=dim ** -0.5), prefixes, members, fresh, padding=2).check()


@pytest.mark.parametrize("dim,dtype", [(64, nnv.BF16), (64, nnv.F16), (128, nnv.F16), (128, nnv.BF16), (256, nnv.F16), (256, nnv.BF16)])
def test_prefixes_of_many_pairs(dim, dtype):
    """Groups of enough rows and heads for the kernel that holds 128 pairs, one of them nearly none."""
    for heads, block in (((16, 1), 16), ((40, 2), 64)):
        d = layer(head_dim=dim, q_heads=heads[0], kv_heads=heads[1], block_tokens=block, dtype=dtype, scale=dim ** -0.5)
        Shared(d, [130, 5, 300], [[1, 2, 17, 40] * 3, [3], [9] * 10], 1, padding=1).check()


@pytest.mark.parametrize("dim,dtype", [(64, nnv.BF16), (128, nnv.F16), (128, nnv.BF16), (256, nnv.BF16)])
def test_prompts_behind_a_prefix(dim, dtype):
    """Many rows of a request: its own tokens go to the kernel for many pairs too."""
    for block in (16, 128):
        d = layer(head_dim=dim, q_heads=16, kv_heads=1, block_tokens=block, dtype=dtype, scale=dim ** -0.5)
        Shared(d, [150, 64], [[70, 3, 40], [100, 1]], [70, 3, 40, 100, 1], padding=3).check()


@pytest.mark.parametrize("dim,heads", [(64, (32, 2)), (128, (64, 8)), (256, (48, 4))], ids=str)
def test_prompts_whose_last_tiles_are_split(dim, heads):
    """Tiles of 128 pairs that fill the chip less than once, and once and a part; requests of a row or two beside them."""
    for members in ([[90, 1, 130, 64], [200, 3]], [[500, 1, 700, 300], [2, 450]]):
        rows = [min(n, 400) for m in members for n in m]
        s = Shared(layer(head_dim=dim, q_heads=heads[0], kv_heads=heads[1], block_tokens=32, dtype=nnv.F16 if dim == 64 else nnv.BF16, scale=dim ** -0.5), [1100, 333], members,
                   [0 if n == 3 else n for n in rows], padding=2)
        few = list(range(0, s.rows, 1 + s.rows // 60))
        got = s.run()
        assert np.array_equal(got, s.run())
        s.check_rows(got, few)


@pytest.mark.parametrize("heads,dim", [((16, 1), 64), ((40, 2), 128), ((16, 2), 256)], ids=str)
def test_requests_of_some_rows_each(heads, dim):
    """Own tokens of 32 to 255 pairs a request by 128 pairs, beside prefixes that all share."""
    s = Shared(layer(q_heads=heads[0], kv_heads=heads[1], block_tokens=16, head_dim=dim, scale=dim ** -0.5), [150, 70], [[9, 30, 2, 77] * 6, [40, 8] * 5], [7, 3, 1, 9, 4, 12] * 6, padding=1)
    s.check()


@pytest.mark.parametrize("fresh", [[60, 9, 12], [30, 1, 1]], ids=str)
def test_rows_within_the_prefix(fresh):
    """Tokens of the prefix itself among the step's rows, as where its first request takes it in."""
    for heads in ((16, 1), (4, 2)):
        Shared(layer(q_heads=heads[0], kv_heads=heads[1], block_tokens=16, head_dim=64), [50], [[0, 4, 7]], fresh).check()


@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 0), (32, 4), (40, 60), (64, 1), (100, 40), (4096, 4), (50, 1000), (150, 101)])
def test_windows(window, sinks):
    for heads, fresh in (((8, 2), 1), ((16, 1), 1), ((16, 1), 45)):
        d = layer(q_heads=heads[0], kv_heads=heads[1], block_tokens=32, window=window, sinks=sinks)
        Shared(d, [100, 33], [[1, 60, 200], [5, 40]], fresh, padding=1).check()


def test_requests_of_no_group():
    for heads in ((8, 2), (16, 1)):
        Shared(layer(q_heads=heads[0], kv_heads=heads[1], block_tokens=16), [40, 64], [[3, 9], [1]], 1, before=[20, 300], loose=[7, 1, 100], padding=2).check()
    s = Shared(layer(block_tokens=16), [], [], 1, loose=[7, 90, 700])
    s.check(s.run(n_groups=0))
    s.groups, s.shared = [3, 3, 3], [50, 60]               # groups of no requests
    s.check()


def test_no_groups_and_no_requests():
    """Without groups the call is attention over the cache, byte by byte; without requests rows are zeros."""
    for fresh in (1, 60):
        s = Shared(layer(block_tokens=16), [], [], fresh, loose=[7, 90, 700], padding=1)
        n, out = len(s.lengths), torch.zeros(s.rows, 8, 128, dtype=torch.bfloat16, device=DEV)
        ws = torch.zeros(nnv.nnv_kv_attention_workspace_bytes(s.d, n, s.rows) + 16, dtype=torch.uint8, device=DEV)
        nnv.nnv_kv_attention(s.d, n, s.rows, s.q.to(DEV), ints(s.table), ints(s.starts), ints(s.lengths), ints(s.positions), s.cache, out, ws)
        torch.cuda.synchronize()
        assert np.array_equal(s.run(n_groups=0), out.double().cpu().numpy())
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)
    out = torch.full((3, 8, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    for groups in (0, 2):
        out.fill_(7)
        nnv.nnv_kv_attention_shared(s.d, 0, 3, groups, s.q[:3].to(DEV), None, ints([0]), None, ints([5, 0, -1]), ints([0, 0, 0]), ints([9, 9]), s.cache, out, ws)
        torch.cuda.synchronize()
        assert (out == 0).all()


def test_prefixes_of_nothing_and_of_more_than_is_held():
    s = Shared(layer(block_tokens=16), [0], [[30, 200]], 1)
    s.check()
    for value in (-7, -2 ** 31):
        s.shared = [value]
        s.check()
    # more than the first request holds: all that it holds is in common
    s = Shared(layer(block_tokens=16), [48], [[0, 9, 20]], 1)
    for value in (49, 10 ** 6, 2 ** 31 - 1):
        s.shared = [value]
        s.check()


def test_groups_with_empty_ones_between():
    s = Shared(layer(block_tokens=16, head_dim=64), [40, 64], [[3, 9], [1, 70]], 1)
    s.groups, s.shared = [0, 0, 2, 2, 4, 4], [5, 40, 11, 64, 3]
    s.check()


def test_many_groups():
    """More groups, and more requests, than a wavefront looks at in one round."""
    g = np.random.default_rng(3)
    for n in (63, 64, 65, 150):
        members = [[int(v) for v in g.integers(0, 30, int(g.integers(1, 4)))] for _ in range(n)]
        Shared(layer(block_tokens=16, head_dim=64, q_heads=4, kv_heads=2), [int(v) for v in g.integers(1, 90, n)], members, 1, loose=[5]).check()


def test_long_prefixes_are_split_and_joined():
    for heads, members, fresh in (((8, 1), [[1, 700]], 1), ((16, 1), [[1, 9, 700, 30] * 3], 1), ((16, 1), [[3, 1100]], 40)):
        s = Shared(layer(q_heads=heads[0], kv_heads=heads[1], block_tokens=64, head_dim=64), [9001], members, fresh)
        first = s.check()
        assert np.array_equal(first, s.run())


def test_blocks_that_are_none():
    for heads in ((8, 2), (16, 1)):
        s = Shared(layer(q_heads=heads[0], kv_heads=heads[1], block_tokens=16), [70], [[40, 30, 5]], 3, padding=2)
        s.positions[1] = -1
        s.table[0][1], s.table[1][5] = -5, 10 ** 8            # tokens 16 .. 31 of the prefix, 80 .. 95 of the second request
        got = s.run()
        assert (got[1] == 0).all()
        s.check(got, hidden=[np.arange(16, 32), np.r_[16:32, 80:96], np.arange(16, 32)])


@pytest.mark.parametrize("scale", [-0.1, 0.0])
def test_factors_that_are_not_positive(scale):
    Shared(layer(block_tokens=16, scale=scale), [70, 20], [[40, 30, 5], [1]], 1).check()


def test_numbers_out_of_range_do_no_harm():
    big = 2 ** 31 - 1
    for heads in ((8, 2), (16, 1)):
        s = Shared(layer(q_heads=heads[0], kv_heads=heads[1], block_tokens=16), [70, 20], [[40, 30, 5], [1]], 4)
        good = s.groups, s.shared, s.starts, s.lengths
        for groups in ([-5, 2, big], [big, -9, 3], [4, 2, 0], [0, 9, 4]):
            s.groups = groups
            s.run()
        s.groups = good[0]
        for starts, lengths in (([0, 50, -9, 3, 10 ** 9], [10 ** 9, -5, big, 0]), ([14, 9, 5, 2, 0], [big] * 4)):
            s.starts, s.lengths = starts, lengths
            s.run()


def test_queries_that_are_not_numbers():
    s = Shared(layer(block_tokens=16, head_dim=64, q_heads=4, kv_heads=2), [70], [[40, 30, 5]], 1)
    want = s.check()
    s.q[1, 2, 5] = float("nan")
    got = s.run()
    assert np.isnan(got[1, 2]).all()
    keep = np.ones(got.shape[:2], bool)
    keep[1, 2] = False
    assert np.array_equal(got[keep], want[keep])


def test_another_stream_and_graph():
    s = Shared(layer(block_tokens=16, head_dim=64), [70, 20], [[40, 30, 5], [1]], 1)
    n = len(s.lengths)
    ws = torch.zeros(nnv.nnv_kv_attention_shared_workspace_bytes(s.d, n, s.rows, 2), dtype=torch.uint8, device=DEV)
    q, out = s.q.to(DEV), torch.zeros(s.rows, 8, 64, dtype=torch.bfloat16, device=DEV)
    arrays = [ints(v) for v in (s.table, s.starts, s.lengths, s.positions, s.groups, s.shared)]
    call = lambda: nnv.nnv_kv_attention_shared(s.d, n, s.rows, 2, q, *arrays, s.cache, out, ws)  # noqa: E731
    want = s.check()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert np.array_equal(out.double().cpu().numpy(), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn in range(3):
        s.q = torch.randn(s.q.shape, generator=torch.Generator().manual_seed(turn)).to(s.q.dtype)
        q.copy_(s.q)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(out.double().cpu().numpy(), s.check())
