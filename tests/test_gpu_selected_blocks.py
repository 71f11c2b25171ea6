"""Bounds of cache blocks, the selection by them and attention over selected blocks, against their definitions.

Bounds and selections are exact.  Attention's tolerance is that of attention over the whole cache: a float32 score is off by at most score_bound(), its
weight by that factor, twice where numerator and denominator differ; weights are rounded to the 16-bit type (half a step each), sums over n tokens and the joins are
float32 (n + 64 roundings, at most 2^-23 each on the matrix cores), the store adds half a step."""
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


class Scene:
    """Requests of given lengths with their last rows as queries, blocks in no order, and 0xFF wherever nothing is held."""

    def __init__(self, d, lengths, fresh, seed=1, padding=0, std=1.5):
        self.d, self.lengths, self.fresh = d, lengths, fresh
        g = torch.Generator().manual_seed(seed)
        block, kv, dim, t = d.block_tokens, d.kv_heads, d.head_dim, T[d.dtype]
        need = [-(-n // block) for n in lengths]
        d.blocks, d.table_blocks = sum(need) + 2, max(need + [1])
        order = torch.randperm(d.blocks, generator=g).tolist()
        self.table = [[order.pop() for _ in range(k)] + [10 ** 8] * (d.table_blocks - k) for k in need]
        total = sum(lengths)
        x = torch.randn(total, 2 * kv, dim, generator=g) + torch.randn(total // 50 + 1, 2 * kv, dim, generator=g).repeat_interleave(50, 0)[:total]
        x = x.to(t)
        self.k, self.v = x[:, :kv], x[:, kv:]
        slots = [self.table[i][j // block] * block + j % block for i, n in enumerate(lengths) for j in range(n)]
        self.cache = torch.full((nnv.nnv_kv_cache_bytes(d),), 0xFF, dtype=torch.uint8, device=DEV)
        if total:
            kd, vd = self.k.to(DEV).contiguous(), self.v.to(DEV).contiguous()
            nnv.nnv_qk_norm_rope(d, total, None, 0, kd, kv * dim, vd, kv * dim, None, None, None, ints([0] * total), ints(slots, torch.int64), None, None, self.cache)
        self.rows = sum(fresh) + padding
        self.q = torch.randn(self.rows, d.q_heads, dim, generator=g).mul(std).to(t)
        self.starts = [0]
        for f in fresh:
            self.starts.append(self.starts[-1] + f)
        self.positions = [n - f + r for n, f in zip(lengths, fresh) for r in range(f)] + [-1] * padding
        half = d.dtype == nnv.F16
        self.held_k, self.held_v = (OS.round_head(c.double().numpy(), half) for c in (self.k, self.v))

    def plan(self):
        return ints(self.table or [0]), ints(self.starts), ints(self.lengths or [0])

    # ---- bounds
    def all_bounds(self):
        """What every block's bounds are, from the tokens."""
        d, at = self.d, 0
        out = np.zeros((d.blocks, d.kv_heads, 2, d.head_dim))
        for i, n in enumerate(self.lengths):
            for b in range(-(-n // d.block_tokens)):
                if 0 <= self.table[i][b] < d.blocks:
                    out[self.table[i][b]] = OS.bounds(self.held_k[at + b * d.block_tokens: at + min(n, (b + 1) * d.block_tokens)])
            at += n
        return out

    def check_bounds(self):
        d = self.d
        out = torch.full((d.blocks + 1, d.kv_heads, 2, d.head_dim), 7.0, dtype=torch.bfloat16, device=DEV)
        print(f"case bounds lengths={self.lengths[:6]} fresh={self.fresh[:6]} heads={d.kv_heads} dim={d.head_dim} block={d.block_tokens} type={d.dtype}", flush=True)
        nnv.nnv_kv_bounds(d, len(self.lengths), self.rows, *self.plan(), self.cache, out)
        torch.cuda.synchronize()
        want = np.full(out.shape, 7.0)
        every = self.all_bounds()
        for i, (n, f) in enumerate(zip(self.lengths, self.fresh)):
            if f:
                for b in range((n - f) // d.block_tokens, -(-n // d.block_tokens)):
                    if 0 <= self.table[i][b] < d.blocks:
                        want[self.table[i][b]] = every[self.table[i][b]]
        assert np.array_equal(out.double().cpu().numpy(), want)

    # ---- selection
    def select(self, keep, first, last, bounds, need=None):
        d = self.d
        need = nnv.nnv_kv_select_workspace_bytes(d, len(self.lengths), self.rows)
        ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device=DEV)
        out = torch.full((self.rows + 1, d.kv_heads, keep), -7, dtype=torch.int32, device=DEV)
        print(f"case select lengths={self.lengths[:6]} fresh={self.fresh[:6]} heads={d.q_heads}/{d.kv_heads} dim={d.head_dim} block={d.block_tokens} keep={keep} "
              f"first={first} last={last} type={d.dtype} width={d.table_blocks}", flush=True)
        nnv.nnv_kv_select(d, len(self.lengths), self.rows, keep, first, last, self.q.to(DEV), *self.plan(), ints(self.positions), bounds, out, ws, need)
        torch.cuda.synchronize()
        assert (out[-1] == -7).all() and (ws[need:] == 0xFF).all(), "written behind the buffers"
        return out[:-1]

    def check_select(self, keep, first=0, last=0, bounds=None):
        d = self.d
        if bounds is None:
            bounds = torch.from_numpy(self.all_bounds()).to(torch.bfloat16).to(DEV)
        got = self.select(keep, first, last, bounds)
        held = bounds.double().cpu().numpy()
        want = np.full(got.shape, -1)
        for i, n in enumerate(self.lengths):
            there = [0 <= b < d.blocks for b in self.table[i]]
            of = held[[b if t else 0 for b, t in zip(self.table[i], there)]]
            for r in range(self.starts[i], self.starts[i + 1]):
                seen = min(self.positions[r], n - 1)
                visible = seen // d.block_tokens + 1 if seen >= 0 else 0
                s = OS.block_scores(self.q[r].double().numpy(), of[:visible], d.scale < 0) if visible else np.zeros((d.kv_heads, 0))
                want[r] = OS.select(s, visible, keep, first, last, there)
        assert np.array_equal(got.cpu().numpy(), want)
        return got

    # ---- attention
    def attend(self, selected):
        d, keep = self.d, selected.shape[-1]
        need = nnv.nnv_kv_attention_blocks_workspace_bytes(d, len(self.lengths), self.rows, keep)
        ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device=DEV)
        out = torch.full((self.rows + 1, d.q_heads, d.head_dim), 7.0, dtype=T[d.dtype], device=DEV)
        print(f"case blocks lengths={self.lengths[:6]} fresh={self.fresh[:6]} heads={d.q_heads}/{d.kv_heads} dim={d.head_dim} block={d.block_tokens} keep={keep} "
              f"type={d.dtype} workspace={need}", flush=True)
        nnv.nnv_kv_attention_blocks(d, len(self.lengths), self.rows, keep, self.q.to(DEV), *self.plan(), ints(self.positions), selected, self.cache, out, ws, need)
        torch.cuda.synchronize()
        assert (out[-1] == 7).all() and (ws[need:] == 0xFF).all(), "written behind the buffers"
        return out[:-1].double().cpu().numpy()

    def check_attend(self, selected):
        d, got = self.d, self.attend(selected)
        lists, u, at, used = selected.cpu().numpy(), torch.finfo(T[d.dtype]).eps / 2, 0, 0
        group = d.q_heads // d.kv_heads
        for i, (n, f) in enumerate(zip(self.lengths, self.fresh)):
            for r in range(self.starts[i], self.starts[i + 1]):
                for h in range(d.kv_heads):
                    tokens = [b * d.block_tokens + j for b in lists[r, h] if 0 <= b < d.table_blocks and 0 <= self.table[i][b] < d.blocks for j in range(d.block_tokens)]
                    tokens = at + np.array([t for t in tokens if t < n and t <= self.positions[r]], int)
                    heads = slice(h * group, (h + 1) * group)
                    ref, size, most = OS.attention(self.q[r:r + 1, heads].double().numpy(), self.held_k[tokens][:, h:h + 1], self.held_v[tokens][:, h:h + 1],
                                                   [len(tokens)], d.scale)
                    bound = (u + 2 * OS.score_bound(d.head_dim, most) + (len(tokens) + 64) * 2.0 ** -23) * size * (1 + 2.0 ** -6) + u * (1 + 2.0 ** -6) * np.abs(ref)
                    worst = (np.abs(got[r:r + 1, heads] - ref) / (bound + float(torch.finfo(T[d.dtype]).tiny))).max()
                    assert worst <= 1, f"row {r} of request {i} of {n}: {worst:.3f} of the bound"
            at += n
            used += f
        assert (got[used:] == 0).all()
        return got

    def lists(self, keep, seed=3):
        """Any blocks of a row's request, none twice, ascending, -1 behind the last."""
        g = np.random.default_rng(seed)
        out = np.full((self.rows, self.d.kv_heads, keep), -1, np.int32)
        for i, n in enumerate(self.lengths):
            for r in range(self.starts[i], self.starts[i + 1]):
                for h in range(self.d.kv_heads):
                    visible = self.positions[r] // self.d.block_tokens + 1
                    some = np.sort(g.permutation(max(visible, 0))[:keep])
                    out[r, h, :len(some)] = some
        return torch.from_numpy(out).to(DEV)


LENGTHS = [([1], [1]), ([16, 17, 15], [1, 1, 1]), ([300, 0, 64, 700], [1, 0, 1, 1]), ([257, 100, 3], [40, 100, 3]), ([500, 40], [3, 17])]


# ---- bounds

@pytest.mark.parametrize("lengths,fresh", LENGTHS, ids=str)
@pytest.mark.parametrize("block", [16, 32, 64, 128, 256])
def test_bounds(lengths, fresh, block):
    for dim, kv, dtype in ((64, 3, nnv.F16), (128, 2, nnv.BF16), (256, 1, nnv.BF16)):
        Scene(layer(head_dim=dim, q_heads=kv, kv_heads=kv, block_tokens=block, dtype=dtype), lengths, fresh, padding=2).check_bounds()


def test_bounds_of_many_requests():
    g = np.random.default_rng(2)
    for n in (63, 64, 65, 300):
        lengths = [int(v) for v in g.integers(0, 90, n)]
        fresh = [int(g.integers(0, v + 1)) if g.random() < 0.5 else min(1, v) for v in lengths]
        Scene(layer(head_dim=64, block_tokens=16), lengths, fresh, padding=3).check_bounds()


def test_bounds_where_blocks_are_none_and_keys_are_extreme():
    s = Scene(layer(block_tokens=16, dtype=nnv.BF16, head_dim=64), [100, 50], [100, 50])
    s.table[0][2], s.table[1][0] = -4, 10 ** 8
    s.check_bounds()
    for dtype in (nnv.F16, nnv.BF16):
        s = Scene(layer(block_tokens=16, dtype=dtype, head_dim=64), [48], [48])
        k = s.k.clone()
        top = float(torch.finfo(T[dtype]).max)
        k[0, 0, :3] = torch.tensor([float("nan"), float("inf"), -float("inf")])
        k[20, 1], k[33, :, :32], k[34, :, 32:] = top, 0, 2.0 ** -14
        k[35] = -2.0 ** -24 if dtype == nnv.F16 else -2.0 ** -130
        slots = [s.table[0][j // 16] * 16 + j % 16 for j in range(48)]
        kd, vd = k.to(DEV).contiguous(), s.v.to(DEV).contiguous()
        nnv.nnv_qk_norm_rope(s.d, 48, None, 0, kd, 128, vd, 128, None, None, None, ints([0] * 48), ints(slots, torch.int64), None, None, s.cache)
        s.held_k = OS.round_head(k.double().numpy(), dtype == nnv.F16)
        s.check_bounds()


def test_bounds_follow_the_tokens_of_one_block():
    """A block that takes a token after the other: its bounds hold those that are there, whatever lay behind."""
    s = Scene(layer(block_tokens=16, head_dim=64), [16], [1])
    for n in range(1, 17):
        s.lengths = [n]
        s.check_bounds()


# ---- selection

@pytest.mark.parametrize("lengths,fresh", [([1], [1]), ([300, 0, 64, 700], [1, 0, 1, 1]), ([257, 100, 3], [40, 100, 3]), ([2000, 40], [3, 17])], ids=str)
@pytest.mark.parametrize("heads,dim,dtype", [((8, 2), 128, nnv.BF16), ((3, 3), 64, nnv.F16), ((5, 1), 256, nnv.BF16), ((16, 1), 64, nnv.BF16), ((40, 2), 128, nnv.F16), ((2, 1), 64, nnv.F16)], ids=str)
def test_selection(lengths, fresh, heads, dim, dtype):
    s = Scene(layer(head_dim=dim, q_heads=heads[0], kv_heads=heads[1], block_tokens=16, dtype=dtype), lengths, fresh, padding=2)
    for keep, first, last in ((1, 0, 0), (3, 1, 2), (7, 0, 4), (40, 2, 1)):
        s.check_select(keep, first, last)


@pytest.mark.parametrize("count", [512, 513, 2048, 2049, 8192, 8193])
def test_selection_among_many_blocks(count):
    """Table widths around those that the kernels' registers are cut for; bounds of a few values, so that many scores are equal."""
    s = Scene(layer(block_tokens=16, head_dim=64, q_heads=2, kv_heads=1), [count * 16 - 3], [2])
    g = torch.Generator().manual_seed(count)
    pool = torch.sort(torch.randint(-2, 3, (40, 1, 2, 64), generator=g).to(torch.bfloat16), 2, descending=True).values
    bounds = pool[torch.randint(40, (s.d.blocks,), generator=g)].contiguous().to(DEV)
    for keep, first, last in ((1, 0, 0), (33, 1, 2), (300, 0, 0), (count - 1, 1, 1), (count + 5, 0, 1)):
        s.check_select(keep, first, last, bounds)


@pytest.mark.parametrize("heads,lengths,fresh", [((16, 8), [8300, 3000] + [1, 40, 700, 16] * 9, [1] * 38), ((128, 8), [8300, 50], [20, 14]), ((64, 8), [600, 8300], [9, 60]),
                                                 ((136, 8), [8300], [33])], ids=["single", "wide heads", "rows together", "seventeen heads"])
def test_selection_in_one_launch(heads, lengths, fresh):
    """As many rows and heads as keep the chip busy with a workgroup each."""
    s = Scene(layer(block_tokens=16, head_dim=64, q_heads=heads[0], kv_heads=heads[1]), lengths, fresh, padding=3)
    assert 512 < s.d.table_blocks <= 1024
    s.positions[2] = -1
    for keep, first, last in ((7, 1, 2), (600, 0, 0)):
        s.check_select(keep, first, last)


@pytest.mark.parametrize("count", [300, 513, 1025, 2049])
def test_selection_of_many_rows_among_many_blocks(count):
    """A wavefront to a row and head, for each number of keys that its lanes hold; bounds of a few values, so that many scores are equal."""
    s = Scene(layer(block_tokens=16, head_dim=64, q_heads=8, kv_heads=8), [count * 16 - 5, 100], [66, 3], padding=1)
    g = torch.Generator().manual_seed(count)
    pool = torch.sort(torch.randint(-2, 3, (200, 8, 2, 64), generator=g).to(torch.bfloat16), 2, descending=True).values
    bounds = pool[torch.randint(200, (s.d.blocks,), generator=g)].contiguous().to(DEV)
    s.positions[4] = -1
    s.table[0][3] = -1
    for keep, first, last in ((9, 1, 2), (count - 2, 0, 1)):
        s.check_select(keep, first, last, bounds)


def test_selection_of_equal_scores():
    s = Scene(layer(block_tokens=16, head_dim=64), [400, 90], [3, 1])
    for value in (0.0, -0.0, 1.5):
        bounds = torch.full((s.d.blocks, 2, 2, 64), value, dtype=torch.bfloat16, device=DEV)
        s.check_select(5, 1, 1, bounds)
        s.check_select(4, 0, 0, bounds)
    s.q[:] = 0
    s.check_select(6, 0, 2)


def test_selection_of_negative_factors_and_of_none():
    for scale in (-0.1, 0.0):
        Scene(layer(block_tokens=16, scale=scale), [300, 20], [2, 1]).check_select(5, 1, 0)


def test_selection_where_blocks_are_none():
    s = Scene(layer(block_tokens=16, head_dim=64), [300, 200], [4, 30], padding=3)
    s.positions[1] = s.positions[10] = -1
    s.table[0][0], s.table[0][7], s.table[0][18] = -5, 10 ** 8, s.d.blocks
    s.table[1] = [-1] * len(s.table[1])
    for keep, first, last in ((5, 1, 1), (40, 0, 0), (2, 0, 0)):
        s.check_select(keep, first, last)


def test_selection_by_queries_that_are_not_numbers():
    s = Scene(layer(block_tokens=16, head_dim=64, q_heads=4, kv_heads=2), [300], [5])
    s.q[1, 0, 3] = float("inf")
    s.q[2, 2:, 0] = -float("inf")
    s.check_select(4, 0, 1)
    s.q[3] = float("nan")
    got = s.select(4, 0, 1, torch.from_numpy(s.all_bounds()).to(torch.bfloat16).to(DEV)).cpu().numpy()
    blocks = np.arange(19)
    for h in range(2):
        assert len(set(got[3, h])) == 4 and np.isin(got[3, h], blocks).all() and (np.diff(got[3, h]) > 0).all()


def test_selection_positions_behind_the_length():
    s = Scene(layer(block_tokens=16, head_dim=64), [100, 33], [1, 1])
    s.positions = [2 ** 31 - 1, 500]
    s.check_select(3, 1, 1)


def test_selection_of_rows_in_several_parts():
    """More scores than are kept at a time."""
    s = Scene(layer(block_tokens=16, head_dim=64, q_heads=8, kv_heads=8), [400, 130], [128, 130])
    s.d.table_blocks = 32768
    s.table = [row + [-1] * (32768 - len(row)) for row in s.table]
    assert nnv.nnv_kv_select_workspace_bytes(s.d, 2, s.rows) == 128 * 8 * 32768 * 8 < s.rows * 8 * 32768 * 8
    bounds = torch.from_numpy(s.all_bounds()).to(torch.bfloat16).to(DEV)
    got = s.select(5, 1, 1, bounds).cpu().numpy()
    s.table = [row[:25] for row in s.table]
    s.d.table_blocks = 25
    assert np.array_equal(got, s.check_select(5, 1, 1, bounds).cpu().numpy())


# ---- attention

@pytest.mark.parametrize("lengths,fresh", LENGTHS, ids=str)
@pytest.mark.parametrize("block", [16, 32, 64, 256])
def test_attention(lengths, fresh, block):
    for dim, heads, dtype in ((64, (6, 3), nnv.F16), (128, (8, 2), nnv.BF16), (256, (5, 1), nnv.BF16)):
        s = Scene(layer(head_dim=dim, q_heads=heads[0], kv_heads=heads[1], block_tokens=block, dtype=dtype, scale=dim ** -0.5), lengths, fresh, padding=2)
        for keep in (1, 3, 8):
            s.check_attend(s.lists(keep))


@pytest.mark.parametrize("heads", [(1, 1), (16, 1), (17, 1), (40, 2), (35, 7), (64, 1)], ids=str)
@pytest.mark.parametrize("dtype", [nnv.F16, nnv.BF16])
def test_attention_of_groups(heads, dtype):
    s = Scene(layer(q_heads=heads[0], kv_heads=heads[1], block_tokens=32, dtype=dtype), [270, 5], [3, 1])
    s.check_attend(s.lists(5))


@pytest.mark.parametrize("block,keep", [(16, 300), (16, 129), (64, 70), (256, 17)])
def test_attention_over_lists_that_are_split(block, keep):
    """Longer lists than a wavefront looks up at a time, in several splits; the same from run to run."""
    s = Scene(layer(head_dim=64, block_tokens=block, q_heads=4, kv_heads=1), [block * 300 + 5 if block < 256 else 5000, 900], [2, 1])
    assert nnv.nnv_kv_attention_blocks_workspace_bytes(s.d, 2, 3, keep) > 0
    lists = s.lists(keep)
    first = s.check_attend(lists)
    assert np.array_equal(first, s.attend(lists))


def test_attention_over_long_lists_of_many_rows():
    """As many rows as need no splits, each over more than one round of lookups."""
    s = Scene(layer(head_dim=64, block_tokens=16, q_heads=16, kv_heads=16), [4000], [70])
    lists = s.lists(240)
    assert nnv.nnv_kv_attention_blocks_workspace_bytes(s.d, 1, 70, 240) == 0
    got = s.attend(lists)
    for r in (0, 1, 35, 69):
        one = Scene(layer(head_dim=64, block_tokens=16, q_heads=16, kv_heads=16), [4000], [70])
        one.q[:r], one.q[r + 1:] = 0, 0
        assert np.array_equal(one.attend(lists)[r], got[r])
    rows = [0, 69]
    s.q, s.positions, s.rows = s.q[rows], [s.positions[r] for r in rows], 2
    s.starts, s.fresh = [0, 2], [2]
    s.check_attend(lists[rows].contiguous())


def test_attention_over_lists_of_any_kind():
    """Orders other than ascending, blocks given twice, behind the position, behind the table, negative ones between others, nothing at all."""
    s = Scene(layer(block_tokens=16, head_dim=64, q_heads=4, kv_heads=2), [300, 40], [3, 1], padding=1)
    none, big = -2 ** 31, 2 ** 31 - 1
    lists = [[[5, 3, 18, 0, 1], [2, 2, 2, 7, 7]], [[-1, -1, 4, -1, 9], [none, big, 18, 10 ** 6, 19]], [[none] * 5, [big] * 5],
             [[2, 1, 0, 0, 3], [100, -7, 2, 2, 1]], [[0, 1, 2, 3, 4]] * 2]
    got = s.check_attend(ints(lists))
    assert (got[2] == 0).all() and (got[4] == 0).all()


def test_attention_where_blocks_are_none():
    s = Scene(layer(block_tokens=16, head_dim=128), [300, 200], [4, 3], padding=2)
    s.positions[1] = -1
    s.table[0][3], s.table[0][7] = -5, 10 ** 8
    s.table[1] = [-1] * len(s.table[1])
    lists = s.lists(19)
    got = s.check_attend(lists)
    assert (got[1] == 0).all() and (got[4:] == 0).all()


def test_rows_without_any_request():
    d = layer(block_tokens=16, head_dim=64)
    ws = torch.full((1 << 20,), 0xFF, dtype=torch.uint8, device=DEV)
    cache = torch.zeros(nnv.nnv_kv_cache_bytes(d), dtype=torch.uint8, device=DEV)
    bounds = torch.zeros(nnv.nnv_kv_bounds_bytes(d), dtype=torch.uint8, device=DEV)
    q, out = torch.ones(3, 8, 64, dtype=torch.bfloat16, device=DEV), torch.full((3, 8, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    selected = torch.full((3, 2, 4), 7, dtype=torch.int32, device=DEV)
    none, starts, positions = None, ints([0]), ints([5, 0, -1])
    nnv.nnv_kv_bounds(d, 0, 3, none, starts, none, cache, bounds)
    nnv.nnv_kv_select(d, 0, 3, 4, 1, 1, q, none, starts, none, positions, bounds, selected, ws)
    nnv.nnv_kv_attention_blocks(d, 0, 3, 4, q, none, starts, none, positions, selected, cache, out, ws)
    torch.cuda.synchronize()
    assert (selected == -1).all() and (out == 0).all()


def test_all_blocks_are_attention():
    """Lists of all that a row sees: the definition of attention over the whole cache."""
    for fresh in ([1, 1], [70, 5]):
        s = Scene(layer(block_tokens=32), [500, 77], fresh)
        every = torch.arange(16, dtype=torch.int32, device=DEV).expand(s.rows, 2, 16).contiguous()
        s.check_attend(every)


def test_starts_and_lengths_out_of_range_do_no_harm():
    s = Scene(layer(block_tokens=16, head_dim=64), [300, 40], [3, 1])
    bounds = torch.from_numpy(s.all_bounds()).to(torch.bfloat16).to(DEV)
    lists = s.lists(4)
    for starts, lengths in (([0, 50, -9], [10 ** 9, -5]), ([-5, 2, 10 ** 9], [2 ** 31 - 1, 2 ** 31 - 1]), ([4, 2, 0], [300, 40])):
        s.starts, s.lengths = starts, lengths
        s.select(4, 1, 1, bounds)
        s.attend(lists)
        scratch = bounds.clone()
        nnv.nnv_kv_bounds(s.d, 2, s.rows, *s.plan(), s.cache, scratch)
        torch.cuda.synchronize()


def test_the_three_together_in_a_graph_and_on_another_stream():
    s = Scene(layer(block_tokens=16, head_dim=64), [400, 90, 17], [1, 1, 1])
    table, starts, lengths = s.plan()
    q, positions = s.q.to(DEV), ints(s.positions)
    bounds = torch.zeros(nnv.nnv_kv_bounds_bytes(s.d) // 2, dtype=torch.bfloat16, device=DEV).view(-1, 2, 2, 64)
    every = torch.from_numpy(s.all_bounds()).to(torch.bfloat16).to(DEV)
    selected = torch.zeros(3, 2, 6, dtype=torch.int32, device=DEV)
    out = torch.zeros(3, 8, 64, dtype=torch.bfloat16, device=DEV)
    ws = torch.zeros(max(nnv.nnv_kv_select_workspace_bytes(s.d, 3, 3), nnv.nnv_kv_attention_blocks_workspace_bytes(s.d, 3, 3, 6)), dtype=torch.uint8, device=DEV)

    def step():
        nnv.nnv_kv_bounds(s.d, 3, 3, table, starts, lengths, s.cache, bounds)
        nnv.nnv_kv_select(s.d, 3, 3, 6, 1, 2, q, table, starts, lengths, positions, bounds, selected, ws)
        nnv.nnv_kv_attention_blocks(s.d, 3, 3, 6, q, table, starts, lengths, positions, selected, s.cache, out, ws)

    bounds.copy_(every)
    want_lists = s.check_select(6, 1, 2)
    want = s.check_attend(want_lists)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert torch.equal(selected, want_lists) and np.array_equal(out.double().cpu().numpy(), want) and torch.equal(bounds, every)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        s.q = torch.randn(s.q.shape, generator=torch.Generator().manual_seed(turn)).to(s.q.dtype)
        q.copy_(s.q)
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        want_lists = s.check_select(6, 1, 2)
        assert torch.equal(selected, want_lists) and np.array_equal(out.double().cpu().numpy(), s.attend(want_lists))
