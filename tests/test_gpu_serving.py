"""The plan of a step, norms and rotations with the append to a 4-bit cache, and attention over it, against their definitions.

Tolerances.  Plans, codes and held values are exact.  A query's norm and rotation are float32: its sum of dim squares, a root, a quotient and
five products and sums err by at most (dim / 2 + 12) * 2^-24 of the sum of the terms' magnitudes, the store by half a
step.  Attention: a float32 score is off by at most score_bound(), and its weight by that factor, twice where numerator and denominator
differ; weights are rounded to the 16-bit type for the products (half a step each), sums over n tokens and the joins are float32
(n + 64 roundings, at most 2^-23 each on the matrix cores), the store adds half a step."""
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


# ---- plan ---------------------------------------------------------------------------------------

def run_plan(held, fresh, free, count, table, block, blocks, rows):
    n, width = len(held), len(table[0]) if table else 3
    d = layer(block_tokens=block, blocks=blocks, table_blocks=width)
    t = ints(table).reshape(n, width) if n else ints([0])
    out = [torch.full((v + 1,), -7, dtype=w, device=DEV) for v, w in ((n + 1, torch.int32), (n, torch.int32), (rows, torch.int32), (rows, torch.int64), (1, torch.int32))]
    free = ints(list(free) or [0])
    print(f"case plan n={n} rows={rows} block={block} blocks={blocks} count={count}", flush=True)
    for _ in range(2):                                   # a call can be repeated
        nnv.nnv_kv_plan(d, n, rows, ints(held or [0]), ints(fresh or [0]), free, ints([count]), t, *out)
    torch.cuda.synchronize()
    assert all(int(o[-1]) == -7 for o in out)
    got = [t.tolist() if n else [], *[o[:-1].tolist() for o in out]]
    want = OS.plan(held, fresh, free.tolist(), count, table, block, blocks, rows)
    for a, b, name in zip(got, [*want[:5], [want[5]]], ("table", "starts", "lengths", "positions", "slots", "left")):
        assert a == list(b), name


PLANS = {
    "one": ([0], [1], 1), "none": ([], [], 0), "no rows": ([5, 0, 64], [0, 0, 0], 0), "edges": ([15, 16, 17, 0, 31, 63, 64], [1, 1, 1, 16, 1, 1, 0], 21),
    "prompts": ([0, 100, 3, 0], [200, 1, 0, 77], 278), "padded": ([0, 7], [3, 2], 9), "cut": ([0, 7, 2], [3, 4, 2], 5), "negative": ([4, -3, 5], [1, 1, -6], 2),
    "too long": ([1000, 0, 64000], [60000, 2, 2 ** 31 - 1], 60002),
}


@pytest.mark.parametrize("block", [16, 64, 256])
@pytest.mark.parametrize("name", list(PLANS))
def test_plan(name, block):
    held, fresh, rows = PLANS[name]
    width = 40
    g = np.random.default_rng(3)
    blocks = 300
    order = list(map(int, g.permutation(blocks)))
    table = []
    for h in held:
        k = min(width, max(0, -(-h // block)))
        table.append([order.pop() for _ in range(k)] + [-1] * (width - k))
    for count in (len(order), 3, 0, -5, 10 ** 6):
        free = order + [1] * (blocks - len(order))
        run_plan(held, fresh, free, count, table, block, blocks, rows)


@pytest.mark.parametrize("n", [1, 63, 1023, 1024, 1025, 2500])
@pytest.mark.parametrize("share", [1.0, 0.4])
def test_plan_of_many_requests(n, share):
    g = np.random.default_rng(n)
    block, width = 16, 12
    held = [int(v) for v in g.integers(0, 100, n)]
    fresh = [int(v) for v in np.where(g.random(n) < 0.7, 1, g.integers(0, 90, n))]
    need = [-(-h // block) for h in held]
    new = sum(-(-(h + f) // block) for h, f in zip(held, fresh)) - sum(need)
    count = int(share * new) + (1 if share == 1 else 0)
    order = list(map(int, g.permutation(sum(need) + count)))
    table = [[order.pop() for _ in range(k)] + [-1] * (width - k) for k in need]
    if n > 3:
        table[2] = [99999] * width                       # entries that are no block
    run_plan(held, fresh, order, count, table, block, sum(need) + count, sum(fresh) + 5)


@pytest.mark.parametrize("n,share", [(2048, 1.0), (2049, 1.0), (4096, 0.5), (4097, 1.0), (9001, 0.7), (9001, 1.0)])
def test_plan_of_thousands_of_requests(n, share):
    """One chunk of requests filled, one more than that, and several."""
    g = np.random.default_rng(n)
    block, width = 16, 6
    held = [int(v) for v in g.integers(0, 60, n)]
    fresh = [int(v) for v in np.where(g.random(n) < 0.9, 1, g.integers(0, 30, n))]
    need = [-(-h // block) for h in held]
    new = sum(-(-(h + f) // block) for h, f in zip(held, fresh)) - sum(need)
    count = int(share * new)
    order = list(map(int, g.permutation(sum(need) + count)))
    table = [[order.pop() for _ in range(k)] + [-1] * (width - k) for k in need]
    run_plan(held, fresh, order, count, table, block, sum(need) + count, sum(fresh))


@pytest.mark.parametrize("heads", [(1, 1), (3, 1), (7, 7)], ids=str)
@pytest.mark.parametrize("norm", [True, False])
def test_norm_rope_of_odd_heads(heads, norm):
    """Heads that are no multiple of those a thread takes, rotations of half a head in pairs, rows of any stride."""
    d = layer(q_heads=heads[0], kv_heads=heads[1], rotary_dim=64, rotary_interleaved=1, positions=50, block_tokens=16, blocks=4)
    g = torch.Generator().manual_seed(11)
    rows, (q, kv) = 33, heads
    for stride in ((q + 2 * kv) * 128, (q + 2 * kv) * 128 + 3):
        x = torch.randn(rows, stride, generator=g).to(torch.bfloat16)
        weight = 1 + 0.2 * torch.randn(2, 128, generator=g)
        table, pos = angles(50, 64), torch.randint(50, (rows,), generator=g).tolist()
        out = torch.full((rows + 1, q, 128), 7.0, dtype=torch.bfloat16, device=DEV)
        out_k = torch.full((rows + 1, kv, 128), 7.0, dtype=torch.bfloat16, device=DEV)
        # each part from the start of a buffer of its own, so that a stride of any size keeps it aligned
        parts = [p.contiguous() for p in (x, x[:, q * 128:], x[:, (q + kv) * 128:])]
        on = [p.to(DEV) for p in parts]
        w = [t.to(DEV) if norm else None for t in weight]
        cache = torch.zeros(nnv.nnv_kv_cache_bytes(d), dtype=torch.uint8, device=DEV)
        print(f"case rope heads={heads} norm={norm} stride={stride}", flush=True)
        nnv.nnv_qk_norm_rope(d, rows, on[0], on[0].stride(0), on[1], on[1].stride(0), on[2], on[2].stride(0), *w, table.to(DEV), ints(pos), ints(list(range(rows)), torch.int64),
                             out, out_k, cache)
        torch.cuda.synchronize()
        assert (out[-1] == 7).all() and (out_k[-1] == 7).all()
        u = torch.finfo(torch.bfloat16).eps / 2
        for got, part, n, wt, steps in ((out, parts[0], q, weight[0], 64 + 12), (out_k, parts[1], kv, weight[1], 0)):
            ref, size = OS.norm_rope(part[:, : n * 128].double().numpy().reshape(rows, n, 128), wt.double().numpy() if norm else None, d.eps,
                                     table.double().numpy()[pos], 64, True)
            # queries: float32 (see above); keys: float64, of which the float32 of odd last bit is off by a step of 2^-23 at most
            bound = (steps * 2.0 ** -24 + 2.0 ** -23) * size * (1 + 2.0 ** -6) + u * (1 + 2.0 ** -6) * np.abs(ref) + 1e-37
            assert (np.abs(got[:-1].double().cpu().numpy() - ref) <= bound).all()
        held = [torch.empty(rows, kv, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        nnv.nnv_kv_read(d, rows, ints(list(range(rows)), torch.int64), cache, *held)
        v = parts[2][:, : kv * 128].double().numpy().reshape(rows, kv, 128)
        assert np.array_equal(held[1].double().cpu().numpy(), OS.round_head(v, False))


# ---- norms, rotations, append -------------------------------------------------------------------

def angles(positions, rotary, seed=2):
    g = torch.Generator().manual_seed(seed)
    a = torch.rand(positions, rotary // 2, generator=g, dtype=torch.float64) * 6.3
    return torch.cat((a.cos(), a.sin()), 1).float()


def run_rope(d, rows, x, positions, slots, norm, pad=0, k_out=True, cache=None):
    """x: (rows, q_heads + 2 kv_heads, dim) on the host -> q, k outputs, the cache."""
    q, kv, dim, t = d.q_heads, d.kv_heads, d.head_dim, T[d.dtype]
    stride = (q + 2 * kv) * dim + pad
    buf = torch.full((rows, stride), float("nan"), dtype=t)
    buf[:, : stride - pad] = x.reshape(rows, -1)
    buf = buf.to(DEV)
    g = torch.Generator().manual_seed(9)
    weights = [torch.rand(dim, generator=g) + 0.5 for _ in range(2)] if norm else [None, None]
    table = angles(d.positions, d.rotary_dim).to(DEV) if d.rotary_dim else None
    qo = torch.full((rows, q, dim), 7.0, dtype=t, device=DEV)
    ko = torch.full((rows, kv, dim), 7.0, dtype=t, device=DEV) if k_out else None
    cache = torch.full((nnv.nnv_kv_cache_bytes(d),), 0xFF, dtype=torch.uint8, device=DEV) if cache is None else cache
    parts = buf[:, : q * dim], buf[:, q * dim:(q + kv) * dim], buf[:, (q + kv) * dim:]
    print(f"case rope rows={rows} heads={q}/{kv} dim={dim} rotary={d.rotary_dim} interleaved={d.rotary_interleaved} type={d.dtype} norm={norm} pad={pad}", flush=True)
    nnv.nnv_qk_norm_rope(d, rows, parts[0], stride, parts[1], stride, parts[2], stride, *[w if w is None else w.to(DEV) for w in weights], table,
                         ints(positions), ints(slots, torch.int64), qo, ko, cache)
    torch.cuda.synchronize()
    return qo, ko, cache, weights, None if table is None else table.double().cpu().numpy()


def read(d, slots, cache):
    n = len(slots)
    k, v = (torch.full((n, d.kv_heads, d.head_dim), 7.0, dtype=T[d.dtype], device=DEV) for _ in range(2))
    nnv.nnv_kv_read(d, n, ints(slots, torch.int64), cache, k, v)
    torch.cuda.synchronize()
    return k.double().cpu().numpy(), v.double().cpu().numpy()


ROPES = [(64, 64, 0), (64, 32, 1), (64, 30, 0), (128, 128, 0), (128, 128, 1), (128, 64, 0), (128, 72, 0), (128, 22, 1), (128, 0, 0), (256, 256, 0), (256, 128, 1), (256, 2, 0)]


@pytest.mark.parametrize("dtype", [nnv.F16, nnv.BF16])
@pytest.mark.parametrize("dim,rotary,interleaved", ROPES)
def test_norm_rope_append(dim, rotary, interleaved, dtype):
    for heads, norm, block, pad in (((8, 2), True, 16, 0), ((3, 3), False, 256, 8), ((5, 1), True, 64, 3)):
        pad = 0 if pad == 3 and False else pad
        rows = 37
        d = layer(q_heads=heads[0], kv_heads=heads[1], head_dim=dim, block_tokens=block, blocks=600 // block, rotary_dim=rotary, rotary_interleaved=interleaved,
                  positions=50, dtype=dtype)
        g = torch.Generator().manual_seed(dim + rotary)
        x = torch.randn(rows, heads[0] + 2 * heads[1], dim, generator=g).to(T[dtype])
        positions = torch.randint(50, (rows,), generator=g).tolist()
        slots = torch.randperm(d.blocks * block, generator=g)[:rows].tolist()
        positions[3], positions[4], slots[5], slots[6] = -1, 50 if rotary else -9, -1, d.blocks * block
        qo, ko, cache, weights, table = run_rope(d, rows, x, positions, slots, norm, pad)
        xs = x.double().numpy()
        empty = np.array([p < 0 or (rotary > 0 and p >= 50) for p in positions])
        at = np.zeros((rows, max(rotary, 1))) if table is None else table[np.clip(positions, 0, 49)]
        w = [None if v is None else v.double().numpy() for v in weights]
        refs = [OS.norm_rope(p, wt, float(np.float32(1e-6)), at, rotary, interleaved) for p, wt in
                ((xs[:, : heads[0]], w[0]), (xs[:, heads[0]:heads[0] + heads[1]], w[1]))]
        half = torch.finfo(T[dtype]).eps / 2
        tiny = float(torch.finfo(T[dtype]).smallest_normal)
        for got, (ref, size) in zip((qo, ko), refs):
            got = got.double().cpu().numpy()
            assert (got[empty] == 0).all()
            bound = (dim / 2 + 12) * 2.0 ** -24 * size + half * (1 + 2.0 ** -10) * np.abs(ref) + tiny
            assert (np.abs(got - ref)[~empty] <= bound[~empty]).all()
        kept = ~empty & np.array([0 <= s < d.blocks * block for s in slots])
        k, v = read(d, slots, cache)
        assert np.array_equal(k[kept], OS.round_head(refs[1][0], dtype == nnv.F16)[kept])
        assert np.array_equal(v[kept], OS.round_head(xs[:, heads[0] + heads[1]:], dtype == nnv.F16)[kept])
        # nothing else of the cache was written: its bytes are as they were
        per = nnv.nnv_kv_cache_bytes(d)
        assert int((cache == 0xFF).sum()) >= per - kept.sum() * heads[1] * (dim + dim // 16)
        out_of_cache = [i for i, s in enumerate(slots) if not 0 <= s < d.blocks * block]
        assert (k[out_of_cache] == 0).all() and (v[out_of_cache] == 0).all()


@pytest.mark.parametrize("dtype", [nnv.F16, nnv.BF16])
def test_held_values_of_every_kind(dtype):
    """Ties between codes, the borders of a scale, zeros of both signs, the smallest and largest numbers, NaN and infinities."""
    d = layer(q_heads=1, kv_heads=1, head_dim=64, block_tokens=16, blocks=8, dtype=dtype)
    t, rows = T[dtype], 60
    g = torch.Generator().manual_seed(4)
    x = torch.randn(rows, 3, 64, generator=g)
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5, -6, 0.0, -0.0] + [4.0] * 46)
    for r in range(20):
        x[r, 1:] = ties * 2.0 ** (r - 10)
    x[20, 1:] = 0
    x[21, 1:] = torch.finfo(t).tiny
    x[22, 1:] = torch.finfo(t).smallest_normal * 3
    x[23, 1:] = torch.finfo(t).max
    x[24, 1:, 3] = float("inf")
    x[25, 1:, 40] = float("-inf")
    x[26, 1:, 5] = float("nan")
    x[27, 1:] = float("nan")
    for i, v in enumerate((3.484375, 3.5, 6.96875, 7.0, 7.03125, 5.0, 2.5)):
        x[30 + i, 1:] = torch.linspace(-1, 1, 64) * v
    x = x.to(t)
    slots = list(range(rows, 0, -1))
    _, _, cache, _, _ = run_rope(d, rows, x, [0] * rows, slots, False)
    k, v = read(d, slots, cache)
    for got, part in ((k[:, 0], 1), (v[:, 0], 2)):
        want = OS.round_head(x.double().numpy()[:, part], dtype == nnv.F16)
        # values below the 16-bit type's normal range are read back rounded
        same = (got == want) | ((np.abs(want) < torch.finfo(t).tiny) & (np.abs(got - want) <= float(torch.finfo(t).tiny) * float(torch.finfo(t).eps)))
        assert same.all()


def test_rope_without_cache_or_queries():
    d = layer(rotary_dim=128, positions=40)
    g = torch.Generator().manual_seed(8)
    x = torch.randn(20, 12, 128, generator=g).to(torch.bfloat16).to(DEV)
    pos, slots, table = ints(list(range(20))), ints(list(range(20)), torch.int64), angles(40, 128).to(DEV)
    q, k, v = (t.contiguous() for t in x.split((8, 2, 2), 1))
    cache = torch.zeros(nnv.nnv_kv_cache_bytes(d), dtype=torch.uint8, device=DEV)
    both = [torch.empty_like(q), torch.empty_like(k)]
    nnv.nnv_qk_norm_rope(d, 20, q, 1024, k, 256, v, 256, None, None, table, pos, slots, *both, cache)
    only = [torch.empty_like(q), torch.empty_like(k)]
    nnv.nnv_qk_norm_rope(d, 20, q, 1024, None, 0, None, 0, None, None, table, pos, None, only[0], None, None)
    nnv.nnv_qk_norm_rope(d, 20, None, 0, k, 256, None, 0, None, None, table, pos, None, None, only[1], None)
    held = torch.zeros_like(cache)
    nnv.nnv_qk_norm_rope(d, 20, None, 0, k, 256, v, 256, None, None, table, pos, slots, None, None, held)
    torch.cuda.synchronize()
    assert torch.equal(both[0], only[0]) and torch.equal(both[1], only[1]) and torch.equal(cache, held) and cache.any()


# ---- attention ----------------------------------------------------------------------------------

class Scene:
    """Requests of given lengths with their last rows as queries, blocks in no order, and 0xFF wherever nothing is held."""

    def __init__(self, d, lengths, fresh, seed=1, padding=0, stray=0):
        self.d, self.lengths, self.fresh = d, lengths, fresh
        g = torch.Generator().manual_seed(seed)
        block, kv, dim, t = d.block_tokens, d.kv_heads, d.head_dim, T[d.dtype]
        need = [-(-n // block) for n in lengths]
        d.blocks, d.table_blocks = sum(need) + 2, max(need + [1])
        order = torch.randperm(d.blocks, generator=g).tolist()
        table = [[order.pop() for _ in range(k)] + [10 ** 8] * (d.table_blocks - k) for k in need]
        total = sum(lengths)
        x = torch.randn(total, 1 + 2 * kv, dim, generator=g).to(t)
        self.k, self.v = x[:, 1:1 + kv], x[:, 1 + kv:]
        slots = [table[i][j // block] * block + j % block for i, n in enumerate(lengths) for j in range(n)]
        self.cache = torch.full((nnv.nnv_kv_cache_bytes(d),), 0xFF, dtype=torch.uint8, device=DEV)
        if total:
            kd, vd = self.k.to(DEV).contiguous(), self.v.to(DEV).contiguous()
            nnv.nnv_qk_norm_rope(d, total, None, 0, kd, kv * dim, vd, kv * dim, None, None, None, ints([0] * total), ints(slots, torch.int64), None, None, self.cache)
        self.rows = sum(fresh) + padding
        self.q = torch.randn(self.rows, d.q_heads, dim, generator=g).mul(1.5).to(t)
        self.starts = [0]
        for f in fresh:
            self.starts.append(self.starts[-1] + f)
        self.positions = [n - f + r for n, f in zip(lengths, fresh) for r in range(f)] + [-1] * padding
        self.table = table

    def run(self, workspace=None):
        d = self.d
        need = nnv.nnv_kv_attention_workspace_bytes(d, len(self.lengths), self.rows)
        ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device=DEV) if workspace is None else workspace
        out = torch.full((self.rows + 1, d.q_heads, d.head_dim), 7.0, dtype=T[d.dtype], device=DEV)
        print(f"case attend lengths={self.lengths[:6]} fresh={self.fresh[:6]} heads={d.q_heads}/{d.kv_heads} dim={d.head_dim} block={d.block_tokens} "
              f"window={d.window} sinks={d.sinks} type={d.dtype} workspace={need}", flush=True)
        nnv.nnv_kv_attention(d, len(self.lengths), self.rows, self.q.to(DEV), ints(self.table or [0]), ints(self.starts), ints(self.lengths or [0]), ints(self.positions),
                             self.cache, out, ws, need)
        torch.cuda.synchronize()
        assert (out[-1] == 7).all() and (ws[need:] == 0xFF).all(), "written behind the buffers"
        return out[:-1].double().cpu().numpy()

    def check(self, got=None, hidden=None):
        """hidden: per request, tokens that may not be seen."""
        d = self.d
        got = self.run() if got is None else got
        half = d.dtype == nnv.F16
        k, v = OS.round_head(self.k.double().numpy(), half), OS.round_head(self.v.double().numpy(), half)
        u, at, used = torch.finfo(T[d.dtype]).eps / 2, 0, 0
        for i, (n, f) in enumerate(zip(self.lengths, self.fresh)):
            rows = slice(self.starts[i], self.starts[i + 1])
            seen = None if hidden is None else ~np.isin(np.arange(n), hidden[i])
            ref, size, most = OS.attention(self.q[rows].double().numpy(), k[at:at + n], v[at:at + n], self.positions[rows], d.scale, d.window, d.sinks, seen)
            bound = (u + 2 * OS.score_bound(d.head_dim, most) + (n + 64) * 2.0 ** -23) * size * (1 + 2.0 ** -6) + u * (1 + 2.0 ** -6) * np.abs(ref) + float(torch.finfo(T[d.dtype]).tiny)
            worst = (np.abs(got[rows] - ref) / bound).max() if f else 0
            assert worst <= 1, f"request {i} of {n}: {worst:.3f} of the bound"
            at += n
            used += f
        assert (got[used:] == 0).all()
        return got


LENGTHS = [[1], [0], [2, 15, 16, 17], [31, 32, 33, 64, 65], [100, 1, 0, 300], [127, 128, 129], [1000], [63, 700, 255, 256, 257]]


@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda v: "-".join(map(str, v)))
@pytest.mark.parametrize("block", [16, 64, 256])
def test_single_rows(lengths, block):
    for dim, heads, dtype in ((128, (8, 2), nnv.BF16), (64, (6, 6), nnv.F16), (256, (5, 1), nnv.BF16)):
        Scene(layer(head_dim=dim, q_heads=heads[0], kv_heads=heads[1], block_tokens=block, dtype=dtype, scale=dim ** -0.5), lengths, [min(1, n) for n in lengths]).check()


@pytest.mark.parametrize("heads", [(1, 1), (4, 4), (16, 1), (20, 1), (40, 2), (24, 8), (35, 7)], ids=str)
@pytest.mark.parametrize("dtype", [nnv.F16, nnv.BF16])
def test_groups(heads, dtype):
    for fresh in ([1, 1, 1], [3, 0, 5]):
        Scene(layer(q_heads=heads[0], kv_heads=heads[1], block_tokens=32, dtype=dtype), [70, 5, 200], fresh).check()


@pytest.mark.parametrize("dim,dtype", [(64, nnv.BF16), (128, nnv.F16), (128, nnv.BF16), (256, nnv.F16)])
@pytest.mark.parametrize("lengths,fresh", [([40], [40]), ([17, 100, 260], [17, 33, 130]), ([1, 2, 300, 90], [1, 2, 1, 64]), ([300], [70])], ids=str)
def test_many_rows(lengths, fresh, dim, dtype):
    Scene(layer(head_dim=dim, q_heads=4, kv_heads=2, block_tokens=16, dtype=dtype, scale=dim ** -0.5), lengths, fresh, padding=3).check()


# rows and heads of a group enough that requests of 32 pairs and more go to the kernel for many rows, the others beside them
MANY = [([40], [40]), ([17, 100, 260], [17, 33, 130]), ([1, 2, 300, 90, 0], [1, 2, 1, 64, 0]), ([300, 64, 65], [70, 64, 1]), ([5, 129, 1, 500], [0, 128, 1, 3])]


@pytest.mark.parametrize("dim,dtype", [(64, nnv.BF16), (64, nnv.F16), (128, nnv.F16), (128, nnv.BF16), (256, nnv.F16), (256, nnv.BF16)])
@pytest.mark.parametrize("lengths,fresh", MANY, ids=str)
def test_many_pairs(lengths, fresh, dim, dtype):
    for heads, block in (((16, 1), 16), ((40, 2), 64)):
        Scene(layer(head_dim=dim, q_heads=heads[0], kv_heads=heads[1], block_tokens=block, dtype=dtype, scale=dim ** -0.5), lengths, fresh, padding=3).check()


@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 3), (64, 64), (100, 70), (700, 0)])
def test_many_pairs_in_windows(window, sinks):
    Scene(layer(q_heads=16, kv_heads=1, block_tokens=32, window=window, sinks=sinks), [40, 600, 333], [40, 50, 129], padding=1).check()


def test_many_pairs_of_many_requests():
    """More requests than are put in order of their lengths."""
    g = np.random.default_rng(5)
    lengths = [int(v) for v in g.integers(1, 150, 70)]
    fresh = [min(n, int(v)) for n, v in zip(lengths, g.integers(0, 12, 70))]
    Scene(layer(q_heads=16, kv_heads=2, head_dim=64, block_tokens=16), lengths, fresh, padding=2).check()


def test_many_pairs_split_and_joined():
    s = Scene(layer(q_heads=16, kv_heads=1, block_tokens=64, head_dim=64), [9000, 700, 40], [70, 33, 1])
    assert nnv.nnv_kv_attention_workspace_bytes(s.d, 3, 104) > 0
    first = s.check()
    assert np.array_equal(first, s.run())


def test_many_pairs_where_blocks_are_none():
    s = Scene(layer(q_heads=16, kv_heads=1, block_tokens=16), [190, 200], [60, 40], padding=2)
    s.positions[3] = s.positions[70] = -1
    s.table[0][3], s.table[0][7] = -5, 10 ** 8            # tokens 48 .. 63 and 112 .. 127
    s.table[1] = [-1] * len(s.table[1])
    got = s.run()
    assert (got[[3, 70]] == 0).all() and (got[60:] == 0).all()
    s.check(got, hidden=[np.r_[48:64, 112:128], np.arange(200)])


@pytest.mark.parametrize("scale", [-0.1, 0.0])
def test_factors_that_are_not_positive(scale):
    for lengths, fresh in (([100, 20], [1, 1]), ([130, 20], [40, 1])):
        Scene(layer(q_heads=16, kv_heads=1, block_tokens=16, scale=scale), lengths, fresh).check()


@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 0), (32, 4), (33, 33), (64, 1), (100, 40), (4096, 4), (50, 1000)])
def test_windows(window, sinks):
    for lengths, fresh in (([1, 30, 64, 150, 500], [1, 1, 1, 1, 1]), ([30, 200], [30, 90])):
        Scene(layer(q_heads=4, kv_heads=2, head_dim=64, block_tokens=16, window=window, sinks=sinks), lengths, fresh).check()


@pytest.mark.parametrize("lengths,fresh", [([70, 33], [1, 2]), ([300, 20], [70, 1])], ids=str)
def test_sinks_and_windows_of_any_size(lengths, fresh):
    most = 2 ** 31 - 1
    for window, sinks in ((5, most), (most, most), (most, 0)):
        Scene(layer(q_heads=16, kv_heads=1, block_tokens=64, head_dim=64, window=window, sinks=sinks), lengths, fresh).check()


def test_long_requests_are_split_and_joined():
    s = Scene(layer(q_heads=4, kv_heads=1, block_tokens=64), [9000, 33, 5000], [1, 1, 2])
    assert nnv.nnv_kv_attention_workspace_bytes(s.d, 3, 4) > 0
    first = s.check()
    assert np.array_equal(first, s.run())
    s = Scene(layer(q_heads=4, kv_heads=1, block_tokens=64, window=3000, sinks=70), [9000, 33, 5000], [1, 1, 2])
    s.check()


def test_rows_that_see_nothing_and_blocks_that_are_none():
    s = Scene(layer(block_tokens=16), [90, 40, 55], [4, 3, 2], padding=4)
    s.positions[0] = s.positions[5] = -1                 # a whole request's first row, a row between others
    s.table[2] = [10 ** 8] * len(s.table[2])             # no block of the third
    s.table[0][2] = -5                                   # tokens 32 .. 47 of the first
    got = s.run()
    assert (got[[0, 5, 7, 8]] == 0).all()
    s.check(got, hidden=[np.arange(32, 48), [], np.arange(55)])


def test_starts_and_lengths_out_of_range_do_no_harm():
    s = Scene(layer(block_tokens=16), [90, 40], [2, 2])
    s.starts, s.lengths, s.positions = [0, -7, 10 ** 9], [10 ** 9, -5], [10 ** 9, 89, 2, -3]
    assert np.isfinite(s.run()).all()
    s.starts, s.lengths = [3, 2, 1], [90, 40]
    s.run()


@pytest.mark.parametrize("lengths,fresh", [([70, 33], [1, 2]), ([9000, 33], [1, 1]), ([300, 20], [70, 1]), ([9000, 40], [70, 1])], ids=str)
def test_queries_that_are_not_numbers(lengths, fresh):
    """A head of a row is NaN where its query holds a NaN, or an infinity (some of whose products are infinity times 0); the others are what they are."""
    s = Scene(layer(q_heads=16, kv_heads=1, block_tokens=64, head_dim=64), lengths, fresh)
    clean, want = s.q.clone(), s.run()
    s.q[0, 3, 5], s.q[fresh[0], 7, 60], s.q[fresh[0], 1, 0] = float("nan"), float("inf"), -float("inf")
    hit = np.zeros(want.shape[:2], bool)
    hit[0, 3] = hit[fresh[0], 7] = hit[fresh[0], 1] = True
    got = s.run()
    assert np.isnan(got[0, 3]).all() and not np.isfinite(got[hit]).any()
    got[hit], s.q = want[hit], clean
    s.check(got)


def test_rows_that_starts_leave_out_beside_split_requests():
    """Their partial results are whatever the workspace holds; the other rows are what they are without them."""
    s = Scene(layer(q_heads=4, kv_heads=1, block_tokens=64), [9000, 33], [3, 1])
    want = s.run()
    s.starts = [2, 3, 4]
    need = nnv.nnv_kv_attention_workspace_bytes(s.d, 2, 4)
    assert need > 0
    for word in (0x7F7F7F7F, 0x00000060, -1):
        ws = torch.full((need // 4 + 16,), word, dtype=torch.int32, device=DEV)
        ws[need // 4:] = -1
        assert np.array_equal(s.run(ws.view(torch.uint8))[2:], want[2:])


def test_positions_behind_the_length_see_what_is_held():
    s = Scene(layer(block_tokens=16), [50], [1])
    a = s.run()
    s.positions = [4000]
    assert np.array_equal(a, s.run())


def test_another_stream_and_graph():
    s = Scene(layer(q_heads=4, kv_heads=1, block_tokens=64), [3000, 70], [1, 1])
    first = s.run()
    with torch.cuda.stream(torch.cuda.Stream()):
        assert np.array_equal(first, s.run())
    d = s.d
    need = nnv.nnv_kv_attention_workspace_bytes(d, 2, 2)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    q, out = s.q.to(DEV), torch.zeros(2, 4, 128, dtype=torch.bfloat16, device=DEV)
    table, starts, lengths, positions = ints(s.table), ints(s.starts), ints(s.lengths), ints(s.positions)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nnv.nnv_kv_attention(d, 2, 2, q, table, starts, lengths, positions, s.cache, out, ws)
    for n in (3000, 40, 2999, 1):
        lengths[0], positions[0] = n, n - 1
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        s.lengths[0], s.positions[0] = n, n - 1
        assert np.array_equal(got.double().cpu().numpy(), s.run())


def test_a_cache_beyond_32_bits():
    """Blocks whose bytes lie behind 4 GiB of the cache."""
    d = layer(q_heads=2, kv_heads=1, block_tokens=256)
    d.blocks = (1 << 33) // (256 * 136)
    cache = torch.empty(nnv.nnv_kv_cache_bytes(d), dtype=torch.uint8, device=DEV)
    s = Scene(layer(q_heads=2, kv_heads=1, block_tokens=256), [600], [1])
    want = s.run()
    far = [d.blocks - 1, d.blocks // 2 + 7, d.blocks - 9]
    slots = [far[j // 256] * 256 + j % 256 for j in range(600)]
    k, v = s.k.to(DEV).contiguous(), s.v.to(DEV).contiguous()
    nnv.nnv_qk_norm_rope(d, 600, None, 0, k, 128, v, 128, None, None, None, ints([0] * 600), ints(slots, torch.int64), None, None, cache)
    d.table_blocks = 3
    s.d, s.table, s.cache = d, [far], cache
    assert np.array_equal(want, s.run())
