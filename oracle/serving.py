"""The serving operators from their definitions, in float64 on the CPU: the two low-bit formats, products with
8-bit weights, the plan of a step, norms and rotations, attention over tokens held in 4 bits."""
from __future__ import annotations

import numpy as np

E4M3 = np.array(sorted({(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8) if (e, m) != (15, 7)} | {m / 8 * 2.0 ** -6 for m in range(8)}))
E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def nearest(values, grid):
    """Magnitudes rounded to the nearest of an ascending grid of codes, halfway to the even code; signs kept."""
    a = np.minimum(np.abs(values), grid[-1])
    hi = np.clip(np.searchsorted(grid, a), 1, len(grid) - 1)
    lo = hi - 1
    below, above = a - grid[lo], grid[hi] - a
    up = (above < below) | ((above == below) & (hi % 2 == 0))
    return np.copysign(np.where(up, grid[hi], grid[lo]), values)


def scale_e4m3(amax):
    """The smallest power of two s >= 2^-126 with amax <= 448 s, of each."""
    s = np.exp2(np.where(amax > 0, np.maximum(np.frexp(amax / 448.0)[1] - 2, -126), -126).astype(float))
    while True:
        low = amax > 448 * s
        if not low.any():
            return s
        s = np.where(low, 2 * s, s)


def scale_e2m1(amax, half):
    """The smallest power of two s >= 2^-126 with amax < 7 s, of each; at most 2^13 in float16, 2^125 in bfloat16."""
    s = np.exp2(np.where(amax > 0, np.maximum(np.frexp(amax / 7.0)[1] - 2, -126), -126).astype(float))
    for _ in range(3):
        s = np.where(amax >= 7 * s, 2 * s, s)
    return np.minimum(s, 2.0 ** (13 if half else 125))


def round_rows(x):
    """Rows of x as 8 bits hold them: a scale per 128 consecutive values."""
    m, k = x.shape
    p = np.zeros((m, -(-k // 128) * 128))
    p[:, :k] = x
    b = p.reshape(m, -1, 128)
    s = scale_e4m3(np.abs(b).max(-1))[..., None]
    return (nearest(b / s, E4M3) * s).reshape(m, -1)[:, :k]


def round_weights(w):
    """Weights as 8 bits hold them: a scale per 128 x 128."""
    n, k = w.shape
    p = np.zeros((-(-n // 128) * 128, -(-k // 128) * 128))
    p[:n, :k] = w
    b = p.reshape(p.shape[0] // 128, 128, -1, 128)
    s = scale_e4m3(np.abs(b).max((1, 3)))[:, None, :, None]
    return (nearest(b / s, E4M3) * s).reshape(p.shape)[:n, :k]


def linear(x, w, bias=None):
    """-> (y, sum of the products' magnitudes)."""
    xq, wq = round_rows(np.asarray(x, np.float64)), round_weights(np.asarray(w, np.float64))
    y = xq @ wq.T
    return (y if bias is None else y + bias), np.abs(xq) @ np.abs(wq).T


def round_head(x, half):
    """Heads (..., head_dim) as 4 bits hold them: a scale per 32 values; a NaN as 0, an infinity as the largest float32."""
    x = np.nan_to_num(np.asarray(x, np.float64), nan=0.0, posinf=float(np.finfo(np.float32).max), neginf=-float(np.finfo(np.float32).max))
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    s = scale_e2m1(np.abs(g).max(-1), half)[..., None]
    return (nearest(g / s, E2M1) * s).reshape(x.shape)


def plan(held, fresh, free, count, table, block, blocks, rows):
    """-> table, starts, lengths, positions, slots, left."""
    table, width = [list(r) for r in table], (len(table[0]) if len(table) else 0)
    count = max(0, min(count, blocks))
    starts, lengths, positions, slots, used, at, short = [0], [], [-1] * rows, [-1] * rows, 0, 0, False
    for i, (h, f) in enumerate(zip(held, fresh)):
        n = max(f, 0)
        fits = h >= 0 and f >= 0 and h + f <= width * block and at + n <= rows
        have, want = -(-h // block), -(-(h + f) // block)
        need = want - have if fits else 0
        short = short or (need > 0 and used + need > count)
        ok = fits and (need == 0 or not short)
        if ok:
            for j in range(need):
                table[i][have + j] = free[count - 1 - used - j]
            used += need
            for j in range(f):
                positions[at + j] = h + j
                b = table[i][(h + j) // block]
                slots[at + j] = b * block + (h + j) % block if 0 <= b < blocks else -1
        at += n
        starts.append(min(at, rows))
        lengths.append(h + f if ok else max(0, min(h, width * block)))
    return table, starts, lengths, positions, slots, count - used


def norm_rope(x, weight, eps, angles, rotary, interleaved):
    """x (rows, heads, dim); angles (rows, rotary): cosines, then sines -> (values, sum of the terms' magnitudes)."""
    h = np.array(x, np.float64)
    if weight is not None:
        h = h / np.sqrt((h * h).mean(-1, keepdims=True) + eps) * weight
    size = np.abs(h)
    if rotary:
        i = np.arange(rotary // 2)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
        c, s = angles[:, None, : rotary // 2], angles[:, None, rotary // 2:]
        x, y = h[..., a], h[..., b]
        out = h.copy()
        out[..., a], out[..., b] = x * c - y * s, y * c + x * s
        size[..., a], size[..., b] = abs(x * c) + abs(y * s), abs(y * c) + abs(x * s)
        h = out
    return h, size


def attention(q, k, v, positions, scale, window=0, sinks=0, seen=None):
    """q (rows, heads, dim) over one request's tokens k, v (tokens, kv heads, dim) -> (out, sum of weights times
    magnitudes of v, largest sum of magnitudes of a score).  seen: tokens that may be seen at all."""
    rows, heads, dim = q.shape
    n, kv, _ = k.shape
    out, size, most = np.zeros(q.shape), np.zeros(q.shape), 0.0
    for r in range(rows):
        j = np.arange(n)
        see = j <= positions[r]
        if window:
            see &= (positions[r] - j < window) | (j < sinks)
        if seen is not None:
            see &= seen
        if not see.any():
            continue
        for h in range(heads):
            g = h // (heads // kv)
            s = k[see, g] @ q[r, h] * scale
            most = max(most, float((np.abs(k[see, g]) @ np.abs(q[r, h])).max()) * abs(scale))
            p = np.exp(s - s.max())
            p /= p.sum()
            out[r, h], size[r, h] = p @ v[see, g], p @ np.abs(v[see, g])
    return out, size, most


def score_bound(dim, most):
    """How far a float32 score may be from its value, in units of the exponent: products and sums of dim terms, the two scalings."""
    return (dim + 8) * 2.0 ** -23 * most


def bounds(k):
    """k (tokens, heads, dim) as the cache holds them -> (heads, 2, dim): the largest, then the smallest."""
    return np.stack((k.max(0), k.min(0)), 1)


def block_scores(q, block_bounds, negative=False):
    """q (heads, dim) over bounds (blocks, kv heads, 2, dim) -> (kv heads, blocks): what a key within the bounds could give, the largest of a group's heads; a sum
    that is no number counts as -infinity."""
    blocks, kv, _, dim = block_bounds.shape
    out = np.full((kv, blocks), -np.inf)
    with np.errstate(invalid="ignore"):
        for h in range(q.shape[0]):
            g = h // (q.shape[0] // kv)
            a, b = q[h] * block_bounds[:, g, 0], q[h] * block_bounds[:, g, 1]
            s = (-np.fmin(a, b) if negative else np.fmax(a, b)).sum(-1)
            out[g] = np.maximum(out[g], np.where(np.isnan(s), -np.inf, s))
    return out


def select(scores, visible, keep, first, last, there):
    """scores (kv heads, blocks), blocks that a row sees -> (kv heads, keep), -1 behind the last; there: blocks that the cache has."""
    out = np.full((scores.shape[0], keep), -1, np.int64)
    for g in range(scores.shape[0]):
        always = [b for b in range(visible) if there[b] and (b < first or b >= visible - last)]
        others = sorted((b for b in range(visible) if there[b] and b not in always), key=lambda b: (-scores[g, b], b))
        chosen = sorted(always + others[: keep - len(always)])
        out[g, : len(chosen)] = chosen
    return out


def residual_norm(x, y, post, gate, scale, eps, pre):
    """-> (r, norm of r, sum of the magnitudes of r's terms); y, post, gate (a row each) and pre may be None."""
    def norm(v, weight):
        mean = (v * v).mean(-1, keepdims=True) + eps
        return np.where(mean == 0, 0.0, v / np.sqrt(np.where(mean == 0, 1, mean))) * weight

    add = np.zeros_like(x) if y is None else y
    if post is not None and y is not None:
        add = norm(add, post)
    if gate is not None and y is not None:
        add = add * gate
    r = x + scale * add
    return r, None if pre is None else norm(r, pre), np.abs(x) + np.abs(scale * add)
