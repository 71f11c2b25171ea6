"""The operators of a language model's layer as a program serves it, as cases that can be timed and compared.

A step of a serving program takes, per request, the tokens that are new (one of a running request, a
chunk of a new one's prompt) through: the plan of the step (which cache blocks the new tokens get, where
every row of the step lies), products with weights held in 8 bits, norms and rotations of queries and
keys with the keys and values appended to a cache held in 4 bits, and attention over that cache.  The
cases cover those four over the range from a single row to thousands, both 16-bit types (the product
float32 too), ragged lengths, several block sizes, head sizes and groupings, windows with sinks.

Formats.  8 bits: e4m3 codes, values 2^e * code, one e per 128 inputs of a row of x and per 128 x 128 block
of the weights, the smallest with amax <= 448 * 2^e.  4 bits: e2m1 codes (0, .5, 1, 1.5, 2, 3, 4, 6 and their
negatives), one e per 32 values of a head, the smallest with amax < 7 * 2^e, at most 13 where the
cache serves float16.  Both round to nearest, ties to even codes.  The scales are powers of two, so that
codes follow from the inputs without a rounding of their own.

Inputs: activations N(0, 1) with a few channels ten times larger, weights N(0, 1/k), keys and values N(0, 1),
request lengths spread from one token to the longest.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
DEV = "cuda"


def listed():
    return [
        # One more token for each of a few dozen running requests: where the call itself is the cost.
        dict(name="plan_decode", op="plan", requests=64, longest=8192, fresh=1, most_fresh=1, block=64, room=1.0),
        # A step that mixes thousands of running requests with prompts, small blocks, and a free list that does not last.
        dict(name="plan_mixed", op="plan", requests=3000, longest=4096, fresh=1, most_fresh=700, block=16, room=0.7),
        # One row through a layer's input projection: the weights are what is read.
        dict(name="linear_row", op="linear", m=1, k=4096, n=6144, x="bf16", y="bf16", bias=False),
        # A handful of rows, sizes that fill no block and no tile, float32 results (scores of classes).
        dict(name="linear_ragged", op="linear", m=37, k=2000, n=1000, x="f16", y="f32", bias=True),
        # A batch of running requests through a wide projection.
        dict(name="linear_batch", op="linear", m=256, k=8192, n=4096, x="bf16", y="bf16", bias=False),
        # A prompt's chunk through a layer's widest product.
        dict(name="linear_prompt", op="linear", m=4096, k=4096, n=12288, x="bf16", y="bf16", bias=False),
        # Queries and keys of a decoding batch, one row a request.
        dict(name="rope_decode", op="rope", rows=64, q_heads=32, kv_heads=8, dim=128, rotary=128, interleaved=False, norm=True, dtype="bf16", block=64),
        # A long chunk of prompts: small heads, half of each rotated, in neighbouring pairs.
        dict(name="rope_prompt", op="rope", rows=8191, q_heads=24, kv_heads=6, dim=64, rotary=32, interleaved=True, norm=True, dtype="f16", block=32),
        # A single long conversation: one row over one long cache.
        dict(name="attend_one", op="attend", requests=1, longest=32768, fresh=1, q_heads=32, kv_heads=8, dim=128, block=64, window=0, sinks=0, dtype="bf16"),
        # A decoding batch of ragged lengths.
        dict(name="attend_batch", op="attend", requests=64, longest=8192, fresh=1, q_heads=32, kv_heads=8, dim=128, block=64, window=0, sinks=0, dtype="bf16"),
        # Very long requests seen through a window with the first tokens kept, a few guessed tokens checked at a time.
        dict(name="attend_window", op="attend", requests=16, longest=49999, fresh=4, q_heads=16, kv_heads=4, dim=64, block=16, window=4096, sinks=4, dtype="f16"),
        # Chunks of prompts over what their requests have in the cache.
        dict(name="attend_prompt", op="attend", requests=4, longest=6000, fresh=1024, q_heads=32, kv_heads=8, dim=128, block=128, window=0, sinks=0, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    op = rng.choice(("plan", "linear", "linear", "rope", "attend", "attend"))
    dtype, block = rng.choice(("bf16", "bf16", "f16")), rng.choice((16, 32, 64, 128, 256))
    if op == "plan":
        return dict(op=op, requests=_log(rng, 1, 4096), longest=_log(rng, 1, 16384), fresh=1, most_fresh=_log(rng, 1, 512), block=block,
                    room=rng.choice((1.0, 1.0, 0.5)))
    if op == "linear":
        x = rng.choice(("bf16", "bf16", "f16", "f32"))
        k, n = (v - v % rng.choice((1, 16, 128)) for v in (_log(rng, 128, 16384), _log(rng, 128, 16384)))
        return dict(op=op, m=_log(rng, 1, 4096), k=k, n=n, x=x, y=rng.choice((x, x, "f32")), bias=rng.random() < 0.5)
    kv_heads, dim = _log(rng, 1, 16), rng.choice((64, 128, 128, 256))
    q_heads = kv_heads * rng.choice((1, 2, 4, 4, 5, 8, 16))
    if op == "rope":
        rotary = rng.choice((dim, dim, dim // 2, 0))
        return dict(op=op, rows=_log(rng, 1, 8192), q_heads=q_heads, kv_heads=kv_heads, dim=dim, rotary=rotary, interleaved=rng.random() < 0.3,
                    norm=rng.random() < 0.7, dtype=dtype, block=block)
    window = rng.choice((0, 0, 0, _log(rng, 64, 8192)))
    return dict(op=op, requests=_log(rng, 1, 256), longest=_log(rng, 1, 65536), fresh=rng.choice((1, 1, 1, _log(rng, 2, 1024))), q_heads=q_heads,
                kv_heads=kv_heads, dim=dim, block=block, window=window, sinks=rng.choice((0, 4, 17)) if window else 0, dtype=dtype)


def draw(rng):
    """A call of the listed ranges; what would cost more than the largest listed one of its operator, in time or memory, is drawn again."""
    while True:
        case = _draw(rng)
        w = work(case)
        most = max((work(c) for c in listed() if c["op"] == case["op"]), key=lambda v: v["bytes"] + v["flops"] / 50)
        plain = 0
        if case["op"] == "attend":      # what the plain form holds: every request padded to the longest
            padded = case["requests"] * case["longest"] * case["kv_heads"] * case["dim"]
            scores = case["requests"] * case["q_heads"] * min(case["fresh"], case["longest"]) * case["longest"]
            plain = max(padded, scores)
        if w["bytes"] + w["flops"] / 50 <= most["bytes"] + most["flops"] / 50 and plain <= 1 << 30:
            return case


# ---- lengths, which a case has by itself --------------------------------------------------------

def _spread(n, most):
    """n lengths from 1 to most, the longest among them, in no order."""
    return [max(1, min(most, math.ceil(most * (1 - (i * 0.6180339887498949) % 1)))) for i in range(n)]


def _fresh(case):
    """New tokens of each request of a plan: `fresh`, or where prompts are among them up to `most_fresh`, none for some."""
    if case["most_fresh"] <= case["fresh"]:
        return [case["fresh"]] * case["requests"]
    return [case["fresh"] if i % 4 else case["most_fresh"] * ((7 * i) % 13) // 13 for i in range(case["requests"])]


def _attended(case):
    """Per request (tokens held with the new ones, new ones)."""
    return [(n, min(n, case["fresh"])) for n in _spread(case["requests"], case["longest"])]


def _visible(case, last):
    """Tokens that the row at position `last` sees."""
    w, s = case["window"], case["sinks"]
    return last + 1 if not w else min(last + 1, w + min(s, max(0, last + 1 - w)))


def work(case):
    op = case["op"]
    if op == "plan":
        held, fresh = _spread(case["requests"], case["longest"]), _fresh(case)
        blocks = sum(-(-(h + f) // case["block"]) - -(-h // case["block"]) for h, f in zip(held, fresh))
        # lengths in, starts and lengths out, a block read and written per block taken, a table entry read and position and slot written per row
        return {"bytes": 16 * case["requests"] + 8 * blocks + (4 + 12) * sum(fresh), "flops": 0}
    if op == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        size = {"f32": 4, "f16": 2, "bf16": 2}
        return {"bytes": m * k * size[case["x"]] + n * k + (n // 128 + 1) * (k // 128 + 1) + m * n * size[case["y"]], "flops": 2.0 * m * n * k}
    q, kv, d = case["q_heads"], case["kv_heads"], case["dim"]
    held = 2 * kv * (d // 2 + d // 32)                     # bytes of a token in the cache
    if op == "rope":
        # rows in, queries and keys out, the cache written, and read back as 16-bit values
        return {"bytes": case["rows"] * (2 * (q + 2 * kv) * d + 2 * (q + kv) * d + held + held + 4 * kv * d + 4 * case["rotary"] + 12), "flops": 0}
    total, flops = 0, 0
    for n, f in _attended(case):
        seen = _visible(case, n - 1) if f == 1 else min(n, _visible(case, n - 1) + f - 1)
        total += seen * held + 2 * 2 * f * q * d
        flops += sum(_visible(case, n - f + r) for r in range(f)) * 4 * q * d if f <= 64 else 4 * q * d * (_visible(case, n - f) + _visible(case, n - 1)) // 2 * f
    return {"bytes": total, "flops": float(flops)}


# ---- inputs: the same for both forms and for exact() --------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, *shape, dtype=torch.float32, std=1.0):
    return torch.randn(*shape, device=DEV, generator=g).mul_(std).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _blocks(case, lengths, g, spare=0):
    """A block table for requests of these lengths, blocks in no order, and the blocks that it leaves."""
    need = [-(-n // case["block"]) for n in lengths]
    count = sum(need) + spare
    order = torch.randperm(count, device=DEV, generator=g, dtype=torch.int32)
    return need, count, order


def _plan_inputs(case, seed):
    g = _gen(seed)
    held, fresh, block = _spread(case["requests"], case["longest"]), _fresh(case), case["block"]
    wanted = [-(-(h + f) // block) for h, f in zip(held, fresh)]
    need = [-(-h // block) for h in held]
    spare = max(1, int(case["room"] * (sum(wanted) - sum(need)))) + (7 if case["room"] == 1.0 else 0)
    _, count, order = _blocks(case, held, g, spare)
    width = max(wanted)
    cols = torch.arange(width, device=DEV)
    first = torch.tensor(need, device=DEV).cumsum(0) - torch.tensor(need, device=DEV)
    there = cols[None] < torch.tensor(need, device=DEV)[:, None]
    table = torch.where(there, order[(first[:, None] + cols[None]).clamp_(max=count - 1)], -1).to(torch.int32)
    free = order[sum(need):].contiguous()
    turn = torch.randperm(case["requests"], device=DEV, generator=g)
    held, fresh = _ints(held)[turn].contiguous(), _ints(fresh)[turn].contiguous()
    return dict(held=held, fresh=fresh, table=table[turn].contiguous(), free=free, count=_ints([spare]), blocks=count, width=width, rows=sum(_fresh(case)))


def _linear_inputs(case, seed):
    g = _gen(seed)
    x = _normal(g, case["m"], case["k"])
    x[:, torch.randint(case["k"], (max(1, case["k"] // 500),), device=DEV, generator=g)] *= 10
    w = _normal(g, case["n"], case["k"], std=case["k"] ** -0.5)
    return x.to(DTYPES[case["x"]]), w, _normal(g, case["n"], std=0.1) if case["bias"] else None


def _rope_inputs(case, seed):
    g, t = _gen(seed), DTYPES[case["dtype"]]
    q, kv, d, rows, block = case["q_heads"], case["kv_heads"], case["dim"], case["rows"], case["block"]
    qkv = _normal(g, rows, (q + 2 * kv) * d, dtype=t)                       # a projection's output: the three side by side
    held = 4096
    positions = torch.randint(held, (rows,), device=DEV, generator=g, dtype=torch.int32)
    blocks = -(-rows // block) + 3
    slots = torch.randperm(blocks * block, device=DEV, generator=g)[:rows].contiguous()
    half = max(1, case["rotary"] // 2)
    angle = torch.arange(held, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
    table = torch.cat((angle.cos(), angle.sin()), 1).float().contiguous() if case["rotary"] else None
    weights = [1 + _normal(g, d, std=0.2) for _ in range(2)] if case["norm"] else [None, None]
    return dict(qkv=qkv, positions=positions, slots=slots, table=table, q_weight=weights[0], k_weight=weights[1], blocks=blocks, held=held)


def _attend_inputs(case, seed):
    g, t = _gen(seed), DTYPES[case["dtype"]]
    kv, d, block = case["kv_heads"], case["dim"], case["block"]
    both = _attended(case)
    lengths, fresh = [n for n, _ in both], [f for _, f in both]
    need, count, order = _blocks(case, lengths, g, 3)
    width = max(need)
    table = torch.full((len(lengths), width), -1, dtype=torch.int32, device=DEV)
    cols = torch.arange(width, device=DEV)
    first = torch.tensor(need, device=DEV).cumsum(0) - torch.tensor(need, device=DEV)
    there = cols[None] < torch.tensor(need, device=DEV)[:, None]
    table = torch.where(there, order[(first[:, None] + cols[None]).clamp_(max=count - 1)], table)
    k, v = (_normal(g, count * block, kv, d, dtype=t) for _ in range(2))
    rows = sum(fresh)
    q = _normal(g, rows, case["q_heads"], d, dtype=t, std=1.5)
    starts = _ints([0] + fresh).cumsum(0).to(torch.int32)
    lengths, fresh = _ints(lengths), _ints(fresh)
    request = torch.repeat_interleave(torch.arange(len(both), device=DEV), fresh.long(), output_size=rows)
    positions = (torch.arange(rows, device=DEV) - starts[request] + lengths[request] - fresh[request]).to(torch.int32)
    return dict(q=q, k=k, v=v, table=table.contiguous(), starts=starts, lengths=lengths, positions=positions, request=request, blocks=count, width=width, rows=rows)


# ---- the plain form: the two formats ------------------------------------------------------------

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exponent(amax, bits):
    """Of a positive float32: floor(log2), from its bits; -127 for zero and what has no normal form."""
    return (amax.view(torch.int32) >> 23).sub_(127), (amax.view(torch.int32) & 0x7FFFFF) > bits


def _to_e4m3(x):
    """x (..., blocks, values of a block) in float32 -> codes as float8, exponents: amax <= 448 * 2^e = 1.75 * 2^(e + 8)."""
    amax = x.abs().amax(-1)
    e, more = _exponent(amax, 0x600000)
    e = (e - 8 + more.to(torch.int32)).clamp_(min=-126)
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn), e


def _to_e2m1(x, half):
    """x (..., head) in float64 -> codes 0..15 (8: negative), exponents of its groups of 32: amax < 7 * 2^e = 1.75 * 2^(e + 2)."""
    x = x.unflatten(-1, (-1, 32))
    amax = x.abs().amax(-1)
    e = torch.frexp(amax)[1] - 3
    e = e + (torch.ldexp(amax, -e) >= 7).to(torch.int32)
    e = torch.where(amax == 0, -126, e).clamp_(min=-126, max=13 if half else 125)
    v = torch.ldexp(x.abs(), -e[..., None].double())
    code = torch.zeros(v.shape, dtype=torch.uint8, device=v.device)
    for border, even_below in zip((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0), (True, False, True, False, True, False, True)):
        code += v > border if even_below else v >= border
    return (code + 8 * torch.signbit(x).to(torch.uint8)).flatten(-2), e


def _of_e2m1(code, e):
    values = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=code.device)
    return (values[code.long()].unflatten(-1, (-1, 32)) * torch.ldexp(torch.ones((), device=code.device), e)[..., None]).flatten(-2)


def _pad(x, to):
    return torch.nn.functional.pad(x, (0, -x.shape[-1] % to))


def _heads(case, qkv):
    q, kv, d = case["q_heads"], case["kv_heads"], case["dim"]
    return [t.unflatten(-1, (-1, d)) for t in qkv.split((q * d, kv * d, kv * d), -1)]


def _norm_rope(x, weight, table, positions, rotary, interleaved):
    """Norm and rotation of heads in the type of x (rows, heads, dim)."""
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight.to(x.dtype)
    if not rotary:
        return x
    cos, sin = (t.to(x.dtype)[:, None] for t in table[positions.long()].chunk(2, -1))
    turned, rest = x[..., :rotary], x[..., rotary:]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if interleaved else turned.chunk(2, -1)
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.cat((torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1), rest), -1)


def _run_plan(s):
    block, blocks, rows = s["block"], s["blocks"], s["rows"]
    held, fresh, table = s["held"].long(), s["fresh"].long(), s["table"]
    ends = fresh.cumsum(0)
    old, new = -(-held // block), -(-(held + fresh) // block)
    fits = (new <= s["width"]) & (ends <= rows)
    need = torch.where(fits, new - old, 0)
    upto = need.cumsum(0)
    granted = fits & ((need == 0) | (upto <= s["count"]))
    taken = torch.where(granted, need, 0)
    cols = torch.arange(s["width"], device=DEV)
    mine = granted[:, None] & (cols >= old[:, None]) & (cols < new[:, None])
    which = s["count"] - 1 - ((upto - need)[:, None] + cols - old[:, None])
    table = torch.where(mine, s["free"][which.clamp(0, s["free"].numel() - 1)], table)
    starts = torch.cat((torch.zeros(1, dtype=torch.int64, device=DEV), ends)).clamp(max=rows)
    row = torch.arange(rows, device=DEV)
    request = (torch.searchsorted(starts, row, right=True) - 1).clamp(max=held.numel() - 1)
    there = granted[request] & (row < starts[-1])
    position = torch.where(there, held[request] + row - starts[request], 0)
    slot = table[request, position // block].long() * block + position % block
    return dict(table=table, starts=starts.to(torch.int32), lengths=(held + torch.where(granted, fresh, 0)).to(torch.int32),
                positions=torch.where(there, position, -1).to(torch.int32), slots=torch.where(there, slot, -1), left=(s["count"] - taken.sum()).to(torch.int32))


def _run_linear(s):
    x = _pad(s["x"].float(), 128).unflatten(-1, (-1, 128))
    codes, e = _to_e4m3(x)
    x = torch.ldexp(codes.float(), e[..., None]).flatten(-2)
    w = torch.ldexp(s["codes"].float(), s["e"][:, None, :, None]).flatten(0, 1).flatten(1)[: s["n"]]
    y = x @ w.t()
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["y_type"])


def _run_rope(s):
    q, k, v = _heads(s["case"], s["qkv"])
    rope = (s["table"], s["positions"], s["case"]["rotary"], s["case"]["interleaved"])
    t = s["qkv"].dtype
    q = _norm_rope(q.float(), s["q_weight"], *rope)
    k = _norm_rope(k.double(), s["k_weight"], *rope)                  # 64 bits: the codes of keys lie next to borders
    held = [_of_e2m1(*_to_e2m1(x, t == torch.float16)).to(t) for x in (k, v.double())]
    return dict(q=q.to(t), k=k.to(t), held_k=held[0], held_v=held[1])


def _run_attend(s):
    case, block = s["case"], s["case"]["block"]
    kv, d, group = case["kv_heads"], case["dim"], case["q_heads"] // case["kv_heads"]
    most, width = s["most"], s["width"] * block
    token = torch.arange(width, device=DEV)
    slot = s["table"][:, token // block].long() * block + token % block
    held = token < s["lengths"][:, None]
    slot = torch.where(held, slot, 0)
    k, v = (_of_e2m1(s[c][slot], s[e][slot]).transpose(1, 2) for c, e in (("k_codes", "k_e"), ("v_codes", "v_e")))   # (requests, heads, tokens, dim)
    row = s["starts"][:-1, None].long() + torch.arange(most, device=DEV)
    there = row < s["starts"][1:, None]
    row = torch.where(there, row, 0)
    q = s["q"].float()[row].unflatten(2, (kv, group)).permute(0, 2, 1, 3, 4).flatten(2, 3)                              # (requests, heads, rows * group, dim)
    at = torch.where(there, s["positions"][row], -1)[:, :, None]
    seen = held[:, None] & (token <= at)
    if case["window"]:
        seen &= (token > at - case["window"]) | (token < case["sinks"])
    p = (q @ k.transpose(2, 3)).mul_(d ** -0.5)
    seen = seen[:, None].repeat_interleave(group, 2)
    p.masked_fill_(~seen, -math.inf)
    p = torch.exp(p - p.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min))
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / torch.where(total == 0, 1, total)
    out = out.unflatten(2, (most, group)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    return out[s["request"], torch.arange(s["rows"], device=DEV) - s["starts"][s["request"]]].to(s["q"].dtype)


# ---- prepare and run ----------------------------------------------------------------------------

def prepare(case, seed):
    if own:
        return _prepare_own(case, seed)
    if case["op"] == "plan":
        return dict(_plan_inputs(case, seed), run=_run_plan, block=case["block"])
    if case["op"] == "linear":
        x, w, bias = _linear_inputs(case, seed)
        w = torch.nn.functional.pad(w, (0, -case["k"] % 128, 0, -case["n"] % 128)).unflatten(0, (-1, 128)).unflatten(2, (-1, 128))   # (block, row, block, column)
        codes, e = _to_e4m3(w.transpose(1, 2).flatten(2))
        return dict(run=_run_linear, x=x, codes=codes.unflatten(2, (128, 128)).transpose(1, 2).contiguous(), e=e, n=case["n"], bias=bias, y_type=DTYPES[case["y"]])
    if case["op"] == "rope":
        return dict(_rope_inputs(case, seed), run=_run_rope, case=case)
    s = _attend_inputs(case, seed)
    for name in ("k", "v"):
        s[name + "_codes"], s[name + "_e"] = _to_e2m1(s.pop(name).double(), case["dtype"] == "f16")
    return dict(s, run=_run_attend, case=case, most=min(case["fresh"], case["longest"]))


def _types(nnv):
    return {"f32": nnv.F32, "f16": nnv.F16, "bf16": nnv.BF16}


def _attention_desc(nnv, case, s, positions=0):
    return nnv.AttentionDesc(q_heads=case["q_heads"], kv_heads=case["kv_heads"], head_dim=case["dim"], block_tokens=case["block"], blocks=s["blocks"],
                             table_blocks=s.get("width", 1), rotary_dim=case.get("rotary", 0), rotary_interleaved=int(case.get("interleaved", False)),
                             positions=positions, window=case.get("window", 0), sinks=case.get("sinks", 0), dtype=_types(nnv)[case["dtype"]],
                             scale=case["dim"] ** -0.5, eps=1e-6)


def _prepare_own(case, seed):
    import paper_2206_07446_amd as nnv
    if case["op"] == "plan":
        s = _plan_inputs(case, seed)
        n = case["requests"]
        desc = nnv.AttentionDesc(q_heads=1, kv_heads=1, head_dim=64, block_tokens=case["block"], blocks=s["blocks"], table_blocks=s["width"], dtype=nnv.BF16, scale=1.0)
        new = lambda count, dtype=torch.int32: torch.empty(count, dtype=dtype, device=DEV)  # noqa: E731
        return dict(s, run=_own_plan, nnv=nnv, desc=desc, n=n, starts=new(n + 1), lengths=new(n), positions=new(s["rows"]), slots=new(s["rows"], torch.int64), left=new(1))
    if case["op"] == "linear":
        x, w, bias = _linear_inputs(case, seed)
        types = _types(nnv)
        desc = nnv.LinearDesc(n=case["n"], k=case["k"], x_dtype=types[case["x"]], y_dtype=types[case["y"]], raw_dtype=nnv.F32)
        w_tx = torch.empty(nnv.nnv_linear_transformed_bytes(desc), dtype=torch.uint8, device=DEV)
        nnv.nnv_linear_transform_weights(desc, w, w_tx)
        workspace = torch.empty(max(16, nnv.nnv_linear_workspace_bytes(desc, case["m"])), dtype=torch.uint8, device=DEV)
        y = torch.empty(case["m"], case["n"], dtype=DTYPES[case["y"]], device=DEV)
        return dict(run=_own_linear, nnv=nnv, desc=desc, m=case["m"], x=x, w_tx=w_tx, bias=bias, y=y, workspace=workspace)
    if case["op"] == "rope":
        s = _rope_inputs(case, seed)
        desc = _attention_desc(nnv, case, s, s["held"])
        q, kv, d = case["q_heads"], case["kv_heads"], case["dim"]
        new = lambda heads: torch.empty(case["rows"], heads, d, dtype=DTYPES[case["dtype"]], device=DEV)  # noqa: E731
        cache = torch.zeros(nnv.nnv_kv_cache_bytes(desc), dtype=torch.uint8, device=DEV)
        return dict(s, run=_own_rope, nnv=nnv, desc=desc, rows=case["rows"], parts=s["qkv"].split((q * d, kv * d, kv * d), -1), cache=cache, q=new(q), k=new(kv),
                    held_k=new(kv), held_v=new(kv))
    s = _attend_inputs(case, seed)
    desc = _attention_desc(nnv, case, s)
    cache = torch.zeros(nnv.nnv_kv_cache_bytes(desc), dtype=torch.uint8, device=DEV)
    k, v = s.pop("k"), s.pop("v")
    count, stride = k.shape[0], case["kv_heads"] * case["dim"]
    nnv.nnv_qk_norm_rope(desc, count, None, 0, k, stride, v, stride, None, None, None, torch.zeros(count, dtype=torch.int32, device=DEV),
                         torch.arange(count, device=DEV), None, None, cache)
    workspace = torch.empty(max(16, nnv.nnv_kv_attention_workspace_bytes(desc, case["requests"], s["rows"])), dtype=torch.uint8, device=DEV)
    return dict(s, run=_own_attend, nnv=nnv, desc=desc, n=case["requests"], cache=cache, workspace=workspace, out=torch.empty_like(s["q"]))


def _own_plan(s):
    s["nnv"].nnv_kv_plan(s["desc"], s["n"], s["rows"], s["held"], s["fresh"], s["free"], s["count"], s["table"], s["starts"], s["lengths"], s["positions"],
                         s["slots"], s["left"])
    return dict(table=s["table"], starts=s["starts"], lengths=s["lengths"], positions=s["positions"], slots=s["slots"], left=s["left"])


def _own_linear(s):
    s["nnv"].nnv_linear_forward(s["desc"], s["m"], s["x"], s["x"].stride(0), s["w_tx"], s["bias"], s["y"], s["y"].stride(0), s["workspace"])
    return s["y"]


def _own_rope(s):
    (q, k, v), nnv = s["parts"], s["nnv"]
    stride = s["qkv"].stride(0)
    nnv.nnv_qk_norm_rope(s["desc"], s["rows"], q, stride, k, stride, v, stride, s["q_weight"], s["k_weight"], s["table"], s["positions"], s["slots"], s["q"],
                         s["k"], s["cache"])
    nnv.nnv_kv_read(s["desc"], s["rows"], s["slots"], s["cache"], s["held_k"], s["held_v"])
    return dict(q=s["q"], k=s["k"], held_k=s["held_k"], held_v=s["held_v"])


def _own_attend(s):
    s["nnv"].nnv_kv_attention(s["desc"], s["n"], s["rows"], s["q"], s["table"], s["starts"], s["lengths"], s["positions"], s["cache"], s["out"], s["workspace"])
    return s["out"]


def run(state):
    return state["run"](state)


# ---- the definitions, in 64 bits ----------------------------------------------------------------

def _round_e4m3(x):
    """Values that e4m3 with a shared power of two stands for, of blocks along the last axis, in float64."""
    amax = x.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(amax.clamp(min=2.0 ** -140) / 448)))
    scale = torch.where(amax > 448 * scale, 2 * scale, torch.where(amax <= 224 * scale, scale / 2, scale)).clamp(min=2.0 ** -126)   # log2 may be off by its last bit
    v = x / scale
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(v / step) * step * scale


def _round_e2m1(x, half):
    groups = x.reshape(*x.shape[:-1], -1, 32)
    amax = groups.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.floor(torch.log2(amax.clamp(min=2.0 ** -140) / 3.5)))
    scale = torch.where(amax < 3.5 * scale, scale / 2, torch.where(amax >= 7 * scale, 2 * scale, scale)).clamp(2.0 ** -126, 2.0 ** (13 if half else 125))
    v = (groups / scale).clamp(-6.99, 6.99)
    size = v.abs()
    step = 0.5 + 0.5 * (size >= 2) + 1.0 * (size >= 4)
    return (torch.round(v / step) * step * scale).reshape(x.shape)


def _exact_plan(case, s):
    held, fresh, table, free, count = (s[k].tolist() for k in ("held", "fresh", "table", "free", "count"))
    block, rows, at, used = case["block"], s["rows"], 0, 0
    starts, lengths, positions, slots = [0], [], [-1] * rows, [-1] * rows
    short = False
    for i, (h, f) in enumerate(zip(held, fresh)):
        have, want = -(-h // block), -(-(h + f) // block)
        need = want - have
        short = short or (need > 0 and used + need > count[0])
        ok = need == 0 or not short
        if ok:
            table[i][have:want] = [free[count[0] - 1 - used - j] for j in range(need)]
            used += need
            for j in range(f):
                positions[at + j] = h + j
                slots[at + j] = table[i][(h + j) // block] * block + (h + j) % block
        at += f
        starts.append(at)
        lengths.append(h + f if ok else h)
    make = lambda v, t=torch.int32: torch.tensor(v, dtype=t)  # noqa: E731
    return dict(table=make(table), starts=make(starts), lengths=make(lengths), positions=make(positions), slots=make(slots, torch.int64), left=make(count[0] - used))


def _exact_linear(case, x, w, bias):
    k, n = case["k"], case["n"]
    kb, nb = -(-k // 128), -(-n // 128)
    xp = torch.zeros(case["m"], kb * 128, dtype=torch.float64, device=DEV)
    xp[:, :k] = x
    wp = torch.zeros(nb * 128, kb * 128, dtype=torch.float64, device=DEV)
    wp[:n, :k] = w
    xp = _round_e4m3(xp.reshape(-1, kb, 128)).reshape(-1, kb * 128)
    blocks = wp.reshape(nb, 128, kb, 128).permute(0, 2, 1, 3).reshape(nb, kb, -1)
    wp = _round_e4m3(blocks).reshape(nb, kb, 128, 128).permute(0, 2, 1, 3).reshape(nb * 128, -1)
    y = torch.matmul(xp, wp.t())[:, :n]
    return y if bias is None else y + bias.double()


def _exact_rope(case, s):
    d, half, rotary = case["dim"], case["dtype"] == "f16", case["rotary"]
    x = s["qkv"].double().reshape(case["rows"], -1, d)
    nq, nkv = case["q_heads"], case["kv_heads"]
    parts = {"q": x[:, :nq], "k": x[:, nq:nq + nkv]}
    for name, weight in (("q", s["q_weight"]), ("k", s["k_weight"])):
        h = parts[name].clone()
        if weight is not None:
            h /= ((h * h).sum(-1, keepdim=True) / d + 1e-6).sqrt()
            h *= weight.double()
        if rotary:
            turn = torch.complex(*(t.contiguous().double() for t in s["table"][s["positions"].long()].split(rotary // 2, 1)))[:, None]
            index = torch.arange(rotary, device=DEV)
            first, second = (index[0::2], index[1::2]) if case["interleaved"] else (index[: rotary // 2], index[rotary // 2:])
            turned = torch.complex(h[..., first], h[..., second]) * turn
            h[..., first], h[..., second] = turned.real, turned.imag
        parts[name] = h
    return dict(q=parts["q"], k=parts["k"], held_k=_round_e2m1(parts["k"], half), held_v=_round_e2m1(x[:, nq + nkv:], half))


def _exact_attend(case, s):
    block, d, half = case["block"], case["dim"], case["dtype"] == "f16"
    group = case["q_heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    starts = s["starts"].tolist()
    for i, n in enumerate(s["lengths"].tolist()):
        blocks = s["table"][i, : -(-n // block)].long()
        kept = [s[c].unflatten(0, (-1, block))[blocks].flatten(0, 1)[:n].double() for c in ("k", "v")]
        k, v = (_round_e2m1(x, half) for x in kept)
        a, b = starts[i], starts[i + 1]
        for c in range(a, b, 128):
            rows = slice(c, min(b, c + 128))
            at = s["positions"][rows].long()[:, None]
            token = torch.arange(n, device=DEV)[None]
            seen = token <= at
            if case["window"]:
                seen = seen & ((at - token < case["window"]) | (token < case["sinks"]))
            for h in range(case["kv_heads"]):
                q = s["q"][rows, h * group:(h + 1) * group].double()
                scores = torch.matmul(q, k[:, h].t()) / math.sqrt(d)
                weights = torch.softmax(scores.masked_fill(~seen[:, None], -math.inf), -1)
                out[rows, h * group:(h + 1) * group] = torch.matmul(weights, v[:, h])
    return out


def exact(case, seed):
    if case["op"] == "plan":
        return _exact_plan(case, _plan_inputs(case, seed))
    if case["op"] == "linear":
        return _exact_linear(case, *_linear_inputs(case, seed))
    if case["op"] == "rope":
        return _exact_rope(case, _rope_inputs(case, seed))
    return _exact_attend(case, _attend_inputs(case, seed))
