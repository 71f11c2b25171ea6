"""One attention layer of a language model as a serving program runs it, from request lengths to the layer's output
rows: the cold start (weights to 8 bits), a step that takes the requests' prompts in, and steps of one token a request
replayed from a HIP graph.  The layer keeps every buffer, so that a step is seven calls and no allocation.  Its attention is over the whole cache, over
the blocks that each row selects (`keep`), or over prefixes that groups of requests share (`share`); `step_stream` runs it from the residual
stream to the residual stream and the norm for the next layer.

`python -m paper_2206_07446_amd.attention_layer --requests 64 --prompt 512 --steps 64` prints the time of each part; with `--keep 8` or `--shared 4096` too.
"""
from __future__ import annotations

import argparse
import ctypes
import math

import torch

from . import binding as nnv

DTYPES = {nnv.F16: torch.float16, nnv.BF16: torch.bfloat16}
NO_TENSORS = -1                # what a call of sizes that it takes returns without tensors (NNV_E_NULL)
MOST_STREAM = 32768            # values of a row that nnv_residual_norm takes


class AttentionLayer:
    """Weights, cache, block table and buffers for up to `rows` rows a step and `requests` requests of `tokens` tokens (whole blocks of them).
    keep: a row sees so many blocks, the first `first`, the last `last` and those of the largest scores; 0: all.  groups: the most groups of requests that may share a prefix."""

    def __init__(self, hidden, q_heads, kv_heads, head_dim, requests, rows, tokens, block_tokens=64, dtype=nnv.BF16, theta=10000.0, window=0, sinks=0,
                 device="cuda:0", keep=0, first=1, last=2, groups=0):
        if keep and (window or groups or not 0 <= first + last <= keep or min(first, last) < 0):
            raise ValueError("blocks are selected without a window and shared prefixes, the first and last ones among those kept")
        self.keep, self.first, self.last, self.groups, self.n_groups = keep, first, last, groups, 0
        self.device, self.dtype, self.requests, self.rows, self.hidden = torch.device(device), DTYPES[dtype], requests, rows, hidden
        width = -(-tokens // block_tokens)
        self.desc = nnv.AttentionDesc(q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, block_tokens=block_tokens, blocks=nnv._int(requests * width),
                                      table_blocks=width, rotary_dim=head_dim, rotary_interleaved=0, positions=nnv._int(width * block_tokens), window=window, sinks=sinks, dtype=dtype,
                                      scale=head_dim ** -0.5, eps=1e-6)
        self.q_size, self.kv_size = q_heads * head_dim, kv_heads * head_dim
        self.qkv_desc = nnv.LinearDesc(n=self.q_size + 2 * self.kv_size, k=hidden, x_dtype=dtype, y_dtype=dtype, raw_dtype=nnv.F32)
        self.out_desc = nnv.LinearDesc(n=hidden, k=self.q_size, x_dtype=dtype, y_dtype=dtype, raw_dtype=nnv.F32)
        self._fits(nnv._int(rows))
        new = lambda *shape, dtype=self.dtype: torch.empty(*shape, dtype=dtype, device=self.device)  # noqa: E731
        bytes_ = lambda n: new(max(16, n), dtype=torch.uint8)  # noqa: E731
        self.qkv_tx, self.out_tx = (bytes_(nnv.nnv_linear_transformed_bytes(d)) for d in (self.qkv_desc, self.out_desc))
        self.cache = bytes_(nnv.nnv_kv_cache_bytes(self.desc))
        # what a call over m rows needs of its scratch goes up and down with m, where the number of parts that it splits into changes: the most of every size
        need = max(max(nnv.nnv_kv_attention_workspace_bytes(self.desc, requests, m), *(nnv.nnv_linear_workspace_bytes(d, m) for d in (self.qkv_desc, self.out_desc)))
                   for m in range(1, rows + 1))
        if keep:
            self.bounds = torch.zeros(nnv.nnv_kv_bounds_bytes(self.desc) // 2, dtype=torch.bfloat16, device=self.device)
            self.selected = new(rows, kv_heads, keep, dtype=torch.int32)
            need = max(need, *(max(nnv.nnv_kv_select_workspace_bytes(self.desc, requests, m), nnv.nnv_kv_attention_blocks_workspace_bytes(self.desc, requests, m, keep))
                               for m in range(1, rows + 1)))
        if groups:
            need = max(need, *(nnv.nnv_kv_attention_shared_workspace_bytes(self.desc, requests, m, g) for m in range(1, rows + 1) for g in range(1, groups + 1)))
            self.group_ends, self.shared = (torch.zeros(groups + n, dtype=torch.int32, device=self.device) for n in (1, 0))
        self.workspace = bytes_(need)
        self.norm_in, self.norm_next, self.norm_out = (torch.ones(hidden, device=self.device) for _ in range(3))
        self.out = new(rows, hidden)
        self.q_weight, self.k_weight = (torch.ones(head_dim, device=self.device) for _ in range(2))
        half = head_dim // 2
        angle = torch.arange(width * block_tokens, dtype=torch.float64)[:, None] * theta ** (-torch.arange(half, dtype=torch.float64) / half)
        self.rope = torch.cat((angle.cos(), angle.sin()), 1).float().to(self.device)
        self.qkv, self.q, self.attended = new(rows, self.q_size + 2 * self.kv_size), new(rows, q_heads, head_dim), new(rows, q_heads, head_dim)
        ints = lambda n, dtype=torch.int32: torch.zeros(n, dtype=dtype, device=self.device)  # noqa: E731
        self.held, self.fresh, self.lengths, self.starts = ints(requests), ints(requests), ints(requests), ints(requests + 1)
        self.positions, self.slots, self.left = ints(rows), ints(rows, torch.int64), ints(1)
        self.table = torch.full((requests, width), -1, dtype=torch.int32, device=self.device)
        self.free = torch.arange(requests * width, dtype=torch.int32, device=self.device)
        self.count = torch.tensor([requests * width], dtype=torch.int32, device=self.device)

    def _fits(self, rows):
        """Sizes that a call of a step would refuse, after those before it have run, are refused with the layer.  A call looks at its sizes before its tensors, of which there
        are none here (16: an address that is not looked at), so that it never runs."""
        lib, desc, step = nnv.load(), ctypes.byref(self.desc), (ctypes.byref(self.desc), self.requests, rows)
        none = lambda n: (None,) * n  # noqa: E731
        calls = [("nnv_linear_forward", (ctypes.byref(d), rows, None, d.k, None, None, None, d.n, None, 0, None)) for d in (self.qkv_desc, self.out_desc)]
        calls += [("nnv_kv_plan", (*step, *none(11))), ("nnv_qk_norm_rope", (desc, rows, 16, self.q_size, None, 0, None, 0, *none(9))), ("nnv_kv_attention", (*step, *none(8), 0, None))]
        if self.keep:
            calls += [("nnv_kv_bounds", (*step, *none(6))), ("nnv_kv_select", (*step, self.keep, self.first, self.last, *none(8), 0, None)),
                      ("nnv_kv_attention_blocks", (*step, self.keep, *none(9), 0, None))]
        # (what attention over shared prefixes launches goes up and down with the rows; with the groups it goes up, to 64 of them and from there on)
        if self.groups:
            calls += [("nnv_kv_attention_shared", (desc, self.requests, m, g, *none(10), 0, None)) for m in range(1, rows + 1) for g in {self.groups, min(self.groups, 64)}]
        for name, args in calls:
            status = getattr(lib, name)(*args)
            if status != NO_TENSORS:
                raise ValueError(f"{name} does not take {rows} rows of {self.requests} requests of this layer: {nnv.nnv_status_string(status)}")

    def _check(self, rows, *tensors):
        """The calls below take addresses: what their buffers do not hold is refused here."""
        if not 0 <= rows <= self.rows:
            raise ValueError(f"{rows} rows, the layer has buffers for 0 to {self.rows}")
        for t in tensors:
            if not (isinstance(t, torch.Tensor) and t.dtype == self.dtype and t.device == self.qkv.device and t.dim() == 2 and t.shape[0] >= rows
                    and t.shape[1] == self.hidden and t.stride(1) == 1 and (rows <= 1 or t.stride(0) >= self.hidden) and t.data_ptr() % 16 == 0):
                raise ValueError(f"expected {rows} rows or more of {self.hidden} {self.dtype} on {self.qkv.device}, each without gaps, the first 16-byte aligned")

    def transform_weights(self, w_qkv, w_out):
        """Raw float32 weights to the layouts that the products run from."""
        for w, d in ((w_qkv, self.qkv_desc), (w_out, self.out_desc)):
            if not (isinstance(w, torch.Tensor) and w.dtype == torch.float32 and w.device == self.qkv.device and w.shape == (d.n, d.k) and w.is_contiguous()):
                raise ValueError(f"expected contiguous float32 weights of {d.n} x {d.k} on {self.qkv.device}")
        nnv.nnv_linear_transform_weights(self.qkv_desc, w_qkv, self.qkv_tx)
        nnv.nnv_linear_transform_weights(self.out_desc, w_out, self.out_tx)

    def plan(self, rows):
        self._check(rows)
        nnv.nnv_kv_plan(self.desc, self.requests, rows, self.held, self.fresh, self.free, self.count, self.table, self.starts, self.lengths, self.positions,
                        self.slots, self.left)

    def project(self, x, rows):
        self._check(rows, x)
        nnv.nnv_linear_forward(self.qkv_desc, rows, x, x.stride(0), self.qkv_tx, None, self.qkv, self.qkv.stride(0), self.workspace)

    def append(self, rows):
        self._check(rows)
        stride = self.qkv.stride(0)
        q, k, v = self.qkv.split((self.q_size, self.kv_size, self.kv_size), 1)
        nnv.nnv_qk_norm_rope(self.desc, rows, q, stride, k, stride, v, stride, self.q_weight, self.k_weight, self.rope, self.positions, self.slots, self.q,
                             None, self.cache)

    def share(self, ends, tokens):
        """Requests ends[g] to ends[g + 1] - 1 begin with the same tokens[g] tokens (whole blocks), which the first of them holds.  Others that hold nothing yet
        begin behind them from here on; others that hold something have to run behind these very blocks already, so that groups may be added, taken away and given
        another first request while they run.  Requests keep the prefix that they began behind whatever is shared later, since its blocks are entered in their own rows of the
        table: groups say what is read once for all of them.  The first request of a group holds the prefix as long as the group is given: before its place is used again,
        share without it.  A captured step reads as many groups as there were, of those that there are when it is replayed."""
        ends, tokens, block = list(ends), list(tokens), self.desc.block_tokens
        held, table = self.held.tolist(), self.table.cpu()
        if len(tokens) > self.groups or len(ends) != len(tokens) + 1 or sorted(ends) != ends or ends[0] < 0 or ends[-1] > self.requests:
            raise ValueError(f"expected up to {self.groups} groups of the {self.requests} requests, in their order")

        def behind(i, first, n):
            return held[i] >= n and torch.equal(table[i, : n // block], table[first, : n // block]) and bool((table[i, : n // block] >= 0).all())

        for first, end, n in zip(ends, ends[1:], tokens):
            if n < 0 or n % block or (first < end and held[first] < n) or any(held[i] and not behind(i, first, n) for i in range(first + 1, end)):
                raise ValueError(f"{n} tokens: expected whole blocks of {block} that request {first} holds, and others of its group that hold nothing or are behind these")
        for first, end, n in zip(ends, ends[1:], tokens):
            new = [i for i in range(first + 1, end) if held[i] == 0]
            self.held[new] = n
            self.table[new, : n // block] = self.table[first, : n // block]
        if self.groups:                                      # (behind the last: groups of no request)
            self.group_ends.copy_(torch.tensor(ends + ends[-1:] * (self.groups - len(tokens)), dtype=torch.int32))
            self.shared.copy_(torch.tensor(tokens + [0] * (self.groups - len(tokens)), dtype=torch.int32))
        self.n_groups = len(tokens)

    def attend(self, rows):
        self._check(rows)
        if self.keep:
            nnv.nnv_kv_bounds(self.desc, self.requests, rows, self.table, self.starts, self.lengths, self.cache, self.bounds)
            nnv.nnv_kv_select(self.desc, self.requests, rows, self.keep, self.first, self.last, self.q, self.table, self.starts, self.lengths, self.positions,
                              self.bounds, self.selected, self.workspace)
            nnv.nnv_kv_attention_blocks(self.desc, self.requests, rows, self.keep, self.q, self.table, self.starts, self.lengths, self.positions, self.selected,
                                        self.cache, self.attended, self.workspace)
            return
        if self.n_groups:
            nnv.nnv_kv_attention_shared(self.desc, self.requests, rows, self.n_groups, self.q, self.table, self.starts, self.lengths, self.positions,
                                        self.group_ends, self.shared, self.cache, self.attended, self.workspace)
            return
        nnv.nnv_kv_attention(self.desc, self.requests, rows, self.q, self.table, self.starts, self.lengths, self.positions, self.cache, self.attended,
                             self.workspace)

    def finish(self, y, rows):
        self._check(rows, y)
        nnv.nnv_linear_forward(self.out_desc, rows, self.attended, self.q_size, self.out_tx, None, y, y.stride(0), self.workspace)

    def step(self, x, y, rows):
        """Rows of x (the new tokens of request 0, then of request 1, ..., as self.fresh counts them) -> rows of y; what is held grows by them.  A step that its
        buffers do not hold is refused before anything runs."""
        self._check(rows, x, y)
        self.plan(rows)
        self.project(x, rows)
        self.append(rows)
        self.attend(rows)
        self.finish(y, rows)
        self.held.copy_(self.lengths)
        self.count.copy_(self.left)

    def step_stream(self, x, h, rows, begin=False, post=False, gate=None, index=None, scale=1.0):
        """A step on the residual stream x (rows of float32 or 16 bits, updated in place).  h: rows of the layer's type, in it this layer's input as the layer
        before left it (begin: the norm of x by norm_in is taken first), after it the norm by norm_next of the new stream.  What is added is the layer's output,
        behind a norm by norm_out where post is set, times scale and its row of gate, or row index[i] of it.  x and h lie apart from each other and the others, each from the
        first of its rows to the last: not as columns of one buffer."""
        self._check(rows, h)
        if self.hidden > MOST_STREAM:
            raise ValueError(f"a stream has at most {MOST_STREAM} values a row")
        types = {torch.float32: nnv.F32, torch.float16: nnv.F16, torch.bfloat16: nnv.BF16}
        if not (isinstance(x, torch.Tensor) and x.dtype in types and x.device == self.qkv.device and x.dim() == 2 and x.shape[0] >= rows and x.shape[1] == self.hidden
                and x.stride(1) == 1 and (rows <= 1 or x.stride(0) >= self.hidden) and x.data_ptr() % 16 == 0):
            raise ValueError(f"expected a stream of {rows} rows or more of {self.hidden} values on {self.qkv.device}, each without gaps, the first 16-byte aligned")
        gates, stride = (0, 0) if gate is None or gate.dim() != 2 else (gate.shape[0], gate.stride(0))
        if gate is not None and not (isinstance(gate, torch.Tensor) and gate.dtype == self.dtype and gate.device == self.qkv.device and gate.dim() == 2 and gates >= 1
                                     and gate.shape[1] == self.hidden and gate.stride(1) == 1 and (gates == 1 or stride >= self.hidden) and gate.data_ptr() % 16 == 0
                                     and (index is not None or gates == 1 or gates >= rows)):
            raise ValueError(f"expected gates of {self.hidden} {self.dtype} on {self.qkv.device}, one, {rows} or an index for each row")
        if not math.isfinite(scale):
            raise ValueError("expected a finite scale")
        if index is not None and not (isinstance(index, torch.Tensor) and index.dtype == torch.int32 and index.device == self.qkv.device and index.is_contiguous() and index.numel() >= rows):
            raise ValueError(f"expected {rows} int32 or more on {self.qkv.device}")
        # from the first byte to the last of what is written, and of what is read beside it
        span = lambda t, values: (t.data_ptr(), t.data_ptr() + values * t.element_size())  # noqa: E731
        matrix = lambda t, m: span(t, (m - 1) * t.stride(0) + self.hidden)  # noqa: E731
        written, read = [matrix(x, rows), matrix(h, rows)], [matrix(self.out, rows)]
        if gate is not None:
            read += [matrix(gate, gates)] + ([] if index is None else [span(index, rows)])
        if rows and any(a < end and first < b for i, (a, b) in enumerate(written) for first, end in written[:i] + read):
            raise ValueError("expected the stream and the norms apart from each other, from gates and indices and from the layer's own rows")
        desc = nnv.ResidualDesc(n=self.hidden, x_dtype=types[x.dtype], y_dtype=self.desc.dtype, h_dtype=self.desc.dtype, scale=scale, eps=self.desc.eps)
        if begin:
            nnv.nnv_residual_norm(desc, rows, x, x.stride(0), None, 0, None, 0, None, 0, None, self.norm_in, None, 0, h, h.stride(0))
        self.step(h, self.out, rows)
        nnv.nnv_residual_norm(desc, rows, x, x.stride(0), self.out, self.out.stride(0), self.norm_out if post else None, gates, gate, stride, index, self.norm_next,
                              x, x.stride(0), h, h.stride(0))


def _time(f, reps):
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    a.record()
    for _ in range(reps):
        f()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) * 1e3 / reps


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, value in (("hidden", 4096), ("q-heads", 32), ("kv-heads", 8), ("head-dim", 128), ("requests", 64), ("prompt", 512), ("steps", 64)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--keep", type=int, default=0, help="blocks of 64 tokens that a row sees (0: all)")
    ap.add_argument("--shared", type=int, default=0, help="tokens that all requests begin with, in whole blocks of 64")
    a = ap.parse_args(argv)
    torch.manual_seed(220607446)
    rows = max(a.requests * a.prompt, a.shared)
    layer = AttentionLayer(a.hidden, a.q_heads, a.kv_heads, a.head_dim, a.requests, rows, a.shared + a.prompt + a.steps + 8, keep=a.keep, last=min(2, a.keep - 1) if a.keep else 2,
                           groups=1 if a.shared else 0)
    dev = layer.device
    w_qkv = torch.randn(layer.qkv_desc.n, a.hidden, device=dev) * a.hidden ** -0.5
    w_out = torch.randn(a.hidden, layer.q_size, device=dev) * layer.q_size ** -0.5
    x = torch.randn(rows, a.hidden, device=dev).to(layer.dtype)
    y = torch.empty_like(x)
    layer.transform_weights(w_qkv, w_out)                    # the library and the GPU are awake after this
    torch.cuda.synchronize()
    print(f"weights to 8 bits        {_time(lambda: layer.transform_weights(w_qkv, w_out), 3):10.1f} us")
    if a.shared:
        layer.fresh[0] = a.shared
        print(f"prefix,  {a.shared:7d} rows    {_time(lambda: layer.step(x, y, a.shared), 1):10.1f} us")
        layer.share([0, a.requests], [a.shared])
    layer.fresh.fill_(a.prompt)
    rows = a.requests * a.prompt
    print(f"prompts, {rows:7d} rows    {_time(lambda: layer.step(x, y, rows), 1):10.1f} us")
    layer.fresh.fill_(1)
    n = a.requests
    layer.step(x, y, n)
    torch.cuda.synchronize()
    stream, h = x[:n].float(), x[:n].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step_stream(stream, h, n)
    print(f"a token, {n:7d} rows    {_time(graph.replay, a.steps):10.1f} us a replayed step")
    for name, part in (("plan", lambda: layer.plan(n)), ("project", lambda: layer.project(x, n)), ("append", lambda: layer.append(n)),
                       ("attend", lambda: layer.attend(n)), ("finish", lambda: layer.finish(y, n))):
        print(f"  {name:20s}   {_time(part, 50):10.1f} us by itself")
    print(f"tokens held by each      {int(layer.held[0]):10d}")


if __name__ == "__main__":
    main()
