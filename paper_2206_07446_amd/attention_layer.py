"""One attention layer of a language model as a serving program runs it, from request lengths to the layer's output
rows: the cold start (weights to 8 bits), a step that takes the requests' prompts in, and steps of one token a request
replayed from a HIP graph.  The layer keeps every buffer, so that a step is seven calls and no allocation.

`python -m paper_2206_07446_amd.attention_layer --requests 64 --prompt 512 --steps 64` prints the time of each part.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as nnv

DTYPES = {nnv.F16: torch.float16, nnv.BF16: torch.bfloat16}


class AttentionLayer:
    """Weights, cache, block table and buffers for up to `rows` rows a step and `requests` requests of `tokens` tokens (whole blocks of them)."""

    def __init__(self, hidden, q_heads, kv_heads, head_dim, requests, rows, tokens, block_tokens=64, dtype=nnv.BF16, theta=10000.0, window=0, sinks=0,
                 device="cuda:0"):
        self.device, self.dtype, self.requests, self.rows, self.hidden = torch.device(device), DTYPES[dtype], requests, rows, hidden
        width = -(-tokens // block_tokens)
        self.desc = nnv.AttentionDesc(q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, block_tokens=block_tokens, blocks=requests * width,
                                      table_blocks=width, rotary_dim=head_dim, rotary_interleaved=0, positions=width * block_tokens, window=window, sinks=sinks, dtype=dtype,
                                      scale=head_dim ** -0.5, eps=1e-6)
        self.q_size, self.kv_size = q_heads * head_dim, kv_heads * head_dim
        self.qkv_desc = nnv.LinearDesc(n=self.q_size + 2 * self.kv_size, k=hidden, x_dtype=dtype, y_dtype=dtype, raw_dtype=nnv.F32)
        self.out_desc = nnv.LinearDesc(n=hidden, k=self.q_size, x_dtype=dtype, y_dtype=dtype, raw_dtype=nnv.F32)
        new = lambda *shape, dtype=self.dtype: torch.empty(*shape, dtype=dtype, device=self.device)  # noqa: E731
        bytes_ = lambda n: new(max(16, n), dtype=torch.uint8)  # noqa: E731
        self.qkv_tx, self.out_tx = (bytes_(nnv.nnv_linear_transformed_bytes(d)) for d in (self.qkv_desc, self.out_desc))
        self.cache = bytes_(nnv.nnv_kv_cache_bytes(self.desc))
        # what a call over m rows needs of its scratch goes up and down with m, where the number of parts that it splits into changes: the most of every size
        need = max(max(nnv.nnv_kv_attention_workspace_bytes(self.desc, requests, m), *(nnv.nnv_linear_workspace_bytes(d, m) for d in (self.qkv_desc, self.out_desc)))
                   for m in range(1, rows + 1))
        self.workspace = bytes_(need)
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

    def attend(self, rows):
        self._check(rows)
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
    a = ap.parse_args(argv)
    torch.manual_seed(220607446)
    rows = a.requests * a.prompt
    layer = AttentionLayer(a.hidden, a.q_heads, a.kv_heads, a.head_dim, a.requests, rows, a.prompt + a.steps + 8)
    dev = layer.device
    w_qkv = torch.randn(layer.qkv_desc.n, a.hidden, device=dev) * a.hidden ** -0.5
    w_out = torch.randn(a.hidden, layer.q_size, device=dev) * layer.q_size ** -0.5
    x = torch.randn(rows, a.hidden, device=dev).to(layer.dtype)
    y = torch.empty_like(x)
    layer.transform_weights(w_qkv, w_out)                    # the library and the GPU are awake after this
    torch.cuda.synchronize()
    print(f"weights to 8 bits        {_time(lambda: layer.transform_weights(w_qkv, w_out), 3):10.1f} us")
    layer.fresh.fill_(a.prompt)
    print(f"prompts, {rows:7d} rows    {_time(lambda: layer.step(x, y, rows), 1):10.1f} us")
    layer.fresh.fill_(1)
    n = a.requests
    layer.step(x, y, n)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step(x, y, n)
    print(f"a token, {n:7d} rows    {_time(graph.replay, a.steps):10.1f} us a replayed step")
    for name, part in (("plan", lambda: layer.plan(n)), ("project", lambda: layer.project(x, n)), ("append", lambda: layer.append(n)),
                       ("attend", lambda: layer.attend(n)), ("finish", lambda: layer.finish(y, n))):
        print(f"  {name:20s}   {_time(part, 50):10.1f} us by itself")
    print(f"tokens held by each      {int(layer.held[0]):10d}")


if __name__ == "__main__":
    main()
