"""The serving operators without a GPU: what the oracle's formats are, sizes, and every refusal, through the compiled module and
through ctypes.  Pointers here are no memory: a call that is not refused must do nothing."""
import numpy as np
import pytest
import torch

import paper_2206_07446_amd as nnv
from oracle import serving as OS
from paper_2206_07446_amd import binding

NULL, BAD_DESC, UNSUPPORTED, WORKSPACE, ALIGN, ARG = -1, -2, -3, -4, -5, -7
A = 4096


@pytest.fixture(params=["module", "ctypes"])
def calls(request, monkeypatch):
    nnv.load()
    if request.param == "module":
        assert binding._native.__name__ == "_nnvpy"
    else:
        monkeypatch.setattr(binding, "_native", binding._CtypesCalls)


def status(fn, *args):
    with pytest.raises(nnv.NnvError) as e:
        fn(*args, stream=0)
    return e.value.status


def linear(**kw):
    return nnv.LinearDesc(**{**dict(n=256, k=512, x_dtype=nnv.BF16, y_dtype=nnv.BF16, raw_dtype=nnv.F32), **kw})


def layer(**kw):
    return nnv.AttentionDesc(**{**dict(q_heads=8, kv_heads=2, head_dim=128, block_tokens=64, blocks=10, table_blocks=4, dtype=nnv.BF16, scale=0.1, eps=1e-6), **kw})


def test_e4m3_of_the_oracle_is_the_type():
    g = torch.Generator().manual_seed(1)
    x = torch.cat((torch.randn(4000, generator=g, dtype=torch.float64) * 50, torch.tensor(np.r_[OS.E4M3, (OS.E4M3[1:] + OS.E4M3[:-1]) / 2])))
    x = x.clamp(-448, 448).float()                      # halves between codes are float32 values
    assert np.array_equal(OS.nearest(x.double().numpy(), OS.E4M3), x.to(torch.float8_e4m3fn).double().numpy())


def test_scales_of_the_oracle():
    a = np.array([0, 2.0 ** -140, 1, 447, 448, 448.0001, 449, 1e30, 3.4e38])
    s = OS.scale_e4m3(a)
    assert ((a <= 448 * s) & ((a > 224 * s) | (s == 2.0 ** -126))).all()
    a = np.array([0, 2.0 ** -140, 1, 3.4999, 3.5, 6.9999, 7, 1e30, 2.9e38])
    s = OS.scale_e2m1(a, False)
    assert (((a < 7 * s) & (a >= 3.5 * s)) | (s == 2.0 ** -126) & (a < 3.5 * s)).all()
    assert OS.scale_e2m1(np.array([65504.0]), True) == 2.0 ** 13 and OS.scale_e2m1(np.array([3.4e38]), False) == 2.0 ** 125
    assert list(OS.nearest(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5, 6.9]), OS.E2M1)) == [0, 1, 1, 2, 2, 4, 4, -4, 6]


def test_linear_sizes(calls):
    assert nnv.nnv_linear_transformed_bytes(linear()) == 256 * 512 + 256
    assert nnv.nnv_linear_transformed_bytes(linear(n=1, k=1)) == 128 * 256 + 256
    assert nnv.nnv_linear_transformed_bytes(linear(n=129, k=513)) == 256 * 768 + 256
    for m in (0, 1, 16):                                 # a few rows are rounded where they are used
        assert nnv.nnv_linear_workspace_bytes(linear(), m) == 0
    for m in (17, 32, 33, 1000):
        assert nnv.nnv_linear_workspace_bytes(linear(k=500), m) >= (m > 16) * -(-m // 16) * 16 * 512


@pytest.mark.parametrize("bad", [dict(n=0), dict(k=-1), dict(x_dtype=3), dict(y_dtype=-1), dict(raw_dtype=9), dict(n=1 << 23), dict(k=1 << 21)])
def test_linear_descriptors(calls, bad):
    d = linear(**bad)
    assert nnv.nnv_linear_transformed_bytes(d) == 0 and nnv.nnv_linear_workspace_bytes(d, 4) == 0
    assert status(nnv.nnv_linear_transform_weights, d, A, A) == BAD_DESC
    assert status(nnv.nnv_linear_forward, d, 40, A, 512, A, None, A, 256, A, 1 << 30) == BAD_DESC


def test_linear_refusals(calls):
    d, f, big = linear(), nnv.nnv_linear_forward, 1 << 30
    assert status(nnv.nnv_linear_transform_weights, d, None, A) == NULL
    assert status(nnv.nnv_linear_transform_weights, d, A, A + 8) == ALIGN
    f(d, 0, None, 0, None, None, None, 0, None, 0, stream=0)
    assert status(f, d, -1, A, 512, A, None, A, 256, A, big) == ARG
    assert status(f, d, 1 << 20, A, 512, A, None, A, 256, A, big) == ARG
    assert status(f, d, 40, A, 511, A, None, A, 256, A, big) == ARG
    assert status(f, d, 40, A, 512, A, None, A, 255, A, big) == ARG
    for i in (2, 4, 6):
        args = [d, 40, A, 512, A, None, A, 256, A, big]
        args[i] = None
        assert status(f, *args) == NULL
        args[i] = A + 4
        assert status(f, *args) == ALIGN
    assert status(f, d, 40, A, 512, A, A + 2, A, 256, A, big) == ALIGN
    assert status(f, d, 40, A, 512, A, None, A, 256, None, big) == NULL
    assert status(f, d, 40, A, 512, A, None, A, 256, A, 16) == WORKSPACE
    assert status(f, d, 40, A, 512, A, None, A, 256, torch.empty(8)) == WORKSPACE


@pytest.mark.parametrize("bad,want", [(dict(q_heads=0), BAD_DESC), (dict(q_heads=9), BAD_DESC), (dict(q_heads=2048), BAD_DESC), (dict(kv_heads=0), BAD_DESC),
                                      (dict(blocks=0), BAD_DESC), (dict(table_blocks=0), BAD_DESC), (dict(rotary_dim=3, positions=9), BAD_DESC),
                                      (dict(rotary_dim=130, positions=9), BAD_DESC), (dict(rotary_dim=64), BAD_DESC), (dict(rotary_interleaved=2), BAD_DESC),
                                      (dict(window=-1), BAD_DESC), (dict(sinks=-1), BAD_DESC), (dict(scale=float("nan")), BAD_DESC), (dict(eps=-1.0), BAD_DESC),
                                      (dict(dtype=7), BAD_DESC), (dict(table_blocks=1 << 26), BAD_DESC), (dict(dtype=nnv.F32), UNSUPPORTED),
                                      (dict(head_dim=96), UNSUPPORTED), (dict(block_tokens=48), UNSUPPORTED), (dict(block_tokens=8), UNSUPPORTED),
                                      (dict(block_tokens=512), UNSUPPORTED)])
def test_attention_descriptors(calls, bad, want):
    d = layer(**bad)
    assert nnv.nnv_kv_cache_bytes(d) == 0 and nnv.nnv_kv_attention_workspace_bytes(d, 1, 1) == 0
    assert status(nnv.nnv_kv_plan, d, 1, 1, *[A] * 9, A + 64) == want
    assert status(nnv.nnv_qk_norm_rope, d, 1, A, 1024, A, 256, A, 256, None, None, None, A, A, A, None, A) == want
    assert status(nnv.nnv_kv_read, d, 1, A, A, A, A) == want
    assert status(nnv.nnv_kv_attention, d, 1, 1, A, A, A, A, A, A, A, A, 1 << 30) == want


def test_cache_sizes(calls):
    assert nnv.nnv_kv_cache_bytes(layer()) == 10 * 2 * 64 * (128 + 8)
    assert nnv.nnv_kv_cache_bytes(layer(head_dim=64, block_tokens=16, kv_heads=1)) == 10 * 16 * 68
    d = layer(blocks=1 << 20, block_tokens=256, kv_heads=8)
    assert nnv.nnv_kv_cache_bytes(d) == (1 << 28) * 8 * 136          # no 32-bit product


def test_plan_refusals(calls):
    d, f = layer(), nnv.nnv_kv_plan
    good = [A + 64 * i for i in range(10)]
    for n, r in ((-1, 1), (1, -1), (1 << 21, 1), (1, 1 << 25)):
        assert status(f, d, n, r, *good) == ARG
    for i in range(10):
        args = list(good)
        args[i] = None
        assert status(f, d, 1, 1, *args) == NULL
        args[i] = A + 2
        assert status(f, d, 1, 1, *args) == ALIGN
    args = list(good)
    args[8] = A + 4                                                   # slots are of 64 bits
    assert status(f, d, 1, 1, *args) == ALIGN
    args = list(good)
    args[9] = args[3]                                                 # free_left in the place of free_count
    assert status(f, d, 1, 1, *args) == ARG


def test_rope_refusals(calls):
    d, f = layer(rotary_dim=128, positions=99), nnv.nnv_qk_norm_rope
    good = [A, 1024, A, 256, A, 256, A, A, A, A, A, A, A, A]
    f(d, 0, *good, stream=0)
    f(d, 3, None, 0, None, 0, None, 0, None, None, None, None, None, None, None, None, stream=0)
    assert status(f, d, -1, *good) == ARG
    for i, v in ((1, 1023), (3, 255), (5, 255)):
        args = list(good)
        args[i] = v
        assert status(f, d, 2, *args) == ARG
    for i in (4, 8, 9, 10, 11):                                       # v, rope, positions, slots, q_out
        args = list(good)
        args[i] = None
        assert status(f, d, 2, *args) == NULL
    args = list(good)
    args[12] = args[13] = None                                        # keys to nowhere
    assert status(f, d, 2, *args) == NULL
    for i in (0, 2, 4, 6, 7, 8, 11, 12, 13):
        args = list(good)
        args[i] = A + 8
        assert status(f, d, 2, *args) == ALIGN
    args = list(good)
    args[10] = A + 4
    assert status(f, d, 2, *args) == ALIGN
    assert status(f, layer(q_heads=1024, kv_heads=1024, head_dim=256), 1 << 24, *[1 << 30 if i in (1, 3, 5) else v for i, v in enumerate(good)]) == ARG


def test_read_and_attention_refusals(calls):
    d = layer()
    nnv.nnv_kv_read(d, 0, None, None, None, None, stream=0)
    nnv.nnv_kv_read(d, 5, None, None, None, None, stream=0)
    assert status(nnv.nnv_kv_read, d, -1, A, A, A, A) == ARG
    assert status(nnv.nnv_kv_read, d, 1 << 28, A, A, A, A) == ARG
    assert status(nnv.nnv_kv_read, d, 1, None, A, A, A) == NULL
    assert status(nnv.nnv_kv_read, d, 1, A, None, A, A) == NULL
    assert status(nnv.nnv_kv_read, d, 1, A + 4, A, A, A) == ALIGN
    assert status(nnv.nnv_kv_read, d, 1, A, A, A + 8, A) == ALIGN
    f, big = nnv.nnv_kv_attention, 1 << 40
    good = [A] * 7
    f(d, 3, 0, *[None] * 8, 0, stream=0)
    for n, r in ((-1, 1), (1, -1), (1 << 21, 1), (1, 1 << 25)):
        assert status(f, d, n, r, *good, A, big) == ARG
        assert nnv.nnv_kv_attention_workspace_bytes(d, n, r) == 0
    for i in range(7):
        args = list(good)
        args[i] = None
        assert status(f, d, 1, 1, *args, A, big) == NULL
        args[i] = A + 2
        assert status(f, d, 1, 1, *args, A, big) == ALIGN
    # launches of 2^32 threads and more
    assert status(nnv.nnv_kv_read, d, 1 << 26, A, A, A, A) == ARG
    assert nnv.nnv_kv_attention_workspace_bytes(d, 1 << 19, 1 << 23) == 0 and status(f, layer(q_heads=32), 1, 1 << 24, *good, A, big) == ARG
    long = layer(table_blocks=1000)
    need = nnv.nnv_kv_attention_workspace_bytes(long, 1, 1)
    assert need > 0
    assert status(f, long, 1, 1, *good, None, big) == NULL
    assert status(f, long, 1, 1, *good, A, need - 1) == WORKSPACE
    assert status(f, long, 1, 1, *good, A + 8, need) == ALIGN


def test_arguments_of_other_types(calls):
    other = (TypeError, nnv.binding.ctypes.ArgumentError)
    with pytest.raises(other):
        nnv.nnv_linear_forward(layer(), 1, A, 512, A, None, A, 256, A, 1 << 20, stream=0)
    with pytest.raises(other):
        nnv.nnv_kv_read(linear(), 1, A, A, A, A, stream=0)
    with pytest.raises(other):
        nnv.nnv_kv_plan(object(), 1, 1, *[A] * 10, stream=0)
    with pytest.raises(OverflowError):
        nnv.nnv_linear_forward(linear(), 1 << 33, A, 512, A, None, A, 256, A, 1 << 20, stream=0)
    with pytest.raises(AttributeError):
        nnv.nnv_kv_read(layer(), 1, "slots", A, A, A, stream=0)


def test_plan_of_the_oracle():
    table, starts, lengths, positions, slots, left = OS.plan([0, 16, 15, 3], [17, 1, 1, 0], [9, 8, 7, 6], 4, [[-1, -1], [5, -1], [4, -1], [3, -1]], 16, 10, 20)
    assert table == [[6, 7], [5, 8], [4, -1], [3, -1]] and starts == [0, 17, 18, 19, 19] and lengths == [17, 17, 16, 3] and left == 1
    assert positions[16:] == [16, 16, 15, -1] and slots[16:] == [7 * 16, 8 * 16, 4 * 16 + 15, -1]
