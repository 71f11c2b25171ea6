"""Descriptors of a program's own, with fields behind the library's: what the calls read of them is the library's part, through the compiled module and through ctypes."""
import ctypes

import pytest

import paper_2206_07446_amd as nnv
from test_binding_calls import NULL, calls, status  # noqa: F401
from test_serving_host import A


class Layer(nnv.ConvDesc):
    _fields_ = [("index", ctypes.c_int32), ("seconds", ctypes.c_double)]


class Projection(nnv.LinearDesc):
    _fields_ = [("index", ctypes.c_int64)]


class Attention(nnv.AttentionDesc):
    _fields_ = [("index", ctypes.c_int64)]


def test_calls_take_them(calls):  # noqa: F811
    conv = Layer(n=1, c=16, h=32, w=32, k=16, r=3, s=3, stride_h=1, stride_w=1, pad_h=1, pad_w=1, groups=1, dtype=nnv.F32, index=7, seconds=0.5)
    assert status(nnv.nnv_conv_forward, conv, nnv.DIRECT, None, A, None, A, None) == NULL
    assert status(nnv.nnv_transform_weights, conv, nnv.DIRECT, None, A) == NULL
    linear = Projection(n=16, k=16, x_dtype=nnv.F16, y_dtype=nnv.F16, raw_dtype=nnv.F16, index=7)
    assert status(nnv.nnv_linear_transform_weights, linear, None, A) == NULL
    attention = Attention(q_heads=1, kv_heads=1, head_dim=64, block_tokens=16, blocks=1, table_blocks=1, dtype=nnv.BF16, scale=1.0, index=7)
    assert status(nnv.nnv_kv_read, attention, 1, None, A, A, A) == NULL


def test_what_is_no_descriptor_is_refused(calls):  # noqa: F811
    class Other(ctypes.Structure):
        _fields_ = nnv.ConvDesc._fields_

    for wrong in (Other(), object(), nnv.LinearDesc()):
        with pytest.raises((TypeError, ctypes.ArgumentError)):
            nnv.nnv_transform_weights(wrong, nnv.DIRECT, A, A, stream=0)
