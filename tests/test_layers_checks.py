"""The operators of layers.py refuse operands that do not fit before any call into the library (CPU
tensors stand in for GPU ones: shape and type are checked before the device)."""
import pytest
import torch

from paper_2609_19758_amd import layers as fl

H, F = torch.float16, torch.float32


def z(*shape, dtype=H):
    return torch.zeros(*shape, dtype=dtype)


def refuses(match, call, *args, **kw):
    with pytest.raises(ValueError, match=match):
        call(*args, **kw)


def test_gated_refuses():
    X, W = z(3, 8), z(10, 8)
    refuses("expected a tensor of 2 dimensions", fl.gated, z(3, 2, 8), W)
    refuses("X: list", fl.gated, [1], W)
    refuses("X: dtype", fl.gated, z(3, 8, dtype=F), W)
    refuses("W: 9 rows", fl.gated, X, z(9, 8))
    refuses("W: 0 rows", fl.gated, X, z(0, 8))
    refuses("act: 'tanh'", fl.gated, X, W, act="tanh")
    refuses("act: \\[\\]", fl.gated, X, W, act=[])
    refuses("not contiguous", fl.gated, z(8, 3).t(), W)
    refuses("expected a GPU tensor", fl.gated, X, W)


def test_gated_narrow_refuses():
    P = z(3, 10, dtype=F)
    refuses("fmt: 'f32'", fl.gated_narrow, P, "f32")
    refuses("P: 9 columns", fl.gated_narrow, z(3, 9, dtype=F), "fp16")
    refuses("P: 0 columns", fl.gated_narrow, z(3, 0, dtype=F), "fp16")
    refuses("P: dtype", fl.gated_narrow, z(3, 10), "fp16")
    refuses("not contiguous", fl.gated_narrow, z(10, 3, dtype=F).t(), "fp16")
    refuses("act", fl.gated_narrow, P, "fp16", act="relu")
    refuses("expected a GPU tensor", fl.gated_narrow, P, "fp16")


def test_gated_grad_refuses():
    dH = z(3, 5)
    refuses("dH: dtype", fl.gated_grad, z(3, 5, dtype=F), z(3, 10, dtype=F))
    refuses("dH: no columns", fl.gated_grad, z(3, 0), z(3, 0, dtype=F))
    refuses("act", fl.gated_grad, dH, z(3, 10, dtype=F), act=None)
    refuses("expected a GPU tensor", fl.gated_grad, dH, z(3, 10, dtype=F))


def test_gated_products_refuses():
    dP, X, W = z(3, 10), z(3, 8), z(10, 8)
    refuses("dP: dtype", fl.gated_products, z(3, 10, dtype=F), X, W)
    refuses("W: 11 rows", fl.gated_products, dP, X, z(11, 8))
    refuses("dP: shape", fl.gated_products, z(3, 12), X, W)
    refuses("dP: shape", fl.gated_products, dP, z(4, 8), W)
    refuses("expected a GPU tensor", fl.gated_products, dP, X, W)


def test_adapters_refuses():
    C, X, A, B = z(3, 6, dtype=F), z(3, 8), z(2, 4, 8), z(2, 6, 4)
    index, scale = z(3, dtype=torch.int32), z(2, dtype=F)
    refuses("X: dtype", fl.adapters, C, z(3, 8, dtype=F), A, B, index, scale)
    refuses("out: 'bf16'", fl.adapters, C, X, A, B, index, scale, out="bf16")
    refuses("A: 2 adapters of rank 0", fl.adapters, C, X, z(2, 0, 8), z(2, 6, 0), index, scale)
    refuses("A: 2 adapters of rank 257", fl.adapters, C, X, z(2, 257, 8), z(2, 6, 257), index, scale)
    refuses("A: 0 adapters", fl.adapters, C, X, z(0, 4, 8), z(0, 6, 4), index, z(0, dtype=F))
    refuses("A: \\(2, 4\\)", fl.adapters, C, X, z(2, 4), B, index, scale)
    refuses("C: shape", fl.adapters, z(4, 6, dtype=F), X, A, B, index, scale)
    refuses("C: dtype", fl.adapters, z(3, 6), X, A, B, index, scale)
    refuses("expected a GPU tensor", fl.adapters, C, X, A, B, index, scale)


def test_heads_refuses():
    C, pos, freq = z(3, 4 * 8, dtype=F), z(3, dtype=torch.int64), z(4, dtype=F)
    refuses("fmt: 'f32'", fl.heads, C, 2, 1, pos, freq, "f32")
    refuses("C: 32 columns", fl.heads, C, 3, 1, pos, freq, "fp16")
    refuses("C: 32 columns", fl.heads, C, 0, 1, pos, freq, "fp16")
    refuses("C: 32 columns", fl.heads, C, 2, 0, pos, freq, "fp16")
    refuses("C: dtype", fl.heads, z(3, 32), 2, 1, pos, freq, "fp16")
    refuses("expected a GPU tensor", fl.heads, C, 2, 1, pos, freq, "fp16")


def test_head_arguments():
    """Checked after the product's device: on their own here."""
    pos, freq, dev = z(3, dtype=torch.int64), z(4, dtype=F), None
    refuses("heads of 513 entries", fl._head_args, 3, 513, None, None, pos, freq, "half", dev)
    refuses("heads of 0 entries", fl._head_args, 3, 0, None, None, pos, None, "half", dev)
    refuses("pairs: 'odd'", fl._head_args, 3, 8, None, None, pos, freq, "odd", dev)
    refuses("gains for queries or keys only", fl._head_args, 3, 8, z(8, dtype=F), None, pos, freq, "half", dev)
    refuses("gq: shape", fl._head_args, 3, 8, z(7, dtype=F), z(8, dtype=F), pos, freq, "half", dev)
    refuses("4 frequencies for heads of 6", fl._head_args, 3, 6, None, None, pos, freq, "half", dev)
    refuses("freq: dtype", fl._head_args, 3, 8, None, None, pos, z(4), "half", dev)
    refuses("freq: \\(2, 2\\)", fl._head_args, 3, 8, None, None, pos, z(2, 2, dtype=F), "half", dev)
    assert fl._head_args(3, 8, None, None, None, None, "interleaved", dev) == (1, 0, 0, 0, 0, 0)


def test_heads_grad_refuses():
    dq, dk, dv = z(3, 2, 8), z(3, 1, 8), z(3, 1, 8)
    pos, freq = z(3, dtype=torch.int64), z(4, dtype=F)
    refuses("dq: dtype", fl.heads_grad, z(3, 2, 8, dtype=F), dk, dv, None, pos, freq)
    refuses("dq: \\(3, 16\\)", fl.heads_grad, z(3, 16), dk, dv, None, pos, freq)
    refuses("2 query and 0 key heads", fl.heads_grad, dq, z(3, 0, 8), z(3, 0, 8), None, pos, freq)
    refuses("expected a GPU tensor", fl.heads_grad, dq, dk, dv, None, pos, freq)


def test_a_stream_of_another_gpu_is_refused():
    class Stream:
        device, cuda_stream = torch.device("cuda", 1), 7

    refuses("stream: on cuda:1, the operands are on cuda:0", fl._Call, torch.device("cuda", 0), Stream())
