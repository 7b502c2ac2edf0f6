"""Kernels and loops of the operators around a delivered product that only certain sizes reach: products of
operands off 16-byte groups that are too large for padded copies, operands of a few elements, long batches in
which a work-group takes several tokens or blocks of columns.  test_layers_routes.py shows on the CPU that these
sizes reach them.

Tolerances.  u = 2^-24 (FP32's half step).  Products of small integers are exact in FP32 while the sums of their
sizes stay below 2^24: compared for equality.  Adapters: k products and rank terms, each step off by at most 2u
of the sum of sizes, and the few steps after them.  Gradients of the gains: sums over tokens and heads, each step
off by at most 2u (the sum's half step and that of its term), the terms by (hd + 40) u (a norm's sum of hd
squares, its root, a rotation)."""
import math

import pytest
import torch

from test_gpu_layers import HALF, TINY, U, act64, fl, gauss, heads64, ints, rng, step, within  # noqa: F401
from test_layers_routes import ADAPTERS, GAINS, GATED, PRODUCTS

pytestmark = pytest.mark.gpu


def placed(x, shift):
    """x on the GPU, `shift` elements into a buffer whose other elements are NaN."""
    buf = torch.full((x.numel() + shift + 16,), float("nan"), dtype=x.dtype, device="cuda")
    v = buf[shift:shift + x.numel()].view(x.shape)
    v.copy_(x)
    return v


def kept(shape, shift, dtype):
    """An output that begins `shift` elements into a buffer of sevens, and a check that nothing beside it is
    written."""
    n = math.prod(shape)
    buf = torch.full((n + shift + 16,), 7.0, dtype=dtype, device="cuda")
    return buf[shift:shift + n].view(shape), lambda: bool((buf[:shift] == 7).all() and (buf[shift + n:] == 7).all())


@pytest.mark.parametrize("fmt", ["bf16", "fp16"])
@pytest.mark.parametrize("t,d,f,shift", [s[:4] for s in GATED])
def test_gated_at_any_alignment(fl, t, d, f, shift, fmt):  # noqa: F811
    g, h = rng(t + d + f), HALF[fmt]
    X, W = (placed(ints(g, *s, to=h, lo=-2, hi=2), shift) for s in ((t, d), (2 * f, d)))
    (H, beside_h), (P, beside_p) = kept((t, f), shift, h), kept((t, 2 * f), shift, torch.float32)
    fl.gated(X, W, act="gelu_tanh", H=H, P=P)
    assert torch.equal(P.double(), torch.mm(X.double(), W.double().t().contiguous()))
    assert beside_h() and beside_p()
    assert torch.equal(fl.gated_narrow(P.contiguous(), fmt, act="gelu_tanh"), H)
    p = P.double().cpu()
    want = act64(p[:, :f], "gelu_tanh") * p[:, f:]
    x = p[:, :f]
    # as in test_gpu_layers.py: the exponential's argument, a few units, half a step of the half format; past
    # FP16's largest number infinite
    tol = want.abs() * (step(fmt) + (x * x + x.abs() + 16).clamp_max(1e5) * 4 * U) + TINY[fmt] + (x * p[:, f:]).abs() * 2.0 ** -126
    fits = want.abs() < torch.finfo(h).max
    within(torch.where(fits.cuda(), H.double(), 0.0), torch.where(fits, want, 0.0), tol, "H")
    without, none = fl.gated(X, W, act="gelu_tanh", deliver=False)
    assert none is None and torch.equal(without, H)


@pytest.mark.parametrize("fmt", ["bf16", "fp16"])
@pytest.mark.parametrize("t,d,f,shift", [s[:4] for s in PRODUCTS])
def test_backward_products_at_any_alignment(fl, t, d, f, shift, fmt):  # noqa: F811
    g, h = rng(t + d + f), HALF[fmt]
    dP, X, W = (placed(ints(g, *s, to=h, lo=-2, hi=2), shift) for s in ((t, 2 * f), (t, d), (2 * f, d)))
    (dX, beside_x), (dW, beside_w) = kept((t, d), shift, torch.float32), kept((2 * f, d), shift, torch.float32)
    fl.gated_products(dP, X, W, dX=dX, dW=dW)
    assert torch.equal(dX.double(), torch.mm(dP.double(), W.double()))
    assert torch.equal(dW.double(), torch.mm(dP.double().t().contiguous(), X.double()))
    assert beside_x() and beside_w()
    assert torch.equal(fl.gated_products(dP, X, W, need_dw=False)[0], dX)
    assert torch.equal(fl.gated_products(dP, X, W, need_dx=False)[1], dW)
