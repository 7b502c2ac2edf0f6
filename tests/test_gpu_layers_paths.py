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


@pytest.mark.parametrize("fmt", ["bf16", "fp16"])
@pytest.mark.parametrize("t,k,n,count,rank", [s[:5] for s in ADAPTERS])
def test_adapters_of_long_batches(fl, t, k, n, count, rank, fmt):  # noqa: F811
    """Runs of one adapter and, in between, rows of two or three taking turns."""
    g, h = rng(t + k + rank), HALF[fmt]
    X, C = gauss(g, t, k, to=h), gauss(g, t, n)
    A, B = gauss(g, count, rank, k, std=1 / math.sqrt(k), to=h), gauss(g, count, n, rank, std=0.3, to=h)
    i = torch.arange(t)
    first = torch.randint(0, count + 1, (t // 50 + 1,), generator=g)
    index = ((first[i // 50] + i % (i // 50 % 3 + 1)) % (count + 1) - 1).to(torch.int32)
    assert sorted(set(index.tolist())) == list(range(-1, count))
    scale = torch.rand(count, generator=g) * 4 - 2
    Cg, Xg, Ag, Bg, sg = (placed(v, 1) if k % 8 else v.cuda() for v in (C, X, A, B, scale))
    (Y, beside) = kept((t, n), 1, torch.float32)
    fl.adapters(Cg, Xg, Ag, Bg, index.cuda(), sg, out="f32", Y=Y)
    want, size = C.double(), C.double().abs()
    for a in range(count):
        r = (index == a).nonzero().flatten()
        x, p, q, s = X[r].double(), A[a].double().t(), B[a].double().t(), float(scale[a])
        want[r] += s * ((x @ p) @ q)
        size[r] += abs(s) * ((x.abs() @ p.abs()) @ q.abs())
    within(Y, want, size * (k + rank + 8) * 2 * U, "Y")
    assert beside() and torch.equal(Y.cpu()[index == -1], C[index == -1])
    assert torch.equal(fl.adapters(Cg, Xg, Ag, Bg, index.cuda(), sg), Y.to(h))


@pytest.mark.parametrize("fmt,pairs", [("bf16", "half"), ("fp16", "interleaved")])
@pytest.mark.parametrize("t,hq,hkv,hd,rd", [s[:5] for s in GAINS])
def test_gains_of_long_batches(fl, t, hq, hkv, hd, rd, fmt, pairs):  # noqa: F811
    g, h, eps = rng(t + hd), HALF[fmt], 1e-5
    C = gauss(g, t, (hq + 2 * hkv) * hd, std=1.5)
    gains = [gauss(g, hd, std=0.5) + 1, gauss(g, hd, std=0.5) - 1]
    pos = torch.randint(0, 1 << 20, (t,), generator=g)
    freq = torch.pow(10000.0, -torch.arange(rd // 2, dtype=torch.float64) * 2 / rd).float()
    # (a mean of their own, so that the sums grow with the tokens)
    d = [gauss(g, t, n, hd, std=0.5, to=h) + 0.25 for n in (hq, hkv, hkv)]
    kw = dict(eps=eps, pairs=pairs)
    dC, dgq, dgk = fl.heads_grad(*[x.cuda() for x in d], C.cuda(), pos.cuda(), freq.cuda(), gq=gains[0].cuda(),
                                 gk=gains[1].cuda(), **kw)
    leaves = [C.double().requires_grad_(True)] + [x.double().requires_grad_(True) for x in gains]
    out = heads64(leaves[0], hq, hkv, hd, pos, freq, leaves[1], leaves[2], eps, pairs)
    grads = torch.autograd.grad(out, leaves, [x.double() for x in d])
    x = C.double().view(t, -1, hd)
    xr = (x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)).abs()
    for got, want, part, dy in ((dgq, grads[1], xr[:, :hq], d[0]), (dgk, grads[2], xr[:, hq:hq + hkv], d[1])):
        # an entry rotated back: at most sqrt(2) of the head's largest
        size = (part * dy.double().abs().amax(-1, keepdim=True) * 1.5).sum((0, 1))
        # every work-group's sum is of its own tokens and heads, 1/1024 of them, in FP32; their sum in FP64
        terms = -(-t // 1024) * part.shape[1] + 8
        within(got, want, size * (2 * terms + hd + 40) * U, "gain")
    # the last tokens, which a work-group takes after others, are those of a call on them alone
    tail = 100
    alone = fl.heads_grad(*[v[-tail:].contiguous().cuda() for v in d], C[-tail:].contiguous().cuda(),
                          pos[-tail:].contiguous().cuda(), freq.cuda(), gq=gains[0].cuda(), gk=gains[1].cuda(), **kw)
    assert torch.equal(alone[0], dC[-tail:])


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_faulty_products_reach_the_gradient(fl, act):  # noqa: F811
    """Infinite and NaN entries of P show in the entries of dP that they enter, and in no other."""
    f, inf, nan = 4, float("inf"), float("nan")
    P = torch.ones(4, 2 * f)
    P[0, 1], P[1, f + 2], P[2, 3], P[3, f] = inf, nan, nan, -inf
    dH = torch.full((4, f), 2.0, dtype=torch.bfloat16).cuda()
    dP, dPt = fl.gated_grad(dH, P.cuda(), act=act, transpose=True)
    assert torch.equal(dPt.t().isnan(), dP.isnan()) and torch.equal(dPt.t().isinf(), dP.isinf())
    dP = dP.cpu()
    assert dP[0, f + 1] == inf                              # dU = dH act(inf)
    assert torch.isnan(dP[1, 2]) and torch.isnan(dP[2, 3]) and torch.isnan(dP[2, f + 3])
    assert dP[3, 0] == -inf                                 # dG = dH U act'(1), act'(1) > 0
    assert int((~torch.isfinite(dP)).sum()) == 5
    H = fl.gated_narrow(P.cuda(), "bf16", act=act).cpu()
    assert H[0, 1] == inf and torch.isnan(H[1, 2]) and torch.isnan(H[2, 3]) and H[3, 0] == -inf
    assert int((~torch.isfinite(H)).sum()) == 4


def test_the_smallest_eps(fl):  # noqa: F811
    """A head of zeros is zero with the smallest eps there is, and so is its gradient where the output's is."""
    hd, t = 64, 3
    C, gain = torch.zeros(t, 4 * hd).cuda(), torch.ones(hd).cuda()
    pos, freq = torch.arange(t).cuda(), torch.ones(hd // 2).cuda()
    kw = dict(gq=gain, gk=gain, eps=2.0 ** -126)
    q, k, v = fl.heads(C, 2, 1, pos, freq, "bf16", **kw)
    assert not q.any() and not k.any() and not v.any()
    for n in (hd, 33):                                       # both kernels
        z = [torch.zeros(t, m, n, dtype=torch.bfloat16).cuda() for m in (2, 1, 1)]
        g = torch.ones(n).cuda()
        dC, dgq, dgk = fl.heads_grad(*z, torch.zeros(t, 4 * n).cuda(), pos, freq[:8].contiguous(), gq=g, gk=g,
                                     eps=2.0 ** -126)
        assert not dC.any() and not dgq.any() and not dgk.any()
