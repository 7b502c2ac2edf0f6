"""The operators around a delivered product against their definitions in 64 bits.

Tolerances.  u = 2^-24 (FP32's half step); eps/2 of a half format is its half step.
  - products of small integers are exact in FP32 as long as the sums stay below 2^24: compared for
    equality;
  - products of Gaussian data: K terms, each sum's step off by at most a whole unit 2u of the partial
    sum (the matrix instruction may truncate), so K 2u sum |a||b| per entry;
  - an activation's value: the exponential takes its argument with a relative error of 2u, so e^x is
    off by 2u |x| and erfc(-x / sqrt 2) (relative slope at most x^2 + 2) by 2u (x^2 + 2), with a few
    units for the functions themselves: (x^2 + |x| + 16) 4u relative, then half a step of the half
    format, and what is below its smallest number.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"bf16": torch.bfloat16, "fp16": torch.float16}
TINY = {"bf16": 2.0 ** -126, "fp16": 2.0 ** -24}     # a step of the smallest numbers, flushed or not


@pytest.fixture(scope="module")
def fl():
    assert torch.cuda.is_available()
    from paper_2609_19758_amd import fpsketch, layers
    fpsketch.load()
    return layers


def rng(seed):
    return torch.Generator().manual_seed(seed)


def gauss(g, *shape, std=1.0, to=torch.float32):
    return (torch.randn(*shape, generator=g) * std).to(to)


def ints(g, *shape, to, lo=-3, hi=3):
    return torch.randint(lo, hi + 1, shape, generator=g).to(to)


def step(fmt):
    return torch.finfo(HALF[fmt]).eps / 2


def act64(x, name):
    if name == "silu":
        return x * torch.sigmoid(x)
    if name == "gelu":
        return 0.5 * x * torch.special.erfc(-x * math.sqrt(0.5))
    z = 2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)
    return x * torch.sigmoid(z)


def act_slope64(x, name):
    if name == "silu":
        s = torch.sigmoid(x)
        return s + x * s * (1 - s)
    if name == "gelu":
        return (0.5 * torch.special.erfc(-x * math.sqrt(0.5))
                + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi))
    c = 2 * math.sqrt(2 / math.pi)
    s = torch.sigmoid(c * (x + 0.044715 * x ** 3))
    return s + x * s * (1 - s) * c * (1 + 3 * 0.044715 * x * x)


def within(got, want, tol, what):
    d = (got.double().cpu() - want).abs()
    bad = ~(d <= tol)
    assert not bad.any(), (what, int(bad.sum()), float((d / tol).nan_to_num(9e9).max()))


def h_tol(P, f, H, fmt):
    x = P[:, :f]
    return (H.abs() * (step(fmt) + (x * x + x.abs() + 16) * 4 * U) + TINY[fmt]
            + (x * P[:, f:]).abs() * 2.0 ** -126)


# ---- gated feed-forward ----------------------------------------------------------------------

SHAPES = [  # t, d, f: one of everything, tile edges and their neighbours, odd widths, long sums
    (1, 1, 1), (1, 8, 4), (1, 7, 3), (3, 64, 16), (1, 4096, 128), (5, 72, 24), (16, 128, 64),
    (17, 129, 65), (31, 63, 33), (33, 200, 40), (64, 256, 128), (65, 264, 136), (127, 1000, 77),
    (128, 512, 256), (129, 520, 264), (200, 40, 1000), (257, 328, 520), (300, 2048, 24),
    (512, 64, 64), (70, 4104, 8), (2, 9000, 40)]


@pytest.mark.parametrize("fmt", ["bf16", "fp16"])
@pytest.mark.parametrize("t,d,f", SHAPES)
def test_products_of_integers_are_exact(fl, t, d, f, fmt):
    g = rng(t * 31 + d * 7 + f)
    h = HALF[fmt]
    X, W = ints(g, t, d, to=h), ints(g, 2 * f, d, to=h)
    dP = ints(g, t, 2 * f, to=h)
    H, P = fl.gated(X.cuda(), W.cuda())
    assert torch.equal(P.double().cpu(), X.double() @ W.double().t())
    H2, none = fl.gated(X.cuda(), W.cuda(), deliver=False)
    assert none is None and torch.equal(H, H2)
    assert torch.equal(fl.gated_narrow(P, fmt), H)
    dX, dW = fl.gated_products(dP.cuda(), X.cuda(), W.cuda())
    assert torch.equal(dX.double().cpu(), dP.double() @ W.double())
    assert torch.equal(dW.double().cpu(), dP.double().t() @ X.double())


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("fmt", ["bf16", "fp16"])
@pytest.mark.parametrize("t,d,f", [(1, 512, 96), (9, 130, 30), (40, 1024, 64), (150, 320, 200),
                                   (300, 256, 512)])
def test_gated_block_and_its_gradient(fl, t, d, f, fmt, act):
    g = rng(5 * t + d + f)
    h = HALF[fmt]
    X, W = gauss(g, t, d, to=h), gauss(g, 2 * f, d, std=2 / math.sqrt(d), to=h)
    H, P = fl.gated(X.cuda(), W.cuda(), act=act)
    x, w = X.double(), W.double()
    within(P, x @ w.t(), d * 2 * U * (x.abs() @ w.abs().t()), "P")
    p = P.double().cpu()
    want = act64(p[:, :f], act) * p[:, f:]
    within(H, want, h_tol(p, f, want, fmt), "H")
    assert torch.equal(fl.gated_narrow(P, fmt, act=act), H)
    dH = gauss(g, t, f, std=0.5, to=h)
    dP, dPt = fl.gated_grad(dH.cuda(), P, act=act, transpose=True)
    assert torch.equal(dPt, dP.t().contiguous())
    assert torch.equal(fl.gated_grad(dH.cuda(), P, act=act)[0], dP)
    gate, up, dh = p[:, :f], p[:, f:], dH.double()
    # act' is a sum of a term of at most 1 and one that stays below 1.2: its error is that of both
    rel = (gate * gate + gate.abs() + 16) * 4 * U
    for got, want, scale in ((dP[:, :f], dh * up * act_slope64(gate, act), (dh * up).abs() * 2.2),
                             (dP[:, f:], dh * act64(gate, act), (dh * act64(gate, act)).abs())):
        within(got, want, want.abs() * step(fmt) + scale * rel + TINY[fmt], "dP")
    dX, dW = fl.gated_products(dP, X.cuda(), W.cuda())
    dp = dP.double().cpu()
    within(dX, dp @ w, 2 * f * 2 * U * (dp.abs() @ w.abs()) + 1e-30, "dX")
    within(dW, dp.t() @ x, t * 2 * U * (dp.abs().t() @ x.abs()) + 1e-30, "dW")
    assert torch.equal(fl.gated_products(dP, X.cuda(), W.cuda(), need_dw=False)[0], dX)
    assert torch.equal(fl.gated_products(dP, X.cuda(), W.cuda(), need_dx=False)[1], dW)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_gradient_against_differences(fl, act):
    """dP against central differences of the float64 block (step e: error e^2 / 6 of the third
    derivative, at most 1, plus rounding 2^-52 / e), on top of dP's own tolerance."""
    g = rng(77)
    t, f, e = 4, 64, 2.0 ** -14
    P = gauss(g, t, 2 * f, std=2.0)
    dH = gauss(g, t, f, to=torch.float16)
    dP = fl.gated_grad(dH.cuda(), P.cuda(), act=act)[0].double().cpu()
    p, dh = P.double(), dH.double()

    def loss(gate, up):
        return dh * act64(gate, act) * up

    diff = torch.cat((loss(p[:, :f] + e, p[:, f:]) - loss(p[:, :f] - e, p[:, f:]),
                      loss(p[:, :f], p[:, f:] + e) - loss(p[:, :f], p[:, f:] - e)), 1) / (2 * e)
    scale = torch.cat((dh * p[:, f:], dh * act64(p[:, :f], act)), 1).abs()
    within(dP, diff, scale * (2.0 ** -11 * 2.2 + e * e + 64 * 2.0 ** -38 + 400 * U) + TINY["fp16"], "dP")


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_far_values_of_the_gate(fl, act):
    """Gates from the far negative side to overflow: act and act' reach their limits, NaN stays."""
    gate = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 20.0, -20.0, 88.0, -88.0, 200.0, -200.0, 1e4, -1e4,
                         1e18, -1e18, 3e38, -3e38, float("nan")])
    f = gate.numel()
    P = torch.cat((gate, torch.ones(f)))[None].cuda()
    H = fl.gated_narrow(P, "bf16", act=act).double().cpu()[0]
    dP = fl.gated_grad(torch.ones(1, f, dtype=torch.bfloat16).cuda(), P, act=act)[0].double().cpu()[0]
    want, slope = act64(gate.double(), act), act_slope64(gate.double(), act)
    assert torch.isnan(H[-1]) and torch.isnan(dP[f - 1])
    slope = torch.where(gate.double().abs() > 1e3, (gate > 0).double(), slope)
    want = torch.where(gate.double().abs() > 1e3, gate.double().clamp_min(0), want)
    x = gate.double()[:-1]
    rel = (x * x + x.abs() + 16).clamp_max(1e5) * 4 * U
    within(H[:-1], want[:-1], want[:-1].abs() * (step("bf16") + rel) + 2e-36, "H")
    within(dP[f:-1], want[:-1], want[:-1].abs() * (step("bf16") + rel) + 2e-36, "dU")
    within(dP[:f - 1], slope[:-1], slope[:-1].abs() * step("bf16") + rel * 2.2 * (x.abs() < 100) + 2e-36, "dG")


def test_infinite_products_come_through(fl):
    """A faulty product is not hidden: non-finite entries of P reach H and dP."""
    P = torch.ones(2, 8)
    P[0, 1], P[1, 6] = float("inf"), float("nan")
    H = fl.gated_narrow(P.cuda(), "fp16").cpu()
    assert torch.isinf(H[0, 1]) and torch.isnan(H[1, 2])
    assert torch.isfinite(H).sum() == 6


@pytest.mark.parametrize("t,d,f", [(50, 136, 72), (3, 24, 40)])
def test_buffers_off_alignment(fl, t, d, f):
    """Operands and outputs that start at any element of a buffer; what is around them is kept."""
    g = rng(9)
    X, W = ints(g, t, d, to=torch.float16), ints(g, 2 * f, d, to=torch.float16)
    dP = ints(g, t, 2 * f, to=torch.float16)
    H0, P0 = fl.gated(X.cuda(), W.cuda())
    dH0 = H0.clamp(-8, 8)
    g0, gt0 = fl.gated_grad(dH0, P0, transpose=True)
    dX0, dW0 = fl.gated_products(dP.cuda(), X.cuda(), W.cuda())

    def shifted(x, n):
        buf = torch.full((x.numel() + n + 9,), 7, dtype=x.dtype, device="cuda")
        v = buf[n:n + x.numel()].view(x.shape)
        v.copy_(x)
        return buf, v

    for n in (1, 2, 3, 5):
        (_, x), (_, w), (_, dp) = shifted(X, n), shifted(W, n + 1), shifted(dP, n + 2)
        (bh, h), (bp, p) = shifted(torch.zeros_like(H0), n), shifted(torch.zeros_like(P0), n)
        fl.gated(x, w, H=h, P=p)
        assert torch.equal(h, H0) and torch.equal(p, P0)
        (bx, dx), (bw, dw) = shifted(torch.zeros_like(dX0), n), shifted(torch.zeros_like(dW0), n)
        fl.gated_products(dp, x, w, dX=dx, dW=dw)
        assert torch.equal(dx, dX0) and torch.equal(dw, dW0)
        (_, dh), (_, pp) = shifted(dH0, n), shifted(P0, n)
        (bg, gg), (bt, gt) = shifted(torch.zeros_like(g0), n), shifted(torch.zeros_like(gt0), n)
        fl.gated_grad(dh, pp, transpose=True, dP=gg, dPt=gt)
        assert torch.equal(gg, g0) and torch.equal(gt, gt0)
        (bn, hn) = shifted(torch.zeros_like(H0), n)
        assert torch.equal(fl.gated_narrow(pp, "fp16", H=hn), H0)
        for b in (bh, bp, bx, bw, bg, bt, bn):
            assert (b[:n] == 7).all() and (b[-9:] == 7).all()


def test_empty_batch(fl):
    W = torch.ones(8, 16, dtype=torch.float16).cuda()
    X = torch.empty(0, 16, dtype=torch.float16).cuda()
    H, P = fl.gated(X, W)
    assert H.shape == (0, 4) and P.shape == (0, 8)
    assert fl.gated_narrow(P, "fp16").shape == (0, 4)
    dP, dPt = fl.gated_grad(H, P, transpose=True)
    assert dP.shape == (0, 8) and dPt.shape == (8, 0)
    dW = torch.full((8, 16), 3.0, device="cuda")
    dX, dW = fl.gated_products(dP, X, W, dW=dW)
    assert dX.shape == (0, 16) and not dW.any()


# ---- adapters --------------------------------------------------------------------------------


def adapters64(C, X, A, B, index, scale):
    """Y in 64 bits and the sum of absolute terms (of the rank's sums of absolute products)."""
    Y, D = C.double().clone(), C.double().abs()
    for a in range(A.shape[0]):
        r = (index == a).nonzero().flatten()
        x, f, b, s = X[r].double(), A[a].double(), B[a].double(), float(scale[a])
        Y[r] += s * ((x @ f.t()) @ b.t())
        D[r] += abs(s) * ((x.abs() @ f.abs().t()) @ b.abs().t())
    return Y, D


ADAPTERS = [  # t, k, n, count, rank
    (1, 1, 1, 1, 1), (1, 64, 64, 1, 4), (1, 4096, 256, 3, 16), (2, 72, 33, 2, 5), (16, 128, 128, 4, 8),
    (17, 130, 70, 40, 12), (48, 512, 300, 24, 16), (33, 96, 520, 1, 64), (64, 257, 129, 5, 31),
    (200, 320, 264, 6, 32), (333, 640, 200, 3, 128), (130, 64, 1032, 7, 256), (700, 200, 96, 500, 16),
    (65, 2048, 64, 2, 9)]


@pytest.mark.parametrize("fmt", ["bf16", "fp16"])
@pytest.mark.parametrize("t,k,n,count,rank", ADAPTERS)
def test_adapters(fl, t, k, n, count, rank, fmt):
    g = rng(t + 3 * k + n + rank)
    h = HALF[fmt]
    X, C = gauss(g, t, k, to=h), gauss(g, t, n, std=3.0)
    A, B = gauss(g, count, rank, k, std=1 / math.sqrt(k), to=h), gauss(g, count, n, rank, std=0.3, to=h)
    scale = torch.rand(count, generator=g) * 4 - 2
    index = torch.randint(-1, count, (t,), generator=g).to(torch.int32)
    args = [x.cuda() for x in (C, X, A, B, index, scale)]
    want, D = adapters64(C, X, A, B, index, scale)
    # k products and rank terms, each 2u; the rank's sums enter the second product in two half
    # words, which drops at most 2^-16 of each (bf16) or 2^-21 (fp16)
    tol = D * ((k + rank + 8) * 2 * U + (2.0 ** -16 if fmt == "bf16" else 2.0 ** -21))
    y = fl.adapters(*args, out="f32")
    within(y, want, tol, "f32")
    none = index == -1
    assert torch.equal(y.cpu()[none], C[none])
    yh = fl.adapters(*args)
    assert yh.dtype == h
    assert torch.equal(yh, y.to(h))
    assert torch.equal(args[0].cpu(), C)
    # a row's result does not depend on the rows beside it
    p = torch.randperm(t, generator=g)
    again = fl.adapters(args[0][p].contiguous(), args[1][p].contiguous(), args[2], args[3],
                        args[4][p].contiguous(), args[5], out="f32")
    assert torch.equal(again, y[p])


@pytest.mark.parametrize("t", [5, 80])
def test_adapters_of_odd_rows(fl, t):
    """Rows without an adapter, with an index outside, with huge and non-finite entries."""
    g = rng(3)
    k, n, r, count = 128, 192, 16, 4
    X, C = gauss(g, t, k, to=torch.float16), gauss(g, t, n)
    A, B = gauss(g, count, r, k, to=torch.float16), gauss(g, count, n, r, to=torch.float16)
    scale = torch.ones(count)
    index = torch.full((t,), -1, dtype=torch.int32)
    Y = fl.adapters(*[x.cuda() for x in (C, X, A, B, index, scale)], out="f32")
    assert torch.equal(Y.cpu(), C)
    index[0], index[1], index[2], index[3] = count, 2, -7, 1
    X[1, 5] = float("inf")          # V infinite: the row is non-finite, as its definition says
    X[3] *= 500.0                   # V far above fp16's range
    X[3] = X[3].clamp(-60000, 60000)
    A[0, 0, 0] = float("nan")       # an adapter that no row uses
    Y = fl.adapters(*[x.cuda() for x in (C, X, A, B, index, scale)], out="f32").cpu()
    assert torch.isnan(Y[0]).all() and torch.isnan(Y[2]).all()
    assert not torch.isfinite(Y[1]).any()
    assert torch.equal(Y[4:], C[4:])
    want, D = adapters64(C[3:4], X[3:4], A[1:2], B[1:2], torch.zeros(1, dtype=torch.int32), scale[1:2])
    within(Y[3:4], want, D * ((k + r + 8) * 2 * U + 2.0 ** -21), "large V")


def test_adapters_of_small_and_large_scale(fl):
    """fp16 factors whose rank sums lie far below and above fp16's range."""
    g = rng(4)
    t, k, n, r = 24, 64, 64, 8
    C = torch.zeros(t, n)
    for x, a in ((1e-3, 1e-4), (3e-5, 1e-6), (200.0, 300.0)):
        X, A = gauss(g, t, k, std=x, to=torch.float16), gauss(g, 1, r, k, std=a, to=torch.float16)
        B = gauss(g, 1, n, r, to=torch.float16)
        index, scale = torch.zeros(t, dtype=torch.int32), torch.ones(1)
        want, D = adapters64(C, X, A, B, index, scale)
        Y = fl.adapters(*[v.cuda() for v in (C, X, A, B, index, scale)], out="f32")
        within(Y, want, D * ((k + r + 8) * 2 * U + 2.0 ** -21), (x, a))


def test_adapters_empty_batch_and_shifted_buffers(fl):
    g = rng(6)
    t, k, n, r, count = 19, 40, 56, 8, 3
    mats = [gauss(g, t, n), gauss(g, t, k, to=torch.bfloat16), gauss(g, count, r, k, to=torch.bfloat16),
            gauss(g, count, n, r, to=torch.bfloat16),
            torch.randint(0, count, (t,), generator=g).to(torch.int32), torch.ones(count)]
    want = fl.adapters(*[m.cuda() for m in mats])
    for s in (1, 2, 3):
        moved = []
        for m in mats:
            buf = torch.zeros(m.numel() + s, dtype=m.dtype, device="cuda")
            buf[s:].copy_(m.flatten())
            moved.append(buf[s:].view(m.shape))
        buf = torch.full((t * n + s + 5,), 7, dtype=torch.bfloat16, device="cuda")
        Y = fl.adapters(*moved, Y=buf[s:s + t * n].view(t, n))
        assert torch.equal(Y, want)
        assert (buf[:s] == 7).all() and (buf[-5:] == 7).all()
    e = [m.cuda() for m in mats]
    e[0], e[1], e[4] = e[0][:0], e[1][:0], e[4][:0]
    assert fl.adapters(*e).shape == (0, n)


# ---- heads -----------------------------------------------------------------------------------


def heads64(C, hq, hkv, hd, pos, freq, gq, gk, eps, pairs):
    t = C.shape[0]
    x = C.view(t, hq + 2 * hkv, hd)
    out = []
    for y, g in ((x[:, :hq], gq), (x[:, hq:hq + hkv], gk)):
        if g is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + eps) * g
        if freq is not None:
            n = freq.numel()
            ang = (pos.double()[:, None] * freq.double())[:, None, :]
            c, s = ang.cos(), ang.sin()
            if pairs == "half":
                a, b = y[..., :n], y[..., n:2 * n]
                z = torch.cat((a * c - b * s, b * c + a * s), -1)
            else:
                a, b = y[..., 0:2 * n:2], y[..., 1:2 * n:2]
                z = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
            y = torch.cat((z, y[..., 2 * n:]), -1)
        out.append(y)
    return out[0], out[1], x[:, hq + hkv:]


HEADS = [  # t, hq, hkv, hd, rd
    (1, 1, 1, 1, 0), (1, 2, 1, 2, 2), (1, 32, 8, 128, 128), (7, 4, 4, 64, 64), (5, 3, 1, 80, 80),
    (6, 2, 2, 96, 48), (33, 8, 2, 128, 64), (4, 5, 5, 256, 256), (3, 2, 1, 512, 512), (9, 3, 3, 33, 20),
    (200, 4, 1, 64, 32), (2, 6, 2, 40, 10), (70, 1, 1, 128, 6), (12, 16, 16, 72, 72), (3, 1, 2, 500, 100)]


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("fmt,pairs", [("bf16", "half"), ("fp16", "interleaved"), ("fp16", "half"),
                                       ("bf16", "interleaved")])
@pytest.mark.parametrize("t,hq,hkv,hd,rd", HEADS)
def test_heads_and_their_gradient(fl, t, hq, hkv, hd, rd, fmt, pairs, norm):
    g = rng(t + hd + rd + hq)
    eps = 1e-5
    C = gauss(g, t, (hq + 2 * hkv) * hd, std=1.5)
    gq = gauss(g, hd, std=0.5) + 1 if norm else None
    gk = gauss(g, hd, std=0.5) - 1 if norm else None
    pos = torch.randint(0, 1 << 20, (t,), generator=g)
    freq = torch.pow(10000.0, -torch.arange(rd // 2, dtype=torch.float64) * 2 / max(rd, 1)).float()
    dev = [None if x is None else x.cuda() for x in (gq, gk)]
    kw = dict(gq=dev[0], gk=dev[1], eps=eps, pairs=pairs)
    frq = freq.cuda() if rd else None
    q, k, v = fl.heads(C.cuda(), hq, hkv, pos.cuda(), frq, fmt, **kw)

    c64 = C.double().requires_grad_(True)
    g64 = [None if x is None else x.double().requires_grad_(True) for x in (gq, gk)]
    want = heads64(c64, hq, hkv, hd, pos, freq if rd else None, g64[0], g64[1], eps, pairs)
    # the norm: a sum of hd squares and a root, (hd + 8) u; the rotation: sums of two products with
    # sines off by 4u, so 16u of the pair's size, at most the head's largest entry twice
    for got, w, name in zip((q, k, v), want, "qkv"):
        w = w.detach()
        size = w.abs().amax(-1, keepdim=True) * 1.5
        within(got, w, w.abs() * step(fmt) + size * (hd + 40) * U + TINY[fmt], name)

    d = [gauss(g, t, n, hd, std=0.5, to=HALF[fmt]) for n in (hq, hkv, hkv)]
    leaves = [c64] + [x for x in g64 if x is not None]
    grads = torch.autograd.grad(want, leaves, [x.double() for x in d])
    dC, dgq, dgk = fl.heads_grad(*[x.cuda() for x in d], C.cuda() if norm else None, pos.cuda(), frq, **kw)
    w = grads[0].view(t, -1, hd)
    # dx = r (g u - x c): both terms at most the head's largest r g u times 1 + |x r| with
    # |x r| <= sqrt(hd), and c is a sum of hd terms
    if norm:
        x = c64.detach().view(t, -1, hd)
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
        u = torch.cat([y.double() for y in d], 1).abs().amax(-1, keepdim=True) * 1.5
        gm = torch.maximum(g64[0].detach().abs().max(), g64[1].detach().abs().max())
        size = r * gm * u * (1 + (x * r).abs() * (x * r).abs().mean(-1, keepdim=True))
    else:
        size = w.abs().amax(-1, keepdim=True) * 1.5
    within(dC.view(t, -1, hd), w, w.abs() * step(fmt) + size * (2 * hd + 80) * U + TINY[fmt], "dC")
    if norm:
        x = c64.detach().view(t, -1, hd)
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
        for got, w, part, dy in ((dgq, grads[1], (x * r)[:, :hq], d[0]), (dgk, grads[2], (x * r)[:, hq:hq + hkv], d[1])):
            s = (part.abs() * dy.double().abs().amax(-1, keepdim=True) * 1.5).sum((0, 1))
            within(got, w, s * (t * part.shape[1] + hd + 40) * U + 1e-30, "gain")
    else:
        assert dgq is None and dgk is None


def test_heads_of_zeros_and_far_positions(fl):
    """A head of zeros is zero (eps carries it) with a finite gradient; positions up to 2^31."""
    hd, t = 128, 4
    C = torch.zeros(t, 4 * hd)
    C[1:] = gauss(rng(1), t - 1, 4 * hd)
    gain = torch.ones(hd)
    pos = torch.tensor([0, 1, 1 << 24, (1 << 31) - 1])
    freq = torch.pow(10000.0, -torch.arange(64, dtype=torch.float64) / 64).float()
    q, k, v = fl.heads(C.cuda(), 2, 1, pos.cuda(), freq.cuda(), "fp16", gq=gain.cuda(), gk=gain.cuda())
    assert not q[0].any() and not k[0].any()
    want = heads64(C.double(), 2, 1, hd, pos, freq, gain.double(), gain.double(), 1e-6, "half")
    # an angle of 2^31 turns to within 2^31 2^-53 in FP64, both here and in the definition
    for got, w in zip((q, k), want):
        size = w.abs().amax(-1, keepdim=True) * 1.5
        within(got, w, w.abs() * step("fp16") + size * ((hd + 40) * U + 2.0 ** -20) + TINY["fp16"], "far")
    dy = [torch.ones(t, n, hd, dtype=torch.float16).cuda() for n in (2, 1, 1)]
    dC, dgq, _ = fl.heads_grad(*dy, C.cuda(), pos.cuda(), freq.cuda(), gq=gain.cuda(), gk=gain.cuda())
    assert torch.isfinite(dC[0, 3 * hd:]).all() and torch.isfinite(dgq).all()


def test_heads_empty_batch_and_shifted_buffers(fl):
    g = rng(12)
    t, hq, hkv, hd = 6, 4, 2, 64
    C = gauss(g, t, 8 * hd)
    gq, gk = gauss(g, hd) + 1, gauss(g, hd) + 1
    pos, freq = torch.arange(t) + 100, torch.pow(100.0, -torch.arange(hd // 2) / hd)
    d = [gauss(g, t, n, hd, to=torch.bfloat16) for n in (hq, hkv, hkv)]
    kw = dict(gq=gq.cuda(), gk=gk.cuda())
    want = fl.heads(C.cuda(), hq, hkv, pos.cuda(), freq.cuda(), "bf16", **kw)
    gwant = fl.heads_grad(*[x.cuda() for x in d], C.cuda(), pos.cuda(), freq.cuda(), **kw)

    def shifted(x, s, pad=0):
        buf = torch.full((x.numel() + s + pad,), 7, dtype=x.dtype, device="cuda")
        buf[s:s + x.numel()].copy_(x.flatten())
        return buf[s:s + x.numel()].view(x.shape)

    for s in (1, 2, 3):
        outs = [shifted(torch.zeros_like(x), s, 4) for x in want]
        kws = dict(gq=shifted(gq, s), gk=shifted(gk, s))
        got = fl.heads(shifted(C, s), hq, hkv, shifted(pos, s), shifted(freq, s), "bf16", q=outs[0],
                       k=outs[1], v=outs[2], **kws)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        got = fl.heads_grad(*[shifted(x, s) for x in d], shifted(C, s), shifted(pos, s),
                            shifted(freq, s), dC=shifted(torch.zeros_like(gwant[0]), s, 4), **kws)
        assert all(torch.equal(a, b) for a, b in zip(got, gwant))
    e = [x[:0].cuda() for x in d]
    q, k, v = fl.heads(C[:0].cuda(), hq, hkv, pos[:0].cuda(), freq.cuda(), "bf16", **kw)
    assert q.shape == (0, hq, hd)
    dC, dgq, dgk = fl.heads_grad(*e, C[:0].cuda(), pos[:0].cuda(), freq.cuda(), **kw)
    assert dC.shape == (0, 8 * hd) and not dgq.any() and not dgk.any()
