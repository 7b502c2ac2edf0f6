"""The operators around a delivered product as a program runs them: together with the verifier, inside
HIP graphs, on several streams, and at sizes that take the large tiles and offsets past 32 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def fl():
    assert torch.cuda.is_available()
    from paper_2609_19758_amd import fpsketch, layers
    fpsketch.load()
    return layers


@pytest.fixture(scope="module")
def fk(fl):
    from paper_2609_19758_amd import fpsketch
    return fpsketch


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def gauss(g, *shape, std=1.0, to=torch.float32):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(to)


def ints(g, *shape, to):
    return torch.randint(-2, 3, shape, generator=g, device="cuda").to(to)


# ---- large products ------------------------------------------------------------------------


@pytest.mark.parametrize("fmt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("t,d,f", [(4001, 4104, 2056), (4100, 4100, 2055), (2000, 4000, 2104),
                                   (4099, 4104, 40), (520, 8200, 64)])
def test_large_products_are_exact(fl, t, d, f, fmt):
    """Small integers through the large tiles, padded copies and products in parts: sums stay below
    2^24, so every FP32 product is exact."""
    g = gen(t + d + f)
    X, W, dP = ints(g, t, d, to=fmt), ints(g, 2 * f, d, to=fmt), ints(g, t, 2 * f, to=fmt)
    H, P = fl.gated(X, W)
    assert torch.equal(P, (X.double() @ W.double().t()).float())
    assert torch.equal(fl.gated_narrow(P, "fp16" if fmt is torch.float16 else "bf16"), H)
    dX, dW = fl.gated_products(dP, X, W)
    assert torch.equal(dX, (dP.double() @ W.double()).float())
    assert torch.equal(dW, (dP.double().t() @ X.double()).float())


@pytest.mark.parametrize("fmt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("t,d,f", [(333, 1000, 2731), (2000, 256, 512), (500, 2048, 2048), (40, 4000, 1000),
                                   (1500, 1023, 2049), (1, 64, 4096), (7, 4104, 8), (2600, 16, 64)])
def test_one_backward_product_has_the_bits_it_has_beside_the_other(fl, t, d, f, fmt):
    """Both in one launch, and both in parts, where they are small; exact, as their sums stay below 2^24."""
    g = gen(3 * t + d + f)
    X, W, dP = ints(g, t, d, to=fmt), ints(g, 2 * f, d, to=fmt), ints(g, t, 2 * f, to=fmt)
    dX, dW = fl.gated_products(dP, X, W)
    assert torch.equal(dX, (dP.double() @ W.double()).float())
    assert torch.equal(dW, (dP.double().t() @ X.double()).float())
    X, W, dP = gauss(g, t, d, to=fmt), gauss(g, 2 * f, d, to=fmt), gauss(g, t, 2 * f, to=fmt)
    dX, dW = fl.gated_products(dP, X, W)
    assert torch.equal(fl.gated_products(dP, X, W, need_dw=False)[0], dX)
    assert torch.equal(fl.gated_products(dP, X, W, need_dx=False)[1], dW)
    outs = torch.zeros_like(dX), torch.zeros_like(dW)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fl.gated_products(dP, X, W, dX=outs[0], dW=outs[1])
    for _ in range(3):
        for o in outs:
            o.zero_()
        graph.replay()
        again = fl.gated_products(dP, X, W)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], dX) and torch.equal(outs[1], dW)
        assert torch.equal(again[0], dX) and torch.equal(again[1], dW)


@pytest.mark.parametrize("fmt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rank", [248, 255, 256])
def test_long_batches_of_the_widest_adapters(fl, rank, fmt):
    """Tiles of 32 rows at the largest rank, whose sums need more than 64 KiB of LDS; eager and captured."""
    g = gen(rank)
    t, k, n, count = 1060, 192, 200, 3
    X, C = gauss(g, t, k, to=fmt), gauss(g, t, n)
    A, B = gauss(g, count, rank, k, std=1 / math.sqrt(k), to=fmt), gauss(g, count, n, rank, std=0.3, to=fmt)
    index = (torch.arange(t, device="cuda") // 100 % (count + 1) - 1).int()
    scale = torch.tensor([1.5, -0.5, 2.0], device="cuda")
    Y = fl.adapters(C, X, A, B, index, scale, out="f32")
    want, D = C.double(), C.double().abs()
    for a in range(count):
        r = (index == a).nonzero().flatten()
        x, p, q, s = X[r].double(), A[a].double().t().contiguous(), B[a].double().t().contiguous(), float(scale[a])
        want[r] += s * ((x @ p) @ q)
        D[r] += abs(s) * ((x.abs() @ p.abs()) @ q.abs())
    # k products and rank terms, each 2u; the rank's sums enter in two half words (2^-21, bf16 2^-16)
    tol = D * ((k + rank + 8) * 2 * U + (2.0 ** -16 if fmt is torch.bfloat16 else 2.0 ** -21))
    assert bool(((Y.double() - want).abs() <= tol).all())
    out = torch.zeros_like(Y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fl.adapters(C, X, A, B, index, scale, out="f32", Y=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, Y)


@pytest.mark.parametrize("fmt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("t,f,shift", [(1531, 8200, 0), (451, 16400, 1), (1600, 8192, 0), (1600, 8192, 5), (256, 129, 3),
                                       (1023, 64, 0), (2177, 12345, 33), (257, 50000, 0)])
def test_long_gradients_and_their_transposes(fl, t, f, shift, fmt):
    """Rows of the gradient and of its transpose that begin on lines and inside them: the gradient is the one
    without a transpose, and nothing beside either buffer is written."""
    g = gen(t + f)
    dH, P = gauss(g, t, f, std=0.5, to=fmt), gauss(g, t, 2 * f)
    want, _ = fl.gated_grad(dH, P, act="gelu")
    n = 2 * t * f
    bufs = [torch.full((shift + n + 70,), 7.0, dtype=fmt, device="cuda") for _ in range(2)]
    dP, dPt = bufs[0][shift:shift + n].view(t, 2 * f), bufs[1][shift:shift + n].view(2 * f, t)
    fl.gated_grad(dH, P, act="gelu", transpose=True, dP=dP, dPt=dPt)
    assert torch.equal(dP, want)
    assert torch.equal(dPt, want.t())
    for b in bufs:
        assert bool((b[:shift] == 7).all()) and bool((b[shift + n:] == 7).all())


# ---- with the verifier ---------------------------------------------------------------------


def _repair(v, A, B, C, seed):
    """Localizes, checks and applies the faults of a dirty product; the repaired product is clean."""
    recs, n, _ = v.localize(A, B, C, seed=seed)
    assert n == len(recs) > 0
    assert not v.apply(A, B, C, recs, seed=seed + 1)
    return {(i, j) for i, j, *_ in recs}


def _dirty(v, A, B, C):
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    v.probe(A, B, C, d_dirty=flag)
    return bool(flag.item())


def test_a_guarded_feed_forward_step(fl, fk):
    """Forward and backward of a gated block with every product verified; a fault in P is found,
    repaired, and H formed again equals the H of the clean run, as do the gradients."""
    g = gen(1)
    t, d, f = 512, 1024, 768
    h = torch.bfloat16
    X, W = gauss(g, t, d, to=h), gauss(g, 2 * f, d, std=0.02, to=h)
    H, P = fl.gated(X, W)
    clean = P.clone()
    v = fk.Verifier(t, d, 2 * f, "bf16", b_layout=1)
    assert not _dirty(v, X, W, P)
    unit = float(P.abs().mean())
    faults = {(3, 17): 2.0 * unit, (400, 1200): -1.5 * unit, (77, 900): float("inf")}
    for (i, j), x in faults.items():
        P[i, j] += x
    assert _dirty(v, X, W, P)
    assert _repair(v, X, W, P, 5) == set(faults)
    # a repaired entry is the exact product rounded once, the kernel's own a sum of d steps
    assert float((P - clean).abs().max()) <= d * 2 * U * float((X.float().abs() @ W.float().abs().t()).max())
    H2 = fl.gated_narrow(P, "bf16")
    assert float((H2.float() - H.float()).abs().max()) <= 2.0 ** -7 * float(H.float().abs().max())
    same = torch.ones_like(H, dtype=torch.bool)
    for i, j in faults:
        same[i, j % f] = False
    assert torch.equal(H2[same], H[same])

    dH = gauss(g, t, f, std=0.05, to=h)
    dP, dPt = fl.gated_grad(dH, P, transpose=True)
    dX, dW = fl.gated_products(dP, X, W)
    vx = fk.Verifier(t, 2 * f, d, "bf16")
    vw = fk.Verifier(2 * f, t, d, "bf16")
    assert not _dirty(vx, dP, W, dX) and not _dirty(vw, dPt, X, dW)
    for vv, A, B, C in ((vx, dP, W, dX), (vw, dPt, X, dW)):
        keep = C.clone()
        C[11, 29] += 3 * float(C.abs().mean())
        assert _dirty(vv, A, B, C)
        assert _repair(vv, A, B, C, 9) == {(11, 29)}
        assert float((C - keep).abs().max()) <= 1e-4 * float(keep.abs().max())
    for vv in (v, vx, vw):
        vv.close()


def test_a_guarded_attention_input(fl, fk):
    """QKV product: verified, repaired, then adapters or heads from it; both leave C as it is."""
    g = gen(2)
    t, d, hq, hkv, hd = 300, 512, 6, 3, 64
    n = (hq + 2 * hkv) * hd
    h = torch.float16
    X, W = gauss(g, t, d, to=h), gauss(g, n, d, std=0.05, to=h)
    C = torch.mm(X, W.t(), out_dtype=torch.float32)
    v = fk.Verifier(t, d, n, "fp16", b_layout=1)
    clean = C.clone()
    C[5, 8] += 4 * float(C.abs().mean())
    assert _dirty(v, X, W, C)
    assert _repair(v, X, W, C, 3) == {(5, 8)}
    assert torch.equal(C.flatten()[9 + 5 * n:], clean.flatten()[9 + 5 * n:])
    C.copy_(clean)
    A, B = gauss(g, 3, 8, d, std=0.05, to=h), gauss(g, 3, n, 8, std=0.05, to=h)
    index = torch.arange(t, device="cuda", dtype=torch.int32) // 90 - 1
    Y = fl.adapters(C, X, A, B, index, torch.full((3,), 2.0, device="cuda"), out="f32")
    assert torch.equal(C, clean)
    pos = torch.arange(t, device="cuda")
    freq = torch.pow(10000.0, -torch.arange(hd // 2, device="cuda") * 2 / hd)
    q, k, vv = fl.heads(Y, hq, hkv, pos, freq, "fp16")
    x = Y.view(t, -1, hd)
    assert torch.equal(vv, x[:, hq + hkv:].half())
    # without a norm a rotation keeps the length of every pair: two roundings of half a step each
    m = q.float()[..., :hd // 2] ** 2 + q.float()[..., hd // 2:] ** 2
    w = x[:, :hq, :hd // 2] ** 2 + x[:, :hq, hd // 2:] ** 2
    assert ((m - w).abs() <= 4 * 2.0 ** -11 * w + 1e-6).all()
    v.close()


# ---- graphs, streams -----------------------------------------------------------------------


def _everything(fl, s, seed):
    """A pass through every operator at small sizes; the state is made once and passed in."""
    if s is None:
        g = gen(seed)
        h = torch.bfloat16
        t, d, f, n = 70, 200, 88, 96
        s = dict(X=gauss(g, t, d, to=h), W=gauss(g, 2 * f, d, std=0.1, to=h), dH=gauss(g, t, f, to=h),
                 Xs=gauss(g, 5, d, to=h), W3=gauss(g, 2 * f, 201, std=0.1, to=h), X3=gauss(g, t, 201, to=h),
                 C=gauss(g, t, n), Xa=gauss(g, t, 104, to=h), A=gauss(g, 4, 8, 104, std=0.1, to=h),
                 B=gauss(g, 4, n, 8, to=h), index=torch.randint(-1, 4, (t,), generator=g, device="cuda").int(),
                 scale=gauss(g, 4), Q=gauss(g, t, 8 * 32), gain=gauss(g, 32) + 1,
                 pos=torch.arange(t, device="cuda") * 7, freq=gauss(g, 16).abs(),
                 dq=gauss(g, t, 4, 32, to=h), dk=gauss(g, t, 2, 32, to=h))
        torch.cuda.synchronize()
        return s
    H, P = fl.gated(s["X"], s["W"])
    Hs, Ps = fl.gated(s["Xs"], s["W"], act="gelu")
    H3, P3 = fl.gated(s["X3"], s["W3"], act="gelu_tanh")
    N = fl.gated_narrow(P, "bf16")
    dP, dPt = fl.gated_grad(s["dH"], P, transpose=True)
    dX, dW = fl.gated_products(dP, s["X"], s["W"])
    dX3, dW3 = fl.gated_products(dP, s["X3"], s["W3"])
    Y = fl.adapters(s["C"], s["Xa"], s["A"], s["B"], s["index"], s["scale"])
    q, k, v = fl.heads(s["Q"], 4, 2, s["pos"], s["freq"], "bf16", gq=s["gain"], gk=s["gain"])
    dC, dgq, dgk = fl.heads_grad(s["dq"], s["dk"], s["dk"], s["Q"], s["pos"], s["freq"], gq=s["gain"],
                                 gk=s["gain"])
    return [H, P, Hs, Ps, H3, P3, N, dP, dPt, dX, dW, dX3, dW3, Y, q, k, v, dC, dgq, dgk]


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_graph_replays_equal_eager_runs(fl):
    """Captured once, replayed on new inputs with eager work and synchronizations between; two graphs
    replayed one after the other keep their own workspaces."""
    s1, s2 = _everything(fl, None, 1), _everything(fl, None, 2)
    want = {1: _everything(fl, s1, 0), 2: _everything(fl, s2, 0)}
    graphs, outs, ins = [], [], []
    for seed in (1, 2):
        s = _everything(fl, None, seed)
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            _everything(fl, s, 0)                     # (first calls outside the capture)
        side.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            out = _everything(fl, s, 0)
        graphs.append(gr)
        outs.append(out)
        ins.append(s)
    for turn in range(4):
        for i, gr in enumerate(graphs):
            seed = 1 + (i + turn) % 2                  # each graph sees both inputs in turn
            src = s1 if seed == 1 else s2
            for k in ins[i]:
                ins[i][k].copy_(src[k])
            gr.replay()
            assert _same(_everything(fl, src, 0), want[seed])      # the program's own eager work
            torch.cuda.synchronize()
            assert _same(outs[i], want[seed]), (turn, i)


def test_streams(fl):
    """Calls on a stream of their own, given or current, with nothing else ordered between; two streams
    at once do not share workspaces."""
    states = [_everything(fl, None, 11), _everything(fl, None, 12)]
    want = [_everything(fl, s, 0) for s in states]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for s, st in zip(states, streams):
            with torch.cuda.stream(st):
                got.append(_everything(fl, s, 0))
        torch.cuda.synchronize()
        assert all(_same(a, b) for a, b in zip(got, want))
    s = states[0]
    for st in (streams[0], streams[0].cuda_stream):
        H, P = fl.gated(s["X"], s["W"], stream=st)
        Y = fl.adapters(s["C"], s["Xa"], s["A"], s["B"], s["index"], s["scale"], stream=st)
        dP, _ = fl.gated_grad(s["dH"], P, stream=st)
        dX, dW = fl.gated_products(dP, s["X"], s["W"], stream=st)
        torch.cuda.synchronize()
        assert _same([H, P, Y, dP, dX, dW], [want[0][i] for i in (0, 1, 13, 7, 9, 10)])
        assert torch.cuda.current_stream() == torch.cuda.default_stream()


def test_refusals_of_later_operands(fl, fk):
    """What the first operand's device check hides on the CPU: later operands' shapes, types, devices."""
    X, W = torch.zeros(3, 8).half().cuda(), torch.zeros(10, 8).half().cuda()
    for bad, match in ((W.bfloat16(), "W: dtype"), (W[:, :7].contiguous(), "W: shape"), (W.cpu(), "W: on cpu"),
                       (torch.zeros(8, 10).half().cuda().t(), "W: not contiguous")):
        with pytest.raises(ValueError, match=match):
            fl.gated(X, bad)
    with pytest.raises(ValueError, match="P: given with deliver=False"):
        fl.gated(X, W, deliver=False, P=torch.zeros(3, 10, device="cuda"))
    with pytest.raises(ValueError, match="H: shape"):
        fl.gated(X, W, H=torch.zeros(3, 6).half().cuda())
    with pytest.raises(ValueError, match="need_dx, need_dw"):
        fl.gated_products(torch.zeros(3, 10).half().cuda(), X, W, need_dx=False, need_dw=False)
    with pytest.raises(ValueError, match="dX, dW"):
        fl.gated_products(torch.zeros(3, 10).half().cuda(), X, W, need_dx=False,
                          dX=torch.zeros(3, 8, device="cuda"))
    C, index, scale = torch.zeros(3, 6, device="cuda"), torch.zeros(3, device="cuda").int(), torch.ones(2, device="cuda")
    A, B = torch.zeros(2, 4, 8).half().cuda(), torch.zeros(2, 6, 4).half().cuda()
    for i, bad, match in ((4, index.long(), "index: dtype"), (4, index[:2], "index: shape"),
                          (5, scale.double(), "scale: dtype"), (3, B[:, :5].contiguous(), "B: shape"),
                          (2, A.bfloat16(), "A: dtype")):
        args = [C, X, A, B, index, scale]
        args[i] = bad
        with pytest.raises(ValueError, match=match):
            fl.adapters(*args)
    with pytest.raises(fk.FpsketchError, match="overlaps"):
        fl.adapters(C, X, A, B, index, scale, out="f32", Y=C)
    Q, pos, freq = torch.zeros(3, 32, device="cuda"), torch.zeros(3, device="cuda").long(), torch.ones(4, device="cuda")
    with pytest.raises(ValueError, match="pos: dtype"):
        fl.heads(Q, 2, 1, pos.int(), freq, "fp16")
    with pytest.raises(ValueError, match="pos: None"):
        fl.heads(Q, 2, 1, None, freq, "fp16")
    with pytest.raises(fk.FpsketchError, match="eps"):
        fl.heads(Q, 2, 1, pos, freq, "fp16", gq=torch.ones(8, device="cuda"), gk=torch.ones(8, device="cuda"),
                 eps=-1.0)


# ---- offsets past 32 bits ------------------------------------------------------------------


def test_offsets_past_32_bits(fl):
    """Arrays of more than 2^31 elements: the last rows equal those of a call on these rows alone (for
    the products: within the sums' rounding, since the tiles differ)."""
    g = gen(4)
    h = torch.bfloat16
    # 131100 tokens x 2 x 8200: P has 2.15e9 entries
    t, d, f, tail = 131100, 64, 8200, 40
    X, W = gauss(g, t, d, to=h), gauss(g, 2 * f, d, std=0.1, to=h)
    H, P = fl.gated(X, W)
    H1, P1 = fl.gated(X[-tail:], W)
    bound = d * 2 * U * float((X[-tail:].float().abs() @ W.float().abs().t()).max())
    assert float((P[-tail:] - P1).abs().max()) <= 2 * bound
    assert float((P[:tail] - fl.gated(X[:tail], W)[1]).abs().max()) <= 2 * bound
    P1 = P[-tail:].contiguous()
    assert torch.equal(fl.gated_narrow(P1, "bf16"), H[-tail:])
    assert torch.equal(fl.gated_narrow(P, "bf16"), H)
    dP, _ = fl.gated_grad(H, P)
    assert torch.equal(dP[-tail:], fl.gated_grad(H[-tail:].contiguous(), P1)[0])
    del H
    # heads and adapters on the same array as their product: 16400 columns
    A, B = gauss(g, 2, 8, d, to=h), gauss(g, 2, 2 * f, 8, to=h)
    index = (torch.arange(t, device="cuda") % 3 - 1).int()
    scale = torch.ones(2, device="cuda")
    Y = fl.adapters(P, X, A, B, index, scale)
    assert torch.equal(Y[-tail:], fl.adapters(P1, X[-tail:], A, B, index[-tail:].contiguous(), scale))
    del Y
    hd, hq, hkv = 200, 80, 1
    pos, freq = torch.arange(t, device="cuda"), torch.pow(100.0, -torch.arange(100, device="cuda") / 100)
    gain = torch.ones(hd, device="cuda")
    kw = dict(gq=gain, gk=gain)
    q, k, v = fl.heads(P, hq, hkv, pos, freq, "bf16", **kw)
    small = fl.heads(P1, hq, hkv, pos[-tail:].contiguous(), freq, "bf16", **kw)
    assert all(torch.equal(a[-tail:], b) for a, b in zip((q, k, v), small))
    dC, _, _ = fl.heads_grad(q, k, v, P, pos, freq, **kw)
    small = fl.heads_grad(*[x[-tail:].contiguous() for x in (q, k, v)], P1, pos[-tail:].contiguous(), freq, **kw)
    assert torch.equal(dC[-tail:], small[0])
