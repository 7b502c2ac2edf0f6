"""The performance cases of the operators around a delivered product.

A linear layer's product C = A W^T leaves its GEMM in FP32 so that it can be verified, and is then
taken on to the half format that the next layer reads.  The operators of
``paper_2609_19758_amd.layers`` do that together with the layer's own arithmetic:

  gated           gated feed-forward: the stacked projections P = X W^T (gate rows of W, then up
                  rows), delivered in FP32 where ``deliver``, and H = act(P_gate) P_up.
  gated_narrow    H once more from a delivered (and repaired) P.
  gated_grad      the gradient dP of P from that of H; where ``deliver`` its transpose too, which is
                  the first operand of dW when that product is verified.
  gated_products  the products of the backward pass, dX = dP W and dW = dP^T X, delivered in FP32.
  adapters        low-rank adapters of many requests added to a shared projection's product C:
                  Y_i = C_i + scale_a (X_i A_a^T) B_a^T with a = index_i, none where it is -1.
  heads           norm of each query and key head of a QKV product with the position rotation;
                  value heads are narrowed.
  heads_grad      its backward pass: the product's gradient and those of the gains.

``own`` false: elementary torch operations in 32 bits (angles in 64), rounded once at the end.
``own`` true: the framework's calls.  ``exact`` states each operator once more in 64 bits.
"""
import math

import torch

own = False


# ---------------------------------------------------------------------------------------------
# Cases.


def _gated(kind, t, d, f, fmt, act="silu", deliver=True, **kw):
    return {"kind": kind, "t": t, "d": d, "f": f, "fmt": fmt, "act": act, "deliver": deliver, **kw}


def _adapters(t, k, n, count, rank, requests, fmt, out="half", **kw):
    return {"kind": "adapters", "t": t, "k": k, "n": n, "count": count, "rank": rank,
            "requests": requests, "fmt": fmt, "out": out, **kw}


def _heads(kind, t, hq, hkv, hd, rd, fmt, pairs="half", norm=True, far=4096, **kw):
    return {"kind": kind, "t": t, "hq": hq, "hkv": hkv, "hd": hd, "rd": rd, "fmt": fmt,
            "pairs": pairs, "norm": norm, "far": far, **kw}


def listed():
    return [
        # decode: one token through a 4096 x 11008 block, the products kept for the verifier
        _gated("gated", 1, 4096, 11008, "bf16", name="gated_1x4096x11008_bf16"),
        # a decode batch with a few prompt tokens in it, on the wider block
        _gated("gated", 67, 5120, 13824, "fp16", name="gated_67x5120x13824_fp16"),
        # a training step or a long prompt: the largest work
        _gated("gated", 4096, 4096, 11008, "bf16", name="gated_4096x4096x11008_bf16"),
        # after a repair: the activation of a product that was localized and corrected
        _gated("gated_narrow", 2048, 4096, 11008, "bf16", name="gated_narrow_2048x11008_bf16"),
        # backward of a ragged micro-batch: elementwise part ...
        _gated("gated_grad", 1531, 5120, 13824, "fp16", act="gelu_tanh",
               name="gated_grad_1531x13824_fp16"),
        # ... and the two products of a training step
        _gated("gated_products", 2048, 4096, 11008, "bf16",
               name="gated_products_2048x4096x11008_bf16"),
        # backward of a short odd batch on a small odd block
        _gated("gated_products", 333, 1000, 2731, "fp16",
               name="gated_products_333x1000x2731_fp16"),
        # decode: a token each of 48 requests with 24 adapters, on an output projection
        _adapters(48, 4096, 4096, 24, 16, 48, "bf16", name="adapters_48x4096x4096_r16_bf16"),
        # prompts of 12 requests of different lengths on a down projection
        _adapters(4093, 11008, 4096, 8, 64, 12, "fp16", name="adapters_4093x11008x4096_r64_fp16"),
        # decode with grouped key and value heads, far into their sequences
        _heads("heads", 48, 32, 8, 128, 128, "bf16", far=131072, name="heads_48_32q8kv128_bf16"),
        # a prompt through an ungrouped layer
        _heads("heads", 8191, 40, 40, 128, 128, "fp16", far=16384,
               name="heads_8191_40q40kv128_fp16"),
        # the backward pass of a training step, part of each head rotated
        _heads("heads_grad", 4096, 32, 8, 128, 64, "bf16", pairs="interleaved", far=8192,
               name="heads_grad_4096_32q8kv128_bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A layer's width: a multiple of 64 three times out of four, else any integer."""
    v = _log(rng, lo, hi)
    return max(64, v // 64 * 64) if rng.random() < 0.75 and v >= 64 else v


_MOST = 4096 * 4096 * 11008     # t d f of the largest listed block


def draw(rng):
    kind = rng.choice(["gated", "gated", "gated", "gated_narrow", "gated_grad", "gated_products",
                       "gated_products", "adapters", "adapters", "heads", "heads_grad"])
    fmt = rng.choice(["bf16", "fp16"])
    if kind.startswith("gated"):
        d, f = _width(rng, 64, 8192), _width(rng, 64, 16384)
        cap = _MOST // (d * f) // (2 if kind == "gated_products" else 1)
        if kind in ("gated_narrow", "gated_grad"):
            cap = min(cap, 4096 * 11008 // f)
        t = _log(rng, 1, max(1, min(8192, cap)))
        return _gated(kind, t, d, f, fmt, act=rng.choice(["silu", "silu", "gelu", "gelu_tanh"]),
                      deliver=rng.random() < 0.75)
    if kind == "adapters":
        t, k, n = _log(rng, 1, 8192), _width(rng, 64, 13824), _width(rng, 64, 13824)
        rank = rng.choice([4, 8, 16, 16, 32, 64, 12, 31, 128])
        count = _log(rng, 1, 64)
        requests = t if t <= 64 and rng.random() < 0.5 else min(t, _log(rng, 1, 64))
        return _adapters(t, k, n, count, rank, requests, fmt,
                         out="half" if rng.random() < 0.8 else "f32")
    hd = rng.choice([64, 80, 96, 128, 128, 128, 256])
    hkv = rng.choice([1, 2, 4, 8, 16])
    hq = hkv * rng.choice([1, 1, 2, 4, 8])
    rd = hd if rng.random() < 0.7 else hd // 4 * 2
    t = _log(rng, 1, max(1, min(16384, 8191 * 120 * 128 // ((hq + 2 * hkv) * hd))))
    return _heads(kind, t, hq, hkv, hd, rd, fmt, pairs=rng.choice(["half", "half", "interleaved"]),
                  norm=rng.random() < 0.75, far=_log(rng, max(t, 64), 1 << 20))


def work(case):
    kind, t = case["kind"], float(case["t"])
    if kind.startswith("gated"):
        d, f = float(case["d"]), float(case["f"])
        if kind == "gated":
            out = 2 * t * f + (8 * t * f if case["deliver"] else 0)
            return {"bytes": 2 * t * d + 4 * f * d + out, "flops": 4 * t * d * f}
        if kind == "gated_narrow":
            return {"bytes": 10 * t * f, "flops": 10 * t * f}
        if kind == "gated_grad":
            return {"bytes": (18 if case["deliver"] else 14) * t * f, "flops": 20 * t * f}
        return {"bytes": 4 * t * f + 2 * t * d + 4 * f * d + 4 * t * d + 8 * f * d,
                "flops": 8 * t * d * f}
    if kind == "adapters":
        k, n, r = float(case["k"]), float(case["n"]), float(case["rank"])
        met = min(case["count"], case["requests"])
        y = 2 if case["out"] == "half" else 4
        return {"bytes": 4 * t * n + 2 * t * k + y * t * n + 2 * met * r * (k + n) + 4 * t,
                "flops": 2 * t * r * (k + n) + t * n}
    hd = case["hd"]
    w, v = float((case["hq"] + 2 * case["hkv"]) * hd), float(case["hkv"] * hd)
    if kind == "heads":
        return {"bytes": 6 * t * w + 8 * t, "flops": 8 * t * w}
    c = 4 * t * (w - v) if case["norm"] else 0
    return {"bytes": c + 4 * t * w + 8 * t, "flops": 16 * t * w}


# ---------------------------------------------------------------------------------------------
# Inputs.


def _half(fmt):
    return {"bf16": torch.bfloat16, "fp16": torch.float16}[fmt]


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 * seed + 29)


def prepare(case, seed):
    """Activations N(0, 1) against weights N(0, 0.02), products of that scale, gradients N(0, 0.05)
    and gains near 1, all on the GPU."""
    g, h, t = _generator(seed), _half(case["fmt"]), case["t"]

    def mat(*shape, std=1.0, to=h):
        return torch.randn(*shape, generator=g, device="cuda").mul_(std).to(to)

    st = {"case": case}
    kind = case["kind"]
    if kind.startswith("gated"):
        d, f = case["d"], case["f"]
        if kind in ("gated", "gated_products"):
            st["X"], st["W"] = mat(t, d), mat(2 * f, d, std=0.02)
        if kind in ("gated_narrow", "gated_grad"):
            st["P"] = mat(t, 2 * f, std=0.02 * math.sqrt(d), to=torch.float32)
        if kind == "gated_grad":
            st["dH"] = mat(t, f, std=0.05)
        if kind == "gated_products":
            st["dP"] = mat(t, 2 * f, std=0.05)
    elif kind == "adapters":
        k, n, r, count = case["k"], case["n"], case["rank"], case["count"]
        st["X"] = mat(t, k)
        st["C"] = mat(t, n, std=0.02 * math.sqrt(k), to=torch.float32)
        st["A"], st["B"] = mat(count, r, k, std=1.0 / math.sqrt(k)), mat(count, n, r, std=0.02)
        st["scale"] = torch.rand(count, generator=g, device="cuda").add_(0.5)
        # tokens of a request are neighbours; one request in eight runs without an adapter
        cuts = torch.rand(case["requests"] - 1, generator=g, device="cuda").mul_(t).long()
        if case["requests"] == t:
            request = torch.arange(t, device="cuda")
        else:
            request = torch.bucketize(torch.arange(t, device="cuda"), cuts.sort().values, right=True)
        which = torch.randint(0, count, (case["requests"],), generator=g, device="cuda")
        none = torch.rand(case["requests"], generator=g, device="cuda") < 0.125
        st["index"] = torch.where(none, -1, which)[request].to(torch.int32)
    else:
        hq, hkv, hd, rd = case["hq"], case["hkv"], case["hd"], case["rd"]
        st["C"] = mat(t, (hq + 2 * hkv) * hd, std=1.3, to=torch.float32)
        st["gq"] = st["gk"] = None
        if case["norm"]:
            st["gq"] = 1 + mat(hd, std=0.1, to=torch.float32)
            st["gk"] = 1 + mat(hd, std=0.1, to=torch.float32)
        # a prompt's positions follow each other; decoding requests stand anywhere
        if t > 64:
            first = torch.randint(0, case["far"] - t + 1, (1,), generator=g, device="cuda")
            st["pos"] = first + torch.arange(t, device="cuda")
        else:
            st["pos"] = torch.randint(0, case["far"], (t,), generator=g, device="cuda")
        p = torch.arange(rd // 2, device="cuda", dtype=torch.float64)
        st["freq"] = torch.pow(10000.0, -2.0 * p / rd).float()
        if kind == "heads_grad":
            st["dq"] = mat(t, hq, hd, std=0.05)
            st["dk"], st["dv"] = mat(t, hkv, hd, std=0.05), mat(t, hkv, hd, std=0.05)
    torch.cuda.synchronize()
    return st


# ---------------------------------------------------------------------------------------------
# One pass.

_EPS = 1e-6


def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    from paper_2609_19758_amd import layers as fl

    case = st["case"]
    kind = case["kind"]
    if kind == "gated":
        H, P = fl.gated(st["X"], st["W"], act=case["act"], deliver=case["deliver"])
        return {"H": H, "P": P}
    if kind == "gated_narrow":
        return {"H": fl.gated_narrow(st["P"], case["fmt"], act=case["act"])}
    if kind == "gated_grad":
        dP, dPt = fl.gated_grad(st["dH"], st["P"], act=case["act"], transpose=case["deliver"])
        return {"dP": dP, "dPt": dPt}
    if kind == "gated_products":
        dX, dW = fl.gated_products(st["dP"], st["X"], st["W"])
        return {"dX": dX, "dW": dW}
    if kind == "adapters":
        return {"Y": fl.adapters(st["C"], st["X"], st["A"], st["B"], st["index"], st["scale"],
                                 out=case["out"])}
    hq, hkv = case["hq"], case["hkv"]
    kw = {"gq": st["gq"], "gk": st["gk"], "eps": _EPS, "pairs": case["pairs"]}
    if kind == "heads":
        q, k, v = fl.heads(st["C"], hq, hkv, st["pos"], st["freq"], case["fmt"], **kw)
        return {"q": q, "k": k, "v": v}
    dC, dgq, dgk = fl.heads_grad(st["dq"], st["dk"], st["dv"], st["C"], st["pos"], st["freq"], **kw)
    return {"dC": dC, "dgq": dgq, "dgk": dgk}


def _act(x, name):
    if name == "silu":
        return x * torch.sigmoid(x)
    if name == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))


def _act_grad(x, name):
    if name == "silu":
        s = torch.sigmoid(x)
        return s * (1 + x * (1 - s))
    if name == "gelu":
        return (0.5 * (1 + torch.erf(x * math.sqrt(0.5)))
                + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi))
    c = math.sqrt(2 / math.pi)
    th = torch.tanh(c * (x + 0.044715 * x * x * x))
    return 0.5 * (1 + th) + 0.5 * x * (1 - th * th) * c * (1 + 3 * 0.044715 * x * x)


def _turn(x, cos, sin, rd, pairs):
    """The rotation of the first rd entries of the heads x (t x heads x hd) by angles t x rd/2."""
    cos, sin = cos[:, None, :], sin[:, None, :]
    if pairs == "half":
        a, b = x[..., :rd // 2], x[..., rd // 2:rd]
    else:
        a, b = x[..., 0:rd:2], x[..., 1:rd:2]
    a, b = a * cos - b * sin, b * cos + a * sin
    y = torch.cat((a, b), -1) if pairs == "half" else torch.stack((a, b), -1).flatten(-2)
    return torch.cat((y, x[..., rd:]), -1)


def _run_plain(st):
    case = st["case"]
    kind, h = case["kind"], _half(case["fmt"])
    if kind.startswith("gated"):
        f, act = case["f"], case["act"]
        if kind in ("gated", "gated_narrow"):
            P = torch.mm(st["X"].float(), st["W"].float().t()) if kind == "gated" else st["P"]
            H = (_act(P[:, :f], act) * P[:, f:]).to(h)
            if kind == "gated_narrow":
                return {"H": H}
            return {"H": H, "P": P if case["deliver"] else None}
        if kind == "gated_grad":
            g, u, dH = st["P"][:, :f], st["P"][:, f:], st["dH"].float()
            dP = torch.cat((dH * u * _act_grad(g, act), dH * _act(g, act)), 1).to(h)
            return {"dP": dP, "dPt": dP.t().contiguous() if case["deliver"] else None}
        dP = st["dP"].float()
        return {"dX": torch.mm(dP, st["W"].float()), "dW": torch.mm(dP.t(), st["X"].float())}
    if kind == "adapters":
        # every row against every adapter, the columns of other adapters set to zero
        count, r, n = case["count"], case["rank"], case["n"]
        V = torch.mm(st["X"].float(), st["A"].float().reshape(count * r, -1).t())
        mine = st["index"][:, None] == torch.arange(count, device="cuda")
        V = torch.where(mine[:, :, None], V.view(-1, count, r) * st["scale"][:, None], 0.0)
        B = st["B"].float().transpose(1, 2).reshape(count * r, n)
        Y = st["C"] + torch.mm(V.reshape(-1, count * r), B)
        return {"Y": Y.to(h) if case["out"] == "half" else Y}
    hq, hkv, hd, rd, t = case["hq"], case["hkv"], case["hd"], case["rd"], case["t"]
    angle = st["pos"].double()[:, None] * st["freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    C = st["C"].view(t, hq + 2 * hkv, hd)
    xs = (C[:, :hq], C[:, hq:hq + hkv])
    gains = (st["gq"], st["gk"])
    norm, pairs = case["norm"], case["pairs"]
    inv = [torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS) if norm else None for x in xs]
    if kind == "heads":
        q, k = (_turn(x * r * g if norm else x, cos, sin, rd, pairs).to(h)
                for x, r, g in zip(xs, inv, gains))
        return {"q": q, "k": k, "v": C[:, hq + hkv:].to(h)}
    us = [_turn(dy.float(), cos, -sin, rd, pairs) for dy in (st["dq"], st["dk"])]
    dgq = dgk = None
    if norm:
        dgq, dgk = ((u * x * r).sum((0, 1)) for u, x, r in zip(us, xs, inv))
        us = [r * (g * u - x * r * r * (x * g * u).mean(-1, keepdim=True))
              for u, x, r, g in zip(us, xs, inv, gains)]
    dC = torch.cat((us[0].to(h), us[1].to(h), st["dv"]), 1).view(t, -1)
    return {"dC": dC, "dgq": dgq, "dgk": dgk}


# ---------------------------------------------------------------------------------------------
# The definitions in 64 bits.


def _exact_act(x, name):
    if name == "silu":
        return torch.nn.functional.silu(x)
    return torch.nn.functional.gelu(x, approximate="none" if name == "gelu" else "tanh")


def _exact_heads(C, case, pos, freq, gq, gk):
    """q, k, v of a product in 64 bits: the rotation as a complex product."""
    hq, hkv, hd, rd = case["hq"], case["hkv"], case["hd"], case["rd"]
    x = C.reshape(C.shape[0], hq + 2 * hkv, hd)
    angle = pos.double()[:, None, None] * freq.double()
    unit = torch.polar(torch.ones_like(angle), angle)
    out = []
    for y, g in ((x[:, :hq], gq), (x[:, hq:hq + hkv], gk)):
        if g is not None:
            y = y / ((y * y).sum(-1, keepdim=True) / hd + _EPS).sqrt() * g
        z, rest = y[..., :rd], y[..., rd:]
        if case["pairs"] == "half":
            z = z.unflatten(-1, (2, rd // 2)).transpose(-1, -2)
        else:
            z = z.unflatten(-1, (rd // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * unit)
        z = z.transpose(-1, -2).flatten(-2) if case["pairs"] == "half" else z.flatten(-2)
        out.append(torch.cat((z, rest), -1))
    return out[0], out[1], x[:, hq + hkv:]


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("gated"):
        f, act = case["f"], case["act"]
        if kind == "gated_products":
            dP = st["dP"].double()
            return {"dX": dP @ st["W"].double(), "dW": dP.t() @ st["X"].double()}
        P = (st["X"].double() @ st["W"].double().t() if kind == "gated" else st["P"].double())
        if kind == "gated_grad":
            P.requires_grad_(True)
        H = _exact_act(P.narrow(1, 0, f), act) * P.narrow(1, f, f)
        if kind == "gated_grad":
            (dP,) = torch.autograd.grad(H, P, st["dH"].double())
            return {"dP": dP, "dPt": dP.t().contiguous() if case["deliver"] else None}
        if kind == "gated_narrow":
            return {"H": H}
        return {"H": H, "P": P if case["deliver"] else None}
    if kind == "adapters":
        Y = st["C"].double()
        for a in range(case["count"]):
            rows = (st["index"] == a).nonzero().flatten()
            V = st["X"][rows].double() @ st["A"][a].double().t()
            Y[rows] += float(st["scale"][a]) * (V @ st["B"][a].double().t())
        return {"Y": Y}
    C = st["C"].double()
    gq, gk = (None if g is None else g.double() for g in (st["gq"], st["gk"]))
    if kind == "heads":
        q, k, v = _exact_heads(C, case, st["pos"], st["freq"], gq, gk)
        return {"q": q, "k": k, "v": v}
    leaves = [C] + ([gq, gk] if gq is not None else [])
    for x in leaves:
        x.requires_grad_(True)
    grads = torch.autograd.grad(_exact_heads(C, case, st["pos"], st["freq"], gq, gk), leaves,
                                [st[n].double() for n in ("dq", "dk", "dv")])
    dgq, dgk = grads[1:] if gq is not None else (None, None)
    return {"dC": grads[0], "dgq": dgq, "dgk": dgk}
