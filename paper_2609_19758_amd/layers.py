"""Operators around a delivered product (the second part of the C ABI in include/fpsketch.h).

A verified linear layer delivers its product C = A W^T in FP32; these calls take it on to the half
format that the next layer reads, together with the layer's own arithmetic:

  gated, gated_narrow, gated_grad, gated_products   the gated feed-forward block and its backward pass
  adapters                                          low-rank adapters of many requests added to C
  heads, heads_grad                                 head norms with the position rotation

Their own products (P of the block; dX and dW of its backward pass) are delivered in FP32 in the
layouts that ``fpsketch.Verifier`` takes, so the same calls verify and repair them.

As in ``fpsketch``, this is argument marshalling only: every step runs in the library's HIP kernels.
Operands are torch tensors, contiguous and on one GPU; they are checked before the library is
called.  The work is enqueued on ``stream`` (default: torch's current stream of the operands' GPU),
and outputs and workspaces are allocated on that stream, so a call can be captured into a graph.
None of it is recorded by autograd: operands that require gradients are taken as they are and results
carry none; the ``_grad`` and ``_products`` calls are the backward passes, called by name.
"""
from __future__ import annotations

import contextlib

import torch

from . import fpsketch as fk

ACT_CODE = {"silu": 0, "gelu": 1, "gelu_tanh": 2}
PAIRS_CODE = {"half": 0, "interleaved": 1}
MAX_RANK = 256
MAX_HEAD = 512
_HALF_CODE = {torch.float16: fk.F16, torch.bfloat16: fk.BF16}
_FMT = {"fp16": (fk.F16, torch.float16), "bf16": (fk.BF16, torch.bfloat16)}
_F32 = torch.float32


def _code(table: dict, key, what: str):
    try:
        return table[key]
    except (KeyError, TypeError):
        raise ValueError(f"{what}: {key!r}, expected "
                         f"{' or '.join(repr(k) for k in table)}") from None


def _half(x, what: str) -> int:
    """The library's code of tensor x's half format."""
    code = _HALF_CODE.get(x.dtype)
    if code is None:
        raise ValueError(f"{what}: dtype {x.dtype}, expected torch.bfloat16 or torch.float16")
    return code


def _shape(x, what: str, dims: int = 2):
    if not isinstance(x, torch.Tensor) or x.dim() != dims:
        got = tuple(x.shape) if isinstance(x, torch.Tensor) else type(x).__name__
        raise ValueError(f"{what}: {got}, expected a tensor of {dims} dimensions")
    return x.shape


def _check(x, what: str, shape: tuple, dtype, device=None) -> int:
    """x's address.  Raises ValueError unless x has this shape and dtype, is contiguous and lives on
    the GPU `device` (None: any GPU)."""
    if (isinstance(x, torch.Tensor) and x.dtype is dtype and x.shape == shape
            and x.is_contiguous() and x.is_cuda and (device is None or x.device == device)):
        return x.data_ptr()
    _shape(x, what, len(shape))
    if tuple(x.shape) != shape:
        raise ValueError(f"{what}: shape {tuple(x.shape)}, expected {shape}")
    fk._check_tensor(x, what, [shape], [dtype], None)
    raise ValueError(f"{what}: on {x.device}, other operands are on {device}")


def _empty(shape: tuple, dtype, device):
    """A new contiguous tensor of one to three dimensions; with strides given a fifth faster than
    torch.empty, which a small operator notices."""
    inner = shape[-1]
    strides = (1,) if len(shape) == 1 else (inner, 1) if len(shape) == 2 else (shape[1] * inner, inner, 1)
    return torch.empty_strided(shape, strides, dtype=dtype, device=device)


class _Call:
    """The GPU and stream of one call: inside, torch allocates on them; `stream` is passed on."""
    __slots__ = ("device", "stream", "stack")

    def __init__(self, device, stream):
        self.device, self.stack = device, None
        if stream is None and device.index == torch._C._cuda_getDevice():
            self.stream = torch._C._cuda_getCurrentRawStream(device.index)
            return
        if getattr(stream, "device", device) != device:
            raise ValueError(f"stream: on {stream.device}, the operands are on {device}")
        given = None if stream is None else fk._stream(stream)
        self.stack = contextlib.ExitStack()
        self.stack.enter_context(torch.cuda.device(device))
        now = torch.cuda.current_stream().cuda_stream
        self.stream = now if given is None else given
        if self.stream != now:
            self.stack.enter_context(torch.cuda.stream(
                torch.cuda.ExternalStream(self.stream, device=device)))

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        if self.stack is not None:
            self.stack.close()

    def output(self, out, what: str, shape: tuple, dtype):
        """The tensor to write, `out` where it is given, and its address."""
        if out is None:
            out = _empty(shape, dtype, self.device)
            return out, out.data_ptr()
        return out, _check(out, what, shape, dtype, self.device)

    def workspace(self, nbytes: int):
        if nbytes <= 0:
            return None, 0
        w = _empty((nbytes,), torch.uint8, self.device)
        return w, w.data_ptr()


# ---- gated feed-forward --------------------------------------------------------------------


def gated(X, W, act: str = "silu", deliver: bool = True, H=None, P=None, stream=None):
    """H = act(G) U with [G U] = P = X W^T, without another pass over P.  X (t x d) and W (2f x d: f gate rows, then
    f up rows) in one half format; returns H (t x f, that format) and P (t x 2f FP32, the C of a
    ``Verifier(t, d, 2 * f, fmt, b_layout=1)`` with B = W), or None in its place with ``deliver``
    false.  ``H`` and ``P``: buffers to write into."""
    (t, d), rows = _shape(X, "X"), _shape(W, "W")[0]
    a, code, h = _code(ACT_CODE, act, "act"), _half(X, "X"), X.dtype
    f = rows // 2
    if rows % 2 or f == 0:
        raise ValueError(f"W: {rows} rows, expected as many gate rows as up rows")
    x = _check(X, "X", (t, d), h)
    w = _check(W, "W", (rows, d), h, X.device)
    if P is not None and not deliver:
        raise ValueError("P: given with deliver=False")
    lib = fk.load()
    with _Call(X.device, stream) as c:
        H, hp = c.output(H, "H", (t, f), h)
        pp = 0
        if deliver:
            P, pp = c.output(P, "P", (t, rows), _F32)
        n = lib.fpsketch_gated_workspace(x, w, t, d, f)
        ws, wp = c.workspace(n)
        fk._check(lib.fpsketch_gated(x, w, t, d, f, code, a, hp, pp, wp, n, c.stream),
                  "fpsketch_gated")
    return H, P


def gated_narrow(P, fmt: str, act: str = "silu", H=None, stream=None):
    """H = act(G) U (t x f in the half format ``fmt``) from a delivered product P (t x 2f FP32), for
    instance after ``Verifier.apply`` repaired it: bit for bit what ``gated`` gives for that P."""
    t, cols = _shape(P, "P")
    a, (code, h) = _code(ACT_CODE, act, "act"), _code(_FMT, fmt, "fmt")
    f = cols // 2
    if cols % 2 or f == 0:
        raise ValueError(f"P: {cols} columns, expected as many gate columns as up columns")
    p = _check(P, "P", (t, cols), _F32)
    lib = fk.load()
    with _Call(P.device, stream) as c:
        H, hp = c.output(H, "H", (t, f), h)
        fk._check(lib.fpsketch_gated_narrow(p, t, f, code, a, hp, c.stream),
                  "fpsketch_gated_narrow")
    return H


def gated_grad(dH, P, act: str = "silu", transpose: bool = False, dP=None, dPt=None, stream=None):
    """The gradient of P from that of H: dP = [dH U act'(G), dH act(G)] (t x 2f in dH's half format),
    and with ``transpose`` its transpose (2f x t), the A of a ``Verifier(2 * f, t, d, fmt)`` that
    verifies dW; None in its place otherwise."""
    t, f = _shape(dH, "dH")
    a, code, h = _code(ACT_CODE, act, "act"), _half(dH, "dH"), dH.dtype
    if f == 0:
        raise ValueError("dH: no columns")
    dh = _check(dH, "dH", (t, f), h)
    p = _check(P, "P", (t, 2 * f), _F32, dH.device)
    if dPt is not None and not transpose:
        raise ValueError("dPt: given with transpose=False")
    lib = fk.load()
    with _Call(dH.device, stream) as c:
        dP, op = c.output(dP, "dP", (t, 2 * f), h)
        tp = 0
        if transpose:
            dPt, tp = c.output(dPt, "dPt", (2 * f, t), h)
        fk._check(lib.fpsketch_gated_grad(dh, p, t, f, code, a, op, tp, c.stream),
                  "fpsketch_gated_grad")
    return dP, dPt


def gated_products(dP, X, W, need_dx: bool = True, need_dw: bool = True, dX=None, dW=None,
                   stream=None):
    """The products of the backward pass in FP32: dX = dP W (t x d, verified by a
    ``Verifier(t, 2 * f, d, fmt)`` with B = W) and dW = dP^T X (2f x d).  None in the place of one
    that is not needed."""
    _shape(dP, "dP")
    (t, d), rows = _shape(X, "X"), _shape(W, "W")[0]
    code, h, f = _half(dP, "dP"), dP.dtype, rows // 2
    if rows % 2 or f == 0:
        raise ValueError(f"W: {rows} rows, expected as many gate rows as up rows")
    p = _check(dP, "dP", (t, rows), h)
    x = _check(X, "X", (t, d), h, dP.device)
    w = _check(W, "W", (rows, d), h, dP.device)
    if not (need_dx or need_dw):
        raise ValueError("need_dx, need_dw: nothing to compute")
    if (dX is not None and not need_dx) or (dW is not None and not need_dw):
        raise ValueError("dX, dW: a buffer is given for a product that is not needed")
    lib = fk.load()
    with _Call(dP.device, stream) as c:
        xp = gp = 0
        if need_dx:
            dX, xp = c.output(dX, "dX", (t, d), _F32)
        if need_dw:
            dW, gp = c.output(dW, "dW", (rows, d), _F32)
        n = lib.fpsketch_gated_products_workspace(p, x, w, t, d, f, need_dx, need_dw)
        ws, wp = c.workspace(n)
        fk._check(lib.fpsketch_gated_products(p, x, w, t, d, f, code, xp, gp, wp, n, c.stream),
                  "fpsketch_gated_products")
    return dX, dW


# ---- adapters ------------------------------------------------------------------------------


def adapters(C, X, A, B, index, scale, out: str = "half", Y=None, stream=None):
    """Y_i = C_i + scale_a (X_i A_a^T) B_a^T with a = index_i, after C (t x n FP32, the product of the
    shared weight) was verified.  X (t x k), A (count x rank x k) and B (count x n x rank) in one
    half format, index (t int32; -1: no adapter; any other value outside [0, count) makes the row
    NaN), scale (count FP32).  Y is in that format, or FP32 with ``out`` "f32".  C is not
    modified."""
    (t, k), n = _shape(X, "X"), _shape(C, "C")[1]
    count, rank, _ = _shape(A, "A", 3)
    code, h = _half(X, "X"), X.dtype
    if out not in ("half", "f32"):
        raise ValueError(f"out: {out!r}, expected 'half' or 'f32'")
    if not 1 <= rank <= MAX_RANK or count < 1:
        raise ValueError(f"A: {count} adapters of rank {rank}, expected at least one of rank 1 to "
                         f"{MAX_RANK}")
    cp = _check(C, "C", (t, n), _F32)
    dev = C.device
    x = _check(X, "X", (t, k), h, dev)
    ap = _check(A, "A", (count, rank, k), h, dev)
    bp = _check(B, "B", (count, n, rank), h, dev)
    ip = _check(index, "index", (t,), torch.int32, dev)
    sp = _check(scale, "scale", (count,), _F32, dev)
    lib = fk.load()
    with _Call(dev, stream) as c:
        Y, yp = c.output(Y, "Y", (t, n), h if out == "half" else _F32)
        nws = lib.fpsketch_adapters_workspace(t, k, n, count, rank)
        ws, wp = c.workspace(nws)
        fk._check(lib.fpsketch_adapters(cp, x, ap, bp, ip, sp, t, k, n, count, rank, code, yp,
                                        code if out == "half" else fk.F32, wp, nws, c.stream),
                  "fpsketch_adapters")
    return Y


# ---- heads ---------------------------------------------------------------------------------


def _head_args(t, hd, gq, gk, pos, freq, pairs, device):
    """Code of the pairs, rotated entries, and the addresses of gq, gk, pos and freq (0: none)."""
    code = _code(PAIRS_CODE, pairs, "pairs")
    if not 1 <= hd <= MAX_HEAD:
        raise ValueError(f"heads of {hd} entries, expected 1 to {MAX_HEAD}")
    if (gq is None) != (gk is None):
        raise ValueError("gq, gk: gains for queries or keys only")
    q = k = p = w = rd = 0
    if gq is not None:
        q = _check(gq, "gq", (hd,), _F32, device)
        k = _check(gk, "gk", (hd,), _F32, device)
    if freq is not None:
        rd = 2 * _shape(freq, "freq", 1)[0]
        if rd > hd:
            raise ValueError(f"freq: {rd // 2} frequencies for heads of {hd} entries")
        w = _check(freq, "freq", (rd // 2,), _F32, device)
    if rd > 0:
        if pos is None:
            raise ValueError("pos: None with frequencies given")
        p = _check(pos, "pos", (t,), torch.int64, device)
    return code, rd, q, k, p, w


def heads(C, hq: int, hkv: int, pos, freq, fmt: str, gq=None, gk=None, eps: float = 1e-6,
          pairs: str = "half", q=None, k=None, v=None, stream=None):
    """Query, key and value heads of a delivered QKV product C (t x (hq + 2 hkv) hd FP32) in the half
    format ``fmt``: q (t x hq x hd), k and v (t x hkv x hd).  With gains gq, gk (hd FP32) each query
    and key head is normed, x g / sqrt(mean x^2 + eps) (eps 0 or a normal number of FP32); its first
    2 len(freq) entries are rotated by pos_i freq_p (pos t int64, freq FP32; freq None: no rotation), in
    pairs (p, p + len(freq)), or (2p, 2p + 1) with ``pairs`` "interleaved"."""
    t, width = _shape(C, "C")
    dt, h = _code(_FMT, fmt, "fmt")
    if hq < 1 or hkv < 1 or width % (hq + 2 * hkv):
        raise ValueError(f"C: {width} columns for {hq} query and {hkv} key and value heads")
    hd = width // (hq + 2 * hkv)
    cp = _check(C, "C", (t, width), _F32)
    code, rd, gqp, gkp, pp, wp = _head_args(t, hd, gq, gk, pos, freq, pairs, C.device)
    lib = fk.load()
    with _Call(C.device, stream) as c:
        q, qp = c.output(q, "q", (t, hq, hd), h)
        k, kp = c.output(k, "k", (t, hkv, hd), h)
        v, vp = c.output(v, "v", (t, hkv, hd), h)
        fk._check(lib.fpsketch_heads(cp, t, hq, hkv, hd, gqp, gkp, eps, pp, wp, rd, code, dt, qp, kp,
                                     vp, c.stream), "fpsketch_heads")
    return q, k, v


def heads_grad(dq, dk, dv, C, pos, freq, gq=None, gk=None, eps: float = 1e-6, pairs: str = "half",
               dC=None, stream=None):
    """The backward pass of ``heads``: dC (t x (hq + 2 hkv) hd in the half format of dq, dk and dv) and
    the gradients of the gains (hd FP32 each; None without gains, when C is not read and may be
    None)."""
    (t, hq, hd), hkv = _shape(dq, "dq", 3), _shape(dk, "dk", 3)[1]
    dt, h = _half(dq, "dq"), dq.dtype
    if hq < 1 or hkv < 1:
        raise ValueError(f"dq, dk: {hq} query and {hkv} key heads")
    qp = _check(dq, "dq", (t, hq, hd), h)
    dev = dq.device
    kp = _check(dk, "dk", (t, hkv, hd), h, dev)
    vp = _check(dv, "dv", (t, hkv, hd), h, dev)
    width, cp = (hq + 2 * hkv) * hd, 0
    if gq is not None or C is not None:
        cp = _check(C, "C", (t, width), _F32, dev)
    code, rd, gqp, gkp, pp, wp = _head_args(t, hd, gq, gk, pos, freq, pairs, dev)
    lib = fk.load()
    with _Call(dev, stream) as c:
        dC, op = c.output(dC, "dC", (t, width), h)
        dgq = dgk = None
        dgqp = dgkp = n = wsp = 0
        if gq is not None:
            dgq, dgqp = c.output(None, "dgq", (hd,), _F32)
            dgk, dgkp = c.output(None, "dgk", (hd,), _F32)
            n = lib.fpsketch_heads_grad_workspace(t, hq, hkv, hd)
            ws, wsp = c.workspace(n)
        fk._check(lib.fpsketch_heads_grad(qp, kp, vp, cp, t, hq, hkv, hd, gqp, gkp, eps, pp, wp, rd,
                                          code, dt, op, dgqp, dgkp, wsp, n, c.stream),
                  "fpsketch_heads_grad")
    return dC, dgq, dgk
