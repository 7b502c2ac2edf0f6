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
"""
from __future__ import annotations

import contextlib

from . import fpsketch as fk

ACT_CODE = {"silu": 0, "gelu": 1, "gelu_tanh": 2}
PAIRS_CODE = {"half": 0, "interleaved": 1}
MAX_RANK = 256
MAX_HEAD = 512


def _code(table: dict, key, what: str) -> int:
    if key not in table:
        raise ValueError(f"{what}: {key!r}, expected {' or '.join(repr(k) for k in table)}")
    return table[key]


def _fmt(x, what: str) -> str:
    """The half format of tensor x."""
    import torch
    names = {torch.bfloat16: "bf16", torch.float16: "fp16"}
    if x.dtype not in names:
        raise ValueError(f"{what}: dtype {x.dtype}, expected torch.bfloat16 or torch.float16")
    return names[x.dtype]


def _matrix(x, what: str, dims: int = 2):
    import torch
    if not isinstance(x, torch.Tensor) or x.dim() != dims:
        got = tuple(x.shape) if isinstance(x, torch.Tensor) else type(x).__name__
        raise ValueError(f"{what}: {got}, expected a tensor of {dims} dimensions")


def _check(x, what: str, shape, dtype, like=None):
    """Raises ValueError unless x has this shape and dtype, is contiguous and on the GPU of `like`."""
    _matrix(x, what, len(shape))
    if tuple(x.shape) != tuple(shape):
        raise ValueError(f"{what}: shape {tuple(x.shape)}, expected {tuple(shape)}")
    fk._check_tensor(x, what, [tuple(shape)], [dtype], None)
    if like is not None and x.device != like.device:
        raise ValueError(f"{what}: on {x.device}, other operands are on {like.device}")


class _Call:
    """The GPU and stream of one call.  Inside, torch allocates on them; `stream` is passed on."""

    def __init__(self, x, stream):
        self.device, self.given = x.device, stream

    def __enter__(self):
        import torch
        self.stack = contextlib.ExitStack()
        self.stack.enter_context(torch.cuda.device(self.device))
        if self.given is None:
            self.stream = torch.cuda.current_stream().cuda_stream
        else:
            self.stream = fk._stream(self.given)
            if self.stream != torch.cuda.current_stream().cuda_stream:
                self.stack.enter_context(torch.cuda.stream(
                    torch.cuda.ExternalStream(self.stream, device=self.device)))
        return self

    def __exit__(self, *exc):
        return self.stack.__exit__(*exc)

    def empty(self, shape, dtype):
        import torch
        return torch.empty(shape, dtype=dtype, device=self.device)

    def workspace(self, nbytes: int):
        import torch
        return self.empty((nbytes,), torch.uint8) if nbytes > 0 else None


def _output(call, out, what: str, shape, dtype):
    if out is None:
        return call.empty(shape, dtype)
    _check(out, what, shape, dtype)
    if out.device != call.device:
        raise ValueError(f"{what}: on {out.device}, the operands are on {call.device}")
    return out


# ---- gated feed-forward --------------------------------------------------------------------


def gated(X, W, act: str = "silu", deliver: bool = True, H=None, P=None, stream=None):
    """H = act(G) U with [G U] = P = X W^T, in one kernel.  X (t x d) and W (2f x d: f gate rows, then
    f up rows) in one half format; returns H (t x f, that format) and P (t x 2f FP32, the C of a
    ``Verifier(t, d, 2 * f, fmt, b_layout=1)`` with B = W), or None in its place with ``deliver``
    false.  ``H`` and ``P``: buffers to write into."""
    import torch
    _matrix(X, "X")
    _matrix(W, "W")
    a = _code(ACT_CODE, act, "act")
    fmt = _fmt(X, "X")
    (t, d), f = X.shape, W.shape[0] // 2
    if W.shape[0] % 2 or f == 0:
        raise ValueError(f"W: {W.shape[0]} rows, expected as many gate rows as up rows")
    _check(X, "X", (t, d), X.dtype)
    _check(W, "W", (2 * f, d), X.dtype, X)
    if P is not None and not deliver:
        raise ValueError("P: given with deliver=False")
    lib = fk.load()
    with _Call(X, stream) as c:
        H = _output(c, H, "H", (t, f), X.dtype)
        P = _output(c, P, "P", (t, 2 * f), torch.float32) if deliver else None
        n = lib.fpsketch_gated_workspace(t, d, f)
        ws = c.workspace(n)
        fk._check(lib.fpsketch_gated(fk._ptr(X), fk._ptr(W), t, d, f, fk.DTYPE_CODE[fmt], a,
                                     fk._ptr(H), fk._ptr(P), fk._ptr(ws), n, c.stream),
                  "fpsketch_gated")
    return H, P


def gated_narrow(P, fmt: str, act: str = "silu", H=None, stream=None):
    """H = act(G) U (t x f in the half format ``fmt``) from a delivered product P (t x 2f FP32), for
    instance after ``Verifier.apply`` repaired it: bit for bit what ``gated`` gives for that P."""
    import torch
    _matrix(P, "P")
    a, dt = _code(ACT_CODE, act, "act"), _code(fk.DTYPE_CODE, fmt, "fmt")
    if dt == fk.F32:
        raise ValueError("fmt: 'f32', expected 'fp16' or 'bf16'")
    t, f = P.shape[0], P.shape[1] // 2
    if P.shape[1] % 2 or f == 0:
        raise ValueError(f"P: {P.shape[1]} columns, expected as many gate columns as up columns")
    _check(P, "P", (t, 2 * f), torch.float32)
    lib = fk.load()
    with _Call(P, stream) as c:
        H = _output(c, H, "H", (t, f), fk.half_dtype(fmt))
        fk._check(lib.fpsketch_gated_narrow(fk._ptr(P), t, f, dt, a, fk._ptr(H), c.stream),
                  "fpsketch_gated_narrow")
    return H


def gated_grad(dH, P, act: str = "silu", transpose: bool = False, dP=None, dPt=None, stream=None):
    """The gradient of P from that of H: dP = [dH U act'(G), dH act(G)] (t x 2f in dH's half format),
    and with ``transpose`` its transpose (2f x t), the A of a ``Verifier(2 * f, t, d, fmt)`` that
    verifies dW; None in its place otherwise."""
    import torch
    _matrix(dH, "dH")
    a = _code(ACT_CODE, act, "act")
    fmt = _fmt(dH, "dH")
    t, f = dH.shape
    if f == 0:
        raise ValueError("dH: no columns")
    _check(dH, "dH", (t, f), dH.dtype)
    _check(P, "P", (t, 2 * f), torch.float32, dH)
    if dPt is not None and not transpose:
        raise ValueError("dPt: given with transpose=False")
    lib = fk.load()
    with _Call(dH, stream) as c:
        dP = _output(c, dP, "dP", (t, 2 * f), dH.dtype)
        dPt = _output(c, dPt, "dPt", (2 * f, t), dH.dtype) if transpose else None
        fk._check(lib.fpsketch_gated_grad(fk._ptr(dH), fk._ptr(P), t, f, fk.DTYPE_CODE[fmt], a,
                                          fk._ptr(dP), fk._ptr(dPt), c.stream),
                  "fpsketch_gated_grad")
    return dP, dPt


def gated_products(dP, X, W, need_dx: bool = True, need_dw: bool = True, dX=None, dW=None,
                   stream=None):
    """The products of the backward pass in FP32: dX = dP W (t x d, verified by a
    ``Verifier(t, 2 * f, d, fmt)`` with B = W) and dW = dP^T X (2f x d).  None in the place of one
    that is not needed."""
    import torch
    _matrix(dP, "dP")
    _matrix(W, "W")
    _matrix(X, "X")
    fmt = _fmt(dP, "dP")
    (t, d), f = X.shape, W.shape[0] // 2
    if W.shape[0] % 2 or f == 0:
        raise ValueError(f"W: {W.shape[0]} rows, expected as many gate rows as up rows")
    _check(dP, "dP", (t, 2 * f), dP.dtype)
    _check(X, "X", (t, d), dP.dtype, dP)
    _check(W, "W", (2 * f, d), dP.dtype, dP)
    if not (need_dx or need_dw):
        raise ValueError("need_dx, need_dw: nothing to compute")
    if (dX is not None and not need_dx) or (dW is not None and not need_dw):
        raise ValueError("dX, dW: a buffer is given for a product that is not needed")
    lib = fk.load()
    with _Call(dP, stream) as c:
        dX = _output(c, dX, "dX", (t, d), torch.float32) if need_dx else None
        dW = _output(c, dW, "dW", (2 * f, d), torch.float32) if need_dw else None
        n = lib.fpsketch_gated_products_workspace(t, d, f)
        ws = c.workspace(n)
        fk._check(lib.fpsketch_gated_products(fk._ptr(dP), fk._ptr(X), fk._ptr(W), t, d, f,
                                              fk.DTYPE_CODE[fmt], fk._ptr(dX), fk._ptr(dW),
                                              fk._ptr(ws), n, c.stream),
                  "fpsketch_gated_products")
    return dX, dW


# ---- adapters ------------------------------------------------------------------------------


def adapters(C, X, A, B, index, scale, out: str = "half", Y=None, stream=None):
    """Y_i = C_i + scale_a (X_i A_a^T) B_a^T with a = index_i, after C (t x n FP32, the product of the
    shared weight) was verified.  X (t x k), A (count x rank x k) and B (count x n x rank) in one
    half format, index (t int32; -1: no adapter; any other value outside [0, count) makes the row
    NaN), scale (count FP32).  Y is in that format, or FP32 with ``out`` "f32".  C is not
    modified."""
    import torch
    _matrix(X, "X")
    _matrix(C, "C")
    _matrix(A, "A", 3)
    fmt = _fmt(X, "X")
    if out not in ("half", "f32"):
        raise ValueError(f"out: {out!r}, expected 'half' or 'f32'")
    (t, k), n = X.shape, C.shape[1]
    count, rank = A.shape[:2]
    if not 1 <= rank <= MAX_RANK or count < 1:
        raise ValueError(f"A: {count} adapters of rank {rank}, expected at least one of rank 1 to "
                         f"{MAX_RANK}")
    _check(C, "C", (t, n), torch.float32)
    _check(X, "X", (t, k), X.dtype, C)
    _check(A, "A", (count, rank, k), X.dtype, C)
    _check(B, "B", (count, n, rank), X.dtype, C)
    _check(index, "index", (t,), torch.int32, C)
    _check(scale, "scale", (count,), torch.float32, C)
    lib = fk.load()
    with _Call(C, stream) as c:
        Y = _output(c, Y, "Y", (t, n), X.dtype if out == "half" else torch.float32)
        nws = lib.fpsketch_adapters_workspace(t, k, n, count, rank)
        ws = c.workspace(nws)
        fk._check(lib.fpsketch_adapters(fk._ptr(C), fk._ptr(X), fk._ptr(A), fk._ptr(B),
                                        fk._ptr(index), fk._ptr(scale), t, k, n, count, rank,
                                        fk.DTYPE_CODE[fmt], fk._ptr(Y),
                                        fk.DTYPE_CODE[fmt] if out == "half" else fk.F32,
                                        fk._ptr(ws), nws, c.stream),
                  "fpsketch_adapters")
    return Y


# ---- heads ---------------------------------------------------------------------------------


def _head_args(t, hd, gq, gk, pos, freq, pairs, like):
    import torch
    code = _code(PAIRS_CODE, pairs, "pairs")
    if not 1 <= hd <= MAX_HEAD:
        raise ValueError(f"heads of {hd} entries, expected 1 to {MAX_HEAD}")
    if (gq is None) != (gk is None):
        raise ValueError("gq, gk: gains for queries or keys only")
    if gq is not None:
        _check(gq, "gq", (hd,), torch.float32, like)
        _check(gk, "gk", (hd,), torch.float32, like)
    rd = 0
    if freq is not None:
        _matrix(freq, "freq", 1)
        rd = 2 * freq.shape[0]
        if rd > hd:
            raise ValueError(f"freq: {rd // 2} frequencies for heads of {hd} entries")
        _check(freq, "freq", (rd // 2,), torch.float32, like)
    if rd > 0:
        if pos is None:
            raise ValueError("pos: None with frequencies given")
        _check(pos, "pos", (t,), torch.int64, like)
    return code, rd


def heads(C, hq: int, hkv: int, pos, freq, fmt: str, gq=None, gk=None, eps: float = 1e-6,
          pairs: str = "half", q=None, k=None, v=None, stream=None):
    """Query, key and value heads of a delivered QKV product C (t x (hq + 2 hkv) hd FP32) in the half
    format ``fmt``: q (t x hq x hd), k and v (t x hkv x hd).  With gains gq, gk (hd FP32) each query
    and key head is normed, x g / sqrt(mean x^2 + eps); its first 2 len(freq) entries are rotated by
    pos_i freq_p (pos t int64, freq FP32; freq None: no rotation), in pairs (p, p + len(freq)), or
    (2p, 2p + 1) with ``pairs`` "interleaved"."""
    import torch
    _matrix(C, "C")
    dt = _code(fk.DTYPE_CODE, fmt, "fmt")
    if dt == fk.F32:
        raise ValueError("fmt: 'f32', expected 'fp16' or 'bf16'")
    t, width = C.shape
    if hq < 1 or hkv < 1 or width % (hq + 2 * hkv):
        raise ValueError(f"C: {width} columns for {hq} query and {hkv} key and value heads")
    hd = width // (hq + 2 * hkv)
    _check(C, "C", (t, width), torch.float32)
    code, rd = _head_args(t, hd, gq, gk, pos, freq, pairs, C)
    lib = fk.load()
    h = fk.half_dtype(fmt)
    with _Call(C, stream) as c:
        q = _output(c, q, "q", (t, hq, hd), h)
        k = _output(c, k, "k", (t, hkv, hd), h)
        v = _output(c, v, "v", (t, hkv, hd), h)
        fk._check(lib.fpsketch_heads(fk._ptr(C), t, hq, hkv, hd, fk._ptr(gq), fk._ptr(gk),
                                     float(eps), fk._ptr(pos) if rd else 0,
                                     fk._ptr(freq) if rd else 0, rd, code, dt, fk._ptr(q),
                                     fk._ptr(k), fk._ptr(v), c.stream), "fpsketch_heads")
    return q, k, v


def heads_grad(dq, dk, dv, C, pos, freq, gq=None, gk=None, eps: float = 1e-6, pairs: str = "half",
               dC=None, stream=None):
    """The backward pass of ``heads``: dC (t x (hq + 2 hkv) hd in the half format of dq, dk and dv) and
    the gradients of the gains (hd FP32 each; None without gains, when C is not read and may be
    None)."""
    import torch
    _matrix(dq, "dq", 3)
    _matrix(dk, "dk", 3)
    fmt = _fmt(dq, "dq")
    (t, hq, hd), hkv = dq.shape, dk.shape[1]
    if hq < 1 or hkv < 1:
        raise ValueError(f"dq, dk: {hq} query and {hkv} key heads")
    _check(dq, "dq", (t, hq, hd), dq.dtype)
    _check(dk, "dk", (t, hkv, hd), dq.dtype, dq)
    _check(dv, "dv", (t, hkv, hd), dq.dtype, dq)
    width = (hq + 2 * hkv) * hd
    if gq is not None or C is not None:
        _check(C, "C", (t, width), torch.float32, dq)
    code, rd = _head_args(t, hd, gq, gk, pos, freq, pairs, dq)
    lib = fk.load()
    with _Call(dq, stream) as c:
        dC = _output(c, dC, "dC", (t, width), dq.dtype)
        dgq = dgk = ws = None
        n = 0
        if gq is not None:
            dgq, dgk = c.empty((hd,), torch.float32), c.empty((hd,), torch.float32)
            n = lib.fpsketch_heads_grad_workspace(t, hq, hkv, hd)
            ws = c.workspace(n)
        fk._check(lib.fpsketch_heads_grad(fk._ptr(dq), fk._ptr(dk), fk._ptr(dv), fk._ptr(C), t, hq,
                                          hkv, hd, fk._ptr(gq), fk._ptr(gk), float(eps),
                                          fk._ptr(pos) if rd else 0, fk._ptr(freq) if rd else 0,
                                          rd, code, fk.DTYPE_CODE[fmt], fk._ptr(dC), fk._ptr(dgq),
                                          fk._ptr(dgk), fk._ptr(ws), n, c.stream),
                  "fpsketch_heads_grad")
    return dC, dgq, dgk
