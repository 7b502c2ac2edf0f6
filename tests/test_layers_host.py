"""The C entry points of the operators around a delivered product, on the CPU: the built library on the
stand-in for the HIP runtime (layers_runtime.cpp, which runs no kernel and refuses launches outside the
runtime's limits), in a process of its own.  Addresses are made up: nothing is read."""
import ctypes
import itertools
import os
import random
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2609_19758_amd import fpsketch as fk  # noqa: E402

STREAM = 0x1000


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("rt") / "libhostrt.so")
    inc = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__",
                    f"-I{inc}", f"-I{os.path.join(ROOT, 'paper_2609_19758_amd', 'csrc')}",
                    f"-I{os.path.join(ROOT, 'include')}", "-o", out,
                    os.path.join(ROOT, "tests", "layers_runtime.cpp")], check=True)
    return out


@pytest.mark.parametrize("scenario", ["refusals", "launches", "empty", "failures", "overlaps"])
def test_entry_points(runtime, scenario):
    env = dict(os.environ, PYTHONPATH=ROOT)
    res = subprocess.run([sys.executable, os.path.abspath(__file__), runtime, scenario],
                         capture_output=True, text=True, timeout=100, env=env)
    assert res.returncode == 0, res.stdout + res.stderr


# ---- in the process of its own -------------------------------------------------------------


class Host:
    def __init__(self, runtime):
        self.rt = ctypes.CDLL(runtime, mode=ctypes.RTLD_GLOBAL)
        self.rt.rt_log.restype = self.rt.rt_faults.restype = ctypes.c_char_p
        self.lib = ctypes.CDLL(fk.LIB_PATH)
        for name, (res, argtypes) in fk._SIGS.items():
            fn = getattr(self.lib, name)
            fn.restype, fn.argtypes = res, argtypes

    def kernels(self):
        """(name, grid) of the launches since the last reset."""
        got = [(ln.split()[0], int(ln.split()[1])) for ln in self.rt.rt_log().decode().splitlines()]
        self.rt.rt_reset()
        return got

    def error(self):
        return self.lib.fpsketch_last_error().decode()


class Room:
    """Addresses of arrays that do not overlap."""

    def __init__(self, shift=0):
        self.next, self.shift = 1 << 40, shift

    def take(self, nbytes, shift=None):
        p = self.next
        self.next += (nbytes + 4095) // 4096 * 4096 + 4096
        return p + (self.shift if shift is None else shift)


class Gated:
    name = "fpsketch_gated"

    def __init__(self, h, t=100, d=264, f=136, shift=0):
        self.h, self.t, self.d, self.f = h, t, d, f
        r = Room(shift)
        self.a = dict(X=r.take(2 * t * d), W=r.take(4 * f * d), t=t, d=d, f=f, dt=fk.BF16, act=0,
                      H=r.take(2 * t * f), P=r.take(8 * t * f), ws=r.take(1 << 45, 0), n=None)

    def need(self):
        a = self.a
        return self.h.lib.fpsketch_gated_workspace(a["X"], a["W"], a["t"], a["d"], a["f"])

    def __call__(self, **kw):
        a = dict(self.a, **kw)
        n = self.need() if a["n"] is None else a["n"]
        return self.h.lib.fpsketch_gated(a["X"], a["W"], a["t"], a["d"], a["f"], a["dt"], a["act"],
                                         a["H"], a["P"], a["ws"], n, STREAM)


class Narrow:
    name = "fpsketch_gated_narrow"

    def __init__(self, h, t=100, d=0, f=136, shift=0):
        self.h = h
        r = Room(shift)
        self.a = dict(P=r.take(8 * t * f), t=t, f=f, dt=fk.F16, act=1, H=r.take(2 * t * f))

    def need(self):
        return 0

    def __call__(self, **kw):
        a = dict(self.a, **kw)
        return self.h.lib.fpsketch_gated_narrow(a["P"], a["t"], a["f"], a["dt"], a["act"], a["H"], STREAM)


class Grad:
    name = "fpsketch_gated_grad"

    def __init__(self, h, t=100, d=0, f=136, shift=0):
        self.h = h
        r = Room(shift)
        self.a = dict(dH=r.take(2 * t * f), P=r.take(8 * t * f), t=t, f=f, dt=fk.F16, act=2,
                      dP=r.take(4 * t * f), dPt=r.take(4 * t * f))

    def need(self):
        return 0

    def __call__(self, **kw):
        a = dict(self.a, **kw)
        return self.h.lib.fpsketch_gated_grad(a["dH"], a["P"], a["t"], a["f"], a["dt"], a["act"], a["dP"],
                                              a["dPt"], STREAM)


class Products:
    name = "fpsketch_gated_products"

    def __init__(self, h, t=100, d=264, f=136, shift=0):
        self.h = h
        r = Room(shift)
        self.a = dict(dP=r.take(4 * t * f), X=r.take(2 * t * d), W=r.take(4 * f * d), t=t, d=d, f=f,
                      dt=fk.F16, dX=r.take(4 * t * d), dW=r.take(8 * f * d), ws=r.take(1 << 45, 0), n=None)

    def need(self, **kw):
        a = dict(self.a, **kw)
        return self.h.lib.fpsketch_gated_products_workspace(a["dP"], a["X"], a["W"], a["t"], a["d"], a["f"],
                                                            int(bool(a["dX"])), int(bool(a["dW"])))

    def __call__(self, **kw):
        a = dict(self.a, **kw)
        n = self.need(**kw) if a["n"] is None else a["n"]
        return self.h.lib.fpsketch_gated_products(a["dP"], a["X"], a["W"], a["t"], a["d"], a["f"], a["dt"],
                                                  a["dX"], a["dW"], a["ws"], n, STREAM)


class Adapters:
    name = "fpsketch_adapters"

    def __init__(self, h, t=100, d=264, f=136, shift=0, count=5, rank=12):
        self.h = h
        r, k, n = Room(shift), d, f
        self.a = dict(C=r.take(4 * t * n), X=r.take(2 * t * k), A=r.take(2 * count * rank * k),
                      B=r.take(2 * count * rank * n), index=r.take(4 * t), scale=r.take(4 * count), t=t, k=k,
                      nn=n, count=count, rank=rank, dt=fk.BF16, Y=r.take(4 * t * n), ydt=fk.F32,
                      ws=r.take(1 << 45, 0), n=None)

    def need(self):
        a = self.a
        return self.h.lib.fpsketch_adapters_workspace(a["t"], a["k"], a["nn"], a["count"], a["rank"])

    def __call__(self, **kw):
        a = dict(self.a, **kw)
        n = self.need() if a["n"] is None else a["n"]
        return self.h.lib.fpsketch_adapters(a["C"], a["X"], a["A"], a["B"], a["index"], a["scale"], a["t"],
                                            a["k"], a["nn"], a["count"], a["rank"], a["dt"], a["Y"],
                                            a["ydt"], a["ws"], n, STREAM)


class Heads:
    name = "fpsketch_heads"

    def __init__(self, h, t=100, d=0, f=0, shift=0, hq=4, hkv=2, hd=64, rd=32):
        self.h = h
        r = Room(shift)
        self.a = dict(C=r.take(4 * t * (hq + 2 * hkv) * hd), t=t, hq=hq, hkv=hkv, hd=hd, gq=r.take(4 * hd),
                      gk=r.take(4 * hd), eps=1e-6, pos=r.take(8 * t), freq=r.take(2 * rd), rd=rd, pairs=0,
                      dt=fk.F16, q=r.take(2 * t * hq * hd), k=r.take(2 * t * hkv * hd),
                      v=r.take(2 * t * hkv * hd))

    def need(self):
        return 0

    def __call__(self, **kw):
        a = dict(self.a, **kw)
        return self.h.lib.fpsketch_heads(a["C"], a["t"], a["hq"], a["hkv"], a["hd"], a["gq"], a["gk"],
                                         a["eps"], a["pos"], a["freq"], a["rd"], a["pairs"], a["dt"], a["q"],
                                         a["k"], a["v"], STREAM)


class HeadsGrad:
    name = "fpsketch_heads_grad"

    def __init__(self, h, t=100, d=0, f=0, shift=0, hq=4, hkv=2, hd=64, rd=32):
        self.h = h
        r, w = Room(shift), (hq + 2 * hkv) * hd
        self.a = dict(dq=r.take(2 * t * hq * hd), dk=r.take(2 * t * hkv * hd), dv=r.take(2 * t * hkv * hd),
                      C=r.take(4 * t * w), t=t, hq=hq, hkv=hkv, hd=hd, gq=r.take(4 * hd), gk=r.take(4 * hd),
                      eps=1e-6, pos=r.take(8 * t), freq=r.take(2 * rd), rd=rd, pairs=1, dt=fk.BF16,
                      dC=r.take(2 * t * w), dgq=r.take(4 * hd), dgk=r.take(4 * hd), ws=r.take(1 << 45, 0),
                      n=None)

    def need(self):
        a = self.a
        return self.h.lib.fpsketch_heads_grad_workspace(a["t"], a["hq"], a["hkv"], a["hd"])

    def __call__(self, **kw):
        a = dict(self.a, **kw)
        n = self.need() if a["n"] is None else a["n"]
        return self.h.lib.fpsketch_heads_grad(a["dq"], a["dk"], a["dv"], a["C"], a["t"], a["hq"], a["hkv"],
                                              a["hd"], a["gq"], a["gk"], a["eps"], a["pos"], a["freq"],
                                              a["rd"], a["pairs"], a["dt"], a["dC"], a["dgq"], a["dgk"],
                                              a["ws"], n, STREAM)


CALLS = [Gated, Narrow, Grad, Products, Adapters, Heads, HeadsGrad]
POINTERS = {"X", "W", "H", "P", "dH", "dP", "dPt", "dX", "dW", "C", "A", "B", "index", "scale", "Y", "q", "k",
            "v", "gq", "gk", "pos", "freq", "dq", "dk", "dv", "dC", "dgq", "dgk", "ws"}


def pointers(call):
    """Names of a call's array arguments."""
    return [n for n in call.a if n in POINTERS and call.a[n] >= 1 << 40]


OPTIONAL = {("fpsketch_gated", "P"), ("fpsketch_gated_grad", "dPt"), ("fpsketch_gated_products", "dX"),
            ("fpsketch_gated_products", "dW")}


def refusals(h):
    """Every argument that cannot be right is refused before any launch, with a detail."""
    big = 1 << 31

    def refused(call, status, **kw):
        h.rt.rt_reset()
        got = call(**kw)
        assert got == status, (call.name, kw, got, h.error())
        assert call.name in h.error(), (call.name, kw, h.error())
        assert h.kernels() == [], (call.name, kw)

    for C in CALLS:
        call = C(h)
        assert call() == fk.OK, h.error()
        refused(call, fk.EDTYPE, dt=fk.F32)
        refused(call, fk.EDTYPE, dt=7)
        refused(call, fk.ESHAPE, t=-1)
        refused(call, fk.ESHAPE, t=big)
        for n in pointers(call):
            if n == "ws":
                continue
            step = 8 if n == "pos" else 2
            refused(call, fk.EINVAL, **{n: call.a[n] + step // 2})
            if (call.name, n) not in OPTIONAL:
                refused(call, fk.EINVAL, **{n: 0})
            else:
                assert call(**{n: 0}) == fk.OK, (call.name, n, h.error())
        for n in ("d", "f", "k", "nn", "count", "rank", "hq", "hkv", "hd"):
            if n in call.a and n not in pointers(call):
                refused(call, fk.ESHAPE, **{n: 0})
                refused(call, fk.ESHAPE, **{n: -3})
        if "act" in call.a:
            refused(call, fk.EINVAL, act=3)
            refused(call, fk.EINVAL, act=-1)
        if "ws" in call.a and call.need() > 0:
            refused(call, fk.EINVAL, n=call.need() - 1)
            refused(call, fk.EINVAL, ws=0)
            refused(call, fk.EINVAL, ws=call.a["ws"] + 8)
    refused(Gated(h), fk.ESHAPE, d=(1 << 22) + 1)
    refused(Gated(h), fk.ESHAPE, f=(1 << 21) + 1)
    refused(Gated(h), fk.ESHAPE, t=1 << 30, d=1 << 20)
    refused(Products(h), fk.EINVAL, dX=0, dW=0)
    refused(Adapters(h), fk.ESHAPE, rank=257)
    refused(Adapters(h), fk.EDTYPE, ydt=fk.F16)
    refused(Adapters(h), fk.EDTYPE, ydt=9)
    refused(Heads(h), fk.ESHAPE, hd=513)
    for C in (Heads, HeadsGrad):
        refused(C(h), fk.EINVAL, rd=31)
        refused(C(h), fk.EINVAL, rd=66)
        refused(C(h), fk.EINVAL, rd=-2)
        refused(C(h), fk.EINVAL, pairs=2)
        refused(C(h), fk.EINVAL, eps=-1.0)
        refused(C(h), fk.EINVAL, eps=float("nan"))
        assert C(h)(gq=0, gk=0, eps=float("nan")) == fk.OK      # (no norm: eps is not looked at)
        assert C(h)(rd=0, pos=0, freq=0) == fk.OK
    assert HeadsGrad(h)(gq=0, gk=0, C=0, dgq=0, dgk=0, ws=0, n=0) == fk.OK


def launches(h):
    """Launches stay within the runtime's limits over the whole range of sizes and alignments, and the
    workspace that the query names is enough (one byte less is refused)."""
    rng = random.Random(3)
    sizes = [1, 2, 7, 8, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1000, 1024, 2731, 4096, 11008]

    def check(call):
        h.rt.rt_reset()
        assert call() == fk.OK, (call.name, call.a, h.error())
        got = h.kernels()
        assert got and all(g > 0 for _, g in got), (call.name, call.a, got)
        n = call.need()
        if n > 0:
            assert call(n=n - 1) == fk.EINVAL and h.kernels() == []

    for C in (Gated, Narrow, Grad, Products, Adapters):
        for _ in range(300):
            kw = dict(count=rng.choice([1, 2, 64, 1000]), rank=rng.choice([1, 4, 8, 31, 64, 256])) \
                if C is Adapters else {}
            check(C(h, t=rng.choice(sizes), d=rng.choice(sizes), f=rng.choice(sizes),
                    shift=rng.choice([0, 0, 4, 8, 12]), **kw))
    for C in (Heads, HeadsGrad):
        for _ in range(300):
            hd = rng.choice([1, 2, 8, 33, 64, 80, 96, 128, 256, 500, 512])
            check(C(h, t=rng.choice(sizes), hq=rng.choice([1, 3, 32, 200]), hkv=rng.choice([1, 2, 8]), hd=hd,
                    rd=rng.choice([0, hd // 2 // 2 * 2, hd // 2 * 2]), shift=rng.choice([0, 0, 8])))
    seen = set()
    for t, d, f in [(1, 4096, 11008), (67, 5120, 13824), (4096, 4096, 11008), (333, 1000, 2731), (64, 8192, 64)]:
        for C in (Gated, Products):
            h.rt.rt_reset()
            assert C(h, t=t, d=d, f=f)() == fk.OK
            seen |= {re.sub(r".*12_GLOBAL__N_1\d+(\w+?_kernel).*", r"\1", k) for k, _ in h.kernels()}
    assert {"few_kernel", "mm_kernel", "mm_pair_kernel", "mm_sum_kernel", "pad_kernel"} <= seen, seen
    # the longest batches: refused or launched, never a grid the runtime does not take
    for t, d, f in itertools.product([1 << 20, (1 << 31) - 1], [1, 64, 512], [1, 64, 256]):
        for C in (Gated, Narrow, Grad, Products, Adapters):
            h.rt.rt_reset()
            assert C(h, t=t, d=d, f=f)() in (fk.OK, fk.ESHAPE), (C.name, t, d, f, h.error())
    for t in (1 << 20, (1 << 31) - 1):
        for C in (Heads, HeadsGrad):
            h.rt.rt_reset()
            assert C(h, t=t)() in (fk.OK, fk.ESHAPE), (C.name, t, h.error())


def empty(h):
    """An empty batch launches nothing but what writes sums over its rows."""
    for C in CALLS:
        call = C(h, t=0)
        h.rt.rt_reset()
        assert call() == fk.OK, (call.name, h.error())
        got = [k for k, _ in h.kernels()]
        if C is Products:
            assert len(got) == 1 and "mm_" in got[0], got
        elif C is HeadsGrad:
            assert len(got) == 1 and "gains_kernel" in got[0], got
        else:
            assert got == [], (call.name, got)
    # with no addresses at all, as an empty tensor has none
    assert Gated(h, t=0)(X=0, H=0, P=0) == fk.OK
    assert Products(h, t=0)(dP=0, X=0, dX=0) == fk.OK
    assert Adapters(h, t=0)(C=0, X=0, index=0, Y=0) == fk.OK
    assert Heads(h, t=0)(C=0, pos=0, q=0, k=0, v=0) == fk.OK
    assert HeadsGrad(h, t=0)(dq=0, dk=0, dv=0, C=0, pos=0, dC=0) == fk.OK


def failures(h):
    """A launch that fails ends the call with its status; the kernels after it do not run, and the
    next call is whole again."""
    for call in (Gated(h, t=700, d=8192, f=64), Gated(h, t=700, d=255, f=99), Narrow(h), Grad(h),
                 Products(h, t=99, d=64, f=1500), Products(h, t=99, d=65, f=1501), Adapters(h),
                 Adapters(h, t=1, d=1, f=1, count=1, rank=1), Heads(h), HeadsGrad(h)):
        h.rt.rt_reset()
        assert call() == fk.OK
        names = [k for k, _ in h.kernels()]
        for k in dict.fromkeys(names):
            h.rt.rt_fail_kernel(k.encode())
            assert call() == fk.ENOMEM, (call.name, k)
            got = [n for n, _ in h.kernels()]
            assert got == names[:names.index(k) + 1], (call.name, k, got)
            assert call() == fk.OK
            assert [n for n, _ in h.kernels()] == names


def overlaps(h):
    """An output or workspace over an input or over another output is refused."""
    outs = {"H", "P", "dP", "dPt", "dX", "dW", "Y", "q", "k", "v", "dC", "dgq", "dgk", "ws"}
    inputs = {"fpsketch_gated_narrow": {"P"}, "fpsketch_gated_grad": {"P"}, "fpsketch_gated_products": {"dP"}}
    for C in CALLS:
        call = C(h, t=100)
        names = pointers(call)
        for o in names:
            if o not in outs or o in inputs.get(call.name, ()) or (o == "ws" and call.need() == 0):
                continue
            for p in names:
                if p == o or p == "ws":
                    continue
                h.rt.rt_reset()
                assert call(**{o: call.a[p]}) == fk.EINVAL, (call.name, o, p)
                assert re.search("overlap", h.error()), h.error()
                assert h.kernels() == []


if __name__ == "__main__":
    globals()[sys.argv[2]](Host(sys.argv[1]))
