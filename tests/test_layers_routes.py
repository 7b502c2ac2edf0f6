"""Which kernels the sizes of ROUTES launch, on the CPU: the built library on the stand-in for the HIP runtime,
as in test_layers_host.py, in a process of its own.  test_gpu_layers_paths.py compares these calls with exact
results, so a rule that changes must not take the kernels for any alignment out of its reach."""
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
for p in (ROOT, os.path.dirname(os.path.abspath(__file__))):
    if p not in sys.path:
        sys.path.insert(0, p)

from paper_2609_19758_amd import fpsketch as fk  # noqa: E402
from test_layers_host import Adapters, Gated, HeadsGrad, Host, Products, runtime  # noqa: E402,F401

# t, d, f, elements that every operand is shifted by in its buffer, kernels.  Operands off 16-byte groups of more
# than 2^22 elements with little work each go through registers, and those with an operand of fewer than 8
# elements besides, an output a thread.
GATED = [(20, 4095, 4096, 0, {"mm_ragged"}), (8, 7510, 1276, 0, {"mm_ragged"}), (130, 4096, 2100, 2, {"mm_ragged"}),
         (100, 6003, 401, 0, {"mm_ragged"}), (1, 7, 400000, 0, {"tiny"}), (1, 7, 400001, 2, {"tiny"})]
PRODUCTS = [(50, 1555, 4608, 0, {"mm_ragged", "mm"}), (972, 64, 2546, 0, {"mm_ragged"}),
            (200, 4100, 600, 2, {"mm_ragged", "mm"}), (7, 1, 700001, 0, {"mm_ragged", "tiny"}),
            (1, 1000001, 3, 0, {"tiny", "mm"})]
# t, k, n, count, rank
ADAPTERS = [(1100, 257, 200, 5, 12, {"shrink_ragged", "expand"}), (1100, 257, 200, 5, 31, {"shrink_ragged", "expand"}),
            (1100, 257, 203, 5, 64, {"shrink_ragged", "expand"}), (2100, 192, 4100, 3, 128, {"shrink", "expand"})]
# t, hq, hkv, hd, rd: more tokens than work-groups (4 for each of 256 compute units)
GAINS = [(2500, 4, 2, 128, 64, {"heads_grad_vec", "gains"}), (2500, 3, 1, 33, 20, {"heads_grad", "gains"}),
         (2500, 2, 2, 80, 20, {"heads_grad", "gains"}), (2300, 1, 1, 512, 512, {"heads_grad_vec", "gains"})]


@pytest.mark.parametrize("scenario", ["routes", "apart", "registers"])
def test_launches(runtime, scenario):  # noqa: F811
    env = dict(os.environ, PYTHONPATH=ROOT)
    res = subprocess.run([sys.executable, os.path.abspath(__file__), runtime, scenario],
                         capture_output=True, text=True, timeout=100, env=env)
    assert res.returncode == 0, res.stdout + res.stderr


# ---- in the process of its own -------------------------------------------------------------


def launched(h, call):
    h.rt.rt_reset()
    assert call() == fk.OK, (call.name, h.error())
    return [(re.sub(r".*12_GLOBAL__N_1\d+(\w+?)_kernel.*", r"\1", k), g) for k, g in h.kernels()]


def routes(h):
    for C, shapes in ((Gated, GATED), (Products, PRODUCTS)):
        for t, d, f, shift, want in shapes:
            got = {k for k, _ in launched(h, C(h, t=t, d=d, f=f, shift=2 * shift))}
            assert got - {"pad", "mm_sum"} == want, (C.name, t, d, f, shift, got)
    for t, k, n, count, rank, want in ADAPTERS:
        got = dict(launched(h, Adapters(h, t=t, d=k, f=n, count=count, rank=rank)))
        assert set(got) == want, (t, k, n, got)
    # the last one: a work-group takes several blocks of 128 columns
    assert got["expand"] < -(-t // 32) * -(-n // 128), got
    for t, hq, hkv, hd, rd, want in GAINS:
        got = launched(h, HeadsGrad(h, t=t, hq=hq, hkv=hkv, hd=hd, rd=rd))
        assert {k for k, _ in got} == want and got[0][1] < t, (t, hd, got)


def apart(h):
    """A product that does not share its launch is cut for the whole chip: dX in as many parts as it takes to
    give 256 compute units a work-group each (at most 32, of at least 4 steps of 64 k), whatever dW's size."""
    for t, d, f in [(7, 1, 700001), (50, 1555, 4608), (200, 4101, 600), (972, 64, 2546)]:
        got = [(k, g) for k, g in launched(h, Products(h, t=t, d=d, f=f)) if k in ("mm", "mm_ragged")]
        tiles, steps = -(-t // 128) * -(-d // 128), -(-2 * f // 64)
        if got[0][0] == "mm_ragged":
            most = min(32, steps // 4)
            assert got[0][1] >= min(256, tiles * most) * 3 // 4, (t, d, f, got, tiles, steps)


def registers(h):
    """A product through registers, whose steps are mostly waiting, gives every compute unit two work-groups where
    K has the steps for it."""
    for t in (20, 50, 100, 130):
        got = launched(h, Gated(h, t=t, d=4095, f=4096))
        assert got[0][0] == "mm_ragged" and 448 <= got[0][1] <= 512, (t, got)


if __name__ == "__main__":
    globals()[sys.argv[2]](Host(sys.argv[1]))
