"""Scalars of the operators around a delivered product that the entry points refuse, on the CPU: the built
library on the stand-in for the HIP runtime, as in test_layers_host.py, in a process of its own."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
for p in (ROOT, os.path.dirname(os.path.abspath(__file__))):
    if p not in sys.path:
        sys.path.insert(0, p)

from paper_2609_19758_amd import fpsketch as fk  # noqa: E402
from test_layers_host import Heads, HeadsGrad, Host, runtime  # noqa: E402,F401


@pytest.mark.parametrize("scenario", ["eps"])
def test_values(runtime, scenario):  # noqa: F811
    env = dict(os.environ, PYTHONPATH=ROOT)
    res = subprocess.run([sys.executable, os.path.abspath(__file__), runtime, scenario],
                         capture_output=True, text=True, timeout=100, env=env)
    assert res.returncode == 0, res.stdout + res.stderr


# ---- in the process of its own -------------------------------------------------------------


def eps(h):
    """eps is held in FP32: one that is not zero but below FP32's normal numbers would become zero (a head of
    zeros NaN) or have a reciprocal past FP32, and one above them infinite."""
    for C in (Heads, HeadsGrad):
        for bad in (1e-300, 1e-46, 2.0 ** -127, 2.0 ** -126 * (1 - 2.0 ** -30), 2.0 ** 128, 1e300):
            h.rt.rt_reset()
            assert C(h)(eps=bad) == fk.EINVAL, (C.name, bad)
            assert "eps" in h.error() and h.kernels() == []
            assert C(h)(eps=bad, gq=0, gk=0) == fk.OK            # (no norm: eps is not looked at)
        for good in (0.0, 2.0 ** -126, 1e-12, 1.0, 3e38):
            assert C(h)(eps=good) == fk.OK, (C.name, good, h.error())


if __name__ == "__main__":
    globals()[sys.argv[2]](Host(sys.argv[1]))
