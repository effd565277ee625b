"""Scales of 0 and next to it, with scores whose size shows a scale that is not the one given; tolerances as
derived in test_cache_gpu.py."""
import numpy as np
import pytest
import torch

from oracle import cache as C
from test_cache_gpu import BF, F32, U, att_of, compare_attend, make, n64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2609_33390_gb300 import build
    build.build()
    from paper_2609_33390_gb300 import brisk as B
    return B


def inputs(dt, L=3, Hq=4):
    """Scores up to 64 x 1e18 x 4e18 = 2.6e38."""
    x = make(2, L, Hq, 2, 64, 200, 150, dt, [150, 9])
    x["q"].fill_(1e18)
    for k in ("kp", "ko"):
        x[k].clamp_(-1, 1).mul_(4e18)
    return x


# 0: the same weight for all; 1e-39: scores up to 0.3, by a scale that is subnormal in fp32
@pytest.mark.parametrize("scale", [0.0, 1e-39])
@pytest.mark.parametrize("dt", [BF, F32])
def test_scales_next_to_0(B, dt, scale):
    x = inputs(dt)
    att = att_of(B, x, 150)
    r = att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"], scale=scale)
    exact = float(np.float32(scale))
    want = C.attend(*(n64(x[k]) for k in ("q", "kp", "vp", "ko", "vo", "lens")), None, exact)
    compare_attend(r, *want, dt, 64, 350)
    acc = n64(att.weights(x["q"], r["lse"], x["ko"], x["lens"], scale=scale))
    sums, big = C.weights(n64(x["q"]), n64(r["lse"]), n64(x["ko"]), n64(x["lens"]), None, exact, None, 1.0)
    top = np.abs(n64(r["lse"])).max()
    rel = (2 * 64 + 16) * U * big + 2.0 ** -21 + 4 * U * top + (6 + 4) * U
    assert (np.abs(acc - sums) <= rel * sums + 1e-30).all()
    assert att.device_status() == B.OK
