"""What attention over caches in 4 bits rounds, at the bounds that brisk.h states: a weight by 2^-11 of itself (fp32: 2^-22) or
2^-35 of the row's largest weight, a query's channel by 2^-23 of itself (bf16: by nothing) or 2^-39 of the largest of its row.

Scores here are one product, exact before the multiplication by the scale in log2 units: that and its constant cost
2^-25 and the addition of the maximum half a unit in the last place of numbers below 64 (2^-19), the exponential
2^-22: eps = 2^-18 in all. Sums of n terms cost 2 n u (u = 2^-24), the result's rounding 2^-24 (bf16: 2^-8)."""
import numpy as np
import pytest
import torch

from oracle import packed as P
from test_packed_gpu import B, BF, F32, U, i32, n64, raw  # noqa: F401 (B: a fixture)

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -18
ROWS = [1, 6, 40]


def one_channel(B, rows, keys, values, dt):
    """An object, and a cache of entries whose first two channels are `keys` [n, 2] and whose values are `values` [n], as far as
    the format holds them; what it holds."""
    n = len(keys)
    att = B.PackedAttention(1, rows, 1, 1, 16, 0, n, dt)
    k, v = torch.zeros(1, n, 1, 16), torch.zeros(1, n, 1, 16)
    k[0, :, 0, :2] = torch.tensor(keys)
    v[0, :, 0] = torch.tensor(values)[:, None]
    cache = att.store(att.alloc_cache(), k.to(dt).cuda(), v.to(dt).cuda(), i32([0]))
    return att, cache, P.values(*raw(cache, "k"))[0, :, 0, :2], P.values(*raw(cache, "v"))[0, :, 0, 0]


def check(r, s, v, dt, eps, floor):
    """r: a call's results, s [rows, n]: scores, v [n]; eps [rows, 1] of a score, floor of a weight beside the largest."""
    n = s.shape[1] + 16
    top = s.max(1, keepdims=True)
    w = np.exp(s - top)
    z = w.sum(1, keepdims=True)
    out, mass = (w @ v)[:, None] / z, (w @ np.abs(v))[:, None] / z
    each = 2.0 ** -22 if dt == F32 else 2.0 ** -11
    tol = (np.expm1(2 * eps) + each + 2 * n * U) * mass + floor * np.abs(v).sum() / z
    tol = tol + (2.0 ** -24 if dt == F32 else 2.0 ** -8) * (np.abs(out) + tol)
    assert (np.abs(n64(r["out"])[0, :, 0] - out) <= tol).all()
    lse = (top + np.log(z))[:, 0]
    assert (np.abs(n64(r["lse"])[0, :, 0] - lse) <= eps[:, 0] + n * U + 2.0 ** -22 * np.abs(lse)).all()


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("rows", ROWS)
def test_small_weights_beside_a_large_one(B, rows, dt):
    """One entry has nearly all the weight, and a value of 0; many others have 2^-13 to 2^-35 of it each."""
    for down in (9.0, 12.0, 13.5, 15.0, 16.5, 18.0, 19.5, 21.0, 22.5, 24.0):
        att, cache, k, v = one_channel(B, rows, [[0.0, 0.0]] + [[-down, 0.0]] * 63, [0.0] + [1.0] * 63, dt)
        assert (k[1:, 0] == -down).all()
        q = torch.zeros(1, rows, 1, 16)
        q[..., 0] = 1.0 + torch.arange(rows)[None, :, None] / 128       # (bf16 holds them)
        r = att.attend(q.to(dt).cuda(), None, None, cache, i32([64]), scale=1.0)
        s = n64(q)[0, :, 0, :1] * k[:, 0]
        check(r, s, v, dt, np.full((rows, 1), EPS), 2.0 ** -35)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("below", [8, 16, 20, 24, 28, 31, 33, 35])
def test_small_channels_of_a_query_beside_a_large_one(B, rows, below, dt):
    """The row's largest channel meets keys of 0; the scores are those of one `below` powers of two smaller."""
    keys = [[0.0, (-1) ** i * (0.5 + i % 7)] for i in range(40)]
    att, cache, k, v = one_channel(B, rows, keys, [float(i % 5 - 2) for i in range(40)], dt)
    q = torch.zeros(1, rows, 1, 16)
    q[..., 0] = 1.0
    bits = torch.randint(128, 256, (rows,), generator=torch.Generator().manual_seed(below)).float() / 128
    if dt == F32:
        bits += torch.rand(rows, generator=torch.Generator().manual_seed(below)) / 128
    q[0, :, 0, 1] = bits * 2.0 ** -below
    scale = 2.0 ** (below - 2)
    r = att.attend(q.to(dt).cuda(), None, None, cache, i32([40]), scale=scale)
    x = n64(q.to(dt))[0, :, 0, 1:2]
    off = np.maximum(2.0 ** -23 * x, 2.0 ** -39) if dt == F32 else np.where(x < 2.0 ** -31, 2.0 ** -39, 0.0)
    check(r, x * k[:, 1] * scale, v, dt, EPS + off * np.abs(k[:, 1]).max() * scale, 2.0 ** -35)
