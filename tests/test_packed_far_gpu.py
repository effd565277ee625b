"""Entries whose offsets pass 2^32 bytes, with log-sums that are held from both sides."""
import numpy as np
import pytest
import torch

from oracle import packed as P
from test_packed_gpu import B, BF, F32, U, i32, n64, spread_rows  # noqa: F401 (B: a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt, rows", [(BF, 2), (BF, 12), (BF, 40), (F32, 3)])
def test_log_sums_of_a_cache_beyond_32_bits(B, dt, rows):
    S, D, n = 70000, 128, 40
    big = torch.zeros(S, 65536, dtype=torch.uint8, device="cuda")          # 4.6 GB: a row of codes every 64 KB
    cache = {m: big[None, :, None, o:o + 64] for m, o in (("k", 0), ("v", 1024))}
    cache.update({m + "_scales": big[None, :, None, o:o + 8] for m, o in (("k", 2048), ("v", 4096))})
    att = B.PackedAttention(1, rows, 1, 1, D, 0, S, dt)
    new = {m: spread_rows((1, n, 1, D), dt, i).clamp(-4, 4) for i, m in enumerate("kv")}
    att.store(cache, new["k"].cuda(), new["v"].cuda(), i32([S - n]))
    k, v = (P.values(*P.store(n64(new[m])))[0, :, 0] for m in "kv")
    g = torch.Generator().manual_seed(rows)
    q = (torch.randn(1, rows, 1, D, generator=g) * 4).to(dt)
    r = att.attend(q.cuda(), None, None, cache, i32([S]))
    assert att.device_status() == B.OK
    s = n64(q)[0, :, 0] @ k.T * D ** -0.5
    big_s = (np.abs(n64(q)[0, :, 0]) @ np.abs(k).T).max(1) * D ** -0.5
    top = np.maximum(s.max(1), 0)[:, None]             # (all other entries are zeros: scores of 0)
    w, rest = np.exp(s - top), (S - n) * np.exp(-top)
    z = w.sum(1, keepdims=True) + rest
    lse = (top + np.log(z))[:, 0]
    assert (np.log(S) < lse - 1).any()                 # entries beyond count for something
    eps = (2 * D + 20) * U * big_s + 2.0 ** -21
    assert (np.abs(n64(r["lse"])[0, :, 0] - lse) <= eps + (S + 16) * U + 2.0 ** -22 * np.abs(lse)).all()
    mass, out = w @ np.abs(v) / z, w @ v / z
    each = 2.0 ** -22 if dt == F32 else 2.0 ** -11
    tol = (2 * eps[:, None] + each + 2 * (S + 16) * U) * mass + 2.0 ** -35 * np.abs(v).sum(0) / z
    tol = tol + (2.0 ** -24 if dt == F32 else 2.0 ** -8) * np.abs(out)
    assert (np.abs(n64(r["out"])[0, :, 0] - out) <= tol).all()
