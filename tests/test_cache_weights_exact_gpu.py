"""fp32 attention weights where scores are large and exact: what is lost is in the subtraction of the log-sums alone.

Queries and keys are small whole numbers, so that products and sums are exact, and the scale is 1/4. Scores are
about 512, log-sums some 6 above, differences d down to -25. A weight's relative error is then that of d (half a
unit in the last place: u |d|, u = 2^-24), of its way to log2 units (u |d| for the product, u |d| / 2 for the
constant), the hardware exponential's (2^-22), and that of the sum
of `rows` terms: 3 u |d| + 2^-21 + (rows + 4) u."""
import numpy as np
import pytest
import torch

from oracle import cache as C
from test_cache_gpu import F32, U, n64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2609_33390_gb300 import build
    build.build()
    from paper_2609_33390_gb300 import brisk as B
    return B


@pytest.mark.parametrize("L,G", [
    (1, 4), (3, 4), (8, 4),               # up to 32 rows a head
    (16, 4), (9, 5),                      # tiles
])
def test_fp32_weights_of_large_scores_keep_their_bits(B, L, G):
    Bn, Hkv, D, S, scale, dt = 2, 2, 64, 150, 0.25, F32
    g = torch.Generator().manual_seed(L)
    q = torch.randint(-2, 3, (Bn, L, Hkv * G, D), generator=g).float()
    k = torch.randint(-1, 2, (Bn, S, Hkv, D), generator=g).float()
    q[..., :32], k[..., :32] = 8, 8
    s = scale * torch.einsum("blhgd,bshd->blhgs", q.view(Bn, L, Hkv, G, D).double(), k.double())
    assert s.min() > 480 and s.max() < 540
    lse = torch.logsumexp(s, 4).view(Bn, L, Hkv * G).float()
    d = float((s - lse.view(Bn, L, Hkv, G, 1).double()).abs().max())
    assert d < 40
    lens = torch.tensor([150, 131], dtype=torch.int32)
    q, k, lse, lens = q.to(dt).cuda(), k.to(dt).cuda(), lse.cuda(), lens.cuda()
    att = B.PrefixAttention(Bn, L, Hkv * G, Hkv, D, 0, S, dt)
    got = n64(att.weights(q, lse, k, lens, scale=scale))
    assert att.device_status() == B.OK
    want, _ = C.weights(n64(q), n64(lse), n64(k), n64(lens), None, scale, None, 1.0)
    rel = 3 * U * d + 2.0 ** -21 + (L * G + 4) * U
    assert (np.abs(got - want) <= rel * want).all(), np.max(np.abs(got - want) / np.maximum(want, 1e-30)) / rel
