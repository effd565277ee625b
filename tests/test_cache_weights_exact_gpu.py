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


def test_bf16_weights_do_not_lean_to_one_side(B):
    """Scores of 128 positive products, of which every other is small, so that sums have more bits than fp32
    holds: eight partial sums of about 16, 32, .. 130, each cut off towards zero by half a unit in the last place on
    average, which is 2.8e-5 in all (2^-20 + 2 x 2^-19 + 4 x 2^-18 + 2^-17, the unit of 64 to 128 being 2^-17) and as much of
    a weight. With the log-sum taken off half-way, four sums above zero lose 2^-20 + 2 x 2^-19 + 2^-18 = 8.6e-6 of
    one sign and the others about as much of the other; that half of it is left over (scores are 130 +- 7, log-sums 5 to
    20 above) is 4.3e-6. To this come sums of `rows` terms and the exponential."""
    Bn, L, G, Hkv, D, S = 2, 8, 4, 2, 128, 1000
    g = torch.Generator().manual_seed(0)
    q, k = torch.rand(Bn, L, Hkv * G, D, generator=g) + 0.5, torch.rand(Bn, S, Hkv, D, generator=g) + 0.5
    for t in (q, k):
        t[..., 1::2] /= 4
    q[..., ::2] *= 2
    q, k = q.bfloat16(), k.bfloat16()
    s = torch.einsum("blhgd,bshd->blhgs", q.view(Bn, L, Hkv, G, D).double(), k.double())
    lse = torch.logsumexp(s, 4).view(Bn, L, Hkv * G).float().cuda()
    lens = torch.tensor([S, S - 1], dtype=torch.int32).cuda()
    q, k = q.cuda(), k.cuda()
    att = B.PrefixAttention(Bn, L, Hkv * G, Hkv, D, 0, S, torch.bfloat16)
    got = n64(att.weights(q, lse, k, lens, scale=1.0))
    assert att.device_status() == B.OK
    want, _ = C.weights(n64(q), n64(lse), n64(k), n64(lens), None, 1.0, None, 1.0)
    tol = 4.3e-6 + (L * G + 4) * U + 2.0 ** -21
    assert abs(got.sum() / want.sum() - 1) <= tol
    assert np.linalg.norm(got - want) <= tol * np.linalg.norm(want)
