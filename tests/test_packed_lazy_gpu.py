"""Caches whose memory another tensor still shares until one of them is written (lazy clones)."""
import pytest
import torch

from test_packed_gpu import B, BF, F32, i32, spread_rows  # noqa: F401 (B: a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("usual", [True, False])
def test_storing_to_a_lazy_clone_leaves_its_source(B, usual, dt):
    if not hasattr(torch, "_lazy_clone"):
        pytest.skip("this torch has no lazy clones")
    att = B.PackedAttention(2, 1, 2, 2, 64, 0, 30, dt)
    source, want = att.alloc_cache(), att.alloc_cache()
    cache = {n: torch._lazy_clone(t) for n, t in source.items()}
    k, v = (spread_rows((2, 9, 2, 64), dt, i).cuda() for i in range(2))
    stream = None if usual else torch.cuda.current_stream()
    att.store(cache, k, v, i32([3, 21]), stream=stream)
    att.store(want, k, v, i32([3, 21]), stream=stream)
    for n in want:
        assert torch.equal(cache[n], want[n]) and want[n].any(), n
        assert not source[n].any(), n


def test_reading_a_lazy_clone(B):
    att = B.PackedAttention(1, 1, 2, 2, 32, 0, 12, BF)
    cache = att.alloc_cache()
    k, v = (spread_rows((1, 12, 2, 32), BF, i).clamp(-4, 4).cuda() for i in range(2))
    att.store(cache, k, v, i32([0]))
    if not hasattr(torch, "_lazy_clone"):
        pytest.skip("this torch has no lazy clones")
    lazy = {n: torch._lazy_clone(t) for n, t in cache.items()}
    q = torch.randn(1, 1, 2, 32).to(BF).cuda()
    for call in (lambda c: att.load(c, 12, i32([0])), lambda c: att.attend(q, None, None, c, i32([12]))):
        a, b = call(cache), call(lazy)
        for n in a:
            assert torch.equal(a[n], b[n])
