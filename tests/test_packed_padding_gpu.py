"""Bytes of a row of scales that are not in use (4 or 8 bytes, of which the first D / 16 are) change nothing, whatever
they hold: no call writes them, and a cache need not begin as zeros."""
import pytest
import torch

from test_packed_gpu import B, BF, F32, att_of, causal, check, i32, make, spread_rows  # noqa: F401 (B: a fixture)

pytestmark = pytest.mark.gpu


def padded(x, fill):
    """Another cache with the same entries, its unused bytes of scales filled."""
    used = x["q"].shape[-1] // 16
    cache = {n: t.clone() for n, t in x["cache"].items()}
    for n in ("k_scales", "v_scales"):
        rest = cache[n][..., used:]
        if fill == "random":
            g = torch.Generator().manual_seed(7)
            rest.copy_(torch.randint(0, 256, rest.shape, dtype=torch.uint8, generator=g))
        else:
            rest.fill_(fill)
    return cache


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("D", [16, 32, 48, 80, 96, 112])
@pytest.mark.parametrize("L, Hq, Hkv, Pn", [(1, 2, 2, 0), (1, 8, 2, 70), (3, 6, 2, 0), (4, 8, 2, 70), (7, 4, 1, 0), (20, 8, 2, 70)])
def test_attention_does_not_read_them(B, L, Hq, Hkv, Pn, D, dt):
    lens = [200, 37, 0, 130]
    x = make(4, L, Hq, Hkv, D, Pn, 200, dt, lens, causal(lens, L))
    att, r = check(B, x, 200)
    for fill in (255, 248, 227, "random"):
        again = att.attend(x["q"], x["kp"], x["vp"], padded(x, fill), x["lens"], visible=x["vis"])
        assert torch.equal(again["out"], r["out"]) and torch.equal(again["lse"], r["lse"]), fill


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("heads", [4, 8])
def test_units_of_several_heads_do_not_read_them(B, heads, dt):
    lens = [(37 * i) % 300 for i in range(80)]
    x = make(80, 1, heads, heads, 80, 0, 300, dt, lens)
    att, r = check(B, x, 300)
    again = att.attend(x["q"], None, None, padded(x, 255), x["lens"])
    assert torch.equal(again["out"], r["out"]) and torch.equal(again["lse"], r["lse"])


@pytest.mark.parametrize("D", [16, 48, 80, 112])
def test_a_cache_that_did_not_begin_as_zeros(B, D):
    """Written, attended over and read back, in memory that held anything."""
    x = make(2, 3, 4, 2, D, 0, 60, BF, [60, 41])
    rows = [spread_rows((2, 60, 2, D), BF, i).clamp(-4, 4).cuda() for i in range(2)]
    att, got = att_of(B, x, 60), []
    for fill in (0, 255):
        cache = {n: torch.full_like(t, fill) for n, t in x["cache"].items()}
        att.store(cache, *rows, i32([0, 0]))
        got.append((att.attend(x["q"], None, None, cache, x["lens"]), att.load(cache, 60, i32([0, 0]))))
        assert att.device_status() == B.OK
    for a, b in zip(*got):
        for n in a:
            assert torch.isfinite(a[n]).all() and torch.equal(a[n], b[n]), n
