"""The forms that a size takes, named: the prefix's own kernel with every order, mask and kind of entry, the ring of
the fp32 form for few rows at its edges, and sums of weights in place. Which form a size takes is worked out from the
constants in the sources, so that a border that moves cannot leave a form without a test."""
import os
import re

import pytest
import torch

from test_cache_gpu import BF, F32
from test_cache_work_gpu import check, inputs, lens_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2609_33390_gb300 import build
    build.build()
    from paper_2609_33390_gb300 import brisk as B
    return B


def constant(name):
    from paper_2609_33390_gb300 import build
    with open(os.path.join(build.CSRC, "cache.cuh")) as f:
        text = f.read()
    value = re.search(r"\b%s = ([^,;]+)[,;]" % name, text)[1]
    return eval(value, {"CACHE_SMS": 152}) if "CACHE_SMS" in value else int(value)


def apart(size):
    """Whether the prefix has a kernel of its own."""
    Bn, L, Hq, Hkv, D, P, S = size
    R = Bn * L * Hq // Hkv
    units = Hkv * -(-R // constant("PAIR_ROWS")) * -(-P // constant("TC_KT"))
    tiles = -(-S // constant("TC_KT"))
    border = "" if tiles <= constant("JOIN_PARTS") else "_SOME" if tiles <= constant("SOME_TILES") else "_LONG"
    return R > constant("SLOT_ROWS") and units >= constant("APART_UNITS" + border)


def attend(att, x, **how):
    return att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"], visible=x["vis"], **how)


# 594 rows a head: the third tile's second slot has none
ORDERS = (6, 33, 24, 8, 128, 6500, 260)
# own entries of a row: none, one part, two, or more
LONG = (40, 16, 64, 32, 72, 2940, 3000)


def long_inputs(mask, seed=0):
    lens = [0 if i % 3 == 0 else 50 + 9 * i for i in range(40)]
    lens[17] = 3000                                    # 24 tiles, about 10 a CTA
    return inputs(*LONG, lens, mask, BF, seed=seed), lens


@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("order", ["token", "head", "fused"])
def test_the_prefixs_own_kernel_in_all_orders(B, order, mask):
    assert apart(ORDERS) and 0 < 6 * 33 * 3 % 256 <= 128
    check(B, inputs(*ORDERS, lens_of(6, 260), mask, BF, order=order), 260)


@pytest.mark.parametrize("mask", [False, True])
def test_the_prefixs_own_kernel_joins_none_to_many_own_parts(B, mask):
    assert apart(LONG)
    x, _ = long_inputs(mask)
    check(B, x, LONG[6])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_hidden_entries_beside_the_prefixs_own_kernel(B, bad):
    """Entries that a row does not see change none of its bits; what a row sees reaches it."""
    assert apart(LONG)
    x, lens = long_inputs(False)
    Bn, L = LONG[:2]
    x["vis"] = (x["lens"][:, None] - L + 1 + torch.arange(L, device="cuda")).clamp(min=0).int()   # causal
    x["vis"][5, 3] = x["vis"][17, 9] = -1
    att = B.PrefixAttention(*LONG, BF)
    ref = {k: v.clone() for k, v in attend(att, x).items()}
    used = torch.arange(LONG[6], device="cuda")[None] < x["lens"][:, None]
    for k in ("ko", "vo"):
        x[k][~used] = bad
    got = attend(att, x)
    assert all(torch.equal(got[k], ref[k]) for k in ref)
    # the newest entry, which the last position alone sees: a value's column, where own entries have one, two and more
    # parts, and a key
    for b in (1, 2, 17, 38):
        x["vo"][b, lens[b] - 1, :, 3] = bad
    x["ko"][4, lens[4] - 1] = bad
    got = attend(att, x)
    keep = torch.ones(ref["out"].shape, dtype=torch.bool, device="cuda")
    for b in (1, 2, 17, 38):
        keep[b, -1, :, 3] = False
    keep[4, -1] = False
    assert torch.equal(got["out"][keep], ref["out"][keep])
    rows = keep.any(3)
    assert torch.equal(got["lse"][rows], ref["lse"][rows])
    assert not torch.isfinite(got["out"][[1, 2, 17, 38], -1, :, 3]).any()
    assert att.device_status() == B.OK


def test_bad_entries_of_the_prefix_reach_all_rows_but_padding(B):
    assert apart(LONG)
    x, _ = long_inputs(True)
    att = B.PrefixAttention(*LONG, BF)
    ref = {k: v.clone() for k, v in attend(att, x).items()}
    pad = (x["vis"] < 0)[..., None]
    value = x["vp"][200, 5, 7].clone()
    x["vp"][200, 5, 7] = float("nan")                  # key head 5: query heads 10 and 11
    got = attend(att, x)
    hit = torch.zeros_like(ref["out"], dtype=torch.bool)
    hit[:, :, 10:12, 7] = ~pad
    assert torch.equal(got["out"][~hit], ref["out"][~hit]) and torch.equal(got["lse"], ref["lse"])
    assert torch.isnan(got["out"][hit]).all()
    x["vp"][200, 5, 7] = value
    x["kp"][2939] = float("nan")
    got = attend(att, x)
    gone = pad.expand_as(got["lse"])
    assert torch.isnan(got["lse"][~gone]).all() and torch.isnan(got["out"][~gone]).all()
    assert torch.isneginf(got["lse"][gone]).all() and (got["out"][gone] == 0).all()


def test_two_prefix_kernels_on_two_streams(B):
    sizes = [(20, 16, 32, 8, 128, 4000, 300), (70, 1, 32, 8, 128, 29200, 800)]
    assert all(apart(s) for s in sizes)
    xs = [inputs(*s, lens_of(s[0], s[6]), True, BF, seed=i) for i, s in enumerate(sizes)]
    atts = [B.PrefixAttention(*s, BF) for s in sizes]
    streams = [torch.cuda.Stream() for _ in sizes]
    alone = [attend(a, x) for a, x in zip(atts, xs)]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [[attend(a, x, stream=s) for _ in range(3)] for a, x, s in zip(atts, xs, streams)]
        torch.cuda.synchronize()
        for a, rs in zip(alone, got):
            assert all(torch.equal(a[k], r[k]) for r in rs for k in a)
    assert all(a.device_status() == B.OK for a in atts)


def test_a_captured_call_of_all_three_kernels_replays_on_new_inputs(B):
    assert apart(ORDERS)
    x, y = (inputs(*ORDERS, lens_of(6, 260, step), True, BF, seed=s) for s, step in ((0, 37), (1, 53)))
    att = B.PrefixAttention(*ORDERS, BF)
    out = {k: torch.zeros_like(v) for k, v in attend(att, x).items()}
    torch.cuda.synchronize()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        attend(att, x, out=out, stream=s)
    want = {k: v.clone() for k, v in attend(att, y).items()}
    for k in x:
        x[k].copy_(y[k])
    for _ in range(3):
        for v in out.values():
            v.fill_(7)
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], want[k]) for k in want)
    assert att.device_status() == B.OK


@pytest.mark.parametrize("size", [(16, 32, 32, 8, 128, 3000, 250), (80, 8, 16, 4, 64, 6000, 200)])
def test_expired_waits_of_the_prefixs_own_kernel(B, size):
    assert apart(size)
    x = inputs(*size, lens_of(size[0], size[6]), True, BF)
    att = B.PrefixAttention(*size, BF)
    ref = {k: v.clone() for k, v in attend(att, x).items()}
    assert att.device_status() == B.OK
    before = B.set_wait_limit(1)
    try:
        attend(att, x)
        assert att.device_status() == B.ERR_TIMEOUT
    finally:
        B.set_wait_limit(before)
    got = attend(att, x)
    assert att.device_status() == B.OK and all(torch.equal(got[k], ref[k]) for k in ref)


@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("size", [
    (5, 32, 32, 8, 128, 9000, 600),       # several row tiles a head, the last one half full
    (40, 8, 16, 4, 64, 4000, 250),        # narrow heads, 5 row tiles
    (40, 8, 12, 4, 40, 5000, 90),
    (40, 16, 64, 32, 72, 384, 0),         # no own entries
    (300, 1, 32, 8, 128, 4096, 150),      # single tokens
    (1025, 1, 16, 8, 64, 1300, 20),
])
def test_the_prefixs_own_kernel_of_many_sizes(B, size, mask):
    assert apart(size)
    check(B, inputs(*size, lens_of(size[0], size[6]), mask, BF), size[6])


# ---------------------------------------------------------------- fp32, up to 8 rows of a sequence

@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("D", [128, 64, 40])
@pytest.mark.parametrize("L,G", [(1, 2), (1, 3), (2, 2), (1, 7), (4, 2)])      # forms of 2, 4 and 8 rows
@pytest.mark.parametrize("steps,S", [
    (1, 64),                              # a tile a CTA: one step of a warp, or none where the tile ends before its keys
    (2, 128),                             # all three places of the ring
    (3, 190),                             # places used again
    (6, 383),
])
def test_the_ring_of_few_rows(B, steps, S, L, G, D, mask):
    """Whole sequences a CTA (their number keeps all CTAs busy), of which the last tile holds 1 to 64 keys."""
    kt, ctas = constant("SIMT_KT"), 2 * 152
    Hkv, Bn = 4, 76
    assert L * G <= constant("FEW_ROWS") and -(-(Bn * Hkv * -(-S // kt)) // ctas) == steps
    full = S - S % kt if S % kt else S - kt
    lens = [full + 1 + (i * 9) % (S - full) if i % 5 else S for i in range(Bn)]
    lens[7], lens[8], lens[9] = full + 8, min(S, full + 9), 5
    size = (Bn, L, G * Hkv, Hkv, D, 0, S)
    check(B, inputs(*size, lens, mask, F32), S)


# ---------------------------------------------------------------- weights

@pytest.mark.parametrize("dt,L,S", [(BF, 75, 9000), (BF, 140, 4200), (BF, 8, 700), (F32, 20, 700), (F32, 3, 700)])
def test_sums_of_weights_in_place(B, dt, L, S):
    """More than 256 rows a head: later passes read what earlier ones wrote to the sums."""
    Bn, Hq, Hkv, D = 3, 16, 4, 128
    x = inputs(Bn, L, Hq, Hkv, D, 0, S, [S, S // 2 + 3, 0], True, dt)
    att = B.PrefixAttention(Bn, L, Hq, Hkv, D, 0, S, dt)
    lse = attend(att, x)["lse"]
    acc = torch.rand(Bn, Hkv, S, device="cuda")
    want = att.weights(x["q"], lse, x["ko"], x["lens"], acc=acc, decay=0.7, visible=x["vis"])
    got = acc.clone()
    att.weights(x["q"], lse, x["ko"], x["lens"], acc=got, decay=0.7, visible=x["vis"], out=got)
    assert torch.equal(got, want) and att.device_status() == B.OK
