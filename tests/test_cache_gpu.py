"""Attention over a shared prefix and own caches, attention weights and eviction on the GPU against
the float64 oracle.

Tolerances. A score is a sum of D products of stored values in fp32, off by at most about (D + 4) u
times scale * sum |q_d k_d| (u = 2^-24; the products of bf16 values are exact), and scaling and the
hardware exponential add a few u of the score's size: eps = (2D + 16) u big + 2^-21. Sums of n
positive terms in fp32 are off by at most n u relative. lse follows with eps + n u + 2^-22 |lse|;
out with (2 eps + 2 n u) sum p |v|, plus, for bf16, half a unit (2^-9) of every probability and of the
rounded result."""
import math

import numpy as np
import pytest
import torch

from oracle import cache as C

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def B():
    from paper_2609_33390_gb300 import build
    build.build()
    from paper_2609_33390_gb300 import brisk as B
    return B


def n64(t):
    return None if t is None else t.double().cpu().numpy()


def caches(lead, S, Hkv, D, order, dt, g, pad=0):
    """k, v [*lead, S, Hkv, D] as views of token-major, head-major or interleaved memory."""
    n = len(lead)
    rnd = lambda *s: torch.randn(*s, generator=g).to(dt).cuda()
    if order == "fused":
        kv = rnd(*lead, S, 2, Hkv, D + pad)[..., :D]
        return kv.select(n + 1, 0), kv.select(n + 1, 1)
    if order == "head":
        return [rnd(*lead, Hkv, S, D + pad)[..., :D].transpose(n, n + 1) for _ in range(2)]
    return [rnd(*lead, S, Hkv, D + pad)[..., :D] for _ in range(2)]


def make(Bn, L, Hq, Hkv, D, P, S, dt, lens, vis=None, order="token", qpad=0, pad=0, seed=0):
    g = torch.Generator().manual_seed(seed + 1000 * D + 10 * P + S)
    x = {"q": (torch.randn(Bn, L, Hq, D + qpad, generator=g) * 1.5).to(dt).cuda()[..., :D]}
    x["kp"], x["vp"] = caches((), P, Hkv, D, order, dt, g, pad) if P else (None, None)
    x["ko"], x["vo"] = caches((Bn,), S, Hkv, D, order, dt, g, pad) if S else (None, None)
    x["lens"] = torch.tensor(lens, dtype=torch.int32).cuda()
    x["vis"] = None if vis is None else torch.tensor(vis, dtype=torch.int32).cuda()
    return x


def att_of(B, x, S):
    Bn, L, Hq, D = x["q"].shape
    P = 0 if x["kp"] is None else x["kp"].shape[0]
    Hkv = (x["ko"] if x["kp"] is None else x["kp"]).shape[-2]
    return B.PrefixAttention(Bn, L, Hq, Hkv, D, P, S, x["q"].dtype)


def check_attend(B, x, S, want_status=None, att=None):
    att = att or att_of(B, x, S)
    r = att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"], visible=x["vis"])
    assert att.device_status() == (B.OK if want_status is None else want_status)
    out, lse, mass, big = C.attend(n64(x["q"]), n64(x["kp"]), n64(x["vp"]), n64(x["ko"]), n64(x["vo"]),
                                   n64(x["lens"]), n64(x["vis"]), att.scale)
    compare_attend(r, out, lse, mass, big, x["q"].dtype, att.D, att.P + S)
    return att, r, (out, lse, mass, big)


def compare_attend(r, out, lse, mass, big, dt, D, n):
    got_o, got_l = n64(r["out"]), n64(r["lse"])
    eps = (2 * D + 16) * U * big + 2.0 ** -21
    none = np.isneginf(lse)
    assert (np.isneginf(got_l) == none).all()
    assert (got_o[none] == 0).all()
    tol_l = eps + n * U + 2.0 ** -22 * np.abs(np.where(none, 0, lse))
    assert (np.abs(np.where(none, 0, got_l - np.where(none, 0, lse))) <= tol_l).all()
    tol = (2 * eps + 2 * n * U)[..., None] * mass
    if dt == BF:
        tol = tol + 2.0 ** -9 * mass * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(out)
    else:
        tol = tol + 2.0 ** -22 * np.abs(out)
    assert (np.abs(got_o - out) <= tol + 1e-30).all(), np.max(np.abs(got_o - out) / (tol + 1e-30))


def causal(lens, L):
    return [[max(0, n - L + 1 + i) for i in range(L)] for n in lens]


SIZES = [
    # B, L, Hq, Hkv, D, P, S, lens
    (1, 1, 1, 1, 8, 0, 1, [1]),
    (1, 1, 1, 1, 64, 1, 0, [0]),
    (1, 1, 8, 2, 128, 127, 5, [5]),
    (2, 1, 4, 4, 64, 128, 130, [130, 1]),
    (3, 5, 6, 2, 72, 129, 257, [0, 129, 257]),
    (2, 7, 28, 4, 128, 301, 77, [77, 3]),
    (5, 2, 3, 1, 40, 1, 64, [64, 0, 63, 1, 17]),
    (1, 33, 16, 2, 128, 700, 300, [299]),           # 264 rows a key head: a tile and a bit
    (2, 64, 8, 1, 64, 0, 200, [200, 70]),           # 512 rows over own entries alone
    (70, 1, 4, 1, 64, 300, 40, [(7 * i) % 41 for i in range(70)]),   # 280 rows over the prefix
    (4, 3, 5, 5, 120, 64, 128, [128, 128, 64, 65]),
    (2, 4, 24, 8, 128, 2500, 600, [600, 500]),      # keys divided over many CTAs
]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("mask", ["all", "causal"])
@pytest.mark.parametrize("size", SIZES)
def test_attend_matches_oracle(B, size, mask, dt):
    Bn, L, Hq, Hkv, D, P, S, lens = size
    x = make(Bn, L, Hq, Hkv, D, P, S, dt, lens, causal(lens, L) if mask == "causal" else None)
    check_attend(B, x, S)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("order", ["token", "head", "fused"])
@pytest.mark.parametrize("pad", [0, 8])
def test_orders_and_strides(B, order, pad, dt):
    x = make(3, 4, 6, 3, 64, 200, 150, dt, [150, 40, 0], order=order, qpad=pad, pad=pad)
    check_attend(B, x, 150)


@pytest.mark.parametrize("dt", [BF, F32])
def test_query_slice_of_a_fused_projection(B, dt):
    g = torch.Generator().manual_seed(5)
    x = make(2, 3, 8, 2, 64, 90, 60, dt, [60, 33])
    qkv = torch.randn(2, 3, 12, 64, generator=g).to(dt).cuda()
    x["q"] = qkv[:, :, :8]
    check_attend(B, x, 60)
    x["q"] = torch.randn(2, 8, 3, 64, generator=g).to(dt).cuda().transpose(1, 2)
    check_attend(B, x, 60)


@pytest.mark.parametrize("dt", [BF, F32])
def test_rows_that_see_nothing(B, dt):
    vis = [[0, -1, 5, -7], [-1, -1, -1, -1], [3, 0, 0, 900]]
    x = make(3, 4, 4, 2, 64, 0, 140, dt, [140, 100, 0], vis)
    _, r, _ = check_attend(B, x, 140)
    assert torch.isneginf(r["lse"][0, 1]).all() and torch.isneginf(r["lse"][2]).all()
    # with a prefix only padding sees nothing
    x = make(3, 4, 4, 2, 64, 50, 140, dt, [140, 100, 0], vis)
    _, r, _ = check_attend(B, x, 140)
    assert torch.isneginf(r["lse"][1]).all() and torch.isfinite(r["lse"][2]).all()
    # nothing at all anywhere
    x = make(3, 4, 4, 2, 64, 0, 140, dt, [0, 0, 0])
    _, r, _ = check_attend(B, x, 140)
    assert (r["out"] == 0).all() and torch.isneginf(r["lse"]).all()


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("L,G", [(5, 2), (40, 8)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_hidden_entries_do_not_reach_the_rows(B, bad, L, G, dt):
    """Infinities and NaN in entries beyond the lengths, and in entries that some rows see and others
    do not: rows that do not see them are as if they were not there."""
    S, lens = 300, [260, 131, 0]
    vis = causal(lens, L)
    x = make(3, L, 2 * G, 2, 64, 30, S, dt, lens, vis)
    att, r, want = check_attend(B, x, S)
    for b, n in enumerate(lens):
        x["ko"][b, n:] = bad
        x["vo"][b, n:] = bad
    got = att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"], visible=x["vis"])
    for k in ("out", "lse"):
        assert torch.equal(got[k], r[k])
    # the newest entry: only the block's last position sees it
    x["ko"][0, 259] = bad
    x["vo"][1, 130, :, 3] = bad
    got = att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"], visible=x["vis"])
    out, lse, mass, big = (w.copy() for w in want)
    for w, g in ((out, got["out"]), (lse, got["lse"])):
        w[0, -1] = n64(g)[0, -1]                     # sees the bad key: whatever follows from it
    w = n64(got["out"])[1, -1, :, 3]
    assert (~np.isfinite(w)).all()
    out[1, -1, :, 3], mass[1, -1, :, 3] = 0, 0
    got["out"][1, -1, :, 3] = 0
    keep = np.ones(lse.shape, bool)
    keep[0, -1] = False
    sub = {k: got[k].cpu()[torch.from_numpy(keep)] for k in got}
    compare_attend(sub, out[keep], lse[keep], mass[keep], big[keep], dt, 64, 30 + S)


@pytest.mark.parametrize("dt", [BF, F32])
def test_nan_keys_and_queries_that_are_seen_give_nan(B, dt):
    x = make(2, 2, 2, 1, 64, 200, 10, dt, [10, 10])
    x["q"][0, 1, 0] = float("nan")
    att = att_of(B, x, 10)
    r = att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"])
    bad = torch.isnan(r["lse"])
    assert bad[0, 1, 0] and bad.sum() == 1 and torch.isnan(r["out"][0, 1, 0]).all()
    assert torch.isfinite(r["out"]).sum() == r["out"].numel() - 64
    x["q"][0, 1, 0] = 1.0
    x["kp"][77] = float("nan")
    r = att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"])
    assert torch.isnan(r["lse"]).all() and torch.isnan(r["out"]).all()


@pytest.mark.parametrize("dt", [BF, F32])
def test_scores_of_any_size_keep_their_weights(B, dt):
    """Scores far above and below zero, growing and falling along the keys: the running maximum."""
    for sign in (1.0, -1.0):
        x = make(1, 2, 2, 1, 64, 600, 300, dt, [300])
        ramp = sign * torch.linspace(-40, 40, 600).cuda()
        x["q"].fill_(1.0)
        x["kp"].mul_(0.05)
        x["kp"][:, 0, 0] = (ramp * 8).to(dt)
        x["ko"].mul_(0.05)
        x["ko"][0, :, 0, 1] = (sign * torch.linspace(-100, 100, 300) * 8).to(dt).cuda()
        check_attend(B, x, 300)
    # one entry far above all others
    x = make(1, 3, 2, 1, 64, 600, 300, dt, [300])
    x["q"].fill_(2.0)
    x["ko"][0, 211] = 20.0
    check_attend(B, x, 300)


@pytest.mark.parametrize("dt", [BF, F32])
def test_scale(B, dt):
    x = make(2, 2, 4, 2, 64, 100, 100, dt, [100, 9])
    att = att_of(B, x, 100)
    for scale in (0.0, 1.0, 0.01):
        r = att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"], scale=scale)
        want = C.attend(*(n64(x[k]) for k in ("q", "kp", "vp", "ko", "vo", "lens")), None, scale)
        compare_attend(r, *want, dt, 64, 200)


@pytest.mark.parametrize("dt", [BF, F32])
def test_lengths_out_of_range_are_clamped_and_reported(B, dt):
    x = make(2, 2, 4, 2, 64, 40, 60, dt, [75, -3])
    check_attend(B, x, 60, want_status=B.ERR_INVALID_ARG)
    att = att_of(B, x, 60)
    lse = torch.zeros(2, 2, 4, device="cuda")
    att.weights(x["q"], lse, x["ko"], x["lens"])
    assert att.device_status() == B.ERR_INVALID_ARG
    r = att.evict(x["ko"], x["vo"], torch.zeros(2, 2, 60, device="cuda"), x["lens"], 50, 0)
    assert att.device_status() == B.ERR_INVALID_ARG and r["own_len"].tolist() == [50, 0]
    x["lens"].clamp_(0, 60)
    check_attend(B, x, 60, att=att)                  # the next call clears the word


@pytest.mark.parametrize("dt", [BF, F32])
def test_the_same_inputs_give_the_same_bits_on_any_stream(B, dt):
    x = make(6, 9, 8, 2, 128, 900, 400, dt, [400, 1, 37, 250, 0, 399])
    att, r, _ = check_attend(B, x, 400)
    acc = att.weights(x["q"], r["lse"], x["ko"], x["lens"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        again = att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"], stream=s)
        acc2 = att.weights(x["q"], again["lse"], x["ko"], x["lens"], stream=s)
        s.synchronize()
        assert torch.equal(again["out"], r["out"]) and torch.equal(again["lse"], r["lse"])
        assert torch.equal(acc2, acc)


def test_captured_calls_replay_on_new_inputs(B):
    x = make(3, 4, 8, 2, 64, 100, 90, BF, [90, 20, 0], [[1, 2, 3, 4]] * 3)
    y = make(3, 4, 8, 2, 64, 100, 90, BF, [3, 90, 45], [[90] * 4, [-1] * 4, [7, 0, 9, 2]], seed=1)
    att = att_of(B, x, 90)
    out = {"out": torch.zeros(3, 4, 8, 64, dtype=BF, device="cuda"), "lse": torch.zeros(3, 4, 8, device="cuda")}
    acc = torch.zeros(3, 2, 90, device="cuda")
    ev = att.alloc_evicted(30)

    def step(s=None):
        att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"], visible=x["vis"], out=out, stream=s)
        att.weights(x["q"], out["lse"], x["ko"], x["lens"], visible=x["vis"], out=acc, stream=s)
        att.evict(x["ko"], x["vo"], acc, x["lens"], 30, 4, out=ev, stream=s)

    step()
    torch.cuda.synchronize()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        step(s)
    for k in x:
        x[k].copy_(y[k])
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (out["out"], out["lse"], acc, *ev.values())]
    step()
    torch.cuda.synchronize()
    for a, b in zip(got, (out["out"], out["lse"], acc, *ev.values())):
        assert torch.equal(a, b)
    want = C.attend(*(n64(y[k]) for k in ("q", "kp", "vp", "ko", "vo", "lens", "vis")), att.scale)
    compare_attend(out, *want, BF, 64, 190)


# ---------------------------------------------------------------- weights

def check_weights(B, x, S, acc=None, decay=1.0, att=None):
    att = att or att_of(B, x, S)
    r = att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"], visible=x["vis"])
    got = n64(att.weights(x["q"], r["lse"], x["ko"], x["lens"], acc=acc, decay=decay, visible=x["vis"]))
    assert att.device_status() == B.OK
    want, big = C.weights(n64(x["q"]), n64(r["lse"]), n64(x["ko"]), n64(x["lens"]), n64(x["vis"]),
                          att.scale, n64(acc), decay)
    rows = att.L * att.Hq // att.Hkv
    # a weight is off by the score's and the log-sum's rounding, relative; the sum by its terms' number
    top = np.abs(np.where(np.isneginf(n64(r["lse"])), 0, n64(r["lse"]))).max()
    rel = (2 * att.D + 16) * U * big + 2.0 ** -21 + 4 * U * top + (rows + 4) * U
    assert (np.abs(got - want) <= rel * np.abs(want) + 1e-30).all()
    for b in range(att.B):
        assert (got[b, :, int(x["lens"][b]):] == 0).all()
    return got


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("mask", ["all", "causal"])
@pytest.mark.parametrize("size", [s for s in SIZES if s[6] > 0])
def test_weights_match_oracle(B, size, mask, dt):
    Bn, L, Hq, Hkv, D, P, S, lens = size
    x = make(Bn, L, Hq, Hkv, D, P, S, dt, lens, causal(lens, L) if mask == "causal" else None)
    check_weights(B, x, S)
    acc = torch.rand(Bn, Hkv, S, device="cuda")
    check_weights(B, x, S, acc, 0.9)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("order", ["head", "fused"])
def test_weights_orders_padding_and_bad_entries(B, order, dt):
    S, lens, vis = 200, [150, 129, 40], [[-1, 140, 150], [0, 1, 129], [40, 39, -2]]
    x = make(3, 3, 8, 2, 72, 50, S, dt, lens, vis, order=order, pad=8, qpad=8)
    att = att_of(B, x, S)
    got = check_weights(B, x, S, att=att)
    r = att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"], visible=x["vis"])
    acc = torch.full((3, 2, S), float("nan"), device="cuda")
    for b, n in enumerate(lens):
        x["ko"][b, n:] = float("nan")
        acc[b, :, :n] = 0
    x["ko"][0, 145] = float("inf")                   # seen by one position of three
    w = n64(att.weights(x["q"], r["lse"], x["ko"], x["lens"], acc=acc, visible=x["vis"], out=acc))
    same = np.ones(w.shape, bool)
    same[0, :, 145] = False
    np.testing.assert_array_equal(w[same], got[same])


# ---------------------------------------------------------------- eviction

def check_evict(B, x, acc, S, keep, recent, room=None):
    Bn, _, Hkv, D = x["ko"].shape
    att = B.PrefixAttention(Bn, 1, Hkv, Hkv, D, 0, S, x["ko"].dtype)
    out = att.alloc_evicted(keep, room)
    for t in out.values():
        t.fill_(77)
    att.evict(x["ko"], x["vo"], acc, x["lens"], keep, recent, out=out)
    assert att.device_status() == B.OK
    want = C.evict(n64(x["ko"]), n64(x["vo"]), acc.double().cpu().numpy(), n64(x["lens"]), keep, recent)
    for name, w in zip(("k", "v", "acc", "own_len", "kept"), want):
        got = n64(out[name])
        if name in ("k", "v"):
            assert (got[:, keep:] == 77).all()
            got = got[:, :keep]
        np.testing.assert_array_equal(got, w, err_msg=name)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("size", [
    # B, Hkv, D, S, lens, keep, recent
    (1, 1, 8, 1, [1], 1, 0),
    (2, 1, 8, 2, [2, 0], 1, 1),
    (3, 2, 64, 33, [33, 20, 0], 20, 5),
    (2, 3, 72, 1300, [1300, 1025], 1024, 0),
    (2, 2, 128, 5000, [5000, 4097], 1000, 1000),
    (4, 4, 128, 3001, [3001, 2048, 2049, 700], 2048, 100),
    (1, 2, 16, 2100, [2100], 2099, 2098),
    (1, 1, 64, 40000, [39999], 17, 3),
])
@pytest.mark.parametrize("kind", ["random", "ties", "special"])
def test_evict_matches_oracle(B, size, kind, dt):
    Bn, Hkv, D, S, lens, keep, recent = size
    x = make(Bn, 1, Hkv, Hkv, D, 0, S, dt, lens)
    g = torch.Generator().manual_seed(S + keep)
    acc = torch.rand(Bn, Hkv, S, generator=g)
    if kind == "ties":
        acc = torch.floor(acc * 3) * (acc > 0.4)
    if kind == "special":
        pick = torch.randint(0, 12, acc.shape, generator=g)
        for j, v in enumerate((float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 1e-45, -1e-45,
                               3.4028234663852886e38, -1.0)):
            acc = torch.where(pick == j, torch.tensor(v), acc)
    check_evict(B, x, acc.cuda(), S, keep, recent)


@pytest.mark.parametrize("order", ["head", "fused"])
def test_evict_orders_and_larger_targets(B, order):
    x = make(3, 1, 2, 2, 72, 0, 500, BF, [500, 100, 333], order=order, pad=8)
    check_evict(B, x, torch.rand(3, 2, 500, device="cuda"), 500, 200, 10, room=260)


def test_caches_beyond_32_bit_offsets(B):
    """Sequences, tokens and heads whose offsets pass 2^32 elements: a sparse 10 GB pool."""
    Bn, S, Hkv, D = 2, 300, 2, 64
    pool = torch.empty(5_000_000_000, dtype=BF, device="cuda")
    x = make(Bn, 2, 4, 2, D, 10, S, BF, [300, 170])
    for name, off in (("ko", 0), ("vo", 40_000)):
        for strides in ((4_400_000_000, 512, 128), (64, 14_700_000, 128), (128, 512, 4_600_000_000)):
            v = torch.as_strided(pool, (Bn, S, Hkv, D), (*strides, 1), off)
            v.copy_(x[name])
            y = dict(x)
            y[name] = v
            check_attend(B, y, S)
    check_weights(B, y | {"ko": torch.as_strided(pool, (Bn, S, Hkv, D), (64, 14_700_000, 128, 1), 0).copy_(x["ko"])}, S)
    far = torch.as_strided(pool, (Bn, S, Hkv, D), (4_400_000_000, 512, 128, 1), 0)
    far.copy_(x["ko"])
    check_evict(B, dict(x, ko=far), torch.rand(Bn, Hkv, S, device="cuda"), S, 100, 10)


def test_decode_loop_example(B):
    """attend -> weights -> evict over several steps keeps every sequence within its budget, and the
    sums of weights are those of the entries that stayed."""
    Bn, L, Hq, Hkv, D, P, S, keep = 3, 4, 8, 2, 64, 64, 48, 24
    g = torch.Generator(device="cuda").manual_seed(0)
    att = B.PrefixAttention(Bn, L, Hq, Hkv, D, P, S, BF)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF)
    kp, vp = rnd(P, Hkv, D), rnd(P, Hkv, D)
    k, v = torch.zeros(Bn, S, Hkv, D, dtype=BF, device="cuda"), torch.zeros(Bn, S, Hkv, D, dtype=BF, device="cuda")
    spare = att.alloc_evicted(keep, room=S)
    acc = torch.zeros(Bn, Hkv, S, device="cuda")
    n = 0
    lens = torch.zeros(Bn, dtype=torch.int32, device="cuda")
    for step in range(20):
        k[:, n:n + L], v[:, n:n + L] = rnd(Bn, L, Hkv, D), rnd(Bn, L, Hkv, D)
        n += L
        lens += L
        q = rnd(Bn, L, Hq, D)
        r = att.attend(q, kp, vp, k, v, lens)
        att.weights(q, r["lse"], k, lens, acc=acc, out=acc)
        assert torch.isfinite(r["out"]).all() and (acc[:, :, n:] == 0).all()
        if n + L > S:
            att.evict(k, v, acc, lens, keep, L, out=spare)
            k, v, spare["k"], spare["v"] = spare["k"], spare["v"], k, v
            lens.copy_(spare["own_len"])
            acc.zero_()
            acc[:, :, :keep] = spare["acc"]
            n = keep
    assert att.device_status() == B.OK and math.isclose(float(acc.sum()), float(acc[:, :, :n].sum()))
