"""Own caches in 4 bits on the GPU against the float64 oracle: writing, reading back, attention.

What is written and read back is exact. Tolerances of attention: as with unquantised caches, scores are off by
eps = (2D + 16) u big + 2^-21 (u = 2^-24; the entries' products are exact in fp32, with fp32 queries
after rounding these to 2^-22, another 4 u big), and sums of n terms by 2 n u (the tensor cores cut what they add
to a sum: 2 u each). Weights are rounded before they meet the values: own entries' to fp16 (2^-11 each, and 2^-35 of the
largest weight, where fp16 ends), with fp32 to two of them (2^-22), the prefix's, with bf16, to bf16 (2^-8 each).
The result's rounding is 2^-8 (bf16)."""
import numpy as np
import pytest
import torch

from oracle import cache as C
from oracle import packed as P

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


def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def raw(cache, name):
    return cache[name].cpu().numpy(), cache[name + "_scales"].cpu().numpy()


def room(shape, order, pad, fill=None):
    """A uint8 tensor [B, S, Hkv, n] whose rows lie `pad` bytes apart, in the given memory order."""
    Bn, S, H, n = shape
    lead = (Bn, H, S) if order == "head" else (Bn, S, H)
    t = torch.randint(0, 256, (*lead, n + pad), dtype=torch.uint8).cuda() if fill is None else \
        torch.full((*lead, n + pad), fill, dtype=torch.uint8).cuda()
    t = t[..., :n]
    return t.transpose(1, 2) if order == "head" else t


def new_cache(Bn, S, H, D, order="token", pad=0, fill=None):
    w = 4 if D <= 64 else 8
    put = {}
    for name in "kv":
        put[name] = room((Bn, S, H, D // 2), order, 16 * pad, fill)
        put[name + "_scales"] = room((Bn, S, H, w), order, 8 * pad, fill)
    return put


def spread_rows(shape, dt, seed):
    """Rows whose groups' magnitudes range over the format's and beyond, with ties and zeros among them."""
    g = torch.Generator().manual_seed(seed)
    D = shape[-1]
    x = torch.randn(*shape, generator=g).view(*shape[:-1], D // 16, 16)
    x = x * torch.exp2(torch.randint(-17, 15, x.shape[:-1], generator=g).float())[..., None]
    tie = torch.tensor([.25, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, 0])
    ties = torch.rand(x.shape[:-1], generator=g) < 0.2
    s = (8 + torch.randint(0, 8, x.shape[:-1], generator=g).float()) / 8
    x = torch.where(ties[..., None], tie * s[..., None], x)
    x = torch.where((torch.rand(x.shape[:-1], generator=g) < 0.05)[..., None], torch.zeros(()), x)
    return x.view(shape).to(dt)


# ---------------------------------------------------------------- writing and reading back

WRITES = [
    # B, T, S, Hkv, D, order, start, count
    (1, 1, 1, 1, 16, "token", [0], None),
    (1, 1, 5, 8, 128, "token", [4], None),
    (3, 7, 40, 2, 64, "head", [0, 33, 5], [7, 7, 0]),
    (2, 33, 64, 3, 80, "token", [31, 0], [33, 1]),
    (4, 5, 9, 1, 48, "head", [4, 0, 2, 1], [5, 3, 1, 0]),
    (2, 50, 70, 5, 112, "token", [20, 3], [50, 49]),
    (1, 90, 128, 4, 96, "head", [38], [90]),
    (9, 17, 30, 2, 32, "token", [i for i in range(9)], [17 - i for i in range(9)]),
]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("size", WRITES)
def test_store_and_load_are_exact(B, size, dt):
    Bn, T, S, H, D, order, start, count = size
    att = B.PackedAttention(Bn, 1, H, H, D, 0, S, dt)
    for pad in (0, 1):
        cache = new_cache(Bn, S, H, D, order, pad)
        before = {n: t.clone() for n, t in cache.items()}
        k, v = (spread_rows((Bn, T, H, D), dt, 7 * T + i) for i in range(2))
        att.store(cache, k.cuda(), v.cuda(), i32(start), None if count is None else i32(count))
        assert att.device_status() == B.OK
        back = att.load(cache, T, i32(start), None if count is None else i32(count))
        assert att.device_status() == B.OK
        used = [T] * Bn if count is None else count
        for name, x in (("k", k), ("v", v)):
            codes, scales = raw(before, name)
            want = np.zeros((Bn, T, H, D))
            for b in range(Bn):
                c, s = P.store(n64(x)[b, :used[b]])
                at = slice(start[b], start[b] + used[b])
                codes[b, at] = c
                scales[b, at, :, :D // 16] = s[..., :D // 16]
                want[b, :used[b]] = P.values(c, s)
            got_c, got_s = raw(cache, name)
            assert (got_c == codes).all() and (got_s == scales).all()
            assert (n64(back[name]) == want).all()


def test_borders_of_every_scale_and_code(B):
    """Every scale that is written: the numbers half-way between two codes, which go to the even one, and their neighbours
    in fp32; and the largest magnitudes half-way between two scales, with their neighbours."""
    half = np.array([.25, .75, 1.25, 1.75, 2.5, 3.5, 5], np.float32)
    rows = []
    for b in range(8, 227):
        s = np.float32(P.scale_of(b))
        x = half * s                                 # (exact)
        top = np.float32(6) * s
        for y in (x, np.nextafter(x, np.float32(0)), np.nextafter(x, np.float32(1e9))):
            rows.append(np.concatenate([[top, -top], y, -y]))
        if b < 226:
            edge = np.float32(3) * (s + np.float32(P.scale_of(b + 1)))   # six times what lies half-way: exact
            for top in (edge, np.nextafter(edge, np.float32(0)), np.nextafter(edge, np.float32(1e9))):
                rows.append(np.concatenate([[top, -0.0], x, -x]))
    x = torch.from_numpy(np.stack(rows).astype(np.float32)).view(1, -1, 1, 16)
    T = x.shape[1]
    att = B.PackedAttention(1, 1, 1, 1, 16, 0, T, F32)
    cache = new_cache(1, T, 1, 16, fill=0)
    att.store(cache, x.cuda(), (-x).cuda(), i32([0]))
    assert att.device_status() == B.OK
    for name, y in (("k", x), ("v", -x)):
        c, s = P.store(n64(y))
        got_c, got_s = raw(cache, name)
        assert (got_s == s).all() and (got_c == c).all()


def test_every_number_of_bf16_under_every_scale(B):
    """Every scale that is written with every magnitude of 2^-4 to 6 times it (smaller ones are 0), and every finite number
    as the largest of its group."""
    def bf(bits):
        return torch.from_numpy((np.asarray(bits).astype(np.uint32) << 16).view(np.float32)).to(BF)

    every = bf(np.arange(0x7f80))
    rows = []
    for b in range(8, 227):
        s = P.scale_of(b)
        x = every[(every.double() >= s / 16) & (every.double() <= 6 * s)]
        top = torch.full_like(x[:1], 6 * s)          # (exact)
        x = torch.cat([x, x.new_zeros(-len(x) % 15)]).view(-1, 15)
        x[:, ::2] *= -1
        rows.append(torch.cat([top.expand(len(x), 1), x], 1))
    tops = every[:, None] * torch.tensor([1, -.75, .3125, -.125, .0, -.0, .625, -.4375] * 2).to(BF)
    x = torch.cat([*rows, tops]).view(1, -1, 1, 16)
    att = B.PackedAttention(1, 1, 1, 1, 16, 0, x.shape[1], BF)
    cache = new_cache(1, x.shape[1], 1, 16, fill=0)
    att.store(cache, x.cuda(), (-x).cuda(), i32([0]))
    assert att.device_status() == B.OK
    for name, y in (("k", x), ("v", -x)):
        c, s = P.store(n64(y))
        got_c, got_s = raw(cache, name)
        assert (got_s == s).all() and (got_c == c).all()


@pytest.mark.parametrize("dt", [BF, F32])
def test_every_byte_reads_as_the_oracle_has_it(B, dt):
    """All scales, the ones that no call writes among them, with all codes."""
    cache = new_cache(1, 256, 1, 128)
    cache["k_scales"].copy_(torch.arange(256).view(1, 256, 1, 1).expand(1, 256, 1, 8))
    cache["v_scales"].copy_(torch.arange(256).flip(0).view(1, 256, 1, 1).expand(1, 256, 1, 8))
    att = B.PackedAttention(1, 1, 1, 1, 128, 0, 256, dt)
    back = att.load(cache, 256, i32([0]))
    for name in "kv":
        assert (n64(back[name]) == P.values(*raw(cache, name))).all()


@pytest.mark.parametrize("dt", [BF, F32])
def test_what_is_loaded_is_stored_as_it_was(B, dt):
    att = B.PackedAttention(2, 1, 3, 3, 80, 0, 64, dt)
    cache, again = new_cache(2, 64, 3, 80, fill=0), new_cache(2, 64, 3, 80, fill=0)
    k, v = (spread_rows((2, 64, 3, 80), dt, i).cuda() for i in range(2))
    att.store(cache, k, v, i32([0, 0]))
    back = att.load(cache, 64, i32([0, 0]))
    att.store(again, back["k"], back["v"], i32([0, 0]))
    for n in cache:
        assert torch.equal(cache[n], again[n])


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T", [1, 40])
def test_numbers_that_are_none_are_reported(B, dt, T):
    att = B.PackedAttention(1, 1, 2, 2, 32, 0, 64, dt)
    k, v = (spread_rows((1, T, 2, 32), dt, i) for i in range(2))
    k[0, T - 1, 1, 20] = float("nan")
    v[0, 0, 0, 3] = -float("inf")
    v[0, 0, 1, 31] = float("inf")
    cache = new_cache(1, 64, 2, 32, fill=0)
    att.store(cache, k.cuda(), v.cuda(), i32([2]))
    assert att.device_status() == B.ERR_NUMERIC
    for name, x in (("k", k), ("v", v)):
        c, s = P.store(n64(x))
        got_c, got_s = raw(cache, name)
        assert (got_c[:, 2:2 + T] == c).all() and (got_s[:, 2:2 + T] == s).all()
    # not where they are not written
    att.store(cache, k.cuda(), v.cuda(), i32([2]), i32([0]))
    assert att.device_status() == B.OK


@pytest.mark.parametrize("T", [3, 40])
def test_places_out_of_range_are_left_out_and_reported(B, T):
    att = B.PackedAttention(4, 1, 2, 2, 64, 0, 50, BF)
    k, v = (spread_rows((4, T, 2, 64), BF, i).cuda() for i in range(2))
    start, count = [48, -2, 5, 2 ** 31 - 2], [T, T, T + 1, T]
    cache = new_cache(4, 50, 2, 64)
    before = {n: t.clone() for n, t in cache.items()}
    att.store(cache, k, v, i32(start), i32(count))
    assert att.device_status() == B.ERR_INVALID_ARG
    back = att.load(cache, T, i32(start), i32(count))
    assert att.device_status() == B.ERR_INVALID_ARG
    for name, x in (("k", k), ("v", v)):
        codes, scales = raw(before, name)
        want = np.zeros((4, T, 2, 64))
        for b in range(4):
            for t in range(T):
                if 0 <= start[b] + t < 50:
                    codes[b, start[b] + t], scales[b, start[b] + t] = P.store(n64(x)[b, t])
                    want[b, t] = P.values(codes[b, start[b] + t], scales[b, start[b] + t])
        got_c, got_s = raw(cache, name)
        assert (got_c == codes).all() and (got_s == scales).all() and (n64(back[name]) == want).all()
    for n in ([0] * 4, [-3, 0, 0, 0]):               # nothing to write: a start may be anything; a count may not
        att.store(cache, k, v, i32(start), i32(n))
        assert att.device_status() == (B.ERR_INVALID_ARG if n[0] else B.OK)


def test_rows_of_any_stride_are_written_and_filled(B):
    att = B.PackedAttention(2, 1, 3, 3, 64, 0, 30, BF)
    kv = spread_rows((2, 9, 2, 3, 64 + 16), BF, 3).cuda()[..., :64]
    k, v = kv[:, :, 0], kv[:, :, 1]
    cache = new_cache(2, 30, 3, 64)
    att.store(cache, k, v, i32([1, 21]))
    out = {n: torch.full((2, 3, 9, 72), 5.0, dtype=BF).cuda()[..., :64].transpose(1, 2) for n in "kv"}
    att.load(cache, 9, i32([1, 21]), i32([9, 4]), out=out)
    for name, x in (("k", k), ("v", v)):
        want = P.values(*P.store(n64(x)))
        want[1, 4:] = 0
        assert (n64(out[name]) == want).all()
        assert (out[name].transpose(1, 2)._base[..., 64:] == 5).all()


# ---------------------------------------------------------------- attention

def make(Bn, L, Hq, Hkv, D, Pn, S, dt, lens, vis=None, order="token", pad=0, seed=0, fill=None):
    g = torch.Generator().manual_seed(seed + 1000 * D + 10 * Pn + S)
    x = {"q": (torch.randn(Bn, L, Hq, D + 8 * pad, generator=g) * 1.5).to(dt).cuda()[..., :D]}
    x["kp"] = x["vp"] = x["cache"] = x["k"] = x["v"] = None
    if Pn:
        x["kp"], x["vp"] = (torch.randn(Pn, Hkv, D, generator=g).to(dt).cuda() for _ in range(2))
    if S:
        x["cache"] = new_cache(Bn, S, Hkv, D, order, pad, fill)
        for name in "kv":
            rows = torch.randn(Bn, S, Hkv, D, generator=g) * torch.exp(torch.randn(Bn, S, Hkv, 1, generator=g) * 0.3)
            c, s = fast_store(rows)
            x["cache"][name].copy_(c)
            x["cache"][name + "_scales"].copy_(s)
            x[name] = P.values(c.numpy(), s.numpy())
    x["lens"] = i32(lens)
    x["vis"] = None if vis is None else i32(vis)
    return x


def fast_store(rows):
    """Codes and scales of rows, nearly the nearest (these tests take them as they are)."""
    D = rows.shape[-1]
    g = rows.view(*rows.shape[:-1], D // 16, 16)
    b = (torch.log2(g.abs().amax(-1) / 6) * 8 + 120).round().clamp(8, 226).int()
    s = torch.tensor([P.scale_of(i) for i in range(227)])[b.long()]
    grid = torch.tensor(P.GRID)
    i = ((g.abs() / s[..., None])[..., None] - grid).abs().argmin(-1) + 8 * (g < 0)
    i = i.view(rows.shape)
    scales = torch.zeros(*rows.shape[:-1], 4 if D <= 64 else 8, dtype=torch.uint8)
    scales[..., :D // 16] = b
    return (i[..., 0::2] + 16 * i[..., 1::2]).to(torch.uint8), scales


def att_of(B, x, S, Pn=None):
    Bn, L, Hq, D = x["q"].shape
    Hkv = (x["kp"] if x["cache"] is None else x["k"]).shape[-2]
    return B.PackedAttention(Bn, L, Hq, Hkv, D, 0 if x["kp"] is None else x["kp"].shape[0], S, x["q"].dtype)


def wanted(x, scale):
    return C.attend(n64(x["q"]), n64(x["kp"]), n64(x["vp"]), x["k"], x["v"], n64(x["lens"]), n64(x["vis"]), scale)


def compare(r, want, x, S):
    out, lse, mass, big = want
    dt, D = x["q"].dtype, x["q"].shape[-1]
    Pn = 0 if x["kp"] is None else x["kp"].shape[0]
    n = Pn + S + 16
    got_o, got_l = n64(r["out"]), n64(r["lse"])
    eps = (2 * D + 16 + (4 if dt == F32 else 0)) * U * big + 2.0 ** -21
    none = np.isneginf(lse)
    assert (np.isneginf(got_l) == none).all()
    assert (got_o[none] == 0).all()
    tol_l = eps + n * U + 2.0 ** -22 * np.abs(np.where(none, 0, lse))
    assert (np.abs(np.where(none, 0, got_l - np.where(none, 0, lse))) <= tol_l).all()
    weight = 2.0 ** -22 if dt == F32 else (2.0 ** -8 if Pn else 2.0 ** -11)
    top = 0 if x["v"] is None else np.abs(x["v"]).max()
    tol = (2 * eps + 2 * n * U)[..., None] * mass + weight * mass * (1 + 2.0 ** -6) + S * 2.0 ** -35 * top
    tol = tol + (2.0 ** -22 if dt == F32 else 2.0 ** -8) * np.abs(out)
    worst = np.max(np.abs(got_o - out) / (tol + 1e-30)) if out.size else 0
    assert worst <= 1, worst


def check(B, x, S, want_status=None, att=None):
    att = att or att_of(B, x, S)
    r = att.attend(x["q"], x["kp"], x["vp"], x["cache"], x["lens"], visible=x["vis"])
    assert att.device_status() == (B.OK if want_status is None else want_status)
    compare(r, wanted(x, att.scale), x, S)
    return att, r


def causal(lens, L):
    return [[max(0, n - L + 1 + i) for i in range(L)] for n in lens]


SIZES = [
    # B, L, Hq, Hkv, D, P, S, lens
    (1, 1, 1, 1, 16, 0, 1, [1]),
    (1, 1, 1, 1, 64, 1, 0, [0]),
    (1, 1, 8, 2, 128, 127, 5, [5]),
    (1, 1, 4, 1, 128, 0, 17, [17]),
    (2, 1, 4, 4, 64, 128, 130, [130, 1]),
    (3, 5, 6, 2, 80, 129, 257, [0, 129, 257]),
    (2, 7, 28, 4, 128, 301, 77, [77, 3]),
    (5, 2, 3, 1, 48, 1, 64, [64, 0, 63, 1, 17]),
    (1, 33, 16, 2, 128, 700, 300, [299]),
    (2, 64, 8, 1, 64, 0, 200, [200, 70]),
    (70, 1, 4, 1, 64, 300, 40, [(7 * i) % 41 for i in range(70)]),
    (4, 3, 5, 5, 112, 64, 128, [128, 128, 64, 65]),
    (2, 4, 24, 8, 128, 2500, 600, [600, 500]),
    (1, 1, 16, 1, 96, 0, 5000, [4999]),               # one row tile's keys over many CTAs
    (40, 2, 8, 4, 32, 0, 90, [(11 * i) % 91 for i in range(40)]),   # CTAs with many short fragments
    (1, 20, 8, 2, 128, 0, 1500, [1490]),
    (3, 12, 8, 2, 64, 90, 260, [260, 100, 0]),         # 48 rows, and 32, of up to 64 channels
    (3, 8, 8, 2, 48, 90, 260, [260, 100, 0]),
]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("mask", ["all", "causal"])
@pytest.mark.parametrize("size", SIZES)
def test_attend_matches_oracle(B, size, mask, dt):
    Bn, L, Hq, Hkv, D, Pn, S, lens = size
    x = make(Bn, L, Hq, Hkv, D, Pn, S, dt, lens, causal(lens, L) if mask == "causal" else None)
    check(B, x, S)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("order", ["token", "head"])
@pytest.mark.parametrize("D", [64, 80, 128])
def test_attend_takes_any_strides(B, dt, order, D):
    x = make(3, 4, 8, 2, D, 50, 150, dt, [150, 20, 0], causal([150, 20, 0], 4), order, pad=1)
    check(B, x, 150)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("Pn", [0, 40])
def test_rows_that_see_nothing(B, dt, Pn):
    vis = [[-1, 0, 3], [0, 0, 0], [-1, -1, -1], [5, -7, 90]]
    x = make(4, 3, 4, 2, 64, Pn, 90, dt, [90, 90, 40, 60], vis)
    check(B, x, 90)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("rows", [1, 6, 40])
def test_hidden_entries_do_not_matter(B, dt, rows):
    """Bytes that no call writes, in every place that no row sees, and between what only some rows see."""
    lens = [100, 37, 0, 260]
    vis = [[max(0, n - i) for i in range(rows)] for n in lens]
    x = make(4, rows, 2, 1, 128, 30, 260, dt, lens, vis)
    att, r = check(B, x, 260)
    for b, n in enumerate(lens):
        for name in ("k", "v", "k_scales", "v_scales"):
            x["cache"][name][b, n:] = 255
    again = att.attend(x["q"], x["kp"], x["vp"], x["cache"], x["lens"], visible=x["vis"])
    assert torch.equal(again["out"], r["out"]) and torch.equal(again["lse"], r["lse"])
    # a row's bits do not change with entries that it does not see and others do
    for b, n in enumerate(lens):
        if n > 1 and rows > 1:
            x["cache"]["v_scales"][b, n - 1] = 255
    again = att.attend(x["q"], x["kp"], x["vp"], x["cache"], x["lens"], visible=x["vis"])
    assert torch.equal(again["out"][:, 1:], r["out"][:, 1:]) and torch.equal(again["lse"], r["lse"])


@pytest.mark.parametrize("dt", [BF, F32])
def test_queries_of_any_size(B, dt):
    """The queries' scaling by a power of two: tiny, huge and mixed rows, zeros, with the scale that undoes it."""
    for e in (-100, -30, 30, 100):
        x = make(2, 3, 4, 2, 64, 0, 70, dt, [70, 9])
        x["q"] = (x["q"].float() * 2.0 ** e).to(dt)
        x["q"][0, 1] = 0
        att = att_of(B, x, 70)
        scale = 2.0 ** -e * 0.125
        r = att.attend(x["q"], None, None, x["cache"], x["lens"], scale=scale)
        compare(r, wanted(x, scale), x, 70)
    x = make(1, 2, 4, 2, 64, 0, 70, dt, [70])
    x["q"][0, 0] *= torch.exp2(torch.linspace(-30, 10, 64)).to(dt).cuda()
    check(B, x, 70)


@pytest.mark.parametrize("dt", [BF, F32])
def test_queries_that_are_no_numbers_show(B, dt):
    x = make(1, 2, 4, 2, 64, 20, 70, dt, [70])
    x["q"][0, 0, 1, 5] = float("nan")
    att = att_of(B, x, 70)
    r = att.attend(x["q"], x["kp"], x["vp"], x["cache"], x["lens"])
    bad = torch.zeros(1, 2, 4, dtype=torch.bool).cuda()
    bad[0, 0, 1] = True
    assert (torch.isnan(r["lse"]) == bad).all() and (torch.isnan(r["out"]) == bad[..., None]).all()


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("rows", [2, 40])
def test_scores_of_any_size_keep_their_weights(B, dt, rows):
    """Scores growing and falling along the keys: the running maximum; one entry far above all others."""
    for sign in (1.0, -1.0):
        x = make(1, rows, 2, 1, 64, 0, 600, dt, [600])
        x["q"].fill_(1.0)
        ramp = (sign * torch.linspace(-300, 300, 600)).view(1, 600, 1, 1)
        k = torch.zeros(1, 600, 1, 64)
        k[..., :1] = ramp
        c, s = fast_store(k)
        x["cache"]["k"].copy_(c)
        x["cache"]["k_scales"].copy_(s)
        x["k"] = P.values(c.numpy(), s.numpy())
        check(B, x, 600)
    k[0, 211] = 200.0
    c, s = fast_store(k * 0.05)
    x["cache"]["k"].copy_(c)
    x["cache"]["k_scales"].copy_(s)
    x["k"] = P.values(c.numpy(), s.numpy())
    check(B, x, 600)


@pytest.mark.parametrize("dt", [BF, F32])
def test_scale(B, dt):
    x = make(2, 2, 4, 2, 64, 100, 100, dt, [100, 9])
    att = att_of(B, x, 100)
    for scale in (0.0, 1.0, 0.01):
        r = att.attend(x["q"], x["kp"], x["vp"], x["cache"], x["lens"], scale=scale)
        compare(r, wanted(x, scale), x, 100)


@pytest.mark.parametrize("dt", [BF, F32])
def test_lengths_out_of_range_are_clamped_and_reported(B, dt):
    x = make(2, 2, 4, 2, 64, 40, 60, dt, [75, -3])
    att, _ = check(B, x, 60, want_status=B.ERR_INVALID_ARG)
    x["lens"].clamp_(0, 60)
    check(B, x, 60, att=att)                         # the next call clears the word


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("L", [1, 9])
def test_the_same_inputs_give_the_same_bits_on_any_stream(B, dt, L):
    x = make(6, L, 8, 2, 128, 900, 400, dt, [400, 1, 37, 250, 0, 399])
    att, r = check(B, x, 400)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        again = att.attend(x["q"], x["kp"], x["vp"], x["cache"], x["lens"], stream=s)
        s.synchronize()
        assert torch.equal(again["out"], r["out"]) and torch.equal(again["lse"], r["lse"])


def test_a_step_captured_and_replayed(B):
    """Write, attend, read back in one graph, on inputs that change in place; the workspace is shared by two graphs."""
    Bn, L, S, H, D = 3, 4, 120, 2, 64
    att = B.PackedAttention(Bn, L, 8, H, D, 50, S, BF)
    x = make(Bn, L, 8, H, D, 50, S, BF, [0] * Bn)
    rows = {n: spread_rows((Bn, L, H, D), BF, i).cuda() for i, n in enumerate("kv")}
    start, n = i32([90, 20, 0]), i32([94, 24, 4])
    out = {"out": torch.empty_like(x["q"].contiguous()), "lse": torch.empty(Bn, L, 8, device="cuda")}
    back = {m: torch.empty(Bn, L, H, D, dtype=BF, device="cuda") for m in "kv"}

    def step():
        att.store(x["cache"], rows["k"], rows["v"], start)
        att.attend(x["q"], x["kp"], x["vp"], x["cache"], n, out=out)
        att.load(x["cache"], L, start, out=back)

    step()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            step()
        graphs.append(g)
    for turn in range(4):
        for i, m in enumerate("kv"):
            rows[m].copy_(torch.randn(Bn, L, H, D).to(BF))
        start.copy_(i32([(30 * turn + 5 * b) % 110 for b in range(Bn)]))
        n.copy_(start + L)
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        assert att.device_status() == B.OK
        for m in "kv":
            assert (n64(back[m]) == P.values(*P.store(n64(rows[m])))).all()
            x[m] = P.values(*raw(x["cache"], m))
        x["lens"] = n
        compare(out, wanted(x, att.scale), x, S)


def test_calls_on_two_streams_at_once(B):
    """Two objects, each with its own workspace and stream, that run beside each other."""
    x = [make(4, 3, 8, 2, 128, 700, 900, BF, [900, 3, 500, 0], seed=i) for i in range(2)]
    att = [att_of(B, y, 900) for y in x]
    want = [a.attend(y["q"], y["kp"], y["vp"], y["cache"], y["lens"]) for a, y in zip(att, x)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for i in range(2):
            got[i].append(att[i].attend(x[i]["q"], x[i]["kp"], x[i]["vp"], x[i]["cache"], x[i]["lens"],
                                        stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            assert torch.equal(r["out"], want[i]["out"]) and torch.equal(r["lse"], want[i]["lse"])


def test_a_cache_beyond_32_bits(B):
    """Entries whose offsets pass 2^32 bytes, in the codes and in the scales' strides."""
    S, H, D = 70000, 1, 128
    big = torch.zeros(S, 65536, dtype=torch.uint8, device="cuda")          # 4.6 GB: a row of codes every 64 KB
    cache = {n: big[None, :, None, o:o + 64] for n, o in (("k", 0), ("v", 1024))}
    cache.update({n + "_scales": big[None, :, None, o:o + 8] for n, o in (("k", 2048), ("v", 4096))})
    att = B.PackedAttention(1, 1, 2, H, D, 0, S, BF)
    rows = {n: spread_rows((1, 40, H, D), BF, i).clamp(-4, 4).cuda() for i, n in enumerate("kv")}
    at = S - 40
    att.store(cache, rows["k"], rows["v"], i32([at]))
    back = att.load(cache, 40, i32([at]))
    for n in "kv":
        assert (n64(back[n]) == P.values(*P.store(n64(rows[n])))).all()
    q = torch.randn(1, 1, 2, D).to(BF).cuda() * 4
    r = att.attend(q, None, None, cache, i32([S]))
    k, v = (torch.cat([torch.zeros(at, D).double(), back[n][0, :, 0].double().cpu()]) for n in "kv")
    s = q[0, 0].double().cpu() @ k.T * D ** -0.5
    want = torch.softmax(s, 1) @ v
    mass = torch.softmax(s, 1) @ v.abs()
    got = r["out"][0, 0].double().cpu()
    assert ((got - want).abs() <= (2.0 ** -8 + 2 * S * U) * mass + 2.0 ** -8 * want.abs() + 1e-9).all()
    assert (n64(r["lse"][0, 0]) - torch.logsumexp(s, 1).numpy() < 1e-3).all()


@pytest.mark.parametrize("Pn", [0, 300])
def test_a_wait_that_gives_up_is_reported_and_the_next_call_is_right(B, Pn):
    """Many rows a key head (the kernel on the tensor cores, whose waits are bounded): a limit that runs out while the
    tiles are being written, then the default again, with the same bits as before."""
    x = make(6, 16, 8, 2, 128, Pn, 700, BF, [700, 300, 0, 650, 64, 1])
    att, r = check(B, x, 700)
    zeros = {"out": torch.zeros_like(r["out"]), "lse": torch.zeros_like(r["lse"])}
    before = B.set_wait_limit(1)
    try:
        for _ in range(3):
            att.attend(x["q"], x["kp"], x["vp"], x["cache"], x["lens"], out=zeros)
            assert att.device_status() == B.ERR_TIMEOUT
    finally:
        B.set_wait_limit(before)
    again = att.attend(x["q"], x["kp"], x["vp"], x["cache"], x["lens"])
    assert att.device_status() == B.OK
    assert torch.equal(again["out"], r["out"]) and torch.equal(again["lse"], r["lse"])


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("L, Hq, Hkv", [(1, 64, 64), (2, 12, 12), (3, 6, 6), (1, 16, 16), (4, 32, 4), (1, 9, 3)])
def test_heads_share_units_whatever_their_number(B, dt, L, Hq, Hkv):
    """Enough sequences that a unit is of several heads (as many as a power of two divides, up to eight)."""
    lens = [(37 * i) % 300 for i in range(60)]
    x = make(60, L, Hq, Hkv, 64, 0, 300, dt, lens, causal(lens, L))
    check(B, x, 300)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("Pn", [0, 37])
def test_calls_in_their_usual_form_and_with_results_given(B, monkeypatch, dt, Pn):
    """Two ways of marshalling, the same bits; the first looks at nothing in the interpreter."""
    x = make(3, 2, 8, 2, 64, Pn, 40, dt, [40, 0, 17])
    att = att_of(B, x, 40)
    start, count = i32([1, 0, 9]), i32([30, 0, 11])
    given = {"out": torch.empty(3, 2, 8, 64, dtype=dt, device="cuda"), "lse": torch.empty(3, 2, 8, device="cuda")}
    back = {n: torch.empty(3, 30, 2, 64, dtype=dt, device="cuda") for n in "kv"}
    args = (x["q"], x["kp"] if Pn else None, x["vp"] if Pn else None, x["cache"], x["lens"])
    att.attend(*args, visible=i32([[40, 3], [0, 0], [1, 17]]), scale=0.5, out=given)
    att.load(x["cache"], 30, start, count, out=back)
    other = att.alloc_cache()
    att.store(other, back["k"], back["v"], start, count, stream=torch.cuda.current_stream())
    with monkeypatch.context() as m:
        for name in ("_view", "_plain", "_bytes", "_cache"):
            m.setattr(B.PackedAttention, name, None)
        r = att.attend(*args, visible=i32([[40, 3], [0, 0], [1, 17]]), scale=0.5)
        kv = att.load(x["cache"], 30, start, count)
        mine = att.alloc_cache("head")
        assert att.store(mine, kv["k"], kv["v"], start, count) is mine
    for got, want in ((r, given), (kv, back), (mine, other)):
        assert got.keys() == want.keys()
        for n in want:
            assert got[n].dtype == want[n].dtype and torch.equal(got[n], want[n]), n


def test_the_usual_form_refuses_what_the_other_does(B):
    x = make(3, 2, 8, 2, 64, 20, 40, BF, [40, 0, 17])
    att, c = att_of(B, x, 40), x["cache"]
    k = torch.zeros(3, 5, 2, 64, dtype=BF, device="cuda")
    start = i32([0, 0, 0])
    good = dict(q=x["q"], k_prefix=x["kp"], v_prefix=x["vp"], cache=c, own_len=x["lens"], visible=None)
    for name, bad in [("q", x["q"].float()), ("q", x["q"][:, :1]), ("q", x["q"].cpu()), ("q", None),
                      ("k_prefix", x["kp"][:5]), ("v_prefix", None), ("own_len", x["lens"].long()),
                      ("own_len", x["lens"].cpu()), ("own_len", i32([1] * 6)[::2]), ("visible", x["lens"]),
                      ("q", torch.zeros(3, 2, 8, 128, dtype=BF, device="cuda")[..., ::2]), ("cache", None),
                      ("cache", dict(c, k=c["k"].int())), ("cache", dict(c, v_scales=c["v_scales"].cpu())),
                      ("cache", dict(c, k_scales=c["k"])), ("cache", dict(c, v=c["v"][:, :39]))]:
        with pytest.raises(ValueError):
            att.attend(**dict(good, **{name: bad}))
    odd = torch.zeros(3 * 2 * 8 * 64 + 1, dtype=BF, device="cuda")[1:].view(3, 2, 8, 64)
    for bad in (dict(good, q=odd), dict(good, own_len=None), dict(good, scale=-1.0)):
        with pytest.raises(B.BriskError):
            att.attend(**bad)
    with pytest.raises(KeyError):
        att.attend(**dict(good, cache={"k": c["k"]}))
    for bad in ((k.float(), k, start), (k, k[:, :4], start), (k, k, start.long()), (k, k, start, start[:2])):
        with pytest.raises(ValueError):
            att.store(c, *bad)
    with pytest.raises(ValueError):
        att.load(c, 5, start.long())
    for call in (lambda: att.store(c, k[:, :0], k[:, :0], start), lambda: att.load(c, 0, start),
                 lambda: att.store(c, k, k, None), lambda: att.load(c, 5, None)):
        with pytest.raises(B.BriskError):
            call()
    assert att.device_status() == B.OK


# Streams come from a pool of 32 in turn, so that one may be another test's capture stream: these take theirs from the other
# pool, and leave the turns of the tests behind them as they are.
def test_calls_in_their_usual_form_captured(B):
    """Results that the calls allocate while they are captured are the graph's, and are written by every replay."""
    Bn, L, S, H, D = 2, 3, 90, 2, 80
    att = B.PackedAttention(Bn, L, 4, H, D, 33, S, BF)
    x = make(Bn, L, 4, H, D, 33, S, BF, [70, 12])
    rows = {n: spread_rows((Bn, L, H, D), BF, i).cuda() for i, n in enumerate("kv")}
    start = i32([5, 0])
    att.store(x["cache"], rows["k"], rows["v"], start)
    torch.cuda.synchronize()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream(priority=-1)
    with torch.cuda.graph(g, stream=s):
        att.store(x["cache"], rows["k"], rows["v"], start)
        r = att.attend(x["q"], x["kp"], x["vp"], x["cache"], x["lens"])
        back = att.load(x["cache"], L, start)
    for turn in range(3):
        for m in "kv":
            rows[m].copy_(torch.randn(Bn, L, H, D).to(BF))
        start.copy_(i32([7 * turn, 30 * turn]))
        g.replay()
        torch.cuda.synchronize()
        assert att.device_status() == B.OK
        for m in "kv":
            assert (n64(back[m]) == P.values(*P.store(n64(rows[m])))).all()
            x[m] = P.values(*raw(x["cache"], m))
        compare(r, wanted(x, att.scale), x, S)


def test_calls_of_two_threads(B):
    """Two host threads, each with an object and a stream of its own."""
    import threading
    x = [make(3, 2, 8, 2, 64, 50, 200, BF, [200, 3, 77], seed=i) for i in range(2)]
    att = [att_of(B, y, 200) for y in x]
    want = [a.attend(y["q"], y["kp"], y["vp"], y["cache"], y["lens"]) for a, y in zip(att, x)]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        s = torch.cuda.Stream(priority=-1)
        with torch.cuda.stream(s):
            for _ in range(100):
                y = x[i]
                r = att[i].attend(y["q"], y["kp"], y["vp"], y["cache"], y["lens"])
                s.synchronize()
                if not (torch.equal(r["out"], want[i]["out"]) and torch.equal(r["lse"], want[i]["lse"])):
                    wrong.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
