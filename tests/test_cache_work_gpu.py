"""Attention and its weights where the work is divided over all SMs, against a float64 torch form on the
GPU: several row tiles a head, key tiles divided between CTAs and not, rows whose parts one
kernel or another joins, fragments of every length; tolerances as derived in test_cache_gpu.py."""
import pytest
import torch

from test_cache_gpu import BF, F32, U, caches
from test_cache_gpu import check_evict, make
from test_cache_gpu import test_hidden_entries_do_not_reach_the_rows as hidden_entries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2609_33390_gb300 import build
    build.build()
    from paper_2609_33390_gb300 import brisk as B
    return B


def inputs(Bn, L, Hq, Hkv, D, P, S, lens, mask, dt, order="token", seed=0):
    g = torch.Generator().manual_seed(seed)
    x = {"q": torch.randn(Bn, L, Hq, D, generator=g).to(dt).cuda()}
    x["kp"], x["vp"] = caches((), P, Hkv, D, order, dt, g) if P else (None, None)
    x["ko"], x["vo"] = caches((Bn,), S, Hkv, D, order, dt, g) if S else (None, None)
    x["lens"] = torch.tensor(lens, dtype=torch.int32).cuda()
    vis = None
    if mask:
        n = torch.tensor(lens)[:, None]
        vis = (n - L + 1 + torch.arange(L)).clamp(min=0)
        odd = torch.rand(Bn, L, generator=g)
        vis = torch.where(odd < 0.05, torch.full_like(vis, -1), vis)                     # padding
        vis = torch.where(odd > 0.9, (torch.rand(Bn, L, generator=g) * (n + 2)).long(), vis)
        vis = vis.int().cuda()
    x["vis"] = vis
    return x


def attend64(x, scale):
    """out, lse, sum p |v|, largest sum |q_d k_d| by rows; also the own entries' weights by (b, h)."""
    q = x["q"].double()
    Bn, L, Hq, D = q.shape
    kp, vp, ko, vo = (None if x[n] is None else x[n].double() for n in ("kp", "vp", "ko", "vo"))
    Hkv = (ko if kp is None else kp).shape[-2]
    G, P, S = Hq // Hkv, 0 if kp is None else kp.shape[0], 0 if ko is None else ko.shape[1]
    out, mass, = torch.zeros_like(q), torch.zeros_like(q)
    big, lse = torch.zeros(Bn, L, Hq, device="cuda", dtype=torch.float64), None
    lse = torch.full_like(big, -float("inf"))
    acc = torch.zeros(Bn, Hkv, S, device="cuda", dtype=torch.float64)
    for b in range(Bn):
        n = int(x["lens"][b])
        seen = torch.full((L,), n, device="cuda") if x["vis"] is None else x["vis"][b].long().clamp(max=n)
        pad = seen < 0
        cols = torch.arange(P + n, device="cuda")
        hide = (cols[None] >= P + seen.clamp(min=0)[:, None]) | pad[:, None]             # [L, P + n]
        for h in range(Hkv):
            rows = q[b, :, h * G:(h + 1) * G].reshape(L * G, D)
            k = torch.cat([t for t in ((kp[:, h] if P else None), (ko[b, :n, h] if S else None)) if t is not None])
            v = torch.cat([t for t in ((vp[:, h] if P else None), (vo[b, :n, h] if S else None)) if t is not None])
            if k.shape[0] == 0:
                continue
            s = (scale * rows @ k.T).masked_fill(hide.repeat_interleave(G, 0), -float("inf"))
            l = torch.logsumexp(s, 1)
            p = torch.exp(s - torch.where(l == -float("inf"), 0.0, l)[:, None])
            put = lambda to, w: to[b, :, h * G:(h + 1) * G].copy_(w.view(L, G, *w.shape[1:]))
            put(out, p @ v), put(mass, p @ v.abs()), put(lse, l)
            put(big, scale * (rows.abs() @ k.abs().T).amax(1))
            acc[b, h, :n] = p[:, P:].sum(0)
    return out, lse, mass, big, acc


def check(B, x, S, decay=0.5):
    Bn, L, Hq, D = x["q"].shape
    P = 0 if x["kp"] is None else x["kp"].shape[0]
    Hkv = (x["ko"] if x["kp"] is None else x["kp"]).shape[-2]
    dt, n = x["q"].dtype, P + S
    att = B.PrefixAttention(Bn, L, Hq, Hkv, D, P, S, dt)
    att.workspace.fill_(0xff)                          # nothing is expected of it
    out, lse, mass, big, acc = attend64(x, att.scale)
    for _ in range(2):                                 # (and nothing of a call is left for the next)
        r = att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"], visible=x["vis"])
        assert att.device_status() == B.OK
        eps = (2 * D + 16) * U * big + 2.0 ** -21
        none = torch.isneginf(lse)
        assert torch.equal(torch.isneginf(r["lse"]), none) and (r["out"][none] == 0).all()
        tol = eps + n * U + 2.0 ** -22 * lse.masked_fill(none, 0).abs()
        assert ((r["lse"].double() - lse).masked_fill(none, 0).abs() <= tol).all()
        tol = (2 * eps + 2 * n * U)[..., None] * mass
        if dt == BF:
            tol += 2.0 ** -9 * mass * (1 + 2.0 ** -7) + 2.0 ** -8 * out.abs()
        else:
            tol += 2.0 ** -22 * out.abs()
        assert ((r["out"].double() - out).abs() <= tol + 1e-30).all()
    if S == 0:
        return
    old = torch.rand(Bn, Hkv, S, device="cuda")
    got = att.weights(x["q"], r["lse"], x["ko"], x["lens"], acc=old, decay=decay, visible=x["vis"])
    assert att.device_status() == B.OK
    used = torch.arange(S, device="cuda") < x["lens"][:, None, None]
    want = acc + decay * old.double() * used
    # the kernel's log-sums, not the exact ones: their error counts twice
    top = lse.masked_fill(none, 0).abs().max()
    rows = L * Hq // Hkv
    rel = 2 * ((2 * D + 16) * U * big.max() + 2.0 ** -21 + 4 * U * top) + (rows + n + 4) * U
    assert ((got.double() - want).abs() <= rel * want + 1e-30).all()
    assert (got[~used.expand_as(got)] == 0).all()


def lens_of(Bn, S, step=37):
    """Lengths of every kind: none, one, around the tiles' ends, all."""
    some = [S, 0, min(S, 1), min(S, 128), min(S, 129), min(S, 127), S // 2]
    return [some[i] if i < len(some) else (i * step) % (S + 1) for i in range(Bn)]


BF_SIZES = [
    # B, L, Hq, Hkv, D, P, S
    (5, 32, 32, 8, 128, 2001, 700),       # several row tiles a head, the last one half full
    (9, 33, 32, 8, 128, 2001, 700),       # 5 row tiles, 4 or 5 units a CTA
    (40, 8, 16, 4, 64, 4000, 300),        # narrow heads, 5 row tiles
    (40, 8, 12, 4, 40, 5000, 90),
    (40, 16, 64, 32, 72, 384, 200),       # whole items a CTA: the items divided at the CTAs' ends alone
    (40, 16, 64, 32, 72, 384, 0),         # and no own entries
    (300, 1, 32, 8, 128, 4096, 150),      # single tokens
    (1025, 1, 16, 8, 64, 1300, 20),
    (30, 4, 8, 2, 128, 1000, 500),        # several row tiles over the prefix, few units
    (9, 1, 28, 4, 120, 6000, 4000),       # all rows of a head in a slot, long caches
    (2, 64, 8, 2, 128, 0, 3100),          # own entries alone, two row tiles a sequence
    (3, 100, 12, 2, 104, 300, 1500),      # row tiles of a sequence that end inside
    (16, 75, 32, 8, 64, 0, 2600),         # the weights' blocks of queries take turns on several runs of key tiles
]


@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("size", BF_SIZES)
def test_divided_work_bf16(B, size, mask):
    Bn, L, Hq, Hkv, D, P, S = size
    check(B, inputs(*size, lens_of(Bn, S), mask, BF), S)


@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("order", ["head", "fused"])
def test_divided_work_in_other_orders(B, order, mask):
    size = (6, 33, 24, 8, 128, 1900, 260)
    check(B, inputs(*size, lens_of(6, 260), mask, BF, order=order), 260)


@pytest.mark.parametrize("mask", [False, True])
def test_one_sequence_much_longer_than_the_others(B, mask):
    """Its own entries are divided into more parts than the prefix's kernel joins; the others' are not."""
    size = (40, 16, 64, 32, 72, 384, 6000)
    lens = [0 if i % 3 == 0 else 50 + i for i in range(40)]
    lens[17] = 6000
    check(B, inputs(*size, lens, mask, BF), 6000)


@pytest.mark.parametrize("mask", [False, True])
@pytest.mark.parametrize("size", [
    (7, 20, 15, 5, 64, 1500, 900),
    (64, 1, 8, 4, 128, 900, 400),
    (2, 50, 12, 3, 96, 0, 1000),
    (50, 20, 10, 10, 24, 130, 70),
    (3, 1, 1, 1, 8, 5000, 3000),
    (4, 1, 2, 1, 128, 700, 5000),         # up to 8 rows: keys and values straight from memory
    (9, 2, 14, 7, 72, 40, 2000),
    (30, 1, 20, 4, 104, 0, 777),
    (5, 3, 4, 2, 40, 3000, 1025),
    (6, 2, 16, 4, 64, 2001, 600),
    (1, 1, 7, 1, 120, 9000, 9000),
    (5, 5, 10, 5, 56, 300, 400),          # 10
])
def test_divided_work_fp32(B, size, mask):
    Bn, L, Hq, Hkv, D, P, S = size
    check(B, inputs(*size, lens_of(Bn, S), mask, F32), S)


@pytest.mark.parametrize("L,G", [(2, 1), (2, 2), (4, 2)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_hidden_entries_with_few_rows(B, bad, L, G):
    hidden_entries(B, bad, L, G, F32)


@pytest.mark.parametrize("kind", ["random", "ties", "special"])
@pytest.mark.parametrize("S,keep,recent", [(90, 40, 7), (2700, 1100, 300), (5000, 4999, 0), (2100, 1, 1)])
def test_evict_of_many_sequences(B, S, keep, recent, kind):
    Bn, Hkv = 80, 4
    x = make(Bn, 1, Hkv, Hkv, 16, 0, S, BF, lens_of(Bn, S))
    g = torch.Generator().manual_seed(S)
    acc = torch.rand(Bn, Hkv, S, generator=g)
    if kind == "ties":
        acc = torch.floor(acc * 3)
    if kind == "special":
        pick = torch.randint(0, 8, acc.shape, generator=g)
        for j, v in enumerate((float("nan"), float("inf"), -float("inf"), 0.0, -0.0, 1e-45, -1.0)):
            acc = torch.where(pick == j, torch.tensor(v), acc)
    check_evict(B, x, acc.cuda(), S, keep, recent)


def test_two_handles_on_two_streams(B):
    """Calls side by side, each with its own workspace, give what they give alone."""
    sizes = [(20, 16, 32, 8, 128, 2000, 300), (70, 1, 32, 8, 128, 3000, 800)]
    xs = [inputs(*s, lens_of(s[0], s[6]), True, BF, seed=i) for i, s in enumerate(sizes)]
    atts = [B.PrefixAttention(*s, BF) for s in sizes]
    streams = [torch.cuda.Stream() for _ in sizes]

    def run(i, stream=None):
        x, a = xs[i], atts[i]
        r = a.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"], visible=x["vis"], stream=stream)
        w = a.weights(x["q"], r["lse"], x["ko"], x["lens"], visible=x["vis"], stream=stream)
        e = a.evict(x["ko"], x["vo"], w, x["lens"], 200, 50, stream=stream)
        return [r["out"], r["lse"], w, *e.values()]

    alone = [run(i) for i in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [run(i, streams[i]) for i in range(2)]
        torch.cuda.synchronize()
        for a, g in zip(alone, got):
            assert all(torch.equal(s, t) for s, t in zip(a, g))
    assert all(a.device_status() == B.OK for a in atts)


@pytest.mark.parametrize("size", [
    (4, 16, 32, 8, 128, 3000, 900),       # the prefix with the own entries
    (16, 32, 32, 8, 128, 3000, 900),      # the prefix by itself
    (4, 16, 16, 4, 64, 0, 3000),
])
def test_expired_waits_are_reported_and_the_next_call_is_right(B, size):
    Bn, L, Hq, Hkv, D, P, S = size
    x = inputs(*size, [S] * Bn, False, BF)
    att = B.PrefixAttention(*size, BF)
    run = lambda: att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"])
    sums = lambda r: att.weights(x["q"], r["lse"], x["ko"], x["lens"])
    ref = run()
    acc = sums(ref)
    assert att.device_status() == B.OK
    for call in (run, lambda: sums(ref)):
        prev = B.set_wait_limit(1)
        try:
            call()
            assert att.device_status() == B.ERR_TIMEOUT
        finally:
            B.set_wait_limit(prev)
        again = run()
        assert att.device_status() == B.OK
        acc2 = sums(again)
        assert att.device_status() == B.OK
        assert torch.equal(again["out"], ref["out"]) and torch.equal(again["lse"], ref["lse"]) and torch.equal(acc, acc2)


def test_calls_on_a_stream_do_not_wait_for_the_current_one(B):
    """What a call allocates is not written on the current stream, which may be far behind."""
    size = (3, 2, 8, 2, 64, 100, 60)
    x = inputs(*size, [60, 40, 5], False, BF)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def run(stream=None):
        att = B.PrefixAttention(*size, BF)
        if stream is not None:
            torch.cuda._sleep(20_000_000)              # about 10 ms of the current stream
        r = att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"], stream=stream)
        w = att.weights(x["q"], r["lse"], x["ko"], x["lens"], stream=stream)
        e = att.evict(x["ko"], x["vo"], w, x["lens"], 30, 5, stream=stream)
        torch.cuda.synchronize()
        assert att.device_status() == B.OK
        return [r["out"], r["lse"], w, *e.values()]

    for a, b in zip(run(), run(s)):
        assert torch.equal(a, b)
