"""A context cache held in 4 bits: entries quantised as they are written, read back, and attended over.

The own caches of a batch (see operators.py beside this file) fill memory and bandwidth; held in 4 bits
they take 3.6 times fewer bytes. ``kind`` names what a serving program does:

  write    PackedAttention.store, then .load of the same places: a block's keys and values, or a prompt's, are
           quantised into the cache, and what they stand for from now on comes back
  read     PackedAttention.load: a run of every sequence's entries read back
  attend   PackedAttention.attend: queries over the shared prefix (unquantised) and the caches in 4 bits

Format: a row is the D channels of an entry and key head, in groups of 16. A group has a scale s, a byte
that holds bits 14 to 7 of a positive fp16 number (5 bits of exponent, 3 of the significand), and a
channel a code, two a byte (the even channel in the low half): a sign bit over the index of one of the
magnitudes 0, .5, 1, 1.5, 2, 3, 4, 6. The channel's value is that times s. Codes are [B, S, Hkv, D / 2]
bytes, scales [B, S, Hkv, 4] (up to 64 channels) or [B, S, Hkv, 8]. Of a group whose largest magnitude is
a, s is a / 6 rounded to 4 significant bits (nearest, ties to even) within 2^-14 .. 10240, and a channel
gets the nearest value (ties to the even index).

Sizes: as in operators.py; T rows are written or read from place ``start[b]`` on, ``count[b]`` of them
between ``lo`` and ``hi`` (attend: entries in use). ``order`` says how the cache lies in memory, "token"
[B, S, Hkv, ..] or "head" [B, Hkv, S, ..]; ``fused``: keys and values that are written come side by side.
"""
import math

import torch

own = False

F32, F64, U8 = torch.float32, torch.float64, torch.uint8
CHUNK = 1 << 28          # scores, or values, held at once while plain or exact values are made


def _case(name, kind, B, L, Hq, Hkv, D, P, S, lo, hi, dtype="bf16", order="token", mask="causal", T=0,
          fused=False):
    return {"name": name, "kind": kind, "B": B, "L": L, "Hq": Hq, "Hkv": Hkv, "D": D, "P": P, "S": S,
            "lo": lo, "hi": hi, "dtype": dtype, "order": order, "mask": mask, "T": T, "fused": fused}


def listed():
    return [
        # one sequence's committed token
        _case("write_one_token", "write", 1, 1, 8, 8, 128, 0, 512, 1, 1, T=1),
        # the throughput server's block step: 32 positions of 128 sequences, from a fused projection
        _case("write_block", "write", 128, 1, 8, 8, 128, 0, 1024, 32, 32, T=32, fused=True),
        # long prompts of 16 sequences of different lengths
        _case("write_prompt", "write", 16, 1, 8, 8, 128, 0, 4200, 1500, 4096, T=4096, order="head"),
        # fp32, one key head, odd sizes, some sequences write nothing
        _case("write_fp32", "write", 37, 1, 1, 1, 80, 0, 911, 0, 53, "f32", T=53),
        # every sequence's cache read back whole, before it is cut or handed on
        _case("read_caches", "read", 64, 1, 8, 8, 128, 0, 2048, 512, 2048, T=2048),
        # fp32, odd sizes, caches by head
        _case("read_fp32", "read", 9, 1, 3, 3, 112, 0, 2999, 0, 1777, "f32", "head", T=1777),
        # one sequence, one token: a chat's first answers, bound by launches and latency
        _case("attend_one_token", "attend", 1, 1, 32, 8, 128, 512, 256, 100, 100, mask="all"),
        # one sequence's token behind a document
        _case("attend_long_token", "attend", 1, 1, 32, 8, 128, 0, 131072, 130001, 130001, order="head", mask="all"),
        # a throughput server's verification of single tokens: the caches fill the memory bus
        _case("attend_256_tokens", "attend", 256, 1, 32, 8, 128, 2048, 2048, 512, 2048, mask="all"),
        # the throughput server's block step
        _case("attend_128_blocks", "attend", 128, 32, 32, 8, 128, 2048, 2048, 512, 2048, order="head"),
        # seven query heads a key head, odd lengths, blocks of seven with padding
        _case("attend_ragged", "attend", 13, 7, 28, 4, 80, 3001, 777, 0, 777, mask="idle"),
        # the smallest model unquantised, as in evaluation
        _case("attend_fp32", "attend", 4, 8, 8, 8, 64, 1000, 300, 17, 300, "f32", "head"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["write", "write", "read", "attend", "attend", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    Hkv = rng.choice([1, 2, 4, 8, 8, 8])
    Hq = Hkv * (rng.choice([1, 2, 4, 4, 4, 5, 7, 8, 16]) if kind == "attend" else 1)
    D = rng.choice([64, 128, 128, 128, 16 * rng.randint(1, 8)])
    B = _log_int(rng, 1, 256)
    S = _log_int(rng, 16, 16384)
    P = rng.choice([0, _log_int(rng, 1, 8192), _log_int(rng, 1, 8192)]) if kind == "attend" else 0
    L, T = 1, 0
    part = 1.0 if dtype == "bf16" else 0.25
    if kind == "attend":
        # no more than the largest listed cases: 0.75 GB of codes, 0.22 TFLOP (fp32: less)
        L = rng.choice([1, 1, _log_int(rng, 2, 64), _log_int(rng, 2, 64)])
        B = max(1, min(B, int(part * 6.7e8 / (S * Hkv * D))))
        B = max(1, min(B, int(part * part * 2.2e11 / (4.0 * L * Hq * (P + S) * D))))
    else:
        T = _log_int(rng, 1, S)
        B = max(1, min(B, int(part * 6.7e7 / (T * Hkv * D)), int(1.0e9 / (S * Hkv * D))))
    most = T or S
    hi = rng.randint((most + 1) // 2, most)
    lo = rng.randint(0, hi) if B > 1 else hi
    c = _case("", kind, B, L, Hq, Hkv, D, P, S, lo, hi, dtype, rng.choice(["token", "head"]),
              rng.choice(["all", "causal", "causal", "idle"]), T, rng.random() < 0.5)
    del c["name"]
    return c


# ---------------------------------------------------------------- the format, plainly

def _scale_bytes(D):
    return 4 if D <= 64 else 8


def _levels(dev):
    return torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], device=dev)


def _pack(x):
    """Codes [.., D / 2] and scales [.., 4 or 8] (bytes) of rows [.., D]."""
    D = x.shape[-1]
    g = x.float().unflatten(-1, (D // 16, 16))
    s = (g.abs().amax(-1) / 6).clamp_(2.0 ** -14, 10240.0)
    bits = s.view(torch.int32)
    bits = (bits + 0x7ffff + ((bits >> 20) & 1)) >> 20        # exponent and 3 bits, to nearest even
    s = (bits << 20).view(F32).unsqueeze(-1)
    a = g.abs()
    idx = torch.zeros(a.shape, dtype=U8, device=x.device)
    for i, mid in enumerate((.25, .75, 1.25, 1.75, 2.5, 3.5, 5.)):      # (mid * s is exact)
        idx += (a >= mid * s) if i % 2 else (a > mid * s)
    idx += torch.signbit(g).to(U8) * 8
    idx = idx.flatten(-2)
    codes = idx[..., 0::2] + idx[..., 1::2] * 16
    scales = torch.zeros((*x.shape[:-1], _scale_bytes(D)), dtype=U8, device=x.device)
    scales[..., :D // 16] = (bits - (112 << 3)).to(U8)
    return codes, scales


def _unpack(codes, scales):
    """The fp32 values [.., D] that codes and scales stand for."""
    D = codes.shape[-1] * 2
    idx = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()
    mag = _levels(codes.device)[idx & 7]
    val = torch.where(idx > 7, -mag, mag).unflatten(-1, (D // 16, 16))
    b = scales[..., :D // 16].int().clamp(max=226)
    s = torch.where(b < 8, b.float() * 2.0 ** -17, ((b + (112 << 3)) << 20).view(F32))
    return (val * s.unsqueeze(-1)).flatten(-2)


# ---------------------------------------------------------------- inputs

def _dt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else F32


def _spread(c):
    """Rows or entries of the B sequences, evenly from lo to hi (the seed shuffles them)."""
    B, lo, hi = c["B"], c["lo"], c["hi"]
    return [hi if B == 1 else lo + (hi - lo) * b // (B - 1) for b in range(B)]


def _rows(shape, D, tilt, g, dev):
    """Rows as projections give them: a few channels are several times larger than the others."""
    return torch.randn((*shape, D), generator=g, device=dev) * tilt


def _tilt(Hkv, D, g, dev):
    t = torch.rand((Hkv, D), generator=g, device=dev)
    return torch.where(t > 0.95, 4.0 * t, 0.5 + t) * 0.8


def _packed(c, tilts, first, g, dev):
    """A cache of random entries, in the memory order of the case."""
    B, S, Hkv, D = c["B"], c["S"], c["Hkv"], c["D"]
    cache = {}
    for name, tilt in zip("kv", tilts):
        lead = (B, Hkv, S) if c["order"] == "head" else (B, S, Hkv)
        codes = torch.empty((*lead, D // 2), dtype=U8, device=dev)
        scales = torch.empty((*lead, _scale_bytes(D)), dtype=U8, device=dev)
        if c["order"] == "head":
            codes, scales = codes.transpose(1, 2), scales.transpose(1, 2)
        run = max(1, CHUNK // (S * Hkv * D))
        many = max(1, CHUNK // (Hkv * D))
        for b in range(0, B, run):
            for t in range(0, S, many):
                n, m = min(run, B - b), min(many, S - t)
                x = _rows((n, m, Hkv), D, tilt, g, dev)
                if t == 0 and name == "k" and first is not None:
                    x[:, 0] = first
                codes[b:b + n, t:t + m], scales[b:b + n, t:t + m] = _pack(x)
        cache[name], cache[name + "_scales"] = codes, scales
    return cache


def _inputs(c, seed):
    """Everything that the call reads, made from the seed alone. Scores have a spread of about
    1.5, and every head has a direction of its own that the first entry of the context answers to
    (the sink that takes part of the attention in a trained model)."""
    dev = torch.device("cuda")
    g = torch.Generator(dev).manual_seed(int(seed))
    B, L, Hq, Hkv, D, P, S, T = (c[k] for k in ("B", "L", "Hq", "Hkv", "D", "P", "S", "T"))
    dt = _dt(c)
    lens = torch.tensor(_spread(c), dtype=torch.int32, device=dev)
    lens = lens[torch.randperm(B, generator=g, device=dev)].contiguous()
    tilts = [_tilt(Hkv, D, g, dev) for _ in range(2)]
    if c["kind"] != "attend":
        at = torch.rand((B,), generator=g, device=dev) * (S - lens + 1)
        x = {"count": lens, "start": at.floor().int().clamp(max=S).minimum(S - lens).contiguous()}
        if c["kind"] == "read":
            x["cache"] = _packed(c, tilts, None, g, dev)
        elif c["fused"]:
            kv = torch.empty((B, T, 2, Hkv, D), dtype=dt, device=dev)
            kv.copy_(_rows((B, T, 2, Hkv), D, torch.stack(tilts), g, dev))
            x["k"], x["v"] = kv.select(2, 0), kv.select(2, 1)
        else:
            x["k"], x["v"] = (_rows((B, T, Hkv), D, tilt, g, dev).to(dt) for tilt in tilts)
        return x
    x = {"own_len": lens}
    lean = torch.randn((Hkv, 1, D), generator=g, device=dev)
    q = torch.randn((B, L, Hkv, Hq // Hkv, D), generator=g, device=dev) * 1.5 + 0.5 * lean
    x["q"] = q.view(B, L, Hq, D).to(dt)
    first = 1.5 * lean[:, 0]
    x["k_pre"] = x["v_pre"] = None
    if P:
        x["k_pre"], x["v_pre"] = (_rows((P, Hkv), D, tilt, g, dev).to(dt) for tilt in tilts)
        x["k_pre"][0] = first.to(dt)
    x["cache"] = _packed(c, tilts, None if P else first, g, dev)
    at = torch.arange(L, device=dev, dtype=torch.int32)
    vis = (lens[:, None] - L + 1 + at).clamp_(min=0)
    if c["mask"] == "idle":
        used = torch.randint(1, L + 1, (B, 1), generator=g, device=dev)
        vis = torch.where(at < used, vis, torch.full_like(vis, -1))
    x["visible"] = None if c["mask"] == "all" else vis.contiguous()
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    x["case"] = case
    if own:
        from paper_2609_33390_gb300 import brisk
        c = case
        x["att"] = brisk.PackedAttention(c["B"], c["L"], c["Hq"], c["Hkv"], c["D"], c["P"], c["S"],
                                         _dt(c))
        if c["kind"] == "write":
            x["cache"] = x["att"].alloc_cache(c["order"])
    return x


# ---------------------------------------------------------------- plain forms

def _live(x, T):
    return (torch.arange(T, device=x["count"].device) < x["count"][:, None])[..., None, None]


def _plain_write(c, x):
    put = {}
    for name in ("k", "v"):
        rows = torch.zeros_like(x[name], memory_format=torch.contiguous_format)
        run = max(1, CHUNK // (c["T"] * c["Hkv"] * c["D"]))
        for b in range(0, c["B"], run):
            r = _unpack(*_pack(x[name][b:b + run]))
            rows[b:b + run] = r.to(rows.dtype)
        put[name] = torch.where(_live(x, c["T"]), rows, torch.zeros_like(rows))
    return put


def _plain_read(c, x):
    T, dev = c["T"], x["count"].device
    at = torch.minimum(x["start"][:, None].long() + torch.arange(T, device=dev), torch.tensor(c["S"] - 1, device=dev))
    run = max(1, CHUNK // (T * c["Hkv"] * c["D"]))
    put = {}
    for name in ("k", "v"):
        rows = torch.empty((c["B"], T, c["Hkv"], c["D"]), dtype=_dt(c), device=dev)
        for b in range(0, c["B"], run):
            pick = [x["cache"][n][b:b + run].gather(1, at[b:b + run, :, None, None].expand(
                -1, -1, c["Hkv"], x["cache"][n].shape[-1])) for n in (name, name + "_scales")]
            r = _unpack(*pick)
            rows[b:b + run] = r.to(rows.dtype)
        put[name] = torch.where(_live(x, T), rows, torch.zeros_like(rows))
    return put


def _parts(c):
    """Runs of sequences whose scores and values fit the room for them."""
    one = max(c["L"] * c["Hq"] * max(1, c["P"] + c["S"]), c["S"] * c["Hkv"] * c["D"])
    n = max(1, CHUNK // one)
    return [(b, min(c["B"], b + n)) for b in range(0, c["B"], n)]


def _plain_attend(c, x):
    B, L, Hq, Hkv, D, P, S = (c[k] for k in ("B", "L", "Hq", "Hkv", "D", "P", "S"))
    G, dev = Hq // Hkv, x["q"].device
    out = torch.empty((B, L, Hq, D), dtype=_dt(c), device=dev)
    lse = torch.empty((B, L, Hq), device=dev)
    if P:
        kp, vp = x["k_pre"].float().permute(1, 2, 0), x["v_pre"].float().transpose(0, 1)
    for b0, b1 in _parts(c):
        n = b1 - b0
        limit = x["own_len"][b0:b1, None].expand(-1, L)
        live = torch.ones((n, L), dtype=torch.bool, device=dev)
        if x["visible"] is not None:
            live = x["visible"][b0:b1] >= 0
            limit = torch.minimum(limit, x["visible"][b0:b1])
        seen = torch.arange(S, device=dev) < limit[..., None]
        k, v = (_unpack(x["cache"][m][b0:b1], x["cache"][m + "_scales"][b0:b1]) for m in "kv")
        q = x["q"][b0:b1].float().view(n, L, Hkv, G, D)
        qo = q.permute(0, 2, 1, 3, 4).reshape(n, Hkv, L * G, D)
        s = (qo @ k.permute(0, 2, 3, 1) / math.sqrt(D)).view(n, Hkv, L, G, S)
        s.masked_fill_(~seen[:, None, :, None, :], -math.inf)
        m = s.amax(4, keepdim=True)
        if P:
            qp = q.view(n * L, Hkv, G, D).transpose(0, 1).reshape(Hkv, -1, D)
            sp = (qp @ kp / math.sqrt(D)).view(Hkv, n, L, G, P)
            m = torch.maximum(m, sp.amax(4, keepdim=True).transpose(0, 1))
        m = m.clamp_(min=-1e30)
        e = s.sub_(m).exp_()
        z = e.sum(4, keepdim=True)
        o = (e.view(n, Hkv, L * G, S) @ v.transpose(1, 2)).view(n, Hkv, L, G, D)
        if P:
            e = sp.sub_(m.transpose(0, 1)).exp_()
            z = z + e.sum(4, keepdim=True).transpose(0, 1)
            o = o + (e.view(Hkv, -1, P) @ vp).view(Hkv, n, L, G, D).transpose(0, 1)
        live = live[:, None, :, None, None] & (z > 0)
        o = torch.where(live, o / z, torch.zeros_like(o))
        ls = torch.where(live, m + z.log(), torch.full_like(z, -math.inf))
        out[b0:b1] = o.permute(0, 2, 1, 3, 4).reshape(n, L, Hq, D).to(out.dtype)
        lse[b0:b1] = ls[..., 0].permute(0, 2, 1, 3).reshape(n, L, Hq)
    return {"out": out, "lse": lse}


def run(state):
    x, c = state, state["case"]
    kind = c["kind"]
    if not own:
        return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}[kind](c, x)
    att = x["att"]
    if kind == "attend":
        return att.attend(x["q"], x["k_pre"], x["v_pre"], x["cache"], x["own_len"], visible=x["visible"])
    if kind == "write":
        att.store(x["cache"], x["k"], x["v"], x["start"], x["count"])
    return att.load(x["cache"], c["T"], x["start"], x["count"])


# ---------------------------------------------------------------- what is counted

def work(case):
    """Bytes: the entries in use and the queries once, the outputs once (written entries go into the cache and
    come back). Flops: the products of the entries in use (what a causal block hides of itself is counted: it is
    at most L entries); for a written element about the ten steps of its quantisation."""
    c = case
    B, L, Hq, Hkv, D, P, T = (c[k] for k in ("B", "L", "Hq", "Hkv", "D", "P", "T"))
    size = 2 if c["dtype"] == "bf16" else 4
    used, rows, packed = sum(_spread(c)), B * L * Hq, D // 2 + D // 16
    if c["kind"] == "attend":
        return {"bytes": 2 * P * Hkv * D * size + 2 * used * Hkv * packed + 2 * rows * D * size + rows * 4 + B * 4,
                "flops": 4 * D * L * Hq * (B * P + used) + 5 * L * Hq * (B * P + used)}
    back = 2 * used * Hkv * packed + 2 * B * T * Hkv * D * size + 8 * B
    if c["kind"] == "read":
        return {"bytes": back, "flops": 2 * used * Hkv * D}
    return {"bytes": back + 2 * used * Hkv * (D * size + packed), "flops": 2 * used * Hkv * D * 11}


# ---------------------------------------------------------------- 64-bit values

_GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _value64(codes, scales):
    """What a cache's rows stand for, in 64 bits: sign and magnitude by the bits' own arithmetic."""
    n, D = codes.shape[-1], codes.shape[-1] * 2
    out = torch.empty((*codes.shape[:-1], D), dtype=F64, device=codes.device)
    byte = scales[..., :D // 16].double().clamp(max=226)
    e = torch.floor(byte / 8)
    frac = byte - 8 * e
    s = torch.where(e > 0, (1 + frac / 8) * torch.exp2(e - 15), frac / 8 * 2.0 ** -14)
    s = s.repeat_interleave(16, -1)
    for half in (0, 1):
        c = (codes if half == 0 else codes.div(16, rounding_mode="floor")).remainder(16).double()
        sign, c = torch.where(c >= 8, -1.0, 1.0), c.remainder(8)
        ex, mant = torch.floor(c / 2), c.remainder(2)
        mag = torch.where(ex > 0, (1 + mant / 2) * torch.exp2(ex - 1), mant / 2)
        out[..., half::2] = sign * mag * s[..., half::2]
    return out


def _quantised64(x):
    """The nearest values that the format holds, by the definition."""
    D = x.shape[-1]
    g = x.double().unflatten(-1, (D // 16, 16))
    top = g.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top / 6)                               # m in [1/2, 1): 4 significant bits of it
    s = torch.ldexp(torch.round(m * 16) / 16, e).clamp(2.0 ** -14, 10240.0)
    r = g.abs() / s
    best, far = torch.zeros_like(r), r.clone()
    for i, v in enumerate(_GRID):                             # the nearest; of two, the even one
        d = (r - v).abs()
        nearer = (d < far) | ((d == far) & (i % 2 == 0))
        best, far = torch.where(nearer, torch.full_like(best, v), best), torch.where(nearer, d, far)
    return (torch.sign(g) * best * s).flatten(-2)


def exact(case, seed):
    c = case
    x = _inputs(c, seed)
    B, L, Hq, Hkv, D, P, S, T = (c[k] for k in ("B", "L", "Hq", "Hkv", "D", "P", "S", "T"))
    G = Hq // Hkv
    if c["kind"] != "attend":
        dev = x["count"].device
        put = {n: torch.zeros((B, T, Hkv, D), dtype=F64, device=dev) for n in ("k", "v")}
        for b in range(B):
            n, at = int(x["count"][b]), int(x["start"][b])
            for name in ("k", "v"):
                if n and c["kind"] == "write":
                    put[name][b, :n] = _quantised64(x[name][b, :n])
                elif n:
                    put[name][b, :n] = _value64(x["cache"][name][b, at:at + n],
                                                x["cache"][name + "_scales"][b, at:at + n])
        return put
    dev = x["q"].device
    out = torch.zeros((B, L, Hq, D), dtype=F64, device=dev)
    lse = torch.full((B, L, Hq), -math.inf, dtype=F64, device=dev)
    for b in range(B):
        n = int(x["own_len"][b])
        k, v = (_value64(x["cache"][m][b, :n], x["cache"][m + "_scales"][b, :n]) for m in "kv")
        if P:
            k, v = torch.cat([x["k_pre"].double(), k]), torch.cat([x["v_pre"].double(), v])
        if P + n == 0:
            continue
        see = torch.full((L,), P + n, device=dev)
        if x["visible"] is not None:
            vis = x["visible"][b].long()
            see = torch.where(vis < 0, 0, P + vis.clamp(max=n))
        see = see.repeat_interleave(G)[:, None] > torch.arange(P + n, device=dev)
        any_ = see.any(1)
        q = x["q"][b].double().reshape(L, Hkv, G, D).transpose(0, 1).reshape(Hkv, L * G, D)
        for h in range(Hkv):
            s = (q[h] @ k[:, h].T * D ** -0.5).masked_fill(~see, -math.inf)
            ls = torch.logsumexp(s, 1)
            p = torch.where(see, torch.exp(s - torch.where(any_, ls, torch.zeros_like(ls))[:, None]), 0.0)
            heads = slice(h * G, (h + 1) * G)
            out[b, :, heads] = (p @ v[:, h]).view(L, G, D)
            lse[b, :, heads] = ls.view(L, G)
    return {"out": out, "lse": lse}
