"""Attention over a cache with a shared prefix, and the cache's eviction: what a serving program
that feeds the decode tail has them do.

A batch of sequences shares a long prefix (a system prompt, few-shot examples) whose keys and
values are held once; every sequence has a cache of its own behind it. A block step attends from
the L positions of every sequence's block, adds up how much attention each entry of the own caches
got, and now and then drops the entries that got least. ``kind`` names the call:

  attend   PrefixAttention.attend    queries [B, L, Hq, D] over the prefix and the own caches
  weights  PrefixAttention.weights   attention weight every own entry got, added to a running sum
  evict    PrefixAttention.evict     the entries of largest sums and the newest, moved together

Sizes: B sequences, L positions a block, Hq query heads over Hkv key heads of width D, P prefix
entries, room for S own entries a sequence of which ``lo`` to ``hi`` are in use. ``order`` says how
the caches lie in memory: "token" [.., S, Hkv, D], "head" [.., Hkv, S, D], "fused" keys and values
of a token side by side. ``mask``: "all" every position sees every own entry, "causal" the block's
positions see the block up to themselves, "idle" causal, and the last positions of some blocks are
padding that sees nothing at all.
"""
import math

import torch

own = False

F32, F64 = torch.float32, torch.float64
DECAY = 0.98
CHUNK = 1 << 29          # scores held at once while plain or exact values are made


def _case(name, kind, B, L, Hq, Hkv, D, P, S, lo, hi, dtype="bf16", order="token", mask="causal",
          keep=0, recent=0):
    return {"name": name, "kind": kind, "B": B, "L": L, "Hq": Hq, "Hkv": Hkv, "D": D, "P": P,
            "S": S, "lo": lo, "hi": hi, "dtype": dtype, "order": order, "mask": mask,
            "keep": keep, "recent": recent}


def listed():
    return [
        # one sequence, one token: a chat's first answers, bound by launches and latency
        _case("attend_one_token", "attend", 1, 1, 32, 8, 128, 512, 256, 100, 100, mask="all"),
        # one interactive sequence on a full-size model, block by block
        _case("attend_one_block", "attend", 1, 32, 32, 8, 128, 4096, 2048, 1100, 1100),
        # a throughput server's verification of single tokens: the own caches fill the memory bus
        _case("attend_256_tokens", "attend", 256, 1, 32, 8, 128, 2048, 2048, 512, 2048, mask="all"),
        # the throughput server's block step behind a long shared prefix: bound by the products
        _case("attend_128_stream", "attend", 128, 32, 32, 8, 128, 8192, 1024, 256, 1024),
        # seven query heads a key head, odd lengths, caches by head, blocks of seven with padding
        _case("attend_ragged", "attend", 13, 7, 28, 4, 128, 3001, 777, 0, 777, order="head",
              mask="idle"),
        # the smallest model unquantised, as in evaluation
        _case("attend_fp32", "attend", 4, 8, 8, 8, 64, 1000, 300, 17, 300, "f32", "fused"),
        # what a step's blocks looked at, one sequence
        _case("weights_one_block", "weights", 1, 32, 32, 8, 128, 0, 2048, 1100, 1100),
        # the same for the throughput server: every own key is read again
        _case("weights_128_stream", "weights", 128, 32, 32, 8, 128, 0, 4096, 1024, 4096),
        # fp32, one key head for all, odd sizes
        _case("weights_fp32", "weights", 6, 5, 12, 1, 80, 0, 1501, 0, 1501, "f32", "head", "idle"),
        # one sequence's cache cut back to its budget
        _case("evict_one", "evict", 1, 1, 32, 8, 128, 0, 2048, 2048, 2048, keep=1024, recent=64),
        # after a long prompt, every sequence of the batch to its budget; some are below it
        _case("evict_128", "evict", 128, 1, 32, 8, 128, 0, 4096, 1500, 4096, keep=2048, recent=256),
        # fp32, odd sizes, caches by head
        _case("evict_fp32", "evict", 9, 1, 6, 3, 72, 0, 2999, 100, 2999, "f32", "head",
              keep=777, recent=33),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "weights", "weights", "evict", "evict"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    Hkv = rng.choice([1, 2, 4, 8, 8, 8])
    Hq = Hkv * rng.choice([1, 2, 4, 4, 4, 5, 7, 8])
    D = rng.choice([64, 128, 128, 128, 8 * rng.randint(2, 16)])
    B = _log_int(rng, 1, 256)
    L = 1 if kind == "evict" else rng.choice([1, _log_int(rng, 2, 64), _log_int(rng, 2, 64)])
    P = _log_int(rng, 1, 16384) - 1 if kind == "attend" else 0
    S = _log_int(rng, 16, 8192)
    # no more than the largest listed cases: 2.1 GB a cache, 0.55 TFLOP (fp32: a tenth of both)
    part = 1.0 if dtype == "bf16" else 0.1
    B = max(1, min(B, int(part * 1.0e9 / (S * Hkv * D))))
    if kind != "evict":
        B = max(1, min(B, int(part * 5.5e11 / (4.0 * L * Hq * (P + S) * D))))
    hi = rng.randint((S + 1) // 2, S)
    lo = rng.randint(0, hi) if B > 1 else hi
    keep = recent = 0
    if kind == "evict":
        keep = _log_int(rng, 1, S)
        recent = rng.randint(0, keep)
    c = _case("", kind, B, L, Hq, Hkv, D, P, S, lo, hi, dtype,
              rng.choice(["token", "token", "head", "fused"]),
              rng.choice(["all", "causal", "causal", "idle"]), keep, recent)
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs

def _dt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else F32


def _spread(c):
    """Entries in use of the B sequences, evenly from lo to hi (the seed shuffles them)."""
    B, lo, hi = c["B"], c["lo"], c["hi"]
    return [hi if B == 1 else lo + (hi - lo) * b // (B - 1) for b in range(B)]


def _randn(shape, dt, g, dev, scale=1.0):
    t = torch.empty(shape, dtype=dt, device=dev)
    flat = t.view(-1)
    n = 1 << 27
    for s in range(0, flat.numel(), n):
        part = flat[s:s + n]
        part.copy_(torch.randn(part.shape, generator=g, device=dev) * scale)
    return t


def _caches(lead, S, Hkv, D, order, dt, g, dev):
    """Keys and values [*lead, S, Hkv, D] as views of how they lie in memory."""
    n = len(lead)
    if order == "fused":
        kv = _randn((*lead, S, 2, Hkv, D), dt, g, dev)
        return kv.select(n + 1, 0), kv.select(n + 1, 1)
    shape = (*lead, Hkv, S, D) if order == "head" else (*lead, S, Hkv, D)
    k, v = _randn(shape, dt, g, dev), _randn(shape, dt, g, dev)
    return (k.transpose(n, n + 1), v.transpose(n, n + 1)) if order == "head" else (k, v)


def _inputs(c, seed):
    """Everything that the call reads, made from the seed alone. Scores have a spread of about
    1.5, and every head has a direction of its own that the first entry of the context answers to
    (the sink that takes part of the attention in a trained model)."""
    dev = torch.device("cuda")
    g = torch.Generator(dev).manual_seed(int(seed))
    B, L, Hq, Hkv, D, P, S = (c[k] for k in ("B", "L", "Hq", "Hkv", "D", "P", "S"))
    dt = _dt(c)
    lens = torch.tensor(_spread(c), dtype=torch.int32, device=dev)
    lens = lens[torch.randperm(B, generator=g, device=dev)].contiguous()
    x = {"own_len": lens}
    x["k_own"], x["v_own"] = _caches((B,), S, Hkv, D, c["order"], dt, g, dev)
    if c["kind"] == "evict":
        # sums as they come about: most entries got little, a few got much; whole groups that got
        # nothing tie
        a = torch.rand((B, Hkv, S), generator=g, device=dev)
        x["acc"] = torch.where(a < 0.05, torch.zeros_like(a), a.pow(6) * 20)
        return x
    lean = torch.randn((Hkv, 1, D), generator=g, device=dev)
    q = torch.randn((B, L, Hkv, Hq // Hkv, D), generator=g, device=dev) * 1.5 + 0.5 * lean
    x["q"] = q.view(B, L, Hq, D).to(dt)
    first = (1.5 * lean[:, 0]).to(dt)
    if P:
        x["k_pre"], x["v_pre"] = _caches((), P, Hkv, D, c["order"], dt, g, dev)
        x["k_pre"][0] = first
    else:
        x["k_pre"] = x["v_pre"] = None
        x["k_own"][:, 0] = first
    at = torch.arange(L, device=dev, dtype=torch.int32)
    vis = (lens[:, None] - L + 1 + at).clamp_(min=0)
    if c["mask"] == "idle":
        used = torch.randint(1, L + 1, (B, 1), generator=g, device=dev)
        vis = torch.where(at < used, vis, torch.full_like(vis, -1))
    x["visible"] = None if c["mask"] == "all" else vis.contiguous()
    if c["kind"] == "weights":
        x["acc"] = torch.rand((B, Hkv, S), generator=g, device=dev)
        # the rows' log-sums as attention left them, over a prefix that took part of the weight
        lse = torch.empty((B, L, Hq), device=dev)
        for b0, b1 in _parts(c):
            s = _own_scores(c, x, b0, b1, F32)
            lse[b0:b1] = torch.logsumexp(s, 4).permute(0, 2, 1, 3).reshape(b1 - b0, L, Hq)
        x["lse"] = lse + torch.rand((B, L, Hq), generator=g, device=dev)
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    x["case"] = case
    if own:
        from paper_2609_33390_gb300 import brisk
        c = case
        x["att"] = brisk.PrefixAttention(c["B"], c["L"], c["Hq"], c["Hkv"], c["D"], c["P"], c["S"],
                                         _dt(c))
        if c["kind"] == "evict":
            x["spare"] = x["att"].alloc_evicted(c["keep"])
    return x


# ---------------------------------------------------------------- plain forms

def _parts(c):
    """Runs of sequences whose scores fit the room for them."""
    one = c["L"] * c["Hq"] * max(1, c["P"] + c["S"])
    n = max(1, CHUNK // one)
    return [(b, min(c["B"], b + n)) for b in range(0, c["B"], n)]


def _seen(c, x, b0, b1):
    """[n, L, S]: which own entries a position sees; [n, L]: which positions see anything."""
    S, dev = c["S"], x["q"].device
    lens, vis = x["own_len"][b0:b1], x["visible"]
    limit = lens[:, None].expand(-1, c["L"])
    live = torch.ones_like(limit, dtype=torch.bool)
    if vis is not None:
        live = vis[b0:b1] >= 0
        limit = torch.minimum(limit, vis[b0:b1])
    return torch.arange(S, device=dev) < limit[..., None], live


def _own_scores(c, x, b0, b1, dt):
    """[n, Hkv, L, G, S] scores over the own caches, hidden entries at minus infinity."""
    n, L, Hkv, G, D, S = b1 - b0, c["L"], c["Hkv"], c["Hq"] // c["Hkv"], c["D"], c["S"]
    q = x["q"][b0:b1].to(dt).view(n, L, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(n, Hkv, L * G, D)
    k = x["k_own"][b0:b1].to(dt).permute(0, 2, 3, 1)
    s = (q @ k / math.sqrt(D)).view(n, Hkv, L, G, S)
    seen, _ = _seen(c, x, b0, b1)
    return s.masked_fill_(~seen[:, None, :, None, :], -math.inf)


def _plain_attend(c, x):
    B, L, Hq, Hkv, D, P = (c[k] for k in ("B", "L", "Hq", "Hkv", "D", "P"))
    G = Hq // Hkv
    out = torch.empty((B, L, Hq, D), dtype=_dt(c), device=x["q"].device)
    lse = torch.empty((B, L, Hq), device=x["q"].device)
    if P:
        kp, vp = x["k_pre"].float().permute(1, 2, 0), x["v_pre"].float().transpose(0, 1)
    for b0, b1 in _parts(c):
        n = b1 - b0
        s = _own_scores(c, x, b0, b1, F32)
        _, live = _seen(c, x, b0, b1)
        m = s.amax(4, keepdim=True)
        if P:
            q = x["q"][b0:b1].float().view(n * L, Hkv, G, D).transpose(0, 1).reshape(Hkv, -1, D)
            sp = (q @ kp / math.sqrt(D)).view(Hkv, n, L, G, P)
            m = torch.maximum(m, sp.amax(4, keepdim=True).transpose(0, 1))
        m = m.clamp_(min=-1e30)
        e = s.sub_(m).exp_()
        z = e.sum(4, keepdim=True)
        o = (e.view(n, Hkv, L * G, -1) @ x["v_own"][b0:b1].float().transpose(1, 2)).view(n, Hkv, L, G, D)
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


def _plain_weights(c, x):
    B, L, Hq, Hkv, S = (c[k] for k in ("B", "L", "Hq", "Hkv", "S"))
    acc = torch.empty_like(x["acc"])
    at = torch.arange(S, device=acc.device)
    for b0, b1 in _parts(c):
        n = b1 - b0
        s = _own_scores(c, x, b0, b1, F32)
        ls = x["lse"][b0:b1].view(n, L, Hkv, Hq // Hkv).permute(0, 2, 1, 3)[..., None]
        w = s.sub_(ls.clamp(min=-1e30)).exp_().sum((2, 3))
        used = at < x["own_len"][b0:b1, None, None]
        acc[b0:b1] = torch.where(used, DECAY * x["acc"][b0:b1] + w, torch.zeros_like(w))
    return {"acc": acc}


def _plain_evict(c, x):
    S, keep, recent, Hkv, D = c["S"], c["keep"], c["recent"], c["Hkv"], c["D"]
    n = x["own_len"].long()[:, None, None]
    at = torch.arange(S, device=n.device)
    rank = torch.where(at >= n - recent, torch.full_like(x["acc"], math.inf), x["acc"])
    rank = torch.where(at < n, rank, torch.full_like(rank, -math.inf))
    best = rank.sort(dim=2, descending=True, stable=True).indices[..., :keep]
    left = torch.where(best < n, best, torch.full_like(best, S)).sort(2).values
    live = left < S
    left = torch.where(live, left, torch.zeros_like(left))
    acc = torch.where(live, x["acc"].gather(2, left), torch.zeros_like(rank[..., :keep]))
    put = {"acc": acc, "kept": torch.where(live, left, torch.full_like(left, -1)).int(),
           "own_len": x["own_len"].clamp(max=keep)}
    for name in ("k", "v"):
        rows = x[name + "_own"].gather(1, left.transpose(1, 2)[..., None].expand(-1, -1, -1, D))
        put[name] = torch.where(live.transpose(1, 2)[..., None], rows, torch.zeros_like(rows))
    return put


def run(state):
    x, c = state, state["case"]
    kind = c["kind"]
    if not own:
        return {"attend": _plain_attend, "weights": _plain_weights, "evict": _plain_evict}[kind](c, x)
    att = x["att"]
    if kind == "attend":
        return att.attend(x["q"], x["k_pre"], x["v_pre"], x["k_own"], x["v_own"], x["own_len"],
                          visible=x["visible"])
    if kind == "weights":
        return {"acc": att.weights(x["q"], x["lse"], x["k_own"], x["own_len"], x["acc"], DECAY,
                                   visible=x["visible"])}
    return att.evict(x["k_own"], x["v_own"], x["acc"], x["own_len"], c["keep"], c["recent"],
                     out=x["spare"])


# ---------------------------------------------------------------- what is counted

def work(case):
    """Bytes: the entries in use and the queries once, the outputs once. Flops: the products of the
    entries in use (what a causal block hides of itself is counted: it is at most L entries)."""
    c = case
    B, L, Hq, Hkv, D, P = (c[k] for k in ("B", "L", "Hq", "Hkv", "D", "P"))
    size = 2 if c["dtype"] == "bf16" else 4
    lens = _spread(c)
    used, rows = sum(lens), B * L * Hq
    if c["kind"] == "attend":
        return {"bytes": 2 * (P + used) * Hkv * D * size + 2 * rows * D * size + rows * 4 + B * 4,
                "flops": 4 * D * L * Hq * (B * P + used) + 5 * L * Hq * (B * P + used)}
    if c["kind"] == "weights":
        return {"bytes": used * Hkv * (D * size + 4) + B * Hkv * c["S"] * 4 + rows * (D * size + 4),
                "flops": (2 * D + 4) * L * Hq * used}
    kept = sum(min(n, c["keep"]) for n in lens)
    return {"bytes": used * Hkv * 4 + 2 * kept * Hkv * D * size + 2 * B * c["keep"] * Hkv * D * size +
            2 * B * c["keep"] * Hkv * 4, "flops": 4 * used * Hkv}


# ---------------------------------------------------------------- 64-bit values

def _exact_rows(c, x, b):
    """Scores [Hkv, L*G, n] of sequence b over its prefix and own entries in use, in 64 bits, and
    which of them a row sees."""
    L, Hkv, D, n = c["L"], c["Hkv"], c["D"], int(x["own_len"][b])
    G = c["Hq"] // Hkv
    k = x["k_own"][b, :n].double()
    if c["P"]:
        k = torch.cat([x["k_pre"].double(), k])
    q = x["q"][b].double().reshape(L, Hkv, G, D).transpose(0, 1).reshape(Hkv, L * G, D)
    s = torch.einsum("hrd,nhd->hrn", q, k) * D ** -0.5
    see = torch.full((L,), c["P"] + n, device=s.device)
    if x["visible"] is not None:
        v = x["visible"][b].long()
        see = torch.where(v < 0, 0, c["P"] + v.clamp(max=n))
    see = see.repeat_interleave(G)[:, None] > torch.arange(c["P"] + n, device=s.device)
    return s, see


def exact(case, seed):
    c = case
    x = _inputs(c, seed)
    B, L, Hq, Hkv, D, S = (c[k] for k in ("B", "L", "Hq", "Hkv", "D", "S"))
    G, dev = Hq // Hkv, x["k_own"].device
    if c["kind"] == "attend":
        out = torch.zeros((B, L, Hq, D), dtype=F64, device=dev)
        lse = torch.full((B, L, Hq), -math.inf, dtype=F64, device=dev)
        for b in range(B):
            s, see = _exact_rows(c, x, b)
            n = int(x["own_len"][b])
            v = x["v_own"][b, :n].double()
            if c["P"]:
                v = torch.cat([x["v_pre"].double(), v])
            any_ = see.any(1)
            ls = torch.logsumexp(s.masked_fill(~see, -math.inf), 2) if s.shape[2] else \
                torch.full(s.shape[:2], -math.inf, dtype=F64, device=dev)
            p = torch.where(see, torch.exp(s - torch.where(any_, ls, torch.zeros_like(ls))[..., None]), 0.0)
            o = torch.einsum("hrn,nhd->hrd", p, v)
            out[b] = o.view(Hkv, L, G, D).transpose(0, 1).reshape(L, Hq, D)
            lse[b] = ls.view(Hkv, L, G).transpose(0, 1).reshape(L, Hq)
        return {"out": out, "lse": lse}
    if c["kind"] == "weights":
        acc = torch.zeros((B, Hkv, S), dtype=F64, device=dev)
        for b in range(B):
            n = int(x["own_len"][b])
            s, see = _exact_rows(c, x, b)
            ls = x["lse"][b].double().view(L, Hkv, G).transpose(0, 1).reshape(Hkv, L * G)
            p = torch.where(see, torch.exp(s - torch.where(see.any(1), ls, torch.zeros_like(ls))[..., None]), 0.0)
            acc[b, :, :n] = DECAY * x["acc"][b, :, :n].double() + p.sum(1)
        return {"acc": acc}
    keep, recent = c["keep"], c["recent"]
    put = {"acc": torch.zeros((B, Hkv, keep), dtype=F64, device=dev),
           "kept": torch.full((B, Hkv, keep), -1, dtype=torch.int32, device=dev),
           "own_len": x["own_len"].clamp(max=keep)}
    for name in ("k", "v"):
        put[name] = torch.zeros((B, keep, Hkv, D), dtype=F64, device=dev)
    for b in range(B):
        n = int(x["own_len"][b])
        old = max(0, n - recent)              # entries that may go
        room = max(0, min(n, keep) - (n - old))
        by = torch.argsort(x["acc"][b, :, :old].double(), dim=1, descending=True, stable=True)[:, :room]
        late = torch.arange(old, n, device=dev).expand(Hkv, -1)
        ids = torch.cat([by.sort(1).values, late], 1)
        for h in range(Hkv):
            i, m = ids[h], ids.shape[1]
            put["kept"][b, h, :m] = i.int()
            put["acc"][b, h, :m] = x["acc"][b, h, i].double()
            put["k"][b, :m, h] = x["k_own"][b, i, h].double()
            put["v"][b, :m, h] = x["v_own"][b, i, h].double()
    return put
