"""Blocks decoded over own caches in 4 bits: every call that the decoder makes is held against the float64 oracle on the
buffers it was given, with the tolerances of test_packed_gpu.py and test_context_gpu.py."""
import numpy as np
import pytest
import torch

from oracle import cache as C
from oracle import packed as P
from paper_2609_33390_gb300 import synth
from test_context_gpu import Checked
from test_packed_gpu import compare, n64, raw

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def brisk():
    from paper_2609_33390_gb300 import build
    build.build()
    from paper_2609_33390_gb300 import brisk as B
    return B


class CheckedPacked:
    """The decoder's PackedAttention, with each call checked; `calls` counts them."""

    def __init__(self, att):
        self.att, self.calls = att, {"attend": 0, "store": 0, "load": 0}

    def attend(self, q, kp, vp, cache, lens, visible=None):
        r = self.att.attend(q, kp, vp, cache, lens, visible=visible)
        x = {"q": q, "kp": kp if self.att.P else None, "vp": vp, "v": P.values(*raw(cache, "v"))}
        want = C.attend(n64(q), n64(x["kp"]), n64(vp) if self.att.P else None, P.values(*raw(cache, "k")), x["v"],
                        n64(lens), n64(visible), self.att.scale)
        compare(r, want, x, self.att.S)
        self.calls["attend"] += 1
        return r

    def store(self, cache, k, v, start, count=None):
        before = {n: raw(cache, n) for n in "kv"}
        self.att.store(cache, k, v, start, count)
        for name, x in (("k", k), ("v", v)):
            codes, scales = before[name]
            for b in range(x.shape[0]):
                n = x.shape[1] if count is None else int(count[b])
                at = slice(int(start[b]), int(start[b]) + n)
                codes[b, at], s = P.store(n64(x[b, :n]))
                scales[b, at, :, :self.att.D // 16] = s[..., :self.att.D // 16]
            got = raw(cache, name)
            assert (got[0] == codes).all() and (got[1] == scales).all()
        self.calls["store"] += 1
        return cache

    def load(self, cache, T, start, count, out):
        self.att.load(cache, T, start, count, out=out)
        for name in "kv":
            x = P.values(*raw(cache, name))
            for b in range(x.shape[0]):
                x[b, int(count[b]):] = 0
            assert (n64(out[name]) == x).all()
        self.calls["load"] += 1
        return out


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,L,P_,S,keep,Hq,Hkv,D", [
    (3, 4, 50, 24, 12, 4, 2, 64),
    (2, 1, 0, 9, 8, 6, 1, 32),                         # a token a block
    (2, 7, 131, 40, 16, 8, 2, 128),                    # 28 rows a key head
])
def test_decoder_calls_match_the_oracle(brisk, B, L, P_, S, keep, Hq, Hkv, D, dt):
    from paper_2609_33390_gb300 import context
    wl = synth.Workload("context", B=B, L=L, V=512, d=128, K=8, r=32, logits_dtype=dt, hidden_dtype=dt)
    tail = brisk.DecodeTail.for_workload(wl, synth.make_weights(wl, "cuda"))
    tail.prepare()
    dec = context.ContextDecoder(tail, context.layer_weights(wl.d, Hq, Hkv, D, dt, seed=L),
                                 torch.arange(P_, device="cuda") * 7 % wl.V, Hq, Hkv, D, S, keep, 2, 0.9, packed=True)
    dec.attention, dec.entries = CheckedPacked(dec.attention), Checked(dec.entries)
    dec.start(torch.arange(B, dtype=torch.int32, device="cuda"))
    steps, room, cuts = 8, S - 1, 0
    for _ in range(steps):                             # the cuts that the bound on the lengths asks for
        if room < L:
            cuts, room = cuts + 1, S - min(keep, S - room)
        room -= L
    for _ in range(steps):
        out = dec.step()
        assert (out["out_tokens"][:, 0] >= 0).all()
        assert (dec.own_len <= dec.most).all() and dec.most <= S
        assert torch.isfinite(dec.acc).all()
    assert dec.attention.calls == {"attend": steps, "store": 1 + 2 * steps + cuts, "load": steps + cuts}
    assert dec.entries.calls == {"attend": 0, "weights": steps, "evict": cuts} and (cuts > 0 or L == 1)
    assert dec.device_status() == brisk.OK


def test_a_problem_of_a_write_is_reported_once(brisk):
    from paper_2609_33390_gb300 import context
    wl = synth.Workload("context", B=2, L=3, V=512, d=128, K=8, r=32, logits_dtype=torch.bfloat16,
                        hidden_dtype=torch.bfloat16)
    tail = brisk.DecodeTail.for_workload(wl, synth.make_weights(wl, "cuda"))
    tail.prepare()
    dec = context.ContextDecoder(tail, context.layer_weights(wl.d, 4, 2, 32, torch.bfloat16),
                                 torch.arange(10, device="cuda"), 4, 2, 32, 30, 12, packed=True)
    dec.start(torch.arange(2, dtype=torch.int32, device="cuda"))
    for _ in range(2):
        dec.step()
    assert dec.device_status() == brisk.OK
    dec.own_len[1] = 30                                # the block's entries lie behind the cache's end
    dec.step()
    dec.own_len.clamp_(max=12)
    dec.step()
    assert dec.device_status() == brisk.ERR_INVALID_ARG
    dec.step()
    assert dec.device_status() == brisk.OK
