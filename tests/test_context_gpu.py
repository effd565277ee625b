"""Blocks decoded over a shared prompt and bounded own caches: every call that the decoder makes of the
context cache's operators is held against the float64 oracle on the buffers it was given, with
the tolerances derived in test_cache_gpu.py."""
import numpy as np
import pytest
import torch

from oracle import cache as C
from paper_2609_33390_gb300 import synth
from test_cache_gpu import U, compare_attend, n64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def brisk():
    from paper_2609_33390_gb300 import build
    build.build()
    from paper_2609_33390_gb300 import brisk as B
    return B


class Checked:
    """The decoder's PrefixAttention, with each call checked; `calls` counts them."""

    def __init__(self, att):
        self.att, self.calls = att, {"attend": 0, "weights": 0, "evict": 0}
        self.device_status = att.device_status

    def attend(self, q, kp, vp, ko, vo, lens, visible=None):
        r = self.att.attend(q, kp, vp, ko, vo, lens, visible=visible)
        want = C.attend(*(n64(t) for t in (q, kp, vp, ko, vo, lens, visible)), self.att.scale)
        compare_attend(r, *want, q.dtype, self.att.D, self.att.P + self.att.S)
        self.calls["attend"] += 1
        return r

    def weights(self, q, lse, k, lens, acc, decay, visible, out):
        want, big = C.weights(n64(q), n64(lse), n64(k), n64(lens), n64(visible), self.att.scale, n64(acc), decay)
        got = n64(self.att.weights(q, lse, k, lens, acc=acc, decay=decay, visible=visible, out=out))
        rows = self.att.L * self.att.Hq // self.att.Hkv
        rel = (2 * self.att.D + 16) * U * big + 2.0 ** -21 + 4 * U * np.abs(n64(lse)).max() + (rows + 4) * U
        assert (np.abs(got - want) <= rel * np.abs(want) + 1e-30).all()
        self.calls["weights"] += 1
        return out

    def evict(self, k, v, acc, lens, keep, recent, out):
        want = C.evict(n64(k), n64(v), n64(acc), n64(lens), keep, recent)
        self.att.evict(k, v, acc, lens, keep, recent, out=out)
        for name, w in zip(("k", "v", "acc", "own_len", "kept"), want):
            got = n64(out[name])
            np.testing.assert_array_equal(got[:, :keep] if name in ("k", "v") else got, w, err_msg=name)
        self.calls["evict"] += 1
        return out


def decoder(brisk, dt, B, L, P, S, keep, Hq, Hkv, D, recent=2, decay=0.9):
    from paper_2609_33390_gb300 import context
    wl = synth.Workload("context", B=B, L=L, V=512, d=128, K=8, r=32, logits_dtype=dt, hidden_dtype=dt)
    w = synth.make_weights(wl, "cuda")
    tail = brisk.DecodeTail.for_workload(wl, w)
    tail.prepare()
    prompt = torch.arange(P, device="cuda") * 7 % wl.V
    dec = context.ContextDecoder(tail, context.layer_weights(wl.d, Hq, Hkv, D, dt, seed=L), prompt, Hq, Hkv, D,
                                 S, keep, recent, decay)
    dec.start(torch.arange(B, dtype=torch.int32, device="cuda"))
    return dec


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,L,P,S,keep,Hq,Hkv,D", [
    (3, 4, 50, 24, 12, 4, 2, 64),
    (2, 1, 0, 9, 8, 6, 1, 32),                         # a token a block
    (5, 7, 131, 140, 30, 2, 2, 128),                   # the caches last for several blocks
])
def test_decoder_calls_match_the_oracle(brisk, B, L, P, S, keep, Hq, Hkv, D, dt):
    dec = decoder(brisk, dt, B, L, P, S, keep, Hq, Hkv, D)
    dec.attention = Checked(dec.attention)
    steps, room = 24, S - 1
    cuts = 0
    for _ in range(steps):                             # the cuts that the bound on the lengths asks for
        if room < L:
            cuts, room = cuts + 1, S - min(keep, S - room)
        room -= L
    committed = torch.ones(B, dtype=torch.int64, device="cuda")
    for _ in range(steps):
        out = dec.step()
        committed += (out["accepted_len"] + 1).clamp(max=L)
        assert (out["out_tokens"][:, 0] >= 0).all()
        assert (dec.own_len <= dec.most).all() and (dec.own_len <= committed).all() and dec.most <= S
        behind = dec.places >= dec.own_len[:, None, None]
        assert (dec.acc[behind.expand_as(dec.acc)] == 0).all() and torch.isfinite(dec.acc).all()
    assert dec.attention.calls == {"attend": steps, "weights": steps, "evict": cuts} and cuts > 0
    assert dec.device_status() == brisk.OK


def test_decoder_refuses_a_block_that_cannot_fit(brisk):
    with pytest.raises(ValueError):
        decoder(brisk, torch.float32, 2, 4, 10, 15, 12, 2, 1, 16)
