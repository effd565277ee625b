"""Decoders over own caches in 4 bits that share what entries are read back into: the same blocks as with buffers of their
own."""
import pytest
import torch

from paper_2609_33390_gb300 import synth

pytestmark = pytest.mark.gpu

SIZES = dict(B=3, L=4, S=24, keep=12, Hq=4, Hkv=2, D=64)


@pytest.fixture(scope="module")
def brisk():
    from paper_2609_33390_gb300 import build
    build.build()
    from paper_2609_33390_gb300 import brisk as B
    return B


def decoder(brisk, dt, seed, packed=True, scratch=None, **sizes):
    from paper_2609_33390_gb300 import context
    z = dict(SIZES, **sizes)
    wl = synth.Workload("context", B=z["B"], L=z["L"], V=512, d=128, K=8, r=32, logits_dtype=dt, hidden_dtype=dt)
    tail = brisk.DecodeTail.for_workload(wl, synth.make_weights(wl, "cuda"))
    tail.prepare()
    dec = context.ContextDecoder(tail, context.layer_weights(wl.d, z["Hq"], z["Hkv"], z["D"], dt, seed=seed),
                                 torch.arange(50, device="cuda") * (7 + seed) % wl.V, z["Hq"], z["Hkv"], z["D"], z["S"],
                                 z["keep"], 2, 0.9, packed=packed, scratch=scratch)
    dec.start(torch.arange(z["B"], dtype=torch.int32, device="cuda") + seed)
    return dec


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_decoders_that_share_decode_as_alone(brisk, dt):
    alone = [decoder(brisk, dt, seed) for seed in range(3)]
    first = decoder(brisk, dt, 0)
    shared = [first] + [decoder(brisk, dt, seed, scratch=first.scratch) for seed in (1, 2)]
    for d in shared[1:]:
        assert d.k is first.k and d.v is first.v and d.spare is first.spare
    for turn in range(9):                              # (with cuts: a block needs 4 of the 12 places behind those kept)
        for a in alone:
            a.want = a.step()
        for a, d in zip(alone, shared):
            out = d.step()
            for n in out:
                assert torch.equal(out[n], a.want[n]), (turn, n)
            assert torch.equal(d.acc, a.acc) and torch.equal(d.own_len, a.own_len)
            for n in d.cache:
                assert torch.equal(d.cache[n], a.cache[n]), (turn, n)
    assert [d.device_status() for d in alone + shared] == [brisk.OK] * 6


def test_scratch_of_other_sizes_or_of_unpacked_caches_is_refused(brisk):
    bf = torch.bfloat16
    scratch = decoder(brisk, bf, 0).scratch
    for other in (dict(B=2), dict(S=25), dict(keep=13), dict(Hkv=4), dict(D=32)):
        with pytest.raises(ValueError):
            decoder(brisk, bf, 0, scratch=scratch, **other)
    with pytest.raises(ValueError):
        decoder(brisk, torch.float32, 0, scratch=scratch)
    plain = decoder(brisk, bf, 0, packed=False)
    assert plain.scratch is None
    with pytest.raises(ValueError):
        decoder(brisk, bf, 0, packed=False, scratch=scratch)
