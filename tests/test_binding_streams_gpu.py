"""Calls on a stream of their own beside a current stream that is far behind: what they allocate is
neither what the current stream still has to read, nor free before the current stream has read it."""
import pytest
import torch

from paper_2609_33390_gb300 import synth
from test_cache_gpu import BF, make

pytestmark = pytest.mark.gpu

BEHIND = 20_000_000                                    # cycles, about 10 ms


@pytest.fixture(scope="module")
def B():
    from paper_2609_33390_gb300 import build
    build.build()
    from paper_2609_33390_gb300 import brisk
    return brisk


def cache_calls(B):
    x = make(3, 2, 8, 2, 64, 100, 60, BF, [60, 40, 5])
    att = B.PrefixAttention(3, 2, 8, 2, 64, 100, 60, BF)
    lse = torch.full((3, 2, 8), 3.0, device="cuda")
    acc = torch.rand(3, 2, 60, device="cuda")
    return {"attend": lambda s: att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"], stream=s),
            "weights": lambda s: {"acc": att.weights(x["q"], lse, x["ko"], x["lens"], stream=s)},
            "evict": lambda s: att.evict(x["ko"], x["vo"], acc, x["lens"], 30, 5, stream=s)}


def check_beside_a_late_stream(call):
    want = {k: v.clone() for k, v in call(None).items()}
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    # memory that the current stream has yet to read, dropped
    old = {k: torch.full_like(v, 7) for k, v in want.items()}
    read = {k: torch.zeros_like(v) for k, v in want.items()}
    torch.cuda._sleep(BEHIND)
    for k, v in old.items():
        read[k].copy_(v)
    del old, v
    got = call(s)
    torch.cuda.synchronize()
    for k in want:
        assert (read[k] == 7).all() and torch.equal(got[k], want[k])
    # results that the current stream has yet to read, dropped, and the next call
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda._sleep(BEHIND)
    for k in want:
        read[k].copy_(got[k])
    del got
    again = call(s)
    with torch.cuda.stream(s):
        for v in again.values():
            v.fill_(3)
    torch.cuda.synchronize()
    for k in want:
        assert torch.equal(read[k], want[k])


@pytest.mark.parametrize("name", ["attend", "weights", "evict"])
def test_results_do_not_race_with_a_current_stream_that_is_behind(B, name):
    check_beside_a_late_stream(cache_calls(B)[name])


def tail_calls(B):
    wl = synth.Workload("streams", B=3, L=6, V=2048, d=32, K=8, r=16)
    tail = B.DecodeTail.for_workload(wl, synth.make_weights(wl, "cuda"))
    tail.prepare()
    block = synth.make_block(wl, "cuda")
    c = tail.topk(block["logits_q"])
    r = tail.select(block["hidden"], block["h_c"], block["x0"], block["logits_q"], c["cand_ids"], c["cand_logprob"])
    accepted = torch.full((3,), 2, dtype=torch.int32, device="cuda")
    return {"topk": lambda s: tail.topk(block["logits_q"], stream=s),
            "select": lambda s: tail.select(block["hidden"], block["h_c"], block["x0"], block["logits_q"],
                                            c["cand_ids"], c["cand_logprob"], stream=s),
            "verify": lambda s: tail.verify(block["logits_p"], r["sel_tokens"], c["cand_ids"], r["refined"], stream=s),
            "replay": lambda s: tail.replay(block, stream=s),
            "distill_loss": lambda s: tail.distill_loss(block["logits_p"], c["cand_ids"], c["cand_logprob"],
                                                        r["refined"], accepted, stream=s),
            "tail": lambda s: tail.tail(block, stream=s)}


@pytest.mark.parametrize("name", ["topk", "select", "verify", "replay", "distill_loss", "tail"])
def test_results_of_a_tail_do_not_race_with_a_current_stream_that_is_behind(B, name):
    check_beside_a_late_stream(tail_calls(B)[name])


def test_an_object_may_be_dropped_while_its_call_is_pending(B):
    x = make(3, 2, 8, 2, 64, 100, 60, BF, [60, 40, 5])
    new = lambda: B.PrefixAttention(3, 2, 8, 2, 64, 100, 60, BF)
    run = lambda att, s=None: att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"], stream=s)
    want = run(new())
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    att = new()
    n = att.workspace.numel()
    with torch.cuda.stream(s):
        torch.cuda._sleep(BEHIND)
    got = run(att, s)
    del att
    for _ in range(3):
        torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
