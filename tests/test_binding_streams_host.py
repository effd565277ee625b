"""Calls on a stream other than the current one: whose memory their results are, without a GPU. The
library, the streams and the checks of places are stand-ins; the calls' own allocations are watched."""
import contextlib

import pytest
import torch


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


class Watch:
    """What is allocated, under which stream, and which streams its memory is also kept for."""

    def __init__(self):
        self.under, self.made, self.kept = None, [], {}


@pytest.fixture
def B():
    from paper_2609_33390_gb300 import build
    build.build()
    from paper_2609_33390_gb300 import brisk
    return brisk


@pytest.fixture
def watch(B, monkeypatch):
    w, real, here = Watch(), B.lib(), Stream(1)

    class Lib:                                         # sizes are the library's, calls do nothing
        def __getattr__(self, name):
            return getattr(real, name) if name.endswith("_bytes") else lambda *a: B.OK

    @contextlib.contextmanager
    def stream(s):
        before, w.under = w.under, s
        yield
        w.under = before

    def empty(*a, **k):
        t = alloc(*a, **k)
        w.made.append((t, w.under))
        return t

    alloc = torch.empty
    monkeypatch.setattr(B, "lib", lambda: Lib())
    monkeypatch.setattr(B, "_stream", lambda s=None: (here if s is None else s).cuda_stream)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: here)
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: w.kept.setdefault(id(t), []).append(s))
    monkeypatch.setattr(B.PrefixAttention, "_view", lambda self, t, shape, what: (0, 0, 0, 0))
    monkeypatch.setattr(B.PrefixAttention, "_plain", staticmethod(lambda t, shape, dtype, what: None))
    w.here = here
    return w


def cache_calls(B):
    att = B.PrefixAttention(2, 3, 4, 2, 64, 10, 20, torch.bfloat16, device="cpu")
    return {"attend": lambda s: att.attend(*[None] * 6, stream=s),
            "weights": lambda s: {"acc": att.weights(*[None] * 4, stream=s)},
            "evict": lambda s: att.evict(*[None] * 4, 8, 2, stream=s)}


def check_results(watch, call):
    for given, other in ((None, False), (Stream(1), False), (Stream(2), True)):
        watch.made, watch.kept = [], {}
        r = call(given)
        assert r and {id(t) for t in r.values()} == {id(t) for t, _ in watch.made}
        for t, under in watch.made:
            assert under is (given if other else None)
            assert watch.kept.get(id(t), []) == ([watch.here] if other else [])


@pytest.mark.parametrize("name", ["attend", "weights", "evict"])
def test_results_are_memory_of_the_stream_that_writes_them(B, watch, name):
    check_results(watch, cache_calls(B)[name])


def tail_calls(B):
    tail = B.DecodeTail.__new__(B.DecodeTail)
    tail.dims = B.make_dims(2, 3, 512, 16, 4, 16, torch.float32, torch.float32)
    tail.B, tail.L, tail.K, tail.device = 2, 3, 4, torch.device("cpu")
    tail.params, tail.tables, tail.workspace = B.Params(), torch.zeros(1), torch.zeros(1)
    block = {n: None for n in ("logits_q", "logits_p", "hidden", "h_c", "x0", "u_sel", "u_acc")}
    return {"topk": lambda s: tail.topk(None, stream=s),
            "select": lambda s: tail.select(*[None] * 6, stream=s),
            "verify": lambda s: tail.verify(*[None] * 4, stream=s),
            "replay": lambda s: tail.replay(block, stream=s),
            "distill_loss": lambda s: tail.distill_loss(*[None] * 5, stream=s),
            "tail": lambda s: tail.tail(block, stream=s)}


@pytest.mark.parametrize("name", ["topk", "select", "verify", "replay", "distill_loss", "tail"])
def test_results_of_a_tail_are_memory_of_the_stream_that_writes_them(B, watch, name):
    check_results(watch, tail_calls(B)[name])


@pytest.mark.parametrize("calls", [cache_calls, tail_calls])
def test_an_objects_buffers_are_kept_for_the_stream_of_a_call(B, watch, monkeypatch, calls):
    """Dropped with the object, they are not free before the call on the other stream has ended."""
    lent = []
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: lent.append((t, s)))
    other = Stream(2)
    for call in calls(B).values():
        for given in (None, Stream(1), other):
            del lent[:]
            call(given)
            assert sum(s is other for _, s in lent) == (0 if given is not other else 1 if calls is cache_calls else 2)


@pytest.mark.parametrize("capturing", [False, True])
@pytest.mark.parametrize("kind", ["cache", "tail"])
def test_new_buffers_are_settled_before_calls_go_to_any_stream(B, monkeypatch, kind, capturing):
    """The clearing of a workspace, on the current stream, is not still to come when a call runs on another."""
    log = []

    class Current:
        def synchronize(self):
            log.append("waited")

    def make(real):
        def new(*a, device=None, **k):
            log.append("made")
            return real(*a, **k)
        return new

    monkeypatch.setattr(torch, "zeros", make(torch.zeros))
    monkeypatch.setattr(torch, "empty", make(torch.empty))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Current())
    monkeypatch.setattr(B, "make_params", lambda w: B.Params())
    if kind == "cache":
        B.PrefixAttention(2, 3, 4, 2, 64, 10, 20, torch.bfloat16, device="cuda")
    else:
        B.DecodeTail(2, 3, 512, 16, 4, 16, torch.float32, torch.float32, {}, device="cuda")
    assert "made" in log and (log[-1] == "waited") != capturing and log.count("waited") == (not capturing)
