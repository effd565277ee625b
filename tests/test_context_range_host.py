"""What the tail's outputs index in the decoder's buffers stays in range, whatever the outputs hold: the decoder on the
CPU, with stand-ins for the library's calls."""
import pytest
import torch

from paper_2609_33390_gb300 import brisk, context

B, L, V, d, Hq, Hkv, D, S = 2, 3, 50, 16, 4, 2, 8, 9


class Tail:
    """Outputs as given; inputs are kept."""

    def __init__(self):
        self.B, self.L, self.d, self.device = B, L, d, torch.device("cpu")
        self.weights = {n: torch.randn(V, d) for n in ("E_in", "E_out")}
        self.workspace = torch.zeros(256, dtype=torch.uint8)
        self.out = None

    def tail(self, block):
        self.x0 = block["x0"]
        return self.out


class Attention:
    def __init__(self, *a):
        self.workspace = torch.zeros(256, dtype=torch.uint8)

    def attend(self, q, kp, vp, k, v, lens, visible=None):
        return {"out": torch.zeros_like(q), "lse": torch.zeros(q.shape[:3])}

    def weights(self, *a, out, **k):
        return out

    def alloc_evicted(self, keep, room):
        return {"k": torch.zeros(B, room, Hkv, D), "v": torch.zeros(B, room, Hkv, D),
                "acc": torch.zeros(B, Hkv, keep), "own_len": torch.zeros(B, dtype=torch.int32)}

    def evict(self, k, v, acc, lens, keep, recent, out):
        out["own_len"].copy_(lens.clamp(max=keep))


@pytest.fixture
def dec(monkeypatch):
    monkeypatch.setattr(brisk, "PrefixAttention", Attention)
    torch.manual_seed(0)
    w = context.layer_weights(d, Hq, Hkv, D, torch.float32, device="cpu")
    return context.ContextDecoder(Tail(), w, torch.arange(5), Hq, Hkv, D, S, keep=6, recent=1)


def i32(*x):
    return torch.tensor(x, dtype=torch.int32)


@pytest.mark.parametrize("ids", [[5, -1, -1], [2 ** 31 - 1, 7, -1], [V, V - 1, 0], [-2 ** 31, 3, 4]])
@pytest.mark.parametrize("accepted", [0, 2, 3, -1, -2 ** 31, 2 ** 31 - 2])
def test_any_outputs_of_the_tail_stay_in_range(dec, ids, accepted):
    dec.start(i32(1, 3))
    for _ in range(6):
        dec.tail.out = {"out_tokens": i32(ids, ids), "accepted_len": i32(accepted, 1), "next_anchor": i32(ids[0], 3)}
        before, cut = dec.own_len.clone(), dec.most + L > S
        dec.step()
        base = before.clamp(max=dec.keep) if cut else before
        n = int(dec.own_len[0] - base[0])
        assert 1 <= n <= L and int(dec.own_len[1] - base[1]) == 2 and (dec.own_len <= dec.most).all()
        want = dec.e_in[[i if 0 <= i < V else 0 for i in ids]]
        at = int(base[0])
        torch.testing.assert_close(dec.k[0, at:at + L], (want @ dec.w["k"]).view(L, Hkv, D))


@pytest.mark.parametrize("anchor", [2 ** 31 - 1, V, -1])
def test_an_anchor_out_of_range_is_0_as_the_tail_has_it(dec, anchor):
    dec.start(i32(anchor, V - 1))
    torch.testing.assert_close(dec.k[:, 0], (dec.e_in[[0, V - 1]] @ dec.w["k"]).view(B, Hkv, D))
