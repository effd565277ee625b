"""Blocks decoded over a shared prompt and bounded own caches: a one-layer stand-in for the backbone in
front of the decode tail, with the context cache's operators as a backbone's layer uses them.

Every block, `ContextDecoder.step` writes the block's keys and values behind the committed entries,
attends over the prompt and them, hands hidden states and logits to the decode tail, adds up the
attention weight that own entries got, and replaces the block's entries by those of the committed
tokens. Before a block that might not fit, all sequences' caches are cut to the entries of
largest weight. Nothing is read back: the host knows an upper bound of the lengths. Projections are
library products; attention, weights, eviction and the tail are the library's kernels."""
from __future__ import annotations

import torch

from . import brisk


def layer_weights(d, Hq, Hkv, D, dtype, device="cuda", seed=0):
    """Projections of one layer, N(0, 1 / fan-in), the masked positions' embedding, and the verifier's head."""
    g = torch.Generator(device=device).manual_seed(seed)
    new = lambda n, m: (torch.randn(n, m, generator=g, device=device) * n ** -0.5).to(dtype)
    return {"q": new(d, Hq * D), "k": new(d, Hkv * D), "v": new(d, Hkv * D), "o": new(Hq * D, d),
            "p": new(d, d), "mask": torch.randn(d, generator=g, device=device).to(dtype)}


class ContextDecoder:
    """B sequences decoded in blocks of L behind the prompt `prompt` [P] (token ids, shared by all).

    `tail`: the prepared DecodeTail (its weights hold the embedding rows E_in and E_out); `w`: see
    layer_weights. Own caches have room for `S` entries and are cut to `keep`, of which the
    `recent` newest always stay; sums of weights shrink by `decay` a block."""

    def __init__(self, tail, w, prompt, Hq, Hkv, D, S, keep, recent=0, decay=1.0):
        if keep + tail.L > S:
            raise ValueError(f"a block of {tail.L} does not fit behind {keep} of {S} entries")
        self.tail, self.w, self.keep, self.recent, self.decay = tail, w, keep, recent, decay
        self.e_in, self.e_out = tail.weights["E_in"], tail.weights["E_out"]
        B, L, dev, dt = tail.B, tail.L, tail.device, self.e_in.dtype
        self.Hq, self.Hkv, self.D, self.S = Hq, Hkv, D, S
        self.attention = brisk.PrefixAttention(B, L, Hq, Hkv, D, prompt.numel(), S, dt, dev)
        self.k_prefix, self.v_prefix = self._entries(self.e_in[prompt])
        self.k, self.v = (torch.zeros(B, S, Hkv, D, dtype=dt, device=dev) for _ in range(2))
        self.acc = torch.zeros(B, Hkv, S, device=dev)
        self.spare = self.attention.alloc_evicted(keep, room=S)
        self.own_len = torch.zeros(B, dtype=torch.int32, device=dev)
        # a workspace's first word is its last call's status, which the next call of the step overwrites
        self.words = [x.workspace[:4].view(torch.int32) for x in (self.attention, tail)]
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.most = 0                                  # no sequence has more entries
        self.at = torch.arange(L, device=dev, dtype=torch.int32)
        self.places = torch.arange(S, device=dev, dtype=torch.int32)
        self.rows = torch.arange(B, device=dev)[:, None]
        pos = torch.arange(L, device=dev)[:, None] / 10000 ** torch.linspace(0, 1, tail.d, device=dev)
        self.block = (w["mask"] + torch.cos(pos)).to(dt).expand(B, L, tail.d)

    def _entries(self, x):
        shape = (*x.shape[:-1], self.Hkv, self.D)
        return (x @ self.w["k"]).view(shape), (x @ self.w["v"]).view(shape)

    def _write(self, x, where):
        self.k[self.rows, where], self.v[self.rows, where] = self._entries(x)

    def _ids(self, x):
        """Token ids as indices: a row without a finite logit, or a wait that gave up, may leave any number, which
        is 0 then (the tail takes such anchors so, and reports them)."""
        return torch.where((x >= 0) & (x < self.e_in.shape[0]), x, 0).long()

    def start(self, x0):
        """The first anchors [B] (int32) become the own caches' first entries."""
        self.own_len.fill_(1)
        self._write(self.e_in[self._ids(x0)][:, None], self.own_len[:, None].long() - 1)
        self.acc.zero_()
        self.most = 1
        self.x0 = x0

    def _note(self, *words):
        for word in words:
            torch.maximum(self.status, word, out=self.status)

    def _cut(self):
        self.attention.evict(self.k, self.v, self.acc, self.own_len, self.keep, self.recent, out=self.spare)
        self._note(self.words[0])
        self.k, self.v, self.spare["k"], self.spare["v"] = self.spare["k"], self.spare["v"], self.k, self.v
        self.own_len.copy_(self.spare["own_len"])
        self.acc[:, :, :self.keep] = self.spare["acc"]
        self.acc[:, :, self.keep:] = 0
        self.most = min(self.most, self.keep)

    def step(self):
        """One block of every sequence: the decode tail's outputs."""
        t, att = self.tail, self.attention
        if self.most + t.L > self.S:
            self._cut()
        where = (self.own_len[:, None] + self.at).long()
        self._write(self.block, where)
        visible = self.own_len[:, None] + self.at + 1  # a position sees the context and the block up to itself
        in_use = self.own_len + t.L
        q = (self.block @ self.w["q"]).view(t.B, t.L, self.Hq, self.D)
        r = att.attend(q, self.k_prefix, self.v_prefix, self.k, self.v, in_use, visible=visible)
        self._note(self.words[0])
        hidden = self.block + r["out"].view(t.B, t.L, -1) @ self.w["o"]
        out = t.tail({"logits_q": hidden @ self.e_out.T, "logits_p": hidden @ self.w["p"] @ self.e_out.T,
                      "hidden": hidden, "h_c": hidden[:, 0].contiguous(), "x0": self.x0})
        att.weights(q, r["lse"], self.k, in_use, acc=self.acc, decay=self.decay, visible=visible, out=self.acc)
        self._note(*self.words)
        # the committed tokens' entries in place of the block's
        self._write(self.e_in[self._ids(out["out_tokens"])], where)
        self.own_len += (out["accepted_len"] + 1).clamp(1, t.L)
        self.acc.masked_fill_(self.places >= self.own_len[:, None, None], 0)
        self.most += t.L
        self.x0 = out["next_anchor"]
        return out

    def device_status(self) -> int:
        """The worst (largest) status that a call of the steps since the last query left, the tail's and each of the
        attention's (see brisk_last_device_status). Waits for the steps, and begins anew."""
        worst = int(self.status)
        self.status.zero_()
        return worst
