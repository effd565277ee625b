"""ctypes binding of ``libbrisk.so`` (the C ABI in ``include/brisk.h``).

Argument marshalling only: every step of the decode tail runs in the CUDA
library. Tensors are torch CUDA tensors; their data pointers and the current
torch stream are handed to the library. Loading fails loudly when the library
has not been built; nothing here falls back to another implementation.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass
from typing import Dict, Optional

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libbrisk.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_CUDA, ERR_TIMEOUT, ERR_NUMERIC = range(6)
DT_F32, DT_BF16 = 0, 1
SELECT_GREEDY, SELECT_SAMPLE = 0, 1
VERIFY_GREEDY, VERIFY_STOCHASTIC = 0, 1

_vp = ctypes.c_void_p


class Dims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("B", "L", "V", "d", "K", "r", "logits_dtype", "hidden_dtype")]


class Params(ctypes.Structure):
    _fields_ = [(n, _vp) for n in ("E_in", "E_out", "P_h", "P_e", "P_phi", "pos", "W0", "Wz", "Wh",
                                   "W_s", "W_c", "w_g")] + [("b_g", ctypes.c_float),
                                                           ("alpha", ctypes.c_float)]


class TailIO(ctypes.Structure):
    _fields_ = [(n, _vp) for n in ("logits_q", "logits_p", "hidden", "h_ctx", "x0", "u_sel", "u_acc",
                                   "u_res", "cand_ids", "cand_logprob", "lse_q", "sel_tokens",
                                   "refined", "accepted_len", "out_tokens", "correction",
                                   "next_anchor")]


class Events(ctypes.Structure):
    _fields_ = [("sweep_q_begin", _vp), ("sweep_q_end", _vp), ("sweep_p_begin", _vp),
                ("sweep_p_end", _vp)]


class CacheDims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "L", "Hq", "Hkv", "D", "P", "S", "dtype")]


class View(ctypes.Structure):
    _fields_ = [("ptr", _vp), ("seq", ctypes.c_int64), ("tok", ctypes.c_int64),
                ("head", ctypes.c_int64)]


class BriskError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)}")


_lib = None

# (name, restype, argtypes) of every exported entry point
_SIGS = [
    ("brisk_workspace_bytes", ctypes.c_size_t, [ctypes.POINTER(Dims)]),
    ("brisk_tables_bytes", ctypes.c_size_t, [ctypes.POINTER(Dims)]),
    ("brisk_corrector_prepare", ctypes.c_int, [ctypes.POINTER(Dims), ctypes.POINTER(Params), _vp, _vp]),
    ("brisk_topk_candidates", ctypes.c_int, [ctypes.POINTER(Dims), _vp, _vp, _vp, _vp, _vp, _vp]),
    ("brisk_corrector_select", ctypes.c_int,
     [ctypes.POINTER(Dims), ctypes.POINTER(Params), _vp, _vp, _vp, _vp, _vp, _vp, _vp,
      ctypes.c_int32, _vp, _vp, _vp, _vp, _vp]),
    ("brisk_verify_block", ctypes.c_int,
     [ctypes.POINTER(Dims), _vp, _vp, _vp, _vp, ctypes.c_int32, ctypes.c_int32, _vp, _vp, _vp, _vp,
      _vp, _vp, _vp]),
    ("brisk_decode_tail", ctypes.c_int,
     [ctypes.POINTER(Dims), ctypes.POINTER(Params), _vp, ctypes.POINTER(TailIO), ctypes.c_int32,
      ctypes.c_int32, _vp, ctypes.POINTER(Events), _vp]),
    ("brisk_topk_candidates_noalloc", ctypes.c_int,
     [ctypes.POINTER(Dims), _vp, _vp, _vp, _vp, _vp]),
    ("brisk_kernels_per_tail", ctypes.c_int32, [ctypes.POINTER(Dims)]),
    ("brisk_last_device_status", ctypes.c_int, [_vp, ctypes.c_int32, _vp]),
    ("brisk_status_string", ctypes.c_char_p, [ctypes.c_int]),
    ("brisk_set_wait_limit", ctypes.c_int64, [ctypes.c_int64]),
    ("brisk_acceptance_counts", ctypes.c_int, [_vp, ctypes.c_int32, ctypes.c_int32, _vp, _vp]),
    ("brisk_acceptance_weights", ctypes.c_int,
     [ctypes.c_int32, _vp, _vp, _vp, ctypes.c_double, _vp, _vp, _vp]),
    ("brisk_tpf_isd", ctypes.c_double, [ctypes.c_int32, ctypes.c_double]),
    ("brisk_isd_costs", ctypes.c_int, [ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]),
    ("brisk_tail_graph_create", ctypes.c_int,
     [ctypes.POINTER(Dims), ctypes.POINTER(Params), _vp, ctypes.POINTER(TailIO), ctypes.c_int32,
      ctypes.c_int32, _vp, _vp, ctypes.POINTER(_vp)]),
    ("brisk_tail_graph_launch", ctypes.c_int, [_vp, _vp]),
    ("brisk_tail_graph_destroy", None, [_vp]),
    ("brisk_replay_diagnostics", ctypes.c_int,
     [ctypes.POINTER(Dims), ctypes.POINTER(Params), _vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_int32,
      _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    ("brisk_distill_loss", ctypes.c_int,
     [ctypes.POINTER(Dims), _vp, _vp, _vp, _vp, _vp, ctypes.c_float, _vp, _vp, _vp, _vp]),
    ("brisk_cache_workspace_bytes", ctypes.c_size_t, [ctypes.POINTER(CacheDims)]),
    ("brisk_prefix_attend", ctypes.c_int,
     [_vp] * 8 + [ctypes.c_float, _vp, _vp, _vp, _vp]),
    ("brisk_cache_weights", ctypes.c_int,
     [_vp] * 6 + [ctypes.c_float, ctypes.c_float, _vp, _vp, _vp, _vp]),
    ("brisk_cache_evict", ctypes.c_int,
     [_vp] * 5 + [ctypes.c_int32, ctypes.c_int32] + [_vp] * 7),
    ("brisk_packed_workspace_bytes", ctypes.c_size_t, [ctypes.POINTER(CacheDims)]),
    ("brisk_packed_store", ctypes.c_int, [_vp, ctypes.c_int32] + [_vp] * 8),
    ("brisk_packed_load", ctypes.c_int, [_vp, ctypes.c_int32] + [_vp] * 8),
    ("brisk_packed_attend", ctypes.c_int, [_vp] * 8 + [ctypes.c_float, _vp, _vp, _vp, _vp]),
]


_BUILD_IT = "build it with `python -c 'import __graft_entry__ as g; g.build()'`"


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: {_BUILD_IT}")
        h = ctypes.CDLL(LIB_PATH)
        for name, res, args in _SIGS:
            f = getattr(h, name)
            f.restype = res
            f.argtypes = args
        _lib = h
    return _lib


def marshal():
    """The module that marshals calls in their usual form; raises if it has not been built for this interpreter and torch."""
    try:
        from . import _marshal
    except ImportError as e:
        raise RuntimeError(f"the binding's module _marshal is missing, or another torch's ({e}): {_BUILD_IT}") from e
    return _marshal


def set_wait_limit(cycles: int) -> int:
    """Limit (SM cycles) of the library's bounded device-side waits; <= 0 restores the default.
    Returns the previous limit."""
    return int(lib().brisk_set_wait_limit(int(cycles)))


def status_string(s: int) -> str:
    return lib().brisk_status_string(int(s)).decode()


def _check(s: int, where: str) -> None:
    if s != OK:
        raise BriskError(s, where)


def _dt(t: torch.dtype) -> int:
    if t == torch.bfloat16:
        return DT_BF16
    if t == torch.float32:
        return DT_F32
    raise ValueError(f"unsupported dtype {t}")


# Marshalling is part of every small call (20 us of 22 for a distillation loss of 128 blocks), so
# pointers travel as plain integers, which the declared argument types convert, and the current
# stream is looked up by its handle, without a Stream object.
def _p(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return t.data_ptr()


def _stream(stream=None):
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def _results(stream, make):
    """make()'s new tensors (a dict), for a call on ``stream`` to write. They are allocated for that stream:
    memory of the current one may be what a kernel still pending there reads or writes, and would be free
    for it again, once dropped, while the call still writes. Whoever reads them on the current stream
    may drop them without waiting, too."""
    if stream is None or stream.cuda_stream == _stream():
        return make()
    here = torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        new = make()
    for t in new.values():
        t.record_stream(here)
    return new


def _lend(stream, *buffers):
    """An object's own buffers to a call on ``stream``: dropped with the object, they are not free for the current
    stream before the call has ended."""
    if stream is not None and stream.cuda_stream != _stream():
        for t in buffers:
            t.record_stream(stream)


def _settle(device):
    """Waits for what the current stream does with new buffers (their clearing, and what their memory was used
    for before): calls may go to any stream. Not under capture, where the calls are the capture's, too."""
    if device.type == "cuda" and not torch.cuda.is_current_stream_capturing():
        torch.cuda.current_stream(device).synchronize()


def make_dims(B, L, V, d, K, r, logits_dtype, hidden_dtype) -> Dims:
    return Dims(B, L, V, d, K, r, _dt(logits_dtype), _dt(hidden_dtype))


def workspace_bytes(dims: Dims) -> int:
    return int(lib().brisk_workspace_bytes(ctypes.byref(dims)))


def tables_bytes(dims: Dims) -> int:
    return int(lib().brisk_tables_bytes(ctypes.byref(dims)))


def kernels_per_tail(dims: Dims) -> int:
    return int(lib().brisk_kernels_per_tail(ctypes.byref(dims)))


def topk_candidates_noalloc(dims: Dims, logits_q, cand_ids, cand_logprob, lse_q, stream=None) -> int:
    """Step 1 without a workspace, for callers that cannot allocate device memory; the
    library's own fixed scratch array is used instead. Returns the status code."""
    return int(lib().brisk_topk_candidates_noalloc(ctypes.byref(dims), _p(logits_q), _p(cand_ids),
                                                   _p(cand_logprob), _p(lse_q), _stream(stream)))


def make_params(w: Dict[str, object]) -> Params:
    names = ("E_in", "E_out", "P_h", "P_e", "P_phi", "pos", "W0", "Wz", "Wh", "W_s", "W_c", "w_g")
    return Params(*[_p(w[n]) for n in names], float(w["b_g"]), float(w["alpha"]))


class DecodeTail:
    """Device buffers and calls of the decode tail for one problem size and weight set.

    ``weights`` holds the corrector parameters and E_in / E_out as CUDA tensors in the hidden
    dtype (see ``synth.make_weights``). The workspace and the folded tables are allocated once
    here with torch; the library itself never allocates. What a call given a ``stream`` allocates
    itself is that stream's memory (see _results).
    """

    def __init__(self, B, L, V, d, K, r, logits_dtype, hidden_dtype, weights, device="cuda"):
        self.dims = make_dims(B, L, V, d, K, r, logits_dtype, hidden_dtype)
        self.B, self.L, self.V, self.d, self.K, self.r = B, L, V, d, K, r
        self.device = torch.device(device)
        ws = workspace_bytes(self.dims)
        tb = tables_bytes(self.dims)
        if ws == 0 or tb == 0:
            raise BriskError(ERR_INVALID_ARG, "dims")
        self.workspace = torch.zeros(ws, dtype=torch.uint8, device=self.device)
        self.tables = torch.empty(tb, dtype=torch.uint8, device=self.device)
        _settle(self.device)
        self.weights = weights
        self.params = make_params(weights)
        self.prepared = False

    @classmethod
    def for_workload(cls, wl, weights, device="cuda", B=None):
        return cls(wl.B if B is None else B, wl.L, wl.V, wl.d, wl.K, wl.r, wl.logits_dtype,
                   wl.hidden_dtype, weights, device)

    def prepare(self, stream=None):
        _lend(stream, self.tables)
        _check(lib().brisk_corrector_prepare(ctypes.byref(self.dims), ctypes.byref(self.params),
                                             _p(self.tables), _stream(stream)), "prepare")
        self.prepared = True

    def _i32(self, *shape):
        return torch.empty(shape, dtype=torch.int32, device=self.device)

    def _f32(self, *shape):
        return torch.empty(shape, dtype=torch.float32, device=self.device)

    def topk(self, logits_q, stream=None):
        B, L, K = self.B, self.L, self.K
        out = _results(stream, lambda: {"cand_ids": self._i32(B, L, K), "cand_logprob": self._f32(B, L, K),
                                        "lse_q": self._f32(B, L)})
        _lend(stream, self.workspace, self.tables)
        _check(lib().brisk_topk_candidates(ctypes.byref(self.dims), _p(logits_q), _p(out["cand_ids"]),
                                           _p(out["cand_logprob"]), _p(out["lse_q"]), _p(self.workspace),
                                           _stream(stream)), "topk")
        return out

    def select(self, hidden, h_ctx, x0, logits_q, cand_ids, cand_logprob, select_mode=SELECT_GREEDY,
               u_sel=None, stream=None):
        B, L, K = self.B, self.L, self.K
        out = _results(stream, lambda: {"sel_tokens": self._i32(B, L), "refined": self._f32(B, L, K)})
        _lend(stream, self.workspace, self.tables)
        _check(lib().brisk_corrector_select(
            ctypes.byref(self.dims), ctypes.byref(self.params), _p(self.tables), _p(hidden), _p(h_ctx),
            _p(x0), _p(logits_q), _p(cand_ids), _p(cand_logprob), int(select_mode), _p(u_sel),
            _p(out["sel_tokens"]), _p(out["refined"]), _p(self.workspace), _stream(stream)), "select")
        return out

    def verify(self, logits_p, sel_tokens, cand_ids, refined, select_mode=SELECT_GREEDY,
               verify_mode=VERIFY_GREEDY, u_acc=None, u_res=None, stream=None):
        B, L = self.B, self.L
        out = _results(stream, lambda: {"accepted_len": self._i32(B), "out_tokens": self._i32(B, L),
                                        "correction": self._i32(B)})
        _lend(stream, self.workspace, self.tables)
        _check(lib().brisk_verify_block(
            ctypes.byref(self.dims), _p(logits_p), _p(sel_tokens), _p(cand_ids), _p(refined),
            int(select_mode), int(verify_mode), _p(u_acc), _p(u_res), _p(out["accepted_len"]),
            _p(out["out_tokens"]), _p(out["correction"]), _p(self.workspace), _stream(stream)), "verify")
        return out

    def replay(self, block, select_mode=SELECT_GREEDY, stream=None):
        """Same-state replay diagnostics (App. B, Eq. 6) of one block (see synth.make_block)."""
        B, L, K = self.B, self.L, self.K
        out = _results(stream, lambda: {"head_tokens": self._i32(B, L), "flags": self._i32(B, L),
                                        "first_breaker": self._i32(B), "refined": self._f32(B, L, K)})
        _lend(stream, self.workspace, self.tables)
        _check(lib().brisk_replay_diagnostics(
            ctypes.byref(self.dims), ctypes.byref(self.params), _p(self.tables),
            _p(block["hidden"]), _p(block["h_c"]), _p(block["x0"]), _p(block["logits_q"]),
            _p(block["logits_p"]), int(select_mode), _p(block["u_sel"]), _p(block["u_acc"]),
            _p(out["head_tokens"]), _p(out["flags"]), _p(out["first_breaker"]), _p(out["refined"]),
            _p(self.workspace), _stream(stream)), "replay_diagnostics")
        return out

    def distill_loss(self, logits_p, cand_ids, cand_logprob, refined, accepted_len, beta=0.01,
                     with_grad=True, stream=None):
        """Distillation loss of the refinement head (App. C.3, Eq. 10) and its gradient in the
        refined scores."""
        def new():
            loss = {"loss": self._f32(1)}
            return dict(loss, grad=self._f32(self.B, self.L, self.K)) if with_grad else loss
        out = _results(stream, new)
        _lend(stream, self.workspace, self.tables)
        _check(lib().brisk_distill_loss(
            ctypes.byref(self.dims), _p(logits_p), _p(cand_ids), _p(cand_logprob), _p(refined),
            _p(accepted_len), float(beta), _p(out["loss"]), _p(out.get("grad")), _p(self.workspace),
            _stream(stream)), "distill_loss")
        out.setdefault("grad", None)
        return out

    def alloc_outputs(self, full=True):
        B, L, K = self.B, self.L, self.K
        o = {"accepted_len": self._i32(B), "out_tokens": self._i32(B, L), "correction": self._i32(B),
             "next_anchor": self._i32(B)}
        if full:
            o.update(cand_ids=self._i32(B, L, K), cand_logprob=self._f32(B, L, K),
                     lse_q=self._f32(B, L), sel_tokens=self._i32(B, L), refined=self._f32(B, L, K))
        return o

    @staticmethod
    def _io(block, out, x0):
        return TailIO(_p(block["logits_q"]), _p(block["logits_p"]), _p(block["hidden"]),
                      _p(block["h_c"]), _p(block["x0"] if x0 is None else x0), _p(block.get("u_sel")),
                      _p(block.get("u_acc")), _p(block.get("u_res")), _p(out.get("cand_ids")),
                      _p(out.get("cand_logprob")), _p(out.get("lse_q")), _p(out.get("sel_tokens")),
                      _p(out.get("refined")), _p(out["accepted_len"]), _p(out["out_tokens"]),
                      _p(out["correction"]), _p(out.get("next_anchor")))

    def tail(self, block, select_mode=SELECT_GREEDY, verify_mode=VERIFY_GREEDY, out=None, x0=None,
             events=None, stream=None):
        """One fused decode-tail call on the tensors of ``block`` (see ``synth.make_block``)."""
        if out is None:
            out = _results(stream, self.alloc_outputs)
        io = self._io(block, out, x0)
        _lend(stream, self.workspace, self.tables)
        ev = None
        if events is not None:
            ev = ctypes.byref(Events(*[_vp(e.cuda_event) for e in events]))
        _check(lib().brisk_decode_tail(ctypes.byref(self.dims), ctypes.byref(self.params),
                                       _p(self.tables), ctypes.byref(io), int(select_mode),
                                       int(verify_mode), _p(self.workspace), ev, _stream(stream)),
               "decode_tail")
        return out

    def graph(self, block, select_mode=SELECT_GREEDY, verify_mode=VERIFY_GREEDY, out=None,
              chain_anchor=True, stream=None):
        """The decode tail on these buffers captured into a replayable CUDA graph (App. F). With
        chain_anchor the anchor buffer is also the next-anchor output, so replays chain blocks."""
        return TailGraph(self, block, select_mode, verify_mode, out, chain_anchor, stream)

    def device_status(self, clear=True, stream=None) -> int:
        return int(lib().brisk_last_device_status(_p(self.workspace), int(clear), _stream(stream)))


class TailGraph:
    """A captured decode tail (see brisk_tail_graph_create); launch() replays it."""

    def __init__(self, tail, block, select_mode, verify_mode, out, chain_anchor, stream):
        if stream is None:
            raise ValueError("capture needs a non-default stream")
        self.tail = tail
        self.block = block
        self.out = tail.alloc_outputs() if out is None else out
        if chain_anchor:
            self.anchor = block["x0"].clone()
            self.out["next_anchor"] = self.anchor
        else:
            self.anchor = block["x0"]
        self.stream = stream
        self._iob = tail._io(block, self.out, self.anchor)
        # (replays may be pending when the graph and its buffers are dropped)
        _lend(stream, tail.workspace, tail.tables, self.anchor, *(t for t in self.out.values() if t is not None))
        saved = self.anchor.clone()
        torch.cuda.synchronize()
        h = _vp()
        _check(lib().brisk_tail_graph_create(ctypes.byref(tail.dims), ctypes.byref(tail.params),
                                             _p(tail.tables), ctypes.byref(self._iob),
                                             int(select_mode), int(verify_mode),
                                             _p(tail.workspace), _stream(stream), ctypes.byref(h)),
               "tail_graph_create")
        self.handle = h
        # the direct call inside create advanced a chained anchor: start the replays from x0
        with torch.cuda.stream(stream):
            self.anchor.copy_(saved)
        stream.synchronize()

    def launch(self):
        _check(lib().brisk_tail_graph_launch(self.handle, _stream(self.stream)), "tail_graph_launch")
        return self.out

    def close(self):
        if self.handle:
            lib().brisk_tail_graph_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def mode_ids(select_mode: str, verify_mode: str):
    return (SELECT_SAMPLE if select_mode == "sample" else SELECT_GREEDY,
            VERIFY_STOCHASTIC if verify_mode == "stochastic" else VERIFY_GREEDY)


# ---------------------------------------------------------------- acceptance profile

def acceptance_counts(accepted_len: torch.Tensor, L: int, counts: torch.Tensor, stream=None) -> None:
    """Adds one step's accepted lengths ([B] int32, device) to running per-position counts
    (counts: [2L] int64 device tensor used as uint64; reached first, then accepted)."""
    if accepted_len.dtype != torch.int32 or counts.dtype != torch.int64 or counts.numel() != 2 * L:
        raise ValueError("accepted_len int32 [B], counts int64 [2L]")
    _check(lib().brisk_acceptance_counts(_p(accepted_len), int(accepted_len.numel()), int(L),
                                         _p(counts), _stream(stream)), "acceptance_counts")


def acceptance_weights(a, g=None, c=None, eps: float = 1e-8):
    """TPF, w_raw and the mean-one w_bar of a profile a[0..M-1] (host, float64)."""
    import numpy as np
    a = np.ascontiguousarray(a, dtype=np.float64)
    M = a.size
    gg = None if g is None else np.ascontiguousarray(g, dtype=np.float64)
    cc = None if c is None else np.ascontiguousarray(c, dtype=np.float64)
    if (gg is not None and gg.size != M + 1) or (cc is not None and cc.size != M + 1):
        raise ValueError("g and c need M + 1 entries")
    tpf = ctypes.c_double()
    w_raw = np.empty(M)
    w_bar = np.empty(M)
    vp = lambda x: None if x is None else x.ctypes.data_as(ctypes.c_void_p)
    _check(lib().brisk_acceptance_weights(M, vp(a), vp(gg), vp(cc), float(eps), ctypes.byref(tpf),
                                          vp(w_raw), vp(w_bar)), "acceptance_weights")
    return tpf.value, w_raw, w_bar


def isd_costs(M: int):
    """Gains g[0..M] and costs c[0..M] of the ISD instantiation (App. C.1, Eq. 8)."""
    import numpy as np
    g = np.zeros(int(M) + 1, dtype=np.float64)
    c = np.zeros(int(M) + 1, dtype=np.float64)
    _check(lib().brisk_isd_costs(int(M), g.ctypes.data_as(ctypes.c_void_p),
                                 c.ctypes.data_as(ctypes.c_void_p)), "isd_costs")
    return g, c


def tpf_isd(N: int, r: float) -> float:
    return float(lib().brisk_tpf_isd(int(N), float(r)))


# ---------------------------------------------------------------- context cache

_PACK2, _PACK4, _PACK5 = (struct.Struct(f"{4 * n}q").pack_into for n in (2, 4, 5))   # n Views
_NONE = (0, 0, 0, 0)

class PrefixAttention:
    """Attention of a batch's blocks over a shared prefix and the sequences' own caches, the weight
    it gave each own entry, and the eviction by that weight, for one problem size.

    B sequences of L query positions, ``Hq`` query heads over ``Hkv`` key heads of width ``D``, ``P``
    shared prefix entries, room for ``S`` own entries a sequence; queries, keys and values in
    ``dtype`` (bf16 or fp32). Tensors are [.., positions, heads, D] with any strides whose rows
    start on 16 bytes (a transposed cache, a slice of a fused projection); lengths, sums and
    outputs are contiguous. The workspace is allocated once here, so calls of one object must not overlap.
    What a call given a ``stream`` allocates itself is that stream's memory (see _results).
    """

    _VIEWS = 5 * ctypes.sizeof(View)

    @staticmethod
    def _workspace_bytes():
        return lib().brisk_cache_workspace_bytes

    def __init__(self, B, L, Hq, Hkv, D, P, S, dtype, device="cuda"):
        self.dims = CacheDims(B, L, Hq, Hkv, D, P, S, _dt(dtype))
        self.B, self.L, self.Hq, self.Hkv, self.D, self.P, self.S = B, L, Hq, Hkv, D, P, S
        self.dtype, self.device = dtype, torch.device(device)
        ws = int(self._workspace_bytes()(ctypes.byref(self.dims)))
        if ws == 0:
            raise BriskError(ERR_INVALID_ARG, "dims")
        self.workspace = torch.zeros(ws, dtype=torch.uint8, device=self.device)
        _settle(self.device)
        self.scale = D ** -0.5
        self._d = ctypes.addressof(self.dims)
        self._ws = self.workspace.data_ptr()
        # the views of a call's strided tensors, written anew by every call
        self._views = ctypes.create_string_buffer(self._VIEWS)
        at = ctypes.addressof(self._views)
        self._at = [at + i * ctypes.sizeof(View) for i in range(5)]
        self._shape_q, self._shape_pre, self._shape_own = (B, L, Hq, D), (P, Hkv, D), (B, S, Hkv, D)
        self._shape_lse, self._shape_acc, self._shape_b, self._shape_vis = (B, L, Hq), (B, Hkv, S), (B,), (B, L)

    # Marshalling is most of a small call, so a tensor's checks are few comparisons, and the views of a call
    # are packed at once.
    def _view(self, t, shape, what):
        """The tensor's address and strides; None for one that a size of zero leaves out."""
        if t is None:
            if 0 in shape:
                return None
            raise ValueError(f"{what} is missing")
        if t.shape != shape or t.dtype != self.dtype:
            raise ValueError(f"{what}: {tuple(t.shape)} {t.dtype}, not {tuple(shape)} {self.dtype}")
        if not t.is_cuda:
            raise ValueError(f"{what} is not on the GPU")
        st = t.stride()
        if st[-1] != 1:
            raise ValueError(f"{what}: the last dimension must be contiguous")
        return (t.data_ptr(), *st[:3]) if len(st) == 4 else (t.data_ptr(), 0, st[0], st[1])

    @staticmethod
    def _plain(t, shape, dtype, what):
        if t is None:
            return None
        if t.shape != shape or t.dtype != dtype:
            raise ValueError(f"{what}: {tuple(t.shape)} {t.dtype}, not {tuple(shape)} {dtype}")
        if not t.is_cuda:
            raise ValueError(f"{what} is not on the GPU")
        return _p(t)

    def _attended(self):
        return {"out": torch.empty(self._shape_q, dtype=self.dtype, device=self.device),
                "lse": torch.empty(self._shape_lse, dtype=torch.float32, device=self.device)}

    def _weighed(self):
        return {"acc": torch.empty(self._shape_acc, dtype=torch.float32, device=self.device)}

    def attend(self, q, k_prefix, v_prefix, k_own, v_own, own_len, visible=None, scale=None,
               out=None, stream=None):
        """out [B, L, Hq, D] and lse [B, L, Hq] of the queries q [B, L, Hq, D] over k/v_prefix
        [P, Hkv, D] and the entries of k/v_own [B, S, Hkv, D] that own_len [B] and visible [B, L]
        (int32; see brisk_prefix_attend) let them see. scale: D^-1/2 unless given. ``out``: a dict
        of tensors to write to instead of new ones."""
        pre, own, view, plain, at = self._shape_pre, self._shape_own, self._view, self._plain, self._at
        if out is None:
            out = _results(stream, self._attended)
        _PACK5(self._views, 0, *view(q, self._shape_q, "q"), *(view(k_prefix, pre, "k_prefix") or _NONE),
               *(view(v_prefix, pre, "v_prefix") or _NONE), *(view(k_own, own, "k_own") or _NONE),
               *(view(v_own, own, "v_own") or _NONE))
        _lend(stream, self.workspace)
        s = lib().brisk_prefix_attend(
            self._d, at[0], at[1], at[2], at[3], at[4],
            plain(own_len, self._shape_b, torch.int32, "own_len"),
            plain(visible, self._shape_vis, torch.int32, "visible"),
            self.scale if scale is None else scale,
            plain(out["out"], self._shape_q, self.dtype, "out"),
            plain(out["lse"], self._shape_lse, torch.float32, "lse"), self._ws, _stream(stream))
        if s:
            raise BriskError(s, "prefix_attend")
        return out

    def weights(self, q, lse, k_own, own_len, acc=None, decay=1.0, visible=None, scale=None,
                out=None, stream=None):
        """decay * acc plus the attention weight every own entry got from the queries whose
        log-sums ``lse`` attend() left: [B, Hkv, S] fp32, in ``out`` (which may be ``acc``) or a
        new tensor. acc None: zeros."""
        plain, at, f32, i32 = self._plain, self._at, torch.float32, torch.int32
        if out is None:
            out = _results(stream, self._weighed)["acc"]
        _PACK2(self._views, 0, *self._view(q, self._shape_q, "q"),
               *(self._view(k_own, self._shape_own, "k_own") or _NONE))
        _lend(stream, self.workspace)
        s = lib().brisk_cache_weights(
            self._d, at[0], plain(lse, self._shape_lse, f32, "lse"), at[1],
            plain(own_len, self._shape_b, i32, "own_len"),
            plain(visible, self._shape_vis, i32, "visible"), self.scale if scale is None else scale,
            decay, plain(acc, self._shape_acc, f32, "acc"), plain(out, self._shape_acc, f32, "out"),
            self._ws, _stream(stream))
        if s:
            raise BriskError(s, "cache_weights")
        return out

    def alloc_evicted(self, keep, room=None):
        """Targets of evict(): caches [B, room, Hkv, D] (room: ``keep`` unless given), sums and kept
        indices [B, Hkv, keep], lengths [B]; zeros, written on the current stream."""
        return self._evicted(torch.zeros, keep, keep if room is None else room)

    def _evicted(self, make, keep, room):
        B, Hkv, D = self.B, self.Hkv, self.D
        new = lambda shape, dt: make(shape, dtype=dt, device=self.device)
        return {"k": new((B, room, Hkv, D), self.dtype), "v": new((B, room, Hkv, D), self.dtype),
                "acc": new((B, Hkv, keep), torch.float32),
                "own_len": new((B,), torch.int32), "kept": new((B, Hkv, keep), torch.int32)}

    def evict(self, k_own, v_own, acc, own_len, keep, recent, out=None, stream=None):
        """Moves the ``recent`` newest entries and those of largest ``acc`` [B, Hkv, S], ``keep`` in
        all, to the caches of ``out`` (see alloc_evicted and brisk_cache_evict): between two layers,
        one spare pair of caches serves them all in turn."""
        if out is None:
            # (the call writes all of them)
            out = _results(stream, lambda: self._evicted(torch.empty, keep, keep))
        plain, view, at, f32, i32 = self._plain, self._view, self._at, torch.float32, torch.int32
        k_to, B, Hkv = out["k"], self.B, self.Hkv
        room = k_to.shape[1]
        if room < keep:
            raise ValueError(f"the targets hold {room} entries, keep is {keep}")
        own, to, kept = self._shape_own, (B, room, Hkv, self.D), (B, Hkv, keep)
        _PACK4(self._views, 0, *(view(k_own, own, "k_own") or _NONE), *(view(v_own, own, "v_own") or _NONE),
               *view(k_to, to, "k"), *view(out["v"], to, "v"))
        _lend(stream, self.workspace)
        s = lib().brisk_cache_evict(
            self._d, at[0], at[1], plain(acc, self._shape_acc, f32, "acc"),
            plain(own_len, self._shape_b, i32, "own_len"), keep, recent, at[2], at[3],
            plain(out["acc"], kept, f32, "out acc"), plain(out["own_len"], self._shape_b, i32, "out own_len"),
            plain(out["kept"], kept, i32, "kept"), self._ws, _stream(stream))
        if s:
            raise BriskError(s, "cache_evict")
        return out

    def device_status(self, clear=True, stream=None) -> int:
        return int(lib().brisk_last_device_status(self._ws, int(clear), _stream(stream)))


_PACK_ATTEND, _PACK_MOVE = (struct.Struct(f"{n}q").pack_into for n in (3 * 4 + 2 * 8, 2 * 4 + 2 * 8))
_NO_CACHE = (0,) * 16


class PackedAttention(PrefixAttention):
    """PrefixAttention whose own caches are held in 4 bits (see brisk_packed in brisk.h for the format; D a
    multiple of 16): entries are written with store(), read back with load() and attended over with
    attend(). The prefix stays in ``dtype``.

    A cache is a dict of uint8 tensors, ``k`` and ``v`` [B, S, Hkv, D / 2] and ``k_scales`` and
    ``v_scales`` [B, S, Hkv, 4 or 8] (see alloc_cache), of any strides whose rows are contiguous and start
    on 16 bytes (8 where D % 32 is not 0), or on their length; bytes of scales behind the first D / 16 may hold anything. The weights of own entries and the eviction by them
    work on entries in ``dtype``: PrefixAttention's, on what load() gives; storing that again gives the same bytes.
    """

    _VIEWS = 3 * 4 * 8 + 2 * 8 * 8

    @staticmethod
    def _workspace_bytes():
        return lib().brisk_packed_workspace_bytes

    def __init__(self, B, L, Hq, Hkv, D, P, S, dtype, device="cuda"):
        super().__init__(B, L, Hq, Hkv, D, P, S, dtype, device)
        self._shape_codes, self._shape_scales = (B, S, Hkv, D // 2), (B, S, Hkv, 4 if D <= 64 else 8)
        at = self._at[0]
        self._at_attend = [at, at + 32, at + 64, at + 96, at + 160]
        self._at_move = [at, at + 32, at + 64, at + 128]
        # a call in its usual form is marshalled there; the ways below are for results given, other streams, refusals
        quick = marshal()
        self._quick_store, self._quick_load, self._quick_attend = quick.store, quick.load, quick.attend
        entry = lambda f: ctypes.cast(f, _vp).value
        self._f_store, self._f_load = entry(lib().brisk_packed_store), entry(lib().brisk_packed_load)
        self._f_attend = entry(lib().brisk_packed_attend)

    def alloc_cache(self, order="token"):
        """A cache of zeros, written on the current stream: in memory [B, S, Hkv, ..] ("token") or
        [B, Hkv, S, ..] ("head": an entry's neighbours in time lie side by side)."""
        if order not in ("token", "head"):
            raise ValueError(f"order {order!r} is neither 'token' nor 'head'")

        def new(shape):
            if order == "token":
                return torch.zeros(shape, dtype=torch.uint8, device=self.device)
            B, S, H, n = shape
            return torch.zeros((B, H, S, n), dtype=torch.uint8, device=self.device).transpose(1, 2)
        return {"k": new(self._shape_codes), "k_scales": new(self._shape_scales),
                "v": new(self._shape_codes), "v_scales": new(self._shape_scales)}

    def _bytes(self, t, shape, what):
        if t.shape != shape or t.dtype != torch.uint8:
            raise ValueError(f"{what}: {tuple(t.shape)} {t.dtype}, not {tuple(shape)} uint8")
        if not t.is_cuda:
            raise ValueError(f"{what} is not on the GPU")
        st = t.stride()
        if st[3] != 1:
            raise ValueError(f"{what}: the last dimension must be contiguous")
        return t.data_ptr(), st

    def _cache(self, cache):
        """The eight numbers of keys' and of values' brisk_packed."""
        if self.S == 0:
            return _NO_CACHE
        if cache is None:
            raise ValueError("the cache is missing")
        of, codes, scales = self._bytes, self._shape_codes, self._shape_scales
        k, a = of(cache["k"], codes, "k")
        ks, b = of(cache["k_scales"], scales, "k_scales")
        v, c = of(cache["v"], codes, "v")
        vs, d = of(cache["v_scales"], scales, "v_scales")
        return (k, ks, a[0], a[1], a[2], b[0], b[1], b[2], v, vs, c[0], c[1], c[2], d[0], d[1], d[2])

    def store(self, cache, k, v, start, count=None, stream=None):
        """Quantises rows t < count[b] (all T unless given) of k, v [B, T, Hkv, D] into places
        start[b] + t of ``cache`` (start, count [B] int32; see brisk_packed_store)."""
        if stream is None:
            s = self._quick_store(self._f_store, self._d, self.workspace, cache, k, v, start, count)
            if s is not None:
                _check(s, "packed_store")
                return cache
        T = k.shape[1]
        shape, plain, at, i32 = (self.B, T, self.Hkv, self.D), self._plain, self._at_move, torch.int32
        _PACK_MOVE(self._views, 0, *self._view(k, shape, "k"), *self._view(v, shape, "v"), *self._cache(cache))
        _lend(stream, self.workspace)
        s = lib().brisk_packed_store(self._d, T, at[0], at[1], plain(start, self._shape_b, i32, "start"),
                                     plain(count, self._shape_b, i32, "count"), at[2], at[3], self._ws,
                                     _stream(stream))
        if s:
            raise BriskError(s, "packed_store")
        return cache

    def load(self, cache, T, start, count=None, out=None, stream=None):
        """k, v [B, T, Hkv, D]: in rows t < count[b] (all T unless given) what places start[b] + t of
        ``cache`` stand for, else zeros. ``out``: a dict of tensors to write to instead of new ones."""
        if out is None and stream is None:
            r = self._quick_load(self._f_load, self._d, self.workspace, cache, T, start, count)
            if r.__class__ is dict:
                return r
            if r is not None:
                raise BriskError(r, "packed_load")
        H, D, plain, at, i32 = self.Hkv, self.D, self._plain, self._at_move, torch.int32
        shape = (self.B, T, H, D)
        if out is None:
            new = lambda: {"k": torch.empty(shape, dtype=self.dtype, device=self.device),
                           "v": torch.empty(shape, dtype=self.dtype, device=self.device)}
            out = new() if stream is None else _results(stream, new)
            k, v = ((out[n].data_ptr(), T * H * D, H * D, D) for n in "kv")
        else:
            k, v = self._view(out["k"], shape, "k"), self._view(out["v"], shape, "v")
        _PACK_MOVE(self._views, 0, *k, *v, *self._cache(cache))
        _lend(stream, self.workspace)
        s = lib().brisk_packed_load(self._d, T, at[2], at[3], plain(start, self._shape_b, i32, "start"),
                                    plain(count, self._shape_b, i32, "count"), at[0], at[1], self._ws,
                                    _stream(stream))
        if s:
            raise BriskError(s, "packed_load")
        return out

    def attend(self, q, k_prefix, v_prefix, cache, own_len, visible=None, scale=None, out=None, stream=None):
        """PrefixAttention.attend with the own entries in ``cache`` (None if S == 0)."""
        scale = self.scale if scale is None else scale
        if out is None and stream is None:
            r = self._quick_attend(self._f_attend, self._d, self.workspace, scale, q, k_prefix, v_prefix, cache,
                                   own_len, visible)
            if r.__class__ is dict:
                return r
            if r is not None:
                raise BriskError(r, "packed_attend")
        pre, view, plain, at = self._shape_pre, self._view, self._plain, self._at_attend
        if out is None:
            out = self._attended() if stream is None else _results(stream, self._attended)
            to, lse = out["out"].data_ptr(), out["lse"].data_ptr()
        else:
            to = plain(out["out"], self._shape_q, self.dtype, "out")
            lse = plain(out["lse"], self._shape_lse, torch.float32, "lse")
        _PACK_ATTEND(self._views, 0, *view(q, self._shape_q, "q"), *(view(k_prefix, pre, "k_prefix") or _NONE),
                     *(view(v_prefix, pre, "v_prefix") or _NONE), *self._cache(cache))
        _lend(stream, self.workspace)
        s = lib().brisk_packed_attend(
            self._d, at[0], at[1], at[2], at[3], at[4],
            plain(own_len, self._shape_b, torch.int32, "own_len"),
            plain(visible, self._shape_vis, torch.int32, "visible"),
            scale, to, lse, self._ws, _stream(stream))
        if s:
            raise BriskError(s, "packed_attend")
        return out

    def weights(self, *args, **kwargs):
        raise TypeError("weights() of a PrefixAttention takes the entries that load() gives")

    def evict(self, *args, **kwargs):
        raise TypeError("evict() of a PrefixAttention takes the entries that load() gives")
