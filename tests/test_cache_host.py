"""Refusals of the context-cache calls: found on the host, before any CUDA call."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2609_33390_gb300 import build
    build.build()
    from paper_2609_33390_gb300 import brisk
    return brisk


def _dims(lib_mod, **kw):
    d = dict(B=2, L=3, Hq=8, Hkv=2, D=64, P=100, S=50, dtype=lib_mod.DT_BF16)
    d.update(kw)
    return lib_mod.CacheDims(*[d[n] for n, _ in lib_mod.CacheDims._fields_])


def test_workspace_of_valid_and_invalid_sizes(B):
    size = lambda **kw: B.lib().brisk_cache_workspace_bytes(ctypes.byref(_dims(B, **kw)))
    assert size() > 0 and size() % 256 == 0
    for ok in (dict(P=0), dict(S=0), dict(D=8), dict(D=128), dict(B=4096), dict(dtype=B.DT_F32),
               dict(Hq=2), dict(L=1000)):
        assert size(**ok) > 0, ok
    for bad in (dict(B=0), dict(B=4097), dict(L=0), dict(Hq=7), dict(Hq=1), dict(Hkv=0), dict(D=4),
                dict(D=12), dict(D=136), dict(P=-1), dict(S=-1), dict(dtype=2), dict(dtype=-1),
                dict(B=4096, L=1 << 20), dict(P=(1 << 30) + 1)):
        assert size(**bad) == 0, bad
    assert B.lib().brisk_cache_workspace_bytes(None) == 0


def _views(B, d, es=2):
    D, Hkv = d.D, d.Hkv
    fake = 1 << 20                                    # never dereferenced: validation fails first
    q = B.View(fake, d.L * d.Hq * D, d.Hq * D, D)
    pre = B.View(fake, 0, Hkv * D, D)
    own = B.View(fake, d.S * Hkv * D, Hkv * D, D)
    return q, pre, own


def _attend(B, d, q, kp, vp, ko, vo, lens=256, scale=0.1, out=256, ws=256):
    ref = lambda v: None if v is None else ctypes.byref(v)
    return B.lib().brisk_prefix_attend(ctypes.byref(d), ref(q), ref(kp), ref(vp), ref(ko), ref(vo),
                                       lens, None, scale, out, None, ws, None)


def _with(B, v, **kw):
    f = {n: getattr(v, n) for n, _ in B.View._fields_}
    f.update(kw)
    return B.View(f["ptr"], f["seq"], f["tok"], f["head"])


def test_attend_refuses(B):
    d = _dims(B)
    q, pre, own = _views(B, d)
    bad = [
        _attend(B, _dims(B, D=20), q, pre, pre, own, own),
        _attend(B, d, None, pre, pre, own, own),
        _attend(B, d, q, None, pre, own, own),
        _attend(B, d, q, pre, None, own, own),
        _attend(B, d, q, pre, pre, None, own),
        _attend(B, d, q, pre, pre, own, None),
        _attend(B, d, q, pre, pre, own, own, lens=None),
        _attend(B, d, q, pre, pre, own, own, out=None),
        _attend(B, d, q, pre, pre, own, own, out=264),
        _attend(B, d, q, pre, pre, own, own, ws=None),
        _attend(B, d, q, pre, pre, own, own, ws=128),
        _attend(B, d, q, pre, pre, own, own, scale=-1.0),
        _attend(B, d, q, pre, pre, own, own, scale=float("inf")),
        _attend(B, d, q, pre, pre, own, own, scale=float("nan")),
        _attend(B, d, _with(B, q, ptr=q.ptr + 8), pre, pre, own, own),
        _attend(B, d, _with(B, q, tok=q.tok + 4), pre, pre, own, own),
        _attend(B, d, q, _with(B, pre, tok=0), pre, own, own),
        _attend(B, d, q, _with(B, pre, tok=-pre.tok), pre, own, own),
        _attend(B, d, q, pre, _with(B, pre, head=32), own, own),
        _attend(B, d, q, pre, pre, _with(B, own, seq=1 << 50), own),
        _attend(B, d, q, pre, pre, own, _with(B, own, ptr=None)),
    ]
    assert bad == [B.ERR_INVALID_ARG] * len(bad)


def test_weights_refuse(B):
    d = _dims(B)
    q, _, own = _views(B, d)

    def call(d=d, q=q, lse=256, k=own, lens=256, scale=0.1, decay=1.0, out=256, ws=256):
        ref = lambda v: None if v is None else ctypes.byref(v)
        return B.lib().brisk_cache_weights(ctypes.byref(d), ref(q), lse, ref(k), lens, None, scale, decay,
                                           None, out, ws, None)
    bad = [call(d=_dims(B, Hq=9)), call(q=None), call(lse=None), call(k=None), call(lens=None),
           call(scale=float("nan")), call(decay=float("inf")), call(out=None), call(ws=None),
           call(ws=300), call(k=_with(B, own, seq=7))]
    assert bad == [B.ERR_INVALID_ARG] * len(bad)


def test_evict_refuses(B):
    d = _dims(B)
    _, _, own = _views(B, d)
    to = [_with(B, own, ptr=own.ptr * (2 + i)) for i in range(2)]
    kv = [own, _with(B, own, ptr=own.ptr * 5)]

    def call(d=d, k=kv[0], v=kv[1], acc=256, lens=256, keep=10, recent=2, kt=to[0], vt=to[1], acc_to=512,
             len_to=512, kept=768, ws=256):
        ref = lambda x: None if x is None else ctypes.byref(x)
        return B.lib().brisk_cache_evict(ctypes.byref(d), ref(k), ref(v), acc, lens, keep, recent, ref(kt),
                                         ref(vt), acc_to, len_to, kept, ws, None)
    bad = [call(keep=0), call(keep=-1), call(recent=-1), call(recent=11), call(k=None), call(vt=None),
           call(acc=None), call(lens=None), call(acc_to=None), call(len_to=None), call(kept=None),
           call(ws=None), call(kt=kv[0]), call(kt=kv[1]), call(vt=kv[0]), call(vt=to[0]),
           call(acc_to=256), call(len_to=256), call(kt=_with(B, to[0], tok=8)), call(d=_dims(B, B=0))]
    assert bad == [B.ERR_INVALID_ARG] * len(bad)


def test_binding_refuses_shapes_types_and_places(B):
    class Host(B.PrefixAttention):                    # the checks alone, without a workspace
        def __init__(self):
            self.dtype = torch.bfloat16

    h = Host()
    t = torch.zeros(2, 4, 3, 8, dtype=torch.bfloat16)
    for bad in (t.float(), t[:, :3], t.transpose(1, 2), None, t):     # the last: not on the GPU
        with pytest.raises(ValueError):
            h._view(bad, (2, 4, 3, 8), "k")
    assert h._view(None, (2, 0, 3, 8), "k") is None
    i = torch.zeros(2, 4, dtype=torch.int32)
    for bad in (i.long(), i[:, :2], i):
        with pytest.raises(ValueError):
            h._plain(bad, (2, 4), torch.int32, "visible")
    with pytest.raises(ValueError):
        B.PrefixAttention(1, 1, 1, 1, 8, 0, 0, torch.float16, device="cpu")
    with pytest.raises(B.BriskError):
        B.PrefixAttention(1, 1, 3, 2, 8, 0, 0, torch.bfloat16, device="cpu")
