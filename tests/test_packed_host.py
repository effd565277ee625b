"""Refusals of the calls on caches in 4 bits: found on the host, before any CUDA call."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2609_33390_gb300 import build
    build.build()
    from paper_2609_33390_gb300 import brisk
    return brisk


class Packed(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p)] + \
        [(n, ctypes.c_int64) for n in ("seq", "tok", "head", "scale_seq", "scale_tok", "scale_head")]


FAKE = 1 << 20                                       # never dereferenced: the checks fail first


def _dims(lib_mod, **kw):
    d = dict(B=2, L=3, Hq=8, Hkv=2, D=64, P=100, S=50, dtype=lib_mod.DT_BF16)
    d.update(kw)
    return lib_mod.CacheDims(*[d[n] for n, _ in lib_mod.CacheDims._fields_])


def _packed(d, ptr=FAKE, **kw):
    row, w = d.D // 2, 4 if d.D <= 64 else 8
    f = dict(codes=ptr, scales=ptr + 4096, seq=d.S * d.Hkv * row, tok=d.Hkv * row, head=row,
             scale_seq=d.S * d.Hkv * w, scale_tok=d.Hkv * w, scale_head=w)
    f.update(kw)
    return Packed(**f)


def _rows(B, d, T, ptr=FAKE * 8):
    return B.View(ptr, T * d.Hkv * d.D, d.Hkv * d.D, d.D)


def _ref(x):
    return None if x is None else ctypes.byref(x)


def test_workspace_of_valid_and_invalid_sizes(B):
    size = lambda **kw: B.lib().brisk_packed_workspace_bytes(ctypes.byref(_dims(B, **kw)))
    for ok in (dict(), dict(P=0), dict(S=0), dict(D=16), dict(D=128), dict(D=80), dict(B=4096), dict(dtype=B.DT_F32)):
        assert size(**ok) > 0 and size(**ok) % 256 == 0, ok
    for bad in (dict(B=0), dict(L=0), dict(Hq=7), dict(D=8), dict(D=24), dict(D=136), dict(D=144), dict(P=-1),
                dict(S=-1), dict(dtype=2), dict(B=4096, L=1 << 20)):
        assert size(**bad) == 0, bad
    assert B.lib().brisk_packed_workspace_bytes(None) == 0


def test_store_and_load_refuse(B):
    d = _dims(B)
    p, p2 = _packed(d), _packed(d, 2 * FAKE)
    x, y = _rows(B, d, 4), _rows(B, d, 4, FAKE * 16)

    def store(d=d, T=4, k=x, v=y, start=256, kt=p, vt=p2, ws=256):
        return B.lib().brisk_packed_store(ctypes.byref(d), T, _ref(k), _ref(v), start, None, _ref(kt), _ref(vt), ws, None)

    def load(d=d, T=4, k=x, v=y, start=256, kt=p, vt=p2, ws=256):
        return B.lib().brisk_packed_load(ctypes.byref(d), T, _ref(kt), _ref(vt), start, None, _ref(k), _ref(v), ws, None)

    for call in (store, load):
        bad = [call(d=_dims(B, D=24)), call(d=_dims(B, B=0)), call(T=0), call(T=-1), call(T=(1 << 30) + 1), call(k=None),
               call(v=None), call(start=None), call(kt=None), call(vt=None), call(ws=None), call(ws=128),
               call(k=B.View(x.ptr + 8, x.seq, x.tok, x.head)), call(k=B.View(x.ptr, x.seq, x.tok, 60)),
               call(kt=_packed(d, codes=None)), call(vt=_packed(d, scales=None)), call(kt=_packed(d, FAKE + 8)),
               call(kt=_packed(d, scales=FAKE + 2)), call(kt=_packed(d, tok=d.Hkv * 32 + 8)),
               call(kt=_packed(d, scale_tok=0)), call(vt=_packed(d, head=16)), call(vt=_packed(d, scale_head=6)),
               call(kt=_packed(d, seq=1 << 39)), call(kt=_packed(d, tok=-64)), call(kt=_packed(d, tok=1 << 32)),
               call(vt=_packed(d, scale_tok=1 << 32))]
        assert bad == [B.ERR_INVALID_ARG] * len(bad), call.__name__
        e = _dims(B, B=1, L=1, Hkv=1 << 20, Hq=1 << 20, D=128)
        assert call(d=e, T=1, k=_rows(B, e, 1), v=_rows(B, e, 1, FAKE * 16), kt=_packed(e),
                    vt=_packed(e, 2 * FAKE)) == B.ERR_UNSUPPORTED
    # keys and values into one place
    assert store(vt=p) == B.ERR_INVALID_ARG
    assert store(vt=_packed(d, 2 * FAKE, scales=p.scales)) == B.ERR_INVALID_ARG
    assert load(v=x) == B.ERR_INVALID_ARG
    # rows of 40 bytes start on 8, their 8 bytes of scales too
    e = _dims(B, D=80)
    assert store(d=e, k=_rows(B, e, 4), v=_rows(B, e, 4, FAKE * 16), kt=_packed(e, FAKE + 4), vt=_packed(e, 2 * FAKE)) == \
        B.ERR_INVALID_ARG


def test_attend_refuses(B):
    d = _dims(B)
    q = B.View(FAKE, d.L * d.Hq * d.D, d.Hq * d.D, d.D)
    pre = B.View(FAKE, 0, d.Hkv * d.D, d.D)
    k, v = _packed(d), _packed(d, 2 * FAKE)

    def call(d=d, q=q, kp=pre, vp=pre, k=k, v=v, lens=256, scale=0.1, out=256, ws=256):
        return B.lib().brisk_packed_attend(ctypes.byref(d), _ref(q), _ref(kp), _ref(vp), _ref(k), _ref(v), lens, None,
                                           scale, out, None, ws, None)
    bad = [call(d=_dims(B, D=72)), call(q=None), call(kp=None), call(vp=None), call(k=None), call(v=None), call(lens=None),
           call(out=None), call(out=264), call(ws=None), call(ws=128), call(scale=-1.0), call(scale=float("nan")),
           call(scale=3e38), call(q=B.View(FAKE + 8, q.seq, q.tok, q.head)), call(k=_packed(d, FAKE + 8)),
           call(v=_packed(d, scale_seq=2))]
    assert bad == [B.ERR_INVALID_ARG] * len(bad)


def test_binding_refuses_shapes_types_and_places(B):
    class Host(B.PackedAttention):                   # the checks alone, without a workspace
        def __init__(self, S=3):
            self.dtype, self.S = torch.bfloat16, S
            self._shape_codes, self._shape_scales = (2, 3, 4, 32), (2, 3, 4, 4)

    h = Host()
    codes, scales = torch.zeros(2, 3, 4, 32, dtype=torch.uint8), torch.zeros(2, 3, 4, 4, dtype=torch.uint8)
    good = {"k": codes, "v": codes, "k_scales": scales, "v_scales": scales}
    for name, bad in (("k", codes.float()), ("v", codes[:, :2]), ("k", codes.transpose(1, 2)), ("k_scales", codes),
                      ("k", codes)):                 # the last: not on the GPU
        with pytest.raises(ValueError):
            h._cache(dict(good, **{name: bad}))
    with pytest.raises(ValueError):
        h._cache(None)
    assert Host(0)._cache(None) == (0,) * 16
    for D in (8, 24, 136):
        with pytest.raises(B.BriskError):
            B.PackedAttention(1, 1, 1, 1, D, 0, 4, torch.bfloat16, device="cpu")
    with pytest.raises(ValueError):
        B.PackedAttention(1, 1, 1, 1, 16, 0, 4, torch.float16, device="cpu")
    att = B.PackedAttention(1, 1, 1, 1, 16, 0, 4, torch.bfloat16, device="cpu")
    with pytest.raises(ValueError):
        att.alloc_cache("time")
    for call in (att.weights, att.evict):
        with pytest.raises(TypeError):
            call()
    assert att.alloc_cache("head")["k"].shape == (1, 4, 1, 8)


def test_calls_without_a_gpu_are_refused(B):
    att = B.PackedAttention(1, 1, 1, 1, 16, 0, 4, torch.bfloat16, device="cpu")
    c, x, n = att.alloc_cache(), torch.zeros(1, 1, 1, 16, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    for call in (lambda: att.store(c, x, x, n), lambda: att.load(c, 1, n), lambda: att.attend(x, None, None, c, n)):
        with pytest.raises(ValueError, match="not on the GPU"):
            call()
