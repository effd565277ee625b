"""A row's bits are its own: attention and the weights give a row the same bits again, whatever other rows
of the call hold, whatever hidden entries hold, and whatever ran on the GPU in between."""
import pytest
import torch

from test_cache_gpu import BF, F32
from test_cache_forms_gpu import apart
from test_cache_work_gpu import inputs, lens_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2609_33390_gb300 import build
    build.build()
    from paper_2609_33390_gb300 import brisk as B
    return B


def test_some_sizes_have_the_prefixs_own_kernel():
    assert apart((256, 1, 32, 8, 128, 2048, 250)) and apart((35, 4, 28, 4, 64, 6000, 250))
    assert apart((33, 4, 32, 4, 128, 3000, 250))


def attend(att, x):
    return att.attend(x["q"], x["kp"], x["vp"], x["ko"], x["vo"], x["lens"], visible=x["vis"])


@pytest.mark.parametrize("size", [
    # B, L, Hq, Hkv, D, P, S: tiles of 128 or 256 rows that are not full
    (256, 1, 32, 8, 128, 2048, 1500),     # 4 rows of a sequence, full tiles over the prefix
    (256, 1, 32, 8, 128, 2048, 250),      # the latter by the prefix's own kernel
    (205, 4, 1, 1, 128, 11000, 400),      # 52 rows in the prefix's last tile
    (3, 10, 32, 4, 128, 12800, 18),       # 112
    (5, 18, 16, 8, 128, 800, 4600),       # 36 rows of a sequence
    (35, 4, 28, 4, 64, 6000, 250),        # 212 of 256 rows in the last tile of the prefix's own kernel
])
def test_rows_repeat_their_bits_between_other_calls(B, size):
    Bn, L, Hq, Hkv, D, P, S = size
    x = inputs(*size, lens_of(Bn, S), False, BF)
    att = B.PrefixAttention(*size, BF)
    # another call, whose large queries and keys stay behind in shared memory
    y = inputs(40, 8, 32, 8, 128, 4000, 500, lens_of(40, 500), False, BF, seed=1)
    other = B.PrefixAttention(40, 8, 32, 8, 128, 4000, 500, BF)
    ref = attend(att, x)
    for factor in (1.0, 7.0, 0.1, 30.0):
        z = dict(y, q=y["q"] * factor)
        attend(other, z)
        got = attend(att, x)
        assert torch.equal(got["out"], ref["out"]) and torch.equal(got["lse"], ref["lse"])
    assert att.device_status() == B.OK


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("size", [
    (3, 8, 8, 2, 64, 900, 700),           # 32 rows of a sequence, beside the prefix
    (3, 8, 8, 2, 128, 0, 700),
    (33, 4, 32, 4, 128, 3000, 250),       # the prefix's own kernel
])
def test_rows_do_not_depend_on_other_rows(B, size, dt):
    """The last position's queries, and an entry that it alone sees, change; the other rows do not."""
    Bn, L, Hq, Hkv, D, P, S = size
    x = inputs(*size, [S] * Bn, False, dt)
    x["vis"] = torch.arange(S - L + 1, S + 1, dtype=torch.int32).cuda().expand(Bn, L).contiguous()
    att = B.PrefixAttention(*size, dt)
    ref = attend(att, x)
    ref = {k: v[:, :-1].clone() for k, v in ref.items()}
    for factor in (20.0, 0.0, -3.0):
        y = dict(x, q=x["q"].clone())
        y["q"][:, -1] *= factor
        for key in (1.0, 50.0, -50.0):
            y["ko"] = x["ko"].clone()
            y["ko"][:, S - 1] *= key
            got = attend(att, y)
            for k in ref:
                assert torch.equal(got[k][:, :-1], ref[k])


def test_rows_do_not_depend_on_what_padding_holds(B):
    size = (6, 8, 16, 4, 128, 1500, 400)
    x = inputs(*size, lens_of(6, 400), False, BF)
    x["vis"] = x["lens"][:, None].expand(6, 8).clone()
    x["vis"][:, 5:] = -1
    att = B.PrefixAttention(*size, BF)
    ref = attend(att, x)
    for fill in (0.0, 40.0, float("nan"), float("inf")):
        y = dict(x, q=x["q"].clone())
        y["q"][:, 5:] = fill
        got = attend(att, y)
        assert torch.equal(got["out"], ref["out"]) and torch.equal(got["lse"], ref["lse"])
