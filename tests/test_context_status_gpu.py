"""Device-side problems of any call of a decoder's step are there after the step, and after further ones."""
import pytest
import torch

from test_context_gpu import decoder

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def brisk():
    from paper_2609_33390_gb300 import build
    build.build()
    from paper_2609_33390_gb300 import brisk as B
    return B


class Failing:
    """The decoder's PrefixAttention, one call of which goes wrong."""

    def __init__(self, brisk, att, name):
        self.brisk, self.att, self.name, self.left = brisk, att, name, 1

    def _fails(self, name):
        if name != self.name or not self.left:
            return False
        self.left -= 1
        return True

    def attend(self, q, kp, vp, ko, vo, lens, visible=None):
        if self._fails("attend"):
            lens = lens.clone()
            lens[0] = self.att.S + 1                   # clamped and reported
        if self._fails("attend, a wait"):
            zeros = {"out": torch.zeros_like(q), "lse": torch.zeros(q.shape[:3], device="cuda")}
            before = self.brisk.set_wait_limit(1)
            try:
                return self.att.attend(q, kp, vp, ko, vo, lens, visible=visible, out=zeros)
            finally:
                self.brisk.set_wait_limit(before)
        return self.att.attend(q, kp, vp, ko, vo, lens, visible=visible)

    def weights(self, q, lse, k, lens, **how):
        if self._fails("weights"):
            lens = lens.clone()
            lens[0] = -1
        return self.att.weights(q, lse, k, lens, **how)

    def evict(self, k, v, acc, lens, keep, recent, out):
        if self._fails("evict"):
            lens = lens.clone()
            lens[0] = -5
        return self.att.evict(k, v, acc, lens, keep, recent, out=out)


@pytest.mark.parametrize("name", ["attend", "attend, a wait", "weights", "evict"])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_a_problem_of_any_call_is_reported_once(brisk, name, dt):
    if name == "attend, a wait" and dt == torch.float32:
        return                                         # no waits there
    dec = decoder(brisk, dt, 3, 4, 50, 24, 12, 4, 2, 64)
    bad = Failing(brisk, dec.attention, name)
    dec.attention = bad
    for _ in range(8):
        dec.step()
    assert bad.left == 0
    assert dec.device_status() == (brisk.ERR_TIMEOUT if name == "attend, a wait" else brisk.ERR_INVALID_ARG)
    for _ in range(8):
        dec.step()
    assert dec.device_status() == brisk.OK


def test_a_problem_of_the_tail_is_reported_after_further_steps(brisk):
    dec = decoder(brisk, torch.bfloat16, 3, 4, 50, 24, 12, 4, 2, 64)
    dec.x0 = torch.tensor([0, dec.e_in.shape[0], 1], dtype=torch.int32, device="cuda")
    for _ in range(3):
        dec.step()
    assert dec.device_status() == brisk.ERR_INVALID_ARG
    dec.step()
    assert dec.device_status() == brisk.OK
