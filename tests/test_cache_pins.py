"""Pins of the float64 statement of prefix attention, attention weights and eviction (oracle/cache.py)
against closed forms and matrix forms that share no code with it."""
import numpy as np
import pytest

from oracle import cache as C


def _softmax(x):
    e = np.exp(x - x.max(-1, keepdims=True))
    return e / e.sum(-1, keepdims=True)


@pytest.mark.parametrize("P,S", [(0, 7), (5, 0), (4, 6)])
def test_attend_equals_the_matrix_form(P, S):
    g = np.random.default_rng(P * 10 + S)
    B, L, Hkv, G, D = 2, 3, 2, 3, 8
    q = g.standard_normal((B, L, Hkv * G, D))
    kp, vp = g.standard_normal((2, P, Hkv, D))
    ko, vo = g.standard_normal((2, B, S, Hkv, D))
    lens = np.array([S, max(S - 2, 0)])
    out, lse, mass, _ = C.attend(q, kp if P else None, vp if P else None, ko if S else None,
                                 vo if S else None, lens, None, 0.5)
    for b in range(B):
        k = np.concatenate([kp, ko[b, :lens[b]]]).repeat(G, 1)
        v = np.concatenate([vp, vo[b, :lens[b]]]).repeat(G, 1)
        s = 0.5 * np.einsum("ihd,thd->hit", q[b], k)
        np.testing.assert_allclose(out[b], np.einsum("hit,thd->ihd", _softmax(s), v), rtol=1e-12, atol=1e-14)
        np.testing.assert_allclose(lse[b], np.log(np.exp(s).sum(-1)).T, rtol=1e-12)
        assert (mass[b] >= np.abs(out[b]) - 1e-12).all()


def test_equal_keys_average_what_a_position_sees():
    B, L, S, D = 1, 4, 5, 8
    q, ko = np.ones((B, L, 1, D)), np.ones((B, S, 1, D))
    vo = np.arange(S, dtype=float)[None, :, None, None] * np.ones(D)
    vis = np.array([[0, 1, 3, -1]])
    out, lse, _, _ = C.attend(q, None, None, ko, vo, np.array([4]), vis, 1.0)
    assert (out[0, 0] == 0).all() and lse[0, 0, 0] == -np.inf
    assert np.allclose(out[0, 1], 0) and np.isclose(lse[0, 1, 0], D)
    assert np.allclose(out[0, 2], 1) and np.isclose(lse[0, 2, 0], D + np.log(3))
    assert (out[0, 3] == 0).all() and lse[0, 3, 0] == -np.inf
    # more visible entries than are in use: those in use; a prefix is hidden from padding alone
    out, lse, _, _ = C.attend(q, ko[0, :2], vo[0, :2], ko, vo, np.array([2]), vis + 5, 1.0)
    assert np.isclose(lse[0, :, 0], D + np.log(4)).all()
    out, lse, _, _ = C.attend(q, ko[0, :2], vo[0, :2], ko, vo, np.array([2]), vis, 1.0)
    assert np.isclose(lse[0, 0, 0], D + np.log(2)) and lse[0, 3, 0] == -np.inf


def test_weights_of_all_entries_sum_to_the_rows():
    g = np.random.default_rng(3)
    B, L, Hkv, G, D, S = 2, 3, 2, 2, 8, 6
    q, ko = g.standard_normal((B, L, Hkv * G, D)), g.standard_normal((B, S, Hkv, D))
    lens = np.array([6, 4])
    _, lse, _, _ = C.attend(q, None, None, ko, ko, lens, None, 0.3)
    acc, _ = C.weights(q, lse, ko, lens, None, 0.3, None, 1.0)
    np.testing.assert_allclose(acc.sum(-1), L * G, rtol=1e-12)
    assert (acc[1, :, 4:] == 0).all()
    again, _ = C.weights(q, lse, ko, lens, None, 0.3, acc + 7.0, 0.5)
    np.testing.assert_allclose(again[0], 1.5 * acc[0] + 3.5, rtol=1e-12)
    assert (again[1, :, 4:] == 0).all()


def test_eviction_by_hand():
    D = 8
    ko = np.arange(8, dtype=float)[None, :, None, None] * np.ones((1, 8, 1, D))
    acc = np.array([[[1.0, 5.0, 1.0, np.nan, -np.inf, 2.0, 0.0, 9.0]]])
    k, v, a, n, kept = C.evict(ko, -ko, acc, np.array([8]), 4, 1)
    assert kept[0, 0].tolist() == [0, 1, 5, 7] and n.tolist() == [4]
    assert k[0, :, 0, 0].tolist() == [0, 1, 5, 7] and v[0, :, 0, 0].tolist() == [0, -1, -5, -7]
    assert a[0, 0].tolist() == [1, 5, 2, 9]
    assert C.evict(ko, ko, acc, np.array([8]), 3, 3)[4][0, 0].tolist() == [5, 6, 7]
    assert C.evict(ko, ko, acc, np.array([7]), 6, 0)[4][0, 0].tolist() == [0, 1, 2, 4, 5, 6]
    k, _, a, n, kept = C.evict(ko, ko, acc, np.array([2]), 4, 1)
    assert kept[0, 0].tolist() == [0, 1, -1, -1] and n.tolist() == [2]
    assert (k[0, 2:] == 0).all() and (a[0, 0, 2:] == 0).all()
