"""Pins of the fp64 oracle of the losses over a vocabulary: closed forms, differences and invariants."""
import numpy as np
import pytest

from oracle import losses as L


def _problem(rng, n=5, v=11, h=4, k=3):
    x, w = rng.standard_normal((n, h)), rng.standard_normal((v, h))
    return x, w, rng.integers(0, v, n), rng.integers(0, v, (n, k)), rng.standard_normal((n, k))


def test_uniform_logits_give_log_v():
    r = L.linear_xent(np.zeros((3, 2)), np.ones((7, 2)), np.array([0, 6, -100]))
    np.testing.assert_allclose(r.token_loss, [np.log(7), np.log(7), 0.0], rtol=1e-14)
    assert abs(r.loss - np.log(7)) < 1e-14
    np.testing.assert_allclose(r.dz[0], (np.full(7, 1 / 7) - np.eye(7)[0]) / 2, rtol=1e-13, atol=0)
    assert not r.dz[2].any()


def test_two_classes_give_the_logistic_function():
    x, w = np.array([[1.7]]), np.array([[1.0], [0.0]])
    r = L.linear_xent(x, w, np.array([0]), reduction="sum")
    assert abs(r.loss - np.log1p(np.exp(-1.7))) < 1e-15
    assert abs(r.dx[0, 0] + 1 / (1 + np.exp(1.7))) < 1e-15


@pytest.mark.parametrize("kind", ["xent", "distill"])
@pytest.mark.parametrize("reduction", ["sum", "mean"])
def test_gradients_against_differences(kind, reduction):
    rng = np.random.default_rng(3)
    x, w, t, ids, lg = _problem(rng)
    t[1] = -100
    ids[2] = -1
    ids[3, 0] = ids[3, 1]
    a = rng.uniform(0.5, 2.0, 5)

    def f(x, w):
        if kind == "xent":
            return L.linear_xent(x, w, t, reduction=reduction, scale=1.3, weight=a, z_loss=0.05)
        return L.linear_distill(x, w, ids, lg, temperature=2.5, reduction=reduction, scale=1.3, weight=a)

    r = f(x, w)
    for arr, grad, which in ((x, r.dx, 0), (w, r.dw, 1)):
        for i in np.ndindex(*arr.shape):
            d = np.zeros_like(arr)
            d[i] = 1e-5
            up, dn = (f(x + s * d, w) if which == 0 else f(x, w + s * d) for s in (1, -1))
            assert abs((up.loss - dn.loss) / 2e-5 - grad[i]) < 1e-9


def test_one_teacher_logit_is_a_hard_label():
    x, w, t, _, _ = _problem(np.random.default_rng(4))
    a, b = L.linear_xent(x, w, t), L.linear_distill(x, w, t[:, None], np.full((5, 1), 3.0))
    for p, q in zip(a, b):
        np.testing.assert_allclose(p, q, rtol=1e-12, atol=1e-14)


def test_distillation_from_the_students_own_softmax_is_zero():
    rng = np.random.default_rng(5)
    x, w = rng.standard_normal((4, 3)), rng.standard_normal((9, 3))
    ids = np.tile(rng.permutation(9), (4, 1))
    r = L.linear_distill(x, w, ids, np.take_along_axis(x @ w.T, ids, 1), temperature=1.7)
    assert abs(r.token_loss).max() < 1e-14 and abs(r.dz).max() < 1e-15


def test_a_duplicated_id_takes_the_sum_of_its_slots():
    rng = np.random.default_rng(6)
    x, w, _, _, _ = _problem(rng)
    ids = np.array([[2, 2, 7]] * 5)
    a = L.linear_distill(x, w, ids, np.zeros((5, 3)))
    b = L.linear_distill(x, w, np.array([[2, 7]] * 5), np.log(np.array([[2.0, 1.0]] * 5)))
    np.testing.assert_allclose(a.dz, b.dz, rtol=1e-12, atol=1e-15)
    # (the losses differ by q log q of the split slot)
    np.testing.assert_allclose(a.token_loss - b.token_loss, np.full(5, -2 / 3 * np.log(2)), rtol=1e-12)


def test_tokens_that_do_not_count_may_hold_anything():
    x, w, t, ids, lg = _problem(np.random.default_rng(7))
    x[1] = np.nan
    t[1] = -100
    ids[1] = -1
    for r in (L.linear_xent(x, w, t), L.linear_distill(x, w, ids, lg)):
        assert np.isfinite(r.dw).all() and r.token_loss[1] == 0 and not r.dx[1].any()
    r = L.linear_xent(x, w, np.full(5, -100))
    assert r.loss == 0 and not r.dw.any()
