"""CPU: the fp64 versions of the operators on score maps against values worked out by hand,
identities and differences of their losses."""
import numpy as np
import pytest

from oracle import scores as S


def test_top_scores_by_hand():
    z = np.array([1.0, 3.0, -0.0, 3.0, 0.0, -np.inf]).reshape(1, 1, 1, 6)
    v, i, rest = S.top_scores(z, 6, 3, 2.0)
    assert v[0, 0, 0].tolist() == [3.0, 3.0, 1.0] and i[0, 0, 0].tolist() == [1, 3, 0]
    assert rest[0, 0, 0] == pytest.approx(np.log(2.0))             # two zeros, one masked
    v, i, rest = S.top_scores(z, 2, 2, 1.0)
    assert i[0, 0, 0].tolist() == [1, 0] and rest[0, 0, 0] == -np.inf
    v, i, _ = S.top_scores(z, 6, 5, 1.0)
    assert i[0, 0, 0].tolist() == [1, 3, 0, 2, 4]                  # -0 equals 0


def test_distill_by_hand():
    # teacher 3/4, 1/4 on classes 0 and 2 of 3; student 1/2, 1/4, 1/4
    z = np.log([2.0, 1.0, 1.0]).reshape(1, 1, 1, 3)
    top, index = np.log([3.0, 1.0]).reshape(1, 1, 1, 2), np.array([0, 2]).reshape(1, 1, 1, 2)
    loss, grad, _ = S.distill(z, 3, top, index, None, 1.0, None, 2.0)
    assert loss[0] == pytest.approx(2 * (0.75 * np.log(1.5) + 0.25 * np.log(1.0)))
    assert np.allclose(grad[0, 0, 0], [2 * -0.25, 2 * 0.25, 0.0])
    # with a rest of e^0 = 1: 3/5, 1/5, 1/5
    loss, grad, _ = S.distill(z, 3, top, index, np.zeros((1, 1, 1)), 1.0, None, 1.0)
    assert loss[0] == pytest.approx(0.6 * np.log(1.2) + 0.4 * np.log(0.8))
    assert np.allclose(grad[0, 0, 0], [-0.1, 0.05, 0.05])


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("t", [1.0, 2.5])
def test_distill_gradient_by_differences(rest, t):
    r = np.random.default_rng(3)
    z = r.normal(0, 2, (2, 1, 3, 7))
    top, index, left = S.top_scores(r.normal(0, 2, z.shape), 6, 3, t)
    index = index.copy()
    index[0, 0, 0, 1] = -1                                        # left out
    index[1, 0, 2, 2] = index[1, 0, 2, 0]                         # the same class twice
    w = r.random((2, 1, 3))
    f = lambda x: S.distill(x, 6, top, index, left if rest else None, t, w, 0.7)[0].sum()
    grad = S.distill(z, 6, top, index, left if rest else None, t, w, 0.7)[1]
    for at in np.ndindex(*z.shape):
        d = np.zeros_like(z)
        d[at] = 1e-5
        assert (f(z + d) - f(z - d)) / 2e-5 == pytest.approx(grad[at], abs=1e-8)


def test_divergence_of_a_record_from_itself_is_zero():
    z = np.random.default_rng(4).normal(0, 3, (1, 2, 2, 9))
    top, index, rest = S.top_scores(z, 9, 4, 2.0)
    loss, grad, _ = S.distill(z, 9, top, index, rest, 2.0, None, 1.0)
    assert abs(loss[0]) < 1e-14 and np.abs(grad).max() < 1e-14


@pytest.mark.parametrize("classes", [1, 5])
def test_clipped_gradient_by_differences(classes):
    r = np.random.default_rng(5)
    z = r.normal(0, 1.5, (2, 2, 4, 6))
    act = r.integers(0, max(2, classes), (2, 2, 4))
    l, ent = S.log_probs(z, classes, act)
    assert np.all(ent >= 0) and np.all(l <= 0)
    old, ref = l - r.choice([-0.5, -0.1, 0.05, 0.6], l.shape), l + r.normal(0, 0.3, l.shape)
    adv, w = r.normal(0, 1, l.shape), r.random(l.shape)
    args = (classes, act, adv, old, ref, w, 0.2, 0.3, 0.1, 1.3)
    loss, grad, kl, _ = S.clipped_loss(z, *args)
    assert np.all(kl > 0)
    for at in np.ndindex(*z.shape):
        d = np.zeros_like(z)
        d[at] = 1e-5
        up, down = S.clipped_loss(z + d, *args)[0].sum(), S.clipped_loss(z - d, *args)[0].sum()
        assert (up - down) / 2e-5 == pytest.approx(grad[at], abs=1e-8)


def test_first_update_is_the_reinforce_gradient():
    """At the first update the ratio is 1 and nothing is clipped: -A (a - p), as the policy's
    logit gradient."""
    r = np.random.default_rng(6)
    z, act, adv = r.normal(0, 2, (1, 3, 4, 8)), r.integers(0, 2, (1, 3, 4)), r.normal(0, 1, (1, 3, 4))
    l, _ = S.log_probs(z, 1, act)
    _, grad, _, _ = S.clipped_loss(z, 1, act, adv, l, None, None, 0.2, 0.2, 0.0, 1.0)
    p = 1.0 / (1.0 + np.exp(-z[..., 0]))
    assert np.allclose(grad[..., 0], -adv * (act - p)) and not grad[..., 1:].any()


def test_pixels_that_take_no_part():
    z = np.array([[[[-np.inf] * 4, [0.0, np.nan, 1.0, 2.0], [0.0, -np.inf, 1.0, 0.0]]]])
    act = np.array([[[0, 1, 1]]])
    w = np.array([[[1.0, 0.0, 1.0]]])
    loss, grad, kl, _ = S.clipped_loss(z, 4, act, np.ones((1, 1, 3)), np.zeros((1, 1, 3)), np.zeros((1, 1, 3)), w, 0.2,
                                       0.2, 0.1, 1.0)
    assert loss[0] == 0 and not grad.any() and kl[0] == 0
    l, ent = S.log_probs(z, 4, np.array([[[0, 9, 1]]]))
    assert l[0, 0, 0] == -np.inf and l[0, 0, 1] == 0.0 and l[0, 0, 2] == -np.inf and ent[0, 0, 0] == 0.0
    top = np.full((1, 1, 3, 2), -np.inf)
    index = np.zeros((1, 1, 3, 2), int) + np.arange(2)
    loss, grad, _ = S.distill(z, 4, top, index, None, 1.0, w, 1.0)
    assert loss[0] == 0 and not grad.any()
