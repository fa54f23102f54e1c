"""Pins of the 64-bit statements of the output-end operators: gradients against central differences, sampling against enumeration."""
import numpy as np
import pytest

from oracle import lm_oracle as o


def _difference(f, x, step=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += step
        b[i] -= step
        g[i] = (f(a) - f(b)) / (2 * step)
    return g


@pytest.mark.parametrize("d", [1, 2, 9])
def test_norm_gradients_are_those_of_the_norm(d):
    rng = np.random.default_rng(d)
    h, w, dy, ds = rng.standard_normal((3, d)), rng.standard_normal(d), rng.standard_normal((3, d)), rng.standard_normal((3, d))
    value = lambda h_, w_: float(np.sum(dy * o.rms_norm(h_, w_, 1e-2)[0]) + np.sum(ds * h_))  # noqa: E731
    dh, dw = o.rms_norm_backward(dy, h, w, 1e-2, ds)
    # central differences in 64 bits: truncation ~ step^2, rounding ~ 1e-16 / step
    assert np.allclose(dh, _difference(lambda a: value(a, w), h), atol=1e-7)
    assert np.allclose(dw, _difference(lambda a: value(h, a), w), atol=1e-7)


@pytest.mark.parametrize("T", [0.5, 1.0, 3.0])
def test_distillation_gradient_is_that_of_its_loss(T):
    rng = np.random.default_rng(5)
    z, t = rng.standard_normal((4, 7)), rng.standard_normal((4, 3))
    idx = np.array([[0, 3, 6], [2, 2, 5], [1, -1, 4], [-1, 9, -1]])      # plain, an index twice, one entry absent, none
    v = np.array([1.0, 0.5, 2.0, 1.0])
    loss, grad = o.distill(z, idx, t, T, v)
    assert np.allclose(grad, _difference(lambda a: float(o.distill(a, idx, t, T, v)[0].sum()), z), atol=1e-7)
    assert loss[3] == 0 and not grad[3].any()
    # the teacher's own distribution over a full vocabulary has no loss
    same = o.distill(z, np.tile(np.arange(7), (4, 1)), z, T)
    assert np.allclose(same[0], 0, atol=1e-12) and np.allclose(same[1], 0, atol=1e-12)


def test_sampling_keeps_and_draws_what_the_filters_say():
    z = np.log(np.array([0.1, 0.4, 0.2, 0.2, 0.1]))
    draws = lambda **kw: [o.sample_row(z, u, **kw)[2] for u in (0.0, 0.05, 0.2, 0.49, 0.51, 0.75, 0.95)]  # noqa: E731
    assert draws() == [0, 0, 1, 1, 2, 3, 4]
    assert set(draws(top_k=2)) == {1, 2}                 # of two equal ones the lower index
    assert set(draws(top_p=0.59)) == {1, 2} and set(draws(top_p=0.61)) == {1, 2, 3}
    assert set(draws(min_p=0.4)) == {1, 2, 3} and set(draws(min_p=1.0)) == {1}
    assert set(draws(t=0.0)) == {1} and set(draws(top_p=0.0)) == {1}
    assert o.sample_row(np.full(3, -np.inf), 0.5)[2] == -1
    assert o.sample_row(np.array([np.nan, 0.0, -np.inf]), 0.9)[2] == 1
    # shares of many draws
    rng = np.random.default_rng(0)
    got = np.bincount([o.sample_row(z, u, t=2.0)[2] for u in rng.random(4000)], minlength=5) / 4000
    want = np.sqrt(np.exp(z)) / np.sqrt(np.exp(z)).sum()
    assert np.all(np.abs(got - want) < 4 * np.sqrt(want / 4000))
