"""The 64-bit forms of layer norm, token log-probabilities and distillation: their gradients against central differences, and the corners
that the library's header defines."""
import numpy as np
import pytest

from tests import head_ref as R


def _differences(f, x, seed, eps=1e-5):
    """Directional derivatives of f along three directions, and the directions."""
    rng = np.random.default_rng(seed)
    for _ in range(3):
        v = rng.standard_normal(x.shape)
        yield (f(x + eps * v) - f(x - eps * v)) / (2 * eps), v


def test_layernorm_gradients():
    rng = np.random.default_rng(1)
    x, dy = rng.standard_normal((5, 33)) * 2 + 1, rng.standard_normal((5, 33))
    gamma, beta = 1 + 0.2 * rng.standard_normal(33), rng.standard_normal(33)
    dx, dg, db = R.layernorm_grad(dy, x, gamma, 1e-5)
    for want, v in _differences(lambda a: (R.layernorm(a, gamma, beta, 1e-5)[0] * dy).sum(), x, 2):
        assert abs((dx * v).sum() - want) < 1e-7
    for want, v in _differences(lambda a: (R.layernorm(x, a, beta, 1e-5)[0] * dy).sum(), gamma, 3):
        assert abs((dg * v).sum() - want) < 1e-7
    for want, v in _differences(lambda a: (R.layernorm(x, gamma, a, 1e-5)[0] * dy).sum(), beta, 4):
        assert abs((db * v).sum() - want) < 1e-7


@pytest.mark.parametrize("scale", [1.0, 0.6])
def test_logprobs_gradients(scale):
    rng = np.random.default_rng(5)
    z, tokens = rng.standard_normal((6, 40)) * 2, np.array([0, 39, -1, 7, 7, -100])
    g, h = rng.standard_normal(6), rng.standard_normal(6)
    got = R.token_logprobs_grad(z, tokens, scale, g, h)

    def f(a):
        logp, entropy, _, _ = R.token_logprobs(a, tokens, scale, 1)
        return (g * logp + h * entropy).sum()
    for want, v in _differences(f, z, 6):
        assert abs((got * v).sum() - want) < 1e-7


@pytest.mark.parametrize("scale", [1.0, 0.5])
def test_distillation_gradient(scale):
    rng = np.random.default_rng(7)
    z, teacher = rng.standard_normal((5, 30)), rng.standard_normal((5, 6))
    index = rng.integers(0, 30, (5, 6))
    index[0] = 4                                           # one column many times
    index[1, 2:] = -1
    teacher[2, 1] = -np.inf
    w = rng.standard_normal(5)
    got = R.distill_grad(z, teacher, index, scale, w)
    for want, v in _differences(lambda a: (w * R.distill(a, teacher, index, scale)[0]).sum(), z, 8):
        assert abs((got * v).sum() - want) < 1e-7


def test_corners():
    z = np.full((3, 5), -np.inf)
    z[1, 2] = 1.0
    z[2] = -3e38
    logp, h, tl, ti = R.token_logprobs(z, [1, 2, 0], 1.0, 3)
    assert np.isneginf(logp[0]) and logp[1] == 0.0 and abs(logp[2] + np.log(5)) < 1e-12
    assert h[0] == 0 and h[1] == 0 and abs(h[2] - np.log(5)) < 1e-12
    assert ti.tolist() == [[0, 1, 2], [2, 0, 1], [0, 1, 2]] and np.isneginf(tl[0]).all()
    loss, q = R.distill(z, np.zeros((3, 2)), np.array([[0, 1], [-1, -1], [0, 9]]), 1.0)
    assert np.isposinf(loss[0]) and loss[1] == 0 and np.isnan(loss[2])
    d = R.distill_grad(z, np.zeros((3, 2)), np.array([[0, 1], [-1, -1], [0, 9]]), 1.0, np.ones(3))
    assert not d[0].any() and not d[1].any() and np.isnan(d[2]).all()
