"""Fixed points of the 64-bit references in oracle/block_oracle.py (CPU only): the recurrence against its closed form, all gradients against central
differences, the norm and the activations against what they have to keep."""
import math

import numpy as np
import pytest

from oracle import block_oracle as bo


def _differences(loss, arrays, grads, h=1e-6, tol=1e-7):
    for a, g in zip(arrays, grads):
        flat = a.reshape(-1)
        for i in np.random.default_rng(5).permutation(flat.size)[:12]:
            keep = flat[i]
            flat[i] = keep + h
            up = loss()
            flat[i] = keep - h
            down = loss()
            flat[i] = keep
            assert abs((up - down) / (2 * h) - g.reshape(-1)[i]) <= tol * (1 + abs(g.reshape(-1)[i]))


@pytest.mark.parametrize("rest", [False, True])
def test_recurrence_equals_the_sum_over_steps(rest):
    rng = np.random.default_rng(1)
    x, z, h0 = rng.standard_normal((2, 9, 3)), rng.standard_normal((2, 9, 3)), rng.standard_normal((2, 3))
    lg, _ = bo.log_gate(z, 4.0)
    h = bo.recur_fwd(x, lg, rest, h0)
    b = np.cumsum(lg, 1)
    u = x * (1 - np.exp(lg)) if rest else x
    for t in range(9):
        want = np.exp(b[:, t]) * h0 + sum(np.exp(b[:, t] - b[:, s]) * u[:, s] for s in range(t + 1))
        np.testing.assert_allclose(h[:, t + 1], want, rtol=1e-12, atol=1e-12)


def test_gates_from_pre_activations():
    z = np.array([-800.0, -3.0, 0.0, 2.0, 800.0])
    lg, slope = bo.log_gate(z, 2.0)
    np.testing.assert_allclose(lg, [-400.0, -0.5 * math.log1p(math.exp(3.0)), -0.5 * math.log(2.0), -0.5 * math.log1p(math.exp(-2.0)), 0.0], rtol=1e-12, atol=1e-300)
    np.testing.assert_allclose(slope[1:4], [0.5 / (1 + math.exp(s)) for s in (-3.0, 0.0, 2.0)], rtol=1e-12)
    same, one = bo.log_gate(z)
    assert (same == z).all() and (one == 1).all()


@pytest.mark.parametrize("rest", [False, True])
def test_recurrence_gradients_against_differences(rest):
    rng = np.random.default_rng(2)
    x, z, do = rng.standard_normal((3, 2, 6, 3))
    h0, dh = rng.standard_normal((2, 2, 3))

    def loss():
        h = bo.recur_fwd(x, bo.log_gate(z, 3.0)[0], rest, h0)
        return (h[:, 1:] * do).sum() + (h[:, -1] * dh).sum()
    lg, slope = bo.log_gate(z, 3.0)
    dx, dlg, d0 = bo.recur_bwd(x, lg, rest, bo.recur_fwd(x, lg, rest, h0), do, dh)
    _differences(loss, (x, z, h0), (dx, dlg * slope, d0))


def test_norm_gradients_against_differences():
    rng = np.random.default_rng(3)
    x, dy = rng.standard_normal((2, 4, 3, 5))
    w = rng.standard_normal(5)
    y, r = bo.rms_fwd(x, w, 1e-3)
    np.testing.assert_allclose(((y / w) ** 2).mean(-1), 1 - 1e-3 * r[..., 0] ** 2, rtol=1e-12)
    _differences(lambda: (bo.rms_fwd(x, w, 1e-3)[0] * dy).sum(), (x, w), bo.rms_bwd(x, w, 1e-3, dy))


@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
def test_product_gradients_against_differences(kind):
    rng = np.random.default_rng(4)
    x, wg, wu, do = rng.standard_normal((3, 4)), rng.standard_normal((5, 4)), rng.standard_normal((5, 4)), rng.standard_normal((3, 5))
    _differences(lambda: (bo.glu_fwd(x, wg, wu, kind) * do).sum(), (x, wg, wu), bo.glu_bwd(x, wg, wu, kind, do))


def test_activations():
    g = np.array([-30.0, -1.0, 0.0, 1.0, 30.0])
    for kind in ("silu", "gelu", "gelu_tanh"):
        a, s = bo.activation(kind, g)
        np.testing.assert_allclose(a[[2, 4]], [0.0, 30.0], atol=1e-10)
        np.testing.assert_allclose(a[3] - a[1], 1.0, rtol=1e-12)         # a(g) - a(-g) = g
        np.testing.assert_allclose(s[2], 0.5, rtol=1e-12)
    np.testing.assert_allclose(bo.activation("gelu", g)[0][3], 0.8413447460685429, rtol=1e-12)
