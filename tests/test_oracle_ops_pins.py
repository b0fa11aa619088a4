"""Fixed points of the 64-bit references in oracle/ops_oracle.py (CPU only): the recurrence against its closed form, the gradients against
central differences, the rotation against what it has to keep."""
import numpy as np
import pytest

from oracle import ops_oracle as oo


def _decay_case(seed, N=2, T=7, dk=3, dv=4):
    rng = np.random.default_rng(seed)
    q, k = rng.standard_normal((2, N, T, dk))
    v, do = rng.standard_normal((2, N, T, dv))
    return q, k, v, -rng.random((N, T)), rng.standard_normal((N, dk, dv)), do, rng.standard_normal((N, dk, dv))


def test_recurrence_equals_the_sum_over_pairs():
    q, k, v, g, s0, _, _ = _decay_case(1)
    o, S = oo.decay_fwd(q, k, v, g, s0)
    b = np.cumsum(g, 1)
    for t in range(q.shape[1]):
        want = np.exp(b[:, t])[:, None] * np.einsum("nc,ncd->nd", q[:, t], s0)
        for u in range(t + 1):
            want += (np.exp(b[:, t] - b[:, u]) * (q[:, t] * k[:, u]).sum(-1))[:, None] * v[:, u]
        np.testing.assert_allclose(o[:, t], want, rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(np.einsum("nc,ncd->nd", q[:, -1], S[:, -1]), o[:, -1], rtol=1e-12)


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


def test_recurrence_gradients_against_differences():
    q, k, v, g, s0, do, ds = _decay_case(2)

    def loss():
        o, S = oo.decay_fwd(q, k, v, g, s0)
        return (o * do).sum() + (S[:, -1] * ds).sum()
    _, S = oo.decay_fwd(q, k, v, g, s0)
    _differences(loss, (q, k, v, g, s0), oo.decay_bwd(q, k, v, g, S, do, ds))


@pytest.mark.parametrize("gated", [False, True])
def test_norm_gradients_against_differences(gated):
    rng = np.random.default_rng(3)
    x, do, r = rng.standard_normal((3, 4, 2, 5))
    w, b = rng.standard_normal((2, 2, 5))
    r = r if gated else None
    loss = lambda: (oo.norm_fwd(x, w, b, 1e-3, r)[0] * do).sum()  # noqa: E731
    dx, dr, dw, db = oo.norm_bwd(x, w, b, 1e-3, do, r)
    _differences(loss, (x, w, b) + ((r,) if gated else ()), (dx, dw, db) + ((dr,) if gated else ()))


@pytest.mark.parametrize("adjacent", [False, True])
def test_rotation_keeps_lengths_and_differences_of_positions(adjacent):
    rng = np.random.default_rng(4)
    q, k = rng.standard_normal((2, 1, 1, 1, 10))
    turn = lambda x, p: oo.rope(x, np.array(p).reshape(1, 1, 2), (4, 6), 100.0, adjacent, False)  # noqa: E731
    np.testing.assert_allclose((turn(q, (3, 9)) ** 2).sum(), (q ** 2).sum(), rtol=1e-12)
    np.testing.assert_allclose((turn(q, (3, 9)) * turn(k, (1, 4))).sum(), (turn(q, (13, 2)) * turn(k, (11, -3))).sum(), rtol=1e-12)
    back = oo.rope(turn(q, (3, 9)), np.array([[[3, 9]]]), (4, 6), 100.0, adjacent, True)
    np.testing.assert_allclose(back, q, rtol=1e-12, atol=1e-12)
    # the first pair of the first section turns by the position itself
    a, b = (0, 1) if adjacent else (0, 2)
    y = turn(q, (1, 0))
    np.testing.assert_allclose(y[..., a], q[..., a] * np.cos(1.0) - q[..., b] * np.sin(1.0), rtol=1e-12)


def test_scan_orders():
    assert list(oo.visits(6, 2, 3, 2)) == [0, 3, 1, 4, 2, 5]
    assert list(oo.visits(6, 2, 3, 3)) == [5, 2, 4, 1, 3, 0]
    assert list(oo.visits(5, 1, 5, 1, 3)) == [2, 1, 0]
