"""Gated recurrence of channels at the ends of its temperatures, by the formulas and tolerances of test_gpu_recur.py and one term more: e^-z is lost in fp32
below 2^-126, so logarithms of gates, what these lack of one and their slopes are off by n = 2^-126 / tau more.  For 300 steps of |x|, |dO| < 5 and states
entering below 10, states and adjoints stay below 1510; a change of all logarithms by n moves them by n 300 1510 at most, dx by n 301 1510, and
dgate, a slope times a gate and its logarithm (1 at most together) times both, by n 1510^2 (1 + 2 300) < 2^31 n."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla
from tests import test_gpu_recur as tr

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gla.load_library()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("tau", [2.0 ** -64, 2.0 ** -40, 2.0 ** 60, 3e38])
@pytest.mark.parametrize("mean,spread", [(0.0, 3.0), (60.0, 30.0)])
def test_temperatures(tau, mean, spread, rest, monkeypatch):
    """Gates of zero and one and few between, and of one alone."""
    lost = 2.0 ** (31 - 126) / tau

    def close(got, want, size, tol, rounding, name):
        bad = np.abs(got - want) - (tol * size + rounding * np.abs(want) + lost + 1e-30)
        assert np.isfinite(got).all() and bad.max() <= 0, (name, float(bad.max()))

    monkeypatch.setattr(tr, "close", close)
    tr.check(tr.make(2, 300, 6, torch.float32, gla.GATE_PRE, 3, mean=mean, spread=spread), 1, 300, 0, gla.GATE_PRE, tau, rest, torch.float32)
