"""Gated recurrence of channels: waits that may not look at all, so that every unit but the first forms the state that enters it from the inputs, held to the
formulas and tolerances of test_gpu_recur.py (a state then goes through one product a step: T 2^-24 of the same sums, within their T 2^-26 4)."""
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla
from tests import test_gpu_recur as tr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
GRID = (40, 60)
T = GRID[0] * GRID[1]                    # 19 units in two blocks


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gla.load_library()


@pytest.fixture
def no_looks():
    keep = gla.gla_get_option(gla.OPT_LOOK_BACK_POLLS)
    gla.gla_set_option(gla.OPT_LOOK_BACK_POLLS, 0)
    yield
    gla.gla_set_option(gla.OPT_LOOK_BACK_POLLS, keep)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("kind,tau", tr.KINDS)
@pytest.mark.parametrize("scan", [0, 1, 2, 3])
@pytest.mark.parametrize("B,D,dtype", [(3, 5, F32), (2, 12, BF16), (2, 77, BF16), (1, 128, F32)])
def test_from_the_inputs(B, D, dtype, scan, kind, tau, rest, no_looks):
    """Waves of several sequences and of one, one and two channels a lane."""
    tr.check(tr.make(B, T, D, dtype, kind, D + scan), *GRID, scan, kind, tau, rest, F32)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("scan", [0, 1])
@pytest.mark.parametrize("D,dtype", [(10, BF16), (65, F32), (384, BF16)])
def test_from_the_inputs_of_padded_batches(D, dtype, scan, rest, no_looks):
    lens = [T, 0, 2050, 129, 1]
    tr.check(tr.make(len(lens), T, D, dtype, gla.GATE_PRE, D, lens=lens), 1, T, scan, gla.GATE_PRE, 16.0, rest, F32)


@pytest.mark.parametrize("D", [64, 513])
def test_no_look_is_made(D, no_looks):
    """What other units have published by then makes no difference: the same bits each time, and not those of the look-back, which adds in another order."""
    x, z = (torch.randn(1, T, D, device=DEV) for _ in range(2))
    want, _ = gla.gla_recur_fwd(x, z, 1, T)
    for _ in range(5):
        assert torch.equal(gla.gla_recur_fwd(x, z, 1, T)[0], want)
    gla.gla_set_option(gla.OPT_LOOK_BACK_POLLS, 1 << 15)
    back, _ = gla.gla_recur_fwd(x, z, 1, T)
    units = (want != back).view(-1, T, D)[0].any(-1)
    assert not units[:128].any() and all(units[n:n + 128].any() for n in range(128, T - 128, 128))
