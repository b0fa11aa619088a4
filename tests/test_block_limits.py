"""Sizes up to which the operators around the mixer in a block take calls, as include/gla.h states them, and those behind: on the host, before anything is
enqueued (no GPU).  A call that the limits let pass is stopped by what is checked behind them: a tensor that is not aligned."""
import ctypes

import pytest

import paper_2405_18428_amd as gla
from tests import test_block_refusals as tb

UNSUPPORTED, ALIGN = tb.UNSUPPORTED, tb.ALIGN


@pytest.fixture(scope="module")
def lib():
    return gla.load_library()


def sized(call, B, T, D):
    return {**call, "B": B, "T": T, "D": D, "gh": 1, "gw": T, "x": tb.OFF}


# Work-groups, below 2^23 of them: groups of 64 channels for odd D, of 128 for even D, or the columns (channels, or pairs of them) of all sequences, 64 each,
# where few channels let sequences share a group; forward a group for each 128 steps, or one for all steps from 256 x 128 channels on
FORWARD = [
    # (B, T, D): 2^23 - 1 units; 2^23; 2 (2^22 - 1); 2 2^22; 3 2^22; 8 (2^20 - 1); 8 2^20
    ((1, (1 << 30) - 128, 64), ALIGN), ((1, 1 << 30, 64), UNSUPPORTED), ((1, (1 << 29) - 128, 130), ALIGN), ((1, 1 << 29, 130), UNSUPPORTED),
    ((1, (1 << 29) - 128, 129), UNSUPPORTED), ((1, (1 << 27) - 128, 1024), ALIGN), ((1, 1 << 27, 1024), UNSUPPORTED),
    # walked: 64 x 16; 2^16 (64 sequences a group); 2^22; 2^23 - 1; 2^23; 7 2^20; 8 2^20; 127 2^16; 129 2^16
    ((64, 131072, 2048), ALIGN), ((1 << 22, 3, 1), ALIGN), ((1 << 22, 3, 128), ALIGN), (((1 << 23) - 1, 3, 128), ALIGN), ((1 << 23, 3, 128), UNSUPPORTED),
    ((1 << 20, 1 << 20, 896), ALIGN), ((1 << 20, 1 << 20, 1024), UNSUPPORTED), ((1 << 22, 300, 127), ALIGN), ((1 << 22, 300, 129), UNSUPPORTED),
    ((1 << 30, 1 << 30, 1 << 26), UNSUPPORTED),
]
# A group for each 64 steps; where there are several of these, below 2^22 times 64 channels of one sequence as well
BACKWARD = [
    # 2^23 - 1; 2^23; 64 x 64 x 2047; 64 x 64 x 2048; 64 x 128 x 2047; 64 x 16 x 2048
    ((1, (1 << 29) - 64, 64), ALIGN), ((1, 1 << 29, 64), UNSUPPORTED), ((64, (1 << 17) - 64, 8192), ALIGN), ((64, 1 << 17, 8192), UNSUPPORTED),
    ((64, (1 << 17) - 64, 8191), UNSUPPORTED), ((64, 131072, 2048), ALIGN),
    # one round: 2^16, 2^22, 2^23; several: 2^17 and 2^22 sequences, 2^22 - 1, 3 2^20 and 3 2^21 times 64 channels
    ((1 << 22, 64, 1), ALIGN), ((1 << 22, 3, 128), ALIGN), ((1 << 23, 3, 128), UNSUPPORTED), ((1 << 22, 65, 1), UNSUPPORTED), (((1 << 22) - 1, 65, 1), ALIGN),
    ((1 << 20, 65, 130), ALIGN), ((1 << 21, 65, 130), UNSUPPORTED), ((1 << 30, 1 << 30, 1 << 26), UNSUPPORTED),
]


@pytest.mark.parametrize("sizes,status", FORWARD)
def test_recurrence_forward(lib, sizes, status):
    assert lib.gla_recur_fwd(*sized(tb.RECUR, *sizes).values()) == status
    assert status == ALIGN or gla.gla_recur_fwd_workspace_bytes(*sizes) == 0


@pytest.mark.parametrize("sizes,status", BACKWARD)
def test_recurrence_backward(lib, sizes, status):
    assert lib.gla_recur_bwd(*sized(tb.RECUR_BWD, *sizes).values()) == status
    assert status == ALIGN or gla.gla_recur_bwd_workspace_bytes(*sizes) == 0


def test_recurrence_workspaces_of_the_largest_calls():
    """A word of 64 bits a unit and channel, one of 32 a block of 16 units; three numbers a round and channel."""
    T = (1 << 30) - 128
    units = T // 128
    assert gla.gla_recur_fwd_workspace_bytes(1, T, 64) >= 64 * (units * 8 + units // 16 * 4)
    T = (1 << 29) - 64
    assert gla.gla_recur_bwd_workspace_bytes(1, T, 64) >= 3 * 4 * 64 * (T // 64)


PRODUCT = [((1 << 28, 8, 8), ALIGN), (((1 << 28) + 1, 1, 1), UNSUPPORTED), ((1 << 28, 55, 8), ALIGN), ((1 << 28, 56, 8), UNSUPPORTED), ((1 << 28, 8, 55), ALIGN), ((1 << 28, 8, 56), UNSUPPORTED),
           ((1, 1 << 20, 4095), ALIGN), ((1, 1 << 20, 4096), UNSUPPORTED), ((1, 4088, (1 << 20) - 1), ALIGN), ((1, 4088, 1 << 20), UNSUPPORTED), ((1, (1 << 20) + 1, 8), UNSUPPORTED),
           ((1, 8, (1 << 20) + 1), UNSUPPORTED), ((16383, 4, 1 << 20), ALIGN), ((16384, 4, 1 << 20), UNSUPPORTED)]


@pytest.mark.parametrize("sizes,status", PRODUCT)
def test_product(lib, sizes, status):
    m = dict(zip("MKF", sizes), x=tb.OFF)
    assert lib.gla_glu_fwd(*{**tb.GLU, **m}.values()) == status and lib.gla_glu_bwd(*{**tb.GLU_BWD, **m}.values()) == status
    assert (gla.gla_glu_bwd_workspace_bytes(*sizes) > 0) == (status == ALIGN)


# (a subnormal temperature's reciprocal is infinite, and a gate of one NaN; below 2^-64 what fp32 loses of e^-z, 2^-126, begins to show in a gate)
TAUS = [(2.0 ** -64, ALIGN), (3.0e38, ALIGN), (2.0 ** -65, tb.SHAPE), (2.0 ** -127, tb.SHAPE), (1e-45, tb.SHAPE), (-1.0, tb.SHAPE)]


@pytest.mark.parametrize("tau,status", TAUS)
def test_temperatures(lib, tau, status):
    tau = ctypes.c_float(tau)
    for call, args in ((lib.gla_recur_fwd, tb.RECUR), (lib.gla_recur_bwd, tb.RECUR_BWD)):
        assert call(*{**args, "x": tb.OFF, "tau": tau}.values()) == status
        assert call(*{**args, "x": tb.OFF, "tau": tau, "kind": 0}.values()) == ALIGN
    for kind, want in ((1, status), (0, ALIGN)):
        assert lib.gla_recur_step(*{**tb.STEP, "s": tb.OFF, "tau": tau, "kind": kind}.values()) == want


HUGE = (1 << 32) + 5                     # as a C int: 5


@pytest.mark.parametrize("call", ["fwd", "bwd", "step", "qk_fwd", "qk_bwd", "qk_keys", "glu_fwd", "glu_bwd", "glu_columns"])
def test_sizes_that_are_no_c_int_are_refused(call, monkeypatch):
    """They would be cut off to 32 bits on their way into the library, which would then work on a part of the tensors.  (Tensors without memory.)"""
    torch = pytest.importorskip("torch")
    from paper_2405_18428_amd import binding

    class Library:
        def __getattr__(self, name):
            raise AssertionError("the library was reached")
    new = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device="meta")  # noqa: E731
    monkeypatch.setattr(binding, "load_library", Library)
    monkeypatch.setattr(binding, "_want", lambda *args: None)
    monkeypatch.setattr(binding, "_want_rows", lambda *args: None)
    monkeypatch.setattr(binding, "_room", lambda *args: None)
    rows, q, k = new(1, HUGE, 1), new(1, 1, HUGE, 2), new(1, 1, 5, 2)
    x, w = new(HUGE, 1), new(1, 1)
    with pytest.raises(ValueError, match="2\\^31"):
        {"fwd": lambda: gla.gla_recur_fwd(rows, rows, 1, HUGE), "bwd": lambda: gla.gla_recur_bwd(rows, rows, rows, 1, HUGE),
         "step": lambda: gla.gla_recur_step(x, x, new(HUGE, 1, dtype=torch.float32)), "qk_fwd": lambda: gla.gla_qk_norm_fwd(q, None),
         "qk_bwd": lambda: gla.gla_qk_norm_bwd(q, None, q, None), "qk_keys": lambda: gla.gla_qk_norm_fwd(new(1, 1, 5, 2), new(1, HUGE, 5, 2)),
         "glu_fwd": lambda: gla.gla_glu_fwd(x, w, w), "glu_bwd": lambda: gla.gla_glu_bwd(x, w, w, x), "glu_columns": lambda: gla.gla_glu_fwd(w, x, x)}[call]()


def test_option_of_two_numbers():
    """Off at first; only off and on; the backward call's two arrays twice, of bf16 calls."""
    assert gla.gla_get_option(gla.OPT_GLU_SPLIT) == 0
    one, fp32 = (gla.gla_glu_bwd_workspace_bytes(8192, 2048, 8192, t) for t in (gla.DT_BF16, gla.DT_F32))
    for bad in (-1, 2):
        with pytest.raises(gla.GlaError):
            gla.gla_set_option(gla.OPT_GLU_SPLIT, bad)
    gla.gla_set_option(gla.OPT_GLU_SPLIT, 1)
    try:
        assert gla.gla_glu_bwd_workspace_bytes(8192, 2048, 8192) >= one + 2 * 8192 * 8192 * 2
        assert gla.gla_glu_bwd_workspace_bytes(8192, 2048, 8192, gla.DT_F32) == fp32
    finally:
        gla.gla_set_option(gla.OPT_GLU_SPLIT, 0)
    assert gla.gla_glu_bwd_workspace_bytes(8192, 2048, 8192) == one
