"""Calls of the operators around a mixer with one decay a head that are refused on the host, before anything is enqueued (no GPU), and the
sizes of their workspaces."""
import ctypes

import pytest

import paper_2405_18428_amd as gla

vp = ctypes.c_void_p
OK, OFF = vp(4096), vp(4100)
NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def lib():
    return gla.load_library()


FWD = {"q": OK, "k": OK, "v": OK, "g": OK, "kind": 0, "lens": None, "B": 2, "H": 2, "T": 1024, "dk": 32, "dv": 64, "gh": 1, "gw": 1024, "scan": 0,
       "dt": 1, "odt": 1, "layout": 0, "s0": None, "out": OK, "fin": None, "ws": OK, "wsb": 1 << 30, "stream": None}
BWD = {"q": OK, "k": OK, "v": OK, "g": OK, "kind": 0, "lens": None, "do": OK, "s0": None, "ds": None, "B": 2, "H": 2, "T": 1024, "dk": 32, "dv": 64,
       "gh": 1, "gw": 1024, "scan": 0, "dt": 1, "odt": 1, "layout": 0, "dq": OK, "dkg": OK, "dvg": OK, "dg": OK, "ds0": None, "ws": OK, "wsb": 1 << 30,
       "stream": None}
SHARED = [({"q": None}, NULL), ({"v": None}, NULL), ({"g": None}, NULL), ({"B": 0}, SHAPE), ({"H": -1}, SHAPE), ({"T": 0, "gw": 0}, SHAPE),
          ({"gw": 1023}, SHAPE), ({"scan": 4}, SHAPE), ({"scan": -1}, SHAPE), ({"layout": 2}, SHAPE), ({"dt": 2}, SHAPE), ({"odt": -1}, SHAPE),
          ({"kind": 2}, SHAPE), ({"dk": 129}, UNSUPPORTED), ({"dv": 129}, UNSUPPORTED), ({"lens": OK, "scan": 2}, UNSUPPORTED),
          ({"B": 1 << 12, "H": 1 << 12}, UNSUPPORTED), ({"T": (1 << 30) + 1, "gw": (1 << 30) + 1}, UNSUPPORTED), ({"q": OFF}, ALIGN), ({"g": OFF}, ALIGN),
          ({"lens": vp(4097)}, ALIGN), ({"s0": OFF}, ALIGN), ({"ws": None}, WORKSPACE), ({"ws": OFF}, WORKSPACE), ({"wsb": 64}, WORKSPACE)]


@pytest.mark.parametrize("change,status", SHARED + [({"out": None}, NULL), ({"out": OFF}, ALIGN), ({"fin": OFF}, ALIGN)])
def test_decay_fwd(lib, change, status):
    assert lib.gla_decay_fwd(*{**FWD, **change}.values()) == status


@pytest.mark.parametrize("change,status", SHARED + [({"do": None}, NULL), ({"dq": None}, NULL), ({"dkg": None}, NULL), ({"dvg": None}, NULL), ({"do": OFF}, ALIGN),
                                                    ({"ds": OFF}, ALIGN), ({"dg": OFF}, ALIGN), ({"ds0": OFF}, ALIGN), ({"dvg": OFF}, ALIGN)])
def test_decay_bwd(lib, change, status):
    assert lib.gla_decay_bwd(*{**BWD, **change}.values()) == status


STEP = {"q": OK, "k": OK, "v": OK, "g": OK, "kind": 1, "B": 2, "H": 2, "dk": 32, "dv": 64, "dt": 1, "odt": 1, "s": OK, "s1": OK, "out": OK, "stream": None}


@pytest.mark.parametrize("change,status", [({"k": None}, NULL), ({"s": None}, NULL), ({"s1": None}, NULL), ({"out": None}, NULL), ({"B": 0}, SHAPE),
                                           ({"dv": 0}, SHAPE), ({"dt": 3}, SHAPE), ({"odt": 3}, SHAPE), ({"kind": -1}, SHAPE), ({"dk": 129}, UNSUPPORTED),
                                           ({"B": 1 << 22}, UNSUPPORTED), ({"s": OFF}, ALIGN), ({"s1": OFF}, ALIGN), ({"q": vp(4097)}, ALIGN),
                                           ({"g": vp(4098)}, ALIGN), ({"s1": vp(4096 + 64)}, SHAPE), ({"s": vp(4096 + 64)}, SHAPE)])
def test_decay_step(lib, change, status):
    assert lib.gla_decay_step(*{**STEP, **change}.values()) == status


ROPE = {"q": OK, "k": vp(8192), "pos": None, "sec": (16, 16), "axes": 2, "base": ctypes.c_float(10000.0), "pairing": 0, "inverse": 0, "B": 1, "H": 2, "T": 12,
        "d": 32, "gh": 3, "gw": 4, "dt": 1, "layout": 0, "oq": vp(12288), "ok": vp(16384), "stream": None}


@pytest.mark.parametrize("change,status", [({"q": None}, NULL), ({"oq": None}, NULL), ({"ok": None}, NULL), ({"k": None}, NULL), ({"sec": None}, NULL),
                                           ({"axes": 0}, SHAPE), ({"sec": (16, 18)}, SHAPE), ({"sec": (15, 16)}, SHAPE), ({"sec": (0, 16)}, SHAPE),
                                           ({"sec": (2 ** 31 - 2, 16)}, SHAPE), ({"base": ctypes.c_float(0.0)}, SHAPE), ({"base": ctypes.c_float(float("nan"))}, SHAPE),
                                           ({"pairing": 2}, SHAPE), ({"gh": 0}, SHAPE), ({"gw": 5}, SHAPE), ({"T": 13, "axes": 3, "sec": (4, 4, 4)}, SHAPE),
                                           ({"axes": 4, "sec": (4, 4, 4, 4)}, SHAPE), ({"axes": 5, "sec": (2,) * 5, "pos": OK}, UNSUPPORTED), ({"d": 258}, UNSUPPORTED),
                                           ({"q": OFF}, ALIGN), ({"ok": OFF}, ALIGN), ({"pos": vp(4098)}, ALIGN), ({"oq": vp(8192)}, SHAPE), ({"ok": OK}, SHAPE),
                                           ({"ok": vp(12288)}, SHAPE), ({"k": OK, "oq": OK}, SHAPE), ({"B": 1 << 20, "T": 1 << 16, "gh": 1 << 8, "gw": 1 << 8}, UNSUPPORTED)])
def test_rope(lib, change, status):
    a = {**ROPE, **change}
    a["sec"] = None if a["sec"] is None else (ctypes.c_int * len(a["sec"]))(*a["sec"])
    assert lib.gla_rope(*a.values()) == status


NORM = {"x": OK, "w": None, "b": None, "eps": ctypes.c_float(1e-5), "r": None, "B": 2, "H": 2, "T": 8, "D": 64, "dt": 1, "odt": 0, "layout": 0, "out": vp(8192),
        "stream": None}
NORM_BWD = {"x": OK, "do": OK, "w": None, "b": None, "eps": ctypes.c_float(1e-5), "r": None, "B": 2, "H": 2, "T": 8, "D": 64, "dt": 1, "odt": 0, "layout": 0,
            "dx": OK, "dr": None, "dw": None, "db": None, "ws": OK, "wsb": 1 << 30, "stream": None}
NORM_SHARED = [({"x": None}, NULL), ({"B": 0}, SHAPE), ({"D": 0}, SHAPE), ({"eps": ctypes.c_float(-1.0)}, SHAPE), ({"eps": ctypes.c_float(float("nan"))}, SHAPE),
               ({"dt": 2}, SHAPE), ({"odt": 2}, SHAPE), ({"layout": -1}, SHAPE), ({"D": 8193}, UNSUPPORTED), ({"B": 1 << 16, "T": 1 << 16}, UNSUPPORTED),
               ({"H": (1 << 17) + 1}, UNSUPPORTED), ({"x": OFF}, ALIGN), ({"w": OFF}, ALIGN), ({"b": OFF}, ALIGN)]


@pytest.mark.parametrize("change,status", NORM_SHARED + [({"out": None}, NULL), ({"out": OFF}, ALIGN), ({"r": OFF}, ALIGN), ({"out": OK}, SHAPE)])
def test_norm_fwd(lib, change, status):
    assert lib.gla_norm_fwd(*{**NORM, **change}.values()) == status


@pytest.mark.parametrize("change,status", NORM_SHARED + [({"do": None}, NULL), ({"dx": None}, NULL), ({"r": OK}, NULL), ({"dr": OK}, NULL), ({"dw": OK}, NULL),
                                                         ({"do": OFF}, ALIGN), ({"dx": OFF}, ALIGN), ({"ws": None}, WORKSPACE), ({"wsb": 16}, WORKSPACE)])
def test_norm_bwd(lib, change, status):
    assert lib.gla_norm_bwd(*{**NORM_BWD, **change}.values()) == status


def test_workspaces():
    # two fp32 words a token for the flows and a state for each 256 of them; nothing forward where there are more sequences than compute units
    n = gla.gla_decay_bwd_workspace_bytes(40, 8, 1024, 64, 64)
    assert n >= 320 * (1024 * 8 + 4 * 64 * 64 * 4) and n < 2 * 320 * (1024 * 8 + 4 * 64 * 64 * 4)
    assert gla.gla_decay_fwd_workspace_bytes(40, 8, 1024, 64, 64) == 0
    assert gla.gla_decay_fwd_workspace_bytes(1, 16, 65536, 128, 128) >= 16 * 32 * 128 * 128 * 4
    for bad in ((0, 1, 1, 1, 1), (1, 1, 1, 129, 1), (1, 1, 1, 1, 129), (1, 1, -5, 1, 1)):
        assert gla.gla_decay_fwd_workspace_bytes(*bad) == 0 and gla.gla_decay_bwd_workspace_bytes(*bad) == 0
    assert gla.gla_norm_bwd_workspace_bytes(2, 1, 100, 1152) >= 2 * 1152 * 4
    assert gla.gla_norm_bwd_workspace_bytes(2, 1, 100, 8193) == 0
