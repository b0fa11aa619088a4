"""Calls of the operators that stand around the mixer in a block (recurrence of channels, norm and rotation of queries and keys, gated feed-forward
product) that are refused on the host, before anything is enqueued (no GPU), and the sizes of their workspaces."""
import ctypes

import pytest

import paper_2405_18428_amd as gla

vp, cf = ctypes.c_void_p, ctypes.c_float
FAR = 1 << 34


def at(n):
    """Tensors far apart, aligned."""
    return vp(FAR * n)


OFF = vp(FAR * 30 + 4)
NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def lib():
    return gla.load_library()


RECUR = {"x": at(1), "gate": at(2), "kind": 1, "tau": cf(16.0), "rest": 0, "lens": None, "B": 2, "T": 1024, "D": 64, "gh": 1, "gw": 1024, "scan": 0, "dt": 1, "odt": 1,
         "s0": None, "out": at(3), "fin": None, "ws": at(4), "wsb": 1 << 30, "stream": None}
RECUR_BWD = {"x": at(1), "gate": at(2), "kind": 1, "tau": cf(16.0), "rest": 0, "lens": None, "do": at(5), "s0": None, "df": None, "B": 2, "T": 1024, "D": 64, "gh": 1,
             "gw": 1024, "scan": 0, "dt": 1, "odt": 1, "dx": at(6), "dg": at(7), "ds": None, "ws": at(4), "wsb": 1 << 30, "stream": None}
SHARED = [({"x": None}, NULL), ({"gate": None}, NULL), ({"B": 0}, SHAPE), ({"T": 0, "gw": 0}, SHAPE), ({"D": -1}, SHAPE), ({"gw": 1023}, SHAPE), ({"scan": 4}, SHAPE),
          ({"scan": -1}, SHAPE), ({"kind": 2}, SHAPE), ({"dt": 2}, SHAPE), ({"odt": -1}, SHAPE), ({"tau": cf(0.0)}, SHAPE), ({"tau": cf(float("nan"))}, SHAPE),
          ({"tau": cf(float("inf"))}, SHAPE), ({"lens": at(9), "scan": 2}, UNSUPPORTED), ({"T": (1 << 30) + 1, "gw": (1 << 30) + 1}, UNSUPPORTED), ({"D": (1 << 26) + 1}, UNSUPPORTED),
          ({"B": 1 << 20, "D": 1 << 10}, UNSUPPORTED), ({"x": OFF}, ALIGN), ({"gate": OFF}, ALIGN), ({"lens": vp(4097)}, ALIGN), ({"s0": OFF}, ALIGN), ({"ws": None}, WORKSPACE),
          ({"ws": OFF}, WORKSPACE), ({"wsb": 64}, WORKSPACE)]


@pytest.mark.parametrize("change,status", SHARED + [({"out": None}, NULL), ({"out": OFF}, ALIGN), ({"fin": OFF}, ALIGN), ({"out": vp(FAR + 16)}, SHAPE),
                                                    ({"out": at(1), "odt": 0}, SHAPE), ({"out": vp(FAR * 2 - 16)}, SHAPE), ({"s0": at(3)}, SHAPE), ({"fin": at(3)}, SHAPE),
                                                    ({"fin": at(1)}, SHAPE), ({"s0": at(8), "fin": vp(FAR * 8 + 16)}, SHAPE)])
def test_recur_fwd(lib, change, status):
    assert lib.gla_recur_fwd(*{**RECUR, **change}.values()) == status


@pytest.mark.parametrize("change,status", SHARED + [({"do": None}, NULL), ({"dx": None}, NULL), ({"dg": None}, NULL), ({"do": OFF}, ALIGN), ({"dx": OFF}, ALIGN), ({"ds": OFF}, ALIGN),
                                                    ({"df": OFF}, ALIGN), ({"dx": at(1)}, SHAPE), ({"dx": at(5)}, SHAPE), ({"dg": at(6)}, SHAPE), ({"dg": vp(FAR * 2 + 16)}, SHAPE),
                                                    ({"s0": at(8), "ds": at(8)}, SHAPE)])
def test_recur_bwd(lib, change, status):
    assert lib.gla_recur_bwd(*{**RECUR_BWD, **change}.values()) == status


STEP = {"x": at(1), "gate": at(2), "kind": 1, "tau": cf(1.0), "rest": 1, "B": 2, "D": 64, "dt": 1, "odt": 1, "s": at(3), "s1": at(3), "out": at(4), "stream": None}


@pytest.mark.parametrize("change,status", [({"x": None}, NULL), ({"gate": None}, NULL), ({"s": None}, NULL), ({"s1": None}, NULL), ({"out": None}, NULL), ({"B": 0}, SHAPE), ({"D": 0}, SHAPE),
                                           ({"kind": -1}, SHAPE), ({"dt": 3}, SHAPE), ({"odt": 3}, SHAPE), ({"tau": cf(-1.0)}, SHAPE), ({"B": 1 << 26}, UNSUPPORTED), ({"s": OFF}, ALIGN),
                                           ({"s1": OFF}, ALIGN), ({"x": vp(FAR + 1)}, ALIGN), ({"gate": vp(FAR + 2), "kind": 0}, ALIGN), ({"s1": vp(FAR * 3 + 16)}, SHAPE), ({"out": at(3)}, SHAPE),
                                           ({"out": at(1)}, SHAPE), ({"s1": at(2)}, SHAPE)])
def test_recur_step(lib, change, status):
    assert lib.gla_recur_step(*{**STEP, **change}.values()) == status


QK = {"q": at(1), "qs": None, "H": 4, "k": at(2), "ks": None, "Hk": 2, "qw": None, "kw": None, "eps": cf(1e-6), "pos": None, "sec": (16, 16), "axes": 2, "base": cf(1e4), "pairing": 0,
      "B": 1, "T": 12, "d": 32, "gh": 3, "gw": 4, "dt": 1, "odt": 1, "layout": 0, "oq": at(3), "ok": at(4), "stream": None}
QK_BWD = {"q": at(1), "qs": None, "H": 4, "k": at(2), "ks": None, "Hk": 2, "dq_": at(5), "dk_": at(6), "qw": at(7), "kw": None, "eps": cf(1e-6), "pos": None, "sec": (16, 16), "axes": 2,
          "base": cf(1e4), "pairing": 0, "B": 1, "T": 12, "d": 32, "gh": 3, "gw": 4, "dt": 1, "odt": 1, "layout": 0, "dq": at(8), "dk": at(9), "dqw": at(10), "dkw": None, "ws": at(11),
          "wsb": 1 << 30, "stream": None}
QK_SHARED = [({"q": None}, NULL), ({"sec": None}, NULL), ({"H": 0}, SHAPE), ({"Hk": -1}, SHAPE), ({"B": 0}, SHAPE), ({"T": 0}, SHAPE), ({"d": 0}, SHAPE), ({"axes": -1}, SHAPE), ({"dt": 2}, SHAPE),
             ({"odt": 5}, SHAPE), ({"layout": 2}, SHAPE), ({"pairing": 2}, SHAPE), ({"eps": cf(-1.0)}, SHAPE), ({"eps": cf(float("nan"))}, SHAPE), ({"eps": cf(float("inf"))}, SHAPE),
             ({"base": cf(0.0)}, SHAPE), ({"sec": (16, 18)}, SHAPE), ({"sec": (15, 16)}, SHAPE), ({"gw": 5}, SHAPE), ({"axes": 4, "sec": (4,) * 4}, SHAPE),
             ({"axes": 5, "sec": (2,) * 5, "pos": at(12)}, UNSUPPORTED), ({"d": 257}, UNSUPPORTED), ({"B": 1 << 16, "T": 1 << 15, "axes": 0}, UNSUPPORTED), ({"H": (1 << 20) + 1}, UNSUPPORTED),
             ({"qs": (-1, 0, 0)}, SHAPE), ({"ks": (0, 0, 1 << 41)}, SHAPE), ({"B": 1 << 24, "qs": (1 << 40, 0, 32)}, SHAPE), ({"B": 1 << 24, "ks": (1 << 17, 0, 32)}, SHAPE), ({"q": vp(FAR + 1)}, ALIGN), ({"qw": OFF}, ALIGN), ({"pos": vp(4098)}, ALIGN), ({"k": None}, NULL)]


def qk_args(d):
    d = dict(d)
    for n in ("qs", "ks"):
        d[n] = None if d[n] is None else (ctypes.c_longlong * 3)(*d[n])
    d["sec"] = None if d["sec"] is None else (ctypes.c_int * len(d["sec"]))(*d["sec"])
    return d.values()


@pytest.mark.parametrize("change,status", QK_SHARED + [({"oq": None}, NULL), ({"ok": None}, NULL), ({"k": None, "ok": None, "kw": at(7)}, NULL), ({"oq": OFF}, ALIGN), ({"ok": OFF}, ALIGN),
                                                       ({"oq": at(2)}, SHAPE), ({"ok": at(3)}, SHAPE), ({"oq": at(1), "odt": 0}, SHAPE), ({"oq": vp(FAR + 16)}, SHAPE),
                                                       ({"oq": at(1), "qs": (0, 32, 128)}, SHAPE), ({"ok": at(1)}, SHAPE)])
def test_qk_norm_fwd(lib, change, status):
    assert lib.gla_qk_norm_fwd(*qk_args({**QK, **change})) == status


@pytest.mark.parametrize("change,status", QK_SHARED + [({"dq_": None}, NULL), ({"dk_": None}, NULL), ({"dq": None}, NULL), ({"dk": None}, NULL),
                                                       ({"k": None, "dk": None, "dk_": None, "dkw": at(12)}, NULL), ({"dq_": OFF}, ALIGN), ({"dq": OFF}, ALIGN), ({"dqw": OFF}, ALIGN),
                                                       ({"dq": at(1)}, SHAPE), ({"dk": at(8)}, SHAPE), ({"dqw": at(7)}, SHAPE), ({"dq": at(6)}, SHAPE), ({"ws": None}, WORKSPACE),
                                                       ({"ws": OFF}, WORKSPACE), ({"wsb": 16}, WORKSPACE)])
def test_qk_norm_bwd(lib, change, status):
    assert lib.gla_qk_norm_bwd(*qk_args({**QK_BWD, **change})) == status


GLU = {"x": at(1), "wg": at(2), "wu": at(3), "M": 10, "K": 60, "F": 100, "act": 0, "dt": 1, "odt": 1, "out": at(4), "pre": None, "ws": at(5), "wsb": 1 << 30, "stream": None}
GLU_BWD = {"x": at(1), "wg": at(2), "wu": at(3), "do": at(6), "pre": None, "M": 10, "K": 60, "F": 100, "act": 0, "dt": 1, "dx": at(7), "dwg": at(8), "dwu": at(9), "ws": at(5), "wsb": 1 << 30,
           "stream": None}
GLU_SHARED = [({"x": None}, NULL), ({"wg": None}, NULL), ({"wu": None}, NULL), ({"M": 0}, SHAPE), ({"K": 0}, SHAPE), ({"F": -4}, SHAPE), ({"act": 3}, SHAPE), ({"act": -1}, SHAPE), ({"dt": 2}, SHAPE),
              ({"K": (1 << 20) + 1}, UNSUPPORTED), ({"F": (1 << 20) + 1}, UNSUPPORTED), ({"M": (1 << 28) + 1}, UNSUPPORTED), ({"K": 1 << 20, "F": 1 << 20}, UNSUPPORTED),
              ({"x": OFF}, ALIGN), ({"wu": OFF}, ALIGN), ({"ws": None}, WORKSPACE), ({"ws": OFF}, WORKSPACE), ({"wsb": 1000}, WORKSPACE)]


@pytest.mark.parametrize("change,status", GLU_SHARED + [({"out": None}, NULL), ({"odt": 2}, SHAPE), ({"out": OFF}, ALIGN), ({"pre": OFF}, ALIGN), ({"out": at(1)}, SHAPE), ({"out": vp(FAR * 2 + 64)}, SHAPE),
                                                        ({"pre": at(4)}, SHAPE), ({"pre": at(3)}, SHAPE)])
def test_glu_fwd(lib, change, status):
    assert lib.gla_glu_fwd(*{**GLU, **change}.values()) == status


@pytest.mark.parametrize("change,status", GLU_SHARED + [({"do": None}, NULL), ({"dwg": None}, NULL), ({"dwu": None}, NULL), ({"dx": None, "dwg": None, "dwu": None}, NULL), ({"do": OFF}, ALIGN),
                                                        ({"pre": OFF}, ALIGN), ({"dx": OFF}, ALIGN), ({"dwu": OFF}, ALIGN), ({"dx": at(1)}, SHAPE), ({"dwg": at(9)}, SHAPE), ({"dx": at(6)}, SHAPE),
                                                        ({"pre": at(7)}, SHAPE)])
def test_glu_bwd(lib, change, status):
    assert lib.gla_glu_bwd(*{**GLU_BWD, **change}.values()) == status


def test_workspaces():
    # forward: a decay and a state of 4 bytes for each 128 steps of a channel, and some more; nothing where channels alone fill the GPU, or for few steps
    n = gla.gla_recur_fwd_workspace_bytes(1, 65536, 2048)
    assert 512 * 2048 * 8 <= n < 512 * 2048 * 9
    assert gla.gla_recur_fwd_workspace_bytes(64, 2048, 2048) == 0 and gla.gla_recur_fwd_workspace_bytes(1, 128, 64) == 0
    assert gla.gla_recur_bwd_workspace_bytes(1, 65536, 2048) == 1024 * 2048 * 12 and gla.gla_recur_bwd_workspace_bytes(4, 64, 2048) == 0
    for bad in ((0, 1, 1), (1, -1, 1), (1, 1, 0), (1, (1 << 30) + 1, 1)):
        assert gla.gla_recur_fwd_workspace_bytes(*bad) == 0 and gla.gla_recur_bwd_workspace_bytes(*bad) == 0
    assert gla.gla_qk_norm_bwd_workspace_bytes(2, 16, 4, 100, 128) >= 2 * 128 * 4
    for bad in ((0, 1, 1, 1, 1), (1, 1, 1, 1, 257), (1, 0, 1, 1, 8), (1, 1, -1, 1, 8)):
        assert gla.gla_qk_norm_bwd_workspace_bytes(*bad) == 0
    # copies only of rows that are no whole pieces of 16 bytes; backward two arrays like the result and the parts of sums
    assert gla.gla_glu_fwd_workspace_bytes(100, 64, 200) == 0 and gla.gla_glu_fwd_workspace_bytes(100, 61, 200) >= (100 + 2 * 200) * 64 * 2
    assert gla.gla_glu_bwd_workspace_bytes(8192, 2048, 8192) >= 2 * 8192 * 8192 * 2
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, (1 << 20) + 1, 1)):
        assert gla.gla_glu_fwd_workspace_bytes(*bad) == 0 and gla.gla_glu_bwd_workspace_bytes(*bad) == 0
