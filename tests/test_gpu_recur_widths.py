"""Gated recurrence of channels at the usual widths and in every variant of its kernels, by the formulas and tolerances of test_gpu_recur.py."""
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla
from tests import test_gpu_recur as tr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gla.load_library()


@pytest.mark.parametrize("kind,tau", tr.KINDS)
@pytest.mark.parametrize("scan", [0, 1])
@pytest.mark.parametrize("T,D,dtype,lens", [(200, 384, BF16, [200, 0, 65, 1]), (700, 384, F32, [333, 700]), (700, 1152, BF16, [1, 700, 640]), (300, 2048, BF16, [129, 0, 300]),
                                            (2100, 128, F32, [2100, 2049, 0, 128])])
def test_padded_batches_of_whole_waves(T, D, dtype, lens, scan, kind, tau):
    """Waves that hold channels of one sequence only: each begins at its own sequence's end in reversed scans."""
    tr.check(tr.make(len(lens), T, D, dtype, kind, T, lens=lens), 1, T, scan, kind, tau, D != 384, F32)


@pytest.mark.parametrize("kind,tau", tr.KINDS)
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("scan", [0, 1])
@pytest.mark.parametrize("B,T,D", [(16, 300, 2048), (300, 20, 130), (130, 260, 255)])
def test_padded_batches_that_are_walked(B, T, D, scan, kind, tau, rest):
    lens = [(37 * b * b + 5) % (T + 1) for b in range(B)]
    lens[:3] = [T, 0, 1]
    tr.check(tr.make(B, T, D, BF16, kind, D, lens=lens), 1, T, scan, kind, tau, rest, F32)


@pytest.mark.parametrize("kind,tau,dtype", [(k, t, d) for k, t in tr.KINDS for d in (BF16, F32)])
@pytest.mark.parametrize("D,gh,gw,scan,rest", [(2049, 64, 64, 3, False), (2049, 1, 4096, 1, True), (4100, 63, 65, 2, True), (4096, 60, 68, 0, False)])
def test_many_rounds_backward(D, gh, gw, scan, rest, kind, tau, dtype):
    """2048 rounds of all groups and more: a wave each."""
    tr.check(tr.make(1, gh * gw, D, dtype, kind, D), gh, gw, scan, kind, tau, rest, F32)


@pytest.mark.parametrize("kind,tau", tr.KINDS)
@pytest.mark.parametrize("scan", [0, 1])
@pytest.mark.parametrize("D,dtype", [(1411, F32), (1536, BF16), (1600, F32)])
def test_many_rounds_backward_of_padded_batches(D, dtype, scan, kind, tau):
    lens = [2100, 0, 1999, 64, 2048]
    tr.check(tr.make(5, 2100, D, dtype, kind, D, lens=lens), 1, 2100, scan, kind, tau, D != 1536, F32)


def lens_of(B, T):
    return torch.tensor(([T, 0, T // 2 + 1, 1, 129] * B)[:B], dtype=torch.int32)


@pytest.mark.parametrize("kind,name", [(gla.GATE_PRE, "x"), (gla.GATE_PRE, "gate"), (gla.GATE_LOG, "gate"), (gla.GATE_LOG, "x")])
@pytest.mark.parametrize("scan,padded", [(0, False), (1, False), (2, False), (3, False), (0, True), (1, True)])
@pytest.mark.parametrize("B,gh,gw,D", [(16, 20, 35, 2048), (40, 10, 26, 511), (3, 10, 20, 130), (2, 50, 101, 256), (5, 45, 60, 37), (1, 83, 99, 514)])
def test_in_place(B, gh, gw, D, scan, padded, kind, name):
    """Over the inputs, and the final state over the initial one: the bits of the call out of place.  Sequences walked by a work-group (the first three), and in units of
    several blocks, where the state handed from one block to the next has to come from an initial state that is still there."""
    T = gh * gw
    p = {n: t.to(DEV) for n, t in tr.make(B, T, D, BF16, kind, 8).items()}
    gh, gw = (1, T) if padded else (gh, gw)
    how = {"scan_dir": scan, "gate_kind": kind, "complement": True, "seq_lens": lens_of(B, T).to(DEV) if padded else None}
    y = p[name].clone()
    _, fin = gla.gla_recur_fwd(p["x"], p["gate"], gh, gw, initial_state=p["s0"], out=y, **how)
    for _ in range(3):
        q = {n: t.clone() for n, t in p.items()}
        out, last = gla.gla_recur_fwd(q["x"], q["gate"], gh, gw, initial_state=q["s0"], out=q[name], final_state=q["s0"], **how)
        assert out is q[name] and last is q["s0"] and torch.equal(out, y) and torch.equal(last, fin)
        # only the state in place
        s = p["s0"].clone()
        apart, last = gla.gla_recur_fwd(p["x"], p["gate"], gh, gw, initial_state=s, final_state=s, out=p[name].clone(), **how)
        assert torch.equal(apart, y) and torch.equal(s, fin)
