"""Gradients of the gated feed-forward product from dg and du as two bf16 numbers each (OPT_GLU_SPLIT), number by number against the 64-bit formulas.

Tolerances as in test_gpu_glu.py, but dg and du are within 2^-16 of themselves instead of 2^-8 (what the first number leaves, 2^-8, is rounded to 2^-8 of itself); sums
are twice as long.  In the 2-norm what is left beside the results' own rounding is below a hundredth of it."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla
from oracle import block_oracle as bo
from tests import test_gpu_glu as tg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gla.load_library()


@pytest.fixture(autouse=True)
def _split():
    gla.gla_set_option(gla.OPT_GLU_SPLIT, 1)
    yield
    gla.gla_set_option(gla.OPT_GLU_SPLIT, 0)


def gradients(x, wg, wu, do, act, kept):
    x, wg, wu, do = (t.to(DEV) for t in (x, wg, wu, do))
    pre = torch.empty(2, *do.shape, device=DEV) if kept else None
    if kept:
        gla.gla_glu_fwd(x, wg, wu, act, pre=pre)
    return gla.gla_glu_bwd(x, wg, wu, do, act, pre=pre)


@pytest.mark.parametrize("kept", [True, False])
@pytest.mark.parametrize("M,K,F", [(1, 1, 1), (2, 8, 16), (3, 7, 5), (33, 65, 200), (64, 96, 127), (127, 384, 65), (129, 200, 250), (257, 520, 260), (1021, 381, 1531), (520, 1150, 1100),
                                   (1500, 1100, 2100), (2100, 2300, 1030), (4200, 2100, 1050), (4096, 4096, 1024)])
def test_as_exact_as_their_rounding(M, K, F, kept):
    act = M % 3 if M < 1000 else 0
    x, wg, wu, do = tg.make(M, K, F, BF16, M)
    got = gradients(x, wg, wu, do, act, kept)
    X, WG, WU, DO = (t.double().numpy() for t in (x, wg, wu, do))
    g, u = X @ WG.T, X @ WU.T
    a, slope = bo.activation(tg.KIND[act], g)
    want = bo.glu_bwd(X, WG, WU, tg.KIND[act], DO)
    sums = lambda n: (n / 4 + 32) * 2.0 ** -24  # noqa: E731
    eg, eu = (sums(K) * (np.abs(X) @ np.abs(w).T) for w in (WG, WU))
    near = 2.0 ** -20 * np.minimum(np.abs(g), 2)
    ea = 1.13 * eg + 2.0 ** -20 * np.abs(a) + near
    dg, du, two = DO * u * slope, DO * a, 2.0 ** -16
    edg = np.abs(DO) * ((np.abs(slope) + near) * eu + np.abs(u) * (0.8 * eg + 2.0 ** -19 + near)) + two * np.abs(dg)
    edu = np.abs(DO) * ea + two * np.abs(du)
    tg.close(got[0], want[0], edg @ np.abs(WG) + edu @ np.abs(WU) + sums(4 * F) * (np.abs(dg) @ np.abs(WG) + np.abs(du) @ np.abs(WU)), 2.0 ** -8, "dx")
    tg.close(got[1], want[1], edg.T @ np.abs(X) + sums(2 * M) * (np.abs(dg).T @ np.abs(X)), 2.0 ** -8, "dw_gate")
    tg.close(got[2], want[2], edu.T @ np.abs(X) + sums(2 * M) * (np.abs(du).T @ np.abs(X)), 2.0 ** -8, "dw_up")
    if M * K > 10000:
        for p, w in zip(got, want):
            w = torch.from_numpy(w).to(DEV)
            assert tg.off(p, w) < 1.02 * tg.off(w.to(BF16), w)


@pytest.mark.parametrize("act", [0, 1, 2])
def test_products_without_end(act):
    """What a number that rounds to infinity leaves is nothing, not NaN; a NaN stays one."""
    x = torch.ones(1, 8, device=DEV, dtype=BF16)
    w = torch.zeros(8, 8, device=DEV, dtype=BF16)
    for value in (3.3e38, float("inf"), float("nan"), 1e-40):
        do = torch.full((1, 8), value, device=DEV, dtype=BF16)
        wg, wu = w.clone(), w.clone()
        wg[:, 0], wu[:, 0] = 4.0, 2.0        # u = 2: dg is past the largest number
        both = []
        for split in (1, 0):
            gla.gla_set_option(gla.OPT_GLU_SPLIT, split)
            both.append(gla.gla_glu_bwd(x, wg, wu, do, act)[1:])
        for p, q in zip(*both):
            assert torch.equal(torch.isnan(p), torch.isnan(q)) and torch.equal(torch.isinf(p), torch.isinf(q)), (value, p, q)


def test_other_calls_take_no_notice():
    """The forward call, fp32 calls, and calls behind it; a workspace for one number each is too small."""
    x, wg, wu, do = (t.to(DEV) for t in tg.make(300, 200, 136, torch.float32, 1))
    sixteen = [t.to(BF16) for t in (x, wg, wu, do)]
    on = [gla.gla_glu_fwd(*sixteen[:3]), *gla.gla_glu_bwd(x, wg, wu, do), *gla.gla_glu_bwd(*sixteen)]
    small = torch.empty(2 * 300 * 136 * 2 + 512, dtype=torch.uint8, device=DEV)
    gla.gla_set_option(gla.OPT_GLU_SPLIT, 0)
    need = gla.gla_glu_bwd_workspace_bytes(300, 200, 136)
    off = [gla.gla_glu_fwd(*sixteen[:3]), *gla.gla_glu_bwd(x, wg, wu, do), *gla.gla_glu_bwd(*sixteen)]
    assert all(torch.equal(a, b) for a, b in zip(on[:4], off[:4])) and not any(torch.equal(a, b) for a, b in zip(on[4:], off[4:]))
    gla.gla_set_option(gla.OPT_GLU_SPLIT, 1)
    assert gla.gla_glu_bwd_workspace_bytes(300, 200, 136) >= need + 2 * 300 * 136 * 2
    with pytest.raises(gla.GlaError):
        gla.gla_glu_bwd(*sixteen, workspace=small)


def test_graph():
    """Captured with the option on, replayed with it off: what was captured."""
    x, wg, wu, do = (t.to(DEV) for t in tg.make(300, 129, 200, BF16, 4))
    want = gla.gla_glu_bwd(x, wg, wu, do, 1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = gla.gla_glu_bwd(x, wg, wu, do, 1)
    gla.gla_set_option(gla.OPT_GLU_SPLIT, 0)
    for _ in range(3):
        for t in held:
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))
        gla.gla_glu_bwd(x, wg, wu, do, 1)
