"""Gated feed-forward product (gla_glu_fwd / gla_glu_bwd) against the 64-bit formulas.

Tolerances.  A product's sum over K is added in fp32, one MFMA after the other and up to 32 numbers inside one: off by at most (K / 4 + 32) 2^-24
of the sum of absolute values |x| |w|, s.  Over the sizes here the roundings are as good as random, but nothing is made of that.  The
activation's own steps are within 2^-20 and its slope is at most 1.13, its second derivative at most 0.8: y = act(g) u is off by
(1.13 |u| sg + |act| su) of the products' errors and 2^-20 |y|, and by 2^-20 |u| min(|g|, 2) where act is near zero (an exponential's argument is
rounded).  dg and du likewise, and bf16 calls round them to 2^-8 of themselves; dx and dw are their sums with weights and rows, whose errors add
up as absolute values, plus their own sums' 2^-24 (terms / 4 + 32).  Results of 16 bits are rounded once, 2^-8."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla
from oracle import block_oracle as bo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
ROUND = {F32: 2.0 ** -23, BF16: 2.0 ** -8}
KIND = {0: "silu", 1: "gelu", 2: "gelu_tanh"}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gla.load_library()


def close(got, want, size, rounding, name):
    got = got.double().cpu().numpy().reshape(want.shape)
    bad = np.abs(got - want) - (size + rounding * np.abs(want) + 1e-30)
    assert np.isfinite(got).all() and bad.max() <= 0, (name, float(bad.max()), np.unravel_index(bad.argmax(), bad.shape))


def make(M, K, F, dtype, seed, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    return randn(M, K).to(dtype), *((randn(F, K) * scale * K ** -0.5).to(dtype) for _ in range(2)), randn(M, F).to(dtype)


def check(M, K, F, dtype, act, seed=0, scale=1.0, out_dtype=None, kept=True, backward=True):
    x, wg, wu, do = make(M, K, F, dtype, seed, scale)
    dx_, dwg_, dwu_, ddo = (t.to(DEV) for t in (x, wg, wu, do))
    pre = torch.full((2, M, F), 77.0, device=DEV)
    y = gla.gla_glu_fwd(dx_, dwg_, dwu_, act, out_dtype=out_dtype, pre=pre if kept else None)
    X, WG, WU, DO = (t.double().numpy() for t in (x, wg, wu, do))
    g, u = X @ WG.T, X @ WU.T
    a, slope = bo.activation(KIND[act], g)
    sums = lambda n: (n / 4 + 32) * 2.0 ** -24  # noqa: E731
    eg, eu = (sums(K) * (np.abs(X) @ np.abs(w).T) for w in (WG, WU))
    if kept:
        close(pre[0], g, eg, 2.0 ** -23, "g")
        close(pre[1], u, eu, 2.0 ** -23, "u")
    near = 2.0 ** -20 * np.minimum(np.abs(g), 2)
    ea = 1.13 * eg + 2.0 ** -20 * np.abs(a) + near
    close(y, bo.glu_fwd(X, WG, WU, KIND[act]), ea * (np.abs(u) + eu) + np.abs(a) * eu, ROUND[y.dtype], "y")
    if not backward:
        return
    dx, dwg, dwu = gla.gla_glu_bwd(dx_, dwg_, dwu_, ddo, act, pre=pre if kept else None)
    assert dx.dtype == dwg.dtype == dwu.dtype == dtype
    wx, wwg, wwu = bo.glu_bwd(X, WG, WU, KIND[act], DO)
    dg, du = DO * u * slope, DO * a
    half = 2.0 ** -8 if dtype is BF16 else 2.0 ** -24
    edg = np.abs(DO) * ((np.abs(slope) + near) * eu + np.abs(u) * (0.8 * eg + 2.0 ** -19 + near)) + half * np.abs(dg)
    edu = np.abs(DO) * ea + half * np.abs(du)
    close(dx, wx, edg @ np.abs(WG) + edu @ np.abs(WU) + sums(2 * F) * (np.abs(dg) @ np.abs(WG) + np.abs(du) @ np.abs(WU)), ROUND[dtype], "dx")
    close(dwg, wwg, edg.T @ np.abs(X) + sums(M) * (np.abs(dg).T @ np.abs(X)), ROUND[dtype], "dw_gate")
    close(dwu, wwu, edu.T @ np.abs(X) + sums(M) * (np.abs(du).T @ np.abs(X)), ROUND[dtype], "dw_up")


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,K,F", [(1, 1, 1), (1, 64, 64), (2, 8, 16), (3, 7, 5), (16, 32, 128), (17, 33, 31), (31, 100, 129), (32, 64, 72), (33, 65, 200), (64, 96, 127),
                                   (65, 72, 136), (127, 384, 65), (128, 128, 128), (129, 200, 250), (200, 63, 300), (255, 381, 77), (256, 64, 256), (257, 520, 260)])
def test_sizes(M, K, F, dtype):
    act = (M + K) % 3
    check(M, K, F, dtype, act, seed=M)
    check(M, K, F, dtype, (act + 1) % 3, seed=M + 1, kept=False)


@pytest.mark.parametrize("dtype,out_dtype", [(BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("M", [5, 300])
def test_other_result_types(M, dtype, out_dtype):
    check(M, 96, 100, dtype, 0, out_dtype=out_dtype, backward=False)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act", [0, 1, 2])
def test_activations_far_from_zero(act, dtype):
    check(40, 48, 56, dtype, act, seed=act, scale=12.0)


@pytest.mark.parametrize("act", [0, 1, 2])
def test_activations_without_end(act):
    """Products up to 1e30: the activation is g or nothing there, and its slope one or nothing."""
    g = torch.tensor([[1e3, 1e10, 1e20, 1e30, -1e3, -1e10, -1e20, -1e30]], device=DEV)
    one, eye = torch.ones(8, 1, device=DEV), torch.zeros(8, 4, device=DEV)
    eye[:, 0] = g[0]
    x = torch.tensor([[1.0, 0, 0, 0]], device=DEV)
    up = torch.tensor([[1.0, 0, 0, 0]], device=DEV) * one
    y = gla.gla_glu_fwd(x, eye, up, act)
    assert torch.equal(y, g.clamp(min=0))
    do = torch.zeros(1, 8, device=DEV)
    for i in range(8):
        do.zero_()[0, i] = 1.0
        dx, dwg, dwu = gla.gla_glu_bwd(x, eye, up, do, act)
        assert float(dwg[i, 0]) == (1.0 if i < 4 else 0.0) and float(dwu[i, 0]) == float(y[0, i]), (i, dwg[i, 0], dwu[i, 0])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,K,F", [(1, 2048, 8192), (7, 1152, 4608), (33, 2048, 1000), (100, 1152, 4608), (1000, 1152, 2000), (3000, 500, 2048), (2100, 2300, 2056), (700, 4100, 1030)])
def test_large(M, K, F, dtype):
    """Many tiles, both tile sizes, sums in parts: against 64 bits on the GPU, by 2-norm.  Sums of n random terms in fp32 are off by less than
    sqrt(n) 2^-24 of their size; results of 16 bits by their rounding, 2^-8 / sqrt(3) at most, gradients of these by sqrt(2) times that."""
    x, wg, wu, do = (t.to(DEV) for t in make(M, K, F, dtype, M))
    pre = torch.empty(2, M, F, device=DEV)
    y = gla.gla_glu_fwd(x, wg, wu, 0, pre=pre)
    leaves = [t.double().requires_grad_(True) for t in (x, wg, wu)]
    g, u = leaves[0] @ leaves[1].t(), leaves[0] @ leaves[2].t()
    want = torch.nn.functional.silu(g) * u
    grads = torch.autograd.grad(want, leaves, do.double())
    most = 2.0 ** -8 / 3 ** 0.5 if dtype is BF16 else 2.0 ** -24 * max(K, 2 * F, M) ** 0.5 * 2
    assert off(pre[0], g.detach()) < 2.0 ** -24 * K ** 0.5 and off(pre[1], u.detach()) < 2.0 ** -24 * K ** 0.5
    assert off(y, want.detach()) < most
    for kept in (pre, None):
        for got, w in zip(gla.gla_glu_bwd(x, wg, wu, do, 0, pre=kept), grads):
            assert off(got, w) < most * 2 ** 0.5
    dx, none, _ = gla.gla_glu_bwd(x, wg, wu, do, 0, pre=pre, want_dw=False)
    nox, dwg, dwu = gla.gla_glu_bwd(x, wg, wu, do, 0, pre=pre, want_dx=False)
    assert none is None and nox is None and off(dx, grads[0]) < most * 2 ** 0.5 and off(dwg, grads[1]) < most * 2 ** 0.5 and off(dwu, grads[2]) < most * 2 ** 0.5


@pytest.mark.parametrize("M", [1, 20, 130])
def test_rows_stay_apart(M):
    """Rows of x that are not finite, and what lies behind the tensors, reach no other row."""
    room = torch.full((M + 300, 72), float("nan"), device=DEV, dtype=BF16)
    x, wg, wu, do = (t.to(DEV) for t in make(M, 72, 136, BF16, 3))
    room[:M] = x
    want = gla.gla_glu_fwd(x, wg, wu)
    assert torch.equal(gla.gla_glu_fwd(room[:M], wg, wu), want)
    if M > 1:
        x[M // 2] = float("nan")
        y = gla.gla_glu_fwd(x, wg, wu)
        keep = torch.arange(M, device=DEV) != M // 2
        assert torch.equal(y[keep], want[keep]) and torch.isnan(y[M // 2]).all()


@pytest.mark.parametrize("M,K,F", [(9, 40, 70), (300, 129, 200)])
def test_shapes_graph_and_streams(M, K, F):
    x, wg, wu, do = (t.to(DEV) for t in make(M, K, F, BF16, 4))
    y = gla.gla_glu_fwd(x, wg, wu, 1)
    assert torch.equal(gla.gla_glu_fwd(x.view(1, 3, M // 3, K), wg, wu, 1).view(M, F), y)
    code = gla.DT_BF16
    ws = torch.empty(max(16, gla.gla_glu_fwd_workspace_bytes(M, K, F, code)), dtype=torch.uint8, device=DEV)
    wb = torch.empty(gla.gla_glu_bwd_workspace_bytes(M, K, F, code), dtype=torch.uint8, device=DEV)
    pre = torch.empty(2, M, F, device=DEV)
    back = gla.gla_glu_bwd(x, wg, wu, do, 1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = [gla.gla_glu_fwd(x, wg, wu, 1, pre=pre, workspace=ws), *gla.gla_glu_bwd(x, wg, wu, do, 1, pre=pre, workspace=wb)]
    for _ in range(3):
        for t in held + [pre]:
            t.fill_(3.0)
        ws.fill_(255)
        wb.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, (y, *back)))
        gla.gla_glu_bwd(x, wu, wg, do, 2, workspace=wb)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [gla.gla_glu_bwd(x, wg, wu, do, 1, stream=s) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for got in outs for a, b in zip(got, back))


def test_refusals():
    x, w, do = torch.zeros(3, 16, device=DEV), torch.zeros(24, 16, device=DEV), torch.zeros(3, 24, device=DEV)
    for args, bad in (((x, w, w[:8]), {}), ((x, w.to(BF16), w), {}), ((x[:, :8], w, w), {}), ((x.cpu(), w, w), {}), ((x, w, w), {"pre": torch.zeros(3, 24, device=DEV)}),
                      ((x, w, w), {"out": torch.zeros(3, 23, device=DEV)}), ((x[0], w, w), {}), ((x, w.t().contiguous().t(), w), {})):
        with pytest.raises((ValueError, TypeError)):
            gla.gla_glu_fwd(*args, **bad)
    room = torch.zeros(2 * 3 * 24 + 3 * 24, device=DEV)
    for bad in ({"act": 3}, {"act": -1}, {"out": room[:72].view(3, 24), "pre": room[4:148].view(2, 3, 24)}):
        with pytest.raises(gla.GlaError):
            gla.gla_glu_fwd(x, w, w, **bad)
    with pytest.raises(gla.GlaError):
        gla.gla_glu_fwd(x[:0], w, w)
    with pytest.raises(gla.GlaError):
        gla.gla_glu_bwd(x, w, w, do, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(gla.GlaError):
        gla.gla_glu_bwd(x, w, w, do, want_dx=False, want_dw=False)
    with pytest.raises(ValueError):
        gla.gla_glu_bwd(x, w, w, do[:2])
