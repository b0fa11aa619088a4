"""Tensors with more than 2^31 elements, and waits that run out.

The recurrence: all rows but the last ones are zero, whose outputs, states and gradients are held to the bounds of test_gpu_recur.py.  Norm and rotation
of queries and keys work on rows by themselves: the last rows have the bits that a call on them alone gives, and so have the products' rows, whose sums
over K go in one order whatever the tiles are; what is summed in parts is held to 2^-8 (bf16)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla
from oracle import block_oracle as bo
from tests.test_gpu_recur import sizes

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gla.load_library()


def host(t):
    return t.double().cpu().numpy()


def close(got, want, size, tol, rounding=2.0 ** -8):
    bad = np.abs(host(got) - want) - (tol * size + rounding * np.abs(want) + 1e-30)
    assert bad.max() <= 0, float(bad.max())


@pytest.mark.parametrize("B,T,D", [(1, (1 << 20) + 77, 2056), (70000, 1000, 36)])
def test_recurrence(B, T, D):
    n = 200
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, do = (torch.zeros(B, T, D, dtype=BF16, device=DEV) for _ in range(2))
    z = torch.full((B, T, D), 1.0, dtype=BF16, device=DEV)
    for t in (x, z, do):
        t[B - 1, T - n:] = torch.randn(n, D, generator=gen, device=DEV).to(BF16)
    y, fin = gla.gla_recur_fwd(x, z, 1, T)
    dx, dz, ds = gla.gla_recur_bwd(x, z, do, 1, T, grad_dtype=BF16, want_d_initial_state=True)
    torch.cuda.synchronize()
    X, Z, DO = (host(t[B - 1, T - n:])[None] for t in (x, z, do))
    lg, slope = bo.log_gate(Z, 16.0)
    zero = np.zeros((1, D))
    h = bo.recur_fwd(X, lg, False, zero)
    wx, wl, _ = bo.recur_bwd(X, lg, False, h, DO, zero)
    W, before = sizes(X, lg, zero)
    V = sizes(DO[:, ::-1], np.concatenate([np.zeros((1, 1, D)), lg[:, :0:-1]], 1), zero)[0][:, ::-1]
    tol = 2.0 ** -18
    close(y[B - 1, T - n:], h[0, 1:], W[0], tol)
    close(fin[B - 1], h[0, -1], W[0, -1], tol, 2.0 ** -23)
    close(dx[B - 1, T - n:], wx[0], V[0], 2 * tol)
    close(dz[B - 1, T - n:], (wl * slope)[0], (slope * (1 + np.abs(lg)) * before * V)[0], 4 * tol)
    assert not y[B - 1, :T - n].any() and not dz[B - 1, :T - n].any() and not y[:B - 1].any() and not dx[:B - 1].any()
    if B == 1:                           # the adjoint goes on to the first step
        decay = np.exp(bo.log_gate(1.0, 16.0)[0])
        close(dx[0, T - n - 1], wx[0, 0] * np.exp(lg[0, 0]), V[0, 0], 2 * tol)
        assert abs(float(ds[0, 0])) <= abs(wx[0, 0, 0]) * decay ** 1000


def test_queries_and_keys():
    T, H, Hk, d, n = 66000, 256, 8, 128, 300
    gen = torch.Generator(device=DEV).manual_seed(2)
    rows = torch.randn(1, T, (H + Hk) * d, generator=gen, device=DEV, dtype=BF16)
    q, k = rows[..., :H * d].unflatten(-1, (H, d)), rows[..., H * d:].unflatten(-1, (Hk, d))
    pos = torch.arange(T, dtype=torch.int32, device=DEV).view(1, T, 1)
    w = 1 + 0.1 * torch.randn(d, generator=gen, device=DEV)
    how = {"sections": (d,), "pairing": 1, "layout": 1}
    yq, yk = gla.gla_qk_norm_fwd(q, k, w, w, **how)
    at = slice(T - n, T)
    wq, wk = gla.gla_qk_norm_fwd(q[:, at], k[:, at], w, w, positions=pos[:, at].contiguous(), **how)
    assert torch.equal(yq[:, at], wq) and torch.equal(yk[:, at], wk)
    dq, dk, dqw, _ = gla.gla_qk_norm_bwd(q, k, yq, yk, w, w, grad_dtype=BF16, **how)
    eq, ek, _, _ = gla.gla_qk_norm_bwd(q[:, at], k[:, at], wq, wk, w, w, grad_dtype=BF16, positions=pos[:, at].contiguous(), **how)
    assert torch.equal(dq[:, at], eq) and torch.equal(dk[:, at], ek) and torch.isfinite(dqw).all()


def test_product():
    M, K, F, n = 270000, 64, 8192, 300
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(M, K, generator=gen, device=DEV, dtype=BF16)
    wg, wu = (0.125 * torch.randn(F, K, generator=gen, device=DEV, dtype=BF16) for _ in range(2))
    pre = torch.empty(2, M, F, device=DEV)
    y = gla.gla_glu_fwd(x, wg, wu, pre=pre)
    last = torch.empty(2, n, F, device=DEV)
    want = gla.gla_glu_fwd(x[M - n:], wg, wu, pre=last)
    assert torch.equal(y[M - n:], want) and torch.equal(pre[:, M - n:], last)
    dx, dwg, _ = gla.gla_glu_bwd(x, wg, wu, y, pre=pre)
    ex, _, _ = gla.gla_glu_bwd(x[M - n:], wg, wu, want, pre=last)
    assert float((dx[M - n:].double() - ex.double()).norm() / ex.double().norm()) < 2.0 ** -8
    # the weights' gradient: all rows together are the first ones and the last ones
    a, b = (gla.gla_glu_bwd(x[s], wg, wu, y[s], pre=pre[:, s].contiguous())[1] for s in (slice(0, M // 2), slice(M // 2, M)))
    assert float((dwg.double() - a.double() - b.double()).norm() / dwg.double().norm()) < 2.0 ** -7


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_product_of_many_odd_rows(dtype):
    """Rows whose copies, a thread for each of 256 columns of four rows of three tensors, would be more than 2^32 threads."""
    M, K, F, n = 23_000_000, 9, 8, 200
    gen = torch.Generator(device=DEV).manual_seed(6)
    x = torch.randn(M, K, generator=gen, device=DEV, dtype=dtype)
    wg, wu = (torch.randn(F, K, generator=gen, device=DEV, dtype=dtype) for _ in range(2))
    y = gla.gla_glu_fwd(x, wg, wu)
    for s in (slice(0, n), slice(M // 2, M // 2 + n), slice(M - n, M)):
        assert torch.equal(y[s], gla.gla_glu_fwd(x[s].clone(), wg, wu))
    dx, _, _ = gla.gla_glu_bwd(x, wg, wu, y, want_dw=False)
    tail = gla.gla_glu_bwd(x[-n:].clone(), wg, wu, y[-n:].clone(), want_dw=False)[0]
    assert float((dx[-n:].double() - tail.double()).norm() / tail.double().norm()) < torch.finfo(dtype).eps


@pytest.mark.parametrize("T,D,lens", [(5000, 512, None), (3000, 1024, [3000, 1, 1700])])
def test_waits_that_run_out(T, D, lens):
    """Units whose waits run out at once form the state that enters them from the inputs."""
    B = 1 if lens is None else len(lens)
    gen = torch.Generator(device=DEV).manual_seed(5)
    x, z = (torch.randn(B, T, D, generator=gen, device=DEV) for _ in range(2))
    s = torch.randn(B, D, generator=gen, device=DEV)
    how = {"initial_state": s, "seq_lens": None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)}
    want = gla.gla_recur_fwd(x, z, 1, T, out=torch.zeros_like(x), **how)
    keep = gla.gla_get_option(gla.OPT_LOOK_BACK_POLLS)
    gla.gla_set_option(gla.OPT_LOOK_BACK_POLLS, 0)
    try:
        got = gla.gla_recur_fwd(x, z, 1, T, out=torch.zeros_like(x), **how)
        torch.cuda.synchronize()
    finally:
        gla.gla_set_option(gla.OPT_LOOK_BACK_POLLS, keep)
    for a, b in zip(got, want):
        assert float((a - b).abs().max()) <= 2.0 ** -18 * float(b.abs().max()) * 4
