"""Backward walks, rotation and norm of tensors with more than 2^31 elements and past what the walks' views with 32-bit offsets reach, sums over many rows,
and calls without the gates' gradient.

The bounds of the recurrence are those of test_gpu_decay.py: 2^-15 (bf16 rows; three splits of 2^-17 and the sums) and 2^-16 (fp32) of the sums over
absolute values, and the rounding of the result."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla
from oracle import ops_oracle as oo

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


def close(got, want, size, tol, rounding):
    bad = np.abs(host(got) - want) - (tol * size + rounding * np.abs(want) + 1e-30)
    assert bad.max() <= 0, float(bad.max())


def check_last_head(T, H, d, dtype, n, gh, gw, scan):
    """Gradients in token order of a call in which only the last n tokens of the last head are not zero."""
    gen = torch.Generator(device=DEV).manual_seed(T)
    q, k, v, do = (torch.zeros(1, T, H, d, dtype=dtype, device=DEV) for _ in range(4))
    for t in (q, k, v, do):
        t[0, T - n:, H - 1] = (0.3 * torch.randn(n, d, generator=gen, device=DEV)).to(dtype)
    g = torch.full((H,), -0.1, device=DEV)
    dq, dk, dv, dg, _ = gla.gla_decay_bwd(q, k, v, g, do, gh, gw, scan, 1, grad_dtype=dtype)
    torch.cuda.synchronize()
    at = oo.visits(T, gh, gw, scan)
    at = at[at >= T - n]
    rows = [host(t[0, :, H - 1][torch.from_numpy(at.copy()).to(DEV)])[None] for t in (q, k, v, do)]
    a, zero = np.full((1, n), float(g[0])), np.zeros((1, d, d))
    if scan >= 2:
        assert n == T                                        # (else other steps would lie between these)
    want = oo.decay_bwd(*rows[:3], a, oo.decay_fwd(*rows[:3], a, zero)[1], rows[3], zero)
    size = [np.abs(x) for x in rows]
    size = oo.decay_bwd(*size[:3], a, oo.decay_fwd(*size[:3], a, zero)[1], size[3], zero)
    tol, rounding = (2.0 ** -15, 2.0 ** -8) if dtype is BF16 else (2.0 ** -16, 2.0 ** -23)
    for got, w, s in zip((dq, dk, dv), want, size):
        close(got[0, :, H - 1][torch.from_numpy(at.copy()).to(DEV)][None], w, s, tol, rounding)
        assert not got[0, :T - n].any() and not got[0, :, :H - 1].any()
    # 2^-14 of one head's gradient: the bound of test_gpu_decay_gates.py for short memories
    assert abs(float(dg[H - 1]) - want[3].sum()) <= 2.0 ** -14 * np.linalg.norm(want[3]) * n ** 0.5 and not dg[:H - 1].any()


def test_backward_behind_2_to_the_31_elements():
    check_last_head(131072 + 40, 130, 128, BF16, 40, 1, 131072 + 40, 0)


@pytest.mark.parametrize("scan", [0, 1])
def test_backward_of_many_heads_in_token_order(scan):
    """Tokens farther apart than the views' factors of 24 bits."""
    check_last_head(70, 66000, 64, F32, 70, 1, 70, scan)


@pytest.mark.parametrize("scan", [2, 3])
@pytest.mark.parametrize("H,gh,gw", [(3000, 40, 50), (3000, 50, 60)])
def test_backward_of_large_grids_in_columns(H, gh, gw, scan):
    """Below and past 2^31 bytes from a sequence's first row to its last."""
    check_last_head(gh * gw, H, 64, F32, gh * gw, gh, gw, scan)


@pytest.mark.parametrize("layout", [0, 1])
def test_rotation_behind_2_to_the_31_elements(layout):
    T, H, d = 131072 + 40, 130, 128
    x = torch.zeros(1, *((H, T) if layout == 0 else (T, H)), d, dtype=BF16, device=DEV)
    rows = x[0, H - 1, -8:] if layout == 0 else x[0, -8:, H - 1]
    rows.copy_(torch.randn(8, d, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV))
    X = host(rows)[None, None]
    y, _ = gla.gla_rope(x, None, (64,), layout=layout)
    torch.cuda.synchronize()
    want = oo.rope(X, np.arange(T - 8, T)[None, :, None], (64,), 10000.0, True, False)[0, 0]
    got = y[0, H - 1, -8:] if layout == 0 else y[0, -8:, H - 1]
    close(got, want, np.abs(X).max(), 2.0 ** -20, 2.0 ** -8)         # (2^-21 of a pair's length, test_gpu_rope.py)
    got.zero_()
    assert not y.any()


@pytest.mark.parametrize("layout,H,T,D", [(0, 1, 270000, 8192), (0, 17, 1000000, 128), (1, 17, 1000000, 128), (1, 6, 5000000, 72)])
def test_norm_behind_2_to_the_31_elements(layout, H, T, D):
    """Rows of zeros but for the last of the last head; their gradient is zero, and so is their part of the weights'."""
    x, do, r = (torch.zeros(1, *((H, T) if layout == 0 else (T, H)), D, dtype=BF16, device=DEV) for _ in range(3))
    last = (lambda t: t[0, H - 1, -8:]) if layout == 0 else (lambda t: t[0, -8:, H - 1])  # noqa: E731
    gen = torch.Generator(device=DEV).manual_seed(2)
    for t in (x, do, r):
        last(t).copy_(torch.randn(8, D, generator=gen, device=DEV))
    w = torch.ones(H, D, device=DEV)
    y = gla.gla_norm_fwd(x, w, r_pre=r, layout=layout)
    dx, dr, dw, db = gla.gla_norm_bwd(x, do, w, r_pre=r, layout=layout, grad_dtype=BF16)
    torch.cuda.synchronize()
    X, DO, R = (host(last(t))[:, None] for t in (x, do, r))
    one, nil = np.ones((1, D)), np.zeros((1, D))
    wy, n, rstd = oo.norm_fwd(X, one, nil, 1e-5, R)
    wx, wr, ww, wb = oo.norm_bwd(X, one, nil, 1e-5, DO, R)
    size = np.abs(DO) * (np.abs(R) + 0.01)
    m = 1 + np.abs(n)
    # the sizes and 2^-15 of test_gpu_norm.py; sums of eight rows
    for got, want, s in ((y, wy, m * (np.abs(R) + 0.01)), (dx, wx, rstd * (size + size.mean(-1, keepdims=True) + m * (size * m).mean(-1, keepdims=True))),
                         (dr, wr, np.abs(DO) * m * 2)):
        close(last(got)[:, None], want, s, 2.0 ** -15, 2.0 ** -8)
        last(got).zero_()
        assert not got.any()
    close(dw[H - 1:], ww, (size * m).sum(0), 2.0 ** -15, 2.0 ** -23)
    close(db[H - 1:], wb, size.sum(0), 2.0 ** -15, 2.0 ** -23)
    assert not dw[:H - 1].any() and not db[:H - 1].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("H,T,D", [(1, 100000, 1152), (16, 30000, 72), (3, 50000, 20), (1, 20000, 4096)])
def test_sums_over_many_rows(H, T, D, gated, layout, dtype):
    """dweight and dbias by relative 2-norm.  Every term is off by some 2^-21 at most (n and the gate by an exponential, a reciprocal and a root of a few units of
    2^-24), at random, and so is their sum of its 2-norm; a group adds up to T / 256 of them in turn and the rest in trees: sqrt(400) / 2 * 2^-24 of what is
    there by then: below 2^-20.  2^-19 in all."""
    gen = torch.Generator(device=DEV).manual_seed(T)
    lead = (1, H, T) if layout == 0 else (1, T, H)
    randn = lambda *s: torch.randn(*s, generator=gen, device=DEV)  # noqa: E731
    x, do, r = ((randn(*lead, D) + 0.5).to(dtype), randn(*lead, D).to(dtype), randn(*lead, D).to(dtype))
    w, b = 1 + 0.3 * randn(H, D), 0.3 * randn(H, D)
    _, _, dw, db = gla.gla_norm_bwd(x, do, w, b, r_pre=r if gated else None, layout=layout)
    torch.cuda.synchronize()
    ww, wb = np.zeros((H, D)), np.zeros((H, D))
    for h in range(H):
        for t0 in range(0, T, 10000):
            X, DO, R = (host((t[0, h, t0:t0 + 10000] if layout == 0 else t[0, t0:t0 + 10000, h])) for t in (x, do, r))
            n = (X - X.mean(-1, keepdims=True)) / np.sqrt(X.var(-1, keepdims=True) + 1e-5)
            dy = DO * R / (1 + np.exp(-R)) if gated else DO
            ww[h] += (dy * n).sum(0)
            wb[h] += dy.sum(0)
    for got, want in ((dw, ww), (db, wb)):
        off = np.linalg.norm(host(got) - want) / np.linalg.norm(want)
        assert off <= 2.0 ** -19, off


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gate", ["head", "token"])
@pytest.mark.parametrize("dk,dv", [(36, 72), (128, 128), (7, 65)])
def test_without_the_gates_gradient(dk, dv, gate, dtype):
    gen = torch.Generator(device=DEV).manual_seed(dk)
    randn = lambda *s: torch.randn(*s, generator=gen, device=DEV)  # noqa: E731
    n, T = 3, 400
    q, k, v, do = ((randn(2, n, T, w) * 0.3).to(dtype) for w in (dk, dk, dv, dv))
    g = -0.1 * torch.rand(*((n,) if gate == "head" else (2, n, T)), generator=gen, device=DEV)
    s0, ds = randn(2, n, dk, dv), randn(2, n, dk, dv)
    got = gla.gla_decay_bwd(q, k, v, g, do, 20, 20, 2, initial_state=s0, d_final_state=ds, want_d_log_decay=False, want_d_initial_state=True)
    assert got[3] is None
    a = host(g[None, :, None].expand(2, n, T) if gate == "head" else g)
    at = oo.visits(T, 20, 20, 2)
    for b in range(2):
        rows = [host(t[b])[:, at] for t in (q, k, v, do)]
        ab = [np.abs(t) for t in rows]
        want = oo.decay_bwd(*rows[:3], a[b][:, at], oo.decay_fwd(*rows[:3], a[b][:, at], host(s0[b]))[1], rows[3], host(ds[b]))
        size = oo.decay_bwd(*ab[:3], a[b][:, at], oo.decay_fwd(*ab[:3], a[b][:, at], np.abs(host(s0[b])))[1], ab[3], np.abs(host(ds[b])))
        tol = 2.0 ** -15 if dtype is BF16 else 2.0 ** -16
        for i in (0, 1, 2):
            close(got[i][b][:, torch.from_numpy(at.copy()).to(DEV)], want[i], size[i], tol, 2.0 ** -23)
        close(got[4][b], want[4], size[4], tol, 2.0 ** -23)
