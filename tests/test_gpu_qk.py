"""Norm and rotation of queries and keys (gla_qk_norm_fwd / gla_qk_norm_bwd) against the 64-bit formulas.

Tolerances.  A row's sum of at most 256 squares goes through 8 products of a lane and 5 steps over lanes: within 16 * 2^-24 of itself, its
root within 2^-20; with the reciprocal root, the weight and the rotation's four roundings every factor of an output is within 2^-19.  Angles are
reduced in 64 bits, sines and cosines within 2^-22 of one.  A turned value is compared with the sum of its two products' absolute values.
dx = r (dn - n mean(dn n)): 2^-18 of r (|dn| + |n| mean |dn n|).  A weight's gradient is a sum over rows that a lane adds one after the other,
64 of a work-group and up to 1024 partial sums: off by (rows / groups + 64 + 32) 2^-24 and 2^-18 of each addend, below 2^-13 of the sum of absolute
values for the rows here.  Results of 16 bits are rounded once, 2^-8."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla
from oracle import block_oracle as bo
from oracle import ops_oracle as oo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
ROUND = {F32: 2.0 ** -23, BF16: 2.0 ** -8}
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gla.load_library()


def close(got, want, size, tol, rounding, name):
    bad = np.abs(got - want) - (tol * size + rounding * np.abs(want) + 1e-30)
    assert np.isfinite(got).all() and bad.max() <= 0, (name, float(bad.max()), np.unravel_index(bad.argmax(), bad.shape))


def spread(x, positions, sections, adjacent):
    """The sum of the absolute values of a turned value's products."""
    y, at = np.abs(x).copy(), 0
    for w in sections:
        for i in range(w // 2):
            c0, c1 = (at + 2 * i, at + 2 * i + 1) if adjacent else (at + i, at + i + w // 2)
            y[..., c0] = y[..., c1] = np.abs(x[..., c0]) + np.abs(x[..., c1])
        at += w
    return y


def check(B, H, Hk, T, d, dtype, out_dtype, layout, sections=(), pairing=0, grid=(0, 0), given=False, packed=False, affine=True, seed=0, far=False):
    gen = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    turn = lambda x: x.transpose(1, 2) if layout == 0 else x  # noqa: E731
    shape = lambda n: (B, n, T, d) if layout == 0 else (B, T, n, d)  # noqa: E731
    if packed:
        rows = (1.5 * randn(B, T, (H + 2 * Hk) * d + 3)).to(dtype).to(DEV)[..., 1:]
        q, k = turn(rows[..., :H * d].unflatten(-1, (H, d))), turn(rows[..., H * d:(H + Hk) * d].unflatten(-1, (Hk, d)))
    else:
        q, k = (1.5 * randn(*shape(H))).to(dtype).to(DEV), (1.5 * randn(*shape(Hk))).to(dtype).to(DEV)
    qw, kw = (1 + 0.3 * randn(d), 1 + 0.3 * randn(d)) if affine else (None, None)
    put = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    axes = len(sections)
    if given:
        lim = 2 ** 31 - 1 if far else 40000
        pos = torch.randint(-lim, lim, (B, T, axes), generator=gen, dtype=torch.int32)
    elif axes:
        n = np.arange(T)
        cell = n % (grid[0] * grid[1]) if axes > 1 else n
        p = [n] if axes == 1 else [cell // grid[1], cell % grid[1]] if axes == 2 else [n // (grid[0] * grid[1]), cell // grid[1], cell % grid[1]]
        pos = torch.from_numpy(np.stack(p, -1))[None].expand(B, T, axes)
    else:
        pos = torch.zeros(B, T, 0)
    dqo, dko = randn(*shape(H)).to(dtype), randn(*shape(Hk)).to(dtype)
    how = {"sections": sections, "eps": EPS, "grid_h": grid[0], "grid_w": grid[1], "positions": put(pos.contiguous()) if given else None, "pairing": pairing,
           "layout": layout}
    yq, yk = gla.gla_qk_norm_fwd(q, k, put(qw), put(kw), out_dtype=out_dtype, **how)
    dq, dk, dqw, dkw = gla.gla_qk_norm_bwd(q, k, put(dqo), put(dko), put(qw), put(kw), grad_dtype=out_dtype, **how)
    torch.cuda.synchronize()
    num = lambda t: t.double().cpu().numpy()  # noqa: E731
    rows = lambda t: num(t if layout == 0 else t.transpose(1, 2))  # noqa: E731
    adjacent, P = pairing == 0, pos.double().numpy()
    for name, x, w, y, dy, dx, dw in (("q", q, qw, yq, dqo, dq, dqw), ("k", k, kw, yk, dko, dk, dkw)):
        X, W, DY = rows(x), np.ones(d) if w is None else num(w), rows(dy)
        n, r = bo.rms_fwd(X, W, EPS)
        close(rows(y), oo.rope(n, P, sections, 10000.0, adjacent, False), spread(n, P, sections, adjacent), 2.0 ** -19, ROUND[out_dtype], name)
        back = oo.rope(DY, P, sections, 10000.0, adjacent, True)
        wx, ww = bo.rms_bwd(X, W, EPS, back)
        size = spread(DY, P, sections, adjacent)
        dn = size * np.abs(W)
        nn = np.abs(X) * r
        close(rows(dx), wx, r * (dn + nn * (dn * nn).mean(-1, keepdims=True)), 2.0 ** -18, ROUND[out_dtype], "d" + name)
        if w is not None:
            close(num(dw), ww, (size * nn).reshape(-1, d).sum(0), 2.0 ** -13, ROUND[F32], name + " weight")
        else:
            assert dw is None


@pytest.mark.parametrize("dtype,out_dtype", [(BF16, BF16), (F32, F32), (BF16, F32)])
@pytest.mark.parametrize("d", [1, 2, 5, 8, 31, 32, 33, 36, 64, 65, 72, 127, 128, 129, 200, 255, 256])
def test_widths(d, dtype, out_dtype):
    check(2, 3, 2, 9, d, dtype, out_dtype, d % 2, seed=d)
    if d > 1:
        w = d // 2 * 2
        check(2, 2, 1, 7, d, dtype, out_dtype, 1, (w,), d % 3 == 0, seed=d, packed=True)
        check(1, 2, 2, 7, d, dtype, out_dtype, 0, (w,), d % 3 != 0, seed=d + 1)


@pytest.mark.parametrize("pairing", [0, 1])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("sections,d,grid,T", [((32, 32), 64, (3, 5), 15), ((16, 56, 56), 128, (2, 3), 18), ((2, 6), 9, (4, 4), 16), ((10, 22), 40, (3, 3), 9),
                                                ((64,), 128, (0, 0), 21), ((128,), 256, (0, 0), 5), ((4, 4, 4), 12, (2, 2), 8)])
def test_sections(sections, d, grid, T, layout, pairing):
    check(2, 4, 2, T, d, BF16, F32, layout, sections, pairing, grid, packed=True, seed=T)
    check(1, 3, 3, T, d, F32, F32, layout, sections, pairing, grid, given=True, affine=False, seed=T + 1)


@pytest.mark.parametrize("B,H,Hk,T", [(1, 1, 1, 1), (64, 16, 4, 1), (1, 40, 1, 3), (3, 7, 5, 50), (2, 16, 16, 1000), (1, 2, 1, 40000)])
def test_rows(B, H, Hk, T):
    check(B, H, Hk, T, 16 if T > 2000 else 64, BF16, F32, 1, (16,), 1, packed=True, seed=H)
    check(B, H, Hk, T, 36, BF16, BF16, 0, (12, 24), 0, given=True, seed=H + 1) if T < 2000 else None


def test_far_positions():
    """The last positions are turned as exactly as the first."""
    check(2, 2, 2, 33, 64, F32, F32, 0, (64,), 1, given=True, far=True)
    check(2, 2, 2, 33, 128, F32, F32, 1, (32, 48, 48), 0, given=True, far=True)


def test_queries_alone_rows_of_zeros_and_eps():
    x = torch.randn(2, 3, 5, 24, device=DEV)
    w = torch.rand(24, device=DEV)
    y, none = gla.gla_qk_norm_fwd(x, None, w, sections=(24,))
    both, _ = gla.gla_qk_norm_fwd(x, x[:, :1], w, sections=(24,))
    assert none is None and torch.equal(y, both)
    dx, dk, dw, dkw = gla.gla_qk_norm_bwd(x, None, x, None, w, sections=(24,))
    assert dk is None and dkw is None and torch.isfinite(dx).all() and torch.isfinite(dw).all()
    assert gla.gla_qk_norm_bwd(x, None, x, None, w, sections=(24,), want_d_weight=False)[2] is None
    z = torch.zeros_like(x)
    assert (gla.gla_qk_norm_fwd(z, None, w)[0] == 0).all() and torch.isfinite(gla.gla_qk_norm_bwd(z, None, x, None, w)[0]).all()
    big = gla.gla_qk_norm_fwd(x, None, eps=100.0)[0]
    want = x / (x.double().square().mean(-1, keepdim=True) + 100.0).sqrt()
    assert float((big - want).abs().max()) < 1e-6


def test_a_nan_stays_in_its_row():
    x = torch.randn(1, 2, 6, 128, device=DEV)
    want, _ = gla.gla_qk_norm_fwd(x, None, sections=(128,), pairing=1)
    x[0, 1, 3, 70] = float("nan")
    y, _ = gla.gla_qk_norm_fwd(x, None, sections=(128,), pairing=1)
    assert torch.isnan(y[0, 1, 3]).all()
    keep = torch.ones(2, 6, dtype=torch.bool)
    keep[1, 3] = False
    assert torch.equal(y[0][keep], want[0][keep])


def test_in_place_broadcast_rows_graph_and_streams():
    B, H, Hk, T, d = 2, 4, 2, 37, 64
    gen = torch.Generator(device=DEV).manual_seed(1)
    q, k = torch.randn(B, T, H, d, generator=gen, device=DEV).to(BF16), torch.randn(B, T, Hk, d, generator=gen, device=DEV).to(BF16)
    w, v = 1 + 0.1 * torch.randn(2, d, generator=gen, device=DEV)
    how = {"sections": (64,), "pairing": 1, "layout": 1}
    y = gla.gla_qk_norm_fwd(q, k, w, v, **how)
    a, b = q.clone(), k.clone()
    z = gla.gla_qk_norm_fwd(a, b, w, v, out_q=a, out_k=b, **how)
    assert z[0] is a and torch.equal(a, y[0]) and torch.equal(b, y[1])
    # one row for all tokens
    same = q[:, :1].expand(B, T, H, d)
    assert torch.equal(gla.gla_qk_norm_fwd(same, None, w, **how)[0], gla.gla_qk_norm_fwd(same.contiguous(), None, w, **how)[0])
    back = gla.gla_qk_norm_bwd(q, k, y[0], y[1], w, v, **how)
    ws = torch.empty(gla.gla_qk_norm_bwd_workspace_bytes(B, H, Hk, T, d), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = [*gla.gla_qk_norm_fwd(q, k, w, v, **how)]
        held += [*gla.gla_qk_norm_bwd(q, k, y[0], y[1], w, v, workspace=ws, **how)]
    for _ in range(3):
        for t in held:
            t.fill_(3.0)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, (*y, *back)))
        gla.gla_qk_norm_bwd(q, k, q, k, v, w, workspace=ws, **how)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [gla.gla_qk_norm_bwd(q, k, y[0], y[1], w, v, stream=s, **how) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for got in outs for a, b in zip(got, back))


def test_refusals():
    q, k = torch.zeros(2, 3, 4, 8, device=DEV), torch.zeros(2, 1, 4, 8, device=DEV)
    w = torch.ones(8, device=DEV)
    for bad in ({"q_weight": w[:4]}, {"q_weight": w.to(BF16)}, {"layout": 2}, {"layout": 1}, {"out_q": q[:1]}, {"out_q": q, "out_k": k.to(BF16)},
                {"positions": torch.zeros(2, 4, 2, dtype=torch.int32, device=DEV), "sections": (8,)}, {"k": k.to(BF16)}, {"k": k.transpose(2, 3)},
                {"k": None, "out_k": k}, {"k": None, "k_weight": w}, {"q": q.cpu()}, {"k": torch.zeros(2, 1, 5, 8, device=DEV)}):
        with pytest.raises((ValueError, TypeError)):
            gla.gla_qk_norm_fwd(**{"q": q, "k": k, **bad})
    for bad in ({"eps": -1.0}, {"eps": float("nan")}, {"sections": (7,)}, {"sections": (6, 4)}, {"sections": (4, 4), "grid_h": 3, "grid_w": 2}, {"sections": (8,), "base": 0.0},
                {"sections": (8,), "pairing": 2}, {"sections": (2, 2, 2, 2)}):
        with pytest.raises(gla.GlaError):
            gla.gla_qk_norm_fwd(q, k, **bad)
    rows = torch.zeros(2, 4, 5 * 8, device=DEV)
    a = rows[..., :24].unflatten(-1, (3, 8)).transpose(1, 2)
    for bad in (rows.flatten()[:192].view(2, 3, 4, 8), rows.flatten()[8:200].view(2, 3, 4, 8)):
        with pytest.raises(gla.GlaError):
            gla.gla_qk_norm_fwd(a, None, out_q=bad)
    with pytest.raises(gla.GlaError):
        gla.gla_qk_norm_fwd(q, k, out_q=torch.empty_like(q), out_k=q[0, 0].view(1, 1, 4, 8).expand(2, 1, 4, 8).contiguous().set_(q.untyped_storage(), 0, (2, 1, 4, 8)))
    with pytest.raises(gla.GlaError):
        gla.gla_qk_norm_fwd(torch.zeros(1, 1, 1, 257, device=DEV), None)
    with pytest.raises(gla.GlaError):
        gla.gla_qk_norm_bwd(q, k, q, k, w, w, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        gla.gla_qk_norm_bwd(q, k, q, None, w, w)
