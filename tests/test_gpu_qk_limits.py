"""Norm of queries and keys without an eps under the root, at numbers of heads that leave lanes of a wave's last turn without a row: rows are not zero, so
all results are finite, and they are held to the formulas and tolerances of test_gpu_qk.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla
from tests import test_gpu_qk as tq

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gla.load_library()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H,Hk", [(1, 1), (3, 1), (6, 4), (16, 5), (17, 16)])
@pytest.mark.parametrize("d", [20, 32, 36, 64, 100, 128, 131, 256])
def test_no_eps(d, H, Hk, dtype, monkeypatch):
    """4, 8, 16 and 32 lanes a row: turns of 16, 8, 4 and 2 heads, the last one of queries, of keys or of both not full."""
    monkeypatch.setattr(tq, "EPS", 0.0)
    w = d // 2 * 2
    tq.check(2, H, Hk, 11, d, dtype, F32, d % 3 == 0, (w,) if d % 8 else (16, w - 16), H % 2, (1, 11), seed=d + H, packed=H > 3)
    tq.check(1, H, Hk, 5, d, dtype, F32, 1, seed=d)


def test_no_eps_of_queries_alone():
    x, dy = (torch.randn(2, 7, 3, 64, device="cuda:0") for _ in range(2))
    w = 1 + 0.1 * torch.randn(64, device="cuda:0")
    dx, _, dw, _ = gla.gla_qk_norm_bwd(x, None, dy, None, w, sections=(64,), eps=0.0)
    near, _, dwn, _ = gla.gla_qk_norm_bwd(x, None, dy, None, w, sections=(64,), eps=1e-12)
    assert torch.isfinite(dx).all() and torch.isfinite(dw).all()
    assert float((dx - near).abs().max()) < 1e-5 and float((dw - dwn).abs().max()) < 1e-4 * np.sqrt(2 * 7 * 3)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [2.0 ** -40, 2.0 ** 40])
def test_no_eps_of_small_and_large_rows(scale, dtype):
    """Squares by a power of two smaller or larger, all of them normal numbers: the same bits, and dx by as much larger or smaller."""
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    x, k, dy, dk = (torch.randn(2, n, 9, 64, generator=gen, device="cuda:0").to(dtype) for n in (6, 2, 6, 2))
    x, k = (torch.where(t.abs() < 2.0 ** -16, 1.0, t).to(dtype) for t in (x, k))
    w, v = 1 + 0.1 * torch.randn(2, 64, generator=gen, device="cuda:0")
    how = {"sections": (64,), "eps": 0.0}
    want, got = (gla.gla_qk_norm_fwd(s * x, s * k, w, v, **how) for s in (1.0, scale))
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.isfinite(got[0]).all()
    want, got = (gla.gla_qk_norm_bwd(s * x, s * k, dy, dk, w, v, **how) for s in (1.0, scale))
    assert all(torch.equal(a * scale, b) for a, b in zip(got[:2], want[:2])) and all(torch.equal(a, b) for a, b in zip(got[2:], want[2:]))
