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
