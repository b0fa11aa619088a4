"""Layer norm at the largest sizes that gla_norm_fwd / gla_norm_bwd take."""
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


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("H,D", [(16384, 4096), (16400, 4097)])
def test_weights_of_2_to_the_26(H, D, layout):
    """Sums for as many weights as a launch with 64 threads for each does not take.  Two rows a head: dweight and dbias are sums of two products, each
    off by 2^-15 of its size (the factors' 2^-16 of test_gpu_norm.py, of n and of the sum)."""
    gen = torch.Generator(device=DEV).manual_seed(H)
    lead = (1, H, 2) if layout == 0 else (1, 2, H)
    x, do = (torch.randn(*lead, D, generator=gen, device=DEV, dtype=F32).to(BF16) for _ in range(2))
    w = 1 + 0.3 * torch.randn(H, D, generator=gen, device=DEV)
    dx, _, dw, db = gla.gla_norm_bwd(x, do, w, None, layout=layout, grad_dtype=BF16)
    torch.cuda.synchronize()
    heads = torch.tensor([0, 1, H // 2, H - 2, H - 1], device=DEV)
    rows = lambda t: (t.transpose(1, 2) if layout == 0 else t)[:, :, heads].double().cpu().numpy()  # noqa: E731
    W = w[heads].double().cpu().numpy()
    X, DO = rows(x), rows(do)
    _, n, rstd = oo.norm_fwd(X, W, np.zeros_like(W), 1e-5)
    wx, _, ww, wb = oo.norm_bwd(X, W, np.zeros_like(W), 1e-5, DO)
    one = 1 + np.abs(n)
    dn = np.abs(DO * W)
    size = rstd * (dn + dn.mean(-1, keepdims=True) + one * (dn * one).mean(-1, keepdims=True))
    for got, want, bound in ((rows(dx), wx, 2.0 ** -15 * size + 2.0 ** -8 * np.abs(wx)),
                             (dw[heads].double().cpu().numpy(), ww, 2.0 ** -15 * (np.abs(DO) * one).sum((0, 1))),
                             (db[heads].double().cpu().numpy(), wb, 2.0 ** -15 * np.abs(DO).sum((0, 1)))):
        assert (np.abs(got - want) <= bound).all()
    assert torch.isfinite(dw).all() and torch.isfinite(db).all()
