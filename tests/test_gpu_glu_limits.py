"""Activations of the gated feed-forward product at the largest fp32 products."""
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gla.load_library()


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("act", [0, 1, 2])
def test_slopes_up_to_the_largest_products(act, kept):
    """The activation is g or nothing there, and its slope one or nothing: products of one element each, gradients without a rounding."""
    g = [1.5e35, 2e35, 1e37, 3e38, -1.5e35, -2e35, -1e37, -3e38]
    x = torch.tensor([[1.0, 0, 0, 0]], device=DEV)
    wg, wu = (torch.zeros(8, 4, device=DEV) for _ in range(2))
    wg[:, 0], wu[:, 0] = torch.tensor(g, device=DEV), 1.0
    pre = torch.empty(2, 1, 8, device=DEV) if kept else None
    y = gla.gla_glu_fwd(x, wg, wu, act, pre=pre)
    assert torch.equal(y, wg[:, 0].clamp(min=0)[None])
    for i in range(8):
        do = torch.zeros(1, 8, device=DEV)
        do[0, i] = 1.0
        dx, dwg, dwu = gla.gla_glu_bwd(x, wg, wu, do, act, pre=pre)
        assert float(dwg[i, 0]) == (1.0 if i < 4 else 0.0) and float(dwu[i, 0]) == float(y[0, i]), (i, dwg[i, 0], dwu[i, 0])
        if i >= 4:
            assert not dx.any(), (i, dx)


@pytest.mark.parametrize("act", [0, 1, 2])
def test_a_nan_product_has_a_nan_slope(act):
    x = torch.tensor([[float("nan")]], device=DEV)
    w = torch.ones(1, 1, device=DEV)
    dx, dwg, dwu = gla.gla_glu_bwd(x, w, w, w, act)
    assert torch.isnan(dx).all() and torch.isnan(dwg).all() and torch.isnan(dwu).all()
    pre = torch.tensor([[[float("nan")]], [[1.0]]], device=DEV)
    _, dwg, dwu = gla.gla_glu_bwd(w, w, w, w, act, pre=pre)
    assert torch.isnan(dwg).all() and torch.isnan(dwu).all()
