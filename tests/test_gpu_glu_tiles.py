"""Gated feed-forward product at sizes whose products are cut in every way there is, number by number against the 64-bit formulas (tolerances of test_gpu_glu.py).

By the model of rounds in gla_glu.hip (forward; dx; both weights' gradients), bf16 and fp32:
 520 x 1150 x 4600   128 x 128; 64 x 64 in parts; 256 x 256 and 64 x 64
 512 x 1152 x 4608   the same with whole tiles
 1500 x 1100 x 2100  128 x 128; 64 x 64 in 2 parts and 128 x 128 in 4; 128 x 128, alone and in 3 parts
 2600 x 2300 x 2500  256 x 256; 128 x 128, alone and in 4 parts; 256 x 256 and 64 x 64
 4200 x 2100 x 1050  256 x 192; 256 x 256, alone and in 3 parts; 128 x 128, alone and in 5 parts
 4096 x 4096 x 1024  128 x 128; 256 x 256; 128 x 128, all whole and alone
 1100 x 1152 x 4608  the framework's own width in a small training step"""
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla
from tests import test_gpu_glu as tg

pytestmark = pytest.mark.gpu
SIZES = [(520, 1150, 4600), (512, 1152, 4608), (1500, 1100, 2100), (2600, 2300, 2500), (4200, 2100, 1050), (4096, 4096, 1024), (1100, 1152, 4608)]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gla.load_library()


@pytest.mark.parametrize("kept", [True, False])
@pytest.mark.parametrize("dtype", [tg.BF16, tg.F32])
@pytest.mark.parametrize("M,K,F", SIZES)
def test_every_tile(M, K, F, dtype, kept):
    tg.check(M, K, F, dtype, 0 if kept else 2, seed=M, kept=kept)
