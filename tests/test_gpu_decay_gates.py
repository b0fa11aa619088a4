"""Gates of gla_decay_fwd / _bwd and their gradient against the 64-bit recurrence."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gla.load_library()


@pytest.mark.parametrize("gate", [-0.2, -0.3, -0.34, -0.5])
def test_weights_of_a_chunk(gate):
    """One key a head, at another step each: outputs are the weights exp(b_i - b_j) of a chunk of 32 steps by themselves.  Weights are below one: up to
    two exponentials of one unit of 2^-24 and their product, 2.5 * 2^-24; their argument b, off by |b| (2^-24 + 2^-25 + 2^-26) (the
    gate's product with log2 e, that constant, the sum), changes exp(-|b|) by less than 0.7 * 2^-24; sums of rests 2^-25: 4 * 2^-24 in all."""
    n = 32
    one = torch.ones(1, n, n, 1, device=DEV)
    k = torch.eye(n, device=DEV).view(1, n, n, 1).contiguous()
    out, _ = gla.gla_decay_fwd(one, k, one, torch.full((n,), gate, device=DEV), 1, n)
    i, j = np.arange(n)[None, :], np.arange(n)[:, None]
    want = np.where(i >= j, np.exp(float(np.float32(gate)) * (i - j)), 0.0)
    worst = np.abs(out.double().cpu().numpy()[0, :, :, 0] - want).max() * 2.0 ** 24
    assert worst <= 4, worst
