"""Gated recurrence of channels near the largest launches: very many sequences, and one of very many steps."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla
from tests import test_gpu_block_far as far

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gla.load_library()


@pytest.mark.parametrize("B,T,D", [((1 << 22) + 5, 3, 1), ((1 << 22) - 1, 65, 1), ((1 << 21) - 1, 66, 2)])
def test_many_sequences(B, T, D):
    """Sequences are walked by themselves: some of the first, the middle and the last have the bits that a call on them alone gives (of as many steps: the waves
    and rounds are the same)."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, z, do = (torch.randn(B, T, D, generator=gen, device=DEV) for _ in range(3))
    s, df = (torch.randn(B, D, generator=gen, device=DEV) for _ in range(2))
    y, fin = gla.gla_recur_fwd(x, z, 1, T, initial_state=s, complement=True)
    back = gla.gla_recur_bwd(x, z, do, 1, T, initial_state=s, d_final_state=df, complement=True, want_d_initial_state=True)
    for at in (slice(0, 100), slice(B // 2, B // 2 + 100), slice(B - 100, B)):
        a, b, c, d, e = (t[at].clone() for t in (x, z, do, s, df))
        w, wf = gla.gla_recur_fwd(a, b, 1, T, initial_state=d, complement=True)
        want = gla.gla_recur_bwd(a, b, c, 1, T, initial_state=d, d_final_state=e, complement=True, want_d_initial_state=True)
        assert torch.equal(y[at], w) and torch.equal(fin[at], wf)
        assert all(torch.equal(g[at], h) for g, h in zip(back, want))
    # step by step in 64 bits, all sequences: memories of at most 66 steps, sums of as many terms below 6 each
    a = torch.nn.functional.logsigmoid(z.double()) / 16
    h, most = s.double(), 0.0
    for t in range(T):
        h = torch.exp(a[:, t]) * h - torch.expm1(a[:, t]) * x[:, t].double()
        most = max(most, float((y[:, t].double() - h).abs().max()))
    assert most <= (2.0 ** -19 + T * 2.0 ** -26) * 6 * 3, most
    assert np.isfinite(float(back[0].sum()) + float(back[1].sum()) + float(back[2].sum()))


def test_many_steps():
    """2^21 units forward, 2^22 rounds backward."""
    far.test_recurrence(1, (1 << 28) + 77, 1)
