"""States that gla_decay_fwd and gla_decay_bwd give back, by relative 2-norm against the 64-bit recurrence: as exact as fp32 arithmetic from bf16 rows too.

Bound: a chunk of 32 or 64 steps adds to a state up to eight products of which each leaves a rounding of 2^-25 rms or less of what is there, and three bf16
numbers leave 2^-26 of a factor; the decays' exponentials are within 2^-23 of themselves.  A memory of up to eight chunks here makes sqrt(64) * 2^-25 of
the first and sqrt(8) * 2^-23 / sqrt(3) of the last, at random: 2^-21."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla
from oracle import ops_oracle as oo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
BOUND = 2.0 ** -21


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gla.load_library()


def off(got, want):
    return np.linalg.norm(got.double().cpu().numpy() - want) / np.linalg.norm(want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gate", ["head", "token"])
@pytest.mark.parametrize("B,T,dk,dv,lens", [(1, 60, 36, 72, None), (1, 700, 128, 128, None), (2, 1500, 64, 128, [1500, 333]), (3, 300, 7, 65, [0, 300, 1]),
                                            (2, 500, 128, 36, None), (70, 130, 32, 64, None)])
@pytest.mark.parametrize("scan", [0, 1])
def test_states(B, T, dk, dv, lens, gate, dtype, scan):
    gen = torch.Generator().manual_seed(T + scan)
    randn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    H = 4
    q, k, v, do = (randn(B, H, T, w).to(dtype) for w in (dk, dk, dv, dv))
    g = -0.02 * torch.rand(*((H,) if gate == "head" else (B, H, T)), generator=gen) - 0.002
    s0, ds = randn(2, B, H, dk, dv)
    n = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    x = [t.to(DEV) for t in (q, k, v, g)]
    fin = gla.gla_decay_fwd(*x, 1, T, scan, seq_lens=n, initial_state=s0.to(DEV), out_dtype=dtype)[1]
    back = [gla.gla_decay_bwd(*x, do.to(DEV), 1, T, scan, seq_lens=n, d_final_state=ds.to(DEV), grad_dtype=dtype, want_d_initial_state=True,
                              want_d_log_decay=want)[4] for want in (True, False)]
    torch.cuda.synchronize()
    want, adjoint = np.zeros(s0.shape), np.zeros(s0.shape)
    a = (g[None, :, None].expand(B, H, T) if gate == "head" else g).double().numpy()
    for b in range(B):
        at = oo.visits(T, 1, T, scan, T if lens is None else lens[b])
        S = s0[b].double().numpy()
        for t in at:
            S = np.exp(a[b][:, t])[:, None, None] * S + k[b, :, t, :, None].double().numpy() * v[b, :, t, None, :].double().numpy()
        want[b] = S
        G = ds[b].double().numpy()
        for t in at[::-1]:
            G = np.exp(a[b][:, t])[:, None, None] * (G + q[b, :, t, :, None].double().numpy() * do[b, :, t, None, :].double().numpy())
        adjoint[b] = G
    assert off(fin, want) <= BOUND, off(fin, want)
    for t in back:
        assert off(t, adjoint) <= BOUND, off(t, adjoint)


def test_states_of_many_pieces():
    """A state handed on from call to call holds what one call gives."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    q, k, v = (torch.randn(1, 4, 4096, 128, generator=gen, device=DEV).to(BF16) for _ in range(3))
    g = torch.full((4,), -0.003, device=DEV)
    whole = gla.gla_decay_fwd(q, k, v, g, 1, 4096)[1].double().cpu().numpy()
    s = torch.zeros(1, 4, 128, 128, device=DEV)
    for t in range(0, 4096, 100):
        x = [y[:, :, t:t + 100].contiguous() for y in (q, k, v)]
        gla.gla_decay_fwd(*x, g, 1, x[0].shape[2], initial_state=s, final_state=s)
    assert off(s, whole) <= 2 * BOUND, off(s, whole)
