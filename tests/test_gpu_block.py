"""The operators as a block uses them.  A mixer's block: slices of a packed projection normed and turned, the recurrence with one decay a head, layer norm of
each head, the gated feed-forward product of the tokens; forward and backward.  A recurrent block: the gated recurrence of channels and the product;
forward, backward, and a padded batch's prompts followed by single tokens.

Forward tolerance: the operators hold 2^-15 of sums of absolute values each or better (their own tests), which for the at most 64 channels and the
memory of some ten tokens here are at most 16 times an output's own size: 4 * 16 * 2^-15 = 2e-3 of the outputs' rms.  The gradients
are held to the 64-bit chain's central differences along random directions, off by at most that share of |gradient| |direction|."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla
from oracle import block_oracle as bo
from oracle import ops_oracle as oo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SHARE = 4 * 16 * 2.0 ** -15
B, T, H, DK, F, TAU, EPS = 2, 150, 3, 32, 80, 4.0, 1e-5
D = H * DK


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gla.load_library()


def inputs(seed):
    rng = np.random.default_rng(seed)
    n = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
    scale = np.float32(D ** -0.5)
    mixer = {"rows": n(B, T, 3 * D), "qw": 1 + np.float32(0.2) * n(DK), "kw": 1 + np.float32(0.2) * n(DK), "g": -0.1 - np.abs(n(H)) * np.float32(0.1),
             "w": 1 + np.float32(0.2) * n(H, DK), "b": np.float32(0.2) * n(H, DK), "wg": n(F, D) * scale, "wu": n(F, D) * scale}
    channels = {"x": n(B, T, D), "z": 1 + n(B, T, D), "s": n(B, D), "wg": n(F, D) * scale, "wu": n(F, D) * scale}
    return mixer, channels, n(B, T, F)


def mixer_reference(p):
    q, k, v = (p["rows"][..., i * D:(i + 1) * D].reshape(B, T, H, DK).transpose(0, 2, 1, 3) for i in range(3))
    pos = np.arange(T)[None, :, None].repeat(B, 0)
    q, k = (oo.rope(bo.rms_fwd(x, p[w], EPS)[0], pos, (DK,), 10000.0, False, False) for x, w in ((q, "qw"), (k, "kw")))
    flat = lambda x: x.reshape(B * H, T, DK)  # noqa: E731
    g = np.broadcast_to(p["g"][None, :, None], (B, H, T)).reshape(B * H, T)
    o = oo.decay_fwd(flat(q) * DK ** -0.5, flat(k), flat(v), g, np.zeros((B * H, DK, DK)))[0].reshape(B, H, T, DK).transpose(0, 2, 1, 3)
    y = oo.norm_fwd(o, p["w"], p["b"], EPS)[0].reshape(B * T, D)
    return bo.glu_fwd(y, p["wg"], p["wu"], "silu").reshape(B, T, F)


QK = {"sections": (DK,), "eps": EPS, "pairing": gla.ROPE_HALVES, "layout": gla.LAYOUT_BTHD}


def mixer(t, dy=None):
    """Outputs, and the gradients of sum(outputs * dy)."""
    q, k, v = (t["rows"][..., i * D:(i + 1) * D].unflatten(-1, (H, DK)) for i in range(3))
    v = v.contiguous()
    qw = t["qw"] * DK ** -0.5            # (the scores' scale in the weight)
    qn, kn = gla.gla_qk_norm_fwd(q, k, qw, t["kw"], **QK)
    o, _ = gla.gla_decay_fwd(qn, kn, v, t["g"], 1, T, layout=1)
    n = gla.gla_norm_fwd(o, t["w"], t["b"], EPS, layout=1)
    tokens = n.view(B, T, D)
    pre = torch.empty(2, B, T, F, device=DEV)
    y = gla.gla_glu_fwd(tokens, t["wg"], t["wu"], pre=pre)
    if dy is None:
        return y
    dn, dwg, dwu = gla.gla_glu_bwd(tokens, t["wg"], t["wu"], dy, pre=pre)
    do, _, dw, db = gla.gla_norm_bwd(o, dn.view(B, T, H, DK), t["w"], t["b"], EPS, layout=1)
    dq, dk, dv, dg, _ = gla.gla_decay_bwd(qn, kn, v, t["g"], do, 1, T, layout=1)
    dq, dk, dqw, dkw = gla.gla_qk_norm_bwd(q, k, dq, dk, qw, t["kw"], **QK)
    rows = torch.cat([x.flatten(-2) for x in (dq, dk, dv)], -1)
    return y, {"rows": rows, "qw": dqw * DK ** -0.5, "kw": dkw, "g": dg, "w": dw, "b": db, "wg": dwg, "wu": dwu}


def channels_reference(p):
    h = bo.recur_fwd(p["x"], bo.log_gate(p["z"], TAU)[0], True, p["s"])[:, 1:]
    return bo.glu_fwd(h.reshape(B * T, D), p["wg"], p["wu"], "gelu_tanh").reshape(B, T, F)


def channels(t, dy=None):
    how = {"tau": TAU, "complement": True, "initial_state": t["s"]}
    h, _ = gla.gla_recur_fwd(t["x"], t["z"], 1, T, **how)
    pre = torch.empty(2, B, T, F, device=DEV)
    y = gla.gla_glu_fwd(h, t["wg"], t["wu"], gla.ACT_GELU_TANH, pre=pre)
    if dy is None:
        return y
    dh, dwg, dwu = gla.gla_glu_bwd(h, t["wg"], t["wu"], dy, gla.ACT_GELU_TANH, pre=pre)
    dx, dz, ds = gla.gla_recur_bwd(t["x"], t["z"], dh, 1, T, want_d_initial_state=True, **how)
    return y, {"x": dx, "z": dz, "s": ds, "wg": dwg, "wu": dwu}


@pytest.mark.parametrize("run,reference,which", [(mixer, mixer_reference, 0), (channels, channels_reference, 1)])
def test_forward_and_gradients(run, reference, which):
    *both, dy = inputs(1)
    p = both[which]
    y, grads = run({n: torch.from_numpy(x).to(DEV) for n, x in p.items()}, torch.from_numpy(dy).to(DEV))
    torch.cuda.synchronize()
    p = {n: x.astype(np.float64) for n, x in p.items()}
    want = reference(p)
    err = np.abs(y.cpu().numpy() - want).max() / np.sqrt((want ** 2).mean())
    assert err <= SHARE, err
    rng = np.random.default_rng(2)
    for name, g in grads.items():
        g = g.double().cpu().numpy()
        for _ in range(3):
            d = rng.standard_normal(g.shape)
            h = 1e-5
            up, down = ((reference({**p, name: p[name] + s * h * d}) * dy).sum() for s in (1, -1))
            slope = (up - down) / (2 * h)
            assert abs(slope - (g * d).sum()) <= SHARE * np.linalg.norm(g) * np.linalg.norm(d), (name, slope, (g * d).sum())


@pytest.mark.parametrize("run,which", [(mixer, 0), (channels, 1)])
def test_training_step_in_a_graph(run, which):
    """Captured whole, replayed with the eager pass in between: the same bits each time."""
    *both, dy = inputs(3)
    t = {n: torch.from_numpy(x).to(DEV) for n, x in both[which].items()}
    dy = torch.from_numpy(dy).to(DEV)

    def step():
        y, grads = run(t, dy)
        return [y, *grads.values()]
    want = [x.clone() for x in step()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(3):
        for x in held:
            x.fill_(9.0)
        again = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, held, again))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_prompts_then_tokens(dtype):
    """A padded batch's prompts in one call, then a token at a time for all: what one call over prompt and tokens gives."""
    gen = torch.Generator().manual_seed(4)
    lens, more = [300, 1, 129], 5
    n, longest = len(lens), max(lens) + more
    x, z = (torch.randn(n, longest, D, generator=gen).to(dtype).to(DEV) for _ in range(2))
    wg, wu = ((torch.randn(F, D, generator=gen) * D ** -0.5).to(dtype).to(DEV) for _ in range(2))
    whole = torch.tensor([c + more for c in lens], dtype=torch.int32, device=DEV)
    h, fin = gla.gla_recur_fwd(x, z, 1, longest, seq_lens=whole, out=torch.zeros_like(x))
    want = gla.gla_glu_fwd(h, wg, wu)
    state = torch.zeros(n, D, device=DEV)
    gla.gla_recur_fwd(x, z, 1, longest, seq_lens=whole - more, initial_state=state, final_state=state)
    rows = torch.arange(n, device=DEV)
    rms = float(want[0, :lens[0]].float().square().mean().sqrt())
    share = SHARE if dtype is torch.float32 else 2.0 ** -5       # (states rounded to 16 bits before the product: 2^-8 of each of its factors, the largest of some hundred)
    for s in range(more):
        at = whole - more + s
        o, _ = gla.gla_recur_step(x[rows, at].contiguous(), z[rows, at].contiguous(), state)
        y = gla.gla_glu_fwd(o, wg, wu)
        assert float((y.float() - want[rows, at].float()).abs().max()) <= share * rms * 4
    assert float((state - fin).abs().max()) <= SHARE * float(fin.abs().max())
