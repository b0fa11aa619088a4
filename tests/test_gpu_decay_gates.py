"""The gates' gradient of gla_decay_bwd against the 64-bit recurrence, by relative 2-norm, so that a gradient of zeros or of another order is
refused, for all scan and memory orders, kinds of gates, lengths and states, and for gates of any strength.

Bounds.  A step's gradient is a sum of up to 256 differences of two flows, each of which is off by e of its size, at random.  Where memories are shortest
a gradient is as large as one flow, so that it is off by at most sqrt(2 * 256) e = 22.6 e of its size (2-norm over all steps); longer memories
make it larger than the flows.  e: fp32 sums of up to 128 products at random 4 * 2^-24 at most (sqrt(128) roundings of 2^-24 / sqrt(3) of partial sums that
grow to the whole: 3.8): 90 * 2^-24 < 2^-17.  bf16 calls split three factors of a product into two numbers, each off by
2^-18 / sqrt(3) rms: e = 2^-18, 22.6 * 2^-18 < 2^-13.
One decay a head: its gradient counts each flow by its place in a block, 256 / sqrt(3) = 148 rms, twice, against a sum of gradients at random: 209 e, with
e = 4 * 2^-24 (bf16 calls take three numbers): 836 * 2^-24 < 2^-14.  With memories of ten steps and more gradients add up over
these and are larger than flows by as much: a tenth, below 2^-17; 2^-16 where padded sequences of less than that stand among the others."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla
from oracle import ops_oracle as oo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
TOKEN = {F32: 2.0 ** -17, BF16: 2.0 ** -13}
HEAD, HEAD_SHORTEST = 2.0 ** -16, 2.0 ** -14


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gla.load_library()


def make(B, H, T, dk, dv, dtype, layout, gate, seed, state=True, scale=0.1):
    gen = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    lead = (B, H, T) if layout == 0 else (B, T, H)
    return {"q": (randn(*lead, dk) * dk ** -0.5).to(dtype), "k": randn(*lead, dk).to(dtype), "v": randn(*lead, dv).to(dtype), "do": randn(*lead, dv).to(dtype),
            "g": -scale * torch.rand(*((H,) if gate == "head" else lead), generator=gen),
            "s0": randn(B, H, dk, dv) if state else None, "ds": randn(B, H, dk, dv) if state else None}


def gradient(c, gh, gw, scan, layout, lens):
    """dlog_decay like c's gates, and dq, dk, dv, in 64 bits."""
    lie = (lambda x: x) if layout == 0 else (lambda x: x.transpose(1, 2))
    q, k, v, do = (lie(c[n]).double().numpy() for n in ("q", "k", "v", "do"))
    B, H, T, dk = q.shape
    g = c["g"].double()
    heads = g.dim() == 1
    g = (g[None, :, None].expand(B, H, T) if heads else lie(g)).numpy()
    zero = np.zeros((B, H, dk, v.shape[3]))
    s0, ds = (zero if c[n] is None else c[n].double().numpy() for n in ("s0", "ds"))
    dg, rows = np.zeros((B, H, T)), [np.zeros(x.shape) for x in (q, k, v)]
    for b in range(B):
        at = oo.visits(T, gh, gw, scan, T if lens is None else min(max(lens[b], 0), T))
        x = [t[b][:, at] for t in (q, k, v, g)]
        S = oo.decay_fwd(*x, s0[b])[1]
        y = oo.decay_bwd(*x, S, do[b][:, at], ds[b])
        dg[b][:, at] = y[3]
        for into, t in zip(rows, y):
            into[b][:, at] = t
    if heads:
        return dg.sum((0, 2)), rows
    return (dg if layout == 0 else dg.swapaxes(1, 2)), rows


def off(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


def check(c, gh, gw, scan, layout, bound, lens=None):
    want, rows = gradient(c, gh, gw, scan, layout, lens)
    assert off(np.zeros_like(want), want) > bound
    d = {n: None if t is None else t.to(DEV) for n, t in c.items()}
    n = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    got = gla.gla_decay_bwd(d["q"], d["k"], d["v"], d["g"], d["do"], gh, gw, scan, layout, n, d["s0"], d["ds"])
    torch.cuda.synchronize()
    dg = got[3].double().cpu().numpy()
    assert off(dg, want) <= bound, (off(dg, want), bound)
    # the step's own part, which is kept out of the gates' gradient, belongs to dq and dk: off by a split's 2^-17 at most
    for x, y in zip(got, rows):
        x = (x if layout == 0 else x.transpose(1, 2)).double().cpu().numpy()
        assert off(x, y) <= 2.0 ** -16
    return dg


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gate", ["head", "token"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("scan", [0, 1, 2, 3])
def test_scan_orders(scan, layout, gate, dtype):
    """More than two blocks of 256 steps, states at both ends."""
    check(make(2, 4, 23 * 25, 32, 48, dtype, layout, gate, seed=scan), 23, 25, scan, layout, HEAD if gate == "head" else TOKEN[dtype])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gate", ["head", "token"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("scan", [0, 1])
def test_padded(scan, layout, gate, dtype):
    """Lengths at and around the ends of chunks and blocks."""
    check(make(7, 4, 600, 24, 40, dtype, layout, gate, seed=10 + scan), 1, 600, scan, layout, HEAD if gate == "head" else TOKEN[dtype],
          [600, 0, 1, 256, 257, 511, 64])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gate", ["head", "token"])
@pytest.mark.parametrize("dk,dv", [(7, 100), (36, 72), (64, 128), (128, 64), (128, 128)])
def test_head_sizes(dk, dv, gate, dtype):
    for state in (False, True):
        check(make(1, 4, 520, dk, dv, dtype, 0, gate, seed=dk + dv, state=state), 1, 520, 0, 0, HEAD if gate == "head" else TOKEN[dtype])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gate", ["head", "token"])
@pytest.mark.parametrize("strength", [-1.0, -4.0, -8.0, -16.0])
def test_strong_gates(strength, gate, dtype):
    """Gradients that vanish with the gate: a step's own product, which no gate scales, leaves no trace in them."""
    c = make(1, 8, 1024, 64, 64, dtype, 0, gate, seed=20, state=False)
    c["g"].fill_(strength)
    check(c, 1, 1024, 0, 0, HEAD_SHORTEST if gate == "head" else TOKEN[dtype])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gates_of_all_strengths(dtype):
    """Gates from zero to -16 beside each other, and closed ones, whose gradient is zero."""
    c = make(2, 4, 700, 64, 64, dtype, 1, "token", seed=21, scale=16.0)
    c["g"][:, ::5] = -float("inf")
    c["g"][:, 1::5] = -1e30
    c["g"][:, 2::5] *= 2.0 ** -10
    dg = check(c, 1, 700, 1, 1, TOKEN[dtype])
    assert not dg[:, ::5].any() and not dg[:, 1::5].any() and dg[:, 2::5].all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gate", ["head", "token"])
def test_closed_gates(gate, dtype):
    """Nothing flows through gates of zero: their gradient is zero, and the others' is what it is without the closed heads."""
    c = make(2, 4, 400, 32, 32, dtype, 0, gate, seed=22)
    (c["g"][1:3] if gate == "head" else c["g"][:, 1:3]).fill_(-float("inf"))
    dg = check(c, 1, 400, 0, 0, HEAD if gate == "head" else TOKEN[dtype])
    assert not (dg[1:3] if gate == "head" else dg[:, 1:3]).any()


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


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gate", ["head", "token"])
@pytest.mark.parametrize("scan", [0, 1])
def test_nan_gate(scan, gate, dtype):
    """A gate that is NaN reaches all that depends on it, and nothing else: states and outputs from its step on, gradients of keys and values before
    it, the gates' gradient; other heads and what lies on the other side have the bits of a call without it."""
    n, t = 600, 300
    c = make(2, 3, n, 24, 40, dtype, 0, gate, seed=30)
    at = 299 if scan else t                 # token of step 300
    d = {m: x.to(DEV) for m, x in c.items()}

    def call(g):
        x = d["q"], d["k"], d["v"], g
        return [*gla.gla_decay_fwd(*x, 1, n, scan, initial_state=d["s0"]),
                *gla.gla_decay_bwd(*x, d["do"], 1, n, scan, initial_state=d["s0"], d_final_state=d["ds"], want_d_initial_state=True)]
    want = call(d["g"])
    g = d["g"].clone()
    (g[1:2] if gate == "head" else g[0, 1, at:at + 1]).fill_(float("nan"))
    got = call(g)
    torch.cuda.synchronize()
    steps = torch.arange(n, device=DEV)
    steps = n - 1 - steps if scan else steps
    after = steps >= t if gate == "token" else steps >= 0
    before = steps < t if gate == "token" else steps < n - 1        # (a head's gate leads from every step to the next)
    for name, x, y in zip(("out", "state", "dq", "dk", "dv", "dg", "ds0"), got, want):
        assert torch.isfinite(y).all(), name
        hit = torch.zeros_like(y, dtype=torch.bool)
        if name == "dg" and gate == "head":
            hit[1] = True
        else:
            which = hit[:, 1] if gate == "head" else hit[:1, 1]
            which[:, {"out": after, "dq": after, "dk": before, "dv": before}[name] if name in ("out", "dq", "dk", "dv") else slice(None)] = True
        assert torch.isnan(x[hit]).all() and torch.equal(x[~hit], y[~hit]), name


@pytest.mark.parametrize("gate", ["head", "token"])
def test_nan_gate_of_a_step(gate):
    q, k, v = (torch.randn(2, 3, w, device=DEV) for w in (24, 24, 40))
    g = torch.full((3,) if gate == "head" else (2, 3), -0.5, device=DEV)
    s = torch.randn(2, 3, 24, 40, device=DEV)
    want, state = gla.gla_decay_step(q, k, v, g, s, state_out=torch.empty_like(s))
    (g[1:2] if gate == "head" else g[0, 1:2]).fill_(float("nan"))
    got, new = gla.gla_decay_step(q, k, v, g, s, state_out=torch.empty_like(s))
    hit = torch.zeros(2, 3, dtype=torch.bool, device=DEV)
    hit[slice(None) if gate == "head" else 0, 1] = True
    for x, y in ((got, want), (new, state)):
        assert torch.isnan(x[hit]).all() and torch.equal(x[~hit], y[~hit])
