"""Rotary positions (gla_rope) at the ends of 32 bits, for long sections and all bases, against angles of 60 digits.

Tolerance: an angle is off by its rounding to 32 bits of half a turn, pi 2^-25, and by 2^-25 / base from a frequency of 2^-63 for each of up to 128 products at
2^31 turns / (2 pi); sine and cosine by 2 units of 2^-24 each, their products' sum by 3 of 2^-25: below 2^-21 and 2^-25 / base of a pair's
length."""
import decimal

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla

D = decimal.Decimal
PI = D("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")


def angles(position, width, base):
    """Of the pairs of a section, in (-pi, pi]."""
    with decimal.localcontext() as ctx:
        ctx.prec = 60
        b, x = D(float(np.float32(base))), []
        ratio, f = (b.ln() * D(-2) / D(width)).exp(), D(1)
        for _ in range(width // 2):
            x.append(float((D(position) * f).remainder_near(2 * PI)))
            f *= ratio
    return np.array(x)


def test_reference():
    """The reference against 64-bit angles where these are exact enough, and against a frequency that is known."""
    for position in (0, 1, -3, 1000):
        x = position * 10000.0 ** (-2.0 * np.arange(16) / 32)
        assert np.abs(np.exp(1j * angles(position, 32, 10000.0)) - np.exp(1j * x)).max() < 1e-12
    assert abs(angles(2 ** 31 - 1, 4, 16.0)[1] - float((D(2 ** 31 - 1) / 4).remainder_near(2 * PI))) < 1e-15


@pytest.mark.gpu
@pytest.mark.parametrize("pairing", [gla.ROPE_ADJACENT, gla.ROPE_HALVES])
@pytest.mark.parametrize("sections", [(256,), (128,), (128, 64, 64), (18, 18), (50,)])
@pytest.mark.parametrize("base", [10000.0, 5e5, 2.0, 1.0, 0.5, 0.01])
def test_far_positions(base, sections, pairing):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    at = [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 12345, -1234567891, 987654321, 1, 0]
    d, T = sum(sections), len(at)
    x = torch.randn(1, 2, T, d, generator=torch.Generator().manual_seed(d))
    pos = torch.tensor(at, dtype=torch.int64).to(torch.int32)[None, :, None].expand(1, T, len(sections)).contiguous()
    y, _ = gla.gla_rope(x.to("cuda:0"), None, sections, positions=pos.to("cuda:0"), base=base, pairing=pairing)
    X, Y = x.double().numpy(), y.double().cpu().numpy()
    first = 0
    for w in sections:
        i = np.arange(w // 2)
        c0, c1 = (first + 2 * i, first + 2 * i + 1) if pairing == gla.ROPE_ADJACENT else (first + i, first + i + w // 2)
        for t in range(T):
            turned = (X[0, :, t, c0] + 1j * X[0, :, t, c1]) * np.exp(1j * angles(at[t], w, base))[:, None]
            off = np.abs(Y[0, :, t, c0] + 1j * Y[0, :, t, c1] - turned)
            bound = (2.0 ** -21 + 2.0 ** -25 / min(base, 1.0)) * np.abs(turned)
            assert (off <= bound).all(), (at[t], w, float((off / np.abs(turned)).max()))
        first += w
