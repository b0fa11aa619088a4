"""Outputs that overlap inputs without being the same tensor are refused on the host, before anything is enqueued (no GPU); in place they are not."""
import ctypes

import pytest

import paper_2405_18428_amd as gla

vp = ctypes.c_void_p
SHAPE = 2
BASE = 1 << 20


@pytest.fixture(scope="module")
def lib():
    return gla.load_library()


@pytest.mark.parametrize("first,last", [(BASE, BASE + 16), (BASE + 16, BASE), (BASE, BASE + 2 * 3 * 32 * 64 * 4 - 16)])
def test_decay_states(lib, first, last):
    x = vp(1 << 30)
    assert lib.gla_decay_fwd(x, x, x, x, 0, None, 2, 3, 600, 32, 64, 1, 600, 0, 1, 1, 0, vp(first), vp(1 << 31), vp(last), vp(1 << 32), 1 << 30, None) == SHAPE
    assert lib.gla_decay_step(x, x, x, x, 0, 2, 3, 32, 64, 1, 1, vp(first), vp(last), vp(1 << 31), None) == SHAPE


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("which", ["q,oq", "k,oq", "q,ok", "k,ok", "oq,ok"])
def test_rope(lib, which, dtype):
    at = {"q": BASE, "k": 2 * BASE, "oq": 3 * BASE, "ok": 4 * BASE}
    a, b = which.split(",")
    size = 2 * 3 * 12 * 32 * (2 if dtype else 4)
    for by in (16, -16, size - 16, 16 - size):
        p = {n: vp(x) for n, x in {**at, b: at[a] + by}.items()}
        assert lib.gla_rope(p["q"], p["k"], None, (ctypes.c_int * 2)(16, 16), 2, ctypes.c_float(1e4), 0, 0, 2, 3, 12, 32, 3, 4, dtype, 0, p["oq"], p["ok"],
                            None) == SHAPE


@pytest.mark.parametrize("x_dtype,out_dtype", [(0, 0), (1, 1), (0, 1), (1, 0)])
@pytest.mark.parametrize("gated", [False, True])
def test_norm(lib, gated, x_dtype, out_dtype):
    n = 2 * 3 * 8 * 64
    read, written = n * (2 if x_dtype else 4), n * (2 if out_dtype else 4)
    x, r = (2 * BASE, BASE) if gated else (BASE, None)          # the one that out overlaps is at BASE
    places = [BASE + 16, BASE - 16, BASE + read - 16, BASE + 16 - written] + ([BASE] if x_dtype != out_dtype else [])
    for out in places:
        assert lib.gla_norm_fwd(vp(x), None, None, ctypes.c_float(1e-5), vp(r), 2, 3, 8, 64, x_dtype, out_dtype, 0, vp(out), None) == SHAPE


@pytest.mark.gpu
@pytest.mark.parametrize("D", [20, 72, 1150, 2050, 8190])
def test_norm_in_place_of_the_gate(D):
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    for dtype in (torch.bfloat16, torch.float32):
        x, r = torch.randn(2, 2, 3, 500 if D < 100 else 40, D, device="cuda:0").to(dtype)
        want = gla.gla_norm_fwd(x, r_pre=r)
        assert gla.gla_norm_fwd(x, r_pre=r, out=r) is r
        torch.cuda.synchronize()
        assert torch.equal(r, want)
