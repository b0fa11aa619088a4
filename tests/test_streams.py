"""Calls on a stream that is not the current one: what they allocate is that stream's memory, and no tensor's memory is handed on before both streams
are done with it."""
import contextlib

import pytest

torch = pytest.importorskip("torch")

import paper_2405_18428_amd as gla
from paper_2405_18428_amd import binding

B, H, GH, GW, DK, DV = 1, 2, 8, 8, 16, 16
T, D = GH * GW, 64
CALLS = ["gla_fwd", "gla_fwd_static", "gla_fwd_ex", "gla_fwd_layout", "gla_fwd_gates", "gla_srem_dwconv", "gla_fwd_multi", "gla_fwd_fused", "gla_fwd_fused_gates",
         "gla_bwd", "gla_bwd_layout", "gla_bwd_gates", "gla_decay_fwd", "gla_decay_bwd", "gla_decay_step", "gla_rope", "gla_norm_fwd", "gla_norm_bwd"]


def arguments(name, new):
    """Positional and keyword arguments of a call; new(*shape, dtype=) makes a tensor."""
    bf, f32 = torch.bfloat16, torch.float32
    q, k, v = new(B, H, T, DK, dtype=bf), new(B, H, T, DK, dtype=bf), new(B, H, T, DV, dtype=bf)
    gate, gate_v, state = new(B, H, T, DK, dtype=f32), new(B, H, T, DV, dtype=f32), new(B, H, DK, DV, dtype=f32)
    qkv = (q, k, v)
    return {
        "gla_fwd": lambda: ((*qkv, gate, GH, GW), {}),
        "gla_fwd_static": lambda: ((*qkv, gate, GH, GW), {"out": new(B, H, T, DV, dtype=f32), "final_state": state}),
        "gla_fwd_ex": lambda: ((*qkv, gate, GH, GW), {}),
        "gla_fwd_layout": lambda: ((*qkv, gate, GH, GW), {"initial_state": state}),
        "gla_fwd_gates": lambda: ((*qkv, gate, gate_v, GH, GW), {}),
        "gla_srem_dwconv": lambda: ((new(B, T, D, dtype=bf), new(D, 3, 3, dtype=f32), new(D, dtype=f32), GH, GW), {}),
        "gla_fwd_multi": lambda: ((*qkv, gate, GH, GW), {}),
        "gla_fwd_fused": lambda: ((*qkv, new(B, H, T, DK, dtype=bf), 16.0, GH, GW), {"r_pre": new(B, H, T, DV, dtype=bf), "ln_weight": new(H, DV, dtype=f32)}),
        "gla_fwd_fused_gates": lambda: ((*qkv, new(B, H, T, DK, dtype=bf), new(B, H, T, DV, dtype=bf), 16.0, GH, GW), {}),
        "gla_bwd": lambda: ((*qkv, gate, new(B, H, T, DV, dtype=bf), GH, GW), {}),
        "gla_bwd_layout": lambda: ((*qkv, gate, new(B, H, T, DV, dtype=bf), GH, GW), {}),
        "gla_bwd_gates": lambda: ((*qkv, gate, gate_v, new(B, H, T, DV, dtype=bf), GH, GW), {}),
        "gla_decay_fwd": lambda: ((*qkv, new(H, dtype=f32), GH, GW), {"initial_state": state}),
        "gla_decay_bwd": lambda: ((*qkv, new(H, dtype=f32), new(B, H, T, DV, dtype=bf), GH, GW), {"d_final_state": state, "want_d_initial_state": True}),
        "gla_decay_step": lambda: ((new(B, H, DK, dtype=bf), new(B, H, DK, dtype=bf), new(B, H, DV, dtype=bf), new(B, H, dtype=f32), state), {}),
        "gla_rope": lambda: ((q, k, (8, 8), GH, GW), {}),
        "gla_norm_fwd": lambda: ((new(B, T, D, dtype=bf), new(D, dtype=f32), new(D, dtype=f32)), {}),
        "gla_norm_bwd": lambda: ((new(B, T, D, dtype=bf), new(B, T, D, dtype=bf), new(D, dtype=f32), new(D, dtype=f32)), {}),
    }[name]()


def tensors(result):
    return [t for t in (result if isinstance(result, tuple) else (result,)) if isinstance(t, torch.Tensor)]


class _OnGpu(torch.Tensor):
    is_cuda = True


class _Stream:
    device_index = -1

    def __init__(self, number):
        self.cuda_stream = number


@pytest.mark.parametrize("name", CALLS)
def test_the_call_runs_on_the_given_stream_and_records_its_tensors(name, monkeypatch):
    """On the CPU, with a library that computes nothing."""
    before, given = _Stream(1), _Stream(2)
    current, recorded, ran = [before], set(), []

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    class Library:
        def __getattr__(self, _):
            return lambda *args: ran.append((current[-1], args[-1])) or 0
    monkeypatch.setattr(torch.cuda, "Stream", _Stream)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda _=None: current[-1])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: recorded.add((t.data_ptr(), s.cuda_stream)))
    monkeypatch.setattr(binding, "load_library", lambda: Library())
    monkeypatch.setattr(binding, "_want", lambda *args: None)
    monkeypatch.setattr(binding, "_on_device_of", lambda _: contextlib.nullcontext())
    binding._torch()
    monkeypatch.setattr(binding, "_raw_stream", lambda _: current[-1].cuda_stream)
    args, kwargs = arguments(name, lambda *shape, dtype: torch.zeros(*shape, dtype=dtype).as_subclass(_OnGpu))
    out = tensors(getattr(gla, name)(*args, **kwargs, stream=given))
    assert current == [before] and ran[-1] == (given, 2) and out
    for t in (*args, *kwargs.values()):
        assert not isinstance(t, torch.Tensor) or (t.data_ptr(), 2) in recorded
    for t in out:
        assert (t.data_ptr(), 1) in recorded


def test_a_stream_of_another_device_is_refused(monkeypatch):
    monkeypatch.setattr(torch.cuda, "Stream", _Stream)
    stream = _Stream(2)
    stream.device_index = 1
    args, _ = arguments("gla_rope", lambda *shape, dtype: torch.zeros(*shape, dtype=dtype))
    with pytest.raises(ValueError, match="stream"):
        gla.gla_rope(*args, stream=stream)


@pytest.mark.gpu
@pytest.mark.parametrize("name", CALLS)
def test_memory_is_kept_while_the_stream_is_busy(name):
    """Tensors dropped while the stream still has work before the call: nothing allocated on the current stream gets their memory; and the results have
    none that the current stream gave back."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    new = lambda *shape, dtype: (-torch.rand(*shape, generator=gen, device="cuda:0")).to(dtype)  # noqa: E731
    args, kwargs = arguments(name, new)
    call = getattr(gla, name)
    want = [t.clone() for t in tensors(call(*[x.clone() if isinstance(x, torch.Tensor) else x for x in args],
                                            **{n: x.clone() if isinstance(x, torch.Tensor) else x for n, x in kwargs.items()}))]
    torch.cuda.synchronize()
    stream, done = torch.cuda.Stream(), torch.cuda.Event()
    load = torch.ones(6144, 6144, device="cuda:0")
    back = [torch.empty_like(t) for t in want]
    given_back = {t.data_ptr() for t in back}
    del back
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for _ in range(40):
            torch.mm(load, load)
    out = tensors(call(*args, **kwargs, stream=stream))
    done.record(stream)
    mine = {t.data_ptr() for t in out}
    passed = {x.data_ptr() for x in (*args, *kwargs.values()) if isinstance(x, torch.Tensor)}
    assert not (mine - passed) & given_back
    sizes = [t.numel() * t.element_size() for t in (*out, *[x for x in (*args, *kwargs.values()) if isinstance(x, torch.Tensor)])]
    with torch.cuda.stream(stream):
        keep = [t.clone() for t in out]
    del out, args, kwargs
    fresh = [torch.full((n,), 77, dtype=torch.uint8, device="cuda:0") for n in sizes for _ in range(2)]
    assert not done.query(), "the stream was not busy for long enough"
    assert not {t.data_ptr() for t in fresh} & (mine | passed)
    torch.cuda.synchronize()
    assert all(int(t.min()) == 77 and int(t.max()) == 77 for t in fresh)
    assert all(torch.equal(a, b) for a, b in zip(keep, want))
