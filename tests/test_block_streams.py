"""Calls of the operators around the mixer on a stream that is not the current one, held to what test_streams.py holds the others to."""
import pytest

torch = pytest.importorskip("torch")

from paper_2405_18428_amd import binding
from tests import test_streams as ts

B, T, D, H, HK, E, F = 2, 300, 64, 4, 2, 32, 96
CALLS = ["gla_recur_fwd", "gla_recur_bwd", "gla_recur_step", "gla_qk_norm_fwd", "gla_qk_norm_bwd", "gla_glu_fwd", "gla_glu_bwd"]


def arguments(name, new):
    bf, f32 = torch.bfloat16, torch.float32
    rows = lambda: new(B, T, D, dtype=bf)  # noqa: E731
    qk = lambda n: new(B, n, T, E, dtype=bf)  # noqa: E731
    w = lambda: new(F, D, dtype=bf)  # noqa: E731
    return {
        "gla_recur_fwd": lambda: ((rows(), rows(), 1, T), {"initial_state": new(B, D, dtype=f32)}),
        "gla_recur_bwd": lambda: ((rows(), rows(), rows(), 1, T), {"d_final_state": new(B, D, dtype=f32), "want_d_initial_state": True}),
        "gla_recur_step": lambda: ((new(B, D, dtype=bf), new(B, D, dtype=bf), new(B, D, dtype=f32)), {}),
        "gla_qk_norm_fwd": lambda: ((qk(H), qk(HK), new(E, dtype=f32), new(E, dtype=f32)), {"sections": (E,)}),
        "gla_qk_norm_bwd": lambda: ((qk(H), qk(HK), qk(H), qk(HK), new(E, dtype=f32), new(E, dtype=f32)), {"sections": (E,)}),
        "gla_glu_fwd": lambda: ((rows(), w(), w()), {"pre": new(2, B, T, F, dtype=f32)}),
        "gla_glu_bwd": lambda: ((rows(), w(), w(), new(B, T, F, dtype=bf)), {}),
    }[name]()


@pytest.mark.parametrize("name", CALLS)
def test_the_call_runs_on_the_given_stream_and_records_its_tensors(name, monkeypatch):
    monkeypatch.setattr(ts, "arguments", arguments)
    monkeypatch.setattr(binding, "_want_rows", lambda *args: None)
    ts.test_the_call_runs_on_the_given_stream_and_records_its_tensors(name, monkeypatch)


@pytest.mark.gpu
@pytest.mark.parametrize("name", CALLS)
def test_memory_is_kept_while_the_stream_is_busy(name, monkeypatch):
    monkeypatch.setattr(ts, "arguments", arguments)
    ts.test_memory_is_kept_while_the_stream_is_busy(name)
