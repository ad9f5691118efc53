"""The factor that a language model's matrices move by: the root of outputs over inputs where a layer has more outputs, else one.
The kernel is stood in for by a record of its arguments, so no GPU is needed."""
import math

import pytest
import torch


@pytest.fixture()
def step():
    from paper_2505_10183_b200 import language_step
    return language_step


class Recorder:
    """Takes the place of the update's kernel; the factor of each shape that it was called with."""

    def __init__(self, monkeypatch, kt):
        self.factors = {}
        monkeypatch.setattr(kt, "kt_orth_update", self)

    def __call__(self, x, out, workspace, steps=5, coefficients=None, scale=1.0, stream=None):
        assert out.shape == x.shape and out.dtype == torch.bfloat16
        self.factors[tuple(x.shape[1:])] = scale
        out.zero_()


# width 256, 4 query heads and 1 of keys and values of 64, hidden 1024: by each layer's inputs and outputs
WANT = {(256, 384): math.sqrt(384 / 256),       # qkv: 256 inputs, 4 + 2 * 1 heads of 64
        (256, 256): 1.0,                        # proj
        (256, 1024): 2.0,                       # up: fourfold
        (1024, 256): 1.0}                       # down


def test_more_outputs_than_inputs_move_by_more(step, monkeypatch):
    """Activations are multiplied from the left, x @ up, so the model's matrices are [inputs, outputs]."""
    recorder = Recorder(monkeypatch, step.kt)
    shape = step.Shape(width=256, heads=4, heads_kv=1, hidden=1024)
    params = step.parameters(shape, 2, 50, 0, "cpu")
    step.Update(2, params, inputs_first=True).step({n: torch.zeros_like(p) for n, p in params.items()})
    assert recorder.factors == {s: pytest.approx(factor, rel=1e-12) for s, factor in WANT.items()}


def test_matrices_of_outputs_by_inputs(step, monkeypatch):
    """Where the caller's matrices are the other way round, as stock linear layers have them, so is the factor."""
    recorder = Recorder(monkeypatch, step.kt)
    shape = step.Shape(width=256, heads=4, heads_kv=1, hidden=1024)
    params = {n: p.t().contiguous() if p.dim() == 2 and n != "embed" else p for n, p in step.parameters(shape, 1, 50, 0, "cpu").items()}
    step.Update(1, params).step({n: torch.zeros_like(p) for n, p in params.items()})
    assert recorder.factors == {(cols, rows): pytest.approx(factor, rel=1e-12) for (rows, cols), factor in WANT.items()}


@pytest.mark.gpu
def test_the_example_moves_so(step, monkeypatch):
    if not torch.cuda.is_available():
        pytest.fail("this test needs a CUDA device")
    torch.cuda.set_device(0)
    recorder = Recorder(monkeypatch, step.kt)
    step.example(64, 256, 1, 300, 8)            # heads of 64, one of keys and values, hidden 1024
    assert recorder.factors == {shape: pytest.approx(factor, rel=1e-12) for shape, factor in WANT.items()}
