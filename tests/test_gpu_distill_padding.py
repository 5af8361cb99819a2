"""Padding of a batch in a distillation step: whatever finite numbers stand there, loss and gradients are the same."""
import pytest
import torch

from paper_2601_04342_amd import binding
from tests.test_gpu_distill import setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fill", [0.0, -3.0, 1e4])
@pytest.mark.parametrize("d", [64, 128])
def test_what_stands_in_padding_does_not_count(d, fill):
    """A clip of two frames in a batch of four: later frames reach neither its own queries nor, at weight 0, a gradient."""
    s = setup(B=2, d=d, seed=7)
    T, HW = s["T"], s["HW"]
    weight = torch.ones(2, T * HW, device="cuda")
    weight[1, 2 * HW:] = 0
    got = []
    for padded in (False, True):
        q, k, v, y = (s[n].clone() for n in ("qr", "kr", "v", "y"))
        if padded:
            for t in (q, k, v):
                t[1, :, 2 * HW:] = fill
            y[1, :, 2 * HW:] = float("nan")
        grads = {n: torch.empty(t.shape, device="cuda") for n, t in s["phi"].items()}
        got.append((binding.distill_gradients(q, k, v, y, s["phi"], grads, T, HW, 1, weight=weight), grads))
    assert torch.isfinite(got[0][0]) and torch.equal(got[0][0], got[1][0])
    assert all(torch.equal(got[0][1][n], got[1][1][n]) and torch.isfinite(got[0][1][n]).all() for n in s["phi"])
