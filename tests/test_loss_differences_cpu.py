"""What the difference test of the head loss's gradient can see; on the CPU."""
import pytest
import torch

from tests.loss_differences import Line
from tests.loss_reference import Reference


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("seed", [1, 2, 3])
def test_wrong_gradients_are_seen(which, dtype, seed):
    line = Line(which, dtype, seed, device="cpu")
    assert abs(line.rise) >= 20 * line.allowed, (line.rise, line.allowed)
    losses = [Reference(*line.at(e), line.targets, line.weights).loss.float() for e in line.ends]
    good = line.gradient.to(dtype)
    assert line.off(losses, good) <= line.allowed
    half = good.clone()
    half[: len(half) // 2] = 0      # (some rows' gradient missing)
    for bad in (torch.zeros_like(good), -good, 0.9 * good, 1.1 * good, half, good.roll(1, 0), good.roll(1, 1)):
        assert line.off(losses, bad) > line.allowed
