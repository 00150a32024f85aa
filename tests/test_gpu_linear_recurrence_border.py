"""linear_recurrence and its gradients where the kernel for many channels takes over: as many channels as are, in vectors of two or one, just
under the line, on it and above it, with few steps and with enough for chunks of time (needs a B200)."""
import pytest

import test_gpu_linear_recurrence as lr

pytestmark = pytest.mark.gpu

# 11000 and 5600 channels, 11200 and 5664 of them with many steps
SHAPES = [(70, 4, 2750), (70, 11, 1002), (70, 7, 801), (70, 8, 700), (300, 8, 1416), (800, 4, 2800), (1500, 8, 708), (1450, 7, 809)]


@pytest.mark.parametrize("mode", (("bf16", True, False, True, "fused"), ("fp32", True, True, False, "plain"), ("bf16", False, True, True, "plain")), ids=str)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_against_every_step_in_64_bits_at_the_border(shape, mode):
    lr.test_against_every_step_in_64_bits((*shape, *mode))
