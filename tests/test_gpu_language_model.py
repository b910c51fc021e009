"""The operators together, as the example trains with them: the loss falls, and equal seeds give equal runs."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [0, 1])
def test_replicas_of_a_small_language_model_learn(dtype):
    from examples.language_model import train
    losses = train(steps=40, dtype=dtype)
    assert abs(losses[0] - math.log(512)) < 1.0          # near uniform at the start
    assert all(math.isfinite(v) for v in losses) and losses[-1] < 0.5 * losses[0]
    assert train(steps=40, dtype=dtype) == losses
