"""The example that runs the losses and the clipping together: training does what training should."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", [0, 1])
def test_updates_lower_both_losses(seed):
    from paper_2605_05802_amd.policy_step import train
    losses, pair_losses, norms = train(seed=seed)
    # at the first update the ratio is 1 and the divergence 0: the loss is minus the mean advantage, which is 0 group by group
    assert abs(losses[0]) < 1e-4
    assert losses[-1] < losses[0] - 0.01 and all(math.isfinite(x) for x in losses)
    assert pair_losses and pair_losses[-1] < pair_losses[0] and all(x > 0 and math.isfinite(x) for x in norms)
