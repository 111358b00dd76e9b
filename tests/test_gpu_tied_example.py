"""The example that runs all uses of the tied weight together learns its task."""
import pytest

pytestmark = pytest.mark.gpu


def test_the_example_learns():
    from examples.tied_training import train
    losses, right = train(steps=150)
    assert losses[0] > 6 and losses[-1] < losses[0] / 3      # a uniform guess over 1000 tokens is at 6.9
    assert right > 0.5
    again, _ = train(steps=3)
    assert again == losses[:3]                               # the same bits from the same seed
