"""The example as a user runs it: write and attention together, turn after turn, against unquantised attention in float32.

An element of a page's head is off by at most half a step: 1/254 of the head's largest magnitude in the page with int8, 2^-4 of the
element with E4M3.  Values are normal with unit variance here, so the largest of 2048 is below 6; outputs are weighted means of them,
so off by at most 6/254 (0.024) and 2^-4 of a mean magnitude of at most 6 (0.38) from V, and by less than as much again from K, whose
scores move by at most a few hundredths.  Their rms is above 0.1 (means of at most 240 values)."""
import pytest
import torch

from examples.rollout_8bit import rollout

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,room", [(torch.int8, 0.5), (torch.uint8, 4.0)])
@pytest.mark.parametrize("heads", [(16, 4, 128), (8, 2, 64)])
def test_rollout_over_an_8_bit_cache(dtype, room, heads):
    assert rollout(dtype, heads=heads) < room


def test_token_by_token():
    assert rollout(torch.int8, turns=((1, 1),) * 40) < 0.5
