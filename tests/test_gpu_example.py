"""The example that uses the operators together: it has to learn, and moments in 8 bits have to serve as well as in 32."""
import math

import pytest

from examples import train_lm

pytestmark = pytest.mark.gpu


def test_training_learns_and_eight_bits_keep_up():
    """Uniform guessing is log 512 = 6.24 nats, the chain's entropy 1.21: 25 rounds have to bring the loss below the middle, and the two forms of
    the moments may end a tenth of a nat apart (a twentieth of what a round's loss varies by between batches, times its early slope)."""
    loss = {bits: train_lm.train(rounds=25, workers=3, bits=bits, out=lambda s: None) for bits in (8, 32)}
    for bits in (8, 32):
        assert all(math.isfinite(x) for x in loss[bits])
        assert loss[bits][-1] < (6.24 + 1.21) / 2 < loss[bits][0]
    assert abs(loss[8][-1] - loss[32][-1]) < 0.1


def test_a_run_repeats_bit_for_bit():
    a, b = (train_lm.train(rounds=4, workers=2, out=lambda s: None, staleness=0) for _ in range(2))
    assert a == b
