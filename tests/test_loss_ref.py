"""The reference of the loss: its gradient against differences, and by a hand-worked case."""
import numpy as np
import pytest

from tests import loss_ref as ref


def test_by_hand():
    z = np.log(np.array([1.0, 2.0, 5.0]))                # softmax 1/8, 2/8, 5/8
    loss, one, two, d, *_ = ref.row(z, 1, [], [], 1.0, 1.0, 0.0)
    assert np.allclose([loss, one, two], [np.log(4.0), np.log(8.0), np.log(8.0)]) and np.allclose(d, [1 / 8, -6 / 8, 5 / 8])
    # a teacher of 1/4, 3/4 on the first and the last: KL = 1/4 log(2) + 3/4 log(6/5); the entry that is not there counts for nothing
    loss, _, _, d, *_ = ref.row(z, -1, [0, 2, -1], np.array([0.0, np.log(3.0), 9.0]), 1.0, 1.0, 1.0)
    assert np.isclose(loss, 0.25 * np.log(2.0) + 0.75 * np.log(1.2)) and np.allclose(d, [1 / 8 - 1 / 4, 2 / 8, 5 / 8 - 3 / 4])


@pytest.mark.parametrize("T", [1.0, 2.5])
def test_gradient_against_differences(T):
    rng = np.random.default_rng(0)
    z, teacher = rng.normal(size=11), rng.normal(size=5)
    args = (3, [3, 7, 7, -1, 0], teacher, T, 0.7, 0.4)          # an index twice, and the label's
    d = ref.row(z, *args)[3]
    for i in range(11):
        hi, lo = z.copy(), z.copy()
        hi[i] += 1e-5
        lo[i] -= 1e-5
        # central differences: h^2 / 6 times a third derivative of order 1, and 1e-16 / h of rounding
        assert abs((ref.row(hi, *args)[0] - ref.row(lo, *args)[0]) / 2e-5 - d[i]) < 1e-8
