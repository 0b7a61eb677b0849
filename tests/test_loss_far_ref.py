"""The reference for large logits: the ordinary one where both hold, and closed forms where only it does."""
import numpy as np

from tests import loss_far_ref as far
from tests import loss_ref as ref


def test_the_same_as_the_ordinary_one():
    rng = np.random.default_rng(0)
    for T in (0.5, 1.0, 3.0):
        z, index, teacher = rng.normal(size=50) * 4, rng.permutation(50)[:6], rng.normal(size=6)
        for lse in (None, (np.float32(ref.log_sum(z)), np.float32(ref.log_sum(z / T)))):
            a, b = (f(z, 7, index, teacher, T, 0.6, 0.4, lse) for f in (far.row, ref.row))
            # an lse that is given is for the gradient alone
            for k in ((0, 1, 2, 3) if lse is None else (3,)):
                assert np.allclose(a[k], b[k], rtol=1e-12, atol=1e-13)
            assert np.allclose(a[6], b[6], rtol=1e-5)


def test_a_row_of_equal_logits_whatever_they_are():
    for value in (0.0, -1e30, 3e38, float(np.finfo(np.float32).min)):
        z = np.full(40, value)
        loss, one, two, d, *_ = far.row(z, 3, [5, 6], [value, value], 2.0, 0.6, 0.4)
        # CE = log 40; KL of 1/2, 1/2 against 1/40 each = log 20
        assert np.isclose(loss, 0.6 * np.log(40) + 0.4 * 4 * np.log(20)) and np.isclose(one, value + np.log(40)) and np.isclose(two, value / 2 + np.log(40))
        want = np.full(40, 0.6 / 40 + 0.8 / 40)
        want[3] -= 0.6
        want[[5, 6]] -= 0.4
        assert np.allclose(d, want)


def test_a_masked_word_with_a_label():
    z = np.array([1.0, 2.0, -1e30])
    loss, _, _, d, *_ = far.row(z, 2, [], [], 1.0, 1.0, 0.0)
    assert np.isclose(loss, 1e30) and np.allclose(d, [1 / (1 + np.e), np.e / (1 + np.e), -1.0])
