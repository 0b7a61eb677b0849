"""The reference of the gated layer: its activations by their usual formulas, its derivatives against differences."""
import numpy as np
import pytest

from tests import ffn_ref as ref


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_activations(kind):
    x = np.linspace(-9.0, 9.0, 181)
    usual = x / (1.0 + np.exp(-x)) if kind == "silu" else 0.5 * x * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (x + 0.044715 * x ** 3)))
    assert np.abs(ref.act(x, kind) - usual).max() < 1e-14
    # central differences: h^2 / 6 times a third derivative below 2, and 1e-16 * 9 / h of rounding
    assert np.abs((ref.act(x + 1e-5, kind) - ref.act(x - 1e-5, kind)) / 2e-5 - ref.slope(x, kind)).max() < 1e-9
