"""The reference of the gated recurrence: its gradients against differences of its forward pass, and by a hand-worked case."""
import numpy as np
import pytest

from tests import scan_ref as ref


def test_by_hand():
    # a = 1/2 throughout: h = (h' + v) / 2
    f, v = np.zeros((3, 1)), np.array([[4.0], [2.0], [8.0]])
    w = ref.forward(f, v, None, [0, 2, 3], np.array([[8.0], [0.0]]))
    assert w["y"].ravel().tolist() == [6.0, 4.0, 4.0] and w["h_last"].ravel().tolist() == [4.0, 4.0]
    d = ref.backward(f, v, None, [0, 2, 3], np.array([[8.0], [0.0]]), np.array([[1.0], [1.0], [2.0]]), None)
    # G = 1, 1.5, 2 from the last row of each; dv = G / 2; df = G (h' - v) / 4; dh0 = G / 2 of the first row
    assert d["dv"].ravel().tolist() == [0.75, 0.5, 1.0] and d["df"].ravel().tolist() == [1.5, 1.0, -4.0] and d["dh0"].ravel().tolist() == [0.75, 1.0]


@pytest.mark.parametrize("gate", [False, True])
def test_gradients_against_differences(gate):
    rng = np.random.default_rng(1)
    rows, cols, bounds = 9, 2, [0, 4, 4, 5, 9]
    x = dict(f=rng.normal(size=(rows, cols)), v=rng.normal(size=(rows, cols)), h0=rng.normal(size=(4, cols)))
    if gate:
        x["o"] = rng.normal(size=(rows, cols))
    dy, dl = rng.normal(size=(rows, cols)), rng.normal(size=(4, cols))

    def loss(p):
        w = ref.forward(p["f"], p["v"], p.get("o"), bounds, p["h0"])
        return (w["y"] * dy).sum() + (w["h_last"] * dl).sum()

    d = ref.backward(x["f"], x["v"], x.get("o"), bounds, x["h0"], dy, dl)
    for name in x:
        for at in np.ndindex(x[name].shape):
            hi, lo = ({k: v.copy() for k, v in x.items()} for _ in range(2))
            hi[name][at] += 1e-5
            lo[name][at] -= 1e-5
            # central differences: the error is h^2 / 6 times a third derivative of order 1, and 1e-16 / h of rounding
            assert abs((loss(hi) - loss(lo)) / 2e-5 - d["d" + name][at]) < 1e-8
