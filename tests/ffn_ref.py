"""The gated feed-forward layer and the gradients of its sums in binary64.  Nothing here is shared with the library."""
import numpy as np

A, B = np.sqrt(2.0 / np.pi), 0.044715


def sigmoid(x):
    return np.where(x >= 0, 1.0 / (1.0 + np.exp(-np.abs(x))), np.exp(-np.abs(x)) / (1.0 + np.exp(-np.abs(x))))


def inner(x, kind):
    """What the sigmoid is taken of, and its derivative: gelu's (1 + tanh(w / 2)) / 2 is sigmoid(w), which keeps its digits where it is small."""
    return (x, np.ones_like(x)) if kind == "silu" else (2.0 * A * (x + B * x ** 3), 2.0 * A * (1.0 + 3.0 * B * x * x))


def act(x, kind):
    return x * sigmoid(inner(x, kind)[0])


def slope(x, kind):
    w, dw = inner(x, kind)
    return sigmoid(w) + x * sigmoid(w) * sigmoid(-w) * dw


# Bounds in binary32.  s = sigmoid(w) = 1 / (1 + 2^(-w log2 e)): the power has a relative error of |w| 2^-23 + 2^-22 and w (three roundings, a constant)
# one of 2^-21 of itself, so s has (1 - s) (|w| (2^-23 + 2^-21) + 2^-22) + 2^-22; act = g s adds 2^-24.  (The power is held to 2^126, or is infinite
# and s is 0, where s is below 2^-126.)
def act_error(x, kind):
    w, _ = inner(x, kind)
    return np.abs(x) * sigmoid(w) * (sigmoid(-w) * (np.abs(w) * 2.0 ** -20.6 + 2.0 ** -22) + 2.0 ** -21) + np.abs(x) * 2.0 ** -126


# slope = s + g s (1 - s) w': 1 - s = e s, with the errors of e and s; two products and a sum; s is not below 2^-126 (e is held to 2^126).
def slope_error(x, kind):
    w, dw = inner(x, kind)
    s, r = sigmoid(w), sigmoid(-w)
    return s * (r * (np.abs(w) * 2.0 ** -20.6 + 2.0 ** -22) + 2.0 ** -21) + np.abs(x * dw) * s * r * (np.abs(w) * 2.0 ** -19 + 2.0 ** -19.5) + (1.0 + np.abs(x * dw)) * 2.0 ** -125
