"""The gated linear recurrence and its gradients in binary64, row by row, with bounds on what a computation in binary32 may be off by.
Nothing here is shared with the library."""
import numpy as np


def sigmoid(x):
    return np.where(x >= 0, 1.0 / (1.0 + np.exp(-np.abs(x))), np.exp(-np.abs(x)) / (1.0 + np.exp(-np.abs(x))))


# Relative errors of binary32: of e = 2^(-x log2 e), whose exponent is rounded twice (|x| 2^-24 each) and whose power is good to 2^-22;
# of a step's product and sum (the quotient 2^-23, its denominator, the products of gates, two additions 2^-24 each: together below 2^-21).
STEP = 2.0 ** -21


def e_error(x):
    return np.abs(x) * 2.0 ** -23 + 2.0 ** -22


def forward(f, v, o, bounds, h0):
    """f, v, o [rows, cols] in binary64 (o may be None), bounds: sequences + 1 rows, h0 [sequences, cols] or None.
    Returns y, h_last, and h with bounds on their errors (in binary32, before any rounding to fewer bits): a dict."""
    rows, cols = f.shape
    n = len(bounds) - 1
    a, r = sigmoid(f), sigmoid(-f)
    gate = np.ones_like(f) if o is None else sigmoid(o)
    h = np.zeros((rows, cols))
    before, err, err_before, size = np.zeros((rows, cols)), np.zeros((rows, cols)), np.zeros((rows, cols)), np.zeros((rows, cols))
    last, last_err = np.zeros((n, cols)), np.zeros((n, cols))
    ea, er = r * e_error(f) + STEP, a * e_error(f) + STEP
    for s in range(n):
        x = h0[s].copy() if h0 is not None else np.zeros(cols)
        e, m = np.zeros(cols), np.abs(x)
        for t in range(bounds[s], bounds[s + 1]):
            before[t], err_before[t] = x, e
            e = a[t] * e + a[t] * ea[t] * m + r[t] * er[t] * np.abs(v[t])
            x = a[t] * x + r[t] * v[t]
            m = a[t] * m + r[t] * np.abs(v[t])
            h[t], err[t], size[t] = x, e, m
        last[s], last_err[s] = x, e
    return dict(h=h, y=h * gate, y_err=err * gate + np.abs(h) * gate * (e_error(np.zeros_like(f) if o is None else o) + STEP), h_last=last, h_last_err=last_err + np.abs(last) * 2.0 ** -24,
                before=before, before_err=err_before, err=err, a=a, r=r, gate=gate)


def backward(f, v, o, bounds, h0, dy, dh_last):
    """Gradients df, dv, do, dh0 with bounds on their errors."""
    w = forward(f, v, o, bounds, h0)
    rows, cols = f.shape
    n = len(bounds) - 1
    a, r, gate, before = w["a"], w["r"], w["gate"], w["before"]
    out = {k: np.zeros((rows, cols)) for k in ("df", "dv", "do", "df_err", "dv_err", "do_err")}
    out["dh0"], out["dh0_err"] = np.zeros((n, cols)), np.zeros((n, cols))
    eo = np.zeros_like(f) if o is None else e_error(o) + STEP
    ea, er = r * e_error(f) + STEP, a * e_error(f) + STEP
    for s in range(n):
        M = dh_last[s].copy() if dh_last is not None else np.zeros(cols)
        e, m = np.zeros(cols), np.abs(M)
        for t in reversed(range(bounds[s], bounds[s + 1])):
            G = dy[t] * gate[t] + M
            Ge = np.abs(dy[t]) * gate[t] * eo[t] + e
            Gm = np.abs(dy[t]) * gate[t] + m
            Ge = Ge + Gm * 2.0 ** -23
            step = before[t] - v[t]
            step_err = w["before_err"][t] + (np.abs(before[t]) + np.abs(v[t])) * 2.0 ** -23
            out["dv"][t], out["dv_err"][t] = G * r[t], Ge * r[t] + Gm * r[t] * er[t]
            out["df"][t] = G * step * a[t] * r[t]
            out["df_err"][t] = a[t] * r[t] * (Ge * np.abs(step) + Gm * step_err + Gm * np.abs(step) * (ea[t] + er[t]))
            if o is not None:
                out["do"][t] = dy[t] * w["h"][t] * gate[t] * (1.0 - gate[t])
                out["do_err"][t] = np.abs(dy[t]) * gate[t] * sigmoid(-o[t]) * (w["err"][t] + np.abs(w["h"][t]) * 2.0 * eo[t])
            M, e, m = a[t] * G, a[t] * Ge + a[t] * ea[t] * Gm, a[t] * Gm
        out["dh0"][s], out["dh0_err"][s] = M, e + np.abs(M) * 2.0 ** -24
    return out
