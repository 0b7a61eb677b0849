"""The loss over a label and a teacher's top logits, and its gradient, in binary64, with bounds on what a computation in binary32 may be off by.
Nothing here is shared with the library."""
import numpy as np

U = 2.0 ** -24


def log_sum(x):
    top = np.max(x)
    if top == -np.inf:
        return -np.inf
    return top + np.log(np.sum(np.exp(x - top)))


def row(z, label, index, teacher, T, wl, wt, lse=None):
    """One row: z [vocab], a label (negative: none), entries `index` and `teacher` (may be empty).
    Returns loss, lse(z), lse(z / T), the gradient for dloss = 1, and the bounds of loss, of the lse's and of the gradient's elements.

    lse: the pair in binary32 that the backward pass starts from, instead of the sums.

    Bounds.  2^x is good to 2^-22; x = z c - k has an error of |z - max| 2^-23 (and a unit's rounding), c one of 2^-25, which moves lse by |lse| 2^-25
    and nearly cancels in a softmax.  A sum has at most 8 * 4 * (vocab / 131072 + 1) terms in a row and 20 joins: 2^-24 each.  From an lse that is
    given in binary32: (|lse| + |z|) 2^-23 in place of that."""
    vocab = len(z)
    one, two = (log_sum(z), log_sum(z / T)) if lse is None else lse
    terms = (32 * (vocab // 131072 + 1) + 20) * U
    far1, far2 = np.abs(z - one), np.abs(z / T - two)
    far1, far2 = np.where(np.isfinite(far1), far1, 0.0), np.where(np.isfinite(far2), far2, 0.0)
    e1, e2 = far1 * 4 * U + 8 * U + terms, far2 * 4 * U + 8 * U + terms
    if lse is not None:
        e1, e2 = (np.abs(one) + far1) * 6 * U + 8 * U, (np.abs(two) + far2) * 6 * U + 8 * U
    loss, loss_err, d, err = 0.0, 2.0 ** -126, np.zeros(vocab), np.full(vocab, 2.0 ** -120)
    if label >= 0:
        p = np.exp(z - one)
        loss += wl * (one - z[label])
        loss_err += wl * ((abs(one - z[label]) + 1) * 6 * U + terms)
        d += wl * p
        err += wl * p * e1
        d[label] -= wl
        err[label] += wl * 2 * U
    there = (np.asarray(index) >= 0) & (np.asarray(teacher) > -np.inf)
    if there.any():
        at, t = np.asarray(index)[there], np.asarray(teacher, dtype=np.float64)[there] / T
        lt = log_sum(t)
        p, q = np.exp(t - lt), np.exp(z / T - two)
        ep = np.abs(t - lt) * 4 * U + 8 * U + 50 * U
        lp, lq = t - lt, z[at] / T - two
        with np.errstate(invalid="ignore"):
            kl = np.where(p > 0, p * (lp - lq), 0.0)
        loss += wt * T * T * kl.sum()
        if np.isfinite(kl).all():
            loss_err += wt * T * T * (np.abs(kl) * (ep + 60 * U) + p * ((np.abs(lp) + np.abs(lq) + 2) * 6 * U + terms + 50 * U)).sum()
        d += wt * T * q
        err += wt * T * q * e2
        np.subtract.at(d, at, wt * T * p)
        np.add.at(err, at, wt * T * p * (ep + len(p) * U))
    lse_err = [abs(x) * 4 * U + 8 * U + terms if np.isfinite(x) else 0.0 for x in (one, two)]
    return loss, one, two, d, loss_err, lse_err, err + np.abs(d) * 8 * U
