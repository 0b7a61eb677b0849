"""The loss of a row whose logits may be anything finite, in binary64: everything from differences to the largest logit, so that nothing is lost next to a large
one.  Bounds as in loss_ref.  Nothing here is shared with the library."""
import numpy as np

U = 2.0 ** -24
FAR = 2.0 ** 20 / np.log2(np.e)      # an lse of this magnitude in binary32 no longer holds the sum's logarithm; the gradient does not start from it


def log_softmax(x):
    """x - lse(x), and log(sum exp(x - max))."""
    top = np.max(x)
    d = x - top
    log_s = np.log(np.sum(np.exp(d)))
    return d - log_s, log_s


def row(z, label, index, teacher, T, wl, wt, lse=None):
    """As loss_ref.row; lse: the pair in binary32 that the backward pass is given.

    Bounds of a softmax's element with exponent d = (z - max) / T - log(sum): |d| 4 U for the exponent and its product, 8 U for the power and quotient, and the
    sum's: 32 terms in a row for each 131072 columns begun and 20 joins.  From an lse in binary32, |lse| + |d| in place of |d|, six roundings."""
    vocab = len(z)
    lp1, s1 = log_softmax(z)
    lp2, s2 = log_softmax(z / T)
    one, two = np.max(z) + s1, np.max(z) / T + s2
    terms = (32 * (vocab // 131072 + 1) + 20) * U
    far1, far2 = (np.where(np.isfinite(x), np.abs(x), 0.0) for x in (lp1, lp2))      # (-infinity: a probability of 0)
    e1, e2 = far1 * 4 * U + 8 * U + terms, far2 * 4 * U + 8 * U + terms
    if lse is not None and max(abs(lse[0]), abs(lse[1])) < FAR:
        e1, e2 = (abs(lse[0]) + far1) * 6 * U + 8 * U, (abs(lse[1]) + far2) * 6 * U + 8 * U
        lp1, lp2 = z - lse[0], z / T - lse[1]
    loss, loss_err, d, err = 0.0, 2.0 ** -126, np.zeros(vocab), np.full(vocab, 2.0 ** -120)
    if label >= 0:
        p = np.exp(lp1)
        loss -= wl * lp1[label]
        loss_err += wl * ((abs(lp1[label]) + 1) * 6 * U + terms)
        d += wl * p
        err += wl * p * e1
        d[label] -= wl
        err[label] += wl * 2 * U
    there = (np.asarray(index) >= 0) & (np.asarray(teacher) > -np.inf)
    if there.any():
        at, t = np.asarray(index)[there], np.asarray(teacher, dtype=np.float64)[there] / T
        lp, _ = log_softmax(t)
        p, q, lq = np.exp(lp), np.exp(lp2), lp2[at]
        ep = np.abs(lp) * 4 * U + 8 * U + 50 * U
        kl = np.where(p > 0, p * (lp - lq), 0.0)
        loss += wt * T * T * kl.sum()
        if np.isfinite(kl).all():
            loss_err += wt * T * T * (np.abs(kl) * (ep + 60 * U) + p * ((np.abs(lp) + np.abs(lq) + 2) * 6 * U + terms + 50 * U)).sum()
        d += wt * T * q
        err += wt * T * q * e2
        np.subtract.at(d, at, wt * T * p)
        np.add.at(err, at, wt * T * p * (ep + len(p) * U))
    lse_err = [abs(x) * 4 * U + 8 * U + terms for x in (one, two)]
    return loss, one, two, d, loss_err, lse_err, err + np.abs(d) * 8 * U
