"""The exchange of answers from its formulas in 64 bits (numpy), and how far 32-bit results may be from it.

U is half a step of float32.  A sum over a row is a chain of at most classes / 64 additions per lane, then a tree:
its relative error is at most (classes / 64 + 32) U, next to the errors of its terms: exp of an exponent d has two
roundings of d (relative error 2 |d| U) and its own (2 U)."""
import numpy as np

U = 2.0 ** -24


def from_lse(z):
    """z - log sum exp z of every row, in two differences: next to a lowest value even 64 bits have no room for the sum's
    logarithm.  -inf where z is -inf, NaN where the row has a NaN."""
    m = z.max(1)
    rest = z - np.where(np.isfinite(m), m, 0.0)[:, None]
    with np.errstate(divide="ignore", invalid="ignore"):
        lp = rest - np.log(np.exp(rest).sum(1))[:, None]
    return np.where(z == -np.inf, -np.inf, lp)


def sum_error(classes):
    # sum_v p_v |d_v| is at most log classes plus the entropy's constant: 2 (log classes + 2) covers the exponents
    return (classes / 64 + 32 + 2 * (np.log(classes) + 2) + 4) * U


def top_logprobs(z, k):
    rows, V = z.shape
    index = np.full((rows, k), -1, np.int32)
    out = np.zeros((rows, k))
    lp = from_lse(z)
    for r in range(rows):
        good = np.flatnonzero(z[r] > -np.inf)                       # neither NaN nor -inf
        order = good[np.argsort(-(z[r, good] + 0.0), kind="stable")][:k]
        index[r, :order.size] = order
        out[r, :order.size] = lp[r, order]
    return index, out


def logprobs_at(z, index):
    filled = (index >= 0) & (index < z.shape[1])
    lp = np.take_along_axis(from_lse(z), np.where(filled, index, 0).astype(np.int64), 1)
    return np.where(filled, lp, 0.0)


def logprob_error(z, lp):
    """x - m and its difference to log S are rounded (|x - m| <= |lp|), log S has the error of S."""
    return (3 * np.abs(lp) + np.log(z.shape[1]) + 8) * U + sum_error(z.shape[1])


class Distill:
    """loss, lse, grad of every row, and bounds on the error of results in 32 bits."""

    def __init__(self, z, index, sum_, members, temperature, weight=None, lse=None):
        rows, V = z.shape
        k = index.shape[1]
        T = float(np.float32(temperature))
        w = np.ones(rows) if weight is None else weight.astype(np.float64)
        filled = (index >= 0) & (index < V) & (sum_ != -np.inf)
        at = np.where(filled, index, 0).astype(np.int64)
        t = np.where(filled, sum_.astype(np.float64) / members / T, -np.inf)
        self.lse, self.loss = np.zeros(rows), np.zeros(rows)
        self.grad = np.zeros((rows, V))
        self.loss_error, self.lse_error = np.zeros(rows), np.zeros(rows)
        self.grad_error = np.zeros((rows, V))
        self.p = np.zeros((rows, k))
        for r in range(rows):
            f = filled[r]
            if w[r] == 0 or not f.any():
                continue
            m = z[r].max()
            own = np.log(np.exp((z[r] - m) / T).sum()) if np.isfinite(m) else -np.inf
            self.lse[r] = m / T + own
            if own == -np.inf:
                continue
            # what is taken off z / T, in two parts: even 64 bits have no room for the second next to a lowest value
            m, own = (m / T, own) if lse is None else (0.0, float(lse[r]))
            tr, v = t[r, f], at[r, f]
            logp = tr - (tr.max() + np.log(np.exp(tr - tr.max()).sum()))
            p = np.exp(logp)
            self.p[r, f] = p
            q = z[r, v] / T - m - own
            self.loss[r] = w[r] * np.where(p > 0, p * (logp - q), 0.0).sum()
            d = z[r] / T - m - own
            soft = np.exp(d)
            g = w[r] / T
            teacher = np.zeros(V)
            np.add.at(teacher, v, p)
            self.grad[r] = g * (soft - teacher)
            # ---- bounds ----
            spread = np.abs(tr - tr.max())
            # t: sum / K / T as two products with rounded reciprocals, four roundings; its softmax as the rows'
            rel_p = (2 * spread + 4 * np.abs(tr) + 4 * np.abs(tr).max() + k + 16) * U
            finite = np.where(np.isfinite(q), np.abs(q), 0.0)
            log_err = (8 * np.abs(tr).max() + 3 * spread + np.log(k + 1) + k + 24 + 4 * finite + np.log(V) + 8) * U + sum_error(V)
            self.lse_error[r] = (4 * abs(self.lse[r]) + 4 * np.abs(z[r, np.isfinite(z[r])]).max() / T + np.log(V) + 8) * U + sum_error(V)
            with np.errstate(invalid="ignore"):
                term = np.where(p > 0, p * np.abs(logp - q), 0.0)
            self.loss_error[r] = abs(w[r]) * ((term * (rel_p + (k + 8) * U)).sum() + (p * log_err).sum())
            far = np.where(np.isfinite(d), np.abs(d), 0.0)
            rel_s = (6 * (far + np.log(V) + 1) + 8) * U + sum_error(V)
            if lse is not None:                                      # z / T - lse in one rounding, 1 / T rounded
                big = np.abs(np.where(np.isfinite(z[r]), z[r], 0.0)) / T
                rel_s = rel_s + 2 * (far + big) * U
            spare = np.zeros(V)
            np.add.at(spare, v, p * (rel_p + (k + 4) * U))
            self.grad_error[r] = abs(g) * (soft * rel_s + spare) + 4 * U * np.abs(self.grad[r]) + 2.0 ** -126 * max(abs(g), 1)

    def stored_error(self, half_step, least):
        """with one rounding to a type: half a step of the value, or of the least subnormal"""
        return self.grad_error + half_step * (np.abs(self.grad) + self.grad_error) + least
