"""Draft verification of one request from its definition, in fp64."""
import numpy as np

TOL = 2.0 ** -20  # of a probability in fp32: see Model.allows


class Model:
    """rows of logits z [n][V], tokens [n], race [V] (None: greedy), u [n], q [n][V] or None."""

    def __init__(self, z, tokens, race, u, heat=1.0, q=None):
        z = np.asarray(z, np.float64)
        n, vocab = z.shape
        self.n, self.race, self.q, self.tokens = n, None if race is None else np.asarray(race, np.float64), q, tokens
        self.greedy = race is None or 0.0 <= heat < 2.0 ** -60
        self.probs, self.close, stands = np.zeros(n), np.zeros(n, bool), np.zeros(n, bool)
        self.rows = []
        for i in range(n):
            x = tokens[i + 1] if i + 1 < n else -1
            some = 0 <= x < vocab
            none = np.isnan(z[i]).any() or z[i].max() == -np.inf
            if not self.greedy:
                none = none or np.isposinf(z[i]).any() or not 0.0 <= heat <= 2.0 ** 40
            if none:
                self.rows.append(None)
                continue
            if self.greedy:
                top = int(z[i].argmax())
                self.rows.append(top)
                if some:
                    self.probs[i] = stands[i] = x == top
                continue
            p = np.exp((z[i] - z[i].max()) / heat)
            p /= p.sum()
            self.rows.append(p)
            if some:
                self.probs[i] = p[x]
                border = u[i] * (1.0 if q is None else float(q[i][x]))
                stands[i] = border < p[x]
                self.close[i] = abs(border - p[x]) <= TOL * p[x]
        self.stands = stands
        self.accepted = 1 + int(np.argmin(stands))  # (the last row's never stands)
        self.next = self.draw(self.accepted - 1)

    def weights(self, i):
        p, x = self.rows[i], self.tokens[i + 1] if i + 1 < self.n else -1
        w = p.copy()
        if 0 <= x < len(p):
            if self.q is None:
                w[x] = 0.0
            else:
                w = np.maximum(p - np.asarray(self.q[i], np.float64), 0.0)
        return w if w.max() > 0 else p

    def draw(self, i):
        if self.rows[i] is None:
            return -1
        if self.greedy:
            return self.rows[i]
        with np.errstate(divide="ignore"):
            r = self.weights(i) / self.race
        return int(r.argmax())

    def allows(self, accepted, following):
        """Whether a kernel in fp32 may answer this.  A term 2^x of a row's sum is off by 2^-22 (the
        exponential) and by x's rounding, 2^-24 |x| ln 2, which for terms that matter (|x| < 40) is 2^-19 at most
        and for those that make most of the sum (|x| < 16) below 2^-20.5; signs alternate.  So p is
        known to 2^-20 or so, w = p - q to that of p, and a ratio to 2^-21 more."""
        i = accepted - 1
        if not 0 <= i < self.n or not all(s or c for s, c in zip(self.stands[:i], self.close[:i])):
            return False
        if self.stands[i] and not self.close[i]:
            return False
        if self.greedy or self.rows[i] is None:
            return following == self.draw(i)
        if not 0 <= following < len(self.rows[i]):
            return False
        w, p = self.weights(i), self.rows[i]
        slack = 2 * TOL * p  # (the kernel's terms and its sum)
        high, low = (w + slack) / self.race * (1 + 2.0 ** -21), np.maximum(w - slack, 0) / self.race * (1 - 2.0 ** -21)
        return bool(w[following] > 0 or self.q is not None) and bool(high[following] >= low.max())
