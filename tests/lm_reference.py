"""The language-model operators' definitions in 64 bits (CPU), and the rounding
that their kernels may add.  A rounding to 32 bits is off by 2^-24 of a value at
the most, one to bfloat16 by 2^-8."""

import numpy as np

EPS = 2.0 ** -24
BF16 = 2.0 ** -8
# n independent roundings of values a_i, each within e |a_i| and of mean 0, stay within
# 8 e sqrt(sum a_i^2) but once in 10^12 (Hoeffding: 2 exp(-8^2 / 2))
SPREAD = 8.0


def out_rounding(ref, bf16):
    return (BF16 if bf16 else EPS) * np.abs(ref)


class Vocab:
    """Log-probabilities, loss and gradients of rows with a target; hidden and weight
    are float64, idle rows of hidden are not looked at."""

    def __init__(self, hidden, weight, t, share=None, mean=True):
        on = t >= 0
        if share is not None:
            on &= share != 0
        self.on, self.h, self.w = on, np.where(on[:, None], hidden, 0.0), weight
        self.t = np.clip(t, 0, len(weight) - 1)
        rows = np.arange(len(t))
        x = self.h @ weight.T
        # products are exact, sums of `width` of them in any order; float32 products leave
        # out planes below 2^-26 of a product and add six sums
        self.dx = (weight.shape[1] + 16) * EPS * (np.abs(self.h) @ np.abs(weight).T)
        top = x.max(1, keepdims=True)
        e = np.exp(x - top)
        s = e.sum(1, keepdims=True)
        self.p = e / s
        spread = np.where(e > 1e-12, top - x, 0.0).max(1)
        self.logp = np.where(on, x[rows, self.t] - top[:, 0] - np.log(s[:, 0]), 0.0)
        # exponentials' arguments, their partial sums, the logarithm: as for logits in memory
        self.own = EPS * (32 + 4 * spread + 2 * np.abs(self.logp))
        self.logp_tol = np.where(on, 2 * self.dx.max(1) + self.own, 0.0)
        w = np.where(on, 1.0 if share is None else share, 0.0)
        self.total = w.sum()
        self.share = w / self.total if mean and self.total else w
        self.loss = -(self.share * self.logp).sum()
        self.loss_tol = (np.abs(self.share) * (self.logp_tol + 4 * EPS * np.abs(self.logp))).sum() + 4 * EPS * abs(self.loss)

    def gradients(self, g, bf16_in, bf16_hidden, bf16_weight):
        """((grad_hidden, tolerance), (grad_weight, tolerance)) for dL/dlogp = g."""
        g = np.where(self.on, g, 0.0)
        G = -g[:, None] * self.p
        G[np.arange(len(g)), self.t] += g
        rel = 2 * self.dx.max(1, keepdims=True) + EPS * 40 + self.own[:, None]
        dG = np.abs(g)[:, None] * self.p * rel + 4 * EPS * np.abs(G)
        out = []
        for left, dl, right, bf16 in ((G, dG, self.w, bf16_hidden), (G.T, dG.T, self.h, bf16_weight)):
            ref = left @ right
            tol = dl @ np.abs(right) + (right.shape[0] + 16) * EPS * (np.abs(left) @ np.abs(right))
            if bf16_in:   # each value of G is rounded to bfloat16 on its way into the product, and where the
                # exponentials are kept they are too: 2 n roundings for n values, sqrt(2) of the spread of n
                tol += SPREAD * BF16 * np.sqrt(2.0 * (left ** 2 @ right ** 2))
            out.append((ref, tol + out_rounding(ref, bf16) + 4 * EPS * np.abs(ref) + 1e-37))
        return out


# additions of a row's values that follow one another in any lane, and across the lanes
SUM = 128


class Norm:
    def __init__(self, x, w, b, eps):
        n = x.shape[1]
        self.x, self.w = x, np.ones(n) if w is None else w
        b = np.zeros(n) if b is None else b
        mean = x.mean(1, keepdims=True)
        d = x - mean
        var = (d ** 2).mean(1, keepdims=True)
        self.mean, self.rstd = mean, 1 / np.sqrt(var + eps)
        self.u = d * self.rstd
        self.y = self.u * self.w + b
        # the mean's sum and its product with 1 / n; the variance's with the mean's error in
        # every difference; the square root, quotient and products
        self.dmean = (SUM + 4) * EPS * np.abs(x).mean(1, keepdims=True)
        dvar = 2 * self.dmean * np.abs(d).mean(1, keepdims=True) + self.dmean ** 2 + (SUM + 8) * EPS * var
        self.rel = 0.5 * dvar * self.rstd ** 2 * 1.01 + 6 * EPS
        self.du = self.rstd * (self.dmean + 2 * EPS * np.abs(d)) + np.abs(self.u) * (self.rel + 2 * EPS)
        self.y_tol = np.abs(self.w) * self.du + 3 * EPS * (np.abs(self.u * self.w) + np.abs(self.y) + np.abs(b)) + 1e-37

    def backward(self, g):
        """{name: (value, tolerance before the last rounding)}"""
        a, u, rstd = g * self.w, self.u, self.rstd
        n, rows = self.x.shape[1], self.x.shape[0]
        m1, m2 = a.mean(1, keepdims=True), (a * u).mean(1, keepdims=True)
        gx = rstd * (a - m1 - u * m2)
        d1 = (SUM + 6) * EPS * np.abs(a).mean(1, keepdims=True)
        d2 = (np.abs(a) * self.du).mean(1, keepdims=True) + (SUM + 8) * EPS * np.abs(a * u).mean(1, keepdims=True)
        gx_tol = rstd * (6 * EPS * (np.abs(a) + np.abs(m1) + np.abs(u * m2)) + d1 + np.abs(u) * d2 + self.du * np.abs(m2)) + \
            np.abs(gx) * self.rel
        gw, gb = (g * u).sum(0), g.sum(0)
        gw_tol = (np.abs(g) * self.du).sum(0) + (rows + 16) * EPS * np.abs(g * u).sum(0)
        gb_tol = (rows + 16) * EPS * np.abs(g).sum(0)
        return {"grad_x": (gx, gx_tol + 1e-37), "grad_weight": (gw, gw_tol + 1e-37), "grad_bias": (gb, gb_tol + 1e-37)}


def embedding(tokens, w, scale):
    rows = scale * w[np.clip(tokens, 0, len(w) - 1)]
    rows[tokens < 0] = 0.0
    rows[tokens >= len(w)] = np.nan
    return rows


def embedding_gradient(tokens, g, classes, scale):
    """(gradient, tolerance before the last rounding)"""
    on = (tokens >= 0) & (tokens < classes)
    out, size, count = np.zeros((classes, g.shape[1])), np.zeros((classes, g.shape[1])), np.zeros(classes)
    np.add.at(out, tokens[on], g[on])
    np.add.at(size, tokens[on], np.abs(g[on]))
    np.add.at(count, tokens[on], 1)
    return scale * out, (count[:, None] + 4) * EPS * abs(scale) * size
