"""The training operators' definitions in 64 bits (CPU), and the rounding that
32-bit kernels may add to them."""

import numpy as np

EPS = 2.0 ** -24
BF16 = 2.0 ** -8      # twice half a unit in the last place of bfloat16, relative
BLOCK, TOP, TINY = 256, 448.0, 2.0 ** -9


def rows(x, t):
    """(p, logp, entropy, spread) of float64 logits; spread: the largest |x_j - M|
    of a class that counts."""
    with np.errstate(all="ignore"):
        top = x.max(1, keepdims=True)
        d = x - top
        e = np.exp(d)
        s = e.sum(1, keepdims=True)
        p = e / s
        logp = d[np.arange(len(x)), np.clip(t, 0, x.shape[1] - 1)] - np.log(s[:, 0])
        entropy = np.log(s[:, 0]) - np.where(p > 0, p * d, 0.0).sum(1)
        spread = np.where(e > 1e-12, -d, 0.0).max(1)
    return p, logp, entropy, spread


def gradient(p, entropy, t, g, h):
    log_p = np.log(np.where(p > 0, p, 1.0))
    y = -p * (g[:, None] + h[:, None] * (log_p + entropy[:, None]))
    y[np.arange(len(p)), t] += g
    return y


def logp_tolerance(logp, spread):
    """x_t - M and log S are rounded (|logp| + spread + log S units), S is a sum
    of exponentials whose arguments were rounded (up to 2 spread units each) and
    whose partial sums were (under 32)."""
    return EPS * (32 + 4 * spread + 2 * np.abs(np.where(np.isfinite(logp), logp, 0.0)))


def gradient_tolerance(p, ref, entropy, spread, t, g, h, bf16):
    """p carries the relative error of an exponential and of S; the target's
    value is a difference of g and g p; bfloat16 rounds once more."""
    size = np.abs(g)[:, None] + np.abs(h)[:, None] * (spread + np.abs(entropy) + 1)[:, None]
    tol = EPS * (32 + 4 * spread)[:, None] * p * size
    tol[np.arange(len(p)), t] += 4 * EPS * np.abs(g)
    return tol + (BF16 * np.abs(ref) if bf16 else 0.0) + 1e-38


def policy(p, logp, entropy, on, old, ref, adv, w, clip, kl_coef, entropy_coef, mean):
    """(stats, g, h) of the policy loss."""
    w = np.where(on, w, 0.0)
    total = w.sum()
    if mean:
        w = w / total if total else w
    lp = np.where(on, logp, 0.0)
    ratio = np.exp(np.where(on, lp - old, 0.0))
    free, bound = ratio * adv, np.clip(ratio, 1 - clip[0], 1 + clip[1]) * adv
    cut = bound < free
    pol = -np.minimum(free, bound)
    k = np.where(on, ref - lp, 0.0) if ref is not None else np.zeros_like(lp)
    kl = np.expm1(k) - k
    loss = pol + kl_coef * kl - entropy_coef * entropy
    keep = w != 0
    stats = np.array([(w[keep] * v[keep]).sum() for v in (loss, pol, kl, entropy, cut.astype(float), ratio)])
    g = np.where(keep, w * (np.where(cut, 0.0, -free) - kl_coef * np.expm1(k)), 0.0)
    return stats, g, np.where(keep, -entropy_coef * w, 0.0)


def preference(logp, on, offsets, ref, beta, smoothing):
    """(stats, g) of the preference loss."""
    reward = []
    for a, b in zip(offsets[:-1], offsets[1:]):
        r = np.arange(a, b)
        r = r[on[a:b]]
        reward.append(beta * (logp[r] - ref[r]).sum())
    reward = np.array(reward)
    good, bad = reward[0::2], reward[1::2]
    m = good - bad
    g = np.zeros(len(logp))
    if len(m) == 0:
        return np.zeros(5), g
    loss = (1 - smoothing) * np.logaddexp(0, -m) + smoothing * np.logaddexp(0, m)
    slope = (smoothing / (1 + np.exp(-m)) - (1 - smoothing) / (1 + np.exp(m))) * beta / len(m)
    for s, (a, b) in enumerate(zip(offsets[:-1], offsets[1:])):
        g[a:b] = slope[s // 2] * (1 if s % 2 == 0 else -1)
    return np.array([v.mean() for v in (loss, (m > 0).astype(float), m, good, bad)]), np.where(on, g, 0.0)


def adamw(w, g, m, v, step, lr, betas, eps, decay):
    """(w, m, v) after a step, and the size of the step itself."""
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    move = lr * m / (1 - betas[0] ** step) / (np.sqrt(v / (1 - betas[1] ** step)) + eps)
    return w * (1 - lr * decay) - move, m, v, np.abs(move)


def block_scale(x):
    """Scale of each element's block of 256."""
    n = len(x)
    pad = np.zeros(-(-n // BLOCK) * BLOCK)
    pad[:n] = np.abs(x)
    return pad.reshape(-1, BLOCK).max(1) / TOP
