"""Plain statements, in 64 bits on the host, of the post-training operators
(numpy; no code shared with the library), with bounds of what 32-bit arithmetic
may be off them by. Test infrastructure only.

Bounds. u = 2^-24. A row's logp is a difference of s (x_y - m), off by 2u of its
size, and log S. S sums V exponentials, each off by 2^-22 of itself (the
hardware's 2^x) and by its exponent's error, 2u times an exponent that weighs in
at no more than about 30 bits (what lies lower is below 2^-30 of the sum): 3e-6;
and by the additions' rounding, some 300 of them in sequence a thread, u each and
of either sign: 20 u, four deviations 5e-6. LOGP = 1e-5 + 2u |logp| covers them.
p_v = 2^(c (x_v - m) - log2 S) is off by its exponent's 3u |exponent| (the smallest
float has exponent -126: 2.3e-5) and by LOGP: P = 4e-5 of itself, and below
2^-126 it may be 0. The gradient's rounding to its type comes on top: half a unit
in the last place, 2^-8 (bfloat16, 8 significant bits) or 2^-11 (half, at least 2^-25) of itself.
"""
import numpy as np

LOGP, P = 1e-5, 4e-5
U = 2.0 ** -24
ROUND = {"f32": (U, 0.0), "bf16": (2.0 ** -8, 0.0), "f16": (2.0 ** -11, 2.0 ** -25)}


def log_softmax(x, scale):
    """Rows of log probabilities; a row of -inf alone stays -inf."""
    z = x.astype(np.float64) * scale
    m = z.max(1, keepdims=True)
    m = np.where(np.isneginf(m), 0.0, m)
    with np.errstate(divide="ignore", invalid="ignore"):
        s = np.exp(z - m).sum(1, keepdims=True)
        out = z - m - np.log(s)
    out[np.isneginf(z).all(1)] = -np.inf
    return out


def token_logp(x, y, scale):
    lp = log_softmax(x, scale)
    return np.where(y >= 0, lp[np.arange(len(y)), np.maximum(y, 0)], 0.0)


def gradient(x, y, coef, scale):
    """d/dx of sum_r coef_r logp_r."""
    p = np.exp(log_softmax(x, scale))
    d = -p * (coef * scale)[:, None]
    d[np.arange(len(y)), np.maximum(y, 0)] += coef * scale
    empty = np.isneginf(x.astype(np.float64)).all(1)
    d[(y < 0) | (coef == 0) | empty] = 0.0
    return d


def gradient_bound(x, y, coef, dcoef, scale, kind):
    """What a 32-bit gradient with slopes off by dcoef may be off `gradient` by."""
    p = np.exp(log_softmax(x, scale))
    k, dk = np.abs(coef * scale)[:, None], np.abs(dcoef * scale)[:, None]
    away = p.copy()                                    # |[v = y] - p|
    at = np.arange(len(y)), np.maximum(y, 0)
    away[at] = 1 - p[at]
    off = dk * away + k * (P * p + 2.0 ** -126)
    off[at] += (k * (2 * LOGP + 4 * U))[:, 0]          # 1 - p_y is off by p_y times logp's error
    rel, low = ROUND[kind]
    return off + rel * (k * away + off) + low


def policy(logp, y, old, adv, w, ref, lo, hi, kl):
    """(loss, token losses, slopes in logp times the weight) from the rows' logp."""
    counts = (y >= 0) & (w != 0) & ~np.isneginf(logp)
    ratio = np.exp(np.where(counts, logp - old, 0.0))
    plain, clipped = ratio * adv, np.clip(ratio, 1 - lo, 1 + hi) * adv
    far = np.where(counts, ref - logp, 0.0) if kl else np.zeros_like(logp)
    each = -np.minimum(plain, clipped) + kl * (np.exp(far) - far - 1)
    slope = -np.where(plain <= clipped, plain, 0.0) + kl * (1 - np.exp(far))
    each, slope = np.where(counts, each, 0.0), np.where(counts, slope, 0.0)
    return (w * each)[counts].sum(), each, np.where(counts, w, 0.0) * slope


def policy_bound(logp, old, adv, ref, kl):
    """Of a token's loss, and of its slope: logp's error through each exponential, and
    the few roundings of the terms (the KL term's three summands may cancel)."""
    d = 2 * LOGP + 2 * U * np.abs(logp) + 8 * U
    ratio = np.exp(logp - old) * np.abs(adv)
    off = ratio * d
    if kl:
        off = off + kl * (np.exp(ref - logp) * (d + 4 * U) + d + 4 * U * (1 + np.abs(ref - logp)))
    return off


def preference(logp, y, off, ref, w, beta, eps, empty):
    """(loss, pair losses, log ratios of the sequences, slope of each row's logp)."""
    pairs = len(off) // 2
    each = np.where((y >= 0) & ~empty, logp - ref, 0.0)
    ratio = np.array([each[off[s]: off[s + 1]].sum() for s in range(2 * pairs)])
    margin = beta * (ratio[0::2] - ratio[1::2])
    loss = (1 - eps) * np.logaddexp(0, -margin) + eps * np.logaddexp(0, margin)
    up, down = 1 / (1 + np.exp(-margin)), 1 / (1 + np.exp(margin))
    slope = w * beta * (eps * up - (1 - eps) * down)
    coef = np.zeros(len(y))
    for s in range(2 * pairs):
        coef[off[s]: off[s + 1]] = slope[s // 2] * (-1 if s % 2 else 1)
    return (w * loss).sum(), loss, ratio, np.where(y >= 0, coef, 0.0)


def dropout_bits(seed, t, worker, site, n):
    """16 bits of SplitMix64's stream for each of n elements, Python integers."""
    mask, gamma = (1 << 64) - 1, 0x9E3779B97F4A7C15

    def mix(z):
        z &= mask
        z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & mask
        z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & mask
        return z ^ (z >> 31)

    key = seed ^ 0x44524F504F555421
    for number in (t, worker + 1, site):
        key = mix(key + gamma * (number + 1))
    out = []
    for i in range((n + 3) // 4):
        z = mix(key + gamma * (i + 1))
        out += [z & 0xFFFF, (z >> 16) & 0xFFFF, (z >> 32) & 0xFFFF, z >> 48]
    return np.array(out[:n], np.int64)
