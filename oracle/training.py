"""The training steps in 64 bits: token log-probabilities, the clipped policy loss
with a KL term, the paired log-ratio preference loss, their gradients with respect
to the logits, and AdamW with 32-bit or 8-bit block-scaled states.

Written from the formulas, one token and one block at a time; shares no code with
the kernels.
"""
import numpy as np


def slots(n_examples, T, n_rows, V, target, weight=None, row_offset=None, length=None):
    """(example, token, row, counts) of every token slot whose outputs are written."""
    got = []
    for i in range(n_examples):
        n = T if length is None else min(max(int(length[i]), 0), T)
        for t in range(T):
            row = i * T + t if row_offset is None else int(row_offset[i]) + t
            if not 0 <= row < n_rows or (row_offset is not None and t >= n):
                continue
            counts = t < n and 0 <= int(target[row]) < V and (weight is None or weight[row] != 0)
            got.append((i, t, row, bool(counts)))
    return got


def log_softmax(z, scale):
    """scale * (z - max) less the logarithm of its exponentials' sum; NaN where the row holds NaN, +inf, or nothing."""
    with np.errstate(invalid="ignore", divide="ignore"):
        x = scale * (np.asarray(z, np.float64) - np.max(z))
        return x - np.log(np.exp(x).sum())


def _d_row(lp, y, c, scale):
    d = -np.exp(lp) * c
    d[y] += c
    return scale * d


def token_logp(logits, target, n_examples, T, scale=1.0, **where):
    logits = np.asarray(logits, np.float64)
    out = {}
    for _, _, row, counts in slots(n_examples, T, *logits.shape, target, **where):
        out[row] = log_softmax(logits[row], scale)[target[row]] if counts else 0.0
    return out


def policy_loss(logits, target, n_examples, T, advantage, scale=1.0, weight=None, row_offset=None, length=None,
                logp_old=None, logp_ref=None, per_token=False, clip_low=0.2, clip_high=0.2, beta=0.0):
    """(loss [n_examples], {row: logp}, {row: dlogits})."""
    logits = np.asarray(logits, np.float64)
    loss, logp, grad = np.zeros(n_examples), {}, {}
    for i, _, row, counts in slots(n_examples, T, *logits.shape, target, weight, row_offset, length):
        if not counts:
            logp[row], grad[row] = 0.0, np.zeros(logits.shape[1])
            continue
        lps = log_softmax(logits[row], scale)
        lp = logp[row] = lps[target[row]]
        w = 1.0 if weight is None else float(weight[row])
        a = float(advantage[row if per_token else i])
        ratio = np.exp(lp - float(logp_old[row])) if logp_old is not None else 1.0
        free, held = -a * ratio, -a * min(max(ratio, 1 - clip_low), 1 + clip_high)
        value, c = max(free, held), free if free >= held else 0.0
        if beta != 0:
            d = float(logp_ref[row]) - lp
            value += beta * (np.inf if d == np.inf else np.expm1(d) - d)
            c -= beta * np.expm1(d)
        loss[i] += w * value
        grad[row] = _d_row(lps, target[row], w * c, scale)
    return loss, logp, grad


def preference_loss(logits, target, n_examples, T, scale=1.0, weight=None, row_offset=None, length=None,
                    logp_ref=None, pair_weight=None, beta=0.1, margin=0.0, label_smoothing=0.0):
    """(loss [n_pairs], log_ratio [n_examples], {row: logp}, {row: dlogits})."""
    logits = np.asarray(logits, np.float64)
    n_pairs, e = n_examples // 2, label_smoothing
    ratio, logp, rows = np.zeros(n_examples), {}, {}
    for i, _, row, counts in slots(n_examples, T, *logits.shape, target, weight, row_offset, length):
        logp[row], rows[row] = 0.0, (i, None, 0.0)
        if counts:
            lps = log_softmax(logits[row], scale)
            logp[row] = lps[target[row]]
            w = 1.0 if weight is None else float(weight[row])
            ratio[i] += w * (logp[row] - (0.0 if logp_ref is None else float(logp_ref[row])))
            rows[row] = (i, lps, w)
    h = beta * (ratio[:n_pairs] - ratio[n_pairs:]) - margin
    pw = np.ones(n_pairs) if pair_weight is None else np.asarray(pair_weight, np.float64)[:n_pairs]
    loss = np.where(pw == 0, 0.0, pw * ((1 - e) * np.logaddexp(0, -h) + e * np.logaddexp(0, h)))
    dh = np.where(pw == 0, 0.0, pw * beta * (e / (1 + np.exp(-h)) - (1 - e) / (1 + np.exp(h))))
    grad = {}
    for row, (i, lps, w) in rows.items():
        c = w * (dh[i] if i < n_pairs else -dh[i - n_pairs])
        grad[row] = np.zeros(logits.shape[1]) if lps is None or c == 0 else _d_row(lps, target[row], c, scale)
    return loss, ratio, logp, grad


# ----------------------------------------------------------------------------
# AdamW
# ----------------------------------------------------------------------------
#: The nonnegative values of the 8-bit format in the order of their codes: three mantissa
#: bits, exponents from 2^-6, steps of 2^-9 below it, 448 the largest.
E4M3 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)])


def e4m3(x):
    """Nearest value of the 8-bit format, ties to the even code."""
    a = np.abs(np.asarray(x, np.float64))
    hi = np.clip(np.searchsorted(E4M3, a), 1, 126)
    lo = hi - 1
    up = (a - E4M3[lo] > E4M3[hi] - a) | ((a - E4M3[lo] == E4M3[hi] - a) & (hi % 2 == 0))
    return np.sign(x) * np.where(up, E4M3[hi], E4M3[lo])


def blocks(x, root=False):
    """(values of the 8-bit format, scales) of x in blocks of 256."""
    q, scales = np.zeros(len(x)), []
    for b in range(0, len(x), 256):
        part = np.asarray(x[b:b + 256], np.float64)
        amax = max(np.abs(part).max(), 2.0 ** -100)
        y = part * (448.0 / amax)
        q[b:b + 256] = e4m3(y)
        if root:
            q[b:b + 256] = np.where(y > 0, np.maximum(q[b:b + 256], 2.0 ** -9), q[b:b + 256])
        scales.append(amax / 448.0)
    return q, np.array(scales)


def adamw(x, g, m, v, step, lr, beta1, beta2, eps, eps_root=0.0, weight_decay=0.0, grad_scale=1.0):
    """(x, m, v) after one step, from and to unquantised states."""
    g = np.asarray(g, np.float64) * grad_scale
    m = beta1 * np.asarray(m, np.float64) + (1 - beta1) * g
    v = beta2 * np.asarray(v, np.float64) + (1 - beta2) * g * g
    x = np.asarray(x, np.float64)
    new = x - lr * weight_decay * x - lr * (m / (1 - beta1 ** step)) / (
        np.sqrt(v / (1 - beta2 ** step) + eps_root) + eps)
    return new, m, v
