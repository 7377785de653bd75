"""The losses on logits in 64 bits, written from their formulas with numpy, one row or pair at a time.

Every function takes plain arrays and returns the values per row or pair, the total and the gradient of the total."""
import numpy as np


def softmax_row(z, s):
    """(lse, log p, H) of one row of logits; a row of which every logit is -infinity has no distribution: (-inf, -infs, 0).
    (log p from differences to the maximum: at the type's lowest value lse alone, in any number of bits here, says nothing.)"""
    u = np.asarray(z, dtype=np.float64) * s
    m = u.max()
    if m == -np.inf:
        return -np.inf, u, 0.0
    with np.errstate(invalid="ignore"):
        lp = u - m
        log_sum = np.log(np.exp(lp).sum())
        lp -= log_sum
        p = np.exp(lp)
        H = -np.sum(p[p > 0] * lp[p > 0]) if not np.isnan(log_sum) else np.nan
    return m + log_sum, lp, H


def token_logprob(z, labels, s):
    """logp, lse, H of every row"""
    out = np.zeros((3, len(labels)))
    for r, y in enumerate(labels):
        if y < 0:
            continue
        lse, lp, H = softmax_row(z[r], s)
        out[:, r] = lp[y] if y < z.shape[1] else np.nan, lse, H
    return out


def token_grad(z, labels, s, d_logp, d_entropy=None):
    g = np.zeros(z.shape)
    for r, y in enumerate(labels):
        if y < 0:
            continue
        lse, lp, H = softmax_row(z[r], s)
        if lse == -np.inf:
            continue
        p = np.exp(lp)
        g[r] = -d_logp[r] * p
        g[r, y] += d_logp[r]
        if d_entropy is not None:
            kept = p > 0
            g[r, kept] -= d_entropy[r] * p[kept] * (lp[kept] + H)
        g[r] *= s
    return g


def kl_term(kind, d):
    """(KL, its derivative) at d = logp - ref"""
    if kind == "k1":
        return d, 1.0
    if kind == "k2":
        return 0.5 * d * d, d
    return np.expm1(-d) + d, -np.expm1(-d)


def policy(z, labels, old, adv, ref, weight, s, low, high, kl_coef, kl_kind, entropy_coef, scale):
    """(total, losses, logp, H, gradient)"""
    n = len(labels)
    loss, logps, ent, grad = np.zeros(n), np.zeros(n), np.zeros(n), np.zeros(z.shape)
    for r, y in enumerate(labels):
        if y < 0 or weight[r] == 0:
            continue
        lse, lp, H = softmax_row(z[r], s)
        logp, p = lp[y], np.exp(lp)
        ratio = np.exp(logp - old[r])
        whole, held = ratio * adv[r], min(max(ratio, 1 - low), 1 + high) * adv[r]
        loss[r] = -min(whole, held)
        slope = -whole if whole <= held else 0.0
        if kl_coef:
            kl, dkl = kl_term(kl_kind, logp - ref[r])
            loss[r] += kl_coef * kl
            slope += kl_coef * dkl
        loss[r] -= entropy_coef * H
        logps[r], ent[r] = logp, H
        if lse == -np.inf:
            continue
        g = -slope * p
        g[y] += slope
        kept = p > 0
        g[kept] += entropy_coef * p[kept] * (lp[kept] + H)
        grad[r] = g * weight[r] * scale * s
    return scale * np.sum(np.where(weight != 0, weight, 0) * np.where(weight != 0, loss, 0)), loss, logps, ent, grad


def distill(z, index, a, teacher_lse, weight, s, scale):
    """(total, losses, gradient)"""
    n, vocab = z.shape
    loss, grad = np.zeros(n), np.zeros(z.shape)
    for r in range(n):
        if weight[r] == 0:
            continue
        entries = [(int(j), float(v)) for j, v in zip(index[r], a[r]) if j >= 0 and v != -np.inf]
        lse, lp, _ = softmax_row(z[r], s)
        p = np.exp(lp)
        if not entries and teacher_lse is None:
            continue
        t = np.array([v * s for _, v in entries])
        if teacher_lse is None:
            q = np.exp(t - t.max())
            logq = t - t.max() - np.log(q.sum())
        else:
            logq = t - teacher_lse[r] if entries else np.zeros(0)
        q = np.exp(logq)
        if lse == -np.inf:
            loss[r] = np.inf if entries else 0.0
            continue
        full = np.zeros(vocab)
        for (j, _), qk, lq in zip(entries, q, logq):
            full[j] += qk
            if qk > 0:
                loss[r] += qk * (lq - lp[j])
        g = p - full if entries else np.zeros(vocab)
        if teacher_lse is not None:
            inside = np.zeros(vocab, dtype=bool)
            inside[[j for j, _ in entries]] = True
            rest = max(0.0, 1.0 - q.sum()) if not inside.all() else 0.0
            u = lp[~inside]
            if u.size and u.max() > -np.inf:
                tail = u.max() + np.log(np.exp(u - u.max()).sum())
                if rest > 0:
                    loss[r] += rest * (np.log(rest) - tail)
                g = p - full
                g[~inside] = p[~inside] - rest * np.exp(u - tail)
            else:
                g = p - full
                if rest > 0:
                    loss[r] = np.inf
        grad[r] = g * weight[r] * scale * s
    return scale * np.sum(np.where(weight != 0, weight, 0) * np.where(weight != 0, loss, 0)), loss, grad


def pair_loss(kind, d, beta, smoothing):
    if kind == "sigmoid":
        softplus = lambda x: np.logaddexp(0.0, x)  # noqa: E731
        return (1 - smoothing) * softplus(-d) + smoothing * softplus(d)
    if kind == "hinge":
        return max(0.0, 1.0 - d)
    return ((d - 0.5) / beta) ** 2


def pair_slope(kind, d, beta, smoothing):
    if kind == "sigmoid":
        return -(1 - smoothing) / (1 + np.exp(d)) + smoothing / (1 + np.exp(-d))
    if kind == "hinge":
        return -1.0 if d < 1 else 0.0
    return 2 * (d - 0.5) / beta ** 2


def preference(logp, ref, offsets, mask, weight, beta, kind, smoothing, margin, normalised, scale):
    """(total, losses, rewards, gradient)"""
    pairs = len(offsets) // 2
    T = len(logp)
    kept = np.ones(T, dtype=bool) if mask is None else np.asarray(mask, dtype=bool)
    diff = np.where(kept, np.asarray(logp, dtype=np.float64) - (0.0 if ref is None else np.asarray(ref, dtype=np.float64)), 0.0)
    R, n = np.zeros(2 * pairs), np.ones(2 * pairs)
    for i in range(2 * pairs):
        span = slice(offsets[i], offsets[i + 1])
        count = kept[span].sum()
        if normalised and count:
            n[i] = count
        R[i] = beta * diff[span].sum() / n[i]
    grad, losses = np.zeros(T), np.zeros(pairs)
    for i in range(pairs):
        d = R[i] - R[pairs + i] - margin
        losses[i] = pair_loss(kind, d, beta, smoothing)
        g = pair_slope(kind, d, beta, smoothing) * weight[i] * scale * beta
        for k, sign in ((i, 1.0), (pairs + i, -1.0)):
            span = slice(offsets[k], offsets[k + 1])
            grad[span] = np.where(kept[span], sign * g / n[k], 0.0)
    return scale * np.sum(weight * losses), losses, R, grad
