"""Products with 4-bit weights, drawn tokens and verified drafts in 64 bits, written from their definitions with numpy, one row or request
at a time."""
import numpy as np


def weights(codes, scale, zero, cols, group):
    """the matrix that codes, scales and zeros stand for"""
    codes = np.asarray(codes)
    w = np.zeros((codes.shape[0], cols))
    for j in range(cols):
        code = (codes[:, j // 2] >> (4 * (j % 2))) & 15
        g = j // group
        w[:, j] = scale[:, g] * (code - (8.0 if zero is None else zero[:, g]))
    return w


def quantized(w, group, symmetric, to_scale):
    """(codes as whole numbers, scale, zero) of a matrix; to_scale: rounding to the scales' type"""
    rows, cols = w.shape
    groups = -(-cols // group)
    q, scale, zero = np.zeros((rows, cols), dtype=np.int64), np.zeros((rows, groups)), np.zeros((rows, groups))
    for r in range(rows):
        for g in range(groups):
            part = w[r, g * group:(g + 1) * group].astype(np.float64)
            low, high = min(0.0, part.min()), max(0.0, part.max())
            s = to_scale(max(high, -low) / 7 if symmetric else (high - low) / 15)
            scale[r, g] = s
            z = 8.0 if symmetric else (np.clip(np.rint(-low / s), 0, 15) if s > 0 else 0.0)
            zero[r, g] = z
            q[r, g * group:(g + 1) * group] = np.clip((np.rint(part / s) if s > 0 else 0) + z, 0, 15)
    return q, scale, zero


def log_softmax(z, s):
    """log p of a row, or None where it has no distribution"""
    u = np.asarray(z, dtype=np.float64) * s
    if np.isnan(u).any() or (u == np.inf).any() or (u == -np.inf).all():
        return None
    u = u - u.max()
    return u - np.log(np.exp(u).sum())


def number(u):
    return min(max(float(u), 0.0), 1 - 2.0 ** -24)


def pick(mass, u):
    """the first entry whose running sum passes u of the whole"""
    running = np.cumsum(mass)
    j = int(np.searchsorted(running, number(u) * running[-1], side="right"))
    return min(j, int(np.nonzero(mass)[0][-1]))


def room(mass, j, u):
    """How far u of the whole is inside entry j's part of the running sum (negative: outside); none for an entry that has no part."""
    if not 0 <= j < len(mass) or not mass[j] > 0:
        return -np.inf
    running = np.cumsum(mass)
    at = number(u) * running[-1]
    last = j == np.nonzero(mass)[0][-1]
    return min(np.inf if last else running[j] - at, at - running[j - 1] if j else np.inf)


def draw(z, u, s):
    """(token, its log-probability, p) of a row"""
    lp = log_softmax(z, s)
    if lp is None or np.isnan(u):
        return -1, np.nan, None
    p = np.exp(lp)
    j = pick(p, u)
    return j, lp[j], p


def verify(z, drafted, u, v, s, draft=None, draft_logp=None, length=None, sq=1.0):
    """(tokens, logp, mass, log p, near) of a request: z (drafts + 1, vocab), draft (drafts, vocab) or None.  mass: what the last token is drawn
    from, and log p there (None: there is none); near: how near a decision was, as a share of q."""
    drafts, vocab = len(drafted), z.shape[1]
    n = drafts if length is None else min(int(length), drafts)
    if n < 0:
        return [], [], None, None, np.inf
    tokens, logp, near = [], [], np.inf
    for t in range(n + 1):
        lp = log_softmax(z[t], s)
        if t == n:
            mass = None
            break
        x = int(drafted[t])
        q = np.zeros(vocab)
        if 0 <= x < vocab:
            if draft is None:
                q[x] = 1.0
            elif draft_logp is None:
                lq = log_softmax(draft[t], sq)
                q = q if lq is None else np.exp(lq)
            elif np.isfinite(draft[t, x]) and np.exp(np.float64(draft_logp[t])) > 0 and np.isfinite(draft_logp[t]):
                q = np.exp((draft[t].astype(np.float64) - float(draft[t, x])) * sq + float(draft_logp[t]))
        if lp is None:
            mass = None
            break
        p = np.exp(lp)
        if 0 <= x < vocab and q[x] > 0:
            near = min(near, abs(u[t] * q[x] - p[x]) / q[x])
            if u[t] * q[x] < p[x]:
                tokens.append(x)
                logp.append(lp[x])
                continue
        mass = np.maximum(p - q, 0.0)
        if not (np.isfinite(q).all() and mass.sum() > 0):
            mass = None
        break
    if lp is None or np.isnan(v):
        return tokens + [-1], logp + [np.nan], None, None, near
    mass = np.exp(lp) if mass is None else mass
    j = pick(mass, v)
    return tokens + [j], logp + [lp[j]], mass, lp, near
