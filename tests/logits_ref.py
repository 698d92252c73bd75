"""Plain 64-bit versions of the operators on rows of logits, one row at a time (numpy)."""
import numpy as np


def lse(y):
    m = np.max(y)
    return m if np.isneginf(m) else m + np.log(np.sum(np.exp(y - m)))


def top(z, k):
    """ids of the k largest: NaN first, then by value, the lower column first."""
    z = np.asarray(z, dtype=np.float64)
    nan = np.isnan(z)
    return np.lexsort((np.arange(z.size), -np.where(nan, 0.0, z), ~nan))[:k].astype(np.int32)


def valid_entries(ids, vocab):
    """Places of the entries that count: in range, and the first of their id."""
    seen, keep = set(), []
    for i, c in enumerate(ids):
        if 0 <= c < vocab and int(c) not in seen:
            seen.add(int(c))
            keep.append(i)
    return np.asarray(keep, dtype=np.int64)


def rest_of(p, qR, t_lse):
    """The teacher's rest; nothing where the student has none and it is no more than rounding t_lse to f32 leaves."""
    pR = max(0.0, 1.0 - p.sum())
    return 0.0 if qR == 0 and pR <= 2.0 ** -22 + 2.0 ** -24 * abs(t_lse) else pR


def distill(z, values, ids, t_lse, tau, kl_share, eta, w):
    """One row: loss, alpha, gradient, and per column the size of the terms that the gradient is a difference of."""
    z = np.asarray(z, dtype=np.float64)
    V = z.size
    keep = valid_entries(ids, V)
    S = np.asarray(ids)[keep].astype(np.int64)
    t = np.asarray(values, dtype=np.float64)[keep] / tau
    c = (float(t_lse) if t_lse is not None else (lse(t) if t.size else -np.inf))
    y = z / tau
    L = lse(y)
    if w == 0 or np.isneginf(c) or np.isneginf(L):
        return 0.0, 0.0, np.zeros(V), np.zeros(V)
    q = np.exp(y - L)
    R = np.ones(V, dtype=bool)
    R[S] = False
    lqR = lse(y[R]) - L if R.any() else -np.inf
    p = np.exp(t - c)
    pR = rest_of(p, np.exp(lqR), float(t_lse)) if t_lse is not None and R.any() else 0.0
    pb, qb = np.append(p, pR), np.append(q[S], np.exp(lqR))
    lq = np.append(y[S] - L, lqR)
    on = pb > 0
    kl = float(np.sum(pb[on] * (np.log(pb[on]) - lq[on])))
    tv = 0.5 * float(np.sum(np.abs(pb - qb)))
    alpha = float(np.sum(np.minimum(pb, qb)))
    lam = kl_share * np.exp(-eta * alpha)
    s = np.sign(qb - pb)
    mean, mass = float(np.sum(s * qb)), float(pb.sum())
    g = np.zeros(V)
    # p_R / q_R q_j as p_R times the column's share of the rest, which is there when q_R is too small for a number
    taken = pR * np.exp(y[R] - lse(y[R])) if pR > 0 and np.isfinite(lqR) else 0.0
    g[R] = q[R] * (lam * mass + 0.5 * (1 - lam) * (s[-1] - mean)) - lam * taken
    g[S] = q[S] * (lam * mass + 0.5 * (1 - lam) * (s[:-1] - mean)) - lam * p
    size = np.zeros(V)
    size[R] = q[R] + taken
    size[S] = q[S] + p
    loss = (lam * kl if lam > 0 else 0.0) + (1 - lam) * tv
    return w * loss, alpha, w / tau * g, abs(w) / tau * size


def distill_undecided(z, values, ids, t_lse, tau, kl_share, eta, w, d):
    """How far the gradient of each column may move where q and p are closer than rounding decides.  With q off by d
    relative, sign(q - p) is open wherever |q - p| <= 2 d (p + q).  Each such sign moves by at most 2, so its own column by
    2 x (1 - lambda) / 2 x q, and the mean by 2 q, hence every column by (1 - lambda) / 2 x q_j x 2 x (the open q's sum)."""
    z = np.asarray(z, dtype=np.float64)
    V = z.size
    keep = valid_entries(ids, V)
    S = np.asarray(ids)[keep].astype(np.int64)
    t = np.asarray(values, dtype=np.float64)[keep] / tau
    c = (float(t_lse) if t_lse is not None else (lse(t) if t.size else -np.inf))
    y = z / tau
    L = lse(y)
    if w == 0 or not np.isfinite(c) or not np.isfinite(L):
        return np.zeros(V)
    q = np.exp(y - L)
    R = np.ones(V, dtype=bool)
    R[S] = False
    p = np.exp(t - c)
    qR = float(np.sum(q[R]))
    pR = rest_of(p, qR, float(t_lse)) if t_lse is not None and R.any() else 0.0
    pb, qb = np.append(p, pR), np.append(q[S], qR)
    open_ = (np.abs(qb - pb) <= 2 * d * (pb + qb)) & (pb + qb > 0)
    half = 0.5 * (1 - kl_share * np.exp(-eta * float(np.sum(np.minimum(pb, qb)))))
    move = half * q * 2 * float(np.sum(qb[open_]))
    move[S] += np.where(open_[:-1], 2 * half * q[S], 0.0)
    if open_[-1]:
        move[R] += 2 * half * q[R]
    return abs(w) / tau * move


def policy(z, action, adv, old, ref, tau, lo, hi, beta, w):
    """One row: loss, logp, gradient, sizes."""
    z = np.asarray(z, dtype=np.float64)
    V = z.size
    y = z / tau
    L = lse(y)
    if w == 0 or not 0 <= action < V or np.isneginf(L):
        return 0.0, 0.0, np.zeros(V), np.zeros(V)
    logp = y[action] - L
    rho = np.exp(logp - old) if old is not None else 1.0
    free, held = rho * adv, min(max(rho, 1 - lo), 1 + hi) * adv
    loss, g = -min(free, held), -free if free <= held else 0.0
    terms = abs(free)
    if ref is not None:
        d = ref - logp
        loss += beta * (np.expm1(d) - d)
        g -= beta * np.expm1(d)
        terms += beta * (1 + np.exp(d))
    q = np.exp(y - L)
    grad = -q * g
    grad[action] += g
    size = q * terms
    size[action] = terms
    return w * loss, logp, w / tau * grad, abs(w) / tau * size
