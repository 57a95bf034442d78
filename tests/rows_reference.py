"""Plain 64-bit forms (numpy) of the operators on rows of logits: the filtered draw and the distillation loss."""
import numpy as np

BELOW_ONE = float(np.nextafter(np.float32(1.0), np.float32(0.0)))


def clamp_uniform(u):
    u = float(u)
    return 0.0 if not u >= 0.0 else min(u, BELOW_ONE)


def kept_ids(x, T=1.0, k=0, p=1.0, m=0.0):
    """(kept ids in id order, their weights exp(z - max), how near a mass border of top-p came to deciding
    otherwise, relative to the mass).  x: float64 [V], the values of the stored logits."""
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64)) + 0.0
    V = x.size
    if not T > 0:
        T, k = 1.0, 1
    top = x.max()
    if top == -np.inf:
        return np.zeros(0, np.int64), np.zeros(0), 1.0
    with np.errstate(invalid="ignore"):
        d = np.where(x == top, 0.0, -np.inf) if top == np.inf else np.where(x == -np.inf, -np.inf, (x - top) / T)
    w = np.exp(d)
    order = np.argsort(-x, kind="stable")
    n, margin = V, 1.0
    if 1 <= k < V:
        n = k
    if p < 1.0:
        cum = np.cumsum(w[order[:n]])
        before = np.concatenate([[0.0], cum[:-1]])
        goal = max(p, 0.0) * cum[-1]
        margin = float(np.min(np.abs(before[1:] - goal)) / cum[-1]) if n > 1 and p > 0 else 1.0
        n = max(1, int(np.sum(before < goal)))
    if m > 0.0:
        n = min(n, max(1, int(np.sum(d[order[:n]] >= np.log(min(m, 1.0))))))
    ids = np.sort(order[:n])
    return ids, w[ids], margin


def draw(x, u, T=1.0, k=0, p=1.0, m=0.0):
    """(token, log-probability among the kept ids, margin): the margin is how near, relative to the mass, a
    border of top-p or of the draw lies to where it would have decided otherwise."""
    ids, w, margin = kept_ids(x, T, k, p, m)
    if ids.size == 0:
        return 0, -np.inf, 1.0
    cum = np.cumsum(w)
    goal = clamp_uniform(u) * cum[-1]
    at = int(np.searchsorted(cum, goal, side="right"))
    at = min(at, int(np.flatnonzero(w)[-1]))
    if w.size > 1:  # the ends of the interval decide nothing
        margin = min(margin, float(np.min(np.abs(cum[:-1] - goal)) / cum[-1]) if goal > 0 else 1.0)
    xx = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    T = T if T > 0 else 1.0
    z = 0.0 if xx.max() == np.inf else (xx[ids[at]] - xx.max()) / T
    return int(ids[at]), float(z - np.log(cum[-1])), margin


def teacher(ids, scores, V, T, tail):
    """(valid places, q of every place, rest) of one row's list."""
    ok = (ids >= 0) & (ids < V)
    s = np.where(ok, scores.astype(np.float64), -np.inf)
    if tail:
        q = np.exp(s)
        every = np.unique(ids[ok]).size == V
        return ok, q, 0.0 if every else max(0.0, 1.0 - q.sum())
    if not (s > -np.inf).any():
        return ok, np.zeros_like(s), 0.0
    q = np.exp((s - s.max()) / T)
    return ok, q / q.sum(), 0.0


def lse(z):
    top = z.max() if z.size else -np.inf
    return top if top == -np.inf else top + np.log(np.exp(z - top).sum())


def distill(x, ids, scores, T=1.0, tail=False, weight=1.0, up=1.0):
    """(loss, log Z, log R, gradient [V]) of one row; x: float64 [V], the values of the stored logits."""
    V = x.size
    z = x.astype(np.float64) / T
    ok, q, rest = teacher(ids, scores, V, T, tail)
    listed = np.zeros(V, bool)
    listed[ids[ok]] = True
    z_all, z_rest = lse(z), lse(z[~listed])
    q_of = np.zeros(V)
    np.add.at(q_of, ids[ok], q[ok])
    if z_all == -np.inf:
        loss = np.inf if (q > 0).any() or rest > 0 else 0.0
        p = np.zeros(V)
        p_in_rest = np.zeros(V)
    else:
        with np.errstate(invalid="ignore", divide="ignore"):
            loss = sum(a * (np.log(a) - (z[i] - z_all)) for a, i in zip(q[ok], ids[ok]) if a > 0)
            if rest > 0:
                loss += rest * (np.log(rest) - (z_rest - z_all))
        p = np.exp(z - z_all)
        p_in_rest = np.exp(z - z_rest) if z_rest > -np.inf else np.zeros(V)
    with np.errstate(invalid="ignore"):  # (listed ids: not the rest's, whatever their share of it would be)
        g = (q.sum() + rest) * p - q_of - np.where(listed, 0.0, rest * p_in_rest)
    if weight == 0:
        return 0.0, z_all, z_rest, np.zeros(V)
    return weight * loss, z_all, z_rest, g * (weight * up / T)
