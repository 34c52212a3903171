"""Plain implementations of the score operators in 64 bits (numpy, row by row), and inputs."""
import numpy as np

INF = float("inf")


def wide(x):
    """Scores as float64: votes by their logarithm, NaN as -inf."""
    if x.dtype == np.uint8:
        with np.errstate(divide="ignore"):
            return np.log(x.astype(np.float64))
    x = x.astype(np.float64)
    return np.where(np.isnan(x), -INF, x)


def best_first(row):
    """Classes of a row, best first, equal ones from the lowest."""
    return np.argsort(-row, kind="stable")


def top_scores(x, k):
    s = wide(x)
    values = np.empty((len(s), k))
    index = np.empty((len(s), k), dtype=np.int32)
    lse = np.empty(len(s))
    for r, row in enumerate(s):
        at = best_first(row)[:k]
        values[r] = row[at]
        index[r] = np.where(row[at] > -INF, at, -1)
        m = row.max()
        with np.errstate(invalid="ignore", divide="ignore"):
            lse[r] = m + np.log(np.where(row == m, 1.0, np.exp(row - m)).sum()) if m > -INF else -INF
    return values, index, lse


def staying(x_row, temperature, top_k, top_p, min_p, shift=0.0):
    """Weights of a row's classes, 0 for those that do not stay (None: an empty row).  shift moves
    the borders of top_p and min_p by so much of the best class's weight."""
    s = wide(x_row[None])[0]
    m = s.max()
    if m == -INF:
        return None
    n = len(s)
    if not temperature > 0:
        top_k, temperature = 1, 1.0
    if top_k < 1 or top_k > n:
        top_k = n
    top_p = float(np.float32(top_p))
    min_p = min(max(float(np.float32(min_p)), 0.0), 1.0) if min_p == min_p else 0.0
    with np.errstate(invalid="ignore"):
        w = np.where(s == m, 1.0, np.exp((s - m) / float(np.float32(temperature))))
    if x_row.dtype == np.uint8 and np.float32(temperature) == 1:
        w = x_row.astype(np.float64)
    order = best_first(s)
    o = w[order].copy()
    first = o[0]
    o[top_k:] = 0
    upto = np.cumsum(o)
    before = np.concatenate([[0.0], upto[:-1]])
    keep = np.ones(n, dtype=bool)
    if top_p < 1:
        keep = before < top_p * upto[-1] + shift * first
        keep[0] = True
    keep &= (o >= min_p * first + shift * first) | (o == first)
    out = np.zeros(n)
    out[order] = np.where(keep, o, 0.0)
    return out


def draw(w, u, shift=0.0):
    """The class that u draws by these weights, the border moved by so much of the best weight."""
    upto = np.cumsum(w)
    goal = min(float(u) if u > 0 else 0.0, 1 - 2.0 ** -24) * upto[-1] + shift * w.max()
    return int(np.argmax(upto > goal)) if goal < upto[-1] else int(np.flatnonzero(w)[-1])


def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Labels."""
    n = len(x)
    t, k, p, m = (np.broadcast_to(v, n) for v in (temperature, top_k, top_p, min_p))
    out = np.empty(n, dtype=np.int32)
    for r in range(n):
        w = staying(x[r], t[r], k[r], p[r], m[r])
        out[r] = -1 if w is None else draw(w, u[r])
    return out


def check_sample(got, x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, note=""):
    """Labels equal to sample()'s, except where a border lies within the weights' rounding.

    A weight is rounded to a multiple of 2^-42 of the best one (off by 2^-43) after its 64-bit
    exponential (2^-45), so sums of up to n weights, and p or u times them, differ from the exact ones by at
    most 2 n (2^-43 + 2^-45) < n 2^-41 of the best weight.  Where a sum of weights is that near to its
    border (votes at temperature 1/2 are squares of whole numbers, half of whose sum can be reached
    exactly), both sides of the border are right.  Votes at temperature 1 have no such room."""
    want = sample(x, u, temperature, top_k, top_p, min_p)
    n = len(x)
    t, k, p, m = (np.broadcast_to(v, n) for v in (temperature, top_k, top_p, min_p))
    for r in np.flatnonzero(got != want):
        delta = x.shape[1] * 2.0 ** -41
        exact = x.dtype == np.uint8 and np.float32(t[r]) == 1
        right = set()
        for a in (-delta, delta):
            w = staying(x[r], t[r], k[r], p[r], m[r], a)
            right |= set() if w is None or exact else {draw(w, u[r], b) for b in (-delta, delta)}
        assert got[r] in right, "%s row %d: %d, not %d %s" % (note, r, got[r], want[r], right)


def distill(x, values, index, temperature, g):
    """Loss and gradient of each row."""
    x = x.astype(np.float64)
    values = values.astype(np.float64)
    n, classes = x.shape
    t = float(np.float32(temperature))
    loss, grad = np.zeros(n), np.zeros((n, classes))
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        for r in range(n):
            on = (index[r] >= 0) & (index[r] < classes) & ~(values[r] == -INF)
            if not on.any() or (x[r] == -INF).all():
                continue
            c, v = index[r][on], values[r][on] / t
            z = x[r] / t
            q = np.exp(z - z.max())
            logq = z - z.max() - np.log(q.sum())
            q /= q.sum()
            v = v - v.max()
            logp = v - np.log(np.exp(v).sum())
            p = np.exp(logp)
            terms = np.where(p == 0, 0.0, p * (logp - logq[c]))
            loss[r] = t * t * terms.sum()
            grad[r] = q
            np.subtract.at(grad[r], c, p)
            grad[r] *= t * float(g[r])
    return loss, grad
