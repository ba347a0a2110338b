"""Networks as experts, from their definition in 64 bits.  Test infrastructure only: shares nothing with the library and is not
imported by the package."""
import numpy as np

BIG = float(np.finfo(np.float32).max)
TINY = 2.0 ** -126


def bounds(first, n_slots):
    """(begin, end) of every expert's slots, and of nobody's."""
    at = [min(max(int(v), 0), n_slots) for v in first]
    return [(a, max(a, b)) for a, b in zip(at, at[1:])] + [(at[-1], n_slots)]


def matmul(x, first, w):
    """(y, the sums of absolute products) of rows x and weights w [experts, out, in]."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    y, size = np.zeros((x.shape[0], w.shape[1])), np.zeros((x.shape[0], w.shape[1]))
    for e, (a, b) in enumerate(bounds(first, x.shape[0])[:-1]):
        y[a:b] = x[a:b] @ w[e].T
        size[a:b] = abs(x[a:b]) @ abs(w[e]).T
    return y, size


def matmul_backward(d_y, x, first, n_experts):
    g, x = np.asarray(d_y, np.float64), np.asarray(x, np.float64)
    d_w = np.zeros((n_experts, g.shape[1], x.shape[1]))
    size = np.zeros_like(d_w)
    for e, (a, b) in enumerate(bounds(first, x.shape[0])[:-1]):
        d_w[e] = g[a:b].T @ x[a:b]
        size[e] = abs(g[a:b]).T @ abs(x[a:b])
    return d_w, size


def quantize(x):
    """(q, scale) of rows of numbers that fp32 holds."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore"):
        size = np.abs(x).max(axis=1)
    scale = np.maximum((size / 127).astype(np.float32), np.float32(TINY))
    bad = ~np.isfinite(x).all(axis=1)
    scale[bad] = np.nan
    with np.errstate(invalid="ignore"):
        q = np.rint(x / scale.astype(np.float64)[:, None])         # 53 bits tell a quotient of two of 24 from a border that it is not on
    q[bad] = 0
    return q.astype(np.int8), scale


def clean(v):
    v = np.asarray(v, np.float64)
    return np.minimum(np.where(np.isnan(v), -np.inf, v), BIG)


def log_share(v, of):
    """v - log of the sum of exp(of), as differences from the largest: logits may be so large that a logarithm is lost beside them."""
    m = of.max()
    return (v - m) - np.log(np.exp(of - m).sum())


def distill(logits, ids, teacher, temperature=1.0, scale=1.0, total=None, d_loss=None):
    """(loss, size of what is added up in it, gradient, size of what is added up in it), row by row."""
    rows, classes = logits.shape
    loss, loss_size = np.zeros(rows), np.zeros(rows)
    grad, grad_size = np.zeros((rows, classes)), np.zeros((rows, classes))
    for r in range(rows):
        x = clean(logits[r]) / temperature
        t = clean(teacher[r]) / temperature
        js = [j for j in range(ids.shape[1]) if 0 <= ids[r, j] < classes and x[ids[r, j]] > -np.inf and t[j] > -np.inf]
        if not js:
            continue
        c = ids[r, js].astype(np.int64)
        log_p = log_share(x, x)
        p = np.exp(log_p)
        rest = np.setdiff1d(np.flatnonzero(x > -np.inf), c)
        with_rest = total is not None and np.isfinite(total[r]) and rest.size > 0
        log_q = np.minimum(t[js] - float(total[r]), 0.0) if with_rest else log_share(t[js], t[js])
        q = np.exp(log_q)
        terms = np.where(q > 0, q * (log_q - log_p[c]), 0.0)
        sizes = np.where(q > 0, q * (abs(log_q) + abs(x[c]) + abs(log_p[c]) + 1), 0.0)
        q_rest = max(0.0, 1.0 - q.sum()) if with_rest else 0.0
        value, size = terms.sum(), sizes.sum()
        share = np.zeros(classes)
        if q_rest > 0:
            log_p_rest = -log_share(np.zeros(1), log_p[rest])[0]
            value += q_rest * (np.log(q_rest) - log_p_rest)
            size += q_rest * (abs(np.log(q_rest)) + abs(log_p_rest)) + 1
            share[rest] = np.exp(log_share(x[rest], x[rest])) * q_rest
        loss[r], loss_size[r] = value * scale, size * abs(scale)
        if d_loss is not None:
            f = float(d_loss[r]) * scale / temperature
            named = np.zeros(classes)
            np.add.at(named, c, q)
            all_q = q.sum() + q_rest
            grad[r] = f * (p * all_q - named - share)
            grad_size[r] = abs(f) * (p * all_q + named + share)
            grad[r][x == -np.inf] = 0
    return loss, loss_size, grad, grad_size
