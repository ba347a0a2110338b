"""Mixtures of family models from their definition, token by token, in 64 bits.  Test infrastructure only: shares
nothing with the library and is not imported by the package."""
import numpy as np

BIG = float(np.finfo(np.float32).max)


def _logits(row):
    x = np.asarray(row, np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    return np.minimum(x, BIG)


def log_scores(x, score):
    """Logarithms of a token's scores; -inf where an expert is masked."""
    if score == "softmax":
        if not np.any(x > -np.inf):
            return np.full_like(x, -np.inf)
        top = x.max()
        return x - top - np.log(np.sum(np.exp(x - top)))
    with np.errstate(over="ignore"):
        return np.minimum(x, 0) - np.log1p(np.exp(-np.abs(x)))


def _best(keys, n):
    """Indices of the n largest keys, ties to the lower index; those of -inf are left out."""
    order = sorted(range(len(keys)), key=lambda i: (-keys[i], i))
    return [i for i in order[:n] if keys[i] > -np.inf]


def route(logits, k, score="softmax", renormalise=True, bias=None, n_groups=1, top_groups=1, group_best=1, scale=1.0):
    tokens, experts = logits.shape
    expert = np.full((tokens, k), -1, np.int32)
    weight = np.zeros((tokens, k))
    for t in range(tokens):
        x = _logits(logits[t])
        a = log_scores(x, score)
        s = np.exp(a)
        if bias is None:
            key, rank = x.copy(), np.where(x > -np.inf, s, -np.inf)
        else:
            key = np.where(x > -np.inf, s + np.asarray(bias, np.float64), -np.inf)
            key = np.where(np.isnan(key), -np.inf, key)
            rank = key
        if n_groups > 1:
            sums = []
            for g in rank.reshape(n_groups, -1):
                v = [u for u in sorted(g, reverse=True)[:group_best] if u > -np.inf]
                sums.append(sum(v) if v else -np.inf)
            taken = _best(sums, top_groups)
            per = experts // n_groups
            for e in range(experts):
                if e // per not in taken:
                    key[e] = -np.inf
        chosen = _best(key, k)
        expert[t, : len(chosen)] = chosen
        if chosen:
            b = x[chosen] if renormalise and score == "softmax" else a[chosen]     # a term common to all falls out
            if renormalise:
                w = np.exp(b - b.max())
                w = w / w.sum()
            else:
                w = np.exp(b)
            weight[t, : len(chosen)] = w * scale
    return expert, weight


def route_backward(logits, expert, d_weight, score="softmax", renormalise=True, scale=1.0):
    """(the gradient, the sum of the absolute values that went into each)"""
    tokens, experts = logits.shape
    d, size = np.zeros((tokens, experts)), np.zeros((tokens, experts))
    for t in range(tokens):
        x = _logits(logits[t])
        s = np.exp(log_scores(x, score))
        js = [j for j in range(expert.shape[1]) if 0 <= expert[t, j] < experts]
        es = [int(expert[t, j]) for j in js]
        dw = np.array([float(d_weight[t, j]) for j in js]) * scale
        if not js:
            continue
        if renormalise:
            a = x[es] if score == "softmax" else log_scores(x, score)[es]
            q = np.exp(a - a.max()) if a.max() > -np.inf else np.zeros(len(es))
            q = q / max(q.sum(), 1e-300)
            for j, e in enumerate(es):
                f = 1.0 if score == "softmax" else 1.0 / (1.0 + np.exp(min(x[e], 700.0)))
                d[t, e] += q[j] * (dw[j] - np.sum(q * dw)) * f
                size[t, e] += q[j] * (abs(dw[j]) + np.sum(q * abs(dw))) * f
        else:
            g, ga = np.zeros(experts), np.zeros(experts)
            for j, e in enumerate(es):
                g[e] += dw[j]
                ga[e] += abs(dw[j])
            if score == "softmax":
                d[t] = s * (g - np.sum(s * g))
                size[t] = s * (ga + np.sum(s * ga))
            else:
                rest = 1.0 / (1.0 + np.exp(np.minimum(x, 700)))
                d[t], size[t] = g * s * rest, ga * s * rest
        d[t][x == -np.inf] = 0
    return d, size


def plan(expert, n_experts):
    flat = np.asarray(expert).reshape(-1)
    order, place = np.full(flat.size, -1, np.int32), np.full(flat.size, -1, np.int32)
    first, at = np.zeros(n_experts + 1, np.int32), 0
    for e in range(n_experts):
        mine = np.flatnonzero(flat == e)
        order[at: at + mine.size] = mine
        place[mine] = np.arange(at, at + mine.size)
        at += mine.size
        first[e + 1] = at
    return first, order, place.reshape(np.shape(expert))


def gather(x, order, k):
    out = np.zeros((order.size, x.shape[1]), np.float64)
    out[order >= 0] = np.asarray(x, np.float64)[order[order >= 0] // k]
    return out


def combine(y, place, weight=None):
    """(the sums, the sums of absolute values)"""
    out = np.zeros((place.shape[0], y.shape[1]))
    size = np.zeros_like(out)
    for t in range(place.shape[0]):
        for j in range(place.shape[1]):
            if place[t, j] >= 0:
                v = np.asarray(y[place[t, j]], np.float64) * (1.0 if weight is None else float(weight[t, j]))
                out[t] += v
                size[t] += abs(v)
    return out, size


def combine_backward(d_out, y, place, weight):
    """(d_y, d_weight, the sums of absolute values in d_weight)"""
    d_y = np.zeros(y.shape)
    d_w, size = np.zeros(place.shape), np.zeros(place.shape)
    for t in range(place.shape[0]):
        g = np.asarray(d_out[t], np.float64)
        for j in range(place.shape[1]):
            if place[t, j] >= 0:
                v = np.asarray(y[place[t, j]], np.float64)
                d_y[place[t, j]] = g * float(weight[t, j])
                d_w[t, j] = np.dot(g, v)
                size[t, j] = np.dot(abs(g), abs(v))
    return d_y, d_w, size


def rows_of(ids, col_base, n_vocab):
    """The table's rows that ids [rows, columns] name; -1 for those outside it."""
    v = np.asarray(ids).astype(np.int64)
    if col_base is not None:
        v = v + np.asarray(col_base, np.int64)[None, :]
    return np.where((v >= 0) & (v < n_vocab), v, -1)


def embed(table, rows, scale):
    out = np.zeros((rows.shape[0], table.shape[1]))
    size = np.zeros_like(out)
    t = np.asarray(table, np.float64)
    for c in range(rows.shape[1]):
        there = rows[:, c] >= 0
        out[there] += t[rows[there, c]]
        size[there] += abs(t[rows[there, c]])
    return out * scale, size * abs(scale)


def embed_backward(d_out, rows, n_vocab, scale):
    out = np.zeros((n_vocab, d_out.shape[1]))
    size = np.zeros_like(out)
    g = np.asarray(d_out, np.float64)
    for c in range(rows.shape[1]):
        there = rows[:, c] >= 0
        np.add.at(out, rows[there, c], g[there])
        np.add.at(size, rows[there, c], abs(g[there]))
    return out * scale, size * abs(scale)
