"""The operators on rows from their definitions, in 64 bits, row by row: what the kernels are compared with.  Inputs are numpy float64 arrays."""
import numpy as np

INF = float("inf")


def softmax(z):
    """Zeros for a row that holds nothing but minus infinity."""
    m = z.max()
    if m == -INF:
        return np.zeros_like(z)
    with np.errstate(invalid="ignore"):
        e = np.exp(z - m)
        return e / e.sum()


def log_scores(x, score):
    """Logarithms of the scores; minus infinity for what is not a member."""
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        if score == "softmax":
            m = x.max()
            return x if m == -INF else x - m - np.log(np.exp(x - m).sum())
        return np.where(x == -INF, -INF, -np.logaddexp(0.0, -x))


def route(gates, k, score="softmax", bias=None, groups=1, kept=None, best=2, renormalise=True, scale=1.0):
    n, E = gates.shape
    kept, size = kept or groups, E // groups
    chosen, weights = np.full((n, k), -1, np.int32), np.zeros((n, k))
    top = float(np.finfo(np.float32).max)
    for i in range(n):
        x = np.where(gates[i] > -INF, np.minimum(gates[i], top), -INF)
        ls = log_scores(x, score)
        s = np.exp(ls)
        c = s + bias if bias is not None else s if groups > 1 else x
        c = np.where((x > -INF) & (c > -INF), c, -INF)
        if groups > 1:
            rank = []
            for g in range(groups):
                part = np.sort(c[g * size:(g + 1) * size])[::-1][:best]
                part = part[part > -INF]
                rank.append(part.sum() if len(part) else -INF)
            stay = sorted(range(groups), key=lambda g: (-rank[g], g))[:kept]
            c = np.where(np.isin(np.arange(E) // size, stay), c, -INF)
        order = [e for e in sorted(range(E), key=lambda e: (-c[e], e)) if c[e] > -INF][:k]
        chosen[i, :len(order)] = order
        if order:
            weights[i, :len(order)] = scale * (softmax(ls[order]) if renormalise else s[order])
    return chosen, weights


def route_backward(gates, chosen, d_weights, score="softmax", renormalise=True, scale=1.0):
    n, E = gates.shape
    out = np.zeros((n, E))
    top = float(np.finfo(np.float32).max)
    for i in range(n):
        x = np.where(gates[i] > -INF, np.minimum(gates[i], top), -INF)
        ls = log_scores(x, score)
        s = np.exp(ls)
        slots = [j for j in range(chosen.shape[1]) if 0 <= chosen[i, j] < E and x[chosen[i, j]] > -INF]
        if not slots:
            continue
        e = chosen[i, slots]
        u = scale * d_weights[i, slots]
        if renormalise:
            r = softmax(ls[e])
            d = r * (u - (r * u).sum())
            if score == "sigmoid":
                d = d * (1 - s[e])
        elif score == "sigmoid":
            d = u * s[e] * (1 - s[e])
        else:
            d = u * s[e]
            out[i] = -s * d.sum()
        np.add.at(out[i], e, d)
    return out


def combine(logits, chosen, weights):
    M, n, C = logits.shape
    out = np.zeros((n, C))
    for i in range(n):
        for j in range(chosen.shape[1]):
            if 0 <= chosen[i, j] < M:
                out[i] += weights[i, j] * softmax(logits[chosen[i, j], i])
    return out


def combine_backward(logits, chosen, weights, d_probs):
    M, n, C = logits.shape
    d_w, d_z = np.zeros(chosen.shape), np.zeros(logits.shape)
    for i in range(n):
        for j in range(chosen.shape[1]):
            m = chosen[i, j]
            if 0 <= m < M:
                p = softmax(logits[m, i])
                d_w[i, j] = (p * d_probs[i]).sum()
                d_z[m, i] += weights[i, j] * p * (d_probs[i] - d_w[i, j])
    return d_w, d_z


def top(values, k, form="value", temperature=1.0):
    n, C = values.shape
    index, value = np.zeros((n, k), np.int32), np.zeros((n, k))
    for i in range(n):
        x = values[i]
        # NaN behind everything, the lowest class first among equal values
        order = np.lexsort((np.arange(C), -np.where(np.isnan(x), 0.0, x), np.isnan(x)))[:k]
        v = x[order]
        with np.errstate(divide="ignore", invalid="ignore"):
            if form == "log":
                v = np.log(v)
            if form == "log_softmax":
                z = x / temperature
                m = np.nanmax(z) if not np.isnan(z).all() else np.nan
                v = v / temperature if m == -INF else v / temperature - m - np.log(np.exp(z - m).sum())
        index[i], value[i] = order, v
    return index, value


def teacher(index, log_probs, classes, tail):
    """q over all classes, which classes are listed, q_0."""
    q, listed = np.zeros(classes), np.zeros(classes, bool)
    here = [j for j in range(len(index)) if 0 <= index[j] < classes]
    if here:
        t = log_probs[here]
        np.add.at(q, index[here], np.exp(t) if tail else softmax(t))
        listed[index[here]] = True
    return q, listed, max(0.0, 1.0 - q.sum()) if tail else 0.0


def distill(logits, index, log_probs, temperature=1.0, tail=False):
    """(loss, gradient of each row's loss)."""
    n, C = logits.shape
    T, loss, grad = temperature, np.zeros(n), np.zeros((n, C))
    for i in range(n):
        q, listed, q0 = teacher(index[i], log_probs[i], C, tail)
        z = logits[i] / T
        if z.max() == -INF:
            continue
        with np.errstate(divide="ignore", invalid="ignore"):
            log_p = z - z.max() - np.log(np.exp(z - z.max()).sum())
            p = np.exp(log_p)
            loss[i] = (np.where(q > 0, q * (np.log(q) - log_p), 0.0)).sum()
            grad[i] = q.sum() * p - q
            p0 = p[~listed].sum()
            if tail and q0 > 0 and p0 > 0:
                loss[i] += q0 * (np.log(q0) - np.log(p0))
                grad[i] += q0 * (p - np.where(listed, 0.0, p / p0))
    return T * T * loss, T * grad
