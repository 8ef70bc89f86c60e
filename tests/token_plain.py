"""The token operators from their definitions, in binary64 with plain loops over rows (numpy), and bounds on what
binary32 sums may differ from them.  Written apart from the library; only tests import it."""
import numpy as np

U = 2.0 ** -24          # rounding error of one binary32 operation, relative
BF16 = 2.0 ** -8        # twice that of one rounding to bfloat16: covers a binary32 value beside a tie


def lookup(table, tokens, scale):
    out = np.zeros((len(tokens), table.shape[1]))
    for t, v in enumerate(tokens):
        if 0 <= v < table.shape[0]:
            out[t] = table[v] * scale
    return out


def table_grad(tokens, dY, V, scale):
    """-> gradient, bound on the error of a binary32 sum in any order"""
    dE, size, n = np.zeros((V, dY.shape[1])), np.zeros((V, dY.shape[1])), np.zeros(V)
    for t, v in enumerate(tokens):
        if 0 <= v < V:
            dE[v] += dY[t]
            size[v] += np.abs(dY[t])
            n[v] += 1
    return dE * scale, (n[:, None] + 1) * U * size * abs(scale) + 1e-44


def capacity(n, E, align):
    """The largest number of rows over all ways to share n entries among E experts: one entry for as many as possible,
    the rest to one of them, is never worse than what the formula says; brute force in the tests for small n."""
    return (n + min(E, n) * (align - 1)) // align * align


def sort_by_expert(ids, E, align):
    flat = np.asarray(ids).reshape(-1)
    rows = capacity(flat.size, E, align)
    members = [[i for i, e in enumerate(flat) if e == x] for x in range(E)]
    offsets, order, slots = [0], np.full(rows, -1, np.int32), np.full(flat.size, -1, np.int32)
    for m in members:
        for r, i in enumerate(m):
            order[offsets[-1] + r] = i
            slots[i] = offsets[-1] + r
        offsets.append(offsets[-1] + -(-len(m) // align) * align)
    return (np.array(offsets, np.int32), np.array([len(m) for m in members], np.int32), order,
            slots.reshape(np.shape(ids)))


def gather(X, order, k):
    out = np.zeros((len(order), X.shape[1]), X.dtype)
    for s, f in enumerate(order):
        if f >= 0:
            out[s] = X[f // k]
    return out


def combine(Ys, slots, weights):
    """-> sum, bound on the error of the binary32 sum"""
    T, k = slots.shape
    out, size = np.zeros((T, Ys.shape[1])), np.zeros((T, Ys.shape[1]))
    for t in range(T):
        for j in range(k):
            if slots[t, j] >= 0:
                term = (1.0 if weights is None else float(weights[t, j])) * Ys[slots[t, j]]
                out[t] += term
                size[t] += np.abs(term)
    return out, (k + 1) * U * size + 1e-44


def combine_grad(Ys, slots, order, weights, dOut):
    """-> dYs, dweights, bound on the error of dweights"""
    T, k = slots.shape
    dYs, dw, bound = np.zeros(Ys.shape), np.zeros((T, k)), np.zeros((T, k))
    for t in range(T):
        for j in range(k):
            s = slots[t, j]
            if s >= 0:
                dYs[s] = float(weights[t, j]) * dOut[t]
                dw[t, j] = Ys[s] @ dOut[t]
                bound[t, j] = (Ys.shape[1] + 1) * U * (np.abs(Ys[s]) @ np.abs(dOut[t])) + 1e-44
    return dYs, dw, bound


def distill(z, ids, teacher, tau, dloss):
    """-> loss, statistics, gradient, and bounds on the error of the loss and of the gradient in binary32.

    A logit's exponent (z - m) * log2(e) / tau carries three roundings and so a share d = 3 |z - m| / tau * U of itself (in
    units of the natural exponent), the exponential two units more; the sum of V of them, added up in lanes of at most
    V / 256 terms in batches and a tree, at most (V / 256 + 40) U relative.  For masked logits the exponential is 0 either way.
    """
    N, V = z.shape
    loss, stats, grad = np.zeros(N), np.zeros((N, 2)), np.zeros((N, V))
    e_loss, e_grad = np.zeros(N), np.zeros((N, V))
    with np.errstate(all="ignore"):
        for n in range(N):
            m = z[n].max() if V else -np.inf
            x = (z[n] - m) / tau
            p = np.exp(x)
            S = p.sum()
            stats[n] = m, (np.log(S) if m > -np.inf else np.nan)
            js = [j for j in range(ids.shape[1]) if 0 <= ids[n, j] < V]
            t = np.array([teacher[n, j] for j in js], dtype=np.float64)
            if len(js) == 0 or t.max() == -np.inf:
                continue
            xt = (t - t.max()) / tau
            q = np.exp(xt)
            q /= q.sum()
            lq, lp = xt - np.log(np.exp(xt).sum()), x[[ids[n, j] for j in js]] - stats[n, 1]
            loss[n] = tau * tau * sum(a * (b - c) for a, b, c in zip(q, lq, lp) if a > 0)
            grad[n] = p / S
            mass = np.zeros(V)
            for a, j in zip(q, js):
                mass[ids[n, j]] += a
            grad[n] = dloss[n] * tau * (p / S - mass)
            near = np.where(p > 0, np.minimum(np.abs(x), 120.0), 0.0)
            sum_error = (V / 256 + 40) * U + (p / S * (3 * near + 2)).sum() * U
            p_error = p / S * ((3 * near + 4) * U + sum_error)
            q_error = mass * (3 * np.minimum(np.abs(xt), 120.0).max() + 2 * len(js) + 8) * U
            e_grad[n] = abs(dloss[n]) * tau * (p_error + q_error) + 4 * U * np.abs(grad[n]) + 1e-37 * abs(dloss[n] * tau)
            size = sum(a * (abs(b) + abs(c)) for a, b, c in zip(q, lq, lp) if a > 0) + abs(stats[n, 1]) + np.log(len(js) + 1)
            e_loss[n] = tau * tau * ((2 * len(js) + 12) * U * size + sum_error)
    return loss, stats, grad, e_loss, e_grad
