"""CPU oracle for the steps that fine-tune a student on long packed sequences -- TEST INFRASTRUCTURE.

Only tests/ may import this file; the HIP path never does, and this file imports nothing from it.

Rotary positions with several axes, softmax attention with a sliding window and sinks over packed sequences and its gradient,
distillation from a teacher's top logits: each from its definition, in fp64, with the whole square of scores in memory.  Beside
the values stand bounds of what an implementation may be off that keeps fp16 tensors, fp32 sums, and passes the probabilities P and
their gradients dS through fp16 before the products that consume them.  A rounding to fp16 is off by at most half a step: 2^-11 of the
value, and 2^-25 below the normal range; one to fp32 by 2^-24 of it.
"""
from __future__ import annotations

import numpy as np

H16, TINY16, H32 = 2.0 ** -11, 2.0 ** -25, 2.0 ** -24


def f64(a):
    return np.asarray(a, dtype=np.float64)


# ------------------------------------------------------------------------------------------------ rotary positions


def rope_axes(x, cos, sin, positions, pair_axis, n_heads, d, inverse=False):
    """x [T x >= n_heads d]; the turned heads [T x n_heads d] and the bound of their error."""
    x, T, half = f64(x)[:, :n_heads * d], len(x), d // 2
    c, s = np.ones((T, half)), np.zeros((T, half))
    for t in range(T):
        for e in range(half):
            p = int(positions[pair_axis[e]][t])
            if 0 <= p < len(cos):
                c[t, e], s[t, e] = cos[p][e], sin[p][e]
    if inverse:
        s = -s
    a, b = np.split(x.reshape(T, n_heads, d), 2, axis=-1)
    c, s = c[:, None], s[:, None]
    y = np.concatenate((a * c - b * s, b * c + a * s), -1)
    terms = np.concatenate((np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)), -1)
    return y.reshape(T, -1), (H16 * np.abs(y) + 2 * H32 * terms + TINY16).reshape(T, -1)


# ------------------------------------------------------------------------------------------------------- attention


def visible(n, window, sinks):
    """[n x n] of which key (column) a query (row) sees."""
    i = np.arange(n)
    gap = i[:, None] - i[None, :]
    return (gap >= 0) & ((gap < window) | (i[None, :] < sinks))


def _heads(qkv, h, g):
    d = qkv.shape[1] // (h + 2 * g)
    x = f64(qkv).reshape(len(qkv), h + 2 * g, d)
    return x, d


def _score_error(q, k, see, d):
    """Bound of the error of a row's scores: fp32 sums of d products, scaled, and the fp32 argument of the exponential."""
    return (d + 16) * H32 * (np.abs(q) @ np.abs(k).T * see).max(1) / np.sqrt(d)


def window_attention_forward(qkv, offsets, h, g, window, sinks):
    """o, lse and the bounds of their errors; rows of no sequence are NaN in all four."""
    x, d = _heads(qkv, h, g)
    T = len(x)
    o, lse = np.full((T, h, d), np.nan), np.full((T, h), np.nan)
    do, dl = o.copy(), lse.copy()
    for a, b in zip(offsets, offsets[1:]):
        if b <= a:
            continue
        n, see = b - a, visible(b - a, window, sinks)
        for i in range(h):
            q, k, v = x[a:b, i], x[a:b, h + i // (h // g)], x[a:b, h + g + i // (h // g)]
            s = np.where(see, q @ k.T / np.sqrt(d), -np.inf)
            m = s.max(1, keepdims=True)
            e = np.exp(s - m)
            total = e.sum(1, keepdims=True)
            p = e / total
            err = _score_error(q, k, see, d) + 4 * H32 * (1 + np.abs(m[:, 0]))
            o[a:b, i], lse[a:b, i] = p @ v, (m + np.log(total))[:, 0]
            # each probability rounded to fp16 relative to a maximum (below the normal range by half its step), the sums, then o
            spread = p @ np.abs(v)
            small = TINY16 * (see @ np.abs(v)) / total
            do[a:b, i] = H16 * np.abs(o[a:b, i]) + (H16 + 2 * err[:, None] + 2 * (n + 16) * H32) * spread * (1 + H16) + small + TINY16
            dl[a:b, i] = 2 * err + 2 * (n + 16) * H32 + 4 * H32 * np.abs(lse[a:b, i])
    return o.reshape(T, -1), lse, do.reshape(T, -1), dl


def window_attention_backward(qkv, o, do, lse, offsets, h, g, window, sinks):
    """dqkv and the bound of its error; rows of no sequence are NaN."""
    x, d = _heads(qkv, h, g)
    T = len(x)
    grad, bound = np.full((2, T, h + 2 * g, d), np.nan)
    o, do, lse = f64(o).reshape(T, h, d), f64(do).reshape(T, h, d), f64(lse)
    for a, b in zip(offsets, offsets[1:]):
        if b <= a:
            continue
        n, see = b - a, visible(b - a, window, sinks)
        grad[a:b], bound[a:b] = 0.0, 0.0
        for i in range(h):
            kv = i // (h // g)
            q, k, v = x[a:b, i], x[a:b, h + kv], x[a:b, h + g + kv]
            u, w = do[a:b, i], o[a:b, i]
            p = np.where(see, np.exp(q @ k.T / np.sqrt(d) - lse[a:b, i, None]), 0.0)
            delta = (u * w).sum(1, keepdims=True)
            ds = p * (u @ v.T - delta) / np.sqrt(d)
            rel = 2 * (_score_error(q, k, see, d) + 4 * H32 * (1 + np.abs(lse[a:b, i])))[:, None]
            dp = (d + 16) * H32 * (np.abs(u) @ np.abs(v).T + (np.abs(u) * np.abs(w)).sum(1, keepdims=True))
            # a probability is held times 2^15; the sums of n terms in fp32
            ep = (H16 + rel) * p * (1 + H16) + see * TINY16 * 2.0 ** -15
            es = ((H16 + rel) * np.abs(ds) + p * dp / np.sqrt(d)) * (1 + H16) + see * TINY16
            sums = (n * (h // g) + 64) * H32
            grad[a:b, i] = ds @ k
            bound[a:b, i] = es @ np.abs(k) + sums * (np.abs(ds) @ np.abs(k))
            grad[a:b, h + kv] += ds.T @ q
            bound[a:b, h + kv] += es.T @ np.abs(q) + sums * (np.abs(ds).T @ np.abs(q))
            grad[a:b, h + g + kv] += p.T @ u
            bound[a:b, h + g + kv] += ep.T @ np.abs(u) + sums * (p.T @ np.abs(u))
    bound += H16 * (np.abs(grad) + bound) + TINY16
    return grad.reshape(T, -1), bound.reshape(T, -1)


# ---------------------------------------------------------------------------------------------------- distillation


def distill(logits, ids, teacher, targets, scale, tau, w):
    """Token losses, logit gradient (times `scale`) and the bounds of their errors."""
    z, t = f64(logits), f64(teacher)
    T, V = z.shape
    loss, grad, el, eg = np.zeros(T), np.zeros((T, V)), np.zeros(T), np.zeros((T, V))
    sums = (V / 256 + 64) * 2 * H32            # a thread's share of a sum of exponentials, each 2 units off
    for r in range(T):
        target = int(targets[r])
        if not 0 <= target < V:
            continue
        m = z[r].max()
        eh, es = np.exp(z[r] - m), np.exp((z[r] - m) / tau)
        q, soft_lse = es / es.sum(), m / tau + np.log(es.sum())
        hard = m + np.log(eh.sum()) - z[r, target]
        one = np.zeros(V)
        one[target] = 1.0
        listed = [(int(i), x / tau) for i, x in zip(ids[r], t[r]) if 0 <= i < V and x > -np.inf]
        want, soft, reach, share = np.zeros(V), 0.0, 0.0, 0.0
        if listed:
            top = max(x for _, x in listed)
            total = sum(np.exp(x - top) for _, x in listed)
            for i, x in listed:
                p = np.exp(x - top) / total
                want[i] += p
                if p > 0:
                    log_p, log_q = x - top - np.log(total), z[r, i] / tau - soft_lse
                    soft += p * (log_p - log_q)
                    reach += p * (abs(log_p) + abs(z[r, i] - m) / tau + np.log(es.sum()))
            share = w
        loss[r] = (1 - w) * hard + share * tau ** 2 * soft
        far = np.log(eh.sum()) + abs(m - z[r, target])
        el[r] = 2 * sums * ((1 - w) * (1 + far) + share * tau ** 2 * (1 + reach) * (1 + 2 * abs(reach))) + 2 * H32 * abs(loss[r])
        grad[r] = scale * ((1 - w) * (eh / eh.sum() - one) + share * tau * (q - want))
        size = scale * ((1 - w) * (eh / eh.sum() * (1 + np.abs(z[r] - m)) + one) + share * tau * (q * (1 + np.abs(z[r] - m) / tau) + want * (1 + reach)))
        eg[r] = H16 * np.abs(grad[r]) + 4 * sums * size + TINY16
    return loss, grad, el, eg
