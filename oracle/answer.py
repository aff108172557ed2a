"""Appends to a paged cache, attention over it and sampling from their definitions, in 64 bits, token by token."""
import numpy as np


def bf16_values(bits):
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def key_at(page_no, head, token, d, Hkv, page, D):
    """Element of the keys' cache that holds element d of a token of a page."""
    return (page_no * Hkv + head) * page * D + ((token // 32) * (D // 8) + d // 8) * 256 + (token % 32) * 8 + d % 8


def value_at(page_no, head, token, d, Hkv, page, D):
    return (page_no * Hkv + head) * page * D + ((token // 8) * D + d) * 8 + token % 8


def page_of(table, s, t, page, n_pages):
    """The page of token t of sequence s, None if it has none."""
    if t < 0 or t // page >= table.shape[1]:
        return None
    p = int(table[s, t // page])
    return p if 0 <= p < n_pages else None


def rows_of(starts, lens, M):
    """(row, sequence, position) of every row of a sequence."""
    for s in range(len(lens)):
        a, b = (min(max(int(v), 0), M) for v in starts[s:s + 2])
        for row in range(a, b):
            yield row, s, max(int(lens[s]), 0) - (b - a) + row - a


def rotate(head, position, freq, layout, magnitude):
    """One head, rotated; and the sum of the sizes of what makes up each element (for the rounding of a calculation in fewer bits)."""
    R = 2 * len(freq)
    out, size = head.copy(), np.zeros_like(head)
    for j, f in enumerate(freq):
        a, b = (j, j + R // 2) if layout == 0 else (2 * j, 2 * j + 1)
        c, s = np.cos(position * f), np.sin(position * f)
        out[a] = magnitude * (head[a] * c - head[b] * s)
        out[b] = magnitude * (head[a] * s + head[b] * c)
        size[a] = size[b] = abs(magnitude) * (abs(head[a]) + abs(head[b]))
    return out, size


def append(x, starts, lens, table, freq, layout, magnitude, M, Hq, Hkv, D, page, n_pages):
    """x: M x (Hq + 2 Hkv) D bits.  Returns {row: (queries, sizes)}, {element of the keys: (value, size)}, {element of the values: bits}."""
    q, k, v = {}, {}, {}
    heads = x.reshape(M, Hq + 2 * Hkv, D)
    values = bf16_values(heads)
    for row, s, t in rows_of(starts, lens, M):
        turned = [rotate(values[row, h], t, freq, layout, magnitude) for h in range(Hq + Hkv)]
        q[row] = np.stack([a for a, _ in turned[:Hq]]).reshape(-1), np.stack([b for _, b in turned[:Hq]]).reshape(-1)
        p = page_of(table, s, t, page, n_pages)
        if p is None:
            continue
        for h in range(Hkv):
            for d in range(D):
                k[key_at(p, h, t % page, d, Hkv, page, D)] = turned[Hq + h][0][d], turned[Hq + h][1][d]
                v[value_at(p, h, t % page, d, Hkv, page, D)] = heads[row, Hq + Hkv + h, d]
    return q, k, v


def attention(q, k, v, starts, lens, table, M, Hq, Hkv, D, page, n_pages, window, scale, max_len):
    """Bits in.  Returns {row: (Hq D outputs, the same sums of sizes)}."""
    qv, out = bf16_values(q).reshape(M, Hq, D), {}
    d = np.arange(D)
    cached = {}

    def key_value(s, t, h):
        if (s, t, h) not in cached:
            p = page_of(table, s, t, page, n_pages)
            cached[s, t, h] = None if p is None else (bf16_values(k[key_at(p, h, t % page, d, Hkv, page, D)]), bf16_values(v[value_at(p, h, t % page, d, Hkv, page, D)]))
        return cached[s, t, h]
    for row, s, position in rows_of(starts, np.minimum(lens, max_len), M):
        y, size = np.zeros((Hq, D)), np.zeros((Hq, D))
        first = max(0, position - window + 1) if window else 0
        for h in range(Hkv):
            seen = [kv for t in range(first, position + 1) if (kv := key_value(s, t, h)) is not None]
            if not seen:
                continue
            keys, vals = np.stack([a for a, _ in seen]), np.stack([b for _, b in seen])
            for e in range(h * Hq // Hkv, (h + 1) * Hq // Hkv):
                with np.errstate(invalid="ignore", over="ignore"):
                    score = keys @ qv[row, e] * scale
                    w = np.exp(score - score.max())
                    w /= w.sum()
                    y[e] = (w[:, None] * vals).sum(0)
                    size[e] = (w[:, None] * np.abs(vals)).sum(0)
        out[row] = y.reshape(-1), size.reshape(-1)
    return out


def sample(logits, temperature, top_k, top_p, min_p, u):
    """One row of logits (floats); the token, -1 if there is none."""
    x = np.where(np.isnan(logits), -np.inf, np.asarray(logits, np.float64))
    order = [int(i) for i in np.lexsort((np.arange(len(x)), -x)) if x[i] > -np.inf]
    if not order:
        return -1
    if not temperature > 0:
        return order[0]
    top = x[order[0]]
    w = {i: 1.0 if x[i] == top else 0.0 if np.isinf(top) else float(np.exp((x[i] - top) / np.float64(temperature))) for i in order}
    if top_k > 0:
        order = order[:top_k]
    if top_p < 1:
        total, run, kept = sum(w[i] for i in order), 0.0, []
        for i in order:
            kept.append(i)
            run += w[i]
            if run >= max(top_p, 0) * total:
                break
        order = kept
    if min_p > 0:
        order = [i for i in order if w[i] >= min(1.0, min_p)]
    order.sort()
    total, run = sum(w[i] for i in order), 0.0
    target = min(max(u, 0.0), 1.0) * total if u == u else 0.0
    for i in order:
        run += w[i]
        if run > target and w[i] > 0:
            return i
    return [i for i in order if w[i] > 0][-1]


def rotary_frequencies(rotary, base, scaling, factor, trained, slow, fast):
    """scaling: 0 none, 1 linear, 2 base, 3 parts."""
    if scaling == 2 and rotary > 2:
        base = base * factor ** (rotary / (rotary - 2))
    out = []
    for j in range(rotary // 2):
        f = base ** (-2 * j / rotary)
        if scaling == 1:
            f /= factor
        if scaling == 3:
            r = min(max((trained * f / (2 * np.pi) - slow) / (fast - slow), 0), 1)
            f = r * f + (1 - r) * f / factor
        out.append(f)
    return out
