"""Plain 64-bit implementations of the operators of include/spec_batch.h, written from their definitions, for the tests."""
import math

import numpy as np


def frequencies(rot, theta=10000.0, scaling="plain", factor=1.0, low=1.0, high=32.0, context=8192.0, magnitude=0.0):
    """(radians a position of every pair, factor of the tables)."""
    f = []
    for j in range(rot // 2):
        t = theta ** (-2.0 * j / rot)
        if scaling == "linear":
            t = t / factor
        elif scaling == "base":
            t = (theta * factor ** (rot / max(rot - 2, 1))) ** (-2.0 * j / rot)
        elif scaling == "bands":
            s = min(max((context * t / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
            t = t * (s + (1 - s) / factor)
        elif scaling == "ramp":
            d = lambda n: rot * math.log(context / (2 * math.pi * n)) / (2 * math.log(theta))
            a, b = max(math.floor(d(high)), 0), min(math.ceil(d(low)), rot - 1)
            g = min(max((j - a) / max(b - a, 0.001), 0.0), 1.0)
            t = t * (1 - g + g / factor)
        f.append(t)
    size = (magnitude or 0.1 * math.log(factor) + 1.0) if scaling == "ramp" else 1.0
    return np.array(f), size


def rotate(h, cos, sin, interleaved):
    """(result, magnitude of its two terms): h float64 [R][heads][hd]; cos, sin [R][rot / 2]."""
    rot = 2 * cos.shape[1]
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    c, s = cos[:, None, :], sin[:, None, :]
    out, mag = h.copy(), np.zeros_like(h)
    a, b = h[..., first], h[..., second]
    out[..., first], out[..., second] = a * c - b * s, b * c + a * s
    mag[..., first], mag[..., second] = np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)
    return out, mag


def attention(q, k_pages, v_pages, row_start, table, own_len, prefix_table, prefix_len, scale, before):
    """float64 q [R][nq][hd], pages [n][nkv][page][hd]; rows of no sequence stay as in `before`.  Returns (out, sum of the terms'
    magnitudes, positions seen, the largest sum of magnitudes behind a score) per row and head."""
    R, nq, hd = q.shape
    n_pages, nkv, page, _ = k_pages.shape
    g = nq // nkv
    out, mag = before.astype(np.float64).copy(), np.zeros((R, nq, hd))
    count, size = np.zeros((R, nq, 1)), np.zeros((R, nq, 1))
    capacity = table.shape[1] * page
    for b in range(len(own_len)):
        r0 = min(max(int(row_start[b]), 0), R)
        r1 = max(r0, min(int(row_start[b + 1]), R))
        n, L = r1 - r0, min(max(int(own_len[b]), 0), capacity)
        for i in range(n):
            places = [(prefix_table[j // page], j % page) for j in range(prefix_len)]
            places += [(table[b, j // page], j % page) for j in range(max(0, L - n + i + 1))]
            places = [(p, j) for p, j in places if 0 <= p < n_pages]
            out[r0 + i] = 0.0
            if not places:
                continue
            pg, at = np.array(places).T
            for h in range(nq):
                k, v = k_pages[pg, h // g, at], v_pages[pg, h // g, at]
                s = k @ q[r0 + i, h] * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                out[r0 + i, h] = w @ v
                mag[r0 + i, h] = w @ np.abs(v)
                size[r0 + i, h] = (np.abs(k) @ np.abs(q[r0 + i, h])).max() * scale
                count[r0 + i, h] = len(w)
    return out, mag, count, size


def verify(p, q, draft_start, drafted, u_accept, u_next):
    """(accepted, next token) of every sequence; p, q float64 rows, q None for drafts without probabilities."""
    A_out, y_out = [], []
    V = p.shape[1]
    for b in range(len(u_next)):
        first, end = int(draft_start[b]), int(draft_start[b + 1])
        if first < 0 or end < first or end > len(drafted):
            A_out.append(-1)
            y_out.append(-1)
            continue
        k, A = end - first, 0
        while A < k:
            x = int(drafted[first + A])
            if not 0 <= x < V:
                break
            give = q[first + A, x] if q is not None else 1.0
            if not float(u_accept[first + A]) * give < p[first + b + A, x]:
                break
            A += 1
        row = p[first + b + A]
        with np.errstate(invalid="ignore"):
            w = np.where(row > 0, row, 0.0)
            if A < k:
                if q is not None:
                    rest = row - q[first + A]
                    rest = np.where(rest > 0, rest, 0.0)
                else:
                    rest = w.copy()
                    if 0 <= drafted[first + A] < V:
                        rest[int(drafted[first + A])] = 0.0
                if rest.sum() > 0:
                    w = rest
        c = np.cumsum(w)
        above = np.nonzero((c > float(u_next[b]) * c[-1]) & (w > 0))[0]
        some = np.nonzero(w > 0)[0]
        A_out.append(A)
        y_out.append(int(above[0]) if len(above) else int(some[-1]) if len(some) else 0)
    return np.array(A_out), np.array(y_out)
