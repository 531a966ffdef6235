"""Plain statements of the calls on pages, for their tests: a sequential simulation of the bookkeeping, the norms, rotation
and attention in 64 bits."""

import math

import numpy as np


def pages_step(table, lens, new_lens, free, n_free, page, n_tok):
    """table [n][width], lens, new_lens, free: lists.  Returns (table, free, n_free, lens, slots, positions, starts, code)."""
    table, free, n = [list(r) for r in table], list(free), len(lens)
    width, cap, code = len(table[0]) if table else 0, len(free), 0
    if not 0 <= n_free <= cap:
        code, n_free = min(code, -1), min(max(n_free, 0), cap)
    room = min(width * page, 2 ** 31 - 1)
    out, starts, row, ok = list(lens), [], 0, [True] * n
    pages = lambda x: -(-x // page)   # noqa: E731
    for r in range(n):
        if not 0 <= lens[r] <= room:
            code, ok[r] = min(code, -1), False
        elif new_lens[r] < 0:
            for j in range(pages(lens[r])):
                if n_free < cap:
                    free[n_free] = table[r][j]
                    n_free += 1
                else:
                    code = min(code, -1)
            out[r] = 0
    for r in range(n):
        x = max(new_lens[r], 0)
        starts.append(min(row, 2 ** 31 - 1))
        if ok[r] and x > 0 and (lens[r] + x > room or row + x > n_tok):
            code, ok[r] = min(code, -3), False
        row += x
    starts.append(min(row, 2 ** 31 - 1))
    top, want, taken = n_free, 0, 0
    slots, positions = [-1] * n_tok, [0] * n_tok
    for r in range(n):
        x = new_lens[r]
        if x <= 0:
            continue
        if ok[r]:
            old, more = pages(lens[r]), pages(lens[r] + x) - pages(lens[r])
            want += more
            if more and want > top:
                code, ok[r] = min(code, -3), False
            else:
                for j in range(more):
                    table[r][old + j] = free[top - 1 - taken]
                    taken += 1
                out[r] = lens[r] + x
        for i in range(min(x, max(n_tok - starts[r], 0))):
            t = starts[r] + i
            if t < n_tok:
                positions[t] = min(max(lens[r] + i, 0), 2 ** 31 - 1)
                if ok[r]:
                    p = table[r][positions[t] // page]
                    if 0 <= p < cap:
                        slots[t] = p * page + positions[t] % page
                    else:
                        code = min(code, -1)
    return table, free, top - taken, out, slots, positions, starts, code


def frequencies(rot, theta):
    return np.array([theta ** (-2.0 * i / rot) for i in range(rot // 2)])


def rotate(x, positions, freq, factor, interleaved, back=False):
    """x [n, heads, d] float64; the first 2 len(freq) elements turn by position * freq (the transposed rotation if back)"""
    half = len(freq)
    angle = np.asarray(positions, np.float64)[:, None] * freq
    z = np.exp((-1j if back else 1j) * angle)[:, None] * factor
    y = x.copy()
    ia, ib = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    w = (x[..., ia] + 1j * x[..., ib]) * z
    y[..., ia], y[..., ib] = w.real, w.imag
    return y


def norm(x, g, eps):
    return x if g is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * g


def norm_rope_grad(x, dy, g, eps, positions, freq, factor, interleaved):
    t = rotate(dy, positions, freq, factor, interleaved, back=True)
    if g is None:
        return t, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r
    return r * (t * g - n * (t * g * n).mean(-1, keepdims=True)), (t * n).sum((0, 1))


def visible(n, window, sinks):
    j = np.arange(n)
    return j[(j < sinks) | (j >= n - window)] if window else j


def attention(q, k_pages, v_pages, table, lens, scale, window=0, sinks=0):
    """q [n, h, d], pages [n_pages, h_kv, page, d] float64 -> (out, lse, sum p |v|)"""
    n, h, d = q.shape
    hk, page = k_pages.shape[1:3]
    out, lse, mag = np.zeros_like(q), np.full((n, h), -math.inf), np.zeros_like(q)
    for r in range(n):
        j = visible(lens[r], window, sinks)
        if len(j) == 0:
            continue
        p = np.asarray(table[r])[j // page]
        for head in range(h):
            m = head // (h // hk)
            k, v = k_pages[p, m, j % page], v_pages[p, m, j % page]
            s = k @ q[r, head] * scale
            top = s.max()
            e = np.exp(s - top)
            out[r, head], lse[r, head] = e @ v / e.sum(), top + math.log(e.sum())
            mag[r, head] = e @ np.abs(v) / e.sum()
    return out, lse, mag
