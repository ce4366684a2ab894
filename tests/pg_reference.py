"""Plain 64-bit forms of the paged cache's operators (include/d2c_pg.h): test infrastructure only."""
import numpy as np


def rotate(x, pos, freq, axis, pairing, inverse=False):
    """x [n, heads, D], pos [axes, n] -> turned by freq[i] * pos[axis[i]]."""
    y = np.array(x, np.float64)
    n = len(freq)
    if n == 0:
        return y
    w = np.asarray(pos, np.float64)[np.asarray(axis)].T * np.asarray(freq, np.float64)      # [rows, pairs]
    c, s = np.cos(w)[:, None], np.sin(w)[:, None] * (-1.0 if inverse else 1.0)
    a, b = (np.arange(n), n + np.arange(n)) if pairing == "halves" else (2 * np.arange(n), 2 * np.arange(n) + 1)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y


def index_of(row_start, length, at, n_rows, cap):
    """(sequence, index, length) of every packed row; sequence -1: none."""
    seq, idx, ln = np.full(n_rows, -1), np.zeros(n_rows, np.int64), np.zeros(n_rows, np.int64)
    for b in range(len(length)):
        lo, hi, n = row_start[b], row_start[b + 1], int(min(max(length[b], 0), cap))
        for r in range(lo, hi):
            seq[r], ln[r] = b, n
            idx[r] = at[r] if at is not None else n - (hi - lo) + (r - lo)
    return seq, idx, ln


def place(seq, idx, ln, pages, page_rows, n_pages):
    """(page, row in it) of each row, page -1 where it has none."""
    page, row = np.full(len(seq), -1), np.zeros(len(seq), np.int64)
    for r in range(len(seq)):
        if seq[r] >= 0 and 0 <= idx[r] < ln[r]:
            p = pages[seq[r], idx[r] // page_rows]
            if 0 <= p < n_pages:
                page[r], row[r] = p, idx[r] % page_rows
    return page, row


def seen(i, length, block, window, origin, numbered):
    """Which of `length` keys the row of index i sees; numbered: at, block or window is given."""
    j = np.arange(length)
    if i < 0 and numbered:
        return np.zeros(length, bool)
    ok = np.ones(length, bool)
    origin = max(0, origin)
    if block:
        end = origin if i < origin else origin + ((i - origin) // block + 1) * block
        ok &= j < end
    if window:
        ok &= j > i - window
        if not block:
            ok &= j < i + window
    return ok


def attention(q, k, v, ok, scale):
    """q [m, H, D], k, v [L, Hkv, D], ok [m, L] -> out [m, H, D], average [m, L], and for the error bounds sum p |v| and the largest sum |q k|."""
    m, H, D = q.shape
    L, Hkv, _ = k.shape
    out, avg, mag, big = np.zeros((m, H, D)), np.zeros((m, L)), np.zeros((m, H, D)), np.zeros((m, H))
    for r in range(m):
        js = np.flatnonzero(ok[r])
        if len(js) == 0:
            continue
        for g in range(Hkv):
            kk, vv = k[js, g], v[js, g]
            heads = np.arange(g * (H // Hkv), (g + 1) * (H // Hkv))
            s = q[r, heads] @ kk.T * scale
            big[r, heads] = (np.abs(q[r, heads]) @ np.abs(kk).T).max(1) * scale
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            out[r, heads], mag[r, heads] = p @ vv, p @ np.abs(vv)
            avg[r, js] += p.sum(0) / H
    return out, avg, mag, big
