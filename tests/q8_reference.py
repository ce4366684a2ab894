"""The 8-bit operators in plain 64-bit numpy, written from their definitions (include/d2c_q8.h)."""
import numpy as np

BLOCK = 64
FMAX = float(np.finfo(np.float32).max)


def scale(a):
    """fl32(a / 127), 0 below 2^-100."""
    a = np.asarray(a, np.float64)
    return np.where(a < 2.0 ** -100, 0.0, (a / 127.0).astype(np.float32).astype(np.float64))


def code(x, s):
    x, s = np.broadcast_arrays(np.asarray(x, np.float64), np.asarray(s, np.float64))
    with np.errstate(invalid="ignore", divide="ignore"):
        c = np.clip(np.rint(np.where(s == 0, 0.0, x / np.where(s == 0, 1.0, s))), -127, 127)
    return np.where(np.isnan(x), 0.0, c).astype(np.int64)


def largest(x):
    """Largest finite magnitude over all but the first two axes' kv heads: x [rows, heads, D] -> [heads]."""
    a = np.abs(np.asarray(x, np.float64))
    a = np.where(a <= FMAX, a, 0.0)                # NaN and infinities count for nothing
    return a.max(axis=(0, 2)) if a.shape[0] else np.zeros(a.shape[1])


class Tensor8:
    """K or V of a cache: codes [blocks * 64, heads, D], scales [blocks, heads]."""

    def __init__(self, rows, heads, dim):
        nb = -(-rows // BLOCK)
        self.codes = np.zeros((nb * BLOCK, heads, dim), np.int64)
        self.scale = np.zeros((nb, heads))

    def update(self, idx, rows, L):
        """rows [m, heads, D] float64 become rows idx."""
        idx, rows = np.asarray(idx, np.int64), np.asarray(rows, np.float64)
        ok = (idx >= 0) & (idx < L)
        idx, rows = idx[ok], rows[ok]
        for b in np.unique(idx // BLOCK):
            at = np.flatnonzero(idx // BLOCK == b)
            lo, hi = b * BLOCK, min(L, (b + 1) * BLOCK)
            new = rows[at]
            want, old = scale(largest(new)), self.scale[b].copy()
            whole = len(at) == hi - lo
            grown = np.maximum(want, (old.astype(np.float32) * np.float32(1.25)).astype(np.float64))
            s = want if whole else np.where(want > old, grown, old)
            if not whole:
                blk = self.codes[lo:hi]
                self.codes[lo:hi] = np.where((s != old)[None, :, None], code(blk * old[None, :, None], s[None, :, None]), blk)
            self.codes[idx[at]] = code(new, s[None, :, None])
            self.scale[b] = s

    def values(self, L=None):
        v = self.codes * np.repeat(self.scale, BLOCK, 0)[:, :, None]
        return v if L is None else v[:L]

    def evict(self, kept):
        heads, dim = self.codes.shape[1:]
        out = Tensor8(len(kept), heads, dim)
        was = self.scale[kept // BLOCK]
        for b in range(out.scale.shape[0]):
            src = slice(b * BLOCK, min(len(kept), (b + 1) * BLOCK))
            out.scale[b] = was[src].max(0)
            c, w, s = self.codes[kept[src]], was[src][:, :, None], out.scale[b][None, :, None]
            out.codes[src] = np.where(w == s, c, code(c * w, s))
        return out


class Cache8:
    def __init__(self, rows, heads, dim):
        self.k, self.v = Tensor8(rows, heads, dim), Tensor8(rows, heads, dim)

    def update(self, idx, new_k, new_v, L):
        self.k.update(idx, new_k, L)
        self.v.update(idx, new_v, L)

    def evict(self, kept):
        out = Cache8.__new__(Cache8)
        out.k, out.v = self.k.evict(kept), self.v.evict(kept)
        return out


def k_bytes(codes):
    """Codes [blocks * 64, heads, D] in the order of the cache's K bytes."""
    nb, (_, h, d) = codes.shape[0] // BLOCK, codes.shape
    return (codes.reshape(nb, BLOCK, h, d // 16, 16).transpose(0, 2, 3, 1, 4).reshape(-1) + 128).astype(np.uint8)


def v_bytes(codes):
    nb, (_, h, d) = codes.shape[0] // BLOCK, codes.shape
    return (codes.reshape(nb, BLOCK // 4, 4, h, d).transpose(0, 3, 1, 4, 2).reshape(-1) + 128).astype(np.uint8)


def attention(q, k, v):
    """q [m, H, D], k / v [L, Hkv, D] -> (out [m, H, D], mean over the heads [m, L], sum p |v| [m, H, D], error bound of a score's exponential).

    The last: a term exp(s - max) computed in fp32 from exactly represented factors is off by at most this share: D products summed
    (2^-24 each of the sum of magnitudes), the scale factors (a few 2^-24 of the score), the difference to the maximum and the exponential."""
    m, H, D = q.shape
    out, total, mag, share = np.zeros((m, H, D)), np.zeros((m, k.shape[0])), np.zeros((m, H, D)), 0.0
    for h in range(H):
        g = h * k.shape[1] // H
        s = q[:, h] @ k[:, g].T / np.sqrt(D)
        sums = np.abs(q[:, h]) @ np.abs(k[:, g]).T / np.sqrt(D)
        share = max(share, float((D + 4) * sums.max() + 6 * np.abs(s).max() + 8) * 2.0 ** -24)
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        out[:, h], mag[:, h] = p @ v[:, g], p @ np.abs(v[:, g])
        total += p
    return out, total / H, mag, share


def linear(a, w):
    """Row and channel scales, codes, and the product as the definition's fp32 operations leave it."""
    def rows(x):
        x = np.asarray(x, np.float64)
        bad = ~np.isfinite(x).all(1)
        s = scale(np.where(bad, 0.0, np.abs(np.where(np.isfinite(x), x, 0.0)).max(1)))
        return code(np.where(bad[:, None], 0.0, x), s[:, None]), np.where(bad, np.nan, s).astype(np.float32)

    (qa, sa), (qw, sw) = rows(a), rows(w)
    total = (qa.astype(np.float64) @ qw.astype(np.float64).T).astype(np.float32)      # whole numbers below 2^53: exact, rounded once
    return (total * sa[:, None]) * sw[None, :], qw, sw


def weigh(avg, weight):
    a = np.nan_to_num(np.asarray(avg, np.float64), nan=0.0, posinf=1.0, neginf=0.0).clip(0, 1)
    return weight + np.floor(a * 2.0 ** 32).astype(np.int64).sum(0)


def keep(weight, protect, n):
    w = np.maximum(np.asarray(weight, np.int64), 0)
    p = np.zeros(len(w), np.int64) if protect is None else (np.asarray(protect) != 0).astype(np.int64)
    order = sorted(range(len(w)), key=lambda i: (-p[i], -int(w[i]), i))
    return np.sort(np.asarray(order[:n], np.int64))
