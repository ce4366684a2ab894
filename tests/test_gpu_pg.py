"""The paged cache on the GPU, through the C ABI, against the plain 64-bit forms of pg_reference.  Pages hold NaN where nothing was
appended, so that a read of what is not there shows."""
import numpy as np
import pytest
import torch

import pg_reference as R
from gpu_util import say

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}          # rounding to T
GEOS = {"mha": (4, 4, 64), "gqa": (8, 2, 64), "dream": (28, 4, 128), "odd": (5, 1, 128), "llada": (32, 32, 128), "three": (6, 2, 128), "thirds": (9, 3, 64),
        "wide": (48, 1, 64)}


def B():
    from paper_2509_23094_amd import binding
    return binding


def tensor(a, dtype):
    t = torch.from_numpy(np.ascontiguousarray(a, np.float32))
    return t.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda().contiguous()


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().double().cpu().numpy()


def rotary(pairs, ladder="shared", pairing="halves", theta=10000.0):
    return B().Rotary(pairs, theta, ladder=ladder, pairing=pairing)


# ------------------------------------------------------------------ rotation

def rotation_bound(x, pos, freq, axis, dtype):
    """Rounding to T, two products and a sum of at most |a| + |b|, sine and cosine within 2^-22, the angle's own 2^-52."""
    turn = np.abs(np.asarray(pos, np.float64)).max() * max(np.abs(freq).max(), 1e-9) * 2.0 ** -51
    size = np.abs(x).max(-1, keepdims=True) * 2
    return HALF[dtype] * np.sqrt(2) * size + size * (2.0 ** -21 + turn)


@pytest.mark.parametrize("pairs,pairing,ladder", [
    ([32], "halves", "shared"), ([8, 12, 12], "halves", "shared"), ([4, 2, 1, 1], "neighbours", "own"), ([16], "neighbours", "shared"),
    ([0, 8], "halves", "own")])
@pytest.mark.parametrize("src,dtype", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("n,heads", [(1, 1), (1, 28), (3, 5), (130, 7), (2500, 3)])
def test_rotate(pairs, pairing, ladder, src, dtype, n, heads):
    say("rotate %s %s %s %s -> %s, %d x %d" % (pairs, pairing, ladder, src, dtype, n, heads))
    rng = np.random.default_rng([n, heads, len(pairs)])
    rot = rotary(pairs, ladder, pairing)
    ctx = B().PgContext(4, 4, 64, dtype, rotary=rot)
    x = tensor(rng.standard_normal((n, heads * 64)), src)
    pos = rng.integers(0, 5000, (len(pairs), n))
    out = torch.full((n, heads * 64), 7.0, dtype=ctx.torch_dtype, device="cuda")
    ctx.d2c_pg_rotate(x, ints(pos), out)
    v = f64(x).reshape(n, heads, 64)
    want = R.rotate(v, pos, rot.freq, rot.axis, pairing)
    assert (np.abs(f64(out).reshape(n, heads, 64) - want) <= rotation_bound(v, pos, rot.freq, rot.axis, dtype)).all()
    still = 2 * len(rot.freq)
    assert torch.equal(out.view(n, heads, 64)[..., still:], x.view(n, heads, 64)[..., still:].to(ctx.torch_dtype))
    # back again
    back = torch.empty_like(out)
    ctx.d2c_pg_rotate(out, ints(pos), back, inverse=True)
    want = R.rotate(f64(out).reshape(n, heads, 64), pos, rot.freq, rot.axis, pairing, inverse=True)
    assert (np.abs(f64(back).reshape(n, heads, 64) - want) <= rotation_bound(v * 2, pos, rot.freq, rot.axis, dtype)).all()


def test_rotate_far_positions():
    """The whole range of 32 bits: the angle is held in 64 bits (2^31 revolutions leave 2^-21 of one at the worst)."""
    rot = rotary([32])
    ctx = B().PgContext(4, 4, 64, "f32", rotary=rot)
    pos = np.array([[0, 1, -1, 1 << 20, 10 ** 7 + 1, (1 << 31) - 1, -(1 << 31), -(1 << 31) + 12345]])
    x = tensor(np.random.default_rng(0).standard_normal((8, 64)), "f32")
    out = torch.empty_like(x)
    ctx.d2c_pg_rotate(x, ints(pos), out)
    v = f64(x).reshape(8, 1, 64)
    for r in range(8):
        want = R.rotate(v[r:r + 1], pos[:, r:r + 1], rot.freq, rot.axis, "halves")
        assert (np.abs(f64(out)[r] - want[0, 0]) <= rotation_bound(v[r:r + 1], pos[:, r:r + 1], rot.freq, rot.axis, "f32")[0, 0]).all()
    assert torch.equal(out[0], x[0])


def test_rotate_in_place_and_pitches():
    rot = rotary([16, 16])
    ctx = B().PgContext(4, 4, 64, "bf16", rotary=rot)
    rng = np.random.default_rng(3)
    wide = tensor(rng.standard_normal((37, 640)), "bf16")
    pos = ints(rng.integers(0, 900, (2, 37)))
    x, want = wide[:, 64:320], torch.empty((37, 256), dtype=torch.bfloat16, device="cuda")
    ctx.d2c_pg_rotate(x, pos, want)
    was = wide.clone()
    ctx.d2c_pg_rotate(x, pos, x)
    assert torch.equal(x, want) and torch.equal(wide[:, :64], was[:, :64]) and torch.equal(wide[:, 320:], was[:, 320:])
    with pytest.raises(B().D2CError, match="overlaps"):
        ctx.d2c_pg_rotate(wide[:, :256], pos, wide[:, 8:264])
    with pytest.raises(B().D2CError, match="overlaps"):
        ctx.d2c_pg_rotate(wide.view(torch.int16)[:, :256].view(torch.bfloat16), pos, wide[:, 320:576])     # between the same rows


def test_rotate_gradient():
    """inverse is the gradient: <dy, rotate(x)> differentiated by x, against differences (the operator is linear)."""
    rot = rotary([8, 16])
    ctx = B().PgContext(2, 2, 64, "f32", rotary=rot)
    rng = np.random.default_rng(5)
    x, dy = (tensor(rng.standard_normal((9, 128)), "f32") for _ in range(2))
    pos = ints(rng.integers(-100, 100, (2, 9)))
    dx, y = torch.empty_like(x), torch.empty_like(x)
    ctx.d2c_pg_rotate(dy, pos, dx, inverse=True)
    ctx.d2c_pg_rotate(x, pos, y)
    base = (f64(y) * f64(dy)).sum()
    for r, c in ((0, 0), (4, 70), (8, 127), (3, 25)):
        moved = x.clone()
        moved[r, c] += 1.0
        step = float(moved[r, c].double() - x[r, c].double())
        ctx.d2c_pg_rotate(moved, pos, y)
        # y's roundings: 256 values of at most about 4 with 2^-22 each, once in each of the two sums; they are the same but for one pair
        assert abs(((f64(y) * f64(dy)).sum() - base) / step - float(dx[r, c])) < 1e-4


# ------------------------------------------------------------------ a batch

class Pool:
    """A handle, a cache of NaN, sequences in pages of no order, and the plain cache beside it."""

    def __init__(self, geo, dtype, page_rows, lengths, seed=0, rot=None, max_rows=4096, spare=2, extra_cols=0, max_batch=None, scale=None):
        self.H, self.Hkv, self.D = GEOS[geo] if isinstance(geo, str) else geo
        self.dtype, self.P, self.rot, self.rng = dtype, page_rows, rot, np.random.default_rng([seed, page_rows])
        self.scale = scale or self.D ** -0.5
        self.ctx = B().PgContext(self.H, self.Hkv, self.D, dtype, page_rows=page_rows, max_rows=max_rows, max_batch=max_batch or max(1, len(lengths)),
                                 rotary=rot)
        need = [max(0, -(-n // page_rows)) for n in lengths]
        self.n_pages = sum(need) + spare
        self.lengths = list(lengths)
        self.pages = np.full((len(lengths), max(need, default=0) + extra_cols), -1, np.int64)
        order = self.rng.permutation(self.n_pages)
        for b, n in enumerate(need):
            self.pages[b, :n], order = order[:n], order[n:]
        self.cache = B().PgCache(self.ctx, self.n_pages)
        self.cache.k.fill_(float("nan"))
        self.cache.v.fill_(float("nan"))
        self.k, self.v = (np.full((self.n_pages, page_rows, self.Hkv, self.D), np.nan) for _ in range(2))

    def batch(self, counts, at=None, origin=None, lead=0, tail=0):
        """Sequences of `counts` rows, with rows of no sequence in front and behind."""
        self.row_start = lead + np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
        self.n_rows, self.at, self.origin = int(self.row_start[-1]) + tail, at, origin
        self.where = R.index_of(self.row_start, self.lengths, at, self.n_rows, self.pages.shape[1] * self.P)
        return B().PgBatch(self.ctx, ints(self.row_start), ints(self.lengths), ints(self.pages), self.n_rows, at=None if at is None else ints(at),
                           origin=None if origin is None else ints(origin))

    def values(self, n, heads, src=None, factor=1.0):
        t = tensor(self.rng.standard_normal((n, heads * self.D)) * factor, src or self.dtype)
        return t, f64(t).reshape(n, heads, self.D)

    def rounded(self, a):
        return f64(tensor(a, self.dtype))

    def append(self, batch, pos=None, src=None, with_q=False, factor=1.0, values=None):
        (k, nk), (v, nv) = values or (self.values(self.n_rows, self.Hkv, src, factor), self.values(self.n_rows, self.Hkv, src, factor))
        q = nq = q_out = None
        if with_q:
            q, nq = self.values(self.n_rows, self.H, src)
            q_out = torch.full((self.n_rows, self.H * self.D), 7.0, dtype=self.ctx.torch_dtype, device="cuda")
        self.ctx.d2c_pg_append(self.cache, batch, k, v, pos=None if pos is None else ints(pos), q=q, q_out=q_out)
        torch.cuda.synchronize()
        seq, idx, ln = self.where
        p = np.asarray(pos) if pos is not None else np.repeat(idx[None], self.rot.n_axes if self.rot else 1, 0)
        if self.rot:
            self.bound = rotation_bound(nk, p, self.rot.freq, self.rot.axis, self.dtype)
            nk = R.rotate(nk, p, self.rot.freq, self.rot.axis, "halves" if self.rot.pairing == 0 else "neighbours")
            if with_q:
                bound = rotation_bound(nq, p, self.rot.freq, self.rot.axis, self.dtype)
                nq = R.rotate(nq, p, self.rot.freq, self.rot.axis, "halves" if self.rot.pairing == 0 else "neighbours")
        else:
            self.bound = HALF[self.dtype] * np.abs(nk).max(2, keepdims=True)
            bound = HALF[self.dtype] * np.abs(nq).max(2, keepdims=True) if with_q else None
        if with_q:
            got = f64(q_out).reshape(self.n_rows, self.H, self.D)
            mine = seq >= 0
            assert (np.abs(got - nq)[mine] <= np.broadcast_to(bound, got.shape)[mine]).all()
            assert (got[~mine] == 7.0).all()
        page, row = R.place(seq, idx, ln, self.pages, self.P, self.n_pages)
        there = page >= 0
        self.k[page[there], row[there]], self.v[page[there], row[there]] = nk[there], self.rounded(nv.reshape(self.n_rows, -1)).reshape(nv.shape)[there]

    def raw(self):
        """The pages as the header lays them out: [n_pages, P, Hkv, D] of K and of V."""
        E = 8 if self.dtype == "bf16" else 4
        units = (self.n_pages, self.Hkv, self.P // 32)
        k = f64(self.cache.k).reshape(*units, self.D // E, 32, E)
        slot = [(t & 19) | (t & 4) << 1 | (t & 8) >> 1 if E == 8 else t for t in range(32)]
        k = k[:, :, :, :, slot].transpose(0, 2, 4, 1, 3, 5).reshape(self.k.shape)
        v = f64(self.cache.v).reshape(*units, 32 // E, self.D, E).transpose(0, 2, 3, 5, 1, 4).reshape(self.v.shape)
        return k, v

    def check(self):
        """Every page, to the bit for V and for K within the rotation's bound; what was not written is still NaN."""
        k, v = self.raw()
        assert np.array_equal(np.isnan(k), np.isnan(self.k))
        assert np.array_equal(v, self.v, equal_nan=True)
        tol = np.nanmax(self.bound) if np.size(self.bound) else 0
        assert (np.abs(k - self.k)[~np.isnan(k)] <= tol).all()
        self.k = k                                     # as stored: what follows starts from the same values

    def fill(self, factor=1.0):
        b = self.batch(self.lengths)
        self.append(b, factor=factor)
        self.k = self.raw()[0]
        return self

    def keys(self, b):
        """K and V of sequence b as the plain cache has them, and which of its rows are there."""
        n = int(min(max(self.lengths[b], 0), self.pages.shape[1] * self.P))
        j = np.arange(n)
        page = self.pages[b, j // self.P] if n else j
        there = (page >= 0) & (page < self.n_pages)
        safe = np.where(there, page, 0)
        return self.k[safe, j % self.P], self.v[safe, j % self.P], there

    def attend(self, batch, block=0, window=0, scale=None, average=False, q=None, avg_cols=None, factor=1.0):
        q, nq = q or self.values(self.n_rows, self.H, factor=factor)
        out = torch.full((self.n_rows, self.H * self.D), 7.0, dtype=self.ctx.torch_dtype, device="cuda")
        cols = avg_cols or max(1, max(self.lengths, default=1))
        avg = torch.full((self.n_rows, cols), 7.0, device="cuda") if average else None
        self.ctx.d2c_pg_attention(self.cache, batch, q, out, block=block, window=window, scale=scale, attn_avg=avg)
        torch.cuda.synchronize()
        self.expect(nq, out, avg, block, window, scale)
        return out, avg

    def expect(self, nq, out, avg, block, window, scale=None):
        seq, idx, _ = self.where
        got = f64(out).reshape(self.n_rows, self.H, self.D)
        ga = None if avg is None else f64(avg)
        scale = scale or self.scale
        numbered = self.at is not None or block > 0 or window > 0
        assert (got[seq < 0] == 7.0).all()
        for b in range(len(self.lengths)):
            rows = np.flatnonzero(seq == b)
            if len(rows) == 0:
                continue
            k, v, there = self.keys(b)
            n = len(there)
            origin = 0 if self.origin is None else int(self.origin[b])
            ok = np.array([R.seen(idx[r], n, block, window, origin, numbered) & there for r in rows]).reshape(len(rows), n)
            o, a, mag, big = R.attention(nq[rows], np.nan_to_num(k), v, ok, scale)
            # a score: D products and sums in fp32, the scale and log2(e) on it; twice in a probability (its own and the sum's).  Sums over
            # a lane's keys, over lanes, waves and splits.  bf16: a probability rounded once.
            score = (self.D + 8) * 2.0 ** -24 * big[..., None]
            rel = 2 * score + (n / 16 + 160) * 2.0 ** -24 + 2.0 ** -20 + (HALF["bf16"] if self.dtype == "bf16" else 0)
            bound = HALF[self.dtype] * np.abs(o) + rel * mag + 1e-30
            with np.errstate(invalid="ignore"):
                bad = ~(np.abs(got[rows] - o) <= bound) & ~((got[rows] == o) | (np.isnan(o) & np.isnan(got[rows])))
            assert not bad.any(), (b, len(rows), n, float(np.nanmax(np.abs(got[rows] - o))), np.argwhere(bad)[:4].tolist())
            if ga is not None:
                cols = min(n, ga.shape[1])
                tol = (2 * score.max(1) + 2.0 ** -19 + (n / 16 + self.H + 160) * 2.0 ** -24) * a[:, :cols] + 1e-30
                assert (np.abs(ga[rows][:, :cols] - a[:, :cols]) <= tol).all(), (b, float(np.abs(ga[rows][:, :cols] - a[:, :cols]).max()))
                assert (ga[rows][:, :cols][~ok[:, :cols]] == 0).all()
                assert (ga[rows][:, cols:] == 7.0).all()
        if ga is not None:
            assert (ga[seq < 0] == 7.0).all()


# ------------------------------------------------------------------ append and read

@pytest.mark.parametrize("src,dtype", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("geo,page_rows", [("mha", 32), ("gqa", 64), ("odd", 128), ("dream", 256)])
@pytest.mark.parametrize("turned", [None, "index", "axes"])
def test_append(src, dtype, geo, page_rows, turned):
    say("append %s %s -> %s pages of %d %s" % (geo, src, dtype, page_rows, turned))
    half = GEOS[geo][2] // 2
    rot = {None: None, "index": rotary([half]), "axes": rotary([8, 8, half - 32], "own", "neighbours")}[turned]
    p = Pool(geo, dtype, page_rows, [70, 1, 0, 33, 300, 257], rot=rot)
    b = p.batch([70, 1, 0, 5, 131, 1], lead=2, tail=3)
    pos = p.rng.integers(-300, 100000, (3, p.n_rows)) if turned == "axes" else None
    p.append(b, pos=pos, src=src, with_q=True)
    p.check()
    # rows read back are the stored bits
    out = [torch.full((p.n_rows, p.Hkv * p.D), 7.0, dtype=p.ctx.torch_dtype, device="cuda") for _ in range(2)]
    p.ctx.d2c_pg_read(p.cache, b, *out)
    seq, idx, ln = p.where
    page, row = R.place(seq, idx, ln, p.pages, p.P, p.n_pages)
    for got, want in zip(out, (p.k, p.v)):
        got = f64(got).reshape(p.n_rows, p.Hkv, p.D)
        assert np.array_equal(got[page >= 0], want[page[page >= 0], row[page >= 0]])
        assert (got[seq < 0] == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_selected_rows_bad_pages_and_bad_indices(dtype):
    """Rows in any order; indices outside the sequence and pages that are not there leave everything else alone, and read as zeros."""
    p = Pool("gqa", dtype, 32, [100, 64, 90], rot=rotary([32]), extra_cols=1)
    p.pages[0, 1], p.pages[2, 0], p.pages[2, 2] = p.n_pages, -5, 1 << 30
    at = [99, 0, 31, 32, 63, 64, -1, 100, 5, -(1 << 31), (1 << 31) - 1, 40, 0, 12, 33, 89, 70]
    b = p.batch([10, 2, 5], at=np.array(at))
    p.append(b, with_q=True)
    p.check()
    out = [torch.full((p.n_rows, p.Hkv * p.D), 7.0, dtype=p.ctx.torch_dtype, device="cuda") for _ in range(2)]
    p.ctx.d2c_pg_read(p.cache, b, *out)
    page, _ = R.place(*p.where, p.pages, p.P, p.n_pages)
    assert all((f64(o)[page < 0] == 0).all() for o in out) and (page < 0).any() and (page >= 0).any()


def test_append_from_a_packed_projection():
    """q, k and v as columns of one [n, d_q + 2 d_kv] projection, as a fused product leaves them; only V or K read."""
    p = Pool("three", "bf16", 64, [130, 7], rot=rotary([64]))
    b = p.batch([130, 7])
    d_q, d_kv = p.H * p.D, p.Hkv * p.D
    x = tensor(p.rng.standard_normal((p.n_rows, d_q + 2 * d_kv)), "f32")
    q, k, v = x[:, :d_q], x[:, d_q:d_q + d_kv], x[:, d_q + d_kv:]
    q_out = torch.empty((p.n_rows, d_q), dtype=torch.bfloat16, device="cuda")
    p.ctx.d2c_pg_append(p.cache, b, k, v, q=q, q_out=q_out)
    got = p.raw()
    want = torch.empty_like(q_out)
    other = Pool("three", "bf16", 64, [130, 7], rot=rotary([64]))
    p.ctx.d2c_pg_append(other.cache, b, k.contiguous(), v.contiguous(), q=q.contiguous(), q_out=want)
    assert torch.equal(q_out, want) and all(np.array_equal(g, w, equal_nan=True) for g, w in zip(got, other.raw()))
    one = [torch.zeros((p.n_rows, d_kv), dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    p.ctx.d2c_pg_read(p.cache, b, one[0], one[1])
    p.ctx.d2c_pg_read(p.cache, b, one[2], None)
    p.ctx.d2c_pg_read(p.cache, b, None, one[3])
    assert torch.equal(one[0], one[2]) and torch.equal(one[1], one[3]) and not torch.equal(one[0], one[1])


def test_append_of_an_aligned_prompt_and_of_an_unaligned_one():
    for first in (0, 3, 8, 13):
        p = Pool("mha", "bf16", 32, [first + 77], rot=rotary([32]))
        p.append(p.batch([77]))
        p.check()


def test_pages_past_32_bits():
    """More than 2^32 values in a cache: pages at its end."""
    H, Hkv, D = GEOS["dream"]
    ctx = B().PgContext(H, Hkv, D, "bf16", page_rows=256, max_rows=8, max_batch=1)
    n_pages = (1 << 32) // (256 * Hkv * D) + 3
    cache = B().PgCache(ctx, n_pages)
    rng = np.random.default_rng(0)
    pages = ints([[n_pages - 1, 0, n_pages - 2]])
    length = 700
    b = B().PgBatch(ctx, ints([0, length]), ints([length]), pages, length)
    k, v = (tensor(rng.standard_normal((length, Hkv * D)), "bf16") for _ in range(2))
    ctx.d2c_pg_append(cache, b, k, v)
    out = [torch.zeros_like(k) for _ in range(2)]
    ctx.d2c_pg_read(cache, b, *out)
    assert torch.equal(out[0], k) and torch.equal(out[1], v)
    q, o = tensor(rng.standard_normal((8, H * D)), "bf16"), torch.zeros((8, H * D), dtype=torch.bfloat16, device="cuda")
    ctx.d2c_pg_attention(cache, B().PgBatch(ctx, ints([0, 8]), ints([length]), pages, 8), q, o, block=1)
    ok = np.array([R.seen(length - 8 + r, length, 1, 0, 0, True) for r in range(8)])
    want, _, mag, _ = R.attention(f64(q).reshape(8, H, D), f64(k).reshape(-1, Hkv, D), f64(v).reshape(-1, Hkv, D), ok, D ** -0.5)
    assert (np.abs(f64(o).reshape(8, H, D) - want) <= HALF["bf16"] * np.abs(want) + 1.1 * HALF["bf16"] * mag).all()


# ------------------------------------------------------------------ attention

MASKS = [dict(), dict(block=1), dict(block=32), dict(block=1, window=40), dict(window=9), dict(block=7, window=1)]


@pytest.mark.parametrize("mask", MASKS, ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("geo,page_rows,lengths,counts", [
    ("mha", 32, [1], [1]), ("dream", 64, [1023], [1]), ("gqa", 32, [257, 33, 32, 31, 1, 0, 300], [1, 2, 0, 31, 1, 3, 40]),
    ("odd", 128, [400, 129, 128], [7, 129, 1]), ("three", 256, [513, 64], [200, 64]), ("mha", 64, [389], [389]),
    ("llada", 64, [130, 97], [70, 97]), ("thirds", 32, [333, 70], [33, 1]), ("wide", 64, [200, 65], [3, 65])])
def test_attention(geo, page_rows, lengths, counts, dtype, mask):
    say("attention %s %s pages of %d, %s rows on %s, %s" % (geo, dtype, page_rows, counts, lengths, mask))
    p = Pool(geo, dtype, page_rows, lengths, seed=len(lengths)).fill()
    b = p.batch(counts, lead=1, tail=2)
    p.attend(b, average=True, **mask)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_of_more_rows_than_the_cache_has(dtype):
    """Without a mask any number of queries may look at a cache; with one, rows with negative indices see nothing."""
    p = Pool("gqa", dtype, 32, [5, 40]).fill()
    b = p.batch([9, 70])
    p.attend(b, average=True)
    p.attend(b, block=1, average=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask", [dict(), dict(block=1), dict(block=16, window=50), dict(window=20)], ids=str)
def test_attention_of_selected_rows(dtype, mask):
    """Indices in any order, twice, negative, past the end; blocks counted from an origin."""
    p = Pool("gqa", dtype, 64, [300, 100, 64], seed=4).fill()
    at = np.concatenate([p.rng.permutation(300)[:61], [-1, 299, 0, 0, 5000, -(1 << 31), (1 << 31) - 1], p.rng.integers(0, 100, 20), [63, 63, 0]])
    b = p.batch([68, 20, 3], at=at, origin=np.array([70, 0, -3]))
    p.attend(b, average=True, **mask)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_origin_past_the_end_and_large_blocks(dtype):
    p = Pool("mha", dtype, 32, [90, 50]).fill()
    p.attend(p.batch([90, 50], origin=np.array([1000, (1 << 31) - 1])), block=1)
    p.attend(p.batch([90, 50], origin=np.array([3, 0])), block=1 << 30, window=1 << 30)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("geo,length,counts", [("odd", 5000, [1]), ("gqa", 9000, [3]), ("dream", 20001, [1]), ("mha", 3500, [60]), ("three", 2500, [130])])
def test_long_caches(dtype, geo, length, counts):
    """Keys split over workgroups and joined."""
    p = Pool(geo, dtype, 128, [length, 40, length // 3], seed=2).fill()
    b = p.batch(counts + [1, 2])
    p.attend(b, block=1)
    p.attend(b, window=length // 2)
    if len(counts) == 1 and counts[0] < 100:
        p.attend(b, average=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("batch", [65, 300, 1024])
def test_many_sequences(dtype, batch):
    rng = np.random.default_rng(batch)
    lengths = rng.integers(0, 60, batch).tolist()
    lengths[batch // 2] = 900
    p = Pool("mha", dtype, 32, lengths).fill()
    counts = np.minimum(rng.integers(0, 4, batch), lengths)
    b = p.batch(counts, tail=5)
    p.attend(b, block=1, average=True)
    p.append(p.batch(counts, tail=5))
    p.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask", [dict(), dict(block=1)], ids=str)
def test_missing_pages_are_not_seen(dtype, mask):
    p = Pool("gqa", dtype, 32, [200, 64, 4000], seed=1).fill()
    p.pages[0, 2], p.pages[0, 5], p.pages[1, 0], p.pages[1, 1] = -1, p.n_pages, -7, 1 << 30
    p.pages[2, 3:90] = -1
    b = p.batch([40, 10, 2])
    p.attend(b, average=True, **mask)


def test_shared_pages_and_lengths_past_the_table():
    """Two sequences share their prompt's pages; a length past the page table counts as what the table holds."""
    p = Pool("dream", "bf16", 64, [192, 200], spare=1).fill()
    p.pages[1, :2] = p.pages[0, :2]
    p.lengths = [1 << 30, 200]
    b = p.batch([3, 5])
    p.attend(b, block=1)
    p.lengths = [-9, 200]
    p.attend(p.batch([3, 5]), average=True, avg_cols=100)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("counts,length", [([40], 300), ([3], 300), ([200], 300), ([2], 6000)])
def test_what_a_row_does_not_see_does_not_change_it(dtype, what, counts, length):
    """K and V of unseen rows hold NaN or infinities: behind a row's own index, before its window, past the length."""
    p = Pool("gqa", dtype, 32, [length, 50], seed=8).fill()
    q = p.values(counts[0] + 20, p.H)
    b = p.batch(counts + [20])
    clean, _ = p.attend(b, block=1, window=30, q=q)
    spot = [length - 1, length - 2, length - 20] + ([length - counts[0], 0] if counts[0] < length else [])
    at = B().PgBatch(p.ctx, ints([0, len(spot)]), ints([length]), ints(p.pages[:1]), len(spot), at=ints(spot))
    t = torch.full((len(spot), p.Hkv * p.D), what, dtype=p.ctx.torch_dtype, device="cuda")
    p.ctx.d2c_pg_append(p.cache, at, t, t)
    out = torch.zeros_like(clean)
    p.ctx.d2c_pg_attention(p.cache, b, q[0], out, block=1, window=30)
    idx = length - counts[0] + np.arange(counts[0])
    for r, i in enumerate(idx):
        hit = any(i - 30 < s <= i for s in spot)
        assert torch.equal(out[r], clean[r]) != hit, (r, i)
    assert torch.equal(out[counts[0]:], clean[counts[0]:])


def test_queries_that_are_not_finite_stay_by_themselves():
    p = Pool("gqa", "bf16", 32, [100]).fill()
    b = p.batch([50])
    q, nq = p.values(50, p.H)
    clean, _ = p.attend(b, block=1, q=(q, nq))
    q[7], q[31, :64] = float("nan"), float("inf")
    out = torch.zeros_like(clean)
    p.ctx.d2c_pg_attention(p.cache, b, q, out, block=1)
    keep = [r for r in range(50) if r not in (7, 31)]
    assert torch.equal(out[keep], clean[keep]) and out[7].isnan().all() and torch.equal(out[31, 64:], clean[31, 64:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_loud_and_quiet_scores(dtype):
    """Scores of thousands (one key takes all) and of nearly nothing (the mean of V)."""
    p = Pool("gqa", dtype, 64, [500, 70]).fill(factor=8.0)
    b = p.batch([45, 70])
    p.attend(b, block=1, factor=16.0)
    p.attend(b, scale=1e-6)
    p.attend(b, scale=3.0, factor=0.01)


def test_pitches():
    """q and out as columns of wider rows."""
    p = Pool("gqa", "bf16", 32, [200, 90]).fill()
    b = p.batch([33, 90])
    wide, to = tensor(p.rng.standard_normal((123, 1024)), "bf16"), torch.full((123, 528), 7.0, dtype=torch.bfloat16, device="cuda")
    q, out = wide[:, 8:8 + 512], to[:, 8:520]
    p.ctx.d2c_pg_attention(p.cache, b, q, out, block=1)
    p.expect(f64(q).reshape(123, 8, 64), out.contiguous(), None, 1, 0)
    assert (to[:, :8] == 7).all() and (to[:, 520:] == 7).all()


def test_bits_repeat():
    p = Pool("dream", "bf16", 64, [5000, 800, 40]).fill()
    b = p.batch([1, 300, 40])
    q = p.values(p.n_rows, p.H)
    first, avg = p.attend(b, block=1, q=q, average=True)
    for _ in range(5):
        out, again = torch.zeros_like(first), torch.zeros_like(avg)
        p.ctx.d2c_pg_attention(p.cache, b, q[0], out, block=1, attn_avg=again)
        assert torch.equal(out, first)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_captured_step_follows_its_lengths(dtype):
    """One graph of append and attention, replayed as sequences grow; eager work and a second handle's graph in between."""
    p = Pool("gqa", dtype, 32, [700, 90, 33], rot=rotary([32])).fill()
    other = Pool("mha", dtype, 64, [400], seed=3).fill()
    p.k = p.raw()[0]
    start, n = ints([0, 1, 2, 3]), 3
    length, pages = ints([600, 60, 5]), ints(p.pages)
    b = B().PgBatch(p.ctx, start, length, pages, n)
    k, v, q, turned, out = (torch.zeros((n, w), dtype=p.ctx.torch_dtype, device="cuda") for w in (p.Hkv * p.D,) * 2 + (p.H * p.D,) * 3)
    avg = torch.zeros((n, 700), device="cuda")
    ob = other.batch([40])
    oq, oo = other.values(40, other.H)[0], torch.zeros((40, other.H * other.D), dtype=p.ctx.torch_dtype, device="cuda")

    def step():
        p.ctx.d2c_pg_append(p.cache, b, k, v, q=q, q_out=turned)
        p.ctx.d2c_pg_attention(p.cache, b, turned, out, block=1, attn_avg=avg)

    graph, graph2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
        other.ctx.d2c_pg_attention(other.cache, ob, oq, oo)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    with torch.cuda.graph(graph2):
        other.ctx.d2c_pg_attention(other.cache, ob, oq, oo)
    want_other = oo.clone()
    for t in range(6):
        length.copy_(ints([600 + 17 * t, 60 + t, 5 + 5 * t]))
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape))
        avg.zero_()
        graph.replay()
        oo.zero_()
        graph2.replay()
        torch.cuda.synchronize()
        got, got_avg, got_q = out.clone(), avg.clone(), turned.clone()
        assert torch.equal(oo, want_other)
        out.zero_()
        avg.zero_()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(got_avg, avg) and torch.equal(got_q, turned)
        p.lengths = length.tolist()
        p.batch([1, 1, 1])
        p.k, p.v = p.raw()
        avg2 = avg.clone()
        for i, ln in enumerate(p.lengths):
            avg2[i, ln:] = 7.0
        p.expect(f64(got_q).reshape(n, p.H, p.D), got, avg2, 1, 0)


def test_streams():
    """Two handles on two streams at once, on tensors of a third."""
    pools = [Pool("dream", "bf16", 64, [3000], seed=s).fill() for s in (1, 2)]
    work = []
    for p in pools:
        b = p.batch([2])
        q = p.values(2, p.H)
        work.append((p, b, q, p.attend(b, block=1, q=q)[0]))
    streams = [torch.cuda.Stream() for _ in pools]
    torch.cuda.synchronize()
    outs = [torch.zeros_like(w[3]) for w in work]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, o, (p, b, q, _) in zip(streams, outs, work):
            with torch.cuda.stream(s):
                p.ctx.d2c_pg_attention(p.cache, b, q[0], o, block=1)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w[3]) for o, w in zip(outs, work))


# ------------------------------------------------------------------ caches of middle length (one launch of wider workgroups)

@pytest.mark.parametrize("mask", [dict(), dict(block=1), dict(block=32, window=300)], ids=str)
@pytest.mark.parametrize("geo,page_rows,lengths,counts", [
    ("dream", 32, [760, 33, 0, 449], [1, 1, 2, 1]),       # each wave several units, one, none
    ("llada", 64, [1500, 64, 1], [70, 1, 1]),             # more than 64 tiles
    ((12, 2, 64), 256, [1400], [200]),
    ("gqa", 32, [500, 700], [3, 40]),
])
def test_middle_caches(geo, page_rows, lengths, counts, mask):
    say("%s %s %s" % (geo, lengths, mask))
    p = Pool(geo, "bf16", page_rows, lengths, seed=4).fill()
    p.attend(p.batch(counts, lead=1, tail=2), average=True, **mask)


def test_middle_caches_of_many_sequences():
    lengths = [(37 * i) % 701 for i in range(60)]
    p = Pool("dream", "bf16", 64, lengths, seed=4).fill()
    p.attend(p.batch([1 if n else 0 for n in lengths]), block=1)


@pytest.mark.parametrize("what", [float("nan"), float("inf")])
@pytest.mark.parametrize("counts,length", [([3], 700), ([100], 600)])
def test_middle_caches_do_not_show_what_is_not_seen(what, counts, length):
    test_what_a_row_does_not_see_does_not_change_it("bf16", what, counts, length)


# ------------------------------------------------------------------ sequences with many products (the kernel for many queries)

def expect_big(p, q, out, avg, block=0, window=0):
    """Pool.expect with the plain form in 64 bits on the GPU: the same bounds."""
    seq, idx, _ = p.where
    numbered = p.at is not None or block > 0 or window > 0
    got, G = out.double().view(p.n_rows, p.H, p.D), p.H // p.Hkv
    assert bool((out[torch.from_numpy(seq < 0).cuda()] == 7.0).all())
    for b in range(len(p.lengths)):
        rows = np.flatnonzero(seq == b)
        if len(rows) == 0:
            continue
        k, v, there = p.keys(b)
        n, origin = len(there), 0 if p.origin is None else int(p.origin[b])
        if n == 0:                           # nothing to see
            assert not bool(got[torch.from_numpy(rows).cuda()].any()) and (avg is None or bool((avg[torch.from_numpy(rows).cuda()] == 7.0).all()))
            continue
        ok = torch.from_numpy(np.array([R.seen(idx[r], n, block, window, origin, numbered) & there for r in rows]).reshape(len(rows), n)).cuda()
        k, v = (torch.from_numpy(np.ascontiguousarray(np.where(there[:, None, None], x, 0.0))).cuda() for x in (k, v))
        sees, where, total = ok.any(1), torch.from_numpy(rows).cuda(), torch.zeros(ok.shape, dtype=torch.float64, device="cuda")
        worst = torch.zeros(len(rows), dtype=torch.float64, device="cuda")
        for h in range(p.H):
            kk, vv, qq = k[:, h // G].contiguous(), v[:, h // G].contiguous(), q[where, h * p.D:(h + 1) * p.D].double()
            s = (qq @ kk.t()) * p.scale
            score = (p.D + 8) * 2.0 ** -24 * ((qq.abs() @ kk.abs().t()) * p.scale).amax(1)
            w = torch.softmax(s.masked_fill(~ok, -float("inf")), 1)
            w[~sees] = 0
            o, mag = w @ vv, w @ vv.abs()
            rel = 2 * score[:, None] + (n / 16 + 160) * 2.0 ** -24 + 2.0 ** -20 + (HALF["bf16"] if p.dtype == "bf16" else 0)
            off = (got[where, h] - o).abs()
            assert bool((off <= HALF[p.dtype] * o.abs() + rel * mag + 1e-30).all()), (b, h, float(off.max()))
            total += w / p.H
            worst = torch.maximum(worst, score)
        if avg is not None:
            tol = (2 * worst[:, None] + 2.0 ** -19 + (n / 16 + p.H + 160) * 2.0 ** -24) * total + 1e-30
            assert bool(((avg[where, :n].double() - total).abs() <= tol).all()) and bool((avg[where, n:] == 7.0).all())
            assert bool((avg[where, :n][~ok] == 0).all())


def attend_big(p, batch, average=False, **mask):
    q = torch.randn((p.n_rows, p.H * p.D), device="cuda", generator=torch.Generator("cuda").manual_seed(5)).to(p.ctx.torch_dtype)
    out = torch.full_like(q, 7.0)
    avg = torch.full((p.n_rows, max(p.lengths)), 7.0, device="cuda") if average else None
    p.ctx.d2c_pg_attention(p.cache, batch, q, out, attn_avg=avg, **mask)
    torch.cuda.synchronize()
    expect_big(p, q, out, avg, **mask)
    return q, out


BIG = {  # (heads, kv heads, head dimension), type, lengths, rows: the first has more than 64e6 (128e6, 256e6) products, the others fewer
    "llada": ((32, 32, 128), "bf16", [3500, 900, 64, 0], [700, 1, 40, 2]),
    "dream": ((28, 4, 128), "bf16", [4001, 4001], [777, 1]),
    "d64": ((32, 8, 64), "bf16", [3333, 100], [1801, 100]),
    "f32": ((32, 32, 128), "f32", [5003, 33], [2601, 33]),
    "f32 d64": ((33, 3, 64), "f32", [5003], [2601]),
}


@pytest.mark.parametrize("mask", [dict(), dict(block=1), dict(block=48)], ids=str)
@pytest.mark.parametrize("name", BIG)
def test_many_products(name, mask):
    geo, dtype, lengths, counts = BIG[name]
    say("many products, %s, %s" % (name, mask))
    p = Pool(geo, dtype, 64, lengths, seed=3).fill()
    attend_big(p, p.batch(counts, lead=1, tail=2), average=name == "dream", **mask)


@pytest.mark.parametrize("geo,counts,lengths", [
    ("llada", [512, 1, 287, 250, 512, 0, 512], [1500, 1500, 1400, 1300, 1450, 9, 700]),      # together; two do not fill their tiles
    ("dream", [110] * 17 + [30, 2], [1000] * 17 + [900, 64]),                                # more than 16 sequences
])
def test_many_products_together(geo, counts, lengths):
    """None of the sequences has many products by itself."""
    p = Pool(geo, "bf16", 64, lengths, seed=13, max_rows=4096).fill()
    b = p.batch(counts, lead=1, tail=2)
    attend_big(p, b, block=1)
    attend_big(p, b, average=True)


def test_many_products_in_a_window():
    p = Pool("llada", "bf16", 32, [4100, 50], seed=5).fill()
    b = p.batch([3001, 50], origin=np.array([7, 0]))
    attend_big(p, b, block=1, window=900)
    attend_big(p, b, block=32, window=901)
    attend_big(p, b, window=450)


def test_many_products_of_selected_rows_and_missing_pages():
    """Indices in no order, some that see nothing; pages that are not there, inside blocks and between them."""
    p = Pool("llada", "bf16", 32, [3200, 40], seed=6).fill()
    p.pages[0, 5], p.pages[0, 10:13], p.pages[0, 99] = -1, p.n_pages, -9
    at = np.concatenate([p.rng.permutation(3200)[:900], [-1, -7, 5000, 3199, 0], p.rng.integers(0, 40, 20)])
    b = p.batch([905, 20], at=at)
    attend_big(p, b, average=True)
    attend_big(p, b, block=1)


@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_many_products_do_not_see_what_they_do_not_see(what):
    p = Pool("llada", "bf16", 32, [3300], seed=7).fill()
    b = p.batch([1000])
    q, clean = attend_big(p, b, block=1)
    spot = [3299, 3100, 2700, 2450]
    at = B().PgBatch(p.ctx, ints([0, len(spot)]), ints([3300]), ints(p.pages[:1]), len(spot), at=ints(spot))
    t = torch.full((len(spot), p.Hkv * p.D), what, dtype=p.ctx.torch_dtype, device="cuda")
    good = [torch.empty_like(t) for _ in range(2)]
    p.ctx.d2c_pg_read(p.cache, at, *good)
    p.ctx.d2c_pg_append(p.cache, at, good[0], t)                  # V alone: the probabilities stay
    out = torch.zeros_like(clean)
    p.ctx.d2c_pg_attention(p.cache, b, q, out, block=1)
    seen = torch.tensor([2300 + r >= min(spot) for r in range(1000)], device="cuda")
    assert torch.equal(out[~seen], clean[~seen])
    if what != what:
        assert bool(out[seen].isnan().all())
    else:
        assert torch.equal(out[seen], torch.full_like(out[seen], what))
    p.ctx.d2c_pg_append(p.cache, at, t, good[1])                  # K alone
    p.ctx.d2c_pg_attention(p.cache, b, q, out, block=1)
    assert torch.equal(out[~seen], clean[~seen])


@pytest.mark.parametrize("geo,dtype,length,m", [("dream", "bf16", 70003, 40), ("dream", "f32", 70003, 140), ("llada", "f32", 3300, 2500)])
def test_many_products_meet_infinities_far_back(geo, dtype, length, m):
    """Some rows see an infinity of V, in a block of keys of which another page is not there; more blocks of keys than are told apart when it is looked for."""
    p = Pool(geo, dtype, 32, [length], seed=11).fill()
    spot = length - 15
    p.pages[0, spot // 32 - 1] = -1
    b = p.batch([m])
    q = torch.randn((m, p.H * p.D), device="cuda", generator=torch.Generator("cuda").manual_seed(5)).to(p.ctx.torch_dtype)
    clean = torch.zeros_like(q)
    p.ctx.d2c_pg_attention(p.cache, b, q, clean, block=1)
    at = B().PgBatch(p.ctx, ints([0, 1]), ints([length]), ints(p.pages[:1]), 1, at=ints([spot]))
    t = torch.zeros((1, p.Hkv * p.D), dtype=p.ctx.torch_dtype, device="cuda")
    keep = [torch.empty_like(t) for _ in range(2)]
    p.ctx.d2c_pg_read(p.cache, at, *keep)
    t[0, ::2], t[0, 1::2] = float("inf"), keep[1][0, 1::2]       # every other dimension
    p.ctx.d2c_pg_append(p.cache, at, keep[0], t)
    out = torch.zeros_like(q)
    p.ctx.d2c_pg_attention(p.cache, b, q, out, block=1)
    seen = torch.arange(length - m, length, device="cuda") >= spot
    assert torch.equal(out[~seen], clean[~seen]) and torch.equal(out[seen][:, 1::2], clean[seen][:, 1::2])
    assert bool((out[seen][:, ::2] == float("inf")).all()) and bool(clean.isfinite().all())


def test_many_products_repeat_to_the_bit_and_follow_their_lengths():
    p = Pool("dream", "bf16", 64, [5000, 700], seed=9).fill()
    b = p.batch([1000, 3])
    q, first = attend_big(p, b, block=1)
    out = torch.zeros_like(first)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.ctx.d2c_pg_attention(p.cache, b, q, out, block=1)
    for n in (5000, 3000, 1001, 5000):
        b.keep[1].copy_(ints([n, 700]))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.zero_()
        p.ctx.d2c_pg_attention(p.cache, b, q, out, block=1)
        assert torch.equal(got, out)
    assert torch.equal(out, first)


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("geo", ["gqa", "dream"])
def test_a_prompt_in_chunks_and_then_tokens(dtype, geo):
    """Two sequences fed chunk by chunk and then token by token: each row equals dense causal attention over rotated rows."""
    total = [150, 97]
    half = GEOS[geo][2] // 2
    p = Pool(geo, dtype, 32, total, rot=rotary([half // 4, half // 4, half // 2]))
    rows = [[(p.rng.standard_normal((n, h * p.D))) for h in (p.H, p.Hkv, p.Hkv)] for n in total]
    done = [0, 0]
    for counts in [(64, 32), (1, 33), (50, 0), (3, 30), (31, 1), (1, 1)]:
        for b in range(2):
            done[b] += counts[b]
        p.lengths = list(done)
        batch = p.batch(counts)
        q, k, v = (tensor(np.concatenate([rows[b][i][done[b] - counts[b]: done[b]] for b in range(2)]), dtype) for i in range(3))
        turned, out = torch.zeros_like(q), torch.zeros_like(q)
        p.ctx.d2c_pg_append(p.cache, batch, k, v, q=q, q_out=turned)
        p.ctx.d2c_pg_attention(p.cache, batch, turned, out, block=1)
        p.k, p.v = p.raw()
        p.expect(f64(turned).reshape(-1, p.H, p.D), out, None, 1, 0)
    assert done == total
    # and the stored keys are the rotated ones
    for b in range(2):
        k, _, _ = p.keys(b)
        plain = f64(tensor(rows[b][1], dtype)).reshape(-1, p.Hkv, p.D)
        pos = np.repeat(np.arange(total[b])[None], 3, 0)
        want = R.rotate(plain, pos, p.rot.freq, p.rot.axis, "halves")
        assert (np.abs(k - want) <= rotation_bound(plain, pos, p.rot.freq, p.rot.axis, dtype)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_selected_refresh_equals_the_contiguous_cache(dtype):
    """The d2Cache step's attention: selected rows refreshed, then attending to everything, with the head average; beside d2c_attention on a
    contiguous cache of the same rows."""
    from paper_2509_23094_amd import workloads as W
    wd = W.DIMS["C1"]
    L, m = 128, 37
    su_dims = W.ModelDims(wd.n_layers, wd.d_model, wd.n_heads, wd.n_kv_heads, wd.head_dim, wd.d_ffn, wd.vocab, dtype=dtype)
    dense = B().Context(su_dims, W.model_weights(su_dims, 0), L)
    p = Pool((wd.n_heads, wd.n_kv_heads, wd.head_dim), dtype, 32, [L]).fill()
    kc, vc = (torch.zeros((L, p.Hkv * p.D), dtype=p.ctx.torch_dtype, device="cuda") for _ in range(2))
    p.ctx.d2c_pg_read(p.cache, p.batch([L]), kc, vc)
    at = np.sort(p.rng.permutation(L)[:m])
    b = p.batch([m], at=at)
    q, (k, nk), (v, nv) = p.values(m, p.H), p.values(m, p.Hkv), p.values(m, p.Hkv)
    p.append(b, values=((k, nk), (v, nv)))
    p.k = p.raw()[0]
    out, avg = p.attend(b, q=q, average=True)
    want, want_avg = torch.zeros_like(out), torch.zeros((m, L), device="cuda")
    dense.d2c_attention(q[0], ints(at), m, k, v, kc, vc, L, want, want_avg)
    tol = 4 * HALF[dtype] if dtype == "bf16" else 1e-5
    assert (f64(out) - f64(want)).std() <= tol * f64(want).std() and np.abs(f64(avg) - f64(want_avg)).max() <= tol * f64(want_avg).max()


# ------------------------------------------------------------------ refusals

def test_refusals():
    Err = B().D2CError
    p = Pool("gqa", "bf16", 32, [100, 40], rot=rotary([32]), max_rows=50, max_batch=2).fill()
    b = p.batch([10, 10])
    q, out = p.values(20, p.H)[0], torch.zeros((20, 512), dtype=torch.bfloat16, device="cuda")
    k = p.values(20, p.Hkv)[0]
    ok = dict(block=1)
    p.ctx.d2c_pg_attention(p.cache, b, q, out, **ok)
    before = out.clone()
    for bad in (dict(block=-1), dict(window=-1), dict(block=(1 << 30) + 1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
                dict(scale=float("nan")), dict(attn_avg=torch.zeros((20, 0), device="cuda")), dict(attn_avg=torch.zeros((19, 100), device="cuda")),
                dict(attn_avg=torch.zeros((20, 200), device="cuda")[:, ::2])):
        with pytest.raises(Err):
            p.ctx.d2c_pg_attention(p.cache, b, q, out, **bad)
    for qq, oo in ((q[:19], out), (q.float(), out), (q, out.float()), (q, q), (q[:, :256], out), (q.t(), out), (q.cpu(), out), (q, out[:, ::2]),
                   (torch.zeros((20, 516), dtype=torch.bfloat16, device="cuda")[:, 4:], out),
                   (torch.zeros((20, 516), dtype=torch.bfloat16, device="cuda")[:, :512], out)):
        with pytest.raises(Err):
            p.ctx.d2c_pg_attention(p.cache, b, qq, oo, **ok)
    # an output inside the cache, or an average over the row starts
    with pytest.raises(Err, match="overlaps"):
        p.ctx.d2c_pg_attention(p.cache, b, q, p.cache.k.view(-1)[: 20 * 512].view(20, 512), **ok)
    with pytest.raises(Err, match="overlaps"):
        p.ctx.d2c_pg_read(p.cache, b, p.cache.v.view(-1)[: 20 * 128].view(20, 128), None)
    with pytest.raises(Err, match="overlaps"):
        p.ctx.d2c_pg_append(p.cache, b, p.cache.v.view(-1)[: 20 * 128].view(20, 128), k)
    with pytest.raises(Err):
        p.ctx.d2c_pg_append(p.cache, b, k, k.float())
    with pytest.raises(Err, match="go together"):
        p.ctx.d2c_pg_append(p.cache, b, k, k, q=q)
    with pytest.raises(Err):
        p.ctx.d2c_pg_append(p.cache, b, k, k, pos=ints(np.zeros((2, 20))))
    # sizes of the handle
    with pytest.raises(Err, match="max_rows"):
        big = p.batch([60, 1])
        p.ctx.d2c_pg_attention(p.cache, big, p.values(61, p.H)[0], torch.zeros((61, 512), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(Err, match="max_batch"):
        three = B().PgBatch(p.ctx, ints([0, 1, 2, 3]), ints([1, 1, 1]), ints(np.zeros((3, 1))), 3)
        p.ctx.d2c_pg_append(p.cache, three, k[:3], k[:3])
    with pytest.raises(Err):
        B().PgBatch(p.ctx, ints([0, 1]), ints([1, 1]), ints(np.zeros((2, 1))), 1)
    with pytest.raises(Err):
        B().PgBatch(p.ctx, torch.tensor([0, 1], device="cuda"), ints([1]), ints([[0]]), 1)
    # another geometry's cache, a handle without a rotation, half a head
    other = B().PgContext(8, 2, 64, "bf16", page_rows=64, max_rows=50, max_batch=2)
    with pytest.raises(Err, match="made for"):
        other.d2c_pg_attention(p.cache, b, q, out)
    with pytest.raises(Err, match="without a rotation"):
        other.d2c_pg_rotate(q, ints(np.zeros((1, 20))), out)
    with pytest.raises(Err, match="whole heads"):
        p.ctx.d2c_pg_rotate(q[:, :96], ints(np.zeros((1, 20))), out[:, :96])
    torch.cuda.synchronize()
    assert torch.equal(out, before)


def test_nothing_to_do():
    p = Pool("gqa", "bf16", 32, [100], max_batch=2).fill()
    none = B().PgBatch(p.ctx, ints([0]), ints([]), torch.zeros((0, 4), dtype=torch.int32, device="cuda"), 5)
    t = torch.full((5, 512), 7.0, dtype=torch.bfloat16, device="cuda")
    p.ctx.d2c_pg_attention(p.cache, none, torch.zeros_like(t), t)
    p.ctx.d2c_pg_append(p.cache, none, t[:, :128].contiguous(), t[:, :128].contiguous())
    empty = B().PgBatch(p.ctx, ints([0, 0]), ints([100]), ints(p.pages), 0)
    e = torch.zeros((0, 512), dtype=torch.bfloat16, device="cuda")
    p.ctx.d2c_pg_attention(p.cache, empty, e, e.clone())
    # sequences without a single page
    bare = B().PgBatch(p.ctx, ints([0, 2, 5]), ints([4, 0]), torch.zeros((2, 0), dtype=torch.int32, device="cuda"), 5)
    p.ctx.d2c_pg_attention(p.cache, bare, torch.ones_like(t), t, block=1)
    torch.cuda.synchronize()
    assert not t.any()
    p.check()


def test_row_starts_that_are_no_row_starts_harm_nothing_else():
    """Starts outside the rows or not ascending: outputs and caches are undefined, memory beside them is not touched."""
    p = Pool("gqa", "bf16", 32, [100, 60, 33], spare=0).fill()
    guard = torch.full((3 * 20, 512), 7.0, dtype=torch.bfloat16, device="cuda")
    q, k = p.values(20, p.H)[0], p.values(20, p.Hkv)[0]
    for starts in ([0, 20, 0, 20], [-5, 7, 9, 4000], [1 << 30, 5, -(1 << 31), (1 << 31) - 1], [0, 500, 500, 20]):
        b = B().PgBatch(p.ctx, ints(starts), ints([100, 60, 33]), ints(p.pages), 20)
        p.ctx.d2c_pg_attention(p.cache, b, q, guard[20:40], block=1)
        p.ctx.d2c_pg_append(p.cache, b, k, k, q=q, q_out=guard[20:40])
        torch.cuda.synchronize()
        assert (guard[:20] == 7).all() and (guard[40:] == 7).all()


def split_pool(counts, seed=0):
    """Three sequences whose caches are long enough that their tiles are split and joined, with a valid batch of `counts` rows."""
    p = Pool("gqa", "bf16", 32, [2000, 1900, 1801], seed=seed).fill()
    batch = p.batch(counts)
    return p, batch, p.values(sum(counts), p.H)[0]


@pytest.mark.parametrize("starts", [[0, 20, 25, 30], [0, 1, 30, 31], [20, 21, 22, 23], [-9, -5, -1, 20], [30, 40, 50, 60], [-5, -4, -3, -2], [0, 20, 20, 20]])
def test_nothing_is_joined_from_the_call_before(starts):
    """A call whose sequences are empty once their starts are taken into the batch, behind one of more rows that was split: nothing of the earlier
    call's splits is joined into this one's output, or behind it."""
    say("records, starts %s" % starts)
    p, whole, q = split_pool([40, 40, 40])
    want = torch.empty_like(q)
    p.ctx.d2c_pg_attention(p.cache, whole, q, want, block=1)
    guard = torch.full((400, 512), 7.0, dtype=torch.bfloat16, device="cuda")
    bad = B().PgBatch(p.ctx, ints(starts), ints(p.lengths), ints(p.pages), 20)
    p.ctx.d2c_pg_attention(p.cache, bad, q[:20], guard[200:220], block=1)
    torch.cuda.synchronize()
    assert (guard[:200] == 7).all() and (guard[220:] == 7).all()
    again = torch.empty_like(want)
    p.ctx.d2c_pg_attention(p.cache, whole, q, again, block=1)
    assert torch.equal(again, want)


@pytest.mark.parametrize("starts", [[40, -(1 << 31), 5, 20], [0, 20, -(1 << 31), (1 << 31) - 1], [(1 << 31) - 1, -(1 << 31), (1 << 31) - 1, 0], [19, -(1 << 31), 18, 20],
                                    [5, 20, 3, 20], [20, 0, 20, 0]])
def test_extreme_row_starts_stay_within_the_rows(starts):
    """Starts whose differences leave 32 bits, with the head average, on caches that are split: only the call's own rows are written."""
    say("extreme starts %s" % starts)
    p, whole, q = split_pool([40, 40, 40], seed=1)
    want, mean = torch.empty_like(q), torch.full((120, 2000), 7.0, device="cuda")
    p.ctx.d2c_pg_attention(p.cache, whole, q, want, block=1, attn_avg=mean)
    guard, beside = torch.full((400, 512), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((400, 2000), 7.0, device="cuda")
    bad = B().PgBatch(p.ctx, ints(starts), ints(p.lengths), ints(p.pages), 20)
    p.ctx.d2c_pg_attention(p.cache, bad, q[:20], guard[200:220], block=1, attn_avg=beside[200:220])
    torch.cuda.synchronize()
    for g in (guard, beside):
        assert (g[:200] == 7).all() and (g[220:] == 7).all()
    again, once = torch.empty_like(want), torch.full_like(mean, 7.0)
    p.ctx.d2c_pg_attention(p.cache, whole, q, again, block=1, attn_avg=once)
    assert torch.equal(again, want) and torch.equal(once, mean)


def test_a_million_tiles():
    """2^20 rows of 32 heads on one: as many tiles as fill whole rounds of workgroups, more than fp32 counts one by one.  Every row sees itself alone,
    those before the cache nothing."""
    n = 1 << 20
    say("%d rows" % n)
    p = Pool((32, 1, 64), "bf16", 32, [512], max_rows=n).fill()
    b = B().PgBatch(p.ctx, ints([0, n]), ints([512]), ints(p.pages), n)
    q, out = torch.ones((n, 2048), dtype=torch.bfloat16, device="cuda"), torch.full((n, 2048), 7.0, dtype=torch.bfloat16, device="cuda")
    p.ctx.d2c_pg_attention(p.cache, b, q, out, block=1, window=1)
    assert torch.equal(out[n - 512:].view(512, 32, 64), tensor(p.keys(0)[1], "bf16").expand(512, 32, 64))
    rest = out[:n - 512].view(torch.int32)
    assert not rest.any(), rest.any(1).nonzero()[:4].tolist()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1e-44, 2.0 ** -126, 2.0 ** 127])
def test_scales_at_the_ends_of_their_range(dtype, scale):
    """Scores of 0 times any scale, behind a mask: every row is the mean of the keys it sees (queries of zeros; a scale that 32 bits hold only as a
    subnormal, and the largest)."""
    p = Pool("gqa", dtype, 32, [70, 33], max_rows=64).fill()
    b = p.batch([40, 3])
    q = (tensor(np.zeros((43, 512)), dtype), np.zeros((43, 8, 64)))
    p.attend(b, block=1, scale=scale, average=True, q=q)
    p.attend(b, block=32, window=40, scale=scale, q=q)


@pytest.mark.parametrize("scale", [2.0 ** 127 * (1 + 2.0 ** -23), 3e38, float("inf")])
def test_scales_above_their_range_are_refused(scale):
    """From there on the product with log2(e) is no number of 32 bits (0 times infinity would be NaN)."""
    p = Pool("gqa", "bf16", 32, [70], max_rows=64).fill()
    b, t = p.batch([3]), torch.full((3, 512), 7.0, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B().D2CError, match="scale"):
        p.ctx.d2c_pg_attention(p.cache, b, torch.zeros_like(t), t, scale=scale)
    torch.cuda.synchronize()
    assert (t == 7).all()
