"""The 8-bit operators on the GPU, through the C ABI, against the plain 64-bit forms of q8_reference: codes, scales, sums, weights and kept
sets bit for bit, attention within bounds that count its roundings."""
import numpy as np
import pytest
import torch

import q8_reference as R
from gpu_util import say

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}          # rounding to T
P_HALF = {"bf16": 2.0 ** -12, "f32": 2.0 ** -22}       # rounding of a probability: fp16 (11 bits), two pieces of it
GEOS = {"mha": (4, 4, 64), "gqa": (8, 2, 64), "dream": (28, 4, 128), "odd": (5, 1, 128), "llada": (32, 32, 128)}


def B():
    from paper_2509_23094_amd import binding
    return binding


def dev(a, dtype):
    t = torch.from_numpy(np.ascontiguousarray(a, np.float32))
    return t.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda().contiguous()


def f64(t):
    return t.detach().double().cpu().numpy()


def rows(rng, m, heads, dim, loud=0.3):
    return rng.standard_normal((m, heads, dim)) * np.exp(loud * rng.standard_normal((m, 1, 1)))


class Case:
    """A handle, a cache with garbage where nothing is written, and the plain cache beside it."""

    def __init__(self, geo, dtype, L, seed=0, max_rows=256, max_batch=1, capacity=None, ctx=None):
        self.H, self.Hkv, self.D = GEOS[geo] if isinstance(geo, str) else geo
        self.dtype, self.L, self.rng = dtype, L, np.random.default_rng([seed, L])
        cap = capacity or L
        self.ctx = ctx or B().Q8Context(self.H, self.Hkv, self.D, dtype, max_seq=max(cap, L), max_rows=max_rows, max_batch=max_batch)
        self.cache = B().Q8Cache(self.ctx, cap)
        for t in (self.cache.k_codes, self.cache.v_codes):
            t.copy_(torch.randint(0, 256, t.shape, dtype=torch.uint8))
        self.ref = R.Cache8(cap, self.Hkv, self.D)

    def new(self, m, factor=1.0):
        """(device tensor, its values) of m rows of K or V."""
        t = dev(rows(self.rng, m, self.Hkv, self.D) * factor, self.dtype).reshape(m, self.Hkv * self.D)
        return t, f64(t).reshape(m, self.Hkv, self.D)

    def update(self, idx, m=None, L=None, factor=1.0, new=None):
        L = self.L if L is None else L
        m = len(idx) if idx is not None else m
        (dk, nk), (dv, nv) = new or (self.new(m, factor), self.new(m, factor))
        di = None if idx is None else torch.tensor(np.asarray(idx), dtype=torch.int32, device="cuda")
        self.ctx.d2c_q8_update([B().Q8Seq(self.cache, L, m, idx=di, new_k=dk, new_v=dv)])
        self.ref.update(np.arange(L - m, L) if idx is None else idx, nk, nv, L)
        torch.cuda.synchronize()

    def fill(self):
        self.update(None, m=self.L)
        return self

    def check(self, L=None):
        """Codes of the first L rows and scales, bit for bit."""
        L = self.L if L is None else L
        nb = -(-L // 64)
        for name, t in (("k", self.ref.k), ("v", self.ref.v)):
            got_s = getattr(self.cache, name + "_scale").cpu().numpy().astype(np.float64)[:nb]
            assert np.array_equal(got_s, t.scale[:nb]), name + " scales"
            raw = getattr(self.cache, name + "_codes").cpu().numpy()
            c = raw.reshape(-1, self.Hkv, self.D // 16, 64, 16).transpose(0, 3, 1, 2, 4) if name == "k" else \
                raw.reshape(-1, self.Hkv, 16, self.D, 4).transpose(0, 2, 4, 1, 3)
            c = c.reshape(-1, self.Hkv, self.D).astype(np.int64) - 128
            assert np.array_equal(c[:L], t.codes[:L]), name + " codes"

    def queries(self, m, factor=1.0):
        return dev(self.rng.standard_normal((m, self.H * self.D)) * factor, self.dtype)

    def expect(self, q, out, avg, L=None):
        L = self.L if L is None else L
        check_attention(q, self.ref.k.values(L), self.ref.v.values(L), out, avg, self)


def check_attention(q, k, v, out, avg, c):
    m = q.shape[0]
    o, a, mag, share = R.attention(f64(q).reshape(m, c.H, c.D), k, v)
    if out is not None:
        # each term's share twice (numerator and denominator), its rounding, D / 64 blocks of fp32 sums, the result's rounding
        n = k.shape[0]
        # a probability is rounded to fp16 times 2^11, relative to a reference that is at most the row's largest.  Where that is a subnormal
        # number (below 2^-14) its rounding is at most half of 2^-24: 2^-25 / 2^11 = 2^-36 of the largest, which is at most the row's sum
        below = 2.0 ** -36 * np.repeat(np.abs(v).sum(0), c.H // c.Hkv, 0)[None]
        tol = HALF[c.dtype] * np.abs(o) + (1 + HALF[c.dtype]) * (mag * (2 * share + P_HALF[c.dtype] + (n ** 0.5 + 70) * 2.0 ** -24) + below) + 1e-30
        err = np.abs(f64(out).reshape(m, c.H, c.D) - o)
        assert (err <= tol).all(), "out: %g times the bound" % (err / tol).max()
    if avg is not None:
        tol = a * (2 * share + (k.shape[0] ** 0.5 + c.H + 16) * 2.0 ** -24) + 1e-30
        err = np.abs(f64(avg) - a)
        assert (err <= tol).all(), "average: %g times the bound" % (err / tol).max()


# ---------------------------------------------------------------------- update and read

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("geo", ["mha", "dream"])
@pytest.mark.parametrize("L", [1, 3, 63, 64, 65, 200, 1000])
def test_fill_and_refresh(geo, dtype, L):
    say(f"q8 update {geo} {dtype} L={L}")
    c = Case(geo, dtype, L).fill()
    c.check()
    for m, factor in ((1, 1.0), (min(L, 3), 2.5), (min(L, 20), 0.1), ((L + 1) // 2, 1.5), (L, 0.7)):
        idx = np.sort(c.rng.permutation(L)[:m])
        c.update(idx, factor=factor)
        c.check()


@pytest.mark.parametrize("L", [4099, 20000])
def test_refresh_of_long_caches(L):
    """Few scattered rows (a workgroup per row) and more rows than blocks (a workgroup per block, its rows searched)."""
    say(f"q8 update long {L}")
    c = Case((2, 1, 64), "bf16", L).fill()
    for m in (5, L // 64, L // 64 + 1, 700, L - 1):
        c.update(np.sort(c.rng.permutation(L)[:m]), factor=1.3)
        c.check()
    c.update(np.arange(64 * 10, 64 * 20), factor=0.2)       # whole blocks among the others
    c.check()


def test_append_row_by_row():
    """A cache that grows: the first row of a block sets its scale, whatever lay there."""
    say("q8 append")
    c = Case("gqa", "bf16", 130, capacity=200)
    c.cache.k_scale.fill_(float("nan"))
    c.cache.v_scale.fill_(1e30)
    c.update(None, m=61, L=61)
    for L in range(62, 131):
        c.update(None, m=1, L=L, factor=1.0 + 0.01 * L)
    c.check(130)


def test_borders_and_values_that_are_not_finite():
    say("q8 borders")
    c = Case("mha", "f32", 128)
    s = float(np.float32(127.0 * 0.75) / np.float32(127))
    x = np.zeros((64, c.Hkv, c.D))
    x[0, :, 0] = 127 * 0.75
    x[1:] = (c.rng.integers(-127, 127, size=(63, c.Hkv, c.D)) + 0.5) * s                       # exactly between two codes
    x[2:4] = np.nextafter(x[2:4].astype(np.float32), np.float32(0))                             # and just beside
    x[4:6] = np.nextafter(x[4:6].astype(np.float32), np.float32(1e9))
    x = x.astype(np.float32)
    d = dev(x, "f32").reshape(64, -1)
    c.update(np.arange(64), new=((d, f64(d).reshape(x.shape)), (d, f64(d).reshape(x.shape))))
    c.check(64)
    y = np.zeros((64, c.Hkv, c.D), np.float32)
    y[3, 0, 5], y[4, 1, 6], y[5, 2, 7], y[6] = np.nan, np.inf, -np.inf, 0.25
    y[7, 3] = 1e-38                                                                             # far below the others
    d = dev(y, "f32").reshape(64, -1)
    c.update(np.arange(64, 128), new=((d, f64(d).reshape(y.shape)), (d, f64(d).reshape(y.shape))))
    c.check(128)
    tiny = np.full((64, c.Hkv, c.D), 1e-36, np.float32)                                         # below 2^-100: zeros, scale 0
    d = dev(tiny, "f32").reshape(64, -1)
    c.update(np.arange(64), new=((d, f64(d).reshape(y.shape)), (d, f64(d).reshape(y.shape))))
    assert (c.cache.k_scale[0] == 0).all()
    c.update([9], factor=1.0)                                                                   # and a row beside them
    c.check(128)
    big = np.full((1, c.Hkv, c.D), 3e38, np.float32)
    d = dev(big, "f32").reshape(1, -1)
    c.update([10], new=((d, f64(d).reshape(big.shape)), (d, f64(d).reshape(big.shape))))
    c.check(128)


@pytest.mark.parametrize("L", [100, 1000])
def test_indices_outside_are_left_out(L):
    say(f"q8 indices outside L={L}")
    c = Case("mha", "bf16", L, capacity=L + 28).fill()
    c.update([-70, -1, 5, 64, L, L + 27, 1 << 30])                                               # L = 1000: fewer than blocks
    c.check()
    c.update(np.r_[[-9], np.arange(0, L, 3), [L, 5000]])                                         # the searched form
    c.check()


@pytest.mark.parametrize("idx", ["all", "one before", "one behind", "gap"])
def test_as_many_indices_as_rows(idx):
    """More than a thousand indices, as many as there are rows: each in its place, or some left out and the others shifted."""
    say(f"q8 as many indices as rows, {idx}")
    L = 1300
    c = Case("gqa", "bf16", L, capacity=L + 28).fill()
    at = np.arange(L)
    c.update({"all": at, "one before": at - 1, "one behind": at + 1, "gap": np.r_[at[:700], at[701:], [L + 3]]}[idx])
    c.check()


def test_batch_of_updates():
    say("q8 batch of 11 updates")
    first = Case("gqa", "bf16", 700, max_batch=11)
    cs = [first] + [Case("gqa", "bf16", 100 + 50 * i, seed=i, ctx=first.ctx) for i in range(10)]
    seqs = []
    for i, c in enumerate(cs):
        c.fill()
        m = 0 if i == 4 else 1 + 9 * i
        (dk, nk), (dv, nv) = c.new(m, 1.5), c.new(m, 1.5)
        idx = np.sort(c.rng.permutation(c.L)[:m])
        seqs.append(B().Q8Seq(c.cache, c.L, m, idx=torch.tensor(idx, dtype=torch.int32, device="cuda"), new_k=dk, new_v=dv))
        c.ref.update(idx, nk, nv, c.L)
    first.ctx.d2c_q8_update(seqs)
    torch.cuda.synchronize()
    for c in cs:
        c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("geo", ["mha", "dream"])
def test_read(geo, dtype):
    say(f"q8 read {geo} {dtype}")
    c = Case(geo, dtype, 201).fill()
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    for idx in (None, [0], [200, 3, 3, 64, 63], [-1, 5, 201, 1 << 30], list(range(0, 201, 7))):
        n = 201 if idx is None else len(idx)
        k, v = (torch.full((n, c.Hkv * c.D), 7.0, dtype=t, device="cuda") for _ in range(2))
        c.ctx.d2c_q8_read(c.cache, 201, None if idx is None else torch.tensor(idx, dtype=torch.int32, device="cuda"), k, v)
        at = np.arange(n) if idx is None else np.asarray(idx)
        ok = (at >= 0) & (at < 201)
        for got, ref in ((k, c.ref.k), (v, c.ref.v)):
            want = np.where(ok[:, None], ref.values().astype(np.float32)[np.where(ok, at, 0)].reshape(n, -1), 0.0)
            assert torch.equal(got.cpu(), torch.from_numpy(want.astype(np.float32)).to(t))
    only = torch.zeros((3, c.Hkv * c.D), dtype=t, device="cuda")
    c.ctx.d2c_q8_read(c.cache, 201, None, None, only)
    assert torch.equal(only.cpu(), torch.from_numpy(c.ref.v.values(3).astype(np.float32).reshape(3, -1)).to(t))


# ---------------------------------------------------------------------- attention

def attend(c, m, L=None, avg=True, q=None, batch=None):
    L = c.L if L is None else L
    q = c.queries(m) if q is None else q
    out = torch.full_like(q, 9.0)
    a = torch.full((m, L), 9.0, device="cuda") if avg else None
    c.ctx.d2c_q8_attention([B().Q8Seq(c.cache, L, m, q=q, out=out, attn_avg=a)])
    torch.cuda.synchronize()
    return q, out, a


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("geo", list(GEOS))
@pytest.mark.parametrize("m,L", [(1, 1), (1, 2), (3, 63), (2, 64), (33, 65), (32, 128), (1, 257), (31, 500), (130, 320), (64, 1030)])
def test_attention(geo, dtype, m, L):
    say(f"q8 attention {geo} {dtype} m={m} L={L}")
    c = Case(geo, dtype, L).fill()
    q, out, avg = attend(c, m)
    c.expect(q, out, avg)
    _, again, _ = attend(c, m, avg=False, q=q)
    assert torch.equal(again, out)                      # the average changes nothing, and the same call gives the same bits


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("geo,m,L", [("dream", 1, 70001), ("odd", 7, 33333), ("llada", 2, 9000), ("mha", 256, 4100)])
def test_attention_long(geo, dtype, m, L):
    say(f"q8 attention long {geo} {dtype} m={m} L={L}")
    c = Case(geo, dtype, L)
    c.update(None, m=L)
    q, out, avg = attend(c, m, avg=m < 100)
    c.expect(q, out, avg)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_refreshes_first_and_a_shorter_length_reads_less(dtype):
    say(f"q8 attention with update {dtype}")
    c = Case("gqa", dtype, 300).fill()
    idx = np.sort(c.rng.permutation(300)[:40])
    (dk, nk), (dv, nv) = c.new(40, 2.0), c.new(40, 2.0)
    q = c.queries(40)
    out, avg = torch.zeros_like(q), torch.zeros((40, 300), device="cuda")
    c.ctx.d2c_q8_attention([B().Q8Seq(c.cache, 300, 40, idx=torch.tensor(idx, dtype=torch.int32, device="cuda"), new_k=dk, new_v=dv, q=q,
                                      out=out, attn_avg=avg)])
    c.ref.update(idx, nk, nv, 300)
    c.check()
    c.expect(q, out, avg)
    q, out, avg = attend(c, 5, L=130)
    c.expect(q, out, avg, L=130)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_batch(dtype):
    """Eleven sequences of different sizes in one call, one of them empty, some without the average."""
    say(f"q8 attention batch {dtype}")
    first = Case("gqa", dtype, 900, max_batch=11, max_rows=600)
    cs = [first] + [Case("gqa", dtype, 1 + 97 * i, seed=i, ctx=first.ctx) for i in range(10)]
    seqs, got = [], []
    for i, c in enumerate(cs):
        c.fill()
        m = 0 if i == 4 else 1 + 11 * i
        q = c.queries(m)
        out, avg = torch.zeros_like(q), torch.zeros((m, c.L), device="cuda") if i % 3 else None
        seqs.append(B().Q8Seq(c.cache, c.L, m, q=q, out=out, attn_avg=avg))
        got.append((q, out, avg))
    first.ctx.d2c_q8_attention(seqs)
    torch.cuda.synchronize()
    for i, (c, (q, out, avg)) in enumerate(zip(cs, got)):
        if i != 4:
            c.expect(q, out, avg)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_of_extreme_sizes(dtype):
    """Loud and silent blocks, one key that takes all, queries far from 1, zeros: nothing overflows and nothing is lost."""
    say(f"q8 attention extremes {dtype}")
    c = Case("mha", dtype, 400).fill()
    c.update(np.arange(64), factor=1e-6)
    c.update(np.arange(64, 128), factor=0.0)
    c.update(np.arange(192, 256), factor=20.0)
    c.check()
    for factor in (1e-30, 1e-3, 1.0, 30.0):
        q = c.queries(19, factor)
        q[3] = 0
        q, out, avg = attend(c, 19, q=q)
        c.expect(q, out, avg)
    q = c.queries(5)
    q[1, 7], q[2, 70], q[3, 200] = float("nan"), float("inf"), -float("inf")
    _, out, avg = attend(c, 5, q=q)
    assert torch.isnan(out[1, : c.D]).all() and torch.isnan(avg[1:4]).all()
    assert torch.isfinite(out[1, c.D:]).all()                                           # the other heads' columns
    c.expect(q[[0, 4]].contiguous(), out[[0, 4]], avg[[0, 4]])


def test_attention_of_a_flat_row_over_a_long_cache():
    """Equal scores: each of 50000 probabilities is 2e-5 of the sum; none may be lost in its rounding."""
    say("q8 attention flat")
    c = Case((2, 1, 64), "bf16", 50000)
    c.update(None, m=50000)
    q = c.queries(3)
    q[0] = 0
    q[1] *= 1e-4
    q, out, avg = attend(c, 3, q=q)
    c.expect(q, out, avg)


# ---------------------------------------------------------------------- linear

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,N,K", [(1, 1, 8), (16, 6144, 2048), (13, 6145, 64), (17, 80, 2048), (1, 16, 64), (2, 17, 72), (15, 33, 256), (16, 768, 1000), (17, 100, 320), (33, 250, 2048),
                                   (64, 64, 4096), (65, 129, 136), (100, 1000, 512), (130, 72, 8192), (200, 300, 640), (257, 513, 576),
                                   (520, 520, 264)])
def test_linear(dtype, m, N, K):
    say(f"q8 linear {dtype} m={m} N={N} K={K}")
    rng = np.random.default_rng([m, N, K])
    a, w = dev(rng.standard_normal((m, K)), dtype), dev(0.02 * rng.standard_normal((N, K)) * np.exp(rng.standard_normal((N, 1))), dtype)
    if m > 3:
        a[1] = 0
        a[2] = 0
        a[2, K // 2] = -5
    ctx = B().Q8Context(4, 4, 64, dtype, max_rows=m, max_k=K, max_n=N)
    p = ctx.d2c_q8_pack(w)
    guard = torch.full((m + 2, N), 123.0, device="cuda")
    out = torch.full((m, N), 9.0, device="cuda")
    ctx.d2c_q8_linear(a, p, out)
    want, _, sw = R.linear(f64(a), f64(w))
    assert np.array_equal(p.scale.cpu().numpy(), sw)
    assert np.array_equal(out.cpu().numpy(), want)
    flat = guard.view(-1)[: m * N].view(m, N)                          # nothing behind the last row or column is written
    ctx.d2c_q8_linear(a, p, flat)
    assert torch.equal(flat, out) and (guard.view(-1)[m * N:] == 123.0).all()


def test_linear_float_rows_of_four_more():
    say("q8 linear f32 K % 8 == 4")
    for m, N, K in ((5, 40, 4), (3, 20, 12), (70, 90, 1028)):
        rng = np.random.default_rng([m, N, K])
        a, w = dev(rng.standard_normal((m, K)), "f32"), dev(rng.standard_normal((N, K)), "f32")
        ctx = B().Q8Context(4, 4, 64, "f32", max_rows=m, max_k=K, max_n=N)
        out = torch.zeros((m, N), device="cuda")
        ctx.d2c_q8_linear(a, ctx.d2c_q8_pack(w), out)
        assert np.array_equal(out.cpu().numpy(), R.linear(f64(a), f64(w))[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [5, 70, 300])
def test_linear_rows_and_channels_that_are_not_finite(dtype, m):
    say(f"q8 linear not finite {dtype} m={m}")
    rng = np.random.default_rng(m)
    N, K = 150, 512
    a, w = dev(rng.standard_normal((m, K)), dtype), dev(rng.standard_normal((N, K)), dtype)
    a[1, 3], a[3, 511], w[7, 0], w[149, 77] = float("nan"), -float("inf"), float("inf"), float("nan")
    ctx = B().Q8Context(4, 4, 64, dtype, max_rows=m, max_k=K, max_n=N)
    out = torch.zeros((m, N), device="cuda")
    ctx.d2c_q8_linear(a, ctx.d2c_q8_pack(w), out)
    assert np.array_equal(out.cpu().numpy(), R.linear(f64(a), f64(w))[0], equal_nan=True)
    assert int(torch.isnan(out).sum()) == 2 * N + 2 * (m - 2)


def test_linear_near_the_largest_sum():
    """All products 127 * 127 over the longest contraction: 1.06e9 still fits the 32-bit sum."""
    say("q8 linear largest sum")
    ctx = B().Q8Context(4, 4, 64, "bf16", max_rows=20, max_k=1 << 16, max_n=48)
    a, w = (torch.ones((r, 1 << 16), dtype=torch.bfloat16, device="cuda") for r in (20, 48))
    w[5] = -1
    out = torch.zeros((20, 48), device="cuda")
    ctx.d2c_q8_linear(a, ctx.d2c_q8_pack(w), out)
    assert np.array_equal(out.cpu().numpy(), R.linear(f64(a), f64(w))[0])


# ---------------------------------------------------------------------- weigh and evict

@pytest.mark.parametrize("m,L", [(1, 1), (3, 63), (17, 64), (64, 65), (130, 1000), (300, 5000), (2, 70000)])
def test_weigh(m, L):
    say(f"q8 weigh m={m} L={L}")
    rng = np.random.default_rng([m, L])
    avg = rng.random((m, L), dtype=np.float32) ** 8
    avg[0, 0] = 1.0
    w = rng.integers(0, 1 << 40, size=L)
    if L > 10:
        avg[0, 1:7] = [np.nan, np.inf, -np.inf, -1.0, 2.0, 1e-12]
    d = torch.from_numpy(w.copy()).cuda()
    ctx = B().Q8Context(4, 4, 64, "f32")
    ctx.d2c_q8_weigh(torch.from_numpy(avg).cuda(), d)
    assert np.array_equal(d.cpu().numpy(), R.weigh(avg, w))


def weights(rng, L, kind):
    if kind == "spread":
        return (np.exp(2 * rng.standard_normal(L)) * 2 ** 30).astype(np.int64)
    if kind == "ties":
        return rng.integers(0, 4, size=L) * (1 << 33)
    if kind == "equal":
        return np.full(L, 12345)
    if kind == "wide":
        return rng.integers(0, (1 << 63) - 1, size=L) >> rng.integers(0, 63, size=L)
    w = rng.integers(-5, 3, size=L)                     # zeros and negative ones
    return w


@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "wide", "negative"])
@pytest.mark.parametrize("L", [1, 2, 64, 65, 1000, 5000, 20481, 140000])
def test_evict(kind, L):
    say(f"q8 evict {kind} L={L}")
    geo = (1, 1, 64) if L > 10000 else "gqa"
    c = Case(geo, "bf16", L).fill()
    w = weights(c.rng, L, kind)
    protect = (c.rng.random(L) < 0.2).astype(np.uint8) * 3
    dw = torch.from_numpy(w).cuda()
    for n, p in ((1, None), (L, None), ((L + 1) // 2, None), ((L + 1) // 2, protect), (max(1, L // 10), protect), (max(1, int((protect > 0).sum())), protect)):
        dst = B().Q8Cache(c.ctx, n)
        kept = torch.full((n,), -1, dtype=torch.int32, device="cuda")
        kw = torch.full((n,), -1, dtype=torch.int64, device="cuda")
        c.ctx.d2c_q8_evict(c.cache, L, dw, None if p is None else torch.from_numpy(p).cuda(), dst, kept, kw)
        want = R.keep(w, p, n)
        assert np.array_equal(kept.cpu().numpy(), want), f"n={n}"
        assert np.array_equal(kw.cpu().numpy(), np.maximum(w[want], 0))
        o = Case.__new__(Case)
        o.__dict__.update(c.__dict__)
        o.cache, o.ref, o.L = dst, c.ref.evict(want), n
        o.check()


# ---------------------------------------------------------------------- together

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_few_steps_together(dtype):
    """Projection of selected rows -> refresh + attention -> weights -> eviction -> the next step on the smaller cache."""
    say(f"q8 together {dtype}")
    d, m, L = 256, 21, 333
    c = Case("gqa", dtype, L, max_rows=64)
    lin = B().Q8Context(c.H, c.Hkv, c.D, dtype, max_rows=64, max_k=d, max_n=c.H * c.D + 2 * c.Hkv * c.D)
    w = dev(0.06 * c.rng.standard_normal((lin.d_q + 2 * lin.d_kv, d)), dtype)
    pack = lin.d2c_q8_pack(w)
    c.fill()
    weight = torch.zeros(L, dtype=torch.int64, device="cuda")
    ref_w, t = np.zeros(L, np.int64), torch.bfloat16 if dtype == "bf16" else torch.float32
    for step in range(4):
        h = dev(c.rng.standard_normal((m, d)), dtype)
        qkv = torch.zeros((m, lin.d_q + 2 * lin.d_kv), device="cuda")
        lin.d2c_q8_linear(h, pack, qkv)
        assert np.array_equal(qkv.cpu().numpy(), R.linear(f64(h), f64(w))[0])
        q, k, v = (x.to(t).contiguous() for x in qkv.split([lin.d_q, lin.d_kv, lin.d_kv], 1))
        idx = np.sort(c.rng.permutation(c.L)[:m])
        out, avg = torch.zeros_like(q), torch.zeros((m, c.L), device="cuda")
        c.ctx.d2c_q8_attention([B().Q8Seq(c.cache, c.L, m, idx=torch.tensor(idx, dtype=torch.int32, device="cuda"), new_k=k, new_v=v, q=q,
                                          out=out, attn_avg=avg)])
        c.ref.update(idx, f64(k).reshape(m, c.Hkv, c.D), f64(v).reshape(m, c.Hkv, c.D), c.L)
        c.check()
        c.expect(q, out, avg)
        c.ctx.d2c_q8_weigh(avg, weight)
        ref_w = R.weigh(f64(avg), ref_w)
        assert np.array_equal(weight.cpu().numpy(), ref_w)
        n = c.L - 40 if step % 2 else c.L
        if n < c.L:
            dst, kept = B().Q8Cache(c.ctx, n), torch.zeros(n, dtype=torch.int32, device="cuda")
            kw = torch.zeros(n, dtype=torch.int64, device="cuda")
            c.ctx.d2c_q8_evict(c.cache, c.L, weight, None, dst, kept, kw)
            want = R.keep(ref_w, None, n)
            assert np.array_equal(kept.cpu().numpy(), want)
            c.cache, c.ref, c.L, weight, ref_w = dst, c.ref.evict(want), n, kw, ref_w[want]
            c.check()


def test_captured_and_replayed_on_another_stream():
    """One graph of all calls, replayed with eager work in between, against eager results."""
    say("q8 graph")
    L, m, n, dtype = 500, 30, 300, "bf16"
    c = Case("gqa", dtype, L, max_rows=64).fill()
    lin = B().Q8Context(8, 2, 64, dtype, max_rows=300, max_k=512, max_n=256)
    w, a = dev(c.rng.standard_normal((256, 512)), dtype), dev(c.rng.standard_normal((300, 512)), dtype)
    pack, y = lin.d2c_q8_pack(w), torch.zeros((300, 256), device="cuda")
    idx = torch.tensor(np.sort(c.rng.permutation(L)[:m]), dtype=torch.int32, device="cuda")
    (dk, _), (dv, _) = c.new(m), c.new(m)
    q = c.queries(m)
    out, avg = torch.zeros_like(q), torch.zeros((m, L), device="cuda")
    weight, kept, kw = torch.zeros(L, dtype=torch.int64, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int64, device="cuda")
    dst = B().Q8Cache(c.ctx, n)
    rk, rv = (torch.zeros((n, c.ctx.d_kv), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    batch = B().Q8Batch(c.ctx, [B().Q8Seq(c.cache, L, m, idx=idx, new_k=dk, new_v=dv, q=q, out=out, attn_avg=avg)])

    def step():
        lin.d2c_q8_linear(a, pack, y)
        c.ctx.d2c_q8_attention(batch)
        c.ctx.d2c_q8_weigh(avg, weight)
        c.ctx.d2c_q8_evict(c.cache, L, weight, None, dst, kept, kw)
        c.ctx.d2c_q8_read(dst, n, None, rk, rv)

    state = [c.cache.k_codes, c.cache.v_codes, c.cache.k_scale, c.cache.v_scale, out, avg, weight, kept, kw, dst.k_codes, dst.v_codes,
             dst.k_scale, dst.v_scale, rk, rv, y]
    start = [t.clone() for t in state]

    def reset(i):
        for t, s in zip(state, start):
            t.copy_(s)
        for t, seed in ((dk, 10), (dv, 20), (q, 30)):
            g = torch.Generator(device="cuda").manual_seed(seed + i)
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))

    want = []
    for i in range(4):
        reset(i)
        step()
        torch.cuda.synchronize()
        want.append([t.clone() for t in state])
    reset(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in (0, 1, 2, 3, 1):
        reset(i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k, (t, s) in enumerate(zip(state, want[i])):
            assert torch.equal(t, s), f"replay {i}, tensor {k}"
        reset((i + 1) % 4)                              # eager work between the replays
        step()
        torch.cuda.synchronize()
        for k, (t, s) in enumerate(zip(state, want[(i + 1) % 4])):
            assert torch.equal(t, s), f"eager {i}, tensor {k}"
    side2 = torch.cuda.Stream()
    reset(2)
    side2.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side2):
        step()
    torch.cuda.synchronize()
    for t, s in zip(state, want[2]):
        assert torch.equal(t, s)


def test_refusals():
    say("q8 refusals")
    b = B()
    c = Case("gqa", "bf16", 100, max_rows=10, max_batch=2).fill()
    ctx, q = c.ctx, c.queries(4)
    out = torch.zeros_like(q)

    def refused(code, f):
        with pytest.raises(b.D2CError) as e:
            f()
        assert e.value.code == code and str(e.value)

    seq = lambda **kw: b.Q8Seq(c.cache, kw.pop("L", 100), kw.pop("m", 4), **kw)
    (dk, _), (dv, _) = c.new(4), c.new(4)
    refused(b.D2C_EINVAL, lambda: ctx.d2c_q8_attention([seq(q=q)]))                                     # no out
    refused(b.D2C_EINVAL, lambda: ctx.d2c_q8_attention([seq(q=q, out=out, new_k=dk)]))                  # no new_v
    refused(b.D2C_EINVAL, lambda: ctx.d2c_q8_update([seq()]))                                           # nothing to write
    refused(b.D2C_EINVAL, lambda: ctx.d2c_q8_attention([seq(q=q, out=out, L=0)]))
    refused(b.D2C_ESHAPE, lambda: ctx.d2c_q8_attention([b.Q8Seq(c.cache, 128, 4, q=q, out=out)]))       # the cache holds it, the handle does not
    refused(b.D2C_ESHAPE, lambda: seq(L=129))                                                           # beyond the cache
    refused(b.D2C_ESHAPE, lambda: ctx.d2c_q8_attention([seq(q=q, out=out)] * 3))                        # more than max_batch
    q11 = c.queries(11)
    refused(b.D2C_ESHAPE, lambda: ctx.d2c_q8_attention([seq(q=q11, out=torch.zeros_like(q11), m=11)]))  # more than max_rows
    refused(b.D2C_EINVAL, lambda: ctx.d2c_q8_update([seq(new_k=dk, new_v=dv, L=3)]))                    # more rows than L
    refused(b.D2C_EINVAL, lambda: ctx.d2c_q8_update([seq(new_k=dk, new_v=dv), seq(new_k=dk, new_v=dv)]))  # one cache twice
    off = torch.zeros(4 * ctx.d_q + 1, dtype=torch.bfloat16, device="cuda")[1:].view(4, ctx.d_q)
    refused(b.D2C_EINVAL, lambda: ctx.d2c_q8_attention([seq(q=off, out=out)]))                          # not 16-byte aligned
    refused(b.D2C_EINVAL, lambda: ctx.d2c_q8_read(c.cache, 100, None, torch.zeros((101, ctx.d_kv), dtype=torch.bfloat16, device="cuda"), None))
    wt, kept = torch.zeros(100, dtype=torch.int64, device="cuda"), torch.zeros(50, dtype=torch.int32, device="cuda")
    refused(b.D2C_EINVAL, lambda: ctx.d2c_q8_evict(c.cache, 100, wt, None, c.cache, kept))              # onto itself
    refused(b.D2C_EINVAL, lambda: ctx.d2c_q8_evict(c.cache, 100, wt, None, b.Q8Cache(ctx, 128), torch.zeros(101, dtype=torch.int32, device="cuda")))
    refused(b.D2C_EINVAL, lambda: ctx.d2c_q8_evict(c.cache, 100, wt.int(), None, b.Q8Cache(ctx, 50), kept))
    refused(b.D2C_ESHAPE, lambda: ctx.d2c_q8_evict(c.cache, 100, wt, None, b.Q8Cache(ctx, 49), torch.zeros(65, dtype=torch.int32, device="cuda")))
    lin = b.Q8Context(4, 4, 64, "bf16", max_rows=8, max_k=64, max_n=32)
    w = torch.zeros((32, 64), dtype=torch.bfloat16, device="cuda")
    p = lin.d2c_q8_pack(w)
    a = torch.zeros((9, 64), dtype=torch.bfloat16, device="cuda")
    refused(b.D2C_ESHAPE, lambda: lin.d2c_q8_linear(a, p, torch.zeros((9, 32), device="cuda")))
    refused(b.D2C_EINVAL, lambda: lin.d2c_q8_linear(a[:8], p, torch.zeros((8, 31), device="cuda")))
    refused(b.D2C_ESHAPE, lambda: lin.d2c_q8_pack(torch.zeros((4, 4), dtype=torch.bfloat16, device="cuda")))
    refused(b.D2C_ESHAPE, lambda: lin.d2c_q8_evict(c.cache, 100, wt, None, b.Q8Cache(ctx, 50), kept))
    c.check()                                                                                            # none of them wrote anything
    ctx.d2c_q8_attention([])
    ctx.d2c_q8_update([seq(m=0)])
    lin.d2c_q8_linear(a[:0], p, torch.zeros((0, 32), device="cuda"))
    c.check()


def test_places_past_32_bits():
    """A cache whose last rows lie more than 4 GiB behind its first: refresh, read, attention, weight, eviction.  All but three rows are
    zeros, so the plain form needs only those three."""
    say("q8 places past 32 bits")
    H, D, L = 32, 128, (1 << 20) + 12345
    idx = np.array([5, (1 << 20) + 3, L - 1])
    rng, t = np.random.default_rng(11), lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()
    ctx = B().Q8Context(H, H, D, "f32", max_seq=L, max_rows=3)
    cache = B().Q8Cache(ctx, L)
    assert cache.k_codes.numel() > 1 << 32
    k, v, q = t(3.0 * rng.standard_normal((3, H * D))), t(rng.standard_normal((3, H * D))), t(rng.standard_normal((3, H * D)))
    out, avg = torch.zeros_like(q), torch.zeros((3, L), device="cuda")
    ctx.d2c_q8_attention([B().Q8Seq(cache, L, 3, idx=torch.tensor(idx, dtype=torch.int32, device="cuda"), new_k=k, new_v=v, q=q, out=out,
                                    attn_avg=avg)])
    ref = R.Cache8(192, H, D)                          # each of the three alone in its block, as it is in the cache
    at = np.array([5, 67, 191])
    ref.update(at, f64(k).reshape(3, H, D), f64(v).reshape(3, H, D), 192)
    rk, rv = torch.zeros((4, H * D), device="cuda"), torch.zeros((4, H * D), device="cuda")
    ctx.d2c_q8_read(cache, L, torch.tensor(list(idx) + [L - 2], dtype=torch.int32, device="cuda"), rk, rv)
    for got, want in ((rk, ref.k), (rv, ref.v)):
        assert np.array_equal(got[:3].cpu().numpy(), want.values()[at].reshape(3, -1).astype(np.float32)) and not got[3].any()
    kk, vv, qq = ref.k.values()[at], ref.v.values()[at], f64(q).reshape(3, H, D)
    s = np.einsum("mhd,nhd->mhn", qq, kk) / D ** 0.5
    sums = np.einsum("mhd,nhd->mhn", np.abs(qq), np.abs(kk)) / D ** 0.5
    share = float((D + 4) * sums.max() + 6 * np.abs(s).max() + 8) * 2.0 ** -24         # as R.attention has it
    den = (L - 3) + np.exp(s).sum(2)
    p = np.exp(s) / den[:, :, None]
    o, mag = np.einsum("mhn,nhd->mhd", p, vv), np.einsum("mhn,nhd->mhd", p, np.abs(vv))
    tol = HALF["f32"] * np.abs(o) + mag * (2 * share + P_HALF["f32"] + (L ** 0.5 + 70) * 2.0 ** -24) * 1.001 + 2.0 ** -36 * np.abs(vv).sum(0)[None]
    assert (np.abs(f64(out).reshape(3, H, D) - o) <= tol).all()
    a = f64(avg)
    for cols, want in ((idx, p.mean(1)), ([0, 1 << 20, L - 2], np.repeat((1 / den).mean(1)[:, None], 3, 1))):
        assert (np.abs(a[:, cols] - want) <= want * (2 * share + (L ** 0.5 + H + 16) * 2.0 ** -24)).all()
    weight = torch.zeros(L, dtype=torch.int64, device="cuda")
    ctx.d2c_q8_weigh(avg, weight)
    assert np.array_equal(weight.cpu().numpy(), R.weigh(a, np.zeros(L, np.int64)))
    weight[torch.from_numpy(idx).cuda()] += 1 << 40
    dst, kept = B().Q8Cache(ctx, 3), torch.zeros(3, dtype=torch.int32, device="cuda")
    ctx.d2c_q8_evict(cache, L, weight, None, dst, kept)
    assert np.array_equal(kept.cpu().numpy(), idx)
    small = ref.evict(at)
    ctx.d2c_q8_read(dst, 3, None, rk[:3], rv[:3])
    for got, want in ((rk, small.k), (rv, small.v)):
        assert np.array_equal(got[:3].cpu().numpy(), want.values(3).reshape(3, -1).astype(np.float32))


def test_a_cache_that_one_sequence_refreshes_and_others_read():
    """All of a call's refreshes come before its attention, in whatever order the sequences stand."""
    say("q8 shared cache")
    c = Case("gqa", "bf16", 400, max_batch=12).fill()
    (dk, nk), (dv, nv) = c.new(7), c.new(7)
    idx = np.sort(c.rng.permutation(400)[:7])
    seqs, got = [], []
    for i in range(12):
        q = c.queries(7)
        out = torch.zeros_like(q)
        new = dict(idx=torch.tensor(idx, dtype=torch.int32, device="cuda"), new_k=dk, new_v=dv) if i == 10 else {}
        seqs.append(B().Q8Seq(c.cache, 400, 7, q=q, out=out, **new))
        got.append((q, out))
    c.ctx.d2c_q8_attention(seqs)
    c.ref.update(idx, nk, nv, 400)
    c.check()
    for q, out in got:
        c.expect(q, out, None)


def test_two_handles_at_once():
    """Two handles on two streams, their calls overlapping in time, give what each gives alone."""
    say("q8 two handles at once")
    cs = [Case("dream", "bf16", 3000 + 500 * i, seed=i).fill() for i in range(2)]
    qs = [c.queries(40 + i) for i, c in enumerate(cs)]
    alone = [attend(c, q.shape[0], q=q)[1:] for c, q in zip(cs, qs)]
    outs = [[(torch.zeros_like(q), torch.zeros((q.shape[0], c.L), device="cuda")) for _ in range(10)] for c, q in zip(cs, qs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    for j in range(10):
        for c, q, o, st in zip(cs, qs, outs, streams):
            with torch.cuda.stream(st):
                c.ctx.d2c_q8_attention([B().Q8Seq(c.cache, c.L, q.shape[0], q=q, out=o[j][0], attn_avg=o[j][1])])
    torch.cuda.synchronize()
    for (x, a), o in zip(alone, outs):
        for y, b in o:
            assert torch.equal(x, y) and torch.equal(a, b)


def test_refusals_of_overlaps_and_other_geometries():
    say("q8 refusals of overlaps")
    b = B()
    c = Case("gqa", "bf16", 200, max_rows=10, max_batch=2).fill()
    ctx = c.ctx

    def refused(code, f):
        with pytest.raises(b.D2CError) as e:
            f()
        assert e.value.code == code and str(e.value)

    q = c.queries(4)
    batch = b.Q8Batch(ctx, [b.Q8Seq(c.cache, 200, 4, q=q, out=torch.zeros_like(q))])
    other = b.Q8Context(8, 4, 64, "bf16", max_seq=300, max_rows=10)
    refused(b.D2C_ESHAPE, lambda: other.d2c_q8_attention(batch))                        # a batch of another handle's geometry
    refused(b.D2C_ESHAPE, lambda: other.d2c_q8_attention([b.Q8Seq(c.cache, 200, 4, q=q, out=torch.zeros_like(q))]))
    rk = torch.zeros((4, other.d_kv), dtype=torch.bfloat16, device="cuda")
    refused(b.D2C_ESHAPE, lambda: other.d2c_q8_read(c.cache, 200, None, rk, None))
    refused(b.D2C_EINVAL, lambda: ctx.d2c_q8_read(c.cache, 200, None, None, None))
    # the second cache begins inside the first
    (dk, _), (dv, _) = c.new(4), c.new(4)
    inner = b.Q8Cache(ctx, 64)
    inner.c.v_codes = c.cache.v_codes.data_ptr() + 64 * ctx.d_kv
    refused(b.D2C_EINVAL, lambda: ctx.d2c_q8_update([b.Q8Seq(c.cache, 200, 4, new_k=dk, new_v=dv), b.Q8Seq(inner, 64, 4, new_k=dk, new_v=dv)]))
    wt = torch.zeros(200, dtype=torch.int64, device="cuda")
    kept = torch.zeros(50, dtype=torch.int32, device="cuda")
    refused(b.D2C_EINVAL, lambda: ctx.d2c_q8_evict(c.cache, 200, wt, None, inner, kept))
    dst = b.Q8Cache(ctx, 50)
    refused(b.D2C_EINVAL, lambda: ctx.d2c_q8_evict(c.cache, 200, wt, None, dst, kept, wt[10:60]))
    refused(b.D2C_EINVAL, lambda: ctx.d2c_q8_evict(c.cache, 200, wt, None, dst, wt[:25].view(torch.int32)))
    lin = b.Q8Context(4, 4, 64, "f32", max_rows=8, max_k=64, max_n=64)
    p = lin.d2c_q8_pack(torch.ones((64, 64), device="cuda"))
    a = torch.ones((8, 64), device="cuda")
    refused(b.D2C_EINVAL, lambda: lin.d2c_q8_linear(a, p, a))
    assert (a == 1).all() and not wt.any() and not kept.any()
    big = torch.zeros(1, device="cuda")
    lib, h, st = b._lib, ctx.handle, torch.cuda.current_stream().cuda_stream
    assert lib.d2c_q8_weigh(h, big.data_ptr(), 1, (1 << 24) + 1, wt.data_ptr(), st) == b.D2C_ESHAPE
    assert lib.d2c_q8_weigh(h, big.data_ptr(), (1 << 24) + 1, 1, wt.data_ptr(), st) == b.D2C_ESHAPE
    assert lib.d2c_q8_read(h, c.cache.ref, 200, kept.data_ptr(), (1 << 24) + 1, rk.data_ptr(), None, st) == b.D2C_ESHAPE
    c.check()


def test_two_graphs_of_one_handle():
    """A product and an attention captured in graphs of their own share the handle's workspace: replayed in turn, with eager calls between."""
    say("q8 two graphs of one handle")
    H, Hkv, D, L, m = 8, 2, 64, 1500, 40
    ctx = B().Q8Context(H, Hkv, D, "bf16", max_seq=L, max_rows=m, max_k=4096, max_n=600)
    c = Case((H, Hkv, D), "bf16", L, ctx=ctx).fill()
    w, a = dev(0.05 * c.rng.standard_normal((600, 4096)), "bf16"), dev(c.rng.standard_normal((m, 4096)), "bf16")
    p, q = ctx.d2c_q8_pack(w), c.queries(m)
    y, out, avg = torch.zeros((m, 600), device="cuda"), torch.zeros_like(q), torch.zeros((m, L), device="cuda")
    batch = B().Q8Batch(ctx, [B().Q8Seq(c.cache, L, m, q=q, out=out, attn_avg=avg)])
    calls = [lambda: ctx.d2c_q8_linear(a, p, y), lambda: ctx.d2c_q8_attention(batch)]
    for f in calls:
        f()
    torch.cuda.synchronize()
    want = [t.clone() for t in (y, out, avg)]
    graphs = []
    for f in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            f()
    for i in range(6):
        for t in (y, out, avg):
            t.fill_(7.0)
        graphs[i % 2].replay()
        graphs[1 - i % 2].replay()
        if i % 3 == 0:
            calls[i % 2]()
        torch.cuda.synchronize()
        for t, x in zip((y, out, avg), want):
            assert torch.equal(t, x), f"replay {i}"


@pytest.mark.parametrize("L", [1, 65, 191, 1100, 5000, 20481])
def test_evict_looks_at_nothing_behind_its_arrays(L):
    """Weights and protection as views of longer arrays that hold large weights and protected rows behind them; what lies behind kept stays."""
    say(f"q8 evict views L={L}")
    c = Case((1, 1, 64), "bf16", L).fill()
    w, p = weights(c.rng, L, "spread"), (c.rng.random(L) < 0.2).astype(np.uint8)
    long_w = torch.full((L + 40000,), (1 << 63) - 1, dtype=torch.int64, device="cuda")
    long_p = torch.full((L + 40000,), 255, dtype=torch.uint8, device="cuda")
    long_w[:L], long_p[:L] = torch.from_numpy(w).cuda(), torch.from_numpy(p).cuda()
    for n, q in ((1, None), ((L + 1) // 2, None), (L, None), (1, p), ((L + 1) // 2, p), (max(1, int(p.sum())), p), (L, p)):
        kept = torch.full((n + 64,), -7, dtype=torch.int32, device="cuda")
        kw = torch.full((n + 64,), -7, dtype=torch.int64, device="cuda")
        c.ctx.d2c_q8_evict(c.cache, L, long_w[:L], None if q is None else long_p[:L], B().Q8Cache(c.ctx, n), kept[:n], kw[:n])
        want = R.keep(w, q, n)
        assert np.array_equal(kept[:n].cpu().numpy(), want), f"n={n}"
        assert np.array_equal(kw[:n].cpu().numpy(), w[want])
        assert (kept[n:] == -7).all() and (kw[n:] == -7).all()


@pytest.mark.parametrize("L", [64, 700, 20001])
def test_float_attention_beside_keys_that_take_nearly_all(L):
    """One key of each block has a value of 0 and a score 20 to 26 bits above the others' 0: the output is what the far smaller probabilities,
    all alike, leave of their bits.  A probability is rounded as two fp16 pieces times 2^15 of the row's largest: where the second is a
    subnormal number, by at most half of 2^-24, that is 2^-40 of the largest, which is at most a block's share of the row's sum.  Of a
    score's 64 products one is not 0."""
    say(f"q8 attention float, small probabilities L={L}")
    D, m = 64, 48
    c = Case((1, 1, D), "f32", L, max_rows=m)
    k, v = np.zeros((L, 1, D)), 1.0 + c.rng.random((L, 1, D))
    k[::64, 0, 0], v[::64] = 3.0, 0.0
    k, v = (dev(x, "f32").reshape(L, D) for x in (k, v))
    c.update(None, m=L, new=((k, f64(k).reshape(L, 1, D)), (v, f64(v).reshape(L, 1, D))))
    c.check()
    q = np.zeros((m, D))
    q[:, 0] = np.linspace(20, 26, m) * np.log(2) * np.sqrt(D) / 3
    q, out, avg = attend(c, m, q=dev(q, "f32"))
    vv = c.ref.v.values(L)
    o, a, mag, _ = R.attention(f64(q).reshape(m, 1, D), c.ref.k.values(L), vv)
    s = 26 * np.log(2)
    share = ((1 + 4) * s + 6 * s + 8) * 2.0 ** -24             # as R.attention has it, of one product
    below = 2.0 ** -40 * vv.sum(0)[None] / -(-L // 64)
    tol = HALF["f32"] * o + (1 + HALF["f32"]) * (mag * (2 * share + P_HALF["f32"] + (L ** 0.5 + 70) * 2.0 ** -24) + below)
    err = np.abs(f64(out).reshape(m, 1, D) - o)
    assert (err <= tol).all(), "out: %g times the bound" % (err / tol).max()
    err = np.abs(f64(avg) - a)
    assert (err <= a * (2 * share + (L ** 0.5 + 17) * 2.0 ** -24)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_size,k_size", [(1e-36, 1e36), (1e-38, 1e37), (1e30, 1e-30), (1e-30, 1e-6)])
def test_attention_of_tiny_queries_on_huge_keys(dtype, q_size, k_size):
    """Queries near the type's smallest numbers and keys that make ordinary scores of them, and the other way round."""
    say(f"q8 attention {dtype} queries of {q_size}, keys of {k_size}")
    c = Case("gqa", dtype, 200)
    k, (dv, nv) = rows(c.rng, 200, c.Hkv, c.D) * k_size, c.new(200)
    dk = dev(k, dtype).reshape(200, c.Hkv * c.D)
    c.update(None, m=200, new=((dk, f64(dk).reshape(k.shape)), (dv, nv)))
    c.check()
    q, out, avg = attend(c, 9, q=c.queries(9, q_size))
    c.expect(q, out, avg)


def test_what_is_written_must_not_overlap_anything():
    """Every call whose output lies over an input or another output is refused, and nothing is written; neighbours are not."""
    say("q8 overlaps")
    b, L, m = B(), 200, 4
    c = Case("gqa", "bf16", L, max_rows=300, max_batch=8).fill()
    ctx, t = c.ctx, torch.bfloat16

    def refused(f):
        with pytest.raises(b.D2CError) as e:
            f()
        assert e.value.code == b.D2C_EINVAL and "overlap" in str(e.value)

    def seq(cache=None, **kw):
        q = c.queries(m)
        args = dict(q=q, out=torch.zeros_like(q), attn_avg=torch.zeros((m, L), device="cuda")) | kw
        return b.Q8Seq(cache or c.cache, L, m, **args)

    attend_ = lambda *s: ctx.d2c_q8_attention(list(s))
    (dk, _), (dv, _) = c.new(m), c.new(m)
    idx = torch.arange(m, dtype=torch.int32, device="cuda")
    fresh = dict(idx=idx, new_k=dk, new_v=dv)
    first = seq()
    refused(lambda: attend_(seq(q=first.q, out=first.q)))
    refused(lambda: attend_(first, seq(out=first.out)))
    refused(lambda: attend_(first, seq(attn_avg=first.attn_avg)))
    refused(lambda: attend_(first, seq(out=first.q)))
    refused(lambda: attend_(seq(attn_avg=torch.zeros(m * max(L, ctx.d_q), device="cuda")[: m * L].view(m, L), out=first.out), first))
    over_k = c.cache.k_codes[: m * ctx.d_q * 2].view(t).view(m, ctx.d_q)
    refused(lambda: attend_(seq(out=over_k)))
    other = b.Q8Cache(ctx, L)
    refused(lambda: attend_(seq(out=over_k, cache=other), seq(**fresh)))
    refused(lambda: ctx.d2c_q8_update([seq(idx=idx, new_k=c.cache.v_codes[: m * ctx.d_kv * 2].view(t).view(m, ctx.d_kv), new_v=dv)]))
    refused(lambda: ctx.d2c_q8_update([seq(idx=c.cache.k_scale.view(-1)[:m].view(torch.int32), new_k=dk, new_v=dv)]))
    refused(lambda: ctx.d2c_q8_update([seq(**fresh), seq(**fresh)]))
    both = b.Q8Cache(ctx, L)
    both.c.v_codes = both.c.k_codes
    refused(lambda: ctx.d2c_q8_update([seq(cache=both, **fresh)]))
    rk, rv = (torch.zeros((m, ctx.d_kv), dtype=t, device="cuda") for _ in range(2))
    refused(lambda: ctx.d2c_q8_read(c.cache, L, idx, rk, rk))
    refused(lambda: ctx.d2c_q8_read(c.cache, L, idx, c.cache.v_codes[: m * ctx.d_kv * 2].view(t).view(m, ctx.d_kv), rv))
    refused(lambda: ctx.d2c_q8_read(c.cache, L, rk.view(-1).view(torch.int32)[:m], rk, rv))
    c.check()

    lin = b.Q8Context(4, 4, 64, "f32", max_rows=300, max_k=64, max_n=64)
    w, a = torch.ones((64, 64), device="cuda"), torch.ones((64, 64), device="cuda")
    p = lin.d2c_q8_pack(w)
    refused(lambda: lin.d2c_q8_linear(a, p, a))
    refused(lambda: lin.d2c_q8_linear(a[:16], p, p.codes.view(torch.float32).view(16, 64)))
    refused(lambda: lin.d2c_q8_linear(a[:1], p, p.scale.view(1, 64)))
    rc = b._lib.d2c_q8_pack(lin.handle, w.data_ptr(), 64, 64, w.data_ptr(), p.scale.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert rc == b.D2C_EINVAL and (w == 1).all() and (a == 1).all()

    weight, kept = torch.zeros(L, dtype=torch.int64, device="cuda"), torch.zeros(50, dtype=torch.int32, device="cuda")
    kw, dst = torch.zeros(50, dtype=torch.int64, device="cuda"), b.Q8Cache(ctx, 50)
    refused(lambda: ctx.d2c_q8_weigh(weight.view(torch.float32)[:L].view(1, L), weight))
    refused(lambda: ctx.d2c_q8_evict(c.cache, L, weight, None, dst, c.cache.k_codes[:200].view(torch.int32), kw))
    refused(lambda: ctx.d2c_q8_evict(c.cache, L, weight, None, dst, dst.k_codes[:200].view(torch.int32), kw))
    refused(lambda: ctx.d2c_q8_evict(c.cache, L, weight, None, dst, kept, c.cache.v_codes[:400].view(torch.int64)))
    c.check()
    assert not weight.any() and not kept.any() and (dst.k_codes == 128).all()

    # neighbours in one allocation, a shared input, and a cache that others read are no overlap
    both = torch.zeros((4 * m, ctx.d_q), dtype=t, device="cuda")
    both[: 2 * m] = c.queries(2 * m)
    s = [seq(q=both[:m], out=both[2 * m: 3 * m]), seq(q=both[m: 2 * m], out=both[3 * m:]), seq(q=both[:m], **fresh)]
    attend_(*s)
    ref = c.ref
    ref.update(np.arange(m), f64(dk).reshape(m, c.Hkv, c.D), f64(dv).reshape(m, c.Hkv, c.D), L)
    c.check()
    for x in s:
        c.expect(x.q, x.out, x.attn_avg)


def test_averages_of_more_tiles_than_a_launch_has_room_for_are_refused():
    """2^23 workgroups of 512 threads do not fit a launch: refused before anything is looked at (the sizes are claimed, no such buffer is)."""
    say("q8 averages too large")
    b = B()
    ctx = b.Q8Context(1, 1, 64, "bf16", max_seq=1 << 24, max_rows=1 << 12, max_batch=2)
    cache, x = b.Q8Cache(ctx, 64), torch.zeros(1024, device="cuda")
    st, p = torch.cuda.current_stream().cuda_stream, x.data_ptr()
    for sizes in ([(1 << 10, 1 << 24)], [(1 << 10, (1 << 23) + 1), (993, 1 << 23)], [(1, 1 << 24), (1 << 11, 1 << 23)]):
        arr = (b.d2c_q8_seq * len(sizes))()
        for s, (m, L) in zip(arr, sizes):
            s.cache, s.q, s.out, s.attn_avg, s.m, s.L = cache.c, p, p, p, m, L
        assert b._lib.d2c_q8_attention(ctx.handle, arr, len(sizes), st) == b.D2C_ESHAPE
        assert b"tiles" in b._lib.d2c_q8_last_error(ctx.handle)
    assert not x.any()


@pytest.mark.parametrize("m,N,K", [(5, 768, 256), (20, 512, 4096), (37, 256, 4096), (300, 512, 256), (100, 1000, 512)])
def test_linear_into_outputs_of_any_alignment(m, N, K):
    """out is float: any multiple of 4 bytes will do."""
    say(f"q8 linear out anywhere m={m} N={N} K={K}")
    rng = np.random.default_rng([m, N, K])
    a, w = dev(rng.standard_normal((m, K)), "bf16"), dev(rng.standard_normal((N, K)), "bf16")
    ctx = B().Q8Context(4, 4, 64, "bf16", max_rows=m, max_k=K, max_n=N)
    p, want = ctx.d2c_q8_pack(w), R.linear(f64(a), f64(w))[0]
    for shift in (0, 1, 2, 3):
        room = torch.full((m * N + 8,), 5.0, device="cuda")
        ctx.d2c_q8_linear(a, p, room[shift: shift + m * N].view(m, N))
        assert np.array_equal(room[shift: shift + m * N].view(m, N).cpu().numpy(), want)
        assert (room[:shift] == 5.0).all() and (room[shift + m * N:] == 5.0).all()


def _linear_sizes():
    from q8_sizes import LINEAR
    return [(key, size) for key, sizes in LINEAR.items() for size in sizes]


@pytest.mark.parametrize("key,size", _linear_sizes(), ids=lambda x: "-".join(map(str, x)))
def test_linear_in_every_kernel(key, size):
    """Each kernel of the product, by sizes that leave a part of its last tiles; rows and channels that are not finite stay among themselves."""
    from q8_sizes import linear
    m, N, K = size
    say(f"q8 linear kernel {key} size {size}")
    p = B().d2c_q8_plan_linear(m, N, K)
    assert (p["kernel"], p["row_tiles"], p["col_tiles"], p["splits"] > 1) == key
    for dtype in ("bf16", "f32") if N * K < 10 ** 8 else ("bf16",):
        t, g = torch.bfloat16 if dtype == "bf16" else torch.float32, torch.Generator(device="cuda").manual_seed(m + N + K)
        a = torch.randn((m, K), generator=g, device="cuda").to(t)
        w = (0.02 * torch.exp(torch.randn((N, 1), generator=g, device="cuda")) * torch.randn((N, K), generator=g, device="cuda")).to(t)
        if m > 5:
            a[1], a[2] = 0, 0
            a[2, K // 2], a[m - 2, K - 1], w[N - 1, 0], w[3, K - 1] = -5, float("nan"), float("inf"), float("nan")
        ctx = B().Q8Context(4, 4, 64, dtype, max_rows=m, max_k=K, max_n=N)
        pack = ctx.d2c_q8_pack(w)
        room = torch.full((m * N + 2048,), 123.0, device="cuda")
        out = room[1024: 1024 + m * N].view(m, N)
        ctx.d2c_q8_linear(a, pack, out)
        want, sw = linear(a, w)
        assert torch.equal(pack.scale.nan_to_num(nan=-1.0), sw.nan_to_num(nan=-1.0))
        assert torch.equal(out.isnan(), want.isnan()) and torch.equal(out.nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))
        assert (room[:1024] == 123.0).all() and (room[1024 + m * N:] == 123.0).all()
        room.fill_(7.0)
        ctx.d2c_q8_linear(a, pack, out)
        assert torch.equal(out.nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))


@pytest.mark.parametrize("L", [4096, 4097, 6144, 6145, 9000, 20480])
def test_evict_where_the_choice_changes_its_form(L):
    """On both sides of the sizes at which keys are held in registers or read again."""
    say(f"q8 evict forms L={L}")
    c = Case((1, 1, 64), "bf16", L).fill()
    for kind in ("spread", "ties", "wide"):
        w, p = weights(c.rng, L, kind), (c.rng.random(L) < 0.1).astype(np.uint8)
        dw, dp = torch.from_numpy(w).cuda(), torch.from_numpy(p).cuda()
        for n, q in ((L // 3, None), (L // 3, p), (L // 50, p), (L, p)):
            dst, kept, kw = B().Q8Cache(c.ctx, n), torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int64, device="cuda")
            c.ctx.d2c_q8_evict(c.cache, L, dw, None if q is None else dp, dst, kept, kw)
            want = R.keep(w, q, n)
            assert np.array_equal(kept.cpu().numpy(), want) and np.array_equal(kw.cpu().numpy(), w[want]), f"{kind} n={n}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_of_the_largest_scores(dtype):
    """Scores up to 2^22: a key that leads by 64 takes all (the scores' own rounding is (D + 10) 2^-24 of 2^22, below 20)."""
    say(f"q8 attention largest scores {dtype}")
    c = Case("gqa", dtype, 300).fill()
    k, v, m = c.ref.k.values(300), c.ref.v.values(300), 40
    q = c.queries(m)
    group = np.arange(c.H) // (c.H // c.Hkv)
    score = lambda q: np.einsum("mhd,nhd->mhn", f64(q).reshape(m, c.H, c.D), k[:, group]) / c.D ** 0.5
    q = (q.float() * float(0.9 * 2 ** 22 / np.abs(score(q)).max())).to(q.dtype)
    s = np.sort(score(q), 2)
    assert 2 ** 21 < np.abs(s).max() < 2 ** 22
    clear, first = s[:, :, -1] - s[:, :, -2] > 64, score(q).argmax(2)
    assert clear.mean() > 0.9
    q, out, avg = attend(c, m, q=q)
    assert torch.isfinite(out).all() and torch.isfinite(avg).all()
    want, got = v[first, group[None]], f64(out).reshape(m, c.H, c.D)
    tol = (HALF[dtype] + P_HALF[dtype] + 2.0 ** -20) * np.abs(want) + 1e-12
    assert (np.abs(got - want) <= tol)[clear].all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_average_of_equal_scores_is_one_over_the_length(dtype):
    """Equal scores: the exponentials are 1 and their sum is L, both exact; two roundings are left, of 1 / L and of its product, and as many
    again are allowed (the instructions' own).  The float output of values that are all 1 likewise, with its sum's product beside them."""
    say(f"q8 average of equal scores {dtype}")
    c = Case((1, 1, 64), dtype, 4200)
    one = dev(np.ones((4200, 64)), dtype)
    c.update(None, m=4200, new=((one, f64(one).reshape(4200, 1, 64)),) * 2)
    value = float(c.ref.v.values(1)[0, 0, 0])
    for L in [1, 3, 7] + list(range(70, 260, 9)) + [1000, 1023, 2500, 4199]:
        q, out, avg = attend(c, 2, L=L, q=torch.zeros((2, 64), dtype=c.ctx.torch_dtype, device="cuda"))
        assert np.abs(f64(avg) * L - 1).max() <= 4 * 2.0 ** -24, L
        if dtype == "f32":
            assert np.abs(f64(out) / value - 1).max() <= (8 + L ** 0.5) * 2.0 ** -24, L


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_of_the_largest_values(dtype):
    """Values of V up to 2^112 / L: sums over the keys stay in float's range."""
    say(f"q8 attention largest values {dtype}")
    for L in (64, 1100):
        c = Case("gqa", dtype, L)
        v = c.rng.uniform(0.5, 1.0, (L, c.Hkv, c.D)) * 2.0 ** 112 / L
        dv = dev(v, dtype).reshape(L, c.Hkv * c.D)
        c.update(None, m=L, new=(c.new(L), (dv, f64(dv).reshape(v.shape))))
        c.check()
        q = c.queries(9)
        q[0] = 0
        q, out, avg = attend(c, 9, q=q)
        c.expect(q, out, avg)
