"""CPU-side checks of the paged cache: the header against the library and the binding, refusals that need no GPU, and what the plain 64-bit
forms (which the GPU tests compare with) promise."""
import ctypes
import itertools
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

import pg_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2509_23094_amd", "libd2c.so")
built = pytest.mark.skipif(not os.path.exists(LIB), reason="libd2c.so not built (run __graft_entry__.build())")


@built
def test_header_library_and_binding_agree():
    from paper_2509_23094_amd import binding as B
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "d2c_pg.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(d2c_pg_[a-z_0-9]+)\s*\(", text)))
    assert names == sorted(B.PG_EXPORTS)
    for n in names:
        assert getattr(B._lib, n) is not None
    for n in ("rotate", "append", "read", "attention"):
        assert hasattr(B.PgContext, "d2c_pg_" + n)
    # 10 whole numbers, 64 doubles, 64 bytes; 5 pointers and 3 whole numbers; ...
    assert [ctypes.sizeof(c) for c in (B.d2c_pg_dims, B.d2c_pg_cache, B.d2c_pg_batch, B.d2c_pg_new, B.d2c_pg_attend)] == [616, 24, 56, 80, 64]


def dims(**more):
    from paper_2509_23094_amd import binding as B
    d = B.d2c_pg_dims(4, 2, 64, B.D2C_BF16, 64, 16, 4, 32, 2, 0)
    for i in range(32):
        d.freq[i], d.axis[i] = 10000.0 ** (-i / 32), i % 2
    for name, value in more.items():
        setattr(d, name, value)
    return d


@built
@pytest.mark.parametrize("field,value,code", [
    ("n_heads", 0, -1), ("n_heads", 2048, -1), ("n_kv_heads", 0, -1), ("n_kv_heads", 3, -1), ("head_dim", 96, -4), ("dtype", 2, -1),
    ("page_rows", 16, -4), ("page_rows", 48, -4), ("page_rows", 512, -4), ("max_rows", -1, -1), ("max_rows", (1 << 20) + 1, -1),
    ("max_batch", -1, -1), ("max_batch", 1025, -1), ("n_pairs", -8, -1), ("n_pairs", 12, -1), ("n_pairs", 40, -1), ("n_axes", 5, -1),
    ("n_axes", 1, -1), ("pairing", 2, -1)])
def test_init_refuses(field, value, code):
    from paper_2509_23094_amd import binding as B
    out = ctypes.c_void_p()
    assert B._lib.d2c_pg_init(ctypes.byref(dims(**{field: value})), ctypes.byref(out)) == code
    assert B._lib.d2c_pg_last_error(None) and not out


@built
@pytest.mark.parametrize("freq", [float("nan"), float("inf"), 65537.0, -65537.0])
def test_init_refuses_frequencies(freq):
    from paper_2509_23094_amd import binding as B
    d, out = dims(), ctypes.c_void_p()
    d.freq[31] = freq
    assert B._lib.d2c_pg_init(ctypes.byref(d), ctypes.byref(out)) == B.D2C_EINVAL
    assert b"frequency" in B._lib.d2c_pg_last_error(None)


@built
def test_null_arguments_are_refused():
    from paper_2509_23094_amd import binding as B
    lib, out = B._lib, ctypes.c_void_p()
    assert lib.d2c_pg_init(None, ctypes.byref(out)) == B.D2C_EINVAL
    assert lib.d2c_pg_init(ctypes.byref(dims()), None) == B.D2C_EINVAL
    assert lib.d2c_pg_destroy(None) == B.D2C_OK
    assert lib.d2c_pg_workspace_bytes(None) == 0
    assert lib.d2c_pg_cache_size(None, 1, None) == B.D2C_EINVAL
    assert lib.d2c_pg_rotate(None, None, 0, 0, 1, 1, None, 0, None, 0, None) == B.D2C_EINVAL
    assert lib.d2c_pg_append(None, None, None, None, None) == B.D2C_EINVAL
    assert lib.d2c_pg_read(None, None, None, None, 0, None, 0, None) == B.D2C_EINVAL
    assert lib.d2c_pg_attention(None, None, None, None, None) == B.D2C_EINVAL


@built
def test_rotary_ladders():
    from paper_2509_23094_amd import binding as B
    r = B.Rotary([2, 3, 3], 10000.0)
    assert r.axis == [0, 0, 1, 1, 1, 2, 2, 2] and r.n_axes == 3
    assert np.allclose(r.freq, 10000.0 ** -(np.arange(8) / 8), rtol=1e-15)
    r = B.Rotary([2, 3, 3], 100.0, ladder="own", pairing="neighbours")
    assert np.allclose(r.freq, 100.0 ** -np.array([0, .5, 0, 1 / 3, 2 / 3, 0, 1 / 3, 2 / 3])) and r.pairing == B.D2C_PG_NEIGHBOURS
    r = B.Rotary(freq=[1.0, 0.5], axis=[3, 0])
    assert r.n_axes == 4
    for bad in (dict(pairs=[8], ladder="third"), dict(pairs=[8], pairing="odd"), dict(), dict(pairs=[8], freq=[1.0]), dict(pairs=[65]),
                dict(pairs=[8] * 5), dict(freq=[1.0], axis=[4]), dict(freq=[1.0], axis=[0, 0]), dict(freq=[1.0], axis=[-1])):
        with pytest.raises(B.D2CError):
            B.Rotary(**bad)


@built
@pytest.mark.parametrize("value", [(1 << 32) + 64, 1 << 32, 1 << 31, -(1 << 31) - 1, (1 << 64) + 1])
def test_binding_refuses_what_32_bits_do_not_hold(value):
    """Nothing goes on with the low 32 bits of a larger number (2^32 + 1 as a block would be causal)."""
    import torch
    from paper_2509_23094_amd import binding as B
    sizes = dict(n_heads=4, n_kv_heads=2, head_dim=64, page_rows=64, max_rows=16, max_batch=4)
    for name in sizes:
        with pytest.raises(B.D2CError, match=name) as e:
            B.PgContext(dtype="bf16", **{**sizes, name: value})
        assert e.value.code == B.D2C_EINVAL
    ctx = object.__new__(B.PgContext)
    ctx.handle, ctx.device = None, 0
    for name in ("block", "window"):
        with pytest.raises(B.D2CError, match=name):
            ctx.d2c_pg_attention(None, None, None, None, **{name: value})
    none = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(B.D2CError, match="n_rows"):
        B.PgBatch(ctx, none, none, none.view(1, 1), value)


@built
@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-46, 1e-50, 5e-324, -1e-50, -1.0, float("nan"), float("-inf")])
def test_binding_refuses_scales_that_are_not_positive_in_32_bits(scale):
    """A positive number that 32 bits round to 0 does not become the default 1 / sqrt(D)."""
    from paper_2509_23094_amd import binding as B
    ctx = object.__new__(B.PgContext)
    ctx.handle = None
    with pytest.raises(B.D2CError, match="scale") as e:
        ctx.d2c_pg_attention(None, None, None, None, scale=scale)
    assert e.value.code == B.D2C_EINVAL


# ------------------------------------------------------------------ the plain forms

def test_plain_rotation():
    """Lengths stay, turns add up, the angle between two rows depends on their distance, the inverse undoes."""
    rng = np.random.default_rng(0)
    x, y = rng.standard_normal((2, 5, 3, 16))
    freq, axis = 100.0 ** -(np.arange(6) / 6), [0, 1, 0, 1, 0, 1]
    for pairing in ("halves", "neighbours"):
        pos = rng.integers(-50, 50, (2, 5))
        t = R.rotate(x, pos, freq, axis, pairing)
        assert np.allclose((t ** 2).sum(2), (x ** 2).sum(2)) and np.array_equal(t[..., 12:], x[..., 12:])
        assert np.allclose(R.rotate(t, pos, freq, axis, pairing), R.rotate(x, 2 * pos, freq, axis, pairing))
        assert np.allclose(R.rotate(t, pos, freq, axis, pairing, inverse=True), x)
        far = (R.rotate(x, pos + 1000, freq, axis, pairing) * R.rotate(y, pos + 1007, freq, axis, pairing)).sum(2)
        assert np.allclose(far, (R.rotate(x, pos, freq, axis, pairing) * R.rotate(y, pos + 7, freq, axis, pairing)).sum(2))


def test_plain_masks():
    def see(*a):
        return np.flatnonzero(R.seen(*a)).tolist()
    assert see(3, 6, 1, 0, 0, True) == [0, 1, 2, 3]
    assert see(3, 6, 4, 0, 0, True) == [0, 1, 2, 3] and see(4, 6, 4, 0, 0, True) == [0, 1, 2, 3, 4, 5]
    assert see(1, 9, 4, 0, 3, True) == [0, 1, 2] and see(3, 9, 4, 0, 3, True) == [0, 1, 2, 3, 4, 5, 6]
    assert see(5, 9, 1, 2, 0, True) == [4, 5] and see(5, 9, 0, 2, 0, True) == [4, 5, 6]
    assert see(-1, 4, 0, 0, 0, True) == [] and see(-1, 4, 0, 0, 0, False) == [0, 1, 2, 3]
    assert see(9, 4, 1, 0, 0, True) == [0, 1, 2, 3] and see(9, 4, 1, 3, 0, True) == []


def test_plain_attention_leaves_out_what_is_not_seen():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((2, 4, 8)), rng.standard_normal((6, 2, 8)), rng.standard_normal((6, 2, 8))
    ok = np.array([[1, 1, 0, 0, 1, 0], [0] * 6], bool)
    out, avg, _, _ = R.attention(q, k, v, ok, 0.3)
    js = [0, 1, 4]
    for h in range(4):
        s = q[0, h] @ k[js, h // 2].T * 0.3
        p = np.exp(s) / np.exp(s).sum()
        assert np.allclose(out[0, h], p @ v[js, h // 2])
    assert np.isclose(avg[0].sum(), 1) and not avg[0][~ok[0]].any() and not out[1].any() and not avg[1].any()
    k[2], v[3] = np.nan, np.inf
    assert np.array_equal(R.attention(q, k, v, ok, 0.3)[0], out)


def test_plain_places():
    seq, idx, ln = R.index_of([1, 3, 3, 5], [4, 0, 70], None, 6, 64)
    assert seq.tolist() == [-1, 0, 0, 2, 2, -1] and idx[1:5].tolist() == [2, 3, 62, 63] and ln[3] == 64
    page, row = R.place(seq, idx, ln, np.array([[5, -1], [0, 0], [7, 9]]), 32, 9)
    assert page.tolist() == [-1, 5, 5, -1, -1, -1] and row[1:3].tolist() == [2, 3]


# ------------------------------------------------------------------ the plans' whole numbers

PLAN = """
#include "%s"
extern "C" void span(int lo, int hi, int n, int* out) { const d2c::PgSpan s = d2c::pg_span(lo, hi, n); out[0] = s.row0; out[1] = s.m; }
extern "C" int whole(int tiles, float share) { return d2c::pg_whole(tiles, share); }
extern "C" int backwards(int wg, int count) { return d2c::pg_backwards(wg, count); }
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """csrc/pg_plan.h, which the kernels use, compiled for the host; overflows of whole numbers end the program."""
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    at = tmp_path_factory.mktemp("plan")
    (at / "plan.cpp").write_text(PLAN % os.path.join(ROOT, "paper_2509_23094_amd", "csrc", "pg_plan.h"))
    subprocess.run(["g++", "-std=c++17", "-O1", "-ftrapv", "-shared", "-fPIC", "-o", str(at / "plan.so"), str(at / "plan.cpp")], check=True)
    return ctypes.CDLL(str(at / "plan.so"))


def test_rows_between_any_two_starts(plan):
    edges = sorted({0, 1, 5, 19, 20, 21, 40, 1 << 20, (1 << 20) + 1, 1 << 30, (1 << 31) - 2, (1 << 31) - 1} | {-1, -5, -(1 << 30), 1 - (1 << 31), -(1 << 31)})
    out = (ctypes.c_int * 2)()
    for n, lo, hi in itertools.product((1, 20, 120, 1 << 20), edges, edges):
        plan.span(lo, hi, n, out)
        row0, end = min(max(lo, 0), n), min(max(hi, 0), n)
        assert list(out) == [row0, max(0, end - row0)], (lo, hi, n)


def test_no_more_tiles_stay_whole_than_there_are(plan):
    """Tiles of kernels for few and many queries that fill whole rounds exactly: the share as make_plan forms it, in fp32."""
    for workgroups, rounds in itertools.product((256, 512), (1, 2, 3, 2047, 2048, 2049, 4096, 40000, 65536)):
        tiles = workgroups * rounds
        share = np.float32(np.float32(tiles) / np.float32(tiles) + np.float32(1e-6))
        assert plan.whole(tiles, ctypes.c_float(share)) == tiles
        if rounds <= 2048:           # (from there on a part of a round is less than a millionth of all)
            less = tiles + workgroups // 2
            share = np.float32(np.float32(tiles) / np.float32(less) + np.float32(1e-6))
            assert tiles <= plan.whole(less, ctypes.c_float(share)) <= tiles + 2
    assert plan.whole(0, ctypes.c_float(1.000001)) == 0


@pytest.mark.parametrize("count", [1, 7, 8, 9, 15, 31, 32, 64, 100, 128, 250, 255, 256, 257, 304])
def test_a_round_that_goes_backwards_leaves_out_no_workgroup(plan, count):
    order = [plan.backwards(wg, count) for wg in range(count)]
    assert sorted(order) == list(range(count))
    assert all(at % 8 == wg % 8 for wg, at in enumerate(order))                  # on its XCD
    if count % 8 == 0:
        assert order[:8] == list(range(count - 8, count))
