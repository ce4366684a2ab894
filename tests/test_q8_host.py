"""CPU-side checks of the 8-bit operators: the header against the library and the binding, refusals that need no GPU, and what the plain
64-bit forms (which the GPU tests compare with) promise."""
import ctypes
import os
import re

import numpy as np
import pytest

import q8_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2509_23094_amd", "libd2c.so")
built = pytest.mark.skipif(not os.path.exists(LIB), reason="libd2c.so not built (run __graft_entry__.build())")


@built
def test_header_library_and_binding_agree():
    from paper_2509_23094_amd import binding as B
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "d2c_q8.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(d2c_q8_[a-z_0-9]+)\s*\(", text)))
    assert names == sorted(B.Q8_EXPORTS)
    for n in names:
        assert getattr(B._lib, n) is not None
    for n in ("update", "attention", "read", "pack", "linear", "weigh", "evict"):
        assert hasattr(B.Q8Context, "d2c_q8_" + n)
    assert ctypes.sizeof(B.d2c_q8_seq) == 10 * 8 + 8 and ctypes.sizeof(B.d2c_q8_dims) == 36


@built
@pytest.mark.parametrize("field,value,code", [
    ("n_heads", 0, -1), ("n_kv_heads", 0, -1), ("n_kv_heads", 3, -1), ("n_heads", 2048, -1), ("head_dim", 96, -4), ("dtype", 2, -1),
    ("max_seq", -1, -1), ("max_seq", (1 << 24) + 1, -1), ("max_rows", -1, -1), ("max_rows", (1 << 16) + 1, -1), ("max_batch", 257, -1),
    ("max_k", (1 << 16) + 1, -1), ("max_n", -5, -1)])
def test_init_refuses(field, value, code):
    from paper_2509_23094_amd import binding as B
    d = B.d2c_q8_dims(4, 4, 64, B.D2C_BF16, 128, 16, 1, 0, 0)
    setattr(d, field, value)
    out = ctypes.c_void_p()
    assert B._lib.d2c_q8_init(ctypes.byref(d), ctypes.byref(out)) == code
    assert B._lib.d2c_q8_last_error(None) and not out


@built
def test_null_arguments_are_refused():
    from paper_2509_23094_amd import binding as B
    lib, out = B._lib, ctypes.c_void_p()
    assert lib.d2c_q8_init(None, ctypes.byref(out)) == B.D2C_EINVAL
    assert lib.d2c_q8_destroy(None) == B.D2C_OK
    assert lib.d2c_q8_workspace_bytes(None) == 0
    assert lib.d2c_q8_update(None, None, 1, None) == B.D2C_EINVAL
    assert lib.d2c_q8_attention(None, None, 1, None) == B.D2C_EINVAL
    assert lib.d2c_q8_read(None, None, 1, None, 1, None, None, None) == B.D2C_EINVAL
    assert lib.d2c_q8_pack(None, None, 1, 8, None, None, None) == B.D2C_EINVAL
    assert lib.d2c_q8_linear(None, None, 1, None, None, 1, 8, None, None) == B.D2C_EINVAL
    assert lib.d2c_q8_weigh(None, None, 1, 1, None, None) == B.D2C_EINVAL
    assert lib.d2c_q8_evict(None, None, 1, None, None, 1, None, None, None, None) == B.D2C_EINVAL
    assert lib.d2c_q8_cache_size(None, 1, None, None) == B.D2C_EINVAL
    assert lib.d2c_q8_weight_bytes(17, 65) == 32 * 128 and lib.d2c_q8_weight_bytes(0, 8) == 0


@built
def test_binding_refuses_tensors_of_another_kind():
    import torch
    from paper_2509_23094_amd import binding as B

    class Ctx:                                   # geometry of a handle, no device needed
        torch_dtype, device, d_kv, d_q, geo = torch.bfloat16, -1, 128, 256, (2, 64, -1)

    class Cache:
        c, geo = B.d2c_q8_cache(), (2, 64, -1)

        def holds(self, L):
            pass

    def batch(**kw):
        return B.Q8Batch(Ctx, [B.Q8Seq(Cache(), 64, 3, **kw)])

    batch(q=torch.zeros(3, 256, dtype=torch.bfloat16))
    for bad in (dict(q=torch.zeros(3, 256)), dict(q=torch.zeros(2, 256, dtype=torch.bfloat16)),
                dict(new_k=torch.zeros(3, 64, dtype=torch.bfloat16)), dict(idx=torch.zeros(3, dtype=torch.int64)),
                dict(attn_avg=torch.zeros(3, 63)), dict(out=torch.zeros(256, 3, dtype=torch.bfloat16).t())):
        with pytest.raises(B.D2CError) as e:
            batch(**bad)
        assert e.value.code == B.D2C_EINVAL
    Cache.geo = (2, 128, -1)                     # a cache of another geometry
    with pytest.raises(B.D2CError) as e:
        batch(q=torch.zeros(3, 256, dtype=torch.bfloat16))
    assert e.value.code == B.D2C_ESHAPE


# ---------------------------------------------------------------------- the plain forms

def test_codes_are_within_half_a_step_and_ties_go_to_even():
    rng = np.random.default_rng(0)
    x = rng.standard_normal(4000).astype(np.float32).astype(np.float64)
    s = R.scale(np.abs(x).max())
    assert np.abs(R.code(x, s) * s - x).max() <= s / 2 * (1 + 1e-12)
    assert list(R.code(np.array([0.5, 1.5, 2.5, -0.5, -1.5, 300.0, np.inf, -np.inf, np.nan]), 1.0)) == [0, 2, 2, 0, -2, 127, 127, -127, 0]
    assert R.scale(2.0 ** -101) == 0 and R.scale(0.0) == 0 and R.code(1e-40, 0.0) == 0


def test_many_small_growths_do_not_carry_a_value_away():
    """A row that is never refreshed beside one that grows by a little 600 times: each growth of the scale is a factor of 1.25 or more
    and rounds by half a step, so the whole drift stays below half a last step / (1 - 1/1.25) = 2.5 of them."""
    t = R.Tensor8(64, 1, 16)
    rng = np.random.default_rng(1)
    first = rng.standard_normal((64, 1, 16))
    t.update(np.arange(64), first, 64)
    size = np.abs(first).max()
    for _ in range(600):
        size *= 1.01
        t.update([7], np.full((1, 1, 16), size), 64)
    others = np.delete(np.arange(64), 7)
    assert np.abs(t.values()[others] - first[others]).max() <= 2.5 * t.scale[0, 0] + 1e-9
    assert abs(t.values()[7, 0, 0] - size) <= t.scale[0, 0] / 2 + 1e-9


def test_a_refreshed_block_takes_the_scale_of_its_rows_again():
    t = R.Tensor8(70, 2, 16)
    t.update(np.arange(70), np.full((70, 2, 16), 8.0), 70)
    t.update(np.arange(64, 70), np.full((6, 2, 16), 0.5), 70)              # all rows below L of the second block
    assert (t.scale[1] == R.scale(0.5)).all() and (t.scale[0] == R.scale(8.0)).all()
    t.update(np.arange(63), np.full((63, 2, 16), 0.5), 70)                 # one row of the first stays
    assert (t.scale[0] == R.scale(8.0)).all()


def test_byte_order_is_the_documented_one():
    rng = np.random.default_rng(2)
    heads, D, nb = 3, 64, 2
    c = rng.integers(-127, 128, size=(nb * 64, heads, D))
    k, v = R.k_bytes(c), R.v_bytes(c)
    for _ in range(200):
        b, h, t, d = rng.integers(nb), rng.integers(heads), rng.integers(64), rng.integers(D)
        base = (b * heads + h) * 64 * D
        assert k[base + d // 16 * 1024 + t * 16 + d % 16] == c[b * 64 + t, h, d] + 128
        assert v[base + t // 4 * 4 * D + d * 4 + t % 4] == c[b * 64 + t, h, d] + 128


def test_keep_orders_protected_weight_and_index():
    assert list(R.keep([5, 9, 5, 1], None, 2)) == [0, 1]
    assert list(R.keep([5, 9, 5, 1], [0, 0, 0, 1], 2)) == [1, 3]
    assert list(R.keep([5, 9, 5, 1], [1, 0, 1, 1], 2)) == [0, 2]
    assert list(R.keep([-3, 0, -1], None, 2)) == [0, 1]


@built
def test_weight_bytes_of_the_largest_sizes():
    from paper_2509_23094_amd import binding as B
    big = (1 << 31) - 1
    for N, K in ((big, 8), (1, big), (big, big), (1 << 20, 1 << 16)):
        assert B._lib.d2c_q8_weight_bytes(N, K) == -(-N // 16) * 16 * (-(-K // 64) * 64)


@built
def test_init_errors_of_two_threads_keep_apart():
    """The text of a failed d2c_q8_init belongs to the thread that called it."""
    import threading
    from paper_2509_23094_amd import binding as B

    def fail(field, value):
        d, out = B.d2c_q8_dims(4, 4, 64, B.D2C_BF16, 128, 16, 1, 0, 0), ctypes.c_void_p()
        setattr(d, field, value)
        assert B._lib.d2c_q8_init(ctypes.byref(d), ctypes.byref(out)) < 0
        return B._lib.d2c_q8_last_error(None)

    mine, seen = fail("head_dim", 96), []
    assert b"head_dim" in mine
    other = threading.Thread(target=lambda: seen.append((B._lib.d2c_q8_last_error(None), fail("dtype", 7))))
    other.start()
    other.join()
    assert seen[0][0] == b"" and b"dtype" in seen[0][1]
    assert B._lib.d2c_q8_last_error(None) == mine


# ---------------------------------------------------------------------- the product's kernels and the sizes that test them

def _linear_kernel(m, N, K):
    from paper_2509_23094_amd import binding as B
    p = B.d2c_q8_plan_linear(m, N, K)
    return (p["kernel"], p["row_tiles"], p["col_tiles"], p["splits"] > 1), p


@built
def test_every_kernel_of_the_product_has_a_tested_size():
    """The sizes that the GPU tests multiply reach the kernels they are listed for, and sizes all over the range reach no other."""
    from q8_sizes import LINEAR
    for key, sizes in LINEAR.items():
        for size in sizes:
            assert _linear_kernel(*size)[0] == key, size
    rng = np.random.default_rng(3)
    sizes = np.exp(rng.uniform(0, 1, (60000, 3)) * np.log([4096, 65536, 8192])).astype(np.int64)
    seen = {_linear_kernel(int(m), int(n), 8 * int(k))[0] for m, n, k in sizes}
    assert seen <= set(LINEAR), seen - set(LINEAR)


@built
def test_linear_plan_covers_the_contraction_and_fits_its_parts():
    rng = np.random.default_rng(4)
    for m, n, k in np.exp(rng.uniform(0, 1, (20000, 3)) * np.log([65536, 1 << 20, 8192])).astype(np.int64):
        m, n, k = int(m), int(n), 8 * int(k)
        (kernel, mt, nt, split), p = _linear_kernel(m, n, k)
        steps = -(-k // 64)
        units = -(-steps // 4) if kernel == 2 else steps                  # what a split takes whole numbers of
        per = -(-units // p["splits"])
        assert p["splits"] >= 1 and per * (p["splits"] - 1) < units, (m, n, k, p)          # none empty
        assert not split or 4 * p["splits"] * m * n <= 32 << 20, (m, n, k, p)
        assert p["waves"] in (8, 16)
        if kernel == 0:
            assert m <= 16 and k <= 2048 and not split
        if kernel == 1:
            assert mt == -(-m // 16) <= 2


@built
def test_linear_plan_rejects_bad_arguments():
    from paper_2509_23094_amd import binding as B
    shape = (ctypes.c_int32 * 5)()
    for m, n, k in ((0, 16, 16), (1, 0, 16), (1, 16, 0), ((1 << 16) + 1, 16, 16), (1, (1 << 20) + 1, 16), (1, 16, (1 << 16) + 1)):
        assert B._lib.d2c_q8_plan_linear(m, n, k, shape) == B.D2C_EINVAL
    assert B._lib.d2c_q8_plan_linear(1, 16, 16, None) == B.D2C_EINVAL


def test_the_product_in_torch_is_the_one_in_numpy():
    import torch
    from q8_sizes import linear
    g = torch.Generator().manual_seed(0)
    a, w = torch.randn((9, 72), generator=g), 0.02 * torch.randn((33, 72), generator=g)
    a[1], a[2, 3], a[4, 5], w[6, 7], a[7] = 0, float("nan"), float("-inf"), float("inf"), 2.0 ** -101
    want, _, sw = R.linear(a.numpy(), w.numpy())
    got, s = linear(a, w)
    assert np.array_equal(got.numpy(), want, equal_nan=True) and np.array_equal(s.numpy(), sw, equal_nan=True)
