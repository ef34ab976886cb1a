"""Products with matrices in 4 bits where nothing may be lost: results that fp32 holds exactly, single inputs of 24 bits, what random rows
are off by on average; inputs and scales at the ends of their ranges."""
import numpy as np
import pytest

import paper_2302_07863_amd as pkg
from tests.hipmem import DeviceArray
from tests.rows import BF16, F16, F32, U32, Rows, normed, pack, scale_words, scales_of, unpack, weights

pytestmark = pytest.mark.gpu


def matrix(rng, n, k, group, zeros, values, scale_dtype=F16):
    """A matrix whose scales are among `values`."""
    groups = -(-k // group)
    codes = rng.integers(0, 256, (n, (k + 1) // 2)).astype(np.uint8)
    scales = scale_words(rng.choice(values, (n, groups)), scale_dtype)
    z = rng.integers(0, 16, (n, groups)).astype(np.uint8) if zeros else None
    return pkg.Quant(n, k, group, codes, scales, scale_dtype, z), weights(codes, scales_of(scales, scale_dtype), z, k, group)


def multiply(q, words, x_dtype, n, **kw):
    rows, k = words.shape
    x, y = Rows(words), Rows(np.zeros((rows, n), np.float32))
    q.matmul(x.ptr, x_dtype, rows, y.ptr, F32, **kw)
    return y.get().astype(np.float64)


# narrow and wide matrices of few and many rows: rows straight from memory, staged whole, in chunks, in blocks
SHAPES = [(1, 40, 512), (1, 5000, 512), (3, 49, 1000), (11, 4200, 136), (16, 130, 8328), (17, 80, 512), (22, 346, 32), (32, 33, 2500), (32, 2048, 1030), (45, 40, 1536),
          (70, 80, 257), (509, 1601, 264), (449, 1700, 2056)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,n,k", SHAPES)
@pytest.mark.parametrize("x_dtype", [F32, BF16, F16])
def test_sums_that_fp32_holds_are_exact(x_dtype, rows, n, k, group):
    """Whole numbers times codes times scales of 1/2 and 1/4 (fp32 rows: 1/2 alone).  A sum on the way to a group's is at most 31/16 of the group's inputs, in 16ths: 31 * 128 * 2047
    are less than 2^23.  One of scaled groups is at most 15/16 of all inputs times 1/2, in 64ths (32nds): 30 * 264 * 2047, 30 * 2000 * 255 and 15 * 4 * 2^18 are less than 2^24.
    18 bits are three parts of 8."""
    rng = np.random.default_rng(rows * 1000 + k + group)
    q, w = matrix(rng, n, k, group, rows % 2 == 1, [0.5, -0.5] if x_dtype == F32 else [0.5, -0.25])
    x = np.zeros((rows, k))
    for row in x:
        at = rng.choice(k, min(k, {F32: 4, BF16: 2000, F16: 264}[x_dtype]), replace=False)
        if x_dtype == F32:
            row[at] = rng.choice([-1, 1], len(at)) * (rng.integers(1 << 16, 1 << 17, len(at)) * 2 + 1)
        else:
            most = 255 if x_dtype == BF16 else 2047
            row[at] = rng.integers(-most, most + 1, len(at))
    words = pack(x, x_dtype)
    assert np.array_equal(unpack(words, x_dtype), x)
    assert np.array_equal(multiply(q, words, x_dtype, n), x @ w.T)


def singles(rng, rows, k):
    """Rows of one input of 24 bits each."""
    x = np.zeros((rows, k))
    x[np.arange(rows), rng.integers(0, k, rows)] = rng.choice([-1.0, 1.0], rows) * (rng.integers(1 << 22, 1 << 23, rows) * 2 + 1) * 2.0 ** rng.integers(-40, 10, rows)
    return x


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,n,k", SHAPES)
def test_single_inputs_of_24_bits(rows, n, k, group):
    """Each part's products are exact, so is the sum of the lower two; their sum with the first is rounded once.  Behind a norm: of the mean three roundings (halved by the
    root), the root, its inverse, two products with the scale, input times gain, the sum: 7.5 half steps."""
    rng = np.random.default_rng(rows + k + group)
    q, w = matrix(rng, n, k, group, rows % 2 == 1, [0.5, -0.25])
    words = pack(singles(rng, rows, k), F32)
    want = unpack(words, F32) @ w.T
    assert np.all(np.abs(multiply(q, words, F32, n) - want) <= U32 * np.abs(want))
    gain = (1.0 + 0.2 * rng.standard_normal(k)).astype(np.float32)
    g = DeviceArray(gain)
    got = multiply(q, words, F32, n, gain=g.ptr.value, eps=1e-6, scale=0.5)
    want = 0.5 * (normed(unpack(words, F32), gain.astype(np.float64), float(np.float32(1e-6))) @ w.T)
    assert np.all(np.abs(got - want) <= 8 * U32 * np.abs(want))


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("rows,n,k", SHAPES + [(3, 24, 40000)])
@pytest.mark.parametrize("x_dtype", [F32, BF16, F16])
def test_random_rows_on_average(x_dtype, rows, n, k, group, norm):
    """Within a group of G inputs of size 1 a sum is some 1.5 sqrt(G), with at most 66 roundings a step of 32 inputs (one a product): off by 1.5 sqrt(G) sqrt(66 G / 32) half steps, of
    a result of 0.29 sqrt(G) (codes less 8, over 16) or more: 84 for 128.  Some 320 scaled groups, then parts, waves and the norm: sqrt(340) more.  (Measured: 5 at most;
    inputs or weights rounded to 8 bits: some 2^14.)"""
    rng = np.random.default_rng(rows + k + group + x_dtype)
    q, w = matrix(rng, n, k, group, rows % 2 == 1, [0.01, 0.0173, -0.0049])
    words = pack(rng.standard_normal((rows, k)), x_dtype)
    gain = (1.0 + 0.2 * rng.standard_normal(k)).astype(np.float32) if norm else None
    g = DeviceArray(gain) if norm else None
    got = multiply(q, words, x_dtype, n, gain=g.ptr.value if norm else None, eps=1e-6)
    want = normed(unpack(words, x_dtype), None if gain is None else gain.astype(np.float64), float(np.float32(1e-6))) @ w.T
    off = np.sqrt(np.mean((got - want) ** 2) / np.mean(want ** 2)) / U32
    assert off <= 105


@pytest.mark.parametrize("rows,n,k", [(2, 48, 256), (7, 48, 250), (20, 300, 264), (509, 1601, 264)])
def test_subnormal_inputs(rows, n, k):
    """bf16 rows to their last bit; of fp32 rows each part is a multiple of 2^-133, so that an input is off by half of that.  The products, multiples of 2^-137, are exact."""
    rng = np.random.default_rng(rows)
    q, w = matrix(rng, n, k, 64, True, [1024.0])
    for e in (-149, -143, -137, -133, -130, -127, -126, -120, -112, -100):
        x = np.zeros((rows, k))
        at = np.arange(rows), rng.integers(0, k, rows)
        x[at] = 2.0 ** e * (1 + rng.integers(0, 1 << 23, rows) / (1 << 23))
        for x_dtype in (F32, BF16):
            words = pack(x, x_dtype)
            xv = unpack(words, x_dtype)
            want = 2.0 ** 60 * (xv @ w.T)
            tol = U32 * np.abs(want) + (2.0 ** 60 * 2.0 ** -134 * np.abs(w.T[at[1]]) if x_dtype == F32 else 0.0)
            assert np.all(np.abs(multiply(q, words, x_dtype, n, scale=2.0 ** 60) - want) <= tol), (e, x_dtype)


@pytest.mark.parametrize("top", [2.0 ** -125, 2.0 ** -110, 1.0, 2.0 ** 100, 2.0 ** 120])
@pytest.mark.parametrize("rows,n,k", [(2, 48, 256), (7, 48, 250), (509, 1601, 264)])
def test_scales_at_the_ends_of_bf16(rows, n, k, top):
    """One power of two a row, a factor beside the matrix: codes, scales and their sums are exact, the factor's product is rounded once."""
    rng = np.random.default_rng(rows)
    q, w = matrix(rng, n, k, 64, True, top * np.array([1.0, -1.59375, 0.0078125 * 1.0078125]), BF16)
    for x_dtype in (F32, BF16):
        x = np.zeros((rows, k))
        x[np.arange(rows), rng.integers(0, k, rows)] = 2.0 ** rng.integers(-6, 0, rows) / top
        words = pack(x, x_dtype)
        assert np.array_equal(unpack(words, x_dtype), x)
        want = float(np.float32(0.7)) * (x @ w.T)
        assert np.all(np.abs(multiply(q, words, x_dtype, n, scale=0.7) - want) <= 1.001 * U32 * np.abs(want))


@pytest.mark.parametrize("rows,n,k", SHAPES)
@pytest.mark.parametrize("x_dtype", [F32, BF16, F16])
def test_rows_with_an_infinite_input(x_dtype, rows, n, k):
    """NaN throughout, but for fp16 rows in blocks: there infinity times a code, NaN where that is none."""
    rng = np.random.default_rng(rows + k)
    q, w = matrix(rng, n, k, 64, True, [0.5, -0.25])
    x = rng.integers(-3, 4, (rows, k)).astype(np.float64)
    bad = np.zeros(rows, bool)
    bad[rng.integers(0, rows, (rows + 2) // 3)] = True
    at = rng.integers(0, k, rows)
    x[bad, at[bad]] = np.inf
    words = pack(x, x_dtype)
    blocks = x_dtype == F16 and rows > 32 and k % 8 == 0 and -(-n // 128) * -(-rows // 64) >= 96
    with np.errstate(invalid="ignore"):
        far = np.inf * w.T[at[bad]] if blocks else np.full((int(bad.sum()), n), np.nan)
    got = multiply(q, words, x_dtype, n)
    assert np.array_equal(got[bad], far, equal_nan=True)
    assert np.array_equal(got[~bad], x[~bad] @ w.T)
    if x_dtype == F32:
        huge = DeviceArray(np.ones(k, np.float32))
        got = multiply(q, pack(np.where(np.isinf(x), 2.0 ** 70, x), F32), F32, n, gain=huge.ptr.value, eps=1e-6)
        assert np.all(got[bad] == 0) and np.all(np.isfinite(got))
