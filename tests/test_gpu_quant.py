"""Products with matrices in 4 bits against the definition in 64 bits: types, groups, ragged sizes, strides, norms, streams, graphs."""
import ctypes as C

import numpy as np
import pytest

import paper_2302_07863_amd as pkg
from paper_2302_07863_amd import binding as b
from tests.hipmem import DeviceArray, hip
from tests.rows import BF16, F16, F32, HALF_STEP, TINY, U32, Graph, Rows, Stream, close, normed, pack, scale_words, scales_of, unpack, weights

pytestmark = pytest.mark.gpu


def matrix(rng, n, k, group, zeros=False, scale_dtype=F16):
    groups = -(-k // group)
    codes = rng.integers(0, 256, (n, (k + 1) // 2)).astype(np.uint8)
    scales = scale_words(0.01 * (0.5 + rng.random((n, groups))) * rng.choice([-1.0, 1.0], (n, groups)), scale_dtype)
    z = rng.integers(0, 16, (n, groups)).astype(np.uint8) if zeros else None
    return codes, scales, z, pkg.Quant(n, k, group, codes, scales, scale_dtype, z), weights(codes, scales_of(scales, scale_dtype), z, k, group), \
        np.abs(scales_of(scales, scale_dtype))[:, np.arange(k) // group]


def tolerance(xh, scale, y, y_dtype):
    """A step of 32 inputs adds two products of at most 2 * 16 * scale * |x| each (in up to three parts, whose sizes add up to |x|), into a
    sum that never holds more than all of them: at most 6 roundings a step if the matrix cores round once an instruction,
    33 times as many if after every product.  Groups, waves and the norm add a rounding of the sum each."""
    most = 64.0 * np.abs(xh) @ scale.T
    steps = -(-xh.shape[1] // 32)
    return (6 * 33 + 2 * steps + 16) * U32 * most + HALF_STEP[y_dtype] * np.abs(y) + TINY[y_dtype]


def check(rng, n, k, group, rows, x_dtype, y_dtype, zeros=False, scale_dtype=F16, norm=False, scale=1.0, x_stride=None, y_stride=None, first=0,
          stream=None, mean=0.0):
    *_, q, w, s = matrix(rng, n, k, group, zeros, scale_dtype)
    words = pack(rng.standard_normal((rows, k)) + mean, x_dtype)
    x = Rows(words, x_stride, first)
    y = Rows(pack(np.zeros((rows, n)), y_dtype), y_stride, first)
    gain = (1.0 + 0.2 * rng.standard_normal(k)).astype(np.float32) if norm else None
    g = DeviceArray(gain) if norm else None
    q.matmul(x.ptr, x_dtype, rows, y.ptr, y_dtype, x.stride, y.stride, g.ptr.value if norm else None, 1e-6, scale, stream)
    xh = normed(unpack(words, x_dtype), None if gain is None else gain.astype(np.float64), 1e-6)
    want = scale * (xh @ w.T)
    got = unpack(y.get(), y_dtype)
    close(got, want, abs(scale) * tolerance(xh, s, want / scale, y_dtype))


@pytest.mark.parametrize("x_dtype", [F32, BF16, F16])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows", [1, 2, 11, 16, 17, 32, 33, 70])
def test_rows_and_groups(x_dtype, group, rows):
    rng = np.random.default_rng(rows * 1000 + group + x_dtype)
    check(rng, 80, 512, group, rows, x_dtype, x_dtype, zeros=group == 64, scale_dtype=BF16 if rows % 2 else F16)


@pytest.mark.parametrize("n,k", [(1, 1), (1, 128), (16, 2), (15, 33), (17, 31), (33, 127), (47, 129), (100, 257), (5, 1000), (250, 1153), (2049, 96)])
@pytest.mark.parametrize("x_dtype,y_dtype", [(F32, F32), (BF16, F32), (F16, BF16), (BF16, F16)])
def test_ragged_sizes(n, k, x_dtype, y_dtype):
    rng = np.random.default_rng(n * 7 + k)
    for rows, group, zeros in ((1, 32, True), (3, 128, False), (19, 64, True)):
        check(rng, n, k, group, rows, x_dtype, y_dtype, zeros=zeros)


@pytest.mark.parametrize("x_dtype", [F32, BF16, F16])
def test_norm_in_front(x_dtype):
    rng = np.random.default_rng(5 + x_dtype)
    for rows, n, k in ((1, 64, 512), (1, 31, 77), (4, 48, 1024), (29, 20, 640), (40, 33, 384)):
        check(rng, n, k, 64, rows, x_dtype, F32, norm=True, scale=0.7, mean=0.5)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_strides_and_addresses(dtype):
    """Rows apart, rows whose addresses are multiples of their type alone, nothing written beside them."""
    rng = np.random.default_rng(9)
    for rows, x_stride, y_stride, first in ((5, 300, 90, 0), (5, 301, 91, 1), (18, 257, 83, 3), (1, 0, 0, 1)):
        check(rng, 83, 257, 32, rows, dtype, dtype, x_stride=x_stride, y_stride=y_stride, first=first)
    # one row of x for all rows of y
    *_, q, w, s = matrix(rng, 40, 96, 32)
    x, y = Rows(pack(rng.standard_normal((1, 96)), dtype)), Rows(pack(np.zeros((6, 40)), F32))
    q.matmul(x.ptr, dtype, 6, y.ptr, F32, x_stride=0)
    got = y.get()
    assert np.all(got == got[0])


def test_values_far_from_zero_lose_nothing():
    """Inputs around 50 (what a code's offset adds is taken off step by step), inputs of very different sizes in a row, subnormal ones."""
    rng = np.random.default_rng(10)
    check(rng, 64, 4096, 128, 2, F32, F32, mean=50.0)
    codes, scales, z, q, w, s = matrix(rng, 64, 256, 32, True)
    x = rng.standard_normal((3, 256)) * 10.0 ** rng.integers(-30, 20, (3, 256))
    x[2] = 1e-40
    for dtype in (F32, BF16):
        words = pack(x, dtype)
        xd, y = Rows(words), Rows(pack(np.zeros((3, 64)), F32))
        q.matmul(xd.ptr, dtype, 3, y.ptr, F32)
        xv = unpack(words, dtype)
        want = xv @ w.T
        close(y.get()[:2], want[:2], tolerance(xv, s, want, F32)[:2])


def test_long_rows():
    rng = np.random.default_rng(11)
    check(rng, 24, 40000, 128, 3, BF16, F32, zeros=True)
    check(rng, 7000, 64, 32, 2, F16, F16)


def test_a_row_that_is_not_finite_stays_alone():
    rng = np.random.default_rng(12)
    *_, q, w, s = matrix(rng, 50, 200, 32)
    for dtype in (F32, BF16, F16):
        x = rng.standard_normal((4, 200))
        clean = Rows(pack(x, dtype))
        y0, y1 = Rows(pack(np.zeros((4, 50)), F32)), Rows(pack(np.zeros((4, 50)), F32))
        q.matmul(clean.ptr, dtype, 4, y0.ptr, F32)
        x[1, 17], x[2, 199] = np.inf, np.nan
        dirty = Rows(pack(x, dtype))
        q.matmul(dirty.ptr, dtype, 4, y1.ptr, F32)
        a, c = y0.get(), y1.get()
        assert np.array_equal(a[[0, 3]], c[[0, 3]])
        assert not np.any(np.isfinite(c[1:3]))


def test_rows_do_not_depend_on_their_company():
    """A row's result is the same bits alone and in any block that runs through the same kernel."""
    rng = np.random.default_rng(13)
    *_, q, w, s = matrix(rng, 96, 640, 64, True)
    x = pack(rng.standard_normal((16, 640)), BF16)
    whole = Rows(pack(np.zeros((16, 96)), F32))
    xd = Rows(x)
    q.matmul(xd.ptr, BF16, 16, whole.ptr, F32)
    again = Rows(pack(np.zeros((16, 96)), F32))
    q.matmul(xd.ptr, BF16, 16, again.ptr, F32)
    assert np.array_equal(whole.get(), again.get())
    part = Rows(pack(np.zeros((9, 96)), F32))
    q.matmul(xd.ptr + 5 * 640 * 2, BF16, 9, part.ptr, F32)
    assert np.array_equal(whole.get()[5:14], part.get())


def test_from_device_memory_and_rounded_from_fp32():
    rng = np.random.default_rng(14)
    w = (0.02 * rng.standard_normal((48, 200))).astype(np.float32)
    x = Rows(pack(rng.standard_normal((3, 200)), F32))
    for zeros in (False, True):
        codes, scales, z = pkg.quant_round(w, 64, BF16, zeros)
        devs = [DeviceArray(a) for a in (codes, scales)] + ([DeviceArray(z)] if zeros else [])
        a = pkg.Quant(48, 200, 64, codes, scales, BF16, z)
        c = pkg.Quant(48, 200, 64, devs[0].ptr.value, devs[1].ptr.value, BF16, devs[2].ptr.value if zeros else None)
        ya, yc = Rows(pack(np.zeros((3, 48)), F32)), Rows(pack(np.zeros((3, 48)), F32))
        a.matmul(x.ptr, F32, 3, ya.ptr, F32)
        c.matmul(x.ptr, F32, 3, yc.ptr, F32)
        assert np.array_equal(ya.get(), yc.get())
        wq = weights(codes, scales_of(scales, BF16), z, 200, 64)
        s = np.abs(scales_of(scales, BF16))[:, np.arange(200) // 64]
        xv = unpack(x.get(), F32)
        close(ya.get(), xv @ wq.T, tolerance(xv, s, xv @ wq.T, F32))


def test_streams_and_captured_launches():
    rng = np.random.default_rng(15)
    *_, q, w, s = matrix(rng, 128, 512, 128, True)
    xs = [pack(rng.standard_normal((7, 512)), BF16) for _ in range(4)]
    x = Rows(xs[0])
    stream = Stream()
    y, eager = Rows(pack(np.zeros((7, 128)), F32)), Rows(pack(np.zeros((7, 128)), F32))
    graph = Graph(stream, lambda st: q.matmul(x.ptr, BF16, 7, y.ptr, F32, stream=st))
    for words in xs:
        stream.sync()
        assert hip().hipMemcpy(x.dev.ptr, np.ascontiguousarray(words).ctypes.data, words.nbytes, 1) == 0
        graph.replay()
        stream.sync()
        q.matmul(x.ptr, BF16, 7, eager.ptr, F32)
        x.host[:words.size] = words.ravel()
        assert np.array_equal(y.get(), eager.get())


def test_refusals_leave_y_alone():
    rng = np.random.default_rng(16)
    *_, q, w, s = matrix(rng, 40, 96, 32)
    x, y = Rows(pack(rng.standard_normal((2, 96)), F32)), Rows(pack(np.zeros((2, 40)), F32))
    for kw in (dict(rows=0), dict(rows=-3), dict(x=None), dict(y=None), dict(x_dtype=3), dict(y_dtype=-1), dict(eps=-1.0), dict(eps=float("nan"))):
        a = dict(x=x.ptr, x_dtype=F32, rows=2, y=y.ptr, y_dtype=F32)
        a.update(kw)
        with pytest.raises(pkg.BildError) as e:
            q.matmul(**a)
        assert e.value.code == b.EINVAL
    assert np.all(y.get() == 0)
    codes, scales = np.zeros((4, 16), np.uint8), np.zeros((4, 1), np.uint16)
    with pytest.raises(pkg.BildError) as e:
        pkg.Quant(4, 32, 32, codes, scales, F16, np.full((4, 1), 16, np.uint8))
    assert e.value.code == b.EINVAL


@pytest.mark.parametrize("rows", [1, 5, 16])
@pytest.mark.parametrize("k", [8, 120, 136, 1000, 1160, 8328])
@pytest.mark.parametrize("x_dtype", [BF16, F16])
def test_narrow_matrices_with_any_number_of_inputs(rows, k, x_dtype):
    """Fewer feature tiles than compute units, few and many tiles of inputs, the last of them in part; rows that do not begin at 16 bytes."""
    rng = np.random.default_rng(k + rows)
    for n, group, zeros in ((16, 32, True), (49, 64, False), (130, 128, True)):
        check(rng, n, k, group, rows, x_dtype, F32 if rows == 5 else x_dtype, zeros=zeros, x_stride=k + 5, first=3)


@pytest.mark.parametrize("x_dtype", [BF16, F16])
@pytest.mark.parametrize("k", [72, 1032])
def test_nothing_behind_a_row_counts(x_dtype, k):
    """NaN in the elements behind a row's last one."""
    rng = np.random.default_rng(k)
    *_, q, w, s = matrix(rng, 40, k, 32)
    wide = np.full((3, k + 9), np.nan)
    wide[:, :k] = rng.standard_normal((3, k))
    x, y = DeviceArray(pack(wide, x_dtype)), Rows(np.zeros((3, 40), np.float32))
    q.matmul(x.ptr.value, x_dtype, 3, y.ptr, F32, x_stride=k + 9)
    xh = unpack(pack(wide[:, :k], x_dtype), x_dtype)
    want = xh @ w.T
    close(y.get().astype(np.float64), want, tolerance(xh, s, want, F32))


@pytest.mark.parametrize("x_dtype,y_dtype", [(BF16, BF16), (F16, F16), (BF16, F32), (F16, BF16)])
@pytest.mark.parametrize("n,k,rows", [(1600, 8, 500), (1601, 264, 509), (2050, 136, 470), (12300, 72, 33), (900, 1160, 833), (1700, 2056, 449)])
def test_many_rows_and_features(n, k, rows, x_dtype, y_dtype):
    """Blocks of rows and features, the last of either in part; inputs that end inside a tile, in one of the four that are multiplied at a time."""
    rng = np.random.default_rng(n + k + rows)
    group = {8: 32, 264: 64, 136: 128, 72: 64, 1160: 32, 2056: 128}[k]
    check(rng, n, k, group, rows, x_dtype, y_dtype, zeros=rows % 2 == 1, scale_dtype=F16, scale=0.5, x_stride=k + 8, y_stride=n + 3)


@pytest.mark.parametrize("x_dtype", [BF16, F16])
def test_blocks_keep_to_their_rows(x_dtype):
    """NaN behind the rows' inputs, an infinite row and an infinite scale of the last group: everything else stays finite."""
    rng = np.random.default_rng(5)
    n, k, rows, group = 1610, 200, 520, 64
    codes, scales, z, _, w, s = matrix(rng, n, k, group, True)
    scales[7, -1] = np.float16(np.inf).view(np.uint16)
    q = pkg.Quant(n, k, group, codes, scales, F16, z)
    wide = np.full((rows, k + 8), np.nan)
    wide[:, :k] = rng.standard_normal((rows, k))
    wide[100, :k] = np.inf
    x, y = DeviceArray(pack(wide, x_dtype)), Rows(np.zeros((rows, n), np.float32))
    q.matmul(x.ptr.value, x_dtype, rows, y.ptr, F32, x_stride=k + 8)
    got = y.get().astype(np.float64)
    assert not np.isfinite(got[100]).any() and not np.isfinite(got[:, 7]).any()
    keep_rows, keep = np.arange(rows) != 100, np.arange(n) != 7
    xh = unpack(pack(wide[keep_rows, :k], x_dtype), x_dtype)
    want = xh @ w[keep].T
    close(got[keep_rows][:, keep], want, tolerance(xh, s[keep], want, F32))


@pytest.mark.parametrize("rows,n,k", [(3, 200, 1000), (500, 1600, 264)])
def test_one_matrix_on_two_streams_and_in_two_graphs(rows, n, k):
    """Calls in flight at once on one handle, replayed with other rows: the bits of calls by themselves."""
    rng = np.random.default_rng(rows)
    *_, q, w, s = matrix(rng, n, k, 64, True)
    xs = [[pack(rng.standard_normal((rows, k)), BF16) for _ in range(2)] for _ in range(3)]
    x, streams = [Rows(v) for v in xs[0]], [Stream(), Stream()]
    y, alone = [Rows(np.zeros((rows, n), np.float32)) for _ in range(2)], Rows(np.zeros((rows, n), np.float32))
    graphs = [Graph(st, lambda h, i=i: q.matmul(x[i].ptr, BF16, rows, y[i].ptr, F32, stream=h)) for i, st in enumerate(streams)]
    for words in xs:
        for i in range(2):
            assert hip().hipMemcpy(x[i].dev.ptr, np.ascontiguousarray(words[i]).ctypes.data, words[i].nbytes, 1) == 0
        for _ in range(3):
            for g in graphs:
                g.replay()
        for st in streams:
            st.sync()
        for i in range(2):
            q.matmul(x[i].ptr, BF16, rows, alone.ptr, F32)
            assert np.array_equal(y[i].get(), alone.get())
            want = unpack(words[i], BF16) @ w.T
            close(alone.get().astype(np.float64), want, tolerance(unpack(words[i], BF16), s, want, F32))


@pytest.mark.parametrize("first,more", [(1, 0), (0, 1), (8, 8)])
def test_blocks_of_rows_at_any_address(first, more):
    rng = np.random.default_rng(first + more)
    check(rng, 1600, 520, 128, 510, F16, F16, x_stride=520 + more, first=first)


@pytest.mark.parametrize("x_dtype,norm", [(F32, False), (F32, True), (BF16, True), (F16, False)])
@pytest.mark.parametrize("rows", [17, 22, 32, 45])
def test_few_inputs_and_long_ones_for_many_rows(rows, x_dtype, norm):
    """More waves than tiles of inputs ask for; rows that LDS holds exactly, nearly, in chunks of unequal length."""
    rng = np.random.default_rng(rows)
    for n, k, group in ((346, 32, 32), (16, 130, 64), (40, 1536, 128), (33, 6752, 32), (33, 2500, 64)):
        check(rng, n, k, group, rows, x_dtype, F32, zeros=rows % 2 == 0, norm=norm, mean=0.1)


def test_scales_of_bf16_far_apart():
    """A factor of 2^32 between the scales fits, with any bits set; what no power of two brings into fp16 is refused."""
    rng = np.random.default_rng(21)
    n, k, group = 48, 256, 64
    codes = rng.integers(0, 256, (n, k // 2)).astype(np.uint8)
    for top in (2.0 ** 60, 1.0, 2.0 ** -80):
        values = top * 2.0 ** -rng.integers(0, 33, (n, k // group)).astype(np.float64) * (1 + rng.integers(0, 128, (n, k // group)) / 128.0)
        values[0, 0], values[1, 1], values[2] = top * 1.9921875, top * 2.0 ** -32 * 1.9921875, 0.0
        scales = scale_words(values, BF16)
        q, s = pkg.Quant(n, k, group, codes, scales, BF16), scales_of(scales, BF16)
        xv = pack(rng.standard_normal((5, k)) / top, F32)
        x, y = Rows(xv), Rows(np.zeros((5, n), np.float32))
        q.matmul(x.ptr, F32, 5, y.ptr, F32)
        xh = unpack(xv, F32)
        want = xh @ weights(codes, s, None, k, group).T
        close(y.get().astype(np.float64), want, tolerance(xh, np.abs(s)[:, np.arange(k) // group], want, F32))
    for least in (2.0 ** -60, 2.0 ** -120):
        values = np.ones((n, k // group))
        values[3, 1] = least
        with pytest.raises(pkg.BildError) as e:
            pkg.Quant(n, k, group, codes, scale_words(values, BF16), BF16)
        assert e.value.code == b.EINVAL


@pytest.mark.parametrize("x_dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,n,ks", [(1, 40, (1, 3, 7)), (5, 300, (1, 7, 9)), (11, 2048, (4097, 4103)), (32, 2048, (1, 7, 1025, 1031, 1537, 1543)), (45, 64, (5, 1025))])
def test_norm_of_fewer_inputs_than_a_piece(rows, n, ks, x_dtype):
    """Rows, or their last part in LDS, of one to seven inputs: what is behind them counts nothing."""
    rng = np.random.default_rng(rows)
    for k in ks:
        check(rng, n, k, 64, rows, x_dtype, F32, norm=True, mean=0.1)
