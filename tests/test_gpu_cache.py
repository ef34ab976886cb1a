"""The cache in 8 bits on the GPU: pages, what is written into them, and attention, against the definition in numpy."""
import ctypes as C

import numpy as np
import pytest

import paper_2302_07863_amd as pkg
from paper_2302_07863_amd import binding as b
from tests.cached import Held, Oracle, invariants, values
from tests.hipmem import H2D, DeviceArray, hip
from tests.rows import BF16, F16, F32, Graph, Rows, Stream, close, pack, unpack

pytestmark = pytest.mark.gpu


def ints(a):
    return DeviceArray(np.asarray(a, np.int32))


def starts_of(rows):
    return np.concatenate(([0], np.cumsum(rows))).astype(np.int32)


def extend(t, rows, sequences=None, cut=None, uniform=False, **kw):
    """On the device and in the definition; whether they have grown."""
    n = len(rows)
    keep = [ints(x) if x is not None else None for x in (sequences, cut)]
    starts, granted = None if uniform else ints(starts_of(rows)), ints([7])
    ok = t.o.extend(rows, sequences, cut, **kw)
    t.cache.extend(n, int(rows[0]) if uniform else 0, sequences=keep[0] and keep[0].ptr.value, cut=keep[1] and keep[1].ptr.value, starts=starts and starts.ptr.value, granted=granted.ptr.value, **kw)
    assert granted.to_host(np.int32, 1)[0] == int(ok)
    return ok


def fork(t, parents, sequences=None, group=0):
    keep = [ints(x) if x is not None else None for x in (sequences, parents)]
    t.o.fork(parents, sequences, group)
    t.cache.fork(len(parents), keep[1].ptr.value, sequences=keep[0] and keep[0].ptr.value, group=group)
    assert pkg.lib() and keep[1].to_host(np.int32, 1) is not None     # (done before the arrays go)


def append(t, rng, layer, rows, dtype=F32, sequences=None, uniform=False, size=1.0, spoil=None):
    o, tokens = t.o, int(np.sum(rows))
    if not tokens:
        return
    words, x = values(rng, (2, tokens, o.heads, o.d), dtype, size)
    if spoil is not None:
        spoil(words, x)
    k, v = DeviceArray(words[0]), DeviceArray(words[1])
    ids, starts = ints(sequences) if sequences is not None else None, None if uniform else ints(starts_of(rows))
    t.cache.append(layer, dtype, len(rows), int(max(max(rows), 1)), k.ptr.value, v.ptr.value, sequences=ids and ids.ptr.value, starts=starts and starts.ptr.value, tokens=0 if uniform else tokens)
    o.append(layer, x[0], x[1], rows, sequences)
    k.to_host(np.uint8, 1)


def attend(t, rng, layer, rows, group=1, dtype=F32, sequences=None, uniform=False, size=1.0, scale=None, stream=None, **kw):
    """One call against the definition, rows with strides of their own; the outputs."""
    o, tokens = t.o, int(np.sum(rows))
    hq = o.heads * group
    words, x = values(rng, (tokens, hq * o.d), dtype, size)
    q, out = Rows(words, hq * o.d + 3, 1), Rows(np.zeros_like(words), hq * o.d + 5, 3)
    lse = Rows(np.full((tokens, hq), 77, np.float32))
    ids, starts = ints(sequences) if sequences is not None else None, None if uniform else ints(starts_of(rows))
    scale = o.d ** -0.5 if scale is None else scale
    t.cache.attend(layer, dtype, len(rows), int(max(max(rows), 1)), hq, q.ptr, out.ptr, scale, lse=lse.ptr, q_token=q.stride, out_token=out.stride,
                   sequences=ids and ids.ptr.value, starts=starts and starts.ptr.value, tokens=0 if uniform else tokens, **kw)
    got, got_lse = unpack(out.get(), dtype).reshape(tokens, hq, o.d), lse.get()
    want, want_lse, tol, ltol = o.attend(layer, x.astype(np.float64).reshape(tokens, hq, o.d), rows, float(np.float32(scale)), sequences, dtype=dtype,
                                         **{k: v for k, v in kw.items() if k in ("window", "sinks", "causal")})
    alive = np.isfinite(want_lse)
    over = np.repeat([not 0 <= s < len(o.lengths) for s in (range(len(rows)) if sequences is None else sequences)], rows)    # (rows of sequences that are passed over stay what they were)
    assert np.all(got_lse[over] == 77) and np.all(got_lse[~over][~alive[~over]] == -np.inf) and np.all(got[~alive] == 0)
    close(got_lse[alive], want_lse[alive], ltol[alive])
    close(got, want, tol)
    return got, got_lse


def cache(seed=0, pages=40, page=32, layers=1, heads=2, d=64, sequences=4, max_pages=16):
    rng = np.random.default_rng(seed)
    return Held(Oracle(pages, page, layers, heads, d, sequences, max_pages)), rng


# ------------------------------------------------------------------------------------------------ pages
@pytest.mark.parametrize("page", [32, 64, 128])
@pytest.mark.parametrize("seed", [1, 2, 3])
def test_pages_through_many_calls(page, seed):
    t, rng = cache(seed, pages=90, page=page, layers=2, heads=3, d=16, sequences=9, max_pages=14)
    o = t.o
    refused = 0
    for step in range(40):
        what = rng.integers(0, 8)
        if what < 5:
            ids = rng.permutation(9)[:rng.integers(1, 10)].astype(np.int32)
            if rng.random() < 0.2:
                ids[0] = rng.choice([-1, 9, 1000])
            rows = rng.integers(0, 2 * page if rng.random() < 0.5 else 3, len(ids))
            cut = None if rng.random() < 0.5 else np.array([rng.integers(-3, (o.lengths[s] if 0 <= s < 9 else 0) + 5) for s in ids])
            ok = extend(t, rows, ids, cut)
            refused += not ok
            append(t, rng, int(rng.integers(0, 2)), rows, sequences=ids)
        elif what < 7:
            ids, group = (rng.permutation(9)[:6], 3) if rng.random() < 0.5 else (None, 0)
            n = 9 if ids is None else 6
            fork(t, rng.integers(-1, group or n, n), ids, group)
        else:
            used = ints([0])
            want = o.compact()
            t.cache.compact(used=used.ptr.value)
            assert used.to_host(np.int32, 1)[0] == want
        t.same()
        invariants(o)
    assert step == 39 and refused < 40


def test_all_or_none():
    t, rng = cache(pages=5, sequences=3, max_pages=4)
    assert extend(t, [32, 33, 0])
    append(t, rng, 0, [32, 33, 0])
    t.same()
    assert not extend(t, [32, 32, 32], cut=[32, 33, 0])       # three pages are asked for, two are there
    t.same()
    append(t, rng, 0, [32, 32, 32])                            # (writes nothing)
    t.same()
    assert not extend(t, [0, 0, 129])                          # longer than a sequence may be
    t.same()
    assert extend(t, [1, 1, 1])
    append(t, rng, 0, [1, 1, 1])
    t.same()
    assert extend(t, [0, 0, 0], cut=[0, 0, 0]) and np.all(t.o.refs == 0)
    t.same()


def test_shared_pages_are_copied_and_the_last_keeps_its_own():
    t, rng = cache(3, pages=12, sequences=5, max_pages=3)
    extend(t, [41], [0])
    append(t, rng, 0, [41], sequences=[0])
    fork(t, [0, 0, 0, -1, 3])
    t.same()
    assert extend(t, [1, 1], [0, 1], uniform=True)             # sequence 2 holds the old page: both are copied
    t.same()
    append(t, rng, 0, [1, 1], sequences=[0, 1], uniform=True)
    t.same()
    fork(t, [0, 0, 2, 2, 0])
    assert extend(t, [2, 2, 2, 2, 2], uniform=True)
    append(t, rng, 0, [2, 2, 2, 2, 2], uniform=True)
    t.same()
    invariants(t.o)
    # a page that somebody else holds is not written, whatever is asked
    fork(t, [0, 0], [0, 1])
    append(t, rng, 0, [1, 1], sequences=[0, 1])
    t.same()


def test_pages_behind_a_window_are_given_back():
    t, rng = cache(5, pages=30, sequences=3, max_pages=64)
    for step in range(60):
        rows = [7, 31, 1]
        assert extend(t, rows, window=50, sinks=33)
        append(t, rng, 0, rows)
        if step % 9 == 0:
            t.same()
            attend(t, rng, 0, rows, group=2, window=50, sinks=33)
    assert np.sum(t.o.table[1] >= 0) <= 2 + 4 and t.o.lengths[1] == 60 * 31
    # a cut into what was given back is refused, the next one from the beginning is not
    assert not extend(t, [1, 1, 1], cut=[420, 700, 60])
    t.same()
    assert extend(t, [5, 5, 5], cut=[0, 0, 0])
    t.same()


def test_large_pools_and_long_lists():
    t, rng = cache(7, pages=20000, page=32, layers=1, heads=1, d=16, sequences=1500, max_pages=40)
    rows = rng.integers(0, 500, 1500)
    rows[700] = 1280
    ok = extend(t, rows)
    t.same(("table", "lengths", "refs"))
    assert ok == (np.sum(-(-rows // 32)) <= 20000)
    ids = rng.permutation(1500)
    extend(t, rng.integers(0, 3, 1500), ids, cut=rng.integers(0, 500, 1500))
    t.same(("table", "lengths", "refs"))
    fork(t, np.arange(1500) // 2)
    t.same(("table", "lengths", "refs"))
    extend(t, np.ones(1500, int), uniform=True)
    t.same(("table", "lengths", "refs"))
    t.o.compact()
    t.cache.compact()
    t.same(("table", "lengths", "refs"))
    invariants(t.o)


# ------------------------------------------------------------------------------------------------ what is written
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("page,heads,d", [(32, 1, 16), (32, 3, 72), (64, 2, 128), (128, 2, 256), (128, 1, 136)])
def test_codes_and_scales(dtype, page, heads, d):
    t, rng = cache(page + d, pages=24, page=page, layers=2, heads=heads, d=d, sequences=3, max_pages=7)
    for rows in ([1, 0, 5], [1, page, 2 * page + 1], [page - 2, 1, 0], [3, 3, 3]):
        extend(t, rows)
        append(t, rng, 1, rows, dtype, size=float(rng.choice([0.01, 1.0, 30.0])))
        t.same()


def test_a_growing_scale_rounds_what_is_there_again():
    t, rng = cache(1, d=32, heads=1)
    for i in range(30):
        extend(t, [1])
        append(t, rng, 0, [1], F32, size=1.2 ** i)
    t.same()
    k = t.get("scales")[t.o.table[0, 0], 0, 0, 0]
    assert k == np.max(t.o.scales)  or k > 1.2 ** 25


@pytest.mark.parametrize("top", [127.0, 100.0, 3.3e-3, 1e-37, 3e-40, 5e26])
def test_values_on_the_border_between_codes(top):
    """Halves, and the neighbours of halves, in the last bit: codes are those of the quotient, whatever it is computed by."""
    t, rng = cache(3, d=64, heads=2)

    def spoil(words, x):
        y = ((rng.integers(-127, 127, x.shape) + np.float32(0.5)) * np.float64(top) / 127).astype(np.float32)
        x[...] = np.nextafter(y, np.float32(np.inf) * rng.choice([-1, 1], x.shape).astype(np.float32), where=rng.random(x.shape) < 0.6, out=y.copy())
        x[:, 0] = np.float32(top)
        words[...] = x

    extend(t, [30, 9, 1, 32])
    append(t, rng, 0, [30, 9, 1, 32], F32, spoil=spoil)
    t.same()


def test_values_at_the_ends_of_fp32():
    t, rng = cache(2, d=16, heads=2)

    def spoil(words, x):
        x[0, 0, 0, :4] = [np.inf, -np.inf, np.nan, 3e38]
        x[0, 1, 0, :3] = [1e-45, -1e-45, 1e-38]                # (a page of nothing else: below)
        x[1, :, 1] = 0.0                                       # zeros throughout
        x[1, 1, 0, :] = np.nan
        words[...] = x

    extend(t, [2])
    append(t, rng, 0, [2], F32, spoil=spoil)
    t.same()
    assert np.all(np.isfinite(t.get("scales")))

    def tiny(words, x):
        x[...] = np.where(rng.random(x.shape) < 0.5, 1e-45, -3e-45)
        words[...] = x

    extend(t, [3], cut=[0])
    append(t, rng, 0, [3], F32, spoil=tiny)
    t.same()
    out, _ = attend(t, rng, 0, [3])
    assert np.all(np.isfinite(out))


# ------------------------------------------------------------------------------------------------ attention
def filled(seed, lengths, dtype=F32, **kw):
    t, rng = cache(seed, sequences=len(lengths), **kw)
    assert extend(t, lengths)
    for layer in range(t.o.layers):
        append(t, rng, layer, lengths)
    t.same()
    return t, rng


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("page,heads,d,group", [(32, 2, 64, 1), (64, 1, 128, 4), (128, 2, 256, 1), (32, 1, 16, 3), (64, 3, 72, 2), (32, 1, 136, 7), (128, 1, 96, 64), (32, 1, 248, 2)])
def test_single_rows(dtype, page, heads, d, group):
    t, rng = filled(d + group, [1, 31, 32, 33, 300], pages=40, page=page, layers=2, heads=heads, d=d, max_pages=10)
    attend(t, rng, 1, [1] * 5, group, dtype, uniform=True)
    attend(t, rng, 0, [1, 1], group, dtype, sequences=[4, 2])
    attend(t, rng, 1, [1] * 5, group, dtype, window=40, sinks=5)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows", [[2, 2, 2], [11, 1, 5], [0, 40, 17], [130, 1, 64], [1, 0, 0]])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (33, 4), (64, 40), (500, 2)])
def test_several_rows(dtype, rows, window, sinks):
    t, rng = filled(rows[0], [150, 64, 97], pages=30, heads=2, d=64)
    group = 1 if rows[0] == 11 else 2
    attend(t, rng, 0, rows, group, dtype, window=window, sinks=sinks)


@pytest.mark.parametrize("d,group,dtype", [(128, 4, BF16), (64, 1, F16), (80, 2, F32), (256, 1, BF16)])
@pytest.mark.parametrize("rows", [200, 333])
def test_prompts(d, group, dtype, rows):
    t, rng = filled(rows + d, [rows + 60, rows], pages=40, page=32, heads=1, d=d, max_pages=20)
    attend(t, rng, 0, [rows, rows], group, dtype, uniform=True)
    attend(t, rng, 0, [rows, 3], group, dtype, window=70, sinks=4)


@pytest.mark.parametrize("page", [32, 64, 128])
@pytest.mark.parametrize("d,dtype", [(128, BF16), (64, F16), (80, BF16), (72, F32), (256, F16), (136, BF16), (248, F32), (16, F16), (128, F32)])
def test_prompts_that_fill_the_chip(page, d, dtype):
    """Rows times query heads that are not whole tiles, cached positions in front, a window whose sinks end inside a tile of keys."""
    t, rng = filled(page + d, [190, 77], pages=16, page=page, heads=16, d=d, max_pages=7)
    attend(t, rng, 0, [133], 8, dtype, sequences=[0], scale=-0.1 if d == 80 else None)
    attend(t, rng, 0, [77, 61], 8, dtype, sequences=[1, 0], window=50, sinks=37)


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 1), (300, 0), (130, 100)])
def test_prompts_between_single_rows(window, sinks):
    """Ragged: prompts, single rows, none, sequences that are not there, lengths shorter than the rows."""
    lengths = [700, 40, 1, 0, 333, 90, 257]
    t, rng = filled(31, lengths, pages=60, page=64, heads=8, d=64, max_pages=12)
    attend(t, rng, 0, [520, 1, 1, 1, 12, 99, 0], 4, BF16, window=window, sinks=sinks)
    # (of a page that is not there nothing counts)
    t.o.table[0, 3], t.o.table[0, 8], t.o.table[5, 0] = -1, 99999, -5
    t = Held(t.o)
    attend(t, rng, 0, [520, 1, 1, 1, 12, 99, 0], 4, F16, window=window, sinks=sinks)
    if not window:
        attend(t, rng, 0, [300, 1, 2, 0, 64, 90, 3], 4, F32, causal=False)


def test_prompts_with_rows_that_are_not_finite():
    t, rng = filled(32, [200], pages=10, d=64, heads=16)
    words, x = values(rng, (200, 128 * 64), BF16)
    x = x.astype(np.float64).reshape(200, 128, 64)
    bad = np.zeros((200, 128), bool)
    for r, h, v in ((0, 0, np.nan), (77, 5, np.inf), (130, 127, -np.inf)):
        words.reshape(200, 128, 64)[r, h, 9] = pack(np.float32([v]), BF16)[0]
        bad[r, h] = True
        x[r, h] = 0
    q, out = Rows(words), Rows(np.zeros_like(words))
    t.cache.attend(0, BF16, 1, 200, 128, q.ptr, out.ptr, 0.125)
    want, _, tol, _ = t.o.attend(0, x, [200], 0.125, dtype=BF16)
    got = unpack(out.get(), BF16).reshape(200, 128, 64)
    assert np.all(np.isnan(got[bad]))
    close(got[~bad], want[~bad], tol[~bad])


def test_without_order():
    t, rng = filled(4, [100, 1, 0, 250], pages=30, d=64)
    for dtype in (F32, BF16):
        attend(t, rng, 0, [5, 2, 3, 40], 2, dtype, causal=False)


def test_rows_that_see_nothing():
    t, rng = filled(6, [40, 0, 3], pages=30, d=64)
    out, lse = attend(t, rng, 0, [2, 3, 5], 2, BF16)            # (a sequence of length 0; rows from before a sequence's beginning)
    assert np.all(lse[2:7] == -np.inf) and np.all(out[2:7] == 0)
    # sequences that are not there have no outputs, and rows behind the last are not touched
    before = np.full((12, 4 * 64), 5, np.float32)
    o = Rows(before)
    q = Rows(rng.standard_normal((12, 4 * 64)).astype(np.float32))
    ids, starts = ints([0, 9, -4]), ints([0, 2, 4, 7])
    t.cache.attend(0, F32, 3, 3, 4, q.ptr, o.ptr, 0.1, sequences=ids.ptr.value, starts=starts.ptr.value, tokens=12)
    got = o.get()
    assert np.all(got[2:] == 5) and np.all(got[:2] != 5)


def test_pages_that_are_not_there_count_for_nobody():
    t, rng = filled(8, [200, 90], pages=30, d=64)
    table = t.o.table.copy()
    table[0, 2], table[0, 5], table[1, 0] = -1, 1000000, -7
    t.o.table[...] = table
    t2 = Held(t.o)
    attend(t2, rng, 0, [3, 2], 2, F32)
    attend(t2, rng, 0, [3, 2], 2, BF16, window=100, sinks=10)
    t2.o.table[...] = -1
    t3 = Held(t.o)
    out, lse = attend(t3, rng, 0, [3, 2], 2, F16)
    assert np.all(out == 0) and np.all(lse == -np.inf)


@pytest.mark.parametrize("dtype,bad", [(F32, np.nan), (F32, np.inf), (BF16, -np.inf), (F16, np.nan)])
def test_a_row_that_is_not_finite_leaves_the_others_alone(dtype, bad):
    t, rng = filled(9, [100], pages=30, d=64, heads=1)
    words, x = values(rng, (4, 2 * 64), dtype)
    words[1, 5] = pack(np.float32([bad]), dtype)[0]
    q, out, lse = Rows(words), Rows(np.zeros_like(words)), Rows(np.zeros((4, 2), np.float32))
    t.cache.attend(0, dtype, 1, 4, 2, q.ptr, out.ptr, 0.125, lse=lse.ptr)
    x = x.astype(np.float64).reshape(4, 2, 64)
    x[1, 0] = 0
    want, want_lse, tol, ltol = t.o.attend(0, x, [4], 0.125, dtype=dtype)
    got, l = unpack(out.get(), dtype).reshape(4, 2, 64), lse.get()
    others = np.ones((4, 2), bool)
    others[1, 0] = False
    assert np.all(np.isnan(got[1, 0])) and np.isnan(l[1, 0])
    close(got[others], want[others], tol[others])
    close(l[others], want_lse[others], ltol[others])


@pytest.mark.parametrize("size,scale", [(1e-30, 1.0), (1e30, 1e-30), (1.0, 0.0), (1.0, -0.3), (60.0, 1.0)])
def test_rows_of_any_size(size, scale):
    t, rng = filled(10, [150], pages=30, d=64)
    for dtype in (F32, BF16):
        attend(t, rng, 0, [3], 2, dtype, size=size, scale=scale)


def test_a_long_sequence_and_many_short_ones():
    lengths = [3] * 60 + [3000] + [200] * 9 + [0] + [1] * 29
    t, rng = filled(11, lengths, pages=400, page=64, heads=1, d=64, max_pages=60)
    attend(t, rng, 0, [1] * 100, 4, BF16, uniform=True)
    attend(t, rng, 0, [1] * 59 + [0, 70] + [2] * 39, 1, F32)
    attend(t, rng, 0, [1] * 100, 1, F16, window=300, sinks=4)


def test_lists_longer_than_a_workgroup():
    t, rng = cache(12, pages=1200, page=32, heads=1, d=16, sequences=600, max_pages=4)
    rows = rng.integers(0, 60, 600)
    assert extend(t, rows)
    append(t, rng, 0, rows)
    t.same()
    attend(t, rng, 0, np.minimum(rows, rng.integers(0, 3, 600)), 1, F32)


def test_replayed_graphs_and_other_streams():
    """A step - grow, append, attend - captured: its numbers come from device memory, and grow from replay to replay."""
    t, rng = filled(13, [30, 60], pages=30, d=64)
    t.o.extend([1, 1])                                          # what the first replay will do
    words, x = values(rng, (3, 2, 2, 64), F32)
    mem = [DeviceArray(w) for w in words]
    out, st = Rows(np.zeros((2, 128), np.float32)), Stream()

    def step(stream):
        t.cache.extend(2, 1, stream=stream)
        t.cache.append(0, F32, 2, 1, mem[1].ptr.value, mem[2].ptr.value, stream=stream)
        t.cache.attend(0, F32, 2, 1, 2, mem[0].ptr.value, out.ptr, 0.125, stream=stream)

    g = Graph(st, step)
    for i in range(6):
        if i:
            t.o.extend([1, 1])
        t.o.append(0, x[1], x[2], [1, 1])
        g.replay()
        st.sync()
        want, _, tol, _ = t.o.attend(0, x[0].astype(np.float64), [1, 1], 0.125)
        close(out.get().reshape(2, 2, 64), want, tol)
        t.same()
        if i == 3:                                              # eager work of the handle's between replays, in order
            fork(t, [1, 1])


def test_two_handles_at_the_same_time():
    both = [filled(s, [700, 800], pages=60, d=128, max_pages=30) for s in (20, 21)]
    streams, outs, wants = [Stream(), Stream()], [], []
    for (t, rng), st in zip(both, streams):
        words, x = values(rng, (2, 256), F32)
        q, out = DeviceArray(words), Rows(np.zeros((2, 256), np.float32))
        wants.append(t.o.attend(0, x.astype(np.float64).reshape(2, 2, 128), [1, 1], 0.1))
        outs.append((q, out))
    for _ in range(20):
        for (t, _), st, (q, out) in zip(both, streams, outs):
            t.cache.attend(0, F32, 2, 1, 2, q.ptr.value, out.ptr, float(np.float32(0.1)), stream=st.h.value)
    for st, (q, out), w in zip(streams, outs, wants):
        st.sync()
        close(out.get().reshape(2, 2, 128), w[0], w[2])


def test_the_same_bits_every_time():
    t, rng = filled(14, [2000, 100, 5], pages=80, d=128, heads=2, max_pages=70)
    words, _ = values(rng, (3, 8 * 128), BF16)
    q, out = DeviceArray(words), DeviceArray(nbytes=words.nbytes)
    seen = set()
    for _ in range(20):
        t.cache.attend(0, BF16, 3, 1, 8, q.ptr.value, out.ptr.value, 0.1)
        seen.add(out.to_host(np.uint8, words.nbytes).tobytes())
    assert len(seen) == 1


def test_calls_that_are_refused():
    t, rng = filled(15, [5, 5], pages=8, d=64)
    c, mem = t.cache, DeviceArray(nbytes=1 << 16)
    p = mem.ptr.value
    calls = [lambda: c.extend(0), lambda: c.extend(3), lambda: c.extend(1, -1), lambda: c.extend(1, 0, window=-1), lambda: c.extend(1, 0, sinks=-1),
             lambda: c.fork(0, p), lambda: c.fork(3, p), lambda: c.fork(1, None), lambda: c.fork(2, p, group=3), lambda: c.fork(2, p, group=-1),
             lambda: c.append(1, F32, 1, 1, p, p), lambda: c.append(-1, F32, 1, 1, p, p), lambda: c.append(0, 3, 1, 1, p, p), lambda: c.append(0, F32, 0, 1, p, p),
             lambda: c.append(0, F32, 3, 1, p, p), lambda: c.append(0, F32, 1, 0, p, p), lambda: c.append(0, F32, 1, 1, None, p), lambda: c.append(0, F32, 1, 1, p, None),
             lambda: c.append(0, F32, 1, 1, p, p, starts=p, tokens=0), lambda: c.append(0, F32, 2, 1 << 30, p, p),
             lambda: c.attend(1, F32, 1, 1, 2, p, p, 1.0), lambda: c.attend(0, -1, 1, 1, 2, p, p, 1.0), lambda: c.attend(0, F32, 1, 1, 3, p, p, 1.0),
             lambda: c.attend(0, F32, 1, 1, 0, p, p, 1.0), lambda: c.attend(0, F32, 1, 1, 130, p, p, 1.0), lambda: c.attend(0, F32, 1, 1, 2, None, p, 1.0),
             lambda: c.attend(0, F32, 1, 1, 2, p, None, 1.0), lambda: c.attend(0, F32, 1, 1, 2, p, p, float("nan")), lambda: c.attend(0, F32, 1, 1, 2, p, p, float("inf")),
             lambda: c.attend(0, F32, 1, 0, 2, p, p, 1.0), lambda: c.attend(0, F32, 3, 1, 2, p, p, 1.0), lambda: c.attend(0, F32, 1, 1, 2, p, p, 1.0, window=-1),
             lambda: c.attend(0, F32, 1, 1, 2, p, p, 1.0, sinks=-1), lambda: c.attend(0, F32, 1, 1, 2, p, p, 1.0, window=4, causal=False),
             lambda: c.attend(0, F32, 1, 1, 2, p, p, 1.0, starts=p, tokens=0), lambda: c.attend(0, F32, 2, 1 << 29, 128, p, p, 1.0)]
    for call in calls:
        with pytest.raises(pkg.BildError) as e:
            call()
        assert e.value.code == b.EINVAL
    bad = b.CacheAttendCall(q=p, out=p, n=1, rows=1, heads=2, scale=1.0, causal=2, q_token=128, q_head=64, out_token=128, out_head=64)
    assert pkg.lib().bild_cache_attend(c.h, C.byref(bad), None) == b.EINVAL
    bad = b.CacheAppendCall(k=p, v=p, n=1, rows=1, reserved=1)
    assert pkg.lib().bild_cache_append(c.h, C.byref(bad), None) == b.EINVAL
    t.same()


# ------------------------------------------------------------------------------------------------ what rows and pages may be like
@pytest.mark.parametrize("page", [32, 64])
@pytest.mark.parametrize("by", [3, 20, 60])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_pages_whose_scales_are_far_apart(page, by, dtype):
    """Each page of the values has a scale of its own, up to 2^(2 by) apart, some 0: for few rows and for prompts."""
    t, rng = filled(page + by, [333], pages=12, page=page, heads=4, d=64, max_pages=12)
    n = len(t.o.scales)
    t.o.scales[:, 0, 1] *= np.exp2(rng.integers(-by, by + 1, (n, 4))).astype(np.float32)
    t.o.scales[1, 0, 1], t.o.scales[3, 0, 0] = 0, 0
    t = Held(t.o)
    attend(t, rng, 0, [3], 2, dtype)
    attend(t, rng, 0, [300], 8, dtype, causal=False)
    attend(t, rng, 0, [333], 4, dtype, window=100 if by < 60 else 0, sinks=7)


@pytest.mark.parametrize("page", [32, 64])
@pytest.mark.parametrize("tall,low", [(80, -100), (89, -120)])
def test_scales_at_both_ends(page, tall, low):
    """A page of next to nothing counts in the sum of the weights like any other."""
    t, rng = filled(page, [200], pages=7, page=page, heads=4, d=64, max_pages=12)
    for order in (0, 1):
        t.o.scales[:, 0, 1] = np.exp2(float(low))
        t.o.scales[order::2, 0, 1] = np.exp2(float(tall))
        t = Held(t.o)
        attend(t, rng, 0, [2], 2, BF16, causal=False)
        attend(t, rng, 0, [200], 8, BF16, causal=False)


def test_infinities_in_the_values():
    """They are limited, so that sums over many of them end as finite as they are."""
    t, rng = cache(40, pages=40, page=64, heads=4, d=64, sequences=2, max_pages=30)
    extend(t, [1500, 300])

    def spoil(words, x):
        x[1, ::2, 1] = np.inf
        x[1, ::3, 2, ::2] = -np.inf
        x[1, :, 3] = 3e38
        words[...] = x

    append(t, rng, 0, [1500, 300], spoil=spoil)
    t.same()
    assert np.max(t.o.scales) == np.float32(2.0 ** 90)
    attend(t, rng, 0, [1, 2], 2, F32, size=3.0)
    out, _ = attend(t, rng, 0, [400, 300], 4, BF16, size=3.0)
    assert np.all(np.isfinite(out)) and np.max(np.abs(out)) > 2.0 ** 85


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [1, 3, 70])
def test_rows_with_strides(dtype, rows):
    """Heads and tokens apart, heads before tokens: keys, values, rows and results in views of larger arrays."""
    t, rng = cache(50 + rows, pages=20, page=32, heads=3, d=40, sequences=2, max_pages=8)
    o, tokens, group = t.o, 2 * rows, 2
    for _ in range(2):
        extend(t, [rows, rows], uniform=True)
        words, x = values(rng, (2, 3, tokens, 43), dtype)       # [k or v][head][token][d and some]
        mem = DeviceArray(words)
        size, off = words.itemsize, 2
        k, v = mem.ptr.value + off * size, mem.ptr.value + (3 * tokens * 43 + off) * size
        t.cache.append(0, dtype, 2, rows, k, v, k_token=43, k_head=43 * tokens, v_token=43, v_head=43 * tokens)
        rows_of = x[..., off:off + 40].transpose(0, 2, 1, 3)
        o.append(0, rows_of[0], rows_of[1], [rows, rows])
        t.same()
    words, x = values(rng, (6, tokens, 45), dtype)
    before = pack(np.full((tokens, 7, 51), 9, np.float32), dtype)
    q, out = DeviceArray(words), DeviceArray(before)
    t.cache.attend(0, dtype, 2, rows, 6, q.ptr.value + 3 * words.itemsize, out.ptr.value + 5 * words.itemsize, 0.2, q_token=45, q_head=45 * tokens, out_token=7 * 51, out_head=51)
    want, _, tol, _ = o.attend(0, x[..., 3:43].transpose(1, 0, 2).astype(np.float64), [rows, rows], float(np.float32(0.2)), dtype=dtype)
    got = unpack(out.to_host(before.dtype, before.size), dtype).reshape(before.shape)
    close(got[:, :6, 5:45], want, tol)
    got[:, :6, 5:45] = 9
    assert np.all(got == 9)                                     # nothing else is written


def test_pools_beyond_32_bits():
    """Pages of 64 MiB, the last of them behind 4 GiB: written, copied, read and moved."""
    layers, heads, d, page, pages = 64, 64, 128, 64, 70
    size = layers * 2 * heads * page * d
    assert size * pages > 1 << 32
    codes = DeviceArray(nbytes=size * pages)
    scales = DeviceArray(np.zeros(pages * layers * 2 * heads, np.float32))
    table, lengths, refs = ints(np.full((3, 2), -1)), ints([0, 0, 0]), np.ones(pages, np.int32)
    refs[[66, 67, 69]] = 0                                      # (the others are somebody's)
    held = ints(refs)
    c = pkg.Cache(pages, page, layers, heads, d, 3, 2, codes=codes.ptr.value, scales=scales.ptr.value, table=table.ptr.value, lengths=lengths.ptr.value, refs=held.ptr.value)
    rng = np.random.default_rng(5)
    o = Oracle(3, page, 1, heads, d, 3, 2)                      # pages 0, 1, 2 for 66, 67, 69; one layer, the last
    for rows, ids in ((40, [0]), (3, [0, 1])):
        if len(ids) == 2:
            parents = ints([0, 0, 2])
            o.fork([0, 0, 2])
            c.fork(3, parents.ptr.value)
        words, x = values(rng, (2, rows * len(ids), heads, d), BF16)
        k, v = DeviceArray(words[0]), DeviceArray(words[1])
        o.extend([rows] * len(ids), ids)
        o.append(0, x[0], x[1], [rows] * len(ids), ids)
        c.extend(len(ids), rows)
        c.append(layers - 1, BF16, len(ids), rows, k.ptr.value, v.ptr.value)
        names = np.array([66, 67, 69, -1])
        assert np.array_equal(table.to_host(np.int32, 6).reshape(3, 2), names[o.table])
    words, x = values(rng, (2, 2 * heads, d), BF16)
    q, out = DeviceArray(words), DeviceArray(nbytes=words.nbytes)
    want, _, tol, _ = o.attend(0, x.astype(np.float64), [1, 1], float(np.float32(0.1)), dtype=BF16)
    for turn in range(2):
        c.attend(layers - 1, BF16, 2, 1, 2 * heads, q.ptr.value, out.ptr.value, 0.1)
        close(unpack(out.to_host(np.uint16, words.size), BF16).reshape(want.shape), want, tol)
        if turn == 0:
            freed = np.array(held.to_host(np.int32, pages))
            freed[[3, 68]] = 0                                  # two in front go: the highest moves into the first
            assert hip().hipMemcpy(held.ptr, np.ascontiguousarray(freed, np.int32).ctypes.data, 4 * pages, H2D) == 0
            used = ints([0])
            c.compact(used=used.ptr.value)
            assert used.to_host(np.int32, 1)[0] == np.sum(freed > 0)
            assert np.all(table.to_host(np.int32, 6) < used.to_host(np.int32, 1)[0])


@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 40)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_prompts_behind_lengths_far_apart(window, sinks, dtype):
    """Keys of long sequences are shared between workgroups, those of short ones are not; sequences that are passed over, without rows, without keys."""
    lengths = [2900, 130, 129, 0, 700, 64, 5, 260]
    t, rng = filled(60, lengths, pages=90, page=64, heads=1, d=64, max_pages=50)
    ids = [5, 0, -1, 3, 1, 7, 4, 6]
    attend(t, rng, 0, [64, 130, 3, 20, 129, 0, 33, 9], 7, dtype, sequences=ids, window=window, sinks=sinks)


def test_prompts_of_more_sequences_than_a_wave():
    lengths = [int(x) for x in np.random.default_rng(8).integers(0, 90, 80)]
    lengths[7], lengths[70] = 1500, 640
    t, rng = filled(61, lengths, pages=200, page=64, heads=2, d=16, max_pages=30)
    rows = [min(x, 70) if i % 3 else 1 for i, x in enumerate(lengths)]
    rows[7], rows[70] = 130, 600
    attend(t, rng, 0, rows, 4, BF16)
    attend(t, rng, 0, [50] * 80, 4, F16, uniform=True)


@pytest.mark.parametrize("heads", [5, 12, 40, 300])
def test_head_counts_that_share_the_chip_unevenly(heads):
    t, rng = filled(heads, [200, 31], pages=12, page=32, heads=heads, d=16, max_pages=8)
    attend(t, rng, 0, [1, 1], 2, BF16, uniform=True)
    attend(t, rng, 0, [40, 2], 2, F32)


@pytest.mark.parametrize("page,rows,length", [(64, 700, 700), (32, 640, 705)])
def test_a_prompt_whose_last_rows_see_most(page, rows, length):
    """Fewer tiles than workgroups have room, and keys from none to all: the last tiles are shared, the first are not."""
    t, rng = filled(page, [length], pages=26, page=page, heads=4, d=16, max_pages=26)
    attend(t, rng, 0, [rows], 16, BF16, uniform=True)


@pytest.mark.parametrize("window,sinks", [((1 << 31) - 1, 0), ((1 << 31) - 1, 3), ((1 << 31) - 1, (1 << 31) - 1), ((1 << 31) - 9, 0), (1 << 30, 0), (97, 0)])
@pytest.mark.parametrize("d,dtype", [(64, BF16), (128, F32), (256, F16)])
def test_windows_that_hide_nothing(window, sinks, d, dtype):
    """Up to the end of their range, where a sequence has more rows than positions: those from before its beginning see nothing, the others all that is in front of them."""
    t, rng = filled(d, [3, 40, 97, 0], pages=10, page=32, heads=2, d=d, max_pages=4)
    attend(t, rng, 0, [8, 1, 2, 5], 2, dtype, window=window, sinks=sinks)       # few rows
    got, lse = attend(t, rng, 0, [130, 90, 97, 70], 2, dtype, window=window, sinks=sinks)  # prompts
    again, lse_again = attend(t, np.random.default_rng(1), 0, [8], 1, dtype, window=window, sinks=sinks)
    open_, lse_open = attend(t, np.random.default_rng(1), 0, [8], 1, dtype)
    assert np.array_equal(lse_again, lse_open) and np.array_equal(again, open_)
    assert np.all(lse[:127] == -np.inf) and np.all(np.isfinite(lse[127:130]))


@pytest.mark.parametrize("sequences", [3, 40])
def test_fewer_sinks_give_back_what_more_have_kept(sequences):
    """What no row from the cut on sees is given back, whatever earlier calls had for sinks and windows: pages in front of a long stretch without any, and in the middle of one."""
    t, rng = cache(62, pages=260, page=32, heads=1, d=16, sequences=sequences, max_pages=700)

    def grow(rows, times, **kw):
        rows = [rows, rows // 2] + [0] * (sequences - 2)
        for _ in range(times):
            assert extend(t, rows, **kw)
            append(t, rng, 0, rows)
        t.same()
        invariants(t.o)

    grow(600, 10, window=100, sinks=1280)
    assert np.sum(t.o.table[0] >= 0) >= 40
    grow(1, 2, window=100, sinks=4)                             # 39 pages behind a hundred and more that are gone
    assert np.sum(t.o.table[0] >= 0) <= 1 + 6
    grow(600, 5, window=1000, sinks=6100)                       # (the window's pages become sinks)
    grow(300, 20, window=1000, sinks=6100)
    held = np.flatnonzero(t.o.table[0] >= 0)
    assert np.any((held > 2) & (held < 191)) and np.max(np.diff(held)) > 64
    grow(1, 1, window=1000)                                     # from the middle, and from the beginning
    assert np.sum(t.o.table[0] >= 0) <= 34
    attend(t, rng, 0, [1] * sequences, window=1000)


def test_codes_in_a_large_pool():
    """More pages than a workgroup looks at in one turn: what is copied, written and packed there, code by code."""
    t, rng = cache(63, pages=9000, page=32, layers=1, heads=1, d=16, sequences=60, max_pages=300)
    t.o.codes[...] = rng.integers(-127, 128, t.o.codes.shape)
    t.o.scales[...] = rng.random(t.o.scales.shape)
    t = Held(t.o)
    assert extend(t, [273 * 32] * 30, list(range(30, 60)))      # (8190 pages in front)
    ids = list(range(30))
    rows = rng.integers(1, 900, 30)
    assert extend(t, rows, ids)
    append(t, rng, 0, rows, sequences=ids)
    t.same()
    fork(t, rng.integers(0, 15, 30), ids)
    assert extend(t, [3] * 30, ids)
    append(t, rng, 0, [3] * 30, sequences=ids)
    t.same()
    assert np.max(t.o.table) > 8192
    assert extend(t, [0] * 6, [3, 4, 5, 31, 40, 59], cut=[0] * 6)
    t.o.compact()
    t.cache.compact()
    t.same()
    invariants(t.o)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_tens_of_thousands_of_positions(dtype):
    t, rng = cache(64, pages=700, page=64, heads=2, d=64, sequences=2, max_pages=640)
    t.o.lengths[:] = 40001, 130
    t.o.table[0, :626], t.o.table[1, :3] = rng.permutation(697)[:626], [697, 698, 699]
    t.o.refs[t.o.table[t.o.table >= 0]] = 1
    t.o.codes[...] = rng.integers(-127, 128, t.o.codes.shape)
    t.o.scales[...] = 0.2 + rng.random(t.o.scales.shape)
    t = Held(t.o)
    attend(t, rng, 0, [1, 1], 4, dtype, uniform=True)
    attend(t, rng, 0, [5, 2], 4, dtype, window=33000, sinks=700)
    attend(t, rng, 0, [40, 1], 4, dtype)                        # a prompt
