"""Rules on logits against the definition in 64 bits: every rule alone and together, types, odd vocabularies, strides, masks that leave nothing,
infinities and NaN, streams and graphs."""
import numpy as np
import pytest

import paper_2302_07863_amd as pkg
from paper_2302_07863_amd import binding as b
from tests.hipmem import DeviceArray, hip
from tests.rows import BF16, F16, F32, HALF_STEP, TINY, U32, Graph, Rows, Stream, mask_words, pack, ruled, unpack

pytestmark = pytest.mark.gpu
I32 = np.int32


class Call:
    """Device copies of a call's arrays, and the expectation of every row."""

    def __init__(self, z, dtype, tokens=None, lengths=None, starts=None, penalties=None, bias_ids=None, bias=None, counts=None, allowed=None, targets=None,
                 stride=None, first=0):
        self.rows, self.vocab = z.shape
        self.dtype, self.words = dtype, pack(z, dtype)
        self.logits, self.out = Rows(self.words, stride, first), Rows(pack(np.zeros(z.shape), dtype), stride, first)
        self.stats = DeviceArray(nbytes=16 * self.rows)
        self.kw, self.keep = {}, []
        r = self.rows

        def dev(a, t):
            a = np.ascontiguousarray(a, dtype=t)
            self.keep.append(DeviceArray(a))
            return self.keep[-1].ptr.value

        def per_row(a):
            return None if a is None else [a[i if len(a) == r and r > 1 or len(a) > 1 else 0] for i in range(r)]

        want = dict(zip(("tokens", "penalties", "bias_ids", "bias", "allowed"), map(per_row, (tokens, penalties, bias_ids, bias, allowed))))
        self.lens = lengths if lengths is not None else ([len(tokens[0])] * r if tokens is not None else None)
        if tokens is not None:
            tokens = np.asarray(tokens, I32)
            self.kw.update(tokens=dev(tokens, I32), tokens_stride=0 if len(tokens) == 1 else tokens.shape[1], max_tokens=tokens.shape[1],
                           lengths=dev(self.lens, I32), penalties=dev(penalties, np.float32), penalties_stride=0 if len(penalties) == 1 else 1)
            if starts is not None:
                self.kw.update(starts=dev(starts, I32))
        if bias_ids is not None:
            bias_ids = np.asarray(bias_ids, I32)
            self.kw.update(bias_ids=dev(bias_ids, I32), bias=dev(bias, np.float32), bias_stride=0 if len(bias_ids) == 1 else bias_ids.shape[1],
                           max_bias=bias_ids.shape[1])
            if counts is not None:
                self.kw.update(bias_counts=dev(counts, I32))
        if allowed is not None:
            words = mask_words(allowed)
            self.kw.update(mask=dev(words, np.uint32), mask_stride=0 if len(words) == 1 else words.shape[1])
        if targets is not None:
            self.kw.update(targets=dev(targets, I32))
        self.targets = targets
        v = unpack(self.words, dtype)
        self.want, self.size = [], []
        for i in range(r):
            n = None if counts is None else min(max(int(counts[i]), 0), bias_ids.shape[1])
            args = dict(tokens=want["tokens"] and want["tokens"][i], length=self.lens is not None and self.lens[i], start=0 if starts is None else starts[i],
                        penalties=want["penalties"] and want["penalties"][i], bias_ids=want["bias_ids"] and want["bias_ids"][i][:n],
                        bias=want["bias"] and want["bias"][i][:n])
            with np.errstate(all="ignore"):
                self.want.append(ruled(v[i], allowed=want["allowed"] and want["allowed"][i], **args))
                # what a rounding can be half a step of: the largest number on the way
                size = np.abs(v[i]) * (max(penalties[0][0], 1 / penalties[0][0]) * 1.5 if penalties is not None else 1.0)
                if penalties is not None:
                    size = size + max(abs(float(p[1])) for p in penalties) * max(self.lens + [0]) + max(abs(float(p[2])) for p in penalties)
                if bias is not None:
                    size = size + np.max(np.abs(np.asarray(bias, np.float64)), initial=0.0)
            self.size.append(size)

    def run(self, rules, stream=None, **kw):
        rules.apply(self.logits.ptr, self.dtype, self.rows, **{**dict(out=self.out.ptr, stats=self.stats.ptr.value, logits_stride=self.logits.stride,
                                                                       out_stride=self.out.stride, stream=stream), **self.kw, **kw})

    def check(self, logits=True, stats=True):
        got = unpack(self.out.get(), self.dtype) if logits else None
        st = self.stats.to_host(b.ROW_STATS_DTYPE, self.rows)
        for i in range(self.rows):
            w, size = self.want[i], self.size[i]
            tol = 5 * U32 * size                          # division or product, count's product, two differences, a sum
            if logits:
                gone = np.isneginf(w)
                assert np.array_equal(np.isneginf(got[i]), gone)
                with np.errstate(invalid="ignore"):
                    bad = np.abs(got[i] - w) > tol + HALF_STEP[self.dtype] * np.abs(w) + TINY[self.dtype]
                bad &= ~gone
                assert not bool(np.any(bad)), (i, int(np.argmax(bad)))
            if stats:
                m = float(np.max(w))
                if m == -np.inf:
                    assert st["argmax"][i] == -1 and st["zmax"][i] == -np.inf and st["lse"][i] == -np.inf
                else:
                    t = float(np.max(tol[np.isfinite(w)]))
                    a = int(st["argmax"][i])
                    assert abs(st["zmax"][i] - m) <= t
                    assert a == int(np.argmax(w)) or (w[a] >= m - 2 * t and w[a] < m), (i, a, int(np.argmax(w)))
                    lse = m + np.log(np.sum(np.exp(w - m)))
                    # an exponential is off by 2^-22 and its argument by tol, a sum by half a step for each of its terms in turn: a thread's, then those of 64 lanes,
                    # 4 waves and the row's workgroups
                    depth = self.vocab / 256 + 40
                    assert abs(st["lse"][i] - lse) <= 2 * t + 2.0 ** -22 + depth * U32 + 2 * U32 * abs(lse), (i, st["lse"][i], lse)
                if self.targets is None or not 0 <= self.targets[i] < self.vocab:
                    assert np.isnan(st["z_target"][i])
                else:
                    v = w[self.targets[i]]
                    assert st["z_target"][i] == v if np.isinf(v) else abs(st["z_target"][i] - v) <= tol[self.targets[i]]


def text(rng, rows, n, vocab):
    return np.minimum(vocab - 1, (vocab ** rng.random((rows, n))).astype(I32) - 1)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", [1, 7, 31, 32, 33, 1000, 2048, 2049, 8191, 32128, 50257])
def test_everything_together(dtype, vocab):
    rng = np.random.default_rng(vocab + dtype)
    rules = pkg.Rules(vocab, 8)
    for rows in (1, 5):
        z = 3 * rng.standard_normal((rows, vocab))
        n, nb = 300, 20
        allowed = rng.random((rows, vocab)) < 0.7
        allowed[0, 0] = True
        call = Call(z, dtype, text(rng, rows, n, vocab), [int(x) for x in rng.integers(0, n + 1, rows)], [int(x) for x in rng.integers(0, 100, rows)],
                    1.2 + rng.random((rows, 3)).astype(np.float32), rng.integers(0, vocab, (rows, nb)), rng.standard_normal((rows, nb)).astype(np.float32),
                    [int(x) for x in rng.integers(0, nb + 1, rows)], allowed, [int(x) for x in rng.integers(-1, vocab + 1, rows)])
        call.run(rules)
        call.check()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_each_rule_alone(dtype):
    rng = np.random.default_rng(1)
    vocab, rows = 4099, 3
    rules = pkg.Rules(vocab, rows)
    z = 3 * rng.standard_normal((rows, vocab))
    for kw in (dict(), dict(tokens=text(rng, rows, 50, vocab), penalties=[[1.5, 0, 0]]), dict(tokens=text(rng, rows, 50, vocab), penalties=[[1, 0.5, 0]]),
               dict(tokens=text(rng, rows, 50, vocab), penalties=[[1, 0, 0.5]], starts=[10, 0, 60]),
               dict(tokens=text(rng, 1, 50, vocab), penalties=[[0.7, -0.5, -1.0]], lengths=[0, 20, 50]),
               dict(bias_ids=rng.integers(0, vocab, (rows, 9)), bias=rng.standard_normal((rows, 9)).astype(np.float32)),
               dict(bias_ids=rng.integers(0, vocab, (1, 1023)), bias=rng.standard_normal((1, 1023)).astype(np.float32)),
               dict(allowed=rng.random((rows, vocab)) < 0.01), dict(allowed=rng.random((1, vocab)) < 0.5)):
        call = Call(z, dtype, targets=[5, vocab - 1, 0], **kw)
        call.run(rules)
        call.check()
    # without rules every bit of the logits stays
    call = Call(z, dtype)
    call.run(rules)
    assert call.out.get().tobytes() == call.words.tobytes()


def test_rows_of_a_review_share_a_sequence():
    rng = np.random.default_rng(2)
    vocab, rows = 32000, 11
    call = Call(rng.standard_normal((rows, vocab)), F32, text(rng, 1, 500, vocab), [490 + i for i in range(rows)], [40] * rows, [[1.3, 0.2, 0.1]],
                targets=[int(t) for t in rng.integers(0, vocab, rows)], allowed=rng.random((rows, vocab)) < 0.5)
    call.run(pkg.Rules(vocab, 32))
    call.check()


def test_ids_outside_repeated_ids_and_lengths_outside():
    rng = np.random.default_rng(3)
    vocab = 700
    rules = pkg.Rules(vocab, 4)
    z = rng.standard_normal((4, vocab))
    tokens = rng.integers(0, vocab, (4, 64))
    tokens[:, 3], tokens[:, 9], tokens[:, 11], tokens[0] = -1, vocab, 2 ** 31 - 1, 5
    ids = np.array([[5, 6, 5, -1, vocab, 6, 5, 699]] * 4)
    bias = np.array([[1, 2, 3, 100, 100, -2, 0.5, 7]] * 4, np.float32)
    call = Call(z, F32, tokens, [64, 200, -5, 10], [0, -3, 2, 10], [[1.1, 0.3, 0.2]] * 4, ids, bias, [8, 3, 99, -1])
    call.run(rules)
    call.check()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_masks_infinities_and_nan(dtype):
    """A row of which nothing is left, one id left, the type's lowest value where masked and where not, what is not a number behind a mask and not."""
    rng = np.random.default_rng(4)
    vocab = 3001
    low = {F32: -3.4028234e38, BF16: -3.3895314e38, F16: -65504.0}[dtype]
    z = rng.standard_normal((9, vocab))
    allowed = rng.random((9, vocab)) < 0.5
    allowed[0] = False
    allowed[1] = False
    allowed[1, 2999] = True
    z[2, ::2], z[3] = low, low
    allowed[3] = True
    allowed[4] = True
    z[4] = -np.inf
    z[5, ~allowed[5]] = np.nan
    z[6, ~allowed[6]] = np.inf
    z[7, 17], allowed[7, 17] = np.nan, True
    z[8, 19], allowed[8, 19] = np.inf, True
    rules = pkg.Rules(vocab, 9)
    call = Call(z[:7], dtype, allowed=allowed[:7], targets=[0, 2999, 1, 3000, 5, 6, 7])
    call.run(rules)
    call.check()
    odd = Call(z[7:], dtype, allowed=allowed[7:])
    odd.run(rules)
    st = odd.stats.to_host(b.ROW_STATS_DTYPE, 2)
    finite = np.where(allowed[7] & np.isfinite(z[7]), unpack(odd.words[0], dtype), -np.inf)
    assert np.isnan(st["lse"][0]) and st["argmax"][0] == int(np.argmax(finite)) and st["zmax"][0] == np.max(finite)
    assert st["zmax"][1] == np.inf and st["lse"][1] == np.inf and st["argmax"][1] == 19
    # all NaN
    none = Call(np.full((1, vocab), np.nan), dtype)
    none.run(rules)
    st = none.stats.to_host(b.ROW_STATS_DTYPE, 1)
    assert np.isnan(st["lse"][0]) and st["argmax"][0] == -1


def test_ties_go_to_the_lowest_id():
    for vocab in (40, 5000, 100003):
        rules = pkg.Rules(vocab, 2)
        z = np.zeros((2, vocab))
        z[1, [vocab // 3, vocab // 3 + 1, vocab - 1]] = 4.0
        for dtype in (F32, F16):
            call = Call(z, dtype)
            call.run(rules)
            st = call.stats.to_host(b.ROW_STATS_DTYPE, 2)
            assert list(st["argmax"]) == [0, vocab // 3]
            call.check()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place_strided_statistics_only_logits_only(dtype):
    rng = np.random.default_rng(5)
    vocab, rows = 1500, 4
    rules = pkg.Rules(vocab, rows)
    kw = dict(tokens=text(rng, rows, 90, vocab), penalties=[[1.4, 0.1, 0.2]], allowed=rng.random((rows, vocab)) < 0.6, targets=[1, 2, 3, 4])
    z = rng.standard_normal((rows, vocab))
    for stride, first in ((vocab, 0), (vocab + 5, 3), (vocab + 1, 1)):
        call = Call(z, dtype, stride=stride, first=first, **kw)
        call.run(rules)
        call.check()
        plain = call.out.get()
        call.run(rules, out=None)
        call.check(logits=False)
        call.run(rules, stats=None)
        call.check(stats=False)
        call.run(rules, out=call.logits.ptr, out_stride=call.logits.stride)
        assert call.logits.get().tobytes() == plain.tobytes()
        call.check(logits=False)


def test_long_histories_and_many_rows():
    rng = np.random.default_rng(6)
    vocab = 20000
    tokens = text(rng, 2, 100000, vocab)
    tokens[1] = 12345                                        # (one id a hundred thousand times)
    call = Call(rng.standard_normal((2, vocab)), F32, tokens, [100000, 100000], [0, 1], [[1.1, 0.001, 0.1]] * 2)
    call.run(pkg.Rules(vocab, 2))
    call.check()
    vocab, rows = 300, 3000
    call = Call(rng.standard_normal((rows, vocab)), BF16, text(rng, rows, 5, vocab), penalties=[[1.1, 0.5, 0.1]] * rows, targets=[int(t) for t in rng.integers(0, vocab, rows)])
    call.run(pkg.Rules(vocab, rows))
    call.check()


def test_one_handle_for_calls_of_every_size_in_turn():
    """What a call leaves in the handle shows in no later one."""
    rng = np.random.default_rng(7)
    vocab = 70001
    rules = pkg.Rules(vocab, 40)
    for rows in (40, 1, 17, 1, 3, 40):
        call = Call(rng.standard_normal((rows, vocab)), F16, allowed=rng.random((1, vocab)) < 0.9, targets=[int(t) for t in rng.integers(0, vocab, rows)])
        call.run(rules)
        call.check()


def test_streams_and_captured_launches():
    rng = np.random.default_rng(8)
    vocab, rows = 32128, 3
    eager_rules, graph_rules = pkg.Rules(vocab, rows), pkg.Rules(vocab, rows)
    stream = Stream()
    z = rng.standard_normal((rows, vocab))
    call = Call(z, F32, text(rng, rows, 60, vocab), [20, 30, 40], penalties=[[1.3, 0.2, 0.4]], targets=[7, 8, 9])
    graph = Graph(stream, lambda st: call.run(graph_rules, stream=st))
    for step in range(4):
        words = pack(rng.standard_normal((rows, vocab)), F32)
        stream.sync()
        assert hip().hipMemcpy(call.logits.dev.ptr, words.ctypes.data, words.nbytes, 1) == 0
        graph.replay()
        stream.sync()
        replayed = call.out.get(), call.stats.to_host(np.uint8, 16 * rows)
        call.run(eager_rules)
        assert np.array_equal(call.out.get(), replayed[0])
        assert np.array_equal(call.stats.to_host(np.uint8, 16 * rows), replayed[1])


def test_refusals():
    rules = pkg.Rules(100, 4)
    call = Call(np.zeros((4, 100)), F32, np.zeros((4, 8), I32), penalties=[[1, 0, 0]], bias_ids=np.zeros((4, 2), I32), bias=np.zeros((4, 2)))
    call.run(rules)
    for kw, code in ((dict(rows=0), b.EINVAL), (dict(rows=5), b.ECAP), (dict(logits=None), b.EINVAL), (dict(out=None, stats=None), b.EINVAL), (dict(dtype=3), b.EINVAL),
                     (dict(lengths=None), b.EINVAL), (dict(penalties=None), b.EINVAL), (dict(penalties_stride=2), b.EINVAL), (dict(bias=None), b.EINVAL),
                     (dict(max_tokens=-1), b.EINVAL), (dict(max_tokens=1 << 20), b.EINVAL), (dict(max_bias=1024), b.EINVAL), (dict(max_bias=-1), b.EINVAL),
                     (dict(out=call.logits.ptr, out_stride=101), b.EINVAL)):
        a = {**dict(logits=call.logits.ptr, dtype=F32, rows=4, out=call.out.ptr, stats=call.stats.ptr.value), **call.kw, **kw}
        with pytest.raises(pkg.BildError) as e:
            rules.apply(**a)
        assert e.value.code == code, kw
    for vocab, rows in ((0, 1), (1, 0), (1 << 25, 1), (10, 65536)):
        with pytest.raises(pkg.BildError) as e:
            pkg.Rules(vocab, rows)
        assert e.value.code == b.EINVAL


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_statistics_of_logits_of_any_size(dtype):
    """Whole rows, whole ranges of workgroups and every other id at one value of any size, beside ordinary logits."""
    rng = np.random.default_rng(9)
    vocab = 9001
    fills = [s * v for v in (65504.0, 1e6, 3e6, 4.3e6, 1e7, 1e9, 3.1e9, 4.4e9, 1e10, 1e12, 1e15, 1e20, 9e29, 1.1e30, 1e38) for s in (-1.0, 1.0)]
    z = rng.standard_normal((4 * len(fills), vocab))
    for i, v in enumerate(fills):
        z[4 * i], z[4 * i + 1, 2000:8000], z[4 * i + 2, ::2] = v, v, v
        z[4 * i + 3] = v * (1 + rng.random(vocab) / 16)
    rules = pkg.Rules(vocab, len(z))
    for rows in (len(z), 4):                                # (ranges of other lengths)
        for first in range(0, len(z), rows):
            call = Call(z[first:first + rows], dtype)
            call.run(rules)
            assert call.out.get().tobytes() == call.words.tobytes()
            st, w = call.stats.to_host(b.ROW_STATS_DTYPE, rows), unpack(call.words, dtype)
            for i in range(rows):
                m = np.max(w[i])
                lse = m + np.log(np.sum(np.exp(w[i] - m)))
                # as in Call.check, with nothing off before the exponentials but a half step of each argument: below 10 on average, as the sum is of 9001
                tol = 2.0 ** -22 + (vocab / 256 + 40 + 20) * U32 + 2 * U32 * abs(lse)
                assert st["zmax"][i] == m and st["argmax"][i] == np.argmax(w[i])
                assert abs(st["lse"][i] - lse) <= tol, (rows, fills[(first + i) // 4], i % 4, st["lse"][i], lse)
