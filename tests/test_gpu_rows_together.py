"""The operators on rows as a decoding step uses them: a norm in front of 4-bit projections, the positions on their results in place, then
a 4-bit head behind a norm, rules on its logits and the statistics; captured once, replayed with other tokens."""
import numpy as np
import pytest

import paper_2302_07863_amd as pkg
from paper_2302_07863_amd import binding as b
from tests.hipmem import DeviceArray, H2D, hip
from tests.rows import BF16, F16, F32, Graph, HALF_STEP, Rows, Stream, U32, close, mask_words, normed, pack, ruled, scales_of, turned, unpack, weights
from tests.test_gpu_quant import tolerance

pytestmark = pytest.mark.gpu


def matrix(rng, n, k, group, zeros):
    codes, scales, z = pkg.quant_round(rng.normal(0, 0.05, (n, k)).astype(np.float32), group, F16, zeros)
    values = scales_of(scales, F16)
    return pkg.Quant(n, k, group, codes, scales, F16, z), (weights(codes, values, z, k, group), np.abs(values)[:, np.arange(k) // group])


def write(dev, host):
    host = np.ascontiguousarray(host)
    assert host.nbytes <= dev.nbytes and hip().hipMemcpy(dev.ptr, host.ctypes.data, host.nbytes, H2D) == 0


@pytest.mark.parametrize("rows", [1, 7, 33])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_step(rows, dtype):
    rng = np.random.default_rng(rows)
    d, heads, kv, d_head, vocab, rot, cap = 320, 5, 2, 64, 5009, 48, 40
    (wqkv, mqkv), (wo, mo), (whead, mhead) = (matrix(rng, n, k, g, z) for n, k, g, z in
                                              (((heads + 2 * kv) * d_head, d, 64, True), (d, heads * d_head, 32, False), (vocab, d, 128, True)))
    gain = rng.uniform(0.5, 1.5, (2, d)).astype(np.float32)
    gains = DeviceArray(gain)
    width = (heads + 2 * kv) * d_head
    word = np.float32 if dtype == F32 else np.uint16
    x = Rows(np.zeros((rows, d), word), d + 8)
    qkv, o = Rows(np.zeros((rows, width), word)), Rows(np.zeros((rows, d), word))
    logits, out = Rows(np.zeros((rows, vocab), np.float32), vocab + 3), Rows(np.zeros((rows, vocab), np.float32))
    positions, tokens, lengths, starts = (DeviceArray(np.zeros(s, np.int32)) for s in (rows, (rows, cap), rows, rows))
    penalties, targets = DeviceArray(np.array([1.3, 0.25, 0.5], np.float32)), DeviceArray(np.zeros(rows, np.int32))
    words = (vocab + 31) // 32
    mask = DeviceArray(np.zeros((rows, words), np.uint32))
    stats = DeviceArray(nbytes=rows * b.ROW_STATS_DTYPE.itemsize)
    rotary, rules = pkg.Rotary(rot_dim=rot, halves=True, base=500000.0), pkg.Rules(vocab, rows)
    size = 4 if dtype == F32 else 2

    def step(stream):
        wqkv.matmul(x.ptr, dtype, rows, qkv.ptr, dtype, x_stride=d + 8, gain=gains.ptr.value, eps=1e-6, stream=stream)
        rotary.apply(d_head, dtype, rows, pkg.RotaryRows(qkv.ptr, qkv.ptr, heads, width, d_head, width, d_head),
                     pkg.RotaryRows(qkv.ptr + heads * d_head * size, qkv.ptr + heads * d_head * size, kv, width, d_head, width, d_head),
                     positions=positions.ptr.value, stream=stream)
        wo.matmul(qkv.ptr, dtype, rows, o.ptr, dtype, x_stride=width, stream=stream)
        whead.matmul(o.ptr, dtype, rows, logits.ptr, F32, y_stride=vocab + 3, gain=gains.ptr.value + 4 * d, eps=1e-6, scale=3.0, stream=stream)
        rules.apply(logits.ptr, F32, rows, out=out.ptr, stats=stats.ptr.value, targets=targets.ptr.value, logits_stride=vocab + 3, tokens=tokens.ptr.value,
                    tokens_stride=cap, lengths=lengths.ptr.value, starts=starts.ptr.value, penalties=penalties.ptr.value, mask=mask.ptr.value, mask_stride=words,
                    max_tokens=cap, stream=stream)

    stream = Stream()
    graph = None
    for turn in range(4):
        xv = rng.normal(0, 1, (rows, d))
        allowed = rng.random((rows, vocab)) < 0.5
        allowed[:, 17] = True
        ids, n, first = rng.integers(0, vocab, (rows, cap)).astype(np.int32), rng.integers(0, cap + 1, rows).astype(np.int32), rng.integers(0, 9, rows).astype(np.int32)
        pos, tgt = rng.integers(0, 100000, rows).astype(np.int32), rng.integers(0, vocab, rows).astype(np.int32)
        xw = pack(xv, dtype)
        x._view(x.host)[...] = xw
        for dev, host in ((x.dev, x.host), (positions, pos), (tokens, ids), (lengths, n), (starts, first), (targets, tgt), (mask, mask_words(allowed))):
            write(dev, host)
        if graph is None:
            step(stream.h.value)
            stream.sync()
            graph = Graph(stream, step)
        else:
            graph.replay()
            stream.sync()
        # each operator from what the one before it left, so that a tolerance is one operator's
        xs, q, os_, z = unpack(x.get(), dtype), unpack(qkv.get(), dtype).reshape(rows, -1, d_head), unpack(o.get(), dtype), logits.get().astype(np.float64)
        f, magnitude = rotary.frequencies()

        def product(a, w, g, y_dtype):
            an = normed(a, g, 1e-6) if g is not None else a
            y = an @ w[0].T
            return y, tolerance(an, w[1], y, y_dtype)

        want, tol = product(xs, mqkv, gain[0].astype(np.float64), dtype)
        want, tol = want.reshape(rows, -1, d_head), tol.reshape(rows, -1, d_head)
        close(q[:, heads + kv:], want[:, heads + kv:], tol[:, heads + kv:])
        turn_tol = np.max(tol, axis=2, keepdims=True) * 2 + np.max(np.abs(want), axis=2, keepdims=True) * (2 * HALF_STEP[dtype] + 4 * U32)
        close(q[:, :heads + kv], turned(want[:, :heads + kv], pos, f, magnitude, True), turn_tol[:, :heads + kv])
        want, tol = product(q[:, :heads].reshape(rows, -1), mo, None, dtype)
        close(os_, want, tol)
        want, tol = product(os_, mhead, gain[1].astype(np.float64), F32)
        close(z, 3.0 * want, 3.0 * tol + 2 * U32 * np.abs(3.0 * want))
        got, st = out.get().astype(np.float64), stats.to_host(b.ROW_STATS_DTYPE, rows)
        for r in range(rows):
            w = ruled(z[r], ids[r], n[r], first[r], (1.3, 0.25, 0.5), allowed=allowed[r])
            np.testing.assert_array_equal(np.isneginf(got[r]), ~allowed[r])
            at = allowed[r]
            # up to four roundings of the value or of one of the penalties it meets; frequency times a count is at most 0.25 * 40
            close(got[r][at], w[at], 4 * U32 * (np.abs(w[at]) + 1.3 * np.abs(z[r][at]) + 10.5))
            assert st["argmax"][r] == int(np.argmax(got[r])) and st["zmax"][r] == np.max(got[r])
            lse = np.log(np.sum(np.exp(got[r] - np.max(got[r])))) + np.max(got[r])
            assert abs(st["lse"][r] - lse) <= 1e-5 + 2 * U32 * abs(lse)
            assert st["z_target"][r] == got[r][tgt[r]]


def test_errors_of_other_calls_are_not_theirs():
    """A refused allocation, the caller's or one of the library's own that has told of it, is not reported again by the calls behind it."""
    import ctypes as C
    import bild_inputs as bi
    from tests.test_gpu_parity import Rig, TOY_VARIANTS
    rng = np.random.default_rng(3)
    R = Rig(bi.toy_pair(**TOY_VARIANTS["f32-relu-tied"]))
    st = R.state(R.cfg.max_new, 3)
    st.encode(R.src)
    x, y, z = (Rows(pack(rng.standard_normal((120, n)), BF16)) for n in (264, 12300, 264))
    rules, rotary, stats = pkg.Rules(264, 120), pkg.Rotary(24), DeviceArray(nbytes=120 * 16)

    def callers():
        p = C.c_void_p()
        assert hip().hipMalloc(C.byref(p), C.c_size_t(1 << 50)) != 0

    def librarys():
        with pytest.raises(pkg.BildError) as e:
            pkg.Quant(1 << 24, 1 << 20, 32, x.ptr, x.ptr, F16)        # (8 TB: nothing is read before there is room for it)
        assert e.value.code == b.ENOMEM

    def steps():
        st.small_step(0.0)
        st.set_rules((1.2, 0.0, 0.0))
        st.small_step(0.0)
        st.set_rules()

    for fail in (callers, librarys):
        calls = [lambda: matrix(rng, 40, 264, 32, True), lambda: pkg.Quant(4, 32, 32, np.zeros((4, 16), np.uint8), np.full((4, 1), 0x3F80, np.uint16), BF16),
                 lambda: rules.apply(z.ptr, BF16, 120, out=z.ptr, stats=stats.ptr.value),
                 lambda: rotary.apply(24, BF16, 120, pkg.RotaryRows(z.ptr, z.ptr, 11, 264, 24, 264, 24))]
        for n, rows in ((40, 3), (12300, 3), (12300, 120), (40, 120)):
            q = matrix(rng, n, 264, 32, True)[0]
            calls.append(lambda q=q, rows=rows: q.matmul(x.ptr, BF16, rows, y.ptr, BF16))
        for call in calls + ([steps] if fail is librarys else []):
            fail()
            call()
