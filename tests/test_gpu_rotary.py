"""Rotary positions of rows against the definition in 64 bits: layouts, parts of a head, scalings, types, strides, in place, gradients;
models whose passes turn by them against the oracle."""
import numpy as np
import pytest

import bild_inputs as bi
import oracle
import paper_2302_07863_amd as pkg
from paper_2302_07863_amd import binding as b
from tests import parity
from tests.hipmem import DeviceArray
from tests.rows import BF16, F16, F32, HALF_STEP, TINY, U32, Graph, Rows, Stream, close, pack, turned, unpack

pytestmark = pytest.mark.gpu


def tolerance(x, want, magnitude, halves, rot, dtype):
    """cos and sin rounded to fp32 (half a step each), a product's rounding, the sum's: 3 half steps of |u| + |v|; then the row type's."""
    both = np.zeros_like(x)
    half = rot // 2
    iu = np.arange(half) if halves else 2 * np.arange(half)
    iv = iu + half if halves else iu + 1
    both[..., iu] = both[..., iv] = np.abs(x[..., iu]) + np.abs(x[..., iv])
    return 3.1 * U32 * magnitude * both + HALF_STEP[dtype] * np.abs(want) + TINY[dtype]


def run(rng, tokens, heads, d_head, dtype, rotary, positions=None, first=0, inverse=False, pad=0, shift=0, in_place=False, stream=None):
    """heads: of queries and keys; pad: words behind every token's heads; shift: words in front of the array."""
    f, m = rotary.frequencies()
    halves, rot = bool(rotary.cfg.layout), rotary.cfg.rot_dim
    pos = np.arange(first, first + tokens) if positions is None else positions
    pd = None if positions is None else DeviceArray(np.asarray(positions, np.int32))
    rows, arrays = [], []
    for h in heads:
        if h == 0:
            rows.append(pkg.RotaryRows())
            arrays.append(None)
            continue
        words = pack(rng.standard_normal((tokens, h * d_head)), dtype)
        src = Rows(words, h * d_head + pad, shift)
        dst = src if in_place else Rows(pack(np.zeros(words.shape), dtype), h * d_head + 2 * pad, shift)
        rows.append(pkg.RotaryRows(src.ptr, dst.ptr, h, src.stride, d_head, dst.stride, d_head))
        arrays.append((words, dst, src))
    rotary.apply(d_head, dtype, tokens, rows[0], rows[1], pd.ptr.value if pd else None, first, inverse, stream)
    for h, a in zip(heads, arrays):
        if a is None:
            continue
        x = unpack(a[0], dtype).reshape(tokens, h, d_head)
        want = turned(x, pos, f, m, halves, inverse)
        got = unpack(a[1].get(), dtype).reshape(tokens, h, d_head)
        close(got, want, tolerance(x, want, m, halves, rot, dtype))
        assert np.array_equal(got[..., rot:], x[..., rot:])


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("d_head,rot", [(128, 128), (64, 64), (80, 32), (128, 2), (96, 94), (40, 38), (2, 2), (17, 6), (256, 256), (1024, 200), (5, 4)])
def test_layouts_and_parts(dtype, halves, d_head, rot):
    rng = np.random.default_rng(d_head * 10 + rot + dtype)
    r = pkg.Rotary(rot, halves)
    for tokens, heads in ((1, (1, 1)), (3, (4, 2)), (37, (2, 1))):
        run(rng, tokens, heads, d_head, dtype, r, first=tokens * 100)
        run(rng, tokens, heads, d_head, dtype, r, first=tokens, pad=3, shift=1)
        run(rng, tokens, heads, d_head, dtype, r, first=5, in_place=True, pad=1)


@pytest.mark.parametrize("kw", [dict(scaling=pkg.ROTARY_LINEAR, factor=4.0), dict(scaling=pkg.ROTARY_BASE, factor=8.0),
                                dict(scaling=pkg.ROTARY_BANDS, factor=8.0, original=8192), dict(scaling=pkg.ROTARY_BANDS, factor=2.0, original=512, low=2.0, high=16.0),
                                dict(scaling=pkg.ROTARY_YARN, factor=16.0, original=4096), dict(scaling=pkg.ROTARY_YARN, factor=4.0, original=2048, magnitude=1.5),
                                dict(base=500000.0)])
def test_scalings_far_out(kw):
    rng = np.random.default_rng(3)
    for halves in (False, True):
        r = pkg.Rotary(128, halves, **kw)
        run(rng, 4, (3, 1), 128, F32, r, positions=[0, 131071, 1 << 20, (1 << 31) - 1])
        run(rng, 2, (2, 2), 128, BF16, r, positions=[-7, -(1 << 31)])


@pytest.mark.parametrize("heads", [(32, 32), (64, 8), (1, 0), (0, 3), (71, 1), (300, 0), (1000, 1)])
def test_heads(heads):
    rng = np.random.default_rng(heads[0])
    for dtype in (F32, BF16):
        run(rng, 5, heads, 64, dtype, pkg.Rotary(64, True), first=9)
        run(rng, 1, heads, 24, dtype, pkg.Rotary(6), first=9)


def test_many_tokens_in_any_order():
    rng = np.random.default_rng(4)
    run(rng, 2111, (4, 2), 64, F16, pkg.Rotary(64), positions=rng.integers(0, 100000, 2111))
    run(rng, 5000, (1, 1), 16, BF16, pkg.Rotary(8, True), positions=np.full(5000, 77))


def test_heads_and_tokens_with_strides():
    """Heads outermost ([head][token][d_head]), and rows of a packed q, k, v buffer turned where they stand."""
    rng = np.random.default_rng(6)
    r = pkg.Rotary(32, True)
    f, m = r.frequencies()
    t, h, d = 9, 5, 32
    words = pack(rng.standard_normal((h * t, d)), F32)
    src, dst = Rows(words), Rows(pack(np.zeros((h * t, d)), F32))
    r.apply(d, F32, t, pkg.RotaryRows(src.ptr, dst.ptr, h, d, t * d, d, t * d))
    x = unpack(words, F32).reshape(h, t, d).transpose(1, 0, 2)
    want = turned(x, np.arange(t), f, m, True)
    got = unpack(dst.get(), F32).reshape(h, t, d).transpose(1, 0, 2)
    close(got, want, tolerance(x, want, m, True, 32, F32))
    hq, hk = 6, 2
    words = pack(rng.standard_normal((t, (hq + 2 * hk) * d)), BF16)
    buf = Rows(words)
    st = buf.stride
    r.apply(d, BF16, t, pkg.RotaryRows(buf.ptr, buf.ptr, hq, st, d, st, d), pkg.RotaryRows(buf.ptr + hq * d * 2, buf.ptr + hq * d * 2, hk, st, d, st, d), first=3)
    x = unpack(words, BF16).reshape(t, -1, d)
    want = turned(x, 3 + np.arange(t), f, m, True)
    want[:, hq + hk:] = x[:, hq + hk:]
    got = unpack(buf.get(), BF16).reshape(t, -1, d)
    close(got, want, tolerance(x, want, m, True, 32, BF16))
    assert np.array_equal(got[:, hq + hk:], x[:, hq + hk:])


def test_inverse_is_the_gradient():
    """inverse turns by minus the angle; <dy, J dx> = <J^T dy, dx>, and differences of the forward give J."""
    rng = np.random.default_rng(7)
    for halves, kw in ((True, dict(scaling=pkg.ROTARY_YARN, factor=4.0, original=512)), (False, dict())):
        r = pkg.Rotary(48, halves, **kw)
        run(rng, 6, (3, 2), 64, F32, r, first=1000, inverse=True)
        t, h, d = 4, 2, 64
        x, dx, dy = (rng.standard_normal((t, h * d)).astype(np.float32) for _ in range(3))

        def fwd(a, inverse=False):
            s, o = Rows(pack(a, F32)), Rows(pack(np.zeros(a.shape), F32))
            r.apply(d, F32, t, pkg.RotaryRows(s.ptr, o.ptr, h, h * d, d, h * d, d), first=33, inverse=inverse)
            return o.get().astype(np.float64)

        gx = fwd(dy, True)
        jdx = fwd(x + dx) - fwd(x)                    # (the map is linear: a difference of any size is exact but for roundings)
        m = r.frequencies()[1]
        # each of the two sides has t * h * d terms with errors of at most 12 half steps of numbers below 2 m (|x| + |dx|) (1 + |dy|)
        lhs, rhs = np.sum(dy * jdx), np.sum(gx * dx)
        assert abs(lhs - rhs) <= 12 * U32 * 4 * m * np.sum((np.abs(x) + np.abs(dx)) * 2 * (1 + np.abs(dy)))


def test_streams_and_captured_launches():
    rng = np.random.default_rng(8)
    r = pkg.Rotary(64, True)
    words = pack(rng.standard_normal((12, 128)), F32)
    src, dst, eager = Rows(words), Rows(pack(np.zeros((12, 128)), F32)), Rows(pack(np.zeros((12, 128)), F32))
    positions = DeviceArray(np.zeros(12, np.int32))
    stream = Stream()

    def launch(out):
        return lambda st: r.apply(64, F32, 12, pkg.RotaryRows(src.ptr, out.ptr, 2, 128, 64, 128, 64), positions=positions.ptr.value, stream=st)

    graph = Graph(stream, launch(dst))
    from tests.hipmem import hip
    for step in range(4):
        pos = (np.arange(12) + 50 * step).astype(np.int32)
        stream.sync()
        assert hip().hipMemcpy(positions.ptr, pos.ctypes.data, pos.nbytes, 1) == 0
        graph.replay()
        stream.sync()
        launch(eager)(None)
        assert np.array_equal(dst.get(), eager.get())


def test_refusals():
    r = pkg.Rotary(64)
    src = Rows(pack(np.zeros((2, 128)), F32))
    good = dict(d_head=64, dtype=F32, tokens=2, q=pkg.RotaryRows(src.ptr, src.ptr, 2, 128, 64, 128, 64))
    r.apply(**good)
    for kw in (dict(tokens=0), dict(d_head=62), dict(d_head=1025), dict(dtype=3), dict(q=pkg.RotaryRows()), dict(q=pkg.RotaryRows(None, src.ptr, 1)),
               dict(q=pkg.RotaryRows(src.ptr, None, 1)), dict(q=pkg.RotaryRows(src.ptr, src.ptr, -1)), dict(first=2 ** 31 - 2, tokens=3),
               dict(q=pkg.RotaryRows(src.ptr, src.ptr, 2, 128, 64, 129, 64)), dict(q=pkg.RotaryRows(src.ptr, src.ptr, 2, 128, 64, 128, 32))):
        with pytest.raises(pkg.BildError) as e:
            r.apply(**{**good, **kw})
        assert e.value.code == b.EINVAL


# ------------------------------------------------------------------------------------------------ models
class Turned(oracle.Model):
    """The oracle's network with the positions of a rotary configuration."""

    def __init__(self, shape, w, rotary):
        super().__init__(shape, w)
        self.r = rotary

    def _qk_pos(self, a, positions):
        f, m = self.r.frequencies()
        x = a.reshape(len(a), self.s.heads, self.s.d_head)
        return turned(x, positions, f, m, bool(self.r.cfg.layout)).reshape(a.shape)


@pytest.mark.parametrize("kw", [dict(), dict(dtype=bi.DT_BF16), dict(dtype=bi.DT_BF16, d=1280, heads=20, d_head=64, d_ff=2560), dict(cross=True)])
@pytest.mark.parametrize("rot", [dict(rot_dim=0, halves=True), dict(rot_dim=8, halves=True, scaling=pkg.ROTARY_YARN, factor=4.0, original=16),
                                 dict(rot_dim=6, scaling=pkg.ROTARY_BANDS, factor=8.0, original=64)])
def test_models_turn_by_them(kw, rot):
    """Prompt, single steps and a review of a model made with rotary positions, logits and cached keys, against the oracle."""
    cfg = bi.toy_pair(**{**dict(act=bi.ACT_SWIGLU, pos=bi.POS_ROPE, cross=False), **kw})
    ws, wl = bi.make_pair_weights(cfg)
    rotary = pkg.Rotary(**{**rot, "rot_dim": rot["rot_dim"] or cfg.large.d_head, "base": 1000.0})
    models = [pkg.Model(pkg.config_from_shape(s), [w[n] for n in bi.tensor_names(s)], rotary.cfg) for s, w in ((cfg.small, ws), (cfg.large, wl))]
    state = pkg.State(pkg.Pair(*models), max_src=40, max_len=80)
    state.debug_enable_logits(True)
    rng = np.random.default_rng(1)
    src = rng.integers(0, cfg.large.vocab, 37 if cfg.large.dtype == bi.DT_BF16 else 21).tolist()
    state.encode(src)
    tol = parity.logit_tol(cfg)
    oracles = [Turned(cfg.small, ws, rotary), Turned(cfg.large, wl, rotary)]
    for _ in range(3):
        state.small_step(0.0)
        y = state.sequence()
        cross = oracles[0].cross_kv(oracles[0].encode(src)) if cfg.small.cross and cfg.small.n_enc else None
        if cfg.small.cross and not cfg.small.n_enc:
            cross = oracles[0].cross_kv(oracles[1].encode(src))
        z = oracles[0].logits_full(y[:-1], cross or [])[-1]
        close(state.debug_logits(pkg.SMALL, 0), z, tol)
    y = state.sequence()
    state.large_verify(float("inf"))
    z = oracles[1].logits_full(y, oracles[1].cross_kv(oracles[1].encode(src)) if cfg.large.cross else [])
    for i in range(4):
        close(state.debug_logits(pkg.LARGE, i), z[len(y) - 4 + i], tol)
    # keys of the first layer are given back in the order the caller knows
    m, s = oracles[1], cfg.large
    pos = np.arange(len(y) - 1)
    k = m._qk_pos(oracle.model.rmsnorm(m.embed(y[:-1], pos), m.w["dec.0.ln1"], s.eps) @ m.w["dec.0.wk"], pos)
    got = state.debug_kv(pkg.LARGE, 0, False, 0, len(pos))
    close(got, k, 1e-4 if s.dtype == bi.DT_F32 else 2.0 ** -8 * np.abs(k) + 1e-4)


def test_a_model_made_with_plain_pairs_is_the_ordinary_one():
    cfg = bi.toy_pair(act=bi.ACT_SWIGLU, pos=bi.POS_ROPE, cross=False)
    ws, wl = bi.make_pair_weights(cfg)
    out = []
    for rotary in (None, pkg.RotaryConfig(0, cfg.large.d_head, 0, 0, cfg.large.rope_base, 1.0, 0, 0, 0)):
        models = [pkg.Model(pkg.config_from_shape(s), [w[n] for n in bi.tensor_names(s)], rotary) for s, w in ((cfg.small, ws), (cfg.large, wl))]
        state = pkg.State(pkg.Pair(*models), max_src=16, max_len=60)
        out.append(state.generate(list(range(3, 15)), 0.5, 2.0, 30)[0])
    assert out[0] == out[1]


def test_a_model_that_host_memory_does_not_hold():
    """No memory for the staging of a tensor is an error of the call, and the process goes on."""
    import gc
    import resource
    gc.collect()                                                      # (what is freed later would make room)
    vocab, d = 1 << 17, 1024                                          # (half a gigabyte of embedding, never touched)
    cfg = b.ModelConfig(n_enc_layers=0, n_dec_layers=1, d_model=d, n_heads=16, d_head=64, d_ff=1024, act=bi.ACT_SWIGLU, pos=bi.POS_ROPE, vocab=vocab, tied_head=1, dtype=0,
                        cross_attn=0, logit_scale=1.0, embed_scale=1.0, norm_eps=1e-6, rope_base=10000.0)
    small = np.zeros((d, d), np.float32)
    tensors = [np.zeros((vocab, d), np.float32)] + [small] * (b.lib().bild_model_num_tensors(cfg) - 1)
    DeviceArray(np.zeros(1, np.float32))                              # (the runtime is there)
    now = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
    was = resource.getrlimit(resource.RLIMIT_AS)
    resource.setrlimit(resource.RLIMIT_AS, (now + (128 << 20), was[1]))
    try:
        codes = []
        for rotary in (None, b.RotaryConfig(1, 64, 0, 0, 10000.0, 1.0, 0, 0, 0)):
            with pytest.raises(pkg.BildError) as e:
                pkg.Model(cfg, tensors, rotary)
            codes.append(e.value.code)
    finally:
        resource.setrlimit(resource.RLIMIT_AS, was)
    assert codes == [b.ENOMEM] * 2


def test_the_largest_angles():
    """Up to 2^48 radians, where a step of the angle is 2^-5: the same 64-bit product here and there, so that its cosine is the same."""
    rng = np.random.default_rng(12)
    for halves in (False, True):
        run(rng, 4, (2, 1), 64, F32, pkg.Rotary(64, halves, base=6e-6), positions=[(1 << 31) - 1, -(1 << 31), 123456789, 3])
