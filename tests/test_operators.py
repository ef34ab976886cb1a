"""Host side of the operators on rows: rounding to 4 bits, rotary frequencies, refusals that come before any device work."""
import ctypes as C

import numpy as np
import pytest

import paper_2302_07863_amd as pkg
from paper_2302_07863_amd import binding as b
from tests.rows import BF16, F16, HALF_STEP, TINY, scales_of, weights


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("n,k", [(1, 1), (3, 31), (16, 128), (5, 129), (33, 200)])
def test_rounding(group, dtype, zeros, n, k):
    rng = np.random.default_rng(n * 100 + k)
    w = (0.02 * rng.standard_normal((n, k)) + (0.03 if zeros else 0.0)).astype(np.float32)
    codes, scales, z = pkg.quant_round(w, group, dtype, zeros)
    s = scales_of(scales, dtype)
    back = weights(codes, s, z, k, group)
    g = np.arange(k) // group
    # half a step, and at the ends of the range what the scale's rounding moves 7 (15) steps by; fp32 divisions before rounding are off by far less
    step = s[:, g]
    slack = (15 if zeros else 7) * step * (2.0 ** -8 if dtype == BF16 else 2.0 ** -11)
    assert np.all(np.abs(back - w) <= 0.5 * step * (1 + 1e-5) + slack + (0.5 * step if zeros else 0)), np.max(np.abs(back - w) / step)
    if not zeros:
        big = np.array([[np.max(np.abs(w[i, g == j])) for j in range(g[-1] + 1)] for i in range(n)])
        assert np.all(np.abs(s - big / 7) <= big / 7 * (2.0 ** -8 if dtype == BF16 else 2.0 ** -11) * 1.001)
    again = pkg.quant_round(np.ascontiguousarray(w.T), group, dtype, zeros, inputs_first=True)
    assert all(np.array_equal(a, c) for a, c in zip((codes, scales), again[:2]))
    if k % 2:
        assert np.all(codes[:, -1] >> 4 == 0)


def test_rounding_of_zero_groups_and_refusals():
    codes, scales, _ = pkg.quant_round(np.zeros((2, 64), np.float32), 32)
    assert np.all(weights(codes, scales_of(scales, F16), None, 64, 32) == 0)
    for bad in (np.inf, np.nan):
        w = np.zeros((2, 64), np.float32)
        w[1, 5] = bad
        with pytest.raises(pkg.BildError) as e:
            pkg.quant_round(w, 32)
        assert e.value.code == b.EINVAL
    with pytest.raises(pkg.BildError):
        pkg.quant_round(np.full((1, 32), 1e6, np.float32), 32, F16)       # (a scale beyond fp16)
    pkg.quant_round(np.full((1, 32), 1e6, np.float32), 32, BF16)
    for kw in (dict(group=16), dict(group=32, scale_dtype=0), dict(group=32, scale_dtype=7), dict(group=0)):
        with pytest.raises(pkg.BildError) as e:
            pkg.quant_round(np.zeros((2, 64), np.float32), **kw)
        assert e.value.code == b.EINVAL


def test_frequencies():
    f, m = pkg.Rotary(64, base=10000.0).frequencies()
    want = 10000.0 ** (-2 * np.arange(32) / 64)
    assert m == 1.0 and np.allclose(f, want, rtol=1e-14)
    assert np.allclose(pkg.Rotary(64, scaling=pkg.ROTARY_LINEAR, factor=4.0).frequencies()[0], want / 4, rtol=1e-14)
    # the changed base leaves the first pair and divides the last one's frequency by the factor
    g = pkg.Rotary(64, scaling=pkg.ROTARY_BASE, factor=8.0).frequencies()[0]
    assert g[0] == 1.0 and abs(g[-1] * 8 / want[-1] - 1) < 1e-12
    turns = 8192 * want / (2 * np.pi)
    g = pkg.Rotary(64, scaling=pkg.ROTARY_BANDS, factor=8.0, original=8192).frequencies()[0]
    assert np.allclose(g[turns >= 4], want[turns >= 4], rtol=1e-14) and np.allclose(g[turns <= 1], want[turns <= 1] / 8, rtol=1e-14)
    mid = (turns > 1) & (turns < 4)
    assert np.any(mid) and np.all((g[mid] < want[mid]) & (g[mid] > want[mid] / 8))
    turns = 4096 * want / (2 * np.pi)
    g, m = pkg.Rotary(64, scaling=pkg.ROTARY_YARN, factor=16.0, original=4096).frequencies()
    assert abs(m - (0.1 * np.log(16.0) + 1)) < 1e-12
    keep = np.floor(64 * np.log(4096 / (32 * 2 * np.pi)) / (2 * np.log(10000.0)))
    assert np.allclose(g[:int(keep) + 1], want[:int(keep) + 1], rtol=1e-14) and np.allclose(g[turns < 0.5], want[turns < 0.5] / 16, rtol=1e-14)
    assert np.all(np.diff(g) < 0)
    assert pkg.Rotary(64, scaling=pkg.ROTARY_YARN, factor=16.0, original=4096, magnitude=1.25).frequencies()[1] == 1.25


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=258), dict(rot_dim=-2), dict(base=0.0), dict(base=float("inf")), dict(base=float("nan")),
                                dict(scaling=5), dict(scaling=-1), dict(scaling=1, factor=0.5), dict(scaling=1, factor=float("nan")), dict(scaling=3, factor=2.0),
                                dict(scaling=3, factor=2.0, original=64, low=2.0, high=2.0), dict(scaling=3, factor=2.0, original=64, low=0.0, high=4.0),
                                dict(scaling=4, factor=2.0, original=64, base=1.0), dict(scaling=4, factor=2.0, original=64, magnitude=-1.0)])
def test_rotary_configurations_that_are_refused(kw):
    with pytest.raises(pkg.BildError) as e:
        pkg.Rotary(**{**dict(rot_dim=64), **kw})
    assert e.value.code == b.EINVAL


def test_null_arguments():
    lib = pkg.lib()
    h = C.c_void_p()
    one = (C.c_uint8 * 64)()
    assert lib.bild_quant_round(None, 1, 32, 0, 32, 2, one, one, None) == b.EINVAL
    assert lib.bild_quant_create(1, 32, 32, None, one, 2, None, C.byref(h)) == b.EINVAL
    assert lib.bild_quant_create(1, 32, 32, one, None, 2, None, C.byref(h)) == b.EINVAL
    assert lib.bild_quant_create(1, 32, 32, one, one, 2, None, None) == b.EINVAL
    for n, k, group, dt in ((0, 32, 32, 2), (1, 0, 32, 2), (1, 32, 48, 2), (1, 32, 32, 0), (1 << 25, 32, 32, 2), (1, 1 << 21, 32, 2)):
        assert lib.bild_quant_create(n, k, group, one, one, dt, None, C.byref(h)) == b.EINVAL
    assert lib.bild_quant_matmul(None, C.byref(b.QuantCall()), None) == b.EINVAL
    assert lib.bild_quant_destroy(None) == b.EINVAL
    assert lib.bild_rotary_frequencies(None, one, None) == b.EINVAL
    assert lib.bild_rotary_create(None, C.byref(h)) == b.EINVAL
    assert lib.bild_rotary_apply(None, C.byref(b.RotaryCall()), None) == b.EINVAL
    assert lib.bild_rotary_destroy(None) == b.EINVAL
    r = pkg.Rotary(64)
    assert lib.bild_rotary_apply(r.h, None, None) == b.EINVAL
    assert lib.bild_rotary_apply(r.h, C.byref(b.RotaryCall()), None) == b.EINVAL
    assert lib.bild_rules_create(0, 1, C.byref(h)) == b.EINVAL
    assert lib.bild_rules_create(1, 1, None) == b.EINVAL
    assert lib.bild_rules_apply(None, C.byref(b.RulesCall()), None) == b.EINVAL
    assert lib.bild_rules_destroy(None) == b.EINVAL
    assert not h.value


def test_models_with_rotary_positions_that_are_refused():
    lib = pkg.lib()
    cfg = b.ModelConfig(n_enc_layers=0, n_dec_layers=1, d_model=64, n_heads=2, d_head=32, d_ff=96, act=2, pos=1, vocab=100, tied_head=1, dtype=0,
                        cross_attn=0, logit_scale=1.0, embed_scale=1.0, norm_eps=1e-6, rope_base=10000.0)
    n = lib.bild_model_num_tensors(C.byref(cfg))
    ptrs, h = (C.c_void_p * n)(), C.c_void_p()
    good = b.RotaryConfig(1, 32, 0, 0, 10000.0, 1.0, 0, 0, 0)
    for c, r, count in ((cfg, None, n), (None, good, n), (cfg, b.RotaryConfig(1, 34, 0, 0, 10000.0, 1.0, 0, 0, 0), n), (cfg, b.RotaryConfig(1, 0, 0, 0, 1e4, 1.0, 0, 0, 0), n),
                        (cfg, good, n - 1), (cfg, good, n)):
        assert lib.bild_model_create_rotary(C.byref(c) if c else None, C.byref(r) if r else None, ptrs, count, C.byref(h)) == b.EINVAL
    cfg.pos = 0
    assert lib.bild_model_create_rotary(C.byref(cfg), C.byref(good), ptrs, n, C.byref(h)) == b.EINVAL
    assert not h.value


def test_a_state_that_is_not_there_takes_no_rules():
    l = b.lib()
    assert l.bild_set_quant_head(None, 1, None) == b.EINVAL
    assert l.bild_set_rules(None, None, None, None, 0) == b.EINVAL
    assert l.bild_set_masks(None, 0, 1, None) == b.EINVAL


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("size", [1e-9, 3e-7, 1e-6, 1e-4, 0.02, 1.0])
def test_no_value_moves_by_more_than_half_a_scale(size, zeros, dtype):
    """With zeros and without, down to groups whose scale is the type's smallest or would be none: half a scale, and of 7 (15) steps what the scale was off by."""
    rng = np.random.default_rng(5)
    n, k, group = 40, 200, 64
    w = (size * (rng.standard_normal((n, k)) + (rng.uniform(-3, 3, (n, 1)) if zeros else 0.0))).astype(np.float32)
    w[:, 64:128] *= 1e-3
    codes, scales, z = pkg.quant_round(w, group, dtype, zeros)
    s, g = scales_of(scales, dtype), np.arange(k) // group
    lo = np.stack([np.minimum(w[:, g == j].min(axis=1), 0) for j in range(g[-1] + 1)], axis=1).astype(np.float64)
    hi = np.stack([np.maximum(w[:, g == j].max(axis=1), 0) for j in range(g[-1] + 1)], axis=1).astype(np.float64)
    best, steps = ((hi - lo) / 15, 15) if zeros else (np.maximum(hi, -lo) / 7, 7)
    short = steps * np.maximum(best - s, 0)                           # (a scale that came out smaller leaves the ends of the range outside)
    off = np.abs(weights(codes, s, z, k, group) - w)
    assert np.all(off <= (0.5 * s * (1 + 1e-5) + short)[:, g]), np.max(off / s[:, g])
    # (rounded to the nearest, near zero to half of the smallest, and never to none)
    assert np.all(s > 0) and np.all(s <= np.maximum(best * (1 + HALF_STEP[dtype] * 1.001) + TINY[dtype] / 2, TINY[dtype]))


def test_host_arrays_of_other_sizes_are_refused(monkeypatch):
    """The library reads as much as the sizes say: an array that has less, or values of another width, does not get there."""
    good = dict(codes=np.zeros((5, 33), np.uint8), scales=np.zeros((5, 3), np.float16), zeros=np.zeros((5, 3), np.uint8))
    for kw in (dict(codes=np.zeros((5, 32), np.uint8)), dict(codes=np.zeros((5, 33), np.int32)), dict(scales=np.zeros((5, 2), np.float16)),
               dict(scales=np.zeros((5, 3), np.float32)), dict(zeros=np.zeros((4, 3), np.uint8)), dict(zeros=np.zeros((5, 3), np.int64)), dict(scales=np.zeros(0, np.uint16))):
        with pytest.raises(pkg.BildError) as e:
            pkg.Quant(5, 65, 32, scale_dtype=F16, **{**good, **kw})
        assert e.value.code == b.EINVAL
    calls = []

    class Library:
        def __getattr__(self, name):
            def call(*args):
                calls.append((name, args, (C.c_float * 3).from_address(args[1])[:] if name == "bild_set_rules" else None))
                return b.OK
            return call if name != "bild_strerror" else lambda code: b""

    class Large:
        cfg = b.ModelConfig(vocab=100)

    class Closed:
        h = None

    monkeypatch.setattr(b, "lib", Library)
    st = pkg.State.__new__(pkg.State)
    st.pair = type("Pair", (), dict(large=Large))
    for call in (lambda: st.set_rules((1.0, 0.0)), lambda: st.set_rules((1.0, 0.0, 0.0, 0.0)), lambda: st.set_rules(1.0), lambda: st.set_masks(0, np.ones((2, 3), np.uint32)),
                 lambda: st.set_masks(0, np.ones((2, 5), np.uint32)), lambda: st.set_masks(0, np.ones(8, np.uint32)), lambda: st.set_quant_head(1, Closed())):
        with pytest.raises(pkg.BildError) as e:
            call()
        assert e.value.code == b.EINVAL and not calls
    st.set_rules(np.arange(1, 7)[::2])                                # (every other value of an array: in one piece by then)
    st.set_masks(3, np.ones(4, np.uint32))
    st.set_masks(3, [[1, 2, 3, 4]] * 2)
    st.set_masks(3, None, 7)
    assert calls[0][0] == "bild_set_rules" and calls[0][2] == [1.0, 3.0, 5.0]
    assert [(name, args[1], args[2]) for name, args, _ in calls[1:]] == [("bild_set_masks", 3, n) for n in (1, 2, 7)]


@pytest.mark.parametrize("kw", [dict(base=1e-20), dict(base=4e-6), dict(rot_dim=4, base=5e-11), dict(base=1e-12, scaling=1, factor=2.0), dict(base=1e-38, scaling=2, factor=1.5)])
def test_frequencies_that_no_angle_can_be_formed_of_are_refused(kw):
    """Angles of 2^48 and more (positions go to 2^31) are beyond what the sines are formed from."""
    kw = {**dict(rot_dim=64), **kw}
    for call in (lambda: pkg.Rotary(**kw), lambda: pkg.Rotary(**{**kw, "halves": True})):
        with pytest.raises(pkg.BildError) as e:
            call()
        assert e.value.code == b.EINVAL
    f, _ = pkg.Rotary(**{**kw, "base": 6e-6}).frequencies() if kw["rot_dim"] == 64 and "scaling" not in kw else pkg.Rotary(4, base=6e-11).frequencies()
    assert 1e5 < np.max(f) <= 131072
