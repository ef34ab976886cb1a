"""The cache's definition in numpy against itself, and refusals that come before any device work."""
import ctypes as C

import numpy as np
import pytest

import paper_2302_07863_amd as pkg
from paper_2302_07863_amd import binding as b
from tests.cached import Oracle, invariants


def test_pages_are_counted_and_kept_apart():
    rng = np.random.default_rng(3)
    o = Oracle(60, 32, 1, 1, 16, 7, 10)
    text = [[] for _ in range(7)]                       # what each sequence should hold
    for step in range(300):
        what = rng.integers(0, 5)
        if what < 3:
            ids = rng.permutation(7)[:rng.integers(1, 8)]
            rows = rng.integers(0, 40, len(ids))
            cut = np.array([rng.integers(0, len(text[s]) + 1) if rng.random() < 0.5 else len(text[s]) for s in ids])
            ok = o.extend(rows, ids, cut)
            for s, c in zip(ids, cut):
                text[s] = text[s][:c]
            if ok:
                x = rng.integers(-127, 128, (int(np.sum(rows)), 1, 16)).astype(np.float32)
                x[:, :, 0] = 127                          # (every scale is 127: codes are the values)
                o.append(0, x, x, rows, ids)
                first = 0
                for s, r in zip(ids, rows):
                    text[s] = text[s] + [row for row in x[first:first + r, 0]]
                    first += r
        elif what == 3:
            ids = rng.permutation(7)[:4]
            parents = rng.integers(-1, 4, 4)
            o.fork(parents, ids)
            old = list(text)
            for s, p in zip(ids, parents):
                text[s] = list(old[ids[p]]) if p >= 0 else []
        else:
            assert o.compact() == np.sum(o.refs > 0)
            assert np.all(o.refs[:np.sum(o.refs > 0)] > 0)
        invariants(o)
        for s in range(7):
            assert o.lengths[s] == len(text[s])
            got, there = o.held(s, 0, 1)
            assert np.all(there)
            if len(text[s]):
                assert np.allclose(got[:, 0], np.array(text[s]), atol=1e-9)


def test_attention_of_the_definition():
    rng = np.random.default_rng(4)
    o = Oracle(9, 32, 2, 2, 16, 2, 4)
    o.extend([70, 5])
    k, v = rng.standard_normal((2, 75, 2, 16)).astype(np.float32)
    o.append(1, k, v, [70, 5])
    q = rng.standard_normal((75, 4, 16))
    out, lse, tol, _ = o.attend(1, q, [70, 5], 0.25, window=20, sinks=3)
    kk, vv = o.held(0, 1, 0)[0], o.held(0, 1, 1)[0]
    assert np.max(np.abs(kk - k[:70])) <= np.max(np.abs(k)) / 254 * 1.001
    for t, h in ((0, 0), (19, 1), (20, 2), (69, 3)):
        see = [j for j in range(t + 1) if j > t - 20 or j < 3]
        z = 0.25 * kk[see, h // 2] @ q[t, h]
        p = np.exp(z) / np.sum(np.exp(z))
        assert np.allclose(out[t, h], p @ vv[see, h // 2]) and np.isclose(lse[t, h], np.log(np.sum(np.exp(z))))
    assert np.all(tol < 1e-3)


def _config(**kw):
    # (the arrays of a configuration that is refused are not looked at)
    return b.CacheConfig(**{**dict(codes=1 << 20, scales=1 << 20, table=1 << 20, lengths=1 << 20, refs=1 << 20, pages=4, page_tokens=32, layers=1, heads=2, d_head=64, sequences=2,
                                   max_pages=2, reserved=0), **kw})


@pytest.mark.parametrize("kw", [dict(codes=None), dict(scales=None), dict(table=None), dict(lengths=None), dict(refs=None), dict(codes=(1 << 20) + 8), dict(scales=(1 << 20) + 2),
                                dict(refs=(1 << 20) + 1), dict(pages=0), dict(pages=(1 << 24) + 1), dict(page_tokens=16), dict(page_tokens=48), dict(page_tokens=256), dict(layers=0),
                                dict(layers=1025), dict(heads=0), dict(heads=1025), dict(d_head=8), dict(d_head=20), dict(d_head=264), dict(d_head=-64), dict(sequences=0),
                                dict(sequences=65536), dict(max_pages=0), dict(max_pages=1 << 26), dict(sequences=65535, max_pages=1 << 13), dict(reserved=1)])
def test_caches_that_are_refused(kw):
    h = C.c_void_p()
    assert pkg.lib().bild_cache_create(C.byref(_config(**kw)), C.byref(h)) == b.EINVAL and not h.value


def test_null_arguments():
    lib, h, one = pkg.lib(), C.c_void_p(), (C.c_uint8 * 256)()
    assert lib.bild_cache_create(None, C.byref(h)) == b.EINVAL
    assert lib.bild_cache_create(C.byref(_config()), None) == b.EINVAL
    assert lib.bild_cache_destroy(None) == b.EINVAL
    assert lib.bild_cache_extend(None, C.byref(b.CacheExtendCall(n=1)), None) == b.EINVAL
    assert lib.bild_cache_fork(None, None, one, 1, 0, None) == b.EINVAL
    assert lib.bild_cache_compact(None, None, None) == b.EINVAL
    assert lib.bild_cache_append(None, C.byref(b.CacheAppendCall()), None) == b.EINVAL
    assert lib.bild_cache_attend(None, C.byref(b.CacheAttendCall()), None) == b.EINVAL
    assert lib.bild_beams_select(None, C.byref(b.BeamsCall()), None) == b.EINVAL
    assert lib.bild_beams_destroy(None) == b.EINVAL
    for vocab, batch, beams in ((0, 1, 1), ((1 << 24) + 1, 1, 1), (10, 0, 1), (10, 1, 0), (10, 1, 65), (10, 1024, 64)):
        assert lib.bild_beams_create(vocab, batch, beams, C.byref(h)) == b.EINVAL
    assert lib.bild_beams_create(10, 1, 1, None) == b.EINVAL
    assert not h.value
