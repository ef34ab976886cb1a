"""Selection over beams and vocabulary against a sort in 64 bits."""
import ctypes as C

import numpy as np
import pytest

import paper_2302_07863_amd as pkg
from paper_2302_07863_amd import binding as b
from tests.hipmem import DeviceArray
from tests.rows import BF16, F16, F32, Graph, Rows, Stream, pack, unpack

pytestmark = pytest.mark.gpu


def choose(z, scores, choices, lengths=None, finished=None, eos=-1, pad=0, penalty=0.0, history=None):
    """z [beams][vocab] in 64 bits: (sum, rank, parent, token, length, ended, history) in order."""
    beams, vocab = z.shape
    found = []
    for j in range(beams):
        length, score = int(lengths[j]) if lengths is not None else 0, float(scores[j])
        if finished is not None and finished[j]:
            rank = score / max(length, 1) ** penalty
            if np.isfinite(rank):
                found.append((-rank, j, pad, score, length, 1))
            continue
        m = np.max(z[j])
        with np.errstate(all="ignore"):
            lse = m + np.log(np.sum(np.exp(z[j] - m)))
        if not np.isfinite(score - lse):
            continue
        total = (score - lse) + z[j]
        over = max(length + 1, 1) ** penalty
        for v in np.lexsort((np.arange(vocab), -total))[:choices]:
            if total[v] > -np.inf:
                found.append((-(total[v] / over), j, int(v), total[v], length + 1, int(v == eos)))
    found = sorted(found)[:choices]
    out = dict(scores=[f[3] for f in found], parents=[f[1] for f in found], tokens=[f[2] for f in found], lengths=[f[4] for f in found], finished=[f[5] for f in found])
    for name, none in (("scores", -np.inf), ("parents", -1), ("tokens", -1), ("lengths", 0), ("finished", 1)):
        out[name] += [none] * (choices - len(found))
    if history is not None:
        out["history"] = [(list(history[p]) if p >= 0 else [-1] * history.shape[1]) + [t] for p, t in zip(out["parents"], out["tokens"])]
    return {k: np.array(v) for k, v in out.items()}


def select(words, dtype, batch, beams, choices, scores, lengths=None, finished=None, eos=-1, pad=0, penalty=0.0, history=None, stride=None, replays=0):
    vocab = words.shape[1]
    logits = Rows(words, stride, 3 if stride else 0)
    dev = {k: DeviceArray(v) for k, v in (("scores", np.float32(scores)), ("lengths", lengths), ("finished", finished)) if v is not None}
    n = batch * choices
    outs = dict(scores=Rows(np.full((1, n), 9, np.float32)), **{k: Rows(np.full((1, n), 9, np.int32)) for k in ("parents", "tokens", "lengths", "finished")})
    kw = dict(eos=eos, pad=pad, penalty=penalty)
    if history is not None:
        hist, hout = Rows(history, history.shape[1] + 2), Rows(np.zeros((n, history.shape[1] + 1), np.int32), history.shape[1] + 5, 1)
        kw.update(history=hist.ptr, history_stride=hist.stride, out_history=hout.ptr, out_history_stride=hout.stride, steps=history.shape[1])
    sel = pkg.Beams(vocab, batch, beams)

    def call(stream=None):
        sel.select(logits.ptr, dtype, batch, choices, dev["scores"].ptr.value, outs["scores"].ptr, outs["parents"].ptr, outs["tokens"].ptr, logits_stride=logits.stride,
                   lengths=dev["lengths"].ptr.value if lengths is not None else None, finished=dev["finished"].ptr.value if finished is not None else None,
                   out_lengths=outs["lengths"].ptr, out_finished=outs["finished"].ptr, stream=stream, **kw)

    if replays:
        st = Stream()
        g = Graph(st, call)
        for _ in range(replays):
            g.replay()
        st.sync()
    else:
        call()
    got = {k: v.get()[0] for k, v in outs.items()}
    if history is not None:
        got["history"] = hout.get()
    z = unpack(words, dtype)
    for e in range(batch):
        at = slice(e * beams, (e + 1) * beams)
        want = choose(z[at], np.float32(scores)[at], choices, *(x[at] if x is not None else None for x in (lengths, finished)), eos=eos, pad=pad, penalty=penalty,
                      history=history[at] if history is not None else None)
        mine = slice(e * choices, (e + 1) * choices)
        for name, w in want.items():
            g = got[name][mine]
            if name == "scores":
                there = np.isfinite(w)
                assert np.array_equal(there, np.isfinite(g)) and np.all(g[~there] == -np.inf)
                # sums of exponentials in fp32: a step each and 20 of adding, then the rounding
                assert np.all(np.abs(g[there] - w[there]) <= 2.0 ** -19 + 2.0 ** -23 * np.abs(w[there]))
            else:
                assert np.array_equal(g, w), (name, e, g, w)
    return got


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("batch,beams,vocab,choices", [(1, 1, 1, 1), (1, 4, 7, 4), (2, 3, 255, 6), (3, 4, 1000, 8), (1, 5, 32128, 5), (2, 8, 50257, 16), (1, 2, 250112, 4), (5, 1, 4097, 64), (1, 12, 20000, 24), (1, 32, 8192, 64), (2, 5, 1009, 10),
                                                       (1, 64, 513, 64)])
def test_sizes(dtype, batch, beams, vocab, choices):
    rng = np.random.default_rng(vocab + beams)
    rows = batch * beams
    words = pack(2.5 * rng.standard_normal((rows, vocab)), dtype)
    scores = -3.0 * rng.random(rows)
    select(words, dtype, batch, beams, choices, scores, stride=vocab + 5)
    lengths = rng.integers(0, 30, rows).astype(np.int32)
    finished = (rng.random(rows) < 0.4).astype(np.int32)
    select(words, dtype, batch, beams, choices, scores - lengths, lengths, finished, eos=int(np.argmax(unpack(words, dtype)[0])), pad=min(2, vocab - 1), penalty=0.7,
           history=rng.integers(0, vocab, (rows, 9)).astype(np.int32))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["zeros", "two values", "steps", "half masked"])
@pytest.mark.parametrize("beams,vocab,choices", [(1, 3000, 5), (4, 32128, 8), (3, 700, 64)])
def test_many_equal_logits(dtype, kind, beams, vocab, choices):
    """Ties go to the lower beam and id; lists that hold them all would be too long."""
    rng = np.random.default_rng(beams)
    z = np.zeros((beams, vocab))
    if kind == "two values":
        z = np.where(rng.random(z.shape) < 0.5, 0.0, -3.0)
    elif kind == "steps":
        z = np.floor(3 * rng.random(z.shape))
    elif kind == "half masked":
        z = np.where(rng.random(z.shape) < 0.5, -np.inf, 1.0)
    scores = np.array([-1.0, -1.0, -0.5, -1.0][:beams])
    select(pack(z, dtype), dtype, 1, beams, choices, scores)
    finished = np.zeros(beams, np.int32)
    finished[-1] = 1
    # (an ended beam that is as good as what others go on with)
    if beams > 1 and kind == "zeros":
        scores[-1] = np.float32(-1.0 - np.log(vocab))
    select(pack(z, dtype), dtype, 1, beams, choices, scores, np.zeros(beams, np.int32), finished)


def test_rows_that_offer_nothing():
    rng = np.random.default_rng(8)
    z = rng.standard_normal((6, 400))
    z[0] = -np.inf
    z[1, 5] = np.nan
    z[2, 7] = np.inf
    z[3, 3:] = -np.inf
    scores = np.array([0.0, 0.0, 0.0, -1.0, -np.inf, np.nan])
    got = select(pack(z, F32), F32, 1, 6, 8, scores)
    assert list(got["parents"]) == [3] * 3 + [-1] * 5 and np.all(got["finished"][3:] == 1)
    got = select(pack(z, F16), F16, 1, 6, 8, scores, np.full(6, 4, np.int32), np.array([0, 1, 0, 0, 1, 1], np.int32), penalty=1.0,
                 history=rng.integers(0, 9, (6, 0)).astype(np.int32))
    assert got["parents"][0] == 1 and got["lengths"][0] == 4
    z[...] = -np.inf
    select(pack(z, F32), F32, 2, 3, 4, scores)


def test_logits_far_from_zero():
    rng = np.random.default_rng(9)
    z = rng.standard_normal((4, 5000)).astype(np.float32)
    for shift in (1e4, -1e4, 3e6):
        select(z + np.float32(shift) if abs(shift) < 1e6 else np.round(z) + np.float32(shift), F32, 1, 4, 8, np.array([-1.0, -2.0, -1.5, -9.0]))


@pytest.mark.parametrize("penalty", [40.0, -40.0, 200.0, -200.0, 1.0])
def test_penalties_and_scores_far_apart(penalty):
    """Ranks beyond what fp32 holds are sorted all the same."""
    rng = np.random.default_rng(11)
    z = rng.standard_normal((4, 3000)).astype(np.float32)
    lengths = np.array([3, 4, 5, 3], np.int32)
    select(z, F32, 1, 4, 8, np.array([-1.0, -2.0, -1.5, -9.0]), lengths, penalty=penalty)
    select(z, F32, 1, 4, 8, np.array([-1e30, -2e38, -1.5, -3e38]), lengths, penalty=penalty)
    z[2, 7:] = -1e37
    select(z, F32, 1, 4, 64, np.array([-1.0, -2.0, -1.5, -9.0]), lengths, penalty=1.0)


def test_replays_and_batches_below_the_most():
    rng = np.random.default_rng(10)
    words = pack(rng.standard_normal((12, 3001)), BF16)
    select(words, BF16, 3, 4, 4, -rng.random(12), replays=3, history=rng.integers(0, 9, (12, 300)).astype(np.int32))


def test_calls_that_are_refused():
    s, mem = pkg.Beams(100, 2, 3), DeviceArray(nbytes=1 << 14)
    p = mem.ptr.value
    ok = dict(logits=p, dtype=F32, batch=1, choices=3, scores=p, out_scores=p, out_parents=p, out_tokens=p)
    for kw, code in ((dict(logits=None), b.EINVAL), (dict(scores=None), b.EINVAL), (dict(out_scores=None), b.EINVAL), (dict(out_parents=None), b.EINVAL), (dict(out_tokens=None), b.EINVAL),
                     (dict(dtype=3), b.EINVAL), (dict(batch=0), b.EINVAL), (dict(batch=3), b.ECAP), (dict(choices=0), b.EINVAL), (dict(choices=65), b.EINVAL),
                     (dict(penalty=float("inf")), b.EINVAL), (dict(penalty=float("nan")), b.EINVAL), (dict(steps=-1), b.EINVAL), (dict(history=p), b.EINVAL), (dict(out_history=p), b.EINVAL),
                     (dict(finished=p, pad=100), b.EINVAL), (dict(finished=p, pad=-1), b.EINVAL)):
        with pytest.raises(pkg.BildError) as e:
            s.select(**{**ok, **kw})
        assert e.value.code == code, kw
    bad = b.BeamsCall(logits=p, scores=p, out_scores=p, out_parents=p, out_tokens=p, batch=1, choices=1, reserved=1)
    assert pkg.lib().bild_beams_select(s.h, C.byref(bad), None) == b.EINVAL


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("beams,choices,vocab,living", [(8, 16, 250112, 1), (16, 16, 32128, 1), (32, 64, 32128, 4), (64, 64, 5001, 2), (12, 12, 1000, 1), (8, 16, 9000, 3)])
def test_few_living_beams(beams, choices, vocab, living, dtype):
    """A first step, where one beam has a score, and last ones, where most have ended: fewer chunks than usual to take a threshold from."""
    rng = np.random.default_rng(beams + living)
    words = pack(2.5 * rng.standard_normal((beams, vocab)), dtype)
    at = rng.permutation(beams)[:living]
    scores = np.full(beams, -np.inf)
    scores[at] = -rng.random(living)
    select(words, dtype, 1, beams, choices, scores)
    finished = np.ones(beams, np.int32)
    finished[at] = 0
    lengths = rng.integers(3, 30, beams).astype(np.int32)
    select(words, dtype, 1, beams, choices, -lengths * (0.5 + rng.random(beams)), lengths, finished, pad=1, penalty=0.6)


def test_beams_whose_scores_are_far_apart():
    """Most of what is chosen goes on from the best beam, whose groups alone are too few."""
    rng = np.random.default_rng(12)
    words = pack(2.5 * rng.standard_normal((32, 32128)), BF16)
    select(words, BF16, 1, 32, 64, -0.7 * np.arange(32))
    select(words, BF16, 1, 32, 64, -3.0 * np.arange(32)[::-1])
