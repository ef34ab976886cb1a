"""Rules on logits and 4-bit heads inside a state's passes, against the oracle whose distributions are changed the same way: the steps of
a generation one by one (tokens, flags, rollback indices, probabilities, logits) and whole generations."""
import numpy as np
import pytest

import bild_inputs as bi
import oracle
import paper_2302_07863_amd as pkg
from paper_2302_07863_amd import binding as b
from tests import parity
from tests import test_gpu_rejection as rejection
from tests import test_gpu_sampling as sampling
from tests.rows import F16, mask_words, ruled, scales_of, weights
from tests.test_gpu_early_exit import EERig, _prefix_toy
from tests.test_gpu_parity import Rig, TOY_VARIANTS

pytestmark = pytest.mark.gpu
INF = float("inf")


class Changed:
    """What a state is told, and the same for the oracle's rows of logits."""

    def __init__(self, R, kind: str):
        vocab, cap = R.cfg.large.vocab, R.n0 + R.cfg.max_new + 1
        rng = np.random.default_rng(11)
        self.n0, self.first, self.penalties, self.bias, self.allowed = R.n0, R.n0 + 1, None, {}, None
        if "penalties" in kind:
            self.penalties = (1.25, 0.375, 0.5)
        if "biases" in kind:
            self.bias = {int(t): float(v) for t, v in zip(rng.choice(vocab, 20, replace=False), rng.uniform(-2, 2, 20))}
        if "masks" in kind:
            self.allowed = rng.random((cap - self.first, vocab)) < 0.4
            self.allowed[:, vocab - 1] = True                         # (a row allows at least this one)
            self.allowed[3] = False
            self.allowed[3, vocab // 3] = True

    def tell(self, st):
        st.set_rules(self.penalties, self.bias)
        if self.allowed is not None:
            st.set_masks(self.first, mask_words(self.allowed))

    def row(self, z, y, position: int):
        mask = None if self.allowed is None or not 0 <= position - self.first < len(self.allowed) else self.allowed[position - self.first]
        return ruled(z, tokens=np.asarray(y) if self.penalties else None, length=position, start=self.n0, penalties=self.penalties,
                     bias_ids=list(self.bias) or None, bias=list(self.bias.values()), allowed=mask)

    def oracle(self, monkeypatch):
        """From here on the oracle's decoders answer with changed rows."""
        was, row = oracle.bild._Cached, self.row

        class Ruled(was):
            def next_logits(self, y):
                return row(super().next_logits(y), y, len(y))

            def block_logits(self, y, first):
                return np.stack([row(z, y, first + i) for i, z in enumerate(super().block_logits(y, first))])

        monkeypatch.setattr(oracle.bild, "_Cached", Ruled)


def same_logits(st, ref, R, fb, rb, worst):
    """The logits a state keeps are the changed ones: up to the oracle's first decision that was not the state's (see parity.py for the others)."""
    tol = parity.logit_tol(R.cfg) * worst
    st.encode(R.src)
    st.debug_enable_logits(True)
    checked = 0
    for rec in ref.trace:
        if rec["kind"] == "small":
            tok, flag, _ = st.small_step(fb)
            rows, same = [(st.debug_logits(pkg.SMALL, 0), rec["z"])], tok == rec["tok"] and bool(flag) == rec["fallback"]
        else:
            out, r, _ = st.large_verify(rb)
            rows, same = [(st.debug_logits(pkg.LARGE, i), rec["z"][i]) for i in range(rec["r"] + 1)], r == rec["r"] and out[-1] == rec["tok"]
        for got, want in rows:
            np.testing.assert_array_equal(np.isneginf(got), np.isneginf(want))
            at = ~np.isneginf(want)
            assert np.max(np.abs(got[at] - want[at])) <= tol
        checked += len(rows)
        if not same:
            break
    st.debug_enable_logits(False)
    return checked


KINDS = ["penalties", "biases", "masks", "penalties biases masks"]


def run(R, rules, monkeypatch, before=None, settings=((0.5, 2.0, 10), (0.2, 0.7, 3))):
    rules.oracle(monkeypatch)
    for fb, rb, nm in settings:
        ref = oracle.bild_generate(R.req, fb, rb, nm, R.cfg.max_new, keep_logits=True)
        st = R.state(R.cfg.max_new, nm)
        if before:
            before(st)
        rules.tell(st)
        st.encode(R.src)
        worst = parity.teacher_forced(st, ref, R.n0, fb, rb, R.cfg, check_logits=False)
        checked = same_logits(st, ref, R, fb, rb, 1.25)               # (a repetition of 1.25 scales what a logit is off by)
        toks, stats = st.generate(R.src, fb, rb, R.cfg.max_new)
        print(worst, checked, parity.compare_generation(toks, stats, ref, fb, rb))
        if rules.allowed is not None:
            assert all(rules.allowed[p - rules.first, t] for p, t in enumerate(toks, R.n0) if p >= rules.first)
        assert st.generate(R.src, fb, rb, R.cfg.max_new)[0] == toks
    for which in ("small", "large"):
        g = oracle.greedy(R.req, which, R.cfg.max_new)
        got = st.greedy(pkg.SMALL if which == "small" else pkg.LARGE, R.src, R.cfg.max_new)
        assert got == g.tokens or min(r["gap"] for r in g.trace) < parity.MARGIN


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", ["f32-relu-tied", "bf16-relu-tied", "f32-rope-swiglu-deconly", "bf16-trunc-geglu", "f32-wide"])
def test_rules_toy_parity(name, kind, monkeypatch):
    R = Rig(bi.toy_pair(**TOY_VARIANTS[name]))
    run(R, Changed(R, kind), monkeypatch)


def test_rules_over_many_ranges_and_long_reviews(monkeypatch):
    """A vocabulary of several workgroups a row, reviews of up to 32 rows."""
    R = Rig(bi.toy_pair(vocab=9001, max_new=70))
    run(R, Changed(R, KINDS[-1]), monkeypatch, settings=((0.0, INF, 31), (0.01, 9.0, 17)))


@pytest.mark.parametrize("name", ["f32-relu-tied", "bf16-relu-tied", "f32-rope-swiglu-deconly"])
def test_rules_early_exit(name, monkeypatch):
    R = EERig(_prefix_toy(name))
    run(R, Changed(R, KINDS[-1]), monkeypatch)


def quant_heads(R, group, zeros):
    """(heads, rig) with both models' LM heads in 4 bits; the oracle's have the values the codes stand for."""
    out = []
    for m in (R.req.small, R.req.large):
        e = np.asarray(m.head, dtype=np.float32)
        codes, scales, z = pkg.quant_round(e, group, F16, zeros)
        m.head = weights(codes, scales_of(scales, F16), z, e.shape[1], group)
        out.append(pkg.Quant(e.shape[0], e.shape[1], group, codes, scales, F16, z))
    return out


@pytest.mark.parametrize("kind", ["", KINDS[-1]])
@pytest.mark.parametrize("name,more", [("f32-relu-tied", {}), ("bf16-relu-tied", {}), ("f32-rope-swiglu-deconly", {}), ("bf16-trunc-geglu", {}), ("f32-wide", {}),
                                       ("bf16-relu-tied", dict(vocab=5003, max_new=70, d=160))])
def test_quant_heads_toy_parity(name, more, kind, monkeypatch):
    R = Rig(bi.toy_pair(**{**TOY_VARIANTS[name], **more}))
    heads = quant_heads(R, 32, bool(kind))

    def before(st):
        for which, h in zip((pkg.SMALL, pkg.LARGE), heads):
            st.set_quant_head(which, h)

    run(R, Changed(R, kind), monkeypatch, before, settings=((0.5, 2.0, 10), (0.0, INF, 31) if more else (0.2, 0.7, 3)))


def test_quant_head_early_exit(monkeypatch):
    R = EERig(_prefix_toy("bf16-relu-tied"))
    heads = quant_heads(R, 64, True)

    def before(st):
        for which, h in zip((pkg.SMALL, pkg.LARGE), heads):
            st.set_quant_head(which, h)

    run(R, Changed(R, KINDS[0]), monkeypatch, before)


# The routes of a pass that hand the final hidden state on in forms of their own: one kernel for the layers (with the head inside, with a row of
# several tiles), separate kernels over high and low planes, the thin products of wide models.
@pytest.mark.parametrize("env", [dict(), dict(BILD_ONE_KERNEL="0"), dict(BILD_PRE_MIN_ROWS="1")])
@pytest.mark.parametrize("d,d_ff,rows", [(512, 1024, 9), (2048, 512, 20), (2560, 512, 7)])
def test_every_route_to_the_head(d, d_ff, rows, env, monkeypatch):
    for k, v in env.items():
        monkeypatch.setenv(k, v)
    cfg = bi.toy_pair(dtype=bi.DT_BF16, d=d, heads=d // 64, d_head=64, d_ff=d_ff, vocab=2100, act=bi.ACT_SWIGLU, pos=bi.POS_ROPE, cross=False, tied=False,
                      n_small=1, n_large=2, max_new=40, embed_scale=14.0, logit_scale=4.0)
    R = Rig(cfg)
    heads = quant_heads(R, 128, True)
    rules = Changed(R, "penalties biases")
    rules.oracle(monkeypatch)
    tol = 1.25 * parity.logit_tol(cfg)
    st = R.state(cfg.max_new, rows)
    for quant in (False, True):
        if quant:
            for which, h in zip((pkg.SMALL, pkg.LARGE), heads):
                st.set_quant_head(which, h)
        rules.tell(st)
        st.debug_enable_logits(True)
        st.encode(R.src)
        R.req.large.head, dequantised = (R.req.large.head, None) if quant else (np.asarray(R.wl["head"], dtype=np.float64), R.req.large.head)
        y = list(R.src)
        for n in (0, 1, rows):
            block = [int(t) for t in bi.make_tokens(cfg.large.vocab, n, seed=40 + n)]
            out, r, nll = st.large_verify(INF, draft=block)
            y += block
            z = [rules.row(v, y, len(y) - n + i) for i, v in enumerate(R.req.large.logits_full(y, [])[len(y) - n - 1:])]
            for i in range(n + 1):
                got = st.debug_logits(pkg.LARGE, i)
                assert np.max(np.abs(got - z[i])) <= tol, (quant, n, i)
                if i < n:
                    assert abs(nll[i] - oracle.policy.nll(z[i], block[i])) <= 2 * tol
            assert out[n] == int(np.argmax(got))
            y.append(out[n])
        if dequantised is not None:
            R.req.large.head = dequantised
    print(st.pass_routes())


@pytest.mark.parametrize("name", ["f32-relu-tied", "f32-rope-swiglu-deconly"])
def test_rules_with_draws(name, monkeypatch):
    """Draws from, and acceptance by, the changed distributions."""
    R = Rig(bi.toy_pair(**TOY_VARIANTS[name]))
    cfg = R.cfg
    rules = Changed(R, KINDS[-1])
    rules.oracle(monkeypatch)
    n = R.n0 + cfg.max_new + 1
    us, ul, ua = (bi.make_uniforms(n, cfg.input_seed, i) for i in range(3))
    margin = sampling._margin(cfg)
    for fb, rb, nm in ((0.5, 2.0, 10), (0.1, 5.0, 4)):
        st = R.state(cfg.max_new, nm)
        rules.tell(st)
        ref = oracle.bild_generate(R.req, fb, rb, nm, cfg.max_new, sampler=oracle.Sampler(sampling.TOP_P, us, ul))
        st.set_sampling(sampling.TOP_P, us, ul)
        st.encode(R.src)
        print(sampling.replay(st, ref, R.n0, fb, rb, margin))
        toks, stats = st.generate(R.src, fb, rb, cfg.max_new)
        sampling.free_running(toks, stats, ref, R.n0, fb, rb, margin)
        assert all(rules.allowed[p - rules.first, t] for p, t in enumerate(toks, R.n0) if p >= rules.first)
        ref = oracle.bild_generate(R.req, 0.0, 0.0, nm, cfg.max_new, sampler=oracle.Sampler(sampling.TOP_P, us, ul, ua), acceptance="rejection")
        st.set_acceptance(pkg.ACCEPT_REJECTION, ua)
        st.encode(R.src)
        print(rejection.replay(st, ref, R.n0, 0.0, margin))
        toks, _ = st.generate(R.src, 0.0, 0.0, cfg.max_new)
        rejection.free_running(toks, ref, R.n0, 0.0, margin)
        assert all(rules.allowed[p - rules.first, t] for p, t in enumerate(toks, R.n0) if p >= rules.first)


def probabilities(st, R):
    st.encode(R.src)
    return [st.small_step(0.0)[2] for _ in range(8)]


@pytest.mark.parametrize("name", ["f32-relu-tied", "bf16-relu-tied", "f32-rope-swiglu-deconly"])
def test_taken_back(name):
    """A state without them again answers as it did, through its captured passes; two settings in turn."""
    R = Rig(bi.toy_pair(**TOY_VARIANTS[name]))
    st = R.state(R.cfg.max_new, 10)
    want = st.generate(R.src, 0.5, 2.0, R.cfg.max_new)
    a, c = Changed(R, KINDS[0]), Changed(R, KINDS[1])
    a.tell(st)
    first, at = st.generate(R.src, 0.5, 2.0, R.cfg.max_new), probabilities(st, R)
    c.tell(st)
    st.generate(R.src, 0.5, 2.0, R.cfg.max_new)
    assert probabilities(st, R) != at
    a.tell(st)
    assert st.generate(R.src, 0.5, 2.0, R.cfg.max_new) == first and probabilities(st, R) == at
    heads = quant_heads(R, 32, False)
    st.set_rules()
    st.set_quant_head(pkg.LARGE, heads[1])
    st.generate(R.src, 0.5, 2.0, R.cfg.max_new)
    st.set_quant_head(pkg.LARGE, None)
    assert st.generate(R.src, 0.5, 2.0, R.cfg.max_new) == want
    masks = Changed(R, "masks")
    masks.tell(st)
    assert st.generate(R.src, 0.5, 2.0, R.cfg.max_new)[0] != want[0]
    st.set_masks(masks.first, None, len(masks.allowed))
    assert st.generate(R.src, 0.5, 2.0, R.cfg.max_new)[0] == want[0]


def test_masks_given_on_the_way():
    """Each token's mask from the tokens before it, as a grammar would have it: here the id has to leave the rest that follows from the
    one before."""
    R = Rig(bi.toy_pair(**TOY_VARIANTS["f32-relu-tied"]))
    vocab, ids = R.cfg.large.vocab, np.arange(R.cfg.large.vocab)
    st = R.state(R.cfg.max_new, 3)
    st.encode(R.src)
    for step in range(12):
        y = st.sequence()
        st.set_masks(len(y), mask_words((ids % 5 == (y[-1] + 1) % 5)[None]))
        st.small_step(0.0) if step % 4 != 3 else st.large_verify(INF)
    y = st.sequence()
    assert len(y) == R.n0 + 12 and all(q % 5 == (p + 1) % 5 for p, q in zip(y[R.n0 - 1:], y[R.n0:]))


def test_refusals():
    R = Rig(bi.toy_pair(**TOY_VARIANTS["f32-relu-tied"]))
    vocab, d = R.cfg.large.vocab, R.cfg.large.d
    st = R.state(R.cfg.max_new, 10)
    want = st.generate(R.src, 0.5, 2.0, R.cfg.max_new)
    e = np.zeros((vocab + 1, d + 1), np.float32)
    heads = []
    for n, k in ((vocab + 1, d), (vocab, d + 1)):
        codes, scales, _ = pkg.quant_round(e[:n, :k], 32)
        heads.append(pkg.Quant(n, k, 32, codes, scales, F16))
    good, none = mask_words(np.ones((2, vocab), bool)), np.zeros((1, len(mask_words(np.ones(vocab, bool)))), np.uint32)
    behind = none.copy()
    behind[0, -1] = 1 << (vocab % 32)                                 # (an id behind the vocabulary)
    cap = st.max_len
    for call in (lambda: st.set_quant_head(0, heads[0]), lambda: st.set_quant_head(3, None), lambda: st.set_quant_head(1, heads[0]),
                 lambda: st.set_quant_head(2, heads[1]), lambda: st.set_rules((0.0, 0.0, 0.0)), lambda: st.set_rules((-1.0, 0.0, 0.0)),
                 lambda: st.set_rules((1.0, INF, 0.0)), lambda: st.set_rules((1.0, 0.0, float("nan"))), lambda: st.set_rules(None, {vocab: 1.0}),
                 lambda: st.set_rules(None, {-1: 1.0}), lambda: st.set_rules(None, {0: INF}), lambda: st.set_masks(-1, good), lambda: st.set_masks(cap - 1, good),
                 lambda: st.set_masks(cap, None, 1), lambda: st.set_masks(0, None, 0), lambda: st.set_masks(2, none), lambda: st.set_masks(2, behind)):
        with pytest.raises(pkg.BildError) as err:
            call()
        assert err.value.code == b.EINVAL
    assert b.lib().bild_set_rules(st.h, None, None, None, 1) == b.EINVAL and b.lib().bild_set_rules(st.h, None, None, None, -1) == b.EINVAL
    assert b.lib().bild_set_rules(st.h, None, np.zeros(1024, np.int32).ctypes.data, np.zeros(1024, np.float32).ctypes.data, 1024) == b.EINVAL
    assert st.generate(R.src, 0.5, 2.0, R.cfg.max_new) == want        # nothing of it counted


@pytest.mark.parametrize("fill", [-1e10, -1e20, 1e12])
def test_biases_of_any_size(fill):
    """All ids but five moved to one far value, then all of them: a step's probability is that of the ids at the top."""
    R = Rig(bi.toy_pair(**TOY_VARIANTS["f32-relu-tied"]))
    vocab = R.cfg.large.vocab
    st = R.state(R.cfg.max_new, 3)
    st.set_rules(None, {t: fill for t in range(5, vocab)})
    st.encode(R.src)
    st.debug_enable_logits(True)
    tok, _, prob = st.small_step(0.0)
    z = st.debug_logits(pkg.SMALL, 0).astype(np.float64)
    assert tok == int(np.argmax(z)) and abs(prob - 1 / np.sum(np.exp(z - z.max()))) <= 1e-5
    st.set_rules(None, {t: fill for t in range(vocab)})               # (every logit is the same now)
    tok, _, prob = st.small_step(0.0)
    assert np.all(st.debug_logits(pkg.SMALL, 0) == np.float32(fill)) and tok == 0 and abs(prob * vocab - 1) <= 1e-5


def test_masks_taken_back_give_the_route_back():
    """Where no position is restricted any more, passes take the kernels that they took before; where one is, its mask counts."""
    R = Rig(bi.toy_pair(dtype=bi.DT_BF16, d=256, heads=4, d_head=64, d_ff=512, truncate=True, n_src=20, max_new=40))
    vocab = R.cfg.large.vocab
    st = R.state(R.cfg.max_new, 10)
    st.encode(R.src)

    def step():
        before, at = st.pass_routes(), len(st.sequence())
        tok = st.small_step(0.0)[0]
        now = st.pass_routes()
        return tok, st.pass_stages(), {k for k in now if now[k] > before[k]}, at

    step()
    _, stages, route, at = step()
    want = st.generate(R.src, 0.5, 2.0, R.cfg.max_new)
    only = np.zeros((1, vocab), bool)
    for allowed in (17, vocab - 1, 3):
        st.encode(R.src)
        first = len(st.sequence())
        only[:] = False
        only[0, allowed] = True
        st.set_masks(first, mask_words(np.repeat(only, 2, axis=0)))
        tok, masked, *_ = step()
        assert tok == allowed and masked > stages
        st.set_masks(first, None, 1)                                  # (the other position is restricted still)
        tok, masked, *_ = step()
        assert tok == allowed and masked > stages
        st.set_masks(first + 1, mask_words(np.ones((1, vocab), bool)))  # (a mask that allows all ids)
        _, again, taken, _ = step()
        assert again == stages and taken == route
        st.set_masks(first, mask_words(only))
        st.set_masks(0, None, st.max_len)
        assert st.generate(R.src, 0.5, 2.0, R.cfg.max_new) == want
        st.encode(R.src)
        _, again, taken, _ = step()
        assert again == stages and taken == route
