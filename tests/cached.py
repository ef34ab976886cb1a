"""The cache in 8 bits for tests: its arrays in device memory with guards around them, and the definition in numpy - pages by plain loops, codes in fp32 as they
are specified, attention in 64 bits."""
from __future__ import annotations

import numpy as np

import paper_2302_07863_amd as pkg
from tests.hipmem import DeviceArray
from tests.rows import BF16, F16, F32, HALF_STEP, U32, unpack

LIMIT = np.float32(2.0 ** 90)
GUARD = 256                                            # words before and behind an array that nobody may touch


class Oracle:
    """What the calls do, one sequence after the other."""

    def __init__(self, pages, page_tokens, layers, heads, d_head, sequences, max_pages):
        self.T, self.layers, self.heads, self.d, self.max_pages, self.pages = page_tokens, layers, heads, d_head, max_pages, pages
        self.codes = np.zeros((pages, layers, 2, heads, page_tokens, d_head), np.int8)
        self.scales = np.zeros((pages, layers, 2, heads), np.float32)
        self.table = np.full((sequences, max_pages), -1, np.int32)
        self.lengths = np.zeros(sequences, np.int32)
        self.refs = np.zeros(pages, np.int32)
        self.fits = True

    def _blocks(self, length):
        return -(-int(length) // self.T)

    def _drop(self, s, blocks):
        for b in blocks:
            p = self.table[s, b]
            if 0 <= p < self.pages:
                self.refs[p] -= 1
            self.table[s, b] = -1

    def extend(self, rows, sequences=None, cut=None, window=0, sinks=0):
        """rows: one number or one a sequence.  True if they have grown."""
        T, cap = self.T, self.max_pages * self.T
        ids = list(range(len(rows))) if sequences is None else list(sequences)
        todo = []
        for i, s in enumerate(ids):
            if not 0 <= s < len(self.lengths):
                continue
            length = int(self.lengths[s])
            keep = min(max(int(cut[i]), 0), length) if cut is not None else length
            self._drop(s, range(self._blocks(keep), self._blocks(length)))
            if window:
                self._drop(s, range(self._blocks(sinks), min(max(keep - window + 1, 0) // T, self._blocks(keep))))
            self.lengths[s] = keep
            todo.append((s, keep, int(rows[i])))
        # what each needs
        refs, free, grown = self.refs.copy(), [p for p in range(self.pages) if self.refs[p] == 0], []
        todo = [t for t in todo if t[2] > 0]
        for s, keep, add in todo:
            if keep + add > cap or (keep % T and not 0 <= self.table[s, keep // T] < self.pages):
                self.fits = False
                return False
        for s, keep, add in todo:
            if keep % T and refs[self.table[s, keep // T]] > 1:
                old = self.table[s, keep // T]
                refs[old] -= 1
                grown.append((s, keep // T, old, keep % T))
            grown += [(s, b, -1, 0) for b in range(self._blocks(keep), self._blocks(keep + add))]
        self.fits = len(grown) <= len(free)
        if not self.fits:
            return False
        was, were = self.codes.copy(), self.scales.copy()
        for (s, b, old, part), p in zip(grown, free):
            if old >= 0:
                self.codes[p, ..., :part, :] = was[old, ..., :part, :]
                self.scales[p] = were[old]
                self.refs[old] -= 1
            self.table[s, b] = p
            self.refs[p] = 1
        for s, keep, add in todo:
            self.lengths[s] = keep + add
        return True

    def fork(self, parents, sequences=None, group=0):
        n = len(parents)
        group = group or n
        ids = list(range(n)) if sequences is None else list(sequences)
        table, lengths = self.table.copy(), self.lengths.copy()
        for i, s in enumerate(ids):
            if not 0 <= s < len(lengths):
                continue
            at = i // group * group + parents[i]
            src = ids[at] if 0 <= parents[i] < group and at < n else -1
            self.table[s], self.lengths[s] = (table[src], lengths[src]) if 0 <= src < len(lengths) else (-1, 0)
        self.refs[:] = 0
        for p in self.table[(self.table >= 0) & (self.table < self.pages)]:
            self.refs[p] += 1

    def compact(self):
        used = int(np.sum(self.refs > 0))
        moves = {a: b for a, b in zip([p for p in range(used, self.pages) if self.refs[p] > 0], [p for p in range(used) if self.refs[p] == 0])}
        for a, b in moves.items():
            self.codes[b], self.scales[b] = self.codes[a], self.scales[a]
            self.refs[b], self.refs[a] = self.refs[a], 0
        for row in self.table:
            for i, p in enumerate(row):
                row[i] = moves.get(int(p), p)
        return used

    def append(self, layer, k, v, rows, sequences=None):
        """k, v [tokens][heads][d_head] as float32 values of the row type."""
        if not self.fits:
            return
        ids = list(range(len(rows))) if sequences is None else list(sequences)
        first = 0
        for s, count in zip(ids, rows):
            if 0 <= s < len(self.lengths) and count:
                length = int(self.lengths[s])
                for b in range(max(length - count, 0) // self.T, self._blocks(length)):
                    p0, p1 = max(length - count, b * self.T), min(length, (b + 1) * self.T)
                    page = self.table[s, b]
                    if p1 <= p0 or not 0 <= page < self.pages or self.refs[page] != 1:
                        continue
                    for which, x in ((0, k), (1, v)):
                        for h in range(self.heads):
                            self._write(page, layer, which, h, p0 - b * self.T, x[first + p0 - (length - count):first + p1 - (length - count), h])
            first += count

    def _write(self, page, layer, which, h, before, x):
        x = np.clip(np.where(np.isnan(x), np.float32(0), x.astype(np.float32)), -LIMIT, LIMIT)
        was = self.scales[page, layer, which, h] if before else np.float32(0)
        scale = np.maximum(was, np.max(np.abs(x)))
        codes = self.codes[page, layer, which, h]
        if scale > was:
            codes[:before] = np.rint(codes[:before].astype(np.float32) * was / scale).astype(np.int8)
        codes[before:before + len(x)] = np.rint(x * np.float32(127) / scale).astype(np.int8) if scale > 0 else 0
        self.scales[page, layer, which, h] = scale

    def held(self, s, layer, which):
        """[positions][heads][d_head] in 64 bits, and which of them have a page."""
        n = int(self.lengths[s])
        out, there = np.zeros((self._blocks(n) * self.T, self.heads, self.d)), np.zeros(self._blocks(n) * self.T, bool)
        for b in range(self._blocks(n)):
            p = self.table[s, b]
            if 0 <= p < self.pages:
                at = slice(b * self.T, (b + 1) * self.T)
                out[at] = (self.codes[p, layer, which].astype(np.float64) * (self.scales[p, layer, which].astype(np.float64)[:, None, None] / 127)).transpose(1, 0, 2)
                there[at] = True
        return out[:n], there[:n]

    def attend(self, layer, q, rows, scale, sequences=None, window=0, sinks=0, causal=True, dtype=F32):
        """q [tokens][heads of q][d_head] in 64 bits: outputs, lse and how far each may be off."""
        ids = list(range(len(rows))) if sequences is None else list(sequences)
        tokens, hq, d = q.shape
        out, lse, tol, ltol = np.zeros(q.shape), np.full((tokens, hq), -np.inf), np.zeros(q.shape), np.zeros((tokens, hq))
        group, first = hq // self.heads, 0
        for s, count in zip(ids, rows):
            if 0 <= s < len(self.lengths) and count:
                k, there = self.held(s, layer, 0)
                v, _ = self.held(s, layer, 1)
                n, at = len(k), np.arange(len(k))
                for t in range(count):
                    pos = n - count + t if causal else n - 1
                    seen = there & (at <= pos)
                    if window:
                        seen &= (at > pos - window) | (at < sinks)
                    if not np.any(seen):
                        continue
                    for h in range(hq):
                        kh, vh, x = k[seen, h // group], v[seen, h // group], q[first + t, h]
                        z = scale * (kh @ x)
                        m = np.max(z)
                        p = np.exp(z - m)
                        total = np.sum(p)
                        p /= total
                        o = p @ vh
                        out[first + t, h], lse[first + t, h] = o, m + np.log(total)
                        # scores: d products and sums in fp32 and the two scalings; q's parts (fp32: 22 bits; what is 2^-31 of the row's largest is lost from 16-bit rows)
                        size = abs(scale) * (np.abs(kh) @ np.abs(x))
                        dz = np.max(size) * ((d + 8) * U32 + (2.0 ** -22 if dtype == F32 else 0)) + abs(scale) * np.max(np.abs(x)) * 2.0 ** -39 * np.max(np.sum(np.abs(kh), axis=1))
                        # weights: exponentials (two steps, and the product's rounding of an exponent of up to 2^7), fp16 or two parts, below 2^-24 of the largest by that; sums of a lane
                        weight = 2 * dz + 2.0 ** -22 + 128 * U32 + (2.0 ** -22 if dtype == F32 else 2.0 ** -11) + (len(kh) / 16 + 80) * U32
                        lost = len(kh) * 2.0 ** -25 * np.max(np.abs(vh), axis=0) / total
                        tol[first + t, h] = weight * (p @ np.abs(vh)) + lost + HALF_STEP[dtype] * np.abs(o) + 1e-37
                        ltol[first + t, h] = dz + 2.0 ** -21 + 128 * U32 + (len(kh) / 16 + 80) * U32 + 4 * U32 * abs(lse[first + t, h])
            first += count
        return out, lse, tol, ltol


class Held:
    """An oracle and the same cache on the device."""

    NAMES = ("codes", "scales", "table", "lengths", "refs")

    def __init__(self, oracle: Oracle):
        self.o = oracle
        self.mem, ptr = {}, {}
        for name in self.NAMES:
            a = getattr(oracle, name)
            guard = np.full(GUARD, 0x5A, np.uint8)
            self.mem[name] = DeviceArray(np.concatenate((guard, np.ascontiguousarray(a).view(np.uint8).reshape(-1), guard)))
            ptr[name] = self.mem[name].ptr.value + GUARD
        self.ptr = ptr
        self.cache = pkg.Cache(oracle.pages, oracle.T, oracle.layers, oracle.heads, oracle.d, len(oracle.lengths), oracle.max_pages, **ptr)

    def get(self, name):
        a = getattr(self.o, name)
        raw = self.mem[name].to_host(np.uint8, self.mem[name].nbytes)
        assert np.all(raw[:GUARD] == 0x5A) and np.all(raw[-GUARD:] == 0x5A), f"written outside {name}"
        return raw[GUARD:-GUARD].view(a.dtype).reshape(a.shape)

    def same(self, names=NAMES):
        for name in names:
            got, want = self.get(name), getattr(self.o, name)
            bad = np.argwhere(got != want)
            assert len(bad) == 0, f"{name}: {len(bad)} differ, first at {bad[0]}: {got[tuple(bad[0])]} for {want[tuple(bad[0])]}"


def invariants(o: Oracle):
    """Every page is held as often as it is counted."""
    held = np.bincount(o.table[o.table >= 0], minlength=o.pages)
    assert np.array_equal(held, o.refs)


def values(rng, shape, dtype, size=1.0):
    """Random rows in the type's words and as the float32 values that these are."""
    from tests.rows import pack
    words = pack((size * rng.standard_normal(shape)).astype(np.float32), dtype)
    return words, unpack(words, dtype).astype(np.float32)


__all__ = ["BF16", "F16", "F32", "Held", "Oracle", "invariants", "values"]
