"""Helpers for the tests of the operators on rows: the three row types in numpy, rows with strides in device memory, captured
launches, and the operators' definitions in 64 bits."""
from __future__ import annotations

import ctypes as C

import numpy as np

from paper_2302_07863_amd import binding as b
from tests.hipmem import DeviceArray, hip

F32, BF16, F16 = b.DT_F32, b.DT_BF16, b.DT_F16
WORD = {F32: np.float32, BF16: np.uint16, F16: np.float16}
U32 = 2.0 ** -24                                     # half a step of fp32, relative
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}   # steps near zero


def close(got, want, tol) -> None:
    off = np.abs(np.asarray(got, dtype=np.float64) - want)
    bad = ~(off <= tol)
    if np.any(bad):
        at = np.unravel_index(np.argmax(np.where(bad, off / np.maximum(tol, 1e-300), 0)), bad.shape)
        raise AssertionError(f"{int(bad.sum())} of {bad.size} values, worst at {tuple(int(i) for i in at)}: {got[at]} for {want[at]}, tolerance {np.broadcast_to(tol, bad.shape)[at]}")


def pack(a, dtype: int) -> np.ndarray:
    """float values as words of the row type (nearest even)."""
    a = np.asarray(a, dtype=np.float32)
    if dtype != BF16:
        return a.astype(WORD[dtype])
    u = a.view(np.uint32).astype(np.uint64)
    up = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(a), np.uint16(0x7FC0), up)


def unpack(words, dtype: int) -> np.ndarray:
    """words of the row type as float64."""
    words = np.asarray(words)
    if dtype != BF16:
        return words.astype(np.float64)
    return (words.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


class Rows:
    """A [rows][cols] array with a row stride and a first element of its own inside a larger device buffer, whose other
    words hold a pattern that nobody may touch."""

    def __init__(self, words: np.ndarray, stride: int | None = None, first: int = 0):
        self.shape, self.word = words.shape, words.dtype
        rows, cols = words.shape
        self.stride, self.first = cols if stride is None else stride, first
        self.host = np.frombuffer(b"\x55" * ((first + (rows - 1) * self.stride + cols + 64) * words.itemsize), dtype=words.dtype).copy()
        self._view(self.host)[...] = words
        self.dev = DeviceArray(self.host)
        self.ptr = self.dev.ptr.value + first * words.itemsize

    def _view(self, flat):
        rows, cols = self.shape
        return np.lib.stride_tricks.as_strided(flat[self.first:], (rows, cols), (self.stride * flat.itemsize, flat.itemsize))

    def get(self) -> np.ndarray:
        """The rows as they are now; every word between and around them has to be what it was."""
        now = self.dev.to_host(self.word, len(self.host))
        out = self._view(now).copy()
        raw = now.copy()
        self._view(raw)[...] = self._view(self.host)
        assert raw.tobytes() == self.host.tobytes(), "a word outside the rows was written"
        return out


class Stream:
    def __init__(self):
        self.h = C.c_void_p()
        assert hip().hipStreamCreateWithFlags(C.byref(self.h), 1) == 0    # (does not wait for the default stream)

    def sync(self):
        assert hip().hipStreamSynchronize(self.h) == 0

    def close(self):
        if self.h:
            hip().hipStreamDestroy(self.h)
            self.h = C.c_void_p()

    __del__ = close


class Graph:
    """What `launch(stream)` puts on a stream, captured."""

    def __init__(self, stream: Stream, launch):
        h = hip()
        h.hipStreamBeginCapture.argtypes = [C.c_void_p, C.c_int]
        h.hipStreamEndCapture.argtypes = [C.c_void_p, C.POINTER(C.c_void_p)]
        h.hipGraphInstantiate.argtypes = [C.POINTER(C.c_void_p), C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t]
        h.hipGraphLaunch.argtypes = [C.c_void_p, C.c_void_p]
        h.hipStreamSynchronize.argtypes = [C.c_void_p]
        h.hipGraphExecDestroy.argtypes = [C.c_void_p]
        h.hipGraphDestroy.argtypes = [C.c_void_p]
        self.stream, self.exec = stream, C.c_void_p()
        g = C.c_void_p()
        assert h.hipStreamBeginCapture(stream.h, 1) == 0                  # (this thread's calls alone)
        launch(stream.h.value)
        assert h.hipStreamEndCapture(stream.h, C.byref(g)) == 0
        assert h.hipGraphInstantiate(C.byref(self.exec), g, None, None, 0) == 0
        h.hipGraphDestroy(g)

    def replay(self):
        assert hip().hipGraphLaunch(self.exec, self.stream.h) == 0

    def close(self):
        if self.exec:
            hip().hipGraphExecDestroy(self.exec)
            self.exec = C.c_void_p()

    __del__ = close


# ------------------------------------------------------------------------------------------------ definitions in 64 bits
def scale_words(a, dtype: int) -> np.ndarray:
    w = pack(a, dtype)
    return w.view(np.uint16)


def scales_of(words, dtype: int) -> np.ndarray:
    return unpack(words.view(np.float16) if dtype == F16 else words, dtype)


def weights(codes, scales, zeros, k: int, group: int) -> np.ndarray:
    """[n][k] of a matrix in 4 bits; scales as float64."""
    q = np.stack((codes & 15, codes >> 4), axis=2).reshape(len(codes), -1)[:, :k].astype(np.float64)
    g = np.arange(k) // group
    z = 8.0 if zeros is None else zeros.astype(np.float64)[:, g]
    return (q - z) * scales[:, g]


def normed(x, gain, eps: float) -> np.ndarray:
    return x if gain is None else x * gain / np.sqrt(np.mean(x * x, axis=1, keepdims=True) + eps)


def turned(x, positions, frequencies, magnitude: float, halves: bool, inverse: bool = False) -> np.ndarray:
    """x [tokens][heads][d_head]"""
    half = len(frequencies)
    a = np.asarray(positions, dtype=np.float64)[:, None] * frequencies * (-1.0 if inverse else 1.0)
    c, s = (magnitude * np.cos(a))[:, None, :], (magnitude * np.sin(a))[:, None, :]
    out = x.copy()
    iu = np.arange(half) if halves else 2 * np.arange(half)
    iv = iu + half if halves else iu + 1
    u, v = x[..., iu], x[..., iv]
    out[..., iu], out[..., iv] = u * c - v * s, u * s + v * c
    return out


def ruled(z, tokens=None, length=None, start=0, penalties=None, bias_ids=None, bias=None, allowed=None):
    """One row of logits after the rules; tokens of the row, the first `length` of which count."""
    z = np.array(z, dtype=np.float64)
    vocab = len(z)
    if tokens is not None:
        length = min(max(int(length), 0), len(tokens))
        rep, freq, pres = (float(p) for p in penalties)
        seen, made = set(), {}
        for i, t in enumerate(np.asarray(tokens[:length]).tolist()):
            if 0 <= t < vocab:
                seen.add(t)
                if i >= start:
                    made[t] = made.get(t, 0) + 1
        for t in seen:
            z[t] = z[t] / rep if z[t] > 0 else z[t] * rep
        for t, c in made.items():
            z[t] = z[t] - freq * c - pres
    if bias_ids is not None:
        last = {int(t): float(v) for t, v in zip(bias_ids, bias) if 0 <= int(t) < vocab}
        for t, v in last.items():
            z[t] += v
    if allowed is not None:
        z[~np.asarray(allowed, dtype=bool)] = -np.inf
    return z


def mask_words(allowed) -> np.ndarray:
    """[..][vocab] truth values as the words of a mask."""
    a = np.asarray(allowed, dtype=bool)
    pad = (-a.shape[-1]) % 32
    a = np.concatenate((a, np.ones(a.shape[:-1] + (pad,), bool)), axis=-1)   # (bits behind the vocabulary: nobody's)
    return np.ascontiguousarray(np.packbits(a, axis=-1, bitorder="little")).view(np.uint32)
