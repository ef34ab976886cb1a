"""Thin ctypes binding of libbild.so: argument marshalling only.  Every step of
the decoding path runs in the library's HIP kernels; there is no Python or CPU
fallback, and a missing library is an error."""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Optional, Sequence

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libbild.so")

OK, EINVAL, ESTATE, ECAP, EHIP, ENOMEM = 0, -1, -2, -3, -4, -5
MAX_ROWS = 32
SMALL, LARGE, BOTH = 1, 2, 3
DT_F32, DT_BF16, DT_F16 = 0, 1, 2
ROTARY_NONE, ROTARY_LINEAR, ROTARY_BASE, ROTARY_BANDS, ROTARY_YARN = 0, 1, 2, 3, 4
ACCEPT_THRESHOLD, ACCEPT_REJECTION = 0, 1


class ModelConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_enc_layers", "n_dec_layers", "d_model", "n_heads", "d_head", "d_ff", "act", "pos", "vocab",
        "tied_head", "dtype", "cross_attn", "bos", "tie_shift")] + [
        (n, C.c_float) for n in ("logit_scale", "embed_scale", "norm_eps", "rope_base")] + [
        ("rel_max_dist", C.c_int32)]


class Stats(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "small_steps", "large_calls", "rows_verified", "fallbacks_conf", "fallbacks_forced", "rollbacks",
        "tokens_discarded", "n_generated")]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class Profile(C.Structure):
    _fields_ = [("launches", (C.c_int64 * 2) * 2), ("bytes", (C.c_int64 * 2) * 2), ("ms", (C.c_double * 2) * 2),
                ("dropped", C.c_int32)]


class QuantCall(C.Structure):
    _fields_ = [("x", C.c_void_p), ("x_stride", C.c_int64), ("y", C.c_void_p), ("y_stride", C.c_int64), ("gain", C.c_void_p),
                ("rows", C.c_int32), ("x_dtype", C.c_int32), ("y_dtype", C.c_int32), ("eps", C.c_float), ("scale", C.c_float)]


class RotaryConfig(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("layout", "rot_dim", "scaling", "original")] + [
        (n, C.c_float) for n in ("base", "factor", "low", "high", "magnitude")]


class RotaryRowsStruct(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("src_token", C.c_int64), ("src_head", C.c_int64), ("dst_token", C.c_int64),
                ("dst_head", C.c_int64), ("heads", C.c_int32), ("reserved", C.c_int32)]


class RotaryRows:
    """Rows that Rotary.apply turns: device pointers, strides in elements."""
    __slots__ = ("fields",)

    def __init__(self, src: Optional[int] = None, dst: Optional[int] = None, heads: int = 0, src_token: int = 0, src_head: int = 0, dst_token: int = 0,
                 dst_head: int = 0):
        self.fields = (src or 0, dst or 0, src_token, src_head, dst_token, dst_head, heads, 0)


_NO_ROWS = RotaryRows()


class RotaryCall(C.Structure):
    _fields_ = [("q", RotaryRowsStruct), ("k", RotaryRowsStruct), ("positions", C.c_void_p)] + [
        (n, C.c_int32) for n in ("first", "tokens", "d_head", "dtype", "inverse", "reserved")]


class RulesCall(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("logits_stride", C.c_int64), ("out", C.c_void_p), ("out_stride", C.c_int64), ("targets", C.c_void_p),
                ("stats", C.c_void_p), ("tokens", C.c_void_p), ("tokens_stride", C.c_int64), ("lengths", C.c_void_p), ("starts", C.c_void_p),
                ("penalties", C.c_void_p), ("penalties_stride", C.c_int64), ("bias_ids", C.c_void_p), ("bias", C.c_void_p),
                ("bias_stride", C.c_int64), ("bias_counts", C.c_void_p), ("mask", C.c_void_p), ("mask_stride", C.c_int64),
                ("rows", C.c_int32), ("dtype", C.c_int32), ("max_tokens", C.c_int32), ("max_bias", C.c_int32)]


# The calls' structs as bytes: one packing costs less than setting a ctypes structure field by field.
_QUANT_CALL = struct.Struct("@PqPqPiiiff4x")
_ROTARY_CALL = struct.Struct("@PPqqqqiiPPqqqqiiPiiiiii")
_RULES_CALL = struct.Struct("@PqPqPPPqPPPqPPqPPqiiii")
assert _QUANT_CALL.size == C.sizeof(QuantCall) and _ROTARY_CALL.size == C.sizeof(RotaryCall) and _RULES_CALL.size == C.sizeof(RulesCall)


class BildError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {code} ({strerror(code)})")
        self.code = code


_lib = None

_SIGS = {
    "bild_model_num_tensors": (C.c_int, [C.POINTER(ModelConfig)]),
    "bild_model_create": (C.c_int, [C.POINTER(ModelConfig), C.POINTER(C.c_void_p), C.c_int, C.POINTER(C.c_void_p)]),
    "bild_model_create_rotary": (C.c_int, [C.POINTER(ModelConfig), C.POINTER(RotaryConfig), C.POINTER(C.c_void_p), C.c_int, C.POINTER(C.c_void_p)]),
    "bild_model_destroy": (C.c_int, [C.c_void_p]),
    "bild_pair_create": (C.c_int, [C.c_void_p, C.c_void_p, C.POINTER(C.c_void_p)]),
    "bild_pair_create_early_exit": (C.c_int, [C.c_void_p, C.c_int, C.c_float, C.POINTER(C.c_void_p)]),
    "bild_pair_destroy": (C.c_int, [C.c_void_p]),
    "bild_state_create": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.POINTER(C.c_void_p)]),
    "bild_state_destroy": (C.c_int, [C.c_void_p]),
    "bild_encode": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int]),
    "bild_small_step": (C.c_int, [C.c_void_p, C.c_float, C.POINTER(C.c_int32), C.POINTER(C.c_int32),
                                  C.POINTER(C.c_float)]),
    "bild_large_verify": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_float, C.c_void_p, C.POINTER(C.c_int32),
                                    C.POINTER(C.c_int32), C.c_void_p]),
    "bild_set_sampling": (C.c_int, [C.c_void_p, C.c_float, C.c_void_p, C.c_void_p, C.c_int]),
    "bild_set_acceptance": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_int]),
    "bild_set_quant_head": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p]),
    "bild_set_rules": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int]),
    "bild_set_masks": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_void_p]),
    "bild_kv_truncate": (C.c_int, [C.c_void_p, C.c_int, C.c_int]),
    "bild_seq_truncate": (C.c_int, [C.c_void_p, C.c_int]),
    "bild_force_tokens": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_int]),
    "bild_generate": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_float, C.c_float, C.c_int, C.c_int32,
                                C.c_void_p, C.POINTER(C.c_int32), C.POINTER(Stats)]),
    "bild_greedy": (C.c_int, [C.c_void_p, C.c_int, C.c_void_p, C.c_int, C.c_int, C.c_int32, C.c_void_p,
                              C.POINTER(C.c_int32)]),
    "bild_head_stats": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]),
    "bild_head_stats_static": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]),
    "bild_quant_round": (C.c_int, [C.c_void_p] + [C.c_int] * 5 + [C.c_void_p] * 3),
    "bild_quant_create": (C.c_int, [C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.POINTER(C.c_void_p)]),
    "bild_quant_destroy": (C.c_int, [C.c_void_p]),
    "bild_quant_matmul": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "bild_rotary_frequencies": (C.c_int, [C.POINTER(RotaryConfig), C.c_void_p, C.POINTER(C.c_double)]),
    "bild_rotary_create": (C.c_int, [C.POINTER(RotaryConfig), C.POINTER(C.c_void_p)]),
    "bild_rotary_destroy": (C.c_int, [C.c_void_p]),
    "bild_rotary_apply": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "bild_rules_create": (C.c_int, [C.c_int, C.c_int, C.POINTER(C.c_void_p)]),
    "bild_rules_destroy": (C.c_int, [C.c_void_p]),
    "bild_rules_apply": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p]),
    "bild_get_lengths": (C.c_int, [C.c_void_p] + [C.POINTER(C.c_int32)] * 4),
    "bild_get_sequence": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.POINTER(C.c_int32)]),
    "bild_debug_enable_logits": (C.c_int, [C.c_void_p, C.c_int]),
    "bild_debug_logits": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_void_p]),
    "bild_debug_kv": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p]),
    "bild_bench_pass": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_float)]),
    "bild_bench_gemm": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_float), C.POINTER(C.c_int64),
                                  C.POINTER(C.c_int64)]),
    "bild_gemm_tally": (C.c_int, [C.c_void_p, C.POINTER(C.c_int64), C.POINTER(C.c_int64), C.c_int]),
    "bild_pass_stages": (C.c_int, [C.c_void_p, C.POINTER(C.c_int32)]),
    "bild_pass_routes": (C.c_int, [C.c_void_p, C.POINTER(C.c_int64)]),
    "bild_debug_pass_spins": (C.c_int, [C.c_void_p, C.c_int]),
    "bild_probe_stream": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_float)]),
    "bild_probe_occupy": (C.c_int, [C.c_void_p, C.c_int, C.c_int]),
    "bild_probe_launch": (C.c_int, [C.c_void_p, C.c_int, C.POINTER(C.c_float)]),
    "bild_debug_tiled_bytes": (C.c_int64, [C.c_int, C.c_int, C.c_int]),
    "bild_debug_tile_matrix": (C.c_int, [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p]),
    "bild_debug_cache_rule": (C.c_int, [C.c_int, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int32)]),
    "bild_debug_wide_split": (C.c_int, [C.c_int] * 6 + [C.POINTER(C.c_int32)]),
    "bild_debug_wide_split_rows": (C.c_int, [C.c_int] * 7 + [C.POINTER(C.c_int32)]),
    "bild_debug_head_route": (C.c_int, [C.c_int] * 4),
    "bild_debug_tile_shape": (C.c_int, [C.c_int] * 5 + [C.POINTER(C.c_int32)]),
    "bild_debug_attn_shape": (C.c_int, [C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int32)]),
    "bild_debug_gemm_shape": (C.c_int, [C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int32)]),
    "bild_probe_copy": (C.c_int, [C.c_void_p, C.c_int64, C.c_int]),
    "bild_profile_begin": (C.c_int, [C.c_void_p, C.c_int]),
    "bild_profile_end": (C.c_int, [C.c_void_p, C.POINTER(Profile)]),
    "bild_pass_bytes": (C.c_int64, [C.c_void_p, C.c_int, C.c_int, C.c_int]),
    "bild_strerror": (C.c_char_p, [C.c_int]),
}


def exported_symbols() -> list:
    return sorted(_SIGS)


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'`")
        l = C.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            fn = getattr(l, name)
            fn.restype, fn.argtypes = res, args
        _lib = l
    return _lib


def strerror(code: int) -> str:
    return lib().bild_strerror(code).decode()


def _check(code: int, what: str):
    if code != OK:
        raise BildError(code, what)


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def config_from_shape(shape) -> ModelConfig:
    """ModelConfig from a bild_inputs.ModelShape-like record (plain field copy)."""
    return ModelConfig(n_enc_layers=shape.n_enc, n_dec_layers=shape.n_dec, d_model=shape.d, n_heads=shape.heads,
                       d_head=shape.d_head, d_ff=shape.d_ff, act=shape.act, pos=shape.pos, vocab=shape.vocab,
                       tied_head=int(shape.tied), dtype=shape.dtype, cross_attn=int(shape.cross), bos=shape.bos,
                       tie_shift=shape.tie_shift, logit_scale=shape.logit_scale, embed_scale=shape.embed_scale,
                       norm_eps=shape.eps, rope_base=shape.rope_base,
                       rel_max_dist=getattr(shape, "rel_max_dist", 0))


class Model:
    h = None

    def __init__(self, cfg: ModelConfig, tensors: Sequence[np.ndarray], rotary: Optional[RotaryConfig] = None):
        """rotary: the positions of a network with pos = BILD_POS_ROPE (None: pairs (2i, 2i + 1) of the whole head, cfg.rope_base)."""
        arrs = [np.ascontiguousarray(t, dtype=np.float32) for t in tensors]
        ptrs = (C.c_void_p * len(arrs))(*[a.ctypes.data for a in arrs])
        h = C.c_void_p()
        if rotary is None:
            _check(lib().bild_model_create(C.byref(cfg), ptrs, len(arrs), C.byref(h)), "bild_model_create")
        else:
            _check(lib().bild_model_create_rotary(C.byref(cfg), C.byref(rotary), ptrs, len(arrs), C.byref(h)), "bild_model_create_rotary")
        self.h, self.cfg = h, cfg

    def close(self):
        if self.h:
            lib().bild_model_destroy(self.h)
            self.h = None

    __del__ = close


ROW_STATS_DTYPE = np.dtype([("zmax", np.float32), ("lse", np.float32), ("argmax", np.int32), ("z_target", np.float32)])


def head_stats(model: Model, x_dev_ptr: int, rows: int, targets_dev_ptr: Optional[int], out_dev_ptr: int,
               stream: Optional[int] = None, entry: str = "bild_head_stats"):
    """Device pointers in, device pointer out (rows records of ROW_STATS_DTYPE); see bild.h."""
    _check(getattr(lib(), entry)(model.h, C.c_void_p(x_dev_ptr), rows, C.c_void_p(targets_dev_ptr or 0),
                                 C.c_void_p(out_dev_ptr), C.c_void_p(stream or 0)), entry)


def _where(a) -> Optional[int]:
    """Address of a host array, or a device pointer as it is."""
    return a.ctypes.data if isinstance(a, np.ndarray) else a


def _sized(a, count: int, itemsize: int, what: str):
    """A host array in one piece, which has to have what the library reads of it; a device pointer as it is."""
    if not isinstance(a, np.ndarray):
        return a
    if a.size != count or a.itemsize != itemsize:
        raise BildError(EINVAL, f"{what}, an array of {a.size} x {a.itemsize} bytes for {count} x {itemsize}")
    return np.ascontiguousarray(a)


def quant_round(w: np.ndarray, group: int, scale_dtype: int = DT_F16, zeros: bool = False, inputs_first: bool = False):
    """Rounds an fp32 matrix ([n][k]; inputs_first: [k][n]) to 4 bits; (codes, scales as 16-bit words, zeros or None), see bild.h."""
    a = np.ascontiguousarray(w, dtype=np.float32)
    n, k = a.shape[::-1] if inputs_first else a.shape
    groups = -(-k // group) if group > 0 else 0
    codes, scales = np.zeros((n, (k + 1) // 2), np.uint8), np.zeros((n, groups), np.uint16)
    z = np.zeros((n, groups), np.uint8) if zeros else None
    _check(lib().bild_quant_round(a.ctypes.data, n, k, int(inputs_first), group, scale_dtype, codes.ctypes.data, scales.ctypes.data,
                                  z.ctypes.data if zeros else None), "bild_quant_round")
    return codes, scales, z


class Quant:
    """A matrix in 4 bits on the device.  codes, scales, zeros: host arrays (uint8, 16-bit, uint8) or device pointers."""
    h = None

    def __init__(self, n: int, k: int, group: int, codes, scales, scale_dtype: int, zeros=None):
        h = C.c_void_p()
        groups = -(-k // group) if group > 0 else 0
        codes, scales, zeros = [_sized(a, n * each, size, "bild_quant_create") for a, each, size in ((codes, (k + 1) // 2, 1), (scales, groups, 2), (zeros, groups, 1))]
        _check(lib().bild_quant_create(n, k, group, _where(codes), _where(scales), scale_dtype, _where(zeros), C.byref(h)), "bild_quant_create")
        self.h, self.n, self.k, self._matmul = h, n, k, lib().bild_quant_matmul   # (looked up once: a call is as long as a small kernel)

    def matmul(self, x: int, x_dtype: int, rows: int, y: int, y_dtype: int, x_stride: Optional[int] = None, y_stride: Optional[int] = None,
               gain: Optional[int] = None, eps: float = 0.0, scale: float = 1.0, stream: Optional[int] = None):
        """Device pointers; strides in elements (None: rows side by side)."""
        call = _QUANT_CALL.pack(x or 0, self.k if x_stride is None else x_stride, y or 0, self.n if y_stride is None else y_stride, gain or 0, rows,
                                x_dtype, y_dtype, eps, scale)
        code = self._matmul(self.h, call, stream)
        if code != OK:
            raise BildError(code, "bild_quant_matmul")

    def close(self):
        if self.h:
            lib().bild_quant_destroy(self.h)
            self.h = None

    __del__ = close


class Rotary:
    h = None

    def __init__(self, rot_dim: int, halves: bool = False, base: float = 10000.0, scaling: int = ROTARY_NONE, factor: float = 1.0,
                 original: int = 0, low: float = 0.0, high: float = 0.0, magnitude: float = 0.0):
        self.cfg = RotaryConfig(int(halves), rot_dim, scaling, original, base, factor, low, high, magnitude)
        h = C.c_void_p()
        _check(lib().bild_rotary_create(C.byref(self.cfg), C.byref(h)), "bild_rotary_create")
        self.h, self._apply = h, lib().bild_rotary_apply

    def frequencies(self):
        f, m = np.zeros(self.cfg.rot_dim // 2, np.float64), C.c_double()
        _check(lib().bild_rotary_frequencies(C.byref(self.cfg), f.ctypes.data, C.byref(m)), "bild_rotary_frequencies")
        return f, m.value

    def apply(self, d_head: int, dtype: int, tokens: int, q: RotaryRows, k: Optional[RotaryRows] = None, positions: Optional[int] = None,
              first: int = 0, inverse: bool = False, stream: Optional[int] = None):
        call = _ROTARY_CALL.pack(*q.fields, *(k or _NO_ROWS).fields, positions or 0, first, tokens, d_head, dtype, int(inverse), 0)
        code = self._apply(self.h, call, stream)
        if code != OK:
            raise BildError(code, "bild_rotary_apply")

    def close(self):
        if self.h:
            lib().bild_rotary_destroy(self.h)
            self.h = None

    __del__ = close


class Rules:
    h = None

    def __init__(self, vocab: int, max_rows: int):
        h = C.c_void_p()
        _check(lib().bild_rules_create(vocab, max_rows, C.byref(h)), "bild_rules_create")
        self.h, self.vocab, self._apply = h, vocab, lib().bild_rules_apply

    def apply(self, logits: int, dtype: int, rows: int, out: Optional[int] = None, stats: Optional[int] = None, targets: Optional[int] = None,
              logits_stride: Optional[int] = None, out_stride: Optional[int] = None, tokens: Optional[int] = None, tokens_stride: int = 0,
              lengths: Optional[int] = None, starts: Optional[int] = None, penalties: Optional[int] = None, penalties_stride: int = 0,
              bias_ids: Optional[int] = None, bias: Optional[int] = None, bias_stride: int = 0, bias_counts: Optional[int] = None,
              mask: Optional[int] = None, mask_stride: int = 0, max_tokens: int = 0, max_bias: int = 0, stream: Optional[int] = None):
        """The fields of bild_rules_call by name: device pointers, strides in elements (None: rows side by side)."""
        call = _RULES_CALL.pack(logits or 0, self.vocab if logits_stride is None else logits_stride, out or 0, self.vocab if out_stride is None else out_stride,
                                targets or 0, stats or 0, tokens or 0, tokens_stride, lengths or 0, starts or 0, penalties or 0, penalties_stride,
                                bias_ids or 0, bias or 0, bias_stride, bias_counts or 0, mask or 0, mask_stride, rows, dtype, max_tokens, max_bias)
        code = self._apply(self.h, call, stream)
        if code != OK:
            raise BildError(code, "bild_rules_apply")

    def close(self):
        if self.h:
            lib().bild_rules_destroy(self.h)
            self.h = None

    __del__ = close


class Pair:
    h = None

    def __init__(self, small: Model, large: Model):
        h = C.c_void_p()
        _check(lib().bild_pair_create(small.h, large.h, C.byref(h)), "bild_pair_create")
        self.h, self.small, self.large = h, small, large

    @classmethod
    def early_exit(cls, large: Model, k: int, small_logit_scale: float) -> "Pair":
        """The small model is the first k decoder layers of `large` with the shared head."""
        h = C.c_void_p()
        _check(lib().bild_pair_create_early_exit(large.h, k, small_logit_scale, C.byref(h)), "bild_pair_create_early_exit")
        self = cls.__new__(cls)
        self.h, self.small, self.large = h, None, large
        return self

    def close(self):
        if self.h:
            lib().bild_pair_destroy(self.h)
            self.h = None

    __del__ = close


class State:
    h = None

    def __init__(self, pair: Pair, max_src: int, max_len: int, n_max: int = 10, stream: Optional[int] = None):
        h = C.c_void_p()
        _check(lib().bild_state_create(pair.h, max_src, max_len, n_max, C.c_void_p(stream or 0), C.byref(h)),
               "bild_state_create")
        self.h, self.pair, self.max_len = h, pair, max_len

    def close(self):
        if self.h:
            lib().bild_state_destroy(self.h)
            self.h = None

    __del__ = close

    def encode(self, src):
        a = _i32(src)
        _check(lib().bild_encode(self.h, a.ctypes.data, len(a)), "bild_encode")

    def small_step(self, alpha_fb: float):
        tok, flag, pm = C.c_int32(), C.c_int32(), C.c_float()
        _check(lib().bild_small_step(self.h, alpha_fb, C.byref(tok), C.byref(flag), C.byref(pm)), "bild_small_step")
        return tok.value, flag.value, pm.value

    def large_verify(self, alpha_rb: float, draft=None):
        if draft is None:
            n, dptr, cap = 0, None, MAX_ROWS
        else:
            d = _i32(draft)
            n, dptr, cap = len(d), d.ctypes.data, len(d) + 1
        out = np.zeros(max(cap, 1), dtype=np.int32)
        nll = np.zeros(MAX_ROWS, dtype=np.float32)
        n_out, r = C.c_int32(), C.c_int32()
        _check(lib().bild_large_verify(self.h, dptr, n, alpha_rb, out.ctypes.data, C.byref(n_out), C.byref(r),
                                       nll.ctypes.data), "bild_large_verify")
        return out[:n_out.value].tolist(), r.value, nll

    def kv_truncate(self, which: int, pos: int):
        _check(lib().bild_kv_truncate(self.h, which, pos), "bild_kv_truncate")

    def set_sampling(self, top_p: float, u_small=None, u_large=None):
        """top_p <= 0 returns to argmax decoding."""
        if top_p <= 0:
            _check(lib().bild_set_sampling(self.h, float(top_p), None, None, 0), "bild_set_sampling")
            return
        a = np.ascontiguousarray(u_small, dtype=np.float32)
        b = np.ascontiguousarray(u_large, dtype=np.float32)
        _check(lib().bild_set_sampling(self.h, float(top_p), a.ctypes.data, b.ctypes.data, min(len(a), len(b))),
               "bild_set_sampling")

    def seq_truncate(self, n_keep: int):
        _check(lib().bild_seq_truncate(self.h, n_keep), "bild_seq_truncate")

    def set_acceptance(self, rule: int, u_accept=None):
        """rule: ACCEPT_THRESHOLD (the paper's rollback policy) or ACCEPT_REJECTION (needs set_sampling first)."""
        if u_accept is None:
            _check(lib().bild_set_acceptance(self.h, int(rule), None, 0), "bild_set_acceptance")
            return
        a = np.ascontiguousarray(u_accept, dtype=np.float32)
        _check(lib().bild_set_acceptance(self.h, int(rule), a.ctypes.data, len(a)), "bild_set_acceptance")

    def set_quant_head(self, which: int, head: Optional["Quant"]):
        """A 4-bit matrix in place of the LM head of model `which` (None: the model's own)."""
        if head is not None and not head.h:                          # (closed: not the model's own)
            raise BildError(EINVAL, "bild_set_quant_head")
        _check(lib().bild_set_quant_head(self.h, which, head.h if head is not None else None), "bild_set_quant_head")
        self._heads = {**getattr(self, "_heads", {}), which: head}   # (borrowed by the state)

    def set_rules(self, penalties=None, bias=None):
        """penalties: (repetition, frequency, presence) or None; bias: {id: value} or None."""
        p = _sized(np.asarray(penalties, dtype=np.float32), 3, 4, "bild_set_rules") if penalties is not None else None
        bias = bias or {}
        ids, values = _i32(list(bias.keys())), np.asarray(list(bias.values()), dtype=np.float32)
        _check(lib().bild_set_rules(self.h, p.ctypes.data if p is not None else None, ids.ctypes.data if len(ids) else None,
                                    values.ctypes.data if len(ids) else None, len(ids)), "bild_set_rules")

    def set_masks(self, first: int, masks=None, n: int = 0):
        """masks [n][ceil(vocab / 32)] uint32 for the tokens at positions first .. first + n - 1; None: all ids at n positions."""
        if masks is not None:
            masks = np.asarray(masks, dtype=np.uint32)
            n = masks.shape[0] if masks.ndim == 2 else 1
            masks = _sized(masks, n * ((self.pair.large.cfg.vocab + 31) // 32), 4, "bild_set_masks")
        _check(lib().bild_set_masks(self.h, first, n, masks.ctypes.data if masks is not None else None), "bild_set_masks")

    def force_tokens(self, first: int, tokens, draft_start: int):
        a = _i32(tokens)
        _check(lib().bild_force_tokens(self.h, first, a.ctypes.data if len(a) else None, len(a), draft_start),
               "bild_force_tokens")

    def generate(self, src, alpha_fb: float, alpha_rb: float, max_new: int, eos: int = -1):
        """src=None continues from the encoded state without re-encoding."""
        a = _i32(src if src is not None else [])
        out = np.zeros(max(max_new, 1), dtype=np.int32)
        n, st = C.c_int32(), Stats()
        _check(lib().bild_generate(self.h, a.ctypes.data if src is not None else None, len(a), alpha_fb, alpha_rb, max_new, eos, out.ctypes.data,
                                   C.byref(n), C.byref(st)), "bild_generate")
        return out[:n.value].tolist(), st.as_dict()

    def greedy(self, which: int, src, max_new: int, eos: int = -1):
        a = _i32(src if src is not None else [])
        out = np.zeros(max(max_new, 1), dtype=np.int32)
        n = C.c_int32()
        _check(lib().bild_greedy(self.h, which, a.ctypes.data if src is not None else None, len(a), max_new, eos, out.ctypes.data, C.byref(n)),
               "bild_greedy")
        return out[:n.value].tolist()

    def lengths(self):
        v = [C.c_int32() for _ in range(4)]
        _check(lib().bild_get_lengths(self.h, *[C.byref(x) for x in v]), "bild_get_lengths")
        return dict(y_len=v[0].value, draft_start=v[1].value, len_small=v[2].value, len_large=v[3].value)

    def sequence(self):
        out = np.zeros(self.max_len + 1, dtype=np.int32)
        n = C.c_int32()
        _check(lib().bild_get_sequence(self.h, out.ctypes.data, len(out), C.byref(n)), "bild_get_sequence")
        return out[:n.value].tolist()

    def debug_enable_logits(self, enable: bool = True):
        _check(lib().bild_debug_enable_logits(self.h, int(enable)), "bild_debug_enable_logits")

    def debug_logits(self, which: int, row: int) -> np.ndarray:
        v = self.pair.large.cfg.vocab
        out = np.zeros(v, dtype=np.float32)
        _check(lib().bild_debug_logits(self.h, which, row, out.ctypes.data), "bild_debug_logits")
        return out

    def debug_kv(self, which: int, layer: int, is_v: bool, pos0: int, n: int) -> np.ndarray:
        """Cached keys or values of one decoder layer, rows pos0..pos0+n-1, as [n][heads*d_head] float32."""
        cfg = (self.pair.large if which == LARGE or self.pair.small is None else self.pair.small).cfg
        out = np.zeros((n, cfg.n_heads * cfg.d_head), dtype=np.float32)
        _check(lib().bild_debug_kv(self.h, which, layer, int(is_v), pos0, n, out.ctypes.data), "bild_debug_kv")
        return out

    def bench_pass(self, which: int, rows: int, reps: int) -> float:
        ms = C.c_float()
        _check(lib().bild_bench_pass(self.h, which, rows, reps, C.byref(ms)), "bild_bench_pass")
        return ms.value

    def bench_gemm(self, which: int, rows: int, reps: int) -> dict:
        ms, n, b = C.c_float(), C.c_int64(), C.c_int64()
        _check(lib().bild_bench_gemm(self.h, which, rows, reps, C.byref(ms), C.byref(n), C.byref(b)), "bild_bench_gemm")
        return dict(ms_per_pass=ms.value, launches=n.value, bytes=b.value)

    def pass_stages(self) -> int:
        n = C.c_int32()
        _check(lib().bild_pass_stages(self.h, C.byref(n)), "bild_pass_stages")
        return n.value

    def pass_routes(self) -> dict:
        out = (C.c_int64 * 4)()
        _check(lib().bild_pass_routes(self.h, out), "bild_pass_routes")
        return dict(zip(("chip", "die", "kernels", "gave_up"), out))

    def debug_pass_spins(self, spins: int):
        _check(lib().bild_debug_pass_spins(self.h, spins), "bild_debug_pass_spins")

    def gemm_tally(self, reset: bool = False) -> dict:
        n, b = C.c_int64(), C.c_int64()
        _check(lib().bild_gemm_tally(self.h, C.byref(n), C.byref(b), int(reset)), "bild_gemm_tally")
        return dict(launches=n.value, bytes=b.value)

    def probe_stream(self, groups: int, kib_per_group: int, reps: int = 8) -> float:
        us = C.c_float()
        _check(lib().bild_probe_stream(self.h, groups, kib_per_group, reps, C.byref(us)), "bild_probe_stream")
        return us.value

    def probe_launch(self, reps: int = 2000) -> float:
        us = C.c_float()
        _check(lib().bild_probe_launch(self.h, reps, C.byref(us)), "bild_probe_launch")
        return us.value

    def probe_copy(self, nbytes: int, reps: int = 1):
        _check(lib().bild_probe_copy(self.h, nbytes, reps), "bild_probe_copy")

    def profile_begin(self, max_records: int = 65536):
        _check(lib().bild_profile_begin(self.h, max_records), "bild_profile_begin")

    def profile_end(self) -> dict:
        p = Profile()
        _check(lib().bild_profile_end(self.h, C.byref(p)), "bild_profile_end")
        out = {}
        for mi, mn in enumerate(("small", "large")):
            for ci, cn in enumerate(("layers", "lm_head")):
                out[f"{mn}.{cn}"] = dict(launches=p.launches[mi][ci], bytes=p.bytes[mi][ci], ms=p.ms[mi][ci])
        out["dropped"] = p.dropped
        return out

    def pass_bytes(self, which: int, t_cache: int, rows: int = 1) -> int:
        return int(lib().bild_pass_bytes(self.h, which, t_cache, rows))


def tile_matrix(src: np.ndarray, src_is_k_by_n: bool, dtype: int) -> np.ndarray:
    """Host re-layout of a matrix into the kernels' streaming tile order (bytes)."""
    a = np.ascontiguousarray(src, dtype=np.float32)
    k, n = a.shape if src_is_k_by_n else a.shape[::-1]
    nbytes = int(lib().bild_debug_tiled_bytes(n, k, dtype))
    if nbytes < 0:
        raise BildError(nbytes, "bild_debug_tiled_bytes")
    out = np.zeros(nbytes, dtype=np.uint8)
    _check(lib().bild_debug_tile_matrix(a.ctypes.data, int(src_is_k_by_n), n, k, dtype, out.ctypes.data), "bild_debug_tile_matrix")
    return out


def gemm_shape(n: int, k: int, rows: int, gated: bool = False, lm_head: bool = False, dtype: int = 1) -> dict:
    out = (C.c_int32 * 8)()
    _check(lib().bild_debug_gemm_shape(n, k, rows, int(gated), int(lm_head), dtype, out), "bild_debug_gemm_shape")
    keys = ("wk", "nwv", "rw", "kc", "blocks", "row_blocks", "lds", "lds_limit")
    return dict(zip(keys, [int(v) for v in out]))


def head_route(d_model: int, vocab: int, rows: int, dtype: int) -> str:
    r = lib().bild_debug_head_route(d_model, vocab, rows, dtype)
    if r < 0:
        raise BildError(r, "bild_debug_head_route")
    return ("short", "sweep", "planes")[r]


def tile_shape(n: int, k: int, rows: int, gated: bool = False, rotary: bool = False) -> dict:
    out = (C.c_int32 * 5)()
    _check(lib().bild_debug_tile_shape(n, k, rows, int(gated), int(rotary), out), "bild_debug_tile_shape")
    return dict(zip(("rows", "features", "slices", "shared", "busiest"), [int(v) for v in out]))


def attn_shape(heads: int, d_head: int, rows: int, nkeys: int, max_splits: int = 8, dtype: int = 1) -> dict:
    out = (C.c_int32 * 4)()
    _check(lib().bild_debug_attn_shape(heads, d_head, rows, nkeys, max_splits, dtype, out), "bild_debug_attn_shape")
    return dict(zip(("splits", "defer", "waves", "lds"), [int(v) for v in out]))


def cache_rule(heads: int, d_head: int, positions: int, nkeys: int) -> dict:
    out = (C.c_int32 * 3)()
    _check(lib().bild_debug_cache_rule(heads, d_head, positions, nkeys, out), "bild_debug_cache_rule")
    return dict(zip(("one_kernel", "splits", "waves"), [int(v) for v in out]))


def wide_split(d_model: int, heads: int, d_ff: int, gated: bool, units: int, keys: int, rows: int = 1) -> dict:
    out = (C.c_int32 * 7)()
    _check(lib().bild_debug_wide_split_rows(d_model, heads, d_ff, int(gated), units, keys, rows, out), "bild_debug_wide_split_rows")
    return dict(zip(("qkv_tiles", "qkv_first", "ffn_tiles", "ffn_first", "heads_first", "ranges", "apart"), [int(v) for v in out]))
