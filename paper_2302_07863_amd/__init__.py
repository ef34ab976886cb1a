"""MI355X-native Big Little Decoder: HIP library (csrc/, built into libbild.so)
and its ctypes binding."""
from . import binding
from .binding import (ACCEPT_REJECTION, ACCEPT_THRESHOLD, BOTH, DT_BF16, DT_F16, DT_F32, LARGE, ROTARY_BANDS, ROTARY_BASE, ROTARY_LINEAR,
                      ROTARY_NONE, ROTARY_YARN, SMALL, Beams, BildError, Cache, CacheConfig, Model, ModelConfig, Pair, Quant, Rotary, RotaryConfig, RotaryRows, Rules, State,
                      Stats, config_from_shape, lib, quant_round)
