// What the kernels of bild_cache_attend share: cache_attend.hip (a few rows a sequence), cache_prompt.hip (prompts).
#pragma once
#include "cache.h"
#include "rows_common.h"

namespace bild {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 32;     // keys of a step of the matrix cores' second product: a page has whole ones
constexpr float kLn2 = 0.6931471805599453f;
// Weights are powers of two relative to a maximum that is moved only when a score is beyond it by this much: they stay below 2^8, far from fp16's end.
constexpr float kSlack = 8.f;

struct AttendArgs {
    CacheView c;
    CacheRows r;
    const void* q;
    void* out;
    float* lse;
    int64_t q_token, q_head, out_token, out_head;
    int layer, heads, group;
    int window, sinks, causal;  // (no window is wider than a sequence can be long: up to 2^30)
    float scale;    // of scores, in powers of two, with what codes and scales are short of: log2 e * 2^9 / 127
    int prompt_from;      // rows of a sequence, times `group`, from which on it is the kernel for prompts'
    int groups, least;  // workgroups of a key head; what one takes at least
    int splits;         // of a prompt tile's keys; most
    float* part;
    unsigned* arrived;
};

// Codes as fp16, times 2^-9: a byte permutation puts two codes ^ 0x80 where they are the bits of subnormals, (c + 128) 2^-24, and a packed product and sum, times 2^15 less 2^-2, makes them
// c 2^-9: exact, an instruction a code.
__device__ __forceinline__ f16x2 two(uint32_t x) {
    const f16x2 by = {(_Float16)32768.f, (_Float16)32768.f}, off = {(_Float16)-0.25f, (_Float16)-0.25f};
    return __builtin_elementwise_fma(__builtin_bit_cast(f16x2, x), by, off);
}
struct Halves {
    f16x2 v[4];
};
__device__ __forceinline__ f16x8 eight(f16x2 a, f16x2 b, f16x2 c, f16x2 d) { return __builtin_bit_cast(f16x8, Halves{{a, b, c, d}}); }
// eight codes (already ^ 0x80) side by side
__device__ __forceinline__ f16x8 eight_of(uint32_t a, uint32_t b) {
    return eight(two(__builtin_amdgcn_perm(0u, a, 0x0c010c00u)), two(__builtin_amdgcn_perm(0u, a, 0x0c030c02u)), two(__builtin_amdgcn_perm(0u, b, 0x0c010c00u)),
                 two(__builtin_amdgcn_perm(0u, b, 0x0c030c02u)));
}
// byte k of two words
__device__ __forceinline__ f16x2 pair_of(uint32_t a, uint32_t b, int k) { return two(__builtin_amdgcn_perm(b, a, 0x0c000c00u | (unsigned)(4 + k) << 16 | (unsigned)k)); }

// Rows of q as fp16 times a power of two that puts the largest magnitude below 2^15 (0, infinities and NaN: 1).
__device__ __forceinline__ int up_of(float big) {
    int up = 0;
    if (big > 0.f && big < INFINITY) {
        frexpf(big, &up);
        up = 15 - up;
    }
    return up;
}

constexpr int kTile = 16;      // rows of a tile of the kernels for few rows
// Blocks that could be read while a workgroup gets to a tile and joins what its waves have of it (us, call, of 16 / 32 / 48: 64 sequences of up to 16384 positions 63.2 / 65.5 / 69.6, 64 of 500
// 28.3 / 28.3 / 32.2, one of 513 12.9 / 14.5 / 14.2).
constexpr int kStart = 16;

// Inclusive prefix sums of a wave: within rows of 16 lanes, then the rows before.
__device__ __forceinline__ int prefix_sum(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);   // row_shr 1
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row_bcast15 into rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // row_bcast31 into rows 2 and 3
    return v;
}

// A sequence's share of the work.
struct Seq {
    int s, first, count, length;  // which, its rows, its positions
    int tiles, sink_blocks, low_block, blocks;
    // of its row j.  (Rows from before its beginning see nothing: all of them are at -1, so that a window can be taken off in 32 bits.)
    __device__ int position(int j, int causal) const { return causal ? max(length - count + j, -1) : length - 1; }
    // what a tile counts for in the line
    __device__ int cost() const { return blocks + kStart; }
};
__device__ __forceinline__ Seq sequence_at(const AttendArgs& a, int i) {
    Seq q;
    q.s = a.r.sequence(i, a.c.sequences);
    a.r.span(i, q.first, q.count);
    if (q.s < 0) q.count = 0;
    q.length = q.s < 0 ? 0 : min(max(a.c.lengths[q.s], 0), a.c.cap());
    const int64_t rows = (int64_t)q.count * a.group;
    q.tiles = rows < a.prompt_from ? (int)((rows + kTile - 1) / kTile) : 0;
    q.low_block = a.window ? max(max(q.length - q.count, 0) - a.window + 1, 0) / kBlock : 0;
    q.sink_blocks = a.window ? min((int)(((int64_t)a.sinks + kBlock - 1) / kBlock), q.low_block) : 0;
    q.blocks = max(q.sink_blocks + (q.length + kBlock - 1) / kBlock - q.low_block, 1);  // (one that has none is written all the same)
    return q;
}

// Floats of a row of partial results: the sums over the values, maximum, sum of weights.
constexpr int part_row(int DP) { return DP + 4; }

__device__ __forceinline__ f32x4 mma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

hipError_t launch_cache_attend_tall(const AttendArgs& a, int dtype, hipStream_t st);  // heads above 128
hipError_t cache_attend_tall_init();
hipError_t launch_cache_prompt(const AttendArgs& a, int dtype, int64_t places, hipStream_t st);
hipError_t cache_prompt_init(int d_head);
size_t prompt_part_floats(int d_head);
constexpr int kPromptRows = 128;  // of a tile of the kernel for prompts
constexpr int kMaxSplits = 16;    // pieces of a tile's keys

}  // namespace bild
