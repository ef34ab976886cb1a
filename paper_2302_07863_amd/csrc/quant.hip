// Products of rows with a matrix in 4 bits (bild_quant_matmul).
//
//   y[r][n] = scale * sum_g s[n][g] * sum_{k in g} (q[n][k] - z[n][g]) x[r][k]
//
// Bound: HBM, half a byte a weight; at a few rows the matrix cores idle.  So the codes go to the matrix cores in as few
// instructions as there are: a code becomes the number 1 + q / 16 (of bf16, or of fp16 for fp16 rows) by putting its four bits on top of a mantissa, one shift
// and one and-or for two weights, and a second product with the constant -(1 + z / 16), the same for all inputs of a group, takes 1 + z / 16
// off again.  Both products are exact and go into the same fp32 accumulator step by step, so what cancels is never
// larger than 32 inputs' sum; scales are applied to the accumulators once a group.  No weight is ever rounded.
//
// Layout: tiles of 16 features x 128 inputs, 1 KiB, in the order of the matrix cores' operand: lane l has feature l % 16, its word j
// the inputs 32 j + 8 (l / 16) + 0 .. 7.  Of these, pair p (2p, 2p + 1) lies 4 p bits above the places where bf16 takes it (bits 3 .. 6 and 19 .. 22), the
// last pair round the end of the word.  Beside it, feature by feature, what one lane needs of a tile besides its codes: the scales as fp16 (which goes into the
// products as it is) times a power of two of the whole matrix and the zeros, four bits a group; a word with groups of 128, two, three with groups of
// 64, 32: one load.  (Apart, as two or more, a wave's four feature tiles of 4096 inputs took 18 instead of 13 us to come in, small as they are.)
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <new>
#include <thread>
#include <type_traits>
#include <vector>

#include "operators.h"
#include "rows_common.h"

using namespace bild;

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kTileK = 128;    // inputs of a tile
constexpr int kMaxWaves = 16;  // of a workgroup (with 8 above two row tiles: 22 rows of fp32 by 250112 x 1024 138 us, with 16 108)
constexpr int kPartRows = 32;  // most rows of a workgroup
// Tiles that a wave has under way (with a group per step of 32 inputs the scales take two thirds of a tile's registers).
constexpr int ahead(int group) { return group == 32 ? 3 : 4; }
constexpr int kDirectWaves = 8, kDirectAhead = 3;  // (with four, six, eight tiles ahead 4096 x 4096 takes 5.7, 6.2, 6.2 us instead of 5.35)
constexpr int kChipUnits = 256;  // compute units
constexpr int kLdsLimit = 160 * 1024;

// Rows as the matrix cores take them.  bf16 and fp16 rows as they are; fp32 rows, and rows with a norm's gain, as three bf16 parts each, whose
// sum is the value to 24 bits.  A part is a row of its own to the matrix cores: up to five such rows cost no more instructions than one.
enum RowsAs : int { AS_BF16 = 0, AS_F16 = 1, AS_PARTS = 2 };

struct QuantArgs {
    const uint4* codes;
    const uint32_t* sides;
    const void* x;
    void* y;
    const float* gain;
    int64_t ldx, ldy;
    int n, k, tn, tk, rows;
    int x_dtype, y_dtype;
    float eps, scale;  // (the scale with what codes and scales are short of: 16 and the scales' power of two)
    int rows_per;  // rows of a workgroup
    int wk, lwk;   // waves that share a feature tile's inputs (a power of two)
    int per;       // feature tiles of a wave, one after the other (1 where there are several chunks)
    int chunk;     // input tiles staged at a time
    int chunks;
    unsigned span_m;  // 2^32 / (waves that a row of a chunk's pieces takes), rounded up; 0: one
    int turns;     // of a wave over them (several chunks: a multiple of ahead())
    const uint4* nothing;  // 16 bytes of zeros
    int sums_at;   // where in LDS the sums lie: behind the rows, or (per 1) in their place
};

// Products of 16 features and 16 rows: a lane gets four rows of one feature, so that it scales them by one number.
template <int AS>
__device__ __forceinline__ f32x4 mac(const uint4& codes, const uint4& x, const f32x4& c) {
    if constexpr (AS == AS_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, codes), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, codes), c, 0, 0, 0);
}
// A wave's products to LDS, [row][feature].
__device__ __forceinline__ void put_sums(f32x4* to, int lane, const f32x4& v) {
    float* p = (float*)to + (lane >> 4) * 64 + (lane & 15);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[16 * i] = v[i];
}

// What turns codes into numbers, in registers: an and-or has room for one constant that is none.
struct CodeBits {
    uint32_t mask, one;
};
template <int AS>
__device__ __forceinline__ CodeBits code_bits() {
    CodeBits b = AS == AS_F16 ? CodeBits{0x03C003C0u, 0x3C003C00u} : CodeBits{0x00780078u, 0x3F803F80u};
    asm("" : "+s"(b.mask));
    asm("" : "+v"(b.one));
    return b;
}
// Eight codes as 1 + q / 16.
template <int AS>
__device__ __forceinline__ uint4 codes_up(uint32_t w, const CodeBits& b) {
    if constexpr (AS == AS_F16)
        return make_uint4(((w << 3) & b.mask) | b.one, ((w >> 1) & b.mask) | b.one, ((w >> 5) & b.mask) | b.one,
                          (__builtin_amdgcn_alignbit(w, w, 9) & b.mask) | b.one);
    else
        return make_uint4((w & b.mask) | b.one, ((w >> 4) & b.mask) | b.one, ((w >> 8) & b.mask) | b.one,
                          (__builtin_amdgcn_alignbit(w, w, 12) & b.mask) | b.one);
}
// -(1 + z / 16), twice
template <int AS>
__device__ __forceinline__ uint32_t zero_up(uint32_t z) {
    return AS == AS_F16 ? 0xBC00BC00u + z * 0x00400040u : 0xBF80BF80u + z * 0x00080008u;
}

// Two values' three bf16 parts.
__device__ __forceinline__ void split3(float a, float b, uint32_t (&p)[3]) {
#pragma unroll
    for (int j = 0; j < 3; ++j) {
        p[j] = pack_bf16x2(a, b);
        a -= __uint_as_float(p[j] << 16);
        b -= __uint_as_float(p[j] & 0xFFFF0000u);
    }
}

__device__ __forceinline__ void store_y(const QuantArgs& a, int row, int n0, const f32x4& v) {
    const int left = a.n - n0;
    if (left <= 0) return;
    const float w[4] = {v[0], v[1], v[2], v[3]};
    const auto put = [&](auto tag) {
        typedef decltype(tag) R;
        RowVec<R, 4> o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o.v[i] = R::down(w[i]);
        typename R::type* p = (typename R::type*)a.y + (int64_t)row * a.ldy + n0;
        if (left >= 4) o.store(p); else o.store_some(p, left);
    };
    if (a.y_dtype == BILD_DT_F32) put(RowF32());
    else if (a.y_dtype == BILD_DT_BF16) put(RowBf16());
    else put(RowF16());
}

// Eight inputs of row r, as they are or times the gain in three parts, to their place in the operand; their squares (with a gain).
template <class R, bool PARTS, bool GAIN>
__device__ __forceinline__ float put_piece(const RowVec<R, 8>& x, const float (&g)[8], char* to, int rows, bool real) {
    if constexpr (!PARTS) {
        uint4 q;
        __builtin_memcpy(&q, x.v, 16);
        if (real) *(uint4*)to = q;
        return 0.f;
    } else {
        float ss = 0.f;
        uint32_t q[4][3];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float a = R::up(x.v[2 * j]), b = R::up(x.v[2 * j + 1]);
            if constexpr (GAIN) {
                ss = __builtin_fmaf(a, a, __builtin_fmaf(b, b, ss));
                a *= g[2 * j];
                b *= g[2 * j + 1];
            }
            split3(a, b, q[j]);
        }
        if (real) {
#pragma unroll
            for (int p = 0; p < 3; ++p) *(uint4*)(to + (size_t)p * rows * 64) = make_uint4(q[0][p], q[1][p], q[2][p], q[3][p]);
        }
        return ss;
    }
}

// The workgroup's rows, inputs of the tiles t0 .. t1 - 1, to LDS in the order of the matrix cores' operand:
// [step of 32 inputs][row of the operand][4 pieces of 8].  Row v of the operand is part v / rows of row v % rows.  Inputs from the k-th on are zero.
// A wave's 64 pieces belong to one row; with a norm it adds up their squares.  `between` runs behind the requests of the first U pieces a thread
// (loads come back in order: what it requests does not keep these waiting).
template <class R, bool PARTS, bool GAIN, int U, class Between>
__device__ __forceinline__ void stage_rows(const QuantArgs& a, char* xs, float (*squares)[kPartRows], int r0, int rows, int t0, int t1, Between&& between) {
    const int nthr = blockDim.x, tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int k0 = t0 * kTileK, pieces = (t1 - t0) * (kTileK / 8), span = (a.chunk * (kTileK / 8) + 63) & ~63;  // (a row has whole waves)
    const int full = min(max((a.k - k0) / 8, 0), pieces);  // pieces that are there as a whole
    const bool tail = (a.k & 7) != 0 && full < pieces;     // one more is there in part
    const int v = PARTS ? 3 * rows : rows;                 // rows of the operand
    // (exact below 2^16 waves; what LDS holds is far less)
    const auto row_of = [&](int i) { return a.span_m ? (int)__umulhi((unsigned)__builtin_amdgcn_readfirstlane(i >> 6), a.span_m) : __builtin_amdgcn_readfirstlane(i >> 6); };
    const auto place = [&](int p, int r) { return xs + ((size_t)((p >> 2) * v + r) * 4 + (p & 3)) * 16; };
    RowVec<R, 8> x[U];
    float g[U][8];
    const auto load = [&](int i0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * nthr + tid, r = min(row_of(i), rows - 1), p = i - r * span;
            __builtin_memset(x[u].v, 0, sizeof(x[u].v));
            if constexpr (GAIN) __builtin_memset(g[u], 0, sizeof(g[u]));  // (times x: zero, also where no piece is there as a whole)
            if (full > 0) {  // (past the end: a valid address, replaced below)
                const int k = k0 + min(p, full - 1) * 8;
                x[u].load((const typename R::type*)a.x + (int64_t)(r0 + r) * a.ldx + k);
                if constexpr (GAIN) {
                    RowVec<RowF32, 8> t;
                    t.load(a.gain + k);
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[u][j] = t.v[j];
                }
            }
        }
    };
    const auto put = [&](int i0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * nthr + tid, r = row_of(i), p = i - r * span;
            if (r >= rows) break;
            if ((GAIN || full < pieces) && p >= full) __builtin_memset(x[u].v, 0, sizeof(x[u].v));
            const float ss = put_piece<R, PARTS, GAIN>(x[u], g[u], place(p, r), rows, p < pieces && !(tail && p == full));
            if constexpr (GAIN) {
                const float all = wave_sum(ss);
                if ((tid & 63) == 0) squares[wave][r] += all;
            }
        }
    };
    load(0);
    __builtin_amdgcn_sched_barrier(0);
    between();
    __builtin_amdgcn_sched_barrier(0);
    put(0);
    for (int i0 = U * nthr; i0 < rows * span; i0 += U * nthr) {
        load(i0);
        put(i0);
    }
    // the piece that the last input lies in (nobody else writes it)
    if (!tail || tid >= rows) return;
    RowVec<R, 8> y;
    RowVec<RowF32, 8> h;
    const int n = a.k & 7, k = a.k - n;
    y.load_some((const typename R::type*)a.x + (int64_t)(r0 + tid) * a.ldx + k, n);
    if constexpr (GAIN) h.load_some(a.gain + k, n);
    const float ss = put_piece<R, PARTS, GAIN>(y, h.v, place(full, tid), rows, true);
    if constexpr (GAIN) squares[0][tid] += ss;
}

// What a lane has of its feature besides codes, of the tile's GT groups.
constexpr int side_words(int gt) { return gt == 4 ? 3 : gt; }
template <int GT>
struct Side {
    uint32_t w[side_words(GT)];
    __device__ __forceinline__ void load(const uint32_t* sides, size_t tile, int feature) {
        __builtin_memcpy(w, sides + (tile * 16 + feature) * side_words(GT), sizeof(w));
    }
    __device__ __forceinline__ float scale(int g) const {
        return (float)__builtin_bit_cast(_Float16, (uint16_t)(GT == 1 ? w[0] : w[g >> 1] >> (16 * (g & 1))));
    }
    __device__ __forceinline__ uint32_t zero(int g) const { return GT == 1 ? w[0] >> 16 : w[side_words(GT) - 1] >> (4 * g) & 15u; }
};

// What a wave has requested of one tile.
template <int GT>
struct Unit {
    uint4 codes;
    Side<GT> side;
};

// A workgroup has up to rows_per rows (NT tiles of 16 rows of the operand) and stages them once, or (CHUNKED) chunk by chunk of the inputs where they do
// not fit.  wk of its waves share a feature tile, each takes every wk-th of the input tiles; a wave goes through `per` feature tiles (CHUNKED: one).  It streams their
// tiles of codes one behind the other, ahead() of them under way.  Nothing is stored before the last one: stores would be counted among the loads that the waves
// wait for.  The sums meet in LDS.
template <int AS, int G, int NT, bool CHUNKED>
__global__ __launch_bounds__(64 * kMaxWaves) void quant_kernel(const QuantArgs a) {
    constexpr int GT = kTileK / G;  // groups of a tile
    constexpr int SG = G / 32;      // steps of a group
    constexpr int kAhead = ahead(G);
    constexpr int PARTS = AS == AS_PARTS ? 3 : 1;
    constexpr int CH = NT == 1 && SG > 1 ? 2 : 1;  // chains of products: of one row tile the odd steps have their own
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float squares[kMaxWaves][kPartRows];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
    const int wk = a.wk, wkid = wave & (wk - 1), wfid = wave >> a.lwk, wf = nw >> a.lwk;
    const int r0 = blockIdx.y * a.rows_per, rows = min(a.rows_per, a.rows - r0), v = PARTS * rows;
    const int f0 = (int)blockIdx.x * wf * a.per + wfid;  // the wave's feature tiles: every wf-th from here (some of the last workgroup's are not there: they load the last one's)
    const int turns = a.turns, segments = CHUNKED ? a.chunks : a.per;
    f32x4* sums = (f32x4*)(lds + a.sums_at);  // [feature tile of a wave][wave][row tile][row][four features]

    // the tile of a segment's turn (past the end: the last one there is)
    int ps = 0, pj = 0;
    const auto request = [&](Unit<GT>& u) {
        const int f = min(f0 + (CHUNKED ? 0 : ps) * wf, a.tn - 1), kt = min((CHUNKED ? ps * a.chunk : 0) + wkid + pj * wk, a.tk - 1);
        const size_t tile = (size_t)f * a.tk + kt;
        u.codes = a.codes[tile * 64 + lane];
        u.side.load(a.sides, tile, lane & 15);
        if (++pj == turns) {
            pj = 0;
            ps = min(ps + 1, segments - 1);
        }
    };
    Unit<GT> ring[kAhead];
    const auto first = [&] {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (CHUNKED || i < segments * turns) request(ring[i]);
    };
    const auto stage = [&](int t0, auto&& between) {
        const int t1 = min(t0 + a.chunk, a.tk);
        if constexpr (AS == AS_PARTS) {
            if (a.x_dtype == BILD_DT_F32 && a.gain) stage_rows<RowF32, true, true, 1>(a, lds, squares, r0, rows, t0, t1, between);
            else if (a.x_dtype == BILD_DT_F32) stage_rows<RowF32, true, false, 2>(a, lds, squares, r0, rows, t0, t1, between);
            else if (a.x_dtype == BILD_DT_BF16) stage_rows<RowBf16, true, true, 1>(a, lds, squares, r0, rows, t0, t1, between);  // (without a gain they are as they are)
            else stage_rows<RowF16, true, true, 1>(a, lds, squares, r0, rows, t0, t1, between);
        } else {  // (16 bits are 16 bits)
            if (rows * ((a.chunk * (kTileK / 8) + 63) & ~63) <= (int)blockDim.x) stage_rows<RowBf16, false, false, 1>(a, lds, squares, r0, rows, t0, t1, between);
            else stage_rows<RowBf16, false, false, 4>(a, lds, squares, r0, rows, t0, t1, between);
        }
    };
    const CodeBits bits = code_bits<AS>();
    f32x4 total[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) total[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    int col[NT];  // the lane's row of the operand (past the last: that one again, its results are nobody's)
#pragma unroll
    for (int t = 0; t < NT; ++t) col[t] = min(t * 16 + (lane & 15), v - 1) * 64 + (lane >> 4) * 16;

    const auto process = [&](const Unit<GT>& u, int at) {  // tile `at` of those staged
        const uint32_t cw[4] = {u.codes.x, u.codes.y, u.codes.z, u.codes.w};
        int xs = at * 4 * v * 64;
        asm volatile("" : "+v"(xs));  // (else the compiler keeps an address for every operand of the tiles ahead in a register)
#pragma unroll
        for (int g = 0; g < GT; ++g) {
            const uint32_t zw = zero_up<AS>(u.side.zero(g));
            const uint4 za = make_uint4(zw, zw, zw, zw);
            f32x4 acc[NT][CH];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int c = 0; c < CH; ++c) acc[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < SG; ++s) {
                const int j = g * SG + s;
                const uint4 ca = codes_up<AS>(cw[j], bits);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const uint4 b = *(const uint4*)(lds + col[t] + (xs + j * v * 64));
                    acc[t][s % CH] = mac<AS>(ca, b, acc[t][s % CH]);
                    acc[t][s % CH] = mac<AS>(za, b, acc[t][s % CH]);
                }
            }
            const float scale = u.side.scale(g);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) total[t][i] = __builtin_fmaf(scale, acc[t][c][i], total[t][i]);
                asm volatile("" : "+v"(total[t]));  // (now: four registers less than a group that waits)
            }
        }
    };
    const auto keep = [&](int s) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            put_sums(sums + ((s * nw + wave) * NT + t) * 64, lane, total[t]);
            total[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };

    if (AS == AS_PARTS && lane < kPartRows) squares[wave][lane] = 0.f;
    stage(0, first);
    lds_barrier();
    if constexpr (CHUNKED) {  // (turns: a multiple of kAhead, what is too much is skipped)
        for (int s = 0; s < segments; ++s) {
            const int t0 = s * a.chunk, n = min(a.chunk, a.tk - t0);
            if (s) {
                lds_barrier();
                stage(t0, [] {});
                lds_barrier();
            }
            for (int j = 0; j < turns; j += kAhead) {
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const int at = wkid + (j + i) * wk;
                    if (at < n) process(ring[i], at);
                    request(ring[i]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        lds_barrier();  // (the sums take the rows' place)
        keep(0);
    } else {
        const int all = segments * turns;
        int s = 0, j = 0;
        const auto turn = [&](const Unit<GT>& u) {
            const int at = wkid + j * wk;
            if (at < a.tk) process(u, at);
            if (++j < turns) return;
            if (a.per > 1) keep(s);
            j = 0;
            s += 1;
        };
        int q = 0;
        for (; all - q > kAhead; q += kAhead) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                turn(ring[i]);
                request(ring[i]);  // (past the end: the last one again)
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (q + i < all) turn(ring[i]);
        if (a.per == 1) {
            lds_barrier();
            keep(0);
        }
    }
    lds_barrier();
    // What the waves have of a row's four features, over its parts, to y.
    const int items = a.per * wf * rows * 4;
    for (int it = threadIdx.x; it < items; it += blockDim.x) {
        const int q = it & 3, fr = it >> 2, fl = fr / rows, r = fr - fl * rows;  // feature tile fl of the workgroup's
        const int p = fl / wf, w0 = (fl - p * wf) << a.lwk;
        f32x4 sum = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int part = PARTS - 1; part >= 0; --part) {
            const int c = part * rows + r;
            const f32x4* from = sums + ((p * nw + w0) * NT + (c >> 4)) * 64 + (c & 15) * 4 + q;
#pragma unroll 4
            for (int w = 0; w < wk; ++w) sum += from[w * NT * 64];
        }
        float s = a.scale;
        if (AS == AS_PARTS && a.gain) {
            float ss = 0.f;
#pragma unroll 8
            for (int w = 0; w < nw; ++w) ss += squares[w][r];
            s *= 1.f / sqrtf(ss / (float)a.k + a.eps);
        }
        store_y(a, r0 + r, ((int)blockIdx.x * wf * a.per + fl) * 16 + q * 4, sum * s);
    }
}

// Up to 16 rows of 16 bits without a gain, one feature tile a workgroup: its wk waves take the rows as they lie in memory, beside the codes of the same inputs.
// Nothing is staged, so nobody waits for anybody before the sums meet.
template <int G>
struct DirectUnit {
    Unit<kTileK / G> w;
    uint4 x[4];
};
template <int AS, int G>
__global__ __launch_bounds__(64 * kDirectWaves) void quant_direct_kernel(const QuantArgs a) {
    constexpr int GT = kTileK / G, SG = G / 32, CH = SG > 1 ? 2 : 1;
    constexpr int D = kDirectAhead;
    __shared__ f32x4 sums[kDirectWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), f = blockIdx.x;
    const int pieces = a.k / 8;  // (k is a multiple of 8)
    const uint16_t* xrow = (const uint16_t*)a.x + (int64_t)min(lane & 15, a.rows - 1) * a.ldx;
    int kt = wave;
    const auto request = [&](DirectUnit<G>& u) {  // (past the last tile: that one again)
        const int t = min(kt, a.tk - 1);
        const size_t tile = (size_t)f * a.tk + t;
        u.w.codes = a.codes[tile * 64 + lane];
        u.w.side.load(a.sides, tile, lane & 15);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            RowVec<RowBf16, 8> v;  // (16 bits are 16 bits)
            v.load(xrow + (size_t)min(t * 16 + j * 4 + (lane >> 4), pieces - 1) * 8);
            __builtin_memcpy(&u.x[j], v.v, 16);
        }
        kt += a.wk;
    };
    const CodeBits bits = code_bits<AS>();
    f32x4 total = f32x4{0.f, 0.f, 0.f, 0.f};
    const auto process = [&](DirectUnit<G>& u, int t) {
        const uint32_t cw[4] = {u.w.codes.x, u.w.codes.y, u.w.codes.z, u.w.codes.w};
        if (t * 16 + 16 > pieces) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (t * 16 + j * 4 + (lane >> 4) >= pieces) u.x[j] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int g = 0; g < GT; ++g) {
            const uint32_t zw = zero_up<AS>(u.w.side.zero(g));
            const uint4 za = make_uint4(zw, zw, zw, zw);
            f32x4 acc[CH];
#pragma unroll
            for (int c = 0; c < CH; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < SG; ++s) {
                const int j = g * SG + s;
                const uint4 ca = codes_up<AS>(cw[j], bits);
                acc[s % CH] = mac<AS>(ca, u.x[j], acc[s % CH]);
                acc[s % CH] = mac<AS>(za, u.x[j], acc[s % CH]);
            }
            const float scale = u.w.side.scale(g);
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) total[i] = __builtin_fmaf(scale, acc[c][i], total[i]);
            asm volatile("" : "+v"(total));
        }
    };
    DirectUnit<G> ring[D];
#pragma unroll
    for (int i = 0; i < D; ++i) request(ring[i]);
    int t = wave, left = a.turns;
    for (; left > D; left -= D) {
#pragma unroll
        for (int i = 0; i < D; ++i) {
            if (t < a.tk) process(ring[i], t);
            t += a.wk;
            request(ring[i]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
#pragma unroll
    for (int i = 0; i < D; ++i) {
        if (i < left && t < a.tk) process(ring[i], t);
        t += a.wk;
    }
    put_sums(sums[wave], lane, total);
    lds_barrier();
    const int q = threadIdx.x & 3, r = threadIdx.x >> 2;  // (16 rows of four: a wave)
    if (r >= a.rows) return;
    f32x4 sum = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int w = 0; w < a.wk; ++w) sum += sums[w][r * 4 + q];
    store_y(a, r, f * 16 + q * 4, sum * a.scale);
}

// ---- blocks of rows
// 64 rows of 16 bits by 128 features a workgroup.  Eight waves: two have the block's halves of the features, 64 x 64 products each, of every fourth input tile, so
// that an operand read from LDS serves four feature tiles and a code taken apart four row tiles.  The rows of four half tiles of inputs at a time go from
// memory to LDS without passing through registers, three halves ahead of their use; codes come two tiles ahead into registers.
// Bound: both what a compute unit multiplies, takes apart and scales and what it can have under way at once: 509 rows of fp16 by 4096 x 4096, groups of 128,
// take 27 us (630 TFLOP/s), 20 to 22 without the loads, 18 the loads alone; a tile ahead instead of three halves and two tiles 29.  The matrix cores alone would need
// 7.  bf16 34 us: it has no subtraction of pairs, so that every product with codes has a second with the zeros.
constexpr int kBlockRows = 64, kBlockFeatures = 128, kBlockSplit = 4;

// fp16 only: 1 + q / 16 less 1 + z / 16, which is (q - z) / 16 exactly (the 16 is in QuantArgs::scale, as for the other forms).  (bf16 has no subtraction of pairs: a second
// product does it, as above.)
template <int AS>
__device__ __forceinline__ uint4 codes_less(uint32_t w, const CodeBits& b, uint32_t z) {
    const uint4 q = codes_up<AS>(w, b);
    if constexpr (AS != AS_F16) return q;
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    const f16x2 less = __builtin_bit_cast(f16x2, z);
    const auto one = [&](uint32_t v) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, v) + less); };
    return make_uint4(one(q.x), one(q.y), one(q.z), one(q.w));
}

// Four feature tiles' codes; what lies beside those of the f-th is in the lanes 16 f .. 16 f + 15.
template <int GT>
struct Four {
    uint4 codes[4];
    Side<GT> side;
};

template <int AS, int G>
__global__ __launch_bounds__(512) void quant_block_kernel(const QuantArgs a) {
    constexpr int GT = kTileK / G, SG = G / 32;
    constexpr int SUM = AS == AS_F16 || SG < 2 ? SG : 2;  // steps between scalings (bf16 has no registers for sums that outlast half a tile)
    constexpr int kStage = kBlockSplit * kBlockRows * 8;  // pieces of 16 bytes: [input tile][row][half a tile's 8]
    __shared__ uint4 x0[kStage], x1[kStage], x2[kStage], x3[kStage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), ks = wave >> 1;
    const int per_die = a.per, fb = (int)(blockIdx.x & 7) * per_die + (int)(blockIdx.x >> 3) % per_die, rb = (int)(blockIdx.x >> 3) / per_die;
    if (fb * (kBlockFeatures / 16) >= a.tn) return;
    const int r0 = rb * kBlockRows, pieces = a.k / 8;
    const int f0 = fb * (kBlockFeatures / 16) + (wave & 1) * 4;

    // Piece p of row r lies at place p ^ (r / 2 & 7): the lanes of an operand have 16 rows and meet all banks.  A wave brings rows 8 w .. 8 w + 7 of every tile.
    const int own = wave * 8 + (lane >> 3), first = (lane & 7) ^ (own >> 1 & 7);
    const uint4* const row = (const uint4*)((const uint16_t*)a.x + (int64_t)min(r0 + own, a.rows - 1) * a.ldx);
    const auto bring = [&](uint4* to, int step, int t) {  // `step`: pieces before it
        const int p = step + t * 16 + first;
        const uint4* from = p < pieces ? row + p : a.nothing;
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)(to + (t * kBlockRows + wave * 8) * 8), 16, 0, 0);
    };
    const auto tile_of = [&](int f, int t0) { return (size_t)min(f0 + f, a.tn - 1) * a.tk + min(t0 + ks, a.tk - 1); };
    const auto request = [&](Four<GT>& u, int t0, int f) {
        u.codes[f] = a.codes[tile_of(f, t0) * 64 + lane];
        if (f == 3) u.side.load(a.sides, tile_of(lane >> 4, t0), lane & 15);
    };
    const CodeBits bits = code_bits<AS>();
    f32x4 total[4][4], acc[4][4];  // [feature tile][row tile]
#pragma unroll
    for (int f = 0; f < 4; ++f)
#pragma unroll
        for (int t = 0; t < 4; ++t) total[f][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    // Half a tile; `feed` runs in eight parts between the products.
    const auto process = [&](auto half, const Four<GT>& u, const Side<GT> (&side)[4], const uint4* x, auto&& feed) {
        constexpr int H = decltype(half)::value;
        const uint4* at = x + (ks * kBlockRows + (lane & 15)) * 8;
        uint4 b[2][4];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int t = 0; t < 4; ++t) b[s][t] = at[t * 128 + ((s * 4 + (lane >> 4)) ^ (lane >> 1 & 7))];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int j = 2 * H + s, g = j / SG;
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const uint32_t cw[4] = {u.codes[f].x, u.codes[f].y, u.codes[f].z, u.codes[f].w};
                const uint32_t zw = zero_up<AS>(side[f].zero(g));
                const uint4 za = make_uint4(zw, zw, zw, zw), ca = codes_less<AS>(cw[j], bits, zw);
                feed(s * 4 + f);
                __builtin_amdgcn_sched_barrier(0x8F);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    acc[f][t] = mac<AS>(ca, b[s][t], j % SUM == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[f][t]);
                    if constexpr (AS != AS_F16) acc[f][t] = mac<AS>(za, b[s][t], acc[f][t]);
                }
                if (j % SUM == SUM - 1) {
                    const float scale = side[f].scale(g);
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) total[f][t][i] = __builtin_fmaf(scale, acc[f][t][i], total[f][t][i]);
                        asm volatile("" : "+v"(total[f][t]));
                    }
                }
            }
        }
    };
    // The rows of half h are there: they were requested three halves ago, since when the wave has had thirteen loads more (four a half and, two tiles ahead, five of
    // codes in the lower one).  Behind the barrier those of all waves are, and nobody reads the half before any more.
    const auto arrive = [] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x007D);  // (vmcnt 13, lgkmcnt 0: what it has read itself)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // Past the end the rows are zeros; so is what lies beside the codes (of the last tile again, it may be infinite).
    Side<GT> side[4];
    const auto spread = [&](const Side<GT>& all, int t0) {
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
            for (int i = 0; i < side_words(GT); ++i)
                side[f].w[i] = t0 + ks < a.tk ? (uint32_t)__builtin_amdgcn_ds_bpermute((f * 16 + (lane & 15)) * 4, (int)all.w[i]) : 0u;
    };
    typedef std::integral_constant<int, 0> Low;
    typedef std::integral_constant<int, 1> High;
    // A tile: its rows in x_low and x_high; to `third` and (when it has been read) x_low come the rows three halves on, to `u2` the codes two tiles on.
    const auto turn = [&](int t0, const Four<GT>& u, Four<GT>& u2, uint4* x_low, const uint4* x_high, uint4* third) {
        arrive();
        spread(u.side, t0);
        process(Low(), u, side, x_low, [&](int part) {
            if (part < 4) bring(third, t0 * 16 + 72, part);
            else request(u2, t0 + 2 * kBlockSplit, part - 4);
        });
        arrive();
        process(High(), u, side, x_high, [&](int part) { if (part < 4) bring(x_low, t0 * 16 + 128, part); });
        return t0 + kBlockSplit < a.tk;
    };
    Four<GT> u0, u1, u2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bring(x0, 0, i);
        request(u0, 0, i);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bring(x1, 8, i);
        request(u1, kBlockSplit, i);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) bring(x2, 64, i);
    for (int t0 = 0;; t0 += 6 * kBlockSplit) {
        if (!turn(t0, u0, u2, x0, x1, x3)) break;
        if (!turn(t0 + kBlockSplit, u1, u0, x2, x3, x1)) break;
        if (!turn(t0 + 2 * kBlockSplit, u2, u1, x0, x1, x3)) break;
        if (!turn(t0 + 3 * kBlockSplit, u0, u2, x2, x3, x1)) break;
        if (!turn(t0 + 4 * kBlockSplit, u1, u0, x0, x1, x3)) break;
        if (!turn(t0 + 5 * kBlockSplit, u2, u1, x2, x3, x1)) break;
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70);  // (vmcnt 0: what is still under way goes where the sums come)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    // The four shares meet in LDS: [wave][feature tile][row][four features], a row tile at a time; a wave has a feature tile of the result.
    f32x4* sums = (f32x4*)x0;
    const int half = wave >> 2, tile = wave & 3;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        if (t) lds_barrier();
#pragma unroll
        for (int f = 0; f < 4; ++f) put_sums(sums + (wave * 4 + f) * 64, lane, total[f][t]);
        lds_barrier();
        f32x4 sum = sums[(half * 4 + tile) * 64 + lane];
#pragma unroll
        for (int k = 1; k < kBlockSplit; ++k) sum += sums[((2 * k + half) * 4 + tile) * 64 + lane];
        const int to = r0 + t * 16 + (lane >> 2);
        if (to < a.rows) store_y(a, to, (fb * (kBlockFeatures / 16) + half * 4 + tile) * 16 + (lane & 3) * 4, sum * a.scale);
    }
}

// What bf16 scales ask of the power of two that makes them fp16: the largest exponent, and the lowest bit that is set.
__global__ __launch_bounds__(256) void quant_range_kernel(const uint16_t* scales, size_t count, int* range) {
    int most = -1024, least = 1024;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (size_t)gridDim.x * 256) {
        const uint32_t h = scales[i] & 0x7FFFu, e = h >> 7, m = h & 0x7Fu;
        if (h == 0 || e == 255) continue;  // (zero, and what is not finite, go through any)
        const uint32_t bits = e ? 0x80u | m : m;
        const int unit = (int)(e ? e : 1) - 127 - 7;
        most = max(most, unit + 31 - __builtin_clz(bits));
        least = min(least, unit + __builtin_ctz(bits));
    }
    atomicMax(range, most);
    atomicMin(range + 1, least);
}

// From rows of codes (two a byte), scales and zeros to tiles.  A thread per lane and tile; `bad`: a zero above 15.
__global__ __launch_bounds__(256) void quant_layout_kernel(const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros, int n, int k, int group, int tk, size_t lanes,
                                                           int bf16_shift, int bf16, uint32_t* to_codes, uint32_t* to_sides, unsigned* bad) {
    const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= lanes) return;
    const int lane = (int)(at & 63);
    const size_t tile = at >> 6;
    const int ft = (int)(tile / tk), kt = (int)(tile - (size_t)ft * tk);
    const int f = ft * 16 + (lane & 15), bytes = (k + 1) / 2;
    for (int j = 0; j < 4; ++j) {
        const int k0 = kt * kTileK + 32 * j + 8 * (lane >> 4);
        uint32_t w = 0;
        for (int p = 0; p < 4; ++p) {
            const int kk = k0 + 2 * p;
            const uint32_t b = f < n && kk < k ? codes[(size_t)f * bytes + kk / 2] : 0u;
            const uint32_t pair = (b & 15u) << 3 | (b >> 4) << 19;  // where bf16 takes them
            w |= p == 0 ? pair : p == 3 ? pair << 12 | pair >> 20 : pair << (4 * p);
        }
        to_codes[at * 4 + j] = w;
    }
    const int gt = kTileK / group, groups = (k + group - 1) / group;
    if (lane >= 16) return;  // feature `lane` of the tile
    uint32_t side[4] = {0, 0, 0, 0};
    for (int g = 0; g < gt; ++g) {
        const int gg = kt * gt + g;
        const bool in = f < n && gg < groups;
        uint16_t s = in ? scales[(size_t)f * groups + gg] : (uint16_t)0;
        if (bf16) s = RowF16::down(ldexpf(bf2f(s), bf16_shift));  // (exact: the caller has seen to it)
        const unsigned z = in && zeros ? zeros[(size_t)f * groups + gg] : 8u;
        if (z > 15u) *bad = 1u;
        side[g >> 1] |= (uint32_t)s << (16 * (g & 1));
        if (gt == 1) side[0] |= (z & 15u) << 16;
        else side[side_words(gt) - 1] |= (z & 15u) << (4 * g);
    }
    for (int i = 0; i < side_words(gt); ++i) to_sides[(tile * 16 + lane) * side_words(gt) + i] = side[i];
}

template <void (*KERNEL)(QuantArgs)>
hipError_t launch_kernel(const QuantArgs& a, dim3 grid, int waves, size_t lds, int device, hipStream_t st) {
    if (lds > 64 * 1024) {  // (more than a workgroup gets without asking)
        static std::atomic<uint64_t> asked{0};  // by device
        const uint64_t bit = 1ull << (device & 63);
        if (device > 63 || !(asked.load(std::memory_order_relaxed) & bit)) {
            const hipError_t e = hipFuncSetAttribute((const void*)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, kLdsLimit - 4096);
            if (e != hipSuccess) return e;
            asked.fetch_or(bit, std::memory_order_relaxed);
        }
    }
    return launch_on(KERNEL, grid, dim3(64 * waves), lds, st, a);
}
template <int AS, int G>
hipError_t launch_rows(const QuantArgs& a, int tiles, dim3 grid, int waves, size_t lds, int device, hipStream_t st) {
#define BILD_Q(NT) \
    return a.chunks > 1 ? launch_kernel<quant_kernel<AS, G, NT, true>>(a, grid, waves, lds, device, st) : launch_kernel<quant_kernel<AS, G, NT, false>>(a, grid, waves, lds, device, st)
    if (tiles == 1) BILD_Q(1);
    if (tiles == 2) BILD_Q(2);
    if constexpr (AS == AS_PARTS) {
        if (tiles == 3) BILD_Q(3);
        BILD_Q(6);
    }
#undef BILD_Q
    return hipErrorInvalidValue;
}
template <int AS>
hipError_t launch_group(const QuantArgs& a, int group, int tiles, dim3 grid, int waves, size_t lds, int device, hipStream_t st) {
    if (group == 32) return launch_rows<AS, 32>(a, tiles, grid, waves, lds, device, st);
    if (group == 64) return launch_rows<AS, 64>(a, tiles, grid, waves, lds, device, st);
    return launch_rows<AS, 128>(a, tiles, grid, waves, lds, device, st);
}

template <int AS>
hipError_t launch_direct(const QuantArgs& a, int group, hipStream_t st) {
    const dim3 grid(a.tn), block(64 * a.wk);
    return launch_on(group == 32 ? quant_direct_kernel<AS, 32> : group == 64 ? quant_direct_kernel<AS, 64> : quant_direct_kernel<AS, 128>, grid, block, 0, st, a);
}

template <int AS>
hipError_t launch_block(const QuantArgs& a, int group, dim3 grid, hipStream_t st) {
    return launch_on(group == 32 ? quant_block_kernel<AS, 32> : group == 64 ? quant_block_kernel<AS, 64> : quant_block_kernel<AS, 128>, grid, dim3(512), 0, st, a);
}

bool shape_ok(int n, int k, int group) { return n >= 1 && k >= 1 && n <= (1 << 24) && k <= (1 << 20) && (group == 32 || group == 64 || group == 128); }

uint16_t to_scale(float v, int dtype) {
    if (dtype == BILD_DT_F16) return __builtin_bit_cast(uint16_t, (_Float16)v);
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    return (uint16_t)((u + (((u >> 16) & 1u) + 0x7FFFu)) >> 16);
}
float from_scale(uint16_t h, int dtype) { return dtype == BILD_DT_F16 ? (float)__builtin_bit_cast(_Float16, h) : __builtin_bit_cast(float, (uint32_t)h << 16); }

// One feature; false: a value that is not finite, or a scale beyond the type.
bool round_feature(const float* w, int64_t step, int k, int group, int dtype, uint8_t* codes, uint16_t* scales, uint8_t* zeros) {
    std::memset(codes, 0, (size_t)(k + 1) / 2);
    for (int g = 0; g * group < k; ++g) {
        const int k0 = g * group, k1 = std::min(k0 + group, k);
        float lo = 0.f, hi = 0.f;
        for (int i = k0; i < k1; ++i) {
            const float v = w[i * step];
            if (!std::isfinite(v)) return false;
            lo = std::min(lo, v);
            hi = std::max(hi, v);
        }
        const float want = zeros ? hi / 15.f - lo / 15.f : std::max(hi, -lo) / 7.f;
        scales[g] = to_scale(want, dtype);
        if (scales[g] == 0 && want > 0.f && dtype == BILD_DT_F16) scales[g] = 1;  // (a scale of none would lose the group; in bf16 only what fp32 itself has as subnormal numbers)
        const float s = from_scale(scales[g], dtype);
        if (!std::isfinite(s)) return false;
        const auto nearest = [&](float v) { return s > 0.f ? (int)std::max(-32.f, std::min(32.f, std::nearbyint(v / s))) : 0; };
        const int z = zeros ? std::max(0, std::min(15, -nearest(lo))) : 8;
        if (zeros) zeros[g] = (uint8_t)z;
        for (int i = k0; i < k1; ++i) codes[i / 2] |= (uint8_t)(std::max(0, std::min(15, nearest(w[i * step]) + z)) << (4 * (i & 1)));
    }
    return true;
}

}  // namespace

namespace bild {

int launch_quant(const bild_quant* w, const bild_quant_call& c, hipStream_t st) {
    QuantArgs a;
    a.codes = w->codes;
    a.sides = w->sides;
    a.x = c.x;
    a.y = c.y;
    a.gain = c.gain;
    a.ldx = c.x_stride;
    a.ldy = c.y_stride;
    a.n = w->n;
    a.k = w->k;
    a.tn = w->tn;
    a.tk = w->tk;
    a.rows = c.rows;
    a.x_dtype = c.x_dtype;
    a.y_dtype = c.y_dtype;
    a.eps = c.eps;
    a.scale = (float)(16.0 * c.scale * std::ldexp(1.0, w->scale_exponent));
    const bool parts = c.gain || c.x_dtype == BILD_DT_F32;
    // Where a compute unit has one feature tile at most, nobody takes the rows from LDS again.  us, staged / straight from memory, bf16, 1 and 11 rows: 1024 x 1024
    // 3.26 / 2.72, 4.00 / 3.02; 4096 x 4096 6.23 / 5.35, 7.97 / 6.34; 4096 x 11008 11.0 / 9.5, 16.4 / 12.9; but 11008 x 4096 (688 feature tiles) 9.7 / 10.2, 11.4 / 13.8,
    // 32000 x 4096 19.0 / 21.8, 19.6 / 28.3 (8 rows).  Four waves, from 64 input tiles on eight: 4096 x 4096 with eight 5.76, 7.46, 4096 x 11008 with four 10.1, 13.0.
    if (!parts && c.rows <= 16 && w->tn <= kChipUnits && w->k % 8 == 0) {
        a.wk = std::min(w->tk, w->tk >= 64 ? kDirectWaves : 4);
        a.turns = (w->tk + a.wk - 1) / a.wk;
        const hipError_t err = c.x_dtype == BILD_DT_F16 ? launch_direct<AS_F16>(a, w->group, st) : launch_direct<AS_BF16>(a, w->group, st);
        return err == hipSuccess ? BILD_OK : BILD_EHIP;
    }
    // More rows than a workgroup stages, from 96 blocks of 64 rows by 128 features on.  us, staged / in blocks, groups of 64 (4096 x 4096, 1024 wide) and 128, fp16: 4096 x 4096 of 128, 256, 1024 rows (64, 128,
    // 512 blocks) 20.1 / 25.3, 30.0 / 26.2, 90.9 / 51.7; 4096 x 11008 of 128, 256, 1024 46.4 / 51.6, 73.9 / 53.6, 213 / 107; 11008 x 4096 of 96 rows (172) 38.0 / 24.8;
    // 32000 x 1024 of 33 and 512 (250, 2000) 18.4 / 13.2, 111 / 92; 1024 x 1024 of 512 and 1024 (64, 128) 7.4 / 12.0, 10.7 / 11.4.
    const int blocks = (w->tn + kBlockFeatures / 16 - 1) / (kBlockFeatures / 16), row_blocks64 = (c.rows + kBlockRows - 1) / kBlockRows;
    if (!parts && c.rows > kPartRows && (int64_t)blocks * row_blocks64 >= 96 && (int64_t)blocks * row_blocks64 <= 1 << 22 && w->k % 8 == 0 && ((uintptr_t)c.x & 15) == 0 && c.x_stride % 8 == 0) {
        a.nothing = (const uint4*)w->nothing;
        a.per = (blocks + 7) / 8;
        const dim3 grid((unsigned)(8 * a.per * row_blocks64));
        const hipError_t err = c.x_dtype == BILD_DT_F16 ? launch_block<AS_F16>(a, w->group, grid, st) : launch_block<AS_BF16>(a, w->group, grid, st);
        return err == hipSuccess ? BILD_OK : BILD_EHIP;
    }
    a.rows_per = std::min(c.rows, kPartRows);
    const int v = a.rows_per * (parts ? 3 : 1);
    const int tiles = v <= 16 ? 1 : v <= 32 ? 2 : v <= 48 ? 3 : 6;
    const int row_blocks = (c.rows + a.rows_per - 1) / a.rows_per, tile_bytes = v * kTileK * 2;
    const int turn = ahead(w->group), most = kMaxWaves, wave_sums = tiles * 1024;
    const int room = kLdsLimit - 4096;  // (beside the squares)
    const int units = std::max(1, kChipUnits / row_blocks);
    // How many waves share a feature tile, and how many tiles a workgroup has beside each other (no more than gives one to every compute unit) and one after the other.
    const bool fits = w->tk * tile_bytes + wave_sums <= room;
    int wf = 1;
    int64_t best = 0;
    for (int wk = 1, l = 0; wk <= most && wk <= w->tk; wk *= 2, ++l) {
        if (!fits && wk * tile_bytes > room) break;  // (of so few input tiles at a time every wave is to have one)
        for (int side = std::min(most / wk, (w->tn + units - 1) / units); side * wk <= most; side *= 2) {
            const int waves = side * wk, sums_room = fits ? std::max(1, (room - w->tk * tile_bytes) / (waves * wave_sums)) : 1;
            const int per = std::max(1, std::min((w->tn + units * side - 1) / (units * side), sums_room));
            const int rounds = (w->tn + units * side * per - 1) / (units * side * per);
            // clocks of a compute unit: rows at 64 bytes each, or as fast as its waves take them apart, a tile as fast as memory brings it or the matrix cores take it, the sums
            // (346 x 32 features, one wave each: 32 rows of fp32 16.8 us; several tiles' waves in a workgroup 7.5)
            const int stage = std::max(v * w->k / 32, a.rows_per * ((w->tk + 3) / 4) * (parts ? 400 : 100) / std::min(waves, 4));
            const int64_t cost = (int64_t)rounds * (stage + per * (10 * ((w->tk + wk - 1) / wk) + 6) * std::max(waves, 12) * std::max(10, 6 * tiles));
            if (best && cost >= best) continue;
            best = cost;
            a.wk = wk;
            a.lwk = l;
            a.per = per;
            wf = side;
        }
    }
    const int waves = wf * a.wk;
    // The rows in LDS, all of them or as many input tiles as there is room for, in chunks of equal turns.
    a.chunk = w->tk;
    if (!fits) {
        a.chunk = room / (a.wk * tile_bytes) * a.wk;
        const int n = (w->tk + a.chunk - 1) / a.chunk;
        a.chunk = ((w->tk + n - 1) / n + a.wk - 1) / a.wk * a.wk;
    }
    a.chunks = (w->tk + a.chunk - 1) / a.chunk;
    const unsigned row_waves = (unsigned)(a.chunk * (kTileK / 8) + 63) / 64;
    a.span_m = row_waves == 1 ? 0u : (unsigned)((0xFFFFFFFFull + row_waves) / row_waves);
    a.turns = (a.chunk + a.wk - 1) / a.wk;
    if (a.chunks > 1) a.turns = (a.turns + turn - 1) / turn * turn;
    a.sums_at = a.per > 1 ? a.chunk * tile_bytes : 0;
    const size_t sums = (size_t)a.per * waves * wave_sums, lds = a.per > 1 ? a.sums_at + sums : std::max((size_t)a.chunk * tile_bytes, sums);
    const dim3 grid((w->tn + wf * a.per - 1) / (wf * a.per), row_blocks);
    const hipError_t err = parts ? launch_group<AS_PARTS>(a, w->group, tiles, grid, waves, lds, w->device, st)
                           : c.x_dtype == BILD_DT_F16 ? launch_group<AS_F16>(a, w->group, tiles, grid, waves, lds, w->device, st)
                                                      : launch_group<AS_BF16>(a, w->group, tiles, grid, waves, lds, w->device, st);
    return err == hipSuccess ? BILD_OK : BILD_EHIP;
}

}  // namespace bild

extern "C" int bild_quant_round(const float* w, int n, int k, int inputs_first, int group, int scale_dtype, uint8_t* codes, void* scales, uint8_t* zeros) {
    if (!w || !codes || !scales || !shape_ok(n, k, group)) return BILD_EINVAL;
    if (scale_dtype != BILD_DT_F16 && scale_dtype != BILD_DT_BF16) return BILD_EINVAL;
    const int groups = (k + group - 1) / group, bytes = (k + 1) / 2;
    const int threads = std::min({16, n, std::max(1, (int)((int64_t)n * k >> 16))});
    std::vector<char> good;
    const auto part = [&](int t) {
        bool ok = true;
        for (int f = t; f < n && ok; f += threads)
            ok = round_feature(inputs_first ? w + f : w + (int64_t)f * k, inputs_first ? n : 1, k, group, scale_dtype, codes + (size_t)f * bytes,
                               (uint16_t*)scales + (size_t)f * groups, zeros ? zeros + (size_t)f * groups : nullptr);
        good[t] = ok;
    };
    try {
        good.resize(threads);
        std::vector<std::thread> others;
        others.reserve(threads);
        int made = 1;
        try {
            for (; made < threads; ++made) others.emplace_back(part, made);
        } catch (...) {  // (no more threads to be had: this one does the rest)
        }
        part(0);
        for (std::thread& o : others) o.join();
        for (; made < threads; ++made) part(made);
    } catch (...) {
        return BILD_ENOMEM;
    }
    return std::all_of(good.begin(), good.end(), [](char g) { return g != 0; }) ? BILD_OK : BILD_EINVAL;
}

extern "C" int bild_quant_create(int n, int k, int group, const uint8_t* codes, const void* scales, int scale_dtype, const uint8_t* zeros, bild_quant** out) {
    if (!codes || !scales || !out || !shape_ok(n, k, group)) return BILD_EINVAL;
    if (scale_dtype != BILD_DT_F16 && scale_dtype != BILD_DT_BF16) return BILD_EINVAL;
    int ndev = 0;
    if (hipGetDeviceCount(&ndev) != hipSuccess || ndev < 1) return BILD_EHIP;
    bild_quant* q = new (std::nothrow) bild_quant();
    if (!q) return BILD_ENOMEM;
    q->n = n;
    q->k = k;
    q->group = group;
    q->tn = (n + 15) / 16;
    q->tk = (k + kTileK - 1) / kTileK;
    const size_t tiles = (size_t)q->tn * q->tk;
    const size_t groups = (size_t)(k + group - 1) / group;
    // what stays, and behind it what was given
    const size_t code_bytes = tiles * 1024, side_bytes = (tiles * 64 * side_words(kTileK / group) + 255) / 256 * 256;
    const size_t raw_codes = (size_t)n * ((k + 1) / 2), raw_scales = (size_t)n * groups * 2, raw_zeros = zeros ? (size_t)n * groups : 0;
    const size_t scales_at = (raw_codes + 255) / 256 * 256, zeros_at = scales_at + (raw_scales + 255) / 256 * 256, bad_at = zeros_at + (raw_zeros + 255) / 256 * 256;
    char* raw = nullptr;
    int rc = BILD_OK;
    if (hipGetDevice(&q->device) != hipSuccess) rc = BILD_EHIP;
    else if (hipMalloc(&q->mem, code_bytes + side_bytes + 256) != hipSuccess) q->mem = nullptr, rc = BILD_ENOMEM;
    else if (hipMalloc((void**)&raw, bad_at + 256) != hipSuccess) raw = nullptr, rc = BILD_ENOMEM;
    if (rc == BILD_OK) {
        q->codes = (const uint4*)q->mem;
        q->sides = (const uint32_t*)((char*)q->mem + code_bytes);
        q->nothing = (char*)q->mem + code_bytes + side_bytes;
        unsigned bad = 0;
        bool ok = hipMemset((void*)q->nothing, 0, 256) == hipSuccess && hipMemcpy(raw, codes, raw_codes, hipMemcpyDefault) == hipSuccess && hipMemcpy(raw + scales_at, scales, raw_scales, hipMemcpyDefault) == hipSuccess &&
                  (!zeros || hipMemcpy(raw + zeros_at, zeros, raw_zeros, hipMemcpyDefault) == hipSuccess) && hipMemset(raw + bad_at, 0, sizeof(unsigned)) == hipSuccess;
        const size_t lanes = tiles * 64;
        const int bf16 = scale_dtype == BILD_DT_BF16;
        if (ok && bf16) {  // fp16 times a power of two: its 11 bits and 40 binary places hold all of them, or the matrix is refused
            int range[2] = {-1024, 1024};
            int* at = (int*)(raw + bad_at + 16);
            ok = hipMemcpy(at, range, sizeof(range), hipMemcpyHostToDevice) == hipSuccess;
            if (ok) {
                const size_t count = (size_t)n * groups;
                ok = launch_on(quant_range_kernel, dim3((unsigned)std::min<size_t>((count + 255) / 256, 1024)), dim3(256), 0, nullptr, (const uint16_t*)(raw + scales_at), count, at) == hipSuccess &&
                     hipMemcpy(range, at, sizeof(range), hipMemcpyDeviceToHost) == hipSuccess;
            }
            // (of the powers of two that do, the one nearest to none: sums of products then stay near the results' size, which fp32 holds)
            if (ok && range[0] >= range[1]) {
                const int least = range[0] - 15, most = range[1] + 24;
                q->scale_exponent = std::max(least, std::min(most, 0));
                bad = least > most;
            }
        }
        if (ok && !bad) {
            ok = launch_on(quant_layout_kernel, dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0, nullptr, (const uint8_t*)raw, (const uint16_t*)(raw + scales_at),
                           zeros ? (const uint8_t*)(raw + zeros_at) : nullptr, n, k, group, q->tk, lanes, -q->scale_exponent, bf16, (uint32_t*)q->codes, (uint32_t*)q->sides,
                           (unsigned*)(raw + bad_at)) == hipSuccess && hipMemcpy(&bad, raw + bad_at, sizeof(bad), hipMemcpyDeviceToHost) == hipSuccess;
        }
        rc = !ok ? BILD_EHIP : bad ? BILD_EINVAL : BILD_OK;
    }
    if (raw) (void)hipFree(raw);
    if (rc != BILD_OK) {
        (void)hipGetLastError();  // (told by rc: not to be found by a later call as well)
        (void)bild_quant_destroy(q);
        return rc;
    }
    *out = q;
    return BILD_OK;
}

extern "C" int bild_quant_destroy(bild_quant* w) {
    if (!w) return BILD_EINVAL;
    if (w->mem) (void)hipFree(w->mem);
    delete w;
    return BILD_OK;
}

extern "C" int bild_quant_matmul(const bild_quant* w, const bild_quant_call* c, void* hip_stream) {
    if (!w || !c || !c->x || !c->y) return BILD_EINVAL;
    if (c->rows < 1 || c->rows > 32 * 65535 || !row_type(c->x_dtype) || !row_type(c->y_dtype) || !(c->eps >= 0.f)) return BILD_EINVAL;
    const OnDevice on(w->device);
    if (!on.ok) return BILD_EHIP;
    return launch_quant(w, *c, (hipStream_t)hip_stream);
}
