// Attention over the cache in 8 bits (bild_cache_attend), all keys or a sliding window with sinks: the kernel for a few rows a sequence, heads up to 128, and the choice between this one, the one for
// prompts (cache_prompt.hip) and the one for larger heads (cache_attend_tall.hip).
//
//   out = sum_j p_j s_v[j] cv_j / 127,  p = softmax_j(scale s_k[j] q ck_j / 127)
//
// Bound: HBM, a byte a value, each key and value read once for all rows and query heads of its key head (up to 16: a tile).  The tile's rows are one operand of the matrix cores.  Scores come out
// transposed, S^T = K Q^T, so that a lane has eight consecutive keys of one row, which is what the second product, O^T = V^T P^T, takes from it: weights go from one to the other in
// registers.  Codes become fp16 by a byte permutation and a packed product and sum (cache_attend.h), with the values' transposition into the bargain: the pairs that the permutation joins are two
// tokens' codes.  A page's scale is applied to scores and to partial sums in fp32.
//
// Work is cut where it is: the 32-token blocks of all sequences and row tiles lie in one line, of which each workgroup of a key head takes an equal piece, wherever sequences begin or
// end (the lengths are in device memory, and a batch's are far apart); a workgroup's eight waves take turns over its blocks, or over tiles that are short.  What several workgroups have
// of a tile the last of them joins, in order.
//
// Measured: 32 heads of 128 over 65537 positions, fp16, 92 us, 5.8 TB/s (reads alone reach 6.1).  64 sequences of up to 16384, 8 key heads: 59 us, 4.0 TB/s: a workgroup gets to two to four
// tiles, and from the beginning of one to its meeting are some 10 us beside its blocks: lengths 1, table and scales 2, first codes 2.4, joining waves 3, meeting and joining parts 3.
// One sequence of 513 positions 7.7 us: the same chain.  What did not help: codes of two blocks on their way (the same to 3 % slower), a piece of the line a wave instead of a workgroup (batches of
// short sequences 5 to 15 % faster, all else 3 to 10 % slower).
//
// Not for heads above 128: an instantiation for 256 of the form before this one, whose line of work the compiler did not know to be the same in all lanes, ended in a memory fault, and its cause was not
// found.  (Instantiations hold some hundred scalar registers in lanes of vector registers; none goes to memory.)
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "cache_attend.h"
#include "last_in.h"

using namespace bild;

namespace {

// (twice as many workgroups of half as many waves have twice as many parts to join)
constexpr int kWaves = 8, kThreads = 64 * kWaves;

// (quotients of what is uniform and nearly always below 2^32: a 64-bit division is a hundred instructions)
__device__ __forceinline__ long long quotient(long long a, long long b) {
    return a < (1ll << 32) && b < (1ll << 32) ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}

// What each workgroup takes of a line: equal pieces, none less than `least` unless it is all there is.
__device__ __forceinline__ long long piece_of(long long line, int groups, int least) {
    const long long pieces = min(max(quotient(line, least), 1ll), (long long)groups);
    return quotient(line + pieces - 1, pieces);
}

// A lane's value, for all of them: what the work is cut by has to be known to be the same in all lanes, or every load of codes would be a loop over the bases it might have.
__device__ __forceinline__ long long lane_of(long long x, int lane) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane);
    return (long long)((uint64_t)hi << 32 | lo);
}

// Registers of a block's codes.
template <int DP>
struct Codes {
    static constexpr int NK = DP / 64, NJ = DP / 16, WV = NJ / 4;
    u32x4 k[2][NK];   // two keys of a lane, 16 codes of each 64
    uint32_t v[8][WV];  // eight values, NJ codes of each
};

// N (2 or 4) floats of a row of partial results.
template <int N>
__device__ __forceinline__ void put_part(__amdgpu_buffer_rsrc_t mem, int off, const float (&o)[N]) {
    if constexpr (N == 2) __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(o[0]), __float_as_uint(o[1])}, mem, off, 0, kPartAux);
    else __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(o[0]), __float_as_uint(o[1]), __float_as_uint(o[2]), __float_as_uint(o[3])}, mem, off, 0, kPartAux);
}
template <int N>
__device__ __forceinline__ void get_part(__amdgpu_buffer_rsrc_t mem, int off, float (&o)[N]) {
    if constexpr (N == 2) {
        const auto y = __builtin_amdgcn_raw_buffer_load_b64(mem, off, 0, kPartAux);
        o[0] = __uint_as_float(y[0]);
        o[1] = __uint_as_float(y[1]);
    } else {
        const auto y = __builtin_amdgcn_raw_buffer_load_b128(mem, off, 0, kPartAux);
#pragma unroll
        for (int u = 0; u < 4; ++u) o[u] = __uint_as_float(y[u]);
    }
}

// ONCE: no other tile has the same keys.
template <class R, int DP, bool ONCE>
__global__ __launch_bounds__(kThreads, 2) void cache_attend_kernel(const AttendArgs a) {
    constexpr bool TWO = R::kDtype == BILD_DT_F32;  // rows and weights in two fp16 parts
    constexpr int NK = DP / 64, KS = DP / 32, NJ = DP / 16, WV = NJ / 4, TERMS = TWO ? 2 : 1, LD = DP + 4;
    // Codes that are read once do not push others out of the caches (us: 32 heads x 65537 positions 103 / 89; where tiles share them, 60 rows of 4 heads over 2000 positions 80 / 96)
    constexpr int kAux = ONCE ? 2 : 0;  // nt
    constexpr int kCols = kThreads / kTile, NC = DP / kCols;  // threads of a row of results, columns of each
    typedef typename R::type V;
    extern __shared__ __attribute__((aligned(16))) float sums[];  // [waves or slots][16 rows][LD]
    __shared__ float tops[kWaves * kTile], weights[kWaves * kTile];
    __shared__ long long scan_sums[kWaves];
    __shared__ int found;
    __shared__ long long found_at;
    __shared__ unsigned share;
    const CacheView& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, g = lane >> 4;
    const int head = blockIdx.y, d = c.d_head;

    // where this workgroup's piece of the line begins; up to 64 sequences, a lane a sequence, each wave finds out for itself
    long long line, chunk, w0, at;
    int i;
    Seq mine_seq;
    const bool in_lanes = a.r.n <= 64;
    const auto seq_of = [&](int k) {
        if (!in_lanes) return sequence_at(a, k);
        Seq q;
        q.s = __builtin_amdgcn_readlane(mine_seq.s, k);
        q.first = __builtin_amdgcn_readlane(mine_seq.first, k);
        q.count = __builtin_amdgcn_readlane(mine_seq.count, k);
        q.length = __builtin_amdgcn_readlane(mine_seq.length, k);
        q.tiles = __builtin_amdgcn_readlane(mine_seq.tiles, k);
        q.sink_blocks = __builtin_amdgcn_readlane(mine_seq.sink_blocks, k);
        q.low_block = __builtin_amdgcn_readlane(mine_seq.low_block, k);
        q.blocks = __builtin_amdgcn_readlane(mine_seq.blocks, k);
        return q;
    };
    const auto up_to = [&](long long x) {  // inclusive prefix sums of a wave
        if (!__any(x >= 1 << 25)) return (long long)prefix_sum((int)x);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const long long y = __shfl_up(x, o, 64);
            if (lane >= o) x += y;
        }
        return x;
    };
    if (in_lanes) {
        mine_seq = sequence_at(a, min(lane, a.r.n - 1));
        if (lane >= a.r.n) mine_seq.tiles = 0;
        const long long mine = (long long)mine_seq.tiles * mine_seq.cost(), x = up_to(mine);
        line = lane_of(x, 63);
        chunk = piece_of(line, a.groups, a.least);
        w0 = blockIdx.x * chunk;
        if (w0 >= line) return;
        i = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(__ballot(w0 < x)));
        at = lane_of(x - mine, i);
    } else {
        const int per = (a.r.n + kThreads - 1) / kThreads, i0 = min(tid * per, a.r.n), i1 = min(i0 + per, a.r.n);
        long long mine = 0;
        for (int k = i0; k < i1; ++k) {
            const Seq q = sequence_at(a, k);
            mine += (long long)q.tiles * q.cost();
        }
        const long long x = up_to(mine);
        if (lane == 63) scan_sums[wave] = x;
        __syncthreads();
        long long before = x - mine;
        line = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            before += w < wave ? scan_sums[w] : 0;
            line += scan_sums[w];
        }
        line = lane_of(line, 0);
        chunk = piece_of(line, a.groups, a.least);
        w0 = blockIdx.x * chunk;
        if (w0 >= line) return;
        if (before <= w0 && w0 < before + mine) {
            int k = i0;
            for (;; ++k) {
                const Seq q = sequence_at(a, k);
                const long long next = before + (long long)q.tiles * q.cost();
                if (w0 < next) break;
                before = next;
            }
            found = k;
            found_at = before;
        }
        __syncthreads();
        i = __builtin_amdgcn_readfirstlane(found);
        at = lane_of(found_at, 0);
    }
    const long long w1 = min(w0 + chunk, line);
    Seq sq = seq_of(i);

    int turn = 0;
    for (long long w = w0; w < w1;) {
        while (w >= at + (long long)sq.tiles * sq.cost()) {
            at += (long long)sq.tiles * sq.cost();
            sq = seq_of(++i);
        }
        const int cost = sq.cost(), tile = (int)quotient(w - at, cost), c0 = (int)((w - at) - (long long)tile * cost), c1 = (int)min((long long)cost, c0 + (w1 - w));
        const long long unit = at + (long long)tile * cost;  // where the tile begins
        // (the same numbers give the same bounds to the workgroups on either side)
        const auto block_of = [&](int at_cost) { return at_cost == cost ? sq.blocks : (int)((double)at_cost * sq.blocks / cost); };
        const int b0 = block_of(c0), b1 = block_of(c1);
        // ---- rows
        const int rows = sq.count * a.group, idx = tile * kTile + n16, mine = min(idx, rows - 1), j = mine / a.group, e = mine - j * a.group;
        const int pos = sq.position(j, a.causal), low = a.window ? pos - a.window : -1;
        // the positions that the tile's rows see
        const int j0 = tile * kTile / a.group, j1 = min((tile * kTile + kTile - 1) / a.group, sq.count - 1);
        const int first_pos = sq.position(j0, a.causal), last_pos = sq.position(j1, a.causal);
        const auto block_at = [&](int b) { return b < sq.sink_blocks ? b : b - sq.sink_blocks + sq.low_block; };
        // ---- a page and its scales for each of the next 64 blocks of this wave, a lane a block
        int pages = -1;
        uint32_t where[2] = {0, 0};  // of the block's keys
        float k_scale = 0.f, v_scale = 0.f;
        // a tile that is no more than a wave's share of the piece is one wave's alone, the next one the next wave's
        const bool whole = c0 == 0 && c1 == cost, alone = whole && sq.blocks <= max(chunk / kWaves, 2ll);
        if (alone && (turn++ & (kWaves - 1)) != wave) {
            w += c1 - c0;
            continue;
        }
        const int step = alone ? 1 : kWaves, begin = alone ? b0 : b0 + wave;
        const auto look_up = [&](int b) {
            const int mine_at = b + step * lane, blk = block_at(mine_at), p0 = blk * kBlock;
            pages = -1;
            if (mine_at < b1 && p0 < sq.length && p0 <= last_pos && (!a.window || p0 + kBlock - 1 > first_pos - a.window || p0 < a.sinks))
                pages = c.table[(int64_t)sq.s * c.max_pages + (p0 >> c.page_shift)];
            if (!c.has(pages)) pages = -1;
            if (pages >= 0) {
                const uint64_t codes = (uint64_t)(c.codes + c.plane(pages, a.layer, 0, head) * c.plane_bytes() + (p0 & (c.page_tokens - 1)) * d);
                where[0] = (uint32_t)codes;
                where[1] = (uint32_t)(codes >> 32);
                k_scale = c.scales[c.plane(pages, a.layer, 0, head)];
                v_scale = c.scales[c.plane(pages, a.layer, 1, head)] * (512.f / 127.f);
            }
        };
        if (begin < b1) look_up(begin);
        const V* x_row = (const V*)a.q + (int64_t)(sq.first + j) * a.q_token + (int64_t)(head * a.group + e) * a.q_head;
        RowVec<R, 8> raw[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) raw[s].load(x_row + min(64 * (s >> 1) + 16 * g, d - 16) + 8 * (s & 1));
        float top = -INFINITY, sum = 0.f;
        f32x4 acc[NJ];
#pragma unroll
        for (int t = 0; t < NJ; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};

        const int64_t to_v = (int64_t)c.heads * c.plane_bytes();
        const int key = (n16 >> 2) * 8 + (n16 & 3);  // the lane's row of the first operand, in two halves: tokens key and key + 4
        const auto load = [&](Codes<DP>& x, uint32_t lo, uint32_t hi) {
            const int8_t* codes = (const int8_t*)((uint64_t)hi << 32 | lo);
            const auto k = make_rsrc(codes, (size_t)(kBlock * d)), v = make_rsrc(codes + to_v, (size_t)(kBlock * d));
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < NK; ++t) {
                    // (rows begin at multiples of 8 bytes)
                    x.k[h][t] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(k, (key + 4 * h) * d + min(64 * t + 16 * g, d - 16), 0, kAux));
                }
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const int off = (8 * g + t) * d + min(n16 * NJ, d - NJ);
                if constexpr (WV == 1) {
                    x.v[t][0] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(v, off, 0, kAux);
                } else {
                    const auto y = __builtin_amdgcn_raw_buffer_load_b64(v, off, 0, kAux);
                    x.v[t][0] = (uint32_t)y[0];
                    x.v[t][1] = (uint32_t)y[1];
                }
            }
        };
        f16x8 q[TERMS][KS];
        float row_scale = 1.f;
        const auto use = [&](Codes<DP>& x, int blk, float ks, float vs) {
            f32x4 z[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                z[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < NK; ++t) {
                    const u32x4 y = x.k[h][t] ^ 0x80808080u;
                    const f16x8 lo = eight_of(y[0], y[1]), hi = eight_of(y[2], y[3]);
#pragma unroll
                    for (int m = 0; m < TERMS; ++m) {
                        z[h] = mma(lo, q[m][2 * t], z[h]);
                        z[h] = mma(hi, q[m][2 * t + 1], z[h]);
                    }
                }
            }
            const float by = ks * a.scale * row_scale;
            const int p0 = blk * kBlock + 8 * g;
            float p[8], big = -INFINITY;
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const int at_pos = p0 + t;
                const bool sees = (at_pos <= pos) & ((at_pos > low) | (at_pos < a.sinks));
                p[t] = sees ? z[t >> 2][t & 3] * by : -INFINITY;
                big = fmaxf(big, p[t]);
            }
            big = quad_rows_max(big);
            if (__any(big > top + kSlack)) {
                const float now = big > top + kSlack ? big : top;
                const float less = now == top ? 1.f : __builtin_amdgcn_exp2f(top - now);
                sum *= less;
#pragma unroll
                for (int t = 0; t < NJ; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[t][r] *= less;
                top = now;
            }
            const float base = top == -INFINITY ? 0.f : top;
            f16x8 w[TERMS];
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const float v = __builtin_amdgcn_exp2f(p[t] - base);
                sum += v;
                w[0][t] = (_Float16)v;
                if (TWO) w[TERMS - 1][t] = (_Float16)(v - (float)w[0][t]);
            }
#pragma unroll
            for (int t = 0; t < 8; ++t)
#pragma unroll
                for (int y = 0; y < WV; ++y) x.v[t][y] ^= 0x80808080u;
#pragma unroll
            for (int t = 0; t < NJ; ++t) {
                const int y = t / 4, k = t % 4;
                const f16x8 v = eight(pair_of(x.v[0][y], x.v[1][y], k), pair_of(x.v[2][y], x.v[3][y], k), pair_of(x.v[4][y], x.v[5][y], k), pair_of(x.v[6][y], x.v[7][y], k));
                f32x4 part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int m = 0; m < TERMS; ++m) part = mma(v, w[m], part);
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[t][r] = __builtin_fmaf(part[r], vs, acc[t][r]);
            }
        };
        // ---- the wave's blocks, the next one's codes on their way
        Codes<DP> one;
        int nth = 0, b = begin - step;  // of the looked up ones
        struct Next {
            int blk;  // -1: no more
            float ks, vs;
        };
        const auto next = [&](Codes<DP>& x) {
            Next r = {-1, 0.f, 0.f};
            for (b += step; b < b1; b += step) {
                if (nth == 64) {
                    look_up(b);
                    nth = 0;
                }
                const int page = __builtin_amdgcn_readlane(pages, nth), was = nth++;
                if (page >= 0) {
                    r.blk = block_at(b);
                    load(x, (uint32_t)__builtin_amdgcn_readlane((int)where[0], was), (uint32_t)__builtin_amdgcn_readlane((int)where[1], was));
                    // (the scales were asked for before: whoever waits for them does not wait for these codes)
                    r.ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k_scale), was));
                    r.vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v_scale), was));
                    break;
                }
            }
            return r;
        };
        Next x = next(one);
        // (the rows while the first codes are on their way)
        {
            // (a piece behind the head's end begins earlier, by eights; what another lane has as well is 0 here)
            const auto has = [&](int s) { return 8 * (s & 1) >= 64 * (s >> 1) + 16 * g - min(64 * (s >> 1) + 16 * g, d - 16); };
            float big = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                float most = 0.f;
#pragma unroll
                for (int t = 0; t < 8; ++t) most = fmaxf(most, fabsf(R::up(raw[s].v[t])));
                big = fmaxf(big, has(s) ? most : 0.f);
            }
            big = quad_rows_max(big);
            const int up = up_of(big);
            row_scale = ldexpf(1.f, -up);
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const bool here = has(s);
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    const float v = here ? ldexpf(R::up(raw[s].v[t]), up) : 0.f;
                    q[0][s][t] = (_Float16)v;
                    if (TWO) q[TERMS - 1][s][t] = (_Float16)(v - (float)q[0][s][t]);
                }
            }
        }
        while (x.blk >= 0) {
            use(one, x.blk, x.ks, x.vs);
            x = next(one);
        }

        // ---- the waves' results joined: a slot of kCols threads a row
        sum = quad_rows_sum(sum);
        if (alone) {
            if (idx < rows) {
                const int64_t t_at = sq.first + j;
                const int h = head * a.group + e;
                const float by = sum == 0.f ? 0.f : 1.f / sum;
                V* out = (V*)a.out + t_at * a.out_token + (int64_t)h * a.out_head;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int dim = (4 * g + r) * NJ;
                    RowVec<R, NJ> y;
#pragma unroll
                    for (int t = 0; t < NJ; ++t) y.v[t] = R::down(acc[t][r] * by);
                    if (dim < d) y.store(out + dim);
                }
                if (a.lse && g == 0) a.lse[t_at * a.heads + h] = sum == 0.f ? -INFINITY : top * kLn2 + logf(sum);
            }
            w += c1 - c0;
            continue;
        }
        const int slot = tid / kCols, col = tid % kCols * NC, valid = min(kTile, rows - tile * kTile);
        if (n16 < valid) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float* to = sums + (wave * kTile + n16) * LD + (4 * g + r) * NJ;
#pragma unroll
                for (int t = 0; t < NJ; t += 4) *(float4*)(to + t) = make_float4(acc[t][r], acc[t + 1][r], acc[t + 2][r], acc[t + 3][r]);
            }
            if (g == 0) {
                tops[wave * kTile + n16] = top;
                weights[wave * kTile + n16] = sum;
            }
        }
        lds_barrier();
        float m = -INFINITY, l = 0.f, o[NC];
#pragma unroll
        for (int t = 0; t < NC; ++t) o[t] = 0.f;
        const auto fold = [&](float pm, float pl, const float* po) {  // (parts that have seen nothing: of weight 0)
            const float now = fmaxf(m, pm), base = now == -INFINITY ? 0.f : now;
            const float was = __builtin_amdgcn_exp2f(m - base), is = __builtin_amdgcn_exp2f(pm - base);
            l = l * was + pl * is;
#pragma unroll
            for (int t = 0; t < NC; ++t) o[t] = o[t] * was + po[t] * is;
            m = now;
        };
        if (slot < valid) {
            float tk[kWaves], by[kWaves];
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                tk[k] = tops[k * kTile + slot];
                m = fmaxf(m, tk[k]);
            }
            const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                by[k] = __builtin_amdgcn_exp2f(tk[k] - base);
                l = __builtin_fmaf(weights[k * kTile + slot], by[k], l);
            }
#pragma unroll
            for (int k = 0; k < kWaves; ++k)
#pragma unroll
                for (int t = 0; t < NC; ++t) o[t] = __builtin_fmaf(sums[(k * kTile + slot) * LD + col + t], by[k], o[t]);
        }
        const auto put = [&](int row) {
            const int jr = (tile * kTile + row) / a.group, er = tile * kTile + row - jr * a.group, h = head * a.group + er;
            const int64_t t_at = sq.first + jr;
            const float by = l == 0.f ? 0.f : 1.f / l;
            // (a last piece of values that is cut began earlier: so many columns hold what the piece before has)
            const int cut = max(col / NJ * NJ + NJ - d, 0), dim = col - cut;
            if (col / NJ * NJ < d) {
                V* out = (V*)a.out + t_at * a.out_token + (int64_t)h * a.out_head + dim;
                RowVec<R, NC> y;
#pragma unroll
                for (int u = 0; u < NC; ++u) y.v[u] = R::down(o[u] * by);
                y.store(out);
            }
            if (a.lse && col == 0) a.lse[t_at * a.heads + h] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
        };
        if (whole) {
            if (slot < valid) put(slot);
            lds_barrier();
        } else {
            // the workgroups that share the tile: in the first of them it begins last, in the others first
            const int from = (int)quotient(unit, chunk), to = (int)quotient(unit + cost - 1, chunk);
            constexpr int kRow = part_row(DP);
            const int64_t place = ((int64_t)head * a.groups + blockIdx.x) * 2 + (blockIdx.x == from);
            const auto mem = make_rsrc(a.part + place * kTile * kRow, sizeof(float) * kTile * kRow);
            if (slot < valid) {
                put_part<NC>(mem, (slot * kRow + col) * 4, o);
                if (col == 0) __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(m), __float_as_uint(l), 0u, 0u}, mem, (slot * kRow + DP) * 4, 0, kPartAux);
            }
            if (last_in(a.arrived + (int64_t)head * a.groups + from, (unsigned)(to - from + 1), &share)) {
                // each row's parts dealt to as many slots as there are
                int lanes = 1;
                while (lanes < valid) lanes <<= 1;
                const int apart = kTile / lanes, row = slot & (lanes - 1), sub = slot / lanes;
                m = -INFINITY;
                l = 0.f;
#pragma unroll
                for (int t = 0; t < NC; ++t) o[t] = 0.f;
                for (int p = from + sub; p <= to && row < valid; p += apart) {
                    const int64_t where = ((int64_t)head * a.groups + p) * 2 + (p == from);
                    const auto src = make_rsrc(a.part + where * kTile * kRow, sizeof(float) * kTile * kRow);
                    float po[NC];
                    const u32x4 ml = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(src, (row * kRow + DP) * 4, 0, kPartAux));
                    get_part<NC>(src, (row * kRow + col) * 4, po);
                    fold(__uint_as_float(ml[0]), __uint_as_float(ml[1]), po);
                }
                if (apart > 1) {
#pragma unroll
                    for (int t = 0; t < NC; ++t) sums[slot * LD + col + t] = o[t];
                    if (col == 0) {
                        tops[slot] = m;
                        weights[slot] = l;
                    }
                    __syncthreads();
                    if (slot < valid) {
                        m = -INFINITY;
                        l = 0.f;
#pragma unroll
                        for (int t = 0; t < NC; ++t) o[t] = 0.f;
                        for (int k = 0; k < apart; ++k) fold(tops[k * lanes + slot], weights[k * lanes + slot], sums + (k * lanes + slot) * LD + col);
                    }
                }
                if (slot < valid) put(slot);
            }
            __syncthreads();
        }
        w += c1 - c0;
    }
}

// Rows (times query heads of a key head) of a sequence from which on they take the kernel for prompts: a whole tile of it, or half a one where there is much of it, rows times query heads of all
// sequences.  (us, this kernel / that one: 16 rows of 4 heads over 2000 positions, 32 sequences of 8 key heads 95 / 69, 64 rows over 8000, 32 key heads 50 / 53, 20 of 4 over 4000, 8 key heads 23 / 33;
// 60 of 4 over 2000, 8 sequences 86 / 46; 8 of 4 over 2000, 32 sequences 55 / 70.)
constexpr int kPromptFrom = 64, kPromptWork = 4096;
// Of the line that a workgroup takes, at least (us, call, of 14 / 20 / 28: one sequence of 513 positions 14.4 / 12.9 / 12.9, of 8000, 8 key heads 20.7 / 20.5 / 22.4).
constexpr int kLeast = 20;

constexpr size_t lds_bytes(int DP) { return sizeof(float) * kWaves * kTile * (DP + 4); }

template <class R, int DP, bool ONCE>
hipError_t launch(const AttendArgs& a, hipStream_t st) {
    return launch_on(cache_attend_kernel<R, DP, ONCE>, dim3(a.groups, a.c.heads), dim3(kThreads), lds_bytes(DP), st, a);
}
template <class R>
hipError_t launch(const AttendArgs& a, hipStream_t st) {
    const bool once = (int64_t)a.r.rows * a.group <= kTile;
    if (a.c.d_head <= 64) return once ? launch<R, 64, true>(a, st) : launch<R, 64, false>(a, st);
    return once ? launch<R, 128, true>(a, st) : launch<R, 128, false>(a, st);
}

}  // namespace

namespace bild {

hipError_t attend_init(int d_head) {
    const void* const half[] = {(const void*)cache_attend_kernel<RowF32, 128, true>,  (const void*)cache_attend_kernel<RowBf16, 128, true>,  (const void*)cache_attend_kernel<RowF16, 128, true>,
                                (const void*)cache_attend_kernel<RowF32, 128, false>, (const void*)cache_attend_kernel<RowBf16, 128, false>, (const void*)cache_attend_kernel<RowF16, 128, false>};
    if (const hipError_t e = cache_prompt_init(d_head); e != hipSuccess) return e;
    return d_head <= 64 ? hipSuccess : d_head <= 128 ? raise_lds_limit(half, (int)lds_bytes(128)) : cache_attend_tall_init();
}

size_t attend_part_floats(int heads, int d_head) {
    return std::max((size_t)heads * attend_groups(heads) * 2 * kTile * part_row(d_head <= 64 ? 64 : d_head <= 128 ? 128 : 256), prompt_part_floats(d_head));
}

}  // namespace bild

extern "C" int bild_cache_attend(bild_cache* c, const bild_cache_attend_call* call, void* hip_stream) {
    if (!c || !call) return BILD_EINVAL;
    const bild_cache_attend_call& k = *call;
    const CacheView& v = c->view;
    if (!k.q || !k.out || !row_type(k.dtype) || k.layer < 0 || k.layer >= v.layers || k.window < 0 || k.sinks < 0 || !std::isfinite(k.scale)) return BILD_EINVAL;
    if (k.n < 1 || k.n > v.sequences || k.rows < 1 || (k.starts && k.tokens < 1) || (k.causal != 0 && k.causal != 1) || (!k.causal && k.window)) return BILD_EINVAL;
    if (k.heads < 1 || k.heads % v.heads || k.heads / v.heads > 64) return BILD_EINVAL;
    const int64_t tokens = k.starts ? k.tokens : (int64_t)k.n * k.rows;
    if (tokens * k.heads > 0x7FFFFFFF) return BILD_EINVAL;
    AttendArgs a;
    std::memset((void*)&a, 0, sizeof(a));
    a.c = v;
    a.r = {k.sequences, k.starts, k.n, k.rows, (int)tokens};
    a.q = k.q;
    a.out = k.out;
    a.lse = k.lse;
    a.q_token = k.q_token;
    a.q_head = k.q_head;
    a.out_token = k.out_token;
    a.out_head = k.out_head;
    a.layer = k.layer;
    a.heads = k.heads;
    a.group = k.heads / v.heads;
    a.window = std::min(k.window, v.cap());  // (a wider one hides no more)
    a.sinks = k.window ? k.sinks : 0;
    a.causal = k.causal;
    a.scale = (float)((double)k.scale * 1.4426950408889634 * 512.0 / 127.0);
    a.groups = attend_groups(v.heads);
    a.least = kLeast;
    const int64_t tiles = k.starts ? tokens * a.group / kPromptRows + k.n : k.n * (((int64_t)k.rows * a.group + kPromptRows - 1) / kPromptRows);
    // Places for workgroups: fewer tiles than the chip has room for share their keys between several.  Up to 64 sequences that goes by each one's length, which the kernel finds out: at most
    // kPromptParts are pieces of tiles.
    a.splits = (int)std::min(std::max(kPromptParts / (tiles * v.heads), (int64_t)1), (int64_t)kMaxSplits);
    const int64_t most = kPromptParts / v.heads, places = k.n > 64 ? tiles * a.splits : k.n > 1 ? tiles + std::min(most, tiles * (kMaxSplits - 1)) : std::max(tiles, std::min(most, tiles * kMaxSplits));
    const int64_t per_head = (int64_t)k.rows * a.group;
    const bool prompts = (per_head >= kPromptRows || (per_head >= kPromptFrom && tokens * k.heads >= kPromptWork)) && places * v.heads <= kMaxGroups;
    a.prompt_from = prompts ? kPromptFrom : 0x7FFFFFFF;
    a.part = c->part;
    a.arrived = c->arrived;
    const OnDevice on(c->device);
    if (!on.ok) return BILD_EHIP;
    hipStream_t st = (hipStream_t)hip_stream;
    if (prompts && launch_cache_prompt(a, k.dtype, places, st) != hipSuccess) return BILD_EHIP;
    if (prompts && !k.starts) return BILD_OK;  // (all are prompts; with starts, how many rows a sequence has is known to the kernels alone)
    if (v.d_head > 128) return launch_cache_attend_tall(a, k.dtype, st) == hipSuccess ? BILD_OK : BILD_EHIP;
    const hipError_t err = k.dtype == BILD_DT_F32 ? launch<RowF32>(a, st) : k.dtype == BILD_DT_BF16 ? launch<RowBf16>(a, st) : launch<RowF16>(a, st);
    return err == hipSuccess ? BILD_OK : BILD_EHIP;
}
