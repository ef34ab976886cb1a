// Attention over the cache in 8 bits (bild_cache_attend) of few rows a sequence, heads above 128: cache_attend.hip's walk over the keys in its first form, with four waves a
// workgroup.  (The form with eight is not built for these heads: an instantiation for heads of 256 ended in a memory fault whose cause was not found.)
// Bound: HBM for long sequences; 16 heads of 256 over 65536 positions 108 us a call, 5.0 TB/s; 8 over 4000 24.8 us, which was not taken apart.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "cache_attend.h"
#include "last_in.h"

using namespace bild;

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// Registers of a block's codes.
template <int DP>
struct Codes {
    static constexpr int NK = DP / 64, NJ = DP / 16, WV = NJ / 4;
    u32x4 k[2][NK];   // two keys of a lane, 16 codes of each 64
    uint32_t v[8][WV];  // eight values, NJ codes of each
};

template <class R, int DP>
__global__ __launch_bounds__(kThreads, DP == 256 ? 1 : 2) void cache_attend_tall_kernel(const AttendArgs a) {
    constexpr bool TWO = R::kDtype == BILD_DT_F32;  // rows and weights in two fp16 parts
    constexpr int NK = DP / 64, KS = DP / 32, NJ = DP / 16, WV = NJ / 4, TERMS = TWO ? 2 : 1, LD = DP + 4;
    typedef typename R::type V;
    extern __shared__ __attribute__((aligned(16))) float sums[];  // [4 waves or 16 slots][16 rows][LD], then maxima and sums of weights
    __shared__ float tops[kWaves * kTile], weights[kWaves * kTile];
    __shared__ long long scan_sums[kWaves];
    __shared__ int found;
    __shared__ Seq found_seq;
    __shared__ long long found_at;
    __shared__ unsigned share;
    const CacheView& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, g = lane >> 4;
    const int head = blockIdx.y, d = c.d_head;

    // where this workgroup's piece of the line begins
    long long w0, w1, line;
    {
        const int per = (a.r.n + kThreads - 1) / kThreads, i0 = min(tid * per, a.r.n), i1 = min(i0 + per, a.r.n);
        long long mine = 0;
        Seq last;
        for (int i = i0; i < i1; ++i) {
            last = sequence_at(a, i);
            mine += (long long)last.tiles * last.cost();
        }
        long long x = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const long long y = __shfl_up(x, o, 64);
            if (lane >= o) x += y;
        }
        if (lane == 63) scan_sums[wave] = x;
        __syncthreads();
        long long before = x - mine;
        line = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            before += w < wave ? scan_sums[w] : 0;
            line += scan_sums[w];
        }
        const long long chunk = max((line + a.groups - 1) / a.groups, (long long)a.least);
        w0 = blockIdx.x * chunk;
        w1 = min(w0 + chunk, line);
        if (w0 >= line) return;
        if (before <= w0 && w0 < before + mine) {
            int i = i0;
            Seq q = last;
            if (per > 1)
                for (;; ++i) {
                    q = sequence_at(a, i);
                    const long long next = before + (long long)q.tiles * q.cost();
                    if (w0 < next) break;
                    before = next;
                }
            found = i;
            found_seq = q;
            found_at = before;
        }
        __syncthreads();
    }
    const long long chunk = max((line + a.groups - 1) / a.groups, (long long)a.least);
    int i = __builtin_amdgcn_readfirstlane(found);
    long long at = found_at;
    Seq sq = found_seq;

    for (long long w = w0; w < w1;) {
        while (w >= at + (long long)sq.tiles * sq.cost()) {
            at += (long long)sq.tiles * sq.cost();
            sq = sequence_at(a, ++i);
        }
        const int cost = sq.cost(), tile = (int)((w - at) / cost), c0 = (int)((w - at) - (long long)tile * cost), c1 = (int)min((long long)cost, c0 + (w1 - w));
        const long long unit = at + (long long)tile * cost;  // where the tile begins
        const int b0 = (int)((long long)c0 * sq.blocks / cost), b1 = (int)((long long)c1 * sq.blocks / cost);
        // ---- rows
        const int rows = sq.count * a.group, idx = tile * kTile + n16, mine = min(idx, rows - 1), j = mine / a.group, e = mine - j * a.group;
        const int pos = sq.position(j, a.causal), low = a.window ? pos - a.window : -1;
        // the positions that the tile's rows see
        const int j0 = tile * kTile / a.group, j1 = min((tile * kTile + kTile - 1) / a.group, sq.count - 1);
        const int first_pos = sq.position(j0, a.causal), last_pos = sq.position(j1, a.causal);
        const auto block_at = [&](int b) { return b < sq.sink_blocks ? b : b - sq.sink_blocks + sq.low_block; };
        // ---- a page and its scales for each of the next 64 blocks of this wave, a lane a block
        int pages = -1;
        float k_scale = 0.f, v_scale = 0.f;
        const auto look_up = [&](int b) {
            const int mine_at = b + kWaves * lane, blk = block_at(mine_at), p0 = blk * kBlock;
            pages = -1;
            if (mine_at < b1 && p0 < sq.length && p0 <= last_pos && (!a.window || p0 + kBlock - 1 > first_pos - a.window || p0 < a.sinks))
                pages = c.table[(int64_t)sq.s * c.max_pages + (p0 >> c.page_shift)];
            if (!c.has(pages)) pages = -1;
            if (pages >= 0) {
                k_scale = c.scales[c.plane(pages, a.layer, 0, head)];
                v_scale = c.scales[c.plane(pages, a.layer, 1, head)] * (512.f / 127.f);
            }
        };
        if (b0 + wave < b1) look_up(b0 + wave);
        f16x8 q[TERMS][KS];
        float row_scale;
        {
            const V* x = (const V*)a.q + (int64_t)(sq.first + j) * a.q_token + (int64_t)(head * a.group + e) * a.q_head;
            RowVec<R, 8> raw[KS];
            float big = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int begin = 64 * (s >> 1) + 16 * g, off = min(begin, d - 16) + 8 * (s & 1);
                raw[s].load(x + off);
#pragma unroll
                for (int t = 0; t < 8; ++t) big = fmaxf(big, off + t >= begin ? fabsf(R::up(raw[s].v[t])) : 0.f);
            }
            big = quad_rows_max(big);
            const int up = up_of(big);
            row_scale = ldexpf(1.f, -up);
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int begin = 64 * (s >> 1) + 16 * g, off = min(begin, d - 16) + 8 * (s & 1);
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    // (a piece behind the head's end begins earlier, and what another lane has as well is 0 here)
                    const float v = off + t >= begin ? ldexpf(R::up(raw[s].v[t]), up) : 0.f;
                    q[0][s][t] = (_Float16)v;
                    if (TWO) q[TERMS - 1][s][t] = (_Float16)(v - (float)q[0][s][t]);
                }
            }
        }
        float top = -INFINITY, sum = 0.f;
        f32x4 acc[NJ];
#pragma unroll
        for (int t = 0; t < NJ; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};

        const int key = (n16 >> 2) * 8 + (n16 & 3);  // the lane's row of the first operand, in two halves: tokens key and key + 4
        const auto load = [&](Codes<DP>& x, int page, int blk) {
            const int in_page = blk * kBlock & (c.page_tokens - 1);
            const auto k = make_rsrc(c.codes + c.plane(page, a.layer, 0, head) * c.plane_bytes(), (size_t)c.plane_bytes());
            const auto v = make_rsrc(c.codes + c.plane(page, a.layer, 1, head) * c.plane_bytes(), (size_t)c.plane_bytes());
            const int base = in_page * d;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < NK; ++t) {
                    // (rows begin at multiples of 8 bytes)
                    x.k[h][t] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(k, (key + 4 * h) * d + min(64 * t + 16 * g, d - 16), base, 0));
                }
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const int off = (8 * g + t) * d + min(n16 * NJ, d - NJ);
                if constexpr (WV == 1) {
                    x.v[t][0] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(v, off, base, 0);
                } else if constexpr (WV == 2) {
                    const auto y = __builtin_amdgcn_raw_buffer_load_b64(v, off, base, 0);
                    x.v[t][0] = (uint32_t)y[0];
                    x.v[t][1] = (uint32_t)y[1];
                } else {
                    const auto y = __builtin_amdgcn_raw_buffer_load_b128(v, off, base, 0);
#pragma unroll
                    for (int w4 = 0; w4 < 4; ++w4) x.v[t][w4] = (uint32_t)y[w4];
                }
            }
        };
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
                const bool sees = at_pos <= pos && (at_pos > low || at_pos < a.sinks);
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
        Codes<DP> one, other;
        int nth = 0, b = b0 + wave - kWaves;  // of the looked up ones
        struct Next {
            int blk;  // -1: no more
            float ks, vs;
        };
        const auto next = [&](Codes<DP>& x) {
            Next r = {-1, 0.f, 0.f};
            for (b += kWaves; b < b1; b += kWaves) {
                if (nth == 64) {
                    look_up(b);
                    nth = 0;
                }
                const int page = __builtin_amdgcn_readlane(pages, nth), was = nth++;
                if (page >= 0) {
                    r.blk = block_at(b);
                    load(x, page, r.blk);
                    // (the scales were asked for before: whoever waits for them does not wait for these codes)
                    r.ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k_scale), was));
                    r.vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v_scale), was));
                    break;
                }
            }
            return r;
        };
        Next x = next(one);
        while (x.blk >= 0) {
            const Next y = next(other);
            use(one, x.blk, x.ks, x.vs);
            if (y.blk < 0) break;
            x = next(one);
            use(other, y.blk, y.ks, y.vs);
        }

        // ---- the waves' results joined: a slot of 16 threads a row
        sum = quad_rows_sum(sum);
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
        __syncthreads();
        const int slot = tid >> 4, col = (tid & 15) * NJ, valid = min(kTile, rows - tile * kTile);
        float m = -INFINITY, l = 0.f, o[NJ];
#pragma unroll
        for (int t = 0; t < NJ; ++t) o[t] = 0.f;
        const auto fold = [&](float pm, float pl, const float* po) {  // (parts that have seen nothing: of weight 0)
            const float now = fmaxf(m, pm), base = now == -INFINITY ? 0.f : now;
            const float was = __builtin_amdgcn_exp2f(m - base), is = __builtin_amdgcn_exp2f(pm - base);
            l = l * was + pl * is;
#pragma unroll
            for (int t = 0; t < NJ; ++t) o[t] = o[t] * was + po[t] * is;
            m = now;
        };
#pragma unroll
        for (int k = 0; k < kWaves; ++k) fold(tops[k * kTile + slot], weights[k * kTile + slot], sums + (k * kTile + slot) * LD + col);
        const auto put = [&](int row) {
            const int jr = (tile * kTile + row) / a.group, er = tile * kTile + row - jr * a.group, h = head * a.group + er;
            const int64_t t_at = sq.first + jr;
            const float by = l == 0.f ? 0.f : 1.f / l;
            RowVec<R, NJ> y;
#pragma unroll
            for (int t = 0; t < NJ; ++t) y.v[t] = R::down(o[t] * by);
            V* out = (V*)a.out + t_at * a.out_token + (int64_t)h * a.out_head;
            if (col < d) y.store(out + min(col, d - NJ));  // (a last piece that is cut begins earlier, as its loads did: the lane before writes the same there)
            if (a.lse && col == 0) a.lse[t_at * a.heads + h] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
        };
        const bool whole = c0 == 0 && c1 == cost;
        if (whole) {
            if (slot < valid) put(slot);
            __syncthreads();
        } else {
            // the workgroups that share the tile: in the first of them it begins last, in the others first
            const int from = (int)(unit / chunk), to = (int)((unit + cost - 1) / chunk);
            constexpr int kRow = part_row(DP);
            const int64_t place = ((int64_t)head * a.groups + blockIdx.x) * 2 + (blockIdx.x == from);
            const auto mem = make_rsrc(a.part + place * kTile * kRow, sizeof(float) * kTile * kRow);
            if (slot < valid) {
#pragma unroll
                for (int t = 0; t < NJ; t += 4)
                    __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(o[t]), __float_as_uint(o[t + 1]), __float_as_uint(o[t + 2]), __float_as_uint(o[t + 3])}, mem,
                                                           (slot * kRow + col + t) * 4, 0, kPartAux);
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
                for (int t = 0; t < NJ; ++t) o[t] = 0.f;
                for (int p = from + sub; p <= to && row < valid; p += apart) {
                    const int64_t where = ((int64_t)head * a.groups + p) * 2 + (p == from);
                    const auto src = make_rsrc(a.part + where * kTile * kRow, sizeof(float) * kTile * kRow);
                    float po[NJ];
                    const u32x4 ml = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(src, (row * kRow + DP) * 4, 0, kPartAux));
#pragma unroll
                    for (int t = 0; t < NJ; t += 4) {
                        const u32x4 y = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(src, (row * kRow + col + t) * 4, 0, kPartAux));
#pragma unroll
                        for (int u = 0; u < 4; ++u) po[t + u] = __uint_as_float(y[u]);
                    }
                    fold(__uint_as_float(ml[0]), __uint_as_float(ml[1]), po);
                }
                if (apart > 1) {
#pragma unroll
                    for (int t = 0; t < NJ; t += 4) *(float4*)(sums + slot * LD + col + t) = make_float4(o[t], o[t + 1], o[t + 2], o[t + 3]);
                    if (col == 0) {
                        tops[slot] = m;
                        weights[slot] = l;
                    }
                    __syncthreads();
                    if (slot < valid) {
                        m = -INFINITY;
                        l = 0.f;
#pragma unroll
                        for (int t = 0; t < NJ; ++t) o[t] = 0.f;
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

constexpr size_t lds_bytes(int DP) { return sizeof(float) * kWaves * kTile * (DP + 4); }

template <class R>
hipError_t launch(const AttendArgs& a, hipStream_t st) {
    return launch_on(cache_attend_tall_kernel<R, 256>, dim3(a.groups, a.c.heads), dim3(kThreads), lds_bytes(256), st, a);
}

}  // namespace

namespace bild {

hipError_t cache_attend_tall_init() {
    const void* const all[] = {(const void*)cache_attend_tall_kernel<RowF32, 256>, (const void*)cache_attend_tall_kernel<RowBf16, 256>, (const void*)cache_attend_tall_kernel<RowF16, 256>};
    return raise_lds_limit(all, (int)lds_bytes(256));
}

hipError_t launch_cache_attend_tall(const AttendArgs& a, int dtype, hipStream_t st) {
    return dtype == BILD_DT_F32 ? launch<RowF32>(a, st) : dtype == BILD_DT_BF16 ? launch<RowBf16>(a, st) : launch<RowF16>(a, st);
}

}  // namespace bild
