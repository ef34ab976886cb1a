// Attention of prompts over the cache in 8 bits (bild_cache_attend): sequences with many rows.
//
//   out = sum_j p_j s_v[j] cv_j / 127,  p = softmax_j(scale s_k[j] q ck_j / 127), a running maximum and sum, rescaled where a tile's maximum is 2^8 beyond it
//
// A workgroup has 128 rows (rows times the query heads of a key head) of a sequence and walks over its keys, 64 at a time: their codes come from memory into registers while the tile before is
// multiplied, become fp16 on their way into LDS (once for all rows), the values transposed.  A wave has 32 rows; scores come out as S^T = K Q^T, so that weights stay in registers as the operand
// of O^T = V^T P^T: lane l has row l % 32 and of each 16 keys the eight of its half, and the values lie in LDS in that order of keys.  Chunks of 16 bytes are swapped within a row of LDS by the
// row's number, so that neither product's reads meet in a bank.  Scores of keys that a row does not see begin as -infinity.  A page's scale of the values goes into the exponent of its weights (one
// sum, no product a value), relative to a power of two that the results are in units of.
//
// Bound: issue slots and the matrix cores, which work by turns more than side by side (busy 51 and 35 % of the time, by counters; LDS 35 %, of which conflicts are a quarter).  2000 rows of 32 heads of 128, 8 key heads, behind 3001 positions (131 GFLOP): some 155 us among other calls, 178
// back to back at the 1.9 to 2.0 GHz that the chip then keeps, 740 to 850 TFLOP/s where a large product reaches 1191; a tile of a wave is some 410 slots (32 products, 34 of four slots) and 1024 cycles of the matrix cores, and takes 2560.  Left out in
// turn, in the form before the loop was cleared of copies of registers (195 us a call), exponentials saved 2 us, taking codes apart 12, all products 36.  What did not help: the next tile's scores beside a tile's exponentials (5 to 10 % slower, at 256 registers), waves'
// priorities, four waves a unit more at 128 registers (spills, 60 % slower).  fp32 rows of heads above 128 keep 55 to 63 registers of a lane in memory.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "cache_attend.h"
#include "last_in.h"

using namespace bild;

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kThreads = 256, kKeys = 64, kUnits = 256;
constexpr int kAhead = 4;  // operands of the scores' products that are asked for before the first of them
constexpr int kSplitLeast = 4;  // tiles of keys that a workgroup has at least

__device__ __forceinline__ f32x16 mma(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float max_xor32(float v) {
    uint32_t a, b;
    pair_xor32(__float_as_uint(v), a, b);
    return fmaxf(__uint_as_float(a), __uint_as_float(b));
}

// PAGES: pages of a tile of keys.
template <class R, int DP, int PAGES>
__global__ __launch_bounds__(kThreads, R::kDtype == BILD_DT_F32 || DP == 256 ? 1 : 2) void cache_prompt_kernel(const AttendArgs a) {
    constexpr bool TWO = R::kDtype == BILD_DT_F32;
    constexpr int TERMS = TWO ? 2 : 1, QS = DP / 16, ND = DP / 32, KC = DP / 64, VI = (DP + 127) / 128;
    constexpr bool SOME = VI * kThreads > 2 * DP;  // of the threads have values on their way
    constexpr int kBuffer = 2 * kKeys * DP;  // fp16 values of a tile's keys and values
    typedef typename R::type V;
    extern __shared__ __attribute__((aligned(16))) _Float16 lds[];  // two buffers: keys [64][DP], values [DP][64]
    const CacheView& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n32 = lane & 31, half = lane >> 5, d = c.d_head;
    __shared__ unsigned share;
    const int head = blockIdx.x % c.heads;  // (dies take workgroups in turn: those of a head have its keys in few L2s)
    // ---- which tile of which sequence, and which piece of its keys.  Places are in the order of sequences, rows and keys; the last rows, which see most, come first, those that come second to
    // the compute units the other way round, so that who has much to do shares its unit with who has little (us, call: 200 rows of 4 heads behind 4000 positions, 8 key heads 52 / 47).
    const auto place_of = [&](int places) {
        const int round = max(kUnits / c.heads, 1), nth = (int)(blockIdx.x / c.heads);
        return places - 1 - (nth >= round && nth < 2 * round ? round + min(places, 2 * round) - 1 - nth : nth);
    };
    int s, first, count, tile, length, split, pieces, part_at, flag_at;
    if (a.r.n <= 64) {
        // a lane a sequence: its tiles, the keys of one, and as many pieces of these as its share of the whole work is, of kPromptParts at most
        int mine_s = a.r.sequence(min(lane, a.r.n - 1), c.sequences), mine_first, mine_count;
        a.r.span(min(lane, a.r.n - 1), mine_first, mine_count);
        const int mine_rows = mine_count * a.group;
        int mine_tiles = lane < a.r.n && mine_s >= 0 && mine_rows >= a.prompt_from ? (mine_rows - 1) / kPromptRows + 1 : 0;
        const int mine_length = mine_s < 0 ? 0 : min(max(c.lengths[mine_s], 0), c.cap());
        int keys = (mine_length + kKeys - 1) / kKeys;
        if (a.window) keys = (int)min((int64_t)keys, ((int64_t)a.sinks + kKeys - 1) / kKeys + ((int64_t)a.window + kPromptRows / a.group) / kKeys + 2);
        const float work = wave_sum((float)mine_tiles * (float)keys);
        const int mine_pieces = min((int)((float)keys * (0.999f * kPromptParts / c.heads) / fmaxf(work, 1.f)), min(kMaxSplits, keys / kSplitLeast));
        // One sequence whose first tiles see few keys and whose last ones see many: the last ones, which have at least two shares, are cut into `high` pieces (us, call: 2500 rows of 8 heads of an
        // empty cache, 2 key heads 75 / 66).
        int low_tiles = mine_tiles, high = 0;
        if (a.r.n == 1 && a.causal && !a.window && mine_pieces <= 1 && mine_tiles > 0) {
            const int seen = max(mine_length - mine_count + min(kPromptRows, mine_rows) / a.group, 0) / kKeys + 1;  // tiles of keys that the first rows see
            const float share = fmaxf((float)mine_tiles * 0.5f * (float)(seen + keys) * (float)c.heads / kPromptParts, (float)kSplitLeast);
            high = min((int)((float)keys / share), kMaxSplits);
            if (high > 1 && keys > seen) {
                low_tiles = min(max((int)ceilf((float)mine_tiles * (2.f * share - (float)seen) / (float)(keys - seen)), 0), mine_tiles);
                low_tiles = max(low_tiles, mine_tiles - max(kPromptParts / c.heads - mine_tiles, 0) / (high - 1));  // (no more places than the launch has, and parts)
            }
        }
        if (lane == 0 && low_tiles < mine_tiles) mine_tiles = low_tiles + (mine_tiles - low_tiles) * high;  // (from here on: places)
        const int mine = max(mine_pieces, 1) * mine_tiles, parts = mine_pieces > 1 ? mine : 0, flags = mine_pieces > 1 ? mine_tiles : 0;
        const int upto = prefix_sum(mine), parts_upto = prefix_sum(parts), flags_upto = prefix_sum(flags), places = __builtin_amdgcn_readlane(upto, 63);
        if ((int)(blockIdx.x / c.heads) >= places) return;
        const int place = place_of(places), at = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(__ballot(place < upto))), local = place - __builtin_amdgcn_readlane(upto - mine, at);
        pieces = max(__builtin_amdgcn_readlane(mine_pieces, at), 1);
        tile = local / pieces;
        split = local - tile * pieces;
        part_at = __builtin_amdgcn_readlane(parts_upto - parts, at) + local - split;
        flag_at = __builtin_amdgcn_readlane(flags_upto - flags, at) + tile;
        low_tiles = __builtin_amdgcn_readlane(low_tiles, 0);
        if (a.r.n == 1 && place >= low_tiles && __builtin_amdgcn_readlane(mine_tiles, 0) > low_tiles) {
            pieces = __builtin_amdgcn_readlane(high, 0);
            flag_at = (place - low_tiles) / pieces;
            split = place - low_tiles - flag_at * pieces;
            part_at = flag_at * pieces;
            tile = low_tiles + flag_at;
        }
        s = __builtin_amdgcn_readlane(mine_s, at);
        first = __builtin_amdgcn_readlane(mine_first, at);
        count = __builtin_amdgcn_readlane(mine_count, at);
        length = __builtin_amdgcn_readlane(mine_length, at);
    } else {
        // entry i of the list has the slots floor(first row * group / 128) + i and those behind, as many as it can have tiles
        const int place = place_of((int)(gridDim.x / c.heads)), slot = place / a.splits;
        int i;
        pieces = a.splits;
        split = place - slot * pieces;
        flag_at = slot;
        part_at = slot * pieces;
        if (a.r.starts) {
            int lo = 0, hi = a.r.n;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                a.r.span(mid, first, count);
                if ((int)((int64_t)first * a.group / kPromptRows) + mid <= slot) lo = mid; else hi = mid;
            }
            i = lo;
            a.r.span(i, first, count);
            tile = slot - (int)((int64_t)first * a.group / kPromptRows) - i;
        } else {
            const int per = (int)(((int64_t)a.r.rows * a.group + kPromptRows - 1) / kPromptRows);
            i = slot / per;
            tile = slot - i * per;
            a.r.span(i, first, count);
        }
        if (tile < 0 || tile * kPromptRows >= count * a.group || count * a.group < a.prompt_from) return;
        s = a.r.sequence(i, c.sequences);
        if (s < 0) return;
        length = min(max(c.lengths[s], 0), c.cap());
    }
    const int rows = count * a.group;
    const int idx0 = tile * kPromptRows + wave * 32, idx = min(idx0 + n32, rows - 1), j = idx / a.group, e = idx - j * a.group;
    const auto pos_of = [&](int at) { return a.causal ? max(length - count + at, -1) : length - 1; };  // (see Seq::position)
    const int pos = pos_of(j), low = a.window ? pos - a.window : -1;
    // ---- the keys that any row of the tile sees, in tiles
    const int wg_first = pos_of(tile * kPromptRows / a.group), wg_last = pos_of(min(tile * kPromptRows + kPromptRows - 1, rows - 1) / a.group);
    const int low_tile = a.window ? max(wg_first - a.window + 1, 0) / kKeys : 0;
    const int sink_tiles = a.window ? min((int)(((int64_t)a.sinks + kKeys - 1) / kKeys), low_tile) : 0;
    const int all_tiles = sink_tiles + max((min(wg_last + 1, length) + kKeys - 1) / kKeys - low_tile, 0);
    // (the first rows of a sequence may see too few keys for as many pieces)
    const int splits = min(pieces, max(all_tiles / kSplitLeast, 1));
    if (split >= splits) return;
    const int t0 = all_tiles * split / splits, tiles = all_tiles * (split + 1) / splits;
    const auto tile_at = [&](int t) { return t < sink_tiles ? t : t - sink_tiles + low_tile; };
    // (of the wave's rows)
    const int first_pos = pos_of(min(idx0, rows - 1) / a.group), last_pos = pos_of(min(idx0 + 31, rows - 1) / a.group);

    // ---- pages and scales of the next 64 tiles, a lane a tile
    int pages[PAGES];
    uint32_t where[PAGES][2];  // of the keys' codes
    float k_scale[PAGES], v_scale[PAGES];
    const auto look_up = [&](int t0) {
        const int t = t0 + lane, key0 = tile_at(t) * kKeys;
#pragma unroll
        for (int p = 0; p < PAGES; ++p) {
            const int k0 = key0 + p * kBlock;
            pages[p] = -1;
            k_scale[p] = v_scale[p] = 0.f;
            if (t < tiles && k0 < length) pages[p] = c.table[(int64_t)s * c.max_pages + (k0 >> c.page_shift)];
            if (!c.has(pages[p])) pages[p] = -1;
            // (a page that is not there: any that is in the pool, and no weight)
            const uint64_t at = (uint64_t)(c.codes + c.plane(max(pages[p], 0), a.layer, 0, head) * c.plane_bytes() + (k0 & (c.page_tokens - 1)) * d);
            where[p][0] = (uint32_t)at;
            where[p][1] = (uint32_t)(at >> 32);
            if (pages[p] >= 0) {
                k_scale[p] = c.scales[c.plane(pages[p], a.layer, 0, head)];
                v_scale[p] = c.scales[c.plane(pages[p], a.layer, 1, head)] * (512.f / 127.f);
            }
        }
    };
    look_up(t0);
    // ---- rows
    f16x8 q[TERMS][QS];
    float row_scale;
    {
        const V* x = (const V*)a.q + (int64_t)(first + j) * a.q_token + (int64_t)(head * a.group + e) * a.q_head;
        RowVec<R, 8> raw[QS];
        float big = 0.f;
#pragma unroll
        for (int t = 0; t < QS; ++t) {
            const int begin = 16 * t + 8 * half;
            raw[t].load(x + min(begin, d - 8));
#pragma unroll
            for (int u = 0; u < 8; ++u) big = fmaxf(big, begin < d ? fabsf(R::up(raw[t].v[u])) : 0.f);
        }
        big = max_xor32(big);
        const int up = up_of(big);
        row_scale = ldexpf(fabsf(a.scale), -up);
#pragma unroll
        for (int t = 0; t < QS; ++t)
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                // (the scale's sign goes into the rows: what scores are multiplied by is not negative)
                const float y = 16 * t + 8 * half < d ? ldexpf(R::up(raw[t].v[u]), up) : 0.f, v = a.scale < 0.f ? -y : y;
                q[0][t][u] = (_Float16)v;
                if (TWO) q[TERMS - 1][t][u] = (_Float16)(v - (float)q[0][t][u]);
            }
    }

    // ---- codes on their way from memory to LDS: where a thread's pieces lie in a page, and (the same for a wave) which page of a tile they are of
    u32x4 kc[KC];
    uint32_t vc[VI][8];
    int k_off[KC], v_off[VI];
#pragma unroll
    for (int u = 0; u < KC; ++u) {
        const int item = u * kThreads + tid, key = item / (DP / 16), ch = item % (DP / 16);
        k_off[u] = (PAGES == 2 ? key & (kBlock - 1) : key) * d + min(16 * ch, d - 16);
    }
#pragma unroll
    for (int u = 0; u < VI; ++u) {
        const int item = u * kThreads + tid, group = item / (DP / 4), dg = item % (DP / 4), k0 = 16 * (group >> 1) + 4 * (group & 1);
        v_off[u] = (PAGES == 2 ? k0 & (kBlock - 1) : k0) * d + min(4 * dg, d - 4);
    }
    const int64_t to_v = (int64_t)c.heads * c.plane_bytes();
    const auto request = [&](int t) {  // (looked up)
        const auto plane = [&](int which, int half_of) {
            const uint64_t lo = (uint32_t)__builtin_amdgcn_readlane((int)where[half_of][0], (t - t0) & 63), hi = (uint32_t)__builtin_amdgcn_readlane((int)where[half_of][1], (t - t0) & 63);
            return make_rsrc((const int8_t*)(hi << 32 | lo) + (which ? to_v : 0), (size_t)(kKeys / PAGES * d));
        };
#pragma unroll
        for (int u = 0; u < KC; ++u) {
            const int first_key = (u * kThreads + wave * 64) / (DP / 16);
            kc[u] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(plane(0, PAGES == 2 && first_key >= kBlock ? PAGES - 1 : 0), k_off[u], 0, 0));
        }
#pragma unroll
        for (int u = 0; u < VI; ++u) {
            const int first_group = (u * kThreads + wave * 64) / (DP / 4);
            if (SOME && first_group >= 8) continue;
            const auto from = plane(1, PAGES == 2 && first_group >= 4 ? PAGES - 1 : 0);
#pragma unroll
            for (int y = 0; y < 8; ++y) vc[u][y] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(from, v_off[u], ((y & 3) + 8 * (y >> 2)) * d, 0);
        }
    };
    const auto k_at = [&](int key, int ch) { return key * DP + 8 * (ch ^ (DP == 64 ? (key >> 1) & 7 : key & 15)); };
    const auto v_at = [&](int dim, int ch) { return kKeys * DP + dim * kKeys + 8 * (ch ^ ((dim >> 1) & 7)); };
    const auto deliver = [&](int buffer) {
        _Float16* to = lds + buffer * kBuffer;
#pragma unroll
        for (int u = 0; u < KC; ++u) {
            const int item = u * kThreads + tid, key = item / (DP / 16), ch = item % (DP / 16);
            const u32x4 y = kc[u] ^ 0x80808080u;
            const bool cut = 16 * ch > d - 16;  // (a last piece that is half as long begins earlier: what belongs in its place is its second half)
            *(f16x8*)(to + k_at(key, 2 * ch)) = eight_of(cut ? y[2] : y[0], cut ? y[3] : y[1]);
            *(f16x8*)(to + k_at(key, 2 * ch + 1)) = eight_of(y[2], y[3]);
        }
#pragma unroll
        for (int u = 0; u < VI; ++u) {
            const int item = u * kThreads + tid, group = item / (DP / 4), dg = item % (DP / 4);
            if (SOME && group >= 8) continue;
            uint32_t y[8];
#pragma unroll
            for (int z = 0; z < 8; ++z) y[z] = vc[u][z] ^ 0x80808080u;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                *(f16x8*)(to + v_at(4 * dg + k, group)) = eight(pair_of(y[0], y[1], k), pair_of(y[2], y[3], k), pair_of(y[4], y[5], k), pair_of(y[6], y[7], k));
        }
    };

    float top = -INFINITY, sum = 0.f, unit = 0.f, per_unit = 0.f, most_v = 0.f;  // (the sums over the values are in `unit`s)
    f32x16 acc[ND];
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[t][r] = 0.f;
    if (t0 < tiles) {
        request(t0);
        deliver(t0 & 1);
    }
    lds_barrier();
    for (int t = t0; t < tiles; ++t) {
        const int key0 = tile_at(t) * kKeys;
        bool there[PAGES];
        float ks[PAGES], vs[PAGES];
#pragma unroll
        for (int p = 0; p < PAGES; ++p) {
            there[p] = __builtin_amdgcn_readlane(pages[p], (t - t0) & 63) >= 0;
            ks[p] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k_scale[p]), (t - t0) & 63));
            vs[p] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v_scale[p]), (t - t0) & 63));
        }
        if (t + 1 < tiles) {
            if (((t + 1 - t0) & 63) == 0) look_up(t + 1);
            request(t + 1);
        }
        __builtin_amdgcn_sched_barrier(0);
        const _Float16* at = lds + (t & 1) * kBuffer;
        const bool seen = key0 <= last_pos && (!a.window || key0 + kKeys - 1 > first_pos - a.window || key0 < a.sinks) && (there[0] || there[PAGES - 1]);
        if (seen) {
            float part, part_log;
            const auto scale_of = [&](int p) {
                // a page's scale goes into its weights, relative to a power of two that the sums are kept in units of
                const float v = vs[p];
                if (__builtin_amdgcn_readfirstlane(v > unit || (v > 0.f && v < unit * 0.0625f))) {
                    most_v = fmaxf(most_v, v);
                    const float now = fmaxf(__uint_as_float((__float_as_uint(v) + 0x7FFFFFu) & 0x7F800000u), most_v * 8.27180613e-25f), less = unit / now;
#pragma unroll
                    for (int u = 0; u < ND; ++u)
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[u][r] *= less;
                    unit = now;
                    per_unit = 1.f / now;
                }
                // (not below 2^-60: there its values count for nothing in fp16, but the sum of the weights is taken from the same numbers)
                part = fmaxf(v * per_unit, 8.67361738e-19f);
                part_log = __builtin_amdgcn_logf(part);
            };
            scale_of(0);
            // (what scores are multiplied by is not 0, so that hidden ones stay -infinity: where it would be, the scores are 0)
            const float by[2] = {fmaxf(ks[0] * row_scale, 1.17549435e-38f), fmaxf(ks[PAGES - 1] * row_scale, 1.17549435e-38f)};
            const bool full = key0 + kKeys - 1 <= first_pos && (!a.window || key0 > last_pos - a.window || key0 + kKeys <= a.sinks) && there[0] && there[PAGES - 1];
            // scores begin as -infinity where the row does not see the key
            f32x16 z[2];
            const auto scores = [&] {
#pragma unroll
                for (int u = 0; u < QS; ++u)
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        const f16x8 k = *(const f16x8*)(at + k_at(32 * m + n32, 2 * u + half));
#pragma unroll
                        for (int w = 0; w < TERMS; ++w) z[m] = mma(k, q[w][u], z[m]);
                    }
                // (the next products' operands come from LDS while these run)
                __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
                for (int u = 0; u < 2 * QS - kAhead; ++u) {
                    __builtin_amdgcn_sched_group_barrier(0x8, TERMS, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x8, kAhead * TERMS, 0);
            };
            if (full) {
                z[0] = z[1] = f32x16{};
                scores();
            } else {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int key = key0 + 32 * m + 8 * (r >> 2) + 4 * half + (r & 3);
                        z[m][r] = (key <= pos) & ((key > low) | (key < a.sinks)) & there[m * (PAGES - 1)] ? 0.f : -INFINITY;
                    }
                }
                scores();
            }
            float big = -INFINITY;
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                float most = z[m][0];
#pragma unroll
                for (int r = 1; r < 16; ++r) most = fmaxf(most, z[m][r]);
                big = fmaxf(big, most * by[m]);
            }
            big = max_xor32(big);
            if (__any(big > top + kSlack)) {
                const float now = big > top + kSlack ? big : top, less = now == top ? 1.f : __builtin_amdgcn_exp2f(top - now);
                sum *= less;
#pragma unroll
                for (int u = 0; u < ND; ++u)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[u][r] *= less;
                top = now;
            }
            const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int p = 0; p < PAGES; ++p) {
                if (p) scale_of(p);
                const float off = part_log - base;
                constexpr int ST = 4 / PAGES;
                f16x8 w[TERMS][ST];
                float sums[2] = {0.f, 0.f};
#pragma unroll
                for (int st = 0; st < ST; ++st) {
                    const int m = (p * ST + st) >> 1;
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(z[m][8 * (st & 1) + u], by[m], off));
                        sums[u & 1] += e;
                        w[0][st][u] = (_Float16)e;
                        if (TWO) w[TERMS - 1][st][u] = (_Float16)(e - (float)w[0][st][u]);
                    }
                }
                sum = __builtin_fmaf(sums[0] + sums[1], __builtin_amdgcn_rcpf(part), sum);
#pragma unroll
                for (int st = 0; st < ST; ++st)
#pragma unroll
                    for (int u = 0; u < ND; ++u) {
                        const f16x8 y = *(const f16x8*)(at + v_at(32 * u + n32, 2 * (p * ST + st) + half));
#pragma unroll
                        for (int x = 0; x < TERMS; ++x) acc[u] = mma(y, w[x][st], acc[u]);
                    }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (t + 1 < tiles) deliver((t + 1) & 1);
        lds_barrier();
    }
    // ---- results
    uint32_t x, y;
    pair_xor32(__float_as_uint(sum), x, y);
    sum = __uint_as_float(x) + __uint_as_float(y);
#pragma unroll
    for (int u = 0; u < ND; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[u][r] *= unit;
    if (splits > 1) {
        // a lane's values lie in memory as it has them, 1 KiB a store of a wave: the last of the tile's workgroups has the same lanes
        constexpr int kPart = kPromptRows * (DP + 4);  // floats: see prompt_part_floats
        const auto place = [&](int sp) { return make_rsrc(a.part + ((int64_t)(part_at + sp) * c.heads + head) * kPart, sizeof(float) * kPart); };
        const auto mine = place(split);
#pragma unroll
        for (int u = 0; u < ND; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(acc[u][4 * r]), __float_as_uint(acc[u][4 * r + 1]), __float_as_uint(acc[u][4 * r + 2]), __float_as_uint(acc[u][4 * r + 3])},
                                                       mine, (((wave * ND + u) * 4 + r) * 64 + lane) * 16, 0, kPartAux);
        if (half == 0) __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(top), __float_as_uint(sum)}, mine, (kPromptRows * DP + 2 * (wave * 32 + n32)) * 4, 0, kPartAux);
        if (!last_in(a.arrived + (int64_t)flag_at * c.heads + head, (unsigned)splits, &share)) return;
        float m = -INFINITY, l = 0.f;
        for (int sp = 0; sp < splits; ++sp) {
            const auto ml = __builtin_amdgcn_raw_buffer_load_b64(place(sp), (kPromptRows * DP + 2 * (wave * 32 + n32)) * 4, 0, kPartAux);
            m = fmaxf(m, __uint_as_float(ml[0]));
        }
        const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int u = 0; u < ND; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[u][r] = 0.f;
        for (int sp = 0; sp < splits; ++sp) {
            const auto from = place(sp);
            const auto ml = __builtin_amdgcn_raw_buffer_load_b64(from, (kPromptRows * DP + 2 * (wave * 32 + n32)) * 4, 0, kPartAux);
            const float by = __builtin_amdgcn_exp2f(__uint_as_float(ml[0]) - base);
            l = __builtin_fmaf(__uint_as_float(ml[1]), by, l);
#pragma unroll
            for (int u = 0; u < ND; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const auto o = __builtin_amdgcn_raw_buffer_load_b128(from, (((wave * ND + u) * 4 + r) * 64 + lane) * 16, 0, kPartAux);
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[u][4 * r + k] = __builtin_fmaf(__uint_as_float(o[k]), by, acc[u][4 * r + k]);
                }
        }
        top = m;
        sum = l;
    }
    if (idx0 + n32 >= rows) return;
    const float by = sum == 0.f ? 0.f : 1.f / sum;
    const int h = head * a.group + e;
    V* out = (V*)a.out + (int64_t)(first + j) * a.out_token + (int64_t)h * a.out_head;
#pragma unroll
    for (int u = 0; u < ND; ++u)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int dim = 32 * u + 2 * r + 4 * half;
            RowVec<R, 4> o;
#pragma unroll
            for (int k = 0; k < 4; ++k) o.v[k] = R::down(acc[u][r + k] * by);
            if (dim < d) o.store(out + dim);
        }
    if (a.lse && half == 0) a.lse[(int64_t)(first + j) * a.heads + h] = sum == 0.f ? -INFINITY : top * kLn2 + logf(sum);
}

constexpr size_t lds_bytes(int DP) { return (size_t)2 * 2 * kKeys * DP * 2; }

template <class R, int DP>
hipError_t launch(const AttendArgs& a, dim3 grid, hipStream_t st) {
    return a.c.page_tokens == 32 ? launch_on(cache_prompt_kernel<R, DP, 2>, grid, dim3(kThreads), lds_bytes(DP), st, a)
                                 : launch_on(cache_prompt_kernel<R, DP, 1>, grid, dim3(kThreads), lds_bytes(DP), st, a);
}
template <class R>
hipError_t launch(const AttendArgs& a, dim3 grid, hipStream_t st) {
    return a.c.d_head <= 64 ? launch<R, 64>(a, grid, st) : a.c.d_head <= 128 ? launch<R, 128>(a, grid, st) : launch<R, 256>(a, grid, st);
}

}  // namespace

namespace bild {

hipError_t cache_prompt_init(int d_head) {
    const void* const half[] = {(const void*)cache_prompt_kernel<RowF32, 128, 1>, (const void*)cache_prompt_kernel<RowBf16, 128, 1>, (const void*)cache_prompt_kernel<RowF16, 128, 1>,
                                (const void*)cache_prompt_kernel<RowF32, 128, 2>, (const void*)cache_prompt_kernel<RowBf16, 128, 2>, (const void*)cache_prompt_kernel<RowF16, 128, 2>};
    const void* const full[] = {(const void*)cache_prompt_kernel<RowF32, 256, 1>, (const void*)cache_prompt_kernel<RowBf16, 256, 1>, (const void*)cache_prompt_kernel<RowF16, 256, 1>,
                                (const void*)cache_prompt_kernel<RowF32, 256, 2>, (const void*)cache_prompt_kernel<RowBf16, 256, 2>, (const void*)cache_prompt_kernel<RowF16, 256, 2>};
    return d_head <= 64 ? hipSuccess : d_head <= 128 ? raise_lds_limit(half, (int)lds_bytes(128)) : raise_lds_limit(full, (int)lds_bytes(256));
}

size_t prompt_part_floats(int d_head) { return (size_t)kPromptParts * kPromptRows * ((d_head <= 64 ? 64 : d_head <= 128 ? 128 : 256) + 4); }

hipError_t launch_cache_prompt(const AttendArgs& a, int dtype, int64_t places, hipStream_t st) {
    const dim3 grid((unsigned)(a.c.heads * places));
    return dtype == BILD_DT_F32 ? launch<RowF32>(a, grid, st) : dtype == BILD_DT_BF16 ? launch<RowBf16>(a, grid, st) : launch<RowF16>(a, grid, st);
}

}  // namespace bild
