// A cache of keys and values in 8 bits, in pages that sequences share: its pages (bild_cache_extend, _fork, _compact) and what is written into them
// (bild_cache_append).  Attention over it: cache_attend.hip.
//
// Tables, lengths and counts of holders live in device memory and are changed there, so that a beam's parents never come to the host.  Who gets which page is a
// matter of order (lowest free page first, in the order of the list); one workgroup settles it with prefix sums, so that it is the same every time.  Counts are whole
// numbers: the order of the atomics shows nowhere.
// Bound: pages that are copied, by memory, 16 bytes a lane; appending, by the reads of the rows; the rest by launches and a few dependent loads.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "cache.h"
#include "rows_common.h"

using namespace bild;

namespace {

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;
// 2^90: sums over 2^30 values in fp32, times weights of up to 2^8 and the scales of codes (2^2) and weights, stay below its largest
constexpr float kLimit = 1.2379400392853803e27f;

// Words of a handle that kernels hand on.
enum : int { W_FITS = 0, W_COPIES, W_USED, W_MOVES, W_COUNT = 16 };

struct ExtendArgs {
    CacheView c;
    CacheRows r;
    const int* cut;
    int* granted;
    int window, sinks;     // (0: nothing is given back behind a window)
    int pieces;            // of a table, each looked through by a wave (see slide)
    int *plan;             // [sequences][4], 16-byte aligned: entries
    int *fresh;            // [pages]: the free pages that are given away, lowest first
    int *asked, *latest;   // [pages], zero between launches: how many of a shared page's holders want to write into it, the last of these + 1
    int* copies;           // [sequences][3]: from, to, positions
    int* words;
};

// Entry i of a list: its sequence, length after the cut, new rows, pages needed before it in the list, shared page that has to be copied (-1: none).
struct Entry {
    int keep, add, before, shared, s;
};

__device__ __forceinline__ int seen(const int* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Exclusive prefix sum over a workgroup of kPlanThreads, and the sum of all; values up to kMany, and sums beyond that are only known to be beyond.
constexpr int kMany = kMaxLimit + 1;
__device__ __forceinline__ int scan(int v, int& total, int* sums) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o, 64);
        if (lane >= o) x = min(x + y, kMany);
    }
    __syncthreads();  // (of the last call's sums)
    if (lane == 63) sums[wave] = x;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) {
        before += w < wave ? sums[w] : 0;
        total += sums[w];
    }
    return before + x - v;
}

// Pages [from, to) of a sequence are given back, by the whole wave, EACH x 64 entries at a time.  Whether there were any.
template <int EACH>
__device__ __forceinline__ bool give_back(const CacheView& c, int64_t row, int from, int to) {
    const int lane = threadIdx.x & 63;
    bool any = false;
    for (int b0 = from; b0 < to; b0 += 64 * EACH) {
        int p[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const int b = b0 + 64 * e + lane;
            p[e] = b < to ? c.table[row + b] : -1;
        }
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            if (p[e] != -1) c.table[row + b0 + 64 * e + lane] = -1;
            if (c.has(p[e])) atomicSub(&c.refs[p[e]], 1);
            any |= p[e] != -1;
        }
    }
    return any;
}

// Positions that entry i's sequence s keeps.
__device__ __forceinline__ int kept(const ExtendArgs& a, int i, int s) {
    const int length = min(max(a.c.lengths[s], 0), a.c.cap());
    return a.cut ? min(max(a.cut[i], 0), length) : length;
}

// What the window of entry u / pieces has left behind, in piece u % pieces of its table, is given back, by the whole wave.  All of it is looked through each time: calls with fewer sinks or
// another window than those before leave pages anywhere in it, and nothing but the table, which is the caller's, says where.
constexpr int kSlideEach = 8;
__device__ __forceinline__ bool slide(const ExtendArgs& a, int u, int pieces) {
    const CacheView& c = a.c;
    const int i = u / pieces, from = (u - i * pieces) * 64 * kSlideEach, s = a.r.sequence(i, c.sequences);
    if (s < 0) return false;
    const int end = max(kept(a, i, s) - a.window + 1, 0) >> c.page_shift, sinks = (int)(((int64_t)a.sinks + c.page_tokens - 1) >> c.page_shift);
    return give_back<kSlideEach>(c, (int64_t)s * c.max_pages, max(from, sinks), min(from + 64 * kSlideEach, end));
}

// One workgroup, as who gets which page is a matter of order: needs are summed over the list, free pages over the pool, both by prefix sums.  Bound: launch and a chain of loads - length, table, count of
// holders - between barriers: 4 beams 6.5 us, 32 beams 8.2.
__global__ __launch_bounds__(kPlanThreads) void cache_extend_kernel(const ExtendArgs a) {
    __shared__ int sums[kPlanWaves];
    __shared__ int wrong, freed;
    __shared__ int given[kPlanThreads];  // the first of the pages that are given away
    const CacheView& c = a.c;
    const int tid = threadIdx.x, lane = tid & 63, n = a.r.n, shift = c.page_shift, mask = c.page_tokens - 1;
    const bool few = n <= 64;  // (a wave has them all)
    if (tid == 0) wrong = freed = 0;
    int counts[8];  // of the pool's first pages, asked for before it is known that they are needed
#pragma unroll
    for (int e = 0; e < 8; ++e) counts[e] = 8 * tid + e < c.pages ? seen(&c.refs[8 * tid + e]) : 1;
    __syncthreads();
    if (a.window > 0)
        for (int u = tid >> 6; u < n * a.pieces; u += kPlanWaves)
            if (slide(a, u, a.pieces)) freed = 1;
    // (a thread's first entry stays in registers, further ones of long lists go through memory)
    Entry mine = {0, 0, 0, -1, -1};
    const auto entry = [&](int i) {
        if (i < kPlanThreads) return mine;
        const int4 q = *(const int4*)(a.plan + 4 * (int64_t)i);
        return Entry{q.x, q.y, q.z, q.w, a.r.sequence(i, c.sequences)};
    };
    const auto put = [&](int i, const Entry& q) {
        if (i < kPlanThreads) mine = q;
        else *(int4*)(a.plan + 4 * (int64_t)i) = make_int4(q.keep, q.add, q.before, q.shared);
    };
    // the cut
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
        const int i = i0 + tid, s = i < n ? a.r.sequence(i, c.sequences) : -1;
        int length = 0, keep = 0, add = 0;
        if (s >= 0) {
            int first;
            length = min(max(c.lengths[s], 0), c.cap());
            keep = kept(a, i, s);
            if (a.r.starts) {
                first = a.r.starts[i];
                add = (int)min(max((int64_t)a.r.starts[i + 1] - first, (int64_t)0), (int64_t)c.cap() + 1);
            } else {
                add = a.r.rows;
            }
            if (keep != length) c.lengths[s] = keep;
        }
        if (i < n) put(i, {keep, s >= 0 ? add : 0, 0, -1, s});
        const int cut0 = (keep + mask) >> shift, cut1 = (length + mask) >> shift;
        if (cut1 > cut0) freed = 1;
        for (unsigned long long todo = __ballot(cut1 > cut0); todo; todo &= todo - 1) {
            const int l = (int)__builtin_ctzll(todo);
            give_back<1>(c, (int64_t)__shfl(s, l, 64) * c.max_pages, __shfl(cut0, l, 64), __shfl(cut1, l, 64));
        }
    }
    __syncthreads();
    // pages that are shared and would be written
    for (int i = tid; i < n; i += kPlanThreads) {
        Entry q = entry(i);
        const int s = q.s, keep = q.keep, add = q.add;
        int shared = -1;
        if (s >= 0 && add > 0) {
            if ((int64_t)keep + add > c.cap()) wrong = 1;
            if (keep & mask) {
                const int p = c.table[(int64_t)s * c.max_pages + (keep >> shift)];
                if (!c.has(p)) {
                    wrong = 1;
                } else {
                    const int holders = seen(&c.refs[p]);
                    if (holders > 1) shared = p;
                    if (few) {
                        // (all lanes that have rows are here)
                        int asked = 0, latest = -1;
                        for (unsigned long long others = __ballot(holders > 1); others; others &= others - 1) {
                            const int l = (int)__builtin_ctzll(others);
                            if (__builtin_amdgcn_readlane(p, l) == p) {
                                ++asked;
                                latest = l;
                            }
                        }
                        if (shared >= 0 && asked == holders && latest == lane) shared = -1;
                    } else if (shared >= 0) {
                        atomicAdd(&a.asked[p], 1);
                        atomicMax(&a.latest[p], i + 1);
                    }
                }
            }
        }
        q.shared = shared;
        put(i, q);
    }
    __threadfence_block();
    __syncthreads();
    int needed = 0;
    const bool fits_so_far = !wrong;
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
        const int i = i0 + tid;
        int need = 0;
        Entry q = {0, 0, 0, -1, -1};
        if (i < n) {
            q = entry(i);
            const int keep = q.keep, add = q.add, p = q.shared;
            if (fits_so_far) need = min(((keep + add + mask) >> shift) - ((keep + mask) >> shift), kMany - 1);
            if (p >= 0) {
                if (!few && seen(&a.asked[p]) == seen(&c.refs[p]) && seen(&a.latest[p]) == i + 1) q.shared = -1;  // (the others get copies)
                else ++need;
            }
        }
        int all;
        const int before = scan(need, all, sums);
        q.before = needed + before;
        if (i < n) put(i, q);
        needed = min(needed + all, kMany);
    }
    __syncthreads();
    for (int i = few ? n : tid; i < n; i += kPlanThreads) {  // (those that keep theirs as well: the count is of all)
        const Entry q = entry(i);
        if (q.s < 0 || q.add <= 0 || !(q.keep & mask)) continue;
        const int p = c.table[(int64_t)q.s * c.max_pages + (q.keep >> shift)];
        if (c.has(p)) a.asked[p] = a.latest[p] = 0;
    }
    // the free pages, lowest first
    bool fits = fits_so_far && needed <= c.pages;
    if (fits && needed > 0) {
        int found = 0;
        for (int p0 = 0; p0 < c.pages && found < needed; p0 += 8 * kPlanThreads) {
            int r[8], mine = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int p = p0 + 8 * tid + e;
                r[e] = p0 == 0 && !freed ? counts[e] : p < c.pages ? seen(&c.refs[p]) : 1;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) mine += r[e] == 0;
            int all, at = scan(mine, all, sums);
            at += found;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (r[e] == 0) {
                    if (at < kPlanThreads) given[at] = p0 + 8 * tid + e;
                    else if (at < needed) a.fresh[at] = p0 + 8 * tid + e;
                    ++at;
                }
            found += all;
        }
        fits = found >= needed;
    }
    __threadfence_block();
    __syncthreads();
    // they are handed out
    int copies = 0;
    for (int i0 = 0; fits && i0 < n; i0 += kPlanThreads) {
        const int i = i0 + tid;
        Entry q = {0, 0, 0, -1, -1};
        if (i < n) q = entry(i);
        const int s = q.s, keep = q.keep, add = q.add, old = s >= 0 ? q.shared : -1;
        int at = q.before;
        int all;
        const int place = scan(old >= 0, all, sums);
        if (old >= 0) {
            const int p = at < kPlanThreads ? given[at] : a.fresh[at];
            ++at;
            c.table[(int64_t)s * c.max_pages + (keep >> shift)] = p;
            atomicSub(&c.refs[old], 1);
            c.refs[p] = 1;
            int* copy = a.copies + 3 * (copies + place);
            copy[0] = old;
            copy[1] = p;
            copy[2] = keep & mask;
        }
        copies += all;
        if (s >= 0 && add > 0) c.lengths[s] = keep + add;
        const int b0 = (keep + mask) >> shift, b1 = add > 0 ? (keep + add + mask) >> shift : b0;
        for (unsigned long long todo = __ballot(b1 > b0); todo; todo &= todo - 1) {
            const int l = (int)__builtin_ctzll(todo);
            const int64_t row = (int64_t)__shfl(s, l, 64) * c.max_pages;
            const int f0 = __shfl(b0, l, 64), f1 = __shfl(b1, l, 64), from = __shfl(at, l, 64);
            for (int b = f0 + lane; b < f1; b += 64) {
                const int k = from + b - f0, p = k < kPlanThreads ? given[k] : a.fresh[k];
                c.table[row + b] = p;
                c.refs[p] = 1;
            }
        }
    }
    if (tid == 0) {
        a.words[W_FITS] = fits;
        a.words[W_COPIES] = copies;
        if (a.granted) *a.granted = fits;
    }
}

// The same of long lists and tables, by more than one workgroup, in front of cache_extend_kernel (us, a call, in front of it / in it: one sequence of 200000 positions, pages of 32 9.9 / 8.7; 16 of
// 50001, pages of 64 8.7 / 8.9; 64 of 2000 8.8 / 10.7; 64 of 50001, pages of 32 11.7 / 28.6; 64 of 2^20, pages of 64 41 / 190).
constexpr int kSlideHere = 32, kSlideGroups = 1024;
__global__ __launch_bounds__(256) void cache_slide_kernel(const ExtendArgs a) {
    const int64_t items = (int64_t)a.r.n * a.pieces;
    for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < items; u += (int64_t)gridDim.x * 4) slide(a, (int)u, a.pieces);
}

// The first positions of pages, a wave a layer, half and head (pieces of a few KiB: enough of them for every compute unit).  Bound: memory; 91 MB read and written 20 us, 4.5 TB/s of 5.41.
__global__ __launch_bounds__(256) void cache_copy_kernel(const CacheView c, const int* copies, const int* words) {
    const int lane = threadIdx.x & 63, planes = c.layers * 2 * c.heads, per = c.plane_bytes();
    const int64_t items = (int64_t)words[W_COPIES] * planes;
    for (int64_t u = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); u < items; u += (int64_t)gridDim.x * 4) {
        const int k = (int)(u / planes), plane = (int)(u - (int64_t)k * planes);
        const int64_t from = (int64_t)copies[3 * k] * planes + plane, to = (int64_t)copies[3 * k + 1] * planes + plane;
        const int bytes = copies[3 * k + 2] * c.d_head;  // (a multiple of 8)
        const int8_t* src = c.codes + from * per;
        int8_t* dst = c.codes + to * per;
        for (int b = lane * 16; b + 16 <= bytes; b += 64 * 16) *(uint4*)(dst + b) = *(const uint4*)(src + b);
        if (lane == 0) {
            if (bytes & 8) *(uint2*)(dst + (bytes & ~15)) = *(const uint2*)(src + (bytes & ~15));
            c.scales[to] = c.scales[from];
        }
    }
}

struct ForkArgs {
    CacheView c;
    const int *sequences, *parents;
    int n, group;
    int* rows;  // [sequences][max_pages]: tables on their way
    int* plan;  // [sequences][4]: new length, -1: stays
};

// Large tables: all rows are read before any is written, so in two launches, a workgroup an entry of the list; counts of holders by atomics on whole numbers.
__global__ __launch_bounds__(256) void cache_fork_read_kernel(const ForkArgs a) {
    const CacheView& c = a.c;
    const int i = blockIdx.x;
    const CacheRows r = {a.sequences, nullptr, a.n, 0, 0};
    const int s = r.sequence(i, c.sequences), parent = a.parents[i], first = i / a.group * a.group;
    const int from = (unsigned)parent < (unsigned)a.group && first + parent < a.n ? r.sequence(first + parent, c.sequences) : -1;
    const bool stays = s < 0 || from == s;
    const int length = from < 0 ? 0 : min(max(c.lengths[from], 0), c.cap());
    if (threadIdx.x == 0) a.plan[4 * i] = stays ? -1 : length;
    if (stays) return;
    const int count = (length + c.page_tokens - 1) >> c.page_shift;
    for (int b = threadIdx.x; b < count; b += 256) {
        int p = c.table[(int64_t)from * c.max_pages + b];
        if (!c.has(p)) p = -1;
        else atomicAdd(&c.refs[p], 1);
        a.rows[(int64_t)i * c.max_pages + b] = p;
    }
}

__global__ __launch_bounds__(256) void cache_fork_write_kernel(const ForkArgs a) {
    const CacheView& c = a.c;
    const int i = blockIdx.x, length = a.plan[4 * i];
    if (length < 0) return;
    const CacheRows r = {a.sequences, nullptr, a.n, 0, 0};
    const int s = r.sequence(i, c.sequences);
    if (s < 0) return;
    const int was = min(max(c.lengths[s], 0), c.cap());
    const int before = (was + c.page_tokens - 1) >> c.page_shift, count = (length + c.page_tokens - 1) >> c.page_shift;
    for (int b = threadIdx.x; b < max(before, count); b += 256) {
        int* entry = c.table + (int64_t)s * c.max_pages + b;
        const int old = b < before ? *entry : -1;
        *entry = b < count ? a.rows[(int64_t)i * c.max_pages + b] : -1;
        if (c.has(old)) atomicSub(&c.refs[old], 1);
    }
    __syncthreads();
    if (threadIdx.x == 0) c.lengths[s] = length;
}

// Small tables: both halves in one workgroup, entries in registers between them: one launch, 3.9 us for 4 beams, 6.0 for 32
// (a whole step of 4 beams, forking in one / two launches 13.9 / 14.9, of 32 33.0 / 33.6).
constexpr int kForkEach = 16;  // entries a thread
__global__ __launch_bounds__(kPlanThreads) void cache_fork_kernel(const ForkArgs a) {
    __shared__ int to[kPlanThreads], from[kPlanThreads], length[kPlanThreads], before[kPlanThreads];
    const CacheView& c = a.c;
    const CacheRows r = {a.sequences, nullptr, a.n, 0, 0};
    const int tid = threadIdx.x, total = a.n * c.max_pages;
    if (tid < a.n) {
        const int s = r.sequence(tid, c.sequences), parent = a.parents[tid], first = tid / a.group * a.group;
        const int src = (unsigned)parent < (unsigned)a.group && first + parent < a.n ? r.sequence(first + parent, c.sequences) : -1;
        const auto pages_of = [&](int q) { return (min(max(c.lengths[q], 0), c.cap()) + c.page_tokens - 1) >> c.page_shift; };
        to[tid] = s == src ? -1 : s;
        from[tid] = src;
        length[tid] = src < 0 ? 0 : min(max(c.lengths[src], 0), c.cap());
        before[tid] = s < 0 ? 0 : pages_of(s);
    }
    __syncthreads();
    int now[kForkEach], old[kForkEach];
#pragma unroll
    for (int e = 0; e < kForkEach; ++e) {
        const int u = e * kPlanThreads + tid, i = u / c.max_pages, b = u - i * c.max_pages;
        now[e] = old[e] = -1;
        if (u >= total || to[i] < 0) continue;
        if (b < (length[i] + c.page_tokens - 1) >> c.page_shift) now[e] = c.table[(int64_t)from[i] * c.max_pages + b];
        if (b < before[i]) old[e] = c.table[(int64_t)to[i] * c.max_pages + b];
        if (!c.has(now[e])) now[e] = -1;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kForkEach; ++e) {
        const int u = e * kPlanThreads + tid, i = u / c.max_pages, b = u - i * c.max_pages;
        if (u >= total || to[i] < 0) continue;
        if (now[e] >= 0) atomicAdd(&c.refs[now[e]], 1);
        if (c.has(old[e])) atomicSub(&c.refs[old[e]], 1);
        if (b < max(before[i], (length[i] + c.page_tokens - 1) >> c.page_shift)) c.table[(int64_t)to[i] * c.max_pages + b] = now[e];
    }
    if (tid < a.n && to[tid] >= 0) c.lengths[to[tid]] = length[tid];
}

struct CompactArgs {
    CacheView c;
    int* moves;  // [pages][2]: from, to
    int* to;     // [pages]
    int* used;
    int* words;
};

// The i-th hole below the number of pages in use takes the i-th page in use above it: one workgroup ranks both by prefix sums over the counts of holders (600 pages 6 us: launch, two passes).
__global__ __launch_bounds__(kPlanThreads) void cache_compact_kernel(const CompactArgs a) {
    __shared__ int sums[kPlanWaves];
    const CacheView& c = a.c;
    const int tid = threadIdx.x;
    int used = 0, all;
    for (int p0 = 0; p0 < c.pages; p0 += 8 * kPlanThreads)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int p = p0 + e * kPlanThreads + tid;
            used += p < c.pages && c.refs[p] > 0;
        }
    scan(used, all, sums);
    used = all;
    int holes = 0, movers = 0;
    for (int p0 = 0; p0 < c.pages; p0 += 8 * kPlanThreads) {
        int r[8], h = 0, m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int p = p0 + 8 * tid + e;
            r[e] = p < c.pages ? c.refs[p] : 0;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int p = p0 + 8 * tid + e;
            h += p < used && r[e] <= 0;
            m += p >= used && p < c.pages && r[e] > 0;
        }
        int all_h, all_m;
        int at_h = holes + scan(h, all_h, sums), at_m = movers + scan(m, all_m, sums);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int p = p0 + 8 * tid + e;
            if (p < used && r[e] <= 0) a.moves[2 * (at_h++) + 1] = p;
            if (p >= used && p < c.pages && r[e] > 0) a.moves[2 * (at_m++)] = p;
        }
        holes += all_h;
        movers += all_m;
    }
    __threadfence_block();
    __syncthreads();
    for (int k = tid; k < movers; k += kPlanThreads) {
        const int from = a.moves[2 * k], to = a.moves[2 * k + 1];
        a.to[from] = to;
        c.refs[to] = c.refs[from];
        c.refs[from] = 0;
    }
    if (tid == 0) {
        a.words[W_USED] = used;
        a.words[W_MOVES] = movers;
        if (a.used) *a.used = used;
    }
}

// Whole pages; the first workgroups' threads turn the tables.
// (us, 150 pages of 512 KiB: pieces of 4 KiB and 2048, 8192 workgroups 17.5, 15.5; of 16 KiB 27.9)
constexpr int kPiece = 4096, kMoveGroups = 8192;  // bytes of a turn
__global__ __launch_bounds__(256) void cache_move_kernel(const CompactArgs a) {
    const CacheView& c = a.c;
    const int tid = threadIdx.x, used = a.words[W_USED], moves = a.words[W_MOVES];
    if (moves == 0) return;
    for (int s = blockIdx.x; s < c.sequences; s += gridDim.x) {
        const int length = min(max(c.lengths[s], 0), c.cap()), count = (length + c.page_tokens - 1) >> c.page_shift;
        for (int b = tid; b < count; b += 256) {
            int* entry = c.table + (int64_t)s * c.max_pages + b;
            const int p = *entry;
            if (p >= used && c.has(p)) *entry = a.to[p];
        }
    }
    const int64_t page_bytes = (int64_t)c.layers * 2 * c.heads * c.plane_bytes(), pieces = (page_bytes + kPiece - 1) / kPiece;
    const int planes = c.layers * 2 * c.heads;
    for (int64_t u = blockIdx.x; u < moves * pieces; u += gridDim.x) {
        const int k = (int)(u / pieces);
        const int64_t from = a.moves[2 * k], to = a.moves[2 * k + 1], b = (u - k * pieces) * kPiece + tid * 16;
        const int8_t* src = c.codes + from * page_bytes;
        int8_t* dst = c.codes + to * page_bytes;
        if (b < page_bytes) *(uint4*)(dst + b) = *(const uint4*)(src + b);  // (a page's bytes: a multiple of 256)
        if (u == k * pieces)
            for (int p = tid; p < planes; p += 256) c.scales[to * planes + p] = c.scales[from * planes + p];
    }
}

struct AppendArgs {
    CacheView c;
    CacheRows r;
    const void *x[2];
    int64_t token[2], head[2];
    int layer;
    const int* words;
};

__device__ __forceinline__ float bounded(float x) { return __builtin_amdgcn_fmed3f(x != x ? 0.f : x, -kLimit, kLimit); }

// A workgroup has the new positions of one page, of keys or values of a head: their largest magnitude, then their codes, nearest to 127 x / scale.  Rows stay in registers between the two.  Bound: the
// chain length - page - rows - maximum; a step 4.2 us, 2000 rows of 8 heads of 128 8.7 (12 MB), 4001 of 16 of 80 14.3 (31 MB).
// KEPT: pieces of eight values that a thread keeps from the first pass for the second.
template <class R, int THREADS, int KEPT>
__global__ __launch_bounds__(THREADS) void cache_append_kernel(const AppendArgs a) {
    constexpr int E = 8;
    typedef typename R::type V;
    __shared__ float tops[THREADS / 64];
    const CacheView& c = a.c;
    const int tid = threadIdx.x, slot = blockIdx.x, head = blockIdx.y, which = blockIdx.z, T = c.page_tokens;
    const int fits = a.words[W_FITS];
    const bool one = !a.r.starts && a.r.rows == 1;
    RowVec<R, E> kept[KEPT];
    // (a single row's place is known before the sequence's length is)
    if (one && tid * E < c.d_head) kept[0].load((const V*)a.x[which] + (int64_t)slot * a.token[which] + (int64_t)head * a.head[which] + tid * E);
    // entry i of the list has the slots floor(first row / T) + 2 i and those behind, as many as it can have pages
    int i, first, count, nth;
    if (a.r.starts) {
        int lo = 0, hi = a.r.n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            a.r.span(mid, first, count);
            if ((first >> c.page_shift) + 2 * mid <= slot) lo = mid; else hi = mid;
        }
        i = lo;
        a.r.span(i, first, count);
        nth = slot - (first >> c.page_shift) - 2 * i;
    } else {
        const int per = ((a.r.rows + T - 2) >> c.page_shift) + 1;
        i = slot / per;
        nth = slot - i * per;
        a.r.span(i, first, count);
    }
    if (nth < 0 || nth > ((count - 1) >> c.page_shift) + 1) return;
    const int s = a.r.sequence(i, c.sequences);
    if (s < 0 || count == 0) return;
    const int length = min(max(c.lengths[s], 0), c.cap()), begin = length - count;  // (rows from before the beginning are not written)
    const int b = (max(begin, 0) >> c.page_shift) + nth;
    if ((b << c.page_shift) >= length) return;
    const int p0 = max(begin, b << c.page_shift), p1 = min(length, (b + 1) << c.page_shift);
    const int page = c.table[(int64_t)s * c.max_pages + b];
    if (!c.has(page)) return;
    const int64_t plane = c.plane(page, a.layer, which, head);
    const int holders = c.refs[page];
    const float held = c.scales[plane];
    if (!fits || holders != 1) return;
    const int before = p0 - (b << c.page_shift), m = p1 - p0, d = c.d_head, per_row = d / E, pieces = m * per_row;
    int8_t* codes = c.codes + plane * c.plane_bytes();
    const V* x = (const V*)a.x[which] + (int64_t)(first + p0 - begin) * a.token[which] + (int64_t)head * a.head[which];
    const float was = before > 0 ? fabsf(bounded(held)) : 0.f;
    const auto at = [&](int u) {
        const int row = u / per_row;
        return x + (int64_t)row * a.token[which] + (u - row * per_row) * E;
    };
    float top = 0.f;
    {
        int row = tid / per_row, piece = tid - row * per_row;
        const int rows_on = THREADS / per_row, pieces_on = THREADS - rows_on * per_row;
#pragma unroll
        for (int k = 0; k < KEPT; ++k) {
            if (k * THREADS + tid < pieces) {
                if (!one) kept[k].load(x + (int64_t)row * a.token[which] + piece * E);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) kept[k].v[e] = 0;
            }
            row += rows_on;
            piece += pieces_on;
            if (piece >= per_row) {
                piece -= per_row;
                ++row;
            }
        }
    }
    const auto largest = [&](const RowVec<R, E>& q) {
#pragma unroll
        for (int e = 0; e < E; ++e) top = fmaxf(top, fabsf(bounded(R::up(q.v[e]))));
    };
#pragma unroll
    for (int k = 0; k < KEPT; ++k) largest(kept[k]);
    for (int u = KEPT * THREADS + tid; u < pieces; u += THREADS) {
        RowVec<R, E> q;
        q.load(at(u));
        largest(q);
    }
    top = wave_max(top);
    if (THREADS > 64) {
        if ((tid & 63) == 0) tops[tid >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) top = fmaxf(top, tops[w]);
    }
    const float scale = fmaxf(was, top);
    // (contraction would change nothing: each is a product, a division, a rounding)
    if (scale > was) {
        for (int u = tid; u < before * per_row; u += THREADS) {
            uint2 q = *(const uint2*)(codes + 8 * u);
            int8_t v[8];
            __builtin_memcpy(v, &q, 8);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (int8_t)rintf((float)v[e] * was / scale);
            __builtin_memcpy(&q, v, 8);
            *(uint2*)(codes + 8 * u) = q;
        }
    }
    // A product with 1 / scale is within 3 * 2^-24 of the quotient, so within 2^-15 of it: where that leaves no doubt about the nearest whole number, it is enough.
    const float per_scale = 1.f / scale;
    const auto put = [&](const RowVec<R, E>& q, int u) {
        int8_t v[8];
        bool sure = true;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float y = bounded(R::up(q.v[e])) * 127.f * per_scale, whole = rintf(y);
            sure &= fabsf(y - whole) < 0.5f - 3.0517578125e-5f;  // (not if it is NaN: a scale of 0, or whose reciprocal is beyond fp32)
            v[e] = (int8_t)whole;
        }
        if (__any(!sure)) {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = scale > 0.f ? (int8_t)rintf(bounded(R::up(q.v[e])) * 127.f / scale) : (int8_t)0;
        }
        uint2 w;
        __builtin_memcpy(&w, v, 8);
        *(uint2*)(codes + (int64_t)before * d + 8 * u) = w;
    };
#pragma unroll
    for (int k = 0; k < KEPT; ++k)
        if (k * THREADS + tid < pieces) put(kept[k], k * THREADS + tid);
    for (int u = KEPT * THREADS + tid; u < pieces; u += THREADS) {
        RowVec<R, E> q;
        q.load(at(u));
        put(q, u);
    }
    if (tid == 0) c.scales[plane] = scale;
}

// A page's threads: as many as keep its pieces, four each (us, a call: 4001 rows of 16 heads of 80, pages of 32, 128 / 256 threads 12.9 / 14.6; 2000 of 8 heads of 128, pages of 64 12.5 / 8.2;
// 4000 of the same in fp32, pages of 128, 256 threads with four / eight 13.2 / 12.0).  few: rows of a decoding step.
template <class R>
hipError_t launch_append(const AppendArgs& a, dim3 grid, bool few, hipStream_t st) {
    const int pieces = a.c.plane_bytes() / 8;
    if (few) return launch_on(cache_append_kernel<R, 64, 4>, grid, dim3(64), 0, st, a);
    if (pieces <= 4 * 128) return launch_on(cache_append_kernel<R, 128, 4>, grid, dim3(128), 0, st, a);
    return pieces <= 4 * 256 ? launch_on(cache_append_kernel<R, 256, 4>, grid, dim3(256), 0, st, a) : launch_on(cache_append_kernel<R, 256, 8>, grid, dim3(256), 0, st, a);
}

bool config_ok(const bild_cache_config& g) {
    if (!g.codes || !g.scales || !g.table || !g.lengths || !g.refs || g.reserved != 0) return false;
    if ((uintptr_t)g.codes % 16 || ((uintptr_t)g.scales | (uintptr_t)g.table | (uintptr_t)g.lengths | (uintptr_t)g.refs) % 4) return false;
    if (g.page_tokens != 32 && g.page_tokens != 64 && g.page_tokens != 128) return false;
    if (g.pages < 1 || g.pages > kMaxLimit || g.layers < 1 || g.layers > 1024 || g.heads < 1 || g.heads > 1024) return false;
    if (g.d_head < 16 || g.d_head > 256 || g.d_head % 8 || g.sequences < 1 || g.sequences > 65535 || g.max_pages < 1) return false;
    return (int64_t)g.max_pages * g.page_tokens <= 1 << 30 && (int64_t)g.sequences * g.max_pages <= 1 << 28;
}

}  // namespace

extern "C" int bild_cache_create(const bild_cache_config* cfg, bild_cache** out) {
    if (!cfg || !out || !config_ok(*cfg)) return BILD_EINVAL;
    const bild_cache_config& g = *cfg;
    bild_cache* c = new (std::nothrow) bild_cache();
    if (!c) return BILD_ENOMEM;
    c->view = {g.codes, g.scales, g.table, g.lengths, g.refs, g.pages, g.page_tokens, g.page_tokens == 32 ? 5 : g.page_tokens == 64 ? 6 : 7, g.layers, g.heads,
               g.d_head, g.sequences, g.max_pages};
    const size_t seqs = (size_t)g.sequences, pages = (size_t)g.pages, counts = attend_counts(g.heads);
    // (asked, latest, counts of arrivals and words begin as zeros)
    const size_t zeros = (2 * pages + counts + W_COUNT + 3) / 4 * 4, ints = zeros + 7 * seqs + 4 * pages + seqs * (size_t)g.max_pages;
    const size_t bytes = (ints * 4 + 255) / 256 * 256, floats = attend_part_floats(g.heads, g.d_head);
    int rc = BILD_OK;
    const int one = 1;
    if (hipGetDevice(&c->device) != hipSuccess || attend_init(g.d_head) != hipSuccess) rc = BILD_EHIP;
    else if (hipMalloc(&c->mem, bytes + 4 * floats) != hipSuccess) c->mem = nullptr, rc = BILD_ENOMEM;
    else {
        c->words = (int*)c->mem;
        c->asked = c->words + W_COUNT;
        c->latest = c->asked + pages;
        c->arrived = (unsigned*)(c->latest + pages);
        c->plan = c->words + zeros;
        c->fresh = c->plan + 7 * seqs;
        c->moves = c->fresh + pages;
        c->rows = c->moves + 3 * pages;
        c->part = (float*)((char*)c->mem + bytes);
        if (hipMemset(c->mem, 0, 4 * zeros) != hipSuccess || hipMemcpy(c->words + W_FITS, &one, 4, hipMemcpyHostToDevice) != hipSuccess ||
            hipStreamSynchronize(nullptr) != hipSuccess)
            rc = BILD_EHIP;
    }
    if (rc != BILD_OK) {
        (void)hipGetLastError();  // (told by rc: not to be found by a later call as well)
        (void)bild_cache_destroy(c);
        return rc;
    }
    *out = c;
    return BILD_OK;
}

extern "C" int bild_cache_destroy(bild_cache* c) {
    if (!c) return BILD_EINVAL;
    if (c->mem) (void)hipFree(c->mem);
    delete c;
    return BILD_OK;
}

extern "C" int bild_cache_extend(bild_cache* c, const bild_cache_extend_call* call, void* hip_stream) {
    if (!c || !call) return BILD_EINVAL;
    const bild_cache_extend_call& k = *call;
    if (k.n < 1 || k.n > c->view.sequences || k.rows < 0 || k.window < 0 || k.sinks < 0) return BILD_EINVAL;
    const int pieces = (c->view.max_pages + 64 * kSlideEach - 1) / (64 * kSlideEach);
    ExtendArgs a = {c->view, {k.sequences, k.starts, k.n, std::min(k.rows, c->view.cap() + 1), 0}, k.cut, k.granted, k.window, k.sinks, pieces, c->plan, c->fresh, c->asked, c->latest,
                    c->plan + 4 * (size_t)c->view.sequences, c->words};
    const OnDevice on(c->device);
    if (!on.ok) return BILD_EHIP;
    hipStream_t st = (hipStream_t)hip_stream;
    if (const int64_t items = (int64_t)k.n * pieces; k.window && items > kSlideHere) {
        if (launch_on(cache_slide_kernel, dim3((unsigned)std::min<int64_t>((items + 3) / 4, kSlideGroups)), dim3(256), 0, st, a) != hipSuccess) return BILD_EHIP;
        a.window = 0;
    }
    if (launch_on(cache_extend_kernel, dim3(1), dim3(kPlanThreads), 0, st, a) != hipSuccess) return BILD_EHIP;
    if (!k.starts && k.rows == 0) return BILD_OK;  // (nothing is copied)
    const int64_t planes = (int64_t)c->view.layers * 2 * c->view.heads, groups = std::min<int64_t>((k.n * planes + 3) / 4, 2048);
    const int* copies = a.copies;
    return launch_on(cache_copy_kernel, dim3((unsigned)groups), dim3(256), 0, st, c->view, copies, c->words) == hipSuccess ? BILD_OK : BILD_EHIP;
}

extern "C" int bild_cache_fork(bild_cache* c, const int32_t* sequences, const int32_t* parents, int n, int group, void* hip_stream) {
    if (!c || !parents || n < 1 || n > c->view.sequences || group < 0 || group > n) return BILD_EINVAL;
    const ForkArgs a = {c->view, sequences, parents, n, group ? group : n, c->rows, c->plan};
    const OnDevice on(c->device);
    if (!on.ok) return BILD_EHIP;
    hipStream_t st = (hipStream_t)hip_stream;
    if (n <= kPlanThreads && (int64_t)n * c->view.max_pages <= kForkEach * kPlanThreads)
        return launch_on(cache_fork_kernel, dim3(1), dim3(kPlanThreads), 0, st, a) == hipSuccess ? BILD_OK : BILD_EHIP;
    if (launch_on(cache_fork_read_kernel, dim3(n), dim3(256), 0, st, a) != hipSuccess) return BILD_EHIP;
    return launch_on(cache_fork_write_kernel, dim3(n), dim3(256), 0, st, a) == hipSuccess ? BILD_OK : BILD_EHIP;
}

extern "C" int bild_cache_compact(bild_cache* c, int32_t* used, void* hip_stream) {
    if (!c) return BILD_EINVAL;
    const CompactArgs a = {c->view, c->moves, c->moves + 2 * (size_t)c->view.pages, used, c->words};
    const OnDevice on(c->device);
    if (!on.ok) return BILD_EHIP;
    hipStream_t st = (hipStream_t)hip_stream;
    if (launch_on(cache_compact_kernel, dim3(1), dim3(kPlanThreads), 0, st, a) != hipSuccess) return BILD_EHIP;
    // (at most half of the pages move; a table a workgroup)
    const CacheView& v = c->view;
    const int64_t pieces = ((int64_t)v.layers * 2 * v.heads * v.plane_bytes() + kPiece - 1) / kPiece, groups = std::min<int64_t>(std::max<int64_t>(v.pages / 2 * pieces, v.sequences), kMoveGroups);
    return launch_on(cache_move_kernel, dim3((unsigned)groups), dim3(256), 0, st, a) == hipSuccess ? BILD_OK : BILD_EHIP;
}

extern "C" int bild_cache_append(bild_cache* c, const bild_cache_append_call* call, void* hip_stream) {
    if (!c || !call) return BILD_EINVAL;
    const bild_cache_append_call& k = *call;
    if (!k.k || !k.v || k.reserved != 0 || !row_type(k.dtype) || k.layer < 0 || k.layer >= c->view.layers) return BILD_EINVAL;
    if (k.n < 1 || k.n > c->view.sequences || k.rows < 1 || (k.starts && k.tokens < 1)) return BILD_EINVAL;
    const int64_t slots = k.starts ? (k.tokens >> c->view.page_shift) + 2 * (int64_t)k.n : k.n * ((((int64_t)k.rows + c->view.page_tokens - 2) >> c->view.page_shift) + 1);
    if ((!k.starts && (int64_t)k.n * k.rows > 0x7FFFFFFF) || slots > kMaxGroups) return BILD_EINVAL;
    const AppendArgs a = {c->view, {k.sequences, k.starts, k.n, k.rows, k.starts ? k.tokens : k.n * k.rows}, {k.k, k.v}, {k.k_token, k.v_token}, {k.k_head, k.v_head}, k.layer, c->words};
    const OnDevice on(c->device);
    if (!on.ok) return BILD_EHIP;
    const dim3 grid((unsigned)slots, c->view.heads, 2);
    const bool few = k.rows <= 4;
    hipStream_t st = (hipStream_t)hip_stream;
    const hipError_t err = k.dtype == BILD_DT_F32 ? launch_append<RowF32>(a, grid, few, st) : k.dtype == BILD_DT_BF16 ? launch_append<RowBf16>(a, grid, few, st)
                                                                                                                : launch_append<RowF16>(a, grid, few, st);
    return err == hipSuccess ? BILD_OK : BILD_EHIP;
}
