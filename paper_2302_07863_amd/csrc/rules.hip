// Rules on logits (bild_rules_apply): penalties for tokens that were there, biases, bit masks, and the softmax statistics of
// what is left, in one pass over the logits.
//
// Bound: memory, every logit read and written once.  A workgroup takes a range of a row's ids and requests all of its logits at once.  What the row's
// tokens and biases say about its ids it collects in a table in LDS, a word per id, from the whole list: a list of some thousand tokens comes from the L2 faster
// than a table of counts for the whole vocabulary could be cleared and filled in memory, and counts are whole numbers, so the order of the LDS atomics
// shows nowhere.  A thread keeps the maximum and the sum of its ids as they come by; the last workgroup of a row joins those of its ranges.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "last_in.h"
#include "operators.h"
#include "rows_common.h"

using namespace bild;

namespace {
// A word of the table: how often the id occurs from `starts` on, whether it occurs at all, which of the biases is its last.
constexpr unsigned kCountBits = 20, kSeen = 1u << kCountBits, kBiasAt = kCountBits + 1;
constexpr unsigned kCountMask = kSeen - 1;
static_assert(kMaxRuleTokens <= (int)kCountMask && kMaxBiases < 1 << (32 - kBiasAt), "a word holds them");
constexpr int kThreads = 256;
constexpr int kMaxRange = kThreads * 16;  // ids of a workgroup, 16 a thread: 16 KiB of table
constexpr int kCountStride = 32;          // words between two rows' counts of arrivals: a line each (side by side, a thousand arrivals took 20 us)

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

struct Penalty {
    float rep, freq, pres;
};

// z after the rules that the table's word asks for.  (Each step rounded for itself: the compiler is not to join products and sums.)
__device__ __forceinline__ float apply(float z, unsigned w, const Penalty& p, const float* bias) {
#pragma clang fp contract(off)
    const unsigned c = w & kCountMask;
    if (c || (w & kSeen)) z = z > 0.f ? z / p.rep : z * p.rep;
    if (c) {
        const float f = p.freq * (float)c;
        z = z - f;
        z = z - p.pres;
    }
    if (w >> kBiasAt) z = z + bias[(w >> kBiasAt) - 1];
    return z;
}

// Sums of exponentials are kept as sums of 2^(z L - M), L = log2 e as fp32 has it, M the whole number above the largest z L: a product and the hardware's exponential a
// term, rounded once, as the product is exact before M is taken off.  In the end the sum is multiplied by 2^(M - m L): a term is e^(z - m) to a factor of 2^((z - m) (L - log2 e)),
// which for a term of e^-20 is off by 2.7e-7 of it.  M comes from a product that is rounded: of maxima below kFar by a quarter at most, so that no term is above 2^(1/4).
// (From 4e9 on by more than the exponential's range.)  Beyond kFar, where logits are half an integer apart and more, terms are the exponentials of their differences.
constexpr float kLog2e = 1.44269502162933349609375f;
constexpr float kFar = 4194304.f;  // 2^22
__device__ __forceinline__ float whole_above(float m) { return m == -INFINITY ? 0.f : ceilf(m * kLog2e); }
__device__ __forceinline__ float term(float z, float whole) { return __builtin_amdgcn_exp2f(__builtin_fmaf(z, kLog2e, -whole)); }
// such a sum as one of e^(z - m)
__device__ __forceinline__ float to_base(float s, float m) {
    return !(fabsf(m) < kFar) ? s : s * __builtin_amdgcn_exp2f(__builtin_fmaf(-m, kLog2e, whole_above(m)));
}

// Statistics of two sets of ids.  (A sum that is NaN stays NaN beside any other; what lies infinitely far below counts nothing.)
__device__ __forceinline__ Stat join(const Stat& a, const Stat& b) {
    Stat r;
    r.m = fmaxf(a.m, b.m);
    r.s = a.s * (a.m == r.m ? 1.f : fexp_full(a.m - r.m)) + b.s * (b.m == r.m ? 1.f : fexp_full(b.m - r.m));
    r.idx = a.m > b.m || (a.m == b.m && a.idx < b.idx) ? a.idx : b.idx;
    return r;
}

__device__ __forceinline__ void put_stats(const RulesArgs& a, int row, const Stat& r, float z_target) {
    bild_row_stats o;
    o.zmax = r.m;
    o.lse = r.m == INFINITY ? INFINITY : r.m == -INFINITY && r.s == 0.f ? -INFINITY : r.m + logf(r.s);
    o.argmax = r.idx == 0x7FFFFFFF ? -1 : r.idx;
    o.z_target = z_target;
    a.stats[row] = o;
}

// last_in (last_in.h) for workgroups whose one wave has stored their partial results.
__device__ __forceinline__ bool last_wave_in(unsigned* counter, unsigned n) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    unsigned before = 0;
    if ((threadIdx.x & 63) == 0) {
        before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (before == n - 1) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    return __builtin_amdgcn_readfirstlane((int)before) == (int)n - 1;
}

// The first n of a row's tokens, dealt to the threads by fours, two of these requested at a time: request(0), then each(f) with f(i, token).
struct Tokens {
    typedef Piece<16, 4> Four;
    static constexpr int U = 2;
    const int* ids;
    int n;
    Four p[U];
    __device__ __forceinline__ void request(int i0) {
        const int full = n >> 2;
        if (full == 0) return;
#pragma unroll
        for (int u = 0; u < U; ++u) p[u] = *(const Four*)(ids + 4 * (int64_t)min(i0 + u * kThreads + (int)threadIdx.x, full - 1));
    }
    template <class F>
    __device__ __forceinline__ void each(F&& f) {
        const int tid = threadIdx.x, full = n >> 2;
        for (int i0 = 0; i0 < full; i0 += U * kThreads) {
            if (i0) request(i0);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * kThreads + tid;
                if (i < full) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) f(4 * i + e, (int)p[u].w[e]);
                }
            }
        }
        if (tid < (n & 3)) f((full << 2) + tid, ids[(full << 2) + tid]);
    }
};

// EACH ids a thread, in pieces of 16 bytes that lie a workgroup's width apart.
template <class R, int EACH>
__global__ __launch_bounds__(kThreads) void rules_kernel(const RulesArgs a) {
    constexpr int E = 16 / R::kBytes, P = EACH / E, W = kThreads / 64;
    typedef typename R::type V;
    extern __shared__ __attribute__((aligned(16))) unsigned table[];  // [range], then the biases, where there are tokens or biases
    __shared__ float tops[W], sums[W];
    __shared__ int ids_at[W];
    static_assert(W == 4, "joined by hand");
    __shared__ float at_target;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), nthr = kThreads;
    const int row = blockIdx.y, v0 = (int)blockIdx.x * a.range, v1 = min(v0 + a.range, a.vocab), n = v1 - v0;
    const bool tabled = a.tokens || a.bias_ids;
    const bool pass = a.len_ptr != nullptr;
    const int next = pass ? *a.len_ptr + a.len_add + row + 1 : 0;  // position of a pass's logits
    const int n_tokens = !a.tokens ? 0 : pass ? min(next, a.max_tokens) : min(max(a.lengths[row], 0), a.max_tokens);
    const int from = !a.tokens ? 0 : pass ? (a.start_ptr ? *a.start_ptr : 1) : a.starts ? a.starts[row] : 0;
    const int n_bias = !a.bias_ids ? 0 : a.bias_counts ? min(max(a.bias_counts[row], 0), a.max_bias) : a.max_bias;
    const int target = pass ? (next < *a.ylen_ptr ? a.y[next] : -1) : a.targets ? a.targets[row] : -1, ti = target - v0;
    const V* in = (const V*)a.logits + (int64_t)row * a.ld + v0;
    V* out = a.out ? (V*)a.out + (int64_t)row * a.ldo + v0 : nullptr;
    const uint32_t* mask = a.mask ? a.mask + (int64_t)(pass ? next : row) * a.mask_stride + (v0 >> 5) : nullptr;
    float* bias = (float*)(table + a.range);

    struct Slot {
        RowVec<R, E> x;
        uint32_t allowed;
    };
    Slot pieces[P];
    const auto request = [&](Slot& q, int turn) {  // (past the end: ids that are there, for nobody)
        const int i = (turn * nthr + tid) * E;
        if (n >= E) q.x.load(in + min(i, n - E));
        if (i < n && i + E > n) q.x.load_some(in + i, n - i);
        q.allowed = ~0u;
        if (mask) q.allowed = mask[min(i, n - 1) >> 5];  // (a range starts with a word of the mask, and no piece has ids of two words)
    };
    // (loads come back in order, and the logits, which need nothing, take longest: everything is requested before anything is waited for)
#pragma unroll
    for (int p = 0; p < P; ++p) request(pieces[p], p);
    Penalty pen = {1.f, 0.f, 0.f};
    if (tabled) {
        const int* bias_ids = a.bias_ids + (int64_t)row * a.bias_stride;
        const float* values = a.bias + (int64_t)row * a.bias_stride;
        int b_id = -1;
        float b_value = 0.f;
        if (tid < n_bias) {
            b_id = bias_ids[tid];
            b_value = values[tid];
        }
        Tokens said = {a.tokens + (int64_t)row * a.tokens_stride, n_tokens, {}};
        said.request(0);
        if (a.tokens) {
            const bild_penalties p = a.penalties[(int64_t)row * a.penalties_stride];
            pen = {p.repetition, p.frequency, p.presence};
        }
        for (int i = tid * 4; i < a.range; i += kThreads * 4) *(uint4*)(table + i) = make_uint4(0, 0, 0, 0);
        lds_barrier();
        if (n_bias > 0) {
            for (int i = tid; i < n_bias; i += kThreads) {
                if (i != tid) {
                    b_id = bias_ids[i];
                    b_value = values[i];
                }
                const unsigned v = (unsigned)b_id - (unsigned)v0;
                bias[i] = b_value;
                if (v < (unsigned)n) atomicMax(&table[v], (unsigned)(i + 1) << kBiasAt);
            }
            lds_barrier();
        }
        said.each([&](int i, int t) {
            const unsigned v = (unsigned)t - (unsigned)v0;
            if (v >= (unsigned)n) return;
            if (i >= from) atomicAdd(&table[v], 1u);
            else atomicOr(&table[v], kSeen);
        });
        lds_barrier();
    }

    float z[P][E];
    float top = -INFINITY;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int i = (p * kThreads + tid) * E;
#pragma unroll
        for (int e = 0; e < E; ++e) z[p][e] = R::up(pieces[p].x.v[e]);
        if (tabled) {
            uint32_t w[E], any = 0u;
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                const uint4 q = *(const uint4*)(table + min(i, a.range - E) + e);
                w[e] = q.x; w[e + 1] = q.y; w[e + 2] = q.z; w[e + 3] = q.w;
                any |= q.x | q.y | q.z | q.w;
            }
            if (i < n && any) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (w[e]) z[p][e] = apply(z[p][e], w[e], pen, bias);
            }
        }
        uint32_t allowed = pieces[p].allowed >> (i & 31);
        const bool edge = i + E > n;
        if (edge) allowed &= i < n ? (1u << (n - i)) - 1u : 0u;
        if (mask || edge) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const uint32_t keep = (uint32_t)((int)(allowed << (31 - e)) >> 31);
                z[p][e] = __uint_as_float((__float_as_uint(z[p][e]) & keep) | (0xFF800000u & ~keep));
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) top = __builtin_amdgcn_fmed3f(top, z[p][e], INFINITY);
    }
    const auto put = [&] {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int i = (p * kThreads + tid) * E;
            RowVec<R, E> y;
#pragma unroll
            for (int e = 0; e < E; ++e) y.v[e] = R::down(z[p][e]);
            if (i + E <= n) y.store(out + i); else y.store_some(out + i, n - i);
        }
    };
    // (the wave that tells of the workgroup's arrival waits for its stores first: its own logits come behind that)
    const bool tells = wave == 0 && a.parts > 1 && a.stats;
    if (out && !tells) put();
    if (!a.stats && !pass) return;
    const float mine = top;
    top = wave_max(top);
    if (lane == 0) tops[wave] = top;
    // the target's logit is with one thread
    if (ti >= 0 && ti < n && ti / E % kThreads == tid) {
        float zt = 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < E; ++e)
                if ((p * kThreads + tid) * E + e == ti) zt = z[p][e];
        at_target = zt;
    }
    lds_barrier();
    Stat r;
    r.m = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    float s = 0.f;
    if (fabsf(r.m) < kFar || r.m == -INFINITY) {
        const float whole = whole_above(r.m);
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < E; ++e) s += term(z[p][e], whole);
    } else {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < E; ++e) s += fexp_full(z[p][e] - r.m);
    }
    s = wave_sum(s);
    int idx = 0x7FFFFFFF;
    if (top == r.m && r.m != -INFINITY) {  // (a wave that has the maximum)
        if (mine == r.m) {
#pragma unroll
            for (int p = P - 1; p >= 0; --p)
#pragma unroll
                for (int e = E - 1; e >= 0; --e)
                    if (z[p][e] == r.m) idx = v0 + (p * kThreads + tid) * E + e;
        }
        for (int o = 32; o > 0; o >>= 1) idx = min(idx, __shfl_xor(idx, o, 64));
    }
    if (lane == 0) {
        sums[wave] = s;
        ids_at[wave] = idx;
    }
    lds_barrier();
    if (wave != 0) return;
    r.s = to_base(sums[0] + sums[1] + sums[2] + sums[3], r.m);
    r.idx = min(min(ids_at[0], ids_at[1]), min(ids_at[2], ids_at[3]));
    if (pass) {  // (a row of which nothing is left: its lowest id, as a token has to be one)
        if (lane == 0) a.part[(size_t)row * a.part_ld + blockIdx.x] = StatPart{r.m, r.s, r.idx == 0x7FFFFFFF ? v0 : r.idx, 0};
        if (lane == 0 && ti >= 0 && ti < n) a.zt[row] = at_target;
        return;
    }
    const bool has = target >= 0 && target < a.vocab;
    float zt = has ? at_target : NAN;  // (where the target is not this range's: not read)
    if (a.parts > 1) {
        const auto parts = make_rsrc(a.part + (size_t)row * a.parts, sizeof(StatPart) * (size_t)a.parts);
        if (lane == 0)
            __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(r.m), __float_as_uint(r.s), (unsigned)r.idx, __float_as_uint(zt)}, parts,
                                                   (int)blockIdx.x * 16, 0, kPartAux);
        const bool last = last_wave_in(a.arrived + (size_t)row * kCountStride, (unsigned)a.parts);
        if (out) put();
        if (!last) return;
        r = stat_neutral();
        for (int p = lane; p < a.parts; p += 64) {
            const u32x4 q = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(parts, p * 16, 0, kPartAux));
            r = join(r, Stat{__uint_as_float(q[0]), __uint_as_float(q[1]), (int)q[2]});
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) r = join(r, stat_shfl_xor(r, o));
        if (has) zt = __uint_as_float((unsigned)__builtin_amdgcn_raw_buffer_load_b32(parts, target / a.range * 16 + 12, 0, kPartAux));
    }
    if (lane == 0) put_stats(a, row, r, zt);
}

// Workgroups of a row: two thousand in all, none with more ids than its threads hold or with less than one piece a thread.  (Ranges of up to 4096 / 8192
// ids, us: 512 x 50257 fp16 29.1 / 32.2, with 1000 tokens a row 40.4 / 46.2, 256 x 128000 bf16 with 1000 53.5 / 65.9; two thousand / one
// thousand workgroups: 11 x 250112 fp32 with 700 tokens 12.6 / 13.6, 64 x 32000 bf16 with 8192 12.9 / 13.1.)
int parts_of(int rows, int vocab) {
    const int least = (vocab + kMaxRange - 1) / kMaxRange, most = std::max(least, (vocab + 2047) / 2048);
    return std::max(least, std::min(most, (2048 + rows - 1) / rows));
}
template <class R>
hipError_t launch(const RulesArgs& a, size_t lds, hipStream_t st) {
    return launch_on(a.range <= kThreads * 8 ? rules_kernel<R, 8> : rules_kernel<R, 16>, dim3(a.parts, a.rows), dim3(kThreads), lds, st, a);
}
size_t parts_cap(int max_rows, int vocab) { return (size_t)max_rows * ((vocab + kMaxRange - 1) / kMaxRange) + 2048 + max_rows; }

}  // namespace

struct bild_rules {
    int vocab = 0, max_rows = 0, device = 0;
    void* mem = nullptr;
    StatPart* part = nullptr;
    unsigned* arrived = nullptr;
};

namespace bild {

hipError_t launch_rules(RulesArgs a, hipStream_t st, int* parts) {
    a.parts = parts_of(a.rows, a.vocab);
    a.range = ((a.vocab + a.parts - 1) / a.parts + 31) / 32 * 32;  // whole words of the mask
    a.parts = (a.vocab + a.range - 1) / a.range;
    if (parts) *parts = a.parts;
    const size_t lds = a.tokens || a.bias_ids ? sizeof(unsigned) * ((size_t)a.range + (a.bias_ids ? a.max_bias : 0)) : 0;
    return a.dtype == BILD_DT_F32 ? launch<RowF32>(a, lds, st) : a.dtype == BILD_DT_BF16 ? launch<RowBf16>(a, lds, st) : launch<RowF16>(a, lds, st);
}

}  // namespace bild

extern "C" int bild_rules_create(int vocab, int max_rows, bild_rules** out) {
    if (!out || vocab < 1 || vocab > (1 << 24) || max_rows < 1 || max_rows > 65535) return BILD_EINVAL;
    bild_rules* r = new (std::nothrow) bild_rules();
    if (!r) return BILD_ENOMEM;
    r->vocab = vocab;
    r->max_rows = max_rows;
    const size_t counts = (sizeof(unsigned) * kCountStride * (size_t)max_rows + 255) / 256 * 256;
    int rc = BILD_OK;
    if (hipGetDevice(&r->device) != hipSuccess) rc = BILD_EHIP;
    else if (hipMalloc(&r->mem, counts + sizeof(StatPart) * parts_cap(max_rows, vocab)) != hipSuccess) r->mem = nullptr, rc = BILD_ENOMEM;
    else if (hipMemset(r->mem, 0, counts) != hipSuccess || hipStreamSynchronize(nullptr) != hipSuccess) rc = BILD_EHIP;
    if (rc != BILD_OK) {
        (void)hipGetLastError();  // (told by rc: not to be found by a later call as well)
        (void)bild_rules_destroy(r);
        return rc;
    }
    r->arrived = (unsigned*)r->mem;
    r->part = (StatPart*)((char*)r->mem + counts);
    *out = r;
    return BILD_OK;
}

extern "C" int bild_rules_destroy(bild_rules* r) {
    if (!r) return BILD_EINVAL;
    if (r->mem) (void)hipFree(r->mem);
    delete r;
    return BILD_OK;
}

extern "C" int bild_rules_apply(bild_rules* r, const bild_rules_call* call, void* hip_stream) {
    if (!r || !call) return BILD_EINVAL;
    const bild_rules_call& c = *call;
    if (!c.logits || (!c.out && !c.stats) || !row_type(c.dtype) || c.rows < 1) return BILD_EINVAL;
    if (c.rows > r->max_rows) return BILD_ECAP;
    if (c.tokens && (!c.lengths || !c.penalties || c.penalties_stride < 0 || c.penalties_stride > 1)) return BILD_EINVAL;
    if (c.bias_ids && !c.bias) return BILD_EINVAL;
    if ((c.tokens && (c.max_tokens < 0 || c.max_tokens > kMaxRuleTokens)) || (c.bias_ids && (c.max_bias < 0 || c.max_bias > kMaxBiases))) return BILD_EINVAL;
    if (c.out == c.logits && c.out_stride != c.logits_stride && c.rows > 1) return BILD_EINVAL;
    RulesArgs a;
    std::memset((void*)&a, 0, sizeof(a));
    a.logits = c.logits;
    a.out = c.out;
    a.ld = c.logits_stride;
    a.ldo = c.out_stride;
    a.targets = c.targets;
    a.stats = c.stats;
    a.tokens = c.tokens;
    a.tokens_stride = c.tokens_stride;
    a.lengths = c.lengths;
    a.starts = c.starts;
    a.penalties = c.penalties;
    a.penalties_stride = c.penalties_stride;
    a.bias_ids = c.bias_ids;
    a.bias = c.bias;
    a.bias_stride = c.bias_stride;
    a.bias_counts = c.bias_counts;
    a.mask = c.mask;
    a.mask_stride = c.mask_stride;
    a.rows = c.rows;
    a.vocab = r->vocab;
    a.dtype = c.dtype;
    a.max_tokens = c.max_tokens;
    a.max_bias = c.max_bias;
    a.part = r->part;
    a.arrived = r->arrived;
    const OnDevice on(r->device);
    if (!on.ok) return BILD_EHIP;
    return launch_rules(a, (hipStream_t)hip_stream) == hipSuccess ? BILD_OK : BILD_EHIP;
}
