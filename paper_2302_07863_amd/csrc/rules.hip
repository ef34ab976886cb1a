// Rules on logits (bild_rules_apply): penalties for tokens that were there, biases, bit masks, and the softmax statistics of
// what is left, in one pass over the logits.
//
// Bound: memory, every logit read and written once.  A workgroup takes a range of a row's ids.  What the row's tokens and
// biases say about its ids it collects in a table in LDS, a word per id, from the whole list: a list of some thousand tokens
// comes from the L2 faster than a table of counts for the whole vocabulary could be cleared and filled in memory, and counts
// are whole numbers, so the order of the LDS atomics shows nowhere.  The last workgroup of a row joins the ranges' statistics.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "last_in.h"
#include "operators.h"
#include "rows_common.h"

using namespace bild;

// A word of the table: how often the id occurs from `starts` on, whether it occurs at all, which of the biases is its last.
namespace {
constexpr unsigned kCountBits = 20, kSeen = 1u << kCountBits, kBiasAt = kCountBits + 1;
constexpr unsigned kCountMask = kSeen - 1;
constexpr int kMaxTokens = (1 << kCountBits) - 1, kMaxBias = (1 << (32 - kBiasAt)) / 2 - 1;  // (1023)
constexpr int kThreads = 256;
constexpr int kMaxRange = 8192;  // ids of a workgroup: 32 KiB of table

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

// Statistics of two sets of ids.  (A sum that is NaN stays NaN beside any other; what lies infinitely far below counts nothing.)
__device__ __forceinline__ Stat join(const Stat& a, const Stat& b) {
    Stat r;
    r.m = fmaxf(a.m, b.m);
    r.s = a.s * (a.m == r.m ? 1.f : fexp_full(a.m - r.m)) + b.s * (b.m == r.m ? 1.f : fexp_full(b.m - r.m));
    r.idx = a.m > b.m || (a.m == b.m && a.idx < b.idx) ? a.idx : b.idx;
    return r;
}
__device__ __forceinline__ Stat join_wave(Stat r) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) r = join(r, stat_shfl_xor(r, o));
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

template <class R>
__global__ __launch_bounds__(kThreads) void rules_kernel(const RulesArgs a) {
    constexpr int E = 16 / R::kBytes;
    typedef typename R::type V;
    extern __shared__ unsigned table[];  // [range] where there are tokens or biases
    __shared__ StatPart share[kThreads / 64];
    __shared__ unsigned word;
    __shared__ float at_target;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = blockIdx.y, v0 = (int)blockIdx.x * a.range, v1 = min(v0 + a.range, a.vocab);
    const bool tabled = a.tokens || a.bias_ids;
    Penalty pen = {1.f, 0.f, 0.f};
    const float* bias = nullptr;
    if (tabled) {
        for (int i = tid; i < v1 - v0; i += kThreads) table[i] = 0u;
        __syncthreads();
        if (a.bias_ids) {
            const int n = a.bias_counts ? min(max(a.bias_counts[row], 0), a.max_bias) : a.max_bias;
            const int* ids = a.bias_ids + (int64_t)row * a.bias_stride;
            bias = a.bias + (int64_t)row * a.bias_stride;
            for (int i = tid; i < n; i += kThreads) {
                const int v = ids[i];
                if (v >= v0 && v < v1) atomicMax(&table[v - v0], (unsigned)(i + 1) << kBiasAt);
            }
            __syncthreads();
        }
        if (a.tokens) {
            const int n = min(max(a.lengths[row], 0), a.max_tokens), from = a.starts ? a.starts[row] : 0;
            const int* ids = a.tokens + (int64_t)row * a.tokens_stride;
            for (int i = tid; i < n; i += kThreads) {
                const int v = ids[i];
                if (v < v0 || v >= v1) continue;
                if (i >= from) atomicAdd(&table[v - v0], 1u);
                else atomicOr(&table[v - v0], kSeen);
            }
            const bild_penalties p = a.penalties[(int64_t)row * a.penalties_stride];
            pen = {p.repetition, p.frequency, p.presence};
            __syncthreads();
        }
    }
    const V* in = (const V*)a.logits + (int64_t)row * a.ld;
    V* out = a.out ? (V*)a.out + (int64_t)row * a.ldo : nullptr;
    const uint32_t* mask = a.mask ? a.mask + (int64_t)row * a.mask_stride : nullptr;
    const int target = a.targets ? a.targets[row] : -1;
    float m = -INFINITY, s = 0.f;
    int idx = 0x7FFFFFFF;
    for (int v = v0 + tid * E; v < v1; v += kThreads * E) {
        const int n = v1 - v;
        RowVec<R, E> x;
        if (n >= E) x.load(in + v); else x.load_some(in + v, n);
        const uint32_t allowed = mask ? mask[v >> 5] >> (v & 31) : ~0u;  // (a range starts with a word, so do eight ids not cross one)
        float z[E];
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            z[i] = R::up(x.v[i]);
            if (tabled) z[i] = apply(z[i], i < n ? table[v + i - v0] : 0u, pen, bias);
            if (!(allowed >> i & 1u) || i >= n) z[i] = -INFINITY;
            if (i < n && v + i == target) at_target = z[i];
            x.v[i] = R::down(z[i]);
            if (z[i] > top) top = z[i];
        }
        if (out) {
            if (n >= E) x.store(out + v); else x.store_some(out + v, n);
        }
        if (a.stats) {  // (equal maxima keep the lower id: ids come in increasing order)
            if (top > m) {
                s = s * fexp_full(m - top);
                m = top;
#pragma unroll
                for (int i = E - 1; i >= 0; --i)
                    if (z[i] == top) idx = v + i;
            }
            const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int i = 0; i < E; ++i) s += fexp_full(z[i] - base);
        }
    }
    if (!a.stats) return;
    Stat r = join_wave(Stat{m, s, idx});
    if (lane == 0) share[wave] = StatPart{r.m, r.s, r.idx, 0};
    __syncthreads();
    r = Stat{share[0].m, share[0].s, share[0].idx};
    for (int w = 1; w < kThreads / 64; ++w) r = join(r, Stat{share[w].m, share[w].s, share[w].idx});
    const bool has = target >= 0 && target < a.vocab;
    float zt = has ? at_target : NAN;  // (where the target is not this range's: not read)
    if (a.parts > 1) {
        typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
        const auto parts = make_rsrc(a.part + (size_t)row * a.parts, sizeof(StatPart) * (size_t)a.parts);
        if (tid == 0)
            __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(r.m), __float_as_uint(r.s), (unsigned)r.idx, __float_as_uint(zt)}, parts,
                                                   (int)blockIdx.x * 16, 0, kPartAux);
        if (!last_in(a.arrived + row, (unsigned)a.parts, &word)) return;
        if (wave != 0) return;
        r = stat_neutral();
        for (int p = lane; p < a.parts; p += 64) {
            const u32x4 q = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(parts, p * 16, 0, kPartAux));
            r = join(r, Stat{__uint_as_float(q[0]), __uint_as_float(q[1]), (int)q[2]});
        }
        r = join_wave(r);
        if (has) zt = __uint_as_float((unsigned)__builtin_amdgcn_raw_buffer_load_b32(parts, target / a.range * 16 + 12, 0, kPartAux));
    }
    if (tid == 0) put_stats(a, row, r, zt);
}

// Workgroups of a row: about a thousand in all, none with more ids than its table holds or with less than one piece a thread.
int parts_of(int rows, int vocab) {
    const int least = (vocab + kMaxRange - 1) / kMaxRange, most = std::max(least, (vocab + 2047) / 2048);
    return std::max(least, std::min(most, (1024 + rows - 1) / rows));
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

hipError_t launch_rules(RulesArgs a, hipStream_t st) {
    // whole words of the mask
    a.range = ((a.vocab + a.parts - 1) / a.parts + 31) / 32 * 32;
    a.parts = (a.vocab + a.range - 1) / a.range;
    const size_t lds = a.tokens || a.bias_ids ? sizeof(unsigned) * (size_t)a.range : 0;
    const dim3 grid(a.parts, a.rows), block(kThreads);
    if (a.dtype == BILD_DT_F32) hipLaunchKernelGGL(rules_kernel<RowF32>, grid, block, lds, st, a);
    else if (a.dtype == BILD_DT_BF16) hipLaunchKernelGGL(rules_kernel<RowBf16>, grid, block, lds, st, a);
    else hipLaunchKernelGGL(rules_kernel<RowF16>, grid, block, lds, st, a);
    return hipGetLastError();
}

}  // namespace bild

extern "C" int bild_rules_create(int vocab, int max_rows, bild_rules** out) {
    if (!out || vocab < 1 || vocab > (1 << 24) || max_rows < 1 || max_rows > 65535) return BILD_EINVAL;
    bild_rules* r = new (std::nothrow) bild_rules();
    if (!r) return BILD_ENOMEM;
    r->vocab = vocab;
    r->max_rows = max_rows;
    const size_t counts = (sizeof(unsigned) * (size_t)max_rows + 255) / 256 * 256;
    int rc = BILD_OK;
    if (hipGetDevice(&r->device) != hipSuccess) rc = BILD_EHIP;
    else if (hipMalloc(&r->mem, counts + sizeof(StatPart) * parts_cap(max_rows, vocab)) != hipSuccess) r->mem = nullptr, rc = BILD_ENOMEM;
    else if (hipMemset(r->mem, 0, counts) != hipSuccess || hipStreamSynchronize(nullptr) != hipSuccess) rc = BILD_EHIP;
    if (rc != BILD_OK) {
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
    if ((c.tokens && (c.max_tokens < 0 || c.max_tokens > kMaxTokens)) || (c.bias_ids && (c.max_bias < 0 || c.max_bias > kMaxBias))) return BILD_EINVAL;
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
    a.parts = parts_of(c.rows, r->vocab);
    const OnDevice on(r->device);
    if (!on.ok) return BILD_EHIP;
    return launch_rules(a, (hipStream_t)hip_stream) == hipSuccess ? BILD_OK : BILD_EHIP;
}
