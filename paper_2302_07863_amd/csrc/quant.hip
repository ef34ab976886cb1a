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
// Layout: tiles of 16 features x 128 inputs, 1 KiB, in the order of the matrix cores' A operand: lane l has feature l % 16, its word j
// the inputs 32 j + 8 (l / 16) + 0 .. 7.  Of these, pair p (2p, 2p + 1) lies in the nibbles p and p + 4, the two halves of the word.  Scales (and
// zeros) of a tile: the four features of an accumulator's lane side by side, one such group per group of inputs.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <thread>
#include <vector>

#include "operators.h"
#include "rows_common.h"

using namespace bild;

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kTileK = 128;   // inputs of a tile
constexpr int kMaxWaves = 8;

// Rows as the matrix cores take them: bf16 and fp16 as they are; fp32, and rows with a norm's gain, as three bf16 parts.
enum RowsAs : int { AS_BF16 = 0, AS_F16 = 1, AS_PARTS = 2 };

struct QuantArgs {
    const uint4* codes;
    const uint16_t* scales;
    const uint8_t* zeros;
    const void* x;
    void* y;
    const float* gain;
    int64_t ldx, ldy;
    int n, k, tn, tk, rows;
    int x_dtype, y_dtype, bf16_scales;
    float eps, scale;
};

template <int AS>
__device__ __forceinline__ f32x4 mac(const uint4& a, const uint4& b, const f32x4& c) {
    if constexpr (AS == AS_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Eight codes as 1 + q / 16.
template <int AS>
__device__ __forceinline__ uint4 codes_up(uint32_t w) {
    if constexpr (AS == AS_F16) {
        constexpr uint32_t m = 0x03C003C0u, one = 0x3C003C00u;
        return make_uint4(((w << 6) & m) | one, ((w << 2) & m) | one, ((w >> 2) & m) | one, ((w >> 6) & m) | one);
    } else {
        constexpr uint32_t m = 0x00780078u, one = 0x3F803F80u;
        return make_uint4(((w << 3) & m) | one, ((w >> 1) & m) | one, ((w >> 5) & m) | one, ((w >> 9) & m) | one);
    }
}
// -(1 + z / 16), twice
template <int AS>
__device__ __forceinline__ uint32_t zero_up(uint32_t z) {
    const uint32_t h = AS == AS_F16 ? 0xBC00u | (z << 6) : 0xBF80u | (z << 3);
    return h | (h << 16);
}

// Eight values of a row in up to three parts that the matrix cores take.
template <int AS>
struct Frag {
    uint4 part[AS == AS_PARTS ? 3 : 1];
};

__device__ __forceinline__ void split3(const float (&v)[8], Frag<AS_PARTS>& f) {
    uint32_t p[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = v[2 * i], b = v[2 * i + 1];
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            const uint32_t h = pack_bf16x2(a, b);
            p[j][i] = h;
            a -= __uint_as_float(h << 16);
            b -= __uint_as_float(h & 0xFFFF0000u);
        }
    }
#pragma unroll
    for (int j = 0; j < 3; ++j) f.part[j] = make_uint4(p[j][0], p[j][1], p[j][2], p[j][3]);
}

template <class R>
__device__ __forceinline__ void up8(const R*, const void* row, int k0, int k, float (&v)[8]) {
    RowVec<R, 8> r;
    const typename R::type* p = (const typename R::type*)row + k0;
    if (k0 + 8 <= k) r.load(p); else r.load_some(p, k - k0);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = R::up(r.v[i]);
}

// Inputs k0 .. k0 + 7 of a row (zero from the k-th on); AS_PARTS: times the gain, squares added to ss.
template <int AS>
__device__ __forceinline__ void load_frag(const QuantArgs& a, const char* row, int k0, Frag<AS>& f, float& ss) {
    if constexpr (AS == AS_PARTS) {
        float v[8];
        if (a.x_dtype == BILD_DT_F32) up8((const RowF32*)nullptr, row, k0, a.k, v);
        else if (a.x_dtype == BILD_DT_BF16) up8((const RowBf16*)nullptr, row, k0, a.k, v);
        else up8((const RowF16*)nullptr, row, k0, a.k, v);
        if (a.gain) {
            float g[8];
            up8((const RowF32*)nullptr, a.gain, k0, a.k, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                ss = __builtin_fmaf(v[i], v[i], ss);
                v[i] *= g[i];
            }
        }
        split3(v, f);
    } else {
        RowVec<RowBf16, 8> r;  // (16 bits are 16 bits)
        const uint16_t* p = (const uint16_t*)row + k0;
        if (k0 + 8 <= a.k) r.load(p); else r.load_some(p, a.k - k0);
        __builtin_memcpy(&f.part[0], r.v, 16);
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

// NT row tiles of 16; the workgroup's waves share a feature tile, each takes every nw-th input tile of it.
template <int AS, int G, int NT>
__global__ __launch_bounds__(64 * kMaxWaves) void quant_kernel(const QuantArgs a) {
    constexpr int GT = kTileK / G;  // groups of a tile
    constexpr int SG = G / 32;      // steps of a group
    __shared__ f32x4 part[kMaxWaves][NT][64];
    __shared__ float squares[kMaxWaves][NT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = blockDim.x >> 6;
    const int ft = blockIdx.x, r0 = blockIdx.y * (16 * NT);
    const int xb = a.x_dtype == BILD_DT_F32 ? 4 : 2;
    const char* row[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) row[t] = (const char*)a.x + (int64_t)min(r0 + t * 16 + (lane & 15), a.rows - 1) * a.ldx * xb;
    f32x4 total[NT];
    float ss[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        total[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        ss[t] = 0.f;
    }
    for (int kt = wave; kt < a.tk; kt += nw) {
        const size_t tile = (size_t)ft * a.tk + kt;
        const uint4 c = a.codes[tile * 64 + lane];
        const uint32_t cw[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
        for (int g = 0; g < GT; ++g) {
            uint32_t zw = zero_up<AS>(8);
            if (a.zeros) zw = zero_up<AS>(a.zeros[((tile * 4 + ((lane & 15) >> 2)) * GT + g) * 4 + (lane & 3)]);
            const uint4 za = make_uint4(zw, zw, zw, zw);
            const uint2 sw = *(const uint2*)(a.scales + ((tile * 4 + (lane >> 4)) * GT + g) * 4);
            f32x4 acc[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < SG; ++s) {
                const int j = g * SG + s;
                const uint4 ca = codes_up<AS>(cw[j]);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    Frag<AS> f;
                    load_frag<AS>(a, row[t], kt * kTileK + j * 32 + 8 * (lane >> 4), f, ss[t]);
#pragma unroll
                    for (int p = (int)(sizeof(f) / 16) - 1; p >= 0; --p) {
                        acc[t] = mac<AS>(ca, f.part[p], acc[t]);
                        acc[t] = mac<AS>(za, f.part[p], acc[t]);
                    }
                }
            }
            const uint32_t sh[4] = {sw.x & 0xFFFFu, sw.x >> 16, sw.y & 0xFFFFu, sw.y >> 16};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float sv = a.bf16_scales ? bf2f(sh[i]) : RowF16::up((uint16_t)sh[i]);
#pragma unroll
                for (int t = 0; t < NT; ++t) total[t][i] = __builtin_fmaf(sv, acc[t][i], total[t][i]);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        part[wave][t][lane] = total[t];
        squares[wave][t][lane] = ss[t];
    }
    __syncthreads();
    for (int t = wave; t < NT; t += nw) {
        f32x4 sum = part[0][t][lane];
        for (int w = 1; w < nw; ++w) sum += part[w][t][lane];
        float f = 16.f * a.scale;
        if (a.gain) {  // (four lanes have a row's inputs)
            float q = 0.f;
            for (int w = 0; w < nw; ++w)
                for (int i = 0; i < 4; ++i) q += squares[w][t][(lane & 15) + 16 * i];
            f *= 1.f / sqrtf(q / (float)a.k + a.eps);
        }
        const int r = r0 + t * 16 + (lane & 15);
        if (r < a.rows) store_y(a, r, ft * 16 + 4 * (lane >> 4), sum * f);
    }
}

// From rows of codes (two a byte), scales and zeros to tiles.  A thread per lane and tile; `bad`: a zero above 15.
__global__ __launch_bounds__(256) void quant_layout_kernel(const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros, int n, int k, int group, int tk, size_t lanes,
                                                           uint32_t* to_codes, uint16_t* to_scales, uint8_t* to_zeros, unsigned* bad) {
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
            w |= (b & 15u) << (4 * p) | (b >> 4) << (4 * p + 16);
        }
        to_codes[at * 4 + j] = w;
    }
    const int gt = kTileK / group, groups = (k + group - 1) / group;
    if (lane < 16)  // feature `lane` of the tile
        for (int g = 0; g < gt; ++g) {
            const int gg = kt * gt + g;
            const bool in = f < n && gg < groups;
            const size_t to = ((tile * 4 + (lane >> 2)) * gt + g) * 4 + (lane & 3);
            to_scales[to] = in ? scales[(size_t)f * groups + gg] : (uint16_t)0;
            if (!zeros) continue;
            const unsigned z = in ? zeros[(size_t)f * groups + gg] : 0u;
            if (z > 15u) *bad = 1u;
            to_zeros[to] = (uint8_t)(z & 15u);
        }
}

template <int AS, int G>
void launch_rows(const QuantArgs& a, int waves, hipStream_t st) {
    if (a.rows <= 16) hipLaunchKernelGGL((quant_kernel<AS, G, 1>), dim3(a.tn), dim3(64 * waves), 0, st, a);
    else hipLaunchKernelGGL((quant_kernel<AS, G, 2>), dim3(a.tn, (a.rows + 31) / 32), dim3(64 * waves), 0, st, a);
}
template <int AS>
void launch_group(const QuantArgs& a, int group, int waves, hipStream_t st) {
    if (group == 32) launch_rows<AS, 32>(a, waves, st);
    else if (group == 64) launch_rows<AS, 64>(a, waves, st);
    else launch_rows<AS, 128>(a, waves, st);
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
    a.scales = w->scales;
    a.zeros = w->zeros;
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
    a.bf16_scales = w->bf16_scales;
    a.eps = c.eps;
    a.scale = c.scale;
    const int waves = std::max(1, std::min(kMaxWaves, w->tk));
    if (c.gain || c.x_dtype == BILD_DT_F32) launch_group<AS_PARTS>(a, w->group, waves, st);
    else if (c.x_dtype == BILD_DT_F16) launch_group<AS_F16>(a, w->group, waves, st);
    else launch_group<AS_BF16>(a, w->group, waves, st);
    return hipGetLastError() == hipSuccess ? BILD_OK : BILD_EHIP;
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
    q->bf16_scales = scale_dtype == BILD_DT_BF16;
    const size_t tiles = (size_t)q->tn * q->tk, tile_scales = 16 * (size_t)(kTileK / group);
    const size_t groups = (size_t)(k + group - 1) / group;
    // what stays, and behind it what was given
    const size_t code_bytes = tiles * 1024, scale_bytes = (tiles * tile_scales * 2 + 255) / 256 * 256, zero_bytes = zeros ? (tiles * tile_scales + 255) / 256 * 256 : 0;
    const size_t raw_codes = (size_t)n * ((k + 1) / 2), raw_scales = (size_t)n * groups * 2, raw_zeros = zeros ? (size_t)n * groups : 0;
    const size_t scales_at = (raw_codes + 255) / 256 * 256, zeros_at = scales_at + (raw_scales + 255) / 256 * 256, bad_at = zeros_at + (raw_zeros + 255) / 256 * 256;
    char* raw = nullptr;
    int rc = BILD_OK;
    if (hipGetDevice(&q->device) != hipSuccess) rc = BILD_EHIP;
    else if (hipMalloc(&q->mem, code_bytes + scale_bytes + zero_bytes) != hipSuccess) q->mem = nullptr, rc = BILD_ENOMEM;
    else if (hipMalloc((void**)&raw, bad_at + 256) != hipSuccess) raw = nullptr, rc = BILD_ENOMEM;
    if (rc == BILD_OK) {
        q->codes = (const uint4*)q->mem;
        q->scales = (const uint16_t*)((char*)q->mem + code_bytes);
        q->zeros = zeros ? (const uint8_t*)q->mem + code_bytes + scale_bytes : nullptr;
        unsigned bad = 0;
        bool ok = hipMemcpy(raw, codes, raw_codes, hipMemcpyDefault) == hipSuccess && hipMemcpy(raw + scales_at, scales, raw_scales, hipMemcpyDefault) == hipSuccess &&
                  (!zeros || hipMemcpy(raw + zeros_at, zeros, raw_zeros, hipMemcpyDefault) == hipSuccess) && hipMemset(raw + bad_at, 0, sizeof(unsigned)) == hipSuccess;
        if (ok) {
            const size_t lanes = tiles * 64;
            hipLaunchKernelGGL(quant_layout_kernel, dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0, nullptr, (const uint8_t*)raw, (const uint16_t*)(raw + scales_at),
                               zeros ? (const uint8_t*)(raw + zeros_at) : nullptr, n, k, group, q->tk, lanes, (uint32_t*)q->codes, (uint16_t*)q->scales,
                               (uint8_t*)q->zeros, (unsigned*)(raw + bad_at));
            ok = hipGetLastError() == hipSuccess && hipMemcpy(&bad, raw + bad_at, sizeof(bad), hipMemcpyDeviceToHost) == hipSuccess;
        }
        rc = !ok ? BILD_EHIP : bad ? BILD_EINVAL : BILD_OK;
    }
    if (raw) (void)hipFree(raw);
    if (rc != BILD_OK) {
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
