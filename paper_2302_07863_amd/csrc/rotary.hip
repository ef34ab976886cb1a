// Rotary positions of rows that the caller holds (bild_rotary_apply), and the frequencies that models share with it.
//
//   (u, v) -> m (u cos a - v sin a, u sin a + v cos a),  a = position * f_i
//
// Bound: memory, each row read and written once; the arithmetic is two products and a sum a value.  A workgroup takes the heads, or part of them, of as many tokens as
// give every thread one piece of 32 bytes.  A thread requests its piece and, while that is on its way, helps to form the tokens' cosines and sines, in 64 bits (an
// angle of 100 000 radians has no correct digit after the sixth in fp32), into LDS.
// us: 4096 tokens of 32 + 32 heads of 128 bf16 (134 MB) pairs 27.4, halves 26.1 (4.9, 5.1 TB/s; a copy of 512 MB reaches 5.4), 94 of 128 turned 34 and 38; 1531
// tokens of packed fp32 heads of 80, 32 turned, 6.0; one token 2.75 to 3.1.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "operators.h"
#include "rows_common.h"

using namespace bild;

namespace {

constexpr int kMaxHalf = 128;      // pairs of a head
constexpr int kThreads = 256;
constexpr int kMaxTokens = 16;     // tokens of a workgroup

struct RotaryArgs {
    const void* src[2];
    void* dst[2];
    int64_t src_token[2], src_head[2], dst_token[2], dst_head[2];
    const int* positions;
    int first, tokens;
    int heads_q, heads;   // of the first array, of both
    int half, rot, d_head;
    int pair_units, units;  // pieces of a head: of its turned part, of all that is written
    int tokens_per, heads_per;
    int again;              // values may be written twice
    unsigned units_m, slab_m;  // of units and units * heads_per (see divide)
    float sign;
    double magnitude;
    double frequency[kMaxHalf];
};

// u / d by a product with m = 2^32 / d rounded up (0: d is 1); exact for u and d below 2^16, since u * (m * d - 2^32) < 2^32.
__device__ __forceinline__ int divide(int u, unsigned m) { return m ? (int)__umulhi((unsigned)u, m) : u; }

// Cosine and sine in 64 bits, good to some 2^-36 (the results are rounded to fp32), of angles up to 2^48: the quarter turn nearest to the angle is taken off in two
// steps, each with one rounding, and what is left, at most pi / 4, goes into the Taylor series.  A third of the library's
// instructions, in a chain that every workgroup waits for.
__device__ __forceinline__ void turn_of(double angle, double& cs, double& sn) {
    const double k = rint(angle * 0.63661977236758134308);  // 2 / pi
    const double r = fma(-k, 6.123233995736766036e-17, fma(-k, 1.57079632679489661923, angle)), q = r * r;
    double s = fma(q, -2.50521083854417187751e-8, 2.75573192239858906526e-6);  // 1 / 11!, 1 / 9!
    s = fma(q, s, -1.98412698412698412698e-4);
    s = fma(q, s, 8.33333333333333333333e-3);
    s = fma(q, s, -0.166666666666666666667);
    s = fma(q * r, s, r);
    double c = fma(q, 2.08767569878680989792e-9, -2.75573192239858906526e-7);  // 1 / 12!, 1 / 10!
    c = fma(q, c, 2.48015873015873015873e-5);
    c = fma(q, c, -1.38888888888888888889e-3);
    c = fma(q, c, 4.16666666666666666667e-2);
    c = fma(q, c, -0.5);
    c = fma(q, c, 1.0);
    const int quarter = (int)(long long)k;
    const double x = quarter & 1 ? s : c, y = quarter & 1 ? c : s;
    cs = (quarter + 1) & 2 ? -x : x;
    sn = quarter & 2 ? -y : y;
}

// A piece of a head are two times 16 bytes: of first and of second halves, of pairs side by side, or of what lies behind the turned part.
template <class R, bool HALVES>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryArgs a) {
    constexpr int E = 16 / R::kBytes;
    typedef typename R::type V;
    typedef RowVec<R, E> Vec;
    __shared__ float2 turn[kMaxTokens * kMaxHalf];
    const int t0 = (int)blockIdx.x * a.tokens_per, nt = min(a.tokens_per, a.tokens - t0);
    const int h0 = (int)blockIdx.y * a.heads_per, nh = min(a.heads_per, a.heads - h0);
    const int slab = a.units * a.heads_per, count = nt * slab;
    struct Unit {
        Vec x, y;
        V* dst;
        int p;  // which of the head's
        int t;  // token; -1: nothing
    };
    // Where the two vectors of a piece begin and how many values they have (of neighbouring lanes either lie side by side).  The last vector of a part whose
    // length is no multiple of one begins earlier, and what it shares with its neighbour is written twice, the same both times; in place it is cut short.
    struct Place {
        int x, y, nx, ny;
    };
    const auto place = [&](int p) {
        int base = 0, len = a.rot, x = p * E, y = (p + a.pair_units) * E;
        if (p >= a.pair_units) {
            base = a.rot;
            len = a.d_head - a.rot;
            x -= a.pair_units * E;
            y = x + (a.units - a.pair_units) * E;
        } else if (HALVES) {
            len = a.half;
            y = x;
        }
        if (a.again && len >= E) {
            x = min(x, len - E);
            y = min(y, len - E);
        }
        return Place{base + x, base + y + (HALVES && base == 0 ? a.half : 0), len - x, len - y};
    };
    const auto request = [&](Unit& q, int u) {
        const int t = divide(u, a.slab_m), r = u - t * slab, hh = divide(r, a.units_m);
        q.t = -1;
        if (u >= count || hh >= nh) return;
        q.p = r - hh * a.units;
        q.t = t;
        const int head = h0 + hh, which = head >= a.heads_q, h = which ? head - a.heads_q : head;
        const V* src = (const V*)a.src[which] + (int64_t)(t0 + t) * a.src_token[which] + (int64_t)h * a.src_head[which];
        q.dst = (V*)a.dst[which] + (int64_t)(t0 + t) * a.dst_token[which] + (int64_t)h * a.dst_head[which];
        const Place at = place(q.p);
        if (at.ny >= E) {
            q.x.load(src + at.x);
            q.y.load(src + at.y);
        } else {
            q.x.load_some(src + at.x, at.nx);
            q.y.load_some(src + at.y, at.ny);
        }
    };
    const auto finish = [&](Unit& q) {
        if (q.t < 0) return;
        const Place at = place(q.p);
        if (q.p < a.pair_units) {
            const float2* tn = turn + q.t * a.half;
            const auto pair = [&](typename R::type& u, typename R::type& v, int i) {
                const float2 c = tn[min(i, a.half - 1)];
                const float fu = R::up(u), fv = R::up(v);
                u = R::down(fu * c.x - fv * c.y);
                v = R::down(fu * c.y + fv * c.x);
            };
#pragma unroll
            for (int i = 0; i < E; ++i) {
                if (HALVES) pair(q.x.v[i], q.y.v[i], at.x + i);
                else if (i < E / 2) pair(q.x.v[2 * i], q.x.v[2 * i + 1], at.x / 2 + i);
                else pair(q.y.v[2 * i - E], q.y.v[2 * i - E + 1], at.y / 2 + i - E / 2);
            }
        }
        if (at.ny >= E) {
            q.x.store(q.dst + at.x);
            q.y.store(q.dst + at.y);
        } else {
            q.x.store_some(q.dst + at.x, at.nx);
            q.y.store_some(q.dst + at.y, at.ny);
        }
    };
    Unit unit;
    request(unit, (int)threadIdx.x);
    __builtin_amdgcn_sched_barrier(0);
    // the rows are on their way meanwhile
    for (int e = threadIdx.x; e < nt * a.half; e += kThreads) {
        const int t = e / a.half, i = e - t * a.half;
        const int pos = a.positions ? a.positions[t0 + t] : a.first + t0 + t;
        double sn, cs;
        turn_of((double)pos * a.frequency[i], cs, sn);
        turn[e] = make_float2((float)(cs * a.magnitude), (float)(sn * a.magnitude) * a.sign);
    }
    lds_barrier();
    finish(unit);
}

__global__ __launch_bounds__(64) void rotary_table_kernel(double2* table, int pairs, const bild_rotary r) {
    const int pos = (int)blockIdx.x;
    for (int i = threadIdx.x; i < pairs; i += 64) {
        double sn = 0.0, cs = 1.0;
        if (2 * i < r.cfg.rot_dim) {
            sincos((double)pos * r.frequency[i], &sn, &cs);
            sn *= r.magnitude;
            cs *= r.magnitude;
        }
        table[(size_t)pos * pairs + i] = make_double2(cs, sn);
    }
}

template <class R>
hipError_t launch(const RotaryArgs& a, bool halves, hipStream_t st) {
    const dim3 grid((a.tokens + a.tokens_per - 1) / a.tokens_per, (a.heads + a.heads_per - 1) / a.heads_per);
    return launch_on(halves ? rotary_kernel<R, true> : rotary_kernel<R, false>, grid, dim3(kThreads), 0, st, a);
}

bool fields_ok(const bild_rotary_config& c) {
    if (c.layout != BILD_ROTARY_PAIRS && c.layout != BILD_ROTARY_HALVES) return false;
    if (c.rot_dim < 2 || c.rot_dim > 2 * kMaxHalf || c.rot_dim % 2) return false;
    if (c.scaling < BILD_ROTARY_NONE || c.scaling > BILD_ROTARY_YARN) return false;
    if (!(c.base > 0.f) || !std::isfinite(c.base)) return false;
    if (c.scaling == BILD_ROTARY_NONE) return true;
    if (!(c.factor >= 1.f) || !std::isfinite(c.factor)) return false;
    if (c.scaling < BILD_ROTARY_BANDS) return true;
    if (c.original < 1 || !std::isfinite(c.low) || !std::isfinite(c.high)) return false;
    if (!(c.low == 0.f && c.high == 0.f) && !(c.low > 0.f && c.high > c.low)) return false;
    if (c.scaling != BILD_ROTARY_YARN) return true;
    return c.base > 1.f && c.magnitude >= 0.f && std::isfinite(c.magnitude);
}

void frequencies(const bild_rotary_config& c, double* f, double* magnitude) {
    constexpr double kTurn = 6.283185307179586476925;
    const int rot = c.rot_dim, half = rot / 2;
    const double factor = c.factor;
    const bool given = c.low != 0.f || c.high != 0.f;
    const double low = given ? c.low : 1.0, high = given ? c.high : c.scaling == BILD_ROTARY_YARN ? 32.0 : 4.0;
    double base = c.base;
    // (one pair turns by one radian a position whatever the base)
    if (c.scaling == BILD_ROTARY_BASE && rot > 2) base *= std::pow(factor, (double)rot / (rot - 2));
    double first = 0, last = 0;
    if (c.scaling == BILD_ROTARY_YARN) {
        const auto pair_of = [&](double turns) { return rot * std::log(c.original / (turns * kTurn)) / (2 * std::log(base)); };
        first = std::max(std::floor(pair_of(high)), 0.0);
        last = std::min(std::ceil(pair_of(low)), rot - 1.0);
    }
    for (int i = 0; i < half; ++i) {
        const double g = std::pow(base, -2.0 * i / rot);
        double keep = 1.0;  // how much of g, against g / factor
        if (c.scaling == BILD_ROTARY_LINEAR) keep = 0.0;
        if (c.scaling == BILD_ROTARY_BANDS) keep = std::min(std::max((c.original * g / kTurn - low) / (high - low), 0.0), 1.0);
        if (c.scaling == BILD_ROTARY_YARN) keep = 1.0 - std::min(std::max((i - first) / std::max(last - first, 0.001), 0.0), 1.0);
        f[i] = c.scaling == BILD_ROTARY_NONE || c.scaling == BILD_ROTARY_BASE ? g : g * keep + g / factor * (1.0 - keep);
    }
    *magnitude = c.scaling != BILD_ROTARY_YARN ? 1.0 : c.magnitude > 0.f ? c.magnitude : 0.1 * std::log(factor) + 1.0;
}

// (turn_of's reduction: angles up to 2^48, of positions up to 2^31.  Only bases below one have such frequencies.)
constexpr double kMaxFrequency = 131072.0;
bool config_ok(const bild_rotary_config& c) {
    if (!fields_ok(c)) return false;
    double f[kMaxHalf], magnitude;
    frequencies(c, f, &magnitude);
    return std::all_of(f, f + c.rot_dim / 2, [](double v) { return v <= kMaxFrequency; });
}

bool rows_ok(const bild_rotary_rows& r) { return r.heads >= 0 && r.reserved == 0 && (r.heads == 0 || (r.src && r.dst)); }

}  // namespace

namespace bild {

hipError_t launch_rotary_table(double2* table, int positions, int d_head, const bild_rotary& r, hipStream_t st) {
    if (!table || positions < 1 || r.cfg.rot_dim > d_head) return hipErrorInvalidValue;
    return launch_on(rotary_table_kernel, dim3(positions), dim3(64), 0, st, table, d_head / 2, r);
}

}  // namespace bild

extern "C" int bild_rotary_frequencies(const bild_rotary_config* cfg, double* f, double* magnitude) {
    if (!cfg || !f || !config_ok(*cfg)) return BILD_EINVAL;
    double m;
    frequencies(*cfg, f, &m);
    if (magnitude) *magnitude = m;
    return BILD_OK;
}

extern "C" int bild_rotary_create(const bild_rotary_config* cfg, bild_rotary** out) {
    if (!cfg || !out || !config_ok(*cfg)) return BILD_EINVAL;
    bild_rotary* r = new (std::nothrow) bild_rotary();
    if (!r) return BILD_ENOMEM;
    r->cfg = *cfg;
    frequencies(*cfg, r->frequency, &r->magnitude);
    *out = r;
    return BILD_OK;
}

extern "C" int bild_rotary_destroy(bild_rotary* r) {
    if (!r) return BILD_EINVAL;
    delete r;
    return BILD_OK;
}

extern "C" int bild_rotary_apply(const bild_rotary* r, const bild_rotary_call* call, void* hip_stream) {
    if (!r || !call) return BILD_EINVAL;
    const bild_rotary_call& c = *call;
    const int rot = r->cfg.rot_dim;
    if (!rows_ok(c.q) || !rows_ok(c.k) || c.reserved != 0 || !row_type(c.dtype)) return BILD_EINVAL;
    if (c.tokens < 1 || c.d_head < rot || c.d_head > 1024) return BILD_EINVAL;
    const int64_t heads = (int64_t)c.q.heads + c.k.heads;
    if (heads < 1 || heads > 65535) return BILD_EINVAL;
    if (!c.positions && (int64_t)c.first + c.tokens - 1 > 0x7FFFFFFF) return BILD_EINVAL;
    RotaryArgs a;
    std::memset((void*)&a, 0, sizeof(a));
    const bild_rotary_rows* rows[2] = {&c.q, &c.k};
    bool in_place = true, any_in_place = false;
    for (int i = 0; i < 2; ++i) {
        const bild_rotary_rows& x = *rows[i];
        a.src[i] = x.src;
        a.dst[i] = x.dst;
        a.src_token[i] = x.src_token;
        a.src_head[i] = x.src_head;
        a.dst_token[i] = x.dst_token;
        a.dst_head[i] = x.dst_head;
        in_place = in_place && (x.heads == 0 || (x.src == x.dst && x.src_token == x.dst_token && x.src_head == x.dst_head));
        any_in_place = any_in_place || (x.heads > 0 && x.src == x.dst);
        if (x.heads > 0 && x.src == x.dst && ((c.tokens > 1 && x.src_token != x.dst_token) || (x.heads > 1 && x.src_head != x.dst_head))) return BILD_EINVAL;
    }
    a.positions = c.positions;
    a.first = c.first;
    a.tokens = c.tokens;
    a.heads_q = c.q.heads;
    a.heads = (int)heads;
    a.half = rot / 2;
    a.rot = rot;
    a.d_head = c.d_head;
    const int e = 16 / row_bytes(c.dtype);
    const bool halves = r->cfg.layout == BILD_ROTARY_HALVES;
    a.pair_units = (rot + 2 * e - 1) / (2 * e);
    a.units = a.pair_units + (in_place ? 0 : (c.d_head - rot + 2 * e - 1) / (2 * e));  // (in place the rest is there already)
    // a piece a thread (two of them: 26.2 against 25.4 us for 134 MB in halves, 3.5 against 2.8 for eleven tokens)
    a.again = !any_in_place;
    a.heads_per = std::min((int)heads, std::max(1, kThreads / a.units));
    a.tokens_per = std::min({c.tokens, kMaxTokens, std::max(1, kThreads / (a.units * a.heads_per))});
    const auto magic = [](int d) { return d == 1 ? 0u : (unsigned)((0xFFFFFFFFull + d) / d); };  // (at most a workgroup's 256 pieces and a head's 130: see divide)
    a.units_m = magic(a.units);
    a.slab_m = magic(a.units * a.heads_per);
    a.sign = c.inverse ? -1.f : 1.f;
    a.magnitude = r->magnitude;
    std::memcpy(a.frequency, r->frequency, sizeof(double) * (size_t)a.half);
    hipStream_t st = (hipStream_t)hip_stream;
    int device = 0;
    if (hipGetDevice(&device) != hipSuccess) return BILD_EHIP;
    if (st && hipStreamGetDevice(st, &device) != hipSuccess) return BILD_EHIP;
    const OnDevice on(device);
    if (!on.ok) return BILD_EHIP;
    const hipError_t err = c.dtype == BILD_DT_F32 ? launch<RowF32>(a, halves, st) : c.dtype == BILD_DT_BF16 ? launch<RowBf16>(a, halves, st) : launch<RowF16>(a, halves, st);
    return err == hipSuccess ? BILD_OK : BILD_EHIP;
}
