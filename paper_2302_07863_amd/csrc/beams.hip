// The best continuations over beams and vocabulary (bild_beams_select), and the beams' histories in their new order.
//
//   rank(b, v) = (score_b + z_bv - lse_b) / length^penalty, the `choices` largest, of equals the lower (b, v)
//
// Bound: memory, every logit read once.  The first kernel reads them: for the softmax's sum, and for the largest of each chunk of 64 consecutive 16-byte pieces.  The k best
// lie in chunks whose maxima are among the k best maxima, so the second kernel, a workgroup a group of beams, looks at some thousand maxima and reads few chunks again.
// What is chosen is decided in 64 bits (of the fp32 sums): a threshold that k maxima reach is taken in fp32, to which ranks are rounded monotonically, so that it loses
// nobody; who reaches it is listed and each counts how many are better.  Lists that are too long are left for a walk in the order of the ids, one workgroup an entry of the batch: right, and slow.
// They are too long where thousands of ranks are equal (flat logits), and where the threshold is low because maxima are taken in groups, each of one beam: where few beams live (a search's first step;
// with fewer than 2 of 8 beams for 16 choices, 4 of 32 for 64, there are not as many groups as choices and no threshold), or most of what is chosen goes on from few beams.  us, a call: 8 beams of 250112
// ids, 16 choices 15, with one living beam 234; 32 beams, 64 choices with scores 0.7 apart from beam to beam 156, with four living 779; of 32128 ids 13, 110, 53, 327.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "operators.h"
#include "rows_common.h"

using namespace bild;

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64, kMaxPieces = 2;
constexpr int kPickThreads = 1024, kPickWaves = kPickThreads / 64;
constexpr int kMaxBeams = 64, kMaxChoices = 64;
constexpr int kListed = 1024;  // candidates, chunks of a list

struct BeamsArgs {
    const void* logits;
    int64_t ld;
    const float* scores;
    const int *lengths, *finished;
    float* out_scores;
    int *out_parents, *out_tokens, *out_lengths, *out_finished;
    const int* history;
    int64_t history_ld;
    int* out_history;
    int64_t out_history_ld;
    int vocab, beams, choices, eos, pad, steps;
    float penalty;
    int parts;     // workgroups of a row
    int chunks;    // of a row
    float* tops;   // [rows][chunks]
    float2* sums;  // [rows][parts][waves]: maximum and sum of e^(z - maximum)
};

template <class R>
struct Piece16 {
    static constexpr int E = 16 / R::kBytes;
    float z[E];
    // the piece at id i of a row of `vocab`; ids behind its end are -infinity
    __device__ __forceinline__ void load(const typename R::type* row, int i, int vocab) {
        RowVec<R, E> x;
        if (i + E <= vocab) {
            x.load(row + i);
#pragma unroll
            for (int e = 0; e < E; ++e) z[e] = R::up(x.v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) z[e] = i + e < vocab ? R::up(row[i + e]) : -INFINITY;
        }
    }
};

// P pieces a thread, a workgroup's width apart: a wave's piece is a chunk.  Bound: memory and, beside it, an exponential a logit: 128 rows of 250112 bf16 (64 MB) 14.6 us, 4.4 TB/s.
template <class R, int P>
__global__ __launch_bounds__(kThreads) void beams_read_kernel(const BeamsArgs a) {
    constexpr int E = 16 / R::kBytes;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = blockIdx.y;
    const typename R::type* in = (const typename R::type*)a.logits + (int64_t)row * a.ld;
    const int first = blockIdx.x * (P * kThreads * E);
    Piece16<R> x[P];
#pragma unroll
    for (int p = 0; p < P; ++p) x[p].load(in, first + (p * kThreads + tid) * E, a.vocab);
    float top = -INFINITY, mine[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        float m = x[p].z[0];
#pragma unroll
        for (int e = 1; e < E; ++e) m = fmaxf(m, x[p].z[e]);
        m = wave_max(m);
        mine[p] = m;
        top = fmaxf(top, m);
    }
    float s = 0.f;
    if (fabsf(top) < kFar || top == -INFINITY) {
        const float whole = whole_above(top);
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < E; ++e) s += term(x[p].z[e], whole);
        s = to_base(wave_sum(s), top);
    } else {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < E; ++e) s += fexp_full(x[p].z[e] - top);
        s = wave_sum(s);
    }
    if (lane == 0) {
        a.sums[((int64_t)row * a.parts + blockIdx.x) * kWaves + wave] = make_float2(top, s);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int chunk = (blockIdx.x * P + p) * kWaves + wave;
            if (chunk < a.chunks) a.tops[(int64_t)row * a.chunks + chunk] = mine[p];
        }
    }
}

struct Candidate {
    double rank;
    float z;
    int beam, id, unused;
};
__device__ __forceinline__ bool better(const Candidate& x, const Candidate& y) {
    return x.rank > y.rank || (x.rank == y.rank && (x.beam < y.beam || (x.beam == y.beam && x.id < y.id)));
}

// The choice: one workgroup an entry of the batch.  Bound: a chain of meetings (sums, maxima, threshold, chunks, ranks, histories): 4 beams of 32128 ids 7.2 us, 16 entries of 8 beams of 250112 13.8,
// 4 of 32 beams and 64 choices 27.
template <class R>
__global__ __launch_bounds__(kPickThreads) void beams_pick_kernel(const BeamsArgs a) {
    constexpr int E = 16 / R::kBytes, CHUNK = 64 * E, KEPT = 4;  // maxima that a thread keeps from the first pass over them for the second
    typedef typename R::type V;
    __shared__ double base[kMaxBeams], over[kMaxBeams];  // rank = (base + z) / over
    __shared__ float base_f[kMaxBeams], by_f[kMaxBeams]; // nearly: (base_f + z) * by_f
    __shared__ float group_tops[kPickThreads / 4], reach;
    __shared__ int n_chunks, n_list, far;
    __shared__ int chunk_list[kListed];
    __shared__ Candidate list[kListed + kMaxChoices + kMaxBeams];
    __shared__ Candidate best[kMaxChoices];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t row0 = (int64_t)blockIdx.x * a.beams;
    const V* logits = (const V*)a.logits + row0 * a.ld;
    const int chunks = a.chunks, all = a.beams * chunks;
    const float* tops = a.tops + row0 * chunks;
    if (tid == 0) n_chunks = n_list = far = 0;
    lds_barrier();
    // Groups of 16 or 4 lanes: four times as many as choices at least, or the threshold would be among the low ones of their maxima (of beams that offer nothing they are empty: see the top).  A wave
    // looks at the maxima of a slice of a beam's chunks, neighbours in groups apart.
    const int width = a.choices <= 16 ? 16 : 4, groups = kPickThreads / width;
    const int slices = (kPickWaves + a.beams - 1) / a.beams, pairs = a.beams * slices, per = (chunks + slices - 1) / slices, swapped = lane / width + 64 / width * (lane & (width - 1));
    const auto each = [&](int pair, auto&& f) {  // f(beam, chunk of it)
        const int b = pair / slices, c0 = (pair - b * slices) * per, c1 = min(c0 + per, chunks);
        for (int c = c0 + swapped; c < c1; c += 64) f(b, c);
    };
    float kept[KEPT];  // of the wave's first pair
    {
        const int b = wave / slices, c0 = (wave - b * slices) * per + swapped;
#pragma unroll
        for (int k = 0; k < KEPT; ++k) kept[k] = tops[min(b * chunks + c0 + 64 * k, all - 1)];
    }
    // ---- what each beam's logits are ranked by: a wave a beam for the sums, then a lane a beam; one wave has what their lengths count for, a lane a beam
    if (wave == kPickWaves - 1 && lane < a.beams) {
        const bool ended = a.finished && a.finished[row0 + lane] != 0;
        const int length = a.lengths ? a.lengths[row0 + lane] : 0;
        const double to = a.penalty == 0.f ? 1.0 : exp((double)a.penalty * log((double)max(ended ? length : length + 1, 1)));
        over[lane] = to;
        by_f[lane] = (float)(1.0 / to);
        if (!ended && !(to < 1e30 && to > 1e-30)) far = 1;  // (beyond what fp32 can sort)
    }
    {
        const int n = a.parts * kWaves;
        const auto part_of = [&](int b) { return a.sums + (row0 + b) * a.parts * kWaves; };
        float2 x[KEPT];
        const auto load = [&](int b) {
#pragma unroll
            for (int k = 0; k < KEPT; ++k) x[k] = part_of(b)[min(lane + 64 * k, n - 1)];
        };
        if (wave < a.beams) load(wave);
        for (int b = wave; b < a.beams; b += kPickWaves) {
            const float2* part = part_of(b);
            float m = -INFINITY;
#pragma unroll
            for (int k = 0; k < KEPT; ++k) m = fmaxf(m, x[k].x);
            for (int p = lane + 64 * KEPT; p < n; p += 64) m = fmaxf(m, part[p].x);
            m = wave_max(m);
            const float from = m == -INFINITY ? 0.f : m;
            double s = 0.0;
#pragma unroll
            for (int k = 0; k < KEPT; ++k)
                if (lane + 64 * k < n) s += (double)(x[k].y * fexp_full(x[k].x - from));
            for (int p = lane + 64 * KEPT; p < n; p += 64) s += (double)(part[p].y * fexp_full(part[p].x - from));
            if (b + kPickWaves < a.beams) load(b + kPickWaves);
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
            if (lane == 0) {
                base_f[b] = m;
                base[b] = s;
            }
        }
    }
    const float score = wave == 0 && lane < a.beams ? a.scores[row0 + lane] : 0.f;
    const bool goes_on = wave == 0 && lane < a.beams && !(a.finished && a.finished[row0 + lane] != 0);
    lds_barrier();
    if (wave == 0 && lane < a.beams) {
        const double at = (double)score - ((double)base_f[lane] + log(base[lane]));
        const bool live = goes_on && fabs(at) < INFINITY;
        base[lane] = live ? at : NAN;  // (NaN: this beam's logits offer nothing)
        base_f[lane] = live ? (float)at : NAN;
        if (live && !(fabs(at) < 1e30)) far = 1;
    }
    lds_barrier();
    const auto rank_of = [&](int b, float z) { return (base[b] + (double)z) / over[b]; };
    // ---- a rank that `choices` chunks reach: of groups' maxima the choices-th.  In fp32: a sum, a product and what the numbers in them are rounded by are off by less than
    // 2^-21 of the largest of them, so that who is below it by twice that is not among the best.
    // (least: -infinity where there are not as many groups; sums beyond fp32 stay in)
    const auto nearly = [&](int b, float z) { return (base_f[b] + z) * by_f[b]; };
    const auto slack = [&](int b, float z) { return (fabsf(base_f[b]) + fabsf(z)) * by_f[b] * 9.5367431640625e-7f; };  // 2^-20
    const auto may = [&](int b, float z, float least) { return z > -INFINITY && base_f[b] == base_f[b] && !(nearly(b, z) + slack(b, z) < least); };
    float top = -INFINITY;
    for (int pair = wave; pair < pairs; pair += kPickWaves)
        each(pair, [&](int b, int c) {
            const int k = (c - swapped - (pair % slices) * per) >> 6;
            const float z = pair == wave && k < KEPT ? (k == 0 ? kept[0] : k == 1 ? kept[1] : k == 2 ? kept[2] : kept[3]) : tops[b * chunks + c];
            top = fmaxf(top, nearly(b, z) - slack(b, z));
        });
    for (int o = width / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    if ((lane & (width - 1)) == 0) group_tops[tid / width] = top;
    lds_barrier();
    {  // the group's threads count who is before it
        const int group = tid / width;
        const float mine = group_tops[group];
        int before = 0;
        for (int other = tid & (width - 1); other < groups; other += width) {
            const float z = group_tops[other];
            before += z > mine || (z == mine && other < group);
        }
        for (int o = width / 2; o > 0; o >>= 1) before += __shfl_xor(before, o, 64);
        if (before == a.choices - 1 && (tid & (width - 1)) == 0) reach = mine;
    }
    lds_barrier();
    const float least = reach;
    for (int pair = wave; pair < pairs; pair += kPickWaves)
        each(pair, [&](int b, int c) {
            const int k = (c - swapped - (pair % slices) * per) >> 6;
            const float z = pair == wave && k < KEPT ? (k == 0 ? kept[0] : k == 1 ? kept[1] : k == 2 ? kept[2] : kept[3]) : tops[b * chunks + c];
            if (may(b, z, least)) {
                const int at = atomicAdd(&n_chunks, 1);
                if (at < kListed) chunk_list[at] = b * chunks + c;
            }
        });
    lds_barrier();
    const int found = far ? kListed + 1 : n_chunks;
    if (found <= kListed)
        for (int u = wave; u < found; u += kPickWaves) {
            const int c = chunk_list[u], b = c / chunks, i = (c - b * chunks) * CHUNK + lane * E;
            Piece16<R> x;
            x.load(logits + (int64_t)b * a.ld, i, a.vocab);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (i + e < a.vocab && may(b, x.z[e], least)) {
                    const int at = atomicAdd(&n_list, 1);
                    if (at < kListed) list[at] = {rank_of(b, x.z[e]), x.z[e], b, i + e, 0};
                }
            }
        }
    lds_barrier();
    // beams that have ended
    const auto ended_beams = [&] {
        if (tid < a.beams && a.finished && a.finished[row0 + tid] != 0) {
            const float score = a.scores[row0 + tid];
            const double r = (double)score / over[tid];
            if (r > -INFINITY) list[atomicAdd(&n_list, 1)] = {r, score, tid, a.pad, 0};
        }
    };
    // the first of the list in order, `best`; afterwards they are the list.  32 threads count who is before one of them.
    const auto settle = [&](int n) {
        for (int u = tid >> 5; u < n; u += kPickThreads / 32) {
            const Candidate mine = list[u];
            int before = 0;
            for (int k0 = 0; k0 < n; k0 += 32) {
                const int k = k0 + (tid & 31);
                before += __builtin_popcountll(__ballot(k < n && better(list[min(k, n - 1)], mine)) >> (lane & 32) & 0xFFFFFFFF);
            }
            if (before < a.choices && (tid & 31) == 0) best[before] = mine;
        }
        __syncthreads();
    };
    if (found <= kListed && n_list <= kListed) {
        lds_barrier();  // (everybody has seen the list's length)
        ended_beams();
        __syncthreads();
        settle(n_list);
    } else {
        // chunk by chunk in the order of their ids: who is not better than the last of the best so far comes too late
        __syncthreads();
        if (tid == 0) n_list = 0;
        __syncthreads();
        ended_beams();
        __syncthreads();
        settle(n_list);
        int n = min(n_list, a.choices);
        for (int u0 = 0; u0 < all; u0 += 64) {
            __syncthreads();
            const int mine = u0 + lane;
            // (the best that a chunk can have: its largest at its first id)
            const auto hopes = [&](int v) {
                const Candidate x = {rank_of(v / chunks, tops[v]), 0.f, v / chunks, v % chunks * CHUNK, 0};
                return x.rank > -INFINITY && (n < a.choices || better(x, best[n - 1]));
            };
            // (the list changes from chunk to chunk: looked at again where it is a chunk's turn)
            for (unsigned long long todo = __ballot(mine < all && hopes(min(mine, all - 1))); todo; todo &= todo - 1) {
                const int u = u0 + (int)__builtin_ctzll(todo), b = u / chunks, i = (u - b * chunks) * CHUNK;
                if (!hopes(u)) continue;
                if (tid < n) list[tid] = best[tid];
                if (tid == 0) n_list = n;
                __syncthreads();
                for (int at = i + tid; at < min(i + CHUNK, a.vocab); at += kPickThreads) {
                    const float z = R::up(logits[(int64_t)b * a.ld + at]);
                    const Candidate x = {rank_of(b, z), z, b, at, 0};
                    if (x.rank > -INFINITY && (n < a.choices || better(x, best[n - 1]))) list[atomicAdd(&n_list, 1)] = x;
                }
                __syncthreads();
                settle(n_list);
                n = min(n_list, a.choices);
                __syncthreads();
            }
        }
        if (tid == 0) n_list = n;
        __syncthreads();
    }
    // ---- results
    const int have = min(n_list, a.choices);
    const int64_t out0 = (int64_t)blockIdx.x * a.choices;
    if (tid < a.choices) {
        const bool none = tid >= have;
        const Candidate x = none ? Candidate{0.0, 0.f, -1, -1, 0} : best[tid];
        const bool ended = !none && a.finished && a.finished[row0 + x.beam] != 0;
        const int length = none || !a.lengths ? 0 : a.lengths[row0 + x.beam];
        const double sum = none ? -INFINITY : ended ? (double)x.z : base[x.beam] + (double)x.z;  // (of one that has ended z is its score)
        a.out_scores[out0 + tid] = (float)sum;
        a.out_parents[out0 + tid] = x.beam;
        a.out_tokens[out0 + tid] = x.id;
        if (a.out_lengths) a.out_lengths[out0 + tid] = none ? 0 : ended ? length : length + 1;
        if (a.out_finished) a.out_finished[out0 + tid] = none || ended || x.id == a.eos;
    }
    if (a.history)
        for (int k = wave; k < a.choices; k += kPickWaves) {
            const int b = k < have ? best[k].beam : -1;
            int* out = a.out_history + (out0 + k) * a.out_history_ld;
            const int* in = a.history + (row0 + max(b, 0)) * a.history_ld;
            for (int t = lane; t < a.steps; t += 64) out[t] = b < 0 ? -1 : in[t];
            if (lane == 0) out[a.steps] = b < 0 ? -1 : best[k].id;
        }
}

// Pieces a thread: two, one where that gives the chip too few workgroups (128 rows of 250112 bf16: four 13.8 us, eight 16, two 13).
int pieces_of(int rows, int vocab, int e) {
    int p = kMaxPieces;
    while (p > 1 && (int64_t)rows * ((vocab + p * kThreads * e - 1) / (p * kThreads * e)) < 512) p /= 2;
    return p;
}
template <class R>
hipError_t launch(BeamsArgs a, int batch, hipStream_t st) {
    constexpr int E = 16 / R::kBytes;
    const int rows = batch * a.beams, p = pieces_of(rows, a.vocab, E);
    a.parts = (a.vocab + p * kThreads * E - 1) / (p * kThreads * E);
    a.chunks = (a.vocab + 64 * E - 1) / (64 * E);
    const dim3 grid(a.parts, rows);
    const hipError_t err = p == 2 ? launch_on(beams_read_kernel<R, 2>, grid, dim3(kThreads), 0, st, a) : launch_on(beams_read_kernel<R, 1>, grid, dim3(kThreads), 0, st, a);
    if (err != hipSuccess) return err;
    return launch_on(beams_pick_kernel<R>, dim3(batch), dim3(kPickThreads), 0, st, a);
}

}  // namespace

struct bild_beams {
    int vocab = 0, max_batch = 0, beams = 0, device = 0;
    void* mem = nullptr;
    float2* sums = nullptr;
    float* tops = nullptr;
};

extern "C" int bild_beams_create(int vocab, int max_batch, int beams, bild_beams** out) {
    if (!out || vocab < 1 || vocab > (1 << 24) || max_batch < 1 || beams < 1 || beams > kMaxBeams || (int64_t)max_batch * beams > 65535) return BILD_EINVAL;
    bild_beams* b = new (std::nothrow) bild_beams();
    if (!b) return BILD_ENOMEM;
    b->vocab = vocab;
    b->max_batch = max_batch;
    b->beams = beams;
    // (fp32: the smallest pieces)
    const size_t rows = (size_t)max_batch * beams, chunks = ((size_t)vocab + 255) / 256, sums = rows * ((chunks + kWaves - 1) / kWaves) * kWaves;
    int rc = BILD_OK;
    if (hipGetDevice(&b->device) != hipSuccess) rc = BILD_EHIP;
    else if (hipMalloc(&b->mem, sums * sizeof(float2) + rows * chunks * sizeof(float)) != hipSuccess) b->mem = nullptr, rc = BILD_ENOMEM;
    if (rc != BILD_OK) {
        (void)hipGetLastError();  // (told by rc: not to be found by a later call as well)
        (void)bild_beams_destroy(b);
        return rc;
    }
    b->sums = (float2*)b->mem;
    b->tops = (float*)(b->sums + sums);
    *out = b;
    return BILD_OK;
}

extern "C" int bild_beams_destroy(bild_beams* b) {
    if (!b) return BILD_EINVAL;
    if (b->mem) (void)hipFree(b->mem);
    delete b;
    return BILD_OK;
}

extern "C" int bild_beams_select(bild_beams* b, const bild_beams_call* call, void* hip_stream) {
    if (!b || !call) return BILD_EINVAL;
    const bild_beams_call& c = *call;
    if (!c.logits || !c.scores || !c.out_scores || !c.out_parents || !c.out_tokens || !row_type(c.dtype) || c.reserved != 0) return BILD_EINVAL;
    if (c.batch < 1 || c.choices < 1 || c.choices > kMaxChoices || !std::isfinite(c.penalty) || c.steps < 0) return BILD_EINVAL;
    if ((c.history != nullptr) != (c.out_history != nullptr)) return BILD_EINVAL;
    if (c.finished && (c.pad < 0 || c.pad >= b->vocab)) return BILD_EINVAL;
    if (c.batch > b->max_batch) return BILD_ECAP;
    BeamsArgs a;
    std::memset((void*)&a, 0, sizeof(a));
    a.logits = c.logits;
    a.ld = c.logits_stride;
    a.scores = c.scores;
    a.lengths = c.lengths;
    a.finished = c.finished;
    a.out_scores = c.out_scores;
    a.out_parents = c.out_parents;
    a.out_tokens = c.out_tokens;
    a.out_lengths = c.out_lengths;
    a.out_finished = c.out_finished;
    a.history = c.history;
    a.history_ld = c.history_stride;
    a.out_history = c.out_history;
    a.out_history_ld = c.out_history_stride;
    a.vocab = b->vocab;
    a.beams = b->beams;
    a.choices = c.choices;
    a.eos = c.eos;
    a.pad = c.pad;
    a.steps = c.steps;
    a.penalty = c.penalty;
    a.sums = b->sums;
    a.tops = b->tops;
    const OnDevice on(b->device);
    if (!on.ok) return BILD_EHIP;
    hipStream_t st = (hipStream_t)hip_stream;
    const hipError_t err = c.dtype == BILD_DT_F32 ? launch<RowF32>(a, c.batch, st) : c.dtype == BILD_DT_BF16 ? launch<RowBf16>(a, c.batch, st) : launch<RowF16>(a, c.batch, st);
    return err == hipSuccess ? BILD_OK : BILD_EHIP;
}
