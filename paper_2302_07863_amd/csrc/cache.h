// The cache in 8 bits as its kernels see it (cache.hip: pages and appending; cache_attend.hip: attention).
#pragma once
#include <algorithm>

#include "operators.h"

namespace bild {

// The caller's arrays and their sizes, as kernel arguments.
struct CacheView {
    int8_t* codes;
    float* scales;
    int* table;
    int* lengths;
    int* refs;
    int pages, page_tokens, page_shift, layers, heads, d_head, sequences, max_pages;

    __host__ __device__ int cap() const { return max_pages << page_shift; }
    // of page p: keys (which 0) or values of a layer and key head
    __host__ __device__ int64_t plane(int p, int layer, int which, int head) const {
        return (((int64_t)p * layers + layer) * 2 + which) * heads + head;
    }
    __host__ __device__ int plane_bytes() const { return page_tokens * d_head; }
    __device__ bool has(int p) const { return (unsigned)p < (unsigned)pages; }
};

// Which sequences a call is about, and how many rows each has.
struct CacheRows {
    const int *sequences, *starts;
    int n, rows, tokens;

    __device__ int sequence(int i, int all) const {  // -1: passed over
        const int s = sequences ? sequences[i] : i;
        return (unsigned)s < (unsigned)all ? s : -1;
    }
    // first row and count of entry i, within 0 .. tokens
    __device__ void span(int i, int& first, int& count) const {
        if (!starts) {
            first = i * rows;
            count = rows;
            return;
        }
        first = min(max(starts[i], 0), tokens);
        count = min(max(starts[i + 1], first), tokens) - first;
    }
};

constexpr int kMaxLimit = 16777216;       // of lists and pools: 2^24
constexpr int kMaxGroups = kMaxLimit - 1;  // workgroups in a direction: their threads are counted in 32 bits

}  // namespace bild

struct bild_cache {
    bild::CacheView view = {};
    int device = 0;
    void* mem = nullptr;
    // cache.hip: see there
    int *plan = nullptr, *fresh = nullptr, *asked = nullptr, *latest = nullptr, *rows = nullptr, *moves = nullptr, *words = nullptr;
    // cache_attend.hip: partial results and counts of arrivals
    float* part = nullptr;
    unsigned* arrived = nullptr;
};

namespace bild {

// Workgroups of a launch: one a compute unit, and one a key head at least.  One more than there are units and it would take twice the time (us, call, 264 / 252 of them: 16 sequences of 3000
// positions, 12 key heads of 128 61 / 43; 280 / 240: 4 of 8000, 40 key heads 101 / 72).
constexpr int kAttendGroups = 256;
inline int attend_groups(int heads) { return std::max(kAttendGroups / heads, 1); }  // of a key head
hipError_t attend_init(int d_head);                      // what its kernels need of the current device
size_t attend_part_floats(int heads, int d_head);        // of bild_cache::part
constexpr int kPromptParts = 512;                        // most workgroups of a launch that shares the keys of tiles of prompts: two a compute unit
inline size_t attend_counts(int heads) { return std::max((size_t)heads * attend_groups(heads), (size_t)kPromptParts); }

}  // namespace bild
