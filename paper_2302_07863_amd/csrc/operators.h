// What the operators on rows (quant.hip, rotary.hip, rules.hip) share with each other and with the decoder passes.
#pragma once
#include "bild_internal.h"

// A matrix in 4 bits: tiles of 16 features x 128 inputs in the order the matrix cores take them.
struct bild_quant {
    int n = 0, k = 0, group = 0;
    int tn = 0, tk = 0;        // feature tiles, input tiles
    int scale_exponent = 0;    // the scales are those stored times 2^this
    void* mem = nullptr;       // one allocation
    const uint4* codes = nullptr;     // [tn][tk][64 lanes]: see quant.hip
    const uint32_t* sides = nullptr;  // [tn][tk][16 features]: fp16 scales and zeros
    const void* nothing = nullptr;    // 256 bytes of zeros
    int device = 0;
};

struct bild_rotary {
    bild_rotary_config cfg;
    double frequency[128];
    double magnitude;
};

namespace bild {

constexpr int kMaxRuleTokens = (1 << 20) - 1, kMaxBiases = 1023;  // of a row (see rules.hip)

// Runs what follows on `device` and puts the caller's current device back.
class OnDevice {
    int was = -1;

public:
    bool ok;
    explicit OnDevice(int device) {
        int now = -1;
        ok = hipGetDevice(&now) == hipSuccess;
        if (ok && now != device) {
            ok = hipSetDevice(device) == hipSuccess;
            if (ok) was = now;
        }
    }
    ~OnDevice() {
        if (was >= 0) (void)hipSetDevice(was);
    }
    OnDevice(const OnDevice&) = delete;
};

// Launches a kernel and returns that launch's own status (hipGetLastError would also give what an earlier call, the caller's perhaps, has left).
template <class T>
struct As {
    typedef T type;
};
template <class... P>
hipError_t launch_on(void (*kernel)(P...), dim3 grid, dim3 block, size_t lds, hipStream_t st, const typename As<P>::type&... a) {
    void* args[] = {(void*)&a...};
    return hipLaunchKernel((const void*)kernel, grid, block, args, lds, st);
}

inline int row_bytes(int dtype) { return dtype == BILD_DT_F32 ? 4 : 2; }
inline bool row_type(int dtype) { return dtype == BILD_DT_F32 || dtype == BILD_DT_BF16 || dtype == BILD_DT_F16; }

// cos and sin of the positions from 0 on, times the magnitude, as the passes' kernels read them: [position][d_head / 2] pairs, those
// behind rot_dim not turned.
hipError_t launch_rotary_table(double2* table, int positions, int d_head, const bild_rotary& r, hipStream_t st);

int launch_quant(const bild_quant* w, const bild_quant_call& c, hipStream_t st);

// Rules on the logits of a row (bild_rules_call), as kernel arguments.
struct RulesArgs {
    const void* logits;
    void* out;
    int64_t ld, ldo;
    const int* targets;
    bild_row_stats* stats;
    const int* tokens;
    int64_t tokens_stride;
    const int *lengths, *starts;
    const bild_penalties* penalties;
    int64_t penalties_stride;
    const int* bias_ids;
    const float* bias;
    int64_t bias_stride;
    const int* bias_counts;
    const uint32_t* mask;
    int64_t mask_stride;
    int rows, vocab, dtype, max_tokens, max_bias;
    int parts, range;   // workgroups of a row, ids of each
    StatPart* part;     // [row][parts]
    // Rows of a decoder pass: row r stands at position *len_ptr + len_add + r of the sequence `tokens` (penalties: what stands up to there; those of
    // generated tokens from *start_ptr on, null: from 1), its logits are for the next position: the mask of that position, as target the token there if
    // there is one.  The ranges' statistics and the target's logit are left for the policy kernel.
    const int *len_ptr, *start_ptr, *ylen_ptr;
    int len_add, part_ld;
    const int* y;
    float* zt;
    unsigned* arrived;  // a line per row, zero between launches
};
// *parts (nullable): partial statistics a row.
hipError_t launch_rules(RulesArgs a, hipStream_t st, int* parts = nullptr);

}  // namespace bild
