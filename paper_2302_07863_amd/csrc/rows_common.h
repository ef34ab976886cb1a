// Device helpers of the operators on rows: values of the three row types, and accesses to rows that are aligned to their
// type only.
#pragma once
#include "kernel_common.h"

namespace bild {

// N bytes at an address that is a multiple of A (the vector memory path takes any; a wave of consecutive pieces touches one line more).
template <int N, int A>
struct __attribute__((packed, aligned(A))) Piece {
    uint32_t w[N / 4];
};

struct RowF32 {
    typedef float type;
    static constexpr int kDtype = BILD_DT_F32, kBytes = 4;
    static __device__ __forceinline__ float up(float v) { return v; }
    static __device__ __forceinline__ float down(float v) { return v; }
};
struct RowBf16 {
    typedef uint16_t type;
    static constexpr int kDtype = BILD_DT_BF16, kBytes = 2;
    static __device__ __forceinline__ float up(uint16_t v) { return bf2f(v); }
    static __device__ __forceinline__ uint16_t down(float v) { return (uint16_t)pack_bf16x2(v, 0.f); }
};
struct RowF16 {
    typedef uint16_t type;
    static constexpr int kDtype = BILD_DT_F16, kBytes = 2;
    static __device__ __forceinline__ float up(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
    static __device__ __forceinline__ uint16_t down(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
};

// E consecutive values of a row (16 bytes of a 16-bit type with E = 8, of fp32 with E = 4).
template <class R, int E>
struct RowVec {
    typename R::type v[E];
    __device__ __forceinline__ void load(const typename R::type* p) {
        static_assert(E * R::kBytes % 4 == 0, "whole words");
        const Piece<E * R::kBytes, R::kBytes> q = *(const Piece<E * R::kBytes, R::kBytes>*)p;
        __builtin_memcpy(v, &q, sizeof(v));
    }
    __device__ __forceinline__ void store(typename R::type* p) const {
        Piece<E * R::kBytes, R::kBytes> q;
        __builtin_memcpy(&q, v, sizeof(v));
        *(Piece<E * R::kBytes, R::kBytes>*)p = q;
    }
    // the first n of them
    __device__ __forceinline__ void load_some(const typename R::type* p, int n) {
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = i < n ? p[i] : (typename R::type)0;
    }
    __device__ __forceinline__ void store_some(typename R::type* p, int n) const {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i < n) p[i] = v[i];
    }
};

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

}  // namespace bild
