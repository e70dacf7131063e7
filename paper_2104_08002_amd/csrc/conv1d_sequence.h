// Shared by the sequence operators: rows read at any element alignment, lane exchanges, the activations.
// Not part of the public ABI.
#pragma once

#include "conv1d_internal.h"

namespace conv1d {

constexpr int kSeqWave = 64;
// threads of one launch: what is more is launched in pieces
constexpr long kSeqMostThreads = 1L << 31;
constexpr float kLog2e = 1.44269504088896340736f;

inline bool seq_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// ---- lanes ----------------------------------------------------------------------------------------------------------
#ifdef HOSTMODEL  // one thread at a time: a lane sees its own value
inline float lane_xor(float v, int) { return v; }
inline double lane_xor(double v, int) { return v; }
inline float exp2_hw(float v) { return std::exp2(v); }
inline float rcp_hw(float v) { return 1.f / v; }
inline void keep_here(float&) {}
inline float lane_next(float v) { return v; }
inline bool wave_all(bool v) { return v; }
inline float lane_first(float v) { return v; }
#else
__device__ __forceinline__ float lane_xor(float v, int mask) { return __shfl_xor(v, mask, kSeqWave); }
__device__ __forceinline__ double lane_xor(double v, int mask) { return __shfl_xor(v, mask, kSeqWave); }
// 2^v and 1 / v to one unit in the last place
__device__ __forceinline__ float exp2_hw(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float rcp_hw(float v) { return __builtin_amdgcn_rcpf(v); }
// The value is found here and not behind a later branch, away from the lane exchange that is one instruction with its addition.
__device__ __forceinline__ void keep_here(float& v) { asm volatile("" : "+v"(v)); }
// v of the next lane (0 in the last), of the first lane
__device__ __forceinline__ float lane_next(float v) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x130, 0xf, 0xf, true));  // wave_shl:1
}
__device__ __forceinline__ bool wave_all(bool v) { return __all(v); }
__device__ __forceinline__ float lane_first(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }
#endif

// ---- rows -----------------------------------------------------------------------------------------------------------
// A row is contiguous along the sequence and begins at any element: vectors are loaded at the alignment of an element,
// which the memory path takes at full rate but for the lines that a vector straddles.
typedef __attribute__((ext_vector_type(8), aligned(2))) unsigned short seq_u16x8;
typedef __attribute__((ext_vector_type(8), aligned(2))) __bf16 seq_bf16x8;
typedef __attribute__((ext_vector_type(8))) float seq_f32x8;
typedef __attribute__((ext_vector_type(4), aligned(4))) float seq_f32x4;

template <bool BF16>
struct RowElem {
    using type = float;
};
template <>
struct RowElem<true> {
    using type = unsigned short;
};

// bfloat16, nearest, ties to even (NaN stays NaN): the hardware's conversion
__device__ __forceinline__ unsigned short float_to_bf16(float v) {
    const __bf16 b = static_cast<__bf16>(v);
    unsigned short u;
    __builtin_memcpy(&u, &b, 2);
    return u;
}

// elements at .. at + 7 of a row, all of them there
template <bool BF16>
__device__ __forceinline__ void row_load8_inside(const void* row, long at, float (&v)[8]) {
    if constexpr (BF16) {
        const seq_u16x8 t = *reinterpret_cast<const seq_u16x8*>(static_cast<const unsigned short*>(row) + at);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = bf16_to_float(t[e]);
    } else {
        const seq_f32x4 a = *reinterpret_cast<const seq_f32x4*>(static_cast<const float*>(row) + at);
        const seq_f32x4 b = *reinterpret_cast<const seq_f32x4*>(static_cast<const float*>(row) + at + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = a[e];
            v[4 + e] = b[e];
        }
    }
}

// elements at .. at + 7 of a row whose elements [0, end) are there; 0 elsewhere
template <bool BF16, typename I>
__device__ __forceinline__ void row_load8(const void* row, I at, I end, float (&v)[8]) {
    if (at >= 0 && at + 8 <= end) {
        row_load8_inside<BF16>(row, at, v);
    } else if (at + 8 > 0 && at < end) {  // some of them: every load from a place that is there, without a branch
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const I i = at + e, j = i < 0 ? 0 : i < end ? i : end - 1;
            const float u = load_elem<BF16>(row, j);
            v[e] = i == j ? u : 0.f;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.f;
    }
}

// the elements of at .. at + 7 that lie in [0, end)
template <bool BF16>
__device__ __forceinline__ void row_store8(void* row, long at, long end, const float (&v)[8]) {
    if constexpr (BF16) {
        const seq_bf16x8 t = __builtin_convertvector((seq_f32x8{v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]}), seq_bf16x8);
        __bf16* o = static_cast<__bf16*>(row) + at;
        if (at + 8 <= end) {
            *reinterpret_cast<seq_bf16x8*>(o) = t;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at + e < end) o[e] = t[e];
        }
    } else {
        float* o = static_cast<float*>(row) + at;
        if (at + 8 <= end) {
            *reinterpret_cast<seq_f32x4*>(o) = seq_f32x4{v[0], v[1], v[2], v[3]};
            *reinterpret_cast<seq_f32x4*>(o + 4) = seq_f32x4{v[4], v[5], v[6], v[7]};
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (at + e < end) o[e] = v[e];
        }
    }
}

template <bool BF16>
__device__ __forceinline__ void store_elem(void* base, long i, float v) {
    if constexpr (BF16) static_cast<unsigned short*>(base)[i] = float_to_bf16(v);
    else static_cast<float*>(base)[i] = v;
}

// positions of sequence n that count: all of them, or lengths[n] brought into [0, L]
__device__ __forceinline__ int seq_length(const int* lengths, long n, int L) {
    return lengths ? clampi(lengths[n], 0, L) : L;
}

// ---- functions ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float sigmoid_of(float v) { return rcp_hw(1.f + exp2_hw(-v * kLog2e)); }

// log(1 + exp(v)) = max(v, 0) + log(1 + u), u = exp(-|v|), and log(1 + u) = 2 atanh(r) = r f(r^2), r = u / (2 + u) <= 1/3.
// f is a polynomial with the least relative error on [0, 1/9] (fitted in 64 bits): 8e-9 with its coefficients as floats.  (The
// logarithm instruction has a bound on its absolute error next to 1, which would leave few bits of the small steps that this is
// used for.)
__device__ __forceinline__ float softplus_of(float v) {
    const float u = exp2_hw(-fabsf(v) * kLog2e);
    const float r = u * rcp_hw(2.f + u), q = r * r;
    float f = 0.28178316354751587f;
    f = fmaf(f, q, 0.27960607409477234f);
    f = fmaf(f, q, 0.40024909377098083f);
    f = fmaf(f, q, 0.6666631698608398f);
    f = fmaf(f, q, 2.f);
    const int m = static_cast<int>(__float_as_uint(v));  // max(v, 0) as a number of its bits; a NaN comes through f r
    return fmaf(f, r, __uint_as_float(static_cast<unsigned>(m < 0 ? 0 : m)));
}

}  // namespace conv1d
