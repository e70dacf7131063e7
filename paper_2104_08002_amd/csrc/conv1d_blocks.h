// Shared by the operators around the layers (embedding, group norm, dropout): division by a launch's sizes, ballots, sums over
// a workgroup.  Not part of the public ABI.
#pragma once

#include "conv1d_sequence.h"

namespace conv1d {

// Division of n < 2^31 by any d < 2^31: with 2^s >= d > 2^(s - 1) and m = ceil(2^(31 + s) / d), n m / 2^(31 + s) is off by less
// than n / 2^31 d < 1 / d, so that its whole part is exact.
struct Div31 {
    unsigned d, m;
    int sh;
};
inline Div31 make_div31(long d) {
    Div31 f{static_cast<unsigned>(d), 0, 0};
    if (d == 1) return f;
    int s = 1;
    while ((1L << s) < d) ++s;
    f.m = static_cast<unsigned>(((1UL << (31 + s)) + d - 1) / d);
    f.sh = s - 1;
    return f;
}
__device__ __forceinline__ int div31(int n, const Div31& f) {
    return f.d == 1 ? n : static_cast<int>(__umulhi(static_cast<unsigned>(n), f.m) >> f.sh);
}

// what a launch may count in 31 bits, with room for the last workgroup's surplus
constexpr long kMostItems = (1L << 31) - (1L << 16);

inline size_t round_up(size_t n, size_t to) { return (n + to - 1) / to * to; }

// ---- lanes ----------------------------------------------------------------------------------------------------------
#ifdef HOSTMODEL  // one thread at a time
inline unsigned long wave_ballot(bool v) { return v ? 1UL : 0UL; }
inline int lane_from(int v, int) { return v; }
inline int lds_add(int* p, int v) {
    const int old = *p;
    *p += v;
    return old;
}
inline void lds_add(float* p, float v) { *p += v; }
inline int popcount64(unsigned long v) { return __builtin_popcountl(v); }
inline int first_bit(unsigned long v) { return __builtin_ctzl(v | (1UL << 63)); }
inline int lane_up(int v, int) { return v; }
inline bool wave_any(bool v) { return v; }
#else
__device__ __forceinline__ unsigned long wave_ballot(bool v) { return __ballot(v); }
__device__ __forceinline__ int lane_from(int v, int lane) { return __shfl(v, lane, kSeqWave); }
__device__ __forceinline__ int lds_add(int* p, int v) { return atomicAdd(p, v); }
__device__ __forceinline__ void lds_add(float* p, float v) { atomicAdd(p, v); }
__device__ __forceinline__ int popcount64(unsigned long v) { return __popcll(v); }
__device__ __forceinline__ int first_bit(unsigned long v) { return __ffsll(static_cast<unsigned long long>(v)) - 1; }
__device__ __forceinline__ bool wave_any(bool v) { return __any(v); }
__device__ __forceinline__ int lane_up(int v, int by) { return __shfl_up(v, by, kSeqWave); }
#endif

// ---- vectors of 8 as they lie in memory ---------------------------------------------------------------------------------
// A load that nothing is done with yet: turned into floats only when they are needed, so that the next loads go out before it has come.
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
template <bool BF16>
struct Raw8 {
    u32x4 v[BF16 ? 1 : 2];
};
// all of them there
template <bool BF16>
__device__ __forceinline__ Raw8<BF16> raw8_inside(const void* row, int l) {
    Raw8<BF16> r;
    if constexpr (BF16) {
        r.v[0] = __builtin_bit_cast(u32x4, *reinterpret_cast<const seq_u16x8*>(static_cast<const unsigned short*>(row) + l));
    } else {
        r.v[0] = __builtin_bit_cast(u32x4, *reinterpret_cast<const seq_f32x4*>(static_cast<const float*>(row) + l));
        r.v[1] = __builtin_bit_cast(u32x4, *reinterpret_cast<const seq_f32x4*>(static_cast<const float*>(row) + l + 4));
    }
    return r;
}
// those before len, 0 behind; an element that is not there is read at a place that is (a row has one at least), without a branch
template <bool BF16>
__device__ __forceinline__ Raw8<BF16> raw8(const void* row, int l, int len) {
    Raw8<BF16> r;
    const int last = max(len, 1) - 1;
    if constexpr (BF16) {
        const unsigned short* p = static_cast<const unsigned short*>(row);
        unsigned u[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = p[min(l + e, last)];
#pragma unroll
        for (int i = 0; i < 4; ++i) r.v[0][i] = (l + 2 * i < len ? u[2 * i] : 0u) | (l + 2 * i + 1 < len ? u[2 * i + 1] << 16 : 0u);
    } else {
        const unsigned* p = static_cast<const unsigned*>(row);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const unsigned u = p[min(l + e, last)];
            r.v[e >> 2][e & 3] = l + e < len ? u : 0u;
        }
    }
    return r;
}
__device__ __forceinline__ void floats_of(const Raw8<true>& x, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(x.v[0][i] << 16);
        v[2 * i + 1] = __uint_as_float(x.v[0][i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void floats_of(const Raw8<false>& x, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(x.v[e >> 2][e & 3]);
}

// A row of `all` elements in vectors of 8.  WHOLE: it is made of whole ones.  Else the last is the row's last 8 elements, of which some are
// the vector's before as well: they are written twice with one value, and sums leave them out of the last (`first_new` elements).  So every
// load is of 8 elements that are there, without a branch or a shift.  A row of fewer than 8 elements is one vector, loaded one by one.
template <bool WHOLE>
__device__ __forceinline__ int vector_at(int vec, int all) {
    return WHOLE || all < 8 ? 8 * vec : min(8 * vec, all - 8);
}
template <bool BF16, bool WHOLE>
__device__ __forceinline__ Raw8<BF16> raw8_row(const void* row, int at, int all) {
    if constexpr (WHOLE) return raw8_inside<BF16>(row, at);
    if (all >= 8) return raw8_inside<BF16>(row, at);
    Raw8<BF16> r{};
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (e < all) {
            if constexpr (BF16) r.v[0][e >> 1] |= static_cast<unsigned>(static_cast<const unsigned short*>(row)[e]) << (16 * (e & 1));
            else r.v[e >> 2][e & 3] = static_cast<const unsigned*>(row)[e];
        }
    return r;
}
// the elements of at .. at + 7 that lie before end
template <bool BF16, bool WHOLE>
__device__ __forceinline__ void vector_store8(void* row, int at, int end, const float (&v)[8]) {
    row_store8<BF16>(row, at, WHOLE ? at + 8 : end, v);
}

// The sums of a and b over a workgroup, in every thread, added in one order; lds: two doubles a wave.
template <int THREADS>
__device__ __forceinline__ void block_sums(double& a, double& b, double* lds) {
#pragma unroll
    for (int m = 1; m < kSeqWave; m <<= 1) {
        a += lane_xor(a, m);
        b += lane_xor(b, m);
    }
    if constexpr (THREADS > kSeqWave) {
        __syncthreads();
        if ((threadIdx.x & (kSeqWave - 1)) == 0) {
            lds[2 * (threadIdx.x >> 6)] = a;
            lds[2 * (threadIdx.x >> 6) + 1] = b;
        }
        __syncthreads();
        a = lds[0];
        b = lds[1];
#pragma unroll
        for (int w = 1; w < THREADS / kSeqWave; ++w) {
            a += lds[2 * w];
            b += lds[2 * w + 1];
        }
    }
}

}  // namespace conv1d
