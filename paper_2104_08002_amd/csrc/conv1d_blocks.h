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
#else
__device__ __forceinline__ unsigned long wave_ballot(bool v) { return __ballot(v); }
__device__ __forceinline__ int lane_from(int v, int lane) { return __shfl(v, lane, kSeqWave); }
__device__ __forceinline__ int lds_add(int* p, int v) { return atomicAdd(p, v); }
__device__ __forceinline__ void lds_add(float* p, float v) { atomicAdd(p, v); }
__device__ __forceinline__ int popcount64(unsigned long v) { return __popcll(v); }
__device__ __forceinline__ int first_bit(unsigned long v) { return __ffsll(static_cast<unsigned long long>(v)) - 1; }
__device__ __forceinline__ int lane_up(int v, int by) { return __shfl_up(v, by, kSeqWave); }
#endif

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
