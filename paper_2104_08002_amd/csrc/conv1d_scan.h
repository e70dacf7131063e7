// The selective scan: arguments and tile shape shared by its forward and backward kernels.  Not part of the public ABI.
//
//   e = dt + dt_bias[d], through softplus if asked;  a[s] = exp(e A[d][s])
//   h[s] = a[s] h[s] + e x B[s];  y = sum_s C[s] h[s] + skip[d] x;  out = y z sigmoid(z)
// for every sample n and channel d, S states each; B and C are shared by the D / G channels of a group.
//
// Lanes.  P neighbouring lanes have one channel, K states each, in registers (S is padded to K P with zeros): 4 lanes of 1, 2 or
// 4 states up to S = 16, 8 or 16 lanes of 4 beyond; a wave has 64 / P channels.  One step costs a lane K exponentials (half the
// rate of a product) and 4 K products, which is what bounds the scan.  (With 4 states a lane for every S, S = 8 has 32 channels a
// wave and room in LDS for 16 steps of them: it took as long as S = 16.)  Rows lie along the sequence, states across lanes: a tile
// of steps goes through LDS, loaded and stored along rows (up to 8 elements a lane), read 4 steps at a time.
// Positions behind a sequence's length have e = 0 and e x = 0, which leaves the state as it is.
#pragma once

#include "conv1d_sequence.h"

namespace conv1d {

constexpr int kSub = 8;       // steps between the states that the forward pass keeps for the backward pass
constexpr int kScanWaves = 4; // most waves of a workgroup
constexpr int kMostStates = 64;

struct ScanArgs {
    const void *x, *dt, *B, *C, *z;  // z: nullptr: no gate
    const float *A, *skip, *dt_bias, *init;
    const int* lengths;
    void* out;
    float* final;      // [N][D][S] or nullptr
    float* saved;      // [N][chunks][D][K P]: the state before every kSub-th step, or nullptr
    float* starts;     // [N][D][nseg][K P]: state before each segment (split only)
    float* sums;       // [N][D][nseg]: sum of e over each segment
    int N, D, L, S, G, Dg, softplus;
    long x_sn, x_sd, dt_sn, dt_sd, z_sn, z_sd, out_sn, out_sd;
    long b_sn, b_sg, b_ss, c_sn, c_sg, c_ss;
    int nseg, seg_len; // the sequence in segments of seg_len steps, a multiple of scan_tile(P)
    int chunks;        // ceil(L / kSub)
    int blocks_d;      // workgroups along the channels of a group
    int first;         // first workgroup of the launch
    // backward
    const void* dout;
    long dout_sn, dout_sd;
    const float* dfinal;
    void *dx, *ddt, *dz, *dB, *dC;   // contiguous, in the type of x
    float* part_bc;    // [2][blocks_d][N][G][S][L]: sums over a workgroup's channels (blocks_d > 1)
    float* part_p;     // [N * nseg][D * (K P + 2)]: what a segment adds to the gradients of A, then of skip, then of dt_bias
    float* carries;    // [N][D][nseg][K P]: what the later segments send into each (split only)
    float* dinit;      // [N][D][S] or nullptr
};

typedef __attribute__((ext_vector_type(4))) float scan_f32x4;  // (16-byte aligned: LDS, and what the kernels keep)

template <int K>
struct States {  // of a lane, aligned
    typedef __attribute__((ext_vector_type(K))) float vec;
    vec v;
    __device__ __forceinline__ float operator[](int k) const { return v[k]; }
};
template <>
struct States<1> {
    float v;
    __device__ __forceinline__ float operator[](int) const { return v; }
};
template <int K>
__device__ __forceinline__ States<K> states_at(const float* p) { return *reinterpret_cast<const States<K>*>(p); }
template <int K>
__device__ __forceinline__ void put_states(float* p, const float (&h)[K]) {
    States<K> s;
    if constexpr (K == 1) {
        s.v = h[0];
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k) s.v[k] = h[k];
    }
    *reinterpret_cast<States<K>*>(p) = s;
}

// steps of a tile, of which the 64 lanes stage the same number of elements each (8, 8, 4 for P = 4, 8, 16; backwards 8, 2, 1: the
// sums over waves want LDS too; with 8 elements on fewer lanes, N = 4, D = 256, L = 8192, S = 64 took 658 us backwards for 579)
constexpr int scan_tile(int P) { return P == 4 ? 32 : 64; }
constexpr int scan_tile_back(int P) { return P == 4 ? 32 : 16; }
// floats of a row in LDS: 16 rows of 4 steps lie in distinct banks
constexpr int scan_stride(int T) { return T + 4; }

// sum over the P lanes of a channel, in all of them
#ifdef HOSTMODEL
template <int P>
inline float channel_sum(float v) { return v; }
#else
template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int P>
__device__ __forceinline__ float channel_sum(float v) {
    if constexpr (P >= 2) v = add_dpp<0xB1>(v);    // quad_perm 1,0,3,2
    if constexpr (P >= 4) v = add_dpp<0x4E>(v);    // quad_perm 2,3,0,1
    if constexpr (P >= 8) v = add_dpp<0x141>(v);   // row_half_mirror: the other quad, whose lanes agree
    if constexpr (P >= 16) v = add_dpp<0x140>(v);  // row_mirror
    return v;
}
#endif

// where a workgroup works: sample, group, segment, its channels
struct ScanPlace {
    long n;
    int g, seg, cb;
};
__device__ __forceinline__ ScanPlace scan_place(const ScanArgs& a) {
    unsigned b = static_cast<unsigned>(a.first) + blockIdx.x, q = b / a.blocks_d;
    ScanPlace p;
    p.cb = static_cast<int>(b - q * a.blocks_d);
    b = q / a.nseg;
    p.seg = static_cast<int>(q - b * a.nseg);
    q = b / a.G;
    p.g = static_cast<int>(b - q * a.G);
    p.n = q;
    return p;
}

// A rate times log2(e), kept finite: a step of 0 (a position behind the end has one) leaves the state whatever the rate is.
__device__ __forceinline__ float rate_of(float A) {
    const float r = A * kLog2e, most = 3.4028234e38f;
    return r > most ? most : r < -most ? -most : r;
}
// A of state s of channel d; 0 where there is no such state
__device__ __forceinline__ float scan_rate(const float* A, int S, long d, int s, bool there) { return there && s < S ? A[d * S + s] : 0.f; }
// ... made rates.  The kernels do so behind the loads of their first tile, which then do not wait for those of A: where the
// sequence is cut into single tiles, a launch is one way through memory shorter.
template <int K>
__device__ __forceinline__ void make_rates(float (&rate)[K]) {
#pragma unroll
    for (int k = 0; k < K; ++k) rate[k] = rate_of(rate[k]);
}

template <bool BF16>
__device__ __forceinline__ const typename RowElem<BF16>::type* scan_row(const void* base, long sn, long sd, long n, long d) {
    return static_cast<const typename RowElem<BF16>::type*>(base) + n * sn + d * sd;
}

// Steps t .. t + V - 1 of a row.  INSIDE: they all count; else those from `end` on are 0, every load comes from one of the row's L
// elements, and none waits for a branch: a launch of single tiles takes as long as its last one.  (With that and the rates made
// behind the first loads, N = 3, D = 49, L = 4999, S = 5 in FP32 takes 53 us forwards and backwards, 57 before.)
template <bool BF16, bool INSIDE, int V>
__device__ __forceinline__ void scan_load(const void* row, int t, int end, int L, float (&v)[V]) {
    if constexpr (INSIDE && V == 8) {
        row_load8_inside<BF16>(row, t, v);
    } else if constexpr (INSIDE) {
        typename RowElem<BF16>::type u[V];
        __builtin_memcpy(u, static_cast<const typename RowElem<BF16>::type*>(row) + t, sizeof u);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = load_elem<BF16>(u, e);
    } else if (wave_all(t >= end)) {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = 0.f;
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = load_elem<BF16>(row, min(t + e, L - 1));
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = t + e < end ? v[e] : 0.f;
    }
}
// those of them that lie before `end`
template <bool BF16, int V>
__device__ __forceinline__ void scan_store(void* row, int t, int end, const float (&v)[V]) {
    if constexpr (V == 8) {
        row_store8<BF16>(row, t, end, v);
    } else {
        typename RowElem<BF16>::type u[V];
#pragma unroll
        for (int e = 0; e < V; ++e) store_elem<BF16>(u, e, v[e]);
        auto* to = static_cast<typename RowElem<BF16>::type*>(row) + t;
        if (t + V <= end) {
            __builtin_memcpy(to, u, sizeof u);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (t + e < end) to[e] = u[e];
        }
    }
}

// B and C (BOTH; else `first` alone) of T steps from t0 on into LDS, [step][SP]; 0 behind `end` and for states that are not
// there.  8 steps of a state a lane; the lane's first loads (begin) go out before the rows', their values are used behind them.
template <bool BF16, int SP, int T, bool BOTH>
struct ScanStates {
    static constexpr int kItems = SP * (T / 8), kAll = BOTH ? 2 * kItems : kItems;
    using E = typename RowElem<BF16>::type;
    const E *first, *second;
    long first_ss, second_ss;
    int S, L;
    float v[8];

    __device__ __forceinline__ void load(int i, int t0, int end) {
        const int s = i & (SP - 1), c = i / SP % (T / 8);
        const bool which = BOTH && i >= kItems;
        if (s < S) {
            const E* row = (which ? second : first) + s * (which ? second_ss : first_ss);
            if (t0 + T <= end) scan_load<BF16, true>(row, t0 + 8 * c, end, L, v);
            else scan_load<BF16, false>(row, t0 + 8 * c, end, L, v);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.f;
        }
    }
    __device__ __forceinline__ void put(int i, float* to_first, float* to_second) const {
        float* to = (BOTH && i >= kItems ? to_second : to_first) + (i / SP % (T / 8)) * (8 * SP) + (i & (SP - 1));
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e * SP] = v[e];
    }
    __device__ __forceinline__ void begin(int t0, int end) {
        if (static_cast<int>(threadIdx.x) < kAll) load(threadIdx.x, t0, end);
    }
    __device__ __forceinline__ void finish(int t0, int end, float* to_first, float* to_second) {
        if (static_cast<int>(threadIdx.x) < kAll) put(threadIdx.x, to_first, to_second);
        for (int i = threadIdx.x + blockDim.x; i < kAll; i += blockDim.x) {
            load(i, t0, end);
            put(i, to_first, to_second);
        }
    }
};

// the lane's part in loading and storing a tile's rows: row lane / LPR of the wave, V elements from V (lane % LPR) on
template <int P, int T>
struct ScanRows {
    static constexpr int CW = kSeqWave / P, V = CW * T / kSeqWave, LPR = T / V, RS = scan_stride(T);
    static_assert(CW * LPR == kSeqWave && V <= 8, "a wave stages a tile at once");
};

template <int V>
__device__ __forceinline__ void lds_put(float* to, const float (&v)[V]) {
    if constexpr (V >= 4) {
#pragma unroll
        for (int e = 0; e < V; e += 4) *reinterpret_cast<scan_f32x4*>(to + e) = scan_f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) to[e] = v[e];
    }
}
template <int V>
__device__ __forceinline__ void lds_get(const float* from, float (&v)[V]) {
    if constexpr (V >= 4) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const scan_f32x4 a = *reinterpret_cast<const scan_f32x4*>(from + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i + e] = a[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = from[e];
    }
}

// 2^x as m 2^n, 1 <= m < 2.  Where e A adds up to more than 88 over a segment (a state that grows), 2^x is no float, and as infinity
// would make NaN of a state of 0 before it, or of the shrinking behind it; m 2^n times a state is infinite only if the product is.
// Exponents end at 2^26, far behind those of any state, so that 16 of them add up in an int.  (NaN stays in m.)  A wave whose decays
// are all at most 1, which is the rule, takes them as floats: N = 1, D = 128 in 938 segments takes 7.1 us so and 7.9 otherwise,
// N = 8, D = 128 in 125 segments 6.0 and 6.3.
struct Decay {
    float m;
    int n;
};
__device__ __forceinline__ Decay decay_of(float x) {
    constexpr float most = 1 << 26;
    const float c = x > most ? most : x < -most ? -most : x, f = floorf(c);
    return Decay{exp2_hw(c - f), static_cast<int>(fmaxf(f, -most))};
}
__device__ __forceinline__ float decayed(const Decay& d, float h, float add) { return fmaf(d.m, ldexpf(h, d.n), add); }
// both, one behind the other, up to 16 of them: m is below 2^16 and is brought back by `normal`
__device__ __forceinline__ void decay_more(Decay& d, const Decay& by) {
    d.m *= by.m;
    d.n += by.n;
}
__device__ __forceinline__ Decay normal(const Decay& d) {
    const int up = static_cast<int>(__float_as_uint(d.m) >> 23) - 127;
    return Decay{ldexpf(d.m, -up), d.n + up};
}

// One (sample, channel) row of segment values joined along the sequence: value[seg] holds what a segment adds, and becomes
// what comes into it from the segments before (BACK: behind) it, `first` into the first; sums[seg]: exp(A sum) is a segment's
// decay, and those of a run multiply to a run's.  SP states times `chunks` runs of kRun segments at a time: a run is joined in
// registers, the runs through LDS.
// Bound by latency and by how much of every line it uses, so that a row's segments lie together: N = 8, D = 128 in 125 segments
// takes 6.0 us, 9.8 with the channels of a segment together.  Runs of 16 join up to 1024 segments of 16 states at once (N = 1,
// D = 128 in 938: 7.1 us, 2.2 more with runs of 8, which are no faster at fewer).
constexpr int kRun = 16;
template <bool BACK>
__global__ __launch_bounds__(1024) void scan_join_kernel(float* value, const float* sums, const float* first, const float* A, int N, int D,
                                                         int S, int SP, int nseg, int chunks) {
    __shared__ float run_decay[1024], run_add[1024], last[1024];
    __shared__ int run_shift[1024];              // the n of a run's decay
    __shared__ bool shrinking[1024 / kSeqWave];  // of every wave
    const unsigned per_row = SP * chunks, row = blockIdx.x * (blockDim.x / per_row) + threadIdx.x / per_row;  // (N D < 2^25)
    const bool there = row < static_cast<unsigned>(N) * D;
    const int in_row = threadIdx.x % per_row, s = in_row % SP, chunk = in_row / SP, base = threadIdx.x - in_row + s;
    const unsigned d = there ? row % D : 0;
    const float rate = rate_of(scan_rate(A, S, d, s, there));
    float h = there && first && s < S ? first[static_cast<long>(row) * S + s] : 0.f;
    for (int from = 0; from < nseg; from += kRun * chunks) {
        Decay f[kRun], decay{1.f, 0};
        float x[kRun], v[kRun], add = 0.f;
        const int i0 = from + kRun * chunk, real = there ? nseg - i0 : 0;  // segments of the run that are there
        const long at = static_cast<long>(row) * nseg + (BACK ? nseg - 1 - i0 : i0);
        constexpr int next = BACK ? -1 : 1;
        const int step = next * SP;
        const float* sum = sums + at;
        float* to = value + at * SP + s;
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
            x[i] = i < real - 1 ? sum[i * next] : 0.f;  // (nothing comes behind the last segment, which has left no values)
            v[i] = i < real - 1 ? to[i * step] : 0.f;
        }
        bool shrinks = true;
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
            x[i] *= rate;
            shrinks = shrinks && x[i] <= 0.f;
        }
        shrinks = wave_all(shrinks);
        if (shrinks) {
#pragma unroll
            for (int i = 0; i < kRun; ++i) {
                f[i] = Decay{exp2_hw(x[i]), 0};
                add = fmaf(f[i].m, add, v[i]);
                decay.m *= f[i].m;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kRun; ++i) {
                f[i] = decay_of(x[i]);
                add = decayed(f[i], add, v[i]);
                decay_more(decay, f[i]);
            }
            decay = normal(decay);
        }
        run_decay[threadIdx.x] = decay.m;
        run_shift[threadIdx.x] = decay.n;
        run_add[threadIdx.x] = add;
        if (threadIdx.x % kSeqWave == 0) shrinking[threadIdx.x / kSeqWave] = shrinks;
        __syncthreads();
        if (wave_all(shrinking[threadIdx.x % (blockDim.x / kSeqWave)])) {
#pragma unroll 8
            for (int c = 0; c < chunk; ++c) h = fmaf(run_decay[base + c * SP], h, run_add[base + c * SP]);
        } else {
            for (int c = 0; c < chunk; ++c) h = decayed(Decay{run_decay[base + c * SP], run_shift[base + c * SP]}, h, run_add[base + c * SP]);
        }
        if (shrinks) {
#pragma unroll
            for (int i = 0; i < kRun; ++i) {
                if (i < real) to[i * step] = h;
                h = fmaf(f[i].m, h, v[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kRun; ++i) {
                if (i < real) to[i * step] = h;
                h = decayed(f[i], h, v[i]);
            }
        }
        if (from + kRun * chunks >= nseg) break;  // (of the whole workgroup)
        if (chunk == chunks - 1) last[base] = h;
        __syncthreads();
        h = last[base];
    }
}

template <bool BACK>
inline hipError_t scan_join_launch(float* value, const float* sums, const float* first, const float* A, int N, int D, int S, int SP, int nseg,
                                   hipStream_t st) {
    int chunks = 1;
    while (chunks * kRun < nseg && chunks * 2 * SP <= 1024) chunks *= 2;
    const int per_row = SP * chunks, threads = per_row > 256 ? per_row : 256;
    return launch_kernel(scan_join_kernel<BACK>, dim3(static_cast<unsigned>(cdiv(static_cast<long>(N) * D, threads / per_row))), dim3(threads), 0, st,
                         value, sums, first, A, N, D, S, SP, nseg, chunks);
}

// host
struct ScanPlan {
    int K, P, waves, blocks_d, nseg, seg_len, chunks;
};
ScanPlan scan_plan(int N, int D, int L, int S, int G, bool back);
hipError_t scan_fwd_launch(const ScanArgs& a, const ScanPlan& p, int bf16, hipStream_t st);
hipError_t scan_bwd_launch(const ScanArgs& a, const ScanPlan& p, int bf16, float* dA, float* dskip, float* dbias, hipStream_t st);

// workgroups of a launch
inline long scan_blocks(const ScanArgs& a) { return static_cast<long>(a.N) * a.G * a.nseg * a.blocks_d; }

}  // namespace conv1d
