// Selective scan, backward.  With dy = dout z sigmoid(z) and g the gradient of the state,
//   g[t] = C[t] dy[t] + a[t+1] g[t+1],   c[t] = a[t] g[t] (what a step sends into the one before it),   q[t] = c[t] h[t-1]
//   dC = sum_d dy h,  dB = sum_d g e x,  dx = e sum_s g B + skip dy,  de = x sum_s g B + sum_s A q,  dA = sum_t e q
//   ddt = de sigmoid(dt + dt_bias) behind a softplus, dz = dout y (silu)'(z), dskip = sum dy x, ddt_bias = sum ddt.
// The forward pass has kept the state before every kSub steps: a workgroup goes through its segment from the end, computes
// kSub states and decays again into registers and walks them backwards.  Where a sequence is cut, the adjoint is joined as
// the forward state is: a launch finds what each segment sends into the one before it, another joins them.
// dB and dC are summed over the channels of a wave by lane exchanges, of a workgroup through LDS, of the workgroups of a
// group by a launch of its own, always in the same order.
#include "conv1d_scan.h"

namespace conv1d {
namespace {

constexpr int kThreads = 256;
constexpr int bwd_tile(int P) { return P >= 4 ? 32 : 16; }

// One value per lane and state k, for dB and dC: the sums over the channels of the wave.  Afterwards the lanes whose place
// within their row of 16 is p < P hold them: q[0] dB, q[1] dC of state 4 p + channel_state(row).
#ifdef HOSTMODEL
template <int P>
inline void wave_sums(const float (&dB)[kK], const float (&dC)[kK], float (&q)[2]) {
    q[0] = dB[0];
    q[1] = dC[0];
}
#else
__device__ __forceinline__ float swap32_add(float u, float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(u), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float swap16_add(float u, float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(u), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
template <int P>
__device__ __forceinline__ void wave_sums(const float (&dB)[kK], const float (&dC)[kK], float (&q)[2]) {
    q[0] = swap16_add(swap32_add(dB[0], dB[1]), swap32_add(dB[2], dB[3]));
    q[1] = swap16_add(swap32_add(dC[0], dC[1]), swap32_add(dC[2], dC[3]));
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        if constexpr (P <= 8) q[j] = add_dpp<0x128>(q[j]);  // row_ror:8
        if constexpr (P <= 4) q[j] = add_dpp<0x124>(q[j]);  // row_ror:4
        if constexpr (P <= 2) q[j] = add_dpp<0x4E>(q[j]);
        if constexpr (P <= 1) q[j] = add_dpp<0xB1>(q[j]);
    }
}
#endif
// rows of 16 lanes: 0, 1, 2, 3 hold state 0, 2, 1, 3
__device__ __forceinline__ int channel_state(int lane) {
    const int row = lane >> 4;
    return (row >> 1) | ((row & 1) << 1);
}

// what a step needs; the walk back leaves its own sums in the place
struct alignas(16) Slot {
    float e, ex, dy, unused;
};

// e, e x and dy of the wave's rows, tile at t0
template <bool BF16, int P>
__device__ __forceinline__ void stage_rows(const ScanArgs& a, const ScanPlace& at, int base, long t0, long len, Slot* mine) {
    constexpr int T = bwd_tile(P), CW = kSeqWave / P, LPR = T / 8, RPP = kSeqWave / LPR, STRIDE = T + 1;
    const int lane = threadIdx.x & (kSeqWave - 1);
#pragma unroll
    for (int r0 = 0; r0 < CW; r0 += RPP) {
        const int row = r0 + lane / LPR, c = 8 * (lane % LPR);
        if (row >= CW) continue;
        const bool real = base + row < a.Dg;
        const long d = static_cast<long>(at.g) * a.Dg + (real ? base + row : 0), end = real ? len : 0;
        float x[8], e[8], dy[8], z[8];
        row_load8<BF16>(scan_row<BF16>(a.x, a.x_sn, a.x_sd, at.n, d), t0 + c, end, x);
        row_load8<BF16>(scan_row<BF16>(a.dt, a.dt_sn, a.dt_sd, at.n, d), t0 + c, end, e);
        row_load8<BF16>(scan_row<BF16>(a.dout, a.dout_sn, a.dout_sd, at.n, d), t0 + c, end, dy);
        if (a.z) row_load8<BF16>(scan_row<BF16>(a.z, a.z_sn, a.z_sd, at.n, d), t0 + c, end, z);
        const float bias = a.dt_bias ? a.dt_bias[d] : 0.f;
        Slot* to = mine + row * STRIDE + c;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float v = e[i] + bias;
            if (a.softplus) v = softplus_of(v);
            v = t0 + c + i < end ? v : 0.f;
            if (a.z) dy[i] *= z[i] * sigmoid_of(z[i]);
            to[i] = Slot{v, v * x[i], dy[i], 0.f};
        }
    }
}

template <bool BF16, int P>
__device__ __forceinline__ void stage_states(const void* from, long base, long ss, int S, long t0, long end, float* to) {
    constexpr int SP = kK * P, T = bwd_tile(P);
    const typename RowElem<BF16>::type* row0 = static_cast<const typename RowElem<BF16>::type*>(from) + base;
    for (int i = threadIdx.x; i < SP * (T / 8); i += blockDim.x) {
        const int s = i & (SP - 1), c = i / SP;
        float v[8];
        if (s < S) {
            row_load8<BF16>(row0 + s * ss, t0 + 8 * c, end, v);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) to[(8 * c + e) * SP + s] = v[e];
    }
}

// what a segment sends into the one before it, from nothing sent into itself, and the sum of its steps
template <bool BF16, int P>
__global__ __launch_bounds__(kScanWaves* kSeqWave) void scan_adjoint_kernel(ScanArgs a) {
    constexpr int SP = kK * P, T = bwd_tile(P), CW = kSeqWave / P, STRIDE = T + 1;
    __shared__ __align__(16) Slot steps[kScanWaves][CW * STRIDE];
    __shared__ __align__(16) float sC[T * SP];
    const ScanPlace at = scan_place(a);
    if (at.seg == 0) return;
    const int lane = threadIdx.x & (kSeqWave - 1), wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int p = lane & (P - 1), cl = lane / P;
    const long len = seq_length(a.lengths, at.n, a.L);
    const int base = (at.cb * waves + wave) * CW;
    const bool there = base + cl < a.Dg;
    const long d = static_cast<long>(at.g) * a.Dg + (there ? base + cl : 0);
    Slot* mine = steps[wave];
    float rate[kK], carry[kK], sum = 0.f;
#pragma unroll
    for (int k = 0; k < kK; ++k) {
        rate[k] = scan_rate(a, d, kK * p + k, there);
        carry[k] = 0.f;
    }
    const long t_begin = static_cast<long>(at.seg) * a.seg_len, t_end = min(static_cast<long>(a.L), t_begin + a.seg_len);
    for (long t0 = t_begin + (t_end - 1 - t_begin) / T * T; t0 >= t_begin; t0 -= T) {
        stage_rows<BF16, P>(a, at, base, t0, len, mine);
        stage_states<BF16, P>(a.C, at.n * a.c_sn + at.g * a.c_sg, a.c_ss, a.S, t0, len, sC);
        __syncthreads();
        const Slot* row = mine + cl * STRIDE;
        for (int t = T - kSub; t >= 0; t -= kSub) {
            float part = 0.f;
#pragma unroll
            for (int i = kSub - 1; i >= 0; --i) {
                const Slot s = row[t + i];
                part += s.e;
#pragma unroll
                for (int k = 0; k < kK; ++k)
                    carry[k] = exp2_hw(s.e * rate[k]) * fmaf(sC[(t + i) * SP + kK * p + k], s.dy, carry[k]);
            }
            sum += part;
        }
        __syncthreads();
    }
    if (!there) return;
    const long i = (at.n * a.nseg + at.seg) * a.D + d;
    *reinterpret_cast<seq_f32x4*>(a.carries + i * SP + kK * p) = seq_f32x4{carry[0], carry[1], carry[2], carry[3]};
    if (p == 0) a.sums[i] = sum;
}

// carries[seg]: what segment seg sends on from nothing -> what is sent into it.  One lane per state.
__global__ __launch_bounds__(kThreads) void scan_join_back_kernel(ScanArgs a, int SP) {
    const long i = static_cast<long>(blockIdx.x) * kThreads + threadIdx.x;
    const long nd = i / SP;
    if (nd >= static_cast<long>(a.N) * a.D) return;
    const int s = static_cast<int>(i - nd * SP);
    const long n = nd / a.D, d = nd - n * a.D;
    const float rate = scan_rate(a, d, s, true);
    float c = a.dfinal && s < a.S ? a.dfinal[nd * a.S + s] : 0.f;
#pragma unroll 8
    for (int seg = a.nseg - 1; seg > 0; --seg) {
        const long at = (n * a.nseg + seg) * a.D + d;
        const float add = a.carries[at * SP + s], decay = exp2_hw(rate * a.sums[at]);
        a.carries[at * SP + s] = c;
        c = fmaf(decay, c, add);
    }
    a.carries[(n * a.nseg * a.D + d) * SP + s] = c;
}

template <bool BF16, int P>
__global__ __launch_bounds__(kScanWaves* kSeqWave) void scan_bwd_kernel(ScanArgs a) {
    constexpr int SP = kK * P, T = bwd_tile(P), CW = kSeqWave / P, STRIDE = T + 1;
    constexpr int LPR = T / 8, RPP = kSeqWave / LPR, PASSES = CW > RPP ? CW / RPP : 1;
    constexpr int RED = SP + 1;
    __shared__ __align__(16) Slot steps[kScanWaves][CW * STRIDE];
    __shared__ __align__(16) float sB[T * SP], sC[T * SP];
    __shared__ float red[kScanWaves][2][kSub * RED];
    const ScanPlace at = scan_place(a);
    const int lane = threadIdx.x & (kSeqWave - 1), wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int p = lane & (P - 1), cl = lane / P;
    const long len = seq_length(a.lengths, at.n, a.L);
    const int base = (at.cb * waves + wave) * CW;
    const bool there = base + cl < a.Dg;
    const long d = static_cast<long>(at.g) * a.Dg + (there ? base + cl : 0);
    Slot* mine = steps[wave];
    float rate[kK], carry[kK], dA[kK], dskip[PASSES], dbias[PASSES];
#pragma unroll
    for (int k = 0; k < kK; ++k) {
        const int s = kK * p + k;
        rate[k] = scan_rate(a, d, s, there);
        dA[k] = 0.f;
        carry[k] = 0.f;
        if (a.nseg > 1) carry[k] = there ? a.carries[((at.n * a.nseg + at.seg) * a.D + d) * SP + s] : 0.f;
        else if (a.dfinal && there && s < a.S) carry[k] = a.dfinal[(at.n * a.D + d) * a.S + s];
    }
#pragma unroll
    for (int q = 0; q < PASSES; ++q) dskip[q] = dbias[q] = 0.f;
    const long t_begin = static_cast<long>(at.seg) * a.seg_len, t_end = min(static_cast<long>(a.L), t_begin + a.seg_len);
    for (long t0 = t_begin + (t_end - 1 - t_begin) / T * T; t0 >= t_begin; t0 -= T) {
        stage_rows<BF16, P>(a, at, base, t0, len, mine);
        stage_states<BF16, P>(a.B, at.n * a.b_sn + at.g * a.b_sg, a.b_ss, a.S, t0, len, sB);
        stage_states<BF16, P>(a.C, at.n * a.c_sn + at.g * a.c_sg, a.c_ss, a.S, t0, len, sC);
        __syncthreads();
        Slot* row = mine + cl * STRIDE;
        for (int t = T - kSub; t >= 0; t -= kSub) {
            if (t0 + t >= a.L) continue;
            float h0[kK], h[kSub][kK], decay[kSub][kK];
            if (there) {
                const seq_f32x4 v = *reinterpret_cast<const seq_f32x4*>(a.saved + ((at.n * a.chunks + (t0 + t) / kSub) * a.D + d) * SP + kK * p);
#pragma unroll
                for (int k = 0; k < kK; ++k) h0[k] = v[k];
            } else {
#pragma unroll
                for (int k = 0; k < kK; ++k) h0[k] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < kSub; ++i) {
                const Slot s = row[t + i];
#pragma unroll
                for (int k = 0; k < kK; ++k) {
                    decay[i][k] = exp2_hw(s.e * rate[k]);
                    h[i][k] = fmaf(decay[i][k], i ? h[i - 1][k] : h0[k], s.ex * sB[(t + i) * SP + kK * p + k]);
                }
            }
            float dA_sub[kK] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = kSub - 1; i >= 0; --i) {
                const Slot s = row[t + i];
                float gb = 0.f, qa = 0.f, y = 0.f, vB[kK], vC[kK], q[2];
#pragma unroll
                for (int k = 0; k < kK; ++k) {
                    const float b = sB[(t + i) * SP + kK * p + k], c = sC[(t + i) * SP + kK * p + k];
                    const float g = fmaf(c, s.dy, carry[k]);
                    y = fmaf(c, h[i][k], y);
                    vC[k] = s.dy * h[i][k];
                    vB[k] = g * s.ex;
                    gb = fmaf(g, b, gb);
                    carry[k] = g * decay[i][k];
                    const float kept = carry[k] * (i ? h[i - 1][k] : h0[k]);
                    qa = fmaf(kept, rate[k], qa);
                    dA_sub[k] = fmaf(kept, s.e, dA_sub[k]);
                }
                gb = channel_sum<P>(gb);
                qa = channel_sum<P>(qa);
                y = channel_sum<P>(y);
                if (p == 0) {
                    row[t + i].e = gb;
                    row[t + i].ex = qa;
                    row[t + i].dy = y;
                }
                wave_sums<P>(vB, vC, q);
                if ((lane & 15) < P) {
                    red[wave][0][i * RED + kK * p + channel_state(lane)] = q[0];
                    red[wave][1][i * RED + kK * p + channel_state(lane)] = q[1];
                }
            }
#pragma unroll
            for (int k = 0; k < kK; ++k) dA[k] += dA_sub[k];
            __syncthreads();
            // over the waves of the workgroup, lanes along the sequence
            for (int i = threadIdx.x; i < 2 * kSub * SP; i += blockDim.x) {
                const int step = i & (kSub - 1), s = (i / kSub) & (SP - 1), which = i / (kSub * SP);
                const long tt = t0 + t + step;
                if (s >= a.S || tt >= a.L) continue;
                float v = 0.f;
                for (int w = 0; w < waves; ++w) v += red[w][which][step * RED + s];
                const long o = ((at.n * a.G + at.g) * a.S + s) * a.L + tt;
                if (a.blocks_d == 1) store_elem<BF16>(which ? a.dC : a.dB, o, v);
                else a.part_bc[(static_cast<long>(which) * a.blocks_d + at.cb) * a.N * a.G * a.S * a.L + o] = v;
            }
            __syncthreads();
        }
        // rows again: the gradients of x, dt and z
#pragma unroll
        for (int q = 0; q < PASSES; ++q) {
            const int r = q * RPP + lane / LPR, c = 8 * (lane % LPR);
            if (r >= CW || base + r >= a.Dg || t0 + c >= a.L) continue;
            const long dr = static_cast<long>(at.g) * a.Dg + base + r, o = (at.n * a.D + dr) * a.L;
            float x[8], v[8], dout[8], z[8], dx[8], ddt[8], dz[8];
            row_load8<BF16>(scan_row<BF16>(a.x, a.x_sn, a.x_sd, at.n, dr), t0 + c, len, x);
            row_load8<BF16>(scan_row<BF16>(a.dt, a.dt_sn, a.dt_sd, at.n, dr), t0 + c, len, v);
            row_load8<BF16>(scan_row<BF16>(a.dout, a.dout_sn, a.dout_sd, at.n, dr), t0 + c, len, dout);
            if (a.z) row_load8<BF16>(scan_row<BF16>(a.z, a.z_sn, a.z_sd, at.n, dr), t0 + c, len, z);
            const float bias = a.dt_bias ? a.dt_bias[dr] : 0.f, skip = a.skip ? a.skip[dr] : 0.f;
            const Slot* from = mine + r * STRIDE + c;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool in = t0 + c + i < len;
                const float gb = from[i].e, qa = from[i].ex;
                float dy = dout[i];
                if (a.z) {
                    const float sig = sigmoid_of(z[i]);
                    dy *= z[i] * sig;
                    dz[i] = in ? dout[i] * fmaf(skip, x[i], from[i].dy) * (sig * fmaf(z[i], 1.f - sig, 1.f)) : 0.f;
                }
                const float raw = v[i] + bias;
                const float e = a.softplus ? softplus_of(raw) : raw;
                float de = fmaf(gb, x[i], qa * (1.f / kLog2e));
                if (a.softplus) de *= sigmoid_of(raw);
                dx[i] = in ? fmaf(gb, e, skip * dy) : 0.f;
                ddt[i] = in ? de : 0.f;
                dskip[q] = in ? fmaf(dy, x[i], dskip[q]) : dskip[q];
                dbias[q] += ddt[i];
            }
            using E = typename RowElem<BF16>::type;
            row_store8<BF16>(static_cast<E*>(a.dx) + o, t0 + c, a.L, dx);
            row_store8<BF16>(static_cast<E*>(a.ddt) + o, t0 + c, a.L, ddt);
            if (a.z) row_store8<BF16>(static_cast<E*>(a.dz) + o, t0 + c, a.L, dz);
        }
    }
    const long part = at.n * a.nseg + at.seg, rows = static_cast<long>(a.N) * a.nseg;
#pragma unroll
    for (int q = 0; q < PASSES; ++q) {
#pragma unroll
        for (int m = 1; m < LPR; m <<= 1) {
            dskip[q] += lane_xor(dskip[q], m);
            dbias[q] += lane_xor(dbias[q], m);
        }
        const int r = q * RPP + lane / LPR;
        if (lane % LPR || r >= CW || base + r >= a.Dg) continue;
        const long dr = static_cast<long>(at.g) * a.Dg + base + r;
        a.part_d[part * a.D + dr] = dskip[q];
        a.part_d[(rows + part) * a.D + dr] = dbias[q];
    }
    if (!there) return;
    *reinterpret_cast<seq_f32x4*>(a.part_a + (part * a.D + d) * SP + kK * p) = seq_f32x4{dA[0], dA[1], dA[2], dA[3]};
    if (a.dinit && at.seg == 0) {
#pragma unroll
        for (int k = 0; k < kK; ++k)
            if (kK * p + k < a.S) a.dinit[(at.n * a.D + d) * a.S + kK * p + k] = carry[k];
    }
}

// dB and dC from the sums of the workgroups along the channels
template <bool BF16>
__global__ __launch_bounds__(kThreads) void scan_sum_states_kernel(const float* part, void* dB, void* dC, long n, int blocks, long first) {
    const long groups = (n + 7) / 8;
    long i = first + static_cast<long>(blockIdx.x) * kThreads + threadIdx.x;
    if (i >= 2 * groups) return;
    const int which = i >= groups;
    i = 8 * (i - which * groups);
    float v[8] = {}, u[8];
    for (int b = 0; b < blocks; ++b) {
        row_load8<false>(part + (static_cast<long>(which) * blocks + b) * n, i, n, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += u[e];
    }
    row_store8<BF16>(which ? dC : dB, i, n, v);
}

// columns of a matrix [rows][cols] summed in 64 bits: 16 columns, 64 shares of the rows a workgroup
constexpr int kCols = 16, kShares = 64;
__global__ __launch_bounds__(kCols* kShares) void scan_sum_rows_kernel(const float* part, float* out, long rows, long cols, int SP, int S) {
    __shared__ double sums[kShares][kCols];
    const int c = threadIdx.x % kCols, share = threadIdx.x / kCols;
    const long col = static_cast<long>(blockIdx.x) * kCols + c;
    double sum = 0.0;
    if (col < cols) {
#pragma unroll 8
        for (long r = share; r < rows; r += kShares) sum += static_cast<double>(part[r * cols + col]);
    }
    sums[share][c] = sum;
    __syncthreads();
    if (share || col >= cols) return;
    for (int i = 1; i < kShares; ++i) sum += sums[i][c];
    const long d = col / SP;
    const int s = static_cast<int>(col - d * SP);
    if (s < S) out[d * S + s] = static_cast<float>(sum);
}

hipError_t sum_rows(const float* part, float* out, long rows, long cols, int SP, int S, hipStream_t st) {
    return launch_kernel(scan_sum_rows_kernel, dim3(static_cast<unsigned>(cdiv(cols, kCols))), dim3(kCols * kShares), 0, st, part, out, rows, cols, SP, S);
}

template <bool BF16, int P>
hipError_t bwd_launch(ScanArgs a, const ScanPlan& p, hipStream_t st) {
    const dim3 block(static_cast<unsigned>(p.waves * kSeqWave));
    const long most = kSeqMostThreads / block.x, blocks = scan_blocks(a);
    for (int stage = p.nseg > 1 ? 0 : 2; stage < 3; ++stage) {
        if (stage == 1) {
            const long threads = static_cast<long>(a.N) * a.D * kK * P;
            a.first = 0;
            const hipError_t e = launch_kernel(scan_join_back_kernel, dim3(static_cast<unsigned>(cdiv(threads, kThreads))), dim3(kThreads), 0, st, a, kK * P);
            if (e != hipSuccess) return e;
            continue;
        }
        for (a.first = 0; a.first < blocks; a.first += most) {
            const long left = blocks - a.first;
            const dim3 grid(static_cast<unsigned>(left < most ? left : most));
            const hipError_t e = launch_kernel(stage == 0 ? scan_adjoint_kernel<BF16, P> : scan_bwd_kernel<BF16, P>, grid, block, 0, st, a);
            if (e != hipSuccess) return e;
        }
    }
    if (p.blocks_d > 1) {
        const long n = static_cast<long>(a.N) * a.G * a.S * a.L, threads = 2 * ((n + 7) / 8);
        for (long first = 0; first < threads; first += kSeqMostThreads) {
            const long left = threads - first;
            const hipError_t e = launch_kernel(scan_sum_states_kernel<BF16>, dim3(static_cast<unsigned>(cdiv(left < kSeqMostThreads ? left : kSeqMostThreads, kThreads))),
                                               dim3(kThreads), 0, st, a.part_bc, a.dB, a.dC, n, p.blocks_d, first);
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

template <bool BF16>
hipError_t bwd_type(const ScanArgs& a, const ScanPlan& p, hipStream_t st) {
    switch (p.P) {
        case 1: return bwd_launch<BF16, 1>(a, p, st);
        case 2: return bwd_launch<BF16, 2>(a, p, st);
        case 4: return bwd_launch<BF16, 4>(a, p, st);
        case 8: return bwd_launch<BF16, 8>(a, p, st);
        default: return bwd_launch<BF16, 16>(a, p, st);
    }
}

}  // namespace

hipError_t scan_bwd_launch(const ScanArgs& a, const ScanPlan& p, int bf16, float* dA, float* dskip, float* dbias, hipStream_t st) {
    hipError_t e = bf16 ? bwd_type<true>(a, p, st) : bwd_type<false>(a, p, st);
    const long rows = static_cast<long>(a.N) * a.nseg;
    const int SP = kK * p.P;
    if (e == hipSuccess) e = sum_rows(a.part_a, dA, rows, static_cast<long>(a.D) * SP, SP, a.S, st);
    if (e == hipSuccess && dskip) e = sum_rows(a.part_d, dskip, rows, a.D, 1, 1, st);
    if (e == hipSuccess && dbias) e = sum_rows(a.part_d + rows * a.D, dbias, rows, a.D, 1, 1, st);
    return e;
}

}  // namespace conv1d
