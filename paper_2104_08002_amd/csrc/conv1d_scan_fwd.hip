// Selective scan, forward, and its form for single tokens.  The recurrence is stated in conv1d_scan.h.
// A sequence is one segment where samples and channels fill the chip.  Otherwise it is cut: a first launch finds what each
// segment adds to its state from a state of zero, a second joins them (the decay over a segment is exp(A sum e)), a third
// scans the segments from their states.  That takes the exponentials twice, 16 issue slots per state and step against 9.
// Bound by instruction issue: N = 8, D = 512, L = 8192, S = 16 in bfloat16 with the states kept takes 113 + 6 + 163 us, 4 clocks an
// instruction on 1024 SIMDs and 3.3 TB/s in the last launch.
#include "conv1d_scan.h"

namespace conv1d {
namespace {

constexpr int kThreads = 256;

// The lane's row of a tile.  INSIDE: the tile lies within the sequence: no masks.
template <bool BF16, int P, int T, bool ENDS>
struct FwdRow {
    using R = ScanRows<P, T>;
    static constexpr int V = R::V;
    using E = typename RowElem<BF16>::type;
    const E *x, *dt, *z;
    E* out;
    float bias, skip;
    bool real;
    int c, at;          // first step of the lane within the tile, its place in LDS
    float u[V], w[V];   // x and z of the tile

    __device__ __forceinline__ FwdRow(const ScanArgs& a, const ScanPlace& p, int base, int lane) {
        const int row = lane / R::LPR;
        c = V * (lane % R::LPR);
        at = row * R::RS + c;
        real = base + row < a.Dg;
        const long d = static_cast<long>(p.g) * a.Dg + (real ? base + row : 0);
        x = scan_row<BF16>(a.x, a.x_sn, a.x_sd, p.n, d);
        dt = scan_row<BF16>(a.dt, a.dt_sn, a.dt_sd, p.n, d);
        bias = a.dt_bias ? a.dt_bias[d] : 0.f;
        if (ENDS) return;
        z = a.z ? scan_row<BF16>(a.z, a.z_sn, a.z_sd, p.n, d) : nullptr;
        out = static_cast<E*>(a.out) + p.n * a.out_sn + d * a.out_sd;
        skip = a.skip ? a.skip[d] : 0.f;
    }
    // e and e x into LDS
    template <bool INSIDE>
    __device__ __forceinline__ void stage(const ScanArgs& a, int t0, int len, float* sE, float* sX) {
        float e[V], ex[V];
        scan_load<BF16, INSIDE>(x, t0 + c, len, a.L, u);
        scan_load<BF16, INSIDE>(dt, t0 + c, len, a.L, e);
        if (!ENDS && z) scan_load<BF16, INSIDE>(z, t0 + c, len, a.L, w);
#pragma unroll
        for (int i = 0; i < V; ++i) e[i] += bias;
        if (a.softplus) {
#pragma unroll
            for (int i = 0; i < V; ++i) e[i] = softplus_of(e[i]);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (!INSIDE) e[i] = t0 + c + i < len ? e[i] : 0.f;
            ex[i] = u[i] * e[i];
        }
        lds_put(sE + at, e);
        lds_put(sX + at, ex);
    }
    // the output from the sums in LDS
    template <bool INSIDE>
    __device__ __forceinline__ void finish(const ScanArgs& a, int t0, int len, const float* sY) const {
        if (!real || t0 + c >= a.L) return;
        float y[V];
        lds_get(sY + at, y);
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = fmaf(skip, u[i], y[i]);
        if (z) {
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] *= w[i] * sigmoid_of(w[i]);
        }
        if (!INSIDE) {
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = t0 + c + i < len ? y[i] : 0.f;
            scan_store<BF16>(out, t0 + c, a.L, y);
        } else {
            scan_store<BF16>(out, t0 + c, t0 + c + V, y);
        }
    }
};

// ENDS: no output but the state each segment adds and the sum of its steps.  (P = 16: LDS holds three workgroups of a CU.)
template <bool BF16, int K, int P, bool ENDS>
__global__ __launch_bounds__(kScanWaves* kSeqWave, P == 16 ? 3 : 4) void scan_fwd_kernel(ScanArgs a) {
    constexpr int SP = K * P, T = scan_tile(P);
    using R = ScanRows<P, T>;
    __shared__ __align__(16) float sE[kScanWaves][R::CW * R::RS], sX[kScanWaves][R::CW * R::RS];  // e (then y) and e x
    __shared__ __align__(16) float sB[T * SP], sC[ENDS ? 4 : T * SP];
    const ScanPlace at = scan_place(a);
    if (ENDS && at.seg == a.nseg - 1) return;             // nothing comes behind the last segment
    const int lane = threadIdx.x & (kSeqWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int p = lane & (P - 1), cl = lane / P;
    const int len = seq_length(a.lengths, at.n, a.L);
    const int base = (at.cb * waves + wave) * R::CW;      // first channel of the wave, within its group
    const bool there = base + cl < a.Dg;                  // (a lane without a channel goes along with the group's first)
    const long d = static_cast<long>(at.g) * a.Dg + (there ? base + cl : 0);

    float rate[K], h[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int s = K * p + k;
        rate[k] = scan_rate(a.A, a.S, d, s, there);
        h[k] = 0.f;
        if (ENDS) continue;
        if (a.nseg > 1) h[k] = there ? a.starts[((at.n * a.D + d) * a.nseg + at.seg) * SP + s] : 0.f;
        else if (a.init && there && s < a.S) h[k] = a.init[(at.n * a.D + d) * a.S + s];
    }
    FwdRow<BF16, P, T, ENDS> row(a, at, base, lane);
    using E = typename RowElem<BF16>::type;
    ScanStates<BF16, SP, T, !ENDS> states{static_cast<const E*>(a.B) + at.n * a.b_sn + at.g * a.b_sg,
                                          static_cast<const E*>(a.C) + at.n * a.c_sn + at.g * a.c_sg, a.b_ss, a.c_ss, a.S, a.L, {}};
    const int t_begin = at.seg * a.seg_len, t_end = min(a.L, t_begin + a.seg_len);
    float sum = 0.f;
    for (int t0 = t_begin; t0 < t_end; t0 += T) {
        const bool inside = t0 + T <= len;                // no masks
        states.begin(t0, len);
        if (inside) row.template stage<true>(a, t0, len, sE[wave], sX[wave]);
        else row.template stage<false>(a, t0, len, sE[wave], sX[wave]);
        states.finish(t0, len, sB, sC);
        if (t0 == t_begin) make_rates(rate);
        __syncthreads();
        float* e_row = sE[wave] + cl * R::RS;
        const float* ex_row = sX[wave] + cl * R::RS;
#pragma unroll 1
        for (int t = 0; t < T; t += kSub) {
            if (!ENDS && a.saved && there && t0 + t < a.L) {
                float* to = a.saved + ((at.n * a.chunks + (t0 + t) / kSub) * a.D + d) * SP + K * p;
                put_states<K>(to, h);
            }
            float part = 0.f;
#pragma unroll
            for (int j = 0; j < kSub; j += 4) {
                const scan_f32x4 e = *reinterpret_cast<const scan_f32x4*>(e_row + t + j), ex = *reinterpret_cast<const scan_f32x4*>(ex_row + t + j);
                float y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const States<K> b = states_at<K>(sB + (t + j + i) * SP + K * p);
                    States<K> o;
                    if (!ENDS) o = states_at<K>(sC + (t + j + i) * SP + K * p);
                    float v = 0.f;
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        h[k] = fmaf(exp2_hw(e[i] * rate[k]), h[k], ex[i] * b[k]);
                        if (!ENDS) v = k ? fmaf(o[k], h[k], v) : o[k] * h[k];
                    }
                    if (ENDS) {
                        part += e[i];
                    } else {
                        y[i] = channel_sum<P>(v);
                        keep_here(y[i]);
                    }
                }
                if (!ENDS && p == 0) *reinterpret_cast<scan_f32x4*>(e_row + t + j) = scan_f32x4{y[0], y[1], y[2], y[3]};
            }
            sum += part;
        }
        __syncthreads();
        if (ENDS) continue;
        if (inside) row.template finish<true>(a, t0, len, sE[wave]);
        else row.template finish<false>(a, t0, len, sE[wave]);
    }
    if (!there) return;
    if (ENDS) {
        const long i = (at.n * a.D + d) * a.nseg + at.seg;
        put_states<K>(a.starts + i * SP + K * p, h);
        if (p == 0) a.sums[i] = sum;
    } else if (a.final && at.seg == a.nseg - 1) {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (K * p + k < a.S) a.final[(at.n * a.D + d) * a.S + K * p + k] = h[k];
    }
}

constexpr int kK = 4;  // states of a lane in the step

struct ScanStepArgs {
    const void *x, *dt, *B, *C, *z;
    const float *A, *skip, *dt_bias;
    float* state;  // [N][D][S]
    void* out;
    long x_sn, dt_sn, z_sn, out_sn, b_sn, b_sg, c_sn, c_sg;
    long rows, first;  // first row of the launch, and all of them: N * D
    int D, S, Dg, softplus;
};

// One token: P lanes per channel as in the scan.  Bound by the state's way through memory.
template <bool BF16, int P>
__global__ __launch_bounds__(kThreads) void scan_step_kernel(ScanStepArgs a) {
    const long thread = static_cast<long>(blockIdx.x) * kThreads + threadIdx.x;
    const int p = static_cast<int>(thread & (P - 1));
    const long row = a.first + thread / P;
    const bool there = row < a.rows;
    const long n = there ? row / a.D : 0, d = there ? row - n * a.D : 0, g = d / a.Dg;
    const float x = load_elem<BF16>(a.x, n * a.x_sn + d);
    float e = load_elem<BF16>(a.dt, n * a.dt_sn + d) + (a.dt_bias ? a.dt_bias[d] : 0.f);
    if (a.softplus) e = softplus_of(e);
    const float ex = e * x;
    float y = 0.f;
    float* state = a.state + (n * a.D + d) * a.S;
    float h[kK];
    const bool whole = (a.S & (kK - 1)) == 0 && kK * p < a.S;
    if (there && whole) {
        const seq_f32x4 v = *reinterpret_cast<const seq_f32x4*>(state + kK * p);
#pragma unroll
        for (int k = 0; k < kK; ++k) h[k] = v[k];
    }
#pragma unroll
    for (int k = 0; k < kK; ++k) {
        const int s = kK * p + k;
        if (!there || s >= a.S) continue;
        if (!whole) h[k] = state[s];
        const float b = load_elem<BF16>(a.B, n * a.b_sn + g * a.b_sg + s), c = load_elem<BF16>(a.C, n * a.c_sn + g * a.c_sg + s);
        h[k] = fmaf(exp2_hw(e * rate_of(a.A[d * a.S + s])), h[k], ex * b);
        y = fmaf(c, h[k], y);
        if (!whole) state[s] = h[k];
    }
    if (there && whole) *reinterpret_cast<seq_f32x4*>(state + kK * p) = seq_f32x4{h[0], h[1], h[2], h[3]};
    y = channel_sum<P>(y);
    if (!there || p) return;
    y = fmaf(a.skip ? a.skip[d] : 0.f, x, y);
    if (a.z) {
        const float z = load_elem<BF16>(a.z, n * a.z_sn + d);
        y *= z * sigmoid_of(z);
    }
    store_elem<BF16>(a.out, n * a.out_sn + d, y);
}

template <bool BF16, int K, int P>
hipError_t fwd_launch(ScanArgs a, const ScanPlan& p, hipStream_t st) {
    const dim3 block(static_cast<unsigned>(p.waves * kSeqWave));
    const long most = kSeqMostThreads / block.x, blocks = scan_blocks(a);
    for (int stage = p.nseg > 1 ? 0 : 2; stage < 3; ++stage) {
        if (stage == 1) {
            const hipError_t e = scan_join_launch<false>(a.starts, a.sums, a.init, a.A, a.N, a.D, a.S, K * P, a.nseg, st);
            if (e != hipSuccess) return e;
            continue;
        }
        for (long first = 0; first < blocks; first += most) {
            a.first = static_cast<int>(first);
            const long left = blocks - first;
            const dim3 grid(static_cast<unsigned>(left < most ? left : most));
            const hipError_t e = launch_kernel(stage == 0 ? scan_fwd_kernel<BF16, K, P, true> : scan_fwd_kernel<BF16, K, P, false>, grid, block, 0, st, a);
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

template <bool BF16, int P>
hipError_t step_launch(ScanStepArgs a, hipStream_t st) {
    constexpr long most = kSeqMostThreads / P;
    for (a.first = 0; a.first < a.rows; a.first += most) {
        const long left = a.rows - a.first, rows = left < most ? left : most;
        const hipError_t e = launch_kernel(scan_step_kernel<BF16, P>, dim3(static_cast<unsigned>(cdiv(rows * P, kThreads))), dim3(kThreads), 0, st, a);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// lanes of a channel in the step, of 4 states each
int lanes_of(int S) {
    int P = 1;
    while (kK * P < S) P *= 2;
    return P;
}

// states of a channel in the scan, with the padding
int padded_states(int S) {
    int SP = 4;
    while (SP < S) SP *= 2;
    return SP;
}

bool scan_ok(const conv1d_scan_t* p) {
    if (!p || !p->x || !p->dt || !p->A || !p->B || !p->C) return false;
    if (p->N < 1 || p->D < 1 || p->L < 1 || p->S < 1 || p->G < 1 || p->D % p->G) return false;
    if (p->dtype != CONV1D_FP32 && p->dtype != CONV1D_BF16) return false;
    const size_t size = p->dtype == CONV1D_BF16 ? 2 : 4;
    for (const void* v : {p->x, p->dt, p->B, p->C, p->z})
        if (!seq_aligned(v, size)) return false;
    for (const void* v : {static_cast<const void*>(p->A), static_cast<const void*>(p->skip), static_cast<const void*>(p->dt_bias),
                          static_cast<const void*>(p->init), static_cast<const void*>(p->lengths)})
        if (!seq_aligned(v, 4)) return false;
    return (p->flags & ~CONV1D_SCAN_SOFTPLUS) == 0;
}

// rows and the lanes of their states are counted in 31 bits
bool scan_sizes_ok(const conv1d_scan_t* p) {
    return p->S <= kMostStates && static_cast<long>(p->N) * p->D <= 0x7fffffffL / 64 && p->L <= 1 << 30;
}

ScanArgs scan_args(const conv1d_scan_t* p, const ScanPlan& plan) {
    ScanArgs a{};
    a.x = p->x; a.dt = p->dt; a.B = p->B; a.C = p->C; a.z = p->z;
    a.A = p->A; a.skip = p->skip; a.dt_bias = p->dt_bias; a.init = p->init; a.lengths = p->lengths;
    a.N = p->N; a.D = p->D; a.L = p->L; a.S = p->S; a.G = p->G; a.Dg = p->D / p->G;
    a.softplus = (p->flags & CONV1D_SCAN_SOFTPLUS) != 0;
    a.x_sn = p->x_sn; a.x_sd = p->x_sd; a.dt_sn = p->dt_sn; a.dt_sd = p->dt_sd; a.z_sn = p->z_sn; a.z_sd = p->z_sd;
    a.b_sn = p->b_sn; a.b_sg = p->b_sg; a.b_ss = p->b_ss; a.c_sn = p->c_sn; a.c_sg = p->c_sg; a.c_ss = p->c_ss;
    a.nseg = plan.nseg; a.seg_len = plan.seg_len; a.chunks = plan.chunks; a.blocks_d = plan.blocks_d;
    return a;
}

size_t round256(size_t n) { return (n + 255) & ~static_cast<size_t>(255); }

// the states and the sums of a split sequence
size_t split_bytes(int N, int D, const ScanPlan& p) {
    const size_t rows = static_cast<size_t>(N) * p.nseg * D;
    return p.nseg > 1 ? round256(rows * p.K * p.P * sizeof(float)) + round256(rows * sizeof(float)) : 0;
}

// where the parts of a backward call's workspace begin
struct BwdSpace {
    size_t carries, sums, params, bc, total;
};
BwdSpace bwd_space(int N, int D, int L, int S, int G, const ScanPlan& p) {
    const size_t rows = static_cast<size_t>(N) * p.nseg * D;
    BwdSpace w{};
    w.carries = 0;
    w.sums = w.carries + (p.nseg > 1 ? round256(rows * p.K * p.P * sizeof(float)) : 0);
    w.params = w.sums + (p.nseg > 1 ? round256(rows * sizeof(float)) : 0);
    w.bc = w.params + round256(rows * (p.K * p.P + 2) * sizeof(float));
    w.total = w.bc + (p.blocks_d > 1 ? round256(2 * sizeof(float) * static_cast<size_t>(p.blocks_d) * N * G * S * L) : 0);
    return w;
}

int status_of(hipError_t e) { return e == hipSuccess ? CONV1D_OK : CONV1D_EHIP; }

}  // namespace

// Segments: as many as give the chip's 1024 SIMDs 8 waves each (2 to 3 turns of what fits beside each other: the turns even out;
// N = 8, D = 512, L = 8192, S = 16 backwards with 3, 5, 8, 10 and 16 waves: 538, 524, 502, 527 and 505 us), none shorter than a
// tile; one where the rows alone do.  A wave alone on its SIMD issues an instruction in 8 clocks, so that few rows want short
// segments: N = 3, D = 49, L = 4999, S = 5 in FP32 takes 17 us in the last launch backwards in segments of 32 steps, 36 in 128.
// Two launches more are worth it from 5 tiles on forwards, 3 backwards (S = 16: a tile takes 4 and 11 us, a cut sequence 14 and
// 25 in all, and a launch 3 of the host's).
ScanPlan scan_plan(int N, int D, int L, int S, int G, bool back) {
    ScanPlan p{};
    const int SP = padded_states(S);
    p.K = SP < 16 ? SP / 4 : 4;
    p.P = SP / p.K;
    const int CW = kSeqWave / p.P, Dg = D / G;
    const int need = cdiv(Dg, CW);
    p.waves = need < kScanWaves ? need : kScanWaves;
    p.blocks_d = cdiv(need, p.waves);
    p.chunks = cdiv(L, kSub);
    const long waves = static_cast<long>(N) * G * p.blocks_d * p.waves, room = 1024L * 8;
    const int unit = scan_tile(p.P);
    const long tiles = cdiv(L, unit);
    long nseg = room / waves;
    if (nseg > tiles) nseg = tiles;
    if (nseg < 1 || tiles < (back ? 3 : 5)) nseg = 1;
    p.seg_len = unit * cdiv(tiles, nseg);
    p.nseg = cdiv(L, p.seg_len);
    return p;
}

hipError_t scan_fwd_launch(const ScanArgs& a, const ScanPlan& p, int bf16, hipStream_t st) {
    switch (p.K * p.P) {
        case 4: return bf16 ? fwd_launch<true, 1, 4>(a, p, st) : fwd_launch<false, 1, 4>(a, p, st);
        case 8: return bf16 ? fwd_launch<true, 2, 4>(a, p, st) : fwd_launch<false, 2, 4>(a, p, st);
        case 16: return bf16 ? fwd_launch<true, 4, 4>(a, p, st) : fwd_launch<false, 4, 4>(a, p, st);
        case 32: return bf16 ? fwd_launch<true, 4, 8>(a, p, st) : fwd_launch<false, 4, 8>(a, p, st);
        default: return bf16 ? fwd_launch<true, 4, 16>(a, p, st) : fwd_launch<false, 4, 16>(a, p, st);
    }
}

}  // namespace conv1d

using namespace conv1d;

extern "C" {

size_t conv1d_scan_fwd_workspace_bytes(int N, int D, int L, int S, int G) {
    if (N < 1 || D < 1 || L < 1 || S < 1 || S > kMostStates || G < 1 || D % G) return 0;
    return split_bytes(N, D, scan_plan(N, D, L, S, G, false));
}

size_t conv1d_scan_saved_bytes(int N, int D, int L, int S) {
    if (N < 1 || D < 1 || L < 1 || S < 1 || S > kMostStates) return 0;
    return sizeof(float) * N * static_cast<size_t>(cdiv(L, kSub)) * D * padded_states(S);
}

int conv1d_scan_fwd(const conv1d_scan_t* p, void* y, long y_sn, long y_sd, float* final, void* saved, void* workspace,
                    size_t workspace_bytes, void* stream) {
    if (!scan_ok(p) || !y) return CONV1D_EINVAL;
    if (!seq_aligned(y, p->dtype == CONV1D_BF16 ? 2 : 4) || !seq_aligned(final, 4) || !seq_aligned(saved, 16) || !seq_aligned(workspace, 256))
        return CONV1D_EINVAL;
    if (!scan_sizes_ok(p)) return CONV1D_EUNSUPPORTED;
    const ScanPlan plan = scan_plan(p->N, p->D, p->L, p->S, p->G, false);
    const size_t need = split_bytes(p->N, p->D, plan);
    if (need && (!workspace || workspace_bytes < need)) return CONV1D_EWORKSPACE;
    ScanArgs a = scan_args(p, plan);
    a.out = y; a.out_sn = y_sn; a.out_sd = y_sd; a.final = final; a.saved = static_cast<float*>(saved);
    if (need) {
        a.starts = static_cast<float*>(workspace);
        a.sums = a.starts + round256(static_cast<size_t>(p->N) * plan.nseg * p->D * plan.K * plan.P * sizeof(float)) / sizeof(float);
    }
    return status_of(scan_fwd_launch(a, plan, p->dtype == CONV1D_BF16, static_cast<hipStream_t>(stream)));
}

size_t conv1d_scan_bwd_workspace_bytes(int N, int D, int L, int S, int G) {
    if (N < 1 || D < 1 || L < 1 || S < 1 || S > kMostStates || G < 1 || D % G) return 0;
    return bwd_space(N, D, L, S, G, scan_plan(N, D, L, S, G, true)).total;
}

int conv1d_scan_bwd(const conv1d_scan_t* p, const void* dy, long dy_sn, long dy_sd, const float* dfinal, const void* saved, void* dx,
                    void* ddt, float* dA, void* dB, void* dC, float* dskip, void* dz, float* ddt_bias, float* dinit, void* workspace,
                    size_t workspace_bytes, void* stream) {
    if (!scan_ok(p) || !dy || !saved || !dx || !ddt || !dA || !dB || !dC) return CONV1D_EINVAL;
    if ((p->z != nullptr) != (dz != nullptr) || (dskip && !p->skip) || (ddt_bias && !p->dt_bias)) return CONV1D_EINVAL;
    const size_t size = p->dtype == CONV1D_BF16 ? 2 : 4;
    for (const void* v : {dy, static_cast<const void*>(dx), static_cast<const void*>(ddt), static_cast<const void*>(dB),
                          static_cast<const void*>(dC), static_cast<const void*>(dz)})
        if (!seq_aligned(v, size)) return CONV1D_EINVAL;
    for (const float* v : {dfinal, static_cast<const float*>(dA), static_cast<const float*>(dskip), static_cast<const float*>(ddt_bias),
                           static_cast<const float*>(dinit)})
        if (!seq_aligned(v, 4)) return CONV1D_EINVAL;
    if (!seq_aligned(saved, 16) || !seq_aligned(workspace, 256)) return CONV1D_EINVAL;
    if (!scan_sizes_ok(p)) return CONV1D_EUNSUPPORTED;
    const ScanPlan plan = scan_plan(p->N, p->D, p->L, p->S, p->G, true);
    const BwdSpace w = bwd_space(p->N, p->D, p->L, p->S, p->G, plan);
    if (!workspace || workspace_bytes < w.total) return CONV1D_EWORKSPACE;
    char* ws = static_cast<char*>(workspace);
    ScanArgs a = scan_args(p, plan);
    a.saved = const_cast<float*>(static_cast<const float*>(saved));
    a.dout = dy; a.dout_sn = dy_sn; a.dout_sd = dy_sd; a.dfinal = dfinal;
    a.dx = dx; a.ddt = ddt; a.dz = dz; a.dB = dB; a.dC = dC; a.dinit = dinit;
    a.carries = reinterpret_cast<float*>(ws + w.carries);
    a.sums = reinterpret_cast<float*>(ws + w.sums);
    a.part_p = reinterpret_cast<float*>(ws + w.params);
    a.part_bc = reinterpret_cast<float*>(ws + w.bc);
    return status_of(scan_bwd_launch(a, plan, p->dtype == CONV1D_BF16, dA, dskip, ddt_bias, static_cast<hipStream_t>(stream)));
}

int conv1d_scan_step(const conv1d_scan_t* p, float* state, void* y, long y_sn, void* stream) {
    if (!scan_ok(p) || !state || !y || p->L != 1 || p->init || p->lengths) return CONV1D_EINVAL;
    if (!seq_aligned(y, p->dtype == CONV1D_BF16 ? 2 : 4) || !seq_aligned(state, 4)) return CONV1D_EINVAL;
    if (!scan_sizes_ok(p)) return CONV1D_EUNSUPPORTED;
    ScanStepArgs a{};
    a.x = p->x; a.dt = p->dt; a.B = p->B; a.C = p->C; a.z = p->z; a.A = p->A; a.skip = p->skip; a.dt_bias = p->dt_bias;
    a.state = state; a.out = y;
    a.x_sn = p->x_sn; a.dt_sn = p->dt_sn; a.z_sn = p->z_sn; a.out_sn = y_sn;
    a.b_sn = p->b_sn; a.b_sg = p->b_sg; a.c_sn = p->c_sn; a.c_sg = p->c_sg;
    a.rows = static_cast<long>(p->N) * p->D;
    a.D = p->D; a.S = p->S; a.Dg = p->D / p->G; a.softplus = (p->flags & CONV1D_SCAN_SOFTPLUS) != 0;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool b = p->dtype == CONV1D_BF16;
    switch (lanes_of(p->S)) {
        case 1: return status_of(b ? step_launch<true, 1>(a, st) : step_launch<false, 1>(a, st));
        case 2: return status_of(b ? step_launch<true, 2>(a, st) : step_launch<false, 2>(a, st));
        case 4: return status_of(b ? step_launch<true, 4>(a, st) : step_launch<false, 4>(a, st));
        case 8: return status_of(b ? step_launch<true, 8>(a, st) : step_launch<false, 8>(a, st));
        default: return status_of(b ? step_launch<true, 16>(a, st) : step_launch<false, 16>(a, st));
    }
}

}  // extern "C"
