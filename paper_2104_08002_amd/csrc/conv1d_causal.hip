// Depthwise causal convolution of S <= 8 taps, one filter per channel:
//   p[n][c][t] = bias[c] + sum_{s<S} w[c][s] * xe[n][c][t + s],   xe = the S - 1 inputs before the sequence, then x
//   y = p, or p * sigmoid(p) (SiLU)
// and its gradients dp = dy * act'(p), dx[j] = sum_s w[s] dp[j + S - 1 - s], dw[s] = sum_{n,t} dp[t] xe[t + s], dbias = sum dp.
// Bound by memory: x read once and y written once (forward), x and dy read and dx written (backward; p is computed again from
// x, which costs S products against another tensor through memory).
#include "conv1d_sequence.h"

namespace conv1d {
namespace {

constexpr int kThreads = 256;
constexpr int kV = 8;    // outputs of a lane per step
constexpr int kMostTaps = 8;

struct CausalArgs {
    const void* x;
    const void* w;         // [C][S]
    const float* bias;     // [C] or nullptr
    const void* init;      // [N][C][S - 1] or nullptr: zeros
    const int* lengths;    // [N] or nullptr
    void* y;
    void* final;           // [N][C][S - 1] or nullptr
    // backward
    const void* dy;
    const void* dfinal;    // [N][C][S - 1] or nullptr
    void* dx;
    void* dinit;           // [N][C][S - 1] or nullptr
    float* partial;        // [C][S + 1][N * pieces] or nullptr
    int N, C, L, silu;
    long x_sn, x_sc, y_sn, y_sc, dy_sn, dy_sc;
    int lg;                // log2 of the lanes of a piece
    int pieces;            // of a row
    long first, units;     // first unit of the launch, and all of them: N * C * pieces
};

// A piece of a row belongs to 2^lg lanes, which take one step (backwards: R) of kV outputs each through it.
struct Piece {
    long n, c, unit;
    int piece, sub;        // which of the row, lane within it
    bool there;
};
__device__ __forceinline__ Piece piece_of(const CausalArgs& a) {
    Piece p;
    const long thread = static_cast<long>(blockIdx.x) * kThreads + threadIdx.x;
    p.unit = a.first + (thread >> a.lg);
    p.sub = static_cast<int>(thread & ((1 << a.lg) - 1));
    p.there = p.unit < a.units;
    const long row = (p.there ? p.unit : 0) / a.pieces;
    p.piece = static_cast<int>((p.there ? p.unit : 0) - row * a.pieces);
    p.n = row / a.C;
    p.c = row - p.n * a.C;
    return p;
}

// xe[at] .. xe[at + 7 + S - 1] for outputs at .. at + 7: the row's elements at - (S - 1) .. at + 7.  INSIDE: they are all there.
template <bool BF16, int S, bool INSIDE>
__device__ __forceinline__ void load_window(const CausalArgs& a, const Piece& p, const void* row, int at, int len, float (&v)[kV + S - 1]) {
    float cur[kV], before[kV];
    if constexpr (INSIDE) {
        row_load8_inside<BF16>(row, at, cur);
        if (S > 1) row_load8_inside<BF16>(row, at - kV, before);
    } else {
        row_load8<BF16>(row, at, len, cur);
        if (S > 1) row_load8<BF16>(row, at - kV, len, before);
        if (S > 1 && at == 0 && a.init) {
#pragma unroll
            for (int s = 0; s < S - 1; ++s) before[kV - (S - 1) + s] = load_elem<BF16>(a.init, (p.n * a.C + p.c) * (S - 1) + s);
        }
    }
#pragma unroll
    for (int s = 0; s < S - 1; ++s) v[s] = before[kV - (S - 1) + s];
#pragma unroll
    for (int e = 0; e < kV; ++e) v[S - 1 + e] = cur[e];
}

template <bool BF16, int S, bool INSIDE>
__device__ __forceinline__ void forward_step(const CausalArgs& a, const Piece& p, const typename RowElem<BF16>::type* x,
                                             typename RowElem<BF16>::type* y, int t, int len, const float (&w)[S], float bias) {
    float v[kV + S - 1], o[kV];
    load_window<BF16, S, INSIDE>(a, p, x, t, len, v);
#pragma unroll
    for (int e = 0; e < kV; ++e) {
        o[e] = bias;
#pragma unroll
        for (int s = 0; s < S; ++s) o[e] = fmaf(w[s], v[e + s], o[e]);
    }
    if (a.silu) {
#pragma unroll
        for (int e = 0; e < kV; ++e) o[e] *= sigmoid_of(o[e]);
    }
    if constexpr (!INSIDE) {
#pragma unroll
        for (int e = 0; e < kV; ++e) o[e] = t + e < len ? o[e] : 0.f;
        if (p.there && t < a.L) row_store8<BF16>(y, t, a.L, o);
    } else {
        row_store8<BF16>(y, t, t + kV, o);
    }
}

// One step a lane: waves enough hide the loads, more steps in flight only take registers (N = 8, C = 128, L = 20000, S = 4 in
// bfloat16: 16 to 18 us, 4.6 to 5.1 TB/s, what a large copy reaches).
template <bool BF16, int S>
__global__ __launch_bounds__(kThreads) void causal_fwd_kernel(CausalArgs a) {
    const Piece p = piece_of(a);
    const int len = p.there ? seq_length(a.lengths, p.n, a.L) : 0;
    using T = typename RowElem<BF16>::type;
    const T* x = static_cast<const T*>(a.x) + p.n * a.x_sn + p.c * a.x_sc;
    T* y = static_cast<T*>(a.y) + p.n * a.y_sn + p.c * a.y_sc;
    float w[S];
#pragma unroll
    for (int s = 0; s < S; ++s) w[s] = load_elem<BF16>(a.w, p.c * S + s);
    const float bias = a.bias ? a.bias[p.c] : 0.f;
    const int t = ((p.piece << a.lg) + p.sub) * kV;
    if (wave_all(t > 0 && t + kV <= len)) forward_step<BF16, S, true>(a, p, x, y, t, len, w, bias);
    else forward_step<BF16, S, false>(a, p, x, y, t, len, w, bias);
    if (S > 1 && a.final && p.there && t == 0) {
        const long at = (p.n * a.C + p.c) * (S - 1);
#pragma unroll
        for (int s = 0; s < S - 1; ++s) {
            const int j = len + s;  // xe[j]
            float e = 0.f;
            if (j >= S - 1) e = load_elem<BF16>(x, j - (S - 1));
            else if (a.init) e = load_elem<BF16>(a.init, at + j);
            store_elem<BF16>(a.final, at + s, e);
        }
    }
}

// act'(p) for p from the S inputs at v
template <int S>
__device__ __forceinline__ float slope_of(const float* v, const float (&w)[S], float bias) {
    float q = bias;
#pragma unroll
    for (int s = 0; s < S; ++s) q = fmaf(w[s], v[s], q);
    const float sig = sigmoid_of(q);
    return fmaf(q * sig, 1.f - sig, sig);
}

// One step of a lane backwards: positions t .. t + 7.  behind: dp of the S - 1 positions behind the wave's step; those of its first
// positions come back in it.
template <bool BF16, int S, bool INSIDE>
__device__ __forceinline__ void backward_step(const CausalArgs& a, const Piece& p, const typename RowElem<BF16>::type* x,
                                              const typename RowElem<BF16>::type* dy, typename RowElem<BF16>::type* dx, int t, int len,
                                              const float (&w)[S], float bias, float (&behind)[S > 1 ? S - 1 : 1], float (&sum)[S + 1]) {
    float v[kV + S - 1], dp[kV + (S > 1 ? S - 1 : 1)], g[kV], o[kV];
    load_window<BF16, S, INSIDE>(a, p, x, t, len, v);
    if constexpr (INSIDE) row_load8_inside<BF16>(dy, t, g);
    else row_load8<BF16>(dy, t, len, g);
#pragma unroll
    for (int e = 0; e < kV; ++e) dp[e] = g[e];
    if (a.silu) {
#pragma unroll
        for (int e = 0; e < kV; ++e) dp[e] *= slope_of<S>(v + e, w, bias);
    }
    if constexpr (!INSIDE) {
#pragma unroll
        for (int e = 0; e < kV; ++e) dp[e] = t + e < len ? dp[e] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < S - 1; ++i) {
        const float next = lane_next(dp[i]);
        dp[kV + i] = p.sub != (1 << a.lg) - 1 ? next : behind[i];
        behind[i] = a.lg == 6 ? lane_first(dp[i]) : 0.f;
    }
#pragma unroll
    for (int e = 0; e < kV; ++e) {
        o[e] = w[0] * dp[e + S - 1];
#pragma unroll
        for (int s = 1; s < S; ++s) o[e] = fmaf(w[s], dp[e + S - 1 - s], o[e]);
    }
    if constexpr (!INSIDE) {
#pragma unroll
        for (int e = 0; e < kV; ++e) o[e] = t + e < len ? o[e] : 0.f;
    }
    const long state = (p.n * a.C + p.c) * (S - 1);
    if (S > 1 && a.dfinal && t + kV + (S - 1) > len && t < len) {
#pragma unroll
        for (int e = 0; e < kV; ++e) {
            const int f = t + e + (S - 1) - len;  // x[j] is element j + S - 1 - len of the final state
            if (f >= 0 && f < S - 1) o[e] += load_elem<BF16>(a.dfinal, state + f);
        }
    }
    if constexpr (INSIDE) row_store8<BF16>(dx, t, t + kV, o);
    else if (p.there && t < a.L) row_store8<BF16>(dx, t, a.L, o);
#pragma unroll
    for (int e = 0; e < kV; ++e) {
#pragma unroll
        for (int s = 0; s < S; ++s) sum[s] = fmaf(dp[e], v[e + s], sum[s]);
        sum[S] += dp[e];
    }
    if (!INSIDE && S > 1 && t == 0 && a.dinit && p.there) {
#pragma unroll
        for (int j = 0; j < S - 1; ++j) {
            float d = 0.f;
#pragma unroll
            for (int s = 0; s <= j; ++s) d = fmaf(w[s], dp[j - s], d);
            if (a.dfinal && j >= len) d += load_elem<BF16>(a.dfinal, state + j - len);
            store_elem<BF16>(a.dinit, state + j, d);
        }
    }
}

// The gradients of x at t .. t + 7 need dp up to t + 7 + S - 1: the next lane has them.  A piece is taken from its end, so that
// the last lane of a wave finds them in the step before (in the first one, all lanes compute those behind the piece).
template <bool BF16, int S, int R>
__global__ __launch_bounds__(kThreads) void causal_bwd_kernel(CausalArgs a) {
    constexpr int H = S > 1 ? S - 1 : 1;
    const Piece p = piece_of(a);
    const int len = p.there ? seq_length(a.lengths, p.n, a.L) : 0;
    using T = typename RowElem<BF16>::type;
    const T* x = static_cast<const T*>(a.x) + p.n * a.x_sn + p.c * a.x_sc;
    const T* dy = static_cast<const T*>(a.dy) + p.n * a.dy_sn + p.c * a.dy_sc;
    T* dx = static_cast<T*>(a.dx) + (p.n * a.C + p.c) * a.L;
    float w[S];
#pragma unroll
    for (int s = 0; s < S; ++s) w[s] = load_elem<BF16>(a.w, p.c * S + s);
    const float bias = a.bias ? a.bias[p.c] : 0.f;
    const int step = kV << a.lg, begin = p.piece * step * R, end = begin + step * R;
    float behind[H] = {};  // dp of the S - 1 positions behind the wave's step
    if (S > 1 && a.lg == 6 && end < len) {
        float u[2 * H];
#pragma unroll
        for (int i = 0; i < 2 * (S - 1); ++i) u[i] = end - (S - 1) + i < len ? load_elem<BF16>(x, end - (S - 1) + i) : 0.f;
#pragma unroll
        for (int i = 0; i < S - 1; ++i)
            if (end + i < len) behind[i] = load_elem<BF16>(dy, end + i) * (a.silu ? slope_of<S>(u + i, w, bias) : 1.f);
    }
    float sum[S + 1];
#pragma unroll
    for (int s = 0; s <= S; ++s) sum[s] = 0.f;
#pragma unroll 1
    for (int t = begin + (R - 1) * step + p.sub * kV; t >= begin; t -= step) {
        if (wave_all(t > 0 && t + kV <= len)) backward_step<BF16, S, true>(a, p, x, dy, dx, t, len, w, bias, behind, sum);
        else backward_step<BF16, S, false>(a, p, x, dy, dx, t, len, w, bias, behind, sum);
    }
    if (!a.partial) return;
    for (int m = 1; m < (1 << a.lg); m <<= 1) {
#pragma unroll
        for (int s = 0; s <= S; ++s) sum[s] += lane_xor(sum[s], m);
    }
    if (p.there && p.sub == 0) {
        const long per = static_cast<long>(a.N) * a.pieces;
#pragma unroll
        for (int s = 0; s <= S; ++s) a.partial[(p.c * (S + 1) + s) * per + p.n * a.pieces + p.piece] = sum[s];
    }
}

// one wave per sum, in 64 bits: the error of a gradient is that of its partial sums
__global__ __launch_bounds__(kSeqWave) void causal_sums_kernel(const float* partial, float* dw, float* dbias, int S, long per, long first) {
    const long i0 = first + blockIdx.x, c = i0 / (S + 1);
    const int s = static_cast<int>(i0 - c * (S + 1));
    const float* from = partial + i0 * per;
    double sum = 0.0;
#pragma unroll 4
    for (long i = threadIdx.x; i < per; i += kSeqWave) sum += static_cast<double>(from[i]);
#pragma unroll
    for (int m = 1; m < kSeqWave; m <<= 1) sum += lane_xor(sum, m);
    if (threadIdx.x) return;
    if (s < S) dw[c * S + s] = static_cast<float>(sum);
    else if (dbias) dbias[c] = static_cast<float>(sum);
}

struct StepArgs {
    const void* x;
    const void* w;
    const float* bias;
    void* state;  // [N][C][S - 1]
    void* y;
    long rows, x_sn, y_sn, first;
    int C, silu;
};

// One lane per channel: a row of S - 1 elements is read and written back, one place further on.
template <bool BF16, int S>
__global__ __launch_bounds__(kThreads) void causal_step_kernel(StepArgs a) {
    const long row = a.first + static_cast<long>(blockIdx.x) * kThreads + threadIdx.x;
    if (row >= a.rows) return;
    const long n = row / a.C, c = row - n * a.C;
    float v[S], w[S];
#pragma unroll
    for (int s = 0; s < S; ++s) w[s] = load_elem<BF16>(a.w, c * S + s);
#pragma unroll
    for (int s = 0; s < S - 1; ++s) v[s] = load_elem<BF16>(a.state, row * (S - 1) + s);
    v[S - 1] = load_elem<BF16>(a.x, n * a.x_sn + c);
    float p = a.bias ? a.bias[c] : 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) p = fmaf(w[s], v[s], p);
    if (a.silu) p *= sigmoid_of(p);
    store_elem<BF16>(a.y, n * a.y_sn + c, p);
#pragma unroll
    for (int s = 0; s < S - 1; ++s) store_elem<BF16>(a.state, row * (S - 1) + s, v[s + 1]);
}

struct Cut {
    int lg, pieces;
};
// lanes of a piece: as many as a row has steps of kV outputs, a wave at most; R steps each
Cut cut_of(int L, int R) {
    Cut c{};
    while (c.lg < 6 && (static_cast<long>(kV) << c.lg) < L) ++c.lg;
    c.pieces = cdiv(L, (static_cast<long>(kV) << c.lg) * R);
    return c;
}

// Steps of a lane backwards: the more, the less is computed twice behind a piece and added up behind the launch, as long as 4096
// waves are left for the chip (N = 8, C = 128, L = 20000, S = 4 in bfloat16: 45, 28 and 27 us with 1, 4 and 8; N = 12, C = 49,
// L = 4999, S = 3 in FP32: 9.0, 10.2 and 14 us).
int back_steps(long rows, int L) {
    for (int R : {8, 4}) {
        const Cut c = cut_of(L, R);
        if (c.lg == 6 && rows * c.pieces >= 4096) return R;
    }
    return 1;
}

template <bool BF16, int S>
hipError_t launch_taps(bool bwd, CausalArgs& a, int R, hipStream_t st) {
    auto kern = !bwd ? causal_fwd_kernel<BF16, S> : R == 8 ? causal_bwd_kernel<BF16, S, 8> : R == 4 ? causal_bwd_kernel<BF16, S, 4> : causal_bwd_kernel<BF16, S, 1>;
    const long most = kSeqMostThreads >> a.lg;
    for (a.first = 0; a.first < a.units; a.first += most) {
        const long left = a.units - a.first, units = left < most ? left : most;
        const hipError_t e = launch_kernel(kern, dim3(static_cast<unsigned>(cdiv(units << a.lg, kThreads))), dim3(kThreads), 0, st, a);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <bool BF16>
hipError_t launch_type(bool bwd, CausalArgs& a, int S, int R, hipStream_t st) {
    switch (S) {
        case 1: return launch_taps<BF16, 1>(bwd, a, R, st);
        case 2: return launch_taps<BF16, 2>(bwd, a, R, st);
        case 3: return launch_taps<BF16, 3>(bwd, a, R, st);
        case 4: return launch_taps<BF16, 4>(bwd, a, R, st);
        case 5: return launch_taps<BF16, 5>(bwd, a, R, st);
        case 6: return launch_taps<BF16, 6>(bwd, a, R, st);
        case 7: return launch_taps<BF16, 7>(bwd, a, R, st);
        case 8: return launch_taps<BF16, 8>(bwd, a, R, st);
        default: return hipErrorInvalidValue;
    }
}

template <bool BF16>
hipError_t step_type(StepArgs& a, int S, hipStream_t st) {
    void (*kern)(StepArgs) = nullptr;
    switch (S) {
        case 1: kern = causal_step_kernel<BF16, 1>; break;
        case 2: kern = causal_step_kernel<BF16, 2>; break;
        case 3: kern = causal_step_kernel<BF16, 3>; break;
        case 4: kern = causal_step_kernel<BF16, 4>; break;
        case 5: kern = causal_step_kernel<BF16, 5>; break;
        case 6: kern = causal_step_kernel<BF16, 6>; break;
        case 7: kern = causal_step_kernel<BF16, 7>; break;
        case 8: kern = causal_step_kernel<BF16, 8>; break;
        default: return hipErrorInvalidValue;
    }
    for (a.first = 0; a.first < a.rows; a.first += kSeqMostThreads) {
        const long left = a.rows - a.first, rows = left < kSeqMostThreads ? left : kSeqMostThreads;
        const hipError_t e = launch_kernel(kern, dim3(static_cast<unsigned>(cdiv(rows, kThreads))), dim3(kThreads), 0, st, a);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

bool layout_ok(const conv1d_causal_t* p) {
    if (!p || !p->x || !p->w || p->N < 1 || p->C < 1 || p->L < 1 || p->S < 1) return false;
    if (p->dtype != CONV1D_FP32 && p->dtype != CONV1D_BF16) return false;
    const size_t size = p->dtype == CONV1D_BF16 ? 2 : 4;
    if (!seq_aligned(p->x, size) || !seq_aligned(p->w, size) || !seq_aligned(p->init, size) || !seq_aligned(p->bias, 4) ||
        !seq_aligned(p->lengths, 4))
        return false;
    return (p->flags & ~CONV1D_CAUSAL_SILU) == 0;
}

// rows are counted in 31 bits (units of a launch too: a piece has a row's share of at least kV elements)
bool sizes_ok(const conv1d_causal_t* p) {
    return p->S <= kMostTaps && p->L <= 1 << 30 && static_cast<long>(p->N) * p->C <= 0x7fffffffL;
}

CausalArgs args_of(const conv1d_causal_t* p, int R) {
    CausalArgs a{};
    a.x = p->x; a.w = p->w; a.bias = p->bias; a.init = p->init; a.lengths = p->lengths;
    a.N = p->N; a.C = p->C; a.L = p->L; a.silu = (p->flags & CONV1D_CAUSAL_SILU) != 0;
    a.x_sn = p->x_sn; a.x_sc = p->x_sc;
    const Cut cut = cut_of(p->L, R);
    a.lg = cut.lg;
    a.pieces = cut.pieces;
    a.units = static_cast<long>(p->N) * p->C * cut.pieces;
    return a;
}

int status_of(hipError_t e) { return e == hipSuccess ? CONV1D_OK : CONV1D_EHIP; }

}  // namespace
}  // namespace conv1d

using namespace conv1d;

extern "C" {

int conv1d_causal_fwd(const conv1d_causal_t* p, void* y, long y_sn, long y_sc, void* final, void* stream) {
    if (!layout_ok(p) || !y) return CONV1D_EINVAL;
    const size_t size = p->dtype == CONV1D_BF16 ? 2 : 4;
    if (!seq_aligned(y, size) || !seq_aligned(final, size)) return CONV1D_EINVAL;
    if (!sizes_ok(p)) return CONV1D_EUNSUPPORTED;
    CausalArgs a = args_of(p, 1);
    a.y = y; a.y_sn = y_sn; a.y_sc = y_sc; a.final = final;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return status_of(p->dtype == CONV1D_BF16 ? launch_type<true>(false, a, p->S, 1, st) : launch_type<false>(false, a, p->S, 1, st));
}

size_t conv1d_causal_bwd_workspace_bytes(int N, int C, int L, int S) {
    if (N < 1 || C < 1 || L < 1 || S < 1 || S > kMostTaps) return 0;
    const Cut cut = cut_of(L, back_steps(static_cast<long>(N) * C, L));
    return sizeof(float) * static_cast<size_t>(C) * (S + 1) * N * cut.pieces;
}

int conv1d_causal_bwd(const conv1d_causal_t* p, const void* dy, long dy_sn, long dy_sc, const void* dfinal, void* dx, float* dw,
                      float* dbias, void* dinit, void* workspace, size_t workspace_bytes, void* stream) {
    if (!layout_ok(p) || !dy || !dx || (dbias && !dw)) return CONV1D_EINVAL;
    const size_t size = p->dtype == CONV1D_BF16 ? 2 : 4;
    if (!seq_aligned(dy, size) || !seq_aligned(dfinal, size) || !seq_aligned(dx, size) || !seq_aligned(dinit, size) || !seq_aligned(dw, 4) ||
        !seq_aligned(dbias, 4) || !seq_aligned(workspace, 4))
        return CONV1D_EINVAL;
    if (!sizes_ok(p)) return CONV1D_EUNSUPPORTED;
    if (dw && (!workspace || workspace_bytes < conv1d_causal_bwd_workspace_bytes(p->N, p->C, p->L, p->S))) return CONV1D_EWORKSPACE;
    const int R = back_steps(static_cast<long>(p->N) * p->C, p->L);
    CausalArgs a = args_of(p, R);
    a.dy = dy; a.dy_sn = dy_sn; a.dy_sc = dy_sc; a.dfinal = dfinal; a.dx = dx; a.dinit = dinit;
    a.partial = dw ? static_cast<float*>(workspace) : nullptr;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const hipError_t e = p->dtype == CONV1D_BF16 ? launch_type<true>(true, a, p->S, R, st) : launch_type<false>(true, a, p->S, R, st);
    if (e != hipSuccess || !dw) return status_of(e);
    const long sums = static_cast<long>(p->C) * (p->S + 1), most = kSeqMostThreads / kSeqWave;
    for (long first = 0; first < sums; first += most) {
        const hipError_t e2 = launch_kernel(causal_sums_kernel, dim3(static_cast<unsigned>(sums - first < most ? sums - first : most)), dim3(kSeqWave), 0, st,
                                            a.partial, dw, dbias, p->S, static_cast<long>(p->N) * a.pieces, first);
        if (e2 != hipSuccess) return status_of(e2);
    }
    return CONV1D_OK;
}

int conv1d_causal_step(const conv1d_causal_t* p, void* state, void* y, long y_sn, void* stream) {
    if (!layout_ok(p) || !y || p->L != 1 || p->init || p->lengths || (p->S > 1 && !state)) return CONV1D_EINVAL;
    const size_t size = p->dtype == CONV1D_BF16 ? 2 : 4;
    if (!seq_aligned(y, size) || !seq_aligned(state, size)) return CONV1D_EINVAL;
    if (!sizes_ok(p)) return CONV1D_EUNSUPPORTED;
    StepArgs a{};
    a.x = p->x; a.w = p->w; a.bias = p->bias; a.state = state; a.y = y;
    a.rows = static_cast<long>(p->N) * p->C; a.x_sn = p->x_sn; a.y_sn = y_sn;
    a.C = p->C; a.silu = (p->flags & CONV1D_CAUSAL_SILU) != 0;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return status_of(p->dtype == CONV1D_BF16 ? step_type<true>(a, p->S, st) : step_type<false>(a, p->S, st));
}

}  // extern "C"
