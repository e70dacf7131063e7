// Selective scan, backward.  With dy = dout z sigmoid(z) and g the gradient of the state,
//   g[t] = C[t] dy[t] + a[t+1] g[t+1],   c[t] = a[t] g[t] (what a step sends into the one before it),   q[t] = c[t] h[t-1]
//   dC = sum_d dy h,  dB = sum_d g e x,  dx = e sum_s g B + skip dy,  de = x sum_s g B + sum_s A q,  dA = sum_t e q
//   ddt = de sigmoid(dt + dt_bias) behind a softplus, dz = dout y (silu)'(z), dskip = sum dy x, ddt_bias = sum ddt.
// The forward pass has kept the state before every kSub steps: a workgroup goes through its segment from the end, computes
// kSub states and decays again into registers and walks them backwards.  Where a sequence is cut, the adjoint is joined as
// the forward state is: a launch finds what each segment sends into the one before it, another joins them.
// dB and dC are summed over the channels of a wave by lane exchanges, of a workgroup through LDS, of the workgroups of a
// group by a launch of its own, always in the same order.
// Bound by instruction issue, about 90 slots a step of a wave (16 channels of 16 states), 60 of them the recurrence, 16 the sums over
// channels, 14 what is done per element.  N = 8, D = 512, L = 8192, S = 16 in bfloat16: 118 us the adjoint, 6 its join, 434 this
// pass, 22 the last sums.
#include "conv1d_scan.h"

namespace conv1d {
namespace {

// What was read from LDS before is read again: kept, it would take the registers that a third and fourth wave need.
__device__ __forceinline__ void reload_lds() { asm volatile("" ::: "memory"); }


template <int K>
__device__ __forceinline__ void load_states(const float* from, float (&v)[K]) {
    const States<K> s = states_at<K>(from);
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = s[k];
}

// Sums over the channels of a wave, of one value per lane for each of K states and 4 steps, value K step + state.  Every level
// adds a pair of values and leaves each lane one of the two; one that finds a single value adds it in all lanes.  Within a row
// of 16 lanes an addition reads its neighbour's bank and writes some banks only: two instructions a pair, so those levels come
// first, where the values are most.  Rows and halves of the wave take an exchange, which costs twice an addition, and an addition.
// (Halves and rows first, banks by selections: 90 issue slots for 4 steps of 4 states, this way 66; the kernel took 5 % longer.)
// The kSums<K, P> values left are those of sum_value.
template <int K, int P>
constexpr int kSums = P <= 4 ? 1 : P == 8 ? K / 2 : K;
template <int K, int P>
__device__ __forceinline__ int sum_value(int lane, int j) {
    const int half = lane >> 5, row = (lane >> 4) & 1, bank = (lane >> 2) & 3, side = (lane >> 3) & 1;
    if (P <= 4) return bank + (K > 1 ? 4 * half : 0) + (K > 2 ? 8 * row : 0);
    return P == 8 ? side + 2 * half + 4 * row + 8 * j : half + 2 * row + 4 * j;
}
#ifdef HOSTMODEL
template <int P>
inline void four_sums(float* v, float* w, float& sv, float& sw) {
    sv = v[0];
    sw = w[0];
}
template <int K, int P>
inline void step_sums(const float (&q)[K], float (&out)[kSums<K, P>]) {
    for (float& o : out) o = q[0];
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
// Four values each of v and w: over the four banks of a row (P <= 4; bank b is left with value b: row_ror:4 adds to every bank
// the one before it, row_ror:8 the two before those), over its two sides (P = 8) and the halves of the wave, over rows and
// halves (P = 16).  A vector instruction's result may be read from another lane two wait states later: the pairs of v and w
// alternate, and the ends, whose neighbours the compiler places, wait.
template <int P>
__device__ __forceinline__ void four_sums(float* v, float* w, float& sv, float& sw) {
    if constexpr (P <= 4) {
        float a = v[0], b = v[2], c = w[0], d = w[2];
        asm("s_nop 1\n\t"
            "v_add_f32_dpp %0, %0, %0 row_ror:4 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %2, %2, %2 row_ror:4 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %1, %1, %1 row_ror:4 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %3, %3, %3 row_ror:4 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %0, %4, %4 row_ror:4 row_mask:0xf bank_mask:0xa\n\t"
            "v_add_f32_dpp %2, %6, %6 row_ror:4 row_mask:0xf bank_mask:0xa\n\t"
            "v_add_f32_dpp %1, %5, %5 row_ror:4 row_mask:0xf bank_mask:0xa\n\t"
            "v_add_f32_dpp %3, %7, %7 row_ror:4 row_mask:0xf bank_mask:0xa\n\t"
            "v_add_f32_dpp %0, %0, %0 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %2, %2, %2 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %0, %1, %1 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
            "v_add_f32_dpp %2, %3, %3 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
            "s_nop 1"
            : "+&v"(a), "+&v"(b), "+&v"(c), "+&v"(d)
            : "v"(v[1]), "v"(v[3]), "v"(w[1]), "v"(w[3]));
        sv = a;
        sw = c;
    } else if constexpr (P == 8) {
        float a = v[0], b = v[2], c = w[0], d = w[2];
        asm("s_nop 1\n\t"
            "v_add_f32_dpp %0, %0, %0 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %2, %2, %2 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %1, %1, %1 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %3, %3, %3 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %0, %4, %4 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
            "v_add_f32_dpp %2, %6, %6 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
            "v_add_f32_dpp %1, %5, %5 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
            "v_add_f32_dpp %3, %7, %7 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
            "s_nop 1"
            : "+&v"(a), "+&v"(b), "+&v"(c), "+&v"(d)
            : "v"(v[1]), "v"(v[3]), "v"(w[1]), "v"(w[3]));
        sv = swap32_add(a, b);
        sw = swap32_add(c, d);
    } else {
        sv = swap16_add(swap32_add(v[0], v[1]), swap32_add(v[2], v[3]));
        sw = swap16_add(swap32_add(w[0], w[1]), swap32_add(w[2], w[3]));
    }
}
// the K of those that 4 steps have, over the rest of the wave
template <int K, int P>
__device__ __forceinline__ void step_sums(const float (&q)[K], float (&out)[kSums<K, P>]) {
    if constexpr (P <= 4) {
        if constexpr (K == 4) {
            out[0] = swap16_add(swap32_add(q[0], q[1]), swap32_add(q[2], q[3]));
        } else {
            const float v = swap32_add(q[0], q[K - 1]);
            out[0] = swap16_add(v, v);
        }
    } else if constexpr (P == 8) {
#pragma unroll
        for (int i = 0; i < K / 2; ++i) out[i] = swap16_add(q[2 * i], q[2 * i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < K; ++i) out[i] = q[i];
    }
}
#endif

// The lane's row: where it begins and what its elements share.
template <bool BF16, int P, int T>
struct BackRow {
    using R = ScanRows<P, T>;
    static constexpr int V = R::V;
    using E = typename RowElem<BF16>::type;
    const E *x, *dt, *dout, *z;
    float bias;
    bool real;
    long d;
    int c, at;  // first step of the lane within the tile, its place in LDS

    __device__ __forceinline__ BackRow(const ScanArgs& a, const ScanPlace& p, int base, int lane) {
        const int row = lane / R::LPR;
        c = V * (lane % R::LPR);
        at = row * R::RS + c;
        real = base + row < a.Dg;
        d = static_cast<long>(p.g) * a.Dg + (real ? base + row : 0);
        x = scan_row<BF16>(a.x, a.x_sn, a.x_sd, p.n, d);
        dt = scan_row<BF16>(a.dt, a.dt_sn, a.dt_sd, p.n, d);
        dout = scan_row<BF16>(a.dout, a.dout_sn, a.dout_sd, p.n, d);
        z = a.z ? scan_row<BF16>(a.z, a.z_sn, a.z_sd, p.n, d) : nullptr;
        bias = a.dt_bias ? a.dt_bias[d] : 0.f;
    }
    // e, dy and (WITH_X) x of the tile at t0 into LDS.  INSIDE: it lies within the sequence.  A lane without a channel (there are
    // some if not `full`) goes along with the group's first, x and dy of 0: it adds nothing to the sums over channels.
    template <bool INSIDE, bool WITH_X>
    __device__ __forceinline__ void stage(const ScanArgs& a, int t0, int len, bool full, float* sE, float* sX, float* sY) const {
        float v[V], g[V], u[V], w[V];
        scan_load<BF16, INSIDE>(dt, t0 + c, len, a.L, v);
        scan_load<BF16, INSIDE>(dout, t0 + c, len, a.L, g);
        if (z) scan_load<BF16, INSIDE>(z, t0 + c, len, a.L, w);
        if (WITH_X) scan_load<BF16, INSIDE>(x, t0 + c, len, a.L, u);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += bias;
        if (a.softplus) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = softplus_of(v[i]);
        }
        if (!INSIDE) {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = t0 + c + i < len ? v[i] : 0.f;
        }
        lds_put(sE + at, v);
        if (z) {
#pragma unroll
            for (int i = 0; i < V; ++i) g[i] *= w[i] * sigmoid_of(w[i]);
        }
        if (!full) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                g[i] = real ? g[i] : 0.f;
                if (WITH_X) u[i] = real ? u[i] : 0.f;
            }
        }
        lds_put(sY + at, g);
        if (WITH_X) lds_put(sX + at, u);
    }
    // the gradients of x, dt and z from what the walk back left in LDS
    template <bool INSIDE>
    __device__ __forceinline__ void finish(const ScanArgs& a, const ScanPlace& p, int t0, int len, const float* sE, const float* sX,
                                           const float* sY, float& dskip, float& dbias) const {
        if (!real || t0 + c >= a.L) return;
        const long o = (p.n * a.D + d) * a.L;
        const int end = INSIDE ? t0 + c + V : a.L;
        const float skip = a.skip ? a.skip[d] : 0.f;
        float u[V], v[V], g[V], w[V];
        scan_load<BF16, INSIDE>(x, t0 + c, len, a.L, u);
        scan_load<BF16, INSIDE>(dout, t0 + c, len, a.L, g);
        if (z) scan_load<BF16, INSIDE>(z, t0 + c, len, a.L, w);
        if (a.softplus) scan_load<BF16, INSIDE>(dt, t0 + c, len, a.L, v);
        if (z) {
            float y[V];
            lds_get(sY + at, y);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float sig = sigmoid_of(w[i]), zs = w[i] * sig;
                y[i] = g[i] * fmaf(skip, u[i], y[i]) * fmaf(zs, 1.f - sig, sig);
                g[i] *= zs;
                if (!INSIDE) y[i] = t0 + c + i < len ? y[i] : 0.f;
            }
            scan_store<BF16>(static_cast<E*>(a.dz) + o, t0 + c, end, y);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) dskip = fmaf(g[i], u[i], dskip);
        lds_get(sE + at, u);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            g[i] = fmaf(skip, g[i], u[i]);
            if (!INSIDE) g[i] = t0 + c + i < len ? g[i] : 0.f;
        }
        scan_store<BF16>(static_cast<E*>(a.dx) + o, t0 + c, end, g);
        lds_get(sX + at, u);
        if (a.softplus) {
#pragma unroll
            for (int i = 0; i < V; ++i) u[i] *= sigmoid_of(v[i] + bias);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (!INSIDE) u[i] = t0 + c + i < len ? u[i] : 0.f;
            dbias += u[i];
        }
        scan_store<BF16>(static_cast<E*>(a.ddt) + o, t0 + c, end, u);
    }
};

// what a segment sends into the one before it, from nothing sent into itself, and the sum of its steps
template <bool BF16, int K, int P>
__global__ __launch_bounds__(kScanWaves* kSeqWave, 4) void scan_adjoint_kernel(ScanArgs a) {
    constexpr int SP = K * P, T = scan_tile(P);
    using R = ScanRows<P, T>;
    __shared__ __align__(16) float sE[kScanWaves][R::CW * R::RS], sY[kScanWaves][R::CW * R::RS];  // e and dy
    __shared__ __align__(16) float sC[T * SP];
    const ScanPlace at = scan_place(a);
    if (at.seg == 0) return;
    const int lane = threadIdx.x & (kSeqWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int p = lane & (P - 1), cl = lane / P;
    const int len = seq_length(a.lengths, at.n, a.L);
    const int base = (at.cb * waves + wave) * R::CW;
    const bool there = base + cl < a.Dg;
    const long d = static_cast<long>(at.g) * a.Dg + (there ? base + cl : 0);
    const BackRow<BF16, P, T> line(a, at, base, lane);
    using E = typename RowElem<BF16>::type;
    ScanStates<BF16, SP, T, false> states{static_cast<const E*>(a.C) + at.n * a.c_sn + at.g * a.c_sg, nullptr, a.c_ss, 0, a.S, a.L, {}};
    float rate[K], carry[K], sum = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        rate[k] = scan_rate(a.A, a.S, d, K * p + k, there);
        carry[k] = 0.f;
    }
    const int t_begin = at.seg * a.seg_len, t_end = min(a.L, t_begin + a.seg_len);
    const int t_last = t_begin + (t_end - 1 - t_begin) / T * T;
    for (int t0 = t_last; t0 >= t_begin; t0 -= T) {
        states.begin(t0, len);
        if (t0 + T <= len) line.template stage<true, false>(a, t0, len, true, sE[wave], nullptr, sY[wave]);
        else line.template stage<false, false>(a, t0, len, true, sE[wave], nullptr, sY[wave]);
        states.finish(t0, len, sC, nullptr);
        if (t0 == t_last) make_rates(rate);
        __syncthreads();
        const float *e_row = sE[wave] + cl * R::RS, *dy_row = sY[wave] + cl * R::RS;
#pragma unroll 1
        for (int t = T - kSub; t >= 0; t -= kSub) {
            float part = 0.f;
#pragma unroll
            for (int j = kSub - 4; j >= 0; j -= 4) {
                __builtin_amdgcn_sched_barrier(0);
                const scan_f32x4 e = *reinterpret_cast<const scan_f32x4*>(e_row + t + j), dy = *reinterpret_cast<const scan_f32x4*>(dy_row + t + j);
#pragma unroll
                for (int i = 3; i >= 0; --i) {
                    const States<K> o = states_at<K>(sC + (t + j + i) * SP + K * p);
                    part += e[i];
#pragma unroll
                    for (int k = 0; k < K; ++k) carry[k] = exp2_hw(e[i] * rate[k]) * fmaf(o[k], dy[i], carry[k]);
                }
            }
            sum += part;
        }
        __syncthreads();
    }
    if (!there) return;
    const long i = (at.n * a.D + d) * a.nseg + at.seg;
    put_states<K>(a.carries + i * SP + K * p, carry);
    if (p == 0) a.sums[i] = sum;
}

template <bool BF16, int K, int P>
__global__ __launch_bounds__(kScanWaves* kSeqWave, 3) void scan_bwd_kernel(ScanArgs a) {
    constexpr int SP = K * P, T = scan_tile_back(P);
    using R = ScanRows<P, T>;
    // e, x and dy of a step; the walk back leaves sum_s e g B, de and sum_s C h in their places
    __shared__ __align__(16) float sE[kScanWaves][R::CW * R::RS], sX[kScanWaves][R::CW * R::RS], sY[kScanWaves][R::CW * R::RS];
    __shared__ __align__(16) float sB[T * SP], sC[T * SP];
    __shared__ __align__(16) float red[kScanWaves][2][SP * R::RS];  // dB and dC of the wave's channels, [state][step]
    const ScanPlace at = scan_place(a);
    const int lane = threadIdx.x & (kSeqWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int p = lane & (P - 1), cl = lane / P;
    const int len = seq_length(a.lengths, at.n, a.L);
    const int base = (at.cb * waves + wave) * R::CW;
    const bool there = base + cl < a.Dg, full = base + R::CW <= a.Dg;
    const long d = static_cast<long>(at.g) * a.Dg + (there ? base + cl : 0);
    const BackRow<BF16, P, T> line(a, at, base, lane);
    using E = typename RowElem<BF16>::type;
    ScanStates<BF16, SP, T, true> states{static_cast<const E*>(a.B) + at.n * a.b_sn + at.g * a.b_sg,
                                         static_cast<const E*>(a.C) + at.n * a.c_sn + at.g * a.c_sg, a.b_ss, a.c_ss, a.S, a.L, {}};
    float rate[K], carry[K], dA[K], dskip = 0.f, dbias = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int s = K * p + k;
        rate[k] = rate_of(scan_rate(a.A, a.S, d, s, there));
        dA[k] = 0.f;
        carry[k] = 0.f;
        if (a.nseg > 1) carry[k] = there ? a.carries[((at.n * a.D + d) * a.nseg + at.seg) * SP + s] : 0.f;
        else if (a.dfinal && there && s < a.S) carry[k] = a.dfinal[(at.n * a.D + d) * a.S + s];
    }
    const int t_begin = at.seg * a.seg_len, t_end = min(a.L, t_begin + a.seg_len);
    // the states that the forward pass kept, from the segment's last; each is loaded while the steps behind it are walked
    const float* kept_at = a.saved + ((at.n * a.chunks + (t_end - 1) / kSub) * a.D + d) * SP + K * p;
    float next[K] = {};
    if (there) load_states<K>(kept_at, next);
    for (int t0 = t_begin + (t_end - 1 - t_begin) / T * T; t0 >= t_begin; t0 -= T) {
        const bool inside = t0 + T <= len;
        states.begin(t0, len);
        if (inside) line.template stage<true, true>(a, t0, len, full, sE[wave], sX[wave], sY[wave]);
        else line.template stage<false, true>(a, t0, len, full, sE[wave], sX[wave], sY[wave]);
        states.finish(t0, len, sB, sC);
        __syncthreads();
        float dA_tile[K] = {};
        float *e_row = sE[wave] + cl * R::RS, *x_row = sX[wave] + cl * R::RS, *dy_row = sY[wave] + cl * R::RS;
#pragma unroll 1
        for (int t = T - kSub; t >= 0; t -= kSub) {
            if (t0 + t >= a.L) continue;
            float first[K], h[kSub][K], decay[kSub][K];
#pragma unroll
            for (int k = 0; k < K; ++k) first[k] = next[k];
#pragma unroll
            for (int j = 0; j < kSub; j += 4) {
                __builtin_amdgcn_sched_barrier(0);
                const scan_f32x4 e = *reinterpret_cast<const scan_f32x4*>(e_row + t + j), x = *reinterpret_cast<const scan_f32x4*>(x_row + t + j);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const States<K> b = states_at<K>(sB + (t + j + i) * SP + K * p);
                    const float ex = e[i] * x[i];
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        decay[j + i][k] = exp2_hw(e[i] * rate[k]);
                        h[j + i][k] = fmaf(decay[j + i][k], j + i ? h[j + i - (j + i ? 1 : 0)][k] : first[k], ex * b[k]);
                    }
                }
            }
#pragma unroll
            for (int j = kSub - 4; j >= 0; j -= 4) {
                reload_lds();
                if (j == 0 && there && t0 + t > t_begin) {
                    kept_at -= static_cast<long>(a.D) * SP;
                    load_states<K>(kept_at, next);
                }
                __builtin_amdgcn_sched_barrier(0);
                const scan_f32x4 e = *reinterpret_cast<const scan_f32x4*>(e_row + t + j), x = *reinterpret_cast<const scan_f32x4*>(x_row + t + j),
                                 dy = *reinterpret_cast<const scan_f32x4*>(dy_row + t + j);
                scan_f32x4 out_x, out_e, out_y;
                float vB[4 * K], vC[4 * K], qB[K], qC[K];
#pragma unroll
                for (int i = 3; i >= 0; --i) {
                    const States<K> b = states_at<K>(sB + (t + j + i) * SP + K * p);
                    const States<K> o = states_at<K>(sC + (t + j + i) * SP + K * p);
                    const float ex = e[i] * x[i];
                    float gb = 0.f, qa = 0.f, y = 0.f;
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        const float g = fmaf(o[k], dy[i], carry[k]);
                        y = k ? fmaf(o[k], h[j + i][k], y) : o[k] * h[j + i][k];
                        vC[K * i + k] = dy[i] * h[j + i][k];
                        vB[K * i + k] = g * ex;
                        gb = k ? fmaf(g, b[k], gb) : g * b[k];
                        carry[k] = g * decay[j + i][k];
                        const float kept = carry[k] * (j + i ? h[j + i - (j + i ? 1 : 0)][k] : first[k]);
                        qa = k ? fmaf(kept, rate[k], qa) : kept * rate[k];
                        dA_tile[k] = fmaf(kept, e[i], dA_tile[k]);
                    }
                    gb = channel_sum<P>(gb);
                    qa = channel_sum<P>(qa);
                    y = channel_sum<P>(y);
                    keep_here(gb);
                    keep_here(qa);
                    keep_here(y);
                    out_y[i] = y;
                    out_x[i] = gb * e[i];
                    out_e[i] = fmaf(gb, x[i], qa * (1.f / kLog2e));
                    if (K * i % 4 == 0) four_sums<P>(vB + K * i, vC + K * i, qB[K * i / 4], qC[K * i / 4]);
                }
                float out_B[kSums<K, P>], out_C[kSums<K, P>];
                step_sums<K, P>(qB, out_B);
                step_sums<K, P>(qC, out_C);
#pragma unroll
                for (int i = 0; i < kSums<K, P>; ++i) {
                    const int value = sum_value<K, P>(lane, i), to = (K * p + value % K) * R::RS + t + j + value / K;
                    red[wave][0][to] = out_B[i];
                    red[wave][1][to] = out_C[i];
                }
                if (p == 0) {
                    *reinterpret_cast<scan_f32x4*>(e_row + t + j) = out_x;
                    *reinterpret_cast<scan_f32x4*>(x_row + t + j) = out_e;
                    *reinterpret_cast<scan_f32x4*>(dy_row + t + j) = out_y;
                }
            }
        }
#pragma unroll
        for (int k = 0; k < K; ++k) dA[k] += dA_tile[k];
        __syncthreads();
        // dB and dC over the waves of the workgroup, 4 steps of a state each
        for (int i = threadIdx.x; i < 2 * SP * (T / 4); i += blockDim.x) {
            const int step = 4 * (i % (T / 4)), s = i / (T / 4) % SP, which = i / (T / 4) / SP, t = t0 + step;
            if (s >= a.S || t >= a.L) continue;
            scan_f32x4 v = *reinterpret_cast<const scan_f32x4*>(&red[0][which][s * R::RS + step]);
            for (int w = 1; w < waves; ++w) v += *reinterpret_cast<const scan_f32x4*>(&red[w][which][s * R::RS + step]);
            if (!inside) {  // 0 behind the end also where 0 has met an infinite state or gradient
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = t + e < len ? v[e] : 0.f;
            }
            const long o = ((at.n * a.G + at.g) * a.S + s) * a.L + t;
            if (a.blocks_d > 1) {
                float* to = a.part_bc + (static_cast<long>(which) * a.blocks_d + at.cb) * a.N * a.G * a.S * a.L + o;
                if (t + 4 <= a.L) {
                    *reinterpret_cast<seq_f32x4*>(to) = v;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (t + e < a.L) to[e] = v[e];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (t + e < a.L) store_elem<BF16>(which ? a.dC : a.dB, o + e, v[e]);
            }
        }
        if (inside) line.template finish<true>(a, at, t0, len, sE[wave], sX[wave], sY[wave], dskip, dbias);
        else line.template finish<false>(a, at, t0, len, sE[wave], sX[wave], sY[wave], dskip, dbias);
        // (the next tile's barrier stands between these reads of `red` and its next values)
    }
    float* part = a.part_p + (at.n * a.nseg + at.seg) * (static_cast<long>(a.D) * (SP + 2));
#pragma unroll
    for (int m = 1; m < R::LPR; m <<= 1) {
        dskip += lane_xor(dskip, m);
        dbias += lane_xor(dbias, m);
    }
    if (lane % R::LPR == 0 && line.real) {
        part[static_cast<long>(a.D) * SP + line.d] = dskip;
        part[static_cast<long>(a.D) * (SP + 1) + line.d] = dbias;
    }
    if (!there) return;
#pragma unroll
    for (int k = 0; k < K; ++k) part[d * SP + K * p + k] = dA[k];
    if (a.dinit && at.seg == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (K * p + k < a.S) a.dinit[(at.n * a.D + d) * a.S + K * p + k] = carry[k];
    }
}

// What is left of sums: the first workgroups add the columns of part_p over its rows in 64 bits (the error of a gradient is that
// of its partial sums), kCols columns and kShares shares of the rows each; the others add dB and dC over the workgroups along
// the channels, 8 elements a lane.
constexpr int kCols = 16, kShares = 64;
struct SumArgs {
    const float *part_p, *part_bc;
    float *dA, *dskip, *dbias;
    void *dB, *dC;
    long rows, n;          // rows of part_p; elements of dB
    int D, S, SP, blocks_d, param_blocks;
    long first;            // first workgroup of the launch
};
template <bool BF16>
__global__ __launch_bounds__(kCols* kShares) void scan_sums_kernel(SumArgs a) {
    __shared__ double sums[kShares][kCols];
    const long block = a.first + blockIdx.x;
    if (block >= a.param_blocks) {
        const long groups = (a.n + 7) / 8;
        long i = (block - a.param_blocks) * (kCols * kShares) + threadIdx.x;
        if (i >= 2 * groups) return;
        const int which = i >= groups;
        i = 8 * (i - which * groups);
        float v[8] = {}, u[8];
        for (int b = 0; b < a.blocks_d; ++b) {
            row_load8<false>(a.part_bc + (static_cast<long>(which) * a.blocks_d + b) * a.n, i, a.n, u);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += u[e];
        }
        row_store8<BF16>(which ? a.dC : a.dB, i, a.n, v);
        return;
    }
    const int c = threadIdx.x % kCols, share = threadIdx.x / kCols;
    const long cols = static_cast<long>(a.D) * (a.SP + 2), col = block * kCols + c;
    double sum = 0.0;
    if (col < cols) {
#pragma unroll 8
        for (long r = share; r < a.rows; r += kShares) sum += static_cast<double>(a.part_p[r * cols + col]);
    }
    sums[share][c] = sum;
    __syncthreads();
    if (share || col >= cols) return;
#pragma unroll 8
    for (int i = 1; i < kShares; ++i) sum += sums[i][c];
    const long d = col / a.SP;
    const int s = static_cast<int>(col - d * a.SP);
    if (d < a.D) {
        if (s < a.S) a.dA[d * a.S + s] = static_cast<float>(sum);
    } else {
        const long j = col - static_cast<long>(a.D) * a.SP;
        float* to = j < a.D ? a.dskip : a.dbias;
        if (to) to[j < a.D ? j : j - a.D] = static_cast<float>(sum);
    }
}

template <bool BF16, int K, int P>
hipError_t bwd_launch(ScanArgs a, const ScanPlan& p, float* dA, float* dskip, float* dbias, hipStream_t st) {
    const dim3 block(static_cast<unsigned>(p.waves * kSeqWave));
    const long most = kSeqMostThreads / block.x, blocks = scan_blocks(a);
    for (int stage = p.nseg > 1 ? 0 : 2; stage < 3; ++stage) {
        if (stage == 1) {
            const hipError_t e = scan_join_launch<true>(a.carries, a.sums, a.dfinal, a.A, a.N, a.D, a.S, K * P, a.nseg, st);
            if (e != hipSuccess) return e;
            continue;
        }
        for (long first = 0; first < blocks; first += most) {
            a.first = static_cast<int>(first);
            const long left = blocks - first;
            const dim3 grid(static_cast<unsigned>(left < most ? left : most));
            const hipError_t e = launch_kernel(stage == 0 ? scan_adjoint_kernel<BF16, K, P> : scan_bwd_kernel<BF16, K, P>, grid, block, 0, st, a);
            if (e != hipSuccess) return e;
        }
    }
    SumArgs u{};
    u.part_p = a.part_p; u.part_bc = a.part_bc;
    u.dA = dA; u.dskip = dskip; u.dbias = dbias; u.dB = a.dB; u.dC = a.dC;
    u.rows = static_cast<long>(a.N) * a.nseg;
    u.n = static_cast<long>(a.N) * a.G * a.S * a.L;
    u.D = a.D; u.S = a.S; u.SP = K * P; u.blocks_d = p.blocks_d;
    u.param_blocks = cdiv(static_cast<long>(a.D) * (u.SP + 2), kCols);
    const long sum_blocks = u.param_blocks + (p.blocks_d > 1 ? (2 * ((u.n + 7) / 8) + kCols * kShares - 1) / (kCols * kShares) : 0);
    constexpr long most_sums = kSeqMostThreads / (kCols * kShares);
    for (u.first = 0; u.first < sum_blocks; u.first += most_sums) {
        const long left = sum_blocks - u.first;
        const hipError_t e = launch_kernel(scan_sums_kernel<BF16>, dim3(static_cast<unsigned>(left < most_sums ? left : most_sums)), dim3(kCols * kShares), 0, st, u);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <bool BF16>
hipError_t bwd_type(const ScanArgs& a, const ScanPlan& p, float* dA, float* dskip, float* dbias, hipStream_t st) {
    switch (p.K * p.P) {
        case 4: return bwd_launch<BF16, 1, 4>(a, p, dA, dskip, dbias, st);
        case 8: return bwd_launch<BF16, 2, 4>(a, p, dA, dskip, dbias, st);
        case 16: return bwd_launch<BF16, 4, 4>(a, p, dA, dskip, dbias, st);
        case 32: return bwd_launch<BF16, 4, 8>(a, p, dA, dskip, dbias, st);
        default: return bwd_launch<BF16, 4, 16>(a, p, dA, dskip, dbias, st);
    }
}

}  // namespace

hipError_t scan_bwd_launch(const ScanArgs& a, const ScanPlan& p, int bf16, float* dA, float* dskip, float* dbias, hipStream_t st) {
    return bf16 ? bwd_type<true>(a, p, dA, dskip, dbias, st) : bwd_type<false>(a, p, dA, dskip, dbias, st);
}

}  // namespace conv1d
