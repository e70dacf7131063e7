// Group norm with an activation behind it, for positions or channels contiguous, forward and backward.
//   mean, var: of a group's C / G channels over the positions of its sequence (m values);  rstd = 1 / sqrt(var + eps)
//   h = (x - mean) rstd,  p = h weight[c] + bias[c],  y = p, max(p, 0) or p sigmoid(p)
//   dp = dy act'(p),  dbias = sum dp,  dweight = sum dp h,  dx = rstd (dp weight - (sum dp weight) / m - h (sum dp weight h) / m)
// Bound by memory.  Groups that fit in the registers of one workgroup are read once; larger ones are read twice, cut into enough
// pieces to fill the chip: one launch adds up each piece, the next joins a group's pieces (every workgroup for itself, in one order)
// and writes.  Values are summed as differences from the group's first one, in 64 bits, so that neither a mean far from 0 nor a
// long group costs digits; mean and rstd are kept in 64 bits, and (x - mean) is taken with the mean as two floats.
#include "conv1d_blocks.h"

namespace conv1d {
namespace {

constexpr int kThreads = 256;
enum { kNone = 0, kRelu = 1, kSilu = 2 };

struct NormArgs {
    const void *x, *dy;
    void *y, *dx;
    const float *weight, *bias;
    const int* lengths;
    double* stats;          // [N][G][2]: mean, rstd
    double* part;           // sums of pieces
    float *dweight, *dbias;
    double eps;
    long x_sn, x_sc, x_sl, y_sn, y_sc, y_sl, dy_sn, dy_sc, dy_sl, dx_sn, dx_sc, dx_sl;
    int N, C, L, G, per;    // per: channels of a group
    int vecs, items;        // vectors of 8 of a row, of a group
    int pieces, piece;      // of a group, and its vectors
    int rows_pieces, rows_piece, lanes;  // backward: pieces of a row, their vectors, lanes that a piece has
    int act, first;
    Div31 by_vecs, by_pieces, by_G, by_C, by_rows_pieces;
};

// a mean as two floats
struct Mean {
    float hi, lo, rstd;
};
__device__ __forceinline__ Mean mean_of(double mean, double rstd) {
    const float hi = static_cast<float>(mean);
    return Mean{hi, static_cast<float>(mean - static_cast<double>(hi)), static_cast<float>(rstd)};
}
// s and q: sums of x - shift and of their squares over m values
__device__ __forceinline__ void stats_of(double s, double q, double m, double shift, double eps, double& mean, double& rstd) {
    const double off = m > 0 ? s / m : 0.0, var = m > 0 ? q / m - off * off : 0.0;
    mean = m > 0 ? shift + off : 0.0;
    rstd = 1.0 / sqrt((var < 0.0 ? 0.0 : var) + eps);  // (a NaN stays one)
}

template <int ACT>
__device__ __forceinline__ float act_of(float p) {
    if (ACT == kRelu) return p > 0.f ? p : (p <= 0.f ? 0.f : p);  // (a NaN stays one)
    if (ACT == kSilu) return p * sigmoid_of(p);
    return p;
}
// dp of dy
template <int ACT>
__device__ __forceinline__ float back_of(float dy, float p) {
    if (ACT == kRelu) return p > 0.f ? dy : (p <= 0.f ? 0.f : p);
    if (ACT == kSilu) {
        const float s = sigmoid_of(p);
        return dy * (s * fmaf(p, 1.f - s, 1.f));
    }
    return dy;
}

// x -> h and p for one channel: h = (x - hi) rstd - lo rstd, p = h w + b
struct Channel {
    float hi, rstd, h0, w, b;
};
__device__ __forceinline__ Channel channel_of(const Mean& m, const float* weight, const float* bias, int c) {
    return Channel{m.hi, m.rstd, -m.lo * m.rstd, weight ? weight[c] : 1.f, bias ? bias[c] : 0.f};
}
__device__ __forceinline__ float h_of(float x, const Channel& k) { return fmaf(x - k.hi, k.rstd, k.h0); }

// The side of 0 that p lies on decides over its gradient: next to 0 it is found in 64 bits.  p is off by a few units of 2^-24 of the
// three numbers that it is added up from, so that the sign of a p of more than 2^-20 of them is right.
__device__ __forceinline__ float relu_side(float p, float x, const Channel& k, double mean, double rstd) {
    if (fabsf(p) <= 9.5367431640625e-07f * (fabsf(k.w) * (fabsf((x - k.hi) * k.rstd) + fabsf(k.h0)) + fabsf(k.b)))
        p = static_cast<float>((static_cast<double>(x) - mean) * rstd * static_cast<double>(k.w) + static_cast<double>(k.b));
    return p;
}

// ---- positions contiguous -------------------------------------------------------------------------------------------------
template <bool BF16>
__device__ __forceinline__ const void* row_at(const void* base, long n, long sn, int c, long sc) {
    return static_cast<const typename RowElem<BF16>::type*>(base) + n * sn + c * sc;
}
template <bool BF16>
__device__ __forceinline__ void* row_at(void* base, long n, long sn, int c, long sc) {
    return static_cast<typename RowElem<BF16>::type*>(base) + n * sn + c * sc;
}

constexpr int kAhead = 4;  // vectors that a lane has in flight

template <bool BF16>
__global__ __launch_bounds__(kThreads) void norm_sums_kernel(NormArgs a) {
    __shared__ double lds[2 * kThreads / kSeqWave];
    const int unit = static_cast<int>(blockIdx.x) + a.first, group = div31(unit, a.by_pieces), piece = unit - group * a.pieces;
    const int n = div31(group, a.by_G), c0 = (group - n * a.G) * a.per, len = seq_length(a.lengths, n, a.L);
    const int from = piece * a.piece, to = min(a.items, from + a.piece);
    double s = 0.0, q = 0.0;
    if (len > 0) {
        const double shift = load_elem<BF16>(row_at<BF16>(a.x, n, a.x_sn, c0, a.x_sc), 0);
        for (int i0 = from + static_cast<int>(threadIdx.x); i0 < to; i0 += kThreads * kAhead) {
            float v[kAhead][8];
            int many[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int i = min(i0 + k * kThreads, a.items - 1), c = div31(i, a.by_vecs), at = 8 * (i - c * a.vecs);
                many[k] = i0 + k * kThreads < to ? len - at : 0;
                row_load8<BF16>(row_at<BF16>(a.x, n, a.x_sn, c0 + c, a.x_sc), at, len, v[k]);
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const double d = e < many[k] ? static_cast<double>(v[k][e]) - shift : 0.0;
                    s += d;
                    q = fma(d, d, q);
                }
            }
        }
    }
    block_sums<kThreads>(s, q, lds);
    if (threadIdx.x == 0) {
        a.part[2L * unit] = s;
        a.part[2L * unit + 1] = q;
    }
}

// joins the sums of a group's `many` pieces
__device__ __forceinline__ void join_pieces(const double* part, int many, double& s, double& q, double* lds) {
    s = q = 0.0;
    for (int i = static_cast<int>(threadIdx.x); i < many; i += kThreads) {
        s += part[2L * i];
        q += part[2L * i + 1];
    }
    block_sums<kThreads>(s, q, lds);
}

template <bool BF16, int ACT>
__global__ __launch_bounds__(kThreads) void norm_apply_kernel(NormArgs a) {
    __shared__ double lds[2 * kThreads / kSeqWave];
    const int unit = static_cast<int>(blockIdx.x) + a.first, group = div31(unit, a.by_pieces), piece = unit - group * a.pieces;
    const int n = div31(group, a.by_G), c0 = (group - n * a.G) * a.per, len = seq_length(a.lengths, n, a.L);
    double s, q, mean, rstd;
    join_pieces(a.part + 2L * group * a.pieces, a.pieces, s, q, lds);
    const double shift = len > 0 ? load_elem<BF16>(row_at<BF16>(a.x, n, a.x_sn, c0, a.x_sc), 0) : 0.f;
    stats_of(s, q, static_cast<double>(len) * a.per, shift, a.eps, mean, rstd);
    if (a.stats && piece == 0 && threadIdx.x == 0) {
        a.stats[2L * group] = mean;
        a.stats[2L * group + 1] = rstd;
    }
    const Mean m = mean_of(mean, rstd);
    const int from = piece * a.piece, to = min(a.items, from + a.piece);
    for (int i0 = from + static_cast<int>(threadIdx.x); i0 < to; i0 += kThreads * kAhead) {
        float v[kAhead][8];
        int at[kAhead], c[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = min(i0 + k * kThreads, a.items - 1), of = div31(i, a.by_vecs);
            at[k] = 8 * (i - of * a.vecs);
            c[k] = c0 + of;
            row_load8<BF16>(row_at<BF16>(a.x, n, a.x_sn, c[k], a.x_sc), at[k], len, v[k]);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i0 + k * kThreads >= to) break;
            const Channel ch = channel_of(m, a.weight, a.bias, c[k]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = act_of<ACT>(fmaf(h_of(v[k][e], ch), ch.w, ch.b));
                v[k][e] = at[k] + e < len ? y : 0.f;
            }
            row_store8<BF16>(row_at<BF16>(a.y, n, a.y_sn, c[k], a.y_sc), at[k], a.L, v[k]);
        }
    }
}

// p, h and dp of a vector
template <int ACT>
__device__ __forceinline__ void back8(const float (&x)[8], const float (&dy)[8], const Channel& ch, double mean, double rstd, int many, float (&h)[8],
                                      float (&dp)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        h[e] = h_of(x[e], ch);
        float p = fmaf(h[e], ch.w, ch.b);
        if (ACT == kRelu) p = relu_side(p, x[e], ch, mean, rstd);
        dp[e] = back_of<ACT>(dy[e], p);
        if (e >= many) h[e] = dp[e] = 0.f;
    }
}

// Sums of dp and dp h over each piece of a row, a.lanes lanes a piece (a power of two).
template <bool BF16, int ACT>
__global__ __launch_bounds__(kThreads) void norm_back_sums_kernel(NormArgs a) {
    __shared__ double lds[2 * kThreads / kSeqWave];
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (a.lanes - 1), teams = kThreads / a.lanes;
    const long unit = (static_cast<long>(blockIdx.x) + a.first) * teams + tid / a.lanes;
    const long units = static_cast<long>(a.N) * a.C * a.rows_pieces;
    const bool there = unit < units;
    const int u = static_cast<int>(there ? unit : units - 1);
    const int row = div31(u, a.by_rows_pieces), piece = u - row * a.rows_pieces, n = div31(row, a.by_C), c = row - n * a.C;
    const int len = seq_length(a.lengths, n, a.L);
    const long group = static_cast<long>(n) * a.G + c / a.per;
    const double mean = a.stats[2 * group], rstd = a.stats[2 * group + 1];
    const Channel ch = channel_of(mean_of(mean, rstd), a.weight, a.bias, c);
    const void *x = row_at<BF16>(a.x, n, a.x_sn, c, a.x_sc), *dy = row_at<BF16>(a.dy, n, a.dy_sn, c, a.dy_sc);
    const int from = piece * a.rows_piece, to = there ? min((len + 7) >> 3, from + a.rows_piece) : 0;
    double s = 0.0, q = 0.0;
    for (int i0 = from + lane; i0 < to; i0 += a.lanes * 2) {
        float v[2][8], g[2][8];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int at = 8 * min(i0 + k * a.lanes, to - 1);
            row_load8<BF16>(x, at, len, v[k]);
            row_load8<BF16>(dy, at, len, g[k]);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float h[8], dp[8], s8 = 0.f, q8 = 0.f;
            const int i = i0 + k * a.lanes;
            back8<ACT>(v[k], g[k], ch, mean, rstd, i < to ? len - 8 * i : 0, h, dp);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s8 += dp[e];
                q8 = fmaf(dp[e], h[e], q8);
            }
            s += static_cast<double>(s8);
            q += static_cast<double>(q8);
        }
    }
    if (a.lanes == kThreads) {
        block_sums<kThreads>(s, q, lds);
    } else {
        for (int m = 1; m < a.lanes; m <<= 1) {
            s += lane_xor(s, m);
            q += lane_xor(q, m);
        }
    }
    if (there && lane == 0) {
        a.part[2 * unit] = s;
        a.part[2 * unit + 1] = q;
    }
}

// dweight and dbias of a channel: its rows' pieces over all samples, one wave a channel
__device__ __forceinline__ void channel_sums(const NormArgs& a, int c, int lane, long n_step, int each) {
    double s = 0.0, q = 0.0;
    const int many = a.N * each;
    for (int i = lane; i < many; i += kSeqWave) {
        const int n = i / each;
        const long at = n * n_step + static_cast<long>(c) * each + (i - n * each);
        s += a.part[2 * at];
        q += a.part[2 * at + 1];
    }
    for (int m = 1; m < kSeqWave; m <<= 1) {
        s += lane_xor(s, m);
        q += lane_xor(q, m);
    }
    if (lane == 0) {
        if (a.dbias) a.dbias[c] = static_cast<float>(s);
        if (a.dweight) a.dweight[c] = static_cast<float>(q);
    }
}
__global__ __launch_bounds__(kThreads) void norm_channels_kernel(NormArgs a) {
    const int c = (static_cast<int>(blockIdx.x) * kThreads + static_cast<int>(threadIdx.x)) / kSeqWave;
    if (c < a.C) channel_sums(a, c, threadIdx.x & (kSeqWave - 1), static_cast<long>(a.C) * a.rows_pieces, a.rows_pieces);
}

// sums of dp weight and dp weight h over a group, of its channels' sums
__device__ __forceinline__ void join_channels(const NormArgs& a, const double* part, int c0, int each, double& s, double& q, double* lds) {
    s = q = 0.0;
    for (int i = static_cast<int>(threadIdx.x); i < a.per * each; i += kThreads) {
        const double w = a.weight ? a.weight[c0 + i / each] : 1.0;
        s = fma(w, part[2L * i], s);
        q = fma(w, part[2L * i + 1], q);
    }
    block_sums<kThreads>(s, q, lds);
}

template <bool BF16, int ACT>
__global__ __launch_bounds__(kThreads) void norm_back_kernel(NormArgs a) {
    __shared__ double lds[2 * kThreads / kSeqWave];
    const int unit = static_cast<int>(blockIdx.x) + a.first, group = div31(unit, a.by_pieces), piece = unit - group * a.pieces;
    const int n = div31(group, a.by_G), c0 = (group - n * a.G) * a.per, len = seq_length(a.lengths, n, a.L);
    double s, q;
    join_channels(a, a.part + 2 * (static_cast<long>(n) * a.C + c0) * a.rows_pieces, c0, a.rows_pieces, s, q, lds);
    const double mean = a.stats[2L * group], rstd = a.stats[2L * group + 1], over = len > 0 ? 1.0 / (static_cast<double>(len) * a.per) : 0.0;
    const Mean m = mean_of(mean, rstd);
    const float s1 = static_cast<float>(s * over), q1 = static_cast<float>(q * over);
    const int from = piece * a.piece, to = min(a.items, from + a.piece);
    for (int i0 = from + static_cast<int>(threadIdx.x); i0 < to; i0 += kThreads * 2) {
        float v[2][8], g[2][8];
        int at[2], c[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = min(i0 + k * kThreads, a.items - 1), of = div31(i, a.by_vecs);
            at[k] = 8 * (i - of * a.vecs);
            c[k] = c0 + of;
            row_load8<BF16>(row_at<BF16>(a.x, n, a.x_sn, c[k], a.x_sc), at[k], len, v[k]);
            row_load8<BF16>(row_at<BF16>(a.dy, n, a.dy_sn, c[k], a.dy_sc), at[k], len, g[k]);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (i0 + k * kThreads >= to) break;
            const Channel ch = channel_of(m, a.weight, a.bias, c[k]);
            float h[8], dp[8];
            back8<ACT>(v[k], g[k], ch, mean, rstd, len - at[k], h, dp);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] = at[k] + e < len ? m.rstd * (fmaf(dp[e], ch.w, -s1) - h[e] * q1) : 0.f;
            row_store8<BF16>(row_at<BF16>(a.dx, n, a.dx_sn, c[k], a.dx_sc), at[k], a.L, v[k]);
        }
    }
}

// ---- channels contiguous --------------------------------------------------------------------------------------------------
// A workgroup has some positions of a sample and up to kWide channels; a lane has 8 neighbouring channels at every tall-th of the
// positions.  Sums go to LDS and from there, a channel after the other, to part[n][piece][c].
constexpr int kWide = 8 * kThreads;

struct Lane {
    int c, l0, tall;   // first channel (C or more: none), first position and step
};
__device__ __forceinline__ Lane lane_of(const NormArgs& a, int block) {
    const int vecs = min(kThreads, (a.C - block * kWide + 7) >> 3), tid = static_cast<int>(threadIdx.x), tall = kThreads / vecs, l = tid / vecs;
    return Lane{l < tall ? block * kWide + 8 * (tid - l * vecs) : a.C, l, tall};
}

// Adds up s and q of the lanes that have the same channels; the sums of channel c go to part[2 c], part[2 c + 1].
__device__ __forceinline__ void channels_out(const NormArgs& a, const Lane& k, int block, const double (&s)[8], const double (&q)[8], double* part,
                                             double (*lds)[2]) {
    const int vecs = min(kThreads, (a.C - block * kWide + 7) >> 3), tid = static_cast<int>(threadIdx.x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        __syncthreads();
        lds[tid][0] = s[e];
        lds[tid][1] = q[e];
        __syncthreads();
        if (tid < vecs && k.c + e < a.C) {
            double u = s[e], v = q[e];
            for (int t = 1; t < k.tall; ++t) {
                u += lds[tid + t * vecs][0];
                v += lds[tid + t * vecs][1];
            }
            part[2L * (k.c + e)] = u;
            part[2L * (k.c + e) + 1] = v;
        }
    }
}

// the channels' groups, from c on
struct Groups {
    int g[8];
};
__device__ __forceinline__ Groups groups_of(const NormArgs& a, int c) {
    Groups r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.g[e] = min(c + e, a.C - 1) / a.per;
    return r;
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void norm_last_sums_kernel(NormArgs a) {
    __shared__ double lds[kThreads][2];
    const int unit = static_cast<int>(blockIdx.x) + a.first, n = div31(unit, a.by_pieces), piece = unit - n * a.pieces, block = static_cast<int>(blockIdx.y);
    const int len = seq_length(a.lengths, n, a.L), from = piece * a.piece, to = min(len, from + a.piece);
    const Lane k = lane_of(a, block);
    double s[8] = {}, q[8] = {};
    if (k.c < a.C && len > 0) {
        const Groups of = groups_of(a, k.c);
        float shift[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) shift[e] = load_elem<BF16>(row_at<BF16>(a.x, n, a.x_sn, 0, 0), of.g[e] * a.per);
        for (int l0 = from + k.l0; l0 < to; l0 += k.tall * kAhead) {
            float v[kAhead][8];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) row_load8<BF16>(row_at<BF16>(a.x, n, a.x_sn, min(l0 + j * k.tall, to - 1), a.x_sl), k.c, a.C, v[j]);
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                if (l0 + j * k.tall >= to) break;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const double d = static_cast<double>(v[j][e]) - static_cast<double>(shift[e]);
                    s[e] += d;
                    q[e] = fma(d, d, q[e]);
                }
            }
        }
    }
    channels_out(a, k, block, s, q, a.part + 2L * unit * a.C, lds);
}

// One workgroup a sample and group.  Forward: mean and rstd.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void norm_last_stats_kernel(NormArgs a) {
    __shared__ double lds[2 * kThreads / kSeqWave];
    const int group = static_cast<int>(blockIdx.x) + a.first, n = div31(group, a.by_G), c0 = (group - n * a.G) * a.per;
    const int len = seq_length(a.lengths, n, a.L);
    double s = 0.0, q = 0.0, mean, rstd;
    const double* part = a.part + 2L * (static_cast<long>(n) * a.pieces * a.C + c0);
    for (int i = static_cast<int>(threadIdx.x); i < a.per * a.pieces; i += kThreads) {
        const int piece = i / a.per;
        const long at = static_cast<long>(piece) * a.C + (i - piece * a.per);
        s += part[2 * at];
        q += part[2 * at + 1];
    }
    block_sums<kThreads>(s, q, lds);
    const double shift = len > 0 ? load_elem<BF16>(row_at<BF16>(a.x, n, a.x_sn, 0, 0), c0) : 0.f;
    stats_of(s, q, static_cast<double>(len) * a.per, shift, a.eps, mean, rstd);
    if (threadIdx.x == 0) {
        a.stats[2L * group] = mean;
        a.stats[2L * group + 1] = rstd;
    }
}

// mean, rstd and parameters of a lane's channels
struct Channels {
    Channel of[8];
    double mean[8], rstd[8];
};
__device__ __forceinline__ void channels_of(const NormArgs& a, int n, int c, Channels& r) {
    const Groups g = groups_of(a, c);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const long group = static_cast<long>(n) * a.G + g.g[e];
        r.mean[e] = a.stats[2 * group];
        r.rstd[e] = a.stats[2 * group + 1];
        r.of[e] = channel_of(mean_of(r.mean[e], r.rstd[e]), a.weight, a.bias, min(c + e, a.C - 1));
    }
}

template <bool BF16, int ACT>
__global__ __launch_bounds__(kThreads) void norm_last_apply_kernel(NormArgs a) {
    const int unit = static_cast<int>(blockIdx.x) + a.first, n = div31(unit, a.by_pieces), piece = unit - n * a.pieces, block = static_cast<int>(blockIdx.y);
    const int len = seq_length(a.lengths, n, a.L), from = piece * a.piece, to = min(a.L, from + a.piece);
    const Lane k = lane_of(a, block);
    if (k.c >= a.C) return;
    Channels ch;
    channels_of(a, n, k.c, ch);
    for (int l0 = from + k.l0; l0 < to; l0 += k.tall * kAhead) {
        float v[kAhead][8];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) row_load8<BF16>(row_at<BF16>(a.x, n, a.x_sn, min(l0 + j * k.tall, to - 1), a.x_sl), k.c, a.C, v[j]);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int l = l0 + j * k.tall;
            if (l >= to) break;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = act_of<ACT>(fmaf(h_of(v[j][e], ch.of[e]), ch.of[e].w, ch.of[e].b));
                v[j][e] = l < len ? y : 0.f;
            }
            row_store8<BF16>(row_at<BF16>(a.y, n, a.y_sn, l, a.y_sl), k.c, a.C, v[j]);
        }
    }
}

template <int ACT>
__device__ __forceinline__ void back_last(const float (&x)[8], const float (&dy)[8], const Channels& ch, float (&h)[8], float (&dp)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        h[e] = h_of(x[e], ch.of[e]);
        float p = fmaf(h[e], ch.of[e].w, ch.of[e].b);
        if (ACT == kRelu) p = relu_side(p, x[e], ch.of[e], ch.mean[e], ch.rstd[e]);
        dp[e] = back_of<ACT>(dy[e], p);
    }
}

template <bool BF16, int ACT>
__global__ __launch_bounds__(kThreads) void norm_last_back_sums_kernel(NormArgs a) {
    __shared__ double lds[kThreads][2];
    const int unit = static_cast<int>(blockIdx.x) + a.first, n = div31(unit, a.by_pieces), piece = unit - n * a.pieces, block = static_cast<int>(blockIdx.y);
    const int len = seq_length(a.lengths, n, a.L), from = piece * a.piece, to = min(len, from + a.piece);
    const Lane k = lane_of(a, block);
    double s[8] = {}, q[8] = {};
    if (k.c < a.C) {
        Channels ch;
        channels_of(a, n, k.c, ch);
        for (int l0 = from + k.l0; l0 < to; l0 += k.tall * 2) {
            float v[2][8], g[2][8];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int l = min(l0 + j * k.tall, to - 1);
                row_load8<BF16>(row_at<BF16>(a.x, n, a.x_sn, l, a.x_sl), k.c, a.C, v[j]);
                row_load8<BF16>(row_at<BF16>(a.dy, n, a.dy_sn, l, a.dy_sl), k.c, a.C, g[j]);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (l0 + j * k.tall >= to) break;
                float h[8], dp[8];
                back_last<ACT>(v[j], g[j], ch, h, dp);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s[e] += static_cast<double>(dp[e]);
                    q[e] = fma(static_cast<double>(dp[e]), static_cast<double>(h[e]), q[e]);
                }
            }
        }
    }
    channels_out(a, k, block, s, q, a.part + 2L * unit * a.C, lds);
}

// Backward: sums[n][c] of the pieces' sums, behind them; one wave a sample and channel.
__global__ __launch_bounds__(kThreads) void norm_last_join_kernel(NormArgs a, double* sums) {
    const long i = (static_cast<long>(blockIdx.x) * kThreads + threadIdx.x) / kSeqWave;
    if (i >= static_cast<long>(a.N) * a.C) return;
    const int n = div31(static_cast<int>(i), a.by_C), c = static_cast<int>(i) - n * a.C, lane = threadIdx.x & (kSeqWave - 1);
    double s = 0.0, q = 0.0;
    for (int p = lane; p < a.pieces; p += kSeqWave) {
        const long at = (static_cast<long>(n) * a.pieces + p) * a.C + c;
        s += a.part[2 * at];
        q += a.part[2 * at + 1];
    }
    for (int m = 1; m < kSeqWave; m <<= 1) {
        s += lane_xor(s, m);
        q += lane_xor(q, m);
    }
    if (lane == 0) {
        sums[2 * i] = s;
        sums[2 * i + 1] = q;
    }
}

// One workgroup a sample and group: the group's sums over m, in place of its channels' (they are read by norm_channels_kernel before).
__global__ __launch_bounds__(kThreads) void norm_last_groups_kernel(NormArgs a, const double* sums, double* groups) {
    __shared__ double lds[2 * kThreads / kSeqWave];
    const int group = static_cast<int>(blockIdx.x) + a.first, n = div31(group, a.by_G), c0 = (group - n * a.G) * a.per;
    const int len = seq_length(a.lengths, n, a.L);
    double s, q;
    join_channels(a, sums + 2L * (static_cast<long>(n) * a.C + c0), c0, 1, s, q, lds);
    const double over = len > 0 ? 1.0 / (static_cast<double>(len) * a.per) : 0.0;
    if (threadIdx.x == 0) {
        groups[2L * group] = s * over;
        groups[2L * group + 1] = q * over;
    }
}

template <bool BF16, int ACT>
__global__ __launch_bounds__(kThreads) void norm_last_back_kernel(NormArgs a, const double* groups) {
    const int unit = static_cast<int>(blockIdx.x) + a.first, n = div31(unit, a.by_pieces), piece = unit - n * a.pieces, block = static_cast<int>(blockIdx.y);
    const int len = seq_length(a.lengths, n, a.L), from = piece * a.piece, to = min(a.L, from + a.piece);
    const Lane k = lane_of(a, block);
    if (k.c >= a.C) return;
    Channels ch;
    channels_of(a, n, k.c, ch);
    const Groups of = groups_of(a, k.c);
    float s1[8], q1[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const long group = static_cast<long>(n) * a.G + of.g[e];
        s1[e] = static_cast<float>(groups[2 * group]);
        q1[e] = static_cast<float>(groups[2 * group + 1]);
    }
    for (int l0 = from + k.l0; l0 < to; l0 += k.tall * 2) {
        float v[2][8], g[2][8];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int l = min(l0 + j * k.tall, to - 1);
            row_load8<BF16>(row_at<BF16>(a.x, n, a.x_sn, l, a.x_sl), k.c, a.C, v[j]);
            row_load8<BF16>(row_at<BF16>(a.dy, n, a.dy_sn, l, a.dy_sl), k.c, a.C, g[j]);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int l = l0 + j * k.tall;
            if (l >= to) break;
            float h[8], dp[8];
            back_last<ACT>(v[j], g[j], ch, h, dp);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[j][e] = l < len ? ch.of[e].rstd * (fmaf(dp[e], ch.of[e].w, -s1[e]) - h[e] * q1[e]) : 0.f;
            row_store8<BF16>(row_at<BF16>(a.dx, n, a.dx_sn, l, a.dx_sl), k.c, a.C, v[j]);
        }
    }
}

// ---- host -----------------------------------------------------------------------------------------------------------
constexpr long kFill = 2048;   // workgroups that keep the chip busy: 8 a compute unit
constexpr int kMostPieces = 512;

int ceil_to(long n, int to) { return static_cast<int>((n + to - 1) / to * to); }

struct Plan {
    bool last;
    int vecs, items, pieces, piece, rows_pieces, rows_piece, lanes, blocks;
    size_t part, sums, groups, bytes;
};
// `last`: channels contiguous
Plan plan_of(int N, int C, int L, int G, bool last, bool back) {
    Plan p{};
    p.last = last;
    const long groups = static_cast<long>(N) * G;
    size_t at = 0;
    const auto take = [&](size_t pairs) {
        const size_t here = at;
        at += round_up(2 * sizeof(double) * pairs, 256);
        return here;
    };
    if (last) {
        p.blocks = cdiv(C, kWide);
        const int vecs = C >= kWide ? kThreads : (C + 7) / 8, tall = kThreads / vecs;
        long pieces = kFill / 2 / (static_cast<long>(N) * p.blocks);
        pieces = pieces < 1 ? 1 : pieces > kMostPieces ? kMostPieces : pieces;
        const long least = 4L * tall;  // positions that are worth a workgroup
        p.piece = ceil_to((L + pieces - 1) / pieces, static_cast<int>(least));
        p.pieces = cdiv(L, p.piece);
        p.part = take(static_cast<size_t>(N) * p.pieces * C);
        if (back) p.sums = take(static_cast<size_t>(N) * C);
        p.groups = take(static_cast<size_t>(groups));  // forward: mean and rstd where the caller wants none
    } else {
        p.vecs = (L + 7) / 8;
        p.items = static_cast<int>(static_cast<long>(C / G) * p.vecs);
        long pieces = kFill / groups;
        pieces = pieces < 1 ? 1 : pieces > kMostPieces ? kMostPieces : pieces;
        p.piece = ceil_to((p.items + pieces - 1) / pieces, kThreads);
        p.pieces = cdiv(p.items, p.piece);
        if (back) {
            const long rows = static_cast<long>(N) * C;
            p.lanes = 8;
            while (p.lanes < 64 && p.lanes < p.vecs) p.lanes *= 2;
            if (p.vecs > 128) p.lanes = kThreads;
            long cut = kFill / rows;
            cut = cut < 1 || p.lanes < kThreads ? 1 : cut > 64 ? 64 : cut;
            p.rows_piece = ceil_to((p.vecs + cut - 1) / cut, p.lanes);
            p.rows_pieces = cdiv(p.vecs, p.rows_piece);
            p.part = take(static_cast<size_t>(rows) * p.rows_pieces);
        } else {
            p.part = take(static_cast<size_t>(groups) * p.pieces);
        }
    }
    p.bytes = at;
    return p;
}

bool shape_ok(const conv1d_norm_t* p) {
    if (!p || !p->x || p->N < 1 || p->C < 1 || p->L < 1 || p->G < 1 || p->C % p->G || !(p->eps >= 0.0)) return false;
    if (p->dtype != CONV1D_FP32 && p->dtype != CONV1D_BF16) return false;
    if (p->flags & ~(CONV1D_NORM_RELU | CONV1D_NORM_SILU) || p->flags == (CONV1D_NORM_RELU | CONV1D_NORM_SILU)) return false;
    return seq_aligned(p->x, p->dtype == CONV1D_BF16 ? 2 : 4) && seq_aligned(p->weight, 4) && seq_aligned(p->bias, 4) && seq_aligned(p->lengths, 4);
}
bool sizes_ok(int N, int C, int L, int G) {
    const long vecs = (L + 7L) / 8;
    return C <= 1 << 20 && L <= 1 << 30 && static_cast<long>(N) * C <= 1 << 25 && static_cast<long>(C / G) * vecs <= 1 << 30;
}
// 1: positions contiguous, 2: channels, 0: neither; an axis of one element has no stride
int order_of(int C, int L, long sc, long sl) {
    if (L == 1 && (C == 1 || sc == 1)) return 2;
    if (L == 1 || sl == 1) return 1;
    return C == 1 || sc == 1 ? 2 : 0;
}
int order_of(const conv1d_norm_t* p) { return order_of(p->C, p->L, p->x_sc, p->x_sl); }
// whether a tensor of these strides can be taken in that order
bool fits(const conv1d_norm_t* p, int order, long sc, long sl) { return order == 2 ? p->C == 1 || sc == 1 : p->L == 1 || sl == 1; }

NormArgs args_of(const conv1d_norm_t* p, const Plan& plan, void* workspace) {
    NormArgs a{};
    a.x = p->x; a.weight = p->weight; a.bias = p->bias; a.lengths = p->lengths; a.eps = p->eps;
    a.x_sn = p->x_sn; a.x_sc = p->x_sc; a.x_sl = p->x_sl;
    a.N = p->N; a.C = p->C; a.L = p->L; a.G = p->G; a.per = p->C / p->G;
    a.vecs = plan.vecs; a.items = plan.items; a.pieces = plan.pieces; a.piece = plan.piece;
    a.rows_pieces = plan.rows_pieces; a.rows_piece = plan.rows_piece; a.lanes = plan.lanes;
    a.part = reinterpret_cast<double*>(static_cast<char*>(workspace) + plan.part);
    a.by_vecs = make_div31(plan.vecs ? plan.vecs : 1);
    a.by_pieces = make_div31(plan.pieces);
    a.by_G = make_div31(p->G);
    a.by_C = make_div31(p->C);
    a.by_rows_pieces = make_div31(plan.rows_pieces ? plan.rows_pieces : 1);
    return a;
}

// all units of a launch, in pieces that a grid may have
template <typename... More>
hipError_t launch_units(void (*kern)(NormArgs, More...), NormArgs& a, long units, int blocks, hipStream_t st, More... more) {
    const long most = kSeqMostThreads / kThreads / blocks;
    for (long u = 0; u < units; u += most) {
        a.first = static_cast<int>(u);
        const hipError_t e = launch_kernel(kern, dim3(static_cast<unsigned>(units - u < most ? units - u : most), static_cast<unsigned>(blocks)), dim3(kThreads), 0, st,
                                           a, more...);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <bool BF16, int ACT>
hipError_t forward(NormArgs& a, const Plan& plan, hipStream_t st) {
    const long groups = static_cast<long>(a.N) * a.G;
    if (!plan.last) {
        const hipError_t e = launch_units(norm_sums_kernel<BF16>, a, groups * plan.pieces, 1, st);
        return e == hipSuccess ? launch_units(norm_apply_kernel<BF16, ACT>, a, groups * plan.pieces, 1, st) : e;
    }
    const long units = static_cast<long>(a.N) * plan.pieces;
    hipError_t e = launch_units(norm_last_sums_kernel<BF16>, a, units, plan.blocks, st);
    if (e == hipSuccess) e = launch_units(norm_last_stats_kernel<BF16>, a, groups, 1, st);
    if (e == hipSuccess) e = launch_units(norm_last_apply_kernel<BF16, ACT>, a, units, plan.blocks, st);
    return e;
}

template <bool BF16, int ACT>
hipError_t backward(NormArgs& a, const Plan& plan, double* sums, double* groups, hipStream_t st) {
    const long many = static_cast<long>(a.N) * a.G, waves = kThreads / kSeqWave;
    const bool channels = a.dweight || a.dbias;
    const dim3 wave_a_channel(static_cast<unsigned>(cdiv(a.C, waves)));
    if (!plan.last) {
        const long teams = kThreads / plan.lanes, rows = static_cast<long>(a.N) * a.C * plan.rows_pieces;
        hipError_t e = launch_units(norm_back_sums_kernel<BF16, ACT>, a, cdiv(rows, teams), 1, st);
        if (e == hipSuccess) e = launch_units(norm_back_kernel<BF16, ACT>, a, many * plan.pieces, 1, st);
        if (e == hipSuccess && channels) e = launch_kernel(norm_channels_kernel, wave_a_channel, dim3(kThreads), 0, st, a);
        return e;
    }
    const long units = static_cast<long>(a.N) * plan.pieces;
    hipError_t e = launch_units(norm_last_back_sums_kernel<BF16, ACT>, a, units, plan.blocks, st);
    if (e == hipSuccess)
        e = launch_kernel(norm_last_join_kernel, dim3(static_cast<unsigned>(cdiv(static_cast<long>(a.N) * a.C, waves))), dim3(kThreads), 0, st, a, sums);
    if (e == hipSuccess) e = launch_units(norm_last_groups_kernel, a, many, 1, st, static_cast<const double*>(sums), groups);
    if (e == hipSuccess) e = launch_units(norm_last_back_kernel<BF16, ACT>, a, units, plan.blocks, st, static_cast<const double*>(groups));
    if (e == hipSuccess && channels) {
        NormArgs c = a;
        c.part = sums;
        c.rows_pieces = 1;
        e = launch_kernel(norm_channels_kernel, wave_a_channel, dim3(kThreads), 0, st, c);
    }
    return e;
}

template <bool BF16>
hipError_t forward(NormArgs& a, const Plan& plan, int act, hipStream_t st) {
    return act == kRelu ? forward<BF16, kRelu>(a, plan, st) : act == kSilu ? forward<BF16, kSilu>(a, plan, st) : forward<BF16, kNone>(a, plan, st);
}
template <bool BF16>
hipError_t backward(NormArgs& a, const Plan& plan, int act, double* sums, double* groups, hipStream_t st) {
    return act == kRelu   ? backward<BF16, kRelu>(a, plan, sums, groups, st)
           : act == kSilu ? backward<BF16, kSilu>(a, plan, sums, groups, st)
                          : backward<BF16, kNone>(a, plan, sums, groups, st);
}

int act_flag(int flags) { return flags & CONV1D_NORM_RELU ? kRelu : flags & CONV1D_NORM_SILU ? kSilu : kNone; }
int status_of(hipError_t e) { return e == hipSuccess ? CONV1D_OK : CONV1D_EHIP; }

size_t workspace_of(int N, int C, int L, int G, bool back) {
    if (N < 1 || C < 1 || L < 1 || G < 1 || C % G || !sizes_ok(N, C, L, G)) return 0;
    const size_t rows = plan_of(N, C, L, G, false, back).bytes, last = plan_of(N, C, L, G, true, back).bytes;
    return rows > last ? rows : last;
}

}  // namespace
}  // namespace conv1d

using namespace conv1d;

extern "C" {

size_t conv1d_norm_fwd_workspace_bytes(int N, int C, int L, int G) { return workspace_of(N, C, L, G, false); }
size_t conv1d_norm_bwd_workspace_bytes(int N, int C, int L, int G) { return workspace_of(N, C, L, G, true); }

int conv1d_norm_fwd(const conv1d_norm_t* p, void* y, long y_sn, long y_sc, long y_sl, double* stats, void* workspace, size_t workspace_bytes, void* stream) {
    if (!shape_ok(p) || !y) return CONV1D_EINVAL;
    const size_t size = p->dtype == CONV1D_BF16 ? 2 : 4;
    const int order = order_of(p);
    if (!seq_aligned(y, size) || !seq_aligned(stats, 8) || !seq_aligned(workspace, 256) || !order || !fits(p, order, y_sc, y_sl)) return CONV1D_EINVAL;
    if (!sizes_ok(p->N, p->C, p->L, p->G)) return CONV1D_EUNSUPPORTED;
    const Plan plan = plan_of(p->N, p->C, p->L, p->G, order == 2, false);
    if (!workspace || workspace_bytes < plan.bytes) return CONV1D_EWORKSPACE;
    NormArgs a = args_of(p, plan, workspace);
    a.y = y; a.y_sn = y_sn; a.y_sc = y_sc; a.y_sl = y_sl;
    a.stats = stats ? stats : plan.last ? reinterpret_cast<double*>(static_cast<char*>(workspace) + plan.groups) : nullptr;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int act = act_flag(p->flags);
    return status_of(p->dtype == CONV1D_BF16 ? forward<true>(a, plan, act, st) : forward<false>(a, plan, act, st));
}

int conv1d_norm_bwd(const conv1d_norm_t* p, const void* dy, long dy_sn, long dy_sc, long dy_sl, const double* stats, void* dx, long dx_sn, long dx_sc, long dx_sl,
                    float* dweight, float* dbias, void* workspace, size_t workspace_bytes, void* stream) {
    if (!shape_ok(p) || !dy || !dx || !stats) return CONV1D_EINVAL;
    const size_t size = p->dtype == CONV1D_BF16 ? 2 : 4;
    const int order = order_of(p);
    if (!seq_aligned(dy, size) || !seq_aligned(dx, size) || !seq_aligned(stats, 8) || !seq_aligned(dweight, 4) || !seq_aligned(dbias, 4) ||
        !seq_aligned(workspace, 256) || !order || !fits(p, order, dy_sc, dy_sl) || !fits(p, order, dx_sc, dx_sl))
        return CONV1D_EINVAL;
    if (!sizes_ok(p->N, p->C, p->L, p->G)) return CONV1D_EUNSUPPORTED;
    const Plan plan = plan_of(p->N, p->C, p->L, p->G, order == 2, true);
    if (!workspace || workspace_bytes < plan.bytes) return CONV1D_EWORKSPACE;
    NormArgs a = args_of(p, plan, workspace);
    a.dy = dy; a.dy_sn = dy_sn; a.dy_sc = dy_sc; a.dy_sl = dy_sl;
    a.dx = dx; a.dx_sn = dx_sn; a.dx_sc = dx_sc; a.dx_sl = dx_sl;
    a.stats = const_cast<double*>(stats);
    a.dweight = dweight; a.dbias = dbias;
    char* ws = static_cast<char*>(workspace);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int act = act_flag(p->flags);
    double *sums = reinterpret_cast<double*>(ws + plan.sums), *groups = reinterpret_cast<double*>(ws + plan.groups);
    return status_of(p->dtype == CONV1D_BF16 ? backward<true>(a, plan, act, sums, groups, st) : backward<false>(a, plan, act, sums, groups, st));
}

}  // extern "C"
