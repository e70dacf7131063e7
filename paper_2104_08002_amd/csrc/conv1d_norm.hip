// Group norm with an activation behind it, for positions or channels contiguous, forward and backward.
//   mean, var: of a group's C / G channels over the positions of its sequence (m values);  rstd = 1 / sqrt(var + eps)
//   h = (x - mean) rstd,  p = h weight[c] + bias[c],  y = p, max(p, 0) or p sigmoid(p)
//   dp = dy act'(p),  dbias = sum dp,  dweight = sum dp h,  dx = rstd (dp weight - (sum dp weight) / m - h (sum dp weight h) / m)
// Bound by memory.  Groups that fit in the registers of one workgroup are read once; larger ones are read twice, cut into enough
// pieces to fill the chip: one launch adds up each piece, the next joins a group's pieces (every workgroup for itself, in one order)
// and writes.  Values are summed as differences from the group's first one, in 64 bits, so that neither a mean far from 0 nor a
// long group costs digits; mean and rstd are kept in 64 bits, and (x - mean) is taken with the mean as two floats.
// 8 x 64 x 20000 bfloat16 in 8 groups: 7 + 9 us forward, 11 + 14 backward (20, 41, 41 and 61 MB: 2.9 to 4.4 TB/s in one turn of the chip);
// 8 x 512 x 8192 with channels next to each other: 15 + 5 + 28 forward, 32 + 5 + 39 backward (67, 134, 134 and 201 MB: 4.2 to 5.1 TB/s).
#include "conv1d_blocks.h"

namespace conv1d {
namespace {

constexpr int kThreads = 256, kJoinThreads = 512;
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
    int first, extra;       // extra: workgroups of each of the grid's rows that add up channels (of one workgroup a group: whether they are wanted)
    Div31 by_vecs, by_pieces, by_G, by_C, by_per, by_rows_pieces;
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

// One channel: with t = x - hi, h = t rstd + h0 and p = t a + b.
struct Channel {
    float hi, a, b, near;
};
__device__ __forceinline__ float start_of(const Mean& m) { return -m.lo * m.rstd; }
// near: the side of 0 that p lies on decides over the ReLU's gradient.  p is off by a few units of 2^-24 of t a, h0 w and the bias; next to
// 0 |t a| is about |b|, and |h0 w| + |bias| is at most |b| + 2 |h0 w|: the sign of a larger p is right, smaller ones are found in 64 bits.
__device__ __forceinline__ Channel channel_of(const Mean& m, float w, float b) {
    const float h0w = start_of(m) * w, c = fmaf(start_of(m), w, b);
    return Channel{m.hi, m.rstd * w, c, 1.9073486328125e-06f * (fabsf(c) + fabsf(h0w))};
}
__device__ __forceinline__ float weight_of(const NormArgs& a, int c) { return a.weight ? a.weight[c] : 1.f; }
__device__ __forceinline__ float bias_of(const NormArgs& a, int c) { return a.bias ? a.bias[c] : 0.f; }

// a number with the sign that p has in 64 bits
__device__ __forceinline__ float side_of(const NormArgs& a, float x, int n, int c) {
    const long group = static_cast<long>(n) * a.G + div31(c, a.by_per);
    const double p = (static_cast<double>(x) - a.stats[2 * group]) * a.stats[2 * group + 1] * static_cast<double>(weight_of(a, c)) + static_cast<double>(bias_of(a, c));
    return p > 0.0 ? 1.f : p <= 0.0 ? -1.f : __builtin_nanf("");
}

// t = x - hi of 8 values, and dp in place of dy; channel e is k[STEP e], number c + STEP e.  (What lies next to 0 is rare: it goes through
// one value at a time, so that it costs the other path no registers.)
template <int ACT, int STEP>
__device__ __forceinline__ void back8(const NormArgs& a, const float (&x)[8], const Channel* k, int n, int c, float (&t)[8], float (&dy)[8]) {
    float p[8];
    bool near = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        t[e] = x[e] - k[STEP * e].hi;
        p[e] = fmaf(t[e], k[STEP * e].a, k[STEP * e].b);
        near |= fabsf(p[e]) <= k[STEP * e].near;
    }
    if (ACT == kRelu) {
        if (wave_any(near)) {
#pragma unroll 1
            for (int i = 0; i < 8; ++i) {
                float v = x[0];
#pragma unroll
                for (int e = 1; e < 8; ++e) v = i == e ? x[e] : v;
                const float side = side_of(a, v, n, min(c + STEP * i, a.C - 1));
#pragma unroll
                for (int e = 0; e < 8; ++e) p[e] = i == e ? side : p[e];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) dy[e] = back_of<ACT>(dy[e], p[e]);
}

// dx = rstd (dp w - s1 - h q1) = dp a + t q + s
struct Back {
    float q, s;
};
__device__ __forceinline__ Back back_const(const Mean& m, double s1, double q1) {
    return Back{static_cast<float>(-q1 * m.rstd * m.rstd), static_cast<float>(-m.rstd * (s1 + q1 * start_of(m)))};
}
// sum of dp h, of the sums of dp t and of dp
__device__ __forceinline__ double with_h(double dpt, double dp, double mean, double rstd) {
    return rstd * (dpt + dp * (static_cast<double>(static_cast<float>(mean)) - mean));
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

// vectors that a lane has in flight
constexpr int kAhead = 4;
template <bool BF16>
constexpr int kAheadBack = BF16 ? 4 : 2;  // of x and of dy

// K vectors of a group, `step` apart from item i0 on (those behind the last are the last): channels, first positions and x
template <bool BF16, int K>
struct Batch {
    Raw8<BF16> x[K];
    int c[K], at[K], fresh[K];  // fresh: the first element that no vector before has
};
template <bool BF16, bool WHOLE, int K>
__device__ __forceinline__ void places_of(const NormArgs& a, int c0, int i0, int step, Batch<BF16, K>& r) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = min(i0 + k * step, a.items - 1), of = div31(i, a.by_vecs);
        r.c[k] = c0 + of;
        r.at[k] = vector_at<WHOLE>(i - of * a.vecs, a.L);
        r.fresh[k] = 8 * (i - of * a.vecs) - r.at[k];
    }
}
template <bool BF16, bool WHOLE, int K>
__device__ __forceinline__ void load_rows(const NormArgs& a, const void* base, int n, long sn, long sc, int len, const Batch<BF16, K>& at, Raw8<BF16> (&r)[K]) {
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (WHOLE || wave_any(at.at[k] < len)) r[k] = raw8_row<BF16, WHOLE>(row_at<BF16>(base, n, sn, at.c[k], sc), at.at[k], a.L);
}

// sums of x - shift and of its squares over one vector's values before len
template <bool BF16, bool WHOLE>
__device__ __forceinline__ void add_values(const Raw8<BF16>& raw, int at, int fresh, int len, double shift, double& s, double& q) {
    float v[8];
    floats_of(raw, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double d = WHOLE || (e >= fresh && at + e < len) ? static_cast<double>(v[e]) - shift : 0.0;
        s += d;
        q = fma(d, d, q);
    }
}
// the group's first value; 0 for an empty sequence
template <bool BF16>
__device__ __forceinline__ double shift_of(const NormArgs& a, int n, int c0, int len) {
    const float v = load_elem<BF16>(row_at<BF16>(a.x, n, a.x_sn, c0, a.x_sc), 0);
    return len > 0 ? v : 0.f;
}

// y of a vector
template <bool BF16, int ACT, bool WHOLE>
__device__ __forceinline__ void apply_vector(const NormArgs& a, const Raw8<BF16>& raw, const Channel& k, int n, int c, int at, int len) {
    float v[8];
    floats_of(raw, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float y = act_of<ACT>(fmaf(v[e] - k.hi, k.a, k.b));
        v[e] = WHOLE || at + e < len ? y : 0.f;
    }
    vector_store8<BF16, WHOLE>(row_at<BF16>(a.y, n, a.y_sn, c, a.y_sc), at, a.L, v);
}

struct Unit {
    int n, group, c0, len, piece;
};
__device__ __forceinline__ Unit unit_of(const NormArgs& a, int unit) {
    Unit r;
    r.group = div31(unit, a.by_pieces);
    r.piece = unit - r.group * a.pieces;
    r.n = div31(r.group, a.by_G);
    r.c0 = (r.group - r.n * a.G) * a.per;
    r.len = seq_length(a.lengths, r.n, a.L);
    return r;
}

template <bool BF16, bool WHOLE>
__global__ __launch_bounds__(kThreads) void norm_sums_kernel(NormArgs a) {
    __shared__ double lds[2 * kThreads / kSeqWave];
    const int unit = static_cast<int>(blockIdx.x) + a.first;
    const Unit u = unit_of(a, unit);
    const int from = u.piece * a.piece, to = min(a.items, from + a.piece);
    const double shift = shift_of<BF16>(a, u.n, u.c0, u.len);
    double s = 0.0, q = 0.0;
    for (int i0 = from + static_cast<int>(threadIdx.x); i0 < to; i0 += kThreads * kAhead) {
        Batch<BF16, kAhead> b;
        places_of<BF16, WHOLE>(a, u.c0, i0, kThreads, b);
        load_rows<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sc, u.len, b, b.x);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (i0 + k * kThreads < to) add_values<BF16, WHOLE>(b.x[k], b.at[k], b.fresh[k], u.len, shift, s, q);
    }
    block_sums<kThreads>(s, q, lds);
    if (threadIdx.x == 0) {
        a.part[2L * unit] = s;
        a.part[2L * unit + 1] = q;
    }
}

__device__ __forceinline__ void keep_stats(const NormArgs& a, int group, double mean, double rstd) {
    if (a.stats && threadIdx.x == 0) {
        a.stats[2L * group] = mean;
        a.stats[2L * group + 1] = rstd;
    }
}

// The first vectors are on their way while the group's sums are joined.
template <bool BF16, int ACT, bool WHOLE>
__global__ __launch_bounds__(kThreads) void norm_apply_kernel(NormArgs a) {
    __shared__ double lds[2 * kThreads / kSeqWave];
    const Unit u = unit_of(a, static_cast<int>(blockIdx.x) + a.first);
    const int from = u.piece * a.piece + static_cast<int>(threadIdx.x), to = min(a.items, (u.piece + 1) * a.piece);
    Batch<BF16, kAhead> b;
    places_of<BF16, WHOLE>(a, u.c0, from, kThreads, b);
    load_rows<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sc, u.len, b, b.x);
    const double shift = shift_of<BF16>(a, u.n, u.c0, u.len);
    double s = 0.0, q = 0.0, mean, rstd;
    const double* part = a.part + 2L * u.group * a.pieces;
    for (int i = static_cast<int>(threadIdx.x); i < a.pieces; i += kThreads) {
        s += part[2L * i];
        q += part[2L * i + 1];
    }
    block_sums<kThreads>(s, q, lds);
    stats_of(s, q, static_cast<double>(u.len) * a.per, shift, a.eps, mean, rstd);
    if (u.piece == 0) keep_stats(a, u.group, mean, rstd);
    const Mean m = mean_of(mean, rstd);
    for (int i0 = from;;) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (i0 + k * kThreads < to)
                apply_vector<BF16, ACT, WHOLE>(a, b.x[k], channel_of(m, weight_of(a, b.c[k]), bias_of(a, b.c[k])), u.n, b.c[k], b.at[k], u.len);
        i0 += kThreads * kAhead;
        if (i0 >= to) break;
        places_of<BF16, WHOLE>(a, u.c0, i0, kThreads, b);
        load_rows<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sc, u.len, b, b.x);
    }
}

// A group whose values THREADS lanes hold in kAhead vectors each.
template <bool BF16, int ACT, bool WHOLE, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_one_kernel(NormArgs a) {
    __shared__ double lds[2 * THREADS / kSeqWave];
    const Unit u = unit_of(a, static_cast<int>(blockIdx.x) + a.first);
    const int tid = static_cast<int>(threadIdx.x);
    Batch<BF16, kAhead> b;
    places_of<BF16, WHOLE>(a, u.c0, tid, THREADS, b);
    load_rows<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sc, u.len, b, b.x);
    const double shift = shift_of<BF16>(a, u.n, u.c0, u.len);
    double s = 0.0, q = 0.0, mean, rstd;
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
        if (tid + k * THREADS < a.items) add_values<BF16, WHOLE>(b.x[k], b.at[k], b.fresh[k], u.len, shift, s, q);
    block_sums<THREADS>(s, q, lds);
    stats_of(s, q, static_cast<double>(u.len) * a.per, shift, a.eps, mean, rstd);
    keep_stats(a, u.group, mean, rstd);
    const Mean m = mean_of(mean, rstd);
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
        if (tid + k * THREADS < a.items)
            apply_vector<BF16, ACT, WHOLE>(a, b.x[k], channel_of(m, weight_of(a, b.c[k]), bias_of(a, b.c[k])), u.n, b.c[k], b.at[k], u.len);
}

// sums of dp and dp t over a vector's positions before len
template <bool BF16, int ACT, bool WHOLE>
__device__ __forceinline__ void back_sums(const NormArgs& a, const Raw8<BF16>& xr, const Raw8<BF16>& gr, const Channel& k, int n, int c, int at, int fresh,
                                          int len, float& s, float& q) {
    float x[8], g[8], t[8];
    floats_of(xr, x);
    floats_of(gr, g);
    back8<ACT, 0>(a, x, &k, n, c, t, g);
    s = q = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        s += WHOLE || (e >= fresh && at + e < len) ? g[e] : 0.f;
        q = WHOLE || (e >= fresh && at + e < len) ? fmaf(g[e], t[e], q) : q;
    }
}
// dx of a vector
template <bool BF16, int ACT, bool WHOLE>
__device__ __forceinline__ void back_vector(const NormArgs& a, const Raw8<BF16>& xr, const Raw8<BF16>& gr, const Channel& k, const Back& back, int n, int c,
                                            int at, int len) {
    float x[8], g[8], t[8];
    floats_of(xr, x);
    floats_of(gr, g);
    back8<ACT, 0>(a, x, &k, n, c, t, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = WHOLE || at + e < len ? fmaf(g[e], k.a, fmaf(t[e], back.q, back.s)) : 0.f;
    vector_store8<BF16, WHOLE>(row_at<BF16>(a.dx, n, a.dx_sn, c, a.dx_sc), at, a.L, x);
}

// Sums of dp and dp h over each piece of a row, a.lanes lanes a piece (a power of two).
template <bool BF16, int ACT, bool WHOLE>
__global__ __launch_bounds__(kThreads) void norm_back_sums_kernel(NormArgs a) {
    __shared__ double lds[2 * kThreads / kSeqWave];
    constexpr int K = kAheadBack<BF16>;
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (a.lanes - 1), teams = kThreads / a.lanes;
    const long unit = (static_cast<long>(blockIdx.x) + a.first) * teams + tid / a.lanes;
    const long units = static_cast<long>(a.N) * a.C * a.rows_pieces;
    const bool there = unit < units;
    const int u = static_cast<int>(there ? unit : units - 1);
    const int row = div31(u, a.by_rows_pieces), piece = u - row * a.rows_pieces, n = div31(row, a.by_C), c = row - n * a.C;
    const int len = seq_length(a.lengths, n, a.L);
    const long group = static_cast<long>(n) * a.G + c / a.per;
    const int from = piece * a.rows_piece + lane, to = there ? min((len + 7) >> 3, (piece + 1) * a.rows_piece) : 0;
    const void *x = row_at<BF16>(a.x, n, a.x_sn, c, a.x_sc), *dy = row_at<BF16>(a.dy, n, a.dy_sn, c, a.dy_sc);
    const double mean = a.stats[2 * group], rstd = a.stats[2 * group + 1];
    const float w = weight_of(a, c), bias = bias_of(a, c);
    double s = 0.0, q = 0.0;
    for (int i0 = from; i0 < to; i0 += a.lanes * K) {
        Raw8<BF16> v[K], g[K];
        int at[K], fresh[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int vec = min(i0 + k * a.lanes, to - 1);
            at[k] = vector_at<WHOLE>(vec, a.L);
            fresh[k] = 8 * vec - at[k];
            v[k] = raw8_row<BF16, WHOLE>(x, at[k], a.L);
            g[k] = raw8_row<BF16, WHOLE>(dy, at[k], a.L);
        }
        const Mean m = mean_of(mean, rstd);
        const Channel ch = channel_of(m, w, bias);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (i0 + k * a.lanes >= to) break;
            float s8, q8;
            back_sums<BF16, ACT, WHOLE>(a, v[k], g[k], ch, n, c, at[k], fresh[k], len, s8, q8);
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
        a.part[2 * unit + 1] = len > 0 ? with_h(q, s, mean, rstd) : 0.0;
    }
}

// dweight and dbias of a channel: its rows' pieces over all samples, one wave a channel.  part: [N][C][each].
__device__ __forceinline__ void channel_sums(const NormArgs& a, int c, const double* part, int each) {
    const int lane = static_cast<int>(threadIdx.x) & (kSeqWave - 1), many = a.N * each;
    double s = 0.0, q = 0.0;
#pragma unroll 2
    for (int i = lane; i < many; i += kSeqWave) {
        const int n = each == 1 ? i : div31(i, a.by_rows_pieces);
        const long at = (static_cast<long>(n) * a.C + c) * each + (i - n * each);
        s += part[2 * at];
        q += part[2 * at + 1];
    }
#pragma unroll
    for (int m = 1; m < kSeqWave; m <<= 1) {
        s += lane_xor(s, m);
        q += lane_xor(q, m);
    }
    if (lane == 0) {
        if (a.dbias) a.dbias[c] = static_cast<float>(s);
        if (a.dweight) a.dweight[c] = static_cast<float>(q);
    }
}
// the first `a.extra` workgroups of each of the grid's rows
__device__ __forceinline__ bool took_channels(const NormArgs& a, const double* part, int each) {
    if (static_cast<int>(blockIdx.x) >= a.extra) return false;
    const int c = (static_cast<int>(blockIdx.y) * a.extra + static_cast<int>(blockIdx.x)) * (kThreads / kSeqWave) + static_cast<int>(threadIdx.x) / kSeqWave;
    if (c < a.C) channel_sums(a, c, part, each);
    return true;
}
__global__ __launch_bounds__(kThreads) void norm_channels_kernel(NormArgs a) { took_channels(a, a.part, 1); }

template <bool BF16, int ACT, bool WHOLE>
__global__ __launch_bounds__(kThreads) void norm_back_kernel(NormArgs a) {
    __shared__ double lds[2 * kThreads / kSeqWave];
    constexpr int K = kAheadBack<BF16>;
    if (took_channels(a, a.part, a.rows_pieces)) return;
    const Unit u = unit_of(a, static_cast<int>(blockIdx.x) - a.extra + a.first);
    const int from = u.piece * a.piece + static_cast<int>(threadIdx.x), to = min(a.items, (u.piece + 1) * a.piece);
    Batch<BF16, K> b;
    Raw8<BF16> g[K];
    places_of<BF16, WHOLE>(a, u.c0, from, kThreads, b);
    load_rows<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sc, u.len, b, b.x);
    load_rows<BF16, WHOLE>(a, a.dy, u.n, a.dy_sn, a.dy_sc, u.len, b, g);
    const double mean = a.stats[2L * u.group], rstd = a.stats[2L * u.group + 1];
    double s = 0.0, q = 0.0;
    const double* part = a.part + 2 * (static_cast<long>(u.n) * a.C + u.c0) * a.rows_pieces;
    for (int i = static_cast<int>(threadIdx.x); i < a.per * a.rows_pieces; i += kThreads) {
        const double w = weight_of(a, u.c0 + div31(i, a.by_rows_pieces));
        s = fma(w, part[2L * i], s);
        q = fma(w, part[2L * i + 1], q);
    }
    block_sums<kThreads>(s, q, lds);
    const double over = u.len > 0 ? 1.0 / (static_cast<double>(u.len) * a.per) : 0.0;
    const Mean m = mean_of(mean, rstd);
    const Back back = back_const(m, s * over, q * over);
    for (int i0 = from;;) {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (i0 + k * kThreads < to) {
                const float w = weight_of(a, b.c[k]);
                back_vector<BF16, ACT, WHOLE>(a, b.x[k], g[k], channel_of(m, w, bias_of(a, b.c[k])), back, u.n, b.c[k], b.at[k], u.len);
            }
        i0 += kThreads * K;
        if (i0 >= to) break;
        places_of<BF16, WHOLE>(a, u.c0, i0, kThreads, b);
        load_rows<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sc, u.len, b, b.x);
        load_rows<BF16, WHOLE>(a, a.dy, u.n, a.dy_sn, a.dy_sc, u.len, b, g);
    }
}

// Backward of a group that THREADS lanes hold; its channels' sums go to part[n][c], for norm_channels_kernel.
template <bool BF16, int ACT, bool WHOLE, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_back_one_kernel(NormArgs a) {
    constexpr int K = kAheadBack<BF16>;
    __shared__ double lds[2 * THREADS / kSeqWave];
    __shared__ float vector[K * THREADS][2];
    const Unit u = unit_of(a, static_cast<int>(blockIdx.x) + a.first);
    const int tid = static_cast<int>(threadIdx.x);
    Batch<BF16, K> b;
    Raw8<BF16> g[K];
    places_of<BF16, WHOLE>(a, u.c0, tid, THREADS, b);
    load_rows<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sc, u.len, b, b.x);
    load_rows<BF16, WHOLE>(a, a.dy, u.n, a.dy_sn, a.dy_sc, u.len, b, g);
    const double mean = a.stats[2L * u.group], rstd = a.stats[2L * u.group + 1];
    const Mean m = mean_of(mean, rstd);
    double s = 0.0, q = 0.0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int i = tid + k * THREADS;
        if (i >= a.items) break;
        const float w = weight_of(a, b.c[k]);
        float s8, q8;
        back_sums<BF16, ACT, WHOLE>(a, b.x[k], g[k], channel_of(m, w, bias_of(a, b.c[k])), u.n, b.c[k], b.at[k], b.fresh[k], u.len, s8, q8);
        vector[i][0] = s8;
        vector[i][1] = q8;
        s = fma(static_cast<double>(w), static_cast<double>(s8), s);
        q = fma(static_cast<double>(w), static_cast<double>(q8), q);
    }
    block_sums<THREADS>(s, q, lds);
    if (a.extra) {
        __syncthreads();  // every vector's sums are there
        // lanes of a channel: as many as there are for all of them, up to a wave
        int lanes = 1;
        while (lanes < kSeqWave && 2 * lanes * a.per <= THREADS) lanes *= 2;
        for (int c0 = 0; c0 < a.per; c0 += THREADS / lanes) {
            const int c = c0 + tid / lanes, lane = tid & (lanes - 1);
            double cs = 0.0, cq = 0.0;
            if (c < a.per)
                for (int i = lane; i < a.vecs; i += lanes) {
                    cs += static_cast<double>(vector[c * a.vecs + i][0]);
                    cq += static_cast<double>(vector[c * a.vecs + i][1]);
                }
            for (int l = 1; l < lanes; l <<= 1) {
                cs += lane_xor(cs, l);
                cq += lane_xor(cq, l);
            }
            if (c < a.per && lane == 0) {
                double* part = a.part + 2 * (static_cast<long>(u.n) * a.C + u.c0 + c);
                part[0] = cs;
                part[1] = u.len > 0 ? with_h(cq, cs, mean, rstd) : 0.0;
            }
        }
    }
    const double over = u.len > 0 ? 1.0 / (static_cast<double>(u.len) * a.per) : 0.0;
    const Back back = back_const(m, s * over, with_h(q, s, mean, rstd) * over);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (tid + k * THREADS >= a.items) break;
        const float w = weight_of(a, b.c[k]);
        back_vector<BF16, ACT, WHOLE>(a, b.x[k], g[k], channel_of(m, w, bias_of(a, b.c[k])), back, u.n, b.c[k], b.at[k], u.len);
    }
}

// ---- channels contiguous --------------------------------------------------------------------------------------------------
// A workgroup has some positions of a sample and up to kWide channels; a lane has 8 neighbouring channels at every tall-th of the
// positions.  Sums go through LDS to part[n][piece][c].
constexpr int kWide = 8 * kThreads;

struct Lane {
    int c, l0, tall, vecs;   // first channel (C or more: none), first position and step, lanes of a position
    int fresh;               // (a group's) the first of its 8 channels that no lane before has
};
template <bool WHOLE>
__device__ __forceinline__ Lane lane_of(const NormArgs& a, int block) {
    Lane r;
    r.vecs = min(kThreads, (a.C - block * kWide + 7) >> 3);
    r.tall = kThreads / r.vecs;
    r.l0 = static_cast<int>(threadIdx.x) / r.vecs;
    r.c = r.l0 < r.tall ? vector_at<WHOLE>(block * (kWide / 8) + static_cast<int>(threadIdx.x) - r.l0 * r.vecs, a.C) : a.C;
    return r;
}

struct LastUnit {
    int unit, n, len, from, piece;
};
__device__ __forceinline__ LastUnit last_unit(const NormArgs& a, int unit) {
    LastUnit r;
    r.unit = unit;
    r.n = div31(unit, a.by_pieces);
    r.piece = unit - r.n * a.pieces;
    r.len = seq_length(a.lengths, r.n, a.L);
    r.from = r.piece * a.piece;
    return r;
}

// Adds up s and q of the lanes that have the same channels; the sums of channel c go to part[2 c], part[2 c + 1].
struct LastLds {
    double v[kThreads][8 + 1];
};
template <bool WHOLE>
__device__ __forceinline__ void channels_out(const NormArgs& a, const Lane& k, const double (&s)[8], const double (&q)[8], double* part, LastLds& lds) {
    const int tid = static_cast<int>(threadIdx.x), block = static_cast<int>(blockIdx.y);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) lds.v[tid][e] = h ? q[e] : s[e];
        __syncthreads();
        // a channel of the workgroup's a lane
        for (int i = tid; i < 8 * k.vecs; i += kThreads) {
            const int c = block * kWide + i, e = c - vector_at<WHOLE>(c >> 3, a.C);
            if (c >= a.C) break;
            double u = 0.0;
            for (int t = 0; t < k.tall; ++t) u += lds.v[(i >> 3) + t * k.vecs][e];
            part[2L * c + h] = u;
        }
    }
}

// the groups of a lane's channels
struct Groups {
    long g[8];   // among all samples'
};
__device__ __forceinline__ Groups groups_of(const NormArgs& a, int n, int c) {
    Groups r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.g[e] = static_cast<long>(n) * a.G + div31(min(c + e, a.C - 1), a.by_per);
    return r;
}

// K positions' vectors of the lane's channels, from l0 on (those behind the last are the last)
template <bool BF16, bool WHOLE, int K>
__device__ __forceinline__ void load_last(const NormArgs& a, const void* base, int n, long sn, long sl, const Lane& k, int l0, int to, Raw8<BF16> (&r)[K]) {
#pragma unroll
    for (int j = 0; j < K; ++j) r[j] = raw8_row<BF16, WHOLE>(row_at<BF16>(base, n, sn, min(l0 + j * k.tall, to - 1), sl), k.c, a.C);
}

template <bool BF16, bool WHOLE>
__global__ __launch_bounds__(kThreads) void norm_last_sums_kernel(NormArgs a) {
    __shared__ LastLds lds;
    const LastUnit u = last_unit(a, static_cast<int>(blockIdx.x) + a.first);
    const int to = min(u.len, u.from + a.piece);
    const Lane k = lane_of<WHOLE>(a, static_cast<int>(blockIdx.y));
    double s[8] = {}, q[8] = {};
    if (k.c < a.C && u.from + k.l0 < to) {
        double shift[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) shift[e] = load_elem<BF16>(row_at<BF16>(a.x, u.n, a.x_sn, 0, 0), div31(min(k.c + e, a.C - 1), a.by_per) * a.per);
        const auto add = [&](const Raw8<BF16>& raw) {
            float v[8];
            floats_of(raw, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const double d = static_cast<double>(v[e]) - shift[e];
                s[e] += d;
                q[e] = fma(d, d, q[e]);
            }
        };
        int l0 = u.from + k.l0;
        for (int end = u.from + k.tall * kAhead; end <= to; end += k.tall * kAhead, l0 += k.tall * kAhead) {  // all lanes have all of them
            Raw8<BF16> raw[kAhead];
            load_last<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sl, k, l0, to, raw);
#pragma unroll
            for (int j = 0; j < kAhead; ++j) add(raw[j]);
        }
#pragma unroll 1
        for (; l0 < to; l0 += k.tall) {
            Raw8<BF16> raw[1];
            load_last<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sl, k, l0, to, raw);
            add(raw[0]);
        }
    }
    channels_out<WHOLE>(a, k, s, q, a.part + 2L * u.unit * a.C, lds);
}

// Sums of the pieces of a sample's channels, for one workgroup a sample and group: of its channels together, and (backward) of each.
// A lane has one channel at a time and every share-th piece.
__device__ __forceinline__ void join_pieces(const NormArgs& a, int n, int c0, double* channels, double& s, double& q, double (*lds)[2]) {
    const int tid = static_cast<int>(threadIdx.x), wide = min(a.per, kJoinThreads), shares = kJoinThreads / wide, share = tid / wide;
    s = q = 0.0;
    for (int c1 = 0; c1 < a.per; c1 += wide) {
        const int c = c1 + tid - share * wide;
        double cs = 0.0, cq = 0.0;
        if (share < shares && c < a.per) {
            const double* part = a.part + 2L * (static_cast<long>(n) * a.pieces * a.C + c0 + c);
#pragma unroll 12
            for (int p = share; p < a.pieces; p += shares) {
                cs += part[2L * p * a.C];
                cq += part[2L * p * a.C + 1];
            }
        }
        if (channels) {
            __syncthreads();
            lds[tid][0] = cs;
            lds[tid][1] = cq;
            __syncthreads();
            if (share == 0 && c < a.per) {
                for (int i = 1; i < shares; ++i) {
                    cs += lds[tid + i * wide][0];
                    cq += lds[tid + i * wide][1];
                }
                channels[2L * (static_cast<long>(n) * a.C + c0 + c)] = cs;
                channels[2L * (static_cast<long>(n) * a.C + c0 + c) + 1] = cq;
                const double w = weight_of(a, c0 + c);
                s = fma(w, cs, s);
                q = fma(w, cq, q);
            }
        } else {
            s += cs;
            q += cq;
        }
    }
}

template <bool BF16>
__global__ __launch_bounds__(kJoinThreads) void norm_last_stats_kernel(NormArgs a) {
    __shared__ double lds[2 * kJoinThreads / kSeqWave];
    const int group = static_cast<int>(blockIdx.x) + a.first, n = div31(group, a.by_G), c0 = (group - n * a.G) * a.per;
    const int len = seq_length(a.lengths, n, a.L);
    const float first = load_elem<BF16>(row_at<BF16>(a.x, n, a.x_sn, 0, 0), c0);
    double s, q, mean, rstd;
    join_pieces(a, n, c0, nullptr, s, q, nullptr);
    block_sums<kJoinThreads>(s, q, lds);
    stats_of(s, q, static_cast<double>(len) * a.per, len > 0 ? first : 0.f, a.eps, mean, rstd);
    keep_stats(a, group, mean, rstd);
}

// Backward: the channels' sums to sums[n][c], the group's over m to groups[n][g].
__global__ __launch_bounds__(kJoinThreads) void norm_last_join_kernel(NormArgs a, double* sums, double* groups) {
    __shared__ double lds[2 * kJoinThreads / kSeqWave], all[kJoinThreads][2];
    const int group = static_cast<int>(blockIdx.x) + a.first, n = div31(group, a.by_G), c0 = (group - n * a.G) * a.per;
    const int len = seq_length(a.lengths, n, a.L);
    double s, q;
    join_pieces(a, n, c0, sums, s, q, all);
    block_sums<kJoinThreads>(s, q, lds);
    const double over = len > 0 ? 1.0 / (static_cast<double>(len) * a.per) : 0.0;
    if (threadIdx.x == 0) {
        groups[2L * group] = s * over;
        groups[2L * group + 1] = q * over;
    }
}

// statistics and parameters of a lane's channels
__device__ __forceinline__ void channels_of(const NormArgs& a, int c, const Groups& g, Channel (&r)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int at = min(c + e, a.C - 1);
        r[e] = channel_of(mean_of(a.stats[2 * g.g[e]], a.stats[2 * g.g[e] + 1]), weight_of(a, at), bias_of(a, at));
    }
}

template <bool BF16, int ACT, bool WHOLE>
__global__ __launch_bounds__(kThreads) void norm_last_apply_kernel(NormArgs a) {
    const LastUnit u = last_unit(a, static_cast<int>(blockIdx.x) + a.first);
    const int to = min(a.L, u.from + a.piece);
    const Lane k = lane_of<WHOLE>(a, static_cast<int>(blockIdx.y));
    if (k.c >= a.C || u.from + k.l0 >= to) return;
    Raw8<BF16> raw[kAhead];
    load_last<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sl, k, u.from + k.l0, to, raw);
    Channel ch[8];
    channels_of(a, k.c, groups_of(a, u.n, k.c), ch);
    const auto put = [&](const Raw8<BF16>& r, int l) {
        float v[8];
        floats_of(r, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float y = act_of<ACT>(fmaf(v[e] - ch[e].hi, ch[e].a, ch[e].b));
            v[e] = l < u.len ? y : 0.f;
        }
        vector_store8<BF16, WHOLE>(row_at<BF16>(a.y, u.n, a.y_sn, l, a.y_sl), k.c, a.C, v);
    };
    const int step = k.tall * kAhead;
    for (int l0 = u.from + k.l0, end = u.from + step;; end += step) {
        if (end <= to) {  // all lanes have all of them
#pragma unroll
            for (int j = 0; j < kAhead; ++j) put(raw[j], l0 + j * k.tall);
        } else {
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (l0 + j * k.tall < to) put(raw[j], l0 + j * k.tall);
        }
        l0 += step;
        if (l0 >= to) break;
        load_last<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sl, k, l0, to, raw);
    }
}

template <bool BF16, int ACT, bool WHOLE>
__global__ __launch_bounds__(kThreads, 4) void norm_last_back_sums_kernel(NormArgs a) {
    __shared__ LastLds lds;
    constexpr int K = 2;
    const LastUnit u = last_unit(a, static_cast<int>(blockIdx.x) + a.first);
    const int to = min(u.len, u.from + a.piece);
    const Lane k = lane_of<WHOLE>(a, static_cast<int>(blockIdx.y));
    double s[8] = {}, q[8] = {};
    if (k.c < a.C && u.from + k.l0 < to) {
        const Groups of = groups_of(a, u.n, k.c);
        Channel ch[8];
        channels_of(a, k.c, of, ch);
        const auto add = [&](const Raw8<BF16>& xr, const Raw8<BF16>& gr, float (&s8)[8], float (&q8)[8]) {
            float x[8], g[8], t[8];
            floats_of(xr, x);
            floats_of(gr, g);
            back8<ACT, 1>(a, x, ch, u.n, k.c, t, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s8[e] += g[e];
                q8[e] = fmaf(g[e], t[e], q8[e]);
            }
        };
        const auto flush = [&](const float (&s8)[8], const float (&q8)[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s[e] += static_cast<double>(s8[e]);
                q[e] += static_cast<double>(q8[e]);
            }
        };
        int l0 = u.from + k.l0;
        for (int end = u.from + k.tall * K; end <= to; end += k.tall * K, l0 += k.tall * K) {  // all lanes have all of them
            Raw8<BF16> xr[K], gr[K];
            load_last<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sl, k, l0, to, xr);
            load_last<BF16, WHOLE>(a, a.dy, u.n, a.dy_sn, a.dy_sl, k, l0, to, gr);
            float s8[8] = {}, q8[8] = {};
#pragma unroll
            for (int j = 0; j < K; ++j) add(xr[j], gr[j], s8, q8);
            flush(s8, q8);
        }
#pragma unroll 1
        for (; l0 < to; l0 += k.tall) {
            Raw8<BF16> xr[1], gr[1];
            load_last<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sl, k, l0, to, xr);
            load_last<BF16, WHOLE>(a, a.dy, u.n, a.dy_sn, a.dy_sl, k, l0, to, gr);
            float s8[8] = {}, q8[8] = {};
            add(xr[0], gr[0], s8, q8);
            flush(s8, q8);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            q[e] = with_h(q[e], s[e], a.stats[2 * of.g[e]], a.stats[2 * of.g[e] + 1]);
        }
    }
    channels_out<WHOLE>(a, k, s, q, a.part + 2L * u.unit * a.C, lds);
}

template <bool BF16, int ACT, bool WHOLE>
__global__ __launch_bounds__(kThreads) void norm_last_back_kernel(NormArgs a, const double* sums, const double* groups) {
    constexpr int K = 2;
    if (took_channels(a, sums, 1)) return;
    const LastUnit u = last_unit(a, static_cast<int>(blockIdx.x) - a.extra + a.first);
    const int to = min(a.L, u.from + a.piece);
    const Lane k = lane_of<WHOLE>(a, static_cast<int>(blockIdx.y));
    if (k.c >= a.C || u.from + k.l0 >= to) return;
    Raw8<BF16> xr[K], gr[K];
    load_last<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sl, k, u.from + k.l0, to, xr);
    load_last<BF16, WHOLE>(a, a.dy, u.n, a.dy_sn, a.dy_sl, k, u.from + k.l0, to, gr);
    const Groups of = groups_of(a, u.n, k.c);
    Channel ch[8];
    channels_of(a, k.c, of, ch);
    Back back[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        back[e] = back_const(mean_of(a.stats[2 * of.g[e]], a.stats[2 * of.g[e] + 1]), groups[2 * of.g[e]], groups[2 * of.g[e] + 1]);
    }
    const auto put = [&](const Raw8<BF16>& xr1, const Raw8<BF16>& gr1, int l) {
        float x[8], g[8], t[8];
        floats_of(xr1, x);
        floats_of(gr1, g);
        back8<ACT, 1>(a, x, ch, u.n, k.c, t, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = l < u.len ? fmaf(g[e], ch[e].a, fmaf(t[e], back[e].q, back[e].s)) : 0.f;
        vector_store8<BF16, WHOLE>(row_at<BF16>(a.dx, u.n, a.dx_sn, l, a.dx_sl), k.c, a.C, x);
    };
    const int step = k.tall * K;
    for (int l0 = u.from + k.l0, end = u.from + step;; end += step) {
        if (end <= to) {  // all lanes have all of them
#pragma unroll
            for (int j = 0; j < K; ++j) put(xr[j], gr[j], l0 + j * k.tall);
        } else {
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (l0 + j * k.tall < to) put(xr[j], gr[j], l0 + j * k.tall);
        }
        l0 += step;
        if (l0 >= to) break;
        load_last<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sl, k, l0, to, xr);
        load_last<BF16, WHOLE>(a, a.dy, u.n, a.dy_sn, a.dy_sl, k, l0, to, gr);
    }
}

// ---- channels contiguous, a workgroup a group ---------------------------------------------------------------------------------
// A lane has 8 neighbouring channels of the group at K positions, tall apart, in registers.
template <bool WHOLE>
__device__ __forceinline__ Lane group_lane(const NormArgs& a, int threads) {
    Lane r;
    r.vecs = (a.per + 7) >> 3;
    r.tall = threads / r.vecs;
    r.l0 = static_cast<int>(threadIdx.x) / r.vecs;
    r.c = r.l0 < r.tall ? vector_at<WHOLE>(static_cast<int>(threadIdx.x) - r.l0 * r.vecs, a.per) : a.per;  // within the group
    r.fresh = r.l0 < r.tall ? 8 * (static_cast<int>(threadIdx.x) - r.l0 * r.vecs) - r.c : 8;
    return r;
}
// K positions' vectors, of a row that is the group's channels at one position
template <bool BF16, bool WHOLE, int K>
__device__ __forceinline__ void load_group(const NormArgs& a, const void* base, int n, long sn, long sl, int c0, const Lane& k, Raw8<BF16> (&r)[K]) {
    using T = typename RowElem<BF16>::type;
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const T* row = static_cast<const T*>(base) + n * sn + min(k.l0 + j * k.tall, a.L - 1) * sl + c0;
        r[j] = raw8_row<BF16, WHOLE>(row, min(k.c, vector_at<WHOLE>(k.vecs - 1, a.per)), a.per);  // (a lane that has no channels reads the last)
    }
}

template <bool BF16, int ACT, bool WHOLE, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_last_one_kernel(NormArgs a) {
    using T = typename RowElem<BF16>::type;
    __shared__ double lds[2 * THREADS / kSeqWave];
    const Unit u = unit_of(a, static_cast<int>(blockIdx.x) + a.first);
    const Lane k = group_lane<WHOLE>(a, THREADS);
    Raw8<BF16> raw[kAhead];
    load_group<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sl, u.c0, k, raw);
    const float first = load_elem<BF16>(row_at<BF16>(a.x, u.n, a.x_sn, 0, 0), u.c0);
    const double shift = u.len > 0 ? first : 0.f;
    float w[8], b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int c = u.c0 + min(k.c + e, a.per - 1);
        w[e] = weight_of(a, c);
        b[e] = bias_of(a, c);
    }
    double s = 0.0, q = 0.0, mean, rstd;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        if (k.l0 + j * k.tall >= u.len || k.c >= a.per) break;
        float v[8];
        floats_of(raw[j], v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double d = WHOLE || (e >= k.fresh && k.c + e < a.per) ? static_cast<double>(v[e]) - shift : 0.0;
            s += d;
            q = fma(d, d, q);
        }
    }
    block_sums<THREADS>(s, q, lds);
    stats_of(s, q, static_cast<double>(u.len) * a.per, shift, a.eps, mean, rstd);
    keep_stats(a, u.group, mean, rstd);
    const Mean m = mean_of(mean, rstd);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
        const int l = k.l0 + j * k.tall;
        if (l >= a.L || k.c >= a.per) break;
        float v[8];
        floats_of(raw[j], v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const Channel ch = channel_of(m, w[e], b[e]);
            const float y = act_of<ACT>(fmaf(v[e] - ch.hi, ch.a, ch.b));
            v[e] = l < u.len ? y : 0.f;
        }
        vector_store8<BF16, WHOLE>(static_cast<T*>(a.y) + u.n * a.y_sn + l * a.y_sl + u.c0, k.c, a.per, v);
    }
}

template <bool BF16, int ACT, bool WHOLE, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_last_back_one_kernel(NormArgs a) {
    using T = typename RowElem<BF16>::type;
    constexpr int K = kAheadBack<BF16>;
    __shared__ double lds[2 * THREADS / kSeqWave];
    __shared__ double all[THREADS][8 + 1];
    const Unit u = unit_of(a, static_cast<int>(blockIdx.x) + a.first);
    const int tid = static_cast<int>(threadIdx.x);
    const Lane k = group_lane<WHOLE>(a, THREADS);
    Raw8<BF16> xr[K], gr[K];
    load_group<BF16, WHOLE>(a, a.x, u.n, a.x_sn, a.x_sl, u.c0, k, xr);
    load_group<BF16, WHOLE>(a, a.dy, u.n, a.dy_sn, a.dy_sl, u.c0, k, gr);
    const double mean = a.stats[2L * u.group], rstd = a.stats[2L * u.group + 1];
    const Mean m = mean_of(mean, rstd);
    Channel ch[8];
    float w[8], s8[8] = {}, q8[8] = {};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int c = u.c0 + min(k.c + e, a.per - 1);
        w[e] = weight_of(a, c);
        ch[e] = channel_of(m, w[e], bias_of(a, c));
    }
#pragma unroll
    for (int j = 0; j < K; ++j) {
        if (k.l0 + j * k.tall >= u.len || k.c >= a.per) break;
        float x[8], dy[8], t[8];
        floats_of(xr[j], x);
        floats_of(gr[j], dy);
        back8<ACT, 1>(a, x, ch, u.n, u.c0 + k.c, t, dy);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool counts = WHOLE || (e >= k.fresh && k.c + e < a.per);
            s8[e] += counts ? dy[e] : 0.f;
            q8[e] = counts ? fmaf(dy[e], t[e], q8[e]) : 0.f;
        }
    }
    double s = 0.0, q = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        s = fma(static_cast<double>(w[e]), static_cast<double>(s8[e]), s);
        q = fma(static_cast<double>(w[e]), static_cast<double>(q8[e]), q);
    }
    block_sums<THREADS>(s, q, lds);
    if (a.extra) {
        double* part = a.part + 2 * (static_cast<long>(u.n) * a.C + u.c0);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) all[tid][e] = h ? with_h(static_cast<double>(q8[e]), static_cast<double>(s8[e]), mean, rstd) : static_cast<double>(s8[e]);
            __syncthreads();
            for (int c = tid; c < a.per; c += THREADS) {
                double sum = 0.0;
                for (int t = 0; t < k.tall; ++t) sum += all[(c >> 3) + t * k.vecs][c - vector_at<WHOLE>(c >> 3, a.per)];
                part[2L * c + h] = u.len > 0 ? sum : 0.0;
            }
        }
    }
    const double over = u.len > 0 ? 1.0 / (static_cast<double>(u.len) * a.per) : 0.0;
    const Back back = back_const(m, s * over, with_h(q, s, mean, rstd) * over);
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const int l = k.l0 + j * k.tall;
        if (l >= a.L || k.c >= a.per) break;
        float x[8], dy[8], t[8];
        floats_of(xr[j], x);
        floats_of(gr[j], dy);
        back8<ACT, 1>(a, x, ch, u.n, u.c0 + k.c, t, dy);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = l < u.len ? fmaf(dy[e], ch[e].a, fmaf(t[e], back.q, back.s)) : 0.f;
        vector_store8<BF16, WHOLE>(static_cast<T*>(a.dx) + u.n * a.dx_sn + l * a.dx_sl + u.c0, k.c, a.per, x);
    }
}

// ---- host -----------------------------------------------------------------------------------------------------------
constexpr long kFill = 2048;   // workgroups that keep the chip busy: 8 a compute unit
constexpr int kMostPieces = 512;

int ceil_to(long n, int to) { return static_cast<int>((n + to - 1) / to * to); }

struct Plan {
    bool last;
    int one;   // threads of a workgroup that has a whole group, or 0
    int vecs, items, pieces, piece, rows_pieces, rows_piece, lanes, blocks;
    size_t part, sums, groups, bytes;
};
// `last`: channels contiguous
Plan plan_of(int N, int C, int L, int G, int dtype, bool last, bool back) {
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
        // A workgroup for each group, where its lanes hold it, as below (a lane has four positions, two for floats backward): 16 groups of 64
        // vectors forward 3.8 us for 11.7, of 1024 4.8 for 12.7; 4096 of 64 7.6 for 27.  Large workgroups do not pay where groups are many:
        // a group's channels are a part of a line, and what the next group needs of it has left the cache (1024 groups of 4096 vectors, 32
        // bytes a position, 70 us for 47; backward of 2048 64 for 48).
        const int K = back && dtype == CONV1D_FP32 ? 2 : kAhead, per = (C / G + 7) / 8;
        const bool many = groups >= kFill / 2;
        for (int threads : {kSeqWave, kThreads, 2 * kThreads, 4 * kThreads}) {
            if (threads == kSeqWave && !many) continue;
            if (threads == 2 * kThreads && many && (back || C / G * (dtype == CONV1D_BF16 ? 2 : 4) < 64)) continue;
            if (threads == 4 * kThreads && (many || back)) continue;
            if (C / G < 8 && static_cast<long>(N) * C * L > 1 << 16) continue;  // (less than a vector: the general way shares lines better)
            if (!p.one && per <= threads && L <= static_cast<long>(K) * (threads / per)) p.one = threads;
        }
        if (p.one > kThreads && groups < (back ? 128 : 32)) p.one = 0;
        if (p.one) {
            p.pieces = 1;
            p.part = take(back ? static_cast<size_t>(N) * C : 0);
            p.bytes = at;
            return p;
        }
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
        // A workgroup for each group: four vectors a lane (two of x and two of dy for floats backward), one wave where groups are small and
        // many.  Two launches, which share a group out, take over where few groups leave the chip idle: 16 groups of 4096 vectors forward
        // 8.4 and 6.4 us, of 2048 backward 10.5 and 7.0 (256 groups: 11.7 and 15.2; 1024 groups of 512: 10.9 and 13.6).
        const int most = back && dtype == CONV1D_FP32 ? 2 : kAhead;
        const bool few = groups < (back ? 128 : 32);
        if (p.items <= most * kSeqWave && groups >= kFill / 2) p.one = kSeqWave;
        else if (p.items <= most * kThreads && (!back || !few || p.items <= 512)) p.one = kThreads;
        else if (p.items <= most * 2 * kThreads && !(back && few)) p.one = 2 * kThreads;
        else if (p.items <= most * 4 * kThreads && !back && !few) p.one = 4 * kThreads;
        if (p.one) {
            p.pieces = 1;
            p.part = take(back ? static_cast<size_t>(N) * C : 0);
            p.bytes = at;
            return p;
        }
        long pieces = kFill / groups;
        pieces = pieces < 1 ? 1 : pieces > kMostPieces ? kMostPieces : pieces;
        // (in whole steps of a workgroup's loads where that leaves enough workgroups)
        const int step = kThreads * (back && dtype == CONV1D_FP32 ? 2 : kAhead);
        p.piece = ceil_to((p.items + pieces - 1) / pieces, kThreads);
        if (2 * p.piece > step) p.piece = ceil_to(p.piece, step);
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
    a.by_per = make_div31(a.per);
    a.by_rows_pieces = make_div31(plan.rows_pieces ? plan.rows_pieces : 1);
    return a;
}

// All units of a launch, in pieces that a grid of `blocks` rows may have; with `extra` workgroups, shared out over the rows, before them in the
// first.  (At most 2^18 of them with one row, and with 2^20 channels 512 in each of 512 rows of 2^14: some are always left for the units.)
template <typename... More>
hipError_t launch_units(void (*kern)(NormArgs, More...), NormArgs& a, int threads, long units, int blocks, int extra, hipStream_t st, More... more) {
    a.extra = cdiv(extra, blocks);
    const long most = kSeqMostThreads / threads / blocks - a.extra;
    for (long u = 0; u < units; u += most, a.extra = 0) {
        a.first = static_cast<int>(u);
        const long some = units - u < most ? units - u : most;
        const hipError_t e = launch_kernel(kern, dim3(static_cast<unsigned>(some + a.extra), static_cast<unsigned>(blocks)), dim3(threads), 0, st, a, more...);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <bool BF16, int ACT, bool WHOLE>
hipError_t forward(NormArgs& a, const Plan& plan, hipStream_t st) {
    const long groups = static_cast<long>(a.N) * a.G;
    const auto one = [&](void (*rows)(NormArgs), void (*last)(NormArgs)) { return launch_units(plan.last ? last : rows, a, plan.one, groups, 1, 0, st); };
    switch (plan.one) {
        case kSeqWave: return one(norm_one_kernel<BF16, ACT, WHOLE, kSeqWave>, norm_last_one_kernel<BF16, ACT, WHOLE, kSeqWave>);
        case kThreads: return one(norm_one_kernel<BF16, ACT, WHOLE, kThreads>, norm_last_one_kernel<BF16, ACT, WHOLE, kThreads>);
        case 2 * kThreads: return one(norm_one_kernel<BF16, ACT, WHOLE, 2 * kThreads>, norm_last_one_kernel<BF16, ACT, WHOLE, 2 * kThreads>);
        case 4 * kThreads: return one(norm_one_kernel<BF16, ACT, WHOLE, 4 * kThreads>, norm_last_one_kernel<BF16, ACT, WHOLE, 4 * kThreads>);
        default: break;
    }
    if (!plan.last) {
        const hipError_t e = launch_units(norm_sums_kernel<BF16, WHOLE>, a, kThreads, groups * plan.pieces, 1, 0, st);
        return e == hipSuccess ? launch_units(norm_apply_kernel<BF16, ACT, WHOLE>, a, kThreads, groups * plan.pieces, 1, 0, st) : e;
    }
    const long units = static_cast<long>(a.N) * plan.pieces;
    hipError_t e = launch_units(norm_last_sums_kernel<BF16, WHOLE>, a, kThreads, units, plan.blocks, 0, st);
    if (e == hipSuccess) e = launch_units(norm_last_stats_kernel<BF16>, a, kJoinThreads, groups, 1, 0, st);
    if (e == hipSuccess) e = launch_units(norm_last_apply_kernel<BF16, ACT, WHOLE>, a, kThreads, units, plan.blocks, 0, st);
    return e;
}

template <bool BF16, int ACT, bool WHOLE>
hipError_t backward(NormArgs& a, const Plan& plan, double* sums, double* groups, hipStream_t st) {
    const long many = static_cast<long>(a.N) * a.G;
    const int channels = a.dweight || a.dbias ? cdiv(a.C, kThreads / kSeqWave) : 0;
    if (plan.one) {
        // (extra: the kernel's own, whether sums of channels are wanted)
        hipError_t e = hipSuccess;
        const long most = kSeqMostThreads / plan.one;
        a.extra = channels;
        for (long u = 0; u < many && e == hipSuccess; u += most) {
            a.first = static_cast<int>(u);
            void (*kern)(NormArgs) = plan.one == kSeqWave   ? (plan.last ? norm_last_back_one_kernel<BF16, ACT, WHOLE, kSeqWave> : norm_back_one_kernel<BF16, ACT, WHOLE, kSeqWave>)
                                     : plan.one == kThreads ? (plan.last ? norm_last_back_one_kernel<BF16, ACT, WHOLE, kThreads> : norm_back_one_kernel<BF16, ACT, WHOLE, kThreads>)
                                     : plan.last            ? norm_last_back_one_kernel<BF16, ACT, WHOLE, 2 * kThreads>
                                                            : norm_back_one_kernel<BF16, ACT, WHOLE, 2 * kThreads>;
            e = launch_kernel(kern, dim3(static_cast<unsigned>(many - u < most ? many - u : most)), dim3(plan.one), 0, st, a);
        }
        if (e == hipSuccess && channels) e = launch_kernel(norm_channels_kernel, dim3(channels), dim3(kThreads), 0, st, a);
        return e;
    }
    if (!plan.last) {
        const long teams = kThreads / plan.lanes, rows = static_cast<long>(a.N) * a.C * plan.rows_pieces;
        const hipError_t e = launch_units(norm_back_sums_kernel<BF16, ACT, WHOLE>, a, kThreads, cdiv(rows, teams), 1, 0, st);
        return e == hipSuccess ? launch_units(norm_back_kernel<BF16, ACT, WHOLE>, a, kThreads, many * plan.pieces, 1, channels, st) : e;
    }
    const long units = static_cast<long>(a.N) * plan.pieces;
    hipError_t e = launch_units(norm_last_back_sums_kernel<BF16, ACT, WHOLE>, a, kThreads, units, plan.blocks, 0, st);
    if (e == hipSuccess) e = launch_units(norm_last_join_kernel, a, kJoinThreads, many, 1, 0, st, sums, groups);
    if (e == hipSuccess)
        e = launch_units(norm_last_back_kernel<BF16, ACT, WHOLE>, a, kThreads, units, plan.blocks, channels, st, static_cast<const double*>(sums),
                         static_cast<const double*>(groups));
    return e;
}

template <bool BF16, bool WHOLE>
hipError_t forward(NormArgs& a, const Plan& plan, int act, hipStream_t st) {
    return act == kRelu   ? forward<BF16, kRelu, WHOLE>(a, plan, st)
           : act == kSilu ? forward<BF16, kSilu, WHOLE>(a, plan, st)
                          : forward<BF16, kNone, WHOLE>(a, plan, st);
}
template <bool BF16, bool WHOLE>
hipError_t backward(NormArgs& a, const Plan& plan, int act, double* sums, double* groups, hipStream_t st) {
    return act == kRelu   ? backward<BF16, kRelu, WHOLE>(a, plan, sums, groups, st)
           : act == kSilu ? backward<BF16, kSilu, WHOLE>(a, plan, sums, groups, st)
                          : backward<BF16, kNone, WHOLE>(a, plan, sums, groups, st);
}

int act_flag(int flags) { return flags & CONV1D_NORM_RELU ? kRelu : flags & CONV1D_NORM_SILU ? kSilu : kNone; }
// rows of whole vectors, all of which count (channels contiguous: positions that do not are passed over anyway)
bool is_whole(const conv1d_norm_t* p, const Plan& plan) {
    if (plan.last) return (plan.one ? p->C / p->G : p->C) % 8 == 0;
    return p->L % 8 == 0 && !p->lengths;
}
int status_of(hipError_t e) { return e == hipSuccess ? CONV1D_OK : CONV1D_EHIP; }

size_t workspace_of(int N, int C, int L, int G, int dtype, long x_sc, long x_sl, bool back) {
    if (N < 1 || C < 1 || L < 1 || G < 1 || C % G || !sizes_ok(N, C, L, G) || (dtype != CONV1D_FP32 && dtype != CONV1D_BF16)) return 0;
    return plan_of(N, C, L, G, dtype, order_of(C, L, x_sc, x_sl) == 2, back).bytes;
}

}  // namespace
}  // namespace conv1d

using namespace conv1d;

extern "C" {

size_t conv1d_norm_fwd_workspace_bytes(int N, int C, int L, int G, int dtype, long x_sc, long x_sl) {
    return workspace_of(N, C, L, G, dtype, x_sc, x_sl, false);
}
size_t conv1d_norm_bwd_workspace_bytes(int N, int C, int L, int G, int dtype, long x_sc, long x_sl) {
    return workspace_of(N, C, L, G, dtype, x_sc, x_sl, true);
}

int conv1d_norm_fwd(const conv1d_norm_t* p, void* y, long y_sn, long y_sc, long y_sl, double* stats, void* workspace, size_t workspace_bytes, void* stream) {
    if (!shape_ok(p) || !y) return CONV1D_EINVAL;
    const size_t size = p->dtype == CONV1D_BF16 ? 2 : 4;
    const int order = order_of(p);
    if (!seq_aligned(y, size) || !seq_aligned(stats, 8) || !seq_aligned(workspace, 256) || !order || !fits(p, order, y_sc, y_sl)) return CONV1D_EINVAL;
    if (!sizes_ok(p->N, p->C, p->L, p->G)) return CONV1D_EUNSUPPORTED;
    const Plan plan = plan_of(p->N, p->C, p->L, p->G, p->dtype, order == 2, false);
    if (workspace_bytes < plan.bytes || (plan.bytes && !workspace)) return CONV1D_EWORKSPACE;
    NormArgs a = args_of(p, plan, workspace);
    a.y = y; a.y_sn = y_sn; a.y_sc = y_sc; a.y_sl = y_sl;
    a.stats = stats ? stats : plan.last && !plan.one ? reinterpret_cast<double*>(static_cast<char*>(workspace) + plan.groups) : nullptr;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int act = act_flag(p->flags);
    const bool whole = is_whole(p, plan);
    if (p->dtype == CONV1D_BF16) return status_of(whole ? forward<true, true>(a, plan, act, st) : forward<true, false>(a, plan, act, st));
    return status_of(whole ? forward<false, true>(a, plan, act, st) : forward<false, false>(a, plan, act, st));
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
    const Plan plan = plan_of(p->N, p->C, p->L, p->G, p->dtype, order == 2, true);
    if (workspace_bytes < plan.bytes || (plan.bytes && !workspace)) return CONV1D_EWORKSPACE;
    NormArgs a = args_of(p, plan, workspace);
    a.dy = dy; a.dy_sn = dy_sn; a.dy_sc = dy_sc; a.dy_sl = dy_sl;
    a.dx = dx; a.dx_sn = dx_sn; a.dx_sc = dx_sc; a.dx_sl = dx_sl;
    a.stats = const_cast<double*>(stats);
    a.dweight = dweight; a.dbias = dbias;
    char* ws = static_cast<char*>(workspace);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int act = act_flag(p->flags);
    double *sums = reinterpret_cast<double*>(ws + plan.sums), *groups = reinterpret_cast<double*>(ws + plan.groups);
    const bool whole = is_whole(p, plan);
    if (p->dtype == CONV1D_BF16) return status_of(whole ? backward<true, true>(a, plan, act, sums, groups, st) : backward<true, false>(a, plan, act, sums, groups, st));
    return status_of(whole ? backward<false, true>(a, plan, act, sums, groups, st) : backward<false, false>(a, plan, act, sums, groups, st));
}

}  // extern "C"
