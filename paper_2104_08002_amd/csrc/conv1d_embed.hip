// Embedding lookup with scaling, and its gradient by sorted tokens.
//   y[n][d][l] = scale table[tokens[n][l]][d],   dtable[v][d] = scale sum over (n, l) with tokens[n][l] = v of dy[n][d][l]
// Bound by memory.  Where positions are contiguous, tiles of positions and channels are turned in LDS: rows of the table are read
// and written along the channels, y and dy along the positions.
// The gradient adds the same positions in the same order in every run.  Few tokens: dy is multiplied with the truth values
// "position l has token v" on the matrix cores, straight from memory.  Many: the positions are sorted by their token (a stable radix
// sort, least digit first) while dy is turned into rows; each lane group adds a chunk of neighbouring rows in float and writes the
// runs that lie in its chunk; what of a run lies in several chunks is joined in 64 bits.
#include "conv1d_blocks.h"
#include "conv1d_split_f32.h"

namespace conv1d {
namespace {

constexpr int kThreads = 256;
constexpr long kFill = 2048;       // workgroups that keep the chip busy: 8 a compute unit
constexpr int kFewRows = 1024, kFewElements = 12288;  // rows of a table that LDS holds some channels of, and how much it holds

// ---- forward --------------------------------------------------------------------------------------------------------
struct LookArgs {
    const void *table, *tokens;
    const int* lengths;
    void* y;
    long tok_sn, y_sn, y_sd, y_sl;
    float scale;
    int wide, N, D, L, V;
    int tiles, blocks;      // of positions, of channels: tiles * blocks workgroups a sample
    long first;             // first workgroup or item of this launch
    int items, per_row;
    Div31 by_blocks, by_tiles, by_row, by_L;
};

// the token at position l of sample n; -1 for none: behind the sequence's end, or no row of the table
__device__ __forceinline__ int token_at(const void* tokens, int wide, long n, long tok_sn, int l, int len, int V) {
    if (l >= len) return -1;
    const long at = n * tok_sn + l;
    const long t = wide ? static_cast<const long*>(tokens)[at] : static_cast<const int*>(tokens)[at];
    return t >= 0 && t < V ? static_cast<int>(t) : -1;
}

constexpr int kTile = 8192;  // positions times channels of a tile: 16 or 32 KB

// A tile of kTile / DT positions and DT channels.  Two elements more than a row's positions: the eight channels that a lane writes, and
// those of its neighbours, begin in different banks.
template <bool BF16, int DT>
__global__ __launch_bounds__(kThreads) void embed_turn_kernel(LookArgs a) {
    using T = typename RowElem<BF16>::type;
    constexpr int P = kTile / DT, S = P + 2, NV = DT / 8;
    __shared__ T lds[DT * S];
    __shared__ int toks[P];
    const int unit = static_cast<int>(blockIdx.x) + static_cast<int>(a.first);
    const int nt = div31(unit, a.by_blocks), d0 = (unit - nt * a.blocks) * DT, n = div31(nt, a.by_tiles), l0 = (nt - n * a.tiles) * P;
    const int tid = static_cast<int>(threadIdx.x), len = seq_length(a.lengths, n, a.L), many = min(DT, a.D - d0);
    for (int p = tid; p < P; p += kThreads) toks[p] = token_at(a.tokens, a.wide, n, a.tok_sn, l0 + p, len, a.V);
    __syncthreads();
#pragma unroll 4
    for (int i = tid; i < P * NV; i += kThreads) {
        const int p = i / NV, d = 8 * (i % NV), tok = toks[p];
        if (d >= many) continue;
        float v[8];
        const int row = clampi(tok, 0, a.V - 1);  // (a row that is there: the load waits for no branch)
        row_load8<BF16>(static_cast<const T*>(a.table) + static_cast<long>(row) * a.D, d0 + d, a.D, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) store_elem<BF16>(lds, (d + e) * S + p, tok < 0 ? 0.f : v[e] * a.scale);
    }
    __syncthreads();
    T* y = static_cast<T*>(a.y) + n * a.y_sn;
#pragma unroll 4
    for (int i = tid; i < DT * (P / 8); i += kThreads) {
        const int d = i / (P / 8), p = 8 * (i % (P / 8));
        if (d >= many || l0 + p >= a.L) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = load_elem<BF16>(lds, d * S + p + e);
        row_store8<BF16>(y + (d0 + d) * a.y_sd, l0 + p, a.L, v);
    }
}

// Few tokens: the workgroup's channels of the whole table, scaled and rounded, lie in LDS (and a row of zeros for no token); a lane has
// 8 positions, whose tokens it keeps.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void embed_few_kernel(LookArgs a) {
    using T = typename RowElem<BF16>::type;
    extern __shared__ char dynamic[];
    T* lds = reinterpret_cast<T*>(dynamic);
    const int unit = static_cast<int>(blockIdx.x) + static_cast<int>(a.first);
    const int nt = div31(unit, a.by_blocks), d0 = (unit - nt * a.blocks) * a.per_row, n = div31(nt, a.by_tiles);
    const int l = ((nt - n * a.tiles) * kThreads + static_cast<int>(threadIdx.x)) * 8;
    const int len = seq_length(a.lengths, n, a.L), many = min(a.per_row, a.D - d0);
    int at[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int t = token_at(a.tokens, a.wide, n, a.tok_sn, l + e, len, a.V);
        at[e] = (t < 0 ? a.V : t) * many;
    }
    for (int i = static_cast<int>(threadIdx.x); i < (a.V + 1) * many; i += kThreads) {
        const int v = i / many;
        const float u = v < a.V ? load_elem<BF16>(a.table, static_cast<long>(v) * a.D + d0 + (i - v * many)) * a.scale : 0.f;
        store_elem<BF16>(lds, i, u);
    }
    __syncthreads();
    if (l >= a.L) return;
    T* y = static_cast<T*>(a.y) + n * a.y_sn + d0 * a.y_sd;
    typedef __attribute__((ext_vector_type(8), aligned(BF16 ? 2 : 4))) T vec8;
#pragma unroll 2
    for (int d = 0; d < many; ++d) {
        vec8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = lds[at[e] + d];
        T* row = y + d * a.y_sd + l;
        if (l + 8 <= a.L) {
            *reinterpret_cast<vec8*>(row) = v;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (l + e < a.L) row[e] = v[e];
        }
    }
}

// Channels next to each other: rows are copied.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void embed_copy_kernel(LookArgs a) {
    using T = typename RowElem<BF16>::type;
    const int item = static_cast<int>(blockIdx.x) * kThreads + static_cast<int>(threadIdx.x);
    if (item >= a.items) return;
    const int of = div31(item, a.by_row), d = 8 * (item - of * a.per_row);
    const int m = static_cast<int>(a.first) + of, n = div31(m, a.by_L), l = m - n * a.L;
    const int tok = token_at(a.tokens, a.wide, n, a.tok_sn, l, seq_length(a.lengths, n, a.L), a.V);
    float v[8];
    row_load8<BF16>(static_cast<const T*>(a.table) + static_cast<long>(max(tok, 0)) * a.D, d, a.D, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = tok < 0 ? 0.f : v[e] * a.scale;
    row_store8<BF16>(static_cast<T*>(a.y) + n * a.y_sn + l * a.y_sl, d, a.D, v);
}

// ---- backward, few tokens: a product with truth values ----------------------------------------------------------------------
// dtable[v][d] = sum over l of dy[d][l] [token l = v]: an A operand is 16 channels of 32 neighbouring positions as they lie in memory, a
// B operand the truth values of those positions for 16 tokens, exact in bfloat16; floats are taken as three bfloat16 numbers whose sum
// they are.  The matrix instruction cuts off what its additions lose, so that a step's products start from 0 and are added to the
// running sum by an ordinary addition.  A value that is not finite would reach every token (0 * NaN): where a sum is not finite, the
// wave goes through its positions again without such values, which are then added where they belong.
constexpr int kFewTokens = 1024;

struct FewArgs {
    const void *dy, *tokens;
    const int* lengths;
    float* part;           // [chunks][tokens and channels, both rounded up to 16]
    float* dtable;
    long tok_sn, dy_sn, dy_sd;
    float scale;
    int wide, N, D, L, V, Vp, Dp, vgroups, dgroups;
    int chunk, samples, per_sample, chunks;  // a chunk: positions of a sample, or all of some samples; chunks of a sample (or of those)
    Div31 by_vgroups, by_dgroups, by_sample;
};

typedef sp::u32x4 u32x4;
typedef sp::f32x4 f32x4;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;

// 8 positions' tokens in 16 bits, 0xffff for none
struct Tokens8 {
    unsigned t[4];
};
__device__ __forceinline__ Tokens8 tokens8(const FewArgs& a, long n, int l, int len) {
    unsigned u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const long at = n * a.tok_sn + min(l + e, a.L - 1);
        bool fine = l + e < len;
        if (a.wide) {
            const long t = static_cast<const long*>(a.tokens)[at];
            fine &= static_cast<unsigned long>(t) < static_cast<unsigned long>(a.V);
            u[e] = static_cast<unsigned>(t);
        } else {
            u[e] = static_cast<unsigned>(static_cast<const int*>(a.tokens)[at]);
            fine &= u[e] < static_cast<unsigned>(a.V);
        }
        u[e] = fine ? u[e] : 0xffffu;
    }
    Tokens8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.t[i] = u[2 * i] | (u[2 * i + 1] << 16);
    return r;
}
// bfloat16 1 where a token is v, 0 elsewhere
__device__ __forceinline__ u32x4 truth8(const Tokens8& k, int v) {
    const u16x2 vv = static_cast<u16x2>(static_cast<unsigned short>(v));
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const u16x2 off = __builtin_elementwise_min(__builtin_bit_cast(u16x2, k.t[i]) ^ vv, static_cast<u16x2>(static_cast<unsigned short>(1)));
        r[i] = __builtin_bit_cast(unsigned, static_cast<u16x2>(0x3f80 - off * static_cast<unsigned short>(0x3f80)));
    }
    return r;
}

// 8 positions of a channel as operands: one for bfloat16, three for float
template <bool BF16>
struct Parts {
    u32x4 p[BF16 ? 1 : 3];
};
template <bool BF16, bool FINITE>
__device__ __forceinline__ Parts<BF16> parts8(const void* row, int l, int len) {
    Parts<BF16> r;
    if constexpr (BF16 && !FINITE) {
        if (l + 8 <= len) {
            const seq_u16x8 v = *reinterpret_cast<const seq_u16x8*>(static_cast<const unsigned short*>(row) + l);
            r.p[0] = __builtin_bit_cast(u32x4, v);
            return r;
        }
    }
    float v[8];
    row_load8<BF16>(row, l, len, v);
    if constexpr (FINITE) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fabsf(v[e]) < INFINITY ? v[e] : 0.f;
    }
    if constexpr (BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r.p[0][i] = sp::pack_hi(v[2 * i], v[2 * i + 1]);
    } else {
        const sp::Split8 s = sp::split8(v);
        r.p[0] = s.l;
        r.p[1] = s.m;
        r.p[2] = s.h;
    }
    return r;
}

constexpr int kWaves = kThreads / kSeqWave;

// A wave's steps of 32 positions: every kWaves-th of its chunk's.
struct Steps {
    int n0, from, to, per, all;  // first sample, positions of each, steps of a sample and of all
};
__device__ __forceinline__ Steps steps_of(const FewArgs& a, int chunk) {
    Steps r;
    const int of = div31(chunk, a.by_sample);
    r.n0 = of * a.samples;
    r.from = (chunk - of * a.per_sample) * a.chunk;
    r.to = min(a.L, r.from + a.chunk);
    r.per = (r.to - r.from + 31) >> 5;
    r.all = r.per * min(a.samples, a.N - r.n0);
    return r;
}

template <bool BF16, bool FINITE, int VB, int DB>
__device__ __forceinline__ void few_sums(const FewArgs& a, const Steps& t, int v0, int d0, f32x4 (&acc)[VB][DB]) {
    using T = typename RowElem<BF16>::type;
    const int lane = static_cast<int>(threadIdx.x) & (kSeqWave - 1);
#pragma unroll
    for (int v = 0; v < VB; ++v)
#pragma unroll
        for (int d = 0; d < DB; ++d) acc[v][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    int i = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kSeqWave), n = t.n0;
    const T* rows[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) rows[d] = static_cast<const T*>(a.dy) + n * a.dy_sn + min(d0 + 16 * d + (lane & 15), a.D - 1) * a.dy_sd;
    for (int before = 0; i < t.all; i += kWaves) {
        while (i - before >= t.per) {
            before += t.per;
            ++n;
#pragma unroll
            for (int d = 0; d < DB; ++d) rows[d] += a.dy_sn;
        }
        const int len = min(t.to, seq_length(a.lengths, n, a.L)), l = t.from + 32 * (i - before) + 8 * (lane >> 4);
        Parts<BF16> x[DB];
#pragma unroll
        for (int d = 0; d < DB; ++d) x[d] = parts8<BF16, FINITE>(rows[d], l, len);
        const Tokens8 k = tokens8(a, n, l, len);
#pragma unroll
        for (int v = 0; v < VB; ++v) {
            const u32x4 one = truth8(k, v0 + 16 * v + (lane & 15));
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                f32x4 s = sp::mfma(x[d].p[0], one, f32x4{0.f, 0.f, 0.f, 0.f});
                if constexpr (!BF16) {
                    s = sp::mfma(x[d].p[1], one, s);
                    s = sp::mfma(x[d].p[2], one, s);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[v][d][e] += s[e];
            }
        }
    }
}

template <bool BF16, int VB, int DB>
__global__ __launch_bounds__(kThreads) void embed_few_sums_kernel(FewArgs a) {
    using T = typename RowElem<BF16>::type;
    __shared__ float lds[VB * 16][DB * 16 + 4];
    const int unit = static_cast<int>(blockIdx.x), cd = div31(unit, a.by_vgroups), v0 = (unit - cd * a.vgroups) * (16 * VB);
    const int chunk = div31(cd, a.by_dgroups), d0 = (cd - chunk * a.dgroups) * (16 * DB);
    const Steps t = steps_of(a, chunk);
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kSeqWave - 1), wave = tid / kSeqWave;
    f32x4 acc[VB][DB];
    few_sums<BF16, false, VB, DB>(a, t, v0, d0, acc);
    bool fine = true;
#pragma unroll
    for (int v = 0; v < VB; ++v)
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) fine &= fabsf(acc[v][d][i]) < INFINITY;
    const bool again = !wave_all(fine);
    if (again) few_sums<BF16, true, VB, DB>(a, t, v0, d0, acc);
    for (int w = 0; w < kWaves; ++w) {
        if (w == wave) {
#pragma unroll
            for (int v = 0; v < VB; ++v)
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    float* at = &lds[16 * v + (lane & 15)][16 * d + 4 * (lane >> 4)];
#pragma unroll
                    for (int i = 0; i < 4; ++i) at[i] = w ? at[i] + acc[v][d][i] : acc[v][d][i];
                }
        }
        __syncthreads();
    }
    if (again) {  // a number added to one that is not finite, or two such numbers: any order gives the same
        for (int i = wave; i < t.all; i += kWaves) {
            const int n = t.n0 + i / t.per, l0 = t.from + 32 * (i % t.per), len = min(t.to, seq_length(a.lengths, n, a.L));
            for (int j = lane; j < 32 * 16 * DB; j += kSeqWave) {
                const int l = l0 + (j & 31), d = d0 + (j >> 5);
                if (l >= len || d >= a.D) continue;
                const int tok = token_at(a.tokens, a.wide, n, a.tok_sn, l, len, a.V);
                const float v = load_elem<BF16>(static_cast<const T*>(a.dy) + n * a.dy_sn + d * a.dy_sd, l);
                if (tok >= v0 && tok < v0 + 16 * VB && !(fabsf(v) < INFINITY)) lds_add(&lds[tok - v0][d - d0], v);
            }
        }
    }
    __syncthreads();
    float* part = a.part + static_cast<long>(chunk) * a.Vp * a.Dp;
    for (int i = tid; i < VB * 16 * DB * 4; i += kThreads) {
        const int v = i / (DB * 4), d = 4 * (i % (DB * 4));
        if (v0 + v < a.Vp && d0 + d < a.Dp)
            *reinterpret_cast<f32x4*>(part + static_cast<long>(v0 + v) * a.Dp + d0 + d) = *reinterpret_cast<const f32x4*>(&lds[v][d]);
    }
}

// 16 neighbouring numbers a workgroup, each the sum of 64 lanes' shares of the chunks
constexpr int kFewJoin = 1024;
__global__ __launch_bounds__(kFewJoin) void embed_few_join_kernel(FewArgs a) {
    __shared__ double lds[kFewJoin / 16][17];
    const int tid = static_cast<int>(threadIdx.x), o = tid & 15, slice = tid >> 4;
    const long at = 16L * blockIdx.x + o;  // of part
    double s = 0.0;
#pragma unroll 4
    for (int c = slice; c < a.chunks; c += kFewJoin / 16) s += a.part[static_cast<long>(c) * a.Vp * a.Dp + at];
    lds[slice][o] = s;
    __syncthreads();
    for (int half = kFewJoin / 32; half > 0; half >>= 1) {
        if (slice < half) lds[slice][o] += lds[slice + half][o];
        __syncthreads();
    }
    const int v = static_cast<int>(at / a.Dp), d = static_cast<int>(at - static_cast<long>(v) * a.Dp);
    if (slice == 0 && v < a.V && d < a.D) a.dtable[static_cast<long>(v) * a.D + d] = static_cast<float>(lds[0][o]) * a.scale;
}

// ---- backward, many tokens: the positions in the order of their tokens ---------------------------------------------------------
// Keys are tokens, V for no token: those come last.  A pass of the sort takes up to 8 bits.  The first launch counts the digits of each
// tile of keys; each pass's launch finds where its tile's keys go (from the counts of all tiles, which are few, or made into places by
// a launch between), puts them there in their order, and counts the next pass's digits where they went.  These launches wait for
// memory most of the time: their other workgroups turn dy into rows and clear the gradient meanwhile.
constexpr int kBins = 256;
constexpr int kSort = 1024, kSortWaves = kSort / kSeqWave;
constexpr int kKeys = 4;          // most keys of a lane
constexpr int kFewTiles = 256;    // up to here every workgroup adds up the counts of all tiles itself

struct SortArgs {
    const void *tokens, *dy;
    const int* lengths;
    long tok_sn, dy_sn, dy_sd;
    int wide, N, D, L, V, M;
    Div31 by_L;
    int *keys[2], *pos[2];        // pass p writes to [p & 1] and reads from the other; the first reads the tokens
    int *counts, *totals;         // [passes][tiles][kBins], [kBins]
    int *owners;                  // [0]: how many runs cross chunks (cleared here), then their chunks
    void* rows;                   // [M][8 * per_row]: dy's columns
    float* dtable;
    long zeros;                   // elements of dtable
    int pass, passes, bits, tiles, per_lane, before;  // pass -1: count; before: counts hold places
    int sorts, turns, jobs, per_row;   // workgroups that sort, tiles to turn, these and pieces to clear
    int first_job, l_tiles, d_blocks;
    Div31 by_d_blocks, by_l_tiles;
};

__device__ __forceinline__ int key_at(const SortArgs& a, int m) {
    if (a.pass > 0) return a.keys[(a.pass & 1) ^ 1][m];
    const int n = div31(m, a.by_L), l = m - n * a.L;
    const int t = token_at(a.tokens, a.wide, n, a.tok_sn, l, seq_length(a.lengths, n, a.L), a.V);
    return t < 0 ? a.V : t;
}

__device__ __forceinline__ void count_digits(const SortArgs& a, int* count) {
    const int tid = static_cast<int>(threadIdx.x), tile = static_cast<int>(blockIdx.x), bins = 1 << a.bits;
    if (tid < kBins) count[tid] = 0;
    if (tile == 0 && tid == 0) a.owners[0] = 0;
    for (int p = 1; p < a.passes; ++p)
        if (tid < kBins) a.counts[(static_cast<long>(p) * a.tiles + tile) * kBins + tid] = 0;
    __syncthreads();
    const long first = static_cast<long>(tile) * a.per_lane * kSort;
    for (int k = 0; k < a.per_lane; ++k) {
        const long m = first + k * kSort + tid;
        if (m < a.M) lds_add(&count[key_at(a, static_cast<int>(m)) & (bins - 1)], 1);
    }
    __syncthreads();
    if (tid < kBins) a.counts[static_cast<long>(tile) * kBins + tid] = count[tid];
}

// exclusive sums of the first kBins threads' numbers over them
__device__ __forceinline__ int bins_before(int v, int* lds) {
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kSeqWave - 1), wave = tid / kSeqWave;
    int sum = v;
#pragma unroll
    for (int m = 1; m < kSeqWave; m <<= 1) {
        const int o = lane_up(sum, m);
        sum += lane >= m ? o : 0;
    }
    if (lane == kSeqWave - 1) lds[wave] = sum;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < kBins / kSeqWave; ++w) before += w < wave ? lds[w] : 0;
    return before + sum - v;
}

struct SortLds {
    int place[kSortWaves][kBins];
    int before[kSort / kBins][kBins], total[kSort / kBins][kBins], waves[kSortWaves];
};

__device__ __forceinline__ void put_keys(const SortArgs& a, SortLds& s) {
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kSeqWave - 1), wave = tid / kSeqWave, tile = static_cast<int>(blockIdx.x);
    const int bins = 1 << a.bits, shift = a.pass * a.bits, digit_of = tid & (kBins - 1), slice = tid / kBins;
    const int* counts = a.counts + static_cast<long>(a.pass) * a.tiles * kBins;
    const long first = static_cast<long>(tile) * a.per_lane * kSort + wave * (a.per_lane * kSeqWave) + lane;
    int key[kKeys], mine[kKeys];
#pragma unroll
    for (int k = 0; k < kKeys; ++k) {
        if (k >= a.per_lane) break;
        const long m = first + k * kSeqWave;
        key[k] = key_at(a, static_cast<int>(m < a.M ? m : a.M - 1));
    }
#pragma unroll
    for (int w = 0; w < kSortWaves; w += kSort / kBins) s.place[w + slice][digit_of] = 0;
    // what lies before this tile's keys of each digit: the same digit in earlier tiles, smaller digits anywhere
    int before = 0, total = 0;
    if (a.before) {
        if (slice == 0) {
            before = counts[static_cast<long>(tile) * kBins + digit_of];
            total = a.totals[digit_of];
        }
    } else {
#pragma unroll 8
        for (int t = slice; t < a.tiles; t += kSort / kBins) {
            const int n = counts[t * kBins + digit_of];
            total += n;
            before += t < tile ? n : 0;
        }
    }
    s.before[slice][digit_of] = before;
    s.total[slice][digit_of] = total;
    __syncthreads();
    // a wave has per_lane * 64 neighbouring keys; lanes with the same digit take their places in the order of the lanes
#pragma unroll
    for (int k = 0; k < kKeys; ++k) {
        if (k >= a.per_lane) break;
        const bool there = first + k * kSeqWave < a.M;
        const int digit = (key[k] >> shift) & (bins - 1);
        unsigned long same = wave_ballot(there);
        for (int bit = 1; bit < bins; bit <<= 1) {
            const bool set = digit & bit;
            const unsigned long with = wave_ballot(set);
            same &= set ? with : ~with;
        }
        const int leader = there ? first_bit(same) : lane, ahead = popcount64(same & ((1UL << lane) - 1));
        int at = 0;
        if (there && lane == leader) at = lds_add(&s.place[wave][digit], popcount64(same));
        mine[k] = lane_from(at, leader) + ahead;
    }
    int base = 0;
    if (tid < kBins) {
        total = 0;
#pragma unroll
        for (int i = 0; i < kSort / kBins; ++i) {
            total += s.total[i][tid];
            base += s.before[i][tid];
        }
    }
    base += bins_before(tid < kBins ? total : 0, s.waves);
    __syncthreads();
    if (tid < kBins) {
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            const int n = s.place[w][tid];
            s.place[w][tid] = base;
            base += n;
        }
    }
    __syncthreads();
    const int out = a.pass & 1;
#pragma unroll
    for (int k = 0; k < kKeys; ++k) {
        const long m = first + k * kSeqWave;
        if (k >= a.per_lane || m >= a.M) break;
        const int to = s.place[wave][(key[k] >> shift) & (bins - 1)] + mine[k];
        const int pos = a.pass > 0 ? a.pos[out ^ 1][m] : static_cast<int>(m);
        if (to < 0 || to >= a.M || pos < 0 || pos >= a.M) continue;  // (never, as long as the tokens do not change meanwhile)
        a.keys[out][to] = key[k];
        a.pos[out][to] = pos;
        if (a.pass + 1 < a.passes) {
            const long tile_to = to / (a.per_lane * kSort), digit = (key[k] >> (shift + a.bits)) & (bins - 1);
            global_add(&a.counts[((a.pass + 1L) * a.tiles + tile_to) * kBins + digit], 1);
        }
    }
}

// Many tiles: counts into places.  A workgroup has 16 digits, 64 shares of the tiles each.
__global__ __launch_bounds__(kSort) void embed_places_kernel(SortArgs a) {
    __shared__ int sum[kSort / 16][16];
    const int tid = static_cast<int>(threadIdx.x), o = tid & 15, share = tid >> 4, digit = 16 * static_cast<int>(blockIdx.x) + o;
    int* counts = a.counts + static_cast<long>(a.pass) * a.tiles * kBins + digit;
    const int each = (a.tiles + kSort / 16 - 1) / (kSort / 16), from = min(a.tiles, share * each), to = min(a.tiles, from + each);
    int n = 0;
#pragma unroll 4
    for (int t = from; t < to; ++t) n += counts[static_cast<long>(t) * kBins];
    sum[share][o] = n;
    __syncthreads();
    int before = 0;
    for (int i = 0; i < kSort / 16; ++i) before += i < share ? sum[i][o] : 0;
    if (share == kSort / 16 - 1) a.totals[digit] = before + n;
    for (int t = from; t < to; ++t) {
        const int v = counts[static_cast<long>(t) * kBins];
        counts[static_cast<long>(t) * kBins] = before;
        before += v;
    }
}

// dy's columns as rows
constexpr int kTurn = 16384;
template <bool BF16, int DT>
struct TurnLds {
    typename RowElem<BF16>::type v[DT * (kTurn / DT + 2)];
};
template <bool BF16, int DT>
__device__ __forceinline__ void turn_tile(const SortArgs& a, int unit, TurnLds<BF16, DT>& lds) {
    using T = typename RowElem<BF16>::type;
    constexpr int P = kTurn / DT, S = P + 2, NV = DT / 8;
    const int nt = div31(unit, a.by_d_blocks), d0 = (unit - nt * a.d_blocks) * DT, n = div31(nt, a.by_l_tiles), l0 = (nt - n * a.l_tiles) * P;
    const int tid = static_cast<int>(threadIdx.x), len = seq_length(a.lengths, n, a.L), many = min(DT, a.D - d0), padded = (many + 7) & ~7;
    if (l0 >= len) return;
    const T* dy = static_cast<const T*>(a.dy) + n * a.dy_sn;
#pragma unroll
    for (int i = tid; i < kTurn / 8; i += kSort) {
        const int d = i / (P / 8), p = 8 * (i % (P / 8));
        if (d >= padded) continue;
        float v[8];
        row_load8<BF16>(dy + (d0 + min(d, many - 1)) * a.dy_sd, l0 + p, len, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) store_elem<BF16>(lds.v, d * S + p + e, v[e]);
    }
    __syncthreads();
    T* rows = static_cast<T*>(a.rows) + (static_cast<long>(n) * a.L + l0) * (8 * a.per_row) + d0;
#pragma unroll
    for (int i = tid; i < P * NV; i += kSort) {
        const int p = i / NV, d = 8 * (i % NV);
        if (d >= many || l0 + p >= len) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = load_elem<BF16>(lds.v, (d + e) * S + p);
        row_store8<BF16>(rows + static_cast<long>(p) * (8 * a.per_row), d, d + 8, v);
    }
}

constexpr long kClear = 16 * kSort;  // floats a workgroup clears

template <bool BF16, int DT>
__global__ __launch_bounds__(kSort) void embed_sort_kernel(SortArgs a) {
    __shared__ union {
        SortLds sort;
        TurnLds<BF16, DT> turn;
    } lds;
    const int block = static_cast<int>(blockIdx.x), tid = static_cast<int>(threadIdx.x);
    if (block < a.sorts) {
        if (a.pass < 0) count_digits(a, lds.sort.place[0]);
        else put_keys(a, lds.sort);
        return;
    }
    const int job = a.first_job + block - a.sorts;
    if (job < a.turns) {
        turn_tile<BF16, DT>(a, job, lds.turn);
        return;
    }
    const float none[8] = {};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const long at = (job - a.turns) * kClear + (k * kSort + tid) * 8L;
        if (at < a.zeros) row_store8<false>(a.dtable, at, a.zeros, none);
    }
}

// ---- backward, many tokens: sums of runs -----------------------------------------------------------------------------------
struct SumArgs {
    const void* rows;        // row m is position m's, stride apart (samples: sample_stride)
    const int *keys, *pos;
    int* owners;
    float *head, *tail;      // [chunks][per_row * 8]: what of a chunk belongs to a run that began before it, that goes on behind it
    float* dtable;
    long sample_stride, stride;
    float scale;
    int D, L, V, M, per_row, chunk, chunks, first, items;
    Div31 by_row, by_L;
};

__device__ __forceinline__ void float_store8(float* row, int at, int end, const float (&v)[8], float scale) {
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = v[e] * scale;
    row_store8<false>(row, at, end, s);
}

template <bool BF16, bool TURNED>
__global__ __launch_bounds__(kThreads) void embed_sums_kernel(SumArgs a) {
    using T = typename RowElem<BF16>::type;
    const int item = static_cast<int>(blockIdx.x) * kThreads + static_cast<int>(threadIdx.x);
    if (item >= a.items) return;
    const int of = div31(item, a.by_row), chunk = a.first + of, d = 8 * (item - of * a.per_row);
    const int from = chunk * a.chunk, to = min(a.M, from + a.chunk);
    int key = a.keys[from];
    if (key >= a.V) return;
    bool began = from == 0 || a.keys[from - 1] != key;
    const int width = 8 * a.per_row;
    float sum[8] = {};
    constexpr int kAhead = 8;
#pragma unroll 1
    for (int i0 = from; i0 < to; i0 += kAhead) {
        float v[kAhead][8];
        int k[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int i = min(i0 + j, a.M - 1), m = a.pos[i];
            k[j] = a.keys[i];
            if constexpr (TURNED) {
                row_load8_inside<BF16>(static_cast<const T*>(a.rows) + m * a.stride, d, v[j]);
            } else {
                const int n = div31(m, a.by_L), l = m - n * a.L;
                row_load8<BF16>(static_cast<const T*>(a.rows) + n * a.sample_stride + l * a.stride, d, a.D, v[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (i0 + j >= to) break;
            if (k[j] != key) {
                if (began) float_store8(a.dtable + static_cast<long>(key) * a.D, d, a.D, sum, a.scale);
                else float_store8(a.head + static_cast<long>(chunk) * width, d, width, sum, 1.f);
                if (k[j] >= a.V) return;
                key = k[j];
                began = true;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += v[j][e];
        }
    }
    if (!began) {
        float_store8(a.head + static_cast<long>(chunk) * width, d, width, sum, 1.f);
    } else if (to < a.M && a.keys[to] == key) {
        float_store8(a.tail + static_cast<long>(chunk) * width, d, width, sum, 1.f);
        if (d == 0) a.owners[1 + global_add(a.owners, 1)] = chunk;
    } else {
        float_store8(a.dtable + static_cast<long>(key) * a.D, d, a.D, sum, a.scale);
    }
}

// Runs that cross chunks, in any order: what the chunks behind the one where a run begins have of it is added to that one's.
struct JoinArgs {
    const int *keys, *owners;
    const float *head, *tail;
    float* dtable;
    float scale;
    int D, V, M, per_row, chunk, chunks;
};
// the first place of a key >= v
__device__ __forceinline__ int place_of(const int* keys, int M, int v) {
    int lo = 0, hi = M;
    while (lo < hi) {
        const int mid = lo + ((hi - lo) >> 1);
        if (keys[mid] < v) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}
__global__ __launch_bounds__(kThreads) void embed_join_kernel(JoinArgs a) {
    __shared__ double lds[kThreads][8];
    const int tid = static_cast<int>(threadIdx.x), width = 8 * a.per_row, cols = min(a.per_row, kThreads), teams = kThreads / cols, team = tid / cols;
    const int many = min(a.owners[0], a.chunks - 1);
    for (int i = static_cast<int>(blockIdx.x); i < many; i += static_cast<int>(gridDim.x)) {
        const int chunk = clampi(a.owners[1 + i], 0, a.chunks - 2), key = a.keys[(chunk + 1) * a.chunk - 1];
        const int last = max(chunk, (place_of(a.keys, a.M, key + 1) - 1) / a.chunk);  // the chunk where it ends
        if (key < 0 || key >= a.V) continue;  // (never)
        for (int c0 = 0; c0 < a.per_row; c0 += cols) {
            const int d = 8 * (c0 + tid - team * cols);
            double sum[8] = {};
            if (team < teams && d < width) {
#pragma unroll 4
                for (int c = chunk + team; c <= last; c += teams) {
                    float v[8];
                    row_load8_inside<false>((c == chunk ? a.tail : a.head) + static_cast<long>(c) * width, d, v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[e] += v[e];
                }
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) lds[tid][e] = sum[e];
            __syncthreads();
            if (team == 0 && d < width) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    double s = sum[e];
                    for (int t = 1; t < teams; ++t) s += lds[tid + t * cols][e];
                    v[e] = static_cast<float>(s);
                }
                float_store8(a.dtable + static_cast<long>(key) * a.D, d, a.D, v, a.scale);
            }
        }
    }
}

// ---- host -----------------------------------------------------------------------------------------------------------
bool shape_ok(const conv1d_embed_t* p) {
    if (!p || !p->tokens || p->N < 1 || p->D < 1 || p->L < 1 || p->V < 1) return false;
    if (p->dtype != CONV1D_FP32 && p->dtype != CONV1D_BF16) return false;
    if ((p->flags & ~CONV1D_EMBED_TOKENS64) != 0) return false;
    return seq_aligned(p->tokens, p->flags & CONV1D_EMBED_TOKENS64 ? 8 : 4) && seq_aligned(p->lengths, 4);
}
bool sizes_ok(int N, int D, int L, int V) {
    return D <= 1 << 20 && V < 1 << 30 && static_cast<long>(N) * L <= 1 << 30;
}
int status_of(hipError_t e) { return e == hipSuccess ? CONV1D_OK : CONV1D_EHIP; }

// positions or channels contiguous; an axis of one element has no stride
bool strides_ok(int D, int L, long sd, long sl) { return D == 1 || L == 1 || sl == 1 || sd == 1; }
// positions contiguous: tiles are turned; else channels are, and rows copied
bool is_turned(int D, int L, long sd, long sl) { return L == 1 ? D > 1 && sd != 1 : sl == 1; }

// DT of a tile: 16 channels leave few lanes idle where there are no more
int tile_channels(int D) { return D <= 16 ? 16 : 64; }
constexpr long kMostBlocks = kSeqMostThreads / kSort - 1;

template <bool BF16>
hipError_t look_up(const conv1d_embed_t* p, LookArgs& a, hipStream_t st) {
    if (!is_turned(p->D, p->L, a.y_sd, a.y_sl)) {
        a.per_row = (p->D + 7) / 8;
        a.by_row = make_div31(a.per_row);
        a.by_L = make_div31(p->L);
        const long M = static_cast<long>(p->N) * p->L, most = kMostItems / a.per_row;
        for (long m = 0; m < M; m += most) {
            a.first = m;
            a.items = static_cast<int>((M - m < most ? M - m : most) * a.per_row);
            const hipError_t e = launch_kernel(embed_copy_kernel<BF16>, dim3(static_cast<unsigned>(cdiv(a.items, kThreads))), dim3(kThreads), 0, st, a);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    void (*kern)(LookArgs) = nullptr;
    size_t lds = 0;
    if (p->V < kFewRows) {
        // as many channels a workgroup as leave enough workgroups, and room for several beside each other
        a.tiles = cdiv(p->L, 8 * kThreads);
        a.per_row = 16;
        while (a.per_row > 4 && (static_cast<long>(p->N) * a.tiles * cdiv(p->D, a.per_row) < kFill || (p->V + 1L) * a.per_row > kFewElements)) a.per_row /= 2;
        a.blocks = cdiv(p->D, a.per_row);
        lds = static_cast<size_t>(p->V + 1) * a.per_row * (BF16 ? 2 : 4);
        kern = embed_few_kernel<BF16>;
    } else {
        const int DT = tile_channels(p->D);
        a.tiles = cdiv(p->L, kTile / DT);
        a.blocks = cdiv(p->D, DT);
        kern = DT == 16 ? embed_turn_kernel<BF16, 16> : embed_turn_kernel<BF16, 64>;
    }
    a.by_tiles = make_div31(a.tiles);
    a.by_blocks = make_div31(a.blocks);
    const long units = static_cast<long>(p->N) * a.tiles * a.blocks;
    if (units > kMostItems) return hipErrorInvalidValue;
    for (long u = 0; u < units; u += kMostBlocks) {
        a.first = u;
        const hipError_t e = launch_kernel(kern, dim3(static_cast<unsigned>(units - u < kMostBlocks ? units - u : kMostBlocks)), dim3(kThreads), lds, st, a);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ---- the gradient's workspace -------------------------------------------------------------------------------------------
struct FewPlan {
    int VB, DB, Vp, Dp, vgroups, dgroups, chunk, samples, per_sample, chunks;
    size_t bytes;
};
FewPlan few_plan(int N, int D, int L, int V) {
    FewPlan p{};
    p.Vp = static_cast<int>(round_up(V, 16));
    p.Dp = static_cast<int>(round_up(D, 16));
    p.VB = p.Vp <= 16 ? 1 : 4;
    p.DB = p.Dp <= 16 ? 1 : 4;
    p.vgroups = cdiv(p.Vp, 16 * p.VB);
    p.dgroups = cdiv(p.Dp, 16 * p.DB);
    // enough workgroups to fill the chip, but no more partial sums than dy has numbers
    const long want = kFill / (static_cast<long>(p.vgroups) * p.dgroups), M = static_cast<long>(N) * L, step = 32 * kWaves;
    long chunk = want > 1 ? (M + want - 1) / want : M;
    if (chunk < p.Vp) chunk = p.Vp;
    if (chunk >= 2L * L) {
        p.samples = static_cast<int>(chunk / L < N ? chunk / L : N);
        p.chunk = L;
    } else {
        p.samples = 1;
        p.chunk = static_cast<int>((chunk + step - 1) / step * step);
    }
    p.per_sample = cdiv(L, p.chunk);
    p.chunks = cdiv(N, p.samples) * p.per_sample;
    p.bytes = sizeof(float) * static_cast<size_t>(p.chunks) * p.Vp * p.Dp;
    return p;
}
// Whether the gradient is taken as a product
bool is_few(int N, int D, int L, int V, bool turned) {
    if (!turned || V > kFewTokens) return false;
    const FewPlan p = few_plan(N, D, L, V);
    return static_cast<long>(p.chunks) * p.vgroups * p.dgroups <= kMostBlocks && static_cast<long>(p.Vp) * p.Dp / 16 <= kMostBlocks;
}

struct Plan {
    int M, bits, passes, tiles, per_lane, chunk, chunks, per_row;
    size_t keys[2], pos[2], counts, totals, owners, rows, head, tail, bytes;
};
Plan plan_of(int N, int D, int L, int V, int dtype, bool turned) {
    Plan p{};
    p.M = N * L;
    int bits = 1;
    while (bits < 31 && (1L << bits) <= V) ++bits;  // the keys 0 ... V
    p.passes = cdiv(bits, 8);
    p.bits = cdiv(bits, p.passes);
    p.per_lane = p.M <= kFewTiles * kSort ? 1 : kKeys;
    p.tiles = cdiv(p.M, p.per_lane * kSort);
    p.per_row = (D + 7) / 8;
    // chunks of 32 rows, of 16 where that leaves the chip idle
    p.chunk = static_cast<long>(p.M) * p.per_row < 32L * kFill * kSeqWave ? 16 : 32;
    p.chunks = cdiv(p.M, p.chunk);
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += round_up(bytes, 256);
        return here;
    };
    const size_t M = static_cast<size_t>(p.M), width = 8 * static_cast<size_t>(p.per_row);
    for (int i = 0; i < 2; ++i) {
        p.keys[i] = take(4 * M);
        p.pos[i] = take(4 * M);
    }
    p.counts = take(4 * static_cast<size_t>(p.passes) * p.tiles * kBins);
    p.totals = take(4 * static_cast<size_t>(kBins));
    p.owners = take(4 * (static_cast<size_t>(p.chunks) + 1));
    p.rows = take(turned ? M * width * (dtype == CONV1D_BF16 ? 2 : 4) : 0);
    p.head = take(4 * width * p.chunks);
    p.tail = take(4 * width * p.chunks);
    p.bytes = at;
    return p;
}

template <bool BF16>
hipError_t few_gradient(const conv1d_embed_t* p, const void* dy, long dy_sn, long dy_sd, float* dtable, const FewPlan& plan, float* ws, hipStream_t st) {
    FewArgs a{};
    a.dy = dy; a.tokens = p->tokens; a.lengths = p->lengths; a.part = ws; a.dtable = dtable;
    a.tok_sn = p->tok_sn; a.dy_sn = dy_sn; a.dy_sd = dy_sd; a.scale = p->scale;
    a.wide = p->flags & CONV1D_EMBED_TOKENS64; a.D = p->D; a.L = p->L; a.V = p->V; a.Vp = plan.Vp; a.Dp = plan.Dp;
    a.N = p->N; a.chunk = plan.chunk; a.samples = plan.samples; a.chunks = plan.chunks; a.per_sample = plan.per_sample; a.vgroups = plan.vgroups; a.dgroups = plan.dgroups;
    a.by_vgroups = make_div31(plan.vgroups);
    a.by_dgroups = make_div31(plan.dgroups);
    a.by_sample = make_div31(plan.per_sample);
    void (*kern)(FewArgs) = plan.VB == 1 ? (plan.DB == 1 ? embed_few_sums_kernel<BF16, 1, 1> : embed_few_sums_kernel<BF16, 1, 4>)
                                         : (plan.DB == 1 ? embed_few_sums_kernel<BF16, 4, 1> : embed_few_sums_kernel<BF16, 4, 4>);
    const unsigned units = static_cast<unsigned>(static_cast<long>(plan.chunks) * plan.vgroups * plan.dgroups);
    const hipError_t e = launch_kernel(kern, dim3(units), dim3(kThreads), 0, st, a);
    if (e != hipSuccess) return e;
    return launch_kernel(embed_few_join_kernel, dim3(static_cast<unsigned>(static_cast<long>(plan.Vp) * plan.Dp / 16)), dim3(kFewJoin), 0, st, a);
}

template <bool BF16>
hipError_t gradient(const conv1d_embed_t* p, const void* dy, long dy_sn, long dy_sd, long dy_sl, float* dtable, bool turned, const Plan& plan, char* ws,
                    hipStream_t st) {
    const int DT = tile_channels(p->D);
    SortArgs a{};
    a.tokens = p->tokens; a.dy = dy; a.lengths = p->lengths; a.tok_sn = p->tok_sn; a.dy_sn = dy_sn; a.dy_sd = dy_sd;
    a.wide = p->flags & CONV1D_EMBED_TOKENS64; a.N = p->N; a.D = p->D; a.L = p->L; a.V = p->V; a.M = plan.M;
    a.by_L = make_div31(p->L);
    for (int i = 0; i < 2; ++i) {
        a.keys[i] = reinterpret_cast<int*>(ws + plan.keys[i]);
        a.pos[i] = reinterpret_cast<int*>(ws + plan.pos[i]);
    }
    a.counts = reinterpret_cast<int*>(ws + plan.counts);
    a.totals = reinterpret_cast<int*>(ws + plan.totals);
    a.owners = reinterpret_cast<int*>(ws + plan.owners);
    a.rows = ws + plan.rows;
    a.dtable = dtable;
    a.zeros = static_cast<long>(p->V) * p->D;
    a.passes = plan.passes; a.bits = plan.bits; a.tiles = plan.tiles; a.per_lane = plan.per_lane; a.per_row = plan.per_row;
    a.before = plan.tiles > kFewTiles;
    a.l_tiles = cdiv(p->L, kTurn / DT);
    a.d_blocks = cdiv(p->D, DT);
    a.by_l_tiles = make_div31(a.l_tiles);
    a.by_d_blocks = make_div31(a.d_blocks);
    const long turns = turned ? static_cast<long>(p->N) * a.l_tiles * a.d_blocks : 0, jobs = turns + (a.zeros + kClear - 1) / kClear;
    if (jobs > kMostItems) return hipErrorInvalidValue;
    a.turns = static_cast<int>(turns);
    void (*sort)(SortArgs) = DT == 16 ? embed_sort_kernel<BF16, 16> : embed_sort_kernel<BF16, 64>;
    long done = 0;
    for (a.pass = -1; a.pass < plan.passes; ++a.pass) {
        hipError_t e = hipSuccess;
        if (a.pass >= 0 && a.before) e = launch_kernel(embed_places_kernel, dim3(kBins / 16), dim3(kSort), 0, st, a);
        // the other work in equal shares, what is too much for a grid in grids of its own
        const long upto = jobs * (a.pass + 2) / (plan.passes + 1);
        a.sorts = plan.tiles;
        do {
            const long some = upto - done < kMostBlocks - a.sorts ? upto - done : kMostBlocks - a.sorts;
            a.first_job = static_cast<int>(done);
            if (e == hipSuccess && a.sorts + some > 0) e = launch_kernel(sort, dim3(static_cast<unsigned>(a.sorts + some)), dim3(kSort), 0, st, a);
            if (e != hipSuccess) return e;
            done += some;
            a.sorts = 0;
        } while (done < upto);
    }
    const int last = (plan.passes - 1) & 1;
    SumArgs s{};
    s.rows = turned ? static_cast<const void*>(ws + plan.rows) : dy;
    s.keys = a.keys[last]; s.pos = a.pos[last]; s.owners = a.owners;
    s.head = reinterpret_cast<float*>(ws + plan.head);
    s.tail = reinterpret_cast<float*>(ws + plan.tail);
    s.dtable = dtable;
    s.sample_stride = dy_sn;
    s.stride = turned ? 8L * plan.per_row : dy_sl;
    s.scale = p->scale; s.D = p->D; s.L = p->L; s.V = p->V; s.M = plan.M; s.per_row = plan.per_row; s.chunk = plan.chunk; s.chunks = plan.chunks;
    s.by_row = make_div31(plan.per_row);
    s.by_L = make_div31(p->L);
    const long most = kMostItems / plan.per_row;
    void (*sums)(SumArgs) = turned ? embed_sums_kernel<BF16, true> : embed_sums_kernel<BF16, false>;
    for (long c = 0; c < plan.chunks; c += most) {
        s.first = static_cast<int>(c);
        s.items = static_cast<int>((plan.chunks - c < most ? plan.chunks - c : most) * plan.per_row);
        const hipError_t e = launch_kernel(sums, dim3(static_cast<unsigned>(cdiv(s.items, kThreads))), dim3(kThreads), 0, st, s);
        if (e != hipSuccess) return e;
    }
    if (plan.chunks < 2) return hipSuccess;
    JoinArgs j{};
    j.keys = s.keys; j.owners = a.owners; j.head = s.head; j.tail = s.tail; j.dtable = dtable; j.scale = p->scale;
    j.D = p->D; j.V = p->V; j.M = plan.M; j.per_row = plan.per_row; j.chunk = plan.chunk; j.chunks = plan.chunks;
    return launch_kernel(embed_join_kernel, dim3(static_cast<unsigned>(plan.chunks - 1 < kFill ? plan.chunks - 1 : kFill)), dim3(kThreads), 0, st, j);
}

}  // namespace
}  // namespace conv1d

using namespace conv1d;

extern "C" {

int conv1d_embed_fwd(const conv1d_embed_t* p, const void* table, void* y, long y_sn, long y_sd, long y_sl, void* stream) {
    if (!shape_ok(p) || !table || !y) return CONV1D_EINVAL;
    const size_t size = p->dtype == CONV1D_BF16 ? 2 : 4;
    if (!seq_aligned(table, size) || !seq_aligned(y, size) || !strides_ok(p->D, p->L, y_sd, y_sl)) return CONV1D_EINVAL;
    if (!sizes_ok(p->N, p->D, p->L, p->V)) return CONV1D_EUNSUPPORTED;
    LookArgs a{};
    a.table = table; a.tokens = p->tokens; a.lengths = p->lengths; a.y = y;
    a.tok_sn = p->tok_sn; a.y_sn = y_sn; a.y_sd = y_sd; a.y_sl = y_sl;
    a.scale = p->scale; a.wide = p->flags & CONV1D_EMBED_TOKENS64; a.N = p->N; a.D = p->D; a.L = p->L; a.V = p->V;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return status_of(p->dtype == CONV1D_BF16 ? look_up<true>(p, a, st) : look_up<false>(p, a, st));
}

size_t conv1d_embed_bwd_workspace_bytes(int N, int D, int L, int V, int dtype) {
    if (N < 1 || D < 1 || L < 1 || V < 1 || !sizes_ok(N, D, L, V) || (dtype != CONV1D_FP32 && dtype != CONV1D_BF16)) return 0;
    const size_t few = is_few(N, D, L, V, true) ? few_plan(N, D, L, V).bytes : plan_of(N, D, L, V, dtype, true).bytes, rest = plan_of(N, D, L, V, dtype, false).bytes;
    return few > rest ? few : rest;  // for dy in either order
}

int conv1d_embed_bwd(const conv1d_embed_t* p, const void* dy, long dy_sn, long dy_sd, long dy_sl, float* dtable, void* workspace, size_t workspace_bytes,
                     void* stream) {
    if (!shape_ok(p) || !dy || !dtable) return CONV1D_EINVAL;
    const size_t size = p->dtype == CONV1D_BF16 ? 2 : 4;
    if (!seq_aligned(dy, size) || !seq_aligned(dtable, 4) || !seq_aligned(workspace, 256) || !strides_ok(p->D, p->L, dy_sd, dy_sl)) return CONV1D_EINVAL;
    if (!sizes_ok(p->N, p->D, p->L, p->V)) return CONV1D_EUNSUPPORTED;
    const bool turned = is_turned(p->D, p->L, dy_sd, dy_sl);
    char* ws = static_cast<char*>(workspace);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool bf16 = p->dtype == CONV1D_BF16;
    if (is_few(p->N, p->D, p->L, p->V, turned)) {
        const FewPlan plan = few_plan(p->N, p->D, p->L, p->V);
        if (!workspace || workspace_bytes < plan.bytes) return CONV1D_EWORKSPACE;
        float* part = reinterpret_cast<float*>(ws);
        return status_of(bf16 ? few_gradient<true>(p, dy, dy_sn, dy_sd, dtable, plan, part, st) : few_gradient<false>(p, dy, dy_sn, dy_sd, dtable, plan, part, st));
    }
    const Plan plan = plan_of(p->N, p->D, p->L, p->V, p->dtype, turned);
    if (!workspace || workspace_bytes < plan.bytes) return CONV1D_EWORKSPACE;
    return status_of(bf16 ? gradient<true>(p, dy, dy_sn, dy_sd, dy_sl, dtable, turned, plan, ws, st)
                          : gradient<false>(p, dy, dy_sn, dy_sd, dy_sl, dtable, turned, plan, ws, st));
}

}  // extern "C"
