// Embedding lookup with scaling, and its gradient by sorted tokens.
//   y[n][d][l] = scale table[tokens[n][l]][d],   dtable[v][d] = scale sum over (n, l) with tokens[n][l] = v of dy[n][d][l]
// Memory is what large calls wait for (4 to 5 of 5.2 TB/s at 8 x 512 x 8192); launches of one turn of the chip reach 3.  Where positions are
// contiguous, tiles of positions and channels are turned in LDS: rows of the table are read and written along the channels, y and dy along
// the positions.
// The gradient adds the same positions in the same order in every run.  Few tokens: dy is multiplied with the truth values
// "position l has token v" on the matrix cores, straight from memory, at most 16 sums of 32 products in float and four waves' together, the
// rest in 64 bits.  Many: the positions are sorted by their token (a stable radix
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

// A tile of kTile / DT positions and DT channels: 8 x 512 x 8192 bfloat16 of 32000 tokens 20 to 23 us, 4.3 to 5 TB/s.  Two elements more than a
// row's positions: the eight channels that a lane writes, and those of its neighbours, begin in different banks.
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

// Few tokens and channels (16 x 15 x 60000 bfloat16, five tokens: 11.7 us, 17.8 by tiles; 36 MB at 3.1 TB/s, 1920 workgroups that read and then
// write once): the workgroup's channels of the whole table, scaled and rounded, lie in LDS (and a row of zeros for no token); a lane has 8
// positions, whose tokens (read side by side, and handed over in LDS) it keeps.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void embed_few_kernel(LookArgs a) {
    using T = typename RowElem<BF16>::type;
    extern __shared__ char dynamic[];
    const int unit = static_cast<int>(blockIdx.x) + static_cast<int>(a.first);
    const int nt = div31(unit, a.by_blocks), d0 = (unit - nt * a.blocks) * a.per_row, n = div31(nt, a.by_tiles);
    const int l = ((nt - n * a.tiles) * kThreads + static_cast<int>(threadIdx.x)) * 8;
    const int len = seq_length(a.lengths, n, a.L), many = min(a.per_row, a.D - d0);
    const int first = l - 8 * static_cast<int>(threadIdx.x);
    unsigned short* toks = reinterpret_cast<unsigned short*>(dynamic);  // 16 bits each
    T* lds = reinterpret_cast<T*>(dynamic + 2 * 8 * kThreads);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int p = e * kThreads + static_cast<int>(threadIdx.x), t = token_at(a.tokens, a.wide, n, a.tok_sn, first + p, len, a.V);
        toks[p] = static_cast<unsigned short>(t < 0 ? a.V : t);
    }
    for (int i = static_cast<int>(threadIdx.x); i < (a.V + 1) * many; i += kThreads) {
        const int v = i / many;
        const float u = v < a.V ? load_elem<BF16>(a.table, static_cast<long>(v) * a.D + d0 + (i - v * many)) * a.scale : 0.f;
        store_elem<BF16>(lds, i, u);
    }
    __syncthreads();
    if (l >= a.L) return;
    const seq_u16x8 mine = *reinterpret_cast<const seq_u16x8*>(toks + 8 * threadIdx.x);
    int at[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) at[e] = min(static_cast<int>(mine[e]), a.V) * many;
    T* y = static_cast<T*>(a.y) + n * a.y_sn + d0 * a.y_sd;
    typedef __attribute__((ext_vector_type(8), aligned(BF16 ? 2 : 4))) T vec8;
#pragma unroll 4
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
// Tens of tokens: 16 x 15 x 60000 bfloat16, five, 12.8 us, 36 MB at 2.8 TB/s, since each of 1888 workgroups has one block, a chain of loads,
// product and stores.  Hundreds: bound by the vector units (12 x 49 x 4999 float, 257: 22 us).
// dtable[v][d] = sum over l of dy[d][l] [token l = v]: an A operand is 16 channels of 32 neighbouring positions as they lie in memory, a B
// operand the truth values of those positions for 16 tokens, exact in bfloat16; floats are taken as three bfloat16 numbers whose sum they are.
// The matrix instruction cuts off what its additions lose, so that a step's products start from 0 and are added to the running sum by ordinary additions;
// of a float, the upper 8 bits by themselves: 32 of them add up to 24 bits and lose nothing as long as their
// exponents are less than 11 apart (all three parts in one sum, 12 x 49 x 4999, 257 tokens: error against 64 bits 1.3e-7 of the norm).  A value that
// is not finite would reach every token (0 * NaN): where a sum is not finite, the workgroup goes through its positions again without such
// values, which are then added where they belong.
constexpr int kFewTokens = 65520;  // (16 bits each, 0xffff is no token)

struct FewArgs {
    const void *dy, *tokens;
    const int* lengths;
    float* part;           // [chunks][tokens and channels, both rounded up to 16]
    float* dtable;
    long tok_sn, dy_sn, dy_sd;
    float scale;
    int wide, N, D, L, V, Vp, Dp, vgroups, dgroups;
    int chunk, samples, per_sample, chunks;  // a chunk: positions of a sample, or all of some samples; chunks of a sample (or of those)
    int slice, slices;                       // chunks that a row of the joining grid has, its rows
    Div31 by_vgroups, by_dgroups, by_sample;
};

typedef sp::f32x4 f32x4;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;

// 8 positions' tokens in 16 bits, 0xffff for none
struct Tokens8 {
    unsigned t[4];
};
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
__device__ __forceinline__ Parts<BF16> parts_of(const Raw8<BF16>& x) {
    Parts<BF16> r;
    if constexpr (BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            unsigned u = x.v[0][i];
            if constexpr (FINITE) u = ((u & 0x7f80u) == 0x7f80u ? 0u : u & 0xffffu) | ((u & 0x7f800000u) == 0x7f800000u ? 0u : u & 0xffff0000u);
            r.p[0][i] = u;
        }
    } else {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = __uint_as_float(x.v[e >> 2][e & 3]);
            if constexpr (FINITE) v[e] = fabsf(v[e]) < INFINITY ? v[e] : 0.f;
        }
        const sp::Split8 s = sp::split8(v);
        r.p[0] = s.l;
        r.p[1] = s.m;
        r.p[2] = s.h;
    }
    return r;
}

constexpr int kWaves = kThreads / kSeqWave;

// A chunk: positions [from, to) of `samples` samples from n0 on, taken in blocks of kWaves waves' U steps of 32 positions.
struct Chunk {
    int n0, samples, from, to;
};
__device__ __forceinline__ Chunk chunk_of(const FewArgs& a, int chunk) {
    Chunk r;
    const int of = div31(chunk, a.by_sample);
    r.n0 = of * a.samples;
    r.samples = min(a.samples, a.N - r.n0);
    r.from = (chunk - of * a.per_sample) * a.chunk;
    r.to = min(a.L, r.from + a.chunk);
    return r;
}
// steps whose loads a wave has in flight, beside as many that it multiplies
template <bool BF16, int DB>
constexpr int kU = BF16 ? (DB == 1 ? 4 : 2) : (DB == 1 ? 2 : 1);
constexpr int kMostBlock = 32 * kWaves * 4;
// Most steps of a wave in one chunk, which bounds the additions in float: chunks are added up in 64 bits.  (Without a bound the
// equal gradients of one token at 160 x 16 x 2^20 positions in 2080 chunks were off by 9.4e-6, 158 half steps of float; with it by less than half
// of one.  Up to some millions of positions it costs up to 6 %, at 32 x 16 x 2^20 bfloat16, 200 tokens, 1.21 ms for 1.05.)
constexpr int kMostSteps = 16;

// A block of the chunk: positions l0 ... of sample n, of which len count.
struct Block {
    int n, l0, len;
};
// the chunk's first block that holds any position, from the given one on; n behind the last sample: none
__device__ __forceinline__ Block settle(const FewArgs& a, const Chunk& t, Block b) {
    while (b.n < t.n0 + t.samples) {
        b.len = min(t.to, seq_length(a.lengths, b.n, a.L));
        if (b.l0 < b.len) break;
        ++b.n;
        b.l0 = t.from;
    }
    return b;
}

template <bool BF16, int U, int DB>
struct FewLoads {
    Raw8<BF16> raw[U][DB];
    int toks[(U * 32 * kWaves + kThreads - 1) / kThreads];
};
template <bool BF16, int U, int DB>
__device__ __forceinline__ void load_block(const FewArgs& a, const Block& b, int d0, FewLoads<BF16, U, DB>& r) {
    using T = typename RowElem<BF16>::type;
    constexpr int BLOCK = 32 * kWaves * U;
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kSeqWave - 1), l = b.l0 + 32 * U * (tid / kSeqWave) + 8 * (lane >> 4);
#pragma unroll
    for (int i = 0; i * kThreads < BLOCK; ++i) r.toks[i] = token_at(a.tokens, a.wide, b.n, a.tok_sn, b.l0 + i * kThreads + tid, b.len, a.V);
    const T* base = static_cast<const T*>(a.dy) + b.n * a.dy_sn;
    const bool inside = b.l0 + BLOCK <= b.len;
#pragma unroll
    for (int d = 0; d < DB; ++d) {
        const T* row = base + min(d0 + 16 * d + (lane & 15), a.D - 1) * a.dy_sd;
        if (inside) {
#pragma unroll
            for (int u = 0; u < U; ++u) r.raw[u][d] = raw8_inside<BF16>(row, l + 32 * u);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) r.raw[u][d] = raw8<BF16>(row, l + 32 * u, b.len);
        }
    }
}

template <bool BF16, bool FINITE, int VB, int DB>
__device__ __forceinline__ void few_sums(const FewArgs& a, const Chunk& t, int v0, int d0, f32x4 (&acc)[VB][DB], unsigned short (*toks)[kMostBlock]) {
    constexpr int U = kU<BF16, DB>, BLOCK = 32 * kWaves * U;
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kSeqWave - 1), mine = 32 * U * (tid / kSeqWave);
#pragma unroll
    for (int v = 0; v < VB; ++v)
#pragma unroll
        for (int d = 0; d < DB; ++d) acc[v][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    Block b = settle(a, t, Block{t.n0, t.from, 0});
    if (b.n >= t.n0 + t.samples) return;
    FewLoads<BF16, U, DB> now, next;
    load_block(a, b, d0, now);
    for (int turn = 0;; turn ^= 1) {
#pragma unroll
        for (int i = 0; i * kThreads < BLOCK; ++i) toks[turn][i * kThreads + tid] = static_cast<unsigned short>(now.toks[i]);
        __syncthreads();  // (the next block writes the other half, the one after that waits behind the next)
        const Block after = settle(a, t, Block{b.n, b.l0 + BLOCK, 0});
        const bool more = after.n < t.n0 + t.samples;
        if (more) load_block(a, after, d0, next);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (b.l0 + mine + 32 * u >= b.len) break;
            const Tokens8 k = *reinterpret_cast<const Tokens8*>(&toks[turn][mine + 32 * u + 8 * (lane >> 4)]);
            Parts<BF16> x[DB];
#pragma unroll
            for (int d = 0; d < DB; ++d) x[d] = parts_of<BF16, FINITE>(now.raw[u][d]);
#pragma unroll
            for (int v = 0; v < VB; ++v) {
                const u32x4 one = truth8(k, v0 + 16 * v + (lane & 15));
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const f32x4 none = f32x4{0.f, 0.f, 0.f, 0.f};
                    f32x4 s = sp::mfma(x[d].p[0], one, none);
                    if constexpr (!BF16) {
                        s = sp::mfma(x[d].p[1], one, s);
                        const f32x4 h = sp::mfma(x[d].p[2], one, none);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[e] += h[e];
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[v][d][e] += s[e];
                }
            }
        }
        if (!more) break;
        now = next;
        b = after;
    }
}

// (three workgroups a compute unit for bfloat16: 8 x 128 x 20000, 64 tokens 25 us for 31 with two; for floats they would spill)
template <bool BF16, int VB, int DB>
__global__ __launch_bounds__(kThreads, BF16 ? 3 : 2) void embed_few_sums_kernel(FewArgs a) {
    using T = typename RowElem<BF16>::type;
    __shared__ float lds[VB * 16][DB * 16 + 4];
    const int unit = static_cast<int>(blockIdx.x), cd = div31(unit, a.by_vgroups), v0 = (unit - cd * a.vgroups) * (16 * VB);
    const int chunk = div31(cd, a.by_dgroups), d0 = (cd - chunk * a.dgroups) * (16 * DB);
    const Chunk t = chunk_of(a, chunk);
    __shared__ unsigned short toks[2][kMostBlock];
    __shared__ int bad;
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kSeqWave - 1), wave = tid / kSeqWave;
    f32x4 acc[VB][DB];
    if (tid == 0) bad = 0;
    __syncthreads();
    few_sums<BF16, false, VB, DB>(a, t, v0, d0, acc, toks);
    bool fine = true;
#pragma unroll
    for (int v = 0; v < VB; ++v)
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) fine &= fabsf(acc[v][d][i]) < INFINITY;
    if (!fine) bad = 1;
    __syncthreads();
    const bool again = bad != 0;  // (of any wave: the tokens are staged by all)
    if (again) few_sums<BF16, true, VB, DB>(a, t, v0, d0, acc, toks);
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
        for (int n = t.n0; n < t.n0 + t.samples; ++n) {
            const int len = min(t.to, seq_length(a.lengths, n, a.L)), many = max(0, len - t.from);
            for (long i = tid; i < static_cast<long>(many) * (16 * DB); i += kThreads) {
                const int d = d0 + static_cast<int>(i / many), l = t.from + static_cast<int>(i % many);
                if (d >= a.D) break;
                const float v = load_elem<BF16>(static_cast<const T*>(a.dy) + n * a.dy_sn + d * a.dy_sd, l);
                if (fabsf(v) < INFINITY) continue;
                const int tok = token_at(a.tokens, a.wide, n, a.tok_sn, l, len, a.V);
                if (tok >= v0 && tok < v0 + 16 * VB) lds_add(&lds[tok - v0][d - d0], v);
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

// 16 neighbouring numbers a workgroup, each the sum of THREADS / 16 lanes' shares of the chunks; where few numbers have many chunks, of those
// that one of a.slices rows of the grid has, left in two floats in the place of its first two.
constexpr int kFewJoin = 1024;
constexpr long kSliceChunks = 1024;  // chunks that are worth a slice (kFill / 4 slices and fewer: the last has more than 500)
template <int THREADS>
__global__ __launch_bounds__(THREADS) void embed_few_join_kernel(FewArgs a) {
    __shared__ double lds[THREADS / 16][17];
    const int tid = static_cast<int>(threadIdx.x), o = tid & 15, share = tid >> 4;
    const int from = static_cast<int>(blockIdx.y) * a.slice, to = min(a.chunks, from + a.slice);
    const long at = 16L * blockIdx.x + o, step = static_cast<long>(a.Vp) * a.Dp;  // of part
    double s = 0.0;
#pragma unroll 4
    for (int c = from + share; c < to; c += THREADS / 16) s += a.part[c * step + at];
    lds[share][o] = s;
    __syncthreads();
#pragma unroll
    for (int half = THREADS / 32; half > 0; half >>= 1) {
        if (share < half) lds[share][o] += lds[share + half][o];
        __syncthreads();
    }
    if (share != 0) return;
    s = lds[0][o];
    const float high = static_cast<float>(s);
    if (a.slices > 1) {
        a.part[from * step + at] = high;
        a.part[(from + 1) * step + at] = fabsf(high) < INFINITY ? static_cast<float>(s - static_cast<double>(high)) : 0.f;
        return;
    }
    const int v = static_cast<int>(at / a.Dp), d = static_cast<int>(at - static_cast<long>(v) * a.Dp);
    if (v < a.V && d < a.D) a.dtable[static_cast<long>(v) * a.D + d] = high * a.scale;
}
// What the slices left, one number a lane.
__global__ __launch_bounds__(kThreads) void embed_few_slices_kernel(FewArgs a) {
    const long at = static_cast<long>(blockIdx.x) * kThreads + threadIdx.x, step = static_cast<long>(a.Vp) * a.Dp;
    if (at >= step) return;
    double s = 0.0;
    for (int i = 0; i < a.slices; ++i) {
        const float* part = a.part + static_cast<long>(i) * a.slice * step + at;
        s += static_cast<double>(part[0]) + static_cast<double>(part[step]);
    }
    const int v = static_cast<int>(at / a.Dp), d = static_cast<int>(at - static_cast<long>(v) * a.Dp);
    if (v < a.V && d < a.D) a.dtable[static_cast<long>(v) * a.D + d] = static_cast<float>(s) * a.scale;
}

// ---- backward, many tokens: the positions in the order of their tokens ---------------------------------------------------------
// Keys are tokens, V for no token: those come last.  A pass of the sort takes up to 8 bits, in two launches: one counts the digits of
// each tile of keys; in the other each workgroup finds where its tile's keys go (from the counts of all tiles, which are few, or made
// into places by a launch between) and puts them there in their order.  These launches wait for memory most of the time: their other
// workgroups turn dy into rows and clear the gradient meanwhile.  (Counting the next pass's digits where the keys are put saves a
// launch, but a frequent token's are all counted in one place: 56 us for 160000 positions, of which 18000 have the same token.)
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
    int *counts, *totals;         // [tiles][kBins], [kBins]
    void* rows;                   // [M][8 * per_row]: dy's columns
    float* dtable;
    long zeros;                   // elements of dtable
    int pass, count, bits, tiles, per_lane, before;  // count: this launch counts; before: counts hold places
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
    __syncthreads();
    const long first = static_cast<long>(tile) * a.per_lane * kSort;
    for (int k = 0; k < a.per_lane; ++k) {
        const long m = first + k * kSort + tid;
        if (m < a.M) lds_add(&count[(key_at(a, static_cast<int>(m)) >> (a.pass * a.bits)) & (bins - 1)], 1);
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
    const int* counts = a.counts;
    const long first = static_cast<long>(tile) * a.per_lane * kSort + wave * (a.per_lane * kSeqWave) + lane;
    int key[kKeys], mine[kKeys], pos[kKeys];
#pragma unroll
    for (int k = 0; k < kKeys; ++k) {
        if (k >= a.per_lane) break;
        const int m = static_cast<int>(min(first + k * kSeqWave, a.M - 1L));
        key[k] = key_at(a, m);
        pos[k] = a.pass > 0 ? a.pos[(a.pass & 1) ^ 1][m] : m;
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
#pragma unroll 16
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
        if (to < 0 || to >= a.M || pos[k] < 0 || pos[k] >= a.M) continue;  // (never, as long as the tokens do not change meanwhile)
        a.keys[out][to] = key[k];
        a.pos[out][to] = pos[k];
    }
}

// Many tiles: counts into places.  A workgroup has 16 digits, 64 shares of the tiles each.
__global__ __launch_bounds__(kSort) void embed_places_kernel(SortArgs a) {
    __shared__ int sum[kSort / 16][16];
    const int tid = static_cast<int>(threadIdx.x), o = tid & 15, share = tid >> 4, digit = 16 * static_cast<int>(blockIdx.x) + o;
    int* counts = a.counts + digit;
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

// dy's columns as rows: with the sort and the clearing 49 us for 8 x 512 x 8192 bfloat16 and 32000 tokens, 200 MB
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
        if (a.count) count_digits(a, lds.sort.place[0]);
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
    float *head, *tail;      // [groups of chunks][per_row * 8]: what of a workgroup's rows belongs to a run that began before them, that goes on behind
    float* dtable;
    long sample_stride, stride;
    float scale;
    int D, L, V, M, per_row, chunk, first;
    int cols, teams, blocks;  // vectors of a row that a workgroup has, its lane groups, workgroups of a row
    Div31 by_blocks, by_L;
};

__device__ __forceinline__ void float_store8(float* row, int at, int end, const float (&v)[8], float scale) {
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = v[e] * scale;
    row_store8<false>(row, at, end, s);
}

// Bound by memory: 131 MB, half of them read again, in 18 us (8 x 512 x 8192, 32000 tokens).
// A workgroup has the chunks of kThreads / cols lane groups, cols of the vectors of a row each; their keys and positions, one behind the
// other, go through LDS, so that a lane's loads of rows wait for nothing else.
constexpr int kMostChunk = 32, kMostTeams = 64, kAheadRows = 8;
__device__ __forceinline__ void keep(f32x4 (&at)[2], const float (&v)[8]) {
    at[0] = f32x4{v[0], v[1], v[2], v[3]};
    at[1] = f32x4{v[4], v[5], v[6], v[7]};
}
// Adds to `sum` the heads of chunk t and of those behind it that its run goes on in, in 64 bits; returns the last one.
__device__ __forceinline__ int join_on(const f32x4 (*heads)[2], const int* passes, int at, int cols, int t, int last, float (&sum)[8]) {
    double s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = sum[e];
    for (;; ++t, at += cols) {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += static_cast<double>(heads[at][e >> 2][e & 3]);
        if (!passes[t] || t >= last) break;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = static_cast<float>(s[e]);
    return t;
}

// Where a sum goes and when is found for every row: the code for it is kept short (one kind of store, no call), because it stands
// kAheadRows times in the loop, and instructions come from memory as well (8 x 128 x 20000, 4096 tokens: 36 us with two kinds of
// stores for whole and cut vectors at either place, 13 so).
template <bool BF16, bool TURNED, bool WHOLE>
__global__ __launch_bounds__(kThreads) void embed_sums_kernel(SumArgs a) {
    using T = typename RowElem<BF16>::type;
    __shared__ int keys[kMostTeams * kMostChunk + 2], pos[kMostTeams * kMostChunk], passes[kMostTeams];
    __shared__ f32x4 heads[kThreads][2];
    const int tid = static_cast<int>(threadIdx.x), unit = static_cast<int>(blockIdx.x) + a.first, group = div31(unit, a.by_blocks), block = unit - group * a.blocks;
    const int team = tid / a.cols, col = block * a.cols + tid - team * a.cols;
    const int first = group * a.teams * a.chunk, rows = min(a.M - first, a.teams * a.chunk);
    for (int i = tid; i < rows + 2; i += kThreads) {  // the keys before and behind too
        const int m = first + i - 1;
        keys[i] = m >= 0 && m < a.M ? a.keys[m] : a.V;
        if (i < rows) pos[i] = a.pos[first + i];
    }
    __syncthreads();
    const bool mine = team < a.teams && team * a.chunk < rows && col < a.per_row;
    const int d = 8 * col, from = mine ? team * a.chunk : 0, to = mine ? min(rows, from + a.chunk) : 0, there = WHOLE ? 8 : min(8, a.D - d);
    const long side = static_cast<long>(group) * (8 * a.per_row) + d;
    int key = mine ? keys[1 + from] : a.V;
    bool began = mine && (first + from == 0 || keys[from] != key);  // the run at hand began in this chunk
    bool open = key < a.V;                                         // and is one
    bool came = open && !began;                                    // the chunk's first run began before it
    float sum[8] = {};
    const auto put = [&](float* o, float scale, bool all, const float (&v)[8]) {
        if constexpr (WHOLE) {
            *reinterpret_cast<seq_f32x4*>(o) = seq_f32x4{v[0] * scale, v[1] * scale, v[2] * scale, v[3] * scale};
            *reinterpret_cast<seq_f32x4*>(o + 4) = seq_f32x4{v[4] * scale, v[5] * scale, v[6] * scale, v[7] * scale};
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (all || e < there) o[e] = v[e] * scale;
        }
    };
#pragma unroll 1
    for (int i0 = from; i0 < to && open; i0 += kAheadRows) {
        Raw8<BF16> raw[kAheadRows];
#pragma unroll
        for (int j = 0; j < kAheadRows; ++j) {
            const int m = clampi(pos[min(i0 + j, to - 1)], 0, a.M - 1);
            if constexpr (TURNED) {
                raw[j] = raw8_inside<BF16>(static_cast<const T*>(a.rows) + m * a.stride, d);
            } else {
                const int n = div31(m, a.by_L), l = m - n * a.L;
                const T* row = static_cast<const T*>(a.rows) + n * a.sample_stride + l * a.stride;
                if constexpr (WHOLE) raw[j] = raw8_inside<BF16>(row, d);
                else raw[j] = raw8<BF16>(row, d, a.D);
            }
        }
#pragma unroll
        for (int j = 0; j < kAheadRows; ++j) {
            const int k = i0 + j < to ? keys[1 + i0 + j] : key;
            if (k != key && open) {
                if (began) put(a.dtable + static_cast<long>(key) * a.D + d, a.scale, false, sum);
                else keep(heads[tid], sum);
                open = k < a.V;
                key = k;
                began = true;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = 0.f;
            }
            float v[8];
            floats_of(raw[j], v);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += i0 + j < to ? v[e] : 0.f;
        }
    }
    // what of a run lies in several chunks of the workgroup is put together here
    const bool goes_on = open && first + to < a.M && keys[1 + to] == key;
    if (open && !began) keep(heads[tid], sum);
    const bool pass = came && !began && goes_on;  // the chunk lies within one run
    if (tid - team * a.cols == 0 && team < a.teams) passes[team] = pass;
    __syncthreads();
    if (!mine) return;
    const int last = (rows - 1) / a.chunk;  // the last chunk that is there
    if (came && team == 0) {
        float head[8] = {};
        join_on(heads, passes, tid, a.cols, 0, last, head);
        put(a.head + side, 1.f, true, head);
    }
    if (!open || !began) return;
    bool behind = goes_on;
    if (goes_on && team < last) {
        const int end = join_on(heads, passes, tid + a.cols, a.cols, team + 1, last, sum);
        behind = passes[end];
    }
    put(behind ? a.tail + side : a.dtable + static_cast<long>(key) * a.D + d, behind ? 1.f : a.scale, behind, sum);
}

// Runs that cross the rows of one workgroup, its chunk here: what the chunks behind the one where a run begins have of it is added to that one's,
// by that chunk's lane group
// where those are few, by the whole workgroup where a run is long.  A chain of trips through memory (7 us), which is why all that may be
// needed is loaded at once.
struct JoinArgs {
    const int* keys;
    const float *head, *tail;
    float* dtable;
    float scale;
    int D, V, M, per_row, chunk, chunks, first;
    int cols, teams;  // vectors of a row that a lane group takes at a time, lane groups of a workgroup
};
constexpr int kJoin = 256, kShort = 16;
// 8 columns of a chunk's share
__device__ __forceinline__ void share(const JoinArgs& a, int c, bool first, int d, float (&v)[8]) {
    row_load8_inside<false>((first ? a.tail : a.head) + static_cast<long>(c) * (8 * a.per_row), d, v);
}
__global__ __launch_bounds__(kJoin) void embed_join_kernel(JoinArgs a) {
    __shared__ double lds[4][kJoin];
    __shared__ int longs[kJoin];
    const int tid = static_cast<int>(threadIdx.x), team = tid / a.cols, lane = tid - team * a.cols, first = a.first + static_cast<int>(blockIdx.x) * a.teams;
    if (tid < a.teams) longs[tid] = 0;
    __syncthreads();
    const int chunk = first + team;
    if (team < a.teams && chunk < a.chunks - 1) {
        const long behind = (static_cast<long>(chunk) + 1) * a.chunk, from = behind - a.chunk;
        // (all that may be needed is on its way at once)
        const int key = a.keys[behind - 1], next = a.keys[behind], begin = a.keys[from], before = a.keys[max(from, 1L) - 1];
        int on_key[kShort];
#pragma unroll
        for (int i = 0; i < kShort; ++i) on_key[i] = a.keys[min((chunk + i + 2L) * a.chunk, a.M - 1L)];
        float ahead[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) share(a, min(chunk + i, a.chunks - 1), i == 0, 8 * lane, ahead[i]);
        const bool earlier = begin == key && from > 0 && before == key;
        if (key >= 0 && key < a.V && next == key && !earlier) {
            bool on[kShort];
#pragma unroll
            for (int i = 0; i < kShort; ++i) on[i] = (chunk + i + 2L) * a.chunk < a.M && on_key[i] == key;
            int many = 1;  // chunks that it goes on in; kShort + 1: that many or more
#pragma unroll
            for (int i = 0; i < kShort; ++i) many += many == i + 1 && on[i];
            if (many > kShort) {
                if (lane == 0) longs[team] = 1;
            } else {
                for (int c0 = lane; c0 < a.per_row; c0 += a.cols) {
                    double sum[8] = {};
                    for (int c = 0; c <= many; c += 4) {  // four shares on their way at a time
                        if (c > 0 || c0 != lane) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) share(a, min(chunk + min(c + i, many), a.chunks - 1), c + i == 0, 8 * c0, ahead[i]);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int e = 0; e < 8; ++e) sum[e] += c + i <= many ? static_cast<double>(ahead[i][e]) : 0.0;
                    }
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(sum[e]);
                    float_store8(a.dtable + static_cast<long>(key) * a.D, 8 * c0, a.D, v, a.scale);
                }
            }
        }
    }
    __syncthreads();
    for (int t = 0; t < a.teams; ++t) {
        if (!longs[t]) continue;
        const int begin = first + t, key = clampi(a.keys[(static_cast<long>(begin) + 1) * a.chunk - 1], 0, a.V - 1);
        int lo = begin + kShort, hi = a.chunks;  // its last chunk is lo or one up to hi - 1
        while (hi - lo > 1) {  // a lane looks at each 64th of them
            const int step = (hi - lo + kSeqWave - 1) / kSeqWave, at = lo + (tid & (kSeqWave - 1)) * step;
            const int on = max(1, popcount64(wave_ballot(at < hi && a.keys[static_cast<long>(at) * a.chunk] == key)));
            lo += (on - 1) * step;
            hi = min(hi, lo + step);
        }
        for (int c0 = 0; c0 < a.per_row; c0 += a.cols) {
            const bool there = team < a.teams && c0 + lane < a.per_row;
            double sum[8] = {};
            if (there) {
#pragma unroll 4
                for (int c = begin + team; c <= min(lo, a.chunks - 1); c += a.teams) {
                    float v[8];
                    share(a, c, c == begin, 8 * (c0 + lane), v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[e] += static_cast<double>(v[e]);
                }
            }
            int half = 1;
            while (half < a.teams) half *= 2;
#pragma unroll
            for (int e0 = 0; e0 < 8; e0 += 4) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < 4; ++e) lds[e][tid] = sum[e0 + e];
                for (int h = half >> 1; h > 0; h >>= 1) {
                    __syncthreads();
                    if (team < h && team + h < a.teams) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) lds[e][tid] += lds[e][tid + h * a.cols];
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e0 + e] = lds[e][tid];
            }
            if (team == 0 && there) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(sum[e]);
                float_store8(a.dtable + static_cast<long>(key) * a.D, 8 * (c0 + lane), a.D, v, a.scale);
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
    // A few channels leave most lanes of a tile's loads idle (16 x 15 x 60000 bfloat16, 5 tokens 11.7 us for 17.8 by tiles, 1000 tokens 19 for 24; 12 x
    // 49 x 4999 float, 256 tokens 8.2 for 8.3); tiles are faster for more (8 x 128 x 20000 bfloat16, 4 tokens 11.5 for 14.6, 1000 tokens 11 for 22).
    if (p->V < kFewRows && (p->D <= 16 || (p->D <= 48 && p->V <= 256))) {
        // as many channels a workgroup as leave enough workgroups, and room for several beside each other
        a.tiles = cdiv(p->L, 8 * kThreads);
        a.per_row = 16;
        while (a.per_row > 4 && (static_cast<long>(p->N) * a.tiles * cdiv(p->D, a.per_row) < kFill || (p->V + 1L) * a.per_row > kFewElements)) a.per_row /= 2;
        a.blocks = cdiv(p->D, a.per_row);
        lds = 2 * 8 * kThreads + static_cast<size_t>(p->V + 1) * a.per_row * (BF16 ? 2 : 4);
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
    int VB, DB, Vp, Dp, vgroups, dgroups, block, chunk, samples, per_sample, chunks;  // block: positions that a workgroup takes at a time
    size_t bytes;
};
FewPlan few_plan(int N, int D, int L, int V, int dtype) {
    FewPlan p{};
    p.Vp = static_cast<int>(round_up(V, 16));
    p.Dp = static_cast<int>(round_up(D, 16));
    p.VB = p.Vp <= 16 ? 1 : 4;
    p.DB = p.Dp <= 16 ? 1 : 4;
    p.vgroups = cdiv(p.Vp, 16 * p.VB);
    p.dgroups = cdiv(p.Dp, 16 * p.DB);
    // enough workgroups to fill the chip once (three of the largest tiles fit a compute unit), but no more partial sums than dy has
    // numbers, as long as a wave's sums in float stay short; in whole blocks
    const long M = static_cast<long>(N) * L, step = 32L * kWaves * (dtype == CONV1D_BF16 ? (p.DB == 1 ? kU<true, 1> : kU<true, 4>) : (p.DB == 1 ? kU<false, 1> : kU<false, 4>));
    p.block = static_cast<int>(step);
    const long want = (p.VB * p.DB == 16 ? 3 * kFill / 8 : kFill) / (static_cast<long>(p.vgroups) * p.dgroups);
    long chunk = want > 1 ? (M + want - 1) / want : M;
    if (chunk < p.Vp) chunk = p.Vp;
    if (chunk > kMostSteps * 32L * kWaves) chunk = kMostSteps * 32L * kWaves;
    if (chunk >= 2L * L) {
        // (a workgroup goes through its samples one behind the other, in blocks of their own: no more than a few for the partial sums' sake)
        const long share = want > 1 ? (M / want + L - 1) / L : N, most = share > 4 ? share : 4;
        p.samples = static_cast<int>(chunk / L < N ? chunk / L : N);
        if (p.samples > most) p.samples = static_cast<int>(most);
        // the steps of a sample that the first wave has
        const int of = static_cast<int>(step / (32 * kWaves)), last = cdiv(static_cast<int>(L % step), 32);
        const int steps = static_cast<int>(L / step) * of + (last < of ? last : of);
        if (p.samples * steps > kMostSteps) p.samples = kMostSteps / steps;
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
// Whether the gradient is taken as a product, by what the two take, in us.
// Product: 12, 6.5e-9 for each token x channel x position of whole blocks (in tiles of 16; floats 1.7e-8), its partial sums' way to memory and
// back, 5e-4 for each workgroup that joins 16 of them, and the blocks that a sample's end cuts: their numbers are loaded one by one, and a
// workgroup goes through its samples in turn.
// Sort: 11, 20 more up to 20000 positions, 10 a pass, clearing the gradient, and the larger of 6.5e-5 a position and 5e-3 a tile that is turned; what
// does not stay in the caches goes to memory and back.
// Measured, product and sort: 8 x 512 x 8192 bfloat16 16 tokens 21 and 49, 128 tokens 40 and 46, 256 tokens 65 and 55; 8 x 128 x 20000 256 tokens
// 43 and 53, 512 tokens 70 and 53; 12 x 49 x 4999 float 256 tokens 32 and 52, 1024 tokens 68 and 51; 16 x 15 x 60000 512 tokens 73 and 104, 1024
// tokens 121 and 106.  Short samples: 20000 x 8 x 16, 600 tokens 1396 and 112; 20000 x 64 x 16, 64 tokens 580 and 114; 4000 x 64 x 4, 64 tokens
// 64 and 42; 1000 x 64 x 200, 64 tokens 36 and 40; 16 x 64 x 100, 64 tokens 14 and 21; 20000 x 16 x 2 float, 16 tokens 53 and 169.  Many tokens, few
// positions: 2 x 110 x 2 float, 31203 tokens 132 and 20; 1 x 55 x 26 bfloat16, 23921 tokens 65 and 22.  (Of 641 sizes the slower way was taken at 182
// for more than 1.2 times the time, up to 12.5, by positions alone, now at 47, up to 2.7.)
bool is_few(int N, int D, int L, int V, int dtype, bool turned) {
    if (!turned || V > kFewTokens) return false;
    const FewPlan p = few_plan(N, D, L, V, dtype);
    const bool bf16 = dtype == CONV1D_BF16;
    const double M = static_cast<double>(N) * L, tile = static_cast<double>(p.Vp) * p.Dp, us_a_byte = 1 / 5.2e6;
    const double whole = M - static_cast<double>(N) * (L % p.block), cut = L % p.block ? static_cast<double>(N) * p.vgroups * p.dgroups : 0;
    const double ends = cut * (p.DB == 1 ? (bf16 ? 8e-3 : 4e-3) : bf16 ? 28e-3 : 15e-3) * (L < 16 ? (L + 8) / 24.0 : 1.0), turns = 3.0 * (p.samples - 1);
    const double product = 12 + whole * tile * (bf16 ? 6.5e-9 : 1.7e-8) + 8 * tile * p.chunks * us_a_byte + 5e-4 * tile / 16 + (ends > turns ? ends : turns);
    const double turned_tiles = static_cast<double>(N) * cdiv(L, kTurn / tile_channels(D)) * cdiv(D, tile_channels(D));
    const double sorts = 6.5e-5 * M > 5e-3 * turned_tiles ? 6.5e-5 * M : 5e-3 * turned_tiles, beyond = M * D * (bf16 ? 2 : 4) - 32e6;
    const double sort = 11 + (M < 20000 ? M / 1000 : 20) + (V < 256 ? 10 : V < 65536 ? 20 : 30) + sorts + 4.0 * V * D * us_a_byte +
                        (beyond > 0 ? 2 * beyond * us_a_byte : 0);
    if (product > sort) return false;
    return static_cast<long>(p.chunks) * p.vgroups * p.dgroups <= kMostBlocks && static_cast<long>(p.Vp) * p.Dp / 16 <= kMostBlocks;
}

struct Plan {
    int M, bits, passes, tiles, per_lane, chunk, per_row, cols, teams, span, spans;  // span: rows of a workgroup that adds
    size_t keys[2], pos[2], counts, totals, rows, head, tail, bytes;
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
    p.chunk = static_cast<long>(p.M) * p.per_row < 16L * kFill * kSeqWave ? 16 : kMostChunk;
    p.cols = p.per_row < kThreads ? p.per_row : kThreads;
    p.teams = kThreads / p.cols < kMostTeams ? kThreads / p.cols : kMostTeams;
    p.span = p.teams * p.chunk;
    p.spans = cdiv(p.M, p.span);
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
    p.counts = take(4 * static_cast<size_t>(p.tiles) * kBins);
    p.totals = take(4 * static_cast<size_t>(kBins));
    p.rows = take(turned ? M * width * (dtype == CONV1D_BF16 ? 2 : 4) : 0);
    p.head = take(4 * width * p.spans);
    p.tail = take(4 * width * p.spans);
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
    // few numbers: large workgroups, and of many chunks several rows of them (64 x 16 numbers of 131072: 2.61 ms in all for 2.86)
    const long joins = static_cast<long>(plan.Vp) * plan.Dp / 16;
    const bool large = joins < kFill / 8;
    const long rows = plan.chunks / kSliceChunks < kFill / 4 / joins ? plan.chunks / kSliceChunks : kFill / 4 / joins;
    a.slices = rows > 1 ? static_cast<int>(rows) : 1;
    a.slice = cdiv(plan.chunks, a.slices);
    a.slices = cdiv(plan.chunks, a.slice);
    const hipError_t j = launch_kernel(large ? embed_few_join_kernel<kFewJoin> : embed_few_join_kernel<kThreads>, dim3(static_cast<unsigned>(joins), static_cast<unsigned>(a.slices)),
                                       dim3(large ? kFewJoin : kThreads), 0, st, a);
    if (j != hipSuccess || a.slices == 1) return j;
    return launch_kernel(embed_few_slices_kernel, dim3(static_cast<unsigned>(cdiv(16 * joins, kThreads))), dim3(kThreads), 0, st, a);
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
    a.rows = ws + plan.rows;
    a.dtable = dtable;
    a.zeros = static_cast<long>(p->V) * p->D;
    a.bits = plan.bits; a.tiles = plan.tiles; a.per_lane = plan.per_lane; a.per_row = plan.per_row;
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
    for (int launch = 0; launch < 2 * plan.passes; ++launch) {
        a.pass = launch / 2;
        a.count = launch % 2 == 0;
        hipError_t e = hipSuccess;
        if (!a.count && a.before) e = launch_kernel(embed_places_kernel, dim3(kBins / 16), dim3(kSort), 0, st, a);
        // the other work in equal shares, what is too much for a grid in grids of its own
        const long upto = jobs * (launch + 1) / (2 * plan.passes);
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
    s.keys = a.keys[last]; s.pos = a.pos[last];
    s.head = reinterpret_cast<float*>(ws + plan.head);
    s.tail = reinterpret_cast<float*>(ws + plan.tail);
    s.dtable = dtable;
    s.sample_stride = dy_sn;
    s.stride = turned ? 8L * plan.per_row : dy_sl;
    s.scale = p->scale; s.D = p->D; s.L = p->L; s.V = p->V; s.M = plan.M; s.per_row = plan.per_row; s.chunk = plan.chunk;
    s.by_L = make_div31(p->L);
    s.cols = plan.cols; s.teams = plan.teams;
    s.blocks = cdiv(plan.per_row, s.cols);
    s.by_blocks = make_div31(s.blocks);
    const long units = static_cast<long>(plan.spans) * s.blocks;
    if (units > kMostItems) return hipErrorInvalidValue;
    void (*sums)(SumArgs) = p->D % 8 ? (turned ? embed_sums_kernel<BF16, true, false> : embed_sums_kernel<BF16, false, false>)
                                     : (turned ? embed_sums_kernel<BF16, true, true> : embed_sums_kernel<BF16, false, true>);
    for (long u = 0; u < units; u += kMostBlocks) {
        s.first = static_cast<int>(u);
        const hipError_t e = launch_kernel(sums, dim3(static_cast<unsigned>(units - u < kMostBlocks ? units - u : kMostBlocks)), dim3(kThreads), 0, st, s);
        if (e != hipSuccess) return e;
    }
    if (plan.spans < 2) return hipSuccess;
    JoinArgs j{};
    j.keys = s.keys; j.head = s.head; j.tail = s.tail; j.dtable = dtable; j.scale = p->scale;
    j.D = p->D; j.V = p->V; j.M = plan.M; j.per_row = plan.per_row; j.chunk = plan.span; j.chunks = plan.spans;
    j.cols = plan.per_row < kJoin ? plan.per_row : kJoin;
    j.teams = kJoin / j.cols;
    return launch_kernel(embed_join_kernel, dim3(static_cast<unsigned>(cdiv(plan.spans - 1, j.teams))), dim3(kJoin), 0, st, j);
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

size_t conv1d_embed_bwd_workspace_bytes(int N, int D, int L, int V, int dtype, long dy_sd, long dy_sl) {
    if (N < 1 || D < 1 || L < 1 || V < 1 || !sizes_ok(N, D, L, V) || (dtype != CONV1D_FP32 && dtype != CONV1D_BF16)) return 0;
    const bool turned = is_turned(D, L, dy_sd, dy_sl);
    return is_few(N, D, L, V, dtype, turned) ? few_plan(N, D, L, V, dtype).bytes : plan_of(N, D, L, V, dtype, turned).bytes;
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
    if (is_few(p->N, p->D, p->L, p->V, p->dtype, turned)) {
        const FewPlan plan = few_plan(p->N, p->D, p->L, p->V, p->dtype);
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
