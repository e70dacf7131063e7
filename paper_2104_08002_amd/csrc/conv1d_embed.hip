// Embedding lookup with scaling, and its gradient by sorted tokens.
//   y[n][d][l] = scale table[tokens[n][l]][d],   dtable[v][d] = scale sum over (n, l) with tokens[n][l] = v of dy[n][d][l]
// Bound by memory.  Where positions are contiguous, tiles of positions and channels are turned in LDS: rows of the table are read
// and written along the channels, y and dy along the positions.
// The gradient adds the same positions in the same order in every run: the positions are sorted by their token (a stable radix
// sort, least digit first), the gradient's columns are written as rows in that order, each lane group adds a chunk of neighbouring
// rows in float and writes the runs that lie in its chunk; what of a run lies in several chunks is joined in 64 bits.
#include "conv1d_blocks.h"

namespace conv1d {
namespace {

constexpr int kThreads = 256;

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

// ---- the positions in the order of their tokens ---------------------------------------------------------------------------
// Keys are tokens, V for no token: those come last.  A pass of the sort takes up to kDigit bits: each workgroup counts the digits of its
// tile, one launch turns each digit's counts into places, and each workgroup puts its tile's keys there, in their order.
constexpr int kDigit = 8, kBins = 1 << kDigit;
constexpr int kKeys = 8, kSortTile = kThreads * kKeys;  // a lane, a workgroup

struct SortArgs {
    const void* tokens;
    const int* lengths;
    long tok_sn;
    int wide, L, V, M;
    Div31 by_L;
    const int *keys_in, *pos_in;  // nullptr: the tokens themselves
    int *keys_out, *pos_out, *rank;  // rank (last pass): where each position went
    int *counts, *totals;         // [bins][tiles], [bins]
    int shift, bins, tiles;
};

__device__ __forceinline__ int key_at(const SortArgs& a, int m) {
    if (a.keys_in) return a.keys_in[m];
    const int n = div31(m, a.by_L), l = m - n * a.L;
    const int t = token_at(a.tokens, a.wide, n, a.tok_sn, l, seq_length(a.lengths, n, a.L), a.V);
    return t < 0 ? a.V : t;
}

__global__ __launch_bounds__(kThreads) void embed_count_kernel(SortArgs a) {
    __shared__ int count[kBins];
    const int tid = static_cast<int>(threadIdx.x);
    count[tid] = 0;
    __syncthreads();
    const long first = static_cast<long>(blockIdx.x) * kSortTile;
#pragma unroll
    for (int k = 0; k < kKeys; ++k) {
        const long m = first + k * kThreads + tid;
        if (m < a.M) lds_add(&count[(key_at(a, static_cast<int>(m)) >> a.shift) & (a.bins - 1)], 1);
    }
    __syncthreads();
    if (tid < a.bins) a.counts[static_cast<long>(tid) * a.tiles + blockIdx.x] = count[tid];
}

// exclusive sums over a workgroup; `all` gets the sum
__device__ __forceinline__ int block_before(int v, int* lds, int& all) {
    const int lane = threadIdx.x & (kSeqWave - 1), wave = threadIdx.x >> 6;
    int sum = v;
#pragma unroll
    for (int m = 1; m < kSeqWave; m <<= 1) {
        const int o = lane_up(sum, m);
        sum += lane >= m ? o : 0;
    }
    __syncthreads();
    if (lane == kSeqWave - 1) lds[wave] = sum;
    __syncthreads();
    int before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kThreads / kSeqWave; ++w) {
        before += w < wave ? lds[w] : 0;
        all += lds[w];
    }
    return before + sum - v;
}

// one workgroup a digit: how many of its keys lie in the tiles before
__global__ __launch_bounds__(kThreads) void embed_places_kernel(SortArgs a) {
    __shared__ int lds[kThreads / kSeqWave];
    int* row = a.counts + static_cast<long>(blockIdx.x) * a.tiles;
    int before = 0;
    for (int t0 = 0; t0 < a.tiles; t0 += kThreads) {
        const int t = t0 + static_cast<int>(threadIdx.x), v = t < a.tiles ? row[t] : 0;
        int all;
        const int at = block_before(v, lds, all);
        if (t < a.tiles) row[t] = before + at;
        before += all;
    }
    if (threadIdx.x == 0) a.totals[blockIdx.x] = before;
}

__global__ __launch_bounds__(kThreads) void embed_put_kernel(SortArgs a) {
    constexpr int W = kThreads / kSeqWave;
    __shared__ int place[W][kBins], lds[W];
    const int tid = static_cast<int>(threadIdx.x), lane = tid & (kSeqWave - 1), wave = tid >> 6;
#pragma unroll
    for (int w = 0; w < W; ++w) place[w][tid] = 0;
    __syncthreads();
    // a wave has kKeys * 64 neighbouring keys; lanes with the same digit take their places in the order of the lanes
    const long first = static_cast<long>(blockIdx.x) * kSortTile + wave * (kKeys * kSeqWave) + lane;
    int key[kKeys], mine[kKeys];
#pragma unroll
    for (int k = 0; k < kKeys; ++k) {
        const long m = first + k * kSeqWave;
        key[k] = key_at(a, static_cast<int>(m < a.M ? m : a.M - 1));
    }
#pragma unroll
    for (int k = 0; k < kKeys; ++k) {
        const bool there = first + k * kSeqWave < a.M;
        const int digit = (key[k] >> a.shift) & (a.bins - 1);
        unsigned long same = wave_ballot(there);
        for (int bit = 1; bit < a.bins; bit <<= 1) {
            const bool set = digit & bit;
            const unsigned long with = wave_ballot(set);
            same &= set ? with : ~with;
        }
        const int leader = there ? first_bit(same) : lane, before = popcount64(same & ((1UL << lane) - 1));
        int at = 0;
        if (there && lane == leader) at = lds_add(&place[wave][digit], popcount64(same));
        mine[k] = lane_from(at, leader) + before;
    }
    __syncthreads();
    int all;
    int base = block_before(tid < a.bins ? a.totals[tid] : 0, lds, all);
    if (tid < a.bins) {
        base += a.counts[static_cast<long>(tid) * a.tiles + blockIdx.x];
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const int n = place[w][tid];
            place[w][tid] = base;
            base += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kKeys; ++k) {
        const long m = first + k * kSeqWave;
        if (m >= a.M) continue;
        const int to = place[wave][(key[k] >> a.shift) & (a.bins - 1)] + mine[k];
        const int pos = a.pos_in ? a.pos_in[m] : static_cast<int>(m);
        if (to < 0 || to >= a.M || pos < 0 || pos >= a.M) continue;  // (never, as long as the tokens do not change meanwhile)
        a.keys_out[to] = key[k];
        a.pos_out[to] = pos;
        if (a.rank) a.rank[pos] = to;
    }
}

// ---- backward: rows in that order -------------------------------------------------------------------------------------
struct TurnArgs {
    const void* dy;
    const int *rank, *keys;
    const int* lengths;
    void* rows;            // [M][per_row * 8]
    long dy_sn, dy_sd, first;
    int D, L, V, M, per_row, tiles, blocks;
    Div31 by_blocks, by_tiles;
};

template <bool BF16, int DT>
__global__ __launch_bounds__(kThreads) void embed_rows_kernel(TurnArgs a) {
    using T = typename RowElem<BF16>::type;
    constexpr int P = kTile / DT, S = P + 2, NV = DT / 8;
    __shared__ T lds[DT * S];
    __shared__ int to[P];
    const int unit = static_cast<int>(blockIdx.x) + static_cast<int>(a.first);
    const int nt = div31(unit, a.by_blocks), d0 = (unit - nt * a.blocks) * DT, n = div31(nt, a.by_tiles), l0 = (nt - n * a.tiles) * P;
    const int tid = static_cast<int>(threadIdx.x), len = seq_length(a.lengths, n, a.L), many = min(DT, a.D - d0);
    if (l0 >= len) return;
    for (int p = tid; p < P; p += kThreads) {
        int r = -1;
        if (l0 + p < len) {
            r = a.rank[static_cast<long>(n) * a.L + l0 + p];
            if (r < 0 || r >= a.M || a.keys[r] >= a.V) r = -1;
        }
        to[p] = r;
    }
    const T* dy = static_cast<const T*>(a.dy) + n * a.dy_sn;
#pragma unroll 4
    for (int i = tid; i < DT * (P / 8); i += kThreads) {
        const int d = i / (P / 8), p = 8 * (i % (P / 8));
        if (d >= many) {
            if (d < ((many + 7) & ~7)) {
#pragma unroll
                for (int e = 0; e < 8; ++e) lds[d * S + p + e] = 0;
            }
            continue;
        }
        float v[8];
        row_load8<BF16>(dy + (d0 + d) * a.dy_sd, l0 + p, len, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) store_elem<BF16>(lds, d * S + p + e, v[e]);
    }
    __syncthreads();
#pragma unroll 4
    for (int i = tid; i < P * NV; i += kThreads) {
        const int p = i / NV, d = 8 * (i % NV), r = to[p];
        if (d >= many || static_cast<unsigned>(r) >= static_cast<unsigned>(a.M)) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = load_elem<BF16>(lds, (d + e) * S + p);
        row_store8<BF16>(static_cast<T*>(a.rows) + static_cast<long>(r) * (8 * a.per_row) + d0, d, d + 8, v);
    }
}

// ---- backward: sums of runs -------------------------------------------------------------------------------------------
constexpr int kChunk = 32;  // rows a lane group adds

struct SumArgs {
    const void* rows;        // in the sorted order, per_row * 8 elements apart; or dy, through pos
    const int *keys, *pos;
    float *head, *tail;      // [chunks][per_row * 8]: what of a chunk belongs to a run that began before it, that goes on behind it
    float* dtable;
    long dy_sn, dy_sl;
    float scale;
    int D, L, V, M, per_row, chunks, first, items, sums, zeros, first_row;  // sums, zeros: workgroups that add chunks, that clear rows
    Div31 by_row, by_L;
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

__device__ __forceinline__ void float_store8(float* row, int at, int end, const float (&v)[8], float scale) {
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = v[e] * scale;
    row_store8<false>(row, at, end, s);
}

template <bool BF16, bool BY_POS>
__global__ __launch_bounds__(kThreads) void embed_sums_kernel(SumArgs a) {
    using T = typename RowElem<BF16>::type;
    if (static_cast<int>(blockIdx.x) >= a.sums) {  // rows of tokens that are not there
        const int i = (static_cast<int>(blockIdx.x) - a.sums) * kThreads + static_cast<int>(threadIdx.x), of = div31(i, a.by_row), v = a.first_row + of;
        if (v >= a.V || i >= a.zeros) return;
        const int at = place_of(a.keys, a.M, v);
        if (at < a.M && a.keys[at] == v) return;
        const float none[8] = {};
        float_store8(a.dtable + static_cast<long>(v) * a.D, 8 * (i - of * a.per_row), a.D, none, 0.f);
        return;
    }
    const int item = static_cast<int>(blockIdx.x) * kThreads + static_cast<int>(threadIdx.x);
    if (item >= a.items) return;
    const int of = div31(item, a.by_row), chunk = a.first + of, d = 8 * (item - of * a.per_row);
    const int from = chunk * kChunk, to = static_cast<int>(min(static_cast<long>(a.M), static_cast<long>(from) + kChunk));
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
            const int i = min(i0 + j, a.M - 1);
            k[j] = a.keys[i];
            if constexpr (BY_POS) {
                const int m = a.pos[i], n = div31(m, a.by_L), l = m - n * a.L;
                row_load8<BF16>(static_cast<const T*>(a.rows) + n * a.dy_sn + l * a.dy_sl, d, a.D, v[j]);
            } else {
                row_load8_inside<BF16>(static_cast<const T*>(a.rows) + static_cast<long>(i) * width, d, v[j]);
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
    const bool goes_on = to < a.M && a.keys[to] == key;
    if (!began) float_store8(a.head + static_cast<long>(chunk) * width, d, width, sum, 1.f);
    else if (goes_on) float_store8(a.tail + static_cast<long>(chunk) * width, d, width, sum, 1.f);
    else float_store8(a.dtable + static_cast<long>(key) * a.D, d, a.D, sum, a.scale);
}

// One workgroup a chunk whose last run goes on: what the chunks behind it have of that run is added to it.
struct JoinArgs {
    const int* keys;
    const float *head, *tail;
    float* dtable;
    float scale;
    int D, V, M, per_row, chunks, first;
};
__global__ __launch_bounds__(kThreads) void embed_join_kernel(JoinArgs a) {
    __shared__ double lds[kThreads][8];
    const int chunk = a.first + static_cast<int>(blockIdx.x);
    const long behind = (static_cast<long>(chunk) + 1) * kChunk;
    if (behind >= a.M) return;
    const int key = a.keys[behind - 1], from = chunk * kChunk;
    if (key >= a.V || a.keys[behind] != key) return;
    if (a.keys[from] == key && from > 0 && a.keys[from - 1] == key) return;  // it began in an earlier chunk
    const int last = (place_of(a.keys, a.M, key + 1) - 1) / kChunk;          // the chunk where it ends
    const int tid = static_cast<int>(threadIdx.x), width = 8 * a.per_row;
    const int cols = min(a.per_row, kThreads), teams = kThreads / cols, team = tid / cols;
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

struct Plan {
    int M, bits, passes, tiles, chunks, per_row;
    size_t keys[2], pos[2], rank, counts, totals, rows, head, tail, bytes;
};
Plan plan_of(int N, int D, int L, int V, int dtype, bool turned) {
    Plan p{};
    p.M = N * L;
    int bits = 1;
    while (bits < 31 && (1L << bits) <= V) ++bits;  // the keys 0 ... V
    p.passes = (bits + kDigit - 1) / kDigit;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.tiles = cdiv(p.M, kSortTile);
    p.chunks = cdiv(p.M, kChunk);
    p.per_row = (D + 7) / 8;
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
    p.rank = take(4 * M);
    p.counts = take(4 * static_cast<size_t>(p.tiles) << p.bits);
    p.totals = take(4 * static_cast<size_t>(kBins));
    p.rows = take(turned ? M * width * (dtype == CONV1D_BF16 ? 2 : 4) : 0);
    p.head = take(4 * width * p.chunks);
    p.tail = take(4 * width * p.chunks);
    p.bytes = at;
    return p;
}

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
    const int DT = tile_channels(p->D);
    a.tiles = cdiv(p->L, kTile / DT);
    a.blocks = cdiv(p->D, DT);
    a.by_tiles = make_div31(a.tiles);
    a.by_blocks = make_div31(a.blocks);
    const long units = static_cast<long>(p->N) * a.tiles * a.blocks, most = kSeqMostThreads / kThreads - 1;
    if (units > kMostItems) return hipErrorInvalidValue;
    for (long u = 0; u < units; u += most) {
        a.first = u;
        const long some = units - u < most ? units - u : most;
        const hipError_t e = launch_kernel(DT == 16 ? embed_turn_kernel<BF16, 16> : embed_turn_kernel<BF16, 64>, dim3(static_cast<unsigned>(some)), dim3(kThreads),
                                           0, st, a);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t sort_tokens(const conv1d_embed_t* p, const Plan& plan, char* ws, int*& keys, int*& pos, hipStream_t st) {
    SortArgs a{};
    a.tokens = p->tokens; a.lengths = p->lengths; a.tok_sn = p->tok_sn;
    a.wide = p->flags & CONV1D_EMBED_TOKENS64; a.L = p->L; a.V = p->V; a.M = plan.M;
    a.by_L = make_div31(p->L);
    a.counts = reinterpret_cast<int*>(ws + plan.counts);
    a.totals = reinterpret_cast<int*>(ws + plan.totals);
    a.bins = 1 << plan.bits;
    a.tiles = plan.tiles;
    for (int pass = 0; pass < plan.passes; ++pass) {
        a.shift = pass * plan.bits;
        a.keys_in = keys;
        a.pos_in = pos;
        keys = a.keys_out = reinterpret_cast<int*>(ws + plan.keys[pass & 1]);
        pos = a.pos_out = reinterpret_cast<int*>(ws + plan.pos[pass & 1]);
        a.rank = pass == plan.passes - 1 ? reinterpret_cast<int*>(ws + plan.rank) : nullptr;
        const dim3 tiles(static_cast<unsigned>(plan.tiles));
        hipError_t e = launch_kernel(embed_count_kernel, tiles, dim3(kThreads), 0, st, a);
        if (e == hipSuccess) e = launch_kernel(embed_places_kernel, dim3(static_cast<unsigned>(a.bins)), dim3(kThreads), 0, st, a);
        if (e == hipSuccess) e = launch_kernel(embed_put_kernel, tiles, dim3(kThreads), 0, st, a);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <bool BF16>
hipError_t gradient(const conv1d_embed_t* p, const void* dy, long dy_sn, long dy_sd, long dy_sl, float* dtable, bool turned, const Plan& plan, char* ws,
                    hipStream_t st) {
    int *keys = nullptr, *pos = nullptr;
    hipError_t e = sort_tokens(p, plan, ws, keys, pos, st);
    if (e != hipSuccess) return e;
    if (turned) {
        TurnArgs t{};
        t.dy = dy; t.keys = keys; t.lengths = p->lengths; t.rows = ws + plan.rows;
        t.rank = reinterpret_cast<int*>(ws + plan.rank);
        t.dy_sn = dy_sn; t.dy_sd = dy_sd;
        t.D = p->D; t.L = p->L; t.V = p->V; t.M = plan.M; t.per_row = plan.per_row;
        const int DT = tile_channels(p->D);
        t.tiles = cdiv(p->L, kTile / DT);
        t.blocks = cdiv(p->D, DT);
        t.by_tiles = make_div31(t.tiles);
        t.by_blocks = make_div31(t.blocks);
        const long units = static_cast<long>(p->N) * t.tiles * t.blocks, most = kSeqMostThreads / kThreads - 1;
        if (units > kMostItems) return hipErrorInvalidValue;
        for (long u = 0; u < units; u += most) {
            t.first = u;
            const long some = units - u < most ? units - u : most;
            e = launch_kernel(DT == 16 ? embed_rows_kernel<BF16, 16> : embed_rows_kernel<BF16, 64>, dim3(static_cast<unsigned>(some)), dim3(kThreads), 0, st, t);
            if (e != hipSuccess) return e;
        }
    }
    SumArgs s{};
    s.rows = turned ? static_cast<const void*>(ws + plan.rows) : dy;
    s.keys = keys; s.pos = pos;
    s.head = reinterpret_cast<float*>(ws + plan.head);
    s.tail = reinterpret_cast<float*>(ws + plan.tail);
    s.dtable = dtable; s.dy_sn = dy_sn; s.dy_sl = dy_sl;
    s.scale = p->scale; s.D = p->D; s.L = p->L; s.V = p->V; s.M = plan.M; s.per_row = plan.per_row; s.chunks = plan.chunks;
    s.by_row = make_div31(plan.per_row);
    s.by_L = make_div31(p->L);
    // half a launch's workgroups for chunks, half for rows to clear
    const long most = kMostItems / 2 / plan.per_row;
    void (*sums)(SumArgs) = turned ? embed_sums_kernel<BF16, false> : embed_sums_kernel<BF16, true>;
    for (long c = 0, v = 0; c < plan.chunks || v < p->V; c += most, v += most) {
        const long cn = c < plan.chunks ? (plan.chunks - c < most ? plan.chunks - c : most) : 0, vn = v < p->V ? (p->V - v < most ? p->V - v : most) : 0;
        s.first = static_cast<int>(c < plan.chunks ? c : 0);
        s.first_row = static_cast<int>(v < p->V ? v : 0);
        s.items = static_cast<int>(cn * plan.per_row);
        s.zeros = static_cast<int>(vn * plan.per_row);
        s.sums = cdiv(s.items, kThreads);
        e = launch_kernel(sums, dim3(static_cast<unsigned>(s.sums + cdiv(s.zeros, kThreads))), dim3(kThreads), 0, st, s);
        if (e != hipSuccess) return e;
    }
    if (plan.chunks < 2) return hipSuccess;
    JoinArgs j{};
    j.keys = keys; j.head = s.head; j.tail = s.tail; j.dtable = dtable; j.scale = p->scale;
    j.D = p->D; j.V = p->V; j.M = plan.M; j.per_row = plan.per_row; j.chunks = plan.chunks;
    const long blocks = plan.chunks - 1, room = kSeqMostThreads / kThreads - 1;
    for (long b = 0; b < blocks; b += room) {
        j.first = static_cast<int>(b);
        e = launch_kernel(embed_join_kernel, dim3(static_cast<unsigned>(blocks - b < room ? blocks - b : room)), dim3(kThreads), 0, st, j);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
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
    return plan_of(N, D, L, V, dtype, true).bytes;
}

int conv1d_embed_bwd(const conv1d_embed_t* p, const void* dy, long dy_sn, long dy_sd, long dy_sl, float* dtable, void* workspace, size_t workspace_bytes,
                     void* stream) {
    if (!shape_ok(p) || !dy || !dtable) return CONV1D_EINVAL;
    const size_t size = p->dtype == CONV1D_BF16 ? 2 : 4;
    if (!seq_aligned(dy, size) || !seq_aligned(dtable, 4) || !seq_aligned(workspace, 256) || !strides_ok(p->D, p->L, dy_sd, dy_sl)) return CONV1D_EINVAL;
    if (!sizes_ok(p->N, p->D, p->L, p->V)) return CONV1D_EUNSUPPORTED;
    const Plan plan = plan_of(p->N, p->D, p->L, p->V, p->dtype, true);
    if (!workspace || workspace_bytes < plan.bytes) return CONV1D_EWORKSPACE;
    const bool turned = is_turned(p->D, p->L, dy_sd, dy_sl);
    char* ws = static_cast<char*>(workspace);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return status_of(p->dtype == CONV1D_BF16 ? gradient<true>(p, dy, dy_sn, dy_sd, dy_sl, dtable, turned, plan, ws, st)
                                             : gradient<false>(p, dy, dy_sn, dy_sd, dy_sl, dtable, turned, plan, ws, st));
}

}  // extern "C"
