// Dropout whose mask is computed from a counter wherever it is needed, with the residual added in the same pass.
// Element (row, l) of the N C rows is kept where word l % 4 of Philox4x32 (Salmon et al., "Parallel Random Numbers: As Easy as
// 1, 2, 3", SC 2011) with the counter (row ceil(L / 4) + l / 4, call) and the given key reaches floor(p 2^32).  Seven rounds, the
// fewest that passed all of its authors' tests of randomness: a round is two 32 x 32 -> 64 products, which run at a quarter of the rate
// (32 x 256 x 8192 bfloat16 without a residual: 44 to 47 us, 50 to 53 with ten rounds).
// Bound by memory: the same with a residual 75 to 78 us, 5.2 TB/s.  A lane has 8 neighbouring positions: two blocks of the generator,
// whatever the row's alignment in memory, and two such vectors, whose loads go out together.
#include "conv1d_blocks.h"

#include <math.h>

namespace conv1d {
namespace {

constexpr int kThreads = 256;
constexpr int kSteps = 2;   // vectors of 8 a lane

struct DropArgs {
    const void *x, *res;
    void* y;
    const int* lengths;
    const long* counter;
    long x_sn, x_sc, r_sn, r_sc, y_sn, y_sc;
    unsigned long call;
    unsigned k0, k1, least;  // kept from `least` on
    float scale;
    int first_row, items;    // of this launch
    int C, L, per_row;       // per_row: vectors of a row
    int none;                // p = 1
    Div31 by_row, by_C;
};

__device__ __forceinline__ void philox(unsigned long block, unsigned long call, unsigned k0, unsigned k1, unsigned (&c)[4]) {
    c[0] = static_cast<unsigned>(block);
    c[1] = static_cast<unsigned>(block >> 32);
    c[2] = static_cast<unsigned>(call);
    c[3] = static_cast<unsigned>(call >> 32);
#pragma unroll
    for (int r = 0; r < 7; ++r) {
        const unsigned long a = static_cast<unsigned long>(c[0]) * 0xD2511F53u, b = static_cast<unsigned long>(c[2]) * 0xCD9E8D57u;
        c[0] = static_cast<unsigned>(b >> 32) ^ c[1] ^ k0;
        c[1] = static_cast<unsigned>(b);
        c[2] = static_cast<unsigned>(a >> 32) ^ c[3] ^ k1;
        c[3] = static_cast<unsigned>(a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

template <bool BF16, bool RES>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropArgs a) {
    const unsigned long call = a.call + (a.counter ? static_cast<unsigned long>(*a.counter) : 0UL);
    const int first = static_cast<int>(blockIdx.x) * kThreads * kSteps + static_cast<int>(threadIdx.x);
    float v[kSteps][8], r[kSteps][8];
    long to[kSteps];
    int at[kSteps], end[kSteps];
    unsigned long block[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int item = min(first + s * kThreads, a.items - 1);
        const int of = div31(item, a.by_row), row = a.first_row + of, n = div31(row, a.by_C), c = row - n * a.C;
        at[s] = 8 * (item - of * a.per_row);
        end[s] = seq_length(a.lengths, n, a.L);
        to[s] = n * a.y_sn + c * a.y_sc;
        block[s] = static_cast<unsigned long>(row) * static_cast<unsigned>((a.L + 3) >> 2) + static_cast<unsigned>(at[s] >> 2);
        const long size = BF16 ? 2 : 4;
        row_load8<BF16>(static_cast<const char*>(a.x) + size * (n * a.x_sn + c * a.x_sc), at[s], end[s], v[s]);
        if constexpr (RES) row_load8<BF16>(static_cast<const char*>(a.res) + size * (n * a.r_sn + c * a.r_sc), at[s], end[s], r[s]);
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        if (first + s * kThreads >= a.items) break;
        unsigned word[2][4];
        philox(block[s], call, a.k0, a.k1, word[0]);
        philox(block[s] + 1, call, a.k0, a.k1, word[1]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool keep = word[e >> 2][e & 3] >= a.least && !a.none && at[s] + e < end[s];
            v[s][e] = keep ? v[s][e] * a.scale : 0.f;
            if constexpr (RES) v[s][e] += r[s][e];
        }
        row_store8<BF16>(static_cast<char*>(a.y) + (BF16 ? 2 : 4) * to[s], at[s], a.L, v[s]);
    }
}

}  // namespace
}  // namespace conv1d

using namespace conv1d;

extern "C" int conv1d_dropout(const conv1d_dropout_t* p, void* y, long y_sn, long y_sc, void* stream) {
    if (!p || !p->x || !y || p->N < 1 || p->C < 1 || p->L < 1 || !(p->p >= 0.0 && p->p <= 1.0)) return CONV1D_EINVAL;
    if (p->dtype != CONV1D_FP32 && p->dtype != CONV1D_BF16) return CONV1D_EINVAL;
    const size_t size = p->dtype == CONV1D_BF16 ? 2 : 4;
    if (!seq_aligned(p->x, size) || !seq_aligned(p->residual, size) || !seq_aligned(y, size) || !seq_aligned(p->lengths, 4) || !seq_aligned(p->counter, 8))
        return CONV1D_EINVAL;
    const long rows = static_cast<long>(p->N) * p->C, per_row = (p->L + 7L) / 8;
    if (p->L > 1 << 30 || rows > 0x7fffffffL) return CONV1D_EUNSUPPORTED;
    DropArgs a{};
    a.x = p->x; a.res = p->residual; a.y = y; a.lengths = p->lengths; a.counter = p->counter;
    a.x_sn = p->x_sn; a.x_sc = p->x_sc; a.r_sn = p->r_sn; a.r_sc = p->r_sc; a.y_sn = y_sn; a.y_sc = y_sc;
    a.call = p->call;
    a.k0 = static_cast<unsigned>(p->key);
    a.k1 = static_cast<unsigned>(p->key >> 32);
    a.none = p->p == 1.0;
    a.least = a.none ? 0xffffffffu : static_cast<unsigned>(floor(p->p * 4294967296.0));
    a.scale = a.none ? 0.f : static_cast<float>(1.0 / (1.0 - p->p));
    a.C = p->C; a.L = p->L; a.per_row = static_cast<int>(per_row);
    a.by_row = make_div31(per_row);
    a.by_C = make_div31(p->C);
    void (*kern)(DropArgs) = p->dtype == CONV1D_BF16 ? (p->residual ? dropout_kernel<true, true> : dropout_kernel<true, false>)
                                                     : (p->residual ? dropout_kernel<false, true> : dropout_kernel<false, false>);
    const long most = kMostItems / per_row;  // rows of a launch
    for (long row = 0; row < rows; row += most) {
        const long some = rows - row < most ? rows - row : most;
        a.first_row = static_cast<int>(row);
        a.items = static_cast<int>(some * per_row);
        const hipError_t e = launch_kernel(kern, dim3(static_cast<unsigned>(cdiv(a.items, kThreads * kSteps))), dim3(kThreads), 0,
                                           static_cast<hipStream_t>(stream), a);
        if (e != hipSuccess) return CONV1D_EHIP;
    }
    return CONV1D_OK;
}
