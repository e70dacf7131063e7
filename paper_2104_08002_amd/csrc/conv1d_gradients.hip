// The norm over many gradient tensors, and their scaling by min(1, most / (norm + 1e-6)).
// Bound by memory: every element is read for the norm, read again and written for the scaling.  A launch takes the addresses
// of up to kTensors tensors among its own arguments, so that nothing is copied to the device and a captured graph holds them.
// Squares are summed in 64 bits: no gradient of either type is too large or too small for its square.
#include "conv1d_sequence.h"

#include <algorithm>
#include <new>

namespace conv1d {
namespace {

constexpr int kThreads = 256;
constexpr int kTensors = 160;                 // of a launch: 20 bytes each of the 4096 that arguments may take
constexpr long kPiece = 8L * kThreads * 8;    // elements of a workgroup: 8 steps of 8 a lane

struct Table {
    void* data[kTensors];
    long count[kTensors];
    int begin[kTensors];   // first workgroup of the tensor within the launch
    unsigned bf16[(kTensors + 31) / 32];
    int tensors;
};
struct Job {
    void* data;
    long from, to;
    bool bf16;
};
__device__ __forceinline__ Job job_of(const Table& t, int block) {
    int lo = 0, hi = t.tensors - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.begin[mid] <= block) lo = mid;
        else hi = mid - 1;
    }
    Job j;
    j.data = t.data[lo];
    j.from = (block - t.begin[lo]) * kPiece;
    j.to = min(t.count[lo], j.from + kPiece);
    j.bf16 = (t.bf16[lo >> 5] >> (lo & 31)) & 1;
    return j;
}

// larger of the two; NaN if one is
__device__ __forceinline__ double larger(double a, double b) { return b > a || b != b ? b : a; }

template <bool MAX, int THREADS>
__device__ __forceinline__ double block_value(double v, double* lds) {
#pragma unroll
    for (int m = 1; m < kSeqWave; m <<= 1) {
        const double o = lane_xor(v, m);
        v = MAX ? larger(v, o) : v + o;
    }
    if ((threadIdx.x & (kSeqWave - 1)) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
    for (int w = 1; w < THREADS / kSeqWave; ++w) v = MAX ? larger(v, lds[w]) : v + lds[w];
    return v;
}

constexpr int kAtOnce = 4;  // steps whose loads a lane has in flight

template <bool BF16, bool MAX>
__device__ __forceinline__ void take(const float (&v)[8], double (&sum)[2], float& most) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (MAX) {
            const float m = fabsf(v[e]);
            most = m > most || m != m ? m : most;
        } else {
            sum[e & 1] = fma(static_cast<double>(v[e]), static_cast<double>(v[e]), sum[e & 1]);
        }
    }
}

template <bool BF16, bool MAX>
__device__ __forceinline__ double piece_value(const Job& j) {
    double sum[2] = {0.0, 0.0};
    float most = 0.f;
    const long at = j.from + 8 * threadIdx.x;
    if (j.to - j.from == kPiece) {
#pragma unroll 1
        for (long i = at; i < j.to; i += 8 * kThreads * kAtOnce) {
            float v[kAtOnce][8];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) row_load8_inside<BF16>(j.data, i + 8 * kThreads * k, v[k]);
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) take<BF16, MAX>(v[k], sum, most);
        }
    } else {
        for (long i = at; i < j.to; i += 8 * kThreads) {
            float v[8];
            row_load8<BF16>(j.data, i, j.to, v);
            take<BF16, MAX>(v, sum, most);
        }
    }
    return MAX ? static_cast<double>(most) : sum[0] + sum[1];
}

template <bool MAX>
__global__ __launch_bounds__(kThreads) void grad_part_kernel(Table t, double* part) {
    __shared__ double lds[kThreads / kSeqWave];
    const Job j = job_of(t, static_cast<int>(blockIdx.x));
    const double v = block_value<MAX, kThreads>(j.bf16 ? piece_value<true, MAX>(j) : piece_value<false, MAX>(j), lds);
    if (threadIdx.x == 0) part[blockIdx.x] = v;
}

constexpr int kJoinThreads = 1024;
template <bool MAX>
__global__ __launch_bounds__(kJoinThreads) void grad_join_kernel(const double* part, long n, float* norm) {
    __shared__ double lds[kJoinThreads / kSeqWave];
    double v = 0.0;
#pragma unroll 8
    for (long i = threadIdx.x; i < n; i += kJoinThreads) v = MAX ? larger(v, part[i]) : v + part[i];
    v = block_value<MAX, kJoinThreads>(v, lds);
    if (threadIdx.x == 0) *norm = static_cast<float>(MAX ? v : sqrt(v));
}

template <bool BF16>
__device__ __forceinline__ void scale_piece(const Job& j, float factor) {
    const long at = j.from + 8 * threadIdx.x;
    if (j.to - j.from == kPiece) {
#pragma unroll 1
        for (long i = at; i < j.to; i += 8 * kThreads * kAtOnce) {
            float v[kAtOnce][8];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) row_load8_inside<BF16>(j.data, i + 8 * kThreads * k, v[k]);
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[k][e] *= factor;
                row_store8<BF16>(j.data, i + 8 * kThreads * k, j.to, v[k]);
            }
        }
    } else {
        for (long i = at; i < j.to; i += 8 * kThreads) {
            float v[8];
            row_load8<BF16>(j.data, i, j.to, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= factor;
            row_store8<BF16>(j.data, i, j.to, v);
        }
    }
}

// A factor of 1 changes nothing: nothing is read or written.
__global__ __launch_bounds__(kThreads) void grad_scale_kernel(Table t, const float* norm, float most) {
    const float factor = static_cast<float>(static_cast<double>(most) / (static_cast<double>(*norm) + 1e-6));
    if (factor >= 1.f) return;
    const Job j = job_of(t, static_cast<int>(blockIdx.x));
    if (j.bf16) scale_piece<true>(j, factor);
    else scale_piece<false>(j, factor);
}

long pieces_of(size_t count) { return static_cast<long>((count + kPiece - 1) / kPiece); }

bool tensors_ok(void* const* data, const size_t* counts, const int* dtypes, int tensors) {
    if (tensors < 0 || (tensors && (!data || !counts || !dtypes))) return false;
    for (int i = 0; i < tensors; ++i) {
        if (dtypes[i] != CONV1D_FP32 && dtypes[i] != CONV1D_BF16) return false;
        if (counts[i] && (!data[i] || !seq_aligned(data[i], dtypes[i] == CONV1D_BF16 ? 2 : 4))) return false;
        if (counts[i] > (1UL << 37)) return false;  // (workgroups of one tensor in one launch)
    }
    return true;
}

// whether two of the tensors share memory, or one with the norm, which every workgroup reads: -1 if that cannot be found out
int overlap(void* const* data, const size_t* counts, const int* dtypes, int tensors, const float* norm) {
    struct Range {
        uintptr_t from, to;
    };
    if (tensors < 1) return 0;
    Range* r = new (std::nothrow) Range[tensors + 1];
    if (!r) return -1;
    int n = 0;
    const uintptr_t norm_at = reinterpret_cast<uintptr_t>(norm);
    r[n++] = Range{norm_at, norm_at + sizeof(float)};
    for (int i = 0; i < tensors; ++i) {
        if (!counts[i]) continue;
        const uintptr_t at = reinterpret_cast<uintptr_t>(data[i]);
        r[n++] = Range{at, at + counts[i] * (dtypes[i] == CONV1D_BF16 ? 2 : 4)};
    }
    std::sort(r, r + n, [](const Range& a, const Range& b) { return a.from < b.from; });
    int found = 0;
    for (int i = 1; i < n; ++i) found |= r[i].from < r[i - 1].to;
    delete[] r;
    return found;
}

// launch(table, workgroups, workgroups before it) for every kTensors of the tensors
template <typename Launch>
hipError_t each_table(void* const* data, const size_t* counts, const int* dtypes, int tensors, Launch launch) {
    Table t{};
    long blocks = 0, before = 0;
    for (int i = 0; i <= tensors; ++i) {
        const long more = i < tensors ? pieces_of(counts[i]) : 0;
        if (t.tensors && (i == tensors || t.tensors == kTensors || blocks + more > kSeqMostThreads / kThreads)) {
            const hipError_t e = launch(t, blocks, before);
            if (e != hipSuccess) return e;
            before += blocks;
            blocks = 0;
            t = Table{};
        }
        if (!more) continue;
        t.data[t.tensors] = data[i];
        t.count[t.tensors] = static_cast<long>(counts[i]);
        t.begin[t.tensors] = static_cast<int>(blocks);
        if (dtypes[i] == CONV1D_BF16) t.bf16[t.tensors >> 5] |= 1u << (t.tensors & 31);
        ++t.tensors;
        blocks += more;
    }
    return hipSuccess;
}

}  // namespace
}  // namespace conv1d

using namespace conv1d;

extern "C" {

size_t conv1d_grad_norm_workspace_bytes(const size_t* counts, int tensors) {
    if (!counts || tensors < 1) return 0;
    size_t n = 0;
    for (int i = 0; i < tensors; ++i) n += static_cast<size_t>(pieces_of(counts[i]));
    return n * sizeof(double);
}

int conv1d_grad_norm(void* const* data, const size_t* counts, const int* dtypes, int tensors, int kind, float* norm, void* workspace,
                     size_t workspace_bytes, void* stream) {
    if (!tensors_ok(data, counts, dtypes, tensors) || !norm || !seq_aligned(norm, 4) || !seq_aligned(workspace, 8)) return CONV1D_EINVAL;
    if (kind != CONV1D_NORM_2 && kind != CONV1D_NORM_MAX) return CONV1D_EINVAL;
    const size_t need = conv1d_grad_norm_workspace_bytes(counts, tensors);
    if (need && (!workspace || workspace_bytes < need)) return CONV1D_EWORKSPACE;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    double* part = static_cast<double*>(workspace);
    const bool max = kind == CONV1D_NORM_MAX;
    hipError_t e = each_table(data, counts, dtypes, tensors, [&](const Table& t, long blocks, long before) {
        return launch_kernel(max ? grad_part_kernel<true> : grad_part_kernel<false>, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, st, t, part + before);
    });
    if (e == hipSuccess)
        e = launch_kernel(max ? grad_join_kernel<true> : grad_join_kernel<false>, dim3(1), dim3(kJoinThreads), 0, st, part,
                          static_cast<long>(need / sizeof(double)), norm);
    return e == hipSuccess ? CONV1D_OK : CONV1D_EHIP;
}

int conv1d_grad_clip(void* const* data, const size_t* counts, const int* dtypes, int tensors, const float* norm, float most, void* stream) {
    if (!tensors_ok(data, counts, dtypes, tensors) || !norm || !seq_aligned(norm, 4) || !(most >= 0.f)) return CONV1D_EINVAL;
    if (overlap(data, counts, dtypes, tensors, norm)) return CONV1D_EINVAL;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const hipError_t e = each_table(data, counts, dtypes, tensors, [&](const Table& t, long blocks, long) {
        return launch_kernel(grad_scale_kernel, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, st, t, norm, most);
    });
    return e == hipSuccess ? CONV1D_OK : CONV1D_EHIP;
}

}  // extern "C"
