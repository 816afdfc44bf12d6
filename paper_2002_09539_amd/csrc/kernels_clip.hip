// The norm of the gradients of a model over all its tensors, per group (one model, or each worker's), and clipping:
//
//   norm_g = sqrt(sum over the tensors of group g of x^2)        out = x min(1, max_norm / norm_g)
//
// Squares and their sums are in fp64: an fp32 of any size has a square that neither overflows nor vanishes there, and the
// matrix-free fp64 rate (two operations for four bytes read) is far from what bounds a stream.  Sums have one order: a
// workgroup's over its chunk, then the chunks of a group in turn.
//
// Two launches: the sums of squares of chunks, then the scaled copy, whose workgroups add up their group's sums themselves (up to 4096
// numbers from the L2; groups of more tensors than that get a launch between).  The gradients are read twice, three
// traversals where two are the least; what bounds both launches is memory.  The copy takes the chunks in the reverse order, each
// on the XCD that has summed it, so that what was read last is found in the caches.  Sixteen groups of 14.7 M fp32: 158 us to sum
// (5.9 TB/s) and 354 to copy, 6 us more in the order of the sums.  Taking the groups in batches that fit the 256 MiB memory-side cache costs
// more in the ends of its many launches than the cache gives: 666 us with one group a launch, the same with the copy of one
// beside the sums of the next, 642 with three; and storing past the caches 647.
#include "element_io.h"
#include "ols_internal.h"

namespace ols {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ int find_tensor(const ClipTable& t, int chunk) {   // the last entry whose first chunk is at most `chunk`
    int lo = 0, hi = t.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (t.first_chunk[mid] <= chunk) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ double block_sum(double v) {   // the result is in every lane
    __shared__ double part[kThreads / 64];
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < kThreads / 64; ++w) s += part[w];
    return s;
}

// the sum of a group's chunks: lane i adds up chunks i, i + 256, .. and the workgroup joins the lanes
__device__ __forceinline__ double group_sum(const double* partial, int64_t first, int64_t count) {
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < count; i += kThreads) s += partial[first + i];
    return block_sum(s);
}
__device__ __forceinline__ double group_norm(const double* partial, int64_t first, int64_t count) { return sqrt(group_sum(partial, first, count)); }

template <typename T>
__global__ __launch_bounds__(kThreads) void clip_squares_kernel(ClipTable t, int64_t chunk_elems, double* partial) {
    const int k = find_tensor(t, blockIdx.x);
    const int64_t chunk = blockIdx.x - t.first_chunk[k];
    const int64_t from = chunk * chunk_elems, to = min(from + chunk_elems, t.numel[k]);
    const T* x = (const T*)t.in[k];
    double sum[4] = {0, 0, 0, 0};
    for (int64_t i = from + threadIdx.x * 8; i < to; i += 4 * kThreads * 8) {
        float v[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t at = i + (int64_t)u * kThreads * 8;
            load_upto8(x + at, (int)max((int64_t)0, min((int64_t)8, to - at)), 0.0f, v[u]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[u] = fma((double)v[u][e], (double)v[u][e], sum[u]);
    }
    const double s = block_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
    if (threadIdx.x == 0) partial[t.first_sum[k] + chunk] = s;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void clip_scale_kernel(ClipTable t, int64_t chunk_elems, const double* partial, float max_norm, float* norms) {
    constexpr int kXcds = 8;                             // workgroup b runs on XCD b % 8
    const int turns = gridDim.x / kXcds, turn = blockIdx.x / kXcds;
    const int at = turn < turns ? (turns - 1 - turn) * kXcds + blockIdx.x % kXcds : blockIdx.x;
    const int k = find_tensor(t, at);
    const int64_t chunk = at - t.first_chunk[k];
    const double norm = group_norm(partial, t.group_first[k], t.group_chunks[k]);
    if (threadIdx.x == 0 && t.first_sum[k] + chunk == t.group_first[k]) norms[t.group[k]] = (float)norm;
    const T* x = (const T*)t.in[k];
    T* out = (T*)t.out[k];
    const bool clip = !(norm <= (double)max_norm);      // a NaN clips: it reaches every element
    if (!clip && x == out) return;
    const double factor = clip ? (double)max_norm / norm : 1.0;
    const float scale = (float)factor;
    const bool tiny = factor < 0x1p-126;                 // no normal fp32: what it keeps of it would be the result's precision
    const int64_t from = chunk * chunk_elems, to = min(from + chunk_elems, t.numel[k]);
    for (int64_t i = from + threadIdx.x * 8; i < to; i += 4 * kThreads * 8) {
        float v[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t at = i + (int64_t)u * kThreads * 8;
            load_upto8(x + at, (int)max((int64_t)0, min((int64_t)8, to - at)), 0.0f, v[u]);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t at = i + (int64_t)u * kThreads * 8;
            if (at >= to) continue;
            if (__builtin_expect(tiny, 0)) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[u][e] = (float)((double)v[u][e] * factor);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[u][e] *= scale;
            }
            store_upto8(out + at, (int)min((int64_t)8, to - at), v[u]);
        }
    }
}

// one workgroup a group, which has read all of its chunks before it writes
__global__ __launch_bounds__(kThreads) void clip_sums_kernel(ClipGroups g, double* partial) {
    const double sum = group_sum(partial, g.first[blockIdx.x], g.count[blockIdx.x]);
    if (threadIdx.x == 0) partial[g.first[blockIdx.x]] = sum;
}

__global__ __launch_bounds__(kThreads) void clip_norms_kernel(ClipGroups g, const double* partial, float* norms) {
    const double norm = group_norm(partial, g.first[blockIdx.x], g.count[blockIdx.x]);
    if (threadIdx.x == 0) norms[g.group[blockIdx.x]] = (float)norm;
}

}  // namespace

hipError_t launch_clip(const ClipTable& t, int dtype, int64_t chunk_elems, int blocks, bool copy, double* partial, float max_norm, float* norms,
                       hipStream_t stream) {
    if (blocks == 0) return hipSuccess;
    if (copy && dtype == OLS_F32) clip_scale_kernel<float><<<blocks, kThreads, 0, stream>>>(t, chunk_elems, partial, max_norm, norms);
    else if (copy) clip_scale_kernel<uint16_t><<<blocks, kThreads, 0, stream>>>(t, chunk_elems, partial, max_norm, norms);
    else if (dtype == OLS_F32) clip_squares_kernel<float><<<blocks, kThreads, 0, stream>>>(t, chunk_elems, partial);
    else clip_squares_kernel<uint16_t><<<blocks, kThreads, 0, stream>>>(t, chunk_elems, partial);
    return hipGetLastError();
}
hipError_t launch_clip_sums(const ClipGroups& g, int groups, double* partial, hipStream_t stream) {
    clip_sums_kernel<<<groups, kThreads, 0, stream>>>(g, partial);
    return hipGetLastError();
}
hipError_t launch_clip_norms(const ClipGroups& g, int groups, const double* partial, float* norms, hipStream_t stream) {
    clip_norms_kernel<<<groups, kThreads, 0, stream>>>(g, partial, norms);
    return hipGetLastError();
}

}  // namespace ols
