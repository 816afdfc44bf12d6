// Rows of logits in the registers of a workgroup: reading and writing them, reductions over them, and their best k.
//
// A workgroup loads its part of a row once, up to 16 vectors of 16 bytes a lane; every pass over it unpacks the logits anew.
//
// Best k: the k-th largest of the lanes' maxima is a bound that at least k logits reach and that few others do: fewer
// than k lanes hold anything above it.  Those above it go to a list in LDS; of those equal to it a wavefront needs only
// its first k in index order.  Every listed logit then counts the listed ones that beat it (larger, or equal and
// earlier), which is its place.
#pragma once
#include <algorithm>

#include "element_io.h"
#include "ols_internal.h"

namespace ols {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kMaxTop = OLS_MAX_TOP;

template <typename T>
struct Vec;   // sixteen bytes of logits in registers
template <>
struct Vec<float> {
    static constexpr int kN = 4;
    __device__ static float get(const u4& v, int e) { return __uint_as_float(v[e]); }
    __device__ static u4 pack(const float (&x)[4]) { return {__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])}; }
    static constexpr unsigned kNone = 0xFF800000u;      // -inf
};
template <>
struct Vec<uint16_t> {
    static constexpr int kN = 8;
    __device__ static float get(const u4& v, int e) { return e % 2 ? bf16_hi(v[e / 2]) : bf16_lo(v[e / 2]); }
    __device__ static u4 pack(const float (&x)[8]) { return {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])}; }
    static constexpr unsigned kNone = 0xFF80FF80u;      // -inf twice
};

template <typename T>
__device__ __forceinline__ u4 load_vec(const T* row, int64_t i, int64_t end) {   // logits [i, i + kN), -inf from `end` on
    constexpr int N = Vec<T>::kN;
    if (i + N <= end) return *(const u4any*)(row + i);
    u4 v = {Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone};
    if (i < end) {
        float x[N];
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = i + e < end ? load1(row + i + e) : -INFINITY;
        v = Vec<T>::pack(x);
    }
    return v;
}
template <typename T>
__device__ __forceinline__ void store_vec(T* row, int64_t i, int64_t end, const float (&x)[Vec<T>::kN]) {
    constexpr int N = Vec<T>::kN;
    if (i + N <= end) {
        *(u4any*)(row + i) = Vec<T>::pack(x);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (i + e < end) store1(row + i + e, x[e]);
    }
}

// Reductions of a wavefront in the vector unit's own data path (a shuffle through LDS costs ten times an operation): lanes of
// a row of 16 by shifts, then the rows' last lanes are handed on.  Lane 63 ends with the result, which all read.
template <int CTRL, int ROWS>
__device__ __forceinline__ float moved(float v, float other) {      // lanes that receive nothing see `other`
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(other), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float lane_of(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, moved<0x111, 0xf>(v, -INFINITY));
    v = fmaxf(v, moved<0x112, 0xf>(v, -INFINITY));
    v = fmaxf(v, moved<0x114, 0xf>(v, -INFINITY));
    v = fmaxf(v, moved<0x118, 0xf>(v, -INFINITY));
    v = fmaxf(v, moved<0x142, 0xa>(v, -INFINITY));
    v = fmaxf(v, moved<0x143, 0xc>(v, -INFINITY));
    return lane_of(v, 63);
}
__device__ __forceinline__ float wave_sum(float v) {
    v += moved<0x111, 0xf>(v, 0.0f);
    v += moved<0x112, 0xf>(v, 0.0f);
    v += moved<0x114, 0xf>(v, 0.0f);
    v += moved<0x118, 0xf>(v, 0.0f);
    v += moved<0x142, 0xa>(v, 0.0f);
    v += moved<0x143, 0xc>(v, 0.0f);
    return lane_of(v, 63);
}

template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double v) {      // lanes that receive nothing see 0
    const unsigned long long b = __double_as_longlong(v);
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)b, CTRL, ROWS, 0xf, false);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(b >> 32), CTRL, ROWS, 0xf, false);
    return __longlong_as_double((long long)((unsigned long long)hi << 32 | lo));
}
__device__ __forceinline__ double wave_sum(double v) {
    v += moved<0x111, 0xf>(v);
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);
    v += moved<0x143, 0xc>(v);
    const unsigned long long b = __double_as_longlong(v);
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)b, 63), hi = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)(b >> 32), 63);
    return __longlong_as_double((long long)((unsigned long long)hi << 32 | lo));
}

// log x in fp64, by log m = 2 atanh((m - 1) / (m + 1)) for m in [sqrt 1/2, sqrt 2) and its series up to the 17th power, which is off by 9e-16
// of the whole at the most.  Not inlined: kernels of one wavefront's work wait for their instructions longer than for the arithmetic.
__device__ __attribute__((noinline)) double log_of(double x) {
    if (!(x > 0.0 && x < (double)INFINITY)) return x == 0.0 ? (double)-INFINITY : x > 0.0 ? x : (double)NAN;
    double m = __builtin_amdgcn_frexp_mant(x);
    int e = __builtin_amdgcn_frexp_exp(x);
    if (m < 0.70710678118654752440) m *= 2.0, e -= 1;
    const double f = (m - 1.0) / (m + 1.0), s = f * f;
    double v = 1.0 / 17;
    v = fma(v, s, 1.0 / 15), v = fma(v, s, 1.0 / 13), v = fma(v, s, 1.0 / 11), v = fma(v, s, 1.0 / 9);
    v = fma(v, s, 1.0 / 7), v = fma(v, s, 1.0 / 5), v = fma(v, s, 1.0 / 3), v = fma(v, s, 1.0);
    return fma((double)e, 0.69314718055994530942, 2.0 * f * v);
}

// places among the listed: value descending, index ascending
__device__ __forceinline__ bool beats(float a, int ia, float b, int ib) { return a > b || (a == b && ia < ib); }

// Writes the best k of `count` listed logits in their order.  Up to 64 are compared by the first wavefront in registers.
template <int THREADS>
__device__ __forceinline__ void write_best(const float* val, const int* idx, int count, int k, float* out_val, int* out_idx) {
    for (int i = threadIdx.x; i < k; i += THREADS)
        if (i >= count) out_val[i] = -INFINITY, out_idx[i] = -1;
    if (count <= 64) {
        if (threadIdx.x >= 64) return;
        const int i = threadIdx.x;
        const float v = i < count ? val[i] : -INFINITY;
        const int at = i < count ? idx[i] : 0x7fffffff;
        int place = 0;
        for (int j = 0; j < count; ++j) place += beats(lane_of(v, j), __builtin_amdgcn_readlane(at, j), v, at) ? 1 : 0;
        if (i < count && place < k) out_val[place] = v, out_idx[place] = at;
        return;
    }
    for (int i = threadIdx.x; i < count; i += THREADS) {
        const float v = val[i];
        const int at = idx[i];
        int place = 0;
#pragma unroll 8
        for (int j = 0; j < count; ++j) place += beats(val[j], idx[j], v, at) ? 1 : 0;
        if (place < k) out_val[place] = v, out_idx[place] = at;
    }
}

// The k-th largest of all lanes' values (k <= 32; -inf where fewer lanes hold more).  Every wavefront puts its k largest into
// `tops`, largest first, and then merges the lists by itself: lane w holds the head of list w.
template <int THREADS>
__device__ __forceinline__ float kth_of_lanes(float mine, int k, float* tops) {
    constexpr int WAVES = THREADS / 64;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    float left = mine;
    for (int i = 0; i < k; ++i) {
        const float top = wave_max(left);
        if (lane == 0) tops[wave * k + i] = top;
        const unsigned long long at = __ballot(left == top);
        if (at && lane == __ffsll(at) - 1) left = -INFINITY;
    }
    __syncthreads();
    int used = 0;
    float head = lane < WAVES ? tops[lane * k] : -INFINITY, bound = -INFINITY;
    for (int i = 0; i < k; ++i) {
        bound = wave_max(head);
        const unsigned long long at = __ballot(head == bound);
        if (at && lane == __ffsll(at) - 1) head = lane < WAVES && ++used < k ? tops[lane * k + used] : -INFINITY;
    }
    return bound;
}

// The best k of what the workgroup holds, as (value, index) pairs in LDS, best first; -1 and -inf where there are fewer.
template <typename T, int THREADS, int NV>
__device__ void best_of_part(const u4 (&v)[NV], float lane_max, int64_t start, int k, float* lds_val, int* lds_idx, float* best_val, int* best_idx) {
    constexpr int N = Vec<T>::kN, WAVES = THREADS / 64;
    __shared__ float tops[WAVES * kMaxTop];
    __shared__ int listed;
    const int lane = threadIdx.x % 64;
    if (threadIdx.x == 0) listed = 0;
    const float limit = kth_of_lanes<THREADS>(lane_max, k, tops);
    int same = 0;               // logits equal to the limit that this wavefront has listed
    if (__ballot(lane_max >= limit && lane_max > -INFINITY)) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float top = Vec<T>::get(v[j], 0);
#pragma unroll
            for (int e = 1; e < N; ++e) top = fmaxf(top, Vec<T>::get(v[j], e));
            if (!__ballot(top >= limit && top > -INFINITY)) continue;
            unsigned above = 0, at = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float x = Vec<T>::get(v[j], e);
                above |= x > limit ? 1u << e : 0u;
                at |= x == limit && x > -INFINITY ? 1u << e : 0u;
            }
            const int64_t first = start + ((int64_t)j * THREADS + threadIdx.x) * N;
            int rank = __popc(at);                       // equal ones of earlier lanes
            if (__ballot(at)) {
                for (int o = 1; o < 64; o <<= 1) {
                    const int u = __shfl_up(rank, o);
                    if (lane >= o) rank += u;
                }
            }
            const int in_vec = __shfl(rank, 63);
            rank += same - __popc(at);
            for (unsigned todo = above | at; todo; todo &= todo - 1) {
                const int e = __ffs(todo) - 1;
                const bool eq = (at >> e) & 1u;
                if (!eq || rank < k) {
                    const int to = atomicAdd(&listed, 1);
                    float x = Vec<T>::get(v[j], 0);
#pragma unroll
                    for (int c = 1; c < N; ++c) x = c == e ? Vec<T>::get(v[j], c) : x;
                    lds_val[to] = x;
                    lds_idx[to] = (int)(first + e);
                }
                rank += eq ? 1 : 0;
            }
            same += in_vec;
        }
    }
    __syncthreads();
    write_best<THREADS>(lds_val, lds_idx, listed, k, best_val, best_idx);
    __syncthreads();
}

// Entries of the list: fewer than k lanes hold logits above the bound (at most NV vectors each), and every wavefront lists
// at most k equal to it.
template <typename T, int THREADS, int NV>
constexpr int list_entries(int k) { return k * NV * Vec<T>::kN + THREADS / 64 * k; }

// Every pass unpacks the logits anew: without this, the compiler keeps them as fp32 from pass to pass, which is twice the
// registers and spills.
template <int NV>
__device__ __forceinline__ void keep_packed(u4 (&v)[NV]) {
#pragma unroll
    for (int j = 0; j < NV; ++j) asm("" : "+v"(v[j]));
}

struct RowPlan {
    int threads, nv, parts;
    int64_t part;
};

// Parts of a row: one, where a workgroup's registers hold it and the rows fill the device by themselves; otherwise so many
// that about kFill workgroups run, of at least 2 vectors per lane.
constexpr int64_t kFill = 512, kMostParts = 256;
inline RowPlan row_plan(int dtype, int64_t rows, int64_t vocab, int threads = 1024) {      // of the largest workgroup
    const int n = dtype == OLS_F32 ? 4 : 8;
    const int64_t unit = 256 * n;                       // one vector per lane of the smallest workgroup
    const int64_t most = (int64_t)threads * 16 * n;     // the largest workgroup's registers
    int64_t parts = (vocab + most - 1) / most;
    if (rows < kFill) parts = std::max(parts, std::min(std::min(kMostParts, (kFill + rows - 1) / rows), (vocab + 2 * unit - 1) / (2 * unit)));
    RowPlan r;
    r.part = (vocab + parts - 1) / parts;
    r.part = (r.part + n - 1) / n * n;
    r.parts = (int)((vocab + r.part - 1) / r.part);
    const int64_t vecs = (r.part + unit - 1) / unit;    // per lane of 256
    r.threads = vecs <= 16 ? 256 : vecs <= 32 ? 512 : 1024;
    const int64_t per = (r.part + r.threads * n - 1) / (r.threads * n);
    r.nv = per <= 2 ? 2 : per <= 4 ? 4 : per <= 8 ? 8 : per <= 10 ? 10 : per <= 13 ? 13 : 16;
    return r;
}

}  // namespace
}  // namespace ols
