// Log probabilities of given tokens under rows of logits, with the row's entropy and its best alternatives, and the
// gradient of the first two at the logits.
//
//   m = max z,  s = sum e^{z - m},  t = sum (z - m) e^{z - m}
//   logsumexp = m + log s      logprob = (z_target - m) - log s      entropy = log s - t / s
//   dz_j = g_lp ([j = target] - p_j) - g_H p_j (log p_j + entropy),        p_j = e^{z_j - m} / s
//
// A logit of -inf is a token that cannot occur: probability 0, never an alternative, gradient 0 (as a target: logprob -inf, gradient
// g_lp, by the formula).  A row of nothing else has logsumexp -inf, logprob -inf, entropy 0, no alternatives and no gradient.  A row
// with a NaN or +inf has no distribution: its results are NaN and it has no alternatives.  Everything is fp32 whatever the storage type.
//
// What bounds them is reading the logits.  A workgroup loads its part of a row ONCE, into registers (up to 16 vectors of
// 16 bytes per lane), and takes maximum, sums, the best k and -- where the caller gives the upstream gradients with the
// call -- the gradient from there: one read and one write per logit instead of the two reads and one write of a loss
// followed by its gradient.  Rows that no workgroup holds, and rows too few to fill the device, are cut into parts whose
// statistics and best k a second launch joins.
//
// The logits stay packed as they were read and are unpacked anew by each pass (kept as fp32 from pass to pass they spill: 1.25 ms
// instead of 0.43 below).  8192 rows of 50 001 bf16 logits, loss and gradient: 430 us (3.8 TB/s; 364 to 396 with rows of 50 000,
// which start on whole vectors, and 4.9 TB/s with 32 000), the gradient alone 356.  1531 rows of 32 003 bf16 with five alternatives:
// 34 us, 25 without.  Four
// rows of 128 000 fp32 with eight: 8 us in 252 parts, 7 to join them.
// How the best k are found stands in logit_rows.h.
#include "logit_rows.h"

namespace ols {

namespace {

constexpr float kFloor = -1.0e4f;      // in units of log 2: e^x is 0 far above it, and 0 times it is 0

struct Stats {   // over some of a row: maximum, sum of e^{z - m}, sum of log2(e^{z - m}) e^{z - m}
    float m, s, t;
};
__device__ __forceinline__ Stats join(const Stats& a, const Stats& b) {
    const float m = fmaxf(a.m, b.m);
    const float base = m == -INFINITY ? 0.0f : m;
    const float da = (a.m - base) * kLog2e, db = (b.m - base) * kLog2e;   // -inf where a side is empty
    const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
    return {m, a.s * fa + b.s * fb, (a.t + a.s * fmaxf(da, kFloor)) * fa + (b.t + b.s * fmaxf(db, kFloor)) * fb};
}

struct RowResult {
    float logprob, entropy, lse;
    bool empty, good;      // good: the row has a distribution
    float s, inv_s, log_s, m;
};
__device__ __forceinline__ RowResult row_result(const Stats& a, float target, bool has_target) {
    RowResult r;
    r.empty = a.m == -INFINITY && a.s == 0.0f;
    r.good = !r.empty && a.s < INFINITY;      // false for a NaN
    r.m = a.m, r.s = a.s;
    r.log_s = kLn2 * __builtin_amdgcn_logf(a.s);
    r.inv_s = 1.0f / a.s;
    r.lse = r.empty ? -INFINITY : r.good ? a.m + r.log_s : NAN;
    r.entropy = r.empty ? 0.0f : r.good ? fmaxf(r.log_s - kLn2 * (a.t * r.inv_s), 0.0f) : NAN;
    r.logprob = !has_target ? 0.0f : r.empty ? -INFINITY : r.good ? (target - a.m) - r.log_s : NAN;
    return r;
}

// p (log p + entropy) and p; zero where the logit is -inf, or so far below the maximum that e^(z - m) is zero
struct GradRow {
    float m, inv_s, log_s, entropy, g_lp, g_h;
    int target;
    bool empty, good;
};
__device__ __forceinline__ float logit_grad(const GradRow& r, float z, int64_t j) {
    const float x = (z - r.m) * kLog2e;
    const float p = __builtin_amdgcn_exp2f(x) * r.inv_s;
    const float logp = fmaxf(x, kFloor) * kLn2 - r.log_s;
    const float d = -p * (r.g_lp + r.g_h * (logp + r.entropy));
    return j == r.target ? r.g_lp + d : d;
}

template <typename T, int THREADS, int NV, bool GRAD>
__global__ __launch_bounds__(THREADS, 4) void logprob_kernel(LogprobParams p) {
    constexpr int N = Vec<T>::kN, WAVES = THREADS / 64;
    extern __shared__ char dyn[];
    __shared__ float red_m[WAVES];
    __shared__ float red_s[WAVES], red_t[WAVES];
    __shared__ float best_val[kMaxTop];
    __shared__ int best_idx[kMaxTop];
    const int64_t row = blockIdx.x;
    const int part = blockIdx.y, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const T* z = (const T*)p.logits + row * p.row_stride;
    const int64_t start = (int64_t)part * p.part, end = min(start + p.part, p.vocab);
    u4 v[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] = load_vec<T>(z, start + ((int64_t)j * THREADS + threadIdx.x) * N, end);
    const int target = p.targets ? p.targets[row] : -1;
    const bool has_target = target >= 0 && target < p.vocab;
    const float z_target = has_target ? load1(z + target) : 0.0f;
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) m = fmaxf(m, Vec<T>::get(v[j], e));
    const float lane_max = m;
    keep_packed(v);
    m = wave_max(m);
    if (lane == 0) red_m[wave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, red_m[w]);
    const float base = m == -INFINITY ? 0.0f : m;
    float s = 0.0f, t = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float s0 = 0.0f, t0 = 0.0f;        // short sums first: fewer roundings of the long ones
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float x = (Vec<T>::get(v[j], e) - base) * kLog2e;
            const float w = __builtin_amdgcn_exp2f(x);
            s0 += w;
            t0 = fmaf(fmaxf(x, kFloor), w, t0);
        }
        s += s0, t += t0;
    }
    s = wave_sum(s), t = wave_sum(t);
    if (lane == 0) red_s[wave] = s, red_t[wave] = t;
    __syncthreads();
    s = t = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += red_s[w], t += red_t[w];
    keep_packed(v);
    const Stats all{m, s, t};
    if (p.top > 0) {
        float* list_val = (float*)dyn;
        int* list_idx = (int*)(list_val + list_entries<T, THREADS, NV>(p.top));
        best_of_part<T, THREADS, NV>(v, lane_max, start, p.top, list_val, list_idx, best_val, best_idx);
    }
    if (p.parts > 1) {
        const int64_t slot = row * p.parts + part;
        if (threadIdx.x == 0) {
            float* o = p.part_stats + 3 * slot;
            o[0] = all.m, o[1] = all.s, o[2] = all.t;
        }
        for (int i = threadIdx.x; i < p.top; i += THREADS) p.part_val[slot * p.top + i] = best_val[i], p.part_idx[slot * p.top + i] = best_idx[i];
        return;
    }
    const RowResult r = row_result(all, z_target, has_target);
    if (threadIdx.x == 0) {
        p.logprob[row] = r.logprob, p.entropy[row] = r.entropy, p.lse[row] = r.lse;
        p.stats[2 * row] = r.m, p.stats[2 * row + 1] = r.s;
    }
    for (int i = threadIdx.x; i < p.top; i += THREADS) {
        const bool there = best_idx[i] >= 0 && r.good;
        p.top_logprob[row * p.top + i] = there ? (best_val[i] - r.m) - r.log_s : r.empty || r.good ? -INFINITY : NAN;
        p.top_index[row * p.top + i] = there ? best_idx[i] : -1;
    }
    if constexpr (GRAD) {
        const GradRow g{r.m, r.inv_s, r.log_s, r.entropy, has_target && p.g_logprob ? p.g_logprob[row] : 0.0f, p.g_entropy ? p.g_entropy[row] : 0.0f,
                        has_target ? target : -1, r.empty, r.good};
        T* d = (T*)p.d_logits + row * p.d_stride;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int64_t i = start + ((int64_t)j * THREADS + threadIdx.x) * N;
            if (i >= end) continue;
            float x[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                x[e] = logit_grad(g, Vec<T>::get(v[j], e), i + e);
                if (!g.good) x[e] = g.empty ? 0.0f : NAN;
            }
            store_vec<T>(d, i, end, x);
        }
    }
}

// Entries of the join's list: of fewer than k parts k each, and k of each of four wavefronts.  With all that the parts hold, 256 of them
// and k = 32 fill more than 64 KiB of LDS, and 600 011 equal logits took 23 ms to put in order instead of 65 us.
__host__ __device__ constexpr int join_entries(int k) { return k * (k + 3); }

// joins the parts of a row
__global__ __launch_bounds__(256) void logprob_join_kernel(LogprobParams p) {
    extern __shared__ char dyn[];
    __shared__ float red[3][4];
    __shared__ float best_val[kMaxTop];
    __shared__ int best_idx[kMaxTop];
    __shared__ float tops[4 * kMaxTop];
    __shared__ int count;
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    if (threadIdx.x == 0) count = 0;
    const float* st = p.part_stats + 3 * row * p.parts;
    Stats a{-INFINITY, 0.0f, 0.0f};
    for (int i = threadIdx.x; i < p.parts; i += 256) a = join(a, Stats{st[3 * i], st[3 * i + 1], st[3 * i + 2]});
    for (int o = 32; o; o >>= 1) {
        const Stats b{__shfl_xor(a.m, o), __shfl_xor(a.s, o), __shfl_xor(a.t, o)};
        a = lane & o ? join(b, a) : join(a, b);        // the same order in every lane
    }
    if (lane == 0) red[0][wave] = a.m, red[1][wave] = a.s, red[2][wave] = a.t;
    __syncthreads();
    a = Stats{red[0][0], red[1][0], red[2][0]};
    for (int w = 1; w < 4; ++w) a = join(a, Stats{red[0][w], red[1][w], red[2][w]});
    const int target = p.targets ? p.targets[row] : -1;
    const bool has_target = target >= 0 && target < p.vocab;
    float z_target = 0.0f;
    if (has_target) {
        const int64_t at = row * p.row_stride + target;
        z_target = p.dtype == OLS_F32 ? ((const float*)p.logits)[at] : of_bf16(((const uint16_t*)p.logits)[at]);
    }
    const RowResult r = row_result(a, z_target, has_target);
    if (threadIdx.x == 0) {
        p.logprob[row] = r.logprob, p.entropy[row] = r.entropy, p.lse[row] = r.lse;
        p.stats[2 * row] = r.m, p.stats[2 * row + 1] = r.s;
    }
    if (p.top == 0) return;
    // The k-th best of the parts' best ones is a limit for the row's k-th best.  Fewer than k parts hold anything above it, and of
    // those equal to it, which lie in the order of their indices, a wavefront needs only its first k.
    const int n = p.parts * p.top, per = (n + 3) / 4, end = min(n, (wave + 1) * per);
    float* val = (float*)dyn;
    int* idx = (int*)(val + join_entries(p.top));
    const float* in_val = p.part_val + row * n;
    const float limit = kth_of_lanes<256>((int)threadIdx.x < p.parts ? in_val[threadIdx.x * p.top] : -INFINITY, p.top, tops);
    int same = 0;
    for (int first = wave * per; first < end; first += 64) {
        const int i = first + lane;
        const float v = i < end ? in_val[i] : -INFINITY;
        const int at = i < end ? p.part_idx[row * n + i] : -1;
        const unsigned long long equal = __ballot(at >= 0 && v == limit);
        if (at >= 0 && (v > limit || (v == limit && same + __popcll(equal & ((1ull << lane) - 1)) < p.top))) {
            const int to = atomicAdd(&count, 1);
            val[to] = v, idx[to] = at;
        }
        same += __popcll(equal);
    }
    __syncthreads();
    write_best<256>(val, idx, count, p.top, best_val, best_idx);
    __syncthreads();
    for (int i = threadIdx.x; i < p.top; i += 256) {
        const bool there = best_idx[i] >= 0 && r.good;
        p.top_logprob[row * p.top + i] = there ? (best_val[i] - r.m) - r.log_s : r.empty || r.good ? -INFINITY : NAN;
        p.top_index[row * p.top + i] = there ? best_idx[i] : -1;
    }
}

// The gradient from the logits and what the forward call left: p = e^(z - m) / s.  From the logsumexp alone, p would carry its
// rounding: 1e-3 of it at logits of 10^4, and all of it where a mask of the type's lowest value leaves nothing else.
template <typename T>
__global__ __launch_bounds__(256) void logprob_grad_kernel(LogprobParams p) {
    constexpr int N = Vec<T>::kN, NV = 4;
    const int64_t row = blockIdx.x;
    const T* z = (const T*)p.logits + row * p.row_stride;
    T* d = (T*)p.d_logits + row * p.d_stride;
    const int64_t start = (int64_t)blockIdx.y * (256 * N * NV);
    u4 v[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] = load_vec<T>(z, start + (j * 256 + threadIdx.x) * N, p.vocab);
    const int target = p.targets ? p.targets[row] : -1;
    const bool has_target = target >= 0 && target < p.vocab;
    const Stats a{p.stats[2 * row], p.stats[2 * row + 1], 0.0f};
    const RowResult r = row_result(a, 0.0f, false);
    const bool empty = r.empty, good = r.good;
    const GradRow g{r.m, r.inv_s, r.log_s, p.entropy ? p.entropy[row] : 0.0f, has_target && p.g_logprob ? p.g_logprob[row] : 0.0f,
                    p.g_entropy ? p.g_entropy[row] : 0.0f, has_target ? target : -1, empty, good};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int64_t i = start + (j * 256 + threadIdx.x) * N;
        if (i >= p.vocab) continue;
        float x[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            x[e] = logit_grad(g, Vec<T>::get(v[j], e), i + e);
            if (!good) x[e] = empty ? 0.0f : NAN;
        }
        store_vec<T>(d, i, p.vocab, x);
    }
}

template <typename T, int THREADS, int NV>
hipError_t launch_rows(const LogprobParams& p, hipStream_t stream) {
    const size_t lds = (size_t)(p.top > 0 ? list_entries<T, THREADS, NV>(p.top) : 0) * 8;
    const dim3 grid((unsigned)p.rows, p.parts);
    if (p.d_logits && p.parts == 1) logprob_kernel<T, THREADS, NV, true><<<grid, THREADS, lds, stream>>>(p);
    else logprob_kernel<T, THREADS, NV, false><<<grid, THREADS, lds, stream>>>(p);
    return hipGetLastError();
}

template <typename T, int NV>
hipError_t launch_long(const LogprobParams& p, const RowPlan& r, hipStream_t stream) {
    if (r.threads == 256) return launch_rows<T, 256, NV>(p, stream);
    return r.threads == 512 ? launch_rows<T, 512, NV>(p, stream) : launch_rows<T, 1024, NV>(p, stream);
}

template <typename T>
hipError_t launch_typed(const LogprobParams& p, const RowPlan& r, hipStream_t stream) {
    if (r.threads == 256) {
        if (r.nv == 2) return launch_rows<T, 256, 2>(p, stream);
        if (r.nv == 4) return launch_rows<T, 256, 4>(p, stream);
        if (r.nv == 8) return launch_rows<T, 256, 8>(p, stream);
    }
    // registers that hold nothing are still gone through: 50 001 logits in 13 vectors a lane instead of 16
    return r.nv <= 10 ? launch_long<T, 10>(p, r, stream) : r.nv == 13 ? launch_long<T, 13>(p, r, stream) : launch_long<T, 16>(p, r, stream);
}

// A launch has fewer than 2^32 threads, a row up to 1024 of them.
constexpr int64_t kMostRows = 1 << 21;
LogprobParams rows_of(const LogprobParams& p, int64_t first) {
    const int64_t bytes = p.dtype == OLS_F32 ? 4 : 2;
    auto at = [&](auto* t, int64_t per) { return t ? t + per * first : t; };
    LogprobParams q = p;
    q.rows = std::min(kMostRows, p.rows - first);
    q.logits = at((const char*)p.logits, p.row_stride * bytes), q.d_logits = at((char*)p.d_logits, p.d_stride * bytes);
    q.targets = at(p.targets, 1), q.g_logprob = at(p.g_logprob, 1), q.g_entropy = at(p.g_entropy, 1);
    q.logprob = at(p.logprob, 1), q.entropy = at(p.entropy, 1), q.lse = at(p.lse, 1), q.stats = at(p.stats, 2);
    q.top_logprob = at(p.top_logprob, p.top), q.top_index = at(p.top_index, p.top);
    return q;
}

template <typename T>
hipError_t launch_grad_typed(const LogprobParams& p, hipStream_t stream) {
    const int64_t span = 256 * 4 * Vec<T>::kN;
    logprob_grad_kernel<T><<<dim3((unsigned)p.rows, (unsigned)((p.vocab + span - 1) / span)), 256, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

int64_t logprob_workspace_bytes(int dtype, int64_t rows, int64_t vocab, int top) {
    if (rows == 0) return 0;
    const RowPlan r = row_plan(dtype, rows, vocab);
    return r.parts > 1 ? rows * r.parts * (12 + 8 * (int64_t)top) : 0;
}

hipError_t launch_logprob_grad(const LogprobParams& p, hipStream_t stream) {
    for (int64_t first = 0; first < p.rows; first += kMostRows) {
        const LogprobParams q = rows_of(p, first);
        const hipError_t e = q.dtype == OLS_F32 ? launch_grad_typed<float>(q, stream) : launch_grad_typed<uint16_t>(q, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_logprob(LogprobParams p, void* ws, hipStream_t stream) {
    if (p.rows == 0) return hipSuccess;
    const RowPlan r = row_plan(p.dtype, p.rows, p.vocab);
    p.parts = r.parts, p.part = r.part;
    for (int64_t first = 0; first < p.rows; first += kMostRows) {
        LogprobParams q = rows_of(p, first);                 // one launch's parts after another's in the same place
        q.part_stats = (float*)ws;
        q.part_val = (float*)ws + 3 * q.rows * r.parts;
        q.part_idx = (int32_t*)(q.part_val + q.rows * r.parts * q.top);
        hipError_t e = q.dtype == OLS_F32 ? launch_typed<float>(q, r, stream) : launch_typed<uint16_t>(q, r, stream);
        if (e == hipSuccess && r.parts > 1) {
            logprob_join_kernel<<<(unsigned)q.rows, 256, (size_t)join_entries(q.top) * 8, stream>>>(q);
            e = hipGetLastError();
            if (e == hipSuccess && q.d_logits) e = launch_logprob_grad(q, stream);
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace ols
