// Distillation from a teacher's top logits: the loss of a student's logits z against lists of the teacher's best tokens, with the
// likelihood of a given token beside it, and the gradient of both at the logits.
//
//   u = z / T,  p = softmax(u),  lists (i_j, v_j) of k entries
//   q_j = softmax over the list of v_j / T,   or with `rest`   q_j = e^{v_j},  q_r = max(0, 1 - sum q),  p_r = sum of p outside the list
//   loss = T^2 (sum q_j (log q_j - log p_{i_j}) + q_r (log q_r - log p_r))
//   W = sum q + q_r:    dloss/dz_i = T (W p_i - sum of q_j with i_j = i)   listed,     T (W p_i - q_r p_i / p_r)   others
//   logprob = z_t - log sum e^z,                 dlogprob/dz_i = [i = t] - e^{z_i} / sum e^z
//
// p_r is the sum over what is not listed, never 1 - sum of the listed: of a student that is sure of its list nothing would be left.
// For that the listed logits are struck out of the registers that hold the row (a bit per logit in LDS says which; a set bit met
// again says that a list names a token twice), the sums are taken over the others against the others' own maximum, and one wavefront
// adds the listed ones.  Maximum and sums are fp32; what a list adds up to and the loss, a difference of like numbers, are fp64.
// Exponents are products with log2 e / T in two terms: its rounding alone would move every far logit the same way.
//
// What bounds it is one read and one write of the logits.  A workgroup holds its part of a row in registers and forms the
// gradient from there; all logits get the gradient of an unlisted one, and behind a barrier the entries of the list and the target
// are written over.  Rows that no workgroup holds and rows too few for the device go in parts, a join and the gradient from memory.
#include "logit_rows.h"

namespace ols {

namespace {

constexpr int kMaxList = OLS_MAX_TEACHER;

// e^{d x} as a power of two: x log2 e = hi + lo, both positive, so that -inf stays -inf
__device__ __forceinline__ float power(float d, float hi, float lo) { return __builtin_amdgcn_exp2f(fmaf(d, hi, d * lo)); }

__device__ __forceinline__ double sum_lanes(double v) {
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

struct Sums {            // over some of a row: maximum, sum of e^{(z - m) / T}, sum of e^{z - m}
    float m, s, s1;
};
__device__ __forceinline__ Sums join(const DistillParams& p, const Sums& a, const Sums& b) {
    const float m = fmaxf(a.m, b.m), base = m == -INFINITY ? 0.0f : m;
    const float da = a.m - base, db = b.m - base;                         // -inf where a side is empty
    return {m, a.s * power(da, p.hi, p.lo) + b.s * power(db, p.hi, p.lo), a.s1 * power(da, p.hi1, p.lo1) + b.s1 * power(db, p.hi1, p.lo1)};
}

// A row's list in LDS: places in the row (-1: none), q, and the student's logits; entry k is the target.
struct List {
    int index[kMaxList + 1];
    float q[kMaxList + 1], z[kMaxList + 1];
    int twice, target_listed;            // a token is named twice; the target is in the list
};

// What one wavefront knows of a list.
struct Teacher {
    double w, rest, self;                // sum of q, q_r, sum of q log q
    float top, scale;                    // q_j = e^{(v_j - top) / T or v_j} scale
};

// Reads entries and target; entries outside [start, end) are none.
template <typename T>
__device__ __forceinline__ void read_list(const DistillParams& p, List& l, int64_t row, const T* z, int64_t start, int64_t end) {
    const int lane = threadIdx.x % 64;
    const int target = p.targets ? p.targets[row] : -1;
    bool met = false;
    for (int i = lane; i < p.k; i += 64) {
        const int at = p.index[row * p.k + i];
        const bool there = at >= start && at < end;
        l.index[i] = there ? at : -1;
        l.z[i] = there ? load1(z + at) : -INFINITY;
        met |= there && at == target;
    }
    const unsigned long long any = __ballot(met);
    if (lane == 0) {
        const bool there = target >= start && target < end;
        l.index[p.k] = there ? target : -1;
        l.z[p.k] = there ? load1(z + target) : -INFINITY;
        l.q[p.k] = 0.0f;
        l.target_listed = any != 0;
    }
}

// One bit per logit of [start, ..), set where it is listed.
__device__ __forceinline__ void mark(const DistillParams& p, List& l, unsigned* bits, int64_t start) {
    bool again = false;
    for (int i = threadIdx.x % 64; i < p.k; i += 64) {
        if (l.index[i] < 0) continue;
        const int at = (int)(l.index[i] - start);
        again |= (atomicOr(&bits[at / 32], 1u << (at % 32)) >> (at % 32)) & 1u;
    }
    const unsigned long long any = __ballot(again);
    if (threadIdx.x % 64 == 0) l.twice = any != 0;
}
// Whether entry i is its token's first.
__device__ __forceinline__ bool first_of(const List& l, int i) {
    for (int j = 0; j < i; ++j)
        if (l.index[j] == l.index[i]) return false;
    return true;
}

// The teacher's probabilities into l.q, by one wavefront.  A NaN or +inf among the values makes them all NaN.
__device__ __forceinline__ Teacher weigh(const DistillParams& p, List& l, int64_t row) {
    const int lane = threadIdx.x % 64;
    const float* value = p.value + row * p.k;
    Teacher t;
    float top = -INFINITY;
    bool some = false, bad = false;
    for (int i = lane; i < p.k; i += 64) {
        if (l.index[i] < 0) continue;
        const float v = value[i];
        some = true, bad |= !(v < INFINITY);
        top = fmaxf(top, v);
    }
    some = __ballot(some) != 0, bad = __ballot(bad) != 0;
    top = wave_max(top);
    t.top = p.rest || top == -INFINITY ? 0.0f : top;
    const double inv_t = p.rest ? 1.0 : 1.0 / (double)p.temperature;
    double w = 0.0, self = 0.0;
    for (int i = lane; i < p.k; i += 64) {
        float q = 0.0f;
        if (l.index[i] >= 0) {
            const double u = ((double)value[i] - t.top) * inv_t, e = exp(u);
            w += e, self += e > 0.0 ? e * u : 0.0;
            q = (float)e;
        }
        l.q[i] = q;
    }
    w = sum_lanes(w), self = sum_lanes(self);
    t.scale = 1.0f, t.rest = 0.0;
    if (p.rest) {
        t.rest = some ? fmax(1.0 - w, 0.0) : 0.0;
    } else if (w > 0.0) {
        t.scale = (float)(1.0 / w);
        self = self / w - log(w);
        for (int i = lane; i < p.k; i += 64) l.q[i] *= t.scale;
        w = 1.0;
    }
    if (bad) w = self = NAN, t.scale = NAN;
    t.w = w, t.self = self;
    return t;
}

// What the gradient needs of a row; p.stats holds it for a later call.
struct Coefs {
    float base;          // maximum of the logits that are not struck out (0 where there is none)
    float others, hard;  // the factors of e^{(z - base) / T} and e^{z - base}
    float m;             // maximum of all
    float listed, inv_s1;     // the factors of e^{(z - m) / T} and e^{z - m}
    float s, s1;         // the sums, against m
    bool empty, held;    // nothing is allowed; the rest counts
};
// u: over what is not struck out, listed: over the others, against the larger maximum
__device__ __forceinline__ Coefs coefs(const DistillParams& p, const Sums& u, const Sums& listed, float w, float rest) {
    Coefs c;
    c.m = fmaxf(u.m, listed.m);
    const float m = c.m == -INFINITY ? 0.0f : c.m;
    const float f = power(u.m - m, p.hi, p.lo), f1 = power(u.m - m, p.hi1, p.lo1);
    c.s = u.s * f + listed.s, c.s1 = u.s1 * f1 + listed.s1;
    c.base = u.m == -INFINITY ? 0.0f : u.m;
    c.empty = c.m == -INFINITY && c.s == 0.0f;
    c.held = rest > 0.0f && u.s > 0.0f;
    const float all = c.held ? w + rest : w;
    c.listed = c.empty ? 0.0f * all : all / c.s;              // a list with a NaN stays one
    c.inv_s1 = c.empty ? 0.0f : 1.0f / c.s1;
    c.others = c.listed * f - (c.held ? rest / u.s : 0.0f);
    c.hard = c.inv_s1 * f1;
    return c;
}

// Sums over the listed tokens, each once, against max(m_u, their own maximum), by one wavefront.
__device__ __forceinline__ Sums sum_list(const DistillParams& p, const List& l, float m_u, bool twice) {
    const int lane = threadIdx.x % 64;
    float m = -INFINITY;
    for (int i = lane; i < p.k; i += 64) m = fmaxf(m, l.z[i]);
    m = wave_max(m);
    const float all = fmaxf(m, m_u), base = all == -INFINITY ? 0.0f : all;
    float s = 0.0f, s1 = 0.0f;
    for (int i = lane; i < p.k; i += 64) {
        if (l.index[i] < 0 || (twice && !first_of(l, i))) continue;
        s += power(l.z[i] - base, p.hi, p.lo), s1 += power(l.z[i] - base, p.hi1, p.lo1);
    }
    return {m, wave_sum(s), wave_sum(s1)};
}

// Loss, likelihood and stats of a row, by one wavefront.
__device__ __forceinline__ void finish_row(const DistillParams& p, const List& l, const Teacher& t, const Sums& u, const Coefs& c, int64_t row) {
    const int lane = threadIdx.x % 64;
    const double inv_t = 1.0 / (double)p.temperature;
    double cross = 0.0;
    bool some = false;
    for (int i = lane; i < p.k; i += 64) {
        if (!(l.q[i] > 0.0f)) continue;                                  // a NaN comes by t.self
        some = true;
        cross += (double)l.q[i] * (((double)l.z[i] - (double)c.m) * inv_t);
    }
    cross = sum_lanes(cross);
    some = __ballot(some) != 0;
    if (lane != 0) return;
    const double log_s = log((double)c.s);
    double loss = t.self - cross + t.w * log_s;
    if (c.held) loss += t.rest * (log(t.rest) - (((double)u.m - (double)c.m) * inv_t + log((double)u.s) - log_s));
    if (c.empty) loss = t.w != t.w ? NAN : some ? INFINITY : 0.0;
    else if (!(c.s < INFINITY)) loss = NAN;
    p.loss[row] = (float)(loss * (double)p.temperature * (double)p.temperature);
    if (p.logprob) {
        float given = 0.0f;
        if (l.index[p.k] >= 0) given = c.empty ? -INFINITY : !(c.s1 < INFINITY) ? NAN : (float)((double)l.z[p.k] - (double)c.m - log((double)c.s1));
        p.logprob[row] = given;
    }
    float* o = p.stats + 8 * row;
    o[0] = c.base, o[1] = c.others, o[2] = c.hard, o[3] = c.m, o[4] = c.listed, o[5] = c.inv_s1, o[6] = t.top, o[7] = c.empty && t.w == t.w ? 0.0f : t.scale;
}

// The gradient of a listed token or of the target (entry k, where it is not listed).
__device__ __forceinline__ float entry_grad(const DistillParams& p, const List& l, const Coefs& c, int i, float g_loss, float g_hard) {
    const bool hard = l.index[p.k] == l.index[i];
    const float at_m = l.z[i] - (c.m == -INFINITY ? 0.0f : c.m);
    float soft;
    if (i == p.k) {
        soft = c.others * power(l.z[i] - c.base, p.hi, p.lo);
    } else {
        float q = l.q[i];
        if (l.twice) {
            q = 0.0f;
            for (int j = 0; j < p.k; ++j) q += l.index[j] == l.index[i] ? l.q[j] : 0.0f;
        }
        soft = c.listed * power(at_m, p.hi, p.lo) - q;
    }
    const float d = g_loss * soft + g_hard * ((hard ? 1.0f : 0.0f) - c.inv_s1 * power(at_m, p.hi1, p.lo1));
    return c.empty ? (soft != soft ? NAN : 0.0f) : d;
}

// Sixteen bytes of logits with the marked ones struck out.
template <typename T>
__device__ __forceinline__ void strike(u4& v, const unsigned* bits, int64_t at) {       // at: the first one's place in the part
    constexpr int N = Vec<T>::kN;
    const unsigned b = (((const uint8_t*)bits)[at / 8] >> (at % 8)) & ((1u << N) - 1);
    if (!b) return;
    float x[N];
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = (b >> e) & 1u ? -INFINITY : Vec<T>::get(v, e);
    v = Vec<T>::pack(x);
}

template <typename T, int NV, int THREADS>
__device__ __forceinline__ void write_grad(const DistillParams& p, u4 (&v)[NV], const Coefs& c, T* d, int64_t start, int64_t end, float g_loss, float g_hard) {
    constexpr int N = Vec<T>::kN;
    const bool two = p.targets && p.temperature != 1.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int64_t i = start + ((int64_t)j * THREADS + threadIdx.x) * N;
        if (i >= end) continue;
        float x[N];
        if (two) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float a = Vec<T>::get(v[j], e) - c.base;
                x[e] = g_loss * (c.others * power(a, p.hi, p.lo)) - g_hard * (c.hard * power(a, p.hi1, p.lo1));
            }
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float w = power(Vec<T>::get(v[j], e) - c.base, p.hi, p.lo);
                x[e] = g_loss * (c.others * w) - g_hard * (c.hard * w);
            }
        }
        store_vec<T>(d, i, end, x);
    }
}

template <typename T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS, 4) void distill_kernel(DistillParams p) {
    constexpr int N = Vec<T>::kN, WAVES = THREADS / 64;
    extern __shared__ unsigned bits[];
    __shared__ List list;
    __shared__ float red_m[WAVES], red_s[WAVES], red_s1[WAVES];
    __shared__ Sums listed;
    __shared__ float list_w, list_rest;
    const int64_t row = blockIdx.x;
    const int part = blockIdx.y, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const T* z = (const T*)p.logits + row * p.row_stride;
    const int64_t start = (int64_t)part * p.part, end = min(start + p.part, p.vocab);
    const bool whole = p.parts == 1;
    u4 v[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] = load_vec<T>(z, start + ((int64_t)j * THREADS + threadIdx.x) * N, end);
    for (int i = threadIdx.x; i < (int)((p.part + 31) / 32); i += THREADS) bits[i] = 0;
    __syncthreads();
    Teacher teacher = {};
    if (wave == 0) {
        read_list<T>(p, list, row, z, start, end);
        in_wave_order();
        mark(p, list, bits, start);
    }
    if (p.rest) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int64_t at = ((int64_t)j * THREADS + threadIdx.x) * N;
            if (start + at < end) strike<T>(v[j], bits, at);
        }
    }
    if (wave == 0 && whole) {
        teacher = weigh(p, list, row);
        if (lane == 0) list_w = (float)teacher.w, list_rest = (float)teacher.rest;
    }
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) m = fmaxf(m, Vec<T>::get(v[j], e));
    keep_packed(v);
    m = wave_max(m);
    if (lane == 0) red_m[wave] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, red_m[w]);
    if (wave == 0 && whole) {
        Sums l{-INFINITY, 0.0f, 0.0f};
        if (p.rest) l = sum_list(p, list, m, list.twice);
        if (lane == 0) listed = l;
    }
    const float base = m == -INFINITY ? 0.0f : m;
    const bool two = p.targets && p.temperature != 1.0f;
    float s = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float s0 = 0.0f;                   // short sums first: fewer roundings of the long ones
#pragma unroll
        for (int e = 0; e < N; ++e) s0 += power(Vec<T>::get(v[j], e) - base, p.hi, p.lo);
        s += s0;
        if (two) {
            s0 = 0.0f;
#pragma unroll
            for (int e = 0; e < N; ++e) s0 += power(Vec<T>::get(v[j], e) - base, p.hi1, p.lo1);
            s1 += s0;
        }
    }
    s = wave_sum(s), s1 = wave_sum(s1);
    if (lane == 0) red_s[wave] = s, red_s1[wave] = s1;
    __syncthreads();
    s = s1 = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += red_s[w], s1 += red_s1[w];
    keep_packed(v);
    const Sums u{m, s, two ? s1 : s};
    if (!whole) {
        if (threadIdx.x == 0) {
            float* o = p.part_sums + 3 * (row * p.parts + part);
            o[0] = u.m, o[1] = u.s, o[2] = u.s1;
        }
        return;
    }
    const Coefs c = coefs(p, u, listed, list_w, list_rest);
    if (wave == 0) finish_row(p, list, teacher, u, c, row);
    if (!p.d_logits) return;
    const float g_loss = p.g_loss ? p.g_loss[row] * p.temperature : 0.0f, g_hard = list.index[p.k] >= 0 && p.g_logprob ? p.g_logprob[row] : 0.0f;
    T* d = (T*)p.d_logits + row * p.d_stride;
    write_grad<T, NV, THREADS>(p, v, c, d, start, end, g_loss, g_hard);
    __syncthreads();
    for (int i = threadIdx.x; i <= p.k; i += THREADS)
        if (list.index[i] >= 0 && !(i == p.k && list.target_listed)) store1(d + list.index[i], entry_grad(p, list, c, i, g_loss, g_hard));
}

// Joins the parts of a row and finishes it.
template <typename T>
__global__ __launch_bounds__(64) void distill_join_kernel(DistillParams p) {
    __shared__ List list;
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x;
    const float* in = p.part_sums + 3 * row * p.parts;
    Sums a{-INFINITY, 0.0f, 0.0f};
    for (int i = lane; i < p.parts; i += 64) a = join(p, a, Sums{in[3 * i], in[3 * i + 1], in[3 * i + 2]});
    for (int o = 32; o; o >>= 1) {
        const Sums b{__shfl_xor(a.m, o), __shfl_xor(a.s, o), __shfl_xor(a.s1, o)};
        a = lane & o ? join(p, b, a) : join(p, a, b);       // the same order in every lane
    }
    read_list<T>(p, list, row, (const T*)p.logits + row * p.row_stride, 0, p.vocab);
    in_wave_order();
    const Teacher teacher = weigh(p, list, row);
    in_wave_order();
    Sums l{-INFINITY, 0.0f, 0.0f};
    if (p.rest) l = sum_list(p, list, a.m, true);
    const Coefs c = coefs(p, a, l, (float)teacher.w, (float)teacher.rest);
    finish_row(p, list, teacher, a, c, row);
}

// The gradient from the logits and what the forward call left.
template <typename T>
__global__ __launch_bounds__(256) void distill_grad_kernel(DistillParams p) {
    constexpr int N = Vec<T>::kN, NV = 4, kSpan = 256 * N * NV;
    __shared__ unsigned bits[kSpan / 32];
    __shared__ List list;
    const int64_t row = blockIdx.x;
    const T* z = (const T*)p.logits + row * p.row_stride;
    T* d = (T*)p.d_logits + row * p.d_stride;
    const int64_t start = (int64_t)blockIdx.y * kSpan, end = min(start + kSpan, p.vocab);
    u4 v[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] = load_vec<T>(z, start + (j * 256 + threadIdx.x) * N, end);
    for (int i = threadIdx.x; i < kSpan / 32; i += 256) bits[i] = 0;
    __syncthreads();
    const float* in = p.stats + 8 * row;
    if (threadIdx.x < 64) {
        read_list<T>(p, list, row, z, start, end);
        in_wave_order();
        mark(p, list, bits, start);
        const float top = in[6], scale = in[7], inv_t = p.rest ? 1.0f : 1.0f / p.temperature;
        for (int i = threadIdx.x; i < p.k; i += 64) {
            const float q = expf((p.value[row * p.k + i] - top) * inv_t) * scale;
            list.q[i] = list.index[i] < 0 || scale == 0.0f ? 0.0f : q;
        }
    }
    Coefs c = {};
    c.base = in[0], c.others = in[1], c.hard = in[2], c.m = in[3], c.listed = in[4], c.inv_s1 = in[5];
    c.empty = c.inv_s1 == 0.0f;
    const int target = p.targets ? p.targets[row] : -1;
    const float g_loss = p.g_loss ? p.g_loss[row] * p.temperature : 0.0f;
    const float g_hard = target >= 0 && target < p.vocab && p.g_logprob ? p.g_logprob[row] : 0.0f;
    __syncthreads();                       // every logit of the list is read: the gradient may lie on them
    write_grad<T, NV, 256>(p, v, c, d, start, end, g_loss, g_hard);
    __syncthreads();
    for (int i = threadIdx.x; i <= p.k; i += 256)
        if (list.index[i] >= 0 && !(i == p.k && list.target_listed)) store1(d + list.index[i], entry_grad(p, list, c, i, g_loss, g_hard));
}

template <typename T, int THREADS, int NV>
hipError_t launch_rows(const DistillParams& p, hipStream_t stream) {
    distill_kernel<T, THREADS, NV><<<dim3((unsigned)p.rows, p.parts), THREADS, (size_t)((p.part + 31) / 32) * 4, stream>>>(p);
    return hipGetLastError();
}
template <typename T, int NV>
hipError_t launch_long(const DistillParams& p, const RowPlan& r, hipStream_t stream) {
    if (r.threads == 256) return launch_rows<T, 256, NV>(p, stream);
    return r.threads == 512 ? launch_rows<T, 512, NV>(p, stream) : launch_rows<T, 1024, NV>(p, stream);
}
template <typename T>
hipError_t launch_typed(const DistillParams& p, const RowPlan& r, hipStream_t stream) {
    if (r.threads == 256) {
        if (r.nv == 2) return launch_rows<T, 256, 2>(p, stream);
        if (r.nv == 4) return launch_rows<T, 256, 4>(p, stream);
        if (r.nv == 8) return launch_rows<T, 256, 8>(p, stream);
    }
    return r.nv <= 10 ? launch_long<T, 10>(p, r, stream) : r.nv == 13 ? launch_long<T, 13>(p, r, stream) : launch_long<T, 16>(p, r, stream);
}

// A launch has fewer than 2^32 threads, a row up to 1024 of them.
constexpr int64_t kMostRows = 1 << 21;
DistillParams rows_of(const DistillParams& p, int64_t first) {
    const int64_t bytes = p.dtype == OLS_F32 ? 4 : 2;
    auto at = [&](auto* t, int64_t per) { return t ? t + per * first : t; };
    DistillParams q = p;
    q.rows = std::min(kMostRows, p.rows - first);
    q.logits = at((const char*)p.logits, p.row_stride * bytes), q.d_logits = at((char*)p.d_logits, p.d_stride * bytes);
    q.value = at(p.value, p.k), q.index = at(p.index, p.k), q.targets = at(p.targets, 1);
    q.g_loss = at(p.g_loss, 1), q.g_logprob = at(p.g_logprob, 1);
    q.loss = at(p.loss, 1), q.logprob = at(p.logprob, 1), q.stats = at(p.stats, 8);
    return q;
}

template <typename T>
hipError_t launch_grad_typed(const DistillParams& p, hipStream_t stream) {
    const int64_t span = 256 * 4 * Vec<T>::kN;
    distill_grad_kernel<T><<<dim3((unsigned)p.rows, (unsigned)((p.vocab + span - 1) / span)), 256, 0, stream>>>(p);
    return hipGetLastError();
}

// log2 e / T as hi + lo, both positive
void split_exponent(double x, float& hi, float& lo) {
    hi = (float)x;
    if ((double)hi >= x) hi = nextafterf(hi, 0.0f);
    lo = (float)(x - (double)hi);
}
DistillParams with_exponents(DistillParams p) {
    constexpr double kLog2 = 1.4426950408889634074;
    split_exponent(kLog2 / (double)p.temperature, p.hi, p.lo);
    split_exponent(kLog2, p.hi1, p.lo1);
    return p;
}

hipError_t grad_rows(const DistillParams& p, hipStream_t stream) {
    return p.dtype == OLS_F32 ? launch_grad_typed<float>(p, stream) : launch_grad_typed<uint16_t>(p, stream);
}

}  // namespace

int64_t distill_workspace_bytes(int dtype, int64_t rows, int64_t vocab) {
    if (rows == 0) return 0;
    const RowPlan r = row_plan(dtype, rows, vocab);
    return r.parts > 1 ? std::min(kMostRows, rows) * r.parts * 12 : 0;
}

hipError_t launch_distill_grad(const DistillParams& params, hipStream_t stream) {
    const DistillParams p = with_exponents(params);
    for (int64_t first = 0; first < p.rows; first += kMostRows) {
        const hipError_t e = grad_rows(rows_of(p, first), stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_distill(const DistillParams& params, void* ws, hipStream_t stream) {
    if (params.rows == 0) return hipSuccess;
    DistillParams p = with_exponents(params);
    const RowPlan r = row_plan(p.dtype, p.rows, p.vocab);
    p.parts = r.parts, p.part = r.part, p.part_sums = (float*)ws;      // one launch's parts after another's in the same place
    for (int64_t first = 0; first < p.rows; first += kMostRows) {
        const DistillParams q = rows_of(p, first);
        hipError_t e = q.dtype == OLS_F32 ? launch_typed<float>(q, r, stream) : launch_typed<uint16_t>(q, r, stream);
        if (e == hipSuccess && r.parts > 1) {
            if (q.dtype == OLS_F32) distill_join_kernel<float><<<(unsigned)q.rows, 64, 0, stream>>>(q);
            else distill_join_kernel<uint16_t><<<(unsigned)q.rows, 64, 0, stream>>>(q);
            e = hipGetLastError();
            if (e == hipSuccess && q.d_logits) e = grad_rows(q, stream);
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace ols
