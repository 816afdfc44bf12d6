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
//
// What bounds it is one read and one write of the logits.  A workgroup holds its part of a row in registers and forms the
// gradient from there; all logits get the gradient of an unlisted one, and behind a barrier the entries of the list and the target
// are written over.  Rows that no workgroup holds and rows too few for the device go in parts, a join and the gradient from memory.
// A pass on 8192 rows of 50 001 bf16 with lists of 32 and targets: 409 us, 4.0 TB/s of that read and write; of 50 000, whose rows all
// begin on vectors, 376 (the loss alone 188 and 154, the gradient from stats 384 and 363).  4096 rows of 128 000 with lists of 100 and
// the rest: 525, 4.0 TB/s (297 and 452).  Lists and losses, launches before and behind the rows', are 6 % of either.
#include "logit_rows.h"

namespace ols {

namespace {

constexpr int kMaxList = OLS_MAX_TEACHER;

// e^{d x} as a power of two: x log2 e and its product with d are rounded, so that the exponent is off by up to 2^-23 of itself
__device__ __forceinline__ float power(float d, float scale) { return __builtin_amdgcn_exp2f(d * scale); }

struct Sums {            // over some of a row: maximum, sum of e^{(z - m) / T}, sum of e^{z - m}
    float m, s, s1;
};
__device__ __forceinline__ Sums join(const DistillParams& p, const Sums& a, const Sums& b) {
    const float m = fmaxf(a.m, b.m), base = m == -INFINITY ? 0.0f : m;
    const float da = a.m - base, db = b.m - base;                         // -inf where a side is empty
    return {m, a.s * power(da, p.scale) + b.s * power(db, p.scale), a.s1 * power(da, p.scale1) + b.s1 * power(db, p.scale1)};
}

// A row's list in LDS: places in the row (-1: none), the teacher's values and then q, and the student's logits.
struct List {
    int index[kMaxList];
    float q[kMaxList], z[kMaxList];
};

// What is known of a row from its list and target alone.
struct Teacher {
    double w, rest, self, cross;         // sum of q, q_r, sums of q log q and of q (z - m) / T
    float m, s, s1;                      // of the listed tokens, each once: largest logit, sums of e^{(z - m) / T} and e^{z - m}
    float z_target;
    float top, scale;                    // q_j = e^{(v_j - top) / T or v_j} scale
    int target;                          // -1: none
    int target_listed, twice, any;       // the target is in the list; a token is named twice; some q is positive
};

// Reads a row's list and target; by one wavefront.  kept: their logits, where the launch may write over them.
template <typename T>
__device__ __forceinline__ void read_list(const DistillParams& p, List& l, Teacher& t, int64_t row, const T* z, const float* kept = nullptr) {
    const int target = p.targets ? p.targets[row] : -1;
    t.target = target >= 0 && target < p.vocab ? target : -1;
    bool met = false;
    for (int i = threadIdx.x % 64; i < p.k; i += 64) {
        const int at = p.index[row * p.k + i];
        const float value = p.value[row * p.k + i];            // under way with the index, not behind what follows from it
        const bool there = at >= 0 && at < p.vocab;
        l.index[i] = there ? at : -1;
        l.q[i] = value;
        l.z[i] = !there ? -INFINITY : kept ? kept[i] : load1(z + at);
        met |= there && at == t.target;
    }
    t.target_listed = __ballot(met) != 0;
    t.z_target = t.target < 0 ? -INFINITY : kept ? kept[p.k] : load1(z + t.target);
    in_wave_order();
}

// The teacher's probabilities into l.q and the sums over the list, by one wavefront.  A NaN or +inf among the values makes them all NaN.
__device__ __forceinline__ void weigh(const DistillParams& p, List& l, Teacher& t) {
    const int lane = threadIdx.x % 64;
    float top = -INFINITY, m = -INFINITY;
    bool some = false, bad = false, again = false;
    for (int i = lane; i < p.k; i += 64) {
        if (l.index[i] < 0) continue;
        const float v = l.q[i];
        some = true, bad |= !(v < INFINITY);
        top = fmaxf(top, v), m = fmaxf(m, l.z[i]);
    }
    some = __ballot(some) != 0, bad = __ballot(bad) != 0;
    top = wave_max(top);
    t.m = wave_max(m);
    t.top = p.rest || top == -INFINITY ? 0.0f : top;
    const float base = t.m == -INFINITY ? 0.0f : t.m;
    const double inv_t = 1.0 / (double)p.temperature, inv_v = p.rest ? 1.0 : inv_t;
    double w = 0.0, self = 0.0, cross = 0.0;
    float s = 0.0f, s1 = 0.0f;
    for (int i = lane; i < p.k; i += 64) {
        float q = 0.0f;
        if (l.index[i] >= 0) {
            const double u = ((double)l.q[i] - t.top) * inv_v, e = exp(u);
            w += e, self += e > 0.0 ? e * u : 0.0, cross += e > 0.0 ? e * (((double)l.z[i] - (double)base) * inv_t) : 0.0;
            q = (float)e;
            bool first = true;
            for (int j = 0; j < i; j += 4) {                   // whether the token was named before
                const int4 at = *(const int4*)(l.index + j);
                first &= !(at.x == l.index[i] || (at.y == l.index[i] && j + 1 < i) || (at.z == l.index[i] && j + 2 < i) || (at.w == l.index[i] && j + 3 < i));
            }
            again |= !first;
            if (first) s += power(l.z[i] - base, p.scale), s1 += power(l.z[i] - base, p.scale1);
        }
        l.q[i] = q;
    }
    w = wave_sum(w), self = wave_sum(self), cross = wave_sum(cross);
    t.s = wave_sum(s), t.s1 = wave_sum(s1);
    t.twice = __ballot(again) != 0;
    t.any = w > 0.0;
    t.scale = 1.0f, t.rest = 0.0;
    if (p.rest) {
        t.rest = some ? fmax(1.0 - w, 0.0) : 0.0;
    } else if (w > 0.0) {
        t.scale = (float)(1.0 / w);
        self = self / w - log_of(w), cross /= w;
        for (int i = lane; i < p.k; i += 64) l.q[i] *= t.scale;
        w = 1.0;
    }
    if (bad) w = self = NAN, t.scale = NAN;
    t.w = w, t.self = self, t.cross = cross;
    in_wave_order();
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
// u: over what is not struck out, which are all where the rest does not count.
__device__ __forceinline__ Coefs coefs(const DistillParams& p, const Sums& u, const Sums& listed, float w, float rest) {
    Coefs c;
    const Sums all = p.rest ? join(p, u, listed) : u;
    c.m = all.m, c.s = all.s, c.s1 = all.s1;
    const float m = c.m == -INFINITY ? 0.0f : c.m;
    c.base = u.m == -INFINITY ? 0.0f : u.m;
    c.empty = c.m == -INFINITY && c.s == 0.0f;
    c.held = rest > 0.0f && u.s > 0.0f;
    const float both = c.held ? w + rest : w;
    c.listed = c.empty ? 0.0f * both : both / c.s;             // a list with a NaN stays one
    c.inv_s1 = c.empty ? 0.0f : 1.0f / c.s1;
    c.others = c.listed * power(u.m - m, p.scale) - (c.held ? rest / u.s : 0.0f);
    c.hard = c.inv_s1 * power(u.m - m, p.scale1);
    return c;
}
__device__ __forceinline__ Coefs coefs(const DistillParams& p, const Sums& u, const Teacher& t) { return coefs(p, u, Sums{t.m, t.s, t.s1}, (float)t.w, (float)t.rest); }

// Loss, likelihood and stats of a row, by one lane.
__device__ __forceinline__ void finish_row(const DistillParams& p, const Teacher& t, const Sums& u, const Coefs& c, int64_t row) {
    const double inv_t = 1.0 / (double)p.temperature, log_s = log_of((double)c.s);
    // t.cross is against the listed tokens' own maximum
    double loss = t.self + t.w * log_s;
    if (t.any) loss -= t.cross + t.w * (((t.m == -INFINITY ? 0.0 : (double)t.m) - (double)c.m) * inv_t);
    if (c.held) loss += t.rest * (log_of(t.rest) - (((double)u.m - (double)c.m) * inv_t + log_of((double)u.s) - log_s));
    if (c.empty) loss = t.w != t.w ? NAN : t.any ? INFINITY : 0.0;
    else if (!(c.s < INFINITY)) loss = NAN;
    p.loss[row] = (float)(loss * (double)p.temperature * (double)p.temperature);
    if (p.logprob) {
        float given = 0.0f;
        if (t.target >= 0) given = c.empty ? -INFINITY : !(c.s1 < INFINITY) ? NAN : (float)((double)t.z_target - (double)c.m - log_of((double)c.s1));
        p.logprob[row] = given;
    }
    float* o = p.stats + 8 * row;
    o[0] = c.base, o[1] = c.others, o[2] = c.hard, o[3] = c.m, o[4] = c.listed, o[5] = c.inv_s1, o[6] = t.top, o[7] = c.empty && t.w == t.w ? 0.0f : t.scale;
}

// The gradient of a listed token (q: of all its entries) or of an unlisted target.
__device__ __forceinline__ float entry_grad(const DistillParams& p, const Coefs& c, float z, bool listed, float q, bool target, float g_loss, float g_hard) {
    const float at_m = z - (c.m == -INFINITY ? 0.0f : c.m);
    const float soft = listed ? c.listed * power(at_m, p.scale) - q : c.others * power(z - c.base, p.scale);
    const float d = g_loss * soft + g_hard * ((target ? 1.0f : 0.0f) - c.inv_s1 * power(at_m, p.scale1));
    return c.empty ? (soft != soft ? NAN : 0.0f) : d;
}

// A row, or a part of one, in the registers of a workgroup: whole vectors, and of what is left of the last one a logit in each of the
// first lanes.  Addresses are a uniform pointer and a lane's offset: kept for every vector, as 64-bit numbers, they spill.
template <typename T, int THREADS, int NV>
struct Held {
    static constexpr int kN = Vec<T>::kN;
    u4 v[NV];
    float tail;                          // -inf where there is none

    __device__ static void load_one(u4& v, int j, const T* row, int length) {
        v = u4{Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone, Vec<T>::kNone};
        if ((int)threadIdx.x < length / kN - j * THREADS) v = *(const u4any*)((const char*)row + (size_t)j * THREADS * 16 + threadIdx.x * 16u);
    }
    __device__ void load_tail(const T* row, int length) { tail = (int)threadIdx.x < length % kN ? load1(row + length / kN * kN + threadIdx.x) : -INFINITY; }
    __device__ void load(const T* row, int length) {
#pragma unroll
        for (int j = 0; j < NV; ++j) load_one(v[j], j, row, length);
        load_tail(row, length);
    }
    // The logits whose bits are set become -inf.
    __device__ void strike(const unsigned* bits, int length) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int at = (j * THREADS + (int)threadIdx.x) * kN;
            if (at + kN > length) continue;
            const unsigned b = (((const uint8_t*)bits)[at / 8] >> (at % 8)) & ((1u << kN) - 1);
            if (!b) continue;
            float x[kN];
#pragma unroll
            for (int e = 0; e < kN; ++e) x[e] = (b >> e) & 1u ? -INFINITY : Vec<T>::get(v[j], e);
            v[j] = Vec<T>::pack(x);
        }
        const int at = length / kN * kN + (int)threadIdx.x;
        if (at < length && (bits[at / 32] >> (at % 32)) & 1u) tail = -INFINITY;
    }
    __device__ float largest() const {
        float m = tail;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < kN; ++e) m = fmaxf(m, Vec<T>::get(v[j], e));
        return m;
    }
};

// What e^{z - base} takes: nothing more, a square, or an exponential of its own.
enum Second { kNone, kSquare, kOther };
__host__ __device__ __forceinline__ Second second_of(const DistillParams& p) { return !p.targets || p.temperature == 1.0f ? kNone : p.temperature == 2.0f ? kSquare : kOther; }

// Adds up e^{(z - base) / T} and, where it is another, e^{z - base}.  Short sums first: fewer roundings of the long ones.
template <Second SECOND>
__device__ __forceinline__ void add_one(const DistillParams& p, float d, float& a, float& b) {
    const float w = power(d, p.scale);
    a += w;
    if constexpr (SECOND == kSquare) b = fmaf(w, w, b);
    if constexpr (SECOND == kOther) b += power(d, p.scale1);
}
template <Second SECOND, typename T, int THREADS, int NV>
__device__ __forceinline__ void add_up(const DistillParams& p, const Held<T, THREADS, NV>& h, float base, float& s, float& s1) {
    add_one<SECOND>(p, h.tail - base, s, s1);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float a = 0.0f, b = 0.0f;
#pragma unroll
        for (int e = 0; e < Vec<T>::kN; ++e) add_one<SECOND>(p, Vec<T>::get(h.v[j], e) - base, a, b);
        s += a, s1 += b;
    }
}

// Writes the gradient of logits that are not listed; a register that is done with is filled from the next row.
template <Second SECOND>
__device__ __forceinline__ float one_grad(const DistillParams& p, float d, float soft, float hard) {
    const float w = power(d, p.scale);
    if constexpr (SECOND == kNone) return soft * w;
    if constexpr (SECOND == kSquare) return w * fmaf(-hard, w, soft);
    return fmaf(-hard, power(d, p.scale1), soft * w);
}
template <Second SECOND, typename T, int THREADS, int NV>
__device__ __forceinline__ void write_grad(const DistillParams& p, Held<T, THREADS, NV>& h, const Coefs& c, T* d, const T* next, int length, float g_loss, float g_hard) {
    constexpr int N = Vec<T>::kN;
    const float hard = g_hard * c.hard, soft = SECOND == kNone ? g_loss * c.others - hard : g_loss * c.others;    // factors of at most about one
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float x[N];
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = one_grad<SECOND>(p, Vec<T>::get(h.v[j], e) - c.base, soft, hard);
        if ((int)threadIdx.x < length / N - j * THREADS) *(u4any*)((char*)d + (size_t)j * THREADS * 16 + threadIdx.x * 16u) = Vec<T>::pack(x);
        if (next) Held<T, THREADS, NV>::load_one(h.v[j], j, next, length);
        __builtin_amdgcn_sched_barrier(0);       // registers
    }
    if ((int)threadIdx.x < length % N) store1(d + length / N * N + threadIdx.x, one_grad<SECOND>(p, h.tail - c.base, soft, hard));
    if (next) h.load_tail(next, length);
}
// The teacher's side of whole rows, a wavefront for each: lists' sums, q and logits go to the workspace.  In a kernel of its own, since fp64
// functions take the registers that hold rows.
template <typename T>
__global__ __launch_bounds__(256) void distill_list_kernel(DistillParams p) {
    __shared__ __align__(16) List lists[4];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t row = (int64_t)blockIdx.x * 4 + wave;
    if (row >= p.rows) return;
    List& l = lists[wave];
    Teacher t;
    read_list<T>(p, l, t, row, (const T*)p.logits + row * p.row_stride);
    weigh(p, l, t);
    if (lane == 0) ((Teacher*)p.teachers)[row] = t;
    for (int i = lane; i < p.k; i += 64) p.list_q[row * p.k + i] = l.q[i], p.list_z[row * p.k + i] = l.z[i];
}
// ... and its end, a lane for each row.
__global__ __launch_bounds__(64) void distill_loss_kernel(DistillParams p) {
    const int64_t row = (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (row >= p.rows) return;
    const Teacher t = ((const Teacher*)p.teachers)[row];
    const float* in = p.part_sums + 3 * row;
    const Sums u{in[0], in[1], in[2]};
    finish_row(p, t, u, coefs(p, u, t), row);
}

// Whole rows: a workgroup takes every gridDim.x-th, and reads the next one while it writes the gradient of this.  Parts of rows: one each.
template <typename T, int THREADS, int NV, Second SECOND>
__global__ __launch_bounds__(THREADS, 4) void distill_kernel(DistillParams p) {
    constexpr int WAVES = THREADS / 64;
    extern __shared__ unsigned bits[];
    __shared__ float red_m[WAVES], red_s[WAVES], red_s1[WAVES];
    const int part = blockIdx.y, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t start = (int64_t)part * p.part, end = min(start + p.part, p.vocab);
    const int length = (int)(end - start);
    const bool whole = p.parts == 1;
    Held<T, THREADS, NV> h;
    h.load((const T*)p.logits + (int64_t)blockIdx.x * p.row_stride + start, length);
    if (p.rest)
        for (int i = threadIdx.x; i < (length + 31) / 32; i += THREADS) bits[i] = 0;
    auto place = [&](int64_t row) {            // of the lane's entry of a list; no list is longer than a workgroup
        if ((int)threadIdx.x >= p.k || row >= p.rows) return -1;
        const int at = p.index[row * p.k + threadIdx.x];
        return at >= start && at < end ? (int)(at - start) : -1;
    };
    int at = place(blockIdx.x);
    if (!whole) {
        // The listed logits and the target's, for the workgroups that finish the row: the gradient of one may lie on what another reads.
        float* kept = p.list_z + (int64_t)blockIdx.x * (p.k + 1);
        const T* z = (const T*)p.logits + (int64_t)blockIdx.x * p.row_stride;
        if (at >= 0) kept[threadIdx.x] = load1(z + start + at);
        const int target = threadIdx.x == 0 && p.targets ? p.targets[blockIdx.x] : -1;
        if (target >= start && target < end) kept[p.k] = load1(z + target);
    }
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        if (p.rest) {
            __syncthreads();                   // the bits are clear
            if (at >= 0) atomicOr(&bits[at / 32], 1u << (at % 32));
            __syncthreads();
            h.strike(bits, length);
        }
        float m = wave_max(h.largest());
        keep_packed(h.v);
        if (lane == 0) red_m[wave] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, red_m[w]);
        float s = 0.0f, s1 = 0.0f;
        add_up<SECOND>(p, h, m == -INFINITY ? 0.0f : m, s, s1);
        keep_packed(h.v);
        s = wave_sum(s), s1 = wave_sum(s1);
        if (lane == 0) red_s[wave] = s, red_s1[wave] = s1;
        __syncthreads();
        s = s1 = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) s += red_s[w], s1 += red_s1[w];
        const Sums u{m, s, SECOND == kNone ? s : s1};
        if (threadIdx.x == 0) {
            float* o = p.part_sums + 3 * (row * p.parts + part);
            o[0] = u.m, o[1] = u.s, o[2] = u.s1;
        }
        if (!whole || !p.d_logits) return;     // without a gradient there is a workgroup for each row
        const T* next = row + gridDim.x < p.rows ? (const T*)p.logits + (row + gridDim.x) * p.row_stride : nullptr;
        const int next_at = place(row + gridDim.x);
        const Teacher& t = ((const Teacher*)p.teachers)[row];
        const Coefs c = coefs(p, u, t);
        const float g_loss = p.g_loss ? p.g_loss[row] * p.temperature : 0.0f, g_hard = t.target >= 0 && p.g_logprob ? p.g_logprob[row] : 0.0f;
        T* d = (T*)p.d_logits + row * p.d_stride;
        const float entry_q = at >= 0 ? p.list_q[row * p.k + threadIdx.x] : 0.0f, entry_z = at >= 0 ? p.list_z[row * p.k + threadIdx.x] : 0.0f;
        write_grad<SECOND>(p, h, c, d, next, length, g_loss, g_hard);
        __syncthreads();                   // the list and the target are written over
        if (at >= 0) {
            float q = entry_q;
            if (t.twice) {
                q = 0.0f;
                for (int j = 0; j < p.k; ++j) q += p.index[row * p.k + j] == at ? p.list_q[row * p.k + j] : 0.0f;
            }
            store1(d + at, entry_grad(p, c, entry_z, true, q, at == t.target, g_loss, g_hard));
        }
        if (threadIdx.x == 0 && t.target >= 0 && !t.target_listed) store1(d + t.target, entry_grad(p, c, t.z_target, false, 0.0f, true, g_loss, g_hard));
        if (p.rest && at >= 0) bits[at / 32] = 0;
        at = next_at;
    }
}

// The rest of a call behind the parts, with JOIN: every workgroup joins the parts of its row, the first one writes its results, and all write
// their logits' gradient.  Otherwise the gradient from what an earlier call left.
template <typename T, bool JOIN>
__global__ __launch_bounds__(256) void distill_finish_kernel(DistillParams p) {
    constexpr int NV = 4, kSpan = 256 * Vec<T>::kN * NV;
    __shared__ __align__(16) List list;
    __shared__ Coefs shared;
    __shared__ int listed, twice;
    const int64_t row = blockIdx.x;
    const T* z = (const T*)p.logits + row * p.row_stride;
    T* d = p.d_logits ? (T*)p.d_logits + row * p.d_stride : nullptr;
    const int64_t start = (int64_t)blockIdx.y * kSpan, end = min(start + kSpan, p.vocab);
    const int length = (int)(end - start), lane = threadIdx.x;
    Held<T, 256, NV> h;
    if (d) h.load(z + start, length);
    const float* in = p.stats + 8 * row;
    Teacher t;
    Sums a{-INFINITY, 0.0f, 0.0f};
    if (lane < 64) {
        const float* sums = JOIN ? p.part_sums + 3 * row * p.parts : nullptr;
        if (JOIN && lane < p.parts) a = Sums{sums[3 * lane], sums[3 * lane + 1], sums[3 * lane + 2]};
        read_list<T>(p, list, t, row, z, JOIN ? p.list_z + row * (p.k + 1) : nullptr);
        if constexpr (JOIN) {
            for (int i = lane + 64; i < p.parts; i += 64) a = join(p, a, Sums{sums[3 * i], sums[3 * i + 1], sums[3 * i + 2]});
            for (int o = 32; o; o >>= 1) {
                const Sums b{__shfl_xor(a.m, o), __shfl_xor(a.s, o), __shfl_xor(a.s1, o)};
                a = lane & o ? join(p, b, a) : join(p, a, b);       // the same order in every lane
            }
            weigh(p, list, t);
            const Coefs c = coefs(p, a, t);
            if (lane == 0) shared = c, listed = t.target_listed, twice = t.twice;
        } else {
            const float top = in[6], scale = in[7], inv_t = p.rest ? 1.0f : 1.0f / p.temperature;
            for (int i = lane; i < p.k; i += 64) {
                const float q = expf((list.q[i] - top) * inv_t) * scale;
                list.q[i] = list.index[i] < 0 || scale == 0.0f ? 0.0f : q;
            }
            if (lane == 0) {
                Coefs c = {};
                c.base = in[0], c.others = in[1], c.hard = in[2], c.m = in[3], c.listed = in[4], c.inv_s1 = in[5], c.empty = c.inv_s1 == 0.0f;
                shared = c, listed = t.target_listed, twice = 1;
            }
        }
    }
    auto finish = [&]() {                      // behind the gradient, which waits for it nowhere
        if (JOIN && blockIdx.y == 0 && lane == 0) finish_row(p, t, a, shared, row);
    };
    if (!d) return finish();
    const int target = p.targets ? p.targets[row] : -1;
    const bool has_target = target >= start && target < end;
    const float z_target = has_target ? load1(z + target) : 0.0f;
    const float g_loss = p.g_loss ? p.g_loss[row] * p.temperature : 0.0f;
    const float g_hard = target >= 0 && target < p.vocab && p.g_logprob ? p.g_logprob[row] : 0.0f;
    __syncthreads();                           // the logits of the part are read: the gradient may lie on them
    const Coefs c = shared;
    const Second second = second_of(p);
    if (second == kNone) write_grad<kNone>(p, h, c, d + start, (const T*)nullptr, length, g_loss, g_hard);
    else if (second == kSquare) write_grad<kSquare>(p, h, c, d + start, (const T*)nullptr, length, g_loss, g_hard);
    else write_grad<kOther>(p, h, c, d + start, (const T*)nullptr, length, g_loss, g_hard);
    __syncthreads();
    for (int i = lane; i < p.k; i += 256) {
        const int at = list.index[i];
        if (at < start || at >= end) continue;
        float q = list.q[i];
        if (twice) {
            q = 0.0f;
            for (int j = 0; j < p.k; ++j) q += list.index[j] == at ? list.q[j] : 0.0f;
        }
        store1(d + at, entry_grad(p, c, list.z[i], true, q, at == target, g_loss, g_hard));
    }
    if (lane == 0 && has_target && !listed) store1(d + target, entry_grad(p, c, z_target, false, 0.0f, true, g_loss, g_hard));
    finish();
}

template <typename T, int THREADS, int NV>
hipError_t launch_rows(const DistillParams& p, hipStream_t stream) {
    const int64_t fill = (int64_t)256 * (1024 / THREADS) * (NV <= 4 ? 2 : 1);     // workgroups that run beside each other
    const dim3 grid((unsigned)(p.parts > 1 || !p.d_logits ? p.rows : std::min(p.rows, fill)), p.parts);
    const size_t lds = p.rest ? (size_t)((p.part + 31) / 32) * 4 : 0;
    const Second second = second_of(p);
    if (second == kNone) distill_kernel<T, THREADS, NV, kNone><<<grid, THREADS, lds, stream>>>(p);
    else if (second == kSquare) distill_kernel<T, THREADS, NV, kSquare><<<grid, THREADS, lds, stream>>>(p);
    else distill_kernel<T, THREADS, NV, kOther><<<grid, THREADS, lds, stream>>>(p);
    return hipGetLastError();
}
template <typename T, int THREADS>
hipError_t launch_threads(const DistillParams& p, const RowPlan& r, hipStream_t stream) {
    if (r.nv == 2) return launch_rows<T, THREADS, 2>(p, stream);
    if constexpr (THREADS > 64) {
        if (r.nv == 8) return launch_rows<T, THREADS, 8>(p, stream);
        if (r.nv == 13) return launch_rows<T, THREADS, 13>(p, stream);
        if (r.nv == 16) return launch_rows<T, THREADS, 16>(p, stream);
    }
    return launch_rows<T, THREADS, 4>(p, stream);
}
template <typename T>
hipError_t launch_typed(const DistillParams& p, const RowPlan& r, hipStream_t stream) {
    if (r.threads == 64) return launch_threads<T, 64>(p, r, stream);
    if (r.threads == 256) return launch_threads<T, 256>(p, r, stream);
    return r.threads == 512 ? launch_threads<T, 512>(p, r, stream) : launch_threads<T, 1024>(p, r, stream);
}

// Short rows take a wavefront each, where it holds them and their list: a row is a chain of waits, and four times as many run beside each
// other (8192 rows of 1000 bf16, all launches: 48 us in workgroups of 256, 28 so).  Wider workgroups for rows that fit narrow ones do not help (700
// rows of 32 000: 46 us in 256 lanes, 51 in 512).
RowPlan distill_plan(int dtype, int64_t rows, int64_t vocab, int k) {
    RowPlan r = row_plan(dtype, rows, vocab);
    const int64_t n = dtype == OLS_F32 ? 4 : 8;
    if (r.parts == 1) {
        const bool short_row = vocab <= 64 * 4 * n && k <= 64;
        r.threads = short_row ? 64 : 256;
        while (!short_row && r.threads < 1024 && vocab > r.threads * 16 * n) r.threads *= 2;
    }
    const int64_t per = (r.part + r.threads * n - 1) / (r.threads * n);
    r.nv = per <= 2 ? 2 : per <= 4 ? 4 : per <= 8 ? 8 : per <= 13 ? 13 : 16;
    return r;
}

// A launch has fewer than 2^32 threads: a row up to 1024 for each of its parts, or 256 for each of its pieces in the gradient from memory.
int64_t most_rows(int dtype, int64_t vocab) { return std::max<int64_t>(1, (1 << 21) / ((vocab + (dtype == OLS_F32 ? 4095 : 8191)) / (dtype == OLS_F32 ? 4096 : 8192))); }
DistillParams rows_of(const DistillParams& p, int64_t first) {
    const int64_t bytes = p.dtype == OLS_F32 ? 4 : 2;
    auto at = [&](auto* t, int64_t per) { return t ? t + per * first : t; };
    DistillParams q = p;
    q.rows = std::min(most_rows(p.dtype, p.vocab), p.rows - first);
    q.logits = at((const char*)p.logits, p.row_stride * bytes), q.d_logits = at((char*)p.d_logits, p.d_stride * bytes);
    q.value = at(p.value, p.k), q.index = at(p.index, p.k), q.targets = at(p.targets, 1);
    q.g_loss = at(p.g_loss, 1), q.g_logprob = at(p.g_logprob, 1);
    q.loss = at(p.loss, 1), q.logprob = at(p.logprob, 1), q.stats = at(p.stats, 8);
    return q;
}

template <typename T, bool JOIN>
hipError_t launch_finish(const DistillParams& p, hipStream_t stream) {
    const int64_t span = 256 * 4 * Vec<T>::kN;
    distill_finish_kernel<T, JOIN><<<dim3((unsigned)p.rows, p.d_logits ? (unsigned)((p.vocab + span - 1) / span) : 1), 256, 0, stream>>>(p);
    return hipGetLastError();
}

DistillParams with_exponents(DistillParams p) {
    constexpr double kLog2 = 1.4426950408889634074;
    p.scale = (float)(kLog2 / (double)p.temperature), p.scale1 = (float)kLog2;
    return p;
}

}  // namespace

// Whole rows: of each what its list adds up to, q and z, and the sums.  Parts: their sums, and the listed logits and the target's.
int64_t distill_workspace_bytes(int dtype, int64_t rows, int64_t vocab, int k) {
    if (rows == 0) return 0;
    const RowPlan r = distill_plan(dtype, rows, vocab, k);
    rows = std::min(most_rows(dtype, vocab), rows);
    return rows * (r.parts > 1 ? r.parts * 12 + 4 * (k + 1) : (int64_t)sizeof(Teacher) + 12 + 8 * k);
}

hipError_t launch_distill_grad(const DistillParams& params, hipStream_t stream) {
    const DistillParams p = with_exponents(params);
    for (int64_t first = 0; first < p.rows; first += most_rows(p.dtype, p.vocab)) {
        const DistillParams q = rows_of(p, first);
        const hipError_t e = q.dtype == OLS_F32 ? launch_finish<float, false>(q, stream) : launch_finish<uint16_t, false>(q, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_distill(const DistillParams& params, void* ws, hipStream_t stream) {
    if (params.rows == 0) return hipSuccess;
    DistillParams p = with_exponents(params);
    const RowPlan r = distill_plan(p.dtype, p.rows, p.vocab, p.k);
    p.parts = r.parts, p.part = r.part;
    for (int64_t first = 0; first < p.rows; first += most_rows(p.dtype, p.vocab)) {
        DistillParams q = rows_of(p, first);                           // one launch's rows after another's in the same place
        hipError_t e = hipSuccess;
        if (r.parts > 1) {
            q.part_sums = (float*)ws, q.list_z = q.part_sums + 3 * q.rows * r.parts;
        } else {
            q.teachers = ws;
            q.part_sums = (float*)((char*)ws + q.rows * sizeof(Teacher)), q.list_q = q.part_sums + 3 * q.rows, q.list_z = q.list_q + q.rows * q.k;
            const unsigned blocks = (unsigned)((q.rows + 3) / 4);
            if (q.dtype == OLS_F32) distill_list_kernel<float><<<blocks, 256, 0, stream>>>(q);
            else distill_list_kernel<uint16_t><<<blocks, 256, 0, stream>>>(q);
            e = hipGetLastError();
        }
        if (e == hipSuccess) e = q.dtype == OLS_F32 ? launch_typed<float>(q, r, stream) : launch_typed<uint16_t>(q, r, stream);
        if (e != hipSuccess) return e;
        if (r.parts > 1) {
            e = q.dtype == OLS_F32 ? launch_finish<float, true>(q, stream) : launch_finish<uint16_t, true>(q, stream);
        } else {
            distill_loss_kernel<<<(unsigned)((q.rows + 63) / 64), 64, 0, stream>>>(q);
            e = hipGetLastError();
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace ols
