// One step of beam search over several requests: which hypotheses go on and with which token, and moving their states.
//
//   logp_iv = (z_iv - m_i) - log sum_v e^{z_iv - m_i}
//   candidates:  (i, v) of value score_i + logp_iv and length length_i + 1;  of an ended hypothesis only itself, (i, 0) of value score_i
//   order:       by value / length^penalty, largest first; ties to the lower hypothesis, then to the lower token
//
// Within a hypothesis that is the order of its logits, which is exact: in a part's list, and in the merge where heads of two parts have the same
// value in fp64 (a score that swallows the logits, logits that are tiny beside it).  Between hypotheses it hangs on the last bits of the
// sums: these are added up in fp64, and candidates are compared in fp64.
//
// The choice reads the logits once: a workgroup holds its part of a hypothesis' row in registers, takes the sum
// and the part's best from there (logit_rows.h), and one wavefront for each request merges the parts' lists, each in order: a lane
// holds the heads of its lists, and every turn takes the best head of all.  Ended hypotheses are not read.  512 hypotheses of 128 000
// bf16 (64 requests, the best 8 of each; a fifth has ended, 105 MB are read): 33 us, 3.2 TB/s, since nothing of a workgroup's own is under way
// while it looks for its best, and 10.7 for the merge; few requests are two launches of 6 to 7 us, latencies.
//
// Moving states is one read and one write of what moves.  A thread holds the same sixteen bytes of all hypotheses of a request: all
// are read before one is written, so that states can be moved in place, and a hypothesis that stays where it is is not touched then.
// Four tensors of 33.5 MB into others: 36 us, 7.4 TB/s of what lies in the caches.
#include "logit_rows.h"

namespace ols {

namespace {

// log2 e is rounded by 2^-26 of itself, which moves a row's logarithm by 1e-8 of its logits' mean distance from the largest: rows of one
// model by nearly the same.
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// A hypothesis that is read: it has a score and has not ended.
__device__ __forceinline__ bool goes_on(const BeamParams& p, int64_t row) {
    return !(p.score[row] == -INFINITY) && !(p.finished && p.finished[row]);
}

// The best k of what a workgroup of 256 holds, as best_of_part does it, from a bound that is quicker to find: of 16, 32 or 64 groups of
// lanes, at least 2 k, the k-th largest of their maxima, which at least k logits reach and few others (of 32 groups the 32nd is the smallest: in the worst of
// 512 parts 300 logits lie above it, whose order took 28 us).  Where more do than the list holds (many equal
// ones, or one lane that holds them all) best_of_part takes over.  512 rows of 128 000 bf16, 8 of each: best_of_part 15 us of 39.
template <typename T, int NV>
__device__ __forceinline__ void best_of_groups(const u4 (&v)[NV], float lane_max, int64_t start, int k, int room, float* list_val, int* list_idx, float* best_val,
                                               int* best_idx) {
    constexpr int N = Vec<T>::kN;
    __shared__ float tops[64];
    __shared__ int listed;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    float m = lane_max;
    m = fmaxf(m, moved<0x111, 0xf>(m, -INFINITY));
    m = fmaxf(m, moved<0x112, 0xf>(m, -INFINITY));
    if (k <= 16) m = fmaxf(m, moved<0x114, 0xf>(m, -INFINITY));
    if (k <= 8) m = fmaxf(m, moved<0x118, 0xf>(m, -INFINITY));
    const int size = k <= 8 ? 16 : k <= 16 ? 8 : 4, groups = 256 / size;       // lane size - 1 of a group has seen all of it
    if (lane % size == size - 1) tops[(wave * 64 + lane) / size] = m;
    if (threadIdx.x == 0) listed = 0;
    __syncthreads();
    const float mine = lane < groups ? tops[lane] : -INFINITY;
    int above = 0, with = 0;                                   // groups above the lane's, and with those equal to it
#pragma unroll 16
    for (int i = 0; i < groups; ++i) {
        const float other = lane_of(mine, i);
        above += other > mine ? 1 : 0, with += other >= mine ? 1 : 0;
    }
    const unsigned long long at = __ballot(lane < groups && above < k && with >= k);
    const float limit = at ? lane_of(mine, __ffsll(at) - 1) : -INFINITY;
    if (__ballot(lane_max >= limit && lane_max > -INFINITY)) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float top = Vec<T>::get(v[j], 0);
#pragma unroll
            for (int e = 1; e < N; ++e) top = fmaxf(top, Vec<T>::get(v[j], e));
            if (!(top >= limit && top > -INFINITY)) continue;
            const int64_t first = start + ((int64_t)j * 256 + threadIdx.x) * N;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float x = Vec<T>::get(v[j], e);
                if (!(x >= limit && x > -INFINITY)) continue;
                const int to = atomicAdd(&listed, 1);
                if (to < room) list_val[to] = x, list_idx[to] = (int)(first + e);
            }
        }
    }
    __syncthreads();
    if (listed > room) {
        best_of_part<T, 256, NV>(v, lane_max, start, k, list_val, list_idx, best_val, best_idx);
        return;
    }
    if (listed <= 64) {
        write_best<256>(list_val, list_idx, listed, k, best_val, best_idx);
    } else {                                                   // four listed ones at a time; there is room for four (k >= 9 here, or many are equal)
        const int count = listed, whole = (count + 3) / 4;
        if ((int)threadIdx.x < 4 * whole - count) list_val[count + threadIdx.x] = -INFINITY, list_idx[count + threadIdx.x] = 0x7fffffff;
        __syncthreads();
        for (int i = threadIdx.x; i < count; i += 256) {
            const float x = list_val[i];
            const int at_x = list_idx[i];
            int place = 0;
#pragma unroll 2
            for (int j = 0; j < whole; ++j) {
                const f4 y = ((const f4*)list_val)[j];
                const int4 at_y = ((const int4*)list_idx)[j];
                place += (beats(y[0], at_y.x, x, at_x) ? 1 : 0) + (beats(y[1], at_y.y, x, at_x) ? 1 : 0) + (beats(y[2], at_y.z, x, at_x) ? 1 : 0) + (beats(y[3], at_y.w, x, at_x) ? 1 : 0);
            }
            if (place < k) best_val[place] = x, best_idx[place] = at_x;
        }
    }
    __syncthreads();
}

template <typename T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS, 4) void beam_part_kernel(BeamParams p) {
    constexpr int N = Vec<T>::kN, WAVES = THREADS / 64;
    extern __shared__ __align__(16) char dyn[];
    __shared__ float red_m[WAVES];
    __shared__ double red_s[WAVES];
    __shared__ float best_val[kMaxTop];
    __shared__ int best_idx[kMaxTop];
    const int64_t row = blockIdx.x;
    if (!goes_on(p, row)) return;
    const int part = blockIdx.y, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const T* z = (const T*)p.logits + row / p.in_beams * p.batch_stride + row % p.in_beams * p.beam_stride;
    const int64_t start = (int64_t)part * p.part, end = min(start + p.part, p.vocab);
    u4 v[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] = load_vec<T>(z, start + ((int64_t)j * THREADS + threadIdx.x) * N, end);
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
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float s0 = 0.0f;
#pragma unroll
        for (int e = 0; e < N; ++e) s0 += exp_of(Vec<T>::get(v[j], e) - base);
        s += (double)s0;
    }
    s = wave_sum(s);
    if (lane == 0) red_s[wave] = s;
    keep_packed(v);
    __syncthreads();
    float* list_val = (float*)dyn;
    const int room = list_entries<T, THREADS, NV>(p.beams);       // a multiple of four
    int* list_idx = (int*)(list_val + room);
    best_of_groups<T, NV>(v, lane_max, start, p.beams, room, list_val, list_idx, best_val, best_idx);
    const int64_t slot = row * p.parts + part;
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int w = 0; w < WAVES; ++w) s += red_s[w];
        p.part_m[slot] = m, p.part_s[slot] = s;
    }
    for (int i = threadIdx.x; i < p.beams; i += THREADS) p.part_val[slot * p.beams + i] = best_val[i], p.part_idx[slot * p.beams + i] = best_idx[i];
}

template <int CTRL, int ROWS>
__device__ __forceinline__ double moved_or_own(double v) {
    const unsigned long long b = __double_as_longlong(v);
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp((int)(unsigned)b, (int)(unsigned)b, CTRL, ROWS, 0xf, false);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp((int)(unsigned)(b >> 32), (int)(unsigned)(b >> 32), CTRL, ROWS, 0xf, false);
    return __longlong_as_double((long long)((unsigned long long)hi << 32 | lo));
}
__device__ __forceinline__ double lane_of(double v, int lane) {
    const unsigned long long b = __double_as_longlong(v);
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)b, lane), hi = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)(b >> 32), lane);
    return __longlong_as_double((long long)((unsigned long long)hi << 32 | lo));
}
__device__ __forceinline__ double wave_max(double v) {
    v = fmax(v, moved_or_own<0x111, 0xf>(v));
    v = fmax(v, moved_or_own<0x112, 0xf>(v));
    v = fmax(v, moved_or_own<0x114, 0xf>(v));
    v = fmax(v, moved_or_own<0x118, 0xf>(v));
    v = fmax(v, moved_or_own<0x142, 0xa>(v));
    v = fmax(v, moved_or_own<0x143, 0xc>(v));
    return lane_of(v, 63);
}

// length^a, a in [0, 16], exact where it is a whole number below 2^53: equal quotients are equal numbers then.  A rounded reciprocal or a multiple
// of a logarithm makes two numbers of two thirds of all pairs of equal averages (lengths up to 59, penalty 1).  So whole powers are products,
// and sixteenths go by roots, which are rounded correctly; a finer fraction of a length below 2^32 is no whole number.
__device__ __forceinline__ double power_of(double length, double a) {
    if (16.0 * a != floor(16.0 * a)) return exp(a * log_of(length));
    double v = 1.0, left = a, root = length;
    for (; left >= 1.0; left -= 1.0) v *= length;
    while (left > 0.0) {
        root = sqrt(root), left *= 2.0;
        if (left >= 1.0) v *= root, left -= 1.0;
    }
    return v;
}

// What is known of a hypothesis.
struct Hypothesis {
    double lead, power, sum;   // what comes to a logit's distance from the largest (-inf: it has no candidates), length^|penalty|, sum of e^{z - top}
    float score, top;
    int length, ended, dead;
    int close;                 // two of its logits may have one value in fp64
};

// A workgroup for each request: its wavefronts add up the parts and rank the heads of the parts' lists, then one merges these, each in order.  A
// lane looks after every 64th list; after a turn only the list that was taken from is ranked anew.  LISTS: all lie in LDS.
template <bool LISTS>
__global__ __launch_bounds__(256) void beam_join_kernel(BeamParams p) {
    __shared__ Hypothesis of[kMaxTop];
    extern __shared__ __align__(8) char dyn[];
    const int64_t batch = blockIdx.x;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, k = p.beams, lists = p.in_beams * p.parts, entries = lists * k;
    double* key = LISTS ? (double*)dyn : p.part_key + batch * lists;      // of each list: its head's rank, -inf where there is none
    uint8_t* used = (uint8_t*)(dyn + (LISTS ? 8 * lists : 0));            // and how many are taken
    const float *val = p.part_val + batch * entries, *part_m = p.part_m + batch * lists;
    const double* part_s = p.part_s + batch * lists;
    const int* idx = p.part_idx + batch * entries;
    for (int l = threadIdx.x; l < lists; l += 256) used[l] = 0;
    if constexpr (LISTS) {                                    // all that is read, in one round trip
        double* s = key + lists + (lists + 7) / 8;
        float *m = (float*)(s + lists), *v = m + lists;
        int* at = (int*)(v + entries);
        for (int i = threadIdx.x; i < lists; i += 256) s[i] = part_s[i], m[i] = part_m[i];
        for (int i = threadIdx.x; i < entries; i += 256) v[i] = val[i], at[i] = idx[i];
        part_s = s, part_m = m, val = v, idx = at;
    }
    if ((int)threadIdx.x < p.in_beams) {
        Hypothesis& h = of[threadIdx.x];
        const int64_t row = batch * p.in_beams + threadIdx.x;
        h.score = p.score[row], h.length = p.length ? p.length[row] : 0;
        h.dead = h.score == -INFINITY, h.ended = !h.dead && p.finished && p.finished[row], h.sum = 1.0;
    }
    __syncthreads();
    for (int i = wave; i < p.in_beams; i += 4) {
        if (of[i].dead || of[i].ended) continue;
        float m = -INFINITY;
        for (int j = lane; j < p.parts; j += 64) m = fmaxf(m, part_m[i * p.parts + j]);
        m = ols::wave_max(m);
        const double base = m == -INFINITY ? 0.0 : (double)m;
        double sum = 0.0;
        for (int j = lane; j < p.parts; j += 64) sum += part_s[i * p.parts + j] * exp((double)part_m[i * p.parts + j] - base);
        sum = wave_sum(sum);
        // Logits are 0 or of sizes in [2^-16, 2^8): they differ by 2^-39 at least, and so do their values, by 2^-50 of themselves if the score is below
        // 2^10, which no rounding makes equal.  Otherwise every turn looks at the logits of the heads that share the best rank.
        bool close = !LISTS;
        if constexpr (LISTS)
            for (int e = lane; e < p.parts * k; e += 64) {
                const unsigned size = __float_as_uint(val[i * p.parts * k + e]) & 0x7fffffffu;
                close |= size - 0x37800000u >= 0x0c000000u && size != 0u && size != 0x7f800000u;      // -inf: none
            }
        close = __ballot(close) != 0;
        if (lane == 0) of[i].top = m, of[i].sum = sum, of[i].close = close;
    }
    __syncthreads();
    bool poisoned = false, look = false;
    if (wave == 0) {
        bool bad = false, close = false;
        if (lane < p.in_beams) {
            Hypothesis& h = of[lane];
            bad = !h.dead && (!(h.score < INFINITY) || !(h.sum < INFINITY));
            h.lead = h.dead || !(h.sum > 0.0) ? (double)-INFINITY : (double)h.score - log_of(h.sum);
            h.power = p.penalty == 0.0 ? 1.0 : power_of((double)max(h.ended ? h.length : h.length + 1, 1), fabs(p.penalty));
        }
        if (lane < p.in_beams && !of[lane].dead && !of[lane].ended) close = of[lane].close || !(fabs(of[lane].lead) < 1024.0);
        poisoned = __ballot(bad) != 0, look = p.parts > 1 && __ballot(close) != 0;
        in_wave_order();
    }
    // The hypothesis of list l: quotients are at least 1 / 2048 off a whole number and below 32, where the product is off by 2^-18.  (Divisions of
    // whole numbers were most of a turn.)
    const float per = 1.0f / (float)p.parts;
    auto owner = [&](int l) { return (int)(((float)l + 0.5f) * per); };
    // Entry `at` of list l: whether it is there, its token and value.  Two round trips to LDS.
    struct Candidate {
        int token;                                            // -1: none
        double value, rank;
    };
    auto candidate = [&](int l, int at) {
        const int i = owner(l), entry = l * k + min(at, k - 1);
        const Hypothesis h = of[i];
        const int said = idx[entry];
        const float z = val[entry];
        Candidate c;
        c.value = h.ended ? h.lead : h.lead + ((double)z - (double)h.top);
        c.rank = p.penalty > 0.0 ? c.value / h.power : c.value * h.power;
        c.token = !(h.lead > -INFINITY) ? -1 : h.ended ? (at == 0 && l == i * p.parts ? 0 : -1) : at < k ? said : -1;
        return c;
    };
    auto rank_of = [&](int l, int at) {
        const Candidate c = candidate(l, at);
        return c.token < 0 ? (double)-INFINITY : c.rank;
    };
    const bool single = lists <= 64;                          // a list for each lane
    if (!single) {
        __syncthreads();
        for (int l = threadIdx.x; l < lists; l += 256) key[l] = rank_of(l, 0);
        __syncthreads();
    }
    if (wave) return;
    // The lane's best list, and of place `lane` of the result its list and entry.
    constexpr int kMine = 9;                                  // lists of a lane whose ranks stay in registers: 512 and a few parts for one request
    const bool held = lists <= 64 * kMine;
    const int per_lane = (lists + 63) / 64;
    double mine[kMine];
#pragma unroll
    for (int j = 0; j < kMine; ++j) mine[j] = held && !single && lane + 64 * j < lists ? key[lane + 64 * j] : -INFINITY;
    if (single && lane < lists) mine[0] = rank_of(lane, 0);
    int list = -1, from = -1, entry = 0;
    double best = -INFINITY;
#pragma unroll 1
    for (int turn = 0; turn < k && !poisoned; ++turn) {
        list = -1, best = -INFINITY;
        if (held) {
#pragma unroll
            for (int j = 0; j < kMine; ++j) {
                if (j >= per_lane) break;
                const bool more = mine[j] > best;             // ties: the lower list
                list = more ? lane + 64 * j : list, best = more ? mine[j] : best;
            }
        } else {
            for (int l = lane; l < lists; l += 64) {
                const double v = key[l];
                if (v > best) list = l, best = v;
            }
        }
        const double first = wave_max(best);
        const unsigned long long at = __ballot(list >= 0 && best == first);
        if (!at) break;
        int who = __ffsll(at) - 1, taken = __builtin_amdgcn_readlane(list, who);
        for (unsigned long long more = at & (at - 1); more; more &= more - 1) {
            const int other = __ffsll(more) - 1, l = __builtin_amdgcn_readlane(list, other);
            if (l < taken) taken = l, who = other;
        }
        if (look && !of[owner(taken)].ended) {                // of the hypothesis' heads of this rank: the largest logit, then the lower list
            const int begin = owner(taken) * p.parts;
            float top = -INFINITY;
            int pick = lists;
            for (int l = begin + ((lane - begin) & 63); l < begin + p.parts; l += 64) {
                if (single ? best != first : key[l] != first) continue;             // single: the lane's best is the list's
                const float z = val[l * k + used[l]];
                if (z > top) top = z, pick = l;
            }
            const float largest = ols::wave_max(top);
            unsigned long long same = __ballot(pick < lists && top == largest);
            for (taken = lists; same; same &= same - 1) taken = min(taken, __builtin_amdgcn_readlane(pick, __ffsll(same) - 1));
            who = taken & 63;
        }
        const int place = used[taken];
        if (lane == turn) from = taken, entry = place;
        if (lane == who) {
            const double rank = rank_of(taken, place + 1);
            used[taken] = (uint8_t)(place + 1);
            if (!single) key[taken] = rank;
#pragma unroll
            for (int j = 0; j < kMine; ++j) mine[j] = taken == lane + 64 * j ? rank : mine[j];
        }
        in_wave_order();
    }
    if (lane >= k) return;
    const int64_t out = batch * k + lane;
    if (from < 0) {
        const int slot = lane < p.in_beams ? lane : 0;
        p.new_score[out] = poisoned ? NAN : -INFINITY, p.token[out] = -1, p.parent[out] = slot, p.new_finished[out] = 0;
        if (p.new_length) p.new_length[out] = of[slot].length;
    } else {
        const Hypothesis& h = of[owner(from)];
        const Candidate c = candidate(from, entry);
        p.new_score[out] = (float)c.value, p.token[out] = h.ended ? p.eos : c.token, p.parent[out] = owner(from);
        p.new_finished[out] = h.ended || (p.eos >= 0 && c.token == p.eos);
        if (p.new_length) p.new_length[out] = h.length + (h.ended ? 0 : 1);
    }
}

template <typename T, int THREADS, int NV>
hipError_t launch_rows(const BeamParams& p, hipStream_t stream) {
    const size_t lds = (size_t)list_entries<T, THREADS, NV>(p.beams) * 8;
    beam_part_kernel<T, THREADS, NV><<<dim3((unsigned)(p.batch * p.in_beams), p.parts), THREADS, lds, stream>>>(p);
    return hipGetLastError();
}
template <typename T>
hipError_t launch_typed(const BeamParams& p, const RowPlan& r, hipStream_t stream) {
    if (r.nv == 2) return launch_rows<T, 256, 2>(p, stream);
    if (r.nv == 4) return launch_rows<T, 256, 4>(p, stream);
    if (r.nv == 8) return launch_rows<T, 256, 8>(p, stream);
    return r.nv == 10 ? launch_rows<T, 256, 10>(p, stream) : r.nv == 13 ? launch_rows<T, 256, 13>(p, stream) : launch_rows<T, 256, 16>(p, stream);
}

// ---- states ---------------------------------------------------------------------------------------------------------------

// BYTES at any address, of up to S hypotheses at once.  Places that are not written read the first row again.
template <int BYTES>
struct Piece;
template <>
struct Piece<16> {
    typedef unsigned int type __attribute__((ext_vector_type(4), aligned(1)));
};
template <>
struct Piece<8> {
    typedef unsigned int type __attribute__((ext_vector_type(2), aligned(1)));
};
template <>
struct Piece<4> {
    typedef unsigned int type __attribute__((aligned(1)));
};
template <>
struct Piece<2> {
    typedef unsigned short type __attribute__((aligned(1)));
};
template <>
struct Piece<1> {
    typedef unsigned char type;
};
template <int BYTES, int S>
struct Pieces {
    typename Piece<BYTES>::type v[S];
    __device__ void read(const char* src, int64_t row, const int (&from)[S]) {
#pragma unroll
        for (int i = 0; i < S; ++i) v[i] = *(const typename Piece<BYTES>::type*)(src + max(from[i], 0) * row);
    }
    __device__ void write(char* dst, int64_t row, const int (&from)[S]) const {
#pragma unroll
        for (int i = 0; i < S; ++i)
            if (from[i] >= 0) *(typename Piece<BYTES>::type*)(dst + i * row) = v[i];
    }
};

// A thread for each sixteen bytes of a request's rows; what is left of a row goes in pieces of eight, four, two and one, all read first.
template <int S>
__global__ __launch_bounds__(256) void beam_move_kernel(BeamMove t) {
    int k = 0;
    while (k + 1 < t.n && (int)blockIdx.x >= t.first_block[k + 1]) ++k;
    const int64_t batch = blockIdx.y, at = ((int64_t)(blockIdx.x - t.first_block[k]) * 256 + threadIdx.x) * 16, left = t.row_bytes[k] - at;
    const int32_t* parent = t.parent + batch * t.out_beams;
    const bool in_place = t.src[k] == t.dst[k];
    int from[S];
#pragma unroll
    for (int i = 0; i < S; ++i) {
        from[i] = i < t.out_beams ? parent[i] : -1;
        if (from[i] >= t.in_beams || (in_place && from[i] == i)) from[i] = -1;
    }
    if (left <= 0) return;
    const char* src = (const char*)t.src[k] + batch * t.src_batch[k] + at;
    char* dst = (char*)t.dst[k] + batch * t.dst_batch[k] + at;
    const int64_t src_row = t.src_beam[k], dst_row = t.dst_beam[k];
    if (left >= 16) {
        Pieces<16, S> p;
        p.read(src, src_row, from);
        p.write(dst, dst_row, from);
        return;
    }
    const int four = left & 8, two = four + (left & 4), one = two + (left & 2);      // where they begin
    Pieces<8, S> p8;
    Pieces<4, S> p4;
    Pieces<2, S> p2;
    Pieces<1, S> p1;
    if (left & 8) p8.read(src, src_row, from);
    if (left & 4) p4.read(src + four, src_row, from);
    if (left & 2) p2.read(src + two, src_row, from);
    if (left & 1) p1.read(src + one, src_row, from);
    if (left & 8) p8.write(dst, dst_row, from);
    if (left & 4) p4.write(dst + four, dst_row, from);
    if (left & 2) p2.write(dst + two, dst_row, from);
    if (left & 1) p1.write(dst + one, dst_row, from);
}

}  // namespace

constexpr int64_t kLds = 152 << 10;       // of a compute unit's 160 KiB, beside what the join declares

// Workgroups of four wavefronts: several run on a compute unit, and one's search for its best overlaps with another's loads.  512 rows of
// 128 000 bf16 in workgroups that hold whole rows: 49 us.
static RowPlan beam_plan(int dtype, int64_t rows, int64_t vocab) { return row_plan(dtype, rows, vocab, 256); }

// All parts of a call lie in the workspace; negative: they are more than a launch numbers (fewer than 2^32 threads, 256 for each).
int64_t beam_workspace_bytes(int dtype, int64_t batch, int in_beams, int beams, int64_t vocab) {
    if (batch == 0) return 0;
    const int64_t rows = batch * in_beams, parts = rows * beam_plan(dtype, rows, vocab).parts;
    return parts >= (1 << 24) ? -1 : parts * (20 + 8 * (int64_t)beams);
}

hipError_t launch_beam(BeamParams p, void* ws, hipStream_t stream) {
    if (p.batch == 0) return hipSuccess;
    const int64_t rows = p.batch * p.in_beams;
    const RowPlan r = beam_plan(p.dtype, rows, p.vocab);
    p.parts = r.parts, p.part = r.part;
    p.part_s = (double*)ws;
    p.part_key = p.part_s + rows * r.parts;
    p.part_m = (float*)(p.part_key + rows * r.parts);
    p.part_val = p.part_m + rows * r.parts;
    p.part_idx = (int32_t*)(p.part_val + rows * r.parts * p.beams);
    hipError_t e = p.dtype == OLS_F32 ? launch_typed<float>(p, r, stream) : launch_typed<uint16_t>(p, r, stream);
    if (e != hipSuccess) return e;
    const int64_t lists = (int64_t)p.in_beams * r.parts, counts = (lists + 7) / 8 * 8, whole = counts + lists * (20 + 8 * (int64_t)p.beams);
    if (whole > kLds) {
        beam_join_kernel<false><<<(unsigned)p.batch, 256, (size_t)counts, stream>>>(p);        // at most 32 KiB
        return hipGetLastError();
    }
    if (whole > (60 << 10)) e = ensure_dynamic_lds((const void*)beam_join_kernel<true>, kLds);
    if (e != hipSuccess) return e;
    beam_join_kernel<true><<<(unsigned)p.batch, 256, (size_t)whole, stream>>>(p);
    return hipGetLastError();
}

hipError_t launch_beam_move(const BeamMove& t, unsigned blocks, int64_t batch, hipStream_t stream) {
    const dim3 grid(blocks, (unsigned)batch);
    if (t.out_beams <= 4) beam_move_kernel<4><<<grid, 256, 0, stream>>>(t);
    else if (t.out_beams <= 8) beam_move_kernel<8><<<grid, 256, 0, stream>>>(t);
    else if (t.out_beams <= 16) beam_move_kernel<16><<<grid, 256, 0, stream>>>(t);
    else beam_move_kernel<32><<<grid, 256, 0, stream>>>(t);
    return hipGetLastError();
}

}  // namespace ols
