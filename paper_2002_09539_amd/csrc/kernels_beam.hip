// One step of beam search over several requests: which hypotheses go on and with which token, and moving their states.
//
//   logp_iv = (z_iv - m_i) - log sum_v e^{z_iv - m_i}
//   candidates:  (i, v) of value score_i + logp_iv and length length_i + 1;  of an ended hypothesis only itself, (i, 0) of value score_i
//   order:       by value / length^penalty, largest first; ties to the lower hypothesis, then to the lower token
//
// Within a hypothesis that is the order of its logits, which is exact.  Between hypotheses it hangs on the last bits of the sums:
// these are added up in fp64 from exponentials whose argument's rounding does not lean to a side, and candidates are compared in fp64.
//
// What bounds the choice is one read of the logits: a workgroup holds its part of a hypothesis' row in registers, takes the sum
// and the part's best from there (logit_rows.h), and one wavefront for each request merges the parts' lists, each in order: a lane
// holds the heads of its lists, and every turn takes the best head of all.  Ended hypotheses are not read.
//
// Moving states is one read and one write of what moves.  A thread holds the same sixteen bytes of all hypotheses of a request: all
// are read before one is written, so that states can be moved in place, and a hypothesis that stays where it is is not touched then.
#include "logit_rows.h"

namespace ols {

namespace {

// e^d as a power of two; log2 e = hi + lo, both positive, so that -inf stays -inf
__device__ __forceinline__ float exp_of(float d) {
    constexpr float kHi = 1.44269502162933349609f, kLo = 1.92596299112661747e-8f;
    return __builtin_amdgcn_exp2f(fmaf(d, kHi, d * kLo));
}

// A hypothesis that is read: it has a score and has not ended.
__device__ __forceinline__ bool goes_on(const BeamParams& p, int64_t row) {
    return !(p.score[row] == -INFINITY) && !(p.finished && p.finished[row]);
}

template <typename T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS, 4) void beam_part_kernel(BeamParams p) {
    constexpr int N = Vec<T>::kN, WAVES = THREADS / 64;
    extern __shared__ char dyn[];
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
    int* list_idx = (int*)(list_val + list_entries<T, THREADS, NV>(p.beams));
    best_of_part<T, THREADS, NV>(v, lane_max, start, p.beams, list_val, list_idx, best_val, best_idx);
    const int64_t slot = row * p.parts + part;
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int w = 0; w < WAVES; ++w) s += red_s[w];
        p.part_m[slot] = m, p.part_s[slot] = s;
    }
    for (int i = threadIdx.x; i < p.beams; i += THREADS) p.part_val[slot * p.beams + i] = best_val[i], p.part_idx[slot * p.beams + i] = best_idx[i];
}

// Largest first; a lane's candidate is one of its lists' heads.
struct Head {
    double key;
    int list;               // -1: none
};
__device__ __forceinline__ bool before(const Head& a, const Head& b) { return a.list >= 0 && (b.list < 0 || a.key > b.key || (a.key == b.key && a.list < b.list)); }

// One wavefront for each request.
__global__ __launch_bounds__(64) void beam_join_kernel(BeamParams p) {
    // Of a hypothesis: what comes to a logit's distance from the largest (-inf: it has no candidates), that one, and length^penalty.
    __shared__ double lead[kMaxTop], sums[kMaxTop], scale[kMaxTop];
    __shared__ float tops[kMaxTop];
    extern __shared__ uint16_t used[];                        // of each list: how many are taken
    const int64_t batch = blockIdx.x;
    const int lane = threadIdx.x, lists = p.in_beams * p.parts, k = p.beams;
    for (int i = 0; i < p.in_beams && p.parts > 1; ++i) {
        const int64_t row = batch * p.in_beams + i;
        if (!goes_on(p, row)) continue;
        float m = -INFINITY;
        for (int j = lane; j < p.parts; j += 64) m = fmaxf(m, p.part_m[row * p.parts + j]);
        m = wave_max(m);
        const double base = m == -INFINITY ? 0.0 : (double)m;
        double sum = 0.0;
        for (int j = lane; j < p.parts; j += 64) sum += p.part_s[row * p.parts + j] * exp((double)p.part_m[row * p.parts + j] - base);
        sum = wave_sum(sum);
        if (lane == 0) tops[i] = m, sums[i] = sum;
    }
    in_wave_order();
    bool bad = false;
    if (lane < p.in_beams) {
        const int64_t row = batch * p.in_beams + lane;
        const float score = p.score[row];
        const bool dead = score == -INFINITY, ended = !dead && !goes_on(p, row);
        if (p.parts == 1 && !dead && !ended) tops[lane] = p.part_m[row], sums[lane] = p.part_s[row];
        const double sum = dead || ended ? 1.0 : sums[lane];
        bad = !dead && (!(score < INFINITY) || !(sum < INFINITY));
        lead[lane] = dead || !(sum > 0.0) ? (double)-INFINITY : (double)score - log(sum);
        const int before = p.length ? p.length[row] : 0, after = ended ? before : before + 1;
        scale[lane] = p.penalty == 0.0 ? 1.0 : pow((double)max(after, 1), p.penalty);
    }
    const bool poisoned = __ballot(bad) != 0;
    for (int l = lane; l < lists; l += 64) used[l] = 0;
    in_wave_order();
    // value and key of the head of list l
    auto value_of = [&](int l, int& token) {
        const int i = l / p.parts, at = used[l];
        const int64_t row = batch * p.in_beams + i, slot = batch * lists + l;
        token = -1;
        if (lead[i] == -INFINITY || at >= k) return (double)-INFINITY;
        if (p.finished && p.finished[row]) {
            if (at > 0 || l % p.parts) return (double)-INFINITY;
            token = 0;
            return lead[i];
        }
        token = p.part_idx[slot * k + at];
        return token < 0 ? (double)-INFINITY : lead[i] + ((double)p.part_val[slot * k + at] - (double)tops[i]);
    };
    auto head_of = [&](int l) {
        int token;
        const double v = value_of(l, token);
        return token < 0 ? Head{0.0, -1} : Head{v / scale[l / p.parts], l};
    };
    auto best_of = [&]() {
        Head h{0.0, -1};
        for (int l = lane; l < lists; l += 64) {
            const Head g = head_of(l);
            if (before(g, h)) h = g;
        }
        return h;
    };
    Head mine = best_of();
    for (int turn = 0; turn < k; ++turn) {
        Head h = mine;
        for (int o = 32; o; o >>= 1) {
            const Head g{__shfl_xor(h.key, o), __shfl_xor(h.list, o)};
            if (before(g, h)) h = g;
        }
        const int64_t out = batch * k + turn;
        if (poisoned || h.list < 0) {
            if (lane == 0) {
                const int slot = turn < p.in_beams ? turn : 0;
                p.new_score[out] = poisoned ? NAN : -INFINITY, p.token[out] = -1, p.parent[out] = slot, p.new_finished[out] = 0;
                if (p.new_length) p.new_length[out] = p.length[batch * p.in_beams + slot];
            }
            continue;
        }
        if (h.list % 64 == lane) {
            int token;
            const double v = value_of(h.list, token);
            const int i = h.list / p.parts;
            const int64_t row = batch * p.in_beams + i;
            const bool ended = p.finished && p.finished[row];
            p.new_score[out] = (float)v, p.token[out] = ended ? p.eos : token, p.parent[out] = i;
            p.new_finished[out] = ended || (p.eos >= 0 && token == p.eos);
            if (p.new_length) p.new_length[out] = p.length[row] + (ended ? 0 : 1);
            used[h.list] += 1;
            mine = best_of();
        }
    }
}

template <typename T, int THREADS, int NV>
hipError_t launch_rows(const BeamParams& p, hipStream_t stream) {
    const size_t lds = (size_t)list_entries<T, THREADS, NV>(p.beams) * 8;
    beam_part_kernel<T, THREADS, NV><<<dim3((unsigned)(p.batch * p.in_beams), p.parts), THREADS, lds, stream>>>(p);
    return hipGetLastError();
}
template <typename T, int NV>
hipError_t launch_long(const BeamParams& p, const RowPlan& r, hipStream_t stream) {
    if (r.threads == 256) return launch_rows<T, 256, NV>(p, stream);
    return r.threads == 512 ? launch_rows<T, 512, NV>(p, stream) : launch_rows<T, 1024, NV>(p, stream);
}
template <typename T>
hipError_t launch_typed(const BeamParams& p, const RowPlan& r, hipStream_t stream) {
    if (r.threads == 256) {
        if (r.nv == 2) return launch_rows<T, 256, 2>(p, stream);
        if (r.nv == 4) return launch_rows<T, 256, 4>(p, stream);
        if (r.nv == 8) return launch_rows<T, 256, 8>(p, stream);
    }
    return r.nv <= 10 ? launch_long<T, 10>(p, r, stream) : r.nv == 13 ? launch_long<T, 13>(p, r, stream) : launch_long<T, 16>(p, r, stream);
}

// ---- states ---------------------------------------------------------------------------------------------------------------

typedef unsigned int u4bytes __attribute__((ext_vector_type(4), aligned(1)));   // sixteen bytes at any address

// The pieces of up to S hypotheses at once in registers; the last piece of a row may be shorter.
template <int S>
__global__ __launch_bounds__(256) void beam_move_kernel(BeamMove t) {
    int k = 0;
    while (k + 1 < t.n && (int)blockIdx.x >= t.first_block[k + 1]) ++k;
    const int64_t batch = blockIdx.y, at = ((int64_t)(blockIdx.x - t.first_block[k]) * 256 + threadIdx.x) * 16, left = t.row_bytes[k] - at;
    if (left <= 0) return;
    const int32_t* parent = t.parent + batch * t.out_beams;
    const char* src = (const char*)t.src[k] + batch * t.src_batch[k] + at;
    char* dst = (char*)t.dst[k] + batch * t.dst_batch[k] + at;
    const bool in_place = t.src[k] == t.dst[k];
    int from[S];
#pragma unroll
    for (int i = 0; i < S; ++i) {
        from[i] = i < t.out_beams ? parent[i] : -1;
        if (from[i] >= t.in_beams || (in_place && from[i] == i)) from[i] = -1;
    }
    if (left >= 16) {
        u4 piece[S];
#pragma unroll
        for (int i = 0; i < S; ++i)
            if (from[i] >= 0) piece[i] = *(const u4bytes*)(src + from[i] * t.src_beam[k]);
#pragma unroll
        for (int i = 0; i < S; ++i)
            if (from[i] >= 0) *(u4bytes*)(dst + i * t.dst_beam[k]) = piece[i];
    } else {
        for (int b = 0; b < left; ++b) {
            char piece[S];
#pragma unroll
            for (int i = 0; i < S; ++i)
                if (from[i] >= 0) piece[i] = src[from[i] * t.src_beam[k] + b];
#pragma unroll
            for (int i = 0; i < S; ++i)
                if (from[i] >= 0) dst[i * t.dst_beam[k] + b] = piece[i];
        }
    }
}

}  // namespace

// All parts of a call lie in the workspace.
int64_t beam_workspace_bytes(int dtype, int64_t batch, int in_beams, int beams, int64_t vocab) {
    if (batch == 0) return 0;
    const int64_t rows = batch * in_beams;
    return rows * row_plan(dtype, rows, vocab).parts * (12 + 8 * (int64_t)beams);
}

hipError_t launch_beam(BeamParams p, void* ws, hipStream_t stream) {
    if (p.batch == 0) return hipSuccess;
    const int64_t rows = p.batch * p.in_beams;
    const RowPlan r = row_plan(p.dtype, rows, p.vocab);
    p.parts = r.parts, p.part = r.part;
    p.part_s = (double*)ws;
    p.part_m = (float*)(p.part_s + rows * r.parts);
    p.part_val = p.part_m + rows * r.parts;
    p.part_idx = (int32_t*)(p.part_val + rows * r.parts * p.beams);
    hipError_t e = p.dtype == OLS_F32 ? launch_typed<float>(p, r, stream) : launch_typed<uint16_t>(p, r, stream);
    if (e != hipSuccess) return e;
    beam_join_kernel<<<(unsigned)p.batch, 64, (size_t)p.in_beams * r.parts * 2, stream>>>(p);
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
