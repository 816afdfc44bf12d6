// Embedding lookup with scaling, and its gradient by sorted tokens, per worker.
//
//   out[n] = scale E[t_n]                         ids outside [0, vocab) are no token: their row of `out` is zero
//   dE[v]  = scale sum_{n : t_n = v} dout[n]       in ascending n, added in fp32, rounded once
//
// Both move bytes and compute nothing to speak of.  The lookup reads one row and writes one per id; a row is spread over
// as many lanes as it has vectors of eight, so that short rows share a workgroup.
//
// The gradient could add rows into the table with atomics, whose order (and so whose rounding) changes from run to run,
// and whose rate collapses on the few ids that make up much of a text.  Here the ids are sorted, stably, so that the rows
// of one id are neighbours in a list and every sum has one order:
//   1. radix sort of (id, position), 9 bits a pass: per-workgroup digit counts, then a stable scatter in which every
//      wavefront ranks 64 ids at a time by matching ballots.  Up to kSortItems ids per worker take one workgroup and
//      one launch for all passes.
//   2. the sorted list is cut into runs of kRun positions; a run that lies inside ONE id is added up by a wavefront of its
//      own into a partial row (an id that makes up 6 % of 32 768 tokens is a sum of 2 000 rows, which one wavefront alone
//      would take 100 us to follow).
//   3. a wavefront per table row finds its segment by bisection and writes scale * (rows before the first whole run, the
//      whole runs' partials, rows after the last), or zeros.  Every row of the table is written once, so no fill precedes.
#include "element_io.h"
#include "ols_internal.h"

namespace ols {

namespace {

constexpr int kThreads = 256;
constexpr int kSortThreads = 1024;          // sixteen wavefronts share a workgroup's ids
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kSortItems = 4096;            // ids of one workgroup of the sort
constexpr int kDigitBits = 9;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kRun = 64;                    // sorted positions of a partial row
constexpr int kRowsPerBlock = 16;           // table rows of a workgroup of the last stage: four per wavefront

template <typename TI, typename TO>
__global__ __launch_bounds__(kThreads) void embed_kernel(EmbedParams p, int lanes) {
    const int64_t n = (int64_t)blockIdx.x * (kThreads / lanes) + threadIdx.x / lanes;
    if (n >= p.tokens) return;
    const int64_t group = blockIdx.y;
    const int id = p.ids[group * p.ids_group + n];
    const bool real = id >= 0 && id < p.vocab;
    const TI* src = (const TI*)p.table + group * p.table_group + (real ? id * p.table_row : 0);
    TO* dst = (TO*)p.out + group * p.out_group + n * p.out_row;
    for (int64_t c = (threadIdx.x % lanes) * 8; c < p.width; c += (int64_t)lanes * 8) {
        const int left = (int)min((int64_t)8, p.width - c);
        float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (real) {
            load_upto8(src + c, left, 0.0f, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= p.scale;
        }
        store_upto8(dst + c, left, v);
    }
}

// ---- sorting ------------------------------------------------------------------------------------------------------------

struct SortParams {
    const int32_t* ids;          // first pass: the caller's ids; later ones: keys_in
    int64_t ids_group;
    const int32_t* keys_in;
    const int32_t* pos_in;
    int32_t* keys_out;
    int32_t* pos_out;
    int32_t* counts;             // [group][block][kDigits]
    int64_t n;                   // ids per group
    int blocks, shift;
    int64_t vocab;
};

__device__ __forceinline__ int key_at(const SortParams& p, int group, int64_t i, bool first) {
    if (!first) return p.keys_in[(int64_t)group * p.n + i];
    const int id = p.ids[(int64_t)group * p.ids_group + i];
    return id >= 0 && id < p.vocab ? id : (int)p.vocab;   // what is no token sorts behind every token
}

// the lanes of the wavefront that hold the same digit; lanes that hold no item match nothing
__device__ __forceinline__ unsigned long long same_digit(int digit, bool valid) {
    unsigned long long m = __ballot(valid);
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
        const bool bit = (digit >> b) & 1;
        const unsigned long long set = __ballot(bit);
        m &= bit ? set : ~set;
    }
    return m;
}

// One stable pass over the items of one workgroup: item i goes behind every item of a smaller digit and every earlier
// item of its own.  `before[d]`: how many items of all workgroups precede this workgroup's first one of digit d.
__device__ void scatter_block(const SortParams& p, int group, int block, bool first, int (*cnt)[kDigits], const int* before) {
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    constexpr int kPerWave = kSortItems / kSortWaves;
    const int64_t base = (int64_t)block * kSortItems + wave * kPerWave;
    for (int i = threadIdx.x; i < kSortWaves * kDigits; i += kSortThreads) (&cnt[0][0])[i] = 0;
    __syncthreads();
    for (int k = 0; k < kPerWave; k += 64) {
        const int64_t i = base + k + lane;
        const bool valid = i < p.n;
        const int digit = valid ? (key_at(p, group, i, first) >> p.shift) & (kDigits - 1) : 0;
        const unsigned long long same = same_digit(digit, valid);
        if (valid && (same & ((1ull << lane) - 1)) == 0) cnt[wave][digit] += __popcll(same);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) {
        int at = before[d];
        for (int w = 0; w < kSortWaves; ++w) {
            const int c = cnt[w][d];
            cnt[w][d] = at;
            at += c;
        }
    }
    __syncthreads();
    for (int k = 0; k < kPerWave; k += 64) {
        const int64_t i = base + k + lane;
        const bool valid = i < p.n;
        const int key = valid ? key_at(p, group, i, first) : 0;
        const int digit = (key >> p.shift) & (kDigits - 1);
        const unsigned long long same = same_digit(digit, valid);
        const int rank = __popcll(same & ((1ull << lane) - 1));
        if (valid) {
            const int64_t at = (int64_t)group * p.n + cnt[wave][digit] + rank;
            p.keys_out[at] = key;
            p.pos_out[at] = first ? (int)i : p.pos_in[(int64_t)group * p.n + i];
        }
        // every lane has read the counter before the first of its digit moves it on (one wavefront, in step)
        __builtin_amdgcn_wave_barrier();
        if (valid && rank == 0) cnt[wave][digit] += __popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
}

// exclusive sum over digits of `total` (in LDS), by the first 512 lanes; the result replaces it
__device__ void scan_digits(int* total) {
    __shared__ int wave_sum[kDigits / 64];
    const int d = threadIdx.x, lane = threadIdx.x % 64;
    int own = 0, sum = 0;
    if (d < kDigits) {
        own = sum = total[d];
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(sum, o);
            if (lane >= o) sum += v;
        }
        if (lane == 63) wave_sum[d / 64] = sum;
    }
    __syncthreads();
    if (d < kDigits) {
        int add = 0;
        for (int w = 0; w < d / 64; ++w) add += wave_sum[w];
        total[d] = add + sum - own;
    }
    __syncthreads();
}

__device__ void count_block(const SortParams& p, int group, int block, bool first, int* hist) {
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) hist[d] = 0;
    __syncthreads();
    for (int k = threadIdx.x; k < kSortItems; k += kSortThreads) {
        const int64_t i = (int64_t)block * kSortItems + k;
        if (i < p.n) atomicAdd(&hist[(key_at(p, group, i, first) >> p.shift) & (kDigits - 1)], 1);
    }
    __syncthreads();
}

// all passes of a worker whose ids one workgroup holds; ping-pong between the two list pairs
__global__ __launch_bounds__(kSortThreads) void sort_one_block_kernel(SortParams p, int32_t* keys_a, int32_t* pos_a, int32_t* keys_b,
                                                                      int32_t* pos_b, int passes) {
    __shared__ int cnt[kSortWaves][kDigits];
    __shared__ int before[kDigits];
    for (int pass = 0; pass < passes; ++pass) {
        const bool to_a = (passes - 1 - pass) % 2 == 0;   // the last pass ends in a
        p.keys_out = to_a ? keys_a : keys_b;
        p.pos_out = to_a ? pos_a : pos_b;
        p.keys_in = to_a ? keys_b : keys_a;
        p.pos_in = to_a ? pos_b : pos_a;
        p.shift = pass * kDigitBits;
        count_block(p, blockIdx.x, 0, pass == 0, before);
        scan_digits(before);
        scatter_block(p, blockIdx.x, 0, pass == 0, cnt, before);
        __threadfence_block();
        __syncthreads();
    }
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortParams p, int first) {
    __shared__ int hist[kDigits];
    count_block(p, blockIdx.y, blockIdx.x, first, hist);
    int32_t* out = p.counts + ((int64_t)blockIdx.y * p.blocks + blockIdx.x) * kDigits;
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) out[d] = hist[d];
}

// Every workgroup adds up the counts of all of them itself (blocks x 2 KiB from the L2) instead of waiting for a scan in a
// launch of its own.
__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(SortParams p, int first) {
    __shared__ int cnt[kSortWaves][kDigits];
    __shared__ int before[kDigits], total[kDigits];
    static_assert(kSortThreads == 2 * kDigits, "two lanes add up a digit's counts");
    const int32_t* counts = p.counts + (int64_t)blockIdx.y * p.blocks * kDigits;
    const int d = threadIdx.x % kDigits, half = threadIdx.x / kDigits, me = blockIdx.x;
    if (half == 0) before[d] = 0, total[d] = 0;
    __syncthreads();
    int less = 0, all = 0;
    for (int b = half; b < p.blocks; b += 2) {
        const int c = counts[(int64_t)b * kDigits + d];
        all += c;
        less += b < me ? c : 0;
    }
    atomicAdd(&before[d], less);
    atomicAdd(&total[d], all);
    __syncthreads();
    scan_digits(total);
    if (half == 0) before[d] += total[d];
    __syncthreads();
    scatter_block(p, blockIdx.y, blockIdx.x, first, cnt, before);
}

// ---- sums over sorted positions -----------------------------------------------------------------------------------------

struct RowsParams {
    EmbedGradParams g;
    const int32_t* keys;
    const int32_t* pos;
    float* partial;      // [group][runs][width]
    int64_t runs;
};

// Adds rows pos[from .. to) of dout, columns c + 512 t + 8 lane .., in that order.  The positions are loaded 64 at a time
// and handed round; four rows' loads are in flight together.
template <typename TI, int NV>
__device__ __forceinline__ void add_rows(const RowsParams& q, int64_t group, int64_t from, int64_t to, int64_t c, int lane, float (&sum)[NV][8]) {
    const int32_t* pos = q.pos + group * q.g.tokens;
    const TI* base = (const TI*)q.g.dout + group * q.g.dout_group;
    for (int64_t i0 = from; i0 < to; i0 += 64) {
        const int have = (int)min((int64_t)64, to - i0);
        const int mine = lane < have ? pos[i0 + lane] : 0;
        for (int k = 0; k < have; k += 4) {
            float v[4][NV][8];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t row = __shfl(mine, min(k + r, have - 1));
#pragma unroll
                for (int t = 0; t < NV; ++t) {
                    const int64_t at = c + 512 * t + 8 * lane;
                    load_upto8(base + row * q.g.dout_row + at, k + r < have ? (int)max((int64_t)0, min((int64_t)8, q.g.width - at)) : 0, 0.0f, v[r][t]);
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (k + r < have) {
#pragma unroll
                    for (int t = 0; t < NV; ++t)
#pragma unroll
                        for (int e = 0; e < 8; ++e) sum[t][e] += v[r][t][e];
                }
        }
    }
}

template <typename TI, int NV>
__global__ __launch_bounds__(kThreads) void embed_runs_kernel(RowsParams q) {
    const int lane = threadIdx.x % 64;
    const int64_t run = (int64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64, group = blockIdx.y;
    const int64_t from = run * kRun, to = from + kRun;
    if (run >= q.runs || to > q.g.tokens) return;
    const int32_t* keys = q.keys + group * q.g.tokens;
    const int id = keys[from];
    if (id != keys[to - 1] || id >= q.g.vocab) return;
    const int64_t c = (int64_t)blockIdx.z * 512 * NV;
    float sum[NV][8] = {};
    add_rows<TI, NV>(q, group, from, to, c, lane, sum);
    float* out = q.partial + (group * q.runs + run) * q.g.width;
#pragma unroll
    for (int t = 0; t < NV; ++t) {
        const int64_t at = c + 512 * t + 8 * lane;
        if (at < q.g.width) store_upto8(out + at, (int)min((int64_t)8, q.g.width - at), sum[t]);
    }
}

template <typename TI, typename TO, int NV>
__global__ __launch_bounds__(kThreads) void embed_rows_kernel(RowsParams q) {
    __shared__ int64_t start[kRowsPerBlock + 1];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t v0 = (int64_t)blockIdx.x * kRowsPerBlock, group = blockIdx.y;
    const int32_t* keys = q.keys + group * q.g.tokens;
    if (threadIdx.x <= kRowsPerBlock) {   // the first position whose id is at least v0 + threadIdx.x
        const int64_t v = v0 + threadIdx.x;
        int64_t lo = 0, hi = q.g.tokens;
        while (lo < hi) {
            const int64_t mid = (lo + hi) / 2;
            if (keys[mid] < v) lo = mid + 1;
            else hi = mid;
        }
        start[threadIdx.x] = lo;
    }
    __syncthreads();
    const int64_t c = (int64_t)blockIdx.z * 512 * NV;
    for (int r = wave; r < kRowsPerBlock; r += kThreads / 64) {
        const int64_t v = v0 + r;
        if (v >= q.g.vocab) break;
        const int64_t from = start[r], to = start[r + 1];
        if (from == to && q.g.accumulate) continue;
        float sum[NV][8] = {};
        if (from < to) {
            const int64_t first = (from + kRun - 1) / kRun, last = to / kRun;   // whole runs [first, last)
            if (first >= last) {
                add_rows<TI, NV>(q, group, from, to, c, lane, sum);
            } else {
                add_rows<TI, NV>(q, group, from, first * kRun, c, lane, sum);
                const float* part = q.partial + (group * q.runs + first) * q.g.width;
                for (int64_t k = 0; k < last - first; k += 4) {
                    float p[4][NV][8];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int t = 0; t < NV; ++t) {
                            const int64_t at = c + 512 * t + 8 * lane;
                            const bool there = k + j < last - first && at < q.g.width;
                            load_upto8(part + (k + j) * q.g.width + at, there ? (int)min((int64_t)8, q.g.width - at) : 0, 0.0f, p[j][t]);
                        }
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int t = 0; t < NV; ++t)
#pragma unroll
                            for (int e = 0; e < 8; ++e) sum[t][e] += p[j][t][e];
                }
                add_rows<TI, NV>(q, group, last * kRun, to, c, lane, sum);
            }
        }
        TO* out = (TO*)q.g.grad + group * q.g.grad_group + v * q.g.grad_row;
#pragma unroll
        for (int t = 0; t < NV; ++t) {
            const int64_t at = c + 512 * t + 8 * lane;
            if (at >= q.g.width) continue;
            const int left = (int)min((int64_t)8, q.g.width - at);
            float o[8];
            if (q.g.accumulate) {
                load_upto8(out + at, left, 0.0f, o);
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = fmaf(q.g.scale, sum[t][e], o[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = q.g.scale * sum[t][e];
            }
            store_upto8(out + at, left, o);
        }
    }
}

int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }

struct GradPlan {
    int64_t blocks, runs, off_keys[2], off_pos[2], off_counts, off_partial, bytes;
};
GradPlan grad_plan(int groups, int64_t tokens, int64_t width) {
    GradPlan p;
    p.blocks = (tokens + kSortItems - 1) / kSortItems;
    p.runs = tokens / kRun;
    int64_t at = 0;
    for (int i = 0; i < 2; ++i) {
        p.off_keys[i] = at, at = up256(at + groups * tokens * 4);
        p.off_pos[i] = at, at = up256(at + groups * tokens * 4);
    }
    p.off_counts = at, at = up256(at + (p.blocks > 1 ? groups * p.blocks * kDigits * 4 : 0));
    p.off_partial = at, at = up256(at + groups * p.runs * width * 4);
    p.bytes = at;
    return p;
}

template <typename TI, typename TO, int NV>
void launch_sums(const RowsParams& q, hipStream_t stream) {
    const int tiles = (int)((q.g.width + 512 * NV - 1) / (512 * NV));
    if (q.runs)
        embed_runs_kernel<TI, NV><<<dim3((unsigned)((q.runs + 3) / 4), q.g.groups, tiles), kThreads, 0, stream>>>(q);
    embed_rows_kernel<TI, TO, NV><<<dim3((unsigned)((q.g.vocab + kRowsPerBlock - 1) / kRowsPerBlock), q.g.groups, tiles), kThreads, 0, stream>>>(q);
}

template <typename TI, typename TO>
void launch_sums(const RowsParams& q, hipStream_t stream) {
    if (q.g.width <= 512) launch_sums<TI, TO, 1>(q, stream);
    else launch_sums<TI, TO, 2>(q, stream);
}

}  // namespace

hipError_t launch_embed(const EmbedParams& p, hipStream_t stream) {
    int lanes = 1;
    while (lanes < kThreads && (int64_t)lanes * 8 < p.width) lanes *= 2;
    const int64_t blocks = (p.tokens + kThreads / lanes - 1) / (kThreads / lanes);
    if (blocks == 0 || p.groups == 0 || p.width == 0) return hipSuccess;
    if (blocks > 0x7fffffff) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks, p.groups);
    if (p.dtype == OLS_F32 && p.out_dtype == OLS_F32) embed_kernel<float, float><<<grid, kThreads, 0, stream>>>(p, lanes);
    else if (p.dtype == OLS_F32) embed_kernel<float, uint16_t><<<grid, kThreads, 0, stream>>>(p, lanes);
    else if (p.out_dtype == OLS_F32) embed_kernel<uint16_t, float><<<grid, kThreads, 0, stream>>>(p, lanes);
    else embed_kernel<uint16_t, uint16_t><<<grid, kThreads, 0, stream>>>(p, lanes);
    return hipGetLastError();
}

int64_t embed_grad_workspace_bytes(int groups, int64_t tokens, int64_t width) { return grad_plan(groups, tokens, width).bytes; }

hipError_t launch_embed_grad(const EmbedGradParams& g, void* ws, hipStream_t stream) {
    if (g.groups == 0 || g.width == 0) return hipSuccess;
    const GradPlan plan = grad_plan(g.groups, g.tokens, g.width);
    char* w = (char*)ws;
    int32_t* keys[2] = {(int32_t*)(w + plan.off_keys[0]), (int32_t*)(w + plan.off_keys[1])};
    int32_t* pos[2] = {(int32_t*)(w + plan.off_pos[0]), (int32_t*)(w + plan.off_pos[1])};
    int bits = 1;
    while (bits < 31 && (g.vocab >> bits) != 0) ++bits;   // the key `vocab` stands for "no token"
    const int passes = (bits + kDigitBits - 1) / kDigitBits;
    if (g.tokens > 0) {
        SortParams s;
        s.ids = g.ids, s.ids_group = g.ids_group, s.n = g.tokens, s.vocab = g.vocab;
        s.counts = (int32_t*)(w + plan.off_counts);
        s.blocks = (int)plan.blocks;
        s.keys_in = s.pos_in = nullptr, s.keys_out = s.pos_out = nullptr, s.shift = 0;
        if (plan.blocks == 1) {
            sort_one_block_kernel<<<g.groups, kSortThreads, 0, stream>>>(s, keys[0], pos[0], keys[1], pos[1], passes);
        } else {
            for (int pass = 0; pass < passes; ++pass) {
                const int to = (passes - 1 - pass) % 2;   // the last pass ends in list 0
                s.keys_in = keys[1 - to], s.pos_in = pos[1 - to], s.keys_out = keys[to], s.pos_out = pos[to];
                s.shift = pass * kDigitBits;
                const dim3 grid((unsigned)plan.blocks, g.groups);
                sort_count_kernel<<<grid, kSortThreads, 0, stream>>>(s, pass == 0);
                sort_scatter_kernel<<<grid, kSortThreads, 0, stream>>>(s, pass == 0);
            }
        }
    }
    RowsParams q;
    q.g = g, q.keys = keys[0], q.pos = pos[0], q.partial = (float*)(w + plan.off_partial), q.runs = plan.runs;
    if (g.vocab > 0) {
        if (g.dtype == OLS_F32 && g.grad_dtype == OLS_F32) launch_sums<float, float>(q, stream);
        else if (g.dtype == OLS_F32) launch_sums<float, uint16_t>(q, stream);
        else if (g.grad_dtype == OLS_F32) launch_sums<uint16_t, float>(q, stream);
        else launch_sums<uint16_t, uint16_t>(q, stream);
    }
    return hipGetLastError();
}

}  // namespace ols
