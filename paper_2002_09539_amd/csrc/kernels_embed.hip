// Embedding lookup with scaling, and its gradient by sorted tokens, per worker.
//
//   out[n] = scale E[t_n]                         ids outside [0, vocab) are no token: their row of `out` is zero
//   dE[v]  = scale sum_{n : t_n = v} dout[n]       in ascending n, added in fp32, rounded once
//
// Both move bytes and compute nothing to speak of.  The lookup reads one row and writes one per id; a row is spread over
// as many lanes as it has vectors of eight, so that short rows share a workgroup.  64 rows of 1024 bf16: 2.6 us, which is a
// launch.
//
// The gradient could add rows into the table with atomics, whose order (and so whose rounding) changes from run to run,
// and whose rate collapses on the few ids that make up much of a text.  Here the ids are sorted, stably, so that the rows
// of one id are neighbours in a list and every sum has one order:
//   1. radix sort of (id, position), 9 bits a pass: per-workgroup digit counts, then a stable scatter in which every
//      wavefront ranks 64 ids at a time by matching ballots.  Up to kSortItems ids per worker take one workgroup and
//      one launch for all passes.
//      The sort occupies a few compute units; the other workgroups of its launches meanwhile clear the table, since most ids
//      of a vocabulary do not occur.
//   2. the sorted list is cut into runs of kRun positions, a wavefront each, so that the work does not depend on how often
//      an id occurs.  A sum that lies inside a run is a row of the gradient; one that reaches over its end goes to a partial
//      row.  (With a wavefront per table row, the row of an id that makes up 6 % of 32 768 tokens took longer than all
//      the others together: 288 us.)
//   3. the partial rows of an id that several runs hold are added up in order.
//
// 32 768 tokens by a law of words, 50 001 rows of 1024, bf16 to fp32: 91 us; sorting 47 in four launches, which write 205 MB beside
// it (31 without; with the table cleared after the sums, by id: 44 more), the runs 24 (63 MB read, 48 written), joining 11.  Sorting in two
// launches that count all ids in every workgroup: 76.  Four workers of 1201 tokens, 5003 rows of 389 fp32: 30 us; 13.4, 12.1 and 4.3.
#include <algorithm>

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
constexpr int kPerWave = kSortItems / kSortWaves, kPerLane = kPerWave / 64;
constexpr int kRun = 16;                    // sorted positions of a run
constexpr int kMostBlocks = 1 << 23;        // of kThreads: a launch has fewer than 2^32 threads

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

// The gradient's rows as workgroups behind those of the sort clear them, a piece each.
struct ClearParams {
    char* out;                   // rows of row_bytes, row_pitch apart; a table without gaps is one long row
    int64_t rows, row_bytes, row_pitch, group_bytes;
    int64_t piece;               // bytes
    int64_t per_row, rows_per;   // pieces of a row, or (short rows) rows of a piece
    int64_t first;               // this launch's first piece
};
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
    ClearParams clear;
};

constexpr int64_t kClearBytes = 65536;       // of one workgroup, more in tables of more than kMostPieces; 32 to 256 KiB take the same time
constexpr int64_t kMostPieces = 1 << 21;     // of kSortThreads: a launch has fewer than 2^32 threads
// bytes [from, to) of a row by some lanes, `lane` of `lanes`
__device__ __forceinline__ void clear_bytes(char* row, int64_t from, int64_t to, int lane, int lanes) {
    for (int64_t at = from + 16 * lane; at < to; at += 16 * lanes) {
        if (at + 16 <= to) {
            *(u4any*)(row + at) = u4any{0u, 0u, 0u, 0u};
        } else {
            for (int64_t e = at; e < to; e += 2) *(uint16_t*)(row + e) = 0;
        }
    }
}
__device__ __forceinline__ bool cleared(const ClearParams& p, int group, int64_t piece) {
    if (piece < 0) return false;
    piece += p.first;
    char* out = p.out + group * p.group_bytes;
    if (p.rows_per == 0) {
        const int64_t r = piece / p.per_row, from = piece % p.per_row * p.piece;
        clear_bytes(out + r * p.row_pitch, from, min(p.row_bytes, from + p.piece), threadIdx.x, kSortThreads);
    } else {
        const int64_t r0 = piece * p.rows_per, r1 = min(p.rows, r0 + p.rows_per);
        for (int64_t r = r0 + threadIdx.x / 64; r < r1; r += kSortWaves) clear_bytes(out + r * p.row_pitch, 0, p.row_bytes, threadIdx.x % 64, 64);
    }
    return true;
}

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

// The items of a lane: kPerLane of its wavefront's, 64 apart, loaded together.
struct Items {
    int key[kPerLane], pos[kPerLane];
    bool valid[kPerLane];
};
__device__ __forceinline__ Items load_items(const SortParams& p, int group, int block, bool first, bool with_pos) {
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    const int64_t base = (int64_t)block * kSortItems + wave * kPerWave + lane;
    Items t;
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) {
        const int64_t i = base + 64 * k;
        t.valid[k] = i < p.n;
        t.key[k] = t.valid[k] ? key_at(p, group, i, first) : 0;
        t.pos[k] = with_pos && t.valid[k] ? (first ? (int)i : p.pos_in[(int64_t)group * p.n + i]) : 0;
    }
    return t;
}

// One stable pass over the items of one workgroup: item i goes behind every item of a smaller digit and every earlier
// item of its own.  `before[d]`: how many items of all workgroups precede this workgroup's first one of digit d.
__device__ void scatter_block(const SortParams& p, int group, const Items& t, int (*cnt)[kDigits], const int* before) {
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    unsigned long long same[kPerLane];
    int digit[kPerLane];
    for (int i = threadIdx.x; i < kSortWaves * kDigits; i += kSortThreads) (&cnt[0][0])[i] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) {
        digit[k] = (t.key[k] >> p.shift) & (kDigits - 1);
        same[k] = same_digit(digit[k], t.valid[k]);
        if (t.valid[k] && (same[k] & ((1ull << lane) - 1)) == 0) cnt[wave][digit[k]] += __popcll(same[k]);
        in_wave_order();
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
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) {
        const int rank = __popcll(same[k] & ((1ull << lane) - 1));
        if (t.valid[k]) {
            const int64_t at = (int64_t)group * p.n + cnt[wave][digit[k]] + rank;
            p.keys_out[at] = t.key[k];
            p.pos_out[at] = t.pos[k];
        }
        // every lane has read the counter before the first of its digit moves it on (one wavefront, in step)
        in_wave_order();
        if (t.valid[k] && rank == 0) cnt[wave][digit[k]] += __popcll(same[k]);
        in_wave_order();
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

__device__ void count_block(const SortParams& p, const Items& t, int* hist) {
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) hist[d] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kPerLane; ++k)
        if (t.valid[k]) atomicAdd(&hist[(t.key[k] >> p.shift) & (kDigits - 1)], 1);
    __syncthreads();
}

// all passes of a worker whose ids one workgroup holds; ping-pong between the two list pairs
__global__ __launch_bounds__(kSortThreads) void sort_one_block_kernel(SortParams p, int32_t* keys_a, int32_t* pos_a, int32_t* keys_b,
                                                                      int32_t* pos_b, int passes) {
    __shared__ int cnt[kSortWaves][kDigits];
    __shared__ int before[kDigits];
    if (cleared(p.clear, blockIdx.y, (int64_t)blockIdx.x - 1)) return;
    for (int pass = 0; pass < passes; ++pass) {
        const bool to_a = (passes - 1 - pass) % 2 == 0;   // the last pass ends in a
        p.keys_out = to_a ? keys_a : keys_b;
        p.pos_out = to_a ? pos_a : pos_b;
        p.keys_in = to_a ? keys_b : keys_a;
        p.pos_in = to_a ? pos_b : pos_a;
        p.shift = pass * kDigitBits;
        const Items t = load_items(p, blockIdx.y, 0, pass == 0, true);
        count_block(p, t, before);
        scan_digits(before);
        scatter_block(p, blockIdx.y, t, cnt, before);
        __threadfence_block();
        __syncthreads();
    }
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortParams p, int first) {
    __shared__ int hist[kDigits];
    if (cleared(p.clear, blockIdx.y, (int64_t)blockIdx.x - p.blocks)) return;
    count_block(p, load_items(p, blockIdx.y, blockIdx.x, first, false), hist);
    int32_t* out = p.counts + ((int64_t)blockIdx.y * p.blocks + blockIdx.x) * kDigits;
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) out[d] = hist[d];
}

// Every workgroup adds up the counts of all of them itself (blocks x 2 KiB from the L2) instead of waiting for a scan in a
// launch of its own.
__global__ __launch_bounds__(kSortThreads) void sort_scatter_kernel(SortParams p, int first) {
    __shared__ int cnt[kSortWaves][kDigits];
    __shared__ int before[kDigits], total[kDigits];
    static_assert(kSortThreads == 2 * kDigits, "two lanes add up a digit's counts");
    if (cleared(p.clear, blockIdx.y, (int64_t)blockIdx.x - p.blocks)) return;
    const int32_t* counts = p.counts + (int64_t)blockIdx.y * p.blocks * kDigits;
    const int d = threadIdx.x % kDigits, half = threadIdx.x / kDigits, me = blockIdx.x;
    const Items t = load_items(p, blockIdx.y, blockIdx.x, first, true);
    if (half == 0) before[d] = 0, total[d] = 0;
    __syncthreads();
    int less = 0, all = 0;
#pragma unroll 4
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
    scatter_block(p, blockIdx.y, t, cnt, before);
}

// ---- sums over sorted positions -----------------------------------------------------------------------------------------

struct RowsParams {
    EmbedGradParams g;
    const int32_t* keys;
    const int32_t* pos;
    int32_t* ends;       // [group][vocab]: one behind the last sorted position of an id that several runs hold
    float* partial;      // [group][run][2][width]: the sum that the run begins in the middle of, and the one that it ends in the middle of
    int64_t runs;
};

// Eight columns from c of a row of the gradient.
template <typename TO>
__device__ __forceinline__ void write_row(const RowsParams& q, int64_t group, int64_t v, int64_t c, const float (&sum)[8]) {
    if (c >= q.g.width) return;
    TO* out = (TO*)q.g.grad + group * q.g.grad_group + v * q.g.grad_row + c;
    const int left = (int)min((int64_t)8, q.g.width - c);
    float o[8];
    if (q.g.accumulate) {
        load_upto8(out, left, 0.0f, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = fmaf(q.g.scale, sum[e], o[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = q.g.scale * sum[e];
    }
    store_upto8(out, left, o);
}

// A wavefront takes a run and 512 columns, eight a lane; B rows are under way together.
template <typename TI, typename TO>
__global__ __launch_bounds__(kThreads) void embed_runs_kernel(RowsParams q) {
    constexpr int B = sizeof(TI) == 2 ? 16 : 8;
    static_assert(kRun % B == 0 && kRun < 64, "whole batches, and a lane per position");
    const int lane = threadIdx.x % 64;
    const int64_t run = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x / 64), group = blockIdx.y;
    if (run >= q.runs) return;
    const int64_t n = q.g.tokens, from = run * kRun;
    const int have = (int)min((int64_t)kRun, n - from);
    const int32_t* keys = q.keys + group * n + from;
    // lane i holds position i's id and row; lane `have` the next run's first id, `before` is the previous run's last
    const int key = lane < have || (lane == have && from + have < n) ? keys[lane] : -1;
    const int row = lane < have ? q.pos[group * n + from + lane] : 0;
    const int before = from > 0 ? keys[-1] : -1;
    const int down = __shfl_down(key, 1);
    const int64_t vocab = q.g.vocab;
    if (blockIdx.z == 0 && lane < have && key < vocab && key == before && down != key) q.ends[group * vocab + key] = (int)(from + lane + 1);
    const int64_t c = (int64_t)blockIdx.z * 512 + 8 * lane;
    const int left = (int)max((int64_t)0, min((int64_t)8, q.g.width - c));
    const TI* base = (const TI*)q.g.dout + group * q.g.dout_group + c;
    float sum[8] = {};
    bool open = __builtin_amdgcn_readlane(key, 0) == before;    // the sum began in an earlier run
    for (int k = 0; k < have; k += B) {
        Raw8<TI> v[B];
#pragma unroll
        for (int r = 0; r < B; ++r) v[r].load(base + __builtin_amdgcn_readlane(row, k + r) * q.g.dout_row, left);   // positions past the end: row 0
#pragma unroll
        for (int r = 0; r < B; ++r) {
            const int i = k + r, id = __builtin_amdgcn_readlane(key, i);
            if (i >= have || id >= vocab) return;               // sorted: what is no token comes last
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += v[r].get(e);
            const bool ends = __builtin_amdgcn_readlane(key, i + 1) != id;
            if (!ends && i + 1 < have) continue;
            if (ends && !open) {
                write_row<TO>(q, group, id, c, sum);
            } else if (left > 0) {
                store_upto8(q.partial + ((group * q.runs + run) * 2 + (open ? 0 : 1)) * q.g.width + c, left, sum);
            }
            open = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
        }
    }
}

// The ids that several runs hold: workgroups of the run that such an id begins in add up its partial rows, 256 columns each.  Every
// wavefront adds a quarter of them in order, sixteen rows under way together (the most frequent id of a text has a hundred and
// more), and the quarters are added in order.
template <typename TO>
__global__ __launch_bounds__(kThreads) void embed_join_kernel(RowsParams q) {
    constexpr int B = 16, C = 4, W = kThreads / 64;
    __shared__ float quarter[W][64 * C];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t run = blockIdx.x, group = blockIdx.y, from = run * kRun, next = from + kRun;
    const int32_t* keys = q.keys + group * q.g.tokens;
    const int id = keys[next], first = keys[from], last = keys[next - 1], before = from > 0 ? keys[from - 1] : -1;
    if (last != id || id >= q.g.vocab || (first == id && before == id)) return;
    const int64_t all = (q.ends[group * q.g.vocab + id] - 1) / kRun - run + 1, each = all <= B ? B : (all + W - 1) / W;
    const int64_t width = q.g.width, c = (int64_t)blockIdx.z * (64 * C) + lane, k1 = min(all, (wave + 1) * each);
    float sum[C] = {};
    for (int64_t k = wave * each; k < k1; k += B) {
        float p[B][C];
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const float* part = q.partial + ((group * q.runs + run + k + j) * 2 + (k + j == 0 ? 1 : 0)) * width + c;
#pragma unroll
            for (int t = 0; t < C; ++t) p[j][t] = k + j < k1 && c + 64 * t < width ? part[64 * t] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < B; ++j)
#pragma unroll
            for (int t = 0; t < C; ++t) sum[t] += p[j][t];
    }
#pragma unroll
    for (int t = 0; t < C; ++t) quarter[wave][64 * t + lane] = sum[t];
    __syncthreads();
    const int64_t at = (int64_t)blockIdx.z * (64 * C) + threadIdx.x;
    static_assert(64 * C == kThreads, "a column each");
    if (at >= width) return;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) v += quarter[w][threadIdx.x];
    TO* out = (TO*)q.g.grad + group * q.g.grad_group + id * q.g.grad_row + at;
    store1(out, q.g.accumulate ? fmaf(q.g.scale, v, load1(out)) : q.g.scale * v);
}

int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }

struct GradPlan {
    int64_t blocks, runs, off_keys[2], off_pos[2], off_counts, off_ends, off_partial, bytes;
};
GradPlan grad_plan(int groups, int64_t tokens, int64_t vocab, int64_t width) {
    GradPlan p;
    p.blocks = (tokens + kSortItems - 1) / kSortItems;
    p.runs = (tokens + kRun - 1) / kRun;
    int64_t at = 0;
    for (int i = 0; i < 2; ++i) {
        p.off_keys[i] = at, at = up256(at + groups * tokens * 4);
        p.off_pos[i] = at, at = up256(at + groups * tokens * 4);
    }
    p.off_counts = at, at = up256(at + (p.blocks > 1 ? groups * p.blocks * kDigits * 4 : 0));
    p.off_ends = at, at = up256(at + groups * vocab * 4);
    p.off_partial = at, at = up256(at + groups * p.runs * 2 * width * 4);
    p.bytes = at;
    return p;
}

template <typename TI, typename TO>
void launch_sums(const RowsParams& q, hipStream_t stream) {
    if (q.runs == 0) return;
    embed_runs_kernel<TI, TO><<<dim3((unsigned)((q.runs + kThreads / 64 - 1) / (kThreads / 64)), q.g.groups, (unsigned)((q.g.width + 511) / 512)), kThreads, 0, stream>>>(q);
    if (q.runs > 1) embed_join_kernel<TO><<<dim3((unsigned)(q.runs - 1), q.g.groups, (unsigned)((q.g.width + 255) / 256)), kThreads, 0, stream>>>(q);
}

}  // namespace

hipError_t launch_embed(const EmbedParams& p, hipStream_t stream) {
    int lanes = 1;
    while (lanes < kThreads && (int64_t)lanes * 8 < p.width) lanes *= 2;
    if (p.tokens == 0 || p.groups == 0 || p.width == 0) return hipSuccess;
    const int per = kThreads / lanes;                          // ids of a workgroup
    const int64_t most = (int64_t)kMostBlocks * per;           // and of a launch
    for (int64_t first = 0; first < p.tokens; first += most) {
        EmbedParams q = p;
        q.tokens = std::min(most, p.tokens - first);
        q.ids = p.ids + first;
        q.out = (char*)p.out + first * p.out_row * (p.out_dtype == OLS_F32 ? 4 : 2);
        const dim3 grid((unsigned)((q.tokens + per - 1) / per), p.groups);
        if (p.dtype == OLS_F32 && p.out_dtype == OLS_F32) embed_kernel<float, float><<<grid, kThreads, 0, stream>>>(q, lanes);
        else if (p.dtype == OLS_F32) embed_kernel<float, uint16_t><<<grid, kThreads, 0, stream>>>(q, lanes);
        else if (p.out_dtype == OLS_F32) embed_kernel<uint16_t, float><<<grid, kThreads, 0, stream>>>(q, lanes);
        else embed_kernel<uint16_t, uint16_t><<<grid, kThreads, 0, stream>>>(q, lanes);
    }
    return hipGetLastError();
}

int64_t embed_grad_workspace_bytes(int groups, int64_t tokens, int64_t vocab, int64_t width) { return grad_plan(groups, tokens, vocab, width).bytes; }

hipError_t launch_embed_grad(const EmbedGradParams& g, void* ws, hipStream_t stream) {
    if (g.groups == 0 || g.width == 0) return hipSuccess;
    const GradPlan plan = grad_plan(g.groups, g.tokens, g.vocab, g.width);
    char* w = (char*)ws;
    int32_t* keys[2] = {(int32_t*)(w + plan.off_keys[0]), (int32_t*)(w + plan.off_keys[1])};
    int32_t* pos[2] = {(int32_t*)(w + plan.off_pos[0]), (int32_t*)(w + plan.off_pos[1])};
    int bits = 1;
    while (bits < 31 && (g.vocab >> bits) != 0) ++bits;   // the key `vocab` stands for "no token"
    const int passes = (bits + kDigitBits - 1) / kDigitBits;
    SortParams s = {};
    s.ids = g.ids, s.ids_group = g.ids_group, s.n = g.tokens, s.vocab = g.vocab;
    s.counts = (int32_t*)(w + plan.off_counts), s.blocks = (int)plan.blocks;
    // every launch of the sort, which occupies a few of the compute units, clears its share of the table
    const int shares = plan.blocks <= 1 ? 1 : 3 * passes;
    ClearParams& c = s.clear;
    int64_t pieces = 0;
    if (!g.accumulate && g.vocab > 0) {
        const int64_t elem = g.grad_dtype == OLS_F32 ? 4 : 2;
        c.out = (char*)g.grad, c.group_bytes = g.grad_group * elem, c.rows = g.vocab, c.row_bytes = g.width * elem, c.row_pitch = g.grad_row * elem;
        if (g.grad_row == g.width) c.row_bytes *= g.vocab, c.rows = 1;
        for (c.piece = kClearBytes;; c.piece *= 2) {
            c.rows_per = c.rows > 1 && c.row_bytes < c.piece ? c.piece / c.row_bytes : 0;
            c.per_row = (c.row_bytes + c.piece - 1) / c.piece;
            pieces = c.rows_per ? (c.rows + c.rows_per - 1) / c.rows_per : c.rows * c.per_row;
            if (pieces <= kMostPieces) break;
        }
    }
    int done = 0;
    auto clear = [&](int n) {
        c.first = pieces * done / shares;
        done += n;
        return (unsigned)(pieces * done / shares - c.first);
    };
    if (plan.blocks <= 1) {          // without ids the passes find none
        const unsigned blocks = 1 + clear(1);
        sort_one_block_kernel<<<dim3(blocks, g.groups), kSortThreads, 0, stream>>>(s, keys[0], pos[0], keys[1], pos[1], g.tokens > 0 ? passes : 0);
    } else {
        for (int pass = 0; pass < passes; ++pass) {
            const int to = (passes - 1 - pass) % 2;   // the last pass ends in list 0
            s.keys_in = keys[1 - to], s.pos_in = pos[1 - to], s.keys_out = keys[to], s.pos_out = pos[to];
            s.shift = pass * kDigitBits;
            const unsigned counting = (unsigned)plan.blocks + clear(1);
            sort_count_kernel<<<dim3(counting, g.groups), kSortThreads, 0, stream>>>(s, pass == 0);
            const unsigned scattering = (unsigned)plan.blocks + clear(2);       // takes twice as long
            sort_scatter_kernel<<<dim3(scattering, g.groups), kSortThreads, 0, stream>>>(s, pass == 0);
        }
    }
    RowsParams q;
    q.g = g, q.keys = keys[0], q.pos = pos[0], q.partial = (float*)(w + plan.off_partial), q.runs = plan.runs, q.ends = (int32_t*)(w + plan.off_ends);
    if (g.dtype == OLS_F32 && g.grad_dtype == OLS_F32) launch_sums<float, float>(q, stream);
    else if (g.dtype == OLS_F32) launch_sums<float, uint16_t>(q, stream);
    else if (g.grad_dtype == OLS_F32) launch_sums<uint16_t, float>(q, stream);
    else launch_sums<uint16_t, uint16_t>(q, stream);
    return hipGetLastError();
}

}  // namespace ols
