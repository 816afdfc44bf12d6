// Gated feed-forward block, forward and backward, per worker:
//
//   a = x Wg,   b = x Wu,   h = act(a) b,   y = h Wd
//   dh = dy Wd^T,   da = dh b act'(a),   db = dh act(a),   dx = da Wg^T + db Wu^T
//   dWg = x^T da,   dWu = x^T db,   dWd = h^T dy
//
// Both first projections, the activation and the product are one kernel: a tile holds the same columns of a and of b in the
// registers of the same lanes.  Likewise dh never exists in memory: its tiles become da and db.  The products are those of
// ffn_gemm.h; storage type fp32 takes them through three bf16 terms per operand (ffn_gemm_f32.h).  An operand whose rows are 16-byte aligned
// bf16 is read where it lies; others are laid out in the workspace first (rounded to bf16 where the weights are fp32 master
// weights of a bf16 block), by a streaming pass, except large fp32 weights of few rows, which the tiles split themselves.
//
// Few rows (answering token by token) leave nothing to multiply but every weight to read once: there a lane owns eight
// columns, 32 lanes share the contraction, and several workgroups share it further, so that nearly all weights are under way
// at once.  One row through 2048 - 5632 - 2048 in bf16: 25 us in three launches (12.5, 8 and 4: the first reads 46 MB at 3.7
// TB/s; with half the workgroups and half the loads in flight 17.5, 11.5 and 3.5).
//
// 8192 rows through 2048 - 5632 - 2048, forward and backward, bf16: 1.73 to 1.84 ms on different cards, 925 to 983 TFLOP/s;
// ffn_gemm.h says what bounds the products.
// The two with an epilogue of their own add the time of its memory traffic, since the tiles of a round end together: 461 MB
// written behind a, b and h, 553 MB read and written behind da and db.
#include <algorithm>

#include "ffn_gemm.h"
#include "ffn_gemm_f32.h"

namespace ols {

namespace ffn {

constexpr int kFewRows = 8;          // at most: weights are read by the vector unit
constexpr int kFewThreads = 256;
constexpr int kFewCols = 64;         // columns of a workgroup: a line of 128 bytes of bf16 weights
constexpr int kFewSlab = 1024;       // contraction indices whose inputs lie in LDS at a time

struct PackJob {
    const void* src;
    int64_t row, group, rows, cols, cols8;
    uint16_t* dst;                   // [group][rows][cols8]
    int dtype, groups;
};
constexpr int64_t kMostBlocks = 1 << 23;   // of 256: a launch has fewer than 2^32 threads, and wraps without an error beyond
constexpr int kMaxPacks = 5;
struct PackParams {                  // all operands of a call in one launch
    PackJob job[kMaxPacks];
};

template <typename T>
__device__ __forceinline__ void read_unit(const PackJob& p, int64_t g, int64_t i, float (&v)[8]) {
    const int64_t units = p.cols8 / 8, r = i / units, c = i % units * 8;
    load_upto8((const T*)p.src + g * p.group + r * p.row + c, (int)min((int64_t)8, p.cols - c), 0.0f, v);
}

// Rows follow one another without gaps, so unit i of eight elements (48 bytes as terms) lies behind unit i - 1.  A wavefront's terms
// pass through LDS and are written as whole lines.
template <bool SPLIT>
__global__ __launch_bounds__(256) void pack_kernel(PackParams all) {
    const PackJob& p = all.job[blockIdx.z];
    const int64_t units = p.rows * (p.cols8 / 8), g = blockIdx.y;
    if (g >= p.groups) return;
    const int lane = threadIdx.x % 64;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i - lane < units; i += (int64_t)gridDim.x * 256) {
        float v[8] = {};
        if constexpr (!SPLIT) {
            if (i >= units) return;
            if (p.dtype == OLS_F32) read_unit<float>(p, g, i, v);
            else read_unit<uint16_t>(p, g, i, v);
            store_terms<false>(p.dst + (g * units + i) * 8, v);
        } else {
            __shared__ __align__(16) uint16_t stage[256 * 24];
            if (i < units) read_unit<float>(p, g, i, v);
            uint16_t* mine = stage + threadIdx.x / 64 * (64 * 24);
            store_terms<true>(mine + lane * 24, v);
            in_wave_order();
            const int64_t first = i - lane, chunks = min((int64_t)64, units - first) * 3;
            u4* out = (u4*)(p.dst + (g * units + first) * 24);
#pragma unroll
            for (int t = 0; t < 3; ++t)
                if (t * 64 + lane < chunks) out[t * 64 + lane] = *(const u4*)(mine + (t * 64 + lane) * 8);
            in_wave_order();
        }
    }
}

// ---- few rows -------------------------------------------------------------------------------------------------------------

struct FewParams {
    int64_t rows, K, N, n8;
    const void *w, *w2;              // w2: the second projection
    int64_t w_row, w2_row, w_group, w2_group;
    const void* x;                   // first stage: [rows][K]
    int64_t x_row, x_group;
    const float* in;                 // second stage: the first one's partial sums [range][group][rows][2 n8_in]
    int in_ranges, act;
    int64_t in8;
    int ranges;
    float* partial;                  // [range][group][rows][panels n8]
};

// R rows at once.  FIRST: x from memory and two weight matrices; otherwise h = act(a) b from the partial sums of a and b.
template <typename TX, typename TW, int R, bool FIRST>
__global__ __launch_bounds__(kFewThreads) void few_kernel(FewParams p) {
    constexpr int PANELS = FIRST ? 2 : 1;
    constexpr bool ROUND = sizeof(TX) == 2 && sizeof(TW) == 4;  // master weights of a bf16 block: as the products of more rows round them
    __shared__ __align__(16) float xs[kFewSlab][R];
    __shared__ float red[kFewThreads / 64][PANELS][R][kFewCols];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, cl = lane % 8, kl = threadIdx.x / 8;
    const int64_t col = (int64_t)blockIdx.x * kFewCols + cl * 8, group = blockIdx.z;
    const int range = blockIdx.y;
    const int64_t from = p.K * range / p.ranges, to = p.K * (range + 1) / p.ranges;
    const int left = (int)max((int64_t)0, min((int64_t)8, p.N - col));
    const TW* w = (const TW*)p.w + group * p.w_group + col;
    const TW* w2 = FIRST ? (const TW*)p.w2 + group * p.w2_group + col : nullptr;
    constexpr int B = sizeof(TW) == 2 ? 8 : 4;                  // indices whose weights are in flight together
    Raw8<TW> u[B][PANELS];
    auto request = [&](int64_t k0, int i, int n) {
#pragma unroll
        for (int j = 0; j < B; ++j) {
            const int64_t k = k0 + i + 32 * j;
            const int have = i + 32 * j < n ? left : 0;
            u[j][0].load(w + k * p.w_row, have);
            if constexpr (FIRST) u[j][1].load(w2 + k * p.w2_row, have);
        }
    };
    float acc[PANELS][R][8] = {};
    for (int64_t k0 = from; k0 < to; k0 += kFewSlab) {
        const int n = (int)min((int64_t)kFewSlab, to - k0);
        request(k0, kl, n);                                     // before the inputs are waited for
        __syncthreads();
        for (int r = 0; r < R; ++r)
            for (int i = threadIdx.x; i < n; i += kFewThreads) {
                float v = 0.0f;
                if (r < p.rows) {
                    if constexpr (FIRST) {
                        v = load1((const TX*)p.x + group * p.x_group + r * p.x_row + k0 + i);
                    } else {
                        float a = 0.0f, b = 0.0f;
                        const float* in = p.in + (group * p.rows + r) * 2 * p.in8 + k0 + i;
                        const int64_t step = (int64_t)gridDim.z * p.rows * 2 * p.in8;
#pragma unroll 4
                        for (int s = 0; s < p.in_ranges; ++s) a += in[s * step], b += in[s * step + p.in8];
                        v = act_value<sizeof(TX) == 4>(p.act, a) * b;
                    }
                }
                xs[i][r] = v;
            }
        __syncthreads();
        for (int i = kl; i < n; i += 32 * B) {
            if (i > kl) request(k0, i, n);
#pragma unroll
            for (int j = 0; j < B; ++j) {
                if (i + 32 * j >= n) continue;
                if constexpr (ROUND) {
#pragma unroll
                    for (int t = 0; t < PANELS; ++t)
#pragma unroll
                        for (int e = 0; e < 8; ++e) u[j][t].v[e] = of_bf16(bf16_of(u[j][t].v[e]));
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float x = xs[i + 32 * j][r];
#pragma unroll
                    for (int t = 0; t < PANELS; ++t)
#pragma unroll
                        for (int e = 0; e < 8; ++e) acc[t][r][e] = fmaf(x, u[j][t].get(e), acc[t][r][e]);
                }
            }
        }
    }
#pragma unroll
    for (int t = 0; t < PANELS; ++t)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float v = acc[t][r][e];
                for (int o = 8; o < 64; o <<= 1) v += __shfl_xor(v, o);
                if (lane < 8) red[wave][t][r][cl * 8 + e] = v;
            }
    __syncthreads();
    for (int i = threadIdx.x; i < PANELS * R * kFewCols; i += kFewThreads) {
        const int c = i % kFewCols, r = i / kFewCols % R, t = i / (kFewCols * R);
        const int64_t n = (int64_t)blockIdx.x * kFewCols + c;
        if (r >= p.rows || n >= p.n8) continue;
        float v = 0.0f;
        for (int k = 0; k < kFewThreads / 64; ++k) v += red[k][t][r][c];
        p.partial[(((int64_t)range * gridDim.z + group) * p.rows + r) * PANELS * p.n8 + t * p.n8 + n] = v;
    }
}

// ---- host -----------------------------------------------------------------------------------------------------------------

int64_t up8(int64_t v) { return (v + 7) / 8 * 8; }
int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }
int64_t tiles_of(int64_t n, int64_t tile) { return (n + tile - 1) / tile; }

struct Arena {
    char* base;
    int64_t at = 0;
    void* take(int64_t bytes) {
        void* p = base + at;
        at = up256(at + bytes);
        return p;
    }
};

// An operand as the products read it: rows of inner8 elements, or of three times as many where each fp32 is three bf16 terms; or
// the caller's tensor itself.
struct View {
    const uint16_t* p = nullptr;
    int64_t pitch = 0, group = 0, inner8 = 0;
    int64_t rest = 0;                  // to the second term, where it is kept
    bool plain = false;                // fp32 as the caller has it
};

bool lies_well(const ols_matrix& m, int dtype, int64_t inner) {
    return dtype == OLS_BF16 && inner % 8 == 0 && m.row % 8 == 0 && m.row <= (1 << 22) && m.group % 8 == 0 && ((uintptr_t)m.dev & 15) == 0;
}

// A small bf16 block of few rows keeps what rounding h, da and db to bf16 leaves over, as a second term: its results are the formula's
// rounded once, where others add roundings of the inner tensors (1.41 times that error, up to 1.6 where few are added up).  It is kept
// where the longer contractions do not show beside the launches (forward and backward, 17 rows, 104 - 5600 - 22: 71 to 80 us with it,
// 74 without), and not where they do (32 rows, 1024 - 2816 - 1024: 86 us with it, 80 without; 8 rows, 2048 - 5632 - 2048: 124, 110).
bool keeps_rest(const ols_ffn& f) { return f.dtype == OLS_BF16 && f.rows <= 32 && f.hidden * (2 * f.width + f.out) <= (1 << 21); }

struct Maker {                         // lays operands out; without a stream it only measures
    const ols_ffn& f;
    Arena& ws;
    hipStream_t stream;
    bool go;
    PackParams packs = {};
    int n_packs = 0;
    bool split() const { return f.dtype == OLS_F32; }
    int terms() const { return split() ? 3 : 1; }

    View operand(const ols_matrix& m, int dtype, int64_t outer, int64_t inner, bool may_lie) {
        View v;
        v.inner8 = up8(inner), v.pitch = terms() * v.inner8;
        if (may_lie && !split() && lies_well(m, dtype, inner)) {
            v.p = (const uint16_t*)m.dev, v.pitch = m.row, v.group = m.group;
            return v;
        }
        const int64_t per = outer * v.pitch;
        const int groups = m.group == 0 ? 1 : f.groups;      // shared by the workers: laid out once
        uint16_t* dst = (uint16_t*)ws.take(2 * per * groups);
        v.p = dst, v.group = groups == 1 ? 0 : per;
        packs.job[n_packs++] = PackJob{m.dev, m.row, m.group, outer, inner, v.inner8, dst, dtype, groups};
        return v;
    }
    hipError_t lay_out() const {       // the operands asked for
        if (!go || n_packs == 0) return hipSuccess;
        int64_t units = 0;
        int groups = 1;
        for (int i = 0; i < n_packs; ++i) {
            units = std::max(units, packs.job[i].rows * (packs.job[i].cols8 / 8));
            groups = std::max(groups, packs.job[i].groups);
        }
        const dim3 grid((unsigned)std::min(kMostBlocks, (units + 255) / 256), groups, n_packs);
        if (split()) pack_kernel<true><<<grid, 256, 0, stream>>>(packs);
        else pack_kernel<false><<<grid, 256, 0, stream>>>(packs);
        return hipGetLastError();
    }
    // A weight.  Large ones of fp32 that at most two rows of tiles read are not laid out: the tiles split them as they read them, which
    // takes them a quarter longer and saves a pass of 10 bytes an element.  Forward, 43 rows, three workers, 1160 - 3726 - 50: 88 us
    // instead of 115; 128 rows, 1024 - 2816 - 1024: 52, 59; 256: 67, 74; 400 rows, three workers, 500 - 1000 - 700: 73.5, 68.7.
    // Forward and backward, four workers, 128 rows, 512 - 1024 - 512 (6.3 M weights): 124, 134; 200 rows, 800 - 2048 - 800 (4.9 M): 137,
    // 140; 512 - 1408 - 512 (2.2 M): 110, 106; 20 rows, 128 - 256 - 128: 74, 68.
    bool plain(const ols_matrix& m) const {
        const int64_t weights = f.hidden * (2 * f.width + f.out) * (m.group ? f.groups : 1);
        return split() && f.rows <= 256 && weights >= (3 << 20) && m.row <= (1 << 20);
    }
    View weight(const ols_matrix& m, int64_t outer, int64_t inner, bool may_lie) {
        if (!may_lie || !plain(m)) return operand(m, f.weight_dtype, outer, inner, may_lie);
        View v;
        v.p = (const uint16_t*)m.dev, v.pitch = m.row, v.group = m.group, v.inner8 = inner, v.plain = true;
        return v;
    }
    // gate and up are read with one pitch: where theirs differ, both are laid out
    bool pair_lies() const {
        if (split()) return plain(f.w_gate) && plain(f.w_up) && f.w_gate.row == f.w_up.row;
        return lies_well(f.w_gate, f.weight_dtype, f.hidden) && lies_well(f.w_up, f.weight_dtype, f.hidden) && f.w_gate.row == f.w_up.row;
    }
    View internal(int64_t rows, int64_t inner, void* at) const {
        View v;
        v.inner8 = up8(inner), v.pitch = terms() * v.inner8, v.group = rows * v.pitch, v.p = (const uint16_t*)at;
        v.rest = keeps_rest(f) ? f.groups * v.group : 0;
        return v;
    }
    int64_t internal_bytes(int64_t rows, int64_t inner) const { return 2 * (keeps_rest(f) ? 2 : terms()) * f.groups * rows * up8(inner); }
};

void set_operands(Job& j, const View& a, const View& b, const View* a2, const View* b2) {
    j.segments = 0, j.seg_second = 0;
    for (int t = 0; t < (a2 ? 2 : 1); ++t) {
        const View &u = t ? *a2 : a, &v = t ? *b2 : b;
        for (int k = 0; k < 1 + (u.rest || v.rest); ++k) {        // at most one of the two is in terms
            const int s = j.segments++;
            j.seg_a[s] = u.p - a.p + (k ? u.rest : 0), j.seg_b[s] = k ? v.rest : 0;
            if (t) j.seg_second |= 1u << s;
        }
    }
    j.a = a.p, j.a_group = a.group, j.a_pitch = a.pitch, j.a_inner8 = a.inner8;
    j.b = b.p, j.b_group = b.group, j.b_pitch = b.pitch, j.b_inner8 = b.inner8;
    if (b2) j.b2 = b2->p, j.b2_group = b2->group;
}

constexpr int kCus = 256;

struct Shape {
    int t = 0;                         // rows and columns of a tile (columns: of both panels together)
    int whole = 0, rest = 0, ranges = 1;
};

int64_t count_tiles(const Job* jobs, int n, int groups, int panels, int t) {
    int64_t tiles = 0;
    for (int i = 0; i < n; ++i) tiles += groups * tiles_of(jobs[i].M, t) * tiles_of(jobs[i].N, t / panels);
    return tiles;
}

// Workgroups of a round.
int64_t slots_of(int t, bool split) { return split || t == 256 ? kCus : 2 * kCus; }

// What a product takes, in microseconds, by tile, and by how the tiles of the last round are cut.  Fitted to products of 32 to 8192
// rows and 256 to 5632 columns over 300 to 8192 indices (within 15 % of most).  A slice of 32 indices takes a workgroup 0.3 us where
// few run, 0.4 with one on every compute unit and 0.6 with two (tiles of 128); 0.75 to 0.95 with one tile of 256.  Examples,
// 2048 x 1024 over 2816: tiles of 128 whole 40.4 us, cut in 2 / 4 / 8: 31.7 / 32.3 / 45.3; of 256, 74.6 whole, cut in 4 / 8: 38.6 / 40.2.
// 2048 x 5632 over 1024: tiles of 128 39.0, of 256 36.2.  64 x 1024 over 4096: tiles of 128 whole 41.4, cut in 16: 12.8.
// An epilogue with an activation takes a tile 10 to 25 us more, and less where it is done by the launch that joins ranges
// (three ragged fp32 workers, 201 x 517 over 131, Gaussian: 39.7 us whole).
//
// The products of fp32 keep the matrix pipes as busy with one workgroup on a compute unit as with two (a slice of 16: 0.5 us where few
// run, 0.62 with one on every compute unit, 1.2 with two), so a round is one per compute unit.  Fitted to products of 16 to 2048 rows
// and 32 to 5248 columns over 64 to 5248 indices.  291 x 1088 over 3192, three workers, 81 tiles: whole 110.7 us, cut in 2 / 3 / 4 / 6:
// 70.0 / 58.2 / 74.1 / 64.1; 2048 x 1024 over 2816, 128 tiles: whole 101.9, cut in 2: 72.4.
double estimate(const Shape& s, int64_t slices, bool activation, bool split) {
    if (split) {
        auto slice_us = [](double blocks) { return 0.5 + 0.12 * std::min(1.0, blocks / kCus); };
        const double filled = std::min(1.0, (double)s.whole / kCus), act = activation ? 2.0 : 0.0;
        double us = 0.0;
        if (s.whole) us += 1.0 + (double)((s.whole + kCus - 1) / kCus) * (slices * slice_us(s.whole) + 4.5 + act * filled);
        if (s.rest) {
            const double blocks = (double)s.rest * s.ranges;
            us += ((double)slices / s.ranges + 0.5) * slice_us(blocks) + 10.0 + blocks * s.t * s.t * 4.0 / 3.5e6;
        }
        return us;
    }
    const int64_t slots = slots_of(s.t, false);
    auto slice_us = [&](double blocks) {
        const double one = std::min(1.0, blocks / kCus), two = std::min(1.0, std::max(0.0, blocks / kCus - 1.0));
        return s.t == 256 ? 0.75 + 0.2 * one : 0.3 + 0.1 * one + 0.2 * two;
    };
    const double ends = s.t == 256 ? 8.0 : 4.0, act = activation ? 12.0 : 0.0;
    double us = 0.0;
    if (s.whole) us += (double)((s.whole + slots - 1) / slots) * (slices * slice_us((double)std::min((int64_t)s.whole, slots)) + ends + act);
    if (s.rest) {
        const double blocks = (double)s.rest * s.ranges;
        us += ((double)slices / s.ranges + 0.5) * slice_us(blocks) + ends + 5.0 + act / 4 + blocks * s.t * s.t * 4.0 / 8e6;
    }
    return us;
}

// The tile, and whether the contractions of the tiles that fill no whole round are cut.
Shape choose(const Job* jobs, int n, int groups, int panels, bool split, bool activation) {
    int64_t slices = (int64_t)1 << 40, work = 1;
    for (int i = 0; i < n; ++i) {
        const int64_t k = tiles_of(jobs[i].K, split ? kBKF32 : kBK);
        slices = std::min(slices, k), work = std::max(work, k * jobs[i].segments);
    }
    Shape best{};
    double best_us = 1e300;
    for (int t = 128; t <= (split ? 128 : 256); t += 128) {          // fp32: two sets of sums leave no registers for large tiles
        const int64_t slots = slots_of(t, split), tiles = count_tiles(jobs, n, groups, panels, t);
        if ((tiles + slots) * (t == 256 ? 512 : 256) >= (int64_t)1 << 32) continue;      // cut, the tiles of a last round fill it at the most
        for (int ranges : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
            Shape s{t, (int)tiles, 0, 1};
            if (ranges > 1) {
                s.whole = (int)(tiles / slots * slots), s.rest = (int)(tiles - s.whole), s.ranges = ranges;
                if (t == 256 && activation) continue;      // 8192 x 5632 over 2048: 488 us whole, 485 and 22 to join with the last tiles cut
                if (s.rest == 0 || slices < ranges || work / ranges < 4 || (int64_t)s.rest * ranges > slots) continue;
            }
            const double us = estimate(s, work, activation, split);
            if (us < best_us) best = s, best_us = us;
        }
    }
    return best;
}

template <bool A_RC, bool B_RC, Epi EPI>
hipError_t product(Job* jobs, int n, int groups, bool split, bool plain, Arena& ws, bool go, hipStream_t stream) {
    constexpr int PANELS = EPI == kUp ? 2 : 1;
    if (n == 0) return hipSuccess;
    const Shape shape = choose(jobs, n, groups, PANELS, split, EPI != kStore);
    const int t = shape.t;
    if (t == 0) return hipErrorInvalidValue;              // more tiles than a launch numbers: known before anything is launched
    GemmArgs p = {};
    p.jobs = n, p.groups = groups, p.whole = shape.whole, p.rest = shape.rest, p.ranges = shape.ranges;
    int first = 0;
    for (int i = 0; i < n; ++i) {
        Job& j = p.job[i];
        j = jobs[i];
        j.tiles_m = (int)tiles_of(j.M, t), j.tiles_n = (int)tiles_of(j.N, t / PANELS);
        p.first[i] = first;
        first += j.tiles_m * j.tiles_n * groups;
    }
    const bool joins = shape.rest > 0;
    if (joins) p.partial = (float*)ws.take((int64_t)4 * shape.rest * shape.ranges * t * t);
    if (!go) return hipSuccess;
    const unsigned blocks = shape.whole + shape.rest * shape.ranges;
    const dim3 join_grid(shape.rest, (unsigned)(t * (t / PANELS / 8) / 256));
    if (split) {
        if constexpr (!A_RC) {                            // the second operand of the others is never a weight
            if (plain) gemm_f32_kernel<A_RC, B_RC, EPI, true><<<blocks, 256, 0, stream>>>(p);
        }
        if (!plain) gemm_f32_kernel<A_RC, B_RC, EPI, false><<<blocks, 256, 0, stream>>>(p);
        if (joins) join_kernel<EPI, true, 128><<<join_grid, 256, 0, stream>>>(p);
    } else if (t == 256) {
        gemm_kernel<A_RC, B_RC, EPI, 256><<<blocks, 512, 0, stream>>>(p);
        if constexpr (EPI == kStore) {                   // with an activation large tiles are not cut (choose)
            if (joins) join_kernel<EPI, false, 256><<<join_grid, 256, 0, stream>>>(p);
        }
    } else {
        gemm_kernel<A_RC, B_RC, EPI, 128><<<blocks, 256, 0, stream>>>(p);
        if (joins) join_kernel<EPI, false, 128><<<join_grid, 256, 0, stream>>>(p);
    }
    return hipGetLastError();
}

// Adds up the ranges of the kernels for few rows.
__global__ __launch_bounds__(256) void few_join_kernel(Epilogue e, const float* partial, int64_t rows, int groups, int ranges) {
    const int64_t units = e.n8 / 8, stride = (int64_t)groups * rows * e.n8, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * units) return;
    const int64_t n = i % units * 8, row = blockIdx.y * rows + i / units;
    float v[8] = {};
#pragma unroll 4
    for (int s = 0; s < ranges; ++s) {
        float x[8];
        load8(partial + s * stride + row * e.n8 + n, x);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += x[k];
    }
    emit<kStore, false>(e, row / rows, row % rows, n, v, v);
}

Epilogue store_to(const ols_matrix& m, int64_t n, int dtype) {
    Epilogue e = {};
    e.n = n, e.n8 = up8(n), e.c = m.dev, e.c_row = m.row, e.c_group = m.group, e.c_f32 = dtype == OLS_F32;
    return e;
}

// what a forward call leaves for the backward one
struct Saved {
    int64_t off_a, off_b, off_h, bytes;
};
Saved saved_layout(const ols_ffn& f) {
    const int64_t elems = f.groups * f.rows * up8(f.hidden);
    Saved s;
    s.off_a = 0;
    s.off_b = up256(elems * 4);
    s.off_h = 2 * s.off_b;
    s.bytes = up256(s.off_h + elems * 2 * (f.dtype == OLS_F32 ? 3 : keeps_rest(f) ? 2 : 1));
    return s;
}

template <typename TX, typename TW, bool FIRST>
void few(const FewParams& p, int groups, hipStream_t stream) {
    const dim3 grid((unsigned)tiles_of(p.n8, kFewCols), p.ranges, groups);
    if (p.rows == 1) few_kernel<TX, TW, 1, FIRST><<<grid, kFewThreads, 0, stream>>>(p);
    else if (p.rows == 2) few_kernel<TX, TW, 2, FIRST><<<grid, kFewThreads, 0, stream>>>(p);
    else if (p.rows <= 4) few_kernel<TX, TW, 4, FIRST><<<grid, kFewThreads, 0, stream>>>(p);
    else few_kernel<TX, TW, 8, FIRST><<<grid, kFewThreads, 0, stream>>>(p);
}
template <bool FIRST>
void few(const FewParams& p, const ols_ffn& f, hipStream_t stream) {
    if (f.dtype == OLS_F32) few<float, float, FIRST>(p, f.groups, stream);
    else if (f.weight_dtype == OLS_F32) few<uint16_t, float, FIRST>(p, f.groups, stream);
    else few<uint16_t, uint16_t, FIRST>(p, f.groups, stream);
}

int few_ranges(int64_t K, int64_t cols, int groups) {
    const int64_t blocks = tiles_of(cols, kFewCols) * groups;
    return (int)std::max((int64_t)1, std::min(1024 / blocks, K / 256));
}

// Forward; with go false only the workspace is measured.
hipError_t forward(const ols_ffn& f, Arena& ws, bool go, hipStream_t stream) {
    if (f.rows == 0) return hipSuccess;
    const int64_t h8 = up8(f.hidden);
    if (f.rows <= kFewRows && !f.saved) {
        FewParams p = {};
        p.rows = f.rows, p.K = f.width, p.N = f.hidden, p.n8 = h8, p.act = f.act;
        p.w = f.w_gate.dev, p.w_row = f.w_gate.row, p.w_group = f.w_gate.group;
        p.w2 = f.w_up.dev, p.w2_row = f.w_up.row, p.w2_group = f.w_up.group;
        p.x = f.x.dev, p.x_row = f.x.row, p.x_group = f.x.group;
        p.ranges = few_ranges(f.width, h8, f.groups);
        p.partial = (float*)ws.take(4 * p.ranges * f.groups * f.rows * 2 * h8);
        FewParams d = {};
        d.rows = f.rows, d.K = f.hidden, d.N = f.out, d.n8 = up8(f.out), d.act = f.act;
        d.w = f.w_down.dev, d.w_row = f.w_down.row, d.w_group = f.w_down.group;
        d.in = p.partial, d.in_ranges = p.ranges, d.in8 = h8;
        d.ranges = few_ranges(f.hidden, d.n8, f.groups);
        d.partial = (float*)ws.take(4 * d.ranges * f.groups * f.rows * d.n8);
        if (!go) return hipSuccess;
        few<true>(p, f, stream);
        few<false>(d, f, stream);
        const Epilogue e = store_to(f.y, f.out, f.dtype);
        few_join_kernel<<<dim3((unsigned)((f.rows * (d.n8 / 8) + 255) / 256), f.groups), 256, 0, stream>>>(e, d.partial, f.rows, f.groups, d.ranges);
        return hipGetLastError();
    }
    Maker mk{f, ws, stream, go};
    const View x = mk.operand(f.x, f.dtype, f.rows, f.width, true);
    const View wg = mk.weight(f.w_gate, f.width, f.hidden, mk.pair_lies());
    const View wu = mk.weight(f.w_up, f.width, f.hidden, mk.pair_lies());
    const View wd = mk.weight(f.w_down, f.hidden, f.out, true);
    hipError_t e = mk.lay_out();
    if (e != hipSuccess) return e;
    const Saved s = saved_layout(f);
    char* saved = (char*)f.saved;
    void* hp = saved ? (void*)(saved + s.off_h) : ws.take(mk.internal_bytes(f.rows, f.hidden));
    const View h = mk.internal(f.rows, f.hidden, hp);

    Job up = {};
    up.M = f.rows, up.N = f.hidden, up.K = f.width;
    set_operands(up, x, wg, nullptr, &wu);
    up.epi.n = f.hidden, up.epi.n8 = h8, up.epi.pitch = up8(f.hidden), up.epi.m = f.rows, up.epi.act = f.act;
    up.epi.a = saved ? (float*)(saved + s.off_a) : nullptr, up.epi.b = saved ? (float*)(saved + s.off_b) : nullptr, up.epi.h = (uint16_t*)hp, up.epi.rest = h.rest;
    e = product<false, true, kUp>(&up, 1, f.groups, mk.split(), wg.plain, ws, go, stream);
    if (e != hipSuccess) return e;
    Job down = {};
    down.M = f.rows, down.N = f.out, down.K = f.hidden;
    set_operands(down, h, wd, nullptr, nullptr);
    down.epi = store_to(f.y, f.out, f.dtype);
    return product<false, true, kStore>(&down, 1, f.groups, mk.split(), wd.plain, ws, go, stream);
}

__global__ __launch_bounds__(256) void zero_kernel(char* p, int64_t row_bytes, int64_t pitch, int64_t rows, int64_t group, int unit) {
    const int64_t per = row_bytes / unit;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * per; i += (int64_t)gridDim.x * 256) {
        char* at = p + blockIdx.y * group + i / per * pitch + i % per * unit;
        if (unit == 4) *(float*)at = 0.0f;
        else *(uint16_t*)at = 0;
    }
}

hipError_t zero(const ols_matrix& m, int64_t rows, int64_t cols, int dtype, int groups, hipStream_t stream) {
    const int unit = dtype == OLS_F32 ? 4 : 2;
    zero_kernel<<<dim3((unsigned)std::min(kMostBlocks, (rows * cols + 255) / 256), groups), 256, 0, stream>>>((char*)m.dev, cols * unit, m.row * unit, rows, m.group * unit, unit);
    return hipGetLastError();
}

// Whether two matrices of f.rows rows of its type span some of the same memory.
bool meet(const ols_matrix& a, int64_t a_cols, const ols_matrix& b, int64_t b_cols, const ols_ffn& f) {
    const int64_t size = f.dtype == OLS_F32 ? 4 : 2;
    auto end = [&](const ols_matrix& m, int64_t cols) { return (uintptr_t)m.dev + ((f.groups - 1) * m.group + (f.rows - 1) * m.row + cols) * size; };
    return (uintptr_t)a.dev < end(b, b_cols) && (uintptr_t)b.dev < end(a, a_cols);
}

hipError_t backward(const ols_ffn& f, Arena& ws, bool go, hipStream_t stream) {
    const ols_matrix* grads[3] = {&f.g_gate, &f.g_up, &f.g_down};
    if (f.rows == 0) {                       // sums over no rows
        for (int i = 0; i < 3 && go; ++i)
            if (grads[i]->dev) {
                const hipError_t e = zero(*grads[i], i < 2 ? f.width : f.hidden, i < 2 ? f.hidden : f.out, f.grad_dtype, f.groups, stream);
                if (e != hipSuccess) return e;
            }
        return hipSuccess;
    }
    Maker mk{f, ws, stream, go};
    const bool to_up = f.dx.dev || f.g_gate.dev || f.g_up.dev, weights_up = f.g_gate.dev || f.g_up.dev;
    const int64_t h8 = up8(f.hidden);
    const Saved s = saved_layout(f);
    char* saved = (char*)f.saved;
    const View h = mk.internal(f.rows, f.hidden, saved + s.off_h);
    const View dy = mk.operand(f.dy, f.dtype, f.rows, f.out, true);
    View x, wg, wu, wd;
    if (weights_up) x = mk.operand(f.x, f.dtype, f.rows, f.width, true);
    if (to_up) wd = mk.weight(f.w_down, f.hidden, f.out, true);
    if (f.dx.dev) {
        wg = mk.weight(f.w_gate, f.width, f.hidden, mk.pair_lies());
        wu = mk.weight(f.w_up, f.width, f.hidden, mk.pair_lies());
    }
    hipError_t e = mk.lay_out();
    if (e != hipSuccess) return e;
    View da, db;
    if (to_up) {
        void* pa = ws.take(mk.internal_bytes(f.rows, f.hidden));
        void* pb = ws.take(mk.internal_bytes(f.rows, f.hidden));
        da = mk.internal(f.rows, f.hidden, pa), db = mk.internal(f.rows, f.hidden, pb);
        Job dh = {};
        dh.M = f.rows, dh.N = f.hidden, dh.K = f.out;
        set_operands(dh, dy, wd, nullptr, nullptr);
        dh.epi.n = f.hidden, dh.epi.n8 = h8, dh.epi.pitch = up8(f.hidden), dh.epi.m = f.rows, dh.epi.act = f.act;
        dh.epi.a = (float*)(saved + s.off_a), dh.epi.b = (float*)(saved + s.off_b), dh.epi.h = (uint16_t*)pa, dh.epi.h2 = (uint16_t*)pb, dh.epi.rest = da.rest;
        e = product<false, false, kGateGrad>(&dh, 1, f.groups, mk.split(), wd.plain, ws, go, stream);
        if (e != hipSuccess) return e;
    }
    auto to_x = [&]() {
        Job dx = {};
        dx.M = f.rows, dx.N = f.width, dx.K = f.hidden;
        set_operands(dx, da, wg, &db, &wu);
        dx.epi = store_to(f.dx, f.width, f.dtype);
        return product<false, false, kStore>(&dx, 1, f.groups, mk.split(), wg.plain, ws, go, stream);
    };
    // The weights' gradients read x and dy, the one at x reads the weights: whichever may lie on what the other reads comes last.
    const bool x_last = f.dx.dev && (meet(f.dx, f.width, f.x, f.width, f) || meet(f.dx, f.width, f.dy, f.out, f));
    if (f.dx.dev && !x_last) {
        e = to_x();
        if (e != hipSuccess) return e;
    }
    Job dw[kMaxJobs] = {};
    int n = 0;
    for (int i = 0; i < 3; ++i) {
        if (!grads[i]->dev) continue;
        Job& j = dw[n++];
        j.M = i < 2 ? f.width : f.hidden, j.N = i < 2 ? f.hidden : f.out, j.K = f.rows;
        set_operands(j, i < 2 ? x : h, i == 0 ? da : i == 1 ? db : dy, nullptr, nullptr);
        j.epi = store_to(*grads[i], j.N, f.grad_dtype);
    }
    e = product<true, true, kStore>(dw, n, f.groups, mk.split(), false, ws, go, stream);
    return e == hipSuccess && x_last ? to_x() : e;
}

}  // namespace ffn

int64_t ffn_saved_bytes(const ols_ffn& f) { return f.rows == 0 ? 0 : ffn::saved_layout(f).bytes; }
int64_t ffn_workspace_bytes(const ols_ffn& f, bool grad) {
    ffn::Arena ws{nullptr};
    const hipError_t e = grad ? ffn::backward(f, ws, false, nullptr) : ffn::forward(f, ws, false, nullptr);
    return e == hipSuccess ? ws.at : -1;
}
hipError_t launch_ffn(const ols_ffn& f, bool grad, hipStream_t stream) {
    ffn::Arena ws{(char*)f.ws};
    return grad ? ffn::backward(f, ws, true, stream) : ffn::forward(f, ws, true, stream);
}

}  // namespace ols
