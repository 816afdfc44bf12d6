// Matrix products of the gated feed-forward block on the bf16 matrix cores (v_mfma_f32_32x32x16_bf16, gfx950).
//
// One kernel body computes C[M][N] = sum over segments of A_s B_s with bf16 operands and fp32 sums, for the operand orders
// that the block needs.  An operand is a matrix of 16-byte aligned rows; it is read either
//   * "KC": the contraction index is the contiguous one (memory [rows][K]), or
//   * "RC": the operand's own index is (memory [K][rows]), transposed by the LDS read.
// Segments make fp32 products out of bf16 ones: an fp32 operand is three bf16 planes that add up to it exactly, and the six
// largest of the nine products of planes are six segments of one longer contraction (split_bf16.h says why six are enough).
// The gradient at the block's input, da Wg^T + db Wu^T, is two segments as well.
//
// A tile's slices of 64 contraction indices go from memory straight into LDS (16 bytes a lane, no registers in between),
// into one of two buffers while the other is multiplied; one barrier a slice.  The direct copy writes a wavefront's lanes
// side by side, so rows cannot be padded against bank conflicts: instead every lane fetches another chunk of its row
// than its place says (place = chunk XOR a function of the row), and the fragment reads look there.  Buffer descriptors end at
// the operand's last element, so rows and columns that a tile hangs over read as zeros.
//
// The products are formed with the operands swapped (MFMA rows = columns of C): a lane then holds four consecutive
// columns of one row of C, which the epilogues read and write as vectors.
#pragma once
#include <type_traits>

#include "element_io.h"
#include "ols_internal.h"

namespace ols {
namespace ffn {

constexpr int kBK = 64;              // contraction indices of a slice
constexpr int kXcds = 8;
constexpr int kMaxSegments = 12;

typedef __attribute__((address_space(3))) void* lds_ptr;

// Addresses in LDS are an array plus ONE integer offset: the compiler tells the two buffers apart (and so does not make a
// fragment read wait for the copies into the other one) only where it finds the array within a few steps of the access.

// What a tile copies of one operand.
struct Operand {
    const uint16_t* base;            // of the group and segment
    int64_t pitch;                   // elements between outer indices (rows of KC, contraction indices of RC)
};

// bytes from (outer o, inner i) to the end of the operand's last line, at most 2^31
__device__ __forceinline__ unsigned bytes_left(int64_t outer, int64_t inner8, int64_t pitch, int64_t o, int64_t i) {
    const int64_t left = o < outer ? 2 * ((outer - 1 - o) * pitch + inner8 - i) : 0;
    return (unsigned)min(max(left, (int64_t)0), (int64_t)0x7ffffff0);
}

// KC tile: LDS [ROWS][64], chunk c (8 elements) of row r at place c ^ (r & 7).
template <int ROWS, int THREADS>
struct TileKC {
    static constexpr int kBytes = ROWS * kBK * 2;
    static constexpr int kCopies = kBytes / 1024 / (THREADS / 64);      // per wavefront
    static_assert(kBytes % (1024 * (THREADS / 64)) == 0, "whole copies");
    static constexpr int64_t kUnit = 1;
    unsigned lane_off;
    int chunk;                       // the lane's chunk within the slice
    __device__ TileKC(int64_t pitch) {
        const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
        chunk = (lane % 8) ^ (lane / 8);
        lane_off = (unsigned)((wave * 8 + lane / 8) * pitch * 2 + chunk * 16);
    }
    // rows [row0, row0 + ROWS), contraction indices [k0, k0 + 64) of [rows][k8]
    __device__ void copy(char* lds, int at, const Operand& m, int64_t rows, int64_t k8, int64_t row0, int64_t k0) const {
        const int wave = threadIdx.x / 64;
        const rsrc_t rs = make_rsrc(m.base + row0 * m.pitch + k0, bytes_left(rows, k8, m.pitch, row0, k0));
        const unsigned off = chunk * 8 < k8 - k0 ? lane_off : 0x7ffffff0u;     // past the row's end: zeros
        const unsigned step = (unsigned)(THREADS / 64 * 8 * m.pitch * 2);
#pragma unroll
        for (int t = 0; t < kCopies; ++t)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)(lds + (at + (t * (THREADS / 64) + wave) * 1024)), 16,
                                                     (int)(off >= 0x7ffffff0u ? off : off + t * step), 0, 0, 0);
    }
    // 32 rows from r0 of the tile at `at`, 16 contraction indices 16 s ..: the lane holds k = 16 s + 8 (lane / 32) + 0..7 of row
    // r0 + lane % 32
    __device__ static int lane_part(int at, int r0, int lane) {
        const int r = r0 + lane % 32;
        return at + r * (kBK * 2) + (((lane / 32) ^ (r & 7)) << 4);
    }
    __device__ static bf16x8 frag(const char* lds, int part, int s) { return __builtin_bit_cast(bf16x8, *(const u4*)(lds + (part ^ (s << 5))));
    }
};

// RC tile: LDS [64][COLS], chunk q of line k at place q ^ swizzle(k): the four lines that a transposing read takes together
// fall on different banks.
template <int COLS, int THREADS>
struct TileRC {
    static constexpr int kBytes = COLS * kBK * 2;
    static constexpr int kChunks = COLS / 8, kLines = 64 / kChunks;     // lines of one copy
    static constexpr int kCopies = kBytes / 1024 / (THREADS / 64);
    static_assert(kBytes % (1024 * (THREADS / 64)) == 0 && 64 % kChunks == 0, "whole copies");
    static constexpr int kShift = COLS >= 128 ? 2 : 1;
    __device__ static int swizzle(int k) { return (k & 3) << kShift; }
    unsigned lane_off;
    int line;
    __device__ TileRC(int64_t pitch) {
        const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
        line = wave * kLines + lane / kChunks;                          // the copies of a lane are a multiple of 4 lines apart
        static_assert((THREADS / 64) * kLines % 4 == 0, "one swizzle per lane");
        lane_off = (unsigned)(line * pitch * 2 + ((lane % kChunks) ^ swizzle(line)) * 16);
    }
    // columns [col0, ..), contraction indices [k0, ..) of [K][cols8]
    __device__ void copy(char* lds, int at, const Operand& m, int64_t cols8, int64_t K, int64_t col0, int64_t k0) const {
        const int wave = threadIdx.x / 64;
        const rsrc_t rs = make_rsrc(m.base + k0 * m.pitch + col0, bytes_left(K, cols8, m.pitch, k0, col0));
        const unsigned step = (unsigned)(THREADS / 64 * kLines * m.pitch * 2);
#pragma unroll
        for (int t = 0; t < kCopies; ++t)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)(lds + (at + (t * (THREADS / 64) + wave) * 1024)), 16, (int)(lane_off + t * step), 0, 0, 0);
    }
    // lane j of each block of 16 points at line j / 4, columns 4 (j % 4) ..; lines k and k + 4 have one swizzle
    __device__ static int lane_part(int at, int c0, int lane) {
        const int blk = lane / 16, j = lane % 16;
        const int k = 8 * (blk / 2) + j / 4, c = c0 + 16 * (blk % 2) + 4 * (j % 4);
        return at + k * (COLS * 2) + (((c / 8) ^ swizzle(k)) << 4) + (c % 8) * 2;
    }
    __device__ static bf16x8 frag(const char* lds, int part, int s) {
        const int p = part + s * (16 * COLS * 2);
        typedef s4v __attribute__((address_space(3))) * lds_s4_ptr;
        const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr)(lds + p));
        const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr)(lds + (p + 4 * COLS * 2)));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};


// ---- what is done with a product ------------------------------------------------------------------------------------------

enum Epi { kUp, kStore, kGateGrad };

struct Epilogue {
    int64_t n;                          // columns that exist
    // kStore
    void* c;
    int64_t c_row, c_group;
    int c_f32;
    // kUp: a and b (where they are kept) and h are written; kGateGrad: a and b are read, da and db are written.  Internal
    // tensors have rows of n8 elements; those of planes have [plane][m][n8] per group.
    int act;
    int64_t m, n8;
    void *a, *b;                        // storage type of the call: fp32 with three planes, bf16 with one
    uint16_t *h, *h2;                   // kUp: h.  kGateGrad: da, db
};

__device__ __forceinline__ float act_value(int act, float a) {
    if (act == OLS_ACT_SILU) return a / (1.0f + expf(-a));
    if (act == OLS_ACT_GELU) return 0.5f * a * (1.0f + erff(a * 0.70710678118654752440f));
    return a <= 0.0f ? 0.0f : a;
}
__device__ __forceinline__ void act_both(int act, float a, float& value, float& slope) {
    if (act == OLS_ACT_SILU) {
        const float g = 1.0f / (1.0f + expf(-a));
        value = a * g, slope = g * (1.0f + a * (1.0f - g));
    } else if (act == OLS_ACT_GELU) {
        const float cdf = 0.5f * (1.0f + erff(a * 0.70710678118654752440f));
        value = a * cdf, slope = cdf + a * expf(-0.5f * a * a) * 0.39894228040143267794f;
    } else {
        value = a <= 0.0f ? 0.0f : a, slope = a > 0.0f ? 1.0f : 0.0f;
    }
}

typedef unsigned int u2any __attribute__((ext_vector_type(2), aligned(2)));
typedef unsigned int u4any4 __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ void store4(uint16_t* p, const float (&v)[4], int left) {
    if (left >= 4) {
        *(u2any*)p = u2any{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = bf16_of(v[e]);
    }
}
__device__ __forceinline__ void store4(float* p, const float (&v)[4], int left) {
    if (left >= 4) {
        *(u4any4*)p = u4any4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = v[e];
    }
}
__device__ __forceinline__ void load4(const uint16_t* p, float (&v)[4]) {    // 8-byte aligned
    const u2 w = *(const u2*)p;
    v[0] = bf16_lo(w[0]), v[1] = bf16_hi(w[0]), v[2] = bf16_lo(w[1]), v[3] = bf16_hi(w[1]);
}
__device__ __forceinline__ void load4(const float* p, float (&v)[4]) {
    const f4 w = *(const f4*)p;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = w[e];
}

// four elements of an internal tensor: one bf16 plane, or the three that add up to the fp32 values
template <bool SPLIT>
__device__ __forceinline__ void store_planes(uint16_t* p, int64_t plane, const float (&v)[4]) {
    if constexpr (!SPLIT) {
        *(u2*)p = u2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    } else {
        const Split8 s = split8(f4{v[0], v[1], v[2], v[3]}, f4{0, 0, 0, 0});
        *(u2*)p = u2{s.hi[0], s.hi[1]};
        *(u2*)(p + plane) = u2{s.mid[0], s.mid[1]};
        *(u2*)(p + 2 * plane) = u2{s.lo[0], s.lo[1]};
    }
}

// Columns n .. n + 3 (n a multiple of 4) of row m; `second`: the product with the other panel.
template <Epi EPI, bool SPLIT>
__device__ __forceinline__ void emit(const Epilogue& e, int64_t group, int64_t m, int64_t n, const float (&v)[4], const float (&second)[4]) {
    using T = typename std::conditional<SPLIT, float, uint16_t>::type;
    constexpr int P = SPLIT ? 3 : 1;
    if constexpr (EPI == kStore) {
        const int64_t left = e.n - n;
        if (left <= 0) return;
        const int64_t at = group * e.c_group + m * e.c_row + n;
        if (e.c_f32) store4((float*)e.c + at, v, (int)min(left, (int64_t)4));
        else store4((uint16_t*)e.c + at, v, (int)min(left, (int64_t)4));
    } else {
        if (n >= e.n8) return;
        const int64_t at = (group * e.m + m) * e.n8 + n, plane = e.m * e.n8, at_planes = (group * P * e.m + m) * e.n8 + n;
        float x[4], y[4];
        if constexpr (EPI == kUp) {
            float a[4], b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool real = n + i < e.n;           // the padding of internal rows is zero whatever the operands hold
                a[i] = real ? v[i] : 0.0f, b[i] = real ? second[i] : 0.0f;
                x[i] = real ? act_value(e.act, a[i]) * b[i] : 0.0f;
            }
            if (e.a) {
                store4((T*)e.a + at, a, 4);
                store4((T*)e.b + at, b, 4);
            }
            store_planes<SPLIT>(e.h + at_planes, plane, x);
        } else {
            float a[4], b[4];
            load4((const T*)e.a + at, a);
            load4((const T*)e.b + at, b);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool real = n + i < e.n;
                float value, slope;
                act_both(e.act, a[i], value, slope);
                x[i] = real ? v[i] * b[i] * slope : 0.0f;
                y[i] = real ? v[i] * value : 0.0f;
            }
            store_planes<SPLIT>(e.h + at_planes, plane, x);
            store_planes<SPLIT>(e.h2 + at_planes, plane, y);
        }
    }
}

// ---- the products -----------------------------------------------------------------------------------------------------------

struct Job {
    const uint16_t *a, *b, *b2;          // b2: kUp's second panel, or the second tensor of segments that say so
    int64_t a_group, b_group, b2_group, a_pitch, b_pitch;
    int64_t M, N, K, a_inner8, b_inner8; // inner extents of the operands as stored, up to 8 elements
    int64_t seg_a[kMaxSegments], seg_b[kMaxSegments];
    unsigned seg_second;                 // bit s: segment s takes b2
    int segments, big;                   // the first `big` segments hold the large products
    int tiles_m, tiles_n;
    float* partial;                      // splits > 1: [split][group][M][columns of all panels]
    Epilogue epi;
};
constexpr int kMaxJobs = 3;
struct GemmArgs {
    Job job[kMaxJobs];
    int jobs, groups, splits, total, chunk;      // total: tiles of all jobs, groups and ranges of K; chunk: of one XCD
    int first[kMaxJobs];                         // each job's first tile
};

template <bool A_RC, bool B_RC, Epi EPI, bool SPLIT, int BM, int BN, int THREADS>
__global__ __launch_bounds__(THREADS, 2) void gemm_kernel(GemmArgs p) {
    constexpr int WAVES = THREADS / 64, WN = BN / 64, WM = WAVES / WN, TM = BM / WM / 32, TN = 2;
    constexpr int PANELS = EPI == kUp ? 2 : 1;
    using TA = typename std::conditional<A_RC, TileRC<BM, THREADS>, TileKC<BM, THREADS>>::type;
    using TB = typename std::conditional<B_RC, TileRC<BN / PANELS, THREADS>, TileKC<BN / PANELS, THREADS>>::type;
    constexpr int kBytes = TA::kBytes + PANELS * TB::kBytes;
    __shared__ __align__(1024) char buf0[kBytes];
    __shared__ __align__(1024) char buf1[kBytes];

    // the hardware deals workgroup b to XCD b % 8: each XCD takes a contiguous range of tiles, whose operands its L2 keeps
    int tile = (int)(blockIdx.x % kXcds) * p.chunk + (int)(blockIdx.x / kXcds);
    if ((int)(blockIdx.x / kXcds) >= p.chunk || tile >= p.total) return;
    int j = 0;
    while (j + 1 < p.jobs && tile >= p.first[j + 1]) ++j;
    const Job& q = p.job[j];
    tile -= p.first[j];
    const int per_group = q.tiles_m * q.tiles_n;
    const int range = tile / (per_group * p.groups);
    const int64_t group = tile / per_group % p.groups;
    tile %= per_group;
    constexpr int kBand = 8;                                  // tiles in bands of eight rows of tiles, down each column of the band
    const int band = tile / (kBand * q.tiles_n), rows_here = min(kBand, q.tiles_m - band * kBand);
    const int in_band = tile - band * kBand * q.tiles_n;
    const int64_t m0 = (int64_t)(band * kBand + in_band % rows_here) * BM;
    const int64_t n0 = (int64_t)(in_band / rows_here) * (BN / PANELS);

    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, wm = wave / WN, wn = wave % WN;
    const TA ta(q.a_pitch);
    const TB tb(q.b_pitch);
    const int slices = (int)((q.K + kBK - 1) / kBK);
    const int from = (int)((int64_t)slices * range / p.splits), here = (int)((int64_t)slices * (range + 1) / p.splits) - from;

    f16v acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][t][r] = 0.0f;

    auto copy = [&](char* lds, int it) {
        const int seg = it / here;
        const int64_t k0 = (int64_t)(from + it - seg * here) * kBK;
        const Operand a{q.a + group * q.a_group + q.seg_a[seg], q.a_pitch};
        const bool second = (q.seg_second >> seg) & 1u;
        const Operand b{(second ? q.b2 + group * q.b2_group : q.b + group * q.b_group) + q.seg_b[seg], q.b_pitch};
        if constexpr (A_RC) ta.copy(lds, 0, a, q.a_inner8, q.K, m0, k0);
        else ta.copy(lds, 0, a, q.M, q.a_inner8, m0, k0);
        if constexpr (B_RC) tb.copy(lds, TA::kBytes, b, q.b_inner8, q.K, n0, k0);
        else tb.copy(lds, TA::kBytes, b, q.N, q.b_inner8, n0, k0);
        if constexpr (PANELS == 2) {
            const Operand b2{q.b2 + group * q.b2_group + q.seg_b[seg], q.b_pitch};
            tb.copy(lds, TA::kBytes + TB::kBytes, b2, q.b_inner8, q.K, n0, k0);
        }
    };
    int part_a[TM], part_b[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) part_a[i] = TA::lane_part(0, wm * (BM / WM) + 32 * i, lane);
#pragma unroll
    for (int t = 0; t < TN; ++t) part_b[t] = TB::lane_part(TA::kBytes + (PANELS == 2 ? t * TB::kBytes : 0), PANELS == 2 ? wn * 32 : wn * 64 + 32 * t, lane);
    // opaque from here on: addresses stay an array plus one offset (see the top of the file)
#pragma unroll
    for (int i = 0; i < TM; ++i) asm("" : "+v"(part_a[i]));
#pragma unroll
    for (int t = 0; t < TN; ++t) asm("" : "+v"(part_b[t]));
    auto multiply = [&](const char* lds) {
        bf16x8 fa[2][TM], fb[2][TN];
        auto fetch = [&](int s, bf16x8 (&x)[TM], bf16x8 (&y)[TN]) {
#pragma unroll
            for (int t = 0; t < TN; ++t) y[t] = TB::frag(lds, part_b[t], s);
#pragma unroll
            for (int i = 0; i < TM; ++i) x[i] = TA::frag(lds, part_a[i], s);
        };
        fetch(0, fa[0], fb[0]);
#pragma unroll
        for (int s = 0; s < kBK / 16; ++s) {
            if (s + 1 < kBK / 16) fetch(s + 1, fa[(s + 1) & 1], fb[(s + 1) & 1]);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int t = 0; t < TN; ++t) acc[i][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[s & 1][t], fa[s & 1][i], acc[i][t], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);     // fragments of two steps at a time, not of the whole slice: registers
        }
    };
    // fp32: the large products come first.  Where their sum is infinite the small ones, products of an infinity with a remainder
    // of zero among them, have nothing to add: such sums are kept as they are (a bit each for +inf and -inf; a NaN stays one).
    const int small_from = SPLIT ? here * q.big : -1, end = here * q.segments;
    unsigned pos[TM][TN] = {}, neg[TM][TN] = {};
    auto mark = [&]() {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    pos[i][t] |= acc[i][t][r] == INFINITY ? 1u << r : 0u;
                    neg[i][t] |= acc[i][t][r] == -INFINITY ? 1u << r : 0u;
                }
    };
    // The slice has landed, and everyone is done with the buffer that the next copy overwrites.
    auto turn = [&]() {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // this wavefront's copies; the others' are behind the barrier
        __syncthreads();
    };
    if (end > 0) copy(buf0, 0);
    for (int it = 0; it < end; it += 2) {
        turn();
        if (it + 1 < end) copy(buf1, it + 1);
        if (SPLIT && it == small_from) mark();
        multiply(buf0);
        if (it + 1 >= end) break;
        turn();
        if (it + 2 < end) copy(buf0, it + 2);
        if (SPLIT && it + 1 == small_from) mark();
        multiply(buf1);
    }
    if constexpr (SPLIT) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][t][r] = (pos[i][t] >> r) & 1u ? INFINITY : (neg[i][t] >> r) & 1u ? -INFINITY : acc[i][t][r];
    }

#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t m = m0 + wm * (BM / WM) + 32 * i + lane % 32;
        if (m >= q.M) continue;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float v[2][4];
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[t][e] = acc[i][t][4 * g + e];
            const int in = 8 * g + 4 * (lane / 32);
            if (p.splits > 1) {
                const int64_t width = PANELS * q.epi.n8;
                float* row = q.partial + ((range * (int64_t)p.groups + group) * q.M + m) * width;
#pragma unroll
                for (int t = 0; t < TN; ++t) {
                    const int64_t n = PANELS == 2 ? n0 + wn * 32 + in : n0 + wn * 64 + 32 * t + in;
                    if (n < q.epi.n8) store4(row + (PANELS == 2 ? t * q.epi.n8 : 0) + n, v[t], 4);
                }
            } else if constexpr (PANELS == 2) {
                emit<EPI, SPLIT>(q.epi, group, m, n0 + wn * 32 + in, v[0], v[1]);
            } else {
#pragma unroll
                for (int t = 0; t < TN; ++t) emit<EPI, SPLIT>(q.epi, group, m, n0 + wn * 64 + 32 * t + in, v[t], v[t]);
            }
        }
    }
}

// Adds up the ranges of K, in order, and does the epilogue's work.
template <Epi EPI, bool SPLIT>
__global__ __launch_bounds__(256) void join_kernel(Epilogue e, const float* partial, int64_t rows, int groups, int splits) {
    constexpr int PANELS = EPI == kUp ? 2 : 1;
    const int64_t quads = e.n8 / 4, width = PANELS * e.n8, stride = (int64_t)groups * rows * width;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= groups * rows * quads) return;
    const int64_t n = i % quads * 4, row = i / quads;
    float v[2][4] = {};
    for (int s = 0; s < splits; ++s)
#pragma unroll
        for (int t = 0; t < PANELS; ++t) {
            float x[4];
            load4(partial + s * stride + row * width + t * e.n8 + n, x);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[t][k] += x[k];
        }
    emit<EPI, SPLIT>(e, row / rows, row % rows, n, v[0], v[PANELS - 1]);
}

}  // namespace ffn
}  // namespace ols
