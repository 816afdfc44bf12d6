// Matrix products of the gated feed-forward block on the bf16 matrix cores (v_mfma_f32_32x32x16_bf16, gfx950).
//
// One kernel body computes C[M][N] = sum over segments of A_s B_s with bf16 operands and fp32 sums, for the operand orders
// that the block needs.  An operand is a matrix of 16-byte aligned rows; it is read either
//   * "KC": the contraction index is the contiguous one (memory [rows][K]), or
//   * "RC": the operand's own index is (memory [K][rows]), transposed by the LDS read.
// The gradient at the block's input, da Wg^T + db Wu^T, is two segments of one contraction; an operand in two terms doubles them.  Products of fp32 operands are
// in ffn_gemm_f32.h, on the same tiles, jobs and epilogues.
//
// A tile's slices of 32 contraction indices go from memory straight into LDS (16 bytes a lane, no registers in between),
// into a ring of four buffers: three slices are under way while one is multiplied.  The direct copy writes a wavefront's
// lanes side by side, so rows cannot be padded against bank conflicts: instead every lane fetches another chunk of its row
// than its place says (place = chunk XOR a function of the row), and the fragment reads look there.  Buffer descriptors end
// at the operand's last element, so rows and columns that a tile hangs over read as zeros.
//
// Each of a slice's two steps first requests the next step's fragments, the second one those of the next slice, in front of
// which stands the only barrier of a slice.
//
// What bounds it, measured warm on products of 8192 rows, 2048 by 5632 (K contiguous in both operands, unless stated): without
// the copies, on what lies in LDS, 1440 TFLOP/s; the copies alone, at 1.5 times the bytes of a 256 x 256 tile, take as long as
// 1200 would; together 1110 (1160 with the second operand RC).  Tiles of 256 x 128, two workgroups a compute unit: 974.  Two
// buffers of 64 indices: 1107.  Four wavefronts of 128 x 128, one a
// SIMD, with a third less to read from LDS: 4 to 15 % slower than eight, also with the reads between the products.  Wavefront priorities,
// fragment reads spread between the MFMAs, other orders of tiles, rotated starts, rows apart by other than their length: nothing,
// or less.  A library's product of these sizes runs at 1100 to 1370.
//
// Results pass through LDS on their way out: what a lane holds after the MFMAs are four columns of a row, and memory wants
// whole lines (with 8-byte pieces, the product with the gradients' epilogue ran at 410 TFLOP/s instead of 540).
#pragma once
#include <type_traits>

#include "element_io.h"
#include "ols_internal.h"

namespace ols {
namespace ffn {

constexpr int kBK = 32;              // contraction indices of a slice
constexpr int kRing = 4;             // buffers
constexpr int kXcds = 8;
constexpr int kMaxSegments = 4;

typedef __attribute__((address_space(3))) void* lds_ptr;

// Addresses in LDS are an array plus ONE integer offset: the compiler tells the two buffers apart (and so does not make a
// fragment read wait for the copies into the other one) only where it finds the array within a few steps of the access.

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }   // the same in every lane: kept as a scalar

// Where the next slice of a tile lies: its first element and the bytes from there to the operand's last one.
struct Cursor {
    const char* at;
    int64_t left;
    int64_t step;                        // bytes from slice to slice
    __device__ rsrc_t window() const { return make_rsrc(at, (unsigned)min(max(left, (int64_t)0), (int64_t)0x7ffffff0)); }
    __device__ void advance() { at += step, left -= step; }
};

// KC tile: LDS [ROWS][32], chunk c (8 elements) of row r at place c ^ (r / 4 & 3): sixteen rows' chunks lie on different banks.
template <int ROWS, int THREADS>
struct TileKC {
    static constexpr int kBytes = ROWS * kBK * 2;
    static constexpr int kCopies = kBytes / 1024 / (THREADS / 64);      // per wavefront
    static_assert(kBytes % (1024 * (THREADS / 64)) == 0 && kBK == 32, "whole copies of sixteen rows");
    unsigned lane_off, step;
    int chunk;                           // the lane's chunk within the slice
    __device__ TileKC(int64_t pitch) {
        const int lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64);
        chunk = (lane % 4) ^ (lane / 16);
        lane_off = (unsigned)((wave * 16 + lane / 4) * pitch * 2 + chunk * 16);
        step = (unsigned)(THREADS / 64 * 16 * pitch * 2);
    }
    // rows [row0, row0 + ROWS), contraction indices from k0 of [rows][k8]
    __device__ static Cursor cursor(const uint16_t* base, int64_t pitch, int64_t rows, int64_t k8, int64_t row0, int64_t k0) {
        return {(const char*)(base + row0 * pitch + k0), 2 * ((rows - 1 - row0) * pitch + k8 - k0), 2 * kBK};
    }
    __device__ void copy(char* lds, int at, const Cursor& c, int64_t k_left) const {
        const int wave = uniform(threadIdx.x / 64);
        const rsrc_t rs = c.window();
        const bool inside = chunk * 8 < k_left;               // past the row's end: beyond any window, zeros
#pragma unroll
        for (int t = 0; t < kCopies; ++t)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)(lds + (at + (t * (THREADS / 64) + wave) * 1024)), 16,
                                                     (int)(inside ? lane_off + t * step : 0x7ffffff0u), 0, 0, 0);
    }
    // 32 rows from r0 of the tile at `at`, 16 contraction indices 16 s ..: the lane holds k = 16 s + 8 (lane / 32) + 0..7 of row
    // r0 + lane % 32
    __device__ static int lane_part(int at, int r0, int lane) {
        const int r = r0 + lane % 32;
        return at + r * (kBK * 2) + (((lane / 32) ^ ((r >> 2) & 3)) << 4);
    }
    __device__ static bf16x8 frag(const char* lds, int part, int s) { return __builtin_bit_cast(bf16x8, *(const u4*)(lds + (part ^ (s << 5)))); }
};

// RC tile: LDS [32][COLS], chunk q of line k at place q ^ swizzle(k): the four lines that a transposing read takes together
// lie on different banks.
template <int COLS, int THREADS>
struct TileRC {
    static constexpr int kBytes = COLS * kBK * 2;
    static constexpr int kChunks = COLS / 8, kLines = 64 / kChunks;     // lines of one copy
    static constexpr int kCopies = kBytes / 1024 / (THREADS / 64);
    static_assert(kBytes % (1024 * (THREADS / 64)) == 0 && 64 % kChunks == 0, "whole copies");
    static constexpr int kShift = COLS >= 128 ? 2 : 1;
    __device__ static int swizzle(int k) { return (k & 3) << kShift; }
    unsigned lane_off, step;
    __device__ TileRC(int64_t pitch) {
        const int lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64);
        const int line = wave * kLines + lane / kChunks;                // the copies of a lane are a multiple of 4 lines apart
        static_assert((THREADS / 64) * kLines % 4 == 0, "one swizzle per lane");
        lane_off = (unsigned)(line * pitch * 2 + ((lane % kChunks) ^ swizzle(line)) * 16);
        step = (unsigned)(THREADS / 64 * kLines * pitch * 2);
    }
    // columns [col0, ..), contraction indices from k0 of [K][cols8]
    __device__ static Cursor cursor(const uint16_t* base, int64_t pitch, int64_t cols8, int64_t K, int64_t col0, int64_t k0) {
        return {(const char*)(base + k0 * pitch + col0), 2 * ((K - 1 - k0) * pitch + cols8 - col0), 2 * kBK * pitch};
    }
    __device__ void copy(char* lds, int at, const Cursor& c, int64_t) const {
        const int wave = uniform(threadIdx.x / 64);
        const rsrc_t rs = c.window();
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
    // tensors have rows of n8 elements, pitch apart, h and its gradients three times that where they are kept as terms.
    int act;
    int64_t m, n8, pitch;
    // a and b stay fp32 in a bf16 block as well: rounded to bf16 they would put the weights' gradients at 1.8 times the error of
    // their own rounding (3.1e-3 against 64 bits where da's and the result's roundings alone make 2.3e-3).
    float *a, *b;
    uint16_t *h, *h2;                   // kUp: h.  kGateGrad: da, db
    int64_t rest;                       // from a bf16 value to the place of what its rounding has left over; 0: that is not kept
};

// The hardware's exponential and reciprocal are good to a unit in the last place each, but the argument's rounding adds 2^-24 |a| to the
// exponential's relative error: 3e-6 of a SiLU far below zero, which is nothing to a bf16's rounding.  (With expf and a correctly rounded
// division the epilogues of large bf16 blocks were bound by the vector unit: 517 and 317 us of the two products that have one.)
// FULL, the SiLU of fp32 blocks, is good to four units in the last place whatever its size: the exponential makes up for what its
// argument's product with log2 e leaves over.  GELU's slope adds its exponential to a distribution function that is good to 2^-24
// absolutely, so the hardware's is enough there.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f); }
__device__ __forceinline__ float full_exp_of(float x) {
    constexpr float kHigh = 1.44269502162933349609f, kLow = 1.92596299112661747e-8f;      // log2 e
    x = fminf(fmaxf(x, -200.0f), 200.0f);                                                  // 0 and infinity; what is left over stays finite
    const float t = x * kHigh, left = fmaf(x, kLow, fmaf(x, kHigh, -t));
    return __builtin_amdgcn_exp2f(t) * fmaf(left, 0.69314718055994530942f, 1.0f);
}
template <bool FULL>
__device__ __forceinline__ float sigmoid(float a) { return __builtin_amdgcn_rcpf(1.0f + (FULL ? full_exp_of(-a) : exp_of(-a))); }

template <bool FULL>
__device__ __forceinline__ float act_value(int act, float a) {
    if (act == OLS_ACT_SILU) return a * sigmoid<FULL>(a);
    if (act == OLS_ACT_GELU) return 0.5f * a * (1.0f + erff(a * 0.70710678118654752440f));
    return a <= 0.0f ? 0.0f : a;
}
template <bool FULL>
__device__ __forceinline__ void act_both(int act, float a, float& value, float& slope) {
    if (act == OLS_ACT_SILU) {
        const float g = sigmoid<FULL>(a);
        value = a * g, slope = g * (1.0f + a * (1.0f - g));
    } else if (act == OLS_ACT_GELU) {
        const float cdf = 0.5f * (1.0f + erff(a * 0.70710678118654752440f));
        value = a * cdf, slope = cdf + a * exp_of(-0.5f * a * a) * 0.39894228040143267794f;
    } else {
        value = a <= 0.0f ? 0.0f : a, slope = a > 0.0f ? 1.0f : 0.0f;
    }
}

// eight elements of an internal tensor: bf16, or the three terms that add up to the fp32 values, side by side
template <bool SPLIT>
__device__ __forceinline__ void store_terms(uint16_t* p, const float (&v)[8], int64_t rest = 0) {
    if constexpr (!SPLIT) {
        const u4 w = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
        *(u4*)p = w;
        if (rest) {
            float r[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float hi = i % 2 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
                r[i] = fabsf(hi) < INFINITY ? v[i] - hi : 0.0f;
            }
            *(u4*)(p + rest) = u4{pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3]), pack_bf16(r[4], r[5]), pack_bf16(r[6], r[7])};
        }
    } else {
        const Split8 s = split8(f4{v[0], v[1], v[2], v[3]}, f4{v[4], v[5], v[6], v[7]});
        *(u4*)p = s.hi;
        *(u4*)(p + 8) = s.mid;
        *(u4*)(p + 16) = s.lo;
    }
}

// Columns n .. n + 7 (n a multiple of 8) of row m; `second`: the product with the other panel.
template <Epi EPI, bool SPLIT>
__device__ __forceinline__ void emit(const Epilogue& e, int64_t group, int64_t m, int64_t n, const float (&v)[8], const float (&second)[8]) {
    constexpr int P = SPLIT ? 3 : 1;
    if (n >= e.n8) return;
    if constexpr (EPI == kStore) {
        const int left = (int)min((int64_t)8, e.n - n);
        const int64_t at = group * e.c_group + m * e.c_row + n;
        if (e.c_f32) store_upto8((float*)e.c + at, left, v);
        else store_upto8((uint16_t*)e.c + at, left, v);
    } else {
        const int64_t at = (group * e.m + m) * e.pitch + n;
        const int real = (int)min((int64_t)8, e.n - n);
        float a[8], b[8], x[8], y[8];
        if constexpr (EPI == kUp) {
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = v[i], b[i] = second[i], x[i] = act_value<SPLIT>(e.act, v[i]) * second[i];
            if (real < 8) {                              // the padding of internal rows is zero whatever the operands hold
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i >= real) a[i] = b[i] = x[i] = 0.0f;
            }
            if (e.a) {
                store8(e.a + at, a);
                store8(e.b + at, b);
            }
            store_terms<SPLIT>(e.h + P * at, x, e.rest);
        } else {
            load8(e.a + at, a);
            load8(e.b + at, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float value, slope;
                act_both<SPLIT>(e.act, a[i], value, slope);
                x[i] = v[i] * b[i] * slope, y[i] = v[i] * value;
            }
            if (real < 8) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i >= real) x[i] = y[i] = 0.0f;
            }
            store_terms<SPLIT>(e.h + P * at, x, e.rest);
            store_terms<SPLIT>(e.h2 + P * at, y, e.rest);
        }
    }
}

// ---- the products -----------------------------------------------------------------------------------------------------------

struct Job {
    const uint16_t *a, *b, *b2;          // b2: kUp's second panel, or the second tensor of segments that say so
    int64_t a_group, b_group, b2_group, a_pitch, b_pitch;
    int64_t M, N, K, a_inner8, b_inner8; // inner extents of the operands as stored, up to 8 elements
    int64_t seg_a[kMaxSegments], seg_b[kMaxSegments];   // from a and b (or b2) to each segment's operands
    unsigned seg_second;                 // bit s: segment s takes b2
    int segments;
    int tiles_m, tiles_n;
    Epilogue epi;
};
constexpr int kMaxJobs = 3;
struct GemmArgs {
    Job job[kMaxJobs];
    int jobs, groups;
    int first[kMaxJobs];                 // each job's first tile
    // Tiles [0, whole) are computed by a workgroup each.  The `rest` behind them would leave most of the device idle in a round of
    // their own: their contractions are cut into `ranges`, whose sums go to `partial` ([range][tile][rows][columns]) and are
    // joined by another launch.
    int whole, rest, ranges;
    float* partial;
};

struct TilePlace {
    int job;
    int64_t group, m0, n0;
};
__device__ __forceinline__ TilePlace place_of(const GemmArgs& p, int tile, int bm, int bn) {
    int j = 0;
    while (j + 1 < p.jobs && tile >= p.first[j + 1]) ++j;
    const Job& q = p.job[j];
    tile -= p.first[j];
    const int per_group = q.tiles_m * q.tiles_n;
    TilePlace t;
    t.job = j, t.group = tile / per_group;
    tile %= per_group;
    constexpr int kBand = 8;             // bands of eight rows of tiles, down each column of the band: what runs together shares operands
    const int band = tile / (kBand * q.tiles_n), rows = min(kBand, q.tiles_m - band * kBand), in_band = tile - band * kBand * q.tiles_n;
    t.m0 = (int64_t)(band * kBand + in_band % rows) * bm, t.n0 = (int64_t)(in_band / rows) * bn;
    return t;
}

// The tile of a workgroup, and the range of its contraction (-1: all of it).  The hardware deals workgroup b to XCD b % 8: each XCD
// takes a contiguous range of tiles, whose operands its L2 keeps.
__device__ __forceinline__ int tile_of_block(const GemmArgs& p, int& range) {
    range = -1;
    if ((int)blockIdx.x < p.whole) {
        const int per = (p.whole + kXcds - 1) / kXcds, full = p.whole % kXcds == 0 ? kXcds : p.whole % kXcds, xcd = blockIdx.x % kXcds;
        return xcd * per - max(0, xcd - full) + blockIdx.x / kXcds;        // the first `full` XCDs take one tile more where it does not divide
    }
    const int u = blockIdx.x - p.whole;
    range = u / p.rest;
    return p.whole + u % p.rest;
}

// A wavefront's part of a tile on its way out, through its own piece of LDS: 32 rows at a time as [32][TN * 32], chunks of 16 bytes
// at place chunk ^ (row & 15).
template <Epi EPI, bool SPLIT, int T, int TM, int TN>
__device__ __forceinline__ void write_tile(const f16v (&acc)[TM][TN], float* stage, const GemmArgs& p, const TilePlace& at, int tile, int range) {
    constexpr int PANELS = EPI == kUp ? 2 : 1;
    constexpr int kCols = TN * 32, kUnits = kCols / 8 / PANELS, kRows = 64 / kUnits;
    const Job& q = p.job[at.job];
    const int lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64), wm = wave / 2, wn = wave % 2;
    const int lane_row = lane % 32, out_row = lane / kUnits, unit = lane % kUnits;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int chunk = 8 * t + 2 * g + lane / 32;
                *(f4*)(stage + lane_row * kCols + 4 * (chunk ^ (lane_row & 15))) = f4{acc[i][t][4 * g], acc[i][t][4 * g + 1], acc[i][t][4 * g + 2], acc[i][t][4 * g + 3]};
            }
        in_wave_order();                                  // written and read by one wavefront: LDS keeps its order
#pragma unroll 1
        for (int r0 = 0; r0 < 32; r0 += kRows) {
            const int r = r0 + out_row;
            float v[PANELS][8];
#pragma unroll
            for (int q2 = 0; q2 < PANELS; ++q2)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int chunk = q2 * (kCols / 4 / PANELS) + 2 * unit + h;
                    const f4 w = *(const f4*)(stage + r * kCols + 4 * (chunk ^ (r & 15)));
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[q2][4 * h + e] = w[e];
                }
            const int row = wm * (32 * TM) + 32 * i + r, col = wn * (T / 2 / PANELS) + 8 * unit;
            if (range >= 0) {
                float* out = p.partial + ((int64_t)range * p.rest + (tile - p.whole)) * (T * T) + (int64_t)row * T + col;
#pragma unroll
                for (int q2 = 0; q2 < PANELS; ++q2) store8(out + q2 * (T / PANELS), v[q2]);
            } else if (at.m0 + row < q.M) {
                emit<EPI, SPLIT>(q.epi, at.group, at.m0 + row, at.n0 + col, v[0], v[PANELS - 1]);
            }
        }
        in_wave_order();
    }
}

// T x T tiles: 256 with eight wavefronts of 64 x 128, 128 with four of 64 x 64.
template <int T>
constexpr int gemm_threads() { return T == 256 ? 512 : 256; }

template <bool A_RC, bool B_RC, Epi EPI, int T>
__global__ __launch_bounds__(gemm_threads<T>(), 2) void gemm_kernel(GemmArgs p) {
    constexpr int THREADS = gemm_threads<T>(), TM = 2, TN = T / 64;
    constexpr int PANELS = EPI == kUp ? 2 : 1;
    using TA = typename std::conditional<A_RC, TileRC<T, THREADS>, TileKC<T, THREADS>>::type;
    using TB = typename std::conditional<B_RC, TileRC<T / PANELS, THREADS>, TileKC<T / PANELS, THREADS>>::type;
    constexpr int kBytes = TA::kBytes + PANELS * TB::kBytes;
    static_assert(kBytes * kRing >= THREADS / 64 * 32 * TN * 32 * 4, "the results of 32 rows of every wavefront are staged in the buffers");
    __shared__ __align__(1024) char buf0[kBytes];
    __shared__ __align__(1024) char buf1[kBytes];
    __shared__ __align__(1024) char buf2[kBytes];
    __shared__ __align__(1024) char buf3[kBytes];

    int range;
    const int tile = tile_of_block(p, range);
    const TilePlace at = place_of(p, tile, T, T / PANELS);
    const Job& q = p.job[at.job];

    const int lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64), wm = wave / 2, wn = wave % 2;
    const TA ta(q.a_pitch);
    const TB tb(q.b_pitch);
    const int slices = (int)((q.K + kBK - 1) / kBK);
    const int from = range < 0 ? 0 : (int)((int64_t)slices * range / p.ranges);
    const int here = (range < 0 ? slices : (int)((int64_t)slices * (range + 1) / p.ranges)) - from;
    const uint16_t* base_a = q.a + at.group * q.a_group;
    const uint16_t* base_b = q.b + at.group * q.b_group;
    const uint16_t* base_b2 = q.b2 + at.group * q.b2_group;

    f16v acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][t][r] = 0.0f;

    int seg = 0, left_slices = here;                      // of the next copy
    int64_t k_left;
    Cursor cur_a, cur_b, cur_b2;
    auto enter = [&]() {                                  // the segment's first slice of this range
        const int64_t k0 = (int64_t)from * kBK;
        const uint16_t* a = base_a + q.seg_a[seg];
        const uint16_t* b = (PANELS == 1 && ((q.seg_second >> seg) & 1u) ? base_b2 : base_b) + q.seg_b[seg];
        cur_a = A_RC ? TA::cursor(a, q.a_pitch, q.a_inner8, q.K, at.m0, k0) : TA::cursor(a, q.a_pitch, q.M, q.a_inner8, at.m0, k0);
        cur_b = B_RC ? TB::cursor(b, q.b_pitch, q.b_inner8, q.K, at.n0, k0) : TB::cursor(b, q.b_pitch, q.N, q.b_inner8, at.n0, k0);
        if constexpr (PANELS == 2) cur_b2 = TB::cursor(base_b2, q.b_pitch, q.b_inner8, q.K, at.n0, k0);
        k_left = (A_RC ? q.K : q.a_inner8) - k0;
    };
    enter();
    auto copy = [&](char* lds) {
        ta.copy(lds, 0, cur_a, k_left);
        tb.copy(lds, TA::kBytes, cur_b, k_left);
        if constexpr (PANELS == 2) tb.copy(lds, TA::kBytes + TB::kBytes, cur_b2, k_left);
        cur_a.advance(), cur_b.advance();
        if constexpr (PANELS == 2) cur_b2.advance();
        k_left -= kBK;
        if (--left_slices == 0) {
            if (++seg < q.segments) left_slices = here, enter();
            else cur_a.left = cur_b.left = cur_b2.left = 0, cur_a.step = cur_b.step = cur_b2.step = 0;   // from here on nothing is read
        }
    };
    int part_a[TM], part_b[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) part_a[i] = TA::lane_part(0, wm * (32 * TM) + 32 * i, lane);
#pragma unroll
    for (int t = 0; t < TN; ++t) {
        constexpr int kPer = TN / PANELS;                 // fragments of a panel
        part_b[t] = TB::lane_part(TA::kBytes + t / kPer * TB::kBytes, wn * (T / 2 / PANELS) + 32 * (t % kPer), lane);
    }
    bf16x8 fa[2][TM], fb[2][TN];
    auto fetch = [&](const char* lds, int s) {            // step s of a slice, 0 or 1
        // opaque: addresses stay an array plus one offset (see the top of the file), and are formed here instead of being kept
        // for every step and buffer
#pragma unroll
        for (int t = 0; t < TN; ++t) {
            int part = part_b[t];
            asm volatile("" : "+v"(part));
            fb[s & 1][t] = TB::frag(lds, part, s);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            int part = part_a[i];
            asm volatile("" : "+v"(part));
            fa[s & 1][i] = TA::frag(lds, part, s);
        }
    };
    auto multiply = [&](int s) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int t = 0; t < TN; ++t) acc[i][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[s & 1][t], fa[s & 1][i], acc[i][t], 0, 0, 0);
    };
    const int end = here * q.segments;
    // In front of slice it + 1: this wavefront's copies of it have landed (those of the two slices behind it may be under way)
    // and its fragments of slice `it` are in registers; behind the barrier that holds for all wavefronts, so slice it + 1 can
    // be read and the buffer of slice `it` overwritten.  Copies past the end (windows of no bytes) keep the count the same.
    constexpr int kPerSlice = TA::kCopies + PANELS * TB::kCopies;
    static_assert(kPerSlice == 4 && kRing == 4, "the counts below are of four copies a slice");
    auto barrier = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto slice = [&](char* lds, char* next) {
        fetch(lds, 1);
        multiply(0);
        __builtin_amdgcn_sched_barrier(0);                // fragments of two steps at a time: registers
        __builtin_amdgcn_s_waitcnt(0x0078);               // vmcnt(8) lgkmcnt(0)
        barrier();
        fetch(next, 0);
        multiply(1);
        copy(lds);                                        // behind the products: 4 to 6 % of the products that read RC tiles
        __builtin_amdgcn_sched_barrier(0);
    };
    copy(buf0);
    copy(buf1);
    copy(buf2);
    copy(buf3);
    __builtin_amdgcn_s_waitcnt(0x0f7c);                   // vmcnt(12)
    barrier();
    fetch(buf0, 0);
    for (int it = 0; it < end; it += kRing) {
        slice(buf0, buf1);
        if (it + 1 < end) slice(buf1, buf2);
        if (it + 2 < end) slice(buf2, buf3);
        if (it + 3 < end) slice(buf3, buf0);
    }
    __builtin_amdgcn_s_waitcnt(0x0070);                   // the copies past the end write zeros into LDS

    __syncthreads();                                      // everyone is done with the operands
    constexpr int kPart = THREADS / 64 / kRing, kFloats = 32 * TN * 32;   // wavefronts that stage in one buffer
    char* bufs[kRing] = {buf0, buf1, buf2, buf3};
    float* stage = (float*)bufs[0] + wave % kPart * kFloats;
#pragma unroll
    for (int i = 1; i < kRing; ++i) stage = wave / kPart == i ? (float*)bufs[i] + wave % kPart * kFloats : stage;
    write_tile<EPI, false, T>(acc, stage, p, at, tile, range);
}

// Adds up the ranges of the tiles whose contraction was cut, in order, and does the epilogue's work.
template <Epi EPI, bool SPLIT, int T>
__global__ __launch_bounds__(256) void join_kernel(GemmArgs p) {
    constexpr int PANELS = EPI == kUp ? 2 : 1, kUnits = T / PANELS / 8;
    const TilePlace at = place_of(p, p.whole + blockIdx.x, T, T / PANELS);
    const Job& q = p.job[at.job];
    const int i = blockIdx.y * 256 + threadIdx.x, row = i / kUnits, col = i % kUnits * 8;
    if (at.m0 + row >= q.M || at.n0 + col >= q.epi.n8) return;
    float v[PANELS][8] = {};
    const float* in = p.partial + (int64_t)blockIdx.x * (T * T) + (int64_t)row * T + col;
#pragma unroll 4
    for (int s = 0; s < p.ranges; ++s)
#pragma unroll
        for (int q2 = 0; q2 < PANELS; ++q2) {
            float x[8];
            load8(in + (int64_t)s * p.rest * (T * T) + q2 * (T / PANELS), x);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[q2][e] += x[e];
        }
    emit<EPI, SPLIT>(q.epi, at.group, at.m0 + row, at.n0 + col, v[0], v[PANELS - 1]);
}

}  // namespace ffn
}  // namespace ols
