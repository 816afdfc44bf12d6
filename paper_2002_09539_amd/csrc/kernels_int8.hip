// Matrix products in 8-bit integers with a scale for every token and every channel, and the quantisers.
//
//   s_r = fp32(max |x_r| / 127),  q_rk = x_rk / s_r to the nearest whole number, halves to even,   y_rc = (sum_k q_rk w_ck) s_r t_c
//
// The sums are whole numbers, exact in 32 bits whatever their order (width < 2^17).
#include <algorithm>

#include "element_io.h"
#include "ffn_gemm.h"
#include "ols_internal.h"

namespace ols {

namespace {

typedef int i4 __attribute__((ext_vector_type(4)));

// ---- quantisers -----------------------------------------------------------------------------------------------------------

// A row's scale, and x / scale rounded.  x times the reciprocal can miss the border between two numbers, so the remainder x - q s
// decides, which is exact in fp32: next to a border it has fewer than 24 bits.  Tiny rows are raised to where the reciprocal exists.
struct RowScale {
    float scale, raise, s, inv;
    __device__ RowScale(float top, bool bad) {
        scale = bad ? NAN : (float)((double)top / 127.0);
        raise = scale < 1e-30f ? 0x1p64f : 1.0f;
        s = scale * raise;
        inv = s > 0.0f ? 1.0f / s : 0.0f;                      // NaN > 0 is false: q is 0
    }
    __device__ int q(float x) const {
        const float v = x * raise;
        float q = rintf(v * inv);
        const float r = fmaf(-q, s, v), half = 0.5f * s;
        const bool odd = ((int)q & 1) != 0;
        if (r > half || (r == half && odd)) q += 1.0f;
        else if (r < -half || (r == -half && odd)) q -= 1.0f;
        q = inv == 0.0f ? 0.0f : fminf(fmaxf(q, -127.0f), 127.0f);
        return (int)q;
    }
};

__device__ __forceinline__ unsigned pack4(const RowScale& s, float a, float b, float c, float d) {
    return (unsigned)(s.q(a) & 255) | (unsigned)(s.q(b) & 255) << 8 | (unsigned)(s.q(c) & 255) << 16 | (unsigned)(s.q(d) & 255) << 24;
}

typedef unsigned u2any __attribute__((ext_vector_type(2), aligned(1)));

// x, or act(x) up, of eight columns
template <typename T>
__device__ __forceinline__ void values(const QuantRows& p, const T* x, const T* up, int64_t c, float (&v)[8]) {
    const int left = (int)min((int64_t)8, p.width - c);
    load_upto8(x + c, left, 0.0f, v);
    if (!up) return;
    float u[8];
    load_upto8(up + c, left, 0.0f, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = ffn::act_value<true>(p.act, v[e]) * u[e];
}

// The scale of a row, by all threads of a workgroup.
template <typename T, int THREADS>
__device__ __forceinline__ RowScale row_scale(const QuantRows& p, const T* x, const T* up, float* tops, int* bads) {
    float top = 0.0f;
    bool bad = false;
    for (int64_t c = threadIdx.x * 8; c < p.width; c += THREADS * 8) {
        float v[8];
        values<T>(p, x, up, c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e])), bad |= !(fabsf(v[e]) < INFINITY);
    }
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const unsigned long long any = __ballot(bad);
    __syncthreads();                                           // the places may still be read for the row before
    if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = top, bads[threadIdx.x / 64] = any != 0;
    __syncthreads();
    top = 0.0f, bad = false;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) top = fmaxf(top, tops[w]), bad |= bads[w] != 0;
    return RowScale(top, bad);
}

__device__ __forceinline__ void store_packed(int8_t* q, int64_t left, unsigned lo, unsigned hi) {
    if (left >= 8) {
        *(u2any*)q = u2any{lo, hi};
    } else {
        for (int e = 0; e < left; ++e) q[e] = (int8_t)((e < 4 ? lo >> (8 * e) : hi >> (8 * (e - 4))) & 255);
    }
}

// A workgroup for each row.  Up to NV vectors of eight a lane stay in registers from the search for the largest value to the rounding;
// NV = 0: longer rows are read again.
template <typename T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void quantize_rows_kernel(QuantRows p) {
    __shared__ float tops[THREADS / 64];
    __shared__ int bads[THREADS / 64];
    const int64_t group = blockIdx.x / p.rows, row = blockIdx.x % p.rows;
    const T* x = (const T*)p.x.dev + group * p.x.group + row * p.x.row;
    const T* up = p.up.dev ? (const T*)p.up.dev + group * p.up.group + row * p.up.row : nullptr;
    int8_t* q = p.q + group * p.q_group + row * p.q_row;
    if constexpr (NV == 0) {
        const RowScale s = row_scale<T, THREADS>(p, x, up, tops, bads);
        if (threadIdx.x == 0) p.scale[group * p.scale_group + row] = s.scale;
        for (int64_t c = threadIdx.x * 8; c < p.padded; c += THREADS * 8) {
            float v[8];
            values<T>(p, x, up, c, v);
            store_packed(q + c, p.padded - c, pack4(s, v[0], v[1], v[2], v[3]), pack4(s, v[4], v[5], v[6], v[7]));
        }
    } else {
        float v[NV][8];
#pragma unroll
        for (int j = 0; j < NV; ++j) values<T>(p, x, up, (int64_t)(j * THREADS + threadIdx.x) * 8, v[j]);
        float top = 0.0f;
        bool bad = false;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[j][e])), bad |= !(fabsf(v[j][e]) < INFINITY);
        for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
        const unsigned long long any = __ballot(bad);
        if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = top, bads[threadIdx.x / 64] = any != 0;
        __syncthreads();
        top = 0.0f, bad = false;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) top = fmaxf(top, tops[w]), bad |= bads[w] != 0;
        const RowScale s(top, bad);
        if (threadIdx.x == 0) p.scale[group * p.scale_group + row] = s.scale;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int64_t c = (int64_t)(j * THREADS + threadIdx.x) * 8;
            if (c < p.padded) store_packed(q + c, p.padded - c, pack4(s, v[j][0], v[j][1], v[j][2], v[j][3]), pack4(s, v[j][4], v[j][5], v[j][6], v[j][7]));
        }
    }
}

template <typename T>
void launch_rows_typed(const QuantRows& p, unsigned blocks, hipStream_t stream) {
    const int64_t units = (p.padded + 7) / 8;
    if (units <= 64) quantize_rows_kernel<T, 64, 1><<<blocks, 64, 0, stream>>>(p);
    else if (units <= 256) quantize_rows_kernel<T, 256, 1><<<blocks, 256, 0, stream>>>(p);
    else if (units <= 512) quantize_rows_kernel<T, 256, 2><<<blocks, 256, 0, stream>>>(p);
    else if (units <= 1024) quantize_rows_kernel<T, 512, 2><<<blocks, 512, 0, stream>>>(p);
    else if (units <= 2048) quantize_rows_kernel<T, 1024, 2><<<blocks, 1024, 0, stream>>>(p);
    else quantize_rows_kernel<T, 1024, 0><<<blocks, 1024, 0, stream>>>(p);
}

constexpr int kTile = 64;               // of a weight: indices and channels of a workgroup
constexpr int64_t kWeightRange = 512;   // indices whose largest values a workgroup finds

// The largest value of each column in a range of rows: a lane for each column; -1 where something is not finite.
template <typename T>
__global__ __launch_bounds__(256) void weight_top_kernel(QuantWeight p, float* top) {
    __shared__ float tops[4][64];
    const int64_t c = (int64_t)blockIdx.x * 64 + threadIdx.x % 64, k0 = (int64_t)blockIdx.y * kWeightRange, group = blockIdx.z;
    const T* w = (const T*)p.w.dev + group * p.w.group + c;
    float t = 0.0f;
    bool bad = false;
    if (c < p.out)
        for (int64_t k = k0 + threadIdx.x / 64; k < min(k0 + kWeightRange, p.width); k += 4) {
            const float v = fabsf(load1(w + k * p.w.row));
            t = fmaxf(t, v), bad |= !(v < INFINITY);
        }
    tops[threadIdx.x / 64][threadIdx.x % 64] = bad ? INFINITY : t;
    __syncthreads();
    if (threadIdx.x < 64 && c < p.out)
        top[((int64_t)blockIdx.y * gridDim.z + group) * p.out + c] = fmaxf(fmaxf(tops[0][threadIdx.x], tops[1][threadIdx.x]), fmaxf(tops[2][threadIdx.x], tops[3][threadIdx.x]));
}

// Rounds and transposes a tile.
template <typename T>
__global__ __launch_bounds__(256) void weight_kernel(QuantWeight p, const float* top, int ranges) {
    __shared__ int8_t tile[kTile][kTile + 4];
    const int64_t c = (int64_t)blockIdx.x * 64 + threadIdx.x % 64, k0 = (int64_t)blockIdx.y * kTile, group = blockIdx.z;
    float t = 0.0f;
    if (c < p.out)
        for (int r = 0; r < ranges; ++r) t = fmaxf(t, top[((int64_t)r * gridDim.z + group) * p.out + c]);
    const RowScale s(t, !(t < INFINITY));
    if (c < p.out) {
        if (blockIdx.y == 0 && threadIdx.x < 64) p.scale[group * p.scale_group + c] = s.scale;
        const T* w = (const T*)p.w.dev + group * p.w.group + c;
        for (int k = threadIdx.x / 64; k < kTile; k += 4) tile[threadIdx.x % 64][k] = k0 + k < p.width ? (int8_t)s.q(load1(w + (k0 + k) * p.w.row)) : 0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kTile * kTile; i += 256) {
        const int64_t ch = (int64_t)blockIdx.x * 64 + i / kTile, k = k0 + i % kTile;
        if (ch < p.out && k < p.width) p.q[group * p.q_group + ch * p.q_row + k] = tile[i / kTile][i % kTile];
    }
}

// ---- products -------------------------------------------------------------------------------------------------------------

struct Product {
    int groups, out_f32;
    int64_t rows, width, out;
    const int8_t *x, *w;
    int64_t x_row, x_group, w_row, w_group;
    const float *x_scale, *w_scale;
    int64_t x_scale_group, w_scale_group;
    void* y;
    int64_t y_row, y_group;
    QuantRows quant;                     // what few rows are quantised from, by the workgroups that multiply them
    // Large products: tiles [0, whole) take a workgroup each, the contractions of the `rest` behind them are cut into `ranges`, whose
    // sums go to `partial` ([range][tile][rows][channels]).
    int tiles_m, tiles_n, whole, rest, ranges;
    int* partial;
};

typedef unsigned u4bytes __attribute__((ext_vector_type(4), aligned(1)));

// sixteen bytes of a row from index k, zeros from `width` on
__device__ __forceinline__ i4 load_16(const int8_t* row, int64_t k, int64_t width, bool there) {
    if (!there || k >= width) return i4{0, 0, 0, 0};
    if (k + 16 <= width) return __builtin_bit_cast(i4, (u4)*(const u4bytes*)(row + k));
    unsigned v[4] = {};
    for (int e = 0; k + e < width; ++e) v[e / 4] |= (unsigned)(uint8_t)row[k + e] << (8 * (e % 4));
    return i4{(int)v[0], (int)v[1], (int)v[2], (int)v[3]};
}

template <int N>
__device__ __forceinline__ void store_scaled(const Product& p, int64_t group, int64_t r, int64_t c, const float (&v)[N]) {   // columns c .. of row r
    const int64_t at = group * p.y_group + r * p.y_row + c;
    const int left = (int)min((int64_t)N, p.out - c);
    if constexpr (N == 8) {
        if (p.out_f32) store_upto8((float*)p.y + at, left, v);
        else store_upto8((uint16_t*)p.y + at, left, v);
    } else {
        for (int e = 0; e < N; ++e) {
            if (e >= left) continue;
            if (p.out_f32) store1((float*)p.y + at + e, v[e]);
            else store1((uint16_t*)p.y + at + e, v[e]);
        }
    }
}

// Few rows: a workgroup for 16 channels and 16 R rows, whose wavefronts share the contraction, 64 indices at a time in turn; up to kAhead
// of its turns' weights are under way before anything is waited for.  FUSED: the workgroup quantises the rows itself, into LDS.
constexpr int kAhead = 8;
template <typename TX, int R, int WAVES, bool FUSED>
__global__ __launch_bounds__(WAVES * 64) void few_kernel(Product p) {
    extern __shared__ __align__(16) char lds[];
    __shared__ float scales[16 * R];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t group = blockIdx.z, c0 = (int64_t)blockIdx.x * 16, r0 = (int64_t)blockIdx.y * (16 * R);
    const int64_t c = min(c0 + lane % 16, p.out - 1);
    const int8_t* w = p.w + group * p.w_group + c * p.w_row;
    const int turns = (int)((p.width + 63) / 64);
    i4 a[kAhead];
    auto request = [&](int first) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int64_t k = ((int64_t)first + j * WAVES + wave) * 64 + 16 * (lane / 16);
            a[j] = load_16(w, k, p.width, true);
        }
    };
    request(0);
    const int pitch = (int)((p.width + 63) / 64 * 64) + 16;        // of a row in LDS: rows on different banks
    if constexpr (FUSED) {
        const int here = (int)min((int64_t)16 * R, p.rows - r0);
        __shared__ float tops[WAVES];
        __shared__ int bads[WAVES];
        for (int r = 0; r < here; ++r) {
            const TX* x = (const TX*)p.quant.x.dev + group * p.quant.x.group + (r0 + r) * p.quant.x.row;
            const TX* up = p.quant.up.dev ? (const TX*)p.quant.up.dev + group * p.quant.up.group + (r0 + r) * p.quant.up.row : nullptr;
            const RowScale s = row_scale<TX, WAVES * 64>(p.quant, x, up, tops, bads);
            if (threadIdx.x == 0) scales[r] = s.scale;
            for (int64_t k = threadIdx.x * 8; k < pitch - 16; k += WAVES * 64 * 8) {
                float v[8];
                values<TX>(p.quant, x, up, k, v);
                *(u2any*)(lds + r * pitch + k) = u2any{pack4(s, v[0], v[1], v[2], v[3]), pack4(s, v[4], v[5], v[6], v[7])};
            }
        }
        __syncthreads();
    }
    i4 acc[R] = {};
    const int8_t* x = p.x + group * p.x_group;
    for (int first = 0; first < turns; first += kAhead * WAVES) {
        if (first) request(first);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int turn = first + j * WAVES + wave;
            if (turn >= turns) continue;
            const int64_t k = (int64_t)turn * 64 + 16 * (lane / 16);
#pragma unroll
            for (int i = 0; i < R; ++i) {
                // rows that do not exist are the last one again: what comes of them is not written
                const int64_t r = min(r0 + 16 * i + lane % 16, p.rows - 1);
                i4 b;
                if constexpr (FUSED) b = *(const i4*)(lds + (int)(r - r0) * pitch + k);
                else b = load_16(x + r * p.x_row, k, p.width, true);
                acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[j], b, acc[i], 0, 0, 0);
            }
        }
    }
    i4* sums = (i4*)lds;                                           // [wave][R][lane]
    __syncthreads();
#pragma unroll
    for (int i = 0; i < R; ++i) sums[(wave * R + i) * 64 + lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < R; i += WAVES) {
        i4 sum = {};
#pragma unroll
        for (int k = 0; k < WAVES; ++k) sum += sums[(k * R + i) * 64 + lane];
        const int64_t r = r0 + 16 * i + lane % 16, o = c0 + 4 * (lane / 16);
        if (r >= p.rows || o >= p.out) continue;
        const float s = FUSED ? scales[r - r0] : p.x_scale[group * p.x_scale_group + r];
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = o + e < p.out ? (float)sum[e] * s * p.w_scale[group * p.w_scale_group + o + e] : 0.0f;
        store_scaled<4>(p, group, r, o, v);
    }
}

// ---- many rows ------------------------------------------------------------------------------------------------------------

constexpr int kSlice = 64;               // indices of a slice: as many bytes as the bf16 tiles' 32
using ffn::Cursor;
using ffn::uniform;
typedef int i16v __attribute__((ext_vector_type(16)));

struct Place {
    int64_t group, m0, n0;
};
__device__ __forceinline__ Place place_of(const Product& p, int tile, int t) {
    const int per_group = p.tiles_m * p.tiles_n;
    Place at;
    at.group = tile / per_group;
    tile %= per_group;
    constexpr int kBand = 8;             // bands of eight rows of tiles, down each column of the band: what runs together shares operands
    const int band = tile / (kBand * p.tiles_n), rows = min(kBand, p.tiles_m - band * kBand), in_band = tile - band * kBand * p.tiles_n;
    at.m0 = (int64_t)(band * kBand + in_band % rows) * t, at.n0 = (int64_t)(in_band / rows) * t;
    return at;
}
// The hardware deals workgroup b to XCD b % 8: each takes a contiguous range of tiles, whose operands its L2 keeps.
__device__ __forceinline__ int tile_of_block(const Product& p, int& range) {
    range = -1;
    if ((int)blockIdx.x < p.whole) {
        const int per = (p.whole + ffn::kXcds - 1) / ffn::kXcds, full = p.whole % ffn::kXcds == 0 ? ffn::kXcds : p.whole % ffn::kXcds, xcd = blockIdx.x % ffn::kXcds;
        return xcd * per - max(0, xcd - full) + blockIdx.x / ffn::kXcds;
    }
    const int u = blockIdx.x - p.whole;
    range = u / p.rest;
    return p.whole + u % p.rest;
}

// T x T tiles: 256 with eight wavefronts of 64 x 128, 128 with four of 64 x 64.  The tiles, their ring in LDS and the order of copies,
// barriers and reads are those of the bf16 products (ffn_gemm.h): sixteen bytes of a lane are sixteen indices here instead of eight.
template <int T>
__global__ __launch_bounds__(ffn::gemm_threads<T>(), 2) void tile_kernel(Product p) {
    constexpr int THREADS = ffn::gemm_threads<T>(), TM = 2, TN = T / 64;
    using Tile = ffn::TileKC<T, THREADS>;
    constexpr int kBytes = 2 * Tile::kBytes;
    __shared__ __align__(1024) char buf0[kBytes];
    __shared__ __align__(1024) char buf1[kBytes];
    __shared__ __align__(1024) char buf2[kBytes];
    __shared__ __align__(1024) char buf3[kBytes];

    int range;
    const int tile = tile_of_block(p, range);
    const Place at = place_of(p, tile, T);
    const int lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64), wm = wave / 2, wn = wave % 2;
    const int64_t k2 = (p.width + 15) / 16 * 8;               // a row's pairs of bytes, up to whole chunks (x holds zeros there)
    const Tile ta(p.x_row / 2), tb(p.w_row / 2);
    const int slices = (int)((p.width + kSlice - 1) / kSlice);
    const int from = range < 0 ? 0 : (int)((int64_t)slices * range / p.ranges);
    const int end = (range < 0 ? slices : (int)((int64_t)slices * (range + 1) / p.ranges)) - from;

    i16v acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][t][r] = 0;

    const int64_t k0 = (int64_t)from * (kSlice / 2);
    Cursor cur_a = Tile::cursor((const uint16_t*)(p.x + at.group * p.x_group), p.x_row / 2, p.rows, k2, at.m0, k0);
    Cursor cur_b = Tile::cursor((const uint16_t*)(p.w + at.group * p.w_group), p.w_row / 2, p.out, k2, at.n0, k0);
    int64_t k_left = k2 - k0;
    int left_slices = end;                                    // of the next copy
    auto copy = [&](char* lds) {
        ta.copy(lds, 0, cur_a, k_left);
        tb.copy(lds, Tile::kBytes, cur_b, k_left);
        cur_a.advance(), cur_b.advance();
        k_left -= kSlice / 2;
        if (--left_slices == 0) cur_a.left = cur_b.left = 0, cur_a.step = cur_b.step = 0;   // from here on nothing is read
    };
    int part_a[TM], part_b[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) part_a[i] = Tile::lane_part(0, wm * (32 * TM) + 32 * i, lane);
#pragma unroll
    for (int t = 0; t < TN; ++t) part_b[t] = Tile::lane_part(Tile::kBytes, wn * (T / 2) + 32 * t, lane);
    i4 fa[2][TM], fb[2][TN];
    auto fetch = [&](const char* lds, int s) {                // step s of a slice, 0 or 1
#pragma unroll
        for (int t = 0; t < TN; ++t) {
            int part = part_b[t];
            asm volatile("" : "+v"(part));
            fb[s & 1][t] = __builtin_bit_cast(i4, Tile::frag(lds, part, s));
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            int part = part_a[i];
            asm volatile("" : "+v"(part));
            fa[s & 1][i] = __builtin_bit_cast(i4, Tile::frag(lds, part, s));
        }
    };
    auto multiply = [&](int s) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int t = 0; t < TN; ++t) acc[i][t] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[s & 1][t], fa[s & 1][i], acc[i][t], 0, 0, 0);
    };
    // Counts as in ffn_gemm.h: four copies a slice and wavefront; copies past the end (windows of no bytes) keep the count the same.
    static_assert(2 * Tile::kCopies == 4 && ffn::kRing == 4, "the counts below are of four copies a slice");
    auto barrier = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto slice = [&](char* lds, char* next) {
        fetch(lds, 1);
        multiply(0);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0078);                   // vmcnt(8) lgkmcnt(0)
        barrier();
        fetch(next, 0);
        multiply(1);
        copy(lds);
        __builtin_amdgcn_sched_barrier(0);
    };
    copy(buf0);
    copy(buf1);
    copy(buf2);
    copy(buf3);
    __builtin_amdgcn_s_waitcnt(0x0f7c);                       // vmcnt(12)
    barrier();
    fetch(buf0, 0);
    for (int it = 0; it < end; it += ffn::kRing) {
        slice(buf0, buf1);
        if (it + 1 < end) slice(buf1, buf2);
        if (it + 2 < end) slice(buf2, buf3);
        if (it + 3 < end) slice(buf3, buf0);
    }
    __builtin_amdgcn_s_waitcnt(0x0070);                       // the copies past the end write zeros into LDS

    __syncthreads();                                          // everyone is done with the operands
    constexpr int kCols = TN * 32, kUnits = kCols / 8, kRows = 64 / kUnits;
    constexpr int kPart = THREADS / 64 / ffn::kRing, kInts = 32 * kCols;   // wavefronts that stage in one buffer
    static_assert(kBytes >= kPart * kInts * 4, "the results of 32 rows of every wavefront are staged in the buffers");
    char* bufs[ffn::kRing] = {buf0, buf1, buf2, buf3};
    int* stage = (int*)bufs[0] + wave % kPart * kInts;
#pragma unroll
    for (int i = 1; i < ffn::kRing; ++i) stage = wave / kPart == i ? (int*)bufs[i] + wave % kPart * kInts : stage;
    const int lane_row = lane % 32, out_row = lane / kUnits, unit = lane % kUnits, col = wn * (T / 2) + 8 * unit;
    float cs[8];
    if (range < 0) load_upto8(p.w_scale + at.group * p.w_scale_group + at.n0 + col, (int)max((int64_t)0, min((int64_t)8, p.out - at.n0 - col)), 0.0f, cs);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int chunk = 8 * t + 2 * g + lane / 32;
                *(i4*)(stage + lane_row * kCols + 4 * (chunk ^ (lane_row & 15))) = i4{acc[i][t][4 * g], acc[i][t][4 * g + 1], acc[i][t][4 * g + 2], acc[i][t][4 * g + 3]};
            }
        in_wave_order();                                      // written and read by one wavefront: LDS keeps its order
#pragma unroll 1
        for (int r0 = 0; r0 < 32; r0 += kRows) {
            const int r = r0 + out_row, row = wm * (32 * TM) + 32 * i + r;
            const i4 lo = *(const i4*)(stage + r * kCols + 4 * ((2 * unit) ^ (r & 15))), hi = *(const i4*)(stage + r * kCols + 4 * ((2 * unit + 1) ^ (r & 15)));
            if (range >= 0) {
                int* out = p.partial + ((int64_t)range * p.rest + (tile - p.whole)) * (T * T) + row * T + col;
                *(i4*)out = lo;
                *(i4*)(out + 4) = hi;
            } else if (at.m0 + row < p.rows && at.n0 + col < p.out) {
                const float s = p.x_scale[at.group * p.x_scale_group + at.m0 + row];
                float v[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (float)lo[e] * s * cs[e], v[4 + e] = (float)hi[e] * s * cs[4 + e];
                store_scaled<8>(p, at.group, at.m0 + row, at.n0 + col, v);
            }
        }
        in_wave_order();
    }
}

// Adds up the ranges of the tiles whose contraction was cut.
template <int T>
__global__ __launch_bounds__(256) void join_kernel(Product p) {
    constexpr int kUnits = T / 8;
    const Place at = place_of(p, p.whole + blockIdx.x, T);
    const int i = blockIdx.y * 256 + threadIdx.x, row = i / kUnits, col = i % kUnits * 8;
    if (at.m0 + row >= p.rows || at.n0 + col >= p.out) return;
    i4 lo = {}, hi = {};
    const int* in = p.partial + (int64_t)blockIdx.x * (T * T) + row * T + col;
#pragma unroll 4
    for (int s = 0; s < p.ranges; ++s) {
        lo += *(const i4*)(in + (int64_t)s * p.rest * (T * T));
        hi += *(const i4*)(in + (int64_t)s * p.rest * (T * T) + 4);
    }
    const float s = p.x_scale[at.group * p.x_scale_group + at.m0 + row];
    float cs[8], v[8];
    load_upto8(p.w_scale + at.group * p.w_scale_group + at.n0 + col, (int)min((int64_t)8, p.out - at.n0 - col), 0.0f, cs);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)lo[e] * s * cs[e], v[4 + e] = (float)hi[e] * s * cs[4 + e];
    store_scaled<8>(p, at.group, at.m0 + row, at.n0 + col, v);
}

// Rows of int8 laid out for the tiles: on 16 bytes, zeros behind `width`.
struct Pack {
    const int8_t* src;
    int64_t row, group, rows, width, pitch;
    int8_t* dst;
};
__global__ __launch_bounds__(256) void pack_int8_kernel(Pack p) {
    const int64_t units = p.pitch / 16, total = p.rows * units;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / units, k = i % units * 16;
        *(i4*)(p.dst + (blockIdx.y * p.rows + r) * p.pitch + k) = load_16(p.src + blockIdx.y * p.group + r * p.row, k, p.width, true);
    }
}

int64_t up16(int64_t v) { return (v + 15) / 16 * 16; }
int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }
int x_groups(const ols_int8& f) { return f.x.group == 0 && (!f.up.dev || f.up.group == 0) ? 1 : f.groups; }    // rows that the workers share: once
constexpr int64_t kMostBlocks = 1 << 21;   // of 1024 threads: a launch has fewer than 2^32

struct Plan {
    int tile;                             // 0: few rows
    int R, waves;                         // few rows: rows of a workgroup / 16, its wavefronts
    bool fused, lay_x, lay_w;             // rows quantised where they are multiplied; operands laid out first
    int tiles_m, tiles_n, whole, rest, ranges;
    int64_t scale_at, w_at, partial_at, ws_bytes;
};

bool lies_well(const ols_matrix& m) { return m.row % 16 == 0 && m.row <= (1 << 22) && m.group % 16 == 0 && ((uintptr_t)m.dev & 15) == 0; }

constexpr int kFewRows = 64;              // at most: weights go straight into registers
constexpr int kCus = 256;

Plan plan_of(const ols_int8& f) {
    Plan p = {};
    const int64_t turns = (f.width + 63) / 64;
    p.ranges = 1;
    if (f.rows <= kFewRows) {
        const int64_t channels = (f.out + 15) / 16 * f.groups;
        p.R = f.rows <= 16 ? 1 : 2;
        const int64_t blocks = channels * ((f.rows + 16 * p.R - 1) / (16 * p.R));
        p.waves = blocks <= 2 * kCus && turns >= 32 ? 16 : turns >= 8 ? 8 : 4;
        p.fused = f.dtype != OLS_I8 && f.rows <= 16 && f.rows * (turns * 64 + 16) <= 32768 && f.rows * f.width * blocks <= (1 << 23);
    } else {
        int64_t tiles = (f.rows + 255) / 256 * ((f.out + 255) / 256) * f.groups;
        p.tile = tiles >= 192 ? 256 : 128;
        p.tiles_m = (int)((f.rows + p.tile - 1) / p.tile), p.tiles_n = (int)((f.out + p.tile - 1) / p.tile);
        tiles = (int64_t)p.tiles_m * p.tiles_n * f.groups;
        p.whole = (int)tiles;
        if (tiles <= kCus) {
            p.ranges = (int)std::max<int64_t>(1, std::min<int64_t>(2 * kCus / tiles, turns / 4));
            if (p.ranges > 1) p.whole = 0, p.rest = (int)tiles;
        }
        p.lay_w = !lies_well(f.w);
    }
    p.lay_x = f.dtype != OLS_I8 ? !p.fused : p.tile != 0 && (!lies_well(f.x) || f.width % 16 != 0);
    int64_t at = p.lay_x ? up256(x_groups(f) * f.rows * up16(f.width)) : 0;
    p.scale_at = at;
    at += p.lay_x ? up256(x_groups(f) * f.rows * 4) : 0;
    p.w_at = at;
    at += p.lay_w ? up256((f.w.group == 0 ? 1 : f.groups) * f.out * up16(f.width)) : 0;
    p.partial_at = at;
    at += p.rest ? (int64_t)p.ranges * p.rest * p.tile * p.tile * 4 : 0;
    p.ws_bytes = at;
    return p;
}

template <typename TX, int R, int WAVES, bool FUSED>
void launch_few_sized(const Product& p, hipStream_t stream) {
    const size_t sums = (size_t)WAVES * R * 1024, rows = FUSED ? (size_t)p.rows * ((p.width + 63) / 64 * 64 + 16) : 0;
    const dim3 grid((unsigned)((p.out + 15) / 16), (unsigned)((p.rows + 16 * R - 1) / (16 * R)), p.groups);
    few_kernel<TX, R, WAVES, FUSED><<<grid, WAVES * 64, std::max(sums, rows), stream>>>(p);
}
template <typename TX, bool FUSED>
void launch_few(const Product& p, const Plan& plan, hipStream_t stream) {
    if constexpr (FUSED) {                // at most 16 rows
        if (plan.waves == 16) launch_few_sized<TX, 1, 16, true>(p, stream);
        else if (plan.waves == 8) launch_few_sized<TX, 1, 8, true>(p, stream);
        else launch_few_sized<TX, 1, 4, true>(p, stream);
    } else if (plan.R == 1) {
        if (plan.waves == 16) launch_few_sized<TX, 1, 16, false>(p, stream);
        else if (plan.waves == 8) launch_few_sized<TX, 1, 8, false>(p, stream);
        else launch_few_sized<TX, 1, 4, false>(p, stream);
    } else {
        if (plan.waves == 16) launch_few_sized<TX, 2, 16, false>(p, stream);
        else if (plan.waves == 8) launch_few_sized<TX, 2, 8, false>(p, stream);
        else launch_few_sized<TX, 2, 4, false>(p, stream);
    }
}

hipError_t launch_pack(const Pack& p, int groups, hipStream_t stream) {
    const int64_t units = p.rows * (p.pitch / 16);
    pack_int8_kernel<<<dim3((unsigned)std::min<int64_t>((units + 255) / 256, (1 << 23) / groups), groups), 256, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_rows(const QuantRows& p, hipStream_t stream) {
    if (p.rows == 0) return hipSuccess;
    const int64_t each = std::max<int64_t>(1, kMostBlocks / p.groups);
    for (int64_t first = 0; first < p.rows; first += each) {
        QuantRows q = p;
        const int64_t bytes = p.dtype == OLS_F32 ? 4 : 2;
        q.rows = std::min(each, p.rows - first);
        q.x.dev = (char*)p.x.dev + first * p.x.row * bytes;
        if (p.up.dev) q.up.dev = (char*)p.up.dev + first * p.up.row * bytes;
        q.q = p.q + first * p.q_row, q.scale = p.scale + first;
        const unsigned blocks = (unsigned)(q.rows * q.groups);
        if (p.dtype == OLS_F32) launch_rows_typed<float>(q, blocks, stream);
        else launch_rows_typed<uint16_t>(q, blocks, stream);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

int64_t quantize_weight_workspace_bytes(int groups, int64_t width, int64_t out) { return (width + kWeightRange - 1) / kWeightRange * groups * out * 4; }

hipError_t launch_quantize_weight(const QuantWeight& p, void* ws, hipStream_t stream) {
    const int ranges = (int)((p.width + kWeightRange - 1) / kWeightRange);
    float* top = (float*)ws;
    const unsigned cols = (unsigned)((p.out + 63) / 64);
    const dim3 first(cols, ranges, p.groups), second(cols, (unsigned)((p.width + kTile - 1) / kTile), p.groups);
    if (p.dtype == OLS_F32) weight_top_kernel<float><<<first, 256, 0, stream>>>(p, top);
    else weight_top_kernel<uint16_t><<<first, 256, 0, stream>>>(p, top);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (p.dtype == OLS_F32) weight_kernel<float><<<second, 256, 0, stream>>>(p, top, ranges);
    else weight_kernel<uint16_t><<<second, 256, 0, stream>>>(p, top, ranges);
    return hipGetLastError();
}

int64_t int8_workspace_bytes(const ols_int8& f) { return f.rows ? plan_of(f).ws_bytes : 0; }

hipError_t launch_int8(const ols_int8& f, hipStream_t stream) {
    const Plan plan = plan_of(f);
    char* ws = (char*)f.ws;
    Product p = {};
    p.groups = f.groups, p.out_f32 = f.out_dtype == OLS_F32, p.rows = f.rows, p.width = f.width, p.out = f.out;
    p.w = (const int8_t*)f.w.dev, p.w_row = f.w.row, p.w_group = f.w.group, p.w_scale = f.w_scale, p.w_scale_group = f.w_scale_group;
    p.y = f.y.dev, p.y_row = f.y.row, p.y_group = f.y.group;
    p.tiles_m = plan.tiles_m, p.tiles_n = plan.tiles_n, p.whole = plan.whole, p.rest = plan.rest, p.ranges = plan.ranges, p.partial = (int*)(ws + plan.partial_at);
    QuantRows& q = p.quant;
    q.groups = x_groups(f), q.dtype = f.dtype, q.act = f.act, q.rows = f.rows, q.width = f.width, q.x = f.x, q.up = f.up;
    q.q = (int8_t*)ws, q.q_row = up16(f.width), q.q_group = f.rows * q.q_row, q.padded = q.q_row, q.scale = (float*)(ws + plan.scale_at), q.scale_group = f.rows;
    hipError_t e = hipSuccess;
    if (plan.lay_x) {
        if (f.dtype == OLS_I8) {
            e = launch_pack({(const int8_t*)f.x.dev, f.x.row, f.x.group, f.rows, f.width, q.q_row, q.q}, q.groups, stream);
        } else {
            e = launch_quantize_rows(q, stream);
            p.x_scale = q.scale, p.x_scale_group = q.groups == 1 ? 0 : f.rows;
        }
        p.x = q.q, p.x_row = q.q_row, p.x_group = q.groups == 1 ? 0 : q.q_group;
    } else {
        p.x = (const int8_t*)f.x.dev, p.x_row = f.x.row, p.x_group = f.x.group;
    }
    if (f.dtype == OLS_I8) p.x_scale = f.x_scale, p.x_scale_group = f.x_scale_group;
    if (e == hipSuccess && plan.lay_w) {
        const int groups = f.w.group == 0 ? 1 : f.groups;
        const int64_t pitch = up16(f.width);
        int8_t* w = (int8_t*)(ws + plan.w_at);
        e = launch_pack({p.w, p.w_row, p.w_group, f.out, f.width, pitch, w}, groups, stream);
        p.w = w, p.w_row = pitch, p.w_group = groups == 1 ? 0 : f.out * pitch;
    }
    if (e != hipSuccess) return e;
    if (!plan.tile) {
        if (plan.fused) {
            if (f.dtype == OLS_F32) launch_few<float, true>(p, plan, stream);
            else launch_few<uint16_t, true>(p, plan, stream);
        } else {
            launch_few<uint16_t, false>(p, plan, stream);
        }
        return hipGetLastError();
    }
    const unsigned blocks = (unsigned)(plan.whole + plan.rest * plan.ranges);
    if (plan.tile == 256) tile_kernel<256><<<blocks, 512, 0, stream>>>(p);
    else tile_kernel<128><<<blocks, 256, 0, stream>>>(p);
    e = hipGetLastError();
    if (e != hipSuccess || !plan.rest) return e;
    const dim3 grid(plan.rest, plan.tile * plan.tile / 8 / 256);
    if (plan.tile == 256) join_kernel<256><<<grid, 256, 0, stream>>>(p);
    else join_kernel<128><<<grid, 256, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace ols
