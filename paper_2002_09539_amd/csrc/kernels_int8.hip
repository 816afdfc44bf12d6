// Matrix products in 8-bit integers with a scale for every token and every channel, and the quantisers.
//
//   s_r = fp32(max |x_r| / 127),  q_rk = x_rk / s_r to the nearest whole number, halves to even,   y_rc = (sum_k q_rk w_ck) s_r t_c
//
// The sums are whole numbers, exact in 32 bits whatever their order (width < 2^17); the two scales are applied to them in fp32, and the
// result is rounded once.
//
// Few rows are bound by the weights' bytes: they go from memory straight into the registers of the matrix instruction (a row of 2048 to
// 32 000, 65 MB: 15.4 us, 4.3 TB/s).  Many rows are bound by the matrix pipes: both operands go through tiles in LDS (8192 rows, 4096 to
// 4096: 138 to 167 us as the clock allows, 1650 to 1990 TOP/s, where a library's product of 8192^3 reaches 2046).  Between them, some
// dozens of tiles, a launch is a chain of waits.
#include <algorithm>

#include "element_io.h"
#include "ffn_gemm.h"
#include "ols_internal.h"

namespace ols {

namespace {

typedef int i4 __attribute__((ext_vector_type(4)));
using ffn::uniform;

// ---- quantisers -----------------------------------------------------------------------------------------------------------

// A row's scale, and x / scale rounded.  x times the reciprocal can miss the border between two numbers, so the remainder x - q s
// decides, which is exact in fp32: next to a border it has fewer than 24 bits.  Eight values whose remainders all stay clear of half a
// step need no more than that; tiny rows are raised to where the reciprocal exists.
__device__ __forceinline__ unsigned size_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }     // in order of size, then infinities, then NaN
struct RowScale {
    float scale, raise, s, inv, clear;
    __device__ RowScale(unsigned top) {        // size_bits of the row's largest value
        scale = top >= 0x7f800000u ? NAN : (float)((double)__uint_as_float(top) / 127.0);
        raise = scale < 1e-30f ? 0x1p64f : 1.0f;
        s = scale * raise;
        inv = s > 0.0f ? 1.0f / s : 0.0f;                      // NaN > 0 is false: q is 0
        clear = raise == 1.0f && s > 0.0f ? 0.5f * s * (1.0f - 0x1p-16f) : 0.0f;
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
    __device__ int mostly(float x) const {     // q(x), most of the time by a look at the remainder
        const float q0 = rintf(x * inv);
        return fabsf(fmaf(-q0, s, x)) < clear ? (int)q0 : q(x);
    }
};

__device__ __forceinline__ unsigned pack4(const RowScale& s, float a, float b, float c, float d) {
    return (unsigned)(s.q(a) & 255) | (unsigned)(s.q(b) & 255) << 8 | (unsigned)(s.q(c) & 255) << 16 | (unsigned)(s.q(d) & 255) << 24;
}
typedef unsigned u2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u2 pack8(const RowScale& s, const float (&v)[8]) {
    float q[8], far = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = rintf(v[e] * s.inv), far = fmaxf(far, fabsf(fmaf(-q[e], s.s, v[e])));
    if (!(far < s.clear)) return u2{pack4(s, v[0], v[1], v[2], v[3]), pack4(s, v[4], v[5], v[6], v[7])};
    u2 w = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e / 4] = __builtin_amdgcn_cvt_pk_u8_f32(q[e] + 128.0f, e % 4, w[e / 4]);
    return w ^ 0x80808080u;
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

template <int THREADS>
__device__ __forceinline__ unsigned largest(unsigned top, unsigned* tops) {      // of all threads of a workgroup
    for (int o = 32; o; o >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, o));
    if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) top = max(top, tops[w]);
    return top;
}
// The scale of a row, by all threads of a workgroup.
template <typename T, int THREADS>
__device__ __forceinline__ RowScale row_scale(const QuantRows& p, const T* x, const T* up, unsigned* tops) {
    unsigned top = 0;
    for (int64_t c = threadIdx.x * 8; c < p.width; c += THREADS * 8) {
        float v[8];
        values<T>(p, x, up, c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, size_bits(v[e]));
    }
    return RowScale(largest<THREADS>(top, tops));
}

__device__ __forceinline__ void store_packed(int8_t* q, int64_t left, u2 w) {
    if (left >= 8) {
        *(u2any*)q = w;
    } else {
        for (int e = 0; e < left; ++e) q[e] = (int8_t)(w[e / 4] >> (8 * (e % 4)) & 255);
    }
}

// A workgroup for each row.  Up to NV vectors of eight a lane stay in registers from the search for the largest value to the rounding;
// NV = 0: longer rows are read again.  Bound by bytes: 8192 rows of 4096 bf16 25.5 us, 3.9 TB/s.
template <typename T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void quantize_rows_kernel(QuantRows p) {
    __shared__ unsigned tops[THREADS / 64];
    const int64_t group = blockIdx.x / p.rows, row = blockIdx.x % p.rows;
    const T* x = (const T*)p.x.dev + group * p.x.group + row * p.x.row;
    const T* up = p.up.dev ? (const T*)p.up.dev + group * p.up.group + row * p.up.row : nullptr;
    int8_t* q = p.q + group * p.q_group + row * p.q_row;
    if constexpr (NV == 0) {
        const RowScale s = row_scale<T, THREADS>(p, x, up, tops);
        if (threadIdx.x == 0) p.scale[group * p.scale_group + row] = s.scale;
        for (int64_t c = threadIdx.x * 8; c < p.padded; c += THREADS * 8) {
            float v[8];
            values<T>(p, x, up, c, v);
            store_packed(q + c, p.padded - c, pack8(s, v));
        }
    } else {
        float v[NV][8];
#pragma unroll
        for (int j = 0; j < NV; ++j) values<T>(p, x, up, (int64_t)(j * THREADS + threadIdx.x) * 8, v[j]);
        unsigned top = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, size_bits(v[j][e]));
        const RowScale s(largest<THREADS>(top, tops));
        if (threadIdx.x == 0) p.scale[group * p.scale_group + row] = s.scale;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int64_t c = (int64_t)(j * THREADS + threadIdx.x) * 8;
            if (c < p.padded) store_packed(q + c, p.padded - c, pack8(s, v[j]));
        }
    }
}

// Few rows are a chain of waits, which many lanes shorten (64 rows of 5632 bf16: 5.3 us in 1024 lanes, 6.8 in 256); of many, narrow workgroups run
// beside each other, and lanes that hold nothing cost (19 315 rows of 4400: 115 us in 1024 lanes, 60 in 256; 8192 of 1000: 14.1 in 256, 11.1 in 64).
// They meet between 512 and 1024 rows (512 of 5632: 6.9 and 7.3; 1024: 10.3 and 8.7).
template <typename T, int THREADS, int NV>
void launch_rows_sized(const QuantRows& p, unsigned blocks, hipStream_t stream) {
    quantize_rows_kernel<T, THREADS, NV><<<blocks, THREADS, 0, stream>>>(p);
}
template <typename T>
void launch_rows_typed(const QuantRows& p, unsigned blocks, hipStream_t stream) {
    const int64_t units = (p.padded + 7) / 8;
    const bool many = blocks >= 1024;
    if (units <= 64) launch_rows_sized<T, 64, 1>(p, blocks, stream);
    else if (many && units <= 128) launch_rows_sized<T, 64, 2>(p, blocks, stream);
    else if (many && units <= 256) launch_rows_sized<T, 128, 2>(p, blocks, stream);
    else if (many && units <= 384) launch_rows_sized<T, 128, 3>(p, blocks, stream);
    else if (units <= 256) launch_rows_sized<T, 256, 1>(p, blocks, stream);
    else if (units <= 512) launch_rows_sized<T, 256, 2>(p, blocks, stream);
    else if (many && units <= 768) launch_rows_sized<T, 256, 3>(p, blocks, stream);
    else if (many && units <= 1024) launch_rows_sized<T, 256, 4>(p, blocks, stream);
    else if (many && units <= 2048) launch_rows_sized<T, 512, 4>(p, blocks, stream);
    else if (units <= 1024) launch_rows_sized<T, 1024, 1>(p, blocks, stream);
    else if (units <= 2048) launch_rows_sized<T, 1024, 2>(p, blocks, stream);
    else launch_rows_sized<T, 1024, 0>(p, blocks, stream);
}

constexpr int kTile = 64;               // of a weight: indices and channels of a workgroup
constexpr int64_t kWeightRange = 256;   // indices whose largest values a workgroup finds

// Both passes over a weight read eight channels a lane, eight rows a wavefront (a channel a lane, two bytes each: 137 us for 2048 x 32 000
// bf16 instead of 83).
// The largest value of each column in a range of rows; infinite where something is not finite.
template <typename T>
__global__ __launch_bounds__(256) void weight_top_kernel(QuantWeight p, float* top) {
    __shared__ unsigned tops[4][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane % 8 * 8, k0 = (int64_t)blockIdx.y * kWeightRange, group = blockIdx.z;
    const T* w = (const T*)p.w.dev + group * p.w.group + k0 * p.w.row + c;
    const int left = (int)max((int64_t)0, min((int64_t)8, p.out - c)), end = (int)min(kWeightRange, p.width - k0);
    unsigned t[8] = {};
    for (int k = wave * 8 + lane / 8; k < end; k += 128) {     // four rows under way
        float v[4][8];
#pragma unroll
        for (int j = 0; j < 4; ++j) load_upto8(w + (int64_t)(k + 32 * j) * p.w.row, k + 32 * j < end ? left : 0, 0.0f, v[j]);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) t[e] = max(t[e], size_bits(v[j][e]));
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        for (int o = 8; o < 64; o <<= 1) t[e] = max(t[e], (unsigned)__shfl_xor((int)t[e], o));
        if (lane < 8) tops[wave][lane * 8 + e] = t[e];
    }
    __syncthreads();
    const int64_t ch = (int64_t)blockIdx.x * 64 + threadIdx.x;
    if (threadIdx.x >= 64 || ch >= p.out) return;
    const unsigned all = max(max(tops[0][threadIdx.x], tops[1][threadIdx.x]), max(tops[2][threadIdx.x], tops[3][threadIdx.x]));
    top[((int64_t)blockIdx.y * gridDim.z + group) * p.out + ch] = all >= 0x7f800000u ? INFINITY : __uint_as_float(all);
}

// Rounds and transposes a tile through LDS; lines are written sixteen bytes a lane.
template <typename T>
__global__ __launch_bounds__(256) void weight_kernel(QuantWeight p, const float* top, int ranges) {
    __shared__ __align__(8) int8_t tile[kTile][kTile + 8];
    __shared__ float tops[64];
    const int64_t c0 = (int64_t)blockIdx.x * 64, c = c0 + threadIdx.x % 8 * 8, k0 = (int64_t)blockIdx.y * kTile, group = blockIdx.z;
    const int left = (int)max((int64_t)0, min((int64_t)8, p.out - c)), k = threadIdx.x / 8;
    const T* w = (const T*)p.w.dev + group * p.w.group + (k0 + k) * p.w.row + c;
    float v[2][8];
#pragma unroll
    for (int j = 0; j < 2; ++j) load_upto8(w + 32 * j * p.w.row, k0 + k + 32 * j < p.width ? left : 0, 0.0f, v[j]);
    if (threadIdx.x < 64) {
        float t = 0.0f;
        if (c0 + threadIdx.x < p.out)
            for (int r = 0; r < ranges; ++r) t = fmaxf(t, top[((int64_t)r * gridDim.z + group) * p.out + c0 + threadIdx.x]);
        tops[threadIdx.x] = t;
        if (blockIdx.y == 0 && c0 + threadIdx.x < p.out) p.scale[group * p.scale_group + c0 + threadIdx.x] = RowScale(size_bits(t)).scale;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int ch = threadIdx.x % 8 * 8 + e;
        const RowScale s(size_bits(tops[ch]));
        tile[ch][k] = (int8_t)s.mostly(v[0][e]);
        tile[ch][k + 32] = (int8_t)s.mostly(v[1][e]);
    }
    __syncthreads();
    const int row = threadIdx.x / 4, chunk = threadIdx.x % 4 * 16;
    const int64_t rest = p.width - k0 - chunk;
    if (c0 + row >= p.out || rest <= 0) return;
    int8_t* q = p.q + group * p.q_group + (c0 + row) * p.q_row + k0 + chunk;
    store_packed(q, rest, *(const u2*)&tile[row][chunk]);
    if (rest > 8) store_packed(q + 8, rest - 8, *(const u2*)&tile[row][chunk + 8]);
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

__device__ __forceinline__ i4 whole_16(const int8_t* at) { return __builtin_bit_cast(i4, (u4)*(const u4bytes*)at); }

// A scale as mantissa and exponent: the product of a sum and one scale need not lie in fp32's range where that with both does.  (Of 512 rows,
// 2048 to 2048, and of 8192, 512 to 4096, fp64 costs 4 and 5 %, this 1 and 2.)
struct Scale {
    float m;
    int e;
    __device__ explicit Scale(float s) : m(__builtin_amdgcn_frexp_mantf(s)), e(__builtin_amdgcn_frexp_expf(s)) {}
};
__device__ __forceinline__ float scaled(int sum, Scale s, Scale t) { return ldexpf((float)sum * s.m * t.m, s.e + t.e); }

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

// Few rows: a workgroup for 16 channels and 16 R rows, whose wavefronts share the contraction in ranges; kAhead turns of 64 indices are
// under way before anything is waited for.  FUSED: the workgroup quantises the one row itself, into LDS, and a launch falls away (1.5 us
// of a call).  Of more rows every workgroup would have more to do than the launch takes (all of a call on the device, quantised here / by
// themselves: 8 rows, 2048 to 2048 9.7 / 8.5 us, 16 rows, 1024 to 8000 12.5 / 9.2).
constexpr int kAhead = 8;
template <typename TX, int R, int WAVES, bool FUSED>
__global__ __launch_bounds__(WAVES * 64) void few_kernel(Product p) {
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64);
    const int64_t group = blockIdx.z, c0 = (int64_t)blockIdx.x * 16;
    // channels and rows that do not exist are the last one again: what comes of them is not written
    const int8_t* w = p.w + group * p.w_group + min(c0 + lane % 16, p.out - 1) * p.w_row + 16 * (lane / 16);
    const int8_t* x[R];
#pragma unroll
    for (int i = 0; i < R; ++i) x[i] = p.x + group * p.x_group + min((int64_t)16 * i + lane % 16, p.rows - 1) * p.x_row + 16 * (lane / 16);
    const int turns = (int)(p.width / 64), from = turns * wave / WAVES, to = turns * (wave + 1) / WAVES;      // whole turns: no bounds to look at
    const int tail = turns * 64;
    constexpr int AX = kAhead / (2 * R);                           // turns whose rows are under way: registers
    i4 a[kAhead], b[FUSED ? 1 : AX][R];
    auto request = [&](int first) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (first + j < to) a[j] = whole_16(w + (int64_t)(first + j) * 64);
    };
    auto request_rows = [&](int first) {
        if constexpr (!FUSED) {
#pragma unroll
            for (int j = 0; j < AX; ++j)
                if (first + j < to) {
#pragma unroll
                    for (int i = 0; i < R; ++i) b[j][i] = whole_16(x[i] + (int64_t)(first + j) * 64);
                }
        }
    };
    request(from);
    i4 a_tail = {};
    const bool has_tail = wave == WAVES - 1 && p.width % 64 != 0;
    const int64_t behind = p.width - tail - 16 * (lane / 16);      // of the lane's sixteen bytes of the tail, those that exist
    if (has_tail) a_tail = load_16(w + tail, 0, behind, true);
    float scale = 0.0f;
    if constexpr (FUSED) {                                         // one row
        __shared__ unsigned tops[WAVES];
        const TX* row = (const TX*)p.quant.x.dev + group * p.quant.x.group;
        const TX* up = p.quant.up.dev ? (const TX*)p.quant.up.dev + group * p.quant.up.group : nullptr;
        const RowScale s = row_scale<TX, WAVES * 64>(p.quant, row, up, tops);
        scale = s.scale;
        for (int64_t k = threadIdx.x * 8; k < (p.width + 63) / 64 * 64; k += WAVES * 64 * 8) {
            float v[8];
            values<TX>(p.quant, row, up, k, v);
            *(u2*)(lds + k) = pack8(s, v);
        }
        __syncthreads();
    }
    i4 acc[R] = {};
    const int row = 16 * (lane / 16);
    for (int first = from; first < to; first += kAhead) {
        if (first > from) request(first);
        if constexpr (FUSED) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (first + j < to) acc[0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[j], *(const i4*)(lds + row + (first + j) * 64), acc[0], 0, 0, 0);
        } else {
#pragma unroll
            for (int h = 0; h < kAhead; h += AX) {
                if (first + h >= to) continue;
                request_rows(first + h);
#pragma unroll
                for (int j = 0; j < AX; ++j)
                    if (first + h + j < to) {
#pragma unroll
                        for (int i = 0; i < R; ++i) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[h + j], b[j][i], acc[i], 0, 0, 0);
                    }
            }
        }
    }
    if (has_tail) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            i4 v;
            if constexpr (FUSED) v = *(const i4*)(lds + row + tail);
            else v = load_16(x[i] + tail, 0, behind, true);
            acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a_tail, v, acc[i], 0, 0, 0);
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
        const int64_t r = 16 * i + lane % 16, o = c0 + 4 * (lane / 16);
        if (r >= p.rows || o >= p.out) continue;
        const Scale s(FUSED ? scale : p.x_scale[group * p.x_scale_group + r]);
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = o + e < p.out ? scaled(sum[e], s, Scale(p.w_scale[group * p.w_scale_group + o + e])) : 0.0f;
        store_scaled<4>(p, group, r, o, v);
    }
}

// ---- many rows ------------------------------------------------------------------------------------------------------------

constexpr int kSlice = 64;               // indices of a slice: as many bytes as the bf16 tiles' 32
using ffn::Cursor;
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

// T x T tiles: 256 with eight wavefronts of 64 x 128, 128 with four of 64 x 64, 64 with four of 32 x 32.  The tiles, their ring in LDS and
// the order of copies, barriers and reads are those of the bf16 products (ffn_gemm.h): sixteen bytes of a lane are sixteen indices here
// instead of eight.  Tiles of 64 have a ring of eight slices, since few of them run.  The scales are requested before the operands, and two
// turns of the results are under way (8192 rows, 512 to 4096: 38.8 us before, 36.2 so; 4096 to 4096: 144 and 139).
template <int T>
__global__ __launch_bounds__(ffn::gemm_threads<T>(), 2) void tile_kernel(Product p) {
    constexpr int THREADS = ffn::gemm_threads<T>(), TM = T == 64 ? 1 : 2, TN = T / 64, D = T == 64 ? 8 : 4;
    using Tile = ffn::TileKC<T, THREADS>;
    constexpr int kBytes = 2 * Tile::kBytes, kMore = D == 8 ? kBytes : 16;
    __shared__ __align__(1024) char buf0[kBytes];
    __shared__ __align__(1024) char buf1[kBytes];
    __shared__ __align__(1024) char buf2[kBytes];
    __shared__ __align__(1024) char buf3[kBytes];
    __shared__ __align__(1024) char buf4[kMore];
    __shared__ __align__(1024) char buf5[kMore];
    __shared__ __align__(1024) char buf6[kMore];
    __shared__ __align__(1024) char buf7[kMore];

    int range;
    const int tile = tile_of_block(p, range);
    const Place at = place_of(p, tile, T);
    const int lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64), wm = wave / 2, wn = wave % 2;
    // A row's pairs of bytes, up to whole chunks.  x holds zeros there; of w the rest of the chunk that holds the row's last weight is read, sixteen
    // bytes on sixteen, and counts for nothing.
    const int64_t k2 = (p.width + 15) / 16 * 8;
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

    // The scales of the results, requested before the operands: a lane for each of the wavefront's rows, and eight channels of each lane.
    constexpr int kCols = TN * 32, kUnits = kCols / 8, kRows = 64 / kUnits;
    const int out_row = lane / kUnits, unit = lane % kUnits, col = wn * (T / 2) + 8 * unit;
    float row_scale = 0.0f, cs[8] = {};
    if (range < 0) {
        const int64_t row = at.m0 + wm * (32 * TM) + lane % (32 * TM);
        if (row < p.rows) row_scale = p.x_scale[at.group * p.x_scale_group + row];
        load_upto8(p.w_scale + at.group * p.w_scale_group + at.n0 + col, (int)max((int64_t)0, min((int64_t)8, p.out - at.n0 - col)), 0.0f, cs);
    }

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
    // Counts as in ffn_gemm.h; copies past the end (windows of no bytes) keep the count the same.
    constexpr int kPerSlice = 2 * Tile::kCopies;
    static_assert((D - 1) * kPerSlice < 16, "counts of four bits");
    auto barrier = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto slice = [&](char* lds, char* next) {
        fetch(lds, 1);
        multiply(0);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0x0070 | (D - 2) * kPerSlice);   // vmcnt, lgkmcnt(0): the next slice has landed
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
    if constexpr (D == 8) {
        copy(buf4);
        copy(buf5);
        copy(buf6);
        copy(buf7);
    }
    __builtin_amdgcn_s_waitcnt(0x0f70 | (D - 1) * kPerSlice);       // vmcnt
    barrier();
    fetch(buf0, 0);
    for (int it = 0; it < end; it += D) {
        slice(buf0, buf1);
        if (it + 1 < end) slice(buf1, buf2);
        if (it + 2 < end) slice(buf2, buf3);
        if (it + 3 < end) slice(buf3, D == 8 ? buf4 : buf0);
        if constexpr (D == 8) {
            if (it + 4 < end) slice(buf4, buf5);
            if (it + 5 < end) slice(buf5, buf6);
            if (it + 6 < end) slice(buf6, buf7);
            if (it + 7 < end) slice(buf7, buf0);
        }
    }
    __builtin_amdgcn_s_waitcnt(0x0070);                       // the copies past the end write zeros into LDS

    __syncthreads();                                          // everyone is done with the operands
    constexpr int kPart = THREADS / 64 / 4, kInts = 32 * kCols, kSwizzle = kCols >= 64 ? 15 : 7;   // wavefronts that stage in one buffer
    static_assert(kBytes >= kPart * kInts * 4, "the results of 32 rows of every wavefront are staged in the buffers");
    char* bufs[4] = {buf0, buf1, buf2, buf3};
    int* stage = (int*)bufs[0] + wave % kPart * kInts;
#pragma unroll
    for (int i = 1; i < 4; ++i) stage = wave / kPart == i ? (int*)bufs[i] + wave % kPart * kInts : stage;
    const int lane_row = lane % 32;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int chunk = 8 * t + 2 * g + lane / 32;
                *(i4*)(stage + lane_row * kCols + 4 * (chunk ^ (lane_row & kSwizzle))) = i4{acc[i][t][4 * g], acc[i][t][4 * g + 1], acc[i][t][4 * g + 2], acc[i][t][4 * g + 3]};
            }
        in_wave_order();                                      // written and read by one wavefront: LDS keeps its order
#pragma unroll 2
        for (int r0 = 0; r0 < 32; r0 += kRows) {
            const int r = r0 + out_row, row = wm * (32 * TM) + 32 * i + r;
            const Scale s(__shfl(row_scale, 32 * i + r));
            const i4 lo = *(const i4*)(stage + r * kCols + 4 * ((2 * unit) ^ (r & kSwizzle))), hi = *(const i4*)(stage + r * kCols + 4 * ((2 * unit + 1) ^ (r & kSwizzle)));
            if (range >= 0) {
                int* out = p.partial + ((int64_t)range * p.rest + (tile - p.whole)) * (T * T) + row * T + col;
                *(i4*)out = lo;
                *(i4*)(out + 4) = hi;
            } else if (at.m0 + row < p.rows && at.n0 + col < p.out) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = scaled(lo[e], s, Scale(cs[e])), v[4 + e] = scaled(hi[e], s, Scale(cs[4 + e]));
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
    const Scale s(p.x_scale[at.group * p.x_scale_group + at.m0 + row]);
    float cs[8], v[8];
    load_upto8(p.w_scale + at.group * p.w_scale_group + at.n0 + col, (int)min((int64_t)8, p.out - at.n0 - col), 0.0f, cs);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = scaled(lo[e], s, Scale(cs[e])), v[4 + e] = scaled(hi[e], s, Scale(cs[4 + e]));
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
    bool fused, lay_x, lay_w;             // rows quantised where they are multiplied; operands laid out first, in every call (4096 x 4096 weights: 7 us)
    int tiles_m, tiles_n, whole, rest, ranges;
    int64_t scale_at, w_at, partial_at, ws_bytes;
};

bool lies_well(const ols_matrix& m) { return m.row % 16 == 0 && m.row <= (1 << 22) && m.group % 16 == 0 && ((uintptr_t)m.dev & 15) == 0; }

// Whether y lies away from the one row of each group that m holds.
bool away(const ols_int8& f, const ols_matrix& m) {
    const char *a = (const char*)m.dev, *y = (const char*)f.y.dev;
    const int64_t size = f.dtype == OLS_F32 ? 4 : 2, y_size = f.out_dtype == OLS_F32 ? 4 : 2;
    return a >= y + ((f.groups - 1) * f.y.group + f.out) * y_size || y >= a + ((f.groups - 1) * m.group + f.width) * size;
}

constexpr int kCus = 256;
// Up to this many rows weights go straight into registers.  Products alone, in us, few_kernel / tiles: 32 rows, 2048 to 2048: 6.6 / 9.5; to
// 11 264: 12.3 / 11.7; 64 rows, 5632 to 2048: 11.3 / 11.2, 2048 to 11 264: 15.9 / 11.7, to 32 000: 36 / 18.
constexpr int kFewRows = 32;
constexpr int kFewWaves = 4096;           // of all workgroups together, where the contraction is long enough

// What a product in tiles takes, in microseconds: a start (of later rounds a part of it is hidden), and for each round of tiles its slices,
// which take longer the more tiles run beside each other; cut contractions add a launch and their sums' traffic.
// Fitted to products of 64 to 8192 rows and 56 to 32 000 channels over 100 to 8192 indices.  Tiles of 64 / 128 / 256 whole: 512 rows, 2048 to
// 2048: 11.8 / 16.8 / 33; 1024, 2048 to 5632: 38 / 24.5 / 35; 1319, 1184 to 13 224: 81 / 53 / 55; 4096, 1536 to 4096: 77 / 44 / 36.  128 rows, 5632 to 2048 in tiles of 64, cut in 1 / 2 / 4 / 8: 22.5 /
// 17.2 / 13.2 / 14.7.  2000 rows, 512 to 2000, where tiles of 64 take two rounds: 14.7 / 10.4 / 16.9.
struct Cost {
    int tile, slots;                      // tiles of a round
    double start, again, least, more;     // of the first round and of others; a slice: least + more x (share of the slots that are taken)
};
constexpr Cost kCosts[3] = {{64, 2 * kCus, 4.6, 3.0, 0.17, 0.14}, {128, 2 * kCus, 6.0, 4.0, 0.30, 0.42}, {256, kCus, 9.6, 7.0, 0.45, 0.75}};

double cost_of(const Cost& c, int64_t tiles, int64_t slices, int ranges) {
    const int64_t rounds = tiles / c.slots, rest = tiles % c.slots;
    double us = c.start - c.again + (double)rounds * (c.again + (double)slices * (c.least + c.more));
    if (!rest) return us;
    const int64_t run = rest * ranges, last = run % c.slots ? run % c.slots : c.slots;
    us += (double)((run + c.slots - 1) / c.slots) * c.again;
    us += (double)((slices + ranges - 1) / ranges) * ((double)((run - 1) / c.slots) * (c.least + c.more) + c.least + c.more * (double)last / c.slots);
    return ranges == 1 ? us : us + 3.0 + (double)run * c.tile * c.tile * 8 / 4e6;
}

Plan plan_of(const ols_int8& f) {
    Plan p = {};
    const int64_t turns = (f.width + 63) / 64;
    p.ranges = 1;
    if (f.rows <= kFewRows) {
        p.R = f.rows <= 16 ? 1 : 2;
        const int64_t blocks = (f.out + 15) / 16 * f.groups;
        p.waves = 2;
        while (p.waves < 16 && 2 * p.waves * blocks <= kFewWaves && 4 * p.waves <= turns) p.waves *= 2;
        p.fused = f.dtype != OLS_I8 && f.rows == 1 && f.width <= 32768 && f.width * blocks <= (1 << 23);
        p.fused = p.fused && away(f, f.x) && (!f.up.dev || away(f, f.up));      // while some quantise, others write
    } else {
        double best = 1e30;
        for (const Cost& c : kCosts) {
            const int64_t tiles_m = (f.rows + c.tile - 1) / c.tile, tiles_n = (f.out + c.tile - 1) / c.tile, tiles = tiles_m * tiles_n * f.groups;
            if (tiles >= (1 << 23)) continue;                  // a launch has fewer than 2^32 threads
            for (int ranges = 1; ranges <= 16 && (ranges == 1 || 4 * ranges <= turns); ranges *= 2) {
                const double us = cost_of(c, tiles, turns, ranges);
                if (us >= best) continue;
                best = us;
                p.tile = c.tile, p.tiles_m = (int)tiles_m, p.tiles_n = (int)tiles_n, p.ranges = ranges;
                p.rest = ranges > 1 ? (int)(tiles % c.slots) : 0, p.whole = (int)tiles - p.rest;
            }
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
    const size_t sums = (size_t)WAVES * R * 1024, row = FUSED ? (size_t)(p.width + 63) / 64 * 64 : 0;
    few_kernel<TX, R, WAVES, FUSED><<<dim3((unsigned)((p.out + 15) / 16), 1, p.groups), WAVES * 64, std::max(sums, row), stream>>>(p);
}
template <typename TX, int R, bool FUSED>
void launch_few_waves(const Product& p, const Plan& plan, hipStream_t stream) {
    if (plan.waves == 16) launch_few_sized<TX, R, 16, FUSED>(p, stream);
    else if (plan.waves == 8) launch_few_sized<TX, R, 8, FUSED>(p, stream);
    else if (plan.waves == 4) launch_few_sized<TX, R, 4, FUSED>(p, stream);
    else launch_few_sized<TX, R, 2, FUSED>(p, stream);
}
template <typename TX, bool FUSED>
void launch_few(const Product& p, const Plan& plan, hipStream_t stream) {
    if (FUSED || plan.R == 1) launch_few_waves<TX, 1, FUSED>(p, plan, stream);      // fused: one row
    else if constexpr (!FUSED) launch_few_waves<TX, 2, false>(p, plan, stream);
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
    else if (plan.tile == 128) tile_kernel<128><<<blocks, 256, 0, stream>>>(p);
    else tile_kernel<64><<<blocks, 256, 0, stream>>>(p);
    e = hipGetLastError();
    if (e != hipSuccess || !plan.rest) return e;
    const dim3 grid(plan.rest, plan.tile * plan.tile / 8 / 256);
    if (plan.tile == 256) join_kernel<256><<<grid, 256, 0, stream>>>(p);
    else if (plan.tile == 128) join_kernel<128><<<grid, 256, 0, stream>>>(p);
    else join_kernel<64><<<grid, 256, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace ols
