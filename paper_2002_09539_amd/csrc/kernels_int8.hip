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

// A workgroup for each row: its largest value, then what is rounded, read again.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantRows p) {
    __shared__ float tops[4];
    __shared__ int bads[4];
    const int64_t group = blockIdx.x / p.rows, row = blockIdx.x % p.rows;
    const T* x = (const T*)p.x.dev + group * p.x.group + row * p.x.row;
    const T* up = p.up.dev ? (const T*)p.up.dev + group * p.up.group + row * p.up.row : nullptr;
    float top = 0.0f;
    bool bad = false;
    for (int64_t c = threadIdx.x * 8; c < p.width; c += 256 * 8) {
        float v[8];
        values<T>(p, x, up, c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e])), bad |= !(fabsf(v[e]) < INFINITY);
    }
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const unsigned long long any = __ballot(bad);
    if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = top, bads[threadIdx.x / 64] = any != 0;
    __syncthreads();
    const RowScale s(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])), bads[0] | bads[1] | bads[2] | bads[3]);
    if (threadIdx.x == 0) p.scale[group * p.scale_group + row] = s.scale;
    int8_t* q = p.q + group * p.q_group + row * p.q_row;
    for (int64_t c = threadIdx.x * 8; c < p.padded; c += 256 * 8) {
        float v[8];
        values<T>(p, x, up, c, v);
        const unsigned lo = pack4(s, v[0], v[1], v[2], v[3]), hi = pack4(s, v[4], v[5], v[6], v[7]);
        const int left = (int)min((int64_t)8, p.padded - c);
        if (left >= 8) {
            *(u2any*)(q + c) = u2any{lo, hi};
        } else {
            for (int e = 0; e < left; ++e) q[c + e] = (int8_t)((e < 4 ? lo >> (8 * e) : hi >> (8 * (e - 4))) & 255);
        }
    }
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
};

// sixteen bytes of a row from index k, zeros from `width` on
__device__ __forceinline__ i4 load_16(const int8_t* row, int64_t k, int64_t width, bool there) {
    typedef unsigned u4bytes __attribute__((ext_vector_type(4), aligned(1)));
    if (!there || k >= width) return i4{0, 0, 0, 0};
    if (k + 16 <= width) return __builtin_bit_cast(i4, (u4)*(const u4bytes*)(row + k));
    unsigned v[4] = {};
    for (int e = 0; k + e < width; ++e) v[e / 4] |= (unsigned)(uint8_t)row[k + e] << (8 * (e % 4));
    return i4{(int)v[0], (int)v[1], (int)v[2], (int)v[3]};
}

// A wavefront for 16 channels and 64 rows.
__global__ __launch_bounds__(256) void product_kernel(Product p) {
    constexpr int R = 4;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t group = blockIdx.z, c0 = ((int64_t)blockIdx.x * 4 + wave) * 16, r0 = (int64_t)blockIdx.y * (16 * R);
    if (c0 >= p.out) return;
    const int64_t c = c0 + lane % 16;
    const int8_t* w = p.w + group * p.w_group + c * p.w_row;
    const int8_t* x = p.x + group * p.x_group + (r0 + lane % 16) * p.x_row;
    i4 acc[R] = {};
    for (int64_t k = 16 * (lane / 16); k - 16 * (lane / 16) < p.width; k += 64) {
        const i4 a = load_16(w, k, p.width, c < p.out);
#pragma unroll
        for (int i = 0; i < R; ++i) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, load_16(x + 16 * i * p.x_row, k, p.width, r0 + 16 * i + lane % 16 < p.rows), acc[i], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int64_t r = r0 + 16 * i + lane % 16;
        if (r >= p.rows) continue;
        const float s = p.x_scale[group * p.x_scale_group + r];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t o = c0 + 4 * (lane / 16) + e;
            if (o >= p.out) continue;
            const float v = (float)acc[i][e] * s * p.w_scale[group * p.w_scale_group + o];
            const int64_t at = group * p.y_group + r * p.y_row + o;
            if (p.out_f32) store1((float*)p.y + at, v);
            else store1((uint16_t*)p.y + at, v);
        }
    }
}

int64_t up16(int64_t v) { return (v + 15) / 16 * 16; }
int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }
int x_groups(const ols_int8& f) { return f.x.group == 0 && (!f.up.dev || f.up.group == 0) ? 1 : f.groups; }    // rows that the workers share: once
constexpr int64_t kMostBlocks = 1 << 23;   // of 256 threads: a launch has fewer than 2^32

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
        if (p.dtype == OLS_F32) quantize_rows_kernel<float><<<blocks, 256, 0, stream>>>(q);
        else quantize_rows_kernel<uint16_t><<<blocks, 256, 0, stream>>>(q);
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

int64_t int8_workspace_bytes(const ols_int8& f) {
    if (f.rows == 0 || f.dtype == OLS_I8) return 0;
    return up256(x_groups(f) * f.rows * up16(f.width)) + up256(x_groups(f) * f.rows * 4);
}

hipError_t launch_int8(const ols_int8& f, hipStream_t stream) {
    Product p = {};
    p.groups = f.groups, p.out_f32 = f.out_dtype == OLS_F32, p.rows = f.rows, p.width = f.width, p.out = f.out;
    p.w = (const int8_t*)f.w.dev, p.w_row = f.w.row, p.w_group = f.w.group, p.w_scale = f.w_scale, p.w_scale_group = f.w_scale_group;
    p.y = f.y.dev, p.y_row = f.y.row, p.y_group = f.y.group;
    if (f.dtype == OLS_I8) {
        p.x = (const int8_t*)f.x.dev, p.x_row = f.x.row, p.x_group = f.x.group, p.x_scale = f.x_scale, p.x_scale_group = f.x_scale_group;
    } else {
        QuantRows q = {};
        q.groups = x_groups(f), q.dtype = f.dtype, q.act = f.act, q.rows = f.rows, q.width = f.width, q.x = f.x, q.up = f.up;
        q.q = (int8_t*)f.ws, q.q_row = up16(f.width), q.q_group = f.rows * q.q_row, q.padded = q.q_row;
        q.scale = (float*)((char*)f.ws + up256(q.groups * q.q_group)), q.scale_group = f.rows;
        const hipError_t e = launch_quantize_rows(q, stream);
        if (e != hipSuccess) return e;
        p.x = q.q, p.x_row = q.q_row, p.x_group = q.groups == 1 ? 0 : q.q_group, p.x_scale = q.scale, p.x_scale_group = q.groups == 1 ? 0 : f.rows;
    }
    product_kernel<<<dim3((unsigned)((p.out + 63) / 64), (unsigned)((p.rows + 63) / 64), p.groups), 256, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace ols
