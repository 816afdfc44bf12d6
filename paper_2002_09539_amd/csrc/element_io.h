// Reading and writing runs of elements of either storage type (fp32, bf16) as fp32 values.
//
// Rows of caller-owned tensors start wherever the caller's strides put them: a row of 50 001 bf16 logits leaves the next
// one on an odd element.  Global memory takes 16-byte accesses at any address on gfx950, so the vectors here are declared
// with the alignment of one element and every row takes the wide path; only the last, partial vector of a row goes
// element by element (nothing outside a row is touched).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "split_bf16.h"

namespace ols {

// Orders what the lanes of one wavefront write and read in LDS, which the hardware does in the order of its instructions.
__device__ __forceinline__ void in_wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

typedef unsigned int u4any __attribute__((ext_vector_type(4), aligned(2)));   // sixteen bytes at any element's address

__device__ __forceinline__ uint16_t bf16_of(float v) { return (uint16_t)pack_bf16(v, 0.0f); }   // to nearest even
__device__ __forceinline__ float of_bf16(uint16_t v) { return __uint_as_float((unsigned)v << 16); }

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const uint16_t* p) { return of_bf16(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = bf16_of(v); }

// eight elements
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const u4any a = *(const u4any*)p, b = *(const u4any*)(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(a[e]), v[4 + e] = __uint_as_float(b[e]);
}
__device__ __forceinline__ void load8(const uint16_t* p, float (&v)[8]) {
    const u4any a = *(const u4any*)p;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[2 * e] = bf16_lo(a[e]), v[2 * e + 1] = bf16_hi(a[e]);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    u4any a, b;
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] = __float_as_uint(v[e]), b[e] = __float_as_uint(v[4 + e]);
    *(u4any*)p = a;
    *(u4any*)(p + 4) = b;
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
    u4any a;
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
    *(u4any*)p = a;
}

// `left` (0 .. 8 or more) elements of a run of eight; the others read as `fill` and are not written
template <typename T>
__device__ __forceinline__ void load_upto8(const T* p, int left, float fill, float (&v)[8]) {
    if (left >= 8) {
        load8(p, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < left ? load1(p + e) : fill;
    }
}
template <typename T>
__device__ __forceinline__ void store_upto8(T* p, int left, const float (&v)[8]) {
    if (left >= 8) {
        store8(p, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) store1(p + e, v[e]);
    }
}

// Eight elements as they lie in memory, for loads in flight: bf16 takes half the registers until it is used.
template <typename T>
struct Raw8;
template <>
struct Raw8<uint16_t> {
    u4 a;
    __device__ void load(const uint16_t* p, int left) {
        if (left >= 8) {
            a = *(const u4any*)p;
        } else {
            float v[8];
            load_upto8(p, left, 0.0f, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) a[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
        }
    }
    __device__ float get(int e) const { return e % 2 ? bf16_hi(a[e / 2]) : bf16_lo(a[e / 2]); }
};
template <>
struct Raw8<float> {
    float v[8];
    __device__ void load(const float* p, int left) { load_upto8(p, left, 0.0f, v); }
    __device__ float get(int e) const { return v[e]; }
};

}  // namespace ols
