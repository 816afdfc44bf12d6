// The feed-forward block's products of fp32 operands, on the bf16 matrix cores.
//
// An fp32 operand lies as three bf16 terms that add up to it exactly, eight elements' first terms, second and third side by side
// (48 bytes); split_bf16.h says why the six largest of the nine products of terms are enough.  A slice of 16 contraction indices
// brings all three terms of both operands into LDS, and every fragment serves two or three products: with the six products as
// six passes over whole slices, each fragment read for one product only, LDS bounded them at half the rate.
//
// Tiles are 128 x 128, two workgroups of four wavefronts a compute unit, three slices of 24 KB each: one is in registers, one is
// read from LDS while its predecessor is multiplied, two are under way.  The small products come first and a term's registers
// take the next slice's as soon as they are done with.
//
// What bounds it: the matrix pipes at the clock that their power leaves.  The weights' gradients of 4096 rows, 1024 by 2816: 70.9
// GFLOP in 320 us, 221 TFLOP/s of fp32 products (1330 of bf16 ones; a library's fp32 product reaches 154); eight workers of 2325
// rows, 1182 by 400: 297 us instead of 472 by six passes.  The copies in front of the products: 3 % slower; next slice's first terms
// in registers of their own, so that no read is waited for, or wavefront priorities: nothing.
//
// The product of the first terms has accumulators of its own.  An infinite operand has remainders of zero, and the small
// products would turn infinity times zero into NaN: where the large sum is not finite it is the result.
#pragma once
#include "ffn_gemm.h"

namespace ols {
namespace ffn {

constexpr int kBKF32 = 16;

// KC: LDS [128 rows][6 chunks]: of row r (contraction half, term) at place (3 half + term) ^ (r / 8 & 1), so that sixteen rows'
// chunks lie on different banks.
struct TermsKC {
    static constexpr int kBytes = 128 * 6 * 16;
    unsigned off[3];
    int half[3];
    __device__ explicit TermsKC(int64_t pitch) {
        const int lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64);
#pragma unroll
        for (int t = 0; t < 3; ++t) {
            const int i = t * 64 + lane, r = i / 6, c = (i % 6) ^ ((r >> 3) & 1);
            half[t] = c / 3, off[t] = (unsigned)((wave * 32 + r) * pitch * 2 + c * 16);
        }
    }
    __device__ static Cursor cursor(const uint16_t* base, int64_t pitch, int64_t rows, int64_t k8, int64_t row0, int64_t k0) {
        return {(const char*)(base + row0 * pitch + 3 * k0), 2 * ((rows - 1 - row0) * pitch + 3 * (k8 - k0)), 2 * 3 * kBKF32};
    }
    __device__ void copy(char* lds, int at, const Cursor& c, int64_t k_left) const {
        const int wave = uniform(threadIdx.x / 64);
        const rsrc_t rs = c.window();
#pragma unroll
        for (int t = 0; t < 3; ++t)                           // past the row's end: beyond any window, zeros
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)(lds + (at + (wave * 3 + t) * 1024)), 16,
                                                     (int)(half[t] * 8 < k_left ? off[t] : 0x7ffffff0u), 0, 0, 0);
    }
    __device__ static int lane_part(int at, int r0, int lane, int term) {
        const int r = r0 + lane % 32;
        return at + r * 96 + (((3 * (lane / 32) + term) ^ ((r >> 3) & 1)) << 4);
    }
    __device__ static bf16x8 frag(const char* lds, int part) { return __builtin_bit_cast(bf16x8, *(const u4*)(lds + part)); }
};

// RC: LDS [16][COLS / 8 chunks][3 terms], the chunks of line k at place chunk ^ swizzle(k).  With 64 columns the even and the odd lines
// lie on different banks by themselves.  PANELS operands side by side, copied by as many parts of the workgroup.
template <int COLS, int PANELS>
struct TermsRC {
    static constexpr int kBytes = COLS * 6 * 16, kLine = COLS / 8 * 3;
    static_assert(COLS * PANELS == 128, "three copies per wavefront");
    __device__ static int swizzle(int k) { return COLS == 128 ? (k & 3) << 2 : (k & 2) << 1; }
    unsigned off[3];
    __device__ explicit TermsRC(int64_t pitch) {
        const int lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64) % (4 / PANELS);
#pragma unroll
        for (int t = 0; t < 3; ++t) {
            const int i = (wave * 3 + t) * 64 + lane, k = i / kLine, s = i % kLine;
            off[t] = (unsigned)(k * pitch * 2 + (3 * ((s / 3) ^ swizzle(k)) + s % 3) * 16);
        }
    }
    __device__ static Cursor cursor(const uint16_t* base, int64_t pitch, int64_t cols8, int64_t K, int64_t col0, int64_t k0) {
        return {(const char*)(base + k0 * pitch + 3 * col0), 2 * ((K - 1 - k0) * pitch + 3 * (cols8 - col0)), 2 * kBKF32 * pitch};
    }
    __device__ void copy(char* lds, int at, const Cursor& c, int64_t) const {
        const int wave = uniform(threadIdx.x / 64);
        const rsrc_t rs = c.window();
#pragma unroll
        for (int t = 0; t < 3; ++t)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr)(lds + (at + (wave * 3 + t) * 1024)), 16, (int)off[t], 0, 0, 0);
    }
    __device__ static int lane_part(int at, int c0, int lane, int term) {
        const int blk = lane / 16, j = lane % 16;
        const int k = 8 * (blk / 2) + j / 4, c = c0 + 16 * (blk % 2) + 4 * (j % 4);
        return at + k * (kLine * 16) + ((3 * ((c / 8) ^ swizzle(k)) + term) << 4) + (c % 8) * 2;
    }
    __device__ static bf16x8 frag(const char* lds, int part) {
        typedef s4v __attribute__((address_space(3))) * lds_s4_ptr;
        const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr)(lds + part));
        const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr)(lds + (part + 4 * kLine * 16)));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

template <bool A_RC, bool B_RC, Epi EPI>
__global__ __launch_bounds__(256, 2) void gemm_f32_kernel(GemmArgs p) {
    constexpr int PANELS = EPI == kUp ? 2 : 1;
    static_assert(PANELS == 1 || B_RC, "two panels are read line by line");
    using TA = typename std::conditional<A_RC, TermsRC<128, 1>, TermsKC>::type;
    using TB = typename std::conditional<B_RC, TermsRC<128 / PANELS, PANELS>, TermsKC>::type;
    constexpr int kBytes = TA::kBytes + PANELS * TB::kBytes;
    static_assert(kBytes == 24576, "two wavefronts' results are staged in a buffer");
    __shared__ __align__(1024) char buf0[kBytes];
    __shared__ __align__(1024) char buf1[kBytes];
    __shared__ __align__(1024) char buf2[kBytes];

    int range;
    const int tile = tile_of_block(p, range);
    const TilePlace at = place_of(p, tile, 128, 128 / PANELS);
    const Job& q = p.job[at.job];
    const int lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64), wm = wave / 2, wn = wave % 2;
    const TA ta(q.a_pitch);
    const TB tb(q.b_pitch);
    const int slices = (int)((q.K + kBKF32 - 1) / kBKF32);
    const int from = range < 0 ? 0 : (int)((int64_t)slices * range / p.ranges);
    const int here = (range < 0 ? slices : (int)((int64_t)slices * (range + 1) / p.ranges)) - from;
    const uint16_t* base_a = q.a + at.group * q.a_group;
    const uint16_t* base_b = q.b + at.group * q.b_group;
    const uint16_t* base_b2 = q.b2 + at.group * q.b2_group;

    f16v big[2][2], small[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) big[i][t][r] = 0.0f, small[i][t][r] = 0.0f;

    int seg = 0, left_slices = here;                      // of the next copy
    int64_t k_left;
    Cursor cur_a, cur_b;
    auto enter = [&]() {                                  // the segment's first slice of this range
        const int64_t k0 = (int64_t)from * kBKF32;
        const uint16_t* a = seg ? base_a + q.second_a : base_a;
        const uint16_t* b = (PANELS == 1 ? seg != 0 : wave >= 2) ? base_b2 : base_b;
        cur_a = A_RC ? TA::cursor(a, q.a_pitch, q.a_inner8, q.K, at.m0, k0) : TA::cursor(a, q.a_pitch, q.M, q.a_inner8, at.m0, k0);
        cur_b = B_RC ? TB::cursor(b, q.b_pitch, q.b_inner8, q.K, at.n0, k0) : TB::cursor(b, q.b_pitch, q.N, q.b_inner8, at.n0, k0);
        k_left = (A_RC ? q.K : q.a_inner8) - k0;
    };
    enter();
    auto copy = [&](char* lds) {
        ta.copy(lds, 0, cur_a, k_left);
        tb.copy(lds, TA::kBytes, cur_b, k_left);
        cur_a.advance(), cur_b.advance();
        k_left -= kBKF32;
        if (--left_slices == 0) {
            if (++seg < q.segments) left_slices = here, enter();
            else cur_a.left = cur_b.left = 0, cur_a.step = cur_b.step = 0;   // from here on nothing is read
        }
    };
    int part_a[2][3], part_b[2][3];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int n = 0; n < 3; ++n) {
            part_a[i][n] = TA::lane_part(0, wm * 64 + 32 * i, lane, n);
            part_b[i][n] = PANELS == 2 ? TB::lane_part(TA::kBytes + i * TB::kBytes, wn * 32, lane, n) : TB::lane_part(TA::kBytes, wn * 64 + 32 * i, lane, n);
        }
    bf16x8 fa[3][2], fb[3][2];
    auto fetch = [&](const char* lds, int n) {            // the fragments of a term
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int part = part_b[i][n];                      // opaque: an array plus one offset
            asm volatile("" : "+v"(part));
            fb[n][i] = TB::frag(lds, part);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int part = part_a[i][n];
            asm volatile("" : "+v"(part));
            fa[n][i] = TA::frag(lds, part);
        }
    };
    auto multiply = [&](f16v (&to)[2][2], int x, int y) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int t = 0; t < 2; ++t) to[i][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[y][t], fa[x][i], to[i][t], 0, 0, 0);
    };
    const int end = here * q.segments;
    // In front of a slice's products: its fragments are in registers, and this wavefront's copies of the next one have landed (those of
    // the one behind it may be under way); behind the barrier that holds for all wavefronts, so the next slice can be read and this
    // one's buffer overwritten.  Copies past the end (windows of no bytes) keep the count the same.
    auto slice = [&](char* lds, char* next) {
        __builtin_amdgcn_s_waitcnt(0x0076);               // vmcnt(6) lgkmcnt(0)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        multiply(small, 2, 0);
        multiply(small, 0, 2);
        copy(lds);
        __builtin_amdgcn_sched_barrier(0);
        fetch(next, 2);
        multiply(small, 1, 1);
        multiply(small, 1, 0);
        multiply(small, 0, 1);
        __builtin_amdgcn_sched_barrier(0);
        fetch(next, 1);
        multiply(big, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        fetch(next, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    copy(buf0);
    copy(buf1);
    copy(buf2);
    __builtin_amdgcn_s_waitcnt(0x0f7c);                   // vmcnt(12)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    fetch(buf0, 2);
    fetch(buf0, 1);
    fetch(buf0, 0);
    for (int it = 0; it < end; it += 3) {
        slice(buf0, buf1);
        if (it + 1 < end) slice(buf1, buf2);
        if (it + 2 < end) slice(buf2, buf0);
    }
    __builtin_amdgcn_s_waitcnt(0x0070);                   // the copies past the end write zeros into LDS
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) big[i][t][r] = fabsf(big[i][t][r]) < INFINITY ? big[i][t][r] + small[i][t][r] : big[i][t][r];
    __syncthreads();                                      // everyone is done with the operands
    float* stage = (float*)(wave < 2 ? buf0 : buf1) + wave % 2 * (32 * 64);
    write_tile<EPI, true, 128>(big, stage, p, at, tile, range);
}

}  // namespace ffn
}  // namespace ols
