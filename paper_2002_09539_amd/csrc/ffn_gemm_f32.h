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
// PLAIN: the second operand is the caller's fp32 tensor; a lane splits eight elements of a slice on their way to LDS, and two slices
// are under way in registers.
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

// The same places in LDS for an operand that lies in memory as plain fp32: a lane takes eight elements of a slice into registers and
// writes their terms.
struct PlainKC {
    unsigned off;
    int half, place[3];
    __device__ explicit PlainKC(int64_t pitch) {
        const int r = threadIdx.x / 2;
        half = threadIdx.x % 2, off = (unsigned)(r * pitch * 4 + half * 32);
#pragma unroll
        for (int n = 0; n < 3; ++n) place[n] = r * 96 + (((3 * half + n) ^ ((r >> 3) & 1)) << 4);
    }
    __device__ static Cursor cursor(const float* base, int64_t pitch, int64_t rows, int64_t K, int64_t row0, int64_t k0) {
        return {(const char*)(base + row0 * pitch + k0), 4 * ((rows - 1 - row0) * pitch + K - k0), 4 * kBKF32};
    }
    __device__ bool has(int e, int64_t k_left) const { return half * 8 + e < k_left; }    // behind it lies the next row
};
template <int COLS, int PANELS>
struct PlainRC {
    unsigned off;
    int place[3];
    __device__ explicit PlainRC(int64_t pitch) {
        using T = TermsRC<COLS, PANELS>;
        const int i = threadIdx.x % (256 / PANELS), k = i / (COLS / 8), c = i % (COLS / 8);
        off = (unsigned)(k * pitch * 4 + c * 32);
#pragma unroll
        for (int n = 0; n < 3; ++n) place[n] = uniform(threadIdx.x / 64) / (4 / PANELS) * T::kBytes + k * (T::kLine * 16) + ((3 * (c ^ T::swizzle(k)) + n) << 4);
    }
    __device__ static Cursor cursor(const float* base, int64_t pitch, int64_t cols, int64_t K, int64_t col0, int64_t k0) {
        return {(const char*)(base + k0 * pitch + col0), 4 * ((K - 1 - k0) * pitch + cols - col0), 4 * kBKF32 * pitch};
    }
    __device__ bool has(int, int64_t) const { return true; }                               // lines past the last one read as zeros
};
struct PlainUnit {
    u4 lo, hi;
};
template <typename P>
__device__ __forceinline__ PlainUnit plain_request(const P& p, const Cursor& c) {
    const rsrc_t rs = c.window();
    return {__builtin_amdgcn_raw_buffer_load_b128(rs, (int)p.off, 0, 0), __builtin_amdgcn_raw_buffer_load_b128(rs, (int)(p.off + 16), 0, 0)};
}
template <typename P>
__device__ __forceinline__ void plain_place(const P& p, const PlainUnit& u, int64_t k_left, char* lds) {
    f4 a = __builtin_bit_cast(f4, u.lo), b = __builtin_bit_cast(f4, u.hi);
    if (k_left < kBKF32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) a[e] = p.has(e, k_left) ? a[e] : 0.0f, b[e] = p.has(e + 4, k_left) ? b[e] : 0.0f;
    }
    const Split8 s = split8(a, b);
    *(u4*)(lds + p.place[0]) = s.hi;
    *(u4*)(lds + p.place[1]) = s.mid;
    *(u4*)(lds + p.place[2]) = s.lo;
}

template <bool A_RC, bool B_RC, Epi EPI, bool PLAIN>
__global__ __launch_bounds__(256, 2) void gemm_f32_kernel(GemmArgs p) {
    constexpr int PANELS = EPI == kUp ? 2 : 1;
    static_assert(PANELS == 1 || B_RC, "two panels are read line by line");
    using TA = typename std::conditional<A_RC, TermsRC<128, 1>, TermsKC>::type;
    using TB = typename std::conditional<B_RC, TermsRC<128 / PANELS, PANELS>, TermsKC>::type;
    using PB = typename std::conditional<B_RC, PlainRC<128 / PANELS, PANELS>, PlainKC>::type;
    static_assert(TA::kBytes == 12288 && PANELS * TB::kBytes == 12288, "a wavefront's results are staged in a buffer");
    __shared__ __align__(1024) char a0[12288];
    __shared__ __align__(1024) char a1[12288];
    __shared__ __align__(1024) char a2[12288];
    __shared__ __align__(1024) char b0[12288];
    __shared__ __align__(1024) char b1[12288];
    __shared__ __align__(1024) char b2[12288];

    int range;
    const int tile = tile_of_block(p, range);
    const TilePlace at = place_of(p, tile, 128, 128 / PANELS);
    const Job& q = p.job[at.job];
    const int lane = threadIdx.x % 64, wave = uniform(threadIdx.x / 64), wm = wave / 2, wn = wave % 2;
    const TA ta(q.a_pitch);
    const typename std::conditional<PLAIN, PB, TB>::type tb(q.b_pitch);
    const int slices = (int)((q.K + kBKF32 - 1) / kBKF32);
    const int from = range < 0 ? 0 : (int)((int64_t)slices * range / p.ranges);
    const int here = (range < 0 ? slices : (int)((int64_t)slices * (range + 1) / p.ranges)) - from;
    const int64_t k0 = (int64_t)from * kBKF32;

    f16v big[2][2], small[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) big[i][t][r] = 0.0f, small[i][t][r] = 0.0f;

    // the next slice of each operand to be read: its segment, the slices left there, the contraction indices left in a row
    struct Walk {
        Cursor cur;
        int seg, slices;
        int64_t k_left;
    };
    Walk wa, wb;
    auto enter_a = [&]() {
        const uint16_t* a = q.a + at.group * q.a_group + q.seg_a[wa.seg];
        wa.cur = A_RC ? TA::cursor(a, q.a_pitch, q.a_inner8, q.K, at.m0, k0) : TA::cursor(a, q.a_pitch, q.M, q.a_inner8, at.m0, k0);
        wa.slices = here, wa.k_left = (A_RC ? q.K : q.a_inner8) - k0;
    };
    auto enter_b = [&]() {
        const bool second = PANELS == 1 ? ((q.seg_second >> wb.seg) & 1u) != 0 : wave >= 2;
        if constexpr (PLAIN) {
            const float* b = second ? (const float*)q.b2 + at.group * q.b2_group : (const float*)q.b + at.group * q.b_group;
            wb.cur = PB::cursor(b, q.b_pitch, B_RC ? q.b_inner8 : q.N, q.K, at.n0, k0);
        } else {
            const uint16_t* b = second ? q.b2 + at.group * q.b2_group : q.b + at.group * q.b_group;
            wb.cur = B_RC ? TB::cursor(b, q.b_pitch, q.b_inner8, q.K, at.n0, k0) : TB::cursor(b, q.b_pitch, q.N, q.b_inner8, at.n0, k0);
        }
        wb.slices = here, wb.k_left = (B_RC || PLAIN ? q.K : q.b_inner8) - k0;
    };
    wa.seg = wb.seg = 0;
    enter_a(), enter_b();
    auto next = [&](Walk& w, auto& enter) {
        w.cur.advance();
        w.k_left -= kBKF32;
        if (--w.slices == 0) {
            if (++w.seg < q.segments) enter();
            else w.cur.left = 0, w.cur.step = 0;          // from here on nothing is read
        }
    };
    auto copy = [&](char* la, char* lb) {
        ta.copy(la, 0, wa.cur, wa.k_left);
        next(wa, enter_a);
        if constexpr (!PLAIN) {
            tb.copy(lb, 0, wb.cur, wb.k_left);
            next(wb, enter_b);
        }
    };
    // PLAIN: two slices are under way in registers
    PlainUnit unit[2];
    int64_t unit_k[2];
    auto request = [&](int n) {
        if constexpr (PLAIN) {
            unit[n] = plain_request(tb, wb.cur), unit_k[n] = wb.k_left;
            next(wb, enter_b);
        }
    };
    auto place = [&](int n, char* lb) {
        if constexpr (PLAIN) plain_place(tb, unit[n], unit_k[n], lb);
    };
    int part_a[2][3], part_b[2][3];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int n = 0; n < 3; ++n) {
            part_a[i][n] = TA::lane_part(0, wm * 64 + 32 * i, lane, n);
            part_b[i][n] = PANELS == 2 ? TB::lane_part(i * TB::kBytes, wn * 32, lane, n) : TB::lane_part(0, wn * 64 + 32 * i, lane, n);
        }
    bf16x8 fa[3][2], fb[3][2];
    auto fetch = [&](const char* la, const char* lb, int n) {   // the fragments of a term
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int part = part_b[i][n];                      // opaque: an array plus one offset
            asm volatile("" : "+v"(part));
            fb[n][i] = TB::frag(lb, part);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int part = part_a[i][n];
            asm volatile("" : "+v"(part));
            fa[n][i] = TA::frag(la, part);
        }
    };
    auto multiply = [&](f16v (&to)[2][2], int x, int y) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int t = 0; t < 2; ++t) to[i][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[y][t], fa[x][i], to[i][t], 0, 0, 0);
    };
    const int end = here * q.segments;
    auto barrier = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // In front of slice it's products: its fragments are in registers, and this wavefront's copies of slice it + 1 have landed (those
    // of slice it + 2 may be under way); behind the barrier that holds for all wavefronts, so slice it + 1 can be read and the buffers
    // of slice it overwritten.  Copies past the end (windows of no bytes) keep the count the same.  PLAIN: the terms of slice it + 2
    // are written to the buffer that slice it - 1 had, and slice it + 4 is requested.
    auto slice = [&](char* la, char* lb, char* la1, char* lb1, char* lb2, int n) {
        if constexpr (PLAIN) __builtin_amdgcn_s_waitcnt(0x0077);    // vmcnt(7) lgkmcnt(0): requests of two slices and the copies between
        else __builtin_amdgcn_s_waitcnt(0x0076);                    // vmcnt(6) lgkmcnt(0)
        barrier();
        multiply(small, 2, 0);
        multiply(small, 0, 2);
        copy(la, lb);
        place(n, lb2);
        request(n);
        __builtin_amdgcn_sched_barrier(0);
        fetch(la1, lb1, 2);
        multiply(small, 1, 1);
        multiply(small, 1, 0);
        multiply(small, 0, 1);
        __builtin_amdgcn_sched_barrier(0);
        fetch(la1, lb1, 1);
        multiply(big, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        fetch(la1, lb1, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    copy(a0, b0);
    copy(a1, b1);
    copy(a2, b2);
    request(0);
    request(1);
    place(0, b0);
    request(0);
    place(1, b1);
    request(1);
    if constexpr (PLAIN) __builtin_amdgcn_s_waitcnt(0x0074);        // vmcnt(4) lgkmcnt(0): the second pair of requests
    else __builtin_amdgcn_s_waitcnt(0x0f7c);                        // vmcnt(12)
    barrier();
    fetch(a0, b0, 2);
    fetch(a0, b0, 1);
    fetch(a0, b0, 0);
    // nested, not side by side: the compiler then knows in all but the first of them which requests are behind those it waits for
    for (int it = 0; it < end; it += PLAIN ? 6 : 3) {
        slice(a0, b0, a1, b1, b2, 0);
        if (it + 1 < end) {
            slice(a1, b1, a2, b2, b0, 1);
            if (it + 2 < end) {
                slice(a2, b2, a0, b0, b1, 0);
                if constexpr (PLAIN) {
                    if (it + 3 < end) {
                        slice(a0, b0, a1, b1, b2, 1);
                        if (it + 4 < end) {
                            slice(a1, b1, a2, b2, b0, 0);
                            if (it + 5 < end) slice(a2, b2, a0, b0, b1, 1);
                        }
                    }
                }
            }
        }
    }
    __builtin_amdgcn_s_waitcnt(0x0070);                   // the copies past the end write zeros into LDS
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) big[i][t][r] = fabsf(big[i][t][r]) < INFINITY ? big[i][t][r] + small[i][t][r] : big[i][t][r];
    __syncthreads();                                      // everyone is done with the operands
    float* stage = (float*)(wave == 0 ? a0 : wave == 1 ? a1 : wave == 2 ? a2 : b0);
    write_tile<EPI, true, 128>(big, stage, p, at, tile, range);
}

}  // namespace ffn
}  // namespace ols
