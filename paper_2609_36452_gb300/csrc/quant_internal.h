// quant_internal.h - the 4-bit head's parameters and the device helpers that its kernels share.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "rpd_internal.h"

namespace rpd {

constexpr int kQuantMaxD = 32768;       // a row of activations fits a CTA's shared memory
constexpr int kQuantMaxV = 1 << 24;
constexpr int kQuantPairRows = 32;      // matrix rows of a pair of tiles of the packed codes
constexpr int kQuantPadPairs = 4;       // pairs are padded to a multiple of this many (128 rows)

struct QuantParams {
    const uint4 *codes;  // [pairs][blocks][2][32]: a pair's tiles of 16 rows x 64 columns
    const void *meta;    // scales (and zero points), [pairs][groups][2][8][2]
    int pairs;           // pairs of tiles that hold a row
    int blocks;          // 64-column blocks of a row, an even number
    int groups;          // groups of a row, padding included
    int d, V;
    const void *x;       // [rows] rows, x_stride elements apart
    const void *gain;    // [d] or null
    long long x_stride;
    int x_type, x_align, gain_align;  // RPD_TYPE_*; bytes (16, 8, 4, 2) at whose multiples rows (the gain) begin
    int rows, per;       // activation rows; of them, as many as a CTA works on at a time
    float eps;
    void *out;           // [rows] rows of V, out_stride elements apart
    long long out_stride;
    int out_type;
    long long wait_cycles;  // of the wide kernel's waits
    int stall;              // diagnostics: its activations are not asked for
};

template <bool kZeros>
struct MetaVec {
    typedef uint32_t type;  // two 16-bit scales
};
template <>
struct MetaVec<true> {
    typedef uint2 type;  // scale and zero point of a row in each word
};

// cp.async: 16 bytes a lane, past L1; commit closes a group of copies, wait<N> returns once all but the
// last N groups have landed.
__device__ __forceinline__ void copy_async(uint32_t to, const void *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Loads from shared memory by its own addresses (a pointer that the compiler cannot trace back to shared memory is
// read by generic loads, which wait like those from global memory).
__device__ __forceinline__ uint4 lds128(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t at) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
    return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t at) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at));
    return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t at) {
    unsigned short v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at));
    return v;
}
__device__ __forceinline__ void lds_meta(uint32_t at, uint32_t &m) { m = lds32(at); }
__device__ __forceinline__ void lds_meta(uint32_t at, uint2 &m) { m = lds64(at); }

template <bool kF16>
__device__ __forceinline__ float scale_low(uint32_t word) {
    return kF16 ? __low2float(*reinterpret_cast<const __half2 *>(&word)) : __uint_as_float(word << 16);
}
template <bool kF16>
__device__ __forceinline__ float scale_high(uint32_t word) {
    return kF16 ? __high2float(*reinterpret_cast<const __half2 *>(&word)) : __uint_as_float(word & 0xFFFF0000u);
}

// Scales of rows g and g + 8 of a tile, and -z 2^-9 twice as fp16 (z = 8 where no zero points are stored).  A stored
// zero point is that fp16 number in the upper half of its row's word.
constexpr uint32_t kMinusZeroDefault = 0xA400A400u;  // -2^-6 twice

template <bool kF16>
__device__ __forceinline__ void unpack_meta(uint32_t m, float &s_lo, float &s_hi, uint32_t &z_lo, uint32_t &z_hi) {
    s_lo = scale_low<kF16>(m);
    s_hi = scale_high<kF16>(m);
    z_lo = z_hi = kMinusZeroDefault;
}
template <bool kF16>
__device__ __forceinline__ void unpack_meta(uint2 m, float &s_lo, float &s_hi, uint32_t &z_lo, uint32_t &z_hi) {
    s_lo = scale_low<kF16>(m.x);
    s_hi = scale_low<kF16>(m.y);
    z_lo = __byte_perm(m.x, 0, 0x3232);
    z_hi = __byte_perm(m.y, 0, 0x3232);
}

// Pair i (columns 2i, 2i + 1) of a word of codes as two fp16 numbers: masked in place, they are the subnormals q 2^-24
// (pairs 0 and 2) and q 2^-20 (1 and 3), exact.
__device__ __forceinline__ uint32_t code_pair(uint32_t word, int i) {
    return (i < 2 ? word : word >> 8) & (i & 1 ? 0x00F000F0u : 0x000F000Fu);
}

// The pair as (q - z) 2^-9, exact too (one fused multiply-add for both).
__device__ __forceinline__ uint32_t weight_pair(uint32_t word, int i, uint32_t minus_zero) {
    const uint32_t q = code_pair(word, i), up = i & 1 ? 0x68006800u : 0x78007800u;  // 2^11, 2^15
    const __half2 r = __hfma2(*reinterpret_cast<const __half2 *>(&q), *reinterpret_cast<const __half2 *>(&up),
                              *reinterpret_cast<const __half2 *>(&minus_zero));
    return *reinterpret_cast<const uint32_t *>(&r);
}

// Elements [col, col + 8) of a row of d 16-bit elements, zero beyond its end; `align`: bytes (16, 8, 4 or 2) at whose
// multiples every row begins.
template <typename T>
__device__ __forceinline__ uint4 load_chunk(const T *row, int col, int d, int align) {
    if (col + 8 <= d && align > 2) {
        if (align == 16) return *reinterpret_cast<const uint4 *>(row + col);
        if (align == 8) {
            const uint2 *v = reinterpret_cast<const uint2 *>(row + col);
            return make_uint4(v[0].x, v[0].y, v[1].x, v[1].y);
        }
        const uint32_t *v = reinterpret_cast<const uint32_t *>(row + col);
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
    const uint16_t *e = reinterpret_cast<const uint16_t *>(row);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = col + 2 * i;
        w[i] = (c < d ? e[c] : 0u) | (c + 1 < d ? static_cast<uint32_t>(e[c + 1]) : 0u) << 16;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ float2 pair_value(uint32_t v, __nv_bfloat16) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}
__device__ __forceinline__ float2 pair_value(uint32_t v, __half) {
    return __half22float2(*reinterpret_cast<const __half2 *>(&v));
}
__device__ __forceinline__ float2 pair_round(float2 f, __nv_bfloat16) {
    return __bfloat1622float2(__floats2bfloat162_rn(f.x, f.y));
}
__device__ __forceinline__ float2 pair_round(float2 f, __half) { return __half22float2(__floats2half2_rn(f.x, f.y)); }

// Eight columns of u from those of x, with a gain rn(g x): the operand of a readout with a norm is rounded to
// the activations' type (the product of two such numbers is exact in fp32), its factor rho is not.  Returns
// the sum of x^2.
template <typename T>
__device__ __forceinline__ float make_u(const uint4 &x, bool has_gain, const uint4 &gain, float2 (&u)[4]) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w}, gw[4] = {gain.x, gain.y, gain.z, gain.w};
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        u[i] = pair_value(w[i], T());
        if (has_gain) {
            const float2 gf = pair_value(gw[i], T());
            ss = fmaf(u[i].x, u[i].x, fmaf(u[i].y, u[i].y, ss));
            u[i] = pair_round(make_float2(u[i].x * gf.x, u[i].y * gf.y), T());
        }
    }
    return ss;
}

// The power of two at or below x (1 for 0).
__device__ __forceinline__ int exponent_of(float x) { return x > 0.f ? ilogbf(x) : 0; }

// A row's factor rho 2^E under a norm, rho = (ss / d + eps)^-1/2, as it usually is.  ss: the sum of x^2 as make_u adds it
// up, top: the largest |u|.
__device__ __forceinline__ float norm_factor(float ss, float d, float eps, int E) { return ldexpf(rsqrtf(ss / d + eps), E); }

// Whether it is not: fp32 has not held the sum (it is infinite, or below 2^-90, where squares under 2^-126 may be what counts;
// above, what 32768 of these lose is below 2^-44 of it), or rho 2^E may lie under 2^-126 (rho itself is at least 2^-64).
// Rows of zeros, such as a batch is padded with, have products of 0 whatever finite rho is.
__device__ __forceinline__ bool norm_unusual(float ss, float top, float eps, int E) {
    return (!(ss >= 0x1p-90f && ss <= 3e38f) || E < -62) && ss == ss && !(top == 0.f && eps > 0.f);
}

// Then the warp, all of it, goes through the row twice more, for (x 2^-F)^2 with F the exponent of its largest |x|.  E is
// raised until rho 2^E is a normal number: smaller, it would lose bits that a logit has.  (Activations are then
// smaller by as much and off by up to 2^-39 2^E, which times rho is some 2^-165: under half of fp32's smallest number for
// weights of a sum below 2^15.)
struct NormFactor {
    float factor;
    int E;
};
template <typename T>
__device__ __noinline__ NormFactor norm_factor_unusual(const T *x, int chunks, int d, int align, float eps, float top, int E) {
    const int lane = threadIdx.x & 31;
    float most = 0.f;
    for (int c = lane; c < chunks; c += 32) {
        const uint4 v = load_chunk(x, c * 8, d, align);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = pair_value(w[i], T());
            most = fmaxf(most, fmaxf(fabsf(f.x), fabsf(f.y)));
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    if (top == 0.f) return {most > 0.f ? 1.f : rsqrtf(eps), E};  // (eps = 0: products of 0, and 0 / 0 for a row of zeros)
    const int F = exponent_of(fminf(most, 3e38f));
    const float f0 = ldexpf(1.f, -F / 2), f1 = ldexpf(1.f, -F + F / 2);  // (2^-F itself may lie outside fp32)
    float sum = 0.f;
    for (int c = lane; c < chunks; c += 32) {
        const uint4 v = load_chunk(x, c * 8, d, align);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = pair_value(w[i], T());
            const float a = f.x * f0 * f1, b = f.y * f0 * f1;
            sum = fmaf(a, a, fmaf(b, b, sum));
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    // rho = 2^-F (sum / d + eps 2^-2F)^-1/2, the sum at least 1; where eps 2^-2F leaves fp32, eps is all that counts
    const float e = ldexpf(eps, -2 * F);
    const bool held = e <= 3e38f;
    const float r = held ? rsqrtf(sum / static_cast<float>(d) + e) : rsqrtf(eps);
    const int R = held ? -F : 0;  // rho = r 2^R
    E = max(E, -126 - R - ilogbf(r));
    return {ldexpf(r, R + E), E};
}

// Activations as the tensor core gets them: u 2^(14 - E) in fp16, E the exponent of the row's largest u.  Exact from 2^-28
// of the largest element on; a smaller one is off by at most 2^-39 of the largest.
__device__ __forceinline__ void scale_u(const float2 (&u)[4], int E, uint4 &out) {
    const int e = 14 - E;  // in two factors: the power itself may lie outside fp32
    const float f0 = ldexpf(1.f, e / 2), f1 = ldexpf(1.f, e - e / 2);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 h = __floats2half2_rn(u[i].x * f0 * f1, u[i].y * f0 * f1);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    out = make_uint4(w[0], w[1], w[2], w[3]);
}

// What a row's sums are multiplied with besides 2^E rho: 2^(9 - 14).
constexpr float kWeightFactor = 0.03125f;

__device__ __forceinline__ void store_out(void *out, int type, long long at, float v) {
    if (type == RPD_TYPE_F32)
        static_cast<float *>(out)[at] = v;
    else if (type == RPD_TYPE_BF16)
        static_cast<__nv_bfloat16 *>(out)[at] = __float2bfloat16_rn(v);
    else
        static_cast<__half *>(out)[at] = __float2half_rn(v);
}

// The kernel for more rows (k_quant_wide.cu): as many passes over the codes as there are `kWideMaxRows` rows.
constexpr int kWideMaxRows = 64;
// maps: boxes of 4 and of 2 pairs x 128 columns of the packed codes.
long long quant_wide_workspace(int rows, int blocks, int pairs, int num_sms);
cudaError_t quant_wide(const CUtensorMap *maps, const QuantParams &p, int group, bool zeros, bool f16, int num_sms,
                       void *workspace, cudaStream_t s);

}  // namespace rpd
