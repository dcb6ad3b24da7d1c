// quant_internal.h - the 4-bit head's parameters and the device helpers that its kernels share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "rpd_internal.h"

namespace rpd {

constexpr int kQuantMaxD = 65536;       // a row of activations fits a CTA's shared memory
constexpr int kQuantMaxV = 1 << 24;
constexpr int kQuantTileRows = 16;      // matrix rows of a tile of the packed codes
constexpr int kQuantPadTiles = 8;       // tiles are padded to a multiple of this many (128 rows)

struct QuantParams {
    const uint4 *codes;  // [row_tiles][blocks][32]
    const void *meta;    // scales (and zero points), [row_tiles][groups][8][2]
    int row_tiles;       // tiles of 16 matrix rows that hold a row
    int blocks;          // 64-column blocks of a row, a whole number of groups
    int groups;          // groups of a row, padding included
    int scale_f16;       // the scales are fp16, else bf16
    int d, V;
    const void *x;       // [rows] rows, x_stride elements apart
    const void *gain;    // [d] or null
    long long x_stride;
    int x_type, x_vectors, gain_vectors;  // RPD_TYPE_*; rows (the gain) can be read 16 bytes at a time
    int rows;
    float eps;
    void *out;           // [rows] rows of V, out_stride elements apart
    long long out_stride;
    int out_type;
};

constexpr uint32_t kBiasBf16 = 0x43004300u;  // 128: adding q in 0..15 is setting its lowest four bits
constexpr uint32_t kBiasHalf = 0x64006400u;  // 1024, likewise
constexpr uint32_t kZeroDefault = 0x00080008u;

template <bool kZeros>
struct MetaVec {
    typedef uint32_t type;  // two 16-bit scales
};
template <>
struct MetaVec<true> {
    typedef uint2 type;  // scale and zero point of a row in each word
};

// Codes are read once a call: their lines are not kept in L1.
__device__ __forceinline__ uint4 ld_stream(const uint4 *p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}

__device__ __forceinline__ float scale_value(uint32_t bits16, int f16) {
    return f16 ? __half2float(__ushort_as_half(static_cast<unsigned short>(bits16)))
               : __uint_as_float(bits16 << 16);
}

template <typename T>
constexpr uint32_t quant_bias() {
    return kBiasBf16;
}
template <>
constexpr uint32_t quant_bias<__half>() {
    return kBiasHalf;
}

// Scales of rows g and g + 8 of a tile, and their zero points with the bias of the dequantisation.
template <typename T>
__device__ __forceinline__ void unpack_meta(uint32_t m, int f16, float &s_lo, float &s_hi, uint32_t &z_lo,
                                            uint32_t &z_hi) {
    s_lo = scale_value(m & 0xFFFFu, f16);
    s_hi = scale_value(m >> 16, f16);
    z_lo = z_hi = quant_bias<T>() | kZeroDefault;
}
template <typename T>
__device__ __forceinline__ void unpack_meta(uint2 m, int f16, float &s_lo, float &s_hi, uint32_t &z_lo,
                                            uint32_t &z_hi) {
    s_lo = scale_value(m.x & 0xFFFFu, f16);
    s_hi = scale_value(m.y & 0xFFFFu, f16);
    z_lo = quant_bias<T>() | (m.x >> 16) * 0x00010001u;
    z_hi = quant_bias<T>() | (m.y >> 16) * 0x00010001u;
}

// Two neighbouring columns (pair i of a word) of the codes as q - z in the activations' type; exact.
template <typename T>
__device__ __forceinline__ uint32_t dequant_pair(uint32_t word, int i, uint32_t bias_zero);
template <>
__device__ __forceinline__ uint32_t dequant_pair<__nv_bfloat16>(uint32_t word, int i, uint32_t bias_zero) {
    const uint32_t v = ((word >> (4 * i)) & 0x000F000Fu) | kBiasBf16;
    const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&v),
                                     *reinterpret_cast<const __nv_bfloat162 *>(&bias_zero));
    return *reinterpret_cast<const uint32_t *>(&r);
}
template <>
__device__ __forceinline__ uint32_t dequant_pair<__half>(uint32_t word, int i, uint32_t bias_zero) {
    const uint32_t v = ((word >> (4 * i)) & 0x000F000Fu) | kBiasHalf;
    const __half2 r =
        __hsub2(*reinterpret_cast<const __half2 *>(&v), *reinterpret_cast<const __half2 *>(&bias_zero));
    return *reinterpret_cast<const uint32_t *>(&r);
}

// Elements [col, col + 8) of a row of d 16-bit elements, zero beyond its end.
template <typename T>
__device__ __forceinline__ uint4 load_chunk(const T *row, int col, int d, int vectors) {
    if (vectors && col + 8 <= d) return *reinterpret_cast<const uint4 *>(row + col);
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
__device__ __forceinline__ uint32_t pair_round(float2 f, __nv_bfloat16) {
    const __nv_bfloat162 r = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ uint32_t pair_round(float2 f, __half) {
    const __half2 r = __floats2half2_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t *>(&r);
}

// v = rn(v * gain), returning the sum of v^2 before: the operand of a readout with a norm is
// rounded to the activations' type (the product of two such numbers is exact in fp32), the factor rho is
// not.
template <typename T>
__device__ __forceinline__ float norm_chunk(uint4 &v, const uint4 &gain) {
    uint32_t *w = reinterpret_cast<uint32_t *>(&v);
    const uint32_t *gw = reinterpret_cast<const uint32_t *>(&gain);
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 x = pair_value(w[i], T()), gf = pair_value(gw[i], T());
        ss = fmaf(x.x, x.x, fmaf(x.y, x.y, ss));
        w[i] = pair_round(make_float2(x.x * gf.x, x.y * gf.y), T());
    }
    return ss;
}

__device__ __forceinline__ void store_out(void *out, int type, long long at, float v) {
    if (type == RPD_TYPE_F32)
        static_cast<float *>(out)[at] = v;
    else if (type == RPD_TYPE_BF16)
        static_cast<__nv_bfloat16 *>(out)[at] = __float2bfloat16_rn(v);
    else
        static_cast<__half *>(out)[at] = __float2half_rn(v);
}

}  // namespace rpd
