// logits_row.cuh - a row of logits as the kernels read it: 16-byte vectors between single elements, their values, and the bits
// of a mask of allowed tokens.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace rpd {

constexpr float kNoLogit = -__builtin_huge_valf();

template <typename T>
struct Row {
    static constexpr int kVec = 16 / sizeof(T);
    const T *p;
    int V;
    int peel;  // elements before the first 16-byte boundary
    int vecs;  // whole vectors from there
    __device__ Row(const void *base, long long offset, int n) : p(static_cast<const T *>(base) + offset), V(n) {
        peel = min(n, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(p) & 15)) % 16 / sizeof(T)));
        vecs = (n - peel) / kVec;
    }
};

__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float value(__half v) { return __half2float(v); }

__device__ __forceinline__ void unpack(const uint4 &v, float (&z)[4], float) {
    z[0] = __uint_as_float(v.x);
    z[1] = __uint_as_float(v.y);
    z[2] = __uint_as_float(v.z);
    z[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ void unpack(const uint4 &v, float (&z)[8], __nv_bfloat16) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        z[2 * i] = __uint_as_float(w[i] << 16);
        z[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void unpack(const uint4 &v, float (&z)[8], __half) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
        z[2 * i] = f.x;
        z[2 * i + 1] = f.y;
    }
}

// Bits [at, at + 32) of a row of allowed tokens (0 beyond its last word).
__device__ __forceinline__ uint32_t allowed_bits(const uint32_t *mask, int at, int words) {
    const int w = at >> 5;
    const uint32_t lo = mask[w];
    const uint32_t hi = w + 1 < words ? mask[w + 1] : 0u;
    return __funnelshift_r(lo, hi, at & 31);
}

}  // namespace rpd
