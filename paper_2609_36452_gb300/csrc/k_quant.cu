// k_quant.cu - the 4-bit head: products of a few activations with a [V][d] matrix of 4-bit codes,
// a scale (and optionally a zero point) for every `group` columns of a row.
//
//   y[r][v] = rho_r * sum_G s[v][G] * sum_{k in G} (q[v][k] - z[v][G]) * u[r][k]
//
// with u = x and rho = 1, or - with a gain g - the readout's normalisation (App. A.2):
// u = rn(g * x) in the activations' type and rho_r = (mean_k x^2 + eps)^-1/2, applied after the
// sum, as the 16-bit head does it.
//
// Precision.  q - z is a whole number of at most 5 bits: exact in bf16 and fp16, and so is its product
// with u in fp32.  A group's products are summed in fp32 by the tensor core, the sum is multiplied by
// the scale and added to the row's running sum in fp32.  Scales are never rounded into the weights.
//
// What bounds it: reading the codes once.  One row of a 126464 x 4096 head is 259 MB of codes and 8 MB
// of scales.  Dequantising on the way to the multipliers costs about 1.4 instructions a weight and lane
// (shift, mask and bias in one LOP3, subtraction in pairs), 20 us of the device's issue slots.
//
// k_quant_rows: up to 16 rows.  A warp multiplies tiles of 16 matrix rows (M of the m16n8k16 MMA) by 8
// or 16 activation rows (N), so that a dequantised fragment is used for all of them from registers.  The
// codes are stored in fragment order, 512 contiguous bytes for 16 rows x 64 columns, which every lane
// reads as one 16-byte vector, several of them ahead.  A CTA owns a range of tiles and its warps
// divide the range's column blocks evenly, over tile borders: one tile's row sums then come from
// several warps and are joined in shared memory in warp order.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>

#include "op_host.h"
#include "ptx.cuh"
#include "quant_internal.h"

namespace rpd {
namespace {

// ------------------------------------------------------------------------------ layout of the codes

// One 16-byte vector of the packed codes a thread: the place of lane (t, g) of tile (vt, kb) holds
// rows 16 vt + g (words 0, 1) and 16 vt + g + 8 (words 2, 3), columns 64 kb + 8 t + {0..7} (words 0, 2)
// and 32 columns further (words 1, 3).  Nibble i of a word is column 2i, nibble i + 4 column 2i + 1, so
// that (word >> 4i) & 0x000F000F is a pair of neighbouring columns in the halves of a register.
__global__ void k_quant_pack(const uint8_t *codes, uint4 *packed, int V, int d, int tiles, int blocks) {
    const long long n = static_cast<long long>(tiles) * blocks * 32;
    const int row_bytes = (d + 1) / 2;
    for (long long i = blockIdx.x * static_cast<long long>(blockDim.x) + threadIdx.x; i < n;
         i += static_cast<long long>(gridDim.x) * blockDim.x) {
        const int place = static_cast<int>(i & 31), t = place >> 3, g = place & 7;
        const long long tile = i >> 5;
        const int kb = static_cast<int>(tile % blocks);
        const int vt = static_cast<int>(tile / blocks);
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int v = vt * 16 + g + (j >> 1) * 8;
            const int byte = (kb * 64 + (j & 1) * 32 + t * 8) / 2;
            uint32_t word = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const uint32_t c =
                    v < V && byte + b < row_bytes ? codes[static_cast<long long>(v) * row_bytes + byte + b] : 0u;
                word |= (c & 15u) << (4 * b) | (c >> 4) << (16 + 4 * b);
            }
            w[j] = word;
        }
        packed[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// Scales (and zero points) in the order of the tiles: [tile][group][g][2] for rows g and g + 8.  With
// zero points an entry is 32 bits: the scale, and the zero point in the upper half.
template <bool kZeros>
__global__ void k_quant_pack_scales(const uint16_t *scales, const uint8_t *zeros, void *packed, int V, int groups,
                                    int tiles, int padded_groups) {
    const long long n = static_cast<long long>(tiles) * padded_groups * 16;
    for (long long i = blockIdx.x * static_cast<long long>(blockDim.x) + threadIdx.x; i < n;
         i += static_cast<long long>(gridDim.x) * blockDim.x) {
        const int hi = static_cast<int>(i & 1), g = static_cast<int>(i >> 1) & 7;
        const long long tg = i >> 4;
        const int grp = static_cast<int>(tg % padded_groups);
        const int v = static_cast<int>(tg / padded_groups) * 16 + hi * 8 + g;
        const bool in = v < V && grp < groups;
        const long long at = static_cast<long long>(v) * groups + grp;
        const uint32_t s = in ? scales[at] : 0u;
        if (kZeros)
            static_cast<uint32_t *>(packed)[i] = s | (in ? static_cast<uint32_t>(zeros[at]) & 15u : 8u) << 16;
        else
            static_cast<uint16_t *>(packed)[i] = static_cast<uint16_t>(s);
    }
}

// ------------------------------------------------------------------------------ few rows

constexpr int kRowsWarps = 16;
constexpr int kRowsThreads = 32 * kRowsWarps;

__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1,
                                          __nv_bfloat16) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9},"
        " {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9},"
        " {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The lane's part of the activations into shared memory: rows of u, `row_bytes` apart, zero beyond
// column d, and the factors rho.  Every thread takes part; ends with a barrier.
template <typename T>
__device__ void stage_rows(const QuantParams &p, uint8_t *xs, int row_bytes, float *red, float *rho) {
    const T *gain = static_cast<const T *>(p.gain);
    const int chunks = p.blocks * 8;  // of 8 elements
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int r = 0; r < p.rows; ++r) {
        const T *x = static_cast<const T *>(p.x) + r * p.x_stride;
        float ss = 0.f;
        for (int c = threadIdx.x; c < chunks; c += kRowsThreads) {
            uint4 v = load_chunk(x, c * 8, p.d, p.x_vectors);
            if (gain) ss += norm_chunk<T>(v, load_chunk(gain, c * 8, p.d, p.gain_vectors));
            *reinterpret_cast<uint4 *>(xs + static_cast<size_t>(r) * row_bytes + c * 16) = v;
        }
        if (gain) {
#pragma unroll
            for (int o = 16; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            if (lane == 0) red[r * kRowsWarps + warp] = ss;
        }
    }
    __syncthreads();
    if (threadIdx.x < p.rows) {
        float ss = 0.f;
        if (gain)
            for (int w = 0; w < kRowsWarps; ++w) ss += red[threadIdx.x * kRowsWarps + w];
        rho[threadIdx.x] = gain ? rsqrtf(ss / static_cast<float>(p.d) + p.eps) : 1.f;
    }
    __syncthreads();
}

// A finished tile's logits: fragment element (g, 2t) of the MMA's result is matrix row g, activation 2t.
template <int kN8>
__device__ __forceinline__ void store_tile(const QuantParams &p, int tile, const float (&run)[kN8][4],
                                           const float *rho, int g, int t) {
#pragma unroll
    for (int n = 0; n < kN8; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = n * 8 + 2 * t + (i & 1), v = tile * kQuantTileRows + g + (i >> 1) * 8;
            if (r < p.rows && v < p.V) store_out(p.out, p.out_type, r * p.out_stride + v, run[n][i] * rho[r]);
        }
}

template <typename T, int kGroup, int kN8, bool kZeros>
__global__ void __launch_bounds__(kRowsThreads, 1) k_quant_rows(const QuantParams p) {
    constexpr int kUnitBlocks = kGroup == 128 ? 2 : 1;  // 64-column blocks of a unit of work
    constexpr int kUnitGroups = kGroup == 32 ? 2 : 1;
    constexpr int kAhead = kGroup == 128 ? 4 : 6;       // units whose codes are in flight
    typedef typename MetaVec<kZeros>::type Meta;        // scales (and zero points) of rows g and g + 8
    extern __shared__ __align__(128) uint8_t smem[];
    float *join = reinterpret_cast<float *>(smem);  // [warp][4 kN8][lane]
    float *red = join + kRowsWarps * 4 * kN8 * 32;
    float *rho = red + 16 * kRowsWarps;
    uint8_t *xs = reinterpret_cast<uint8_t *>(rho + 16);
    // a row and 64 bytes: the two rows that a quarter of a warp reads at once lie in different banks
    const int row_bytes = p.blocks * 128 + 64;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;

    pdl_trigger();
    // this CTA's tiles, this warp's units of them
    const int tile0 = static_cast<int>(static_cast<long long>(p.row_tiles) * blockIdx.x / gridDim.x);
    const int tile1 = static_cast<int>(static_cast<long long>(p.row_tiles) * (blockIdx.x + 1) / gridDim.x);
    const int per_tile = p.blocks / kUnitBlocks;
    const int units = (tile1 - tile0) * per_tile;
    const int u0 = units * warp / kRowsWarps, u1 = units * (warp + 1) / kRowsWarps;
    const uint4 *codes = p.codes + (static_cast<long long>(tile0) * p.blocks) * 32 + t * 8 + g;
    const Meta *meta = static_cast<const Meta *>(p.meta) + static_cast<long long>(tile0) * p.groups * 8 + g;

    uint4 code[kAhead][kUnitBlocks];
    Meta m[kAhead][kUnitGroups];
    auto fetch = [&](int slot, int u) {
        if (u < u1) {
#pragma unroll
            for (int b = 0; b < kUnitBlocks; ++b) code[slot][b] = ld_stream(codes + static_cast<long long>(u * kUnitBlocks + b) * 32);
#pragma unroll
            for (int k = 0; k < kUnitGroups; ++k) m[slot][k] = __ldg(meta + static_cast<long long>(u * kUnitGroups + k) * 8);
        }
    };
#pragma unroll
    for (int s = 0; s < kAhead; ++s) fetch(s, u0 + s);

    pdl_wait();  // the weights were laid out long ago; the activations may be the predecessor's
    stage_rows<T>(p, xs, row_bytes, red, rho);

    float run[kN8][4];
#pragma unroll
    for (int n = 0; n < kN8; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) run[n][i] = 0.f;
    int in_tile = u0 % per_tile, tile = tile0 + u0 / per_tile;
    bool head = in_tile != 0;  // the tile at hand was begun by an earlier warp
    const uint8_t *xrow = xs + static_cast<size_t>(g) * row_bytes + t * 16;

    for (int u = u0; u < u1; u += kAhead) {
#pragma unroll
        for (int s = 0; s < kAhead; ++s) {
            if (u + s < u1) {
#pragma unroll
                for (int k = 0; k < kUnitGroups; ++k) {
                    float c[kN8][4];
#pragma unroll
                    for (int n = 0; n < kN8; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) c[n][i] = 0.f;
                    float s_lo, s_hi;
                    uint32_t z_lo, z_hi;
                    unpack_meta<T>(m[s][k], p.scale_f16, s_lo, s_hi, z_lo, z_hi);
                    // 32-column halves of this group: (block, half)
#pragma unroll
                    for (int h = 0; h < kGroup / 32; ++h) {
                        const int b = kGroup == 32 ? 0 : h >> 1, half = kGroup == 32 ? k : h & 1;
                        const uint4 q = code[s][b];
                        const uint32_t lo = half ? q.y : q.x, hi = half ? q.w : q.z;
                        uint4 xv[kN8];
#pragma unroll
                        for (int n = 0; n < kN8; ++n) {
                            xv[n] = make_uint4(0, 0, 0, 0);
                            if (n * 8 + g < p.rows)
                                xv[n] = *reinterpret_cast<const uint4 *>(
                                    xrow + static_cast<size_t>(n) * 8 * row_bytes +
                                    (in_tile * kUnitBlocks + b) * 128 + half * 64);
                        }
#pragma unroll
                        for (int step = 0; step < 2; ++step) {
                            const uint32_t a[4] = {dequant_pair<T>(lo, 2 * step, z_lo), dequant_pair<T>(hi, 2 * step, z_hi),
                                                   dequant_pair<T>(lo, 2 * step + 1, z_lo),
                                                   dequant_pair<T>(hi, 2 * step + 1, z_hi)};
#pragma unroll
                            for (int n = 0; n < kN8; ++n)
                                mma_16816(c[n], a, step ? xv[n].z : xv[n].x, step ? xv[n].w : xv[n].y, T());
                        }
                    }
#pragma unroll
                    for (int n = 0; n < kN8; ++n) {
                        run[n][0] = fmaf(c[n][0], s_lo, run[n][0]);
                        run[n][1] = fmaf(c[n][1], s_lo, run[n][1]);
                        run[n][2] = fmaf(c[n][2], s_hi, run[n][2]);
                        run[n][3] = fmaf(c[n][3], s_hi, run[n][3]);
                    }
                }
                fetch(s, u + s + kAhead);
                if (++in_tile == per_tile) {  // the tile's last columns
                    if (head) {
#pragma unroll
                        for (int n = 0; n < kN8; ++n)
#pragma unroll
                            for (int i = 0; i < 4; ++i) join[((warp * kN8 + n) * 4 + i) * 32 + lane] = run[n][i];
                    } else {
                        store_tile<kN8>(p, tile, run, rho, g, t);
                    }
                    head = false;
                    in_tile = 0;
                    ++tile;
#pragma unroll
                    for (int n = 0; n < kN8; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) run[n][i] = 0.f;
                }
            }
        }
    }
    if (head && in_tile) {  // the warp's whole range lies inside one tile
#pragma unroll
        for (int n = 0; n < kN8; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) join[((warp * kN8 + n) * 4 + i) * 32 + lane] = run[n][i];
    }
    __syncthreads();
    if (!head && in_tile) {  // a tile that this warp began and later warps went on with
        const int end = (tile - tile0 + 1) * per_tile;
        for (int w = warp + 1; w < kRowsWarps; ++w) {
            if (units * w / kRowsWarps >= end) break;  // (a warp without units in the tile has left zeros)
#pragma unroll
            for (int n = 0; n < kN8; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) run[n][i] += join[((w * kN8 + n) * 4 + i) * 32 + lane];
        }
        store_tile<kN8>(p, tile, run, rho, g, t);
    }
}

constexpr int kRowsMax = 16;                 // activation rows of a launch
constexpr int kRowsSmem = 224 * 1024;        // of the 227 KB a CTA may have

size_t rows_smem(int n8, int rows, int blocks) {
    return static_cast<size_t>(kRowsWarps) * 4 * n8 * 32 * 4 + 16 * kRowsWarps * 4 + 16 * 4 +
           static_cast<size_t>(rows) * (blocks * 128 + 64);
}

template <typename T, int kGroup, int kN8, bool kZeros>
cudaError_t launch_rows(const QuantParams &p, int num_sms, cudaStream_t s) {
    void (*kernel)(QuantParams) = k_quant_rows<T, kGroup, kN8, kZeros>;
    // (cheap, and per device: set on every call)
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRowsSmem);
    if (e != cudaSuccess) return e;
    return launch_pdl(kernel, dim3(std::min(num_sms, p.row_tiles)), dim3(kRowsThreads),
                      rows_smem(kN8, p.rows, p.blocks), s, p);
}

template <typename T, int kGroup>
cudaError_t launch_rows_group(const QuantParams &p, bool zeros, int num_sms, cudaStream_t s) {
    if (p.rows <= 8)
        return zeros ? launch_rows<T, kGroup, 1, true>(p, num_sms, s) : launch_rows<T, kGroup, 1, false>(p, num_sms, s);
    return zeros ? launch_rows<T, kGroup, 2, true>(p, num_sms, s) : launch_rows<T, kGroup, 2, false>(p, num_sms, s);
}

template <typename T>
cudaError_t launch_rows_type(const QuantParams &p, int group, bool zeros, int num_sms, cudaStream_t s) {
    return group == 32   ? launch_rows_group<T, 32>(p, zeros, num_sms, s)
           : group == 64 ? launch_rows_group<T, 64>(p, zeros, num_sms, s)
                         : launch_rows_group<T, 128>(p, zeros, num_sms, s);
}

}  // namespace
}  // namespace rpd

using namespace rpd;

struct rpd_quant {
    int d = 0, V = 0, group = 0;
    int device = 0, num_sms = 0;
    int row_tiles = 0, pad_tiles = 0, blocks = 0, groups = 0;  // groups: padding included
    uint4 *codes = nullptr;
    void *meta = nullptr;
    bool set = false, zeros = false, scale_f16 = false;
};

extern "C" {

rpd_quant *rpd_quant_create(int d, int V, int group) {
    if (d < 1 || V < 1) {
        op_fail(RPD_ERR_INVALID_ARGUMENT, "d and V must be >= 1 (got %d, %d)", d, V);
        return nullptr;
    }
    if (group != 32 && group != 64 && group != 128) {
        op_fail(RPD_ERR_UNSUPPORTED, "group must be 32, 64 or 128 (got %d)", group);
        return nullptr;
    }
    if (d > kQuantMaxD || V > kQuantMaxV) {
        op_fail(RPD_ERR_UNSUPPORTED, "d must be <= %d and V <= %d (got %d, %d)", kQuantMaxD, kQuantMaxV, d, V);
        return nullptr;
    }
    rpd_quant *q = new (std::nothrow) rpd_quant();
    if (!q) {
        op_fail(RPD_ERR_OUT_OF_MEMORY, "out of host memory");
        return nullptr;
    }
    cudaError_t e = cudaGetDevice(&q->device);
    if (e == cudaSuccess) e = cudaSetDevice(q->device);  // binds the primary context to this thread
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&q->num_sms, cudaDevAttrMultiProcessorCount, q->device);
    if (e != cudaSuccess) {
        op_cuda_fail(e, "device query");
        delete q;
        return nullptr;
    }
    if (check_device(q->device) != RPD_OK) {
        delete q;
        return nullptr;
    }
    q->d = d;
    q->V = V;
    q->group = group;
    const int unit = group > 64 ? group : 64;
    q->blocks = (d + unit - 1) / unit * (unit / 64);
    q->groups = q->blocks * 64 / group;
    q->row_tiles = (V + kQuantTileRows - 1) / kQuantTileRows;
    q->pad_tiles = (q->row_tiles + kQuantPadTiles - 1) / kQuantPadTiles * kQuantPadTiles;
    return q;
}

int rpd_quant_set_weights(rpd_quant *q, const void *codes, const void *scales, int scale_type, const void *zeros,
                          void *stream_ptr) {
    if (!q || !codes || !scales) return op_fail(RPD_ERR_INVALID_ARGUMENT, "null argument");
    if (scale_type != RPD_TYPE_BF16 && scale_type != RPD_TYPE_F16)
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "scales must be bf16 or fp16");
    if (!aligned_to(scales, 2)) return op_fail(RPD_ERR_INVALID_ARGUMENT, "scales must be 2-byte aligned");
    DeviceGuard dg(q->device);
    if (dg.err != cudaSuccess) return op_cuda_fail(dg.err, "cudaSetDevice");
    if (!pointer_usable(codes, q->device, false) || !pointer_usable(scales, q->device, false) ||
        (zeros && !pointer_usable(zeros, q->device, false)))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "codes, scales and zeros must be device memory on the head's device");
    cudaStream_t s = static_cast<cudaStream_t>(stream_ptr);
    const size_t code_bytes = static_cast<size_t>(q->pad_tiles) * q->blocks * 512;
    const size_t meta_bytes = static_cast<size_t>(q->pad_tiles) * q->groups * (zeros ? 64 : 32);
    // Freeing the previous layout waits for the device: no call may still be reading it.
    q->set = false;
    if (q->codes) cudaFree(q->codes);
    if (q->meta) cudaFree(q->meta);
    q->codes = nullptr;
    q->meta = nullptr;
    cudaError_t e = cudaMalloc(&q->codes, code_bytes);
    if (e == cudaSuccess) e = cudaMalloc(&q->meta, meta_bytes);
    if (e == cudaSuccess) {
        const int groups = (q->d + q->group - 1) / q->group;
        k_quant_pack<<<q->num_sms * 8, 256, 0, s>>>(static_cast<const uint8_t *>(codes), q->codes, q->V, q->d,
                                                    q->pad_tiles, q->blocks);
        if (zeros)
            k_quant_pack_scales<true><<<q->num_sms * 4, 256, 0, s>>>(static_cast<const uint16_t *>(scales),
                                                                     static_cast<const uint8_t *>(zeros), q->meta,
                                                                     q->V, groups, q->pad_tiles, q->groups);
        else
            k_quant_pack_scales<false><<<q->num_sms * 4, 256, 0, s>>>(static_cast<const uint16_t *>(scales), nullptr,
                                                                      q->meta, q->V, groups, q->pad_tiles, q->groups);
        e = cudaGetLastError();
        if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    }
    if (e != cudaSuccess) {
        if (q->codes) cudaFree(q->codes);
        if (q->meta) cudaFree(q->meta);
        q->codes = nullptr;
        q->meta = nullptr;
        return op_cuda_fail(e, "layout of the 4-bit weights");
    }
    q->zeros = zeros != nullptr;
    q->scale_f16 = scale_type == RPD_TYPE_F16;
    q->set = true;
    return RPD_OK;
}

int64_t rpd_quant_workspace(const rpd_quant *q, int rows) {
    if (!q || rows < 0) {
        op_fail(RPD_ERR_INVALID_ARGUMENT, "null head or negative rows");
        return -1;
    }
    return 0;
}

int rpd_quant_logits(const rpd_quant *q, const void *x, int x_type, int64_t x_stride, int rows, const void *gain,
                     float eps, void *out, int out_type, int64_t out_stride, void *workspace,
                     int64_t workspace_bytes, void *stream_ptr) {
    if (!q) return op_fail(RPD_ERR_INVALID_ARGUMENT, "null head");
    if (!q->set) return op_fail(RPD_ERR_NO_HEAD, "rpd_quant_set_weights has not been called");
    if (x_type != RPD_TYPE_BF16 && x_type != RPD_TYPE_F16)
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "x must be bf16 or fp16");
    if (!type_size(out_type)) return op_fail(RPD_ERR_INVALID_ARGUMENT, "out must be bf16, fp16 or fp32");
    if (rows < 0) return op_fail(RPD_ERR_INVALID_ARGUMENT, "rows must be >= 0");
    if (rows == 0) return RPD_OK;
    if (!x || !out) return op_fail(RPD_ERR_INVALID_ARGUMENT, "null buffer");
    if (rows > 1 && (x_stride < q->d || out_stride < q->V))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "rows overlap: x_stride must be >= %d and out_stride >= %d", q->d, q->V);
    if (gain && (!(eps >= 0.f) || !std::isfinite(eps)))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "eps must be finite and >= 0");
    if (!aligned_to(x, 2) || (gain && !aligned_to(gain, 2)) || !aligned_to(out, type_size(out_type)))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "x, gain and out must be aligned to their elements");
    (void)workspace;
    (void)workspace_bytes;
    DeviceGuard dg(q->device);
    if (dg.err != cudaSuccess) return op_cuda_fail(dg.err, "cudaSetDevice");
    if (!pointer_usable(x, q->device, false) || !pointer_usable(out, q->device, false) ||
        (gain && !pointer_usable(gain, q->device, false)))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "x, gain and out must be device memory on the head's device");
    QuantParams p{};
    p.codes = q->codes;
    p.meta = q->meta;
    p.row_tiles = q->row_tiles;
    p.blocks = q->blocks;
    p.groups = q->groups;
    p.scale_f16 = q->scale_f16 ? 1 : 0;
    p.d = q->d;
    p.V = q->V;
    p.gain = gain;
    p.x_stride = x_stride;
    p.x_vectors = aligned16(x) && (rows == 1 || x_stride % 8 == 0);
    p.gain_vectors = gain && aligned16(gain);
    p.eps = eps;
    p.out_stride = out_stride;
    p.out_type = out_type;
    cudaStream_t s = static_cast<cudaStream_t>(stream_ptr);
    // as many rows a launch as their activations fit into shared memory (at d = 65536 it is one)
    int most = kRowsMax;
    while (rows_smem(2, most, q->blocks) > kRowsSmem) --most;
    for (int r = 0; r < rows; r += most) {
        p.rows = std::min(most, rows - r);
        p.x = static_cast<const uint16_t *>(x) + r * x_stride;
        p.out = static_cast<char *>(out) + r * out_stride * type_size(out_type);
        const cudaError_t e = x_type == RPD_TYPE_BF16
                                  ? launch_rows_type<__nv_bfloat16>(p, q->group, q->zeros, q->num_sms, s)
                                  : launch_rows_type<__half>(p, q->group, q->zeros, q->num_sms, s);
        if (e != cudaSuccess) return op_cuda_fail(e, "4-bit head launch");
    }
    return RPD_OK;
}

void rpd_quant_destroy(rpd_quant *q) {
    if (!q) return;
    DeviceGuard dg(q->device);
    if (q->codes) cudaFree(q->codes);
    if (q->meta) cudaFree(q->meta);
    delete q;
}

}  // extern "C"
