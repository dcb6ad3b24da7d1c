// k_quant.cu - the 4-bit head: products of a few activations with a [V][d] matrix of 4-bit codes,
// a scale (and optionally a zero point) for every `group` columns of a row.
//
//   y[r][v] = rho_r * sum_G s[v][G] * sum_{k in G} (q[v][k] - z[v][G]) * u[r][k]
//
// with u = x and rho = 1, or - with a gain g - the readout's normalisation (App. A.2):
// u = rn(g * x) in the activations' type and rho_r = (mean_k x^2 + eps)^-1/2, applied after the
// sum, as the 16-bit head does it.
//
// Precision.  A pair of codes, masked in place, is two fp16 subnormals q 2^-24 (or 2^-20), and one fused multiply-add
// makes (q - z) 2^-9 of both, exactly.  Activations are fp16 numbers that a power of two a row has brought into range
// (quant_internal.h: scale_u).  Products and sums of a group are fp32, and a group's sum is multiplied by its scale and
// added to the row's in fp32: nothing is rounded into the weights.  Logits of d = 4096 are up to 1.3e-7 of their norm off.
// (Without the multiply-add, the subnormals themselves to the tensor core and the zero point's part -z sum u added to
// the sum, they were up to 1.7e-6 off: the tensor core lines its addends up by the operands' exponents, and a
// subnormal's has up to ten places less than that says.  It was no faster.)
//
// What bounds it: reading the codes once.  One row of a 126464 x 4096 head in groups of 128 is 259 MB of codes and 8 MB
// of scales, 39.4 us at 6780 GB/s; it takes 45.8 (5.8 TB/s), 8 rows 49.4, 9 rows 63.7, 16 rows 66.0.  As bf16 numbers
// 128 + q less 128 + z (three instructions a pair of codes, 87 for 512 bytes in all) one row took 66 us.
//
// k_quant_rows: up to 16 rows a CTA (many rows of a head that fills the device: k_quant_wide.cu).  A warp multiplies pairs of tiles of 16 matrix rows (M of the
// m16n8k16 MMA) by 8 or 16 activation rows (N), so that a fragment of codes is used for all of these, and a
// fragment of activations for both tiles, from registers (with one tile at a time the reads of shared memory were the
// limit: 52.6 us).  The codes are stored in fragment order, 1 KB for 32 rows x 64 columns, which a warp copies through
// a ring of its own in shared memory (asked for in registers instead, the copies in flight are limited by the six
// scoreboards of a warp: 66 us again).  A CTA owns a range of pairs and its warps divide the range's column blocks
// evenly, over their borders: a pair's sums then may come from several warps and are joined in shared memory in
// warp order.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <utility>

#include "op_host.h"
#include "ptx.cuh"
#include "quant_internal.h"

namespace rpd {
namespace {

// ------------------------------------------------------------------------------ layout of the codes

// One 16-byte vector of the packed codes a thread: the place of lane (t, g) of tile `which` of (pair, kb) holds rows
// 32 pair + 16 which + g (words 0, 1) and 8 rows further (words 2, 3), columns 64 kb + 8 t + {0..7} (words 0, 2)
// and 32 columns further (words 1, 3).  Nibble i of a word is column 2i, nibble i + 4 column 2i + 1, so that
// (word >> 4i) & 0x000F000F is a pair of neighbouring columns in the halves of a register.
__global__ void k_quant_pack(const uint8_t *codes, uint4 *packed, int V, int d, int pairs, int blocks) {
    const long long n = static_cast<long long>(pairs) * blocks * 64;
    const int row_bytes = (d + 1) / 2;
    for (long long i = blockIdx.x * static_cast<long long>(blockDim.x) + threadIdx.x; i < n;
         i += static_cast<long long>(gridDim.x) * blockDim.x) {
        const int place = static_cast<int>(i & 31), t = place >> 3, g = place & 7, which = static_cast<int>(i >> 5) & 1;
        const int kb = static_cast<int>((i >> 6) % blocks);
        const int pair = static_cast<int>((i >> 6) / blocks);
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int v = pair * kQuantPairRows + which * 16 + g + (j >> 1) * 8;
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

// Scales (and zero points) in the order of the pairs: [pair][group][tile][g][2] for rows g and g + 8 of a tile.
// With zero points an entry is 32 bits: the scale, and in the upper half -z 2^-9 in fp16.
template <bool kZeros>
__global__ void k_quant_pack_scales(const uint16_t *scales, const uint8_t *zeros, void *packed, int V, int groups,
                                    int pairs, int padded_groups) {
    const long long n = static_cast<long long>(pairs) * padded_groups * 32;
    for (long long i = blockIdx.x * static_cast<long long>(blockDim.x) + threadIdx.x; i < n;
         i += static_cast<long long>(gridDim.x) * blockDim.x) {
        const int hi = static_cast<int>(i & 1), g = static_cast<int>(i >> 1) & 7, which = static_cast<int>(i >> 4) & 1;
        const int grp = static_cast<int>((i >> 5) % padded_groups);
        const int v = static_cast<int>((i >> 5) / padded_groups) * kQuantPairRows + which * 16 + hi * 8 + g;
        const bool in = v < V && grp < groups;
        const long long at = static_cast<long long>(v) * groups + grp;
        const uint32_t s = in ? scales[at] : 0u;
        if (kZeros)
            static_cast<uint32_t *>(packed)[i] =
                s | static_cast<uint32_t>(__half_as_ushort(__float2half_rn(in ? (zeros[at] & 15) * -0x1p-9f : 0.f))) << 16;
        else
            static_cast<uint16_t *>(packed)[i] = static_cast<uint16_t>(s);
    }
}

// ------------------------------------------------------------------------------ few rows

constexpr int kRowsWarps = 16;
constexpr int kRowsThreads = 32 * kRowsWarps;

__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9},"
        " {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The launch's activations in shared memory: rows of `row_bytes` as scale_u leaves them, zero beyond column d; and
// what a row's logits are multiplied with.  The warps divide the rows, or a row, evenly.  Ends with a barrier.
struct RowsSmem {
    uint8_t *x;
    float *factor, *red;
    int row_bytes;
};

// f(chunk index, u) for the chunks of 8 columns of a row that fall to this lane: 32 neighbouring chunks a
// warp at a time, the lane's next ones asked for before the first is used.  Lanes beyond the last chunk
// get zeros.
template <typename T, typename F>
__device__ __forceinline__ void for_chunks(const QuantParams &p, const T *x, int first, int step, const F &f) {
    constexpr int kBatch = 4;
    const int chunks = p.blocks * 8;
    const T *gain = static_cast<const T *>(p.gain);
    for (int c0 = first; c0 < chunks; c0 += kBatch * step) {
        uint4 v[kBatch], g[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int c = c0 + j * step + (threadIdx.x & 31);
            v[j] = g[j] = make_uint4(0, 0, 0, 0);
            if (c < chunks) {
                v[j] = load_chunk(x, c * 8, p.d, p.x_align);
                if (gain) g[j] = load_chunk(gain, c * 8, p.d, p.gain_align);
            }
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (c0 + j * step < chunks) f(c0 + j * step + static_cast<int>(threadIdx.x & 31), v[j], g[j]);
    }
}

template <typename T>
__device__ void stage_rows(const QuantParams &p, const RowsSmem &s, int first, int rows) {
    const int chunks = p.blocks * 8;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int per_row = kRowsWarps;  // warps that share a row
    while (per_row * rows > kRowsWarps && per_row > 1) per_row >>= 1;
    const int part = warp % per_row;
    for (int r = warp / per_row; r < rows; r += kRowsWarps / per_row) {
        float ss = 0.f, top = 0.f;
        for_chunks(p, static_cast<const T *>(p.x) + (first + r) * p.x_stride, part * 32, per_row * 32,
                   [&](int, const uint4 &v, const uint4 &g) {
                       float2 u[4];
                       ss += make_u<T>(v, p.gain != nullptr, g, u);
#pragma unroll
                       for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(u[i].x), fabsf(u[i].y)));
                   });
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            ss += __shfl_xor_sync(0xffffffffu, ss, o);
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        }
        if (lane == 0) {
            s.red[(r * kRowsWarps + part) * 2] = ss;
            s.red[(r * kRowsWarps + part) * 2 + 1] = top;
        }
    }
    __syncthreads();
    for (int r = warp / per_row; r < rows; r += kRowsWarps / per_row) {
        float ss = 0.f, top = 0.f;
        for (int w = 0; w < per_row; ++w) {
            ss += s.red[(r * kRowsWarps + w) * 2];
            top = fmaxf(top, s.red[(r * kRowsWarps + w) * 2 + 1]);
        }
        int E = exponent_of(top);
        if (p.gain && norm_unusual(ss, top, p.eps, E)) {  // (the row's warps all do it, for E)
            const NormFactor f = norm_factor_unusual(static_cast<const T *>(p.x) + (first + r) * p.x_stride, chunks, p.d,
                                                     p.x_align, p.eps, top, E);
            E = f.E;
            if (part == 0 && lane == 0) s.factor[r] = f.factor;
        } else if (part == 0 && lane == 0) {
            s.factor[r] = p.gain ? norm_factor(ss, static_cast<float>(p.d), p.eps, E) : ldexpf(1.f, E);
        }
        uint8_t *xs = s.x + static_cast<size_t>(r) * s.row_bytes;
        for_chunks(p, static_cast<const T *>(p.x) + (first + r) * p.x_stride, part * 32, per_row * 32,
                   [&](int c, const uint4 &v, const uint4 &g) {
                       float2 u[4];
                       uint4 w;
                       make_u<T>(v, p.gain != nullptr, g, u);
                       scale_u(u, E, w);
                       if (c < chunks) *reinterpret_cast<uint4 *>(xs + c * 16) = w;
                   });
    }
    __syncthreads();
}

// A finished pair's logits: fragment element (g, 2t) of the MMA's result is matrix row g, activation 2t.
template <int kN8>
__device__ __forceinline__ void store_pair(const QuantParams &p, int pair, const float (&run)[2][kN8][4],
                                           const float *factor, int first, int rows, int g, int t) {
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int n = 0; n < kN8; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = n * 8 + 2 * t + (i & 1), v = pair * kQuantPairRows + which * 16 + g + (i >> 1) * 8;
                if (r < rows && v < p.V)
                    store_out(p.out, p.out_type, (first + r) * p.out_stride + v, run[which][n][i] * kWeightFactor * factor[r]);
            }
}

// Units (groups, or for groups of 32 columns two) that a warp copies and waits for at a time: 2 KB of codes.
template <int kGroup, bool kZeros>
struct RowsStage {
    static constexpr int kUnitBlocks = kGroup == 128 ? 2 : 1;  // 64-column blocks of a unit of work
    static constexpr int kUnitGroups = kGroup == 32 ? 2 : 1;
    static constexpr int kUnits = 2 / kUnitBlocks;
    static constexpr int kCodeBytes = 2048;
    static constexpr int kMetaUnit = kUnitGroups * (kZeros ? 128 : 64);
    static constexpr int kBytes = kCodeBytes + kUnits * kMetaUnit;
};

template <int kGroup, int kN8, bool kZeros, bool kF16>
__global__ void __launch_bounds__(kRowsThreads, 1) k_quant_rows(const QuantParams p, const int depth) {
    typedef RowsStage<kGroup, kZeros> Stage;
    typedef typename MetaVec<kZeros>::type Meta;  // scales (and zero points) of rows g and g + 8
    constexpr int kUnitBlocks = Stage::kUnitBlocks, kUnitGroups = Stage::kUnitGroups;
    extern __shared__ __align__(128) uint8_t smem[];
    RowsSmem sm;
    sm.red = reinterpret_cast<float *>(smem);
    sm.factor = sm.red + 2 * 16 * kRowsWarps;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    // a row and 64 bytes: the two rows that a quarter of a warp reads at once lie in different banks
    sm.row_bytes = p.blocks * 128 + 64;
    uint8_t *ring = reinterpret_cast<uint8_t *>(sm.factor + 16);
    sm.x = ring + kRowsWarps * depth * Stage::kBytes;
    float *join = reinterpret_cast<float *>(sm.x);  // [warp][8 kN8][lane], when nobody reads the activations any more

    pdl_trigger();
    const int row0 = blockIdx.y * p.per, rows = min(p.per, p.rows - row0);
    // this CTA's pairs of tiles, this warp's units of them
    const int pair0 = static_cast<int>(static_cast<long long>(p.pairs) * blockIdx.x / gridDim.x);
    const int pair1 = static_cast<int>(static_cast<long long>(p.pairs) * (blockIdx.x + 1) / gridDim.x);
    const int per_pair = p.blocks / kUnitBlocks;
    const int units = (pair1 - pair0) * per_pair;
    const int u0 = units * warp / kRowsWarps, u1 = units * (warp + 1) / kRowsWarps;
    // Both streams are contiguous over the CTA's pairs.  A lane copies the vectors of codes that it reads.
    const int place = (t * 8 + g) * 16;
    const uint8_t *codes = reinterpret_cast<const uint8_t *>(p.codes) +
                           (static_cast<long long>(pair0) * p.blocks + static_cast<long long>(u0) * kUnitBlocks) * 1024 + place;
    const uint8_t *meta = static_cast<const uint8_t *>(p.meta) +
                          (static_cast<long long>(pair0) * per_pair + u0) * Stage::kMetaUnit + lane * 16;
    const uint32_t ring_at = smem_u32(ring) + warp * depth * Stage::kBytes;
    int ahead = u1 - u0;  // units that are not yet asked for
    auto fetch = [&](int slot) {
        if (ahead > 0) {
            const uint32_t to = ring_at + slot * Stage::kBytes;
#pragma unroll
            for (int b = 0; b < 4; ++b)
                if (b / (2 * kUnitBlocks) < ahead) copy_async(to + b * 512 + place, codes + b * 512);
            if (lane * 16 < min(ahead, Stage::kUnits) * Stage::kMetaUnit)
                copy_async(to + Stage::kCodeBytes + lane * 16, meta);
            codes += Stage::kCodeBytes;
            meta += Stage::kUnits * Stage::kMetaUnit;
            ahead -= Stage::kUnits;
        }
        copy_commit();
    };
    for (int s = 0; s < depth - 1; ++s) fetch(s);

    pdl_wait();  // the weights were laid out long ago; the activations may be the predecessor's
    if (p.x_type == RPD_TYPE_BF16)
        stage_rows<__nv_bfloat16>(p, sm, row0, rows);
    else
        stage_rows<__half>(p, sm, row0, rows);

    float run[2][kN8][4], first[2][kN8][4];  // first: of a pair that an earlier warp began
#pragma unroll
    for (int i = 0; i < 8 * kN8; ++i) run[i / (4 * kN8)][i / 4 % kN8][i % 4] = first[i / (4 * kN8)][i / 4 % kN8][i % 4] = 0.f;
    int in_pair = u0 % per_pair, pair = pair0 + u0 / per_pair;
    const bool joins = in_pair != 0;
    bool head = joins;  // the pair at hand was begun by an earlier warp
    // Lanes of activations beyond the last read the last one's elements: their columns of the result
    // are never stored.
    uint32_t xrow[kN8];
#pragma unroll
    for (int n = 0; n < kN8; ++n)
        xrow[n] = smem_u32(sm.x) + min(n * 8 + g, rows - 1) * sm.row_bytes + t * 16;

    int slot = 0, refill = depth - 1;
    for (int u = u0; u < u1; u += Stage::kUnits) {
        if (depth >= 6)
            copy_wait<4>();
        else if (depth >= 4)
            copy_wait<2>();
        else
            copy_wait<0>();
        __syncwarp();  // every lane's copies are seen, and every lane is done with the slot before
        fetch(refill);
        const uint32_t stage = ring_at + slot * Stage::kBytes;
        refill = slot;
        slot = slot + 1 == depth ? 0 : slot + 1;
#pragma unroll
        for (int j = 0; j < Stage::kUnits; ++j) {
            if (u + j < u1) {
                uint4 q[2];
#pragma unroll
                for (int k = 0; k < kUnitGroups; ++k) {
                    float s_lo[2], s_hi[2], c[2][kN8][4];
                    uint32_t z_lo[2], z_hi[2];
#pragma unroll
                    for (int which = 0; which < 2; ++which) {
                        Meta m;
                        lds_meta(stage + Stage::kCodeBytes + (((j * kUnitGroups + k) * 2 + which) * 8 + g) * sizeof(Meta), m);
                        unpack_meta<kF16>(m, s_lo[which], s_hi[which], z_lo[which], z_hi[which]);
#pragma unroll
                        for (int n = 0; n < kN8; ++n)
#pragma unroll
                            for (int i = 0; i < 4; ++i) c[which][n][i] = 0.f;
                    }
                    // 32-column halves of this group: (block, half); a fragment of activations for both tiles
#pragma unroll
                    for (int h = 0; h < kGroup / 32; ++h) {
                        const int b = kGroup == 32 ? 0 : h >> 1, half = kGroup == 32 ? k : h & 1;
                        uint4 xv[kN8];
#pragma unroll
                        for (int n = 0; n < kN8; ++n)
                            xv[n] = lds128(xrow[n] + (in_pair * kUnitBlocks + b) * 128 + half * 64);
#pragma unroll
                        for (int which = 0; which < 2; ++which) {
                            if (kGroup == 32 ? k == 0 : half == 0)
                                q[which] = lds128(stage + (j * kUnitBlocks + b) * 1024 + which * 512 + place);
                            const uint32_t lo = half ? q[which].y : q[which].x, hi = half ? q[which].w : q[which].z;
#pragma unroll
                            for (int step = 0; step < 2; ++step) {
                                const uint32_t a[4] = {
                                    weight_pair(lo, 2 * step, z_lo[which]), weight_pair(hi, 2 * step, z_hi[which]),
                                    weight_pair(lo, 2 * step + 1, z_lo[which]), weight_pair(hi, 2 * step + 1, z_hi[which])};
#pragma unroll
                                for (int n = 0; n < kN8; ++n)
                                    mma_16816(c[which][n], a, step ? xv[n].z : xv[n].x, step ? xv[n].w : xv[n].y);
                            }
                        }
                    }
#pragma unroll
                    for (int which = 0; which < 2; ++which)
#pragma unroll
                        for (int n = 0; n < kN8; ++n) {
                            run[which][n][0] = fmaf(c[which][n][0], s_lo[which], run[which][n][0]);
                            run[which][n][1] = fmaf(c[which][n][1], s_lo[which], run[which][n][1]);
                            run[which][n][2] = fmaf(c[which][n][2], s_hi[which], run[which][n][2]);
                            run[which][n][3] = fmaf(c[which][n][3], s_hi[which], run[which][n][3]);
                        }
                }
                if (++in_pair == per_pair) {  // the pair's last columns
                    if (!head) store_pair<kN8>(p, pair, run, sm.factor, row0, rows, g, t);
#pragma unroll
                    for (int i = 0; i < 8 * kN8; ++i) {
                        float &r = run[i / (4 * kN8)][i / 4 % kN8][i % 4];
                        if (head) first[i / (4 * kN8)][i / 4 % kN8][i % 4] = r;
                        r = 0.f;
                    }
                    head = false;
                    in_pair = 0;
                    ++pair;
                }
            }
        }
    }
    __syncthreads();
    if (joins) {  // (where the warp's whole range lies inside one pair, its sums are still in run)
#pragma unroll
        for (int i = 0; i < 8 * kN8; ++i)
            join[(warp * 8 * kN8 + i) * 32 + lane] =
                head ? run[i / (4 * kN8)][i / 4 % kN8][i % 4] : first[i / (4 * kN8)][i / 4 % kN8][i % 4];
    }
    __syncthreads();
    if (!head && in_pair) {  // a pair that this warp began and later warps went on with
        const int end = (pair - pair0 + 1) * per_pair;
        for (int w = warp + 1; w < kRowsWarps; ++w) {
            if (units * w / kRowsWarps >= end) break;  // (a warp without units in the pair has left zeros)
#pragma unroll
            for (int i = 0; i < 8 * kN8; ++i) run[i / (4 * kN8)][i / 4 % kN8][i % 4] += join[(w * 8 * kN8 + i) * 32 + lane];
        }
        store_pair<kN8>(p, pair, run, sm.factor, row0, rows, g, t);
    }
}

constexpr int kRowsMax = 16;                 // activation rows of a CTA
// More rows are the other kernel's, unless every CTA for them has an SM to itself (rows_of_cta).  126464 x 4096: 16 rows
// 66.0 us here (95 there), 17 rows 96.2 there (120 here); 15872 x 4096: 21.9 (27), and 26.7 (34).  2000 x 4096: 32 rows,
// 126 CTAs, 16.6 us here (23.6), 48 rows, which would be 189, 24.7 there (31.4).  From d = 4480 on 16 rows are two groups
// here and more, each of which reads the codes again; that is not weighed.
constexpr int kRowsMost = 16;
constexpr int kRowsSmem = 224 * 1024;        // of the 227 KB a CTA may have

// Shared memory besides the ring of codes (the activations' part is big enough for the partial sums that follow).
size_t rows_smem(int n8, int rows, int blocks) {
    return (2 * 16 * kRowsWarps + 16) * 4 +
           std::max(static_cast<size_t>(rows) * (blocks * 128 + 64), static_cast<size_t>(kRowsWarps) * 8 * n8 * 32 * 4);
}

constexpr int kRowsRing = kRowsWarps * 2 * (2048 + 4 * 128);  // its least: two stages of any kind a warp

template <int kGroup, int kN8, bool kZeros, bool kF16>
cudaError_t launch_rows(const QuantParams &p, int num_sms, cudaStream_t s) {
    void (*kernel)(QuantParams, int) = k_quant_rows<kGroup, kN8, kZeros, kF16>;
    // (cheap, and per device: set on every call)
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRowsSmem);
    if (e != cudaSuccess) return e;
    const size_t fixed = rows_smem(kN8, p.per, p.blocks);
    const int stage = kRowsWarps * RowsStage<kGroup, kZeros>::kBytes;
    const int fits = static_cast<int>((kRowsSmem - fixed) / stage);
    const int depth = fits >= 6 ? 6 : fits >= 4 ? 4 : 2;
    return launch_pdl(kernel, dim3(std::min(num_sms, p.pairs), (p.rows + p.per - 1) / p.per), dim3(kRowsThreads), fixed + depth * stage, s, p,
                      depth);
}

template <int kGroup, int kN8>
cudaError_t launch_rows_scales(const QuantParams &p, bool zeros, bool f16, int num_sms, cudaStream_t s) {
    if (f16)
        return zeros ? launch_rows<kGroup, kN8, true, true>(p, num_sms, s) : launch_rows<kGroup, kN8, false, true>(p, num_sms, s);
    return zeros ? launch_rows<kGroup, kN8, true, false>(p, num_sms, s) : launch_rows<kGroup, kN8, false, false>(p, num_sms, s);
}

template <int kN8>
cudaError_t launch_rows_group(const QuantParams &p, int group, bool zeros, bool f16, int num_sms, cudaStream_t s) {
    return group == 32   ? launch_rows_scales<32, kN8>(p, zeros, f16, num_sms, s)
           : group == 64 ? launch_rows_scales<64, kN8>(p, zeros, f16, num_sms, s)
                         : launch_rows_scales<128, kN8>(p, zeros, f16, num_sms, s);
}

}  // namespace
}  // namespace rpd

using namespace rpd;

// The weights of a head in its own order, in device memory.
struct QuantLayout {
    uint4 *codes = nullptr;
    void *meta = nullptr;
    cudaError_t allocate(size_t code_bytes, size_t meta_bytes) {  // both or neither
        cudaError_t e = cudaMalloc(&codes, code_bytes);
        if (e == cudaSuccess) e = cudaMalloc(&meta, meta_bytes);
        if (e != cudaSuccess) release();
        return e;
    }
    cudaError_t release() {  // what could not be freed is kept
        cudaError_t e = cudaFree(codes);
        if (e == cudaSuccess) {
            codes = nullptr;
            e = cudaFree(meta);
            if (e == cudaSuccess) meta = nullptr;
        }
        return e;
    }
};

struct rpd_quant {
    int d = 0, V = 0, group = 0;
    int device = 0, num_sms = 0;
    int pairs = 0, pad_pairs = 0, blocks = 0, groups = 0;  // groups: padding included
    QuantLayout layout;
    bool set = false, zeros = false, scale_f16 = false;
    int64_t wait_us = 2000000;  // of the wide kernel's waits
    bool stall = false;
    CUtensorMap maps[2];  // the codes, a row a pair
};

namespace {

long long rows_ctas(const rpd_quant *q, int rows, int per) {
    return ((rows - 1ll) / per + 1) * std::min(q->pairs, q->num_sms);
}

// Activation rows of a CTA of k_quant_rows: as many as fit into its shared memory (16 up to d = 4096, two at d = 32768), but
// eight where every CTA has an SM to itself all the same (2000 x 4096: 16 rows 10.7 us, as one CTA's 16.1).
int rows_of_cta(const rpd_quant *q, int rows) {
    int most = std::min(kRowsMax, std::max(rows, 1));
    while (rows_smem(most > 8 ? 2 : 1, most, q->blocks) + kRowsRing > kRowsSmem) --most;
    return most > 8 && rows_ctas(q, rows, 8) <= q->num_sms ? 8 : most;
}

// Boxes of 4 and of 2 pairs x 128 columns of the packed codes.
int encode_codes(const rpd_quant *q, uint4 *codes, CUtensorMap *maps) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return op_fail(RPD_ERR_CUDA, "cuTensorMapEncodeTiled entry point unavailable");
    cuuint64_t dims[2] = {static_cast<cuuint64_t>(q->blocks) * 128, static_cast<cuuint64_t>(q->pad_pairs)};
    cuuint64_t strides[1] = {static_cast<cuuint64_t>(q->blocks) * 1024};
    cuuint32_t box[2] = {256, 4}, step[2] = {1, 1};
    CUresult r = CUDA_SUCCESS;
    for (int i = 0; i < 2 && r == CUDA_SUCCESS; ++i, box[1] /= 2)
        r = fn(&maps[i], CU_TENSOR_MAP_DATA_TYPE_UINT64, 2, codes, dims, strides, box, step,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? RPD_OK : op_fail(RPD_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", static_cast<int>(r));
}

}  // namespace

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
    q->blocks = (d + 127) / 128 * 2;
    q->groups = q->blocks * 64 / group;
    q->pairs = (V + kQuantPairRows - 1) / kQuantPairRows;
    q->pad_pairs = (q->pairs + kQuantPadPairs - 1) / kQuantPadPairs * kQuantPadPairs;
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
    cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(s, &capturing);
    if (e != cudaSuccess) return op_cuda_fail(e, "cudaStreamIsCapturing");
    if (capturing != cudaStreamCaptureStatusNone)
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "the weights cannot be set while the stream is being captured");
    const size_t code_bytes = static_cast<size_t>(q->pad_pairs) * q->blocks * 1024;
    const size_t meta_bytes = static_cast<size_t>(q->pad_pairs) * q->groups * (zeros ? 128 : 64);
    RelaxedCapture rc;
    // The new layout is made beside the one that is there, which a failure then leaves as it was.  Only where the device
    // has no room for both is the old one freed first.
    QuantLayout made;
    e = made.allocate(code_bytes, meta_bytes);
    if (e == cudaErrorMemoryAllocation && q->set) {
        cudaGetLastError();
        q->set = false;
        e = q->layout.release();
        if (e == cudaSuccess) e = made.allocate(code_bytes, meta_bytes);
    }
    if (e != cudaSuccess) return op_cuda_fail(e, "memory for the 4-bit weights");
    const int groups = (q->d + q->group - 1) / q->group;
    e = launch_plain(k_quant_pack, q->num_sms * 8, 256, s, static_cast<const uint8_t *>(codes), made.codes, q->V, q->d,
                     q->pad_pairs, q->blocks);
    if (e == cudaSuccess)
        e = launch_plain(zeros ? k_quant_pack_scales<true> : k_quant_pack_scales<false>, q->num_sms * 4, 256, s,
                         static_cast<const uint16_t *>(scales), static_cast<const uint8_t *>(zeros), made.meta, q->V,
                         groups, q->pad_pairs, q->groups);
    const cudaError_t done = cudaStreamSynchronize(s);  // (whatever was launched may not outlive its memory)
    if (e == cudaSuccess) e = done;
    CUtensorMap maps[2];
    const int code = e != cudaSuccess ? op_cuda_fail(e, "layout of the 4-bit weights") : encode_codes(q, made.codes, maps);
    if (code != RPD_OK) {
        made.release();
        return code;
    }
    std::swap(q->layout, made);
    std::copy(maps, maps + 2, q->maps);
    q->zeros = zeros != nullptr;
    q->scale_f16 = scale_type == RPD_TYPE_F16;
    q->set = true;
    made.release();  // waits for the device: no call may still be reading it
    cudaGetLastError();
    return RPD_OK;
}

int64_t rpd_quant_workspace(const rpd_quant *q, int rows) {
    if (!q || rows < 0) {
        op_fail(RPD_ERR_INVALID_ARGUMENT, "null head or negative rows");
        return -1;
    }
    return rows <= kRowsMost || rows_ctas(q, rows, rows_of_cta(q, rows)) <= q->num_sms
               ? 0
               : quant_wide_workspace(rows, q->blocks, q->pairs, q->num_sms);
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
    const int64_t need = rpd_quant_workspace(q, rows);
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned_to(workspace, 256)))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "workspace: %lld bytes at a 256-byte boundary needed",
                       static_cast<long long>(need));
    DeviceGuard dg(q->device);
    if (dg.err != cudaSuccess) return op_cuda_fail(dg.err, "cudaSetDevice");
    if (!pointer_usable(x, q->device, false) || !pointer_usable(out, q->device, false) ||
        (gain && !pointer_usable(gain, q->device, false)) || (need > 0 && !pointer_usable(workspace, q->device, false)))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "x, gain, out and workspace must be device memory on the head's device");
    QuantParams p{};
    p.codes = q->layout.codes;
    p.meta = q->layout.meta;
    p.pairs = q->pairs;
    p.blocks = q->blocks;
    p.groups = q->groups;
    p.x_type = x_type;
    p.d = q->d;
    p.V = q->V;
    p.gain = gain;
    p.x_stride = x_stride;
    p.x_align = common_align(reinterpret_cast<uintptr_t>(x) | (rows > 1 ? static_cast<uintptr_t>(x_stride) * 2 : 0));
    p.gain_align = common_align(reinterpret_cast<uintptr_t>(gain));
    p.eps = eps;
    p.out_stride = out_stride;
    p.out_type = out_type;
    p.x = x;
    p.out = out;
    p.rows = rows;
    p.wait_cycles = q->wait_us * kWaitCyclesPerUs;
    p.stall = q->stall ? 1 : 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream_ptr);
    cudaError_t e;
    if (need > 0) {
        e = quant_wide(q->maps, p, q->group, q->zeros, q->scale_f16, q->num_sms, workspace, s);
    } else {
        p.per = rows_of_cta(q, rows);
        e = p.per <= 8 ? launch_rows_group<1>(p, q->group, q->zeros, q->scale_f16, q->num_sms, s)
                       : launch_rows_group<2>(p, q->group, q->zeros, q->scale_f16, q->num_sms, s);
    }
    return e == cudaSuccess ? RPD_OK : op_cuda_fail(e, "4-bit head launch");
}

int rpd_quant_set_wait_limit(rpd_quant *q, int64_t microseconds) {
    if (!q) return op_fail(RPD_ERR_INVALID_ARGUMENT, "null head");
    if (microseconds < 1000 || microseconds > kMaxWaitUs)
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "the wait limit must be 1000 .. %lld us", static_cast<long long>(kMaxWaitUs));
    q->wait_us = microseconds;
    return RPD_OK;
}

int rpd_quant_inject_stall(rpd_quant *q, int on) {
    if (!q) return op_fail(RPD_ERR_INVALID_ARGUMENT, "null head");
    q->stall = on != 0;
    return RPD_OK;
}

void rpd_quant_destroy(rpd_quant *q) {
    if (!q) return;
    DeviceGuard dg(q->device);
    RelaxedCapture rc;
    q->layout.release();
    cudaGetLastError();
    delete q;
}

}  // extern "C"
