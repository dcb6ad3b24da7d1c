// k_fp8.cu - the 8-bit head: products of activations with a [V][d] matrix of e4m3 codes that has a scale for
// every 128 x 128 of them, and the quantiser that makes such operands.
//
//   y[r][v] = rho_r * sum_B sw[v / 128][B] * sx[r][B] * sum_{k in B} qw[v][k] * qx[r][k]
//
// B runs over blocks of 128 columns; u = x, or rn(g x) with rho_r = (mean_k x^2 + eps)^-1/2 under a norm;
// sx[r][B] = max_{k in B} |u| / 448 and qx = e4m3(u / sx), the division and the quotient in fp32.
//
// Precision.  Codes enter the tensor core as they are (a product of two has 8 bits); a block's sum is fp32 in tensor
// memory, is multiplied by the two scales and added to the row's in fp32 registers.  rho enters once, at the end.
//
// k_fp8_rows rounds the activations (a CTA a row) and lays them out as the product's operand.  k_fp8_head multiplies:
// 128 activations are the MMA's M, so that a thread of the epilogue has one row, whose two scales are one factor for
// all of its columns (with the matrix as M it would be a factor a column: a 16-byte load from shared memory for every
// four multiply-adds); 256 matrix rows are N.  A block's product goes into one half of tensor memory while
// eight warps read the other.  Of rows that are not there nothing is copied or read, so that one kernel does for one row
// too; more than 128 go to pairs of CTAs, each of which keeps half of the matrix rows' stage and its own activations.
//
// What bounds it.  Few rows: reading the codes.  126464 x 4096 is 518 MB, 77.6 us at 6683 GB/s: one row takes 83.0, 128 rows (32 MB
// of logits) 103.  Many: no one thing.  1024 rows of 152064 x 3584 are 1116 GFLOP in 447 to 491 us, some 940 cycles for every 256 x 256
// x 128, of which the MMAs are 528; the warp that issues them waits 261 for a stage and 253 for an accumulator (time stamps around its
// waits).  Without the epilogue's reads of accumulators a launch of 447 us took 349, without its stores 421, without both 325.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
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

constexpr float kFp8Most = 448.f;           // e4m3's largest number
constexpr int kFp8Block = 128;              // columns of a scale
constexpr int kFp8RowsTile = 128;           // activations of a CTA's tile (M)
constexpr int kFp8ColsTile = 256;           // matrix rows of a tile (N)
constexpr int kFp8TileBytes = kFp8ColsTile * kFp8Block;  // codes of a tile and block
constexpr int kFp8RowsBytes = kFp8RowsTile * kFp8Block;
constexpr int kFp8Threads = 12 * 32;        // three warpgroups, between which the registers are divided anew
constexpr int kFp8EpilogueRegs = 224, kFp8OtherRegs = 56;  // 256 * 224 + 128 * 56 of the launch's 384 * 168
constexpr int kFp8TmaCodes = 8, kFp8TmaRows = 9, kFp8Mma = 10;  // warps; 0 - 7 are the epilogue
constexpr int kFp8FewRows = 24;             // activations whose logits are handed to all of the epilogue's threads, a column each
constexpr int kFp8FewPitch = kFp8ColsTile + 1;
constexpr int kFp8BoxBytes = kFp8RowsTile * 128;  // of logits on their way out: 64 (32 in fp32) columns x 128 rows
constexpr int kFp8StageOut = 4 * kFp8BoxBytes;
constexpr int kFp8Smem = 226 * 1024;
constexpr int kFp8MaxRows = 1 << 14;         // of a launch

// ------------------------------------------------------------------------------ layout

// Codes in the order of the product: [tile][block][256 rows][128 bytes], 16-byte pieces swizzled within 8 rows; zero
// beyond V and d.
__global__ void k_fp8_pack(const uint8_t *codes, uint4 *packed, int V, int d, long long tiles, int blocks) {
    const long long n = tiles * blocks * kFp8ColsTile * 8;
    const bool whole = d % 16 == 0 && reinterpret_cast<uintptr_t>(codes) % 16 == 0;
    for (long long i = blockIdx.x * static_cast<long long>(blockDim.x) + threadIdx.x; i < n;
         i += static_cast<long long>(gridDim.x) * blockDim.x) {
        const int piece = static_cast<int>(i & 7), row = static_cast<int>(i >> 3) & (kFp8ColsTile - 1);
        const long long at = i >> 11;  // tile and block
        const int kb = static_cast<int>(at % blocks), col = kb * kFp8Block + piece * 16;
        const long long v = at / blocks * kFp8ColsTile + row;
        uint4 w = make_uint4(0, 0, 0, 0);
        if (v < V && col < d) {
            const uint8_t *from = codes + v * d + col;
            if (whole) {
                w = *reinterpret_cast<const uint4 *>(from);
            } else {
                uint32_t b[4] = {0, 0, 0, 0};
                for (int j = 0; j < min(16, d - col); ++j) b[j >> 2] |= static_cast<uint32_t>(from[j]) << (8 * (j & 3));
                w = make_uint4(b[0], b[1], b[2], b[3]);
            }
        }
        packed[(i & ~7ll) + (piece ^ (row & 7))] = w;
    }
}

// Scales beside them: [tile][block][2].
__global__ void k_fp8_pack_scales(const float *scales, float *packed, int rows, long long tiles, int blocks) {
    const long long n = tiles * blocks * 2;
    for (long long i = blockIdx.x * static_cast<long long>(blockDim.x) + threadIdx.x; i < n;
         i += static_cast<long long>(gridDim.x) * blockDim.x) {
        const long long row = (i >> 1) / blocks * 2 + (i & 1);
        packed[i] = row < rows ? scales[row * blocks + (i >> 1) % blocks] : 0.f;
    }
}

// ------------------------------------------------------------------------------ activations

// Eight numbers over a scale as e4m3 codes: the fp32 quotient, rounded.  Of a product with the rounded reciprocal, off by a last
// place at most, the rest x - q s is exact, and q + (rest) / s rounded once is the quotient rounded (Markstein, IBM J. Res. Dev. 34,
// 1990): three operations where a division is some fifteen (a head of 126464 x 4096 took 865 us with these).  (q s - x taken away,
// not x - q s added: so that -0 stays -0.)  The rest has to stay above fp32's smallest number wherever a code is not 0, which blocks of
// tiny numbers do not give: they are divided.
__device__ __forceinline__ uint2 fp8_codes(const float2 (&u)[4], float scale, float inverse) {
    float2 t[4];
    if (scale >= 0x1p-60f && scale <= 0x1p100f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float qx = __fmul_rn(u[i].x, inverse), qy = __fmul_rn(u[i].y, inverse);
            t[i] = make_float2(__fmaf_rn(-__fmaf_rn(qx, scale, -u[i].x), inverse, qx), __fmaf_rn(-__fmaf_rn(qy, scale, -u[i].y), inverse, qy));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = make_float2(u[i].x / scale, u[i].y / scale);
    }
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __nv_cvt_float2_to_fp8x2(t[i], __NV_SATFINITE, __NV_E4M3);
    return make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
}

struct Fp8RowsParams {
    const void *x, *gain;
    long long x_stride;
    int d, blocks, x_align, gain_align;
    float eps;
    uint8_t *codes;  // [tile][block][128 rows][128 bytes], swizzled
    float *scales;   // [tile][block][128], times 2^-E
    float *factor;   // [row]: 2^E, or rho 2^E
    int *counters;   // cleared
    int num_counters;
};

// One row: its codes, its scales relative to 2^E (E the exponent of its largest element, so that sums stay in
// range whatever the row's size) and what its logits are multiplied with.  A block of 128 columns is 16 lanes'.
template <typename T>
__global__ void __launch_bounds__(256) k_fp8_rows(const Fp8RowsParams p) {
    __shared__ float red[2][8];
    __shared__ float scale_of[kQuantMaxD / kFp8Block];
    const int r = blockIdx.x, tile = r / kFp8RowsTile, slot = r % kFp8RowsTile;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, chunks = p.blocks * 16;
    const T *x = static_cast<const T *>(p.x) + r * p.x_stride;
    const T *gain = static_cast<const T *>(p.gain);
    uint8_t *codes = p.codes + (static_cast<long long>(tile) * p.blocks * kFp8RowsTile + slot) * kFp8Block;
    pdl_trigger();
    pdl_wait();
    if (r == 0)
        for (int i = threadIdx.x; i < p.num_counters; i += 256) p.counters[i] = 0;
    float ss = 0.f, top = 0.f;
    for (int first = 0; first < chunks; first += 256) {
        const int c = first + threadIdx.x;
        float2 u[4] = {};
        float amax = 0.f;
        if (c < chunks) {
            ss += make_u<T>(load_chunk(x, c * 8, p.d, p.x_align), gain != nullptr,
                            gain ? load_chunk(gain, c * 8, p.d, p.gain_align) : make_uint4(0, 0, 0, 0), u);
#pragma unroll
            for (int i = 0; i < 4; ++i) amax = fmaxf(amax, fmaxf(fabsf(u[i].x), fabsf(u[i].y)));
        }
#pragma unroll
        for (int o = 8; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        if (c < chunks) {
            top = fmaxf(top, amax);
            const float scale = amax / kFp8Most;
            const float by = scale > 0.f ? scale : 1.f;
            const uint2 q = fp8_codes(u, by, 1.f / by);
            const int kb = c >> 4, piece = (c >> 1) & 7;
            *reinterpret_cast<uint2 *>(codes + static_cast<long long>(kb) * kFp8RowsBytes + (piece ^ (slot & 7)) * 16 + (c & 1) * 8) = q;
            if ((c & 15) == 0) scale_of[kb] = scale;
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        ss += __shfl_xor_sync(0xffffffffu, ss, o);
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    if (lane == 0) {
        red[0][warp] = ss;
        red[1][warp] = top;
    }
    __syncthreads();
    ss = top = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
        ss += red[0][w];
        top = fmaxf(top, red[1][w]);
    }
    int E = exponent_of(top);
    float factor = gain ? norm_factor(ss, static_cast<float>(p.d), p.eps, E) : ldexpf(1.f, E);
    if (gain && norm_unusual(ss, top, p.eps, E)) {
        const NormFactor f = norm_factor_unusual(x, chunks, p.d, p.x_align, p.eps, top, E);
        E = f.E;
        factor = f.factor;
    }
    if (threadIdx.x == 0) p.factor[r] = factor;
    for (int kb = threadIdx.x; kb < p.blocks; kb += 256)
        p.scales[(static_cast<long long>(tile) * p.blocks + kb) * kFp8RowsTile + slot] = ldexpf(scale_of[kb], -E);
}

// ------------------------------------------------------------------------------ the product

// How a launch divides the tiles (256 matrix rows x the rows of a CTA or pair): `workers` CTAs (pairs) take `waves` whole
// tiles each, and of the `tail` tiles that are left equal numbers of blocks, so that none is idle.  A tile that
// several have worked on is added up, in the workers' order, by the one that is done last.
struct Fp8Plan {
    int blocks, row_tiles;         // row tiles: of 128, or pairs' of 256 rows
    int workers, waves, tail, units;  // units: tail * blocks
    int tail_workers;              // the first so many share the tail: each has a unit at least
    int partial_rows;              // rows of a partial sum
};

struct Fp8Params {
    Fp8Plan plan;
    const uint8_t *codes;     // [tile][block][256][128]
    const float *code_scales; // [tile][block][2]
    const uint8_t *x;         // [row tile of 128][block][128][128]
    const float *x_scales;    // [row tile of 128][block][128]
    const float *factor;      // [row]
    int *counters;            // [tail tile][CTA of a pair]
    float *partials;          // [worker][2][CTA of a pair][2][32][partial rows][4]
    void *out;
    long long out_stride;
    int out_type;
    bool out_tma;             // there is a map_out
    int rows, V;
    long long wait_cycles;
    int stall;
};

// A worker's share of a tile: blocks [kb0, kb1).
struct Fp8Segment {
    int tile, kb0, kb1, tail;  // tail: the tile's number among the tail's, or -1
};
__device__ __forceinline__ int fp8_first_unit(const Fp8Plan &p, int worker) {
    return p.tail ? static_cast<int>(static_cast<long long>(p.units) * worker / p.tail_workers) : 0;
}
struct Fp8Walk {
    int unit, end, wave = 0;
    __device__ __forceinline__ Fp8Walk(const Fp8Plan &p, int worker)
        : unit(fp8_first_unit(p, min(worker, p.tail_workers))), end(fp8_first_unit(p, min(worker + 1, p.tail_workers))) {}
    __device__ __forceinline__ bool next(const Fp8Plan &p, int worker, Fp8Segment &s) {
        if (unit < end) {
            s.tail = unit / p.blocks;
            s.tile = p.waves * p.workers + s.tail;
            s.kb0 = unit - s.tail * p.blocks;
            s.kb1 = min(p.blocks, s.kb0 + end - unit);
            unit += s.kb1 - s.kb0;
            return true;
        }
        if (wave == p.waves) return false;
        s.tile = wave++ * p.workers + worker;
        s.tail = -1;
        s.kb0 = 0;
        s.kb1 = p.blocks;
        return true;
    }
};
// The worker that has a unit of the tail.
__device__ __forceinline__ int fp8_worker_of(const Fp8Plan &p, int unit) {
    return static_cast<int>(((unit + 1ll) * p.tail_workers - 1) / p.units);
}
// Where a worker leaves its part of a tail tile: 0 if that is its first, else 1 (whole tiles between the two stay in registers).
__device__ __forceinline__ int fp8_slot_of(const Fp8Plan &p, int worker, int tail) {
    return fp8_first_unit(p, worker) / p.blocks == tail ? 0 : 1;
}

// D (+)= A B^T, both operands e4m3 in shared memory, K = 32; from a converged warp by its elected lane.
template <bool kPair>
__device__ __forceinline__ void umma_f8_warp(uint32_t d, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    if (kPair)
        asm volatile(
            "{\n"
            " .reg .pred e, p;\n"
            " elect.sync _|e, 0xffffffff;\n"
            " setp.ne.b32 p, %4, 0;\n"
            " @e tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n"
            "}\n" ::"r"(d),
            "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n"
            " .reg .pred e, p;\n"
            " elect.sync _|e, 0xffffffff;\n"
            " setp.ne.b32 p, %4, 0;\n"
            " @e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n"
            "}\n" ::"r"(d),
            "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
            : "memory");
}
// kind::f8f6f4: fp32 accumulator, e4m3 A and B, both K-major.
constexpr uint32_t idesc_e4m3(int m, int n) { return (1u << 4) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(m >> 4) << 24); }

template <bool kPair>
__device__ __forceinline__ void fp8_commit(uint64_t *bar) {
    if (kPair)
        umma_commit_pair_multicast_warp(bar, 3);
    else
        umma_commit_warp(bar);
}

// Arrive on a barrier of the pair's even CTA.  What is handed over is tensor memory that has been read, nothing in memory: with
// release semantics at cluster scope the arrival waited for every load and store before it, a fence a block of columns.
__device__ __forceinline__ void mbar_arrive_relaxed(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// 32 columns of the accumulator on their way to a thread's registers, which are theirs after tmem_arrived.
__device__ __forceinline__ void tmem_ask_x32(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32"
        " {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_arrived(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;\n"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :
                 : "memory");
}

__device__ __forceinline__ int ld_shared_cluster(uint32_t cluster_addr) {
    int v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_addr) : "memory");
    return v;
}
__device__ __forceinline__ void mbar_complete_tx(uint64_t *bar, uint32_t bytes) {
    asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}

__device__ __forceinline__ uint32_t pair_of(float a, float b, int type) {
    if (type == RPD_TYPE_BF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// Logits from shared memory to their rows, a warp a row: 256 bytes, of which `cols` numbers are there.  545 rows of
// 126464 x 4096 in bf16 at an odd stride take 356 us so, 920 where every thread wrote its own row's; two numbers a store,
// from the row's first whole word on, took 404.
template <typename T>
__device__ __forceinline__ void fp8_store_rows(const uint8_t *stage, T *out, long long stride, int rows, int cols) {
    constexpr int kBytes = sizeof(T), kBox = 128 / kBytes;  // columns of a box
    const int warp = (threadIdx.x >> 5) & 3, lane = threadIdx.x & 31;
#pragma unroll 4
    for (int r = warp; r < rows; r += 4) {
        T *to = out + r * stride;
#pragma unroll
        for (int j = 0; j < 256 / kBytes / 32; ++j) {
            const int c = j * 32 + lane, byte = c % kBox * kBytes;
            if (c < cols)
                to[c] = *reinterpret_cast<const T *>(stage + c / kBox * kFp8BoxBytes + r * 128 + (((byte >> 4) ^ (r & 7)) << 4) + (byte & 15));
        }
    }
}

// Shared by a CTA's roles.
template <int kStages>
struct Fp8Shared {
    // done: the stage's MMAs are complete; acc_full: with them the accumulator
    uint64_t full[kStages], done[kStages], acc_full[2], acc_empty[2], drained;
    uint32_t tmem;
    int issued_of[2];  // stages that the TMA warps have asked for: codes; activations
    int give_up[2];    // whether a wait has run out, and its limit in 1024 cycles
    int last;
};

// After a wait that ran out: copies in flight land before the memory goes.  In a pair the even CTA's barriers count both's.
// Arrivals and bytes of stages that not every TMA warp has asked for are made up; none is more than kStages ahead.
template <bool kPair, int kStages>
__device__ __noinline__ void fp8_drain(Fp8Shared<kStages> &sm, const int (&codes)[2], const int (&rows)[2], const uint32_t (&bytes)[2],
                                       volatile int *abort) {
    const int any = max(max(codes[0], codes[1]), max(rows[0], rows[1]));
    for (int i = max(0, any - kStages); i < any; ++i) {
        uint64_t *bar = &sm.full[i % kStages];
#pragma unroll
        for (int role = 0; role < 2; ++role) {
            const bool mine = (role ? rows[0] : codes[0]) > i, peers = (role ? rows[1] : codes[1]) > i;
            if (mine && !peers && kPair) mbar_complete_tx(bar, bytes[role]);
            if (!mine && peers && kPair) mbar_arrive_expect_tx(bar, bytes[role]);
            if (!mine && !(peers && kPair)) mbar_arrive(bar);
        }
    }
    for (int i = max(0, any - kStages); i < any; ++i) wait_drained(&sm.full[i % kStages], (i / kStages) & 1, abort);
}

template <bool kPair>
__global__ void __launch_bounds__(kFp8Threads, 1)
    k_fp8_head(const __grid_constant__ CUtensorMap map_codes, const __grid_constant__ CUtensorMap map_x,
               const __grid_constant__ CUtensorMap map_out, const Fp8Params p) {
    constexpr int kCtas = kPair ? 2 : 1;
    constexpr int kCodeBytes = kFp8TileBytes / kCtas, kStageBytes = kFp8RowsBytes + kCodeBytes;
    constexpr int kStages = (kFp8Smem - 2048 - kFp8StageOut) / kStageBytes;
    static_assert(kFp8FewRows * kFp8FewPitch * 4 <= kFp8StageOut, "few rows' logits fit there too");
    extern __shared__ uint8_t smem_raw[];
    __shared__ Fp8Shared<kStages> sm;
    volatile int *abort = sm.give_up;
    uint8_t *smem = smem_raw + (1024 - (smem_u32(smem_raw) & 1023)) % 1024;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = kPair ? static_cast<int>(cluster_ctarank()) : 0, worker = blockIdx.x / kCtas;
    const Fp8Plan &plan = p.plan;

    pdl_trigger();
    if (warp == kFp8Mma) {
        if (kPair)
            tmem_alloc_pair(&sm.tmem, 512);
        else
            tmem_alloc(&sm.tmem, 512);
    }
    if (threadIdx.x == 0) {
        sm.give_up[0] = 0;
        sm.give_up[1] = static_cast<int>(p.wait_cycles >> 10);
        sm.issued_of[0] = sm.issued_of[1] = 0;
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&sm.full[i], 2);
            mbar_init(&sm.done[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sm.acc_full[i], 1);
            mbar_init(&sm.acc_empty[i], 8 * kCtas);
        }
        mbar_init(&sm.drained, 1);
        fence_mbar_init();
    }
    tc_fence_before_sync();
    __syncthreads();
    if (kPair) cluster_sync();
    tc_fence_after_sync();
    const uint32_t tmem = sm.tmem;
    Fp8Walk walk(plan, worker);
    Fp8Segment seg;

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFp8OtherRegs));
        if (warp == kFp8TmaCodes || warp == kFp8TmaRows) {
            // ---- TMA, a warp for the codes and one for the activations
            if (lane == 0) {
                const bool codes = warp == kFp8TmaCodes;
                if (!codes) {  // codes were laid out long ago: theirs need not wait
                    pdl_wait();
                    proxy_fence_global();
                }
                Cursor s;
                int issued = 0;
                bool ok = codes || !p.stall;
                while (ok && walk.next(plan, worker, seg)) {
                    const int col_tile = seg.tile / plan.row_tiles, row_tile = (seg.tile % plan.row_tiles) * kCtas + rank;
                    const int atoms = (min(kFp8RowsTile, p.rows - row_tile * kFp8RowsTile) + 7) / 8;  // of 8 rows; single CTAs' tiles have a row
                    for (int kb = seg.kb0; kb < seg.kb1; ++kb) {
                        if (issued == kStages) pdl_wait();
                        if (issued >= kStages) ok = wait_phase(&sm.done[s.at], s.phase ^ 1u, abort);
                        if (!ok) break;
                        uint8_t *to = smem + s.at * kStageBytes;
                        const long long code_block = static_cast<long long>(col_tile) * plan.blocks + kb;
                        const long long row_block = static_cast<long long>(row_tile) * plan.blocks + kb;
                        if (kPair) {
                            // the even CTA's barrier counts both CTAs' bytes
                            if (rank == 0) mbar_arrive_expect_tx(&sm.full[s.at], 2 * (codes ? kCodeBytes : kFp8RowsBytes));
                            const uint32_t bar = mapa_shared(smem_u32(&sm.full[s.at]), 0);
                            if (codes)
                                tma_load_2d_pair(to + kFp8RowsBytes, &map_codes, bar, 0, static_cast<int>(code_block * kFp8ColsTile) + rank * 128);
                            else
                                tma_load_2d_pair(to, &map_x, bar, 0, static_cast<int>(row_block * kFp8RowsTile));
                        } else if (codes) {
                            mbar_arrive_expect_tx(&sm.full[s.at], kFp8TileBytes);
                            bulk_copy(to + kFp8RowsBytes, p.codes + code_block * kFp8TileBytes, kFp8TileBytes, &sm.full[s.at]);
                        } else {  // (rows behind the last stay whatever they are: a row of A is a row of D)
                            mbar_arrive_expect_tx(&sm.full[s.at], atoms * 1024);
                            bulk_copy(to, p.x + row_block * kFp8RowsBytes, atoms * 1024, &sm.full[s.at]);
                        }
                        ++issued;
                        s.next(kStages);
                    }
                }
                sm.issued_of[codes ? 0 : 1] = issued;
            }
            __syncwarp();
        } else if (warp == kFp8Mma) {
            // ---- MMA issue, in a pair by the even CTA (every branch is warp-uniform)
            if (rank == 0) {
                const uint32_t idesc = idesc_e4m3(kFp8RowsTile * kCtas, kFp8ColsTile), base = __shfl_sync(0xffffffffu, tmem, 0);
                const uint64_t a_base = smem_desc_sw128(smem_u32(smem)), b_base = smem_desc_sw128(smem_u32(smem) + kFp8RowsBytes);
                Cursor s;
                uint32_t acc = 0, acc_phase = 1;  // of the two accumulators: they are used in turn
                bool ok = true;
                pdl_wait();
                while (ok && walk.next(plan, worker, seg)) {
                    for (int kb = seg.kb0; kb < seg.kb1; ++kb) {
                        ok = wait_phase_warp(&sm.full[s.at], s.phase, abort) && wait_phase_warp(&sm.acc_empty[acc], acc_phase, abort);
                        if (!ok) break;
                        tc_fence_after_sync();
                        const uint32_t at = static_cast<uint32_t>(s.at * kStageBytes) / 16;
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            umma_f8_warp<kPair>(base + acc * 256, a_base + at + k * 2, b_base + at + k * 2, idesc, k != 0);
                        fp8_commit<kPair>(&sm.done[s.at]);
                        fp8_commit<kPair>(&sm.acc_full[acc]);
                        acc_phase ^= acc;
                        acc ^= 1;
                        s.next(kStages);
                    }
                }
                // everything issued has to be done before TMEM is given back
                if (kPair)
                    umma_commit_pair_multicast_warp(&sm.drained, 1);
                else
                    umma_commit_warp(&sm.drained);
                wait_drained(&sm.drained, 0, abort);
            }
            __syncwarp();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kFp8EpilogueRegs));
        // ---- epilogue: a thread a row of activations and 128 of the tile's columns
        const int half = warp >> 2, slot = (warp & 3) * 32 + lane;
        const uint32_t from = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + half * 128;
        const uint32_t empty[2] = {kPair ? mapa_shared(smem_u32(&sm.acc_empty[0]), 0) : 0u, kPair ? mapa_shared(smem_u32(&sm.acc_empty[1]), 0) : 0u};
        uint32_t acc = 0, acc_phase = 0;
        bool ok = true;
        pdl_wait();
        while (walk.next(plan, worker, seg)) {
            const int col_tile = seg.tile / plan.row_tiles, row_tile = (seg.tile % plan.row_tiles) * kCtas + rank;
            const int live = min(kFp8RowsTile, p.rows - row_tile * kFp8RowsTile);  // in a pair it may be negative
            const bool reads = (warp & 3) * 32 < live;                              // uniform in the warp
            const float *xs = p.x_scales + (static_cast<long long>(row_tile) * plan.blocks + seg.kb0) * kFp8RowsTile + slot;
            const float *ws = p.code_scales + (static_cast<long long>(col_tile) * plan.blocks + seg.kb0) * 2 + half;
            float run[128];
#pragma unroll
            for (int i = 0; i < 128; ++i) run[i] = 0.f;
            float sx = 0.f, sw = 0.f;
            if (slot < live) {
                sx = __ldcg(xs);
                sw = *ws;
            }
            for (int kb = seg.kb0; kb < seg.kb1 && ok; ++kb) {
                const float f = sx * sw;
                xs += kFp8RowsTile;
                ws += 2;
                if (slot < live && kb + 1 < seg.kb1) {
                    sx = __ldcg(xs);
                    sw = *ws;
                }
                ok = wait_phase_warp(&sm.acc_full[acc], acc_phase, abort);
                if (!ok) break;
                tc_fence_after_sync();
                const auto release = [&] {  // all of the accumulator is in registers
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) {
                        if (kPair)
                            mbar_arrive_relaxed(empty[acc]);
                        else
                            mbar_arrive(&sm.acc_empty[acc]);
                    }
                };
                if (reads) {
                    uint32_t v[2][32];  // one part is multiplied while the next is on its way
                    tmem_ask_x32(from + acc * 256, v[0]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        tmem_arrived(v[c & 1]);
                        if (c < 3)
                            tmem_ask_x32(from + acc * 256 + (c + 1) * 32, v[(c + 1) & 1]);
                        else
                            release();
#pragma unroll
                        for (int i = 0; i < 32; ++i) run[c * 32 + i] = fmaf(f, __uint_as_float(v[c & 1][i]), run[c * 32 + i]);
                    }
                } else {
                    release();
                }
                acc_phase ^= acc;
                acc ^= 1;
            }
            if (!ok)
#pragma unroll
                for (int i = 0; i < 128; ++i) run[i] = __int_as_float(0x7FFFFFFF);
            if (seg.kb1 - seg.kb0 < plan.blocks) {
                // part of a tile: the last of its workers adds the parts up
                const long long part = 2ll * 32 * plan.partial_rows;  // in float4
                const int slot_of = fp8_slot_of(plan, worker, seg.tail);
                float4 *mine = reinterpret_cast<float4 *>(p.partials) + ((worker * 2 + slot_of) * kCtas + rank) * part +
                               half * 32ll * plan.partial_rows + slot;
                if (slot < live)
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const float4 v = make_float4(run[4 * i], run[4 * i + 1], run[4 * i + 2], run[4 * i + 3]);
                        mine[static_cast<long long>(i) * plan.partial_rows] = v;
                    }
                const int w0 = fp8_worker_of(plan, seg.tail * plan.blocks), w1 = fp8_worker_of(plan, (seg.tail + 1) * plan.blocks - 1);
                const int slot0 = fp8_slot_of(plan, w0, seg.tail);  // the others' shares begin in this tile: theirs is 0
                __threadfence();
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (threadIdx.x == 0) sm.last = counter_add_acq_rel(&p.counters[seg.tail * kCtas + rank], 1) == w1 - w0;
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (!sm.last) continue;
                __threadfence();
                if (!kPair && p.rows <= kFp8FewRows) {
                    // a thread a column: the parts of four rows are on their way at once
                    const int v = col_tile * kFp8ColsTile + threadIdx.x;
                    const float *from = p.partials + static_cast<long long>(threadIdx.x >> 2) * plan.partial_rows * 4 + (threadIdx.x & 3);
                    for (int r = 0; r < p.rows; r += 4) {
                        float y[4] = {0.f, 0.f, 0.f, 0.f};
                        for (int w = w0; w <= w1; w += 8) {
                            float x[8][4];
#pragma unroll
                            for (int i = 0; i < 8; ++i)
#pragma unroll
                                for (int j = 0; j < 4; ++j)
                                    x[i][j] = w + i <= w1 && r + j < p.rows
                                                  ? __ldcg(from + (2ll * (w + i) + (w + i == w0 ? slot0 : 0)) * part * 4 + (r + j) * 4)
                                                  : 0.f;
#pragma unroll
                            for (int i = 0; i < 8; ++i)
#pragma unroll
                                for (int j = 0; j < 4; ++j) y[j] += x[i][j];
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (r + j < p.rows && v < p.V)
                                store_out(p.out, p.out_type, (r + j) * p.out_stride + v, y[j] * __ldcg(p.factor + r + j));
                    }
                    continue;
                }
#pragma unroll
                for (int i = 0; i < 128; ++i) run[i] = 0.f;
                if (slot < live)
                    for (int w = w0; w <= w1; ++w) {
                        const float4 *theirs = reinterpret_cast<const float4 *>(p.partials) +
                                               ((w * 2 + (w == w0 ? slot0 : 0)) * kCtas + rank) * part +
                                               half * 32ll * plan.partial_rows + slot;
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const float4 v = __ldcg(theirs + static_cast<long long>(i) * plan.partial_rows);
                            run[4 * i] += v.x;
                            run[4 * i + 1] += v.y;
                            run[4 * i + 2] += v.z;
                            run[4 * i + 3] += v.w;
                        }
                    }
            }
            if (!kPair && p.rows <= kFp8FewRows) {
                // by way of shared memory: a thread has one row, of which it would write 128 columns by itself
                float *stage = reinterpret_cast<float *>(smem + kStages * kStageBytes);
                if (slot < live) {
                    const float factor = __ldcg(p.factor + slot);
#pragma unroll
                    for (int i = 0; i < 128; ++i) stage[slot * kFp8FewPitch + half * 128 + i] = run[i] * factor;
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
                const int v = col_tile * kFp8ColsTile + threadIdx.x;
                if (v < p.V)
                    for (int r = 0; r < p.rows; ++r) store_out(p.out, p.out_type, r * p.out_stride + v, stage[r * kFp8FewPitch + threadIdx.x]);
                asm volatile("bar.sync 1, 256;" ::: "memory");
                continue;
            }
            // Logits leave by way of shared memory, 256 bytes of each row at a time: by TMA, which goes on while the next tile is
            // added up, or a warp a row, where addresses do not fit that or the row ends in them (TMA writes 16 bytes at
            // least, and what follows a row is the caller's).  With stores of 32 bytes a thread 1024 rows of 152064 x 3584 took 537
            // us, by TMA 443.
            uint8_t *stage = smem + kStages * kStageBytes + half * (kFp8StageOut / 2);
            const bool first = threadIdx.x % 128 == 0, wide = p.out_type == RPD_TYPE_F32;
            const float factor = slot < live ? __ldcg(p.factor + static_cast<long long>(row_tile) * kFp8RowsTile + slot) : 0.f;
#pragma unroll
            for (int pass = 0; pass < 2; ++pass) {
                if (pass && !wide) break;
                if (first) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                asm volatile("bar.sync %0, 128;" ::"r"(2 + half) : "memory");
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    uint32_t w[4];
                    if (wide)
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(run[64 * pass + 4 * i + j] * factor);
                    else
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[j] = pair_of(run[8 * i + 2 * j] * factor, run[8 * i + 2 * j + 1] * factor, p.out_type);
                    *reinterpret_cast<uint4 *>(stage + (i >> 3) * kFp8BoxBytes + slot * 128 + (((i & 7) ^ (slot & 7)) * 16)) =
                        make_uint4(w[0], w[1], w[2], w[3]);
                }
                const int v0 = col_tile * kFp8ColsTile + half * 128 + pass * 64;
                if (p.out_tma && v0 + (wide ? 64 : 128) <= p.V) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    asm volatile("bar.sync %0, 128;" ::"r"(2 + half) : "memory");
                    if (first && live > 0) {
#pragma unroll
                        for (int b = 0; b < 2; ++b)
                            asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(
                                             reinterpret_cast<uint64_t>(&map_out)),
                                         "r"(v0 + b * (wide ? 32 : 64)), "r"(row_tile * kFp8RowsTile), "r"(smem_u32(stage + b * kFp8BoxBytes))
                                         : "memory");
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                } else {
                    asm volatile("bar.sync %0, 128;" ::"r"(2 + half) : "memory");
                    const long long at = static_cast<long long>(row_tile) * kFp8RowsTile * p.out_stride + v0;
                    if (wide)
                        fp8_store_rows(stage, static_cast<uint32_t *>(p.out) + at, p.out_stride, live, p.V - v0);
                    else
                        fp8_store_rows(stage, static_cast<uint16_t *>(p.out) + at, p.out_stride, live, p.V - v0);
                }
            }
        }
        if (threadIdx.x % 128 == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    tc_fence_before_sync();
    __syncthreads();
    if (kPair) cluster_sync();
    tc_fence_after_sync();
    if (threadIdx.x == 0 && rank == 0) {
        int codes[2] = {sm.issued_of[0], sm.issued_of[0]}, rows[2] = {sm.issued_of[1], sm.issued_of[1]};
        bool aborted = *abort != 0;
        if (kPair) {
            aborted |= ld_shared_cluster(mapa_shared(smem_u32(&sm.give_up[0]), 1)) != 0;
            codes[1] = ld_shared_cluster(mapa_shared(smem_u32(&sm.issued_of[0]), 1));
            rows[1] = ld_shared_cluster(mapa_shared(smem_u32(&sm.issued_of[1]), 1));
        }
        const uint32_t bytes[2] = {kCodeBytes, kFp8RowsBytes};
        if (aborted) fp8_drain<kPair>(sm, codes, rows, bytes, abort);
    }
    if (kPair) cluster_sync();
    if (warp == kFp8Mma) {
        if (kPair)
            tmem_dealloc_pair(tmem, 512);
        else
            tmem_free(tmem, 512);
    }
}

// Rows from which on CTAs work in pairs: more than a tile of one.
bool fp8_pairs(int rows) { return rows > kFp8RowsTile; }

struct Fp8Layout {
    Fp8Plan plan;
    int grid;
    long long codes, scales, factor, counters, partials, bytes;  // where the parts of the workspace begin, and its size
    Fp8Layout(int rows, int V, int blocks, int num_sms) {
        const int ctas = fp8_pairs(rows) ? 2 : 1, most = std::max(1, num_sms / ctas);
        const long long tiles128 = (rows + kFp8RowsTile - 1ll) / kFp8RowsTile;
        plan.blocks = blocks;
        plan.row_tiles = static_cast<int>((tiles128 + ctas - 1) / ctas);
        const int tiles = (V + kFp8ColsTile - 1) / kFp8ColsTile * plan.row_tiles;
        plan.workers = tiles >= most ? most : std::clamp(static_cast<int>(static_cast<long long>(tiles) * blocks / kLeast), tiles, most);
        plan.waves = tiles / plan.workers;
        plan.tail = tiles % plan.workers;
        plan.units = plan.tail * blocks;
        plan.tail_workers = std::clamp(plan.units / kLeast, plan.tail, plan.workers);
        plan.partial_rows = std::min(rows, kFp8RowsTile);
        grid = plan.workers * ctas;
        const long long padded = static_cast<long long>(plan.row_tiles) * ctas;
        codes = 0;
        scales = codes + padded * blocks * kFp8RowsBytes;
        factor = scales + padded * blocks * kFp8RowsTile * 4;
        counters = factor + padded * kFp8RowsTile * 4;
        partials = counters + (plan.tail * ctas * 4 + 255) / 256 * 256;
        bytes = partials + (plan.tail ? static_cast<long long>(plan.tail_workers) * 2 * ctas * kFp8ColsTile * plan.partial_rows * 4 : 0);
    }
    // Blocks of shared tiles that a worker has at least (as long as every tile has a worker): 50021 x 1001, 13 rows take 15.5 us
    // with 8, 20 with 4; 4096 x 4096, one row 11.4 with 8, 10.2 with 4, 14.1 with 16, 128 rows 21.7, 29.0 and 22.4.
    static constexpr int kLeast = 8;
};

// Of a call: more rows than a launch takes are several launches, one after the other.
long long fp8_workspace(int rows, int V, int blocks, int num_sms) {
    if (rows == 0) return 0;
    long long bytes = Fp8Layout(std::min(rows, kFp8MaxRows), V, blocks, num_sms).bytes;
    if (rows > kFp8MaxRows && rows % kFp8MaxRows) bytes = std::max(bytes, Fp8Layout(rows % kFp8MaxRows, V, blocks, num_sms).bytes);
    return bytes;
}

// Boxes of 128 rows of 128 bytes.
int fp8_encode(const void *base, long long rows, CUtensorMap *map) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return op_fail(RPD_ERR_CUDA, "cuTensorMapEncodeTiled entry point unavailable");
    cuuint64_t dims[2] = {128, static_cast<cuuint64_t>(rows)}, strides[1] = {128};
    cuuint32_t box[2] = {128, 128}, step[2] = {1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, step,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? RPD_OK : op_fail(RPD_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", static_cast<int>(r));
}

// Boxes of 128 rows x 128 bytes of logits, swizzled as the epilogue writes them.
int fp8_encode_out(void *out, int size, int rows, int V, long long stride, CUtensorMap *map) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return op_fail(RPD_ERR_CUDA, "cuTensorMapEncodeTiled entry point unavailable");
    cuuint64_t dims[2] = {static_cast<cuuint64_t>(V), static_cast<cuuint64_t>(rows)}, strides[1] = {static_cast<cuuint64_t>(stride) * size};
    cuuint32_t box[2] = {128u / size, 128}, step[2] = {1, 1};
    const CUresult r = fn(map, size == 2 ? CU_TENSOR_MAP_DATA_TYPE_UINT16 : CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, out, dims, strides, box, step,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? RPD_OK : op_fail(RPD_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", static_cast<int>(r));
}

template <bool kPair>
cudaError_t launch_fp8(const CUtensorMap &codes, const CUtensorMap &x, const CUtensorMap &out, const Fp8Params &p, int grid, cudaStream_t s) {
    cudaError_t e = cudaFuncSetAttribute(k_fp8_head<kPair>, cudaFuncAttributeMaxDynamicSharedMemorySize, kFp8Smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(kFp8Threads);
    cfg.dynamicSmemBytes = kFp8Smem - 1024;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kPair ? 2 : 1;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k_fp8_head<kPair>, codes, x, out, p);
}

// ------------------------------------------------------------------------------ the quantiser

// Eight neighbouring numbers of a row as they are.
template <typename T>
struct Eight {
    uint4 v;
    __device__ __forceinline__ void load(const T *row, int col, int cols, int align) { v = load_chunk(row, col, cols, align); }
    __device__ __forceinline__ void clear() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void get(float2 (&u)[4]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = pair_value(w[i], T());
    }
};
template <>
struct Eight<float> {
    float2 v[4];
    __device__ __forceinline__ void load(const float *row, int col, int cols, int align) {
        if (col + 8 <= cols && align == 16) {
            const float4 a = reinterpret_cast<const float4 *>(row + col)[0], b = reinterpret_cast<const float4 *>(row + col)[1];
            v[0] = make_float2(a.x, a.y);
            v[1] = make_float2(a.z, a.w);
            v[2] = make_float2(b.x, b.y);
            v[3] = make_float2(b.z, b.w);
            return;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = make_float2(col + 2 * i < cols ? row[col + 2 * i] : 0.f, col + 2 * i + 1 < cols ? row[col + 2 * i + 1] : 0.f);
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = make_float2(0.f, 0.f);
    }
    __device__ __forceinline__ void get(float2 (&u)[4]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = v[i];
    }
};

__device__ __forceinline__ void store_codes(uint8_t *row, int col, int cols, bool vec, uint2 q) {
    if (vec && col + 8 <= cols) {
        *reinterpret_cast<uint2 *>(row + col) = q;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (col + i < cols) row[col + i] = static_cast<uint8_t>((i < 4 ? q.x : q.y) >> (8 * (i & 3)));
}
// The same where 8-byte stores do not fit, 16 lanes having a row's block: whole words, of a lane's codes and the next one's.  Every lane
// of the warp calls it.  20832 x 2120 bf16 in blocks of 128 rows, codes at an odd stride: 45 us, byte by byte 82; 35 where 8 bytes fit.
__device__ __forceinline__ void store_codes_words(bool there, uint8_t *row, int col, int cols, uint2 q) {
    const uint32_t next = __shfl_down_sync(0xffffffffu, q.x, 1, 16);
    if (!there) return;
    const int in_block = col & (kFp8Block - 1);
    if (col - in_block + kFp8Block > cols) {
        store_codes(row, col, cols, false, q);
        return;
    }
    uint8_t *to = row + col;
    const int skip = static_cast<int>(-reinterpret_cast<uintptr_t>(to) & 3);  // bytes before the first whole word: of the lane before
    uint32_t *words = reinterpret_cast<uint32_t *>(to + skip);
    words[0] = __funnelshift_r(q.x, q.y, 8 * skip);
    if (in_block + 8 < kFp8Block || skip == 0)
        words[1] = __funnelshift_r(q.y, next, 8 * skip);
    else
#pragma unroll
        for (int i = 1; i < 4; ++i)
            if (i >= skip) to[4 + i] = static_cast<uint8_t>(q.y >> (8 * i));
    if (in_block == 0)
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < skip) to[i] = static_cast<uint8_t>(q.x >> (8 * i));
}

struct Fp8QuantizeParams {
    const void *x;
    long long x_stride, codes_stride;
    int rows, cols, x_align, vec;
    uint8_t *codes;
    float *scales;
};

template <typename T, int n>
__device__ __forceinline__ float largest_of(const Eight<T> (&x)[n]) {
    float amax = 0.f;
#pragma unroll
    for (int j = 0; j < n; ++j) {
        float2 u[4];
        x[j].get(u);
#pragma unroll
        for (int k = 0; k < 4; ++k) amax = fmaxf(amax, fmaxf(fabsf(u[k].x), fabsf(u[k].y)));
    }
    return amax;
}

// Blocks of 128 columns of a row: 16 lanes have one, the grid's next one is found without a division.
template <typename T>
__global__ void __launch_bounds__(256) k_fp8_quantize_rows(const Fp8QuantizeParams p) {
    const int lanes = threadIdx.x >> 4, col = (threadIdx.x & 15) * 8, blocks = (p.cols + kFp8Block - 1) / kFp8Block;
    const long long n = static_cast<long long>(p.rows) * blocks, step = gridDim.x * 16ll;
    long long i = blockIdx.x * 16ll + lanes, row = i / blocks;
    int block = static_cast<int>(i - row * blocks);
    const long long step_rows = step / blocks;
    const int step_blocks = static_cast<int>(step - step_rows * blocks);
    pdl_trigger();
    pdl_wait();
    for (long long first = blockIdx.x * 16ll; first < n; first += step, i += step) {
        const int at = block * kFp8Block + col;
        Eight<T> x[1];
        if (i < n)
            x[0].load(static_cast<const T *>(p.x) + row * p.x_stride, at, p.cols, p.x_align);
        else
            x[0].clear();
        float amax = largest_of(x);
#pragma unroll
        for (int o = 8; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        const float scale = amax / kFp8Most, by = scale > 0.f ? scale : 1.f;
        float2 u[4];
        x[0].get(u);
        const uint2 q = fp8_codes(u, by, 1.f / by);
        uint8_t *to = p.codes + row * p.codes_stride;
        if (i < n && col == 0) p.scales[i] = scale;
        if (!p.vec)
            store_codes_words(i < n, to, at, p.cols, q);
        else if (i < n)
            store_codes(to, at, p.cols, true, q);
        row += step_rows;
        block += step_blocks;
        if (block >= blocks) {
            block -= blocks;
            ++row;
        }
    }
}

// Blocks of 128 x 128: a CTA has one, whose numbers stay in registers (8 rows a thread, 8 columns each) between its largest
// and its codes, while the next one's are on their way: 262 us for a head of 126464 x 4096.  (Without that, at two to four CTAs
// an SM, 370 to 330.)
template <typename T>
__global__ void __launch_bounds__(256, 2) k_fp8_quantize_blocks(const Fp8QuantizeParams p) {
    constexpr int kRows = kFp8Block / 16;
    __shared__ float red[2][8];
    const int lanes = threadIdx.x >> 4, col = (threadIdx.x & 15) * 8, blocks = (p.cols + kFp8Block - 1) / kFp8Block;
    const long long n = (p.rows + kFp8Block - 1ll) / kFp8Block * blocks;
    const auto load = [&](Eight<T> (&x)[kRows], long long i) {
        const long long high = i / blocks;
        const int at = static_cast<int>(i - high * blocks) * kFp8Block + col;
        const int row = static_cast<int>(high) * kFp8Block + lanes;
        const T *from = static_cast<const T *>(p.x) + row * p.x_stride;
#pragma unroll
        for (int j = 0; j < kRows; ++j, from += 16 * p.x_stride) {
            if (row + 16 * j < p.rows)
                x[j].load(from, at, p.cols, p.x_align);
            else
                x[j].clear();
        }
    };
    pdl_trigger();
    pdl_wait();
    Eight<T> x[kRows], next[kRows];
    load(x, blockIdx.x);
    int turn = 0;
    for (long long i = blockIdx.x; i < n; i += gridDim.x, turn ^= 1) {
        if (i + gridDim.x < n) load(next, i + gridDim.x);
        float amax = largest_of(x);
#pragma unroll
        for (int o = 16; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        if ((threadIdx.x & 31) == 0) red[turn][threadIdx.x >> 5] = amax;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) amax = fmaxf(amax, red[turn][w]);
        const float scale = amax / kFp8Most, by = scale > 0.f ? scale : 1.f, inverse = 1.f / by;
        if (threadIdx.x == 0) p.scales[i] = scale;
        const long long high = i / blocks;
        const int at = static_cast<int>(i - high * blocks) * kFp8Block + col;
        const int row = static_cast<int>(high) * kFp8Block + lanes;
        uint8_t *to = p.codes + row * p.codes_stride;
        if (p.vec) {
#pragma unroll
            for (int j = 0; j < kRows; ++j, to += 16 * p.codes_stride) {
                float2 u[4];
                x[j].get(u);
                if (row + 16 * j < p.rows) store_codes(to, at, p.cols, true, fp8_codes(u, by, inverse));
            }
        } else {
#pragma unroll
            for (int j = 0; j < kRows; ++j, to += 16 * p.codes_stride) {
                float2 u[4];
                x[j].get(u);
                store_codes_words(row + 16 * j < p.rows, to, at, p.cols, fp8_codes(u, by, inverse));
            }
        }
#pragma unroll
        for (int j = 0; j < kRows; ++j) x[j] = next[j];
    }
}

template <typename T>
cudaError_t launch_quantize(const Fp8QuantizeParams &p, int high, int num_sms, cudaStream_t s) {
    const long long blocks = (p.cols + kFp8Block - 1ll) / kFp8Block;
    if (high == 1)
        return launch_pdl(k_fp8_quantize_rows<T>, dim3(static_cast<unsigned>(std::min<long long>((p.rows * blocks + 15) / 16, num_sms * 32ll))),
                          dim3(256), 0, s, p);
    return launch_pdl(k_fp8_quantize_blocks<T>,
                      dim3(static_cast<unsigned>(std::min<long long>((p.rows + kFp8Block - 1ll) / kFp8Block * blocks, num_sms * 2ll))), dim3(256), 0,
                      s, p);
}

}  // namespace
}  // namespace rpd

using namespace rpd;

struct rpd_fp8 {
    int d = 0, V = 0, device = 0, num_sms = 0, blocks = 0;
    long long tiles = 0;
    uint8_t *codes = nullptr;
    float *scales = nullptr;
    bool set = false;
    int64_t wait_us = 2000000;
    bool stall = false;
    CUtensorMap map;  // the codes
};

extern "C" {

rpd_fp8 *rpd_fp8_create(int d, int V) {
    if (d < 1 || V < 1) {
        op_fail(RPD_ERR_INVALID_ARGUMENT, "d and V must be >= 1 (got %d, %d)", d, V);
        return nullptr;
    }
    if (d > kQuantMaxD || V > kQuantMaxV) {
        op_fail(RPD_ERR_UNSUPPORTED, "d must be <= %d and V <= %d (got %d, %d)", kQuantMaxD, kQuantMaxV, d, V);
        return nullptr;
    }
    rpd_fp8 *h = new (std::nothrow) rpd_fp8();
    if (!h) {
        op_fail(RPD_ERR_OUT_OF_MEMORY, "out of host memory");
        return nullptr;
    }
    cudaError_t e = cudaGetDevice(&h->device);
    if (e == cudaSuccess) e = cudaSetDevice(h->device);  // binds the primary context to this thread
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&h->num_sms, cudaDevAttrMultiProcessorCount, h->device);
    if (e != cudaSuccess) {
        op_cuda_fail(e, "device query");
        delete h;
        return nullptr;
    }
    if (check_device(h->device) != RPD_OK) {
        delete h;
        return nullptr;
    }
    h->d = d;
    h->V = V;
    h->blocks = (d + kFp8Block - 1) / kFp8Block;
    h->tiles = (V + kFp8ColsTile - 1) / kFp8ColsTile;
    if (h->tiles * h->blocks * kFp8ColsTile >= 1ll << 31) {  // rows of the codes' tensor map (a copy would be 256 GB)
        op_fail(RPD_ERR_UNSUPPORTED, "a head of %d x %d is too large", V, d);
        delete h;
        return nullptr;
    }
    return h;
}

int rpd_fp8_set_weights(rpd_fp8 *h, const void *codes, const float *scales, void *stream_ptr) {
    if (!h || !codes || !scales) return op_fail(RPD_ERR_INVALID_ARGUMENT, "null argument");
    if (!aligned_to(scales, 4)) return op_fail(RPD_ERR_INVALID_ARGUMENT, "scales must be 4-byte aligned");
    DeviceGuard dg(h->device);
    if (dg.err != cudaSuccess) return op_cuda_fail(dg.err, "cudaSetDevice");
    if (!pointer_usable(codes, h->device, false) || !pointer_usable(scales, h->device, false))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "codes and scales must be device memory on the head's device");
    cudaStream_t s = static_cast<cudaStream_t>(stream_ptr);
    cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(s, &capturing);
    if (e != cudaSuccess) return op_cuda_fail(e, "cudaStreamIsCapturing");
    if (capturing != cudaStreamCaptureStatusNone)
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "the weights cannot be set while the stream is being captured");
    RelaxedCapture rc;
    // The layout's size is the head's: made once, and filled again by later calls.
    if (!h->codes) {
        e = cudaMalloc(&h->codes, static_cast<size_t>(h->tiles) * h->blocks * kFp8TileBytes);
        if (e == cudaSuccess) {
            e = cudaMalloc(&h->scales, static_cast<size_t>(h->tiles) * h->blocks * 2 * sizeof(float));
            if (e != cudaSuccess) {
                cudaFree(h->codes);
                h->codes = nullptr;
            }
        }
        if (e != cudaSuccess) return op_cuda_fail(e, "memory for the 8-bit weights");
        const int code = fp8_encode(h->codes, h->tiles * h->blocks * kFp8ColsTile, &h->map);
        if (code != RPD_OK) {
            cudaFree(h->codes);
            cudaFree(h->scales);
            h->codes = nullptr;
            h->scales = nullptr;
            return code;
        }
    }
    e = launch_plain(k_fp8_pack, h->num_sms * 8, 256, s, static_cast<const uint8_t *>(codes), reinterpret_cast<uint4 *>(h->codes), h->V,
                     h->d, h->tiles, h->blocks);
    if (e == cudaSuccess)
        e = launch_plain(k_fp8_pack_scales, h->num_sms * 4, 256, s, scales, h->scales, (h->V + 127) / 128, h->tiles, h->blocks);
    const cudaError_t done = cudaStreamSynchronize(s);  // nothing of the caller's is read after the call
    if (e == cudaSuccess) e = done;
    h->set = e == cudaSuccess;
    return e == cudaSuccess ? RPD_OK : op_cuda_fail(e, "layout of the 8-bit weights");
}

int64_t rpd_fp8_workspace(const rpd_fp8 *h, int rows) {
    if (!h || rows < 0) {
        op_fail(RPD_ERR_INVALID_ARGUMENT, "null head or negative rows");
        return -1;
    }
    return fp8_workspace(rows, h->V, h->blocks, h->num_sms);
}

int rpd_fp8_logits(const rpd_fp8 *h, const void *x, int x_type, int64_t x_stride, int rows, const void *gain, float eps, void *out,
                   int out_type, int64_t out_stride, void *workspace, int64_t workspace_bytes, void *stream_ptr) {
    if (!h) return op_fail(RPD_ERR_INVALID_ARGUMENT, "null head");
    if (!h->set) return op_fail(RPD_ERR_NO_HEAD, "rpd_fp8_set_weights has not been called");
    if (x_type != RPD_TYPE_BF16 && x_type != RPD_TYPE_F16) return op_fail(RPD_ERR_INVALID_ARGUMENT, "x must be bf16 or fp16");
    if (!type_size(out_type)) return op_fail(RPD_ERR_INVALID_ARGUMENT, "out must be bf16, fp16 or fp32");
    if (rows < 0) return op_fail(RPD_ERR_INVALID_ARGUMENT, "rows must be >= 0");
    if (rows == 0) return RPD_OK;
    if (!x || !out) return op_fail(RPD_ERR_INVALID_ARGUMENT, "null buffer");
    if (rows > 1 && (x_stride < h->d || out_stride < h->V))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "rows overlap: x_stride must be >= %d and out_stride >= %d", h->d, h->V);
    if (gain && (!(eps >= 0.f) || !std::isfinite(eps))) return op_fail(RPD_ERR_INVALID_ARGUMENT, "eps must be finite and >= 0");
    if (!aligned_to(x, 2) || (gain && !aligned_to(gain, 2)) || !aligned_to(out, type_size(out_type)))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "x, gain and out must be aligned to their elements");
    const int64_t need = fp8_workspace(rows, h->V, h->blocks, h->num_sms);
    if (!workspace || workspace_bytes < need || !aligned_to(workspace, 256))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "workspace: %lld bytes at a 256-byte boundary needed", static_cast<long long>(need));
    DeviceGuard dg(h->device);
    if (dg.err != cudaSuccess) return op_cuda_fail(dg.err, "cudaSetDevice");
    if (!pointer_usable(x, h->device, false) || !pointer_usable(out, h->device, false) || (gain && !pointer_usable(gain, h->device, false)) ||
        !pointer_usable(workspace, h->device, false))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "x, gain, out and workspace must be device memory on the head's device");
    cudaStream_t s = static_cast<cudaStream_t>(stream_ptr);
    // (more rows than a launch takes: one launch after the other, each with the whole workspace)
    for (long long first = 0; first < rows; first += kFp8MaxRows) {
        const int n = static_cast<int>(std::min<long long>(rows - first, kFp8MaxRows));
        const Fp8Layout at(n, h->V, h->blocks, h->num_sms);
        uint8_t *w = static_cast<uint8_t *>(workspace);
        Fp8RowsParams q{};
        q.x = static_cast<const uint16_t *>(x) + first * x_stride;
        q.gain = gain;
        q.x_stride = x_stride;
        q.d = h->d;
        q.blocks = h->blocks;
        q.x_align = common_align(reinterpret_cast<uintptr_t>(x) | (rows > 1 ? static_cast<uintptr_t>(x_stride) * 2 : 0));
        q.gain_align = common_align(reinterpret_cast<uintptr_t>(gain));
        q.eps = eps;
        q.codes = w + at.codes;
        q.scales = reinterpret_cast<float *>(w + at.scales);
        q.factor = reinterpret_cast<float *>(w + at.factor);
        q.counters = reinterpret_cast<int *>(w + at.counters);
        q.num_counters = at.plan.tail * (fp8_pairs(n) ? 2 : 1);
        cudaError_t e = x_type == RPD_TYPE_BF16 ? launch_pdl(k_fp8_rows<__nv_bfloat16>, dim3(n), dim3(256), 0, s, q)
                                                : launch_pdl(k_fp8_rows<__half>, dim3(n), dim3(256), 0, s, q);
        if (e != cudaSuccess) return op_cuda_fail(e, "8-bit head launch");
        Fp8Params p{};
        p.plan = at.plan;
        p.codes = h->codes;
        p.code_scales = h->scales;
        p.x = q.codes;
        p.x_scales = q.scales;
        p.factor = q.factor;
        p.counters = q.counters;
        p.partials = reinterpret_cast<float *>(w + at.partials);
        p.out = static_cast<uint8_t *>(out) + first * out_stride * type_size(out_type);
        p.out_stride = out_stride;
        p.out_type = out_type;
        p.rows = n;
        p.V = h->V;
        p.wait_cycles = h->wait_us * kWaitCyclesPerUs;
        p.stall = h->stall ? 1 : 0;
        CUtensorMap map = h->map, map_out = h->map;
        // more rows than few, and addresses that TMA takes
        if (n > kFp8FewRows && aligned_to(p.out, 16) && out_stride * type_size(out_type) % 16 == 0) {
            const int code = fp8_encode_out(p.out, type_size(out_type), n, h->V, out_stride, &map_out);
            if (code != RPD_OK) return code;
            p.out_tma = true;
        }
        if (fp8_pairs(n)) {
            const int code = fp8_encode(q.codes, (at.scales - at.codes) / 128, &map);
            if (code != RPD_OK) return code;
            e = launch_fp8<true>(h->map, map, map_out, p, at.grid, s);
        } else {
            e = launch_fp8<false>(h->map, map, map_out, p, at.grid, s);
        }
        if (e != cudaSuccess) return op_cuda_fail(e, "8-bit head launch");
    }
    return RPD_OK;
}

int rpd_fp8_set_wait_limit(rpd_fp8 *h, int64_t microseconds) {
    if (!h) return op_fail(RPD_ERR_INVALID_ARGUMENT, "null head");
    if (microseconds < 1000 || microseconds > kMaxWaitUs)
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "the wait limit must be 1000 .. %lld us", static_cast<long long>(kMaxWaitUs));
    h->wait_us = microseconds;
    return RPD_OK;
}

int rpd_fp8_inject_stall(rpd_fp8 *h, int on) {
    if (!h) return op_fail(RPD_ERR_INVALID_ARGUMENT, "null head");
    h->stall = on != 0;
    return RPD_OK;
}

void rpd_fp8_destroy(rpd_fp8 *h) {
    if (!h) return;
    DeviceGuard dg(h->device);
    RelaxedCapture rc;
    cudaFree(h->codes);
    cudaFree(h->scales);
    cudaGetLastError();
    delete h;
}

int rpd_fp8_quantize(const void *x, int x_type, int64_t x_stride, int rows, int cols, int block_rows, void *codes, int64_t codes_stride,
                     float *scales, void *stream_ptr) {
    const int size = type_size(x_type);
    if (!size) return op_fail(RPD_ERR_INVALID_ARGUMENT, "x must be bf16, fp16 or fp32");
    if (rows < 0 || cols < 0) return op_fail(RPD_ERR_INVALID_ARGUMENT, "rows and cols must be >= 0");
    if (block_rows != 1 && block_rows != 128) return op_fail(RPD_ERR_UNSUPPORTED, "block_rows must be 1 or 128 (got %d)", block_rows);
    if (rows == 0 || cols == 0) return RPD_OK;
    if (!x || !codes || !scales) return op_fail(RPD_ERR_INVALID_ARGUMENT, "null buffer");
    if (rows > 1 && (x_stride < cols || codes_stride < cols))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "rows overlap: strides must be >= %d", cols);
    if (!aligned_to(x, size) || !aligned_to(scales, 4))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "x and scales must be aligned to their elements");
    cudaPointerAttributes a{};
    if (cudaPointerGetAttributes(&a, x) != cudaSuccess || (a.type != cudaMemoryTypeDevice && a.type != cudaMemoryTypeManaged)) {
        cudaGetLastError();
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "x must be device memory");
    }
    DeviceGuard dg(a.device);
    if (dg.err != cudaSuccess) return op_cuda_fail(dg.err, "cudaSetDevice");
    if (!pointer_usable(codes, a.device, false) || !pointer_usable(scales, a.device, false))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "codes and scales must be device memory on the device of x");
    const int ready = check_device(a.device);
    if (ready != RPD_OK) return ready;
    int num_sms = 0;
    cudaError_t e = cudaDeviceGetAttribute(&num_sms, cudaDevAttrMultiProcessorCount, a.device);
    if (e != cudaSuccess) return op_cuda_fail(e, "device query");
    Fp8QuantizeParams p{};
    p.x = x;
    p.x_stride = x_stride;
    p.codes_stride = codes_stride;
    p.rows = rows;
    p.cols = cols;
    p.x_align = common_align(reinterpret_cast<uintptr_t>(x) | (rows > 1 ? static_cast<uintptr_t>(x_stride) * size : 0));
    p.vec = aligned_to(codes, 8) && (rows == 1 || codes_stride % 8 == 0);
    p.codes = static_cast<uint8_t *>(codes);
    p.scales = scales;
    cudaStream_t s = static_cast<cudaStream_t>(stream_ptr);
    e = x_type == RPD_TYPE_F32    ? launch_quantize<float>(p, block_rows, num_sms, s)
        : x_type == RPD_TYPE_BF16 ? launch_quantize<__nv_bfloat16>(p, block_rows, num_sms, s)
                                  : launch_quantize<__half>(p, block_rows, num_sms, s);
    return e == cudaSuccess ? RPD_OK : op_cuda_fail(e, "quantiser launch");
}

}  // extern "C"
