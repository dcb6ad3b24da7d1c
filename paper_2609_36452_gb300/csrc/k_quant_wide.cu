// k_quant_wide.cu - the 4-bit head for more than a few activations: the same sums as k_quant_rows
// (k_quant.cu), on the fifth-generation tensor cores.
//
// The weights of 128 matrix rows are the MMA's A operand (M), read from tensor memory where four warps have put
// (q - z) 2^-9 as fp16, exactly, a thread a matrix row; the activations are B (N: 32 or 64 of them a pass), as scale_u
// leaves them, staged in shared memory with 128-byte swizzling.  A group's product is summed in TMEM; eight other
// warps read it and add it, scaled, to running sums in registers, so that scales stay exact as in the kernel for few
// rows.
//
// A CTA (one an SM) has a pass of up to 64 activation rows and a contiguous range of pairs of 16-row tiles.  It works
// on 256 matrix rows at a time, as two halves that share every stage of activations: a stage is 128 columns of both (16 KB
// of codes, 8 or 16 KB of activations).
//
// What bounds it: not HBM (one pass over a 126464 x 4096 head is 39 us; 17 rows take 96.2, 32 rows 98.7, 33 rows 109, 64
// rows 113, 128 rows 218, and with stored zero points 20 rows 107), nor the tensor cores (an MMA of M = 128 and N =
// 32 / 64 with A in TMEM takes 18 / 32 cycles, 15 us a pass in all), but what a stage costs its roles one after the other: 1550 cycles
// where the codes' share of HBM is 700.  Of 93 us, measured when the operand still was the masked codes, 22 went without
// the stores to TMEM, 6 without the epilogue's arithmetic, 5 without the MMAs; copies and hand-overs alone took 59.
// Tried and no faster: two sets of warps for the operand, two issuers, three operands in flight, 128 rows at a time
// with six in flight (109 us).
//
// (The masked codes themselves as subnormal operands, and -z sum u added by the epilogue, were 3 us faster, 12 with
// stored zero points, but for the reason given in k_quant.cu logits of d = 4096 were 9e-7 of their norm off in place of
// 2.1e-7.)
//
// Roles: warps 0-3 weights to TMEM (lanes by warp % 4), warps 4-11 epilogue (half = warp / 4 - 1), warps 12 and 13 TMA (codes;
// activations), warp 14 MMA issue and TMEM.  Every wait is bounded (from when the kernels before this one are done: a role
// waits for these before its first bounded wait); where one runs out the CTA's remaining logits are NaN.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "ptx.cuh"
#include "quant_internal.h"

namespace rpd {
namespace {

constexpr int kWideThreads = 15 * 32;
constexpr int kWideTmaCodes = 12, kWideTmaRows = 13, kWideMma = 14;  // warps
constexpr int kWideHalf = 4;                        // pairs of tiles (32 matrix rows) of a half (128 TMEM lanes)
constexpr int kWideUnit = 2 * kWideHalf;
constexpr int kWidePairBytes = 2048;                // codes of a pair and stage: [block][tile][512 bytes]
constexpr int kWideCodeBytes = kWideUnit * kWidePairBytes;
constexpr int kWideMaxStages = 8;
constexpr int kWideSlots = 2;                       // A operands in TMEM: 128 columns each (two halves)
constexpr int kWideAccCols = 256;                   // TMEM columns before the A operands: two accumulators
constexpr int kWideSmem = 226 * 1024;
constexpr int kMetaChunk = 4;                       // groups whose scales a warp copies at a time
constexpr int kMetaSlots = 4;

struct WideParams {
    QuantParams q;           // q.per rows a pass: blockIdx.x's
    const uint8_t *x;        // [passes][blocks][n][128 bytes], swizzled
    const float *factor;     // [passes][n]
    int stages;              // at least kWideSlots
};

// ------------------------------------------------------------------------------ activations

// One row of a pass: its fp16 elements in the order of the main kernel's stages, and its factor.  Rows that pad the
// pass are zero.
template <typename T>
__global__ void __launch_bounds__(256) k_quant_wide_x(const QuantParams p, int n, uint8_t *xs, float *factor) {
    __shared__ float red[2][8];
    const int slot = blockIdx.x % n, pass = blockIdx.x / n, r = pass * p.per + slot;
    const bool live = slot < p.per && r < p.rows;
    const int chunks = p.blocks * 8, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const T *x = static_cast<const T *>(p.x) + r * p.x_stride;
    const T *gain = static_cast<const T *>(p.gain);
    pdl_trigger();
    pdl_wait();
    float ss = 0.f, top = 0.f;
    if (live)
        for (int c = threadIdx.x; c < chunks; c += 256) {
            float2 u[4];
            ss += make_u<T>(load_chunk(x, c * 8, p.d, p.x_align), gain != nullptr,
                            gain ? load_chunk(gain, c * 8, p.d, p.gain_align) : make_uint4(0, 0, 0, 0), u);
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(u[i].x), fabsf(u[i].y)));
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
    if (gain && live && norm_unusual(ss, top, p.eps, E)) {
        const NormFactor f = norm_factor_unusual(x, chunks, p.d, p.x_align, p.eps, top, E);
        E = f.E;
        if (threadIdx.x == 0) factor[pass * n + slot] = f.factor;
    } else if (threadIdx.x == 0) {
        factor[pass * n + slot] = gain ? norm_factor(ss, static_cast<float>(p.d), p.eps, E) : ldexpf(1.f, E);
    }
    for (int c = threadIdx.x; c < chunks; c += 256) {
        uint4 w = make_uint4(0, 0, 0, 0);
        if (live) {
            float2 u[4];
            make_u<T>(load_chunk(x, c * 8, p.d, p.x_align), gain != nullptr,
                      gain ? load_chunk(gain, c * 8, p.d, p.gain_align) : make_uint4(0, 0, 0, 0), u);
            scale_u(u, E, w);
        }
        const long long row = (static_cast<long long>(pass) * p.blocks + c / 8) * n + slot;
        *reinterpret_cast<uint4 *>(xs + row * 128 + ((c % 8) ^ (slot % 8)) * 16) = w;
    }
}

// ------------------------------------------------------------------------------ PTX

__device__ __forceinline__ void bulk_copy(void *to, const void *from, uint32_t bytes, uint64_t *bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                     smem_u32(to)),
                 "l"(from), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ void tensor_copy_2d(void *to, const CUtensorMap *map, int x, int y, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::
            "r"(smem_u32(to)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void tmem_alloc(uint32_t *slot, uint32_t cols) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t cols) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(cols) : "memory");
}
// D (+)= A (tensor memory) * B^T (shared memory), issued from a converged warp by its elected lane.
__device__ __forceinline__ void umma_f16_ts_warp(uint32_t d, uint32_t a, uint64_t b_desc, uint32_t idesc,
                                                 uint32_t accumulate) {
    asm volatile(
        "{\n"
        " .reg .pred e, p;\n"
        " elect.sync _|e, 0xffffffff;\n"
        " setp.ne.b32 p, %4, 0;\n"
        " @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
        "}\n" ::"r"(d),
        "r"(a), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void umma_commit_warp(uint64_t *bar) {
    asm volatile(
        "{\n"
        " .reg .pred e;\n"
        " elect.sync _|e, 0xffffffff;\n"
        " @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n"
        "}\n" ::"r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void tmem_st_32x32b_x32(uint32_t at, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0],"
        " {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16,"
        " %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// kind::f16: fp32 accumulator, fp16 A and B, M = 128.
__device__ __forceinline__ uint32_t idesc_f16(int n) {
    return (1u << 4) | (static_cast<uint32_t>(n >> 3) << 17) | (128u >> 4 << 24);
}

// Bounded waits for the phase of parity `parity`, by the SM's clock: give up, and raise *abort, after abort[1] times 1024
// cycles or once another role has raised it.  (The limit is read where it is needed: as a number of 64 bits from the
// parameters it cost the loops of 64 rows registers, 152064 x 3584 in groups of 32 7 us of 170.)
__device__ __forceinline__ bool try_wait_long(uint32_t bar, uint32_t parity) {  // sleeps up to 2 us
    uint32_t ok;
    asm volatile(
        "{\n"
        " .reg .pred p;\n"
        " mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n"
        " selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(2000)
        : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool wait_phase(uint64_t *bar, uint32_t parity, volatile int *abort) {
    const uint32_t a = smem_u32(bar);
    if (try_wait_long(a, parity)) return true;
    const long long t0 = clock64();
    while (!try_wait_long(a, parity)) {
        if (*abort) return false;
        if (clock64() - t0 > static_cast<long long>(abort[1]) << 10) {
            *abort = 1;
            return false;
        }
    }
    return true;
}
// By a converged warp, which stays so.
__device__ __forceinline__ bool wait_phase_warp(uint64_t *bar, uint32_t parity, volatile int *abort) {
    return __all_sync(0xffffffffu, wait_phase(bar, parity, abort));
}
// On the way out: whatever the abort flag says.
__device__ __forceinline__ void wait_drained(uint64_t *bar, uint32_t parity, volatile int *abort) {
    const uint32_t a = smem_u32(bar);
    const long long t0 = clock64();
    while (!mbar_try_wait(a, parity) && clock64() - t0 < static_cast<long long>(abort[1]) << 10) {
    }
}

// ------------------------------------------------------------------------------ the product

// Copies in flight land before the memory goes.  Stages that only one of the two TMA warps has asked for lack an arrival;
// neither is more than `stages` of them ahead.
__device__ __noinline__ void drain_copies(uint64_t *full, int stages, const int *issued_of, volatile int *abort) {
    const int both = min(issued_of[0], issued_of[1]), any = max(issued_of[0], issued_of[1]);
    for (int i = both; i < any; ++i) mbar_arrive(&full[i % stages]);
    for (int i = max(0, any - stages); i < any; ++i) wait_drained(&full[i % stages], (i / stages) & 1, abort);
}

// A place in a ring of barriers.
struct Cursor {
    int at = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next(int n, int by = 1) {
        at += by;
        if (at >= n) {
            at -= n;
            phase ^= 1u;
        }
    }
};

constexpr int meta_group_bytes(bool zeros) { return zeros ? 128 : 64; }  // of a pair and group

// Scales (and zero points) of a warp's pairs on their way through shared memory: chunks of kMetaChunk groups,
// kMetaSlots - 1 of them ahead and on into the next unit.  Every lane calls it.
template <bool kZeros, int kPairs>
struct MetaRing {
    static constexpr int kGroupBytes = meta_group_bytes(kZeros), kPairBytes = kMetaChunk * kGroupBytes;
    static constexpr int kSlotBytes = kPairs * kPairBytes, kBytes = kMetaSlots * kSlotBytes;
    const uint8_t *meta;
    uint32_t ring;
    int pair, last, groups, end;  // the next chunk's first pair (others kWideHalf on), bounds
    int chunk = 0, slot_in = 0, slot_out = 0;
    __device__ MetaRing(const QuantParams &q, uint32_t ring_at, int first, int unit_end)
        : meta(static_cast<const uint8_t *>(q.meta)), ring(ring_at), pair(first), last(q.pairs - 1), groups(q.groups),
          end(unit_end) {
        for (int i = 0; i < kMetaSlots - 1; ++i) fetch();
    }
    __device__ __forceinline__ void fetch() {
        if (pair < end) {
            const int count = min(kMetaChunk, groups - chunk * kMetaChunk);
            const uint32_t to = ring + slot_in * kSlotBytes;
#pragma unroll
            for (int h = 0; h < kPairs; ++h) {
                const int at = (threadIdx.x & 31) * 16;
                const long long from = static_cast<long long>(min(pair + h * kWideHalf, last)) * groups + chunk * kMetaChunk;
                if (at < count * kGroupBytes) copy_async(to + h * kPairBytes + at, meta + from * kGroupBytes + at);
            }
            if (++chunk * kMetaChunk >= groups) {
                chunk = 0;
                pair += kWideUnit;
            }
            slot_in = (slot_in + 1) % kMetaSlots;
        }
        copy_commit();
    }
    __device__ __forceinline__ uint32_t next() {  // where the next chunk is
        copy_wait<kMetaSlots - 2>();
        __syncwarp();  // every lane's copies are seen, and every lane is done with the chunk before
        fetch();
        const uint32_t at = ring + slot_out * kSlotBytes;
        slot_out = (slot_out + 1) % kMetaSlots;
        return at;
    }
};
static_assert(kMetaChunk * meta_group_bytes(true) <= 512, "a chunk of a pair is one copy a lane");

// Shared memory for the epilogue's scales and, where zero points are stored, the weights' warps'.
constexpr int meta_bytes(bool zeros) {
    return zeros ? 8 * MetaRing<true, 1>::kBytes + 4 * MetaRing<true, 2>::kBytes : 8 * MetaRing<false, 1>::kBytes;
}

template <int kGroup, bool kZeros, bool kF16, int n>
__global__ void __launch_bounds__(kWideThreads, 1)
    k_quant_wide(const __grid_constant__ CUtensorMap map4, const __grid_constant__ CUtensorMap map2, const WideParams p) {
    extern __shared__ uint8_t smem_raw[];
    // done: the stage's MMAs are complete (its memory, its A operand and, with groups of 128 columns, the accumulator)
    __shared__ uint64_t full[kWideMaxStages], done[kWideMaxStages], a_full[kWideSlots], acc_full[2], acc_empty[2],
        drained;
    __shared__ uint32_t tmem_slot;
    __shared__ float factor[kWideMaxRows];
    __shared__ int issued_of[2];  // stages that the TMA warps have asked for: codes; activations
    __shared__ int give_up[2];  // whether a wait has run out, and its limit in 1024 cycles
    volatile int *abort = give_up;
    uint8_t *smem = smem_raw + (1024 - (smem_u32(smem_raw) & 1023)) % 1024;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int stage_bytes = n * 256 + kWideCodeBytes;
    const int steps = p.q.blocks / 2;  // stages of a unit
    const uint32_t meta_ring = smem_u32(smem) + p.stages * stage_bytes;
    const int pair0 = static_cast<int>(static_cast<long long>(p.q.pairs) * blockIdx.y / gridDim.y);
    const int pair1 = static_cast<int>(static_cast<long long>(p.q.pairs) * (blockIdx.y + 1) / gridDim.y);

    pdl_trigger();
    if (warp == kWideMma) tmem_alloc(&tmem_slot, 512);
    if (threadIdx.x == 0) {
        give_up[0] = 0;
        issued_of[0] = issued_of[1] = (pair1 - pair0 + kWideUnit - 1) / kWideUnit * steps;  // unless a wait runs out
        give_up[1] = static_cast<int>(p.q.wait_cycles >> 10);
        for (int i = 0; i < p.stages; ++i) {
            mbar_init(&full[i], 2);
            mbar_init(&done[i], 1);
        }
        for (int i = 0; i < kWideSlots; ++i) mbar_init(&a_full[i], 4);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&acc_full[i], 1);
            mbar_init(&acc_empty[i], 8);
        }
        mbar_init(&drained, 1);
        fence_mbar_init();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;

    if (warp == kWideTmaCodes || warp == kWideTmaRows) {
        // ---- TMA, a warp for the codes and one for the activations (a copy takes its thread some 120 cycles)
        if (lane == 0) {
            const bool codes = warp == kWideTmaCodes;
            const uint8_t *x = p.x + static_cast<long long>(blockIdx.x) * p.q.blocks * n * 128;
            if (!codes) {  // codes were laid out long ago: theirs need not wait
                pdl_wait();
                proxy_fence_global();
            }
            Cursor s;
            int issued = 0;
            bool ok = codes || !p.q.stall;
            for (int unit = pair0; unit < pair1 && ok; unit += kWideUnit) {
                const int pairs = min(pair1 - unit, kWideUnit);
                const int rest = pairs % 4;  // copies of four pairs; of two where no more are left
                const int bytes = (pairs - rest + (rest > 2 ? 4 : rest ? 2 : 0)) * kWidePairBytes;
                for (int kb = 0; kb < steps; ++kb) {
                    if (issued == p.stages) pdl_wait();
                    if (issued >= p.stages) ok = wait_phase(&done[s.at], s.phase ^ 1u, abort);
                    if (!ok) break;
                    uint8_t *to = smem + s.at * stage_bytes;
                    if (codes) {
                        mbar_arrive_expect_tx(&full[s.at], bytes);
                        for (int t = 0; t < pairs; t += 4)
                            tensor_copy_2d(to + n * 256 + t * kWidePairBytes, pairs - t > 2 ? &map4 : &map2, kb * 256, unit + t,
                                           &full[s.at]);
                    } else {
                        mbar_arrive_expect_tx(&full[s.at], n * 256);
                        bulk_copy(to, x + static_cast<long long>(kb) * n * 256, n * 256, &full[s.at]);
                    }
                    ++issued;
                    s.next(p.stages);
                }
            }
            if (!ok) issued_of[codes ? 0 : 1] = issued;
        }
        __syncwarp();
    } else if (warp == kWideMma) {
        // ---- MMA issue (every branch is warp-uniform)
        // A stage is straight-line code: what it waits for, sixteen MMAs (or eight), commits.
        constexpr int kGroups = 128 / kGroup, kSteps = 8 / kGroups;  // groups of a stage, 16-column steps of a group
        const uint32_t idesc = idesc_f16(n), base = __shfl_sync(0xffffffffu, tmem, 0);
        const uint64_t b_base = smem_desc_sw128(smem_u32(smem));
        Cursor s, a;
        uint32_t acc_phase = 1;  // of the two accumulators: they are used in turn
        int acc_next = 0;
        bool ok = true;
        pdl_wait();
        for (int unit = pair0; unit < pair1 && ok; unit += kWideUnit) {
            const bool two = pair1 - unit > kWideHalf;
            for (int kb = 0; kb < steps; ++kb) {
                // (the warps that arrive here have seen the whole stage land, activations too)
                ok = wait_phase_warp(&a_full[a.at], a.phase, abort);
                if (!ok) break;
                const uint64_t b = b_base + static_cast<uint32_t>(s.at * stage_bytes) / 16;
                const uint32_t a_at = base + kWideAccCols + a.at * 128;
#pragma unroll 1
                for (int grp = 0; grp < kGroups; ++grp) {
                    ok = ok && wait_phase_warp(&acc_empty[acc_next], acc_phase, abort);
                    if (ok) {
                        tc_fence_after_sync();
                        const uint32_t d = base + acc_next * 128;
#pragma unroll
                        for (int j = 0; j < kSteps; ++j) {
                            const int k = grp * kSteps + j;  // columns 16 k .. of the stage
                            umma_f16_ts_warp(d, a_at + k * 8, b + (k / 4) * (n * 8) + (k % 4) * 2, idesc, j != 0);
                        }
                        if (two)
#pragma unroll
                            for (int j = 0; j < kSteps; ++j) {
                                const int k = grp * kSteps + j;
                                umma_f16_ts_warp(d + 64, a_at + 64 + k * 8, b + (k / 4) * (n * 8) + (k % 4) * 2, idesc, j != 0);
                            }
                        if (kGroup != 128) umma_commit_warp(&acc_full[acc_next]);
                        acc_phase ^= acc_next;
                        acc_next ^= 1;
                    }
                }
                if (!ok) break;
                umma_commit_warp(&done[s.at]);
                s.next(p.stages);
                a.next(kWideSlots);
            }
        }
        // everything issued has to be done before TMEM is given back
        umma_commit_warp(&drained);
        wait_drained(&drained, 0, abort);
        __syncwarp();
    } else if (warp < 4) {
        // ---- weights to TMEM: a thread a matrix row of each half
        const int row = warp * 32 + lane;
        // words 2 hi and 2 hi + 1 of the vectors of lanes (t, g), t = 0..3
        const uint32_t place = smem_u32(smem) + n * 256 + (row >> 5) * kWidePairBytes + ((row >> 4) & 1) * 512 +
                               (row & 7) * 16 + ((row >> 3) & 1) * 8;
        const uint32_t to = tmem + (static_cast<uint32_t>(warp * 32) << 16) + kWideAccCols;
        Cursor s, a, before;  // before: the stage that had the A operand last, two ago
        typedef MetaRing<kZeros, 2> Ring;  // zero points of both halves' rows
        constexpr int kGroups = 128 / kGroup;  // of a stage
        const uint32_t entry = ((lane >> 4) * 16 + (row & 7) * 2 + ((row >> 3) & 1)) * (Ring::kGroupBytes / 32);
        Ring ring(p.q, meta_ring + 8 * MetaRing<kZeros, 1>::kBytes + warp * Ring::kBytes, pair0 + warp, kZeros ? pair1 : 0);
        uint32_t zeros_at = 0;
        int i = 0;
        bool ok = true;
        pdl_wait();
        for (int unit = pair0; unit < pair1 && ok; unit += kWideUnit) {
            const bool two = pair1 - unit > kWideHalf;
            for (int kb = 0; kb < steps; ++kb, ++i) {
                ok = wait_phase_warp(&full[s.at], s.phase, abort);
                if (!ok) break;
                const uint32_t from = place + s.at * stage_bytes;
                uint2 w[16];
#pragma unroll
                for (int t = 0; t < 8; ++t) w[t] = lds64(from + (t >> 2) * 1024 + (t & 3) * 128);
                if (two)
#pragma unroll
                    for (int t = 0; t < 8; ++t)
                        w[8 + t] = lds64(from + kWideHalf * kWidePairBytes + (t >> 2) * 1024 + (t & 3) * 128);
                uint32_t z[2][kGroups];
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {  // (here, their way from shared memory is hidden by the wait below: 1 us)
                    z[0][g] = z[1][g] = kMinusZeroDefault;
                    if (kZeros) {
                        const int in_chunk = (kb * kGroups + g) % kMetaChunk;
                        if (in_chunk == 0) zeros_at = ring.next() + entry;
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            z[h][g] = __byte_perm(lds32(zeros_at + h * Ring::kPairBytes + in_chunk * Ring::kGroupBytes), 0, 0x3232);
                    }
                }
                if (i >= kWideSlots) {
                    ok = wait_phase_warp(&done[before.at], before.phase, abort);
                    if (!ok) break;
                    before.next(p.stages);
                    tc_fence_after_sync();
                }
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    if (b < 2 || two) {
                        uint32_t v[32];
#pragma unroll
                        for (int t = 0; t < 4; ++t)
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                // columns 64 (b % 2) of the stage on, and 32 further
                                v[t * 4 + k] = weight_pair(w[4 * b + t].x, k, z[b / 2][b % 2 * 64 / kGroup]);
                                v[16 + t * 4 + k] = weight_pair(w[4 * b + t].y, k, z[b / 2][(b % 2 * 64 + 32) / kGroup]);
                            }
                        tmem_st_32x32b_x32(to + a.at * 128 + b * 32, v);
                    }
                }
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&a_full[a.at]);
                s.next(p.stages);
                a.next(kWideSlots);
            }
        }
        copy_wait<0>();  // (after a wait that ran out, chunks may be on their way)
    } else {
        // ---- epilogue: a thread a matrix row, all activations
        constexpr int cols = n;
        const int half = (warp >> 2) - 1, row = (warp & 3) * 32 + lane;
        const uint32_t from = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + half * 64;
        typedef MetaRing<kZeros, 1> Ring;
        const uint32_t entry = ((lane >> 4) * 16 + (row & 7) * 2 + ((row >> 3) & 1)) * (Ring::kGroupBytes / 32);
        const int groups = p.q.groups;
        // (a half that has no rows in the last unit follows it all the same, on the last pair's scales)
        Ring ring(p.q, meta_ring + (warp - 4) * Ring::kBytes, pair0 + half * kWideHalf + (warp & 3),
                  pair0 + (pair1 - pair0 + kWideUnit - 1) / kWideUnit * kWideUnit);
        pdl_wait();  // the factors are the predecessor's
        if (threadIdx.x - 128 < n) factor[threadIdx.x - 128] = p.factor[static_cast<long long>(blockIdx.x) * n + threadIdx.x - 128];
        asm volatile("bar.sync 1, 256;" ::: "memory");
        Cursor acc, s;
        bool ok = true;
        for (int unit = pair0; unit < pair1; unit += kWideUnit) {
            f32x2 run[cols / 2];
#pragma unroll
            for (int i = 0; i < cols / 2; ++i) run[i] = pack2(0.f, 0.f);
            for (int first = 0; first < groups && ok; first += kMetaChunk) {
                uint32_t meta_at = ring.next() + entry;
                const int count = min(kMetaChunk, groups - first);
                for (int j = 0; j < count; ++j) {
                    const float scale = scale_low<kF16>(kZeros ? lds32(meta_at) : lds16(meta_at));
                    const f32x2 s2 = pack2(scale, scale);
                    ok = kGroup == 128 ? wait_phase_warp(&done[s.at], s.phase, abort)
                                       : wait_phase_warp(&acc_full[acc.at], acc.phase, abort);
                    if (!ok) break;
                    tc_fence_after_sync();
#pragma unroll
                    for (int c = 0; c < cols / 32; ++c) {
                        float v[32];
                        tmem_ld_32x32b_x32(from + acc.at * 128 + c * 32, v);
                        if (c == cols / 32 - 1) {  // all of the accumulator is read
                            tc_fence_before_sync();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&acc_empty[acc.at]);
                        }
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            run[c * 16 + i] = fma2(s2, pack2(v[2 * i], v[2 * i + 1]), run[c * 16 + i]);
                    }
                    meta_at += Ring::kGroupBytes;
                    acc.next(2);
                    if (kGroup == 128) s.next(p.stages);
                }
            }
            const int pair = unit + half * kWideHalf + (row >> 5), v = pair * kQuantPairRows + lane;
            if (pair < pair1 && v < p.q.V) {
                int pass;  // (read here: kept in a register through the loop above, it cost 20 rows 3 us)
                asm volatile("mov.u32 %0, %%ctaid.x;" : "=r"(pass));
                const int row0 = pass * p.q.per, rows = min(p.q.per, p.q.rows - row0);
#pragma unroll
                for (int i = 0; i < cols / 2; ++i) {
                    float y[2];
                    unpack2(run[i], y[0], y[1]);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int r = 2 * i + k;
                        if (r < rows)
                            store_out(p.q.out, p.q.out_type, (row0 + r) * p.q.out_stride + v,
                                      ok ? y[k] * kWeightFactor * factor[r] : __int_as_float(0x7FFFFFFF));
                    }
                }
            }
        }
        copy_wait<0>();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (*abort && threadIdx.x == 0) drain_copies(full, p.stages, issued_of, abort);
    if (warp == kWideMma) tmem_free(tmem, 512);
}

template <int kGroup, bool kZeros, bool kF16, int n>
cudaError_t launch_wide(const CUtensorMap *maps, WideParams p, int passes, int num_sms, cudaStream_t s) {
    void (*kernel)(const CUtensorMap, const CUtensorMap, const WideParams) = k_quant_wide<kGroup, kZeros, kF16, n>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kWideSmem);
    if (e != cudaSuccess) return e;
    constexpr int stage = n * 256 + kWideCodeBytes, ring = meta_bytes(kZeros);
    constexpr int stages = (kWideSmem - 1024 - ring) / stage;
    static_assert(stages >= kWideSlots, "an A operand's last stage is still in the ring when it is waited for");
    p.stages = std::min(kWideMaxStages, stages);
    return launch_pdl(kernel, dim3(passes, std::min(num_sms, p.q.pairs)), dim3(kWideThreads),
                      static_cast<size_t>(p.stages) * stage + ring + 1024, s, maps[0], maps[1], p);
}

template <int kGroup, int n>
cudaError_t launch_wide_scales(const CUtensorMap *maps, const WideParams &p, bool zeros, bool f16, int passes,
                               int num_sms, cudaStream_t s) {
    if (f16)
        return zeros ? launch_wide<kGroup, true, true, n>(maps, p, passes, num_sms, s) : launch_wide<kGroup, false, true, n>(maps, p, passes, num_sms, s);
    return zeros ? launch_wide<kGroup, true, false, n>(maps, p, passes, num_sms, s) : launch_wide<kGroup, false, false, n>(maps, p, passes, num_sms, s);
}

template <int n>
cudaError_t launch_wide_group(const CUtensorMap *maps, const WideParams &p, int group, bool zeros, bool f16, int passes,
                              int num_sms, cudaStream_t s) {
    return group == 32   ? launch_wide_scales<32, n>(maps, p, zeros, f16, passes, num_sms, s)
           : group == 64 ? launch_wide_scales<64, n>(maps, p, zeros, f16, passes, num_sms, s)
                         : launch_wide_scales<128, n>(maps, p, zeros, f16, passes, num_sms, s);
}

cudaError_t launch_x(const QuantParams &p, int n, int passes, uint8_t *xs, float *factor, cudaStream_t s) {
    return p.x_type == RPD_TYPE_BF16
               ? launch_pdl(k_quant_wide_x<__nv_bfloat16>, dim3(passes * n), dim3(256), 0, s, p, n, xs, factor)
               : launch_pdl(k_quant_wide_x<__half>, dim3(passes * n), dim3(256), 0, s, p, n, xs, factor);
}

// Passes over the codes, their rows and what these are padded to: 64, or 32 where that makes no more passes or they all
// run side by side.  (126464 x 4096: 33 rows, padded to 64, take 109 us, 32 rows as 32 take 98.7; 1022 x 1254: 80
// rows 12.6, as two passes of 64 in turn 26.6.)
struct WidePasses {
    int passes, per_pass, n;
    WidePasses(int rows, int pairs, int num_sms) {
        passes = rows / 32 + (rows % 32 != 0);
        n = static_cast<long long>(passes) * pairs <= num_sms ? 32 : kWideMaxRows;
        if (n == kWideMaxRows) passes = rows / n + (rows % n != 0);
        per_pass = rows / passes + (rows % passes != 0);
        if (per_pass <= 32) n = 32;
    }
};

}  // namespace

long long quant_wide_workspace(int rows, int blocks, int pairs, int num_sms) {
    const WidePasses w(rows, pairs, num_sms);
    return static_cast<long long>(w.passes) * w.n * (blocks * 128ll + 4ll);
}

cudaError_t quant_wide(const CUtensorMap *maps, const QuantParams &p, int group, bool zeros, bool f16, int num_sms,
                       void *workspace, cudaStream_t s) {
    const WidePasses w(p.rows, p.pairs, num_sms);
    uint8_t *xs = static_cast<uint8_t *>(workspace);
    WideParams q{};
    q.q = p;
    q.q.per = w.per_pass;
    q.x = xs;
    float *factor = reinterpret_cast<float *>(xs + static_cast<size_t>(w.passes) * w.n * p.blocks * 128);
    q.factor = factor;
    const cudaError_t e = launch_x(q.q, w.n, w.passes, xs, factor, s);
    if (e != cudaSuccess) return e;
    return w.n == 32 ? launch_wide_group<32>(maps, q, group, zeros, f16, w.passes, num_sms, s)
                     : launch_wide_group<64>(maps, q, group, zeros, f16, w.passes, num_sms, s);
}

}  // namespace rpd
