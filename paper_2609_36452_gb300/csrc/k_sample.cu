// k_sample.cu - a token from every row of logits by one given random number, under limits: top-k, top-p, min-p.
//
// Tokens are ordered by their logits (of equal ones the lower index first); w = e^((z - max) / T).  Top-k keeps the first
// k, top-p a token while the weights before it are less than p times the sum (of those top-k keeps), min-p
// those with w >= min_p.  The token is the first at which the running sum of kept weights exceeds u times their sum.
//
// Precision.  Borders of a running sum over 10^5 tokens lie some 10^-6 of it apart, and closer: sums that carry fp32's
// errors find another token in one row of a thousand.  Weights are therefore integers: 2^y by a table of 512 values and
// a cubic, right to 2^-31 relative and without bias, in units of 2^-54 (and less) of the largest; the few that
// hold more than 2^-10 of the sum are made in 64 bits.  Sums of integers do not depend on their order.
//
// A cluster of up to eight CTAs has a row, in shared memory where it fits there: the row is read from HBM once, whatever
// its limits ask for.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "logits_row.cuh"
#include "op_host.h"
#include "ptx.cuh"

namespace rpd {
namespace {

constexpr int kSampleThreads = 512;
constexpr int kSampleWarps = kSampleThreads / 32;
constexpr int kSampleMaxCluster = 8;
constexpr int kSampleTable = 512;
constexpr float kLowest = -3.402823466e38f;

struct SampleParams {
    rpd_sample_args a;
    int words;       // 32-bit words of a row of masks
    int slice;       // tokens of a CTA, a multiple of 32
    int sum_bits;    // units of a row's sum of weights: 2^-sum_bits of the largest
};

// 2^(i / 512) in units of 2^-31.
struct SampleTable {
    uint32_t v[kSampleTable];
    constexpr SampleTable() : v() {
        for (int i = 0; i < kSampleTable; ++i) {
            const double x = i * (0.6931471805599453 / kSampleTable);
            double term = 1, sum = 1;
            for (int n = 1; n < 24; ++n) {
                term *= x / n;
                sum += term;
            }
            v[i] = static_cast<uint32_t>(sum * 2147483648.0 + 0.5);
        }
    }
};
__device__ const SampleTable g_sample_table;

__device__ __forceinline__ uint32_t order_key(float z) {  // of floats, -0 as 0
    const uint32_t b = __float_as_uint(z + 0.f);
    return b ^ (static_cast<uint32_t>(static_cast<int>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// ------------------------------------------------------------------------------ a CTA's part of a row

__device__ __forceinline__ uint32_t no_logit_pair(float) { return 0xFF800000u; }
__device__ __forceinline__ uint32_t no_logit_pair(__nv_bfloat16) { return 0xFF80FF80u; }
__device__ __forceinline__ uint32_t no_logit_pair(__half) { return 0xFC00FC00u; }

// A vector with the tokens that are not allowed taken out.
template <typename T>
__device__ __forceinline__ uint4 keep_allowed(const uint4 &v, uint32_t bits) {
    const uint32_t none = no_logit_pair(T());
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t keep;
        if (sizeof(T) == 4)
            keep = (bits >> i) & 1u ? 0xFFFFFFFFu : 0u;
        else
            keep = ((bits >> (2 * i)) & 1u ? 0xFFFFu : 0u) | ((bits >> (2 * i + 1)) & 1u ? 0xFFFF0000u : 0u);
        w[i] = (w[i] & keep) | (none & ~keep);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Tokens [v0, v0 + row.V) of a row.  Resident: a copy in shared memory, at the same distance from a 16-byte boundary, in which
// tokens that are not allowed are -infinity.
template <typename T, bool kResident>
struct Slice {
    static constexpr int N = Row<T>::kVec;
    Row<T> row;
    int v0;
    const uint32_t *mask;
    int words;
    uint8_t *buf;
    __device__ Slice(const SampleParams &p, long long r, int rank, uint8_t *buffer)
        : row(p.a.logits, r * p.a.row_stride + min(p.a.V, rank * p.slice), max(0, min(p.slice, p.a.V - rank * p.slice))),
          v0(min(p.a.V, rank * p.slice)), mask(p.a.allowed ? p.a.allowed + r * p.words : nullptr), words(p.words),
          buf(buffer + (reinterpret_cast<uintptr_t>(row.p) & 15)) {}
    __device__ __forceinline__ uint4 global_vec(int i) const {
        return reinterpret_cast<const uint4 *>(row.p + row.peel)[i];
    }
    __device__ __forceinline__ uint4 allowed_vec(uint4 raw, int i) const {
        return mask ? keep_allowed<T>(raw, allowed_bits(mask, v0 + row.peel + i * N, words)) : raw;
    }
    __device__ __forceinline__ float global_at(int j) const {
        const int v = v0 + j;
        return mask && !((mask[v >> 5] >> (v & 31)) & 1u) ? kNoLogit : value(row.p[j]);
    }
    __device__ __forceinline__ float at(int j) const {
        return kResident ? value(reinterpret_cast<const T *>(buf)[j]) : global_at(j);
    }
    __device__ __forceinline__ int loose() const { return row.V - row.vecs * N; }  // tokens outside vectors
    __device__ __forceinline__ int loose_at(int i) const { return i < row.peel ? i : i + row.vecs * N; }
    // f(logit, token) for every token; threads interleave.
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        for (int i = threadIdx.x; i < row.vecs; i += kSampleThreads) {
            const uint4 raw = kResident ? *reinterpret_cast<const uint4 *>(buf + (row.peel + i * N) * sizeof(T))
                                        : allowed_vec(global_vec(i), i);
            float z[N];
            unpack(raw, z, T());
#pragma unroll
            for (int k = 0; k < N; ++k) f(z[k], v0 + row.peel + i * N + k);
        }
        if (static_cast<int>(threadIdx.x) < loose()) {
            const int j = loose_at(threadIdx.x);
            f(at(j), v0 + j);
        }
    }
};
static_assert(kSampleThreads >= 2 * 8, "tokens outside vectors are a thread's each");

// Largest and smallest logit of the slice, and whether one is NaN or +infinity.  A resident slice is copied on the way.
struct SampleRange {
    float top = kNoLogit, low = -kNoLogit;
    bool bad = false;
    __device__ __forceinline__ void add(float z) {
        bad |= !(z < -kNoLogit);
        top = fmaxf(top, z);
        low = fminf(low, z < kLowest ? -kNoLogit : z);
    }
};
template <typename T, bool kResident>
__device__ __forceinline__ SampleRange load_slice(const Slice<T, kResident> &s) {
    constexpr int N = Row<T>::kVec, kUnroll = 4;
    SampleRange r;
    for (int i = threadIdx.x; i < s.row.vecs; i += kSampleThreads * kUnroll) {
        uint4 raw[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (i + u * kSampleThreads < s.row.vecs) raw[u] = s.global_vec(i + u * kSampleThreads);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int at = i + u * kSampleThreads;
            if (at < s.row.vecs) {
                raw[u] = s.allowed_vec(raw[u], at);
                if (kResident) *reinterpret_cast<uint4 *>(s.buf + (s.row.peel + at * N) * sizeof(T)) = raw[u];
                float z[N];
                unpack(raw[u], z, T());
#pragma unroll
                for (int k = 0; k < N; ++k) r.add(z[k]);
            }
        }
    }
    if (static_cast<int>(threadIdx.x) < s.loose()) {
        const int j = s.loose_at(threadIdx.x);
        const float z = s.global_at(j);
        if (kResident) {
            const uint32_t none = no_logit_pair(T());
            T *to = reinterpret_cast<T *>(s.buf) + j;
            *to = z == kNoLogit ? *reinterpret_cast<const T *>(&none) : s.row.p[j];
        }
        r.add(z);
    }
    return r;
}

// ------------------------------------------------------------------------------ weights

// 2^((z - top) c) in units of 2^-bits, c = log2 e / T as the sum of two floats.  y = (z - A) c is a product and its
// error; k is y to the nearest 1/512, the rest |r| <= 2^-9 (after that of the largest logit is taken off), and 2^y =
// 2^(whole part of k) table[k mod 512] (1 + r ln 2 + ...).  A = 0, or the largest logit where that times c leaves
// the range of k: logits that count are then within a factor of two of it, and the difference is exact.
struct SampleWeights {
    float A, c_hi, c_lo, rest_top, floor, big;
    int k_top;  // as the bits of the shifted product
    float c;
    double top, inverse_T;
    static constexpr float kShift = 1.5f * (1 << 14);  // floats near it have steps of 1/512
    // y = d c to the nearest 1 / 512 (its bits), and the rest.  (Every operation rounds by itself: the largest logit's rest is
    // to be the same number wherever it is made.)
    __device__ __forceinline__ int split(float d, float &rest) const {
        const float y = __fmul_rn(d, c_hi), t = __fadd_rn(y, kShift);
        rest = __fadd_rn(__fsub_rn(y, __fsub_rn(t, kShift)), fmaf(d, c_lo, fmaf(d, c_hi, -y)));
        return __float_as_int(t);
    }
    __device__ void set(float top_logit, double T) {
        top = top_logit;
        inverse_T = 1.0 / T;
        const double c64 = 1.4426950408889634 / T;
        c_hi = c = static_cast<float>(c64);
        c_lo = static_cast<float>(c64 - c_hi);
        A = fabsf(top_logit) * c < 0x1p12f ? 0.f : top_logit;
        k_top = split(top_logit - A, rest_top);
        big = -kNoLogit;
    }
    // Logits at and below `floor` weigh nothing: under 2^-bits.
    __device__ void set_floor(int bits) { floor = fmaxf(kLowest, __double2float_rd(top - bits / static_cast<double>(c))); }
    // Of a sum of about `sum` times the largest weight, those that hold 2^-10 and more.
    __device__ void set_big(float sum) { big = static_cast<float>(top - (10.0 - log2f(sum)) / c); }
    __device__ __forceinline__ uint64_t of(float z, int bits, const uint32_t *table) const {
        float r;
        const int k = split(fmaxf(z, floor) - A, r) - k_top;
        r = __fsub_rn(r, rest_top);
        // r ln 2 + r^2 ln^2 2 / 2 + r^3 ln^3 2 / 6 in units of 2^-31, to the nearest
        float q = fmaf(r, 1.1919417e8f, 5.158825e8f);
        q = fmaf(r, q, 1.488522236e9f);
        q = fmaf(r, q, 12582912.f);
        const uint32_t one_q = static_cast<uint32_t>(__float_as_int(q)) + (0x80000000u - 0x4B400000u);
        const uint64_t m = static_cast<uint64_t>(table[k & (kSampleTable - 1)]) * one_q;  // 2^62 to 2^63
        return m >> (62 - bits - (k >> 9));
    }
    // With the big ones in 64 bits; 0 at the floor.
    __device__ __forceinline__ uint64_t exact_of(float z, int bits, const uint32_t *table) const {
        if (z >= big) return __double2ull_rn(exp((z - top) * inverse_T) * static_cast<double>(1ull << bits));
        return z > floor ? of(z, bits, table) : 0ull;
    }
};

// ------------------------------------------------------------------------------ shared memory

// A kept prefix of the order: logits above `key`, and those at it up to token `last`.
struct SampleCut {
    uint32_t key;
    int last;
    __device__ __forceinline__ bool keeps(uint32_t k, int v) const { return k > key || (k == key && v <= last); }
};

struct SampleShared {
    uint32_t table[kSampleTable];
    SampleWeights w;
    uint64_t mass[256];
    uint32_t count[256];
    float range[2][kSampleWarps];
    float top, low;            // the slice's, then the row's
    int bad;
    float sums[kSampleWarps];
    float sum;
    double sum64[kSampleWarps];
    int counts[kSampleWarps];
    // what the first CTA of the cluster has found
    uint64_t above;            // of the bins above the border's
    uint64_t bin_mass;
    int above_count, bin_count, bin;
    int tie;                   // the token of a tie that the border falls on
};

__device__ __forceinline__ double ld_cluster_f64(uint32_t a) {
    double v;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint64_t ld_cluster_u64(uint32_t a) {
    uint64_t v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
template <typename V>
__device__ __forceinline__ uint32_t peer(const V *p, int rank) { return mapa_shared(smem_u32(p), rank); }

// All threads of the row.
__device__ __forceinline__ void row_sync(int ranks) {
    if (ranks > 1)
        cluster_sync();
    else
        __syncthreads();
}

// ------------------------------------------------------------------------------ any border, in four passes

// What a border's place is told by: the first token at which the running count reaches `count`, or the running sum
// of weights reaches (strictly: exceeds) `mass`.
struct SampleTarget {
    bool by_count, strictly;
    int count;
    double mass;
};

// The border among the tokens that `within` keeps: eight bits of the logit's key a pass, by a histogram of counts and
// weights.  Every thread of the row calls it; count and mass become those up to and with the border's token.
template <typename S>
__device__ __noinline__ SampleCut find_border(const S &s, SampleShared &sm, int ranks, int rank, int bits, const SampleCut &within,
                                              const SampleTarget &t, int &count, double &mass, double &weight) {
    uint32_t prefix = 0;
    uint64_t above = 0;
    int above_count = 0, n = 0;
    uint64_t bin_mass = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = threadIdx.x; i < 256; i += kSampleThreads) {
            sm.mass[i] = 0;
            sm.count[i] = 0;
        }
        __syncthreads();
        int run = -1, run_count = 0;  // neighbours that fall into one bin are added at once
        uint64_t run_mass = 0;
        s.each([&](float z, int v) {
            const uint32_t key = order_key(z);
            if (!(z >= kLowest) || !within.keeps(key, v) || (shift < 24 && (key >> (shift + 8)) != prefix)) return;
            const int b = static_cast<int>(key >> shift) & 255;
            if (b != run) {
                if (run >= 0) {
                    atomicAdd(&sm.count[run], run_count);
                    atomicAdd(reinterpret_cast<unsigned long long *>(&sm.mass[run]), static_cast<unsigned long long>(run_mass));
                }
                run = b;
                run_count = 0;
                run_mass = 0;
            }
            ++run_count;
            run_mass += sm.w.exact_of(z, bits, sm.table);
        });
        if (run >= 0) {
            atomicAdd(&sm.count[run], run_count);
            atomicAdd(reinterpret_cast<unsigned long long *>(&sm.mass[run]), static_cast<unsigned long long>(run_mass));
        }
        row_sync(ranks);
        if (rank == 0) {
            if (threadIdx.x < 256) {
                uint64_t m = 0;
                uint32_t c = 0;
                for (int r = 0; r < ranks; ++r) {
                    m += ld_cluster_u64(peer(&sm.mass[threadIdx.x], r));
                    c += ld_cluster_u32(peer(&sm.count[threadIdx.x], r));
                }
                sm.mass[threadIdx.x] = m;
                sm.count[threadIdx.x] = c;
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                uint64_t m = above;
                int c = above_count, found = -1;
                for (int b = 255; b >= 0; --b) {
                    const int bc = static_cast<int>(sm.count[b]);
                    if (bc == 0) continue;
                    found = b;
                    sm.above = m;
                    sm.above_count = c;
                    m += sm.mass[b];
                    c += bc;
                    const double at = static_cast<double>(m);
                    if (t.by_count ? c >= t.count : t.strictly ? at > t.mass : at >= t.mass) break;
                }
                sm.bin = found;  // (the last one that is not empty where roundings let none reach it)
                sm.bin_count = static_cast<int>(sm.count[found]);
                sm.bin_mass = sm.mass[found];
            }
        }
        row_sync(ranks);
        above = ld_cluster_u64(peer(&sm.above, 0));
        bin_mass = ld_cluster_u64(peer(&sm.bin_mass, 0));
        above_count = static_cast<int>(ld_cluster_u32(peer(&sm.above_count, 0)));
        n = static_cast<int>(ld_cluster_u32(peer(&sm.bin_count, 0)));
        prefix = prefix << 8 | ld_cluster_u32(peer(&sm.bin, 0));
        row_sync(ranks);
    }
    // n tokens have the border's logit, and one weight
    weight = static_cast<double>(bin_mass) / n;
    int j = n;
    if (t.by_count) {
        j = min(n, t.count - above_count);
    } else if (weight > 0) {
        const double steps = (t.mass - static_cast<double>(above)) / weight;
        const double place = t.strictly ? floor(steps) + 1 : ceil(steps);
        j = place < 1 ? 1 : place < n ? static_cast<int>(place) : n;
    }
    count = above_count + j;
    mass = static_cast<double>(above) + j * weight;
    SampleCut cut{prefix, 0x7FFFFFFF};
    if (j < n || !t.by_count) {
        // the j-th of them by index: a thread counts neighbouring tokens
        const int per = (s.row.V + kSampleThreads - 1) / kSampleThreads, from = min(s.row.V, static_cast<int>(threadIdx.x) * per);
        const int to = min(s.row.V, from + per);
        int mine = 0;
        for (int i = from; i < to; ++i) mine += order_key(s.at(i)) == prefix && within.keeps(prefix, s.v0 + i);
        int before = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, before, o);
            if ((threadIdx.x & 31) >= o) before += up;
        }
        if ((threadIdx.x & 31) == 31) sm.counts[threadIdx.x >> 5] = before;
        __syncthreads();
        before -= mine;
        int all = 0;
        for (int w = 0; w < kSampleWarps; ++w) {
            if (w < static_cast<int>(threadIdx.x >> 5)) before += sm.counts[w];
            all += sm.counts[w];
        }
        if (threadIdx.x == 0) sm.bin_count = all;
        row_sync(ranks);
        for (int r = 0; r < rank; ++r) before += static_cast<int>(ld_cluster_u32(peer(&sm.bin_count, r)));
        if (before < j && before + mine >= j) {
            int seen = before;
            for (int i = from; i < to; ++i)
                if (order_key(s.at(i)) == prefix && within.keeps(prefix, s.v0 + i) && ++seen == j)
                    st_shared_cluster(peer(&sm.tie, 0), s.v0 + i);
        }
        row_sync(ranks);
        cut.last = static_cast<int>(ld_cluster_u32(peer(&sm.tie, 0)));
        row_sync(ranks);
    }
    return cut;
}

// Weights of the kept tokens and their number, in every thread.
template <typename S>
__device__ __noinline__ double kept_mass(const S &s, SampleShared &sm, int ranks, int bits, const SampleCut &cut, int &count) {
    uint64_t m = 0;
    int c = 0;
    s.each([&](float z, int v) {
        if (z >= kLowest && cut.keeps(order_key(z), v)) {
            m += sm.w.exact_of(z, bits, sm.table);
            ++c;
        }
    });
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        m += __shfl_xor_sync(0xffffffffu, m, o);
        c += __shfl_xor_sync(0xffffffffu, c, o);
    }
    if ((threadIdx.x & 31) == 0) {
        sm.mass[threadIdx.x >> 5] = m;
        sm.counts[threadIdx.x >> 5] = c;
    }
    row_sync(ranks);
    m = 0;
    c = 0;
    for (int r = 0; r < ranks; ++r)
        for (int w = 0; w < kSampleWarps; ++w) {
            m += ld_cluster_u64(peer(&sm.mass[w], r));
            c += static_cast<int>(ld_cluster_u32(peer(&sm.counts[w], r)));
        }
    row_sync(ranks);
    count = c;
    return static_cast<double>(m);
}

// ------------------------------------------------------------------------------ the kernel

__device__ __forceinline__ float clamp_temperature(float T) { return fminf(fmaxf(T, 1.45e-30f), 1.44e37f); }

template <typename T, bool kResident>
__global__ void __launch_bounds__(kSampleThreads) k_sample_limits(const SampleParams p) {
    extern __shared__ __align__(16) uint8_t buffer[];
    __shared__ SampleShared sm;
    const int ranks = static_cast<int>(cluster_nctarank()), rank = ranks > 1 ? static_cast<int>(cluster_ctarank()) : 0;
    const long long r = blockIdx.x / ranks;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_trigger();
    for (int i = threadIdx.x; i < kSampleTable; i += kSampleThreads) sm.table[i] = g_sample_table.v[i];
    pdl_wait();
    const Slice<T, kResident> s(p, r, rank, buffer);
    SampleRange range = load_slice(s);
    const float T_row = p.a.temperature ? p.a.temperature[r] : 1.f, u = p.a.uniform ? p.a.uniform[r] : 0.f;
    const float top_p = p.a.top_p ? p.a.top_p[r] : 1.f, min_p = p.a.min_p ? p.a.min_p[r] : 0.f;
    const int top_k = p.a.top_k ? p.a.top_k[r] : 0;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        range.top = fmaxf(range.top, __shfl_xor_sync(0xffffffffu, range.top, o));
        range.low = fminf(range.low, __shfl_xor_sync(0xffffffffu, range.low, o));
    }
    range.bad = __any_sync(0xffffffffu, range.bad);
    if (lane == 0) {
        sm.range[0][warp] = range.top;
        sm.range[1][warp] = range.bad ? kNoLogit : range.low;  // a smallest logit of -infinity says so
    }
    __syncthreads();
    float top = kNoLogit, low = -kNoLogit;
    for (int w = 0; w < kSampleWarps; ++w) {
        top = fmaxf(top, sm.range[0][w]);
        low = fminf(low, sm.range[1][w]);
    }
    if (ranks > 1) {
        if (threadIdx.x == 0) {
            sm.top = top;
            sm.low = low;
        }
        cluster_sync();
        for (int q = 0; q < ranks; ++q) {
            top = fmaxf(top, __uint_as_float(ld_cluster_u32(peer(&sm.top, q))));
            low = fminf(low, __uint_as_float(ld_cluster_u32(peer(&sm.low, q))));
        }
    }
    const bool ok = low != kNoLogit && top != kNoLogit && T_row >= 0.f && (T_row == 0.f || (p.a.uniform && u >= 0.f && u < 1.f)) &&
                    top_p == top_p && min_p <= 1.f;
    SampleCut all{0u, 0x7FFFFFFF}, cut = all, token{0u, -1};
    int kept = 0;
    double prob = 0;
    if (ok && T_row == 0.f) {
        // the largest logit, and of several the first
        cut = {order_key(top), 0x7FFFFFFF};
        if (threadIdx.x == 0) sm.tie = 0x7FFFFFFF;
        row_sync(ranks);
        s.each([&](float z, int v) {
            if (order_key(z) == cut.key) atomicMin(&sm.tie, v);
        });
        row_sync(ranks);
        for (int q = 0; q < ranks; ++q) cut.last = min(cut.last, static_cast<int>(ld_cluster_u32(peer(&sm.tie, q))));
        token = cut;
        kept = 1;
        prob = 1;
        row_sync(ranks);
    } else if (ok) {
        const int bits = p.sum_bits;
        const float T_used = clamp_temperature(T_row);
        if (threadIdx.x == 0) {
            sm.w.set(top, T_used);
            sm.w.set_floor(bits);
        }
        __syncthreads();
        float sum = 0.f;
        s.each([&](float z, int) { sum += ex2((z - top) * sm.w.c); });
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) sm.sums[warp] = sum;
        __syncthreads();
        if (threadIdx.x == 0) {
            sum = 0.f;
            for (int w = 0; w < kSampleWarps; ++w) sum += sm.sums[w];
            sm.sum = sum;
        }
        row_sync(ranks);
        if (threadIdx.x == 0) {
            sum = 0.f;
            for (int q = 0; q < ranks; ++q) sum += __uint_as_float(ld_cluster_u32(peer(&sm.sum, q)));
            sm.w.set_big(fmaxf(sum, 1.f));
        }
        row_sync(ranks);
        int n;
        double mass = kept_mass(s, sm, ranks, bits, all, n), weight;
        if (top_k > 0 && top_k < n) cut = find_border(s, sm, ranks, rank, bits, cut, {true, false, top_k, 0.0}, n, mass, weight);
        if (top_p < 1.f) cut = find_border(s, sm, ranks, rank, bits, cut, {false, false, 0, top_p * mass}, n, mass, weight);
        if (min_p > 0.f) {
            const float edge = __double2float_ru(top + T_used * log(static_cast<double>(min_p)));
            if (order_key(edge) > cut.key) {
                cut = {order_key(edge), 0x7FFFFFFF};
                mass = kept_mass(s, sm, ranks, bits, cut, n);
            }
        }
        kept = n;
        token = find_border(s, sm, ranks, rank, bits, cut, {false, true, 0, u * mass}, n, prob, weight);
        prob = weight / mass;
    }
    if (rank == 0 && threadIdx.x == 0) {
        p.a.out_token[r] = ok ? token.last : -1;
        p.a.out_status[r] = ok ? RPD_OK : RPD_ERR_INVALID_ARGUMENT;
        if (p.a.out_kept) p.a.out_kept[r] = kept;
        if (p.a.out_prob) p.a.out_prob[r] = static_cast<float>(prob);
    }
    if (p.a.out_allowed) {
        // 32 tokens a warp and word; a lane keeps one of 32 words, so that they are stored together
        uint32_t *out = reinterpret_cast<uint32_t *>(p.a.out_allowed) + r * p.words + s.v0 / 32;
        const int words = (s.row.V + 31) / 32;
        for (int w0 = warp * 32; w0 < words; w0 += kSampleThreads) {
            uint32_t mine = 0;
            for (int i = 0; i < 32; ++i) {
                const int j = (w0 + i) * 32 + lane;
                const float z = j < s.row.V ? s.at(j) : kNoLogit;
                const uint32_t word = __ballot_sync(0xffffffffu, ok && z >= kLowest && cut.keeps(order_key(z), s.v0 + j));
                if (i == lane) mine = word;
            }
            if (w0 + lane < words) out[w0 + lane] = mine;
        }
    }
    if (ranks > 1) cluster_sync();  // shared memory is read by the others until here
}

constexpr int kSampleSmem = 200 * 1024;  // of a slice that stays in shared memory

// CTAs of a row: up to eight, as long as all of them run at once and a CTA has some thousand tokens.
int sample_ranks(long long rows, int V, int num_sms) {
    int ranks = kSampleMaxCluster;
    while (ranks > 1 && (rows * ranks > 2 * num_sms || V < ranks * 2048)) ranks >>= 1;
    return ranks;
}

template <typename T>
cudaError_t launch_sample(SampleParams p, int num_sms, cudaStream_t s) {
    int ranks = sample_ranks(p.a.rows, p.a.V, num_sms);
    const auto slice_of = [&](int n) { return ((p.words + n - 1) / n) * 32; };
    while (ranks < kSampleMaxCluster && slice_of(ranks) * static_cast<long long>(sizeof(T)) > 64 * 1024) ranks *= 2;
    p.slice = slice_of(ranks);
    const long long bytes = p.slice * static_cast<long long>(sizeof(T)) + 32;
    const bool resident = bytes <= kSampleSmem;
    void (*kernel)(const SampleParams) = resident ? k_sample_limits<T, true> : k_sample_limits<T, false>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSampleSmem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.a.rows) * ranks);
    cfg.blockDim = dim3(kSampleThreads);
    cfg.dynamicSmemBytes = resident ? static_cast<size_t>(bytes) : 0;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ranks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

constexpr int kSampleMaxV = 1 << 24;
constexpr int kSampleMaxRows = 1 << 26;

}  // namespace
}  // namespace rpd

using namespace rpd;

extern "C" int rpd_sample(const rpd_sample_args *args, void *stream_ptr) {
    if (!args) return op_fail(RPD_ERR_INVALID_ARGUMENT, "null argument");
    const rpd_sample_args &a = *args;
    if (a.rows < 0 || a.V < 1) return op_fail(RPD_ERR_INVALID_ARGUMENT, "rows must be >= 0 and V >= 1");
    const int size = type_size(a.type);
    if (!size) return op_fail(RPD_ERR_INVALID_ARGUMENT, "logits must be bf16, fp16 or fp32");
    if (a.V > kSampleMaxV || a.rows > kSampleMaxRows)
        return op_fail(RPD_ERR_UNSUPPORTED, "V must be <= %d and rows <= %d", kSampleMaxV, kSampleMaxRows);
    if (a.rows == 0) return RPD_OK;
    if (!a.logits || !a.out_token || !a.out_status) return op_fail(RPD_ERR_INVALID_ARGUMENT, "null buffer");
    if (!a.uniform && !a.temperature)
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "uniform is needed unless every temperature is 0");
    if (a.row_stride < 0) return op_fail(RPD_ERR_INVALID_ARGUMENT, "row_stride must be >= 0");
    const void *words[] = {a.allowed, a.temperature, a.top_k, a.top_p, a.min_p, a.uniform,
                           a.out_token, a.out_status, a.out_kept, a.out_prob, a.out_allowed};
    bool aligned = aligned_to(a.logits, size);
    for (const void *w : words) aligned = aligned && aligned_to(w, 4);
    if (!aligned) return op_fail(RPD_ERR_INVALID_ARGUMENT, "buffers must be aligned to their elements");

    // the device that holds the logits runs the call, whichever is current
    cudaPointerAttributes at{};
    cudaError_t e = cudaPointerGetAttributes(&at, a.logits);
    if (e != cudaSuccess || (at.type != cudaMemoryTypeDevice && at.type != cudaMemoryTypeManaged)) {
        cudaGetLastError();
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "logits must be device memory");
    }
    DeviceGuard dg(at.device);
    if (dg.err != cudaSuccess) return op_cuda_fail(dg.err, "cudaSetDevice");
    if (const int rc = check_device(at.device)) return rc;
    for (const void *w : words)
        if (w && !pointer_usable(w, at.device, false))
            return op_fail(RPD_ERR_INVALID_ARGUMENT, "every buffer must be device memory on the device of the logits");
    int num_sms = 0;
    e = cudaDeviceGetAttribute(&num_sms, cudaDevAttrMultiProcessorCount, at.device);
    if (e != cudaSuccess) return op_cuda_fail(e, "device query");

    SampleParams p{};
    p.a = a;
    p.words = (a.V + 31) / 32;
    int bits = 0;
    while (1 << bits < a.V) ++bits;
    p.sum_bits = std::min(54, 62 - bits);
    cudaStream_t s = static_cast<cudaStream_t>(stream_ptr);
    e = a.type == RPD_TYPE_F32    ? launch_sample<float>(p, num_sms, s)
        : a.type == RPD_TYPE_BF16 ? launch_sample<__nv_bfloat16>(p, num_sms, s)
                                  : launch_sample<__half>(p, num_sms, s);
    return e == cudaSuccess ? RPD_OK : op_cuda_fail(e, "sampling launch");
}
