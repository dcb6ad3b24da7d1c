// k_sample.cu - a token from every row of logits by one given random number, under limits: top-k, top-p, min-p.
//
// Tokens are ordered by their logits (of equal ones the lower index first); w = e^((z - max) / T).  Top-k keeps the first
// k, top-p a token while the weights before it are less than p times the sum (of those top-k keeps), min-p
// those with w >= min_p.  The token is the first at which the running sum of kept weights exceeds u times their sum.
//
// Precision.  Borders of a running sum over 10^5 tokens lie some 10^-6 of it apart, and closer: sums that carry fp32's
// errors find another token in one row of a thousand.  Weights are therefore integers: 2^y by a table of 512 values and
// a cubic, right to 2^-31 relative and without bias, in units of 2^-54 (and more) of the largest; the few that
// hold more than 2^-10 of the sum, and those of a list that decides a row, are made in 64 bits.  Sums of integers do not depend on their order.
//
// A cluster of up to eight CTAs has a row.  One pass brings it from HBM; later ones read it from shared memory, or from L2
// where two slices do not fit an SM.  Most rows are decided by a list of their likeliest tokens (list_likely), others by a
// histogram and a second pass (list_borders), the rest in passes of eight bits (sample_slowly).
//
// What bounds it: not HBM (128 rows of 126464 bf16 logits under top-k, top-p, min-p and a mask, 34 MB, take 33.6 us, 5.1 by bytes; 528 rows
// of 152064 in fp32 under top-p, with the kept tokens' mask, 302 to 319 us, 49.6 by bytes), but some twenty phases with a barrier
// of the row between them, and for rows that need all three passes their arithmetic: 67 instructions a token, at half of the
// issue slots.  Four passes of a 64-bit histogram for every border, the first form, took 956 and 4982 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "logits_row.cuh"
#include "op_host.h"
#include "ptx.cuh"
#include "sample_bins.h"

namespace rpd {
namespace {

constexpr int kSampleThreads = 512;
constexpr int kSampleWarps = kSampleThreads / 32;
constexpr int kSampleMaxCluster = 8;
constexpr int kSampleResident = 1024;      // threads of an SM: 64 registers each
constexpr int kSampleSteps = kSampleMaxCluster * kSampleWarps / 32;  // in which a warp looks at what every warp of the row has left
constexpr int kSampleTable = 512;
constexpr int kSampleBins = 4096;          // of the first histogram
constexpr int kBinParts = 256;             // parts of a bin, of which the mean is kept
constexpr int kBinOctaves = 64;            // what the bins span at most: a bin is a 64th of an octave of weights, or less
constexpr float kBinError = 0x1p-14f;      // of a sum of bins' weights, taken at their tokens' mean places: at most 2^-16 for
                                           // the spread around the mean, 2^-15.5 for the parts and 2^-19 for the units
constexpr int kSampleList = 2048;          // tokens that are sorted
constexpr int kSampleBits = 54;            // sums are in units of 2^-54 of the largest weight, or of more where they would not fit
constexpr float kLowest = -3.402823466e38f;

struct SampleParams {
    rpd_sample_args a;
    int words;       // 32-bit words of a row of masks
    int slice;       // tokens of a CTA, a multiple of 32
    int list_at;     // in shared memory, where the histogram and then the lists are; behind them this CTA's bins of the row
    int upto_at;     // room for running sums of a list
    int bits_at;     // a slice's bits of the mask that goes out; 0 where these are too many
};

// 2^(i / 512) in units of 2^-31, and what is left of it in units of 2^-52 (signed).
struct SampleTable {
    uint32_t v[kSampleTable];
    int rest[kSampleTable];
};
constexpr SampleTable sample_table() {
    SampleTable t{};
    for (int i = 0; i < kSampleTable; ++i) {
        const double x = i * (0.6931471805599453 / kSampleTable);
        double term = 1, sum = 1;
        for (int n = 1; n < 24; ++n) {
            term *= x / n;
            sum += term;
        }
        t.v[i] = static_cast<uint32_t>(sum * 2147483648.0 + 0.5);
        t.rest[i] = static_cast<int>((sum - t.v[i] / 2147483648.0) * 4503599627370496.0);
    }
    return t;
}
__device__ const SampleTable g_sample_table = sample_table();

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

// Largest and smallest of a vector's numbers, pairwise for 16-bit types; the largest is NaN where one is.
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint32_t pair_max(uint32_t a, uint32_t b, __nv_bfloat16) {
    const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ uint32_t pair_max(uint32_t a, uint32_t b, __half) {
    const __half2 r = __hmax2_nan(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ uint32_t pair_max(uint32_t a, uint32_t b, float) {
    return __float_as_uint(max_nan(__uint_as_float(a), __uint_as_float(b)));
}
__device__ __forceinline__ uint32_t pair_min(uint32_t a, uint32_t b, __nv_bfloat16) {
    const __nv_bfloat162 r = __hmin2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ uint32_t pair_min(uint32_t a, uint32_t b, __half) {
    const __half2 r = __hmin2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ uint32_t pair_min(uint32_t a, uint32_t b, float) {
    return __float_as_uint(fminf(__uint_as_float(a), __uint_as_float(b)));
}
template <typename T>
__device__ __forceinline__ uint32_t vec_max(const uint4 &v) {
    return pair_max(pair_max(v.x, v.y, T()), pair_max(v.z, v.w, T()), T());
}
template <typename T>
__device__ __forceinline__ uint32_t vec_min(const uint4 &v) {
    return pair_min(pair_min(v.x, v.y, T()), pair_min(v.z, v.w, T()), T());
}
__device__ __forceinline__ float2 pair_values(uint32_t v, float) { return make_float2(__uint_as_float(v), __uint_as_float(v)); }
__device__ __forceinline__ float2 pair_values(uint32_t v, __nv_bfloat16) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}
__device__ __forceinline__ float2 pair_values(uint32_t v, __half) { return __half22float2(*reinterpret_cast<const __half2 *>(&v)); }

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
    // f(logits, first token) for every vector with a logit of `least` or more, and every token outside of vectors (then other
    // logits are -infinity).
    template <typename F>
    __device__ __forceinline__ void each_vec(float least, F f) const {
        constexpr int kAhead = kResident ? 1 : 4;  // vectors on their way from L2 meanwhile
        const int pieces = row.vecs + loose();
        uint4 raw[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const int i = threadIdx.x + a * kSampleThreads;
            if (!kResident && i < row.vecs) raw[a] = global_vec(i);
        }
#pragma unroll 1
        for (int i = threadIdx.x; i < pieces; i += kSampleThreads) {
            float z[N];
            int first = row.peel + i * N;
            uint4 now;
            if (kResident) {
                if (i < row.vecs) now = *reinterpret_cast<const uint4 *>(buf + first * sizeof(T));
            } else {
                if (i < row.vecs) now = allowed_vec(raw[0], i);
#pragma unroll
                for (int a = 0; a + 1 < kAhead; ++a) raw[a] = raw[a + 1];
                if (i + kAhead * kSampleThreads < row.vecs) raw[kAhead - 1] = global_vec(i + kAhead * kSampleThreads);
            }
            if (i < row.vecs) {
                const float2 most = pair_values(vec_max<T>(now), T());
                if (fmaxf(most.x, most.y) < least) continue;
                unpack(now, z, T());
            } else {
                first = loose_at(i - row.vecs);
                z[0] = at(first);
#pragma unroll
                for (int k = 1; k < N; ++k) z[k] = kNoLogit;
            }
            f(z, v0 + first);
        }
    }
    // f(logit, token) for every token; threads interleave.  (Eight bytes of a resident slice at a time: bodies of f for a whole
    // vector are more code than the instruction caches hold, and every loop here runs some thirty times.)
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        constexpr int n = kResident ? N / 2 : N;
        const int pieces = row.vecs * (N / n);
#pragma unroll 1
        for (int i = threadIdx.x; i < pieces; i += kSampleThreads) {
            const int first = row.peel + i * n;
            float z[N];
            if (kResident) {
                const uint2 raw = *reinterpret_cast<const uint2 *>(buf + first * sizeof(T));
                unpack(make_uint4(raw.x, raw.y, 0, 0), z, T());
            } else {
                unpack(allowed_vec(global_vec(i), i), z, T());
            }
#pragma unroll
            for (int k = 0; k < n; ++k) f(z[k], v0 + first + k);
        }
        const int rest = loose();
#pragma unroll 1
        for (int i = threadIdx.x; i < rest; i += kSampleThreads) {
            const int j = loose_at(i);
            f(at(j), v0 + j);
        }
    }
};
static_assert(kSampleThreads >= 2 * 8, "tokens outside vectors are a thread's each");

// Of a thread's part of a slice: the largest allowed logit, the smallest of any (-infinity if there is one: then the finite ones
// have to be counted), the number of tokens that are not allowed, and about the sum of the weights relative to the
// largest.  The sum is no number where an allowed logit is NaN or +infinity.
template <typename T>
struct SampleRange {
    uint32_t most, least;  // of pairs
    float top = kLowest, sum = 0.f;
    int barred = 0;
    __device__ SampleRange() : most(no_logit_pair(T())), least(no_logit_pair(T()) & 0x7FFF7FFFu) {
        if (sizeof(T) == 4) least = 0x7F800000u;
    }
    __device__ __forceinline__ void add(const uint4 &raw, const uint4 &allowed, bool weigh, float c) {
        constexpr int N = Row<T>::kVec;
        const uint32_t here = vec_max<T>(allowed);
        most = pair_max(most, here, T());
        least = pair_min(least, vec_min<T>(raw), T());
        if (weigh) {
            const float2 two = pair_values(here, T());
            const float larger = max_nan(two.x, two.y);
            if (larger > top) {
                sum *= ex2((top - larger) * c);
                top = larger;
            }
            float z[N];
            unpack(allowed, z, T());
            float part[N / 2];
#pragma unroll
            for (int k = 0; k < N / 2; ++k) part[k] = ex2((z[k] - top) * c) + ex2((z[k + N / 2] - top) * c);
#pragma unroll
            for (int k = N / 4; k; k >>= 1)
#pragma unroll
                for (int i = 0; i < k; ++i) part[i] += part[i + k];
            sum += part[0];
        }
    }
    __device__ __forceinline__ void end(bool weigh) {
        const float2 two = pair_values(most, T());
        const float larger = max_nan(two.x, two.y);
        if (!(larger < -kNoLogit)) sum = __int_as_float(0x7FFFFFFF);
        top = fmaxf(larger, kLowest);
    }
    __device__ __forceinline__ float low() const {
        const float2 two = pair_values(least, T());
        return fminf(two.x, two.y);
    }
};
// Goes through the slice, and copies it where it is resident.
template <typename T, bool kResident>
__device__ __forceinline__ SampleRange<T> load_slice(const Slice<T, kResident> &s, bool weigh, float c) {
    constexpr int N = Row<T>::kVec, kUnroll = 4;
    SampleRange<T> r;
    for (int i = threadIdx.x; i < s.row.vecs; i += kSampleThreads * kUnroll) {
        uint4 raw[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (i + u * kSampleThreads < s.row.vecs) raw[u] = s.global_vec(i + u * kSampleThreads);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int at = i + u * kSampleThreads;
            if (at < s.row.vecs) {
                uint4 allowed = raw[u];
                if (s.mask) {
                    const uint32_t bits = allowed_bits(s.mask, s.v0 + s.row.peel + at * N, s.words);
                    allowed = keep_allowed<T>(allowed, bits);
                    r.barred += N - __popc(bits & ((1u << N) - 1));
                }
                if (kResident) *reinterpret_cast<uint4 *>(s.buf + (s.row.peel + at * N) * sizeof(T)) = allowed;
                r.add(raw[u], allowed, weigh, c);
            }
        }
    }
    if (static_cast<int>(threadIdx.x) < s.loose()) {
        const int j = s.loose_at(threadIdx.x);
        const uint32_t none = no_logit_pair(T());
        const T no_logit = *reinterpret_cast<const T *>(&none), x = s.row.p[j];
        const bool allowed = !s.mask || (s.mask[(s.v0 + j) >> 5] >> ((s.v0 + j) & 31) & 1u);
        alignas(16) T kept[N], any[N];
#pragma unroll
        for (int k = 0; k < N; ++k) kept[k] = no_logit;
        kept[0] = allowed ? x : no_logit;
#pragma unroll
        for (int k = 0; k < N; ++k) any[k] = x;
        if (kResident) reinterpret_cast<T *>(s.buf)[j] = kept[0];
        r.barred += !allowed;
        r.add(*reinterpret_cast<const uint4 *>(any), *reinterpret_cast<const uint4 *>(kept), weigh, c);
    }
    r.end(weigh);
    return r;
}

// ------------------------------------------------------------------------------ weights

// Units of a sum of about `sum` times the largest weight, 1 at least: 2^-54 of the largest weight, or some 2^-59 of the sum.
__device__ __forceinline__ int units_of(float sum) { return min(kSampleBits, 59 - ilogbf(sum)); }
// For n tokens of a list, whose sum is n at most: it fits 2^63 (2^-54 for 512, 2^-52 for 2048).  (An estimate of the sum gave 2048 the
// smaller units too, and every row that is decided by a list 0.2 us more.)
__device__ __forceinline__ int list_units(int n) { return min(kSampleBits, 31 + __clz(n - 1)); }

// 2^((z - top) c) in units of 2^-bits, c = log2 e / T as the sum of two floats.  y = (z - A) c is a product and its
// error; k is y to the nearest 1/512, the rest |r| <= 2^-9 (after that of the largest logit is taken off), and 2^y =
// 2^(whole part of k) table[k mod 512] (1 + r ln 2 + ...).  A = 0, or the largest logit where that times c leaves
// the range of k: logits that count are then within a factor of two of it, and the difference is exact.  From T = 2^96 on logits and
// T are taken 2^-32 times, which is exact for all that counts beside such a T: the floor of the weights, 54 octaves and more
// below the largest logit, is then an fp32 number for every T and logit, and a logit of -infinity, below it, weighs 0; and c_lo
// keeps its digits.
struct SampleWeights {
    float A, c_hi, c_lo, rest_top, least, big;  // A and least as z times shrink
    float shrink;
    int k_top;  // as the bits of the shifted product
    int64_t rest64_top;
    float c, top, temperature;
    static constexpr float kShift = 1.5f * (1 << 14);  // floats near it have steps of 1/512
    // y = d c to the nearest 1 / 512 (its bits), and the rest.  (Every operation rounds by itself: the largest logit's rest is
    // to be the same number wherever it is made.)
    __device__ __forceinline__ int split(float d, float &rest) const {
        const float y = __fmul_rn(d, c_hi), t = __fadd_rn(y, kShift);
        rest = __fadd_rn(__fsub_rn(y, __fsub_rn(t, kShift)), fmaf(d, c_lo, fmaf(d, c_hi, -y)));
        return __float_as_int(t);
    }
    // log2 e / T in two floats: the quotient and what it leaves, divided again.
    __device__ void set_temperature(float T) {
        constexpr float kHigh = 1.44269502f, kLow = 1.92596303e-8f;  // log2 e
        temperature = T;
        c = __fdiv_rn(kHigh, T);
        shrink = T < 0x1p96f ? 1.f : 0x1p-32f;
        T *= shrink;
        c_hi = __fdiv_rn(kHigh, T);
        c_lo = __fdiv_rn(fmaf(-c_hi, T, kHigh) + kLow, T);
    }
    // z times shrink, from A on.
    __device__ __forceinline__ float from_A(float z) const { return fmaf(z, shrink, -A); }
    __device__ void set_top(float top_logit) {
        top = top_logit;
        A = 0.f;
        const float shrunk = from_A(top_logit);
        if (!(fabsf(shrunk) * c_hi < 0x1p12f)) A = shrunk;
        k_top = split(shrunk - A, rest_top);
        rest64_top = rest64(shrunk - A, k_top);
        big = -kNoLogit;
    }
    // Logits so far below weigh nothing: under 2^-bits.
    __device__ void set_floor(int bits) {
        least = from_A(top) - (static_cast<float>(bits) + 0.5f) / c_hi;
    }
    // Of a sum of about `sum` times the largest weight, those that hold 2^-10 and more.
    __device__ void set_big(float sum) { big = top - (10.f - log2f(sum)) / c; }
    __device__ __forceinline__ uint64_t of(float z, int bits, const uint32_t *table) const {
        uint64_t m[2];
        two_of(z, kNoLogit, bits, table, m);
        return m[0];
    }
    // Two at a time.  A logit at the floor and below gets the weight 0: its difference is taken for one of bits + 1/2 octaves,
    // and the shift leaves nothing.
    __device__ __forceinline__ void two_of(float z0, float z1, int bits, const uint32_t *table, uint64_t (&m)[2]) const {
        const f32x2 d = pack2(fmaxf(from_A(z0), least), fmaxf(from_A(z1), least)), c2 = pack2(c_hi, c_hi), shift = pack2(kShift, kShift);
        const f32x2 minus = pack2(-1.f, -1.f);
        const f32x2 y = mul2(d, c2), t = add2(y, shift);
        // (y - (t - shift)) + (d c_lo + (d c_hi - y)) - rest_top
        const f32x2 head = fma2(minus, add2(t, pack2(-kShift, -kShift)), y);
        const f32x2 r = add2(add2(head, fma2(d, pack2(c_lo, c_lo), fma2(d, c2, mul2(minus, y)))), pack2(-rest_top, -rest_top));
        // r ln 2 + r^2 ln^2 2 / 2 + r^3 ln^3 2 / 6 in units of 2^-31, to the nearest
        f32x2 q = fma2(r, pack2(1.1919417e8f, 1.1919417e8f), pack2(5.158825e8f, 5.158825e8f));
        q = fma2(r, q, pack2(1.488522236e9f, 1.488522236e9f));
        q = fma2(r, q, pack2(12582912.f, 12582912.f));
        float tf[2], qf[2];
        unpack2(t, tf[0], tf[1]);
        unpack2(q, qf[0], qf[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int k = __float_as_int(tf[i]) - k_top;
            const uint32_t one_q = static_cast<uint32_t>(__float_as_int(qf[i])) + (0x80000000u - 0x4B400000u);
            m[i] = static_cast<uint64_t>(table[k & (kSampleTable - 1)]) * one_q >> ((62 - bits - (k >> 9)) & 63);  // of 2^62 to 2^63
        }
    }
    // The rest of y in units of 2^-52: the product's and its error.
    __device__ __forceinline__ int64_t rest64(float d, int &k) const {
        const float y = __fmul_rn(d, c_hi), t = __fadd_rn(y, kShift);
        k = __float_as_int(t);
        return __float2ll_rn(__fsub_rn(y, __fsub_rn(t, kShift)) * 0x1p52f) + __float2ll_rn(fmaf(d, c_lo, fmaf(d, c_hi, -y)) * 0x1p52f);
    }
    // 2^(r + k mod 512 / 512) in units of 2^-52, r in these too.
    static __device__ __forceinline__ uint64_t power(int64_t r, int k, const SampleTable *table) {
        const int64_t x = __mul64hi(r << 8, 0x58B90BFBE8E7BCD6ll) >> 7;  // r ln 2: ln 2 in units of 2^-63
        const float xf = static_cast<float>(x) * 0x1p-52f;
        const int64_t p = x + (__mul64hi(x << 6, x << 6) >> 1) + __float2ll_rn(xf * xf * xf * (0.16666667f + xf * 0.041666668f) * 0x1p52f);
        const int at = k & (kSampleTable - 1);
        const int64_t whole = (static_cast<int64_t>(table->v[at]) << 21) + table->rest[at];
        return static_cast<uint64_t>(whole + __mul64hi(whole << 5, p << 7));
    }
    // The same weight with every step in 64 bits, right to some 2^-42.
    __device__ __noinline__ uint64_t in_64_bits(float z, int bits, const SampleTable *table) const {
        const float d = from_A(z);
        if (!(d > least)) return 0;
        int k;
        const int64_t r = rest64(d, k) - rest64_top;
        k -= k_top;
        uint64_t m = power(r, k, table);  // 2^52 to 2^53
        const int down = 52 - bits - (k >> 9);
        return down > 0 ? (m >> min(down - 1, 63)) + 1 >> 1 : m << -down;
    }
    // With the big ones in 64 bits.
    __device__ __forceinline__ uint64_t exact_of(float z, int bits, const SampleTable &table) const {
        if (z >= big) return in_64_bits(z, bits, &table);
        return of(z, bits, table.v);
    }
};

// T ln m, m in (0, 1], as the sum of two floats: logf's number l, and what e^l, in 64 bits, lacks of m.
__device__ __forceinline__ float2 scaled_log(float T, float m, const SampleTable *table) {
    SampleWeights w;
    w.set_temperature(1.f);
    const float l = logf(m);
    int k;
    const int64_t r = w.rest64(l, k);
    k -= __float_as_int(SampleWeights::kShift);
    const int64_t e = static_cast<int64_t>(SampleWeights::power(r, k, table));  // times 2^((k >> 9) - 52)
    const uint32_t b = __float_as_uint(m), field = b >> 23;
    const int64_t whole = field ? (b & 0x7FFFFFu) | 0x800000u : b;
    const int up = static_cast<int>(max(field, 1u)) - 150 + 52 - (k >> 9);  // some 29
    const float off = static_cast<float>((whole << up) - e) / static_cast<float>(e);
    const float high = T * l;
    return make_float2(high, fmaf(T, l, -high) + T * off);
}

// ------------------------------------------------------------------------------ shared memory

// A kept prefix of the order: logits above `key`, and those at it up to token `last`.
struct SampleCut {
    uint32_t key;
    int last;
    __device__ __forceinline__ bool keeps(uint32_t k, int v) const { return k > key || (k == key && v <= last); }
};

// A bin at which a running count or sum passes something, with both before and behind it.
struct SampleFound {
    int bin, count0, count1;
    float sum0, sum1;
};
// What the first histogram leaves to be found out.
struct SamplePlan {
    int slow;               // nothing but the four passes will do
    int gather;             // top-k: every token before `draw1` is listed, and all is decided there
    int by_list;            // top-p: the cut is in the bins from cut0 to cut1
    int by_edge;            // min-p: tokens from `edge` on are kept, and there is no other cut
    float draw0, draw1, cut0, cut1;  // places, in parts of bins
    int cut_count;          // tokens before cut0
    float sum;              // about that of all weights
    int bits;               // units of sums: 2^-bits of the largest weight
};
// An entry of a sorted list, and the weights before it.
struct SampleHit {
    int at;
    uint64_t before, w, entry;
};
struct SampleResult {
    int slow;
    SampleCut cut;
    int token, kept;
    float prob;
};

struct SampleShared {
    SampleTable table;
    SampleWeights w;
    // what lies where the first histogram was, and the lists will be
    struct Scratch {
        uint64_t mass[256];
        uint32_t count[256];
    } *x;
    float range[5][kSampleWarps];  // largest, smallest, sum, n-th of the threads' largest, weights of the n largest
    int finite[kSampleWarps], binned[kSampleWarps];
    float sums[kSampleWarps];
    uint32_t units[kSampleWarps];
    float sum;
    int counts[kSampleWarps];
    // what the first CTA of the cluster has found
    uint64_t above;            // of the bins above the border's
    uint64_t bin_mass;
    int above_count, bin_count, bin;
    int tie;                   // the token of a tie that the border falls on
    float edge;                // the smallest logit that min-p keeps
    // the quick way
    SampleFound found[5];
    float edges[4];            // the smallest logits before the plan's places
    int listed[2], list_at[2]; // entries of this CTA's lists, and where they go in the first one's
    SamplePlan plan;
    SampleResult result;
    // in the first CTA
    uint64_t part[kSampleMaxCluster][3];  // of every CTA: weights of all that count, above the cut's bins, above the draw's
    int part_count[kSampleMaxCluster];
    uint64_t warp_sums[3][kSampleWarps];
    SampleHit hit;
    int first;                 // whether the short way has found the token
};

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
__device__ __forceinline__ void st_cluster_u64(uint32_t a, uint64_t v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory");
}
__device__ __forceinline__ int add_cluster(uint32_t a, int n) {  // returns the value before
    int old;
    asm volatile("atom.relaxed.cluster.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(old) : "r"(a), "r"(n) : "memory");
    return old;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
template <typename V>
__device__ __forceinline__ uint32_t peer(const V *p, int rank) { return mapa_shared(smem_u32(p), rank); }

// All threads of the row.
__device__ __forceinline__ void row_sync(int ranks) {
    if (ranks > 1)
        cluster_sync();
    else
        __syncthreads();
}

// Of all threads of the row, in each of them.
__device__ __forceinline__ int sum_of_row(SampleShared &sm, int ranks, int mine) {
    mine = __reduce_add_sync(0xffffffffu, mine);
    if ((threadIdx.x & 31) == 0) sm.binned[threadIdx.x >> 5] = mine;
    row_sync(ranks);
    int all = 0;
#pragma unroll
    for (int i = 0; i < kSampleSteps; ++i) {
        const int lane = threadIdx.x & 31, q = 32 / kSampleWarps * i + lane / kSampleWarps;
        if (q < ranks) all += static_cast<int>(ld_cluster_u32(peer(&sm.binned[lane % kSampleWarps], q)));
    }
    row_sync(ranks);
    return __reduce_add_sync(0xffffffffu, all);
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
            sm.x->mass[i] = 0;
            sm.x->count[i] = 0;
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
                    atomicAdd(&sm.x->count[run], run_count);
                    atomicAdd(reinterpret_cast<unsigned long long *>(&sm.x->mass[run]), static_cast<unsigned long long>(run_mass));
                }
                run = b;
                run_count = 0;
                run_mass = 0;
            }
            ++run_count;
            run_mass += sm.w.exact_of(z, bits, sm.table);
        });
        if (run >= 0) {
            atomicAdd(&sm.x->count[run], run_count);
            atomicAdd(reinterpret_cast<unsigned long long *>(&sm.x->mass[run]), static_cast<unsigned long long>(run_mass));
        }
        row_sync(ranks);
        if (rank == 0) {
            if (threadIdx.x < 256) {
                uint64_t m = 0;
                uint32_t c = 0;
                for (int r = 0; r < ranks; ++r) {
                    m += ld_cluster_u64(peer(&sm.x->mass[threadIdx.x], r));
                    c += ld_cluster_u32(peer(&sm.x->count[threadIdx.x], r));
                }
                sm.x->mass[threadIdx.x] = m;
                sm.x->count[threadIdx.x] = c;
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                uint64_t m = above;
                int c = above_count, found = -1;
                for (int b = 255; b >= 0; --b) {
                    const int bc = static_cast<int>(sm.x->count[b]);
                    if (bc == 0) continue;
                    found = b;
                    sm.above = m;
                    sm.above_count = c;
                    m += sm.x->mass[b];
                    c += bc;
                    const double at = static_cast<double>(m);
                    if (t.by_count ? c >= t.count : t.strictly ? at > t.mass : at >= t.mass) break;
                }
                sm.bin = found;  // (the last one that is not empty where roundings let none reach it)
                sm.bin_count = static_cast<int>(sm.x->count[found]);
                sm.bin_mass = sm.x->mass[found];
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
        sm.x->mass[threadIdx.x >> 5] = m;
        sm.counts[threadIdx.x >> 5] = c;
    }
    row_sync(ranks);
    m = 0;
    c = 0;
    for (int r = 0; r < ranks; ++r)
        for (int w = 0; w < kSampleWarps; ++w) {
            m += ld_cluster_u64(peer(&sm.x->mass[w], r));
            c += static_cast<int>(ld_cluster_u32(peer(&sm.counts[w], r)));
        }
    row_sync(ranks);
    count = c;
    return static_cast<double>(m);
}

// The tokens that `keep` holds for (or none) as bits: 32 tokens a warp and word; a lane keeps one of 32 words, so that they are
// stored together.
template <typename S, typename F>
__device__ __forceinline__ void write_bits(const S &s, uint32_t *out, bool none, F keep) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, words = (s.row.V + 31) / 32;
    out += s.v0 / 32;
    for (int w0 = warp * 32; w0 < words; w0 += kSampleThreads) {
        uint32_t mine = 0;
        if (!none)
#pragma unroll 1
            for (int i = 0; i < 32; i += 8) {
                float z[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {  // (asked for together: word by word the answers are waited for one by one)
                    const int j = (w0 + i + k) * 32 + lane;
                    z[k] = j < s.row.V ? s.at(j) : kNoLogit;
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const uint32_t word = __ballot_sync(0xffffffffu, keep(z[k], s.v0 + (w0 + i + k) * 32 + lane));
                    if (i + k == lane) mine = word;
                }
            }
        if (w0 + lane < words) out[w0 + lane] = mine;
    }
}

// Every border in four passes.  Leaves the result in every CTA.
template <typename S>
__device__ __noinline__ void sample_slowly(const S &s, SampleShared &sm, int ranks, int rank, float top, float edge, int top_k,
                                           float top_p, float u) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
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
        sum = fmaxf(sum, 1.f);
        sm.plan.bits = units_of(sum);
        sm.w.set_floor(sm.plan.bits);
        sm.w.set_big(sum);
    }
    row_sync(ranks);
    const int bits = sm.plan.bits;
    SampleCut cut{0u, 0x7FFFFFFF};
    int n, place;
    double mass = kept_mass(s, sm, ranks, bits, cut, n), weight, upto;
    if (top_k > 0 && top_k < n) cut = find_border(s, sm, ranks, rank, bits, cut, {true, false, top_k, 0.0}, n, mass, weight);
    if (top_p < 1.f) cut = find_border(s, sm, ranks, rank, bits, cut, {false, false, 0, top_p * mass}, n, mass, weight);
    if (edge != kNoLogit && order_key(edge) > cut.key) {
        cut = {order_key(edge), 0x7FFFFFFF};
        mass = kept_mass(s, sm, ranks, bits, cut, n);
    }
    const SampleCut token = find_border(s, sm, ranks, rank, bits, cut, {false, true, 0, u * mass}, place, upto, weight);
    if (threadIdx.x == 0) sm.result = {0, cut, token.last, n, static_cast<float>(weight / mass)};
    __syncthreads();
}

// ------------------------------------------------------------------------------ the quick way

// A place in the order, in parts of bins: 0 at the largest logit.
__device__ __forceinline__ float sample_place(float z, float top, float scale) { return (top - z) * scale; }

// Entries in ascending order are tokens in theirs.
__device__ __forceinline__ uint64_t sample_entry(float z, int v) { return static_cast<uint64_t>(~order_key(z)) << 32 | static_cast<uint32_t>(v); }

// Up to kSampleThreads entries of each of kLists lists, which lie `apart` entries apart: an entry a thread, exchanged by shuffles
// where its partner is in the same warp.
template <int kLists>
__device__ __forceinline__ void sort_in_registers(uint64_t *list, int apart, int size) {
    const int t = threadIdx.x;
    uint64_t x[kLists];
#pragma unroll
    for (int l = 0; l < kLists; ++l) x[l] = t < size ? list[l * apart + t] : ~0ull;
    for (int k = 2; k <= size; k <<= 1)
        for (int j = k >> 1; j; j >>= 1) {
            const bool low = ((t & k) == 0) == ((t & j) == 0);  // keeps the smaller one
            uint64_t y[kLists];
            if (j >= 32) {
                __syncthreads();
#pragma unroll
                for (int l = 0; l < kLists; ++l)
                    if (t < size) list[l * apart + t] = x[l];
                __syncthreads();
#pragma unroll
                for (int l = 0; l < kLists; ++l) y[l] = t < size ? list[l * apart + (t ^ j)] : ~0ull;
            } else {
#pragma unroll
                for (int l = 0; l < kLists; ++l) y[l] = __shfl_xor_sync(0xffffffffu, x[l], j);
            }
#pragma unroll
            for (int l = 0; l < kLists; ++l)
                if ((y[l] < x[l]) == low) x[l] = y[l];
        }
    __syncthreads();
#pragma unroll
    for (int l = 0; l < kLists; ++l)
        if (t < size) list[l * apart + t] = x[l];
    __syncthreads();
}

// kPer entries a thread, kSampleThreads apart: those exchange in its registers, neighbours by shuffles, the others in shared
// memory.  (All steps there, 66 of them with a barrier each, took 900 rows of 2000 tokens from 112 to 129 us.)
template <int kPer>
__device__ __forceinline__ void sort_long(uint64_t *list) {
    const int t = threadIdx.x;
    uint64_t x[kPer];
#pragma unroll
    for (int l = 0; l < kPer; ++l) x[l] = list[l * kSampleThreads + t];
#pragma unroll 1
    for (int k = 2; k <= kPer * kSampleThreads; k <<= 1) {
#pragma unroll
        for (int d = kPer / 2; d; d >>= 1)
            if (k > d * kSampleThreads)
#pragma unroll
                for (int l = 0; l < kPer; ++l) {
                    if (l & d) continue;
                    const uint64_t a = x[l], b = x[l | d];
                    const bool swap = (b < a) == (((l * kSampleThreads) & k) == 0);
                    x[l] = swap ? b : a;
                    x[l | d] = swap ? a : b;
                }
#pragma unroll 1
        for (int j = min(k, kSampleThreads) >> 1; j; j >>= 1) {
            uint64_t y[kPer];
            if (j >= 32) {
                __syncthreads();
#pragma unroll
                for (int l = 0; l < kPer; ++l) list[l * kSampleThreads + t] = x[l];
                __syncthreads();
#pragma unroll
                for (int l = 0; l < kPer; ++l) y[l] = list[l * kSampleThreads + (t ^ j)];
            } else {
#pragma unroll
                for (int l = 0; l < kPer; ++l) y[l] = __shfl_xor_sync(0xffffffffu, x[l], j);
            }
#pragma unroll
            for (int l = 0; l < kPer; ++l) {
                const bool low = (((l * kSampleThreads + t) & k) == 0) == ((t & j) == 0);
                if ((y[l] < x[l]) == low) x[l] = y[l];
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int l = 0; l < kPer; ++l) list[l * kSampleThreads + t] = x[l];
    __syncthreads();
}

// n0 entries, and n1 from kSampleList / 2 on, by the CTA; each padded to `size`, a power of two (returned).
__device__ __noinline__ int sort_entries(uint64_t *list, int n0, int n1) {
    int size = 32;
    while (size < n0 || size < n1) size <<= 1;
    for (int i = n0 + threadIdx.x; i < size; i += kSampleThreads) list[i] = ~0ull;
    if (n1)
        for (int i = n1 + threadIdx.x; i < size; i += kSampleThreads) list[kSampleList / 2 + i] = ~0ull;
    __syncthreads();
    if (size <= kSampleThreads) {
        if (n1)
            sort_in_registers<2>(list, kSampleList / 2, size);
        else
            sort_in_registers<1>(list, 0, size);
        return size;
    }
    for (int l = 0; l < (n1 ? 2 : 1); ++l) {
        if (size == 2 * kSampleThreads)
            sort_long<2>(list + l * (kSampleList / 2));
        else
            sort_long<kSampleList / kSampleThreads>(list);
    }
    return size;
}

// a f, f in [0, 1) and not -0, rounded down or up.
__device__ __forceinline__ uint64_t times_fraction(uint64_t a, float f, bool up) {
    const uint32_t b = __float_as_uint(f), e = b >> 23;
    const uint64_t m = e ? (b & 0x7FFFFFu) | 0x800000u : b & 0x7FFFFFu;
    const int s = 150 - static_cast<int>(max(e, 1u));  // f = m 2^-s, s >= 24
    const uint64_t hi = __umul64hi(a, m), lo = a * m;
    if (s >= 128) return up && (hi | lo);
    if (s >= 64) {
        const uint64_t q = hi >> (s - 64);
        return q + (up && (lo || (q << (s - 64)) != hi));
    }
    return (hi << (64 - s) | lo >> s) + (up && lo << (64 - s));
}

// a / b to the nearest fp32 number, nearly: numbers as two floats each, the quotient's rest divided again.
__device__ __forceinline__ float quotient(uint64_t a, uint64_t b) {
    const float a_hi = __ull2float_rz(a), b_hi = __ull2float_rz(b);
    const float a_lo = __ull2float_rn(a - __float2ull_rz(a_hi)), b_lo = __ull2float_rn(b - __float2ull_rz(b_hi));
    const float q = a_hi / b_hi;
    return q + (fmaf(-q, b_hi, a_hi) + fmaf(-q, b_lo, a_lo)) / b_hi;
}

// Running sums of the weights of n sorted entries, up to and with each, in shared memory; the sum of all is returned.
__device__ __forceinline__ uint64_t add_up(const uint64_t *list, int n, uint64_t *upto, int bits, SampleShared &sm) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint64_t before = 0;
#pragma unroll 1
    for (int first = 0; first < n; first += kSampleThreads) {
        const int i = first + threadIdx.x;
        uint64_t m = i < n ? sm.w.exact_of(key_value(~static_cast<uint32_t>(list[i] >> 32)), bits, sm.table) : 0ull;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint64_t up = __shfl_up_sync(0xffffffffu, m, o);
            if (lane >= o) m += up;
        }
        if (lane == 31) sm.warp_sums[0][warp] = m;
        __syncthreads();
        uint64_t all = before;
#pragma unroll
        for (int w = 0; w < kSampleWarps; ++w) {
            const uint64_t v = sm.warp_sums[0][w];
            if (w < warp) before += v;
            all += v;
        }
        if (i < n) upto[i] = before + m;
        before = all;
        __syncthreads();
    }
    return before;
}

// The first entry at which the weights, `base` and those before it, reach `target`, or whose logit is below `edge`
// (but not entry 0 if `spare`); or, `through`, the first with which they exceed `target`.  Number n if there is none.
__device__ __forceinline__ SampleHit find_entry(const uint64_t *list, const uint64_t *upto, int n, uint64_t base, uint64_t target, bool through,
                                                bool spare, float edge, SampleShared &sm) {
    __syncthreads();
    if (threadIdx.x == 0) sm.hit = {n, n ? upto[n - 1] : 0ull, 0, ~0ull};
    __syncthreads();
#pragma unroll 1
    for (int i = threadIdx.x; i < n; i += kSampleThreads) {
        const uint64_t with = upto[i], before = i ? upto[i - 1] : 0ull;
        bool now, earlier;  // whether it holds for this entry and for the one before (once it holds it does for all that follow)
        if (through) {
            now = base + with > target;
            earlier = i && base + before > target;
        } else {
            const auto below = [&](int j) { return key_value(~static_cast<uint32_t>(list[j] >> 32)) < edge; };
            now = (base + before >= target || below(i)) && !(spare && i == 0);
            earlier = i && (base + (i > 1 ? upto[i - 2] : 0ull) >= target || below(i - 1)) && !(spare && i == 1);
        }
        if (now && !earlier) sm.hit = {i, before, with - before, list[i]};
    }
    __syncthreads();
    return sm.hit;
}

// A CTA's bins of the row's histogram: counts and weights in units, kPer neighbours a thread; and the running ones before each
// thread's, of the row.
struct SampleBins {
    const uint2 *own;
    int per, first;    // bins of a thread, and the first of this one's among the row's
    int count0, count1, all_count;  // before and behind this thread's, and of the row
    uint32_t units0, units1;
    float unit;        // weight of one
    // The first bin for which the border's condition holds, in every CTA's found[slot] (one thread of the row has it; see
    // BinBorder); what was there stays where it holds for none.
    __device__ __forceinline__ void find(SampleShared &sm, int slot, int ranks, bool by_count, float least, bool more) const {
        const BinBorder border{by_count, more, least, unit};
        if (!border.within(first == 0, count0, units0, count1, units1)) return;
        int i = 0, n = count0, n1 = n;
        uint32_t m = units0, m1 = m;
        for (;; ++i) {
            const uint2 v = own[i];
            n1 = n + static_cast<int>(v.x);
            m1 = m + v.y;
            if (i == per - 1 || border.holds(n1, m1)) break;
            n = n1;
            m = m1;
        }
        tell(sm, slot, ranks, {first + i, n, n1, border.weight(m), border.weight(m1)});
    }
    // The same for a bin that is known.
    __device__ __forceinline__ void find_bin(SampleShared &sm, int slot, int ranks, int bin) const {
        if (bin < first || bin >= first + per) return;
        int n = count0;
        uint32_t m = units0;
        for (int i = 0; i < bin - first; ++i) {
            n += static_cast<int>(own[i].x);
            m += own[i].y;
        }
        const uint2 v = own[bin - first];
        tell(sm, slot, ranks, {bin, n, n + static_cast<int>(v.x), static_cast<float>(m) * unit, static_cast<float>(m + v.y) * unit});
    }
    __device__ __forceinline__ void tell(SampleShared &sm, int slot, int ranks, const SampleFound &f) const {
        for (int q = 0; q < ranks; ++q) {
            const uint32_t to = peer(&sm.found[slot], q);
            st_shared_cluster(to, f.bin);
            st_shared_cluster(to + 4, f.count0);
            st_shared_cluster(to + 8, f.count1);
            st_shared_cluster(to + 12, __float_as_int(f.sum0));
            st_shared_cluster(to + 16, __float_as_int(f.sum1));
        }
    }
};

// The slices' histograms become the row's, a part of the bins a CTA.  `sum`: about that of the row's weights, 1 at least.
__device__ __forceinline__ SampleBins make_bins(SampleShared &sm, const uint32_t *hist, uint8_t *own, int ranks, int rank, float octaves, float sum) {
    const float units = kBinUnits / sum;
    const int per_rank = kSampleBins / ranks, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint2 *mine = reinterpret_cast<uint2 *>(own);
    for (int i = threadIdx.x; i < per_rank; i += kSampleThreads) {
        const int b = rank * per_rank + i;
        uint32_t v[kSampleMaxCluster], n = 0, parts = 0;
#pragma unroll
        for (int q = 0; q < kSampleMaxCluster; ++q) v[q] = q < ranks ? ld_cluster_u32(peer(&hist[b], q)) : 0u;
#pragma unroll
        for (int q = 0; q < kSampleMaxCluster; ++q) {
            n += v[q] >> 20;
            parts += v[q] & 0xFFFFFu;
        }
        const float mean = n ? __fdividef(static_cast<float>(parts), static_cast<float>(n)) + 0.5f : 0.f;
        mine[i] = make_uint2(n, bin_units(static_cast<float>(n) * ex2(-(static_cast<float>(b * kBinParts) + mean) * octaves), units));
    }
    __syncthreads();
    SampleBins bins;
    bins.per = per_rank / kSampleThreads;
    bins.own = mine + threadIdx.x * bins.per;
    bins.first = rank * per_rank + static_cast<int>(threadIdx.x) * bins.per;
    bins.unit = sum / kBinUnits;
    int n = 0;
    uint32_t m = 0;
    for (int i = 0; i < bins.per; ++i) {
        n += static_cast<int>(bins.own[i].x);
        m += bins.own[i].y;
    }
    int n_upto = n;
    uint32_t m_upto = m;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int nu = __shfl_up_sync(0xffffffffu, n_upto, o);
        const uint32_t mu = __shfl_up_sync(0xffffffffu, m_upto, o);
        if (lane >= o) {
            n_upto += nu;
            m_upto += mu;
        }
    }
    if (lane == 31) {
        sm.counts[warp] = n_upto;
        sm.units[warp] = m_upto;
    }
    row_sync(ranks);
    // totals of all warps before this one, in this CTA and those before
    int n_before = 0, n_all = 0;
    uint32_t m_before = 0;
#pragma unroll
    for (int i = 0; i < kSampleSteps; ++i) {
        const int q = 32 / kSampleWarps * i + lane / kSampleWarps, w = lane % kSampleWarps;
        if (q < ranks) {
            const int nw = static_cast<int>(ld_cluster_u32(peer(&sm.counts[w], q)));
            n_all += nw;
            if (q < rank || (q == rank && w < warp)) {
                n_before += nw;
                m_before += ld_cluster_u32(peer(&sm.units[w], q));
            }
        }
    }
    n_all = __reduce_add_sync(0xffffffffu, n_all);
    n_before = __reduce_add_sync(0xffffffffu, n_before);
    m_before = __reduce_add_sync(0xffffffffu, m_before);
    bins.count1 = n_before + n_upto;
    bins.units1 = m_before + m_upto;
    bins.count0 = bins.count1 - n;
    bins.units0 = bins.units1 - m;
    bins.all_count = n_all;
    return bins;
}

// Which bins the borders are in, by the running counts and sums of bins.  Sums are kBinError off at most, so that a border may
// be in either of two bins, or more.  Every thread of the row calls it and knows the plan.
__device__ __forceinline__ SamplePlan plan_borders(SampleShared &sm, const SampleBins &bins, int ranks, float top, float edge, float scale, float sum,
                                                   int expected, int top_k, float top_p, float u) {
    constexpr float kEnd = static_cast<float>(kSampleBins) * kBinParts;
    const auto place_of = [](int bin) { return static_cast<float>(bin) * kBinParts; };
    const float error = kBinError * sum;
    const float edge_place = edge == kNoLogit ? kEnd : fminf(sample_place(edge, top, scale), kEnd);
    SamplePlan plan{};
    plan.sum = sum;
    plan.bits = top_k > 0 ? list_units(top_k) : units_of(sum);
    plan.cut0 = plan.cut1 = -1.f;
    plan.slow = bins.all_count != expected;  // a bin had more tokens than it can count
    if (top_k > 0) {
        bins.find(sm, 0, ranks, true, static_cast<float>(top_k), false);
    } else {
        if (top_p < 1.f) {
            bins.find(sm, 0, ranks, false, top_p * sum - error, false);
            bins.find(sm, 1, ranks, false, top_p * sum + error, false);
        }
        if (edge_place < kEnd) bins.find_bin(sm, 4, ranks, static_cast<int>(edge_place) / kBinParts);
    }
    row_sync(ranks);
    if (top_k > 0) {
        plan.gather = 1;
        plan.draw1 = place_of(sm.found[0].bin + 1);
        plan.slow |= sm.found[0].bin == kSampleBins || sm.found[0].count1 > kSampleList;
        return plan;
    }
    float least = sum, most = sum;  // of the kept weights
    int last = kSampleBins - 1, last_count = bins.all_count;  // bin of a kept token, and tokens up to its end
    plan.by_edge = edge != kNoLogit;
    if (top_p < 1.f) {
        const SampleFound f0 = sm.found[0], f1 = sm.found[1];
        if (edge_place >= place_of(f0.bin)) {
            plan.by_list = 1;
            plan.by_edge = 0;
            plan.cut0 = place_of(f0.bin);
            plan.cut1 = place_of(min(f1.bin + 1, kSampleBins));
            plan.cut_count = f0.count0;
            least = f0.sum0;
            most = f1.bin < kSampleBins ? f1.sum1 : sum;
            if (f1.bin < kSampleBins) {
                last = f1.bin;
                last_count = f1.count1;
            }
            plan.slow |= f0.bin == kSampleBins || last_count - f0.count0 > kSampleList / 2;
        }
    }
    if (plan.by_edge && edge_place < kEnd) {
        const SampleFound f = sm.found[4];
        last = f.bin;
        last_count = f.count1;
        least = f.sum0;
        most = f.sum1;
    }
    least = u * least - error;
    most = u * most + error;
    bins.find(sm, 2, ranks, false, least, true);
    bins.find(sm, 3, ranks, false, most, true);
    row_sync(ranks);
    const SampleFound f0 = sm.found[2], f1 = sm.found[3];
    plan.slow |= f0.bin > last;
    plan.draw0 = place_of(min(f0.bin, last));
    plan.draw1 = place_of(min(f1.bin, last) + 1);
    plan.slow |= (f1.bin > last ? last_count : f1.count1) - f0.count0 > kSampleList / 2;
    return plan;
}

// The smallest logit before a place (infinity: none is): by halves, of the few floats around it where these are enough.
__device__ __forceinline__ float logit_before(float place, float top, float scale) {
    if (!(place > 0.f)) return -kNoLogit;
    const auto before = [&](uint32_t key) { return sample_place(key_value(key), top, scale) < place; };
    const float about = top - place / scale, off = 0x1p-21f * fmaxf(fabsf(top), fabsf(about));
    uint32_t no = order_key(kLowest) - 1, yes = order_key(top);  // not before it; before it
    const float low = about - off, high = about + off;
    if (low >= kLowest && !before(order_key(low))) no = order_key(low);
    if (high < top && before(order_key(high))) yes = order_key(high);
    while (yes - no > 1) {
        const uint32_t mid = no + (yes - no) / 2;
        if (before(mid))
            yes = mid;
        else
            no = mid;
    }
    return key_value(yes);
}

// A token's entry at the end of a list of this CTA.
__device__ __forceinline__ void list_token(int *listed, uint64_t *list, int room, float z, int v) {
    const int at = atomicAdd(listed, 1);
    if (at < room) list[at] = sample_entry(z, v);
}

// A first histogram of the row over 4096 bins, equally wide in the logit, says in which one or two of them each border is;
// a second pass adds the weights before these up, exactly, and lists the tokens in them; the lists go to the first CTA's shared
// memory, which sorts them (solve_lists).  With top-k all tokens that may be kept are listed.  False: the row is not like that (so
// many equal logits that a bin's count or a list runs over, or a k of thousands).  `hist` is clear; kept tokens' bits go to out,
// those in the cut's bins excepted.
template <typename S>
__device__ __forceinline__ bool list_borders(const S &s, SampleShared &sm, uint32_t *hist, uint8_t *own, int ranks, int rank, float top,
                                             float low, float least, float sum, int finite, float edge, int top_k, float top_p, float u,
                                             uint32_t *out, uint32_t *kept_bits) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float c = sm.w.c;
    least = fmaxf(least, kLowest);
    const float span = fminf(fminf(kBinOctaves / c, top - fmaxf(low, least)), 3e38f);
    const float scale = span > 0.f ? fminf((kSampleBins * kBinParts - kBinParts / 2) / span, 1e38f) : 0.f;
    int binned = 0;
    s.each_vec(least, [&](const auto &z, int) {
#pragma unroll
        for (int k = 0; k < S::N; ++k)
            if (z[k] >= least) {
                const int at = static_cast<int>(sample_place(z[k], top, scale));
                if (at < kSampleBins * kBinParts) {
                    atomicAdd(&hist[at / kBinParts], (1u << 20) | (at % kBinParts));  // 4095 tokens fit
                    ++binned;
                }
            }
    });
    const int expected = sum_of_row(sm, ranks, binned);
    sum = fmaxf(sum, 1.f);
    const SampleBins bins = make_bins(sm, hist, own, ranks, rank, scale > 0.f ? c / scale : 0.f, sum);
    SamplePlan plan = plan_borders(sm, bins, ranks, top, edge, scale, sum, expected, top_k, top_p, u);
    if (plan.slow) {
        row_sync(ranks);
        return false;
    }
    if (threadIdx.x < 4) {
        const float place = threadIdx.x == 0 ? plan.draw0 : threadIdx.x == 1 ? plan.draw1 : threadIdx.x == 2 ? plan.cut0 : plan.cut1;
        sm.edges[threadIdx.x] = logit_before(place, top, scale);
    }
    if (threadIdx.x == 0) {
        sm.plan = plan;
        sm.w.set_floor(plan.bits);
        sm.w.set_big(plan.sum);
        if (plan.gather) sm.w.big = kNoLogit;  // (few tokens: all of them in 64 bits)
    }
    __syncthreads();
    uint64_t *list = reinterpret_cast<uint64_t *>(hist), *cut_list = list + kSampleList / 2;
    const float draw0 = sm.edges[0], draw1 = sm.edges[1], cut0 = sm.edges[2], cut1 = sm.edges[3];
    const int bits = plan.bits;
    uint64_t sums[3] = {0, 0, 0};
    int count = 0;
    // Bits of the tokens before the cut's bins; of a list's none yet.
    const auto keep = [&](uint32_t bits_of, int v) {
        const int at = v - s.v0;
        atomicOr(&kept_bits[at >> 5], bits_of << (at & 31));
        if (at % 32 + S::N > 32 && bits_of >> (32 - at % 32)) atomicOr(&kept_bits[(at >> 5) + 1], bits_of >> (32 - at % 32));
    };
    const bool mark = out && kept_bits;
    if (mark) {
        for (int i = threadIdx.x; i < (s.row.V + 31) / 32; i += kSampleThreads) kept_bits[i] = 0;
        __syncthreads();
    }
    if (plan.gather) {
        s.each_vec(draw1, [&](const auto &z, int v) {
#pragma unroll
            for (int k = 0; k < S::N; ++k)
                if (z[k] >= draw1) list_token(&sm.listed[0], list, kSampleList, z[k], v + k);
        });
    } else if (plan.by_edge) {
        s.each_vec(edge, [&](const auto &z, int v) {
            uint32_t kept = 0;
#pragma unroll
            for (int k = 0; k < S::N; ++k)
                if (z[k] >= edge) {
                    const uint64_t m = sm.w.exact_of(z[k], bits, sm.table);
                    kept |= 1u << k;
                    ++count;
                    sums[0] += m;
                    if (z[k] >= draw0)
                        sums[2] += m;
                    else if (z[k] >= draw1)
                        list_token(&sm.listed[0], list, kSampleList / 2, z[k], v + k);
                }
            if (mark) keep(kept, v);
        });
    } else {
        const SampleWeights w = sm.w;
        const float from = plan.by_list ? cut0 : kLowest;
        s.each_vec(kNoLogit, [&](const auto &z, int v) {
            uint32_t kept = 0;
            uint32_t special = 0;  // tokens that are listed, or weighed in 64 bits
#pragma unroll
            for (int k = 0; k < S::N; k += 2) {
                uint64_t m[2];
                w.two_of(z[k], z[k + 1], bits, sm.table.v, m);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float x = z[k + i];
                    const bool before_cut = x >= cut0, before_draw = x >= draw0;
                    sums[0] += m[i];
                    if (before_cut) sums[1] += m[i];
                    if (before_draw) sums[2] += m[i];
                    if (x >= from) kept |= 1u << (k + i);
                    if ((x >= cut1 && !before_cut) || (x >= draw1 && !before_draw) || x >= w.big) special |= 1u << (k + i);
                }
            }
            if (kept && mark) keep(kept, v);
            while (special) {
                const int k = __ffs(special) - 1;
                special &= special - 1;
                const float x = s.at(v - s.v0 + k);
                if (x >= w.big) {
                    const uint64_t more = sm.w.in_64_bits(x, bits, &sm.table) - w.of(x, bits, sm.table.v);
                    sums[0] += more;
                    if (x >= cut0) sums[1] += more;
                    if (x >= draw0) sums[2] += more;
                }
                if (x >= cut1 && x < cut0) list_token(&sm.listed[1], cut_list, kSampleList / 2, x, v + k);
                if (x >= draw1 && x < draw0) list_token(&sm.listed[0], list, kSampleList / 2, x, v + k);
            }
        });
    }
    count = __reduce_add_sync(0xffffffffu, count);
#pragma unroll
    for (int i = 0; i < 3; ++i) {
#pragma unroll
        for (int o = 16; o; o >>= 1) sums[i] += __shfl_xor_sync(0xffffffffu, sums[i], o);
        if (lane == 0) sm.warp_sums[i][warp] = sums[i];
    }
    if (lane == 0) sm.counts[warp] = count;
    __syncthreads();
    if (threadIdx.x < 4) {
        uint64_t m = 0;
        int n = 0;
#pragma unroll
        for (int i = 0; i < kSampleWarps; ++i) {
            n += sm.counts[i];
            m += sm.warp_sums[min(2, static_cast<int>(threadIdx.x))][i];
        }
        if (threadIdx.x < 3)
            st_cluster_u64(peer(&sm.part[rank][threadIdx.x], 0), m);
        else
            st_shared_cluster(peer(&sm.part_count[rank], 0), n);
    }
    if (rank != 0) {  // the lists go behind what the first CTA has
        if (threadIdx.x < 2) sm.list_at[threadIdx.x] = sm.listed[threadIdx.x] ? add_cluster(peer(&sm.listed[threadIdx.x], 0), sm.listed[threadIdx.x]) : 0;
        __syncthreads();
#pragma unroll 1
        for (int which = 0; which < 2; ++which) {
            const int room = plan.gather ? kSampleList : kSampleList / 2, at = sm.list_at[which];
            const uint32_t to = peer(list + which * (kSampleList / 2), 0);
            for (int i = threadIdx.x; i < min(sm.listed[which], room - at); i += kSampleThreads)
                st_cluster_u64(to + (at + i) * 8, list[which * (kSampleList / 2) + i]);
        }
    }
    if (mark) {  // (behind the barrier that the sums have had)
        for (int i = threadIdx.x; i < (s.row.V + 31) / 32; i += kSampleThreads) out[s.v0 / 32 + i] = kept_bits[i];
    } else if (out) {
        const float from = plan.gather ? -kNoLogit : plan.by_list ? cut0 : plan.by_edge ? edge : kLowest;
        write_bits(s, out, plan.gather, [&](float z, int) { return z >= from; });
    }
    return true;
}

// The lists' tokens in order, and so the cut and the token: by the row's first CTA alone.  `upto`: room for running sums.  False:
// a border is not where the histogram had it, which its bounds rule out.
__device__ __forceinline__ bool solve_lists(SampleShared &sm, uint64_t *lists, uint64_t *upto, int ranks, int finite, float edge, int top_k, float top_p,
                                            float u, uint32_t *out) {
    const bool gather = sm.plan.gather, by_list = sm.plan.by_list;
    const int bits = sm.plan.bits, cut_count = sm.plan.cut_count;
    int listed = min(sm.listed[0], gather ? kSampleList : kSampleList / 2);
    const int cut_listed = min(sm.listed[1], kSampleList / 2);
    sort_entries(lists, listed, cut_listed);
    uint64_t all = 0, before_cut = 0, before_draw = 0, mass;
    int kept = 0;
    bool good = sm.listed[0] == listed && sm.listed[1] == cut_listed;
    if (!gather) {
        for (int q = 0; q < ranks; ++q) {
            all += sm.part[q][0];
            before_cut += sm.part[q][1];
            before_draw += sm.part[q][2];
            kept += sm.part_count[q];
        }
        if (!sm.plan.by_edge) kept = finite;
    }
    mass = all;
    if (gather || by_list) {
        const uint64_t *list = gather ? lists : lists + kSampleList / 2;
        const int n = gather ? min(listed, top_k) : cut_listed;
        const uint64_t sum = add_up(list, n, upto, bits, sm);
        const uint64_t target = top_p < 1.f ? times_fraction(gather ? sum : all, fmaxf(top_p, 0.f), true) : ~0ull;
        const SampleHit end = find_entry(list, upto, n, before_cut, target, false, cut_count == 0, edge, sm);
        if (by_list) {
            // the border is here if the first token is before it and the last one is not (or the row's last)
            if (cut_count && before_cut >= target) good = false;
            if (end.at == n && cut_count + n < kept && before_cut + sum < target) good = false;
        }
        kept = cut_count + end.at;
        mass = before_cut + end.before;
        if (out)
            for (int i = threadIdx.x; i < end.at; i += kSampleThreads) {
                const int v = static_cast<int>(list[i] & 0xFFFFFFFFu);
                atomicOr(&out[v >> 5], 1u << (v & 31));
            }
        if (gather) listed = end.at;
    }
    if (!gather) {
        __syncthreads();
        add_up(lists, listed, upto, bits, sm);
    }
    const uint64_t target = times_fraction(mass, u, false);
    const SampleHit hit = find_entry(lists, upto, listed, before_draw, target, true, false, edge, sm);
    if (hit.at == listed || before_draw > target) good = false;
    if (threadIdx.x == 0) sm.result = {!good, {}, static_cast<int>(hit.entry & 0xFFFFFFFFu), kept, quotient(hit.w, mass)};
    __syncthreads();
    return good;
}

// ------------------------------------------------------------------------------ the short way

// Lane j has the j-th largest of the warp's numbers, from 0.
__device__ __forceinline__ float sort_warp(float x) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
        for (int j = k >> 1; j; j >>= 1) {
            const float y = __shfl_xor_sync(0xffffffffu, x, j);
            x = (((lane & k) == 0) == ((lane & j) == 0)) ? fmaxf(x, y) : fminf(x, y);
        }
    return x;
}

// What the short way takes a row for.
struct SampleShort {
    bool by_k, by_sum;  // top-k; top-p without it.  Else min-p alone
    bool whole;         // no kept token is below `from`
    bool all;           // every token is listed: V of them are sorted
    float from;         // logits from there on are listed
    int room;           // for so many
};

// Every token that may be kept is among the largest few of most rows: of those that ask for the first k, or whose probable
// tokens hold top_p, or whose min_p has few above it.  They are listed in the first CTA's shared memory.  -1: too many, or
// they hold too little; else their number.  `mask`, which the kept ones' bits go to, is cleared.
template <typename S>
__device__ __forceinline__ int list_likely(const S &s, SampleShared &sm, const SampleShort &way, uint64_t *list, int ranks, int rank, float top, float c,
                                           float sum, float top_p, uint32_t *out) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float from = way.from;
    float mass = 0.f;
    s.each_vec(from, [&](const auto &z, int v) {
#pragma unroll
        for (int k = 0; k < S::N; ++k)
            if (z[k] >= from) {
                mass += ex2((z[k] - top) * c);
                const int at = atomicAdd(&sm.listed[0], 1);
                if (at < kSampleList) list[at] = sample_entry(z[k], v + k);
            }
    });
#pragma unroll
    for (int o = 16; o; o >>= 1) mass += __shfl_xor_sync(0xffffffffu, mass, o);
    if (lane == 0) sm.sums[warp] = mass;
    row_sync(ranks);
    mass = 0.f;
#pragma unroll
    for (int i = 0; i < kSampleSteps; ++i) {
        const int q = 32 / kSampleWarps * i + lane / kSampleWarps;
        if (q < ranks) mass += __uint_as_float(ld_cluster_u32(peer(&sm.sums[lane % kSampleWarps], q)));
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) mass += __shfl_xor_sync(0xffffffffu, mass, o);
    const int theirs = lane < ranks ? static_cast<int>(ld_cluster_u32(peer(&sm.listed[0], lane))) : 0;
    const int n = __reduce_add_sync(0xffffffffu, theirs), base = __reduce_add_sync(0xffffffffu, lane < rank ? theirs : 0);
    if (n > way.room || (way.by_sum && !way.whole && mass < (top_p + 0x1p-10f) * sum)) return -1;
    if (rank != 0) {
        const uint32_t to = peer(list, 0) + base * 8;
        for (int i = threadIdx.x; i < sm.listed[0]; i += kSampleThreads) st_cluster_u64(to + i * 8, list[i]);
    }
    if (out)
        for (int i = threadIdx.x; i < (s.row.V + 31) / 32; i += kSampleThreads) out[s.v0 / 32 + i] = 0;
    return n;
}

// Every token of a row that the list has room for, at its own place: those that are none sort behind the others.
template <typename S>
__device__ __forceinline__ void list_all(const S &s, uint64_t *list, uint32_t *out) {
    s.each([&](float z, int v) { list[v] = z >= kLowest ? sample_entry(z, v) : ~0ull; });
    if (out)
        for (int i = threadIdx.x; i < (s.row.V + 31) / 32; i += kSampleThreads) out[i] = 0;
}

// The token from a list of n: by the row's first CTA.  A sum of all weights that is only known to lie within `off` of `sum` decides
// as long as both ends do the same; false where they do not.
__device__ __forceinline__ bool solve_likely(SampleShared &sm, const SampleShort &way, uint64_t *list, int n, int V, uint64_t *upto, float edge, int top_k,
                                             float sum, float off, float top_p, float u, uint32_t *out) {
    const int listed = n;
    if (way.by_k) n = min(n, top_k);
    const int bits = way.by_sum ? units_of(fmaxf(sum, 1.f)) : list_units(n);  // (the sum of all has to fit too)
    if (threadIdx.x == 0) {
        sm.w.set_floor(bits);
        sm.w.big = kNoLogit;  // (few tokens: all of them in 64 bits)
    }
    sort_entries(list, way.all ? V : listed, 0);
    const uint64_t mine = add_up(list, n, upto, bits, sm);
    uint64_t low = ~0ull, high = ~0ull;
    if (top_p < 1.f) {
        const float unit = ldexpf(1.f, bits);
        low = high = times_fraction(mine, fmaxf(top_p, 0.f), true);
        if (way.by_sum) {
            low = times_fraction(__float2ull_rd(sum * (1.f - off) * unit), fmaxf(top_p, 0.f), true);
            high = times_fraction(__float2ull_ru(sum * (1.f + off) * unit), fmaxf(top_p, 0.f), true);
        }
    }
    const SampleHit end = find_entry(list, upto, n, 0, low, false, true, edge, sm);
    const bool below = end.at < n && key_value(~static_cast<uint32_t>(end.entry >> 32)) < edge;
    if (way.by_sum && !below && (end.at < n ? end.before < high : !way.whole)) return false;
    if (out)
        for (int i = threadIdx.x; i < end.at; i += kSampleThreads) {
            const int v = static_cast<int>(list[i] & 0xFFFFFFFFu);
            atomicOr(&out[v >> 5], 1u << (v & 31));
        }
    const SampleHit hit = find_entry(list, upto, end.at, 0, times_fraction(end.before, u, false), true, false, edge, sm);
    if (threadIdx.x == 0)
        sm.result = {0, {}, static_cast<int>(hit.entry & 0xFFFFFFFFu), end.at, quotient(hit.w, end.before)};
    __syncthreads();
    return true;
}

// ------------------------------------------------------------------------------ the kernel

__device__ __forceinline__ float clamp_temperature(float T) { return fminf(fmaxf(T, 1.45e-30f), 1.44e37f); }

template <typename T, bool kResident>
__global__ void __launch_bounds__(kSampleThreads, kSampleResident / kSampleThreads) k_sample_limits(const SampleParams p) {
    extern __shared__ __align__(16) uint8_t buffer[];
    __shared__ SampleShared sm;
    const int ranks = static_cast<int>(cluster_nctarank()), rank = ranks > 1 ? static_cast<int>(cluster_ctarank()) : 0;
    const long long r = blockIdx.x / ranks;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t *hist = reinterpret_cast<uint32_t *>(buffer + p.list_at);
    uint8_t *own = buffer + p.list_at + kSampleList * 8;  // this CTA's bins of the row: counts and sums
    static_assert(kSampleBins * 4 <= kSampleList * 8 && sizeof(SampleShared::Scratch) <= kSampleList * 8, "lists take their place");
    pdl_trigger();
    for (int i = threadIdx.x; i < kSampleTable; i += kSampleThreads) {
        sm.table.v[i] = g_sample_table.v[i];
        sm.table.rest[i] = g_sample_table.rest[i];
    }
    for (int i = threadIdx.x; i < kSampleBins / 4; i += kSampleThreads) reinterpret_cast<uint4 *>(hist)[i] = make_uint4(0, 0, 0, 0);
    if (threadIdx.x == 0) {
        sm.x = reinterpret_cast<SampleShared::Scratch *>(hist);
        sm.listed[0] = sm.listed[1] = 0;
        for (int i = 0; i < 5; ++i) sm.found[i] = {kSampleBins, 0, 0, 0.f, 0.f};
    }
    pdl_wait();
    const Slice<T, kResident> s(p, r, rank, buffer);
    // (+ 0: -0 becomes 0, whose bits times_fraction takes)
    const float T_row = p.a.temperature ? p.a.temperature[r] : 1.f, u = p.a.uniform ? p.a.uniform[r] + 0.f : 0.f;
    const float top_p = p.a.top_p ? p.a.top_p[r] + 0.f : 1.f, min_p = p.a.min_p ? p.a.min_p[r] : 0.f;
    const int top_k = p.a.top_k ? p.a.top_k[r] : 0;
    uint32_t *out = p.a.out_allowed ? reinterpret_cast<uint32_t *>(p.a.out_allowed) + r * p.words : nullptr;
    const float T_used = clamp_temperature(T_row), c = 1.44269502f / T_used;
    if (threadIdx.x == 0) sm.w.set_temperature(T_used);
    const bool weigh = T_row != 0.f && !(top_k > 0 && top_k <= kSampleList);
    const SampleRange<T> range = load_slice(s, weigh, c);
    const int warps = ranks * kSampleWarps;
    // so many tokens of every warp's threads, one of each, are not below the number that a warp hands on: the row has 32 or warps
    // times as many
    const int nth = top_k > 0 ? min(32, (top_k + warps - 1) / warps) : max(1, min(32, kSampleBins / ranks / 4 / warps));
    const float sorted = sort_warp(range.top);
    float top = range.top, low = range.low(), nth_top = __shfl_sync(0xffffffffu, sorted, nth - 1);
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
    }
    float sum = range.sum * ex2((range.top - top) * c);
    float likely = lane < nth ? ex2((sorted - top) * c) : 0.f;  // of tokens that are not below what the warp hands on
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        likely += __shfl_xor_sync(0xffffffffu, likely, o);
    }
    int finite = __reduce_add_sync(0xffffffffu, range.barred);  // those that are not, here
    if (lane == 0) {
        sm.range[0][warp] = top;
        sm.range[1][warp] = low;
        sm.range[2][warp] = sum;
        sm.range[3][warp] = nth_top;
        sm.range[4][warp] = likely;
        sm.finite[warp] = finite;
    }
    row_sync(ranks);
    // Under top-p eight CTAs hand on their warps' largest logits, of 128 warps: above the least of them are some 700 tokens (128 times 1 + 1/2 +
    // ... + 1/128), more than a list has room for then, and listing them in vain took a row of 126464 from 25 to 29 us.  Of the
    // largest of each lane's four the least has some 130 above it.
    const bool by_four = top_k <= 0 && ranks == kSampleMaxCluster;
    float tops[kSampleSteps], sums[kSampleSteps], likelies[kSampleSteps], nth_tops[kSampleSteps];
    top = kLowest;
    low = -kNoLogit;
    nth_top = by_four ? kNoLogit : -kNoLogit;
    finite = 0;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < kSampleSteps; ++i) {
        const int q = 32 / kSampleWarps * i + lane / kSampleWarps, w = lane % kSampleWarps;
        tops[i] = kLowest;
        sums[i] = likelies[i] = nth_tops[i] = 0.f;
        if (q < ranks) {
            likelies[i] = __uint_as_float(ld_cluster_u32(peer(&sm.range[4][w], q)));
            tops[i] = __uint_as_float(ld_cluster_u32(peer(&sm.range[0][w], q)));
            sums[i] = __uint_as_float(ld_cluster_u32(peer(&sm.range[2][w], q)));
            low = fminf(low, __uint_as_float(ld_cluster_u32(peer(&sm.range[1][w], q))));
            nth_tops[i] = __uint_as_float(ld_cluster_u32(peer(&sm.range[3][w], q)));
            nth_top = by_four ? fmaxf(nth_top, nth_tops[i]) : fminf(nth_top, nth_tops[i]);
            finite += static_cast<int>(ld_cluster_u32(peer(&sm.finite[w], q)));
        }
        top = fmaxf(top, tops[i]);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
        nth_top = fminf(nth_top, __shfl_xor_sync(0xffffffffu, nth_top, o));
    }
    likely = 0.f;
#pragma unroll
    for (int i = 0; i < kSampleSteps; ++i) {
        const float factor = ex2((tops[i] - top) * c);
        sum += sums[i] * factor;
        if (nth_tops[i] >= nth_top) likely += likelies[i] * factor;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        sum += __shfl_xor_sync(0xffffffffu, sum, o);
        likely += __shfl_xor_sync(0xffffffffu, likely, o);
    }
    finite = p.a.V - __reduce_add_sync(0xffffffffu, finite);
    if (low == kNoLogit && sum == sum) {  // of the allowed ones some may be -infinity
        int count = 0;
        s.each_vec(kLowest, [&](const auto &z, int) {
#pragma unroll
            for (int k = 0; k < Row<T>::kVec; ++k) count += z[k] >= kLowest;
        });
        finite = sum_of_row(sm, ranks, count);
    }
    const bool ok = fabsf(sum) < -kNoLogit && finite > 0 && T_row >= 0.f && (T_row == 0.f || (p.a.uniform && u >= 0.f && u < 1.f)) &&
                    top_p == top_p && min_p <= 1.f;
    bool done = false;  // the mask is written
    SampleCut cut{0xFFFFFFFFu, -1};  // nothing
    if (!ok) {
        if (threadIdx.x == 0) sm.result = {0, cut, -1, 0, 0.f};
    } else if (T_row == 0.f) {
        // the largest logit, and of several the first
        if (threadIdx.x == 0) sm.tie = 0x7FFFFFFF;
        row_sync(ranks);
        cut = {order_key(top), 0x7FFFFFFF};
        s.each_vec(top, [&](const auto &z, int v) {
#pragma unroll
            for (int k = 0; k < Row<T>::kVec; ++k)
                if (z[k] == top) atomicMin(&sm.tie, v + k);
        });
        row_sync(ranks);
        for (int q = 0; q < ranks; ++q) cut.last = min(cut.last, static_cast<int>(ld_cluster_u32(peer(&sm.tie, q))));
        if (threadIdx.x == 0) sm.result = {0, cut, cut.last, 1, 1.f};
    } else {
        const bool by_k = top_k > 0 && top_k < finite;
        if (threadIdx.x == 0) {
            sm.w.set_top(top);
            sm.edge = kNoLogit;
            if (min_p > 0.f) {
                // the first float from top + T ln min_p on
                const float2 log = scaled_log(T_used, min_p, &sm.table);
                const float near = __fadd_rn(top, log.x), part = __fsub_rn(near, top);
                const float rest = __fadd_rn(__fsub_rn(top, __fsub_rn(near, part)), __fsub_rn(log.x, part));  // what the sum has lost
                if (near > kNoLogit) sm.edge = __fadd_ru(near, __fadd_rn(rest, log.y));
            }
        }
        if (!weigh && !by_k) {  // a k that keeps all of few tokens
            float mine = 0.f;
            s.each([&](float z, int) { mine += ex2((z - top) * c); });
#pragma unroll
            for (int o = 16; o; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
            row_sync(ranks);
            if (lane == 0) sm.range[2][warp] = mine;
            row_sync(ranks);
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < kSampleSteps; ++i) {
                const int q = 32 / kSampleWarps * i + lane / kSampleWarps;
                if (q < ranks) sum += __uint_as_float(ld_cluster_u32(peer(&sm.range[2][lane % kSampleWarps], q)));
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        }
        if (by_k) sum = static_cast<float>(top_k);  // more than that it is not
        __syncthreads();
        const float edge = sm.edge;
        // Logits that no border can be at.  Top-k: the n-th largest of a warp's threads' largest, as above.  Top-p, or the draw
        // where there is no limit: what follows a border holds 1 - q of the sum in V tokens at most, and none of these weighs more
        // than the border's.  (2^-12 for the bins' error.)
        float least = kLowest;
        if (by_k) {
            if (top_k <= 32 * warps) least = nth_top;
        } else {
            const float q = top_p < 1.f ? fmaxf(top_p, 0.f) : u, rest = (1.f - q - 0x1p-12f) * sum / static_cast<float>(p.a.V);
            if (edge != kNoLogit && top_p >= 1.f)
                least = edge;
            else if (rest > 0.f)
                least = fmaxf(edge, top + __fdividef(log2f(rest) - 0x1p-6f, c));
        }
        SampleShort way{by_k, !by_k && top_p < 1.f, false, false, 0.f, kSampleList};
        way.from = way.by_k ? least : way.by_sum ? fmaxf(nth_top, edge) : edge;
        way.whole = !way.by_k && way.from == edge;
        if (way.by_sum) way.room = min(kSampleList, kSampleBins / ranks);  // (running sums lie where this CTA's bins would: the slice is needed if that fails)
        // (with top-p only where tokens that will be listed are known to hold it: listed in vain they cost a sixth)
        const bool few = way.by_k ? least > kLowest : way.from > kLowest && (!way.by_sum || way.whole || likely > top_p * sum);
        // Short rows are listed whole (one CTA has them): 136 rows of 300 tokens take 16.4 us so, 24.6 to 30.8 by the histogram; of 1000
        // 20.5 and 24.6 to 32.8; of 2000, as many as there is room for, 30.7 and 41.0 where top-k keeps most of them, else 26.6.
        way.all = !few && (p.a.V <= kSampleList / 2 || (by_k && p.a.V <= kSampleList && top_k >= p.a.V / 2));
        if (few || way.all) {
            uint64_t *list = reinterpret_cast<uint64_t *>(hist);
            int n = finite;
            if (way.all) {
                way.by_sum = false;
                list_all(s, list, out);
            } else {
                n = list_likely(s, sm, way, list, ranks, rank, top, c, sum, top_p, out);
            }
            if (n >= 0) {
                row_sync(ranks);  // (all have looked at the others' numbers, and the list is there)
                if (rank != 0 && !way.by_sum) return;
                // In units of 2^-24 of the sum: additions, one for every four of a thread's tokens; exponents of up to 40 octaves,
                // whose product with c is two roundings off (80); ex2, 4, and a dozen such factors where larger logits turn up (128).
                // Logits more than fp32's largest number below the top are taken for -infinity: where T is as large, they weigh up to
                // 2^-34 each.
                const float off = (static_cast<float>(p.slice / kSampleThreads / 4) + 256.f) * 0x1p-24f + (T_used < 0x1p118f ? 0.f : p.a.V * 0x1p-34f);
                if (rank == 0) {
                    done = solve_likely(sm, way, list, n, p.a.V, reinterpret_cast<uint64_t *>(way.by_sum ? own : buffer + p.upto_at), edge, top_k, sum, off,
                                        top_p, u, out);
                    if (threadIdx.x == 0) sm.first = done;
                }
                if (way.by_sum) {
                    row_sync(ranks);
                    done = ld_cluster_u32(peer(&sm.first, 0)) != 0;
                    if (ranks > 1) cluster_arrive();
                    if (done && rank != 0) return;
                    if (ranks > 1) cluster_wait();
                }
            }
            if (!done) {  // the histogram's place again
                row_sync(ranks);
                for (int i = threadIdx.x; i < kSampleBins / 4; i += kSampleThreads) reinterpret_cast<uint4 *>(hist)[i] = make_uint4(0, 0, 0, 0);
                if (threadIdx.x == 0) sm.listed[0] = 0;
                row_sync(ranks);
            }
        }
        if (done) {
        } else if (list_borders(s, sm, hist, own, ranks, rank, top, low, least, sum, finite, edge, by_k ? top_k : 0, top_p, u, out,
                         p.bits_at ? reinterpret_cast<uint32_t *>(buffer + p.bits_at) : nullptr)) {
            // the rest is the first CTA's; the others' shared memory is not read any more
            if (ranks > 1) {
                cluster_arrive();
                if (rank != 0) return;
                cluster_wait();
            } else {
                __syncthreads();
            }
            done = solve_lists(sm, reinterpret_cast<uint64_t *>(hist), reinterpret_cast<uint64_t *>(buffer + p.upto_at), ranks, finite, edge, top_k, top_p, u, out);
            if (!done) {
                SampleParams whole = p;
                whole.slice = p.words * 32;
                const Slice<T, false> row(whole, r, 0, buffer);
                sample_slowly(row, sm, 1, 0, top, edge, top_k, top_p, u);
                cut = sm.result.cut;
                if (out) write_bits(row, out, false, [&](float z, int v) { return z >= kLowest && cut.keeps(order_key(z), v); });
                done = true;
            }
        } else {
            sample_slowly(s, sm, ranks, rank, top, edge, top_k, top_p, u);
            cut = sm.result.cut;
        }
    }
    if (rank == 0 && threadIdx.x == 0) {
        const SampleResult res = sm.result;
        p.a.out_token[r] = res.token;
        p.a.out_status[r] = ok ? RPD_OK : RPD_ERR_INVALID_ARGUMENT;
        if (p.a.out_kept) p.a.out_kept[r] = res.kept;
        if (p.a.out_prob) p.a.out_prob[r] = res.prob;
    }
    if (done) return;
    if (out) write_bits(s, out, !ok, [&](float z, int v) { return z >= kLowest && cut.keeps(order_key(z), v); });
    if (ranks > 1) cluster_sync();  // shared memory is read by the others until here
}

constexpr int kSampleSmem = 200 * 1024;
constexpr int kSampleSlice = 80 * 1024;  // that stays in shared memory, two of them beside each other; a longer one is read again
constexpr int kSampleMask = 48 * 1024;   // of a slice's bits, at most

// CTAs of a row, two of which an SM holds: as many as run at once, but no slice shorter than some 8000 tokens.  One row of
// 126464 tokens with top-p: 15 to 17 us with eight, 22 with four, 36 with two; 7 rows of 50021: 22.8 with four, 23.0 with eight,
// 28.4 with two; one row of 4096: 9.7 with one, 10.7 with two, 14.3 with four; 128 rows of 126464 with top-k: 33.5 with two, 44.5
// with four, 45 with one; 528 rows of 152064 in fp32 with top-p: 313 with two, 330 with four, 528 with one.
int sample_ranks(long long rows, int V, int num_sms) {
    int ranks = rows * 8 <= 2 * num_sms ? 8 : rows * 4 <= 2 * num_sms ? 4 : 2;
    while (ranks > 1 && V < ranks * 8192) ranks >>= 1;
    return ranks;
}

template <typename T>
cudaError_t launch_sample(SampleParams p, int num_sms, cudaStream_t s) {
    const int ranks = sample_ranks(p.a.rows, p.a.V, num_sms);
    p.slice = (p.words + ranks - 1) / ranks * 32;
    const long long slice_bytes = (p.slice * static_cast<long long>(sizeof(T)) + 47) / 16 * 16;
    const int own_bytes = kSampleBins / ranks * 8;
    const bool resident = slice_bytes <= kSampleSlice;
    p.list_at = resident ? static_cast<int>(slice_bytes) : 0;
    // running sums lie where the slice was, or where this CTA's bins were
    p.upto_at = p.list_at >= kSampleList * 8 ? 0 : p.list_at + kSampleList * 8;
    p.bits_at = p.list_at + kSampleList * 8 + (p.upto_at ? std::max(own_bytes, kSampleList * 8) : own_bytes);
    long long bytes = p.bits_at;
    if (p.a.out_allowed && p.slice / 8 <= kSampleMask)
        bytes += p.slice / 8;
    else
        p.bits_at = 0;
    void (*kernel)(const SampleParams) = resident ? k_sample_limits<T, true> : k_sample_limits<T, false>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSampleSmem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.a.rows) * ranks);
    cfg.blockDim = dim3(kSampleThreads);
    cfg.dynamicSmemBytes = static_cast<size_t>(bytes);
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
    cudaStream_t s = static_cast<cudaStream_t>(stream_ptr);
    e = a.type == RPD_TYPE_F32    ? launch_sample<float>(p, num_sms, s)
        : a.type == RPD_TYPE_BF16 ? launch_sample<__nv_bfloat16>(p, num_sms, s)
                                  : launch_sample<__half>(p, num_sms, s);
    return e == cudaSuccess ? RPD_OK : op_cuda_fail(e, "sampling launch");
}
