// k_verify.cu - drafted tokens checked against a target model's probabilities, from given random
// numbers.
//
// A sequence has n drafted tokens x_0 .. x_{n-1} and n + 1 rows of target logits.  With
// p_i = softmax(z_i / T) over the allowed tokens and q_i = softmax of the draft model's row (or all of it at
// x_i where there is none), draft i is accepted while u_i q_i(x_i) < p_i(x_i).  At the first rejection j
// the next token is drawn from max(p_j - q_j, 0), after n acceptances from p_n: as the winner of a race,
// argmax_v w(v) / e(v) with given exponential variates e.  (A race, because its winner hangs on two
// numbers: the borders of a cumulative sum over 10^5 tokens lie closer than the roundings of any order of
// adding them up in fp32.)  T = 0 puts p_i at its largest logit.
//
// k_verify_rows reads every row of logits once and leaves its largest logit and the sum of the exponentials above it, a
// few slices of a row at a time: bound by HBM (528 rows of 152064 fp32 logits, 321 MB, in 51 us: 6.3 TB/s).
// k_verify_decide, a cluster of CTAs a sequence, joins the slices, finds j, and scans the one row (or two) that the
// next token is drawn from, most of which is still in L2, with the variates, which it has asked into L2 before: some 9
// us, of which 4 are a chain of waits (partial sums, verdicts, scan, join).  Statistics are fp32; differences z - m come
// before the multiplication by 1 / T (with bf16 and fp16 logits they are exact or nearly so).  Without drafts
// (k_sample) a cluster makes the statistics and runs the race in one pass: 128 rows of 126464 bf16 logits under a
// mask, with their variates 99 MB, in 21.1 us from HBM (4.7 TB/s; 18.4 where the same inputs come again and part of them is
// still in L2; as statistics and a second pass 45).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "logits_row.cuh"
#include "op_host.h"
#include "ptx.cuh"

namespace rpd {
namespace {

constexpr int kVerifyThreads = 256;
constexpr int kVerifyWarps = kVerifyThreads / 32;
constexpr int kDecideResident = 1024;  // threads an SM of the kernels that work in clusters
constexpr int kVerifyMaxCluster = 8;  // CTAs that scan one sequence's row, at most
constexpr int kVerifyMaxDrafts = 1024;
constexpr int kVerifyMaxSplits = 32;
constexpr long long kVerifyMaxRows = 1 << 26;  // a grid has as many CTAs: of so many rows none is divided (verify_splits)

struct VerifyParams {
    rpd_verify_args a;
    float4 *partials;  // [B][2 D + 1][splits]: largest logit, sum, lowest index of the largest logit
    int splits;
    int words;         // 32-bit words of a row of `allowed`
};

__device__ __forceinline__ float reciprocal(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// 1 / e of variates, right to a last place or two.  -0 is made 0 first: it is not negative (-log(1 - u) gives it where u
// is 0), so it wins, which its own reciprocal of -infinity would not.
__device__ __forceinline__ float inverse_variate(float e) { return reciprocal(e + 0.f); }
__device__ __forceinline__ void inverse_variates(float e0, float e1, float &r0, float &r1) {
    unpack2(add2(pack2(e0, e1), 0ull), r0, r1);
    r0 = reciprocal(r0);
    r1 = reciprocal(r1);
}

// 1 / T in units of log2, so that e^(x / T) = 2^(x c).  Within bounds where infinite logits give 0 and the
// largest one's 0 stays 0.
__device__ __forceinline__ float exponent_scale(float T) {
    return fminf(fmaxf(1.4426950408889634f / T, 1e-37f), 1e30f);
}

// A draft's own probability, of which there is one a row: exp2f goes down to fp32's smallest number (the terms' 2^x ends
// at 2^-126; p = 0 would reject a draft although u = 0).
__device__ __forceinline__ float probability(float z, float m, float c, float sum) { return exp2f((z - m) * c) / sum; }

// ------------------------------------------------------------------------------ statistics of the rows

// Running maximum and sum (in two halves, for the packed operations).  A sum that is not finite and positive marks a
// row without a distribution: a NaN or an infinite logit makes it NaN, and a row without any finite logit leaves
// it 0.
struct Stat {
    float m = kNoLogit;
    f32x2 s = 0;  // two zeros
    template <int N>
    __device__ __forceinline__ void add(const float (&z)[N], float c) {
        float top = m;
#pragma unroll
        for (int i = 0; i < N; ++i) top = fmaxf(top, z[i]);
        if (top == kNoLogit) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (z[i] != z[i]) s = pack2(z[i], z[i]);
            return;
        }
        if (top > m) {
            const float f = ex2((m - top) * c);
            s = mul2(s, pack2(f, f));
            m = top;
        }
        const f32x2 minus_m = pack2(-m, -m), c2 = pack2(c, c);
#pragma unroll
        for (int i = 0; i + 1 < N; i += 2) {
            float x, y;
            unpack2(mul2(add2(pack2(z[i], z[i + 1]), minus_m), c2), x, y);
            s = add2(s, pack2(ex2(x), ex2(y)));
        }
        if (N % 2) s = add2(s, pack2(ex2((z[N - 1] - m) * c), 0.f));
    }
    __device__ __forceinline__ float sum() const {
        float x, y;
        unpack2(s, x, y);
        return x + y;
    }
    __device__ __forceinline__ void join(float m2, float s2, float c) {
        const float top = fmaxf(m, m2);
        if (top == kNoLogit) {
            s = pack2(sum() + s2, 0.f);
        } else {
            s = pack2(sum() * ex2((m - top) * c) + s2 * ex2((m2 - top) * c), 0.f);
            m = top;
        }
    }
    __device__ __forceinline__ bool ok() const { return sum() > 0.f && sum() < -kNoLogit; }
};

// The largest logit and its lowest index.
struct Best {
    float m = kNoLogit;
    int at = 0x7FFFFFFF;
    bool bad = false;
    __device__ __forceinline__ void add(float z, int i) {
        bad |= z != z;
        if (z > m) {  // a thread's indices rise
            m = z;
            at = i;
        }
    }
    __device__ __forceinline__ void join(float m2, int at2) {
        if (m2 > m || (m2 == m && at2 < at)) {
            m = m2;
            at = at2;
        }
    }
};

// Calls f(z, first index) for the thread's vectors of slice `split` of a row, with the tokens that are
// not allowed at -infinity, and g(z, index) for the elements that no vector holds.
template <typename T, bool kMask, int kThreads, typename F, typename G>
__device__ __forceinline__ void walk_slice(const Row<T> &row, const uint32_t *mask, int words, int split, int splits,
                                           const F &f, const G &g) {
    constexpr int N = Row<T>::kVec;
    constexpr int kUnroll = 4;
    const int v0 = static_cast<int>(static_cast<long long>(row.vecs) * split / splits);
    const int v1 = static_cast<int>(static_cast<long long>(row.vecs) * (split + 1) / splits);
    const uint4 *body = reinterpret_cast<const uint4 *>(row.p + row.peel);
    for (int v = v0 + threadIdx.x; v < v1; v += kThreads * kUnroll) {
        uint4 raw[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (v + u * kThreads < v1) raw[u] = body[v + u * kThreads];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int at = v + u * kThreads;
            if (at < v1) {
                float z[N];
                unpack(raw[u], z, T());
                const int first = row.peel + at * N;
                if (kMask) {
                    const uint32_t bits = allowed_bits(mask, first, words);
#pragma unroll
                    for (int i = 0; i < N; ++i) z[i] = (bits >> i) & 1u ? z[i] : kNoLogit;
                }
                f(z, first);
            }
        }
    }
    // the first slice has the elements before the vectors, the last one those behind
    const int loose = (split == 0 ? row.peel : 0);
    const int behind = row.peel + row.vecs * N;
    const int count = loose + (split == splits - 1 ? row.V - behind : 0);
    if (static_cast<int>(threadIdx.x) < count) {
        const int i = static_cast<int>(threadIdx.x) < loose ? threadIdx.x : behind + threadIdx.x - loose;
        float z = value(row.p[i]);
        if (kMask && !((mask[i >> 5] >> (i & 31)) & 1u)) z = kNoLogit;
        g(z, i);
    }
}

__device__ __forceinline__ int draft_count(const rpd_verify_args &a, int b) {
    return a.lengths ? a.lengths[b] : a.D;
}

__device__ __forceinline__ float temperature_of(const rpd_verify_args &a, int b) {
    return a.temperature ? a.temperature[b] : 1.f;
}

__device__ __forceinline__ long long target_offset(const rpd_verify_args &a, int b, int i) {
    return b * a.target_seq_stride + i * a.target_row_stride;
}
__device__ __forceinline__ long long draft_offset(const rpd_verify_args &a, int b, int i) {
    return b * a.draft_seq_stride + i * a.draft_row_stride;
}
__device__ __forceinline__ const uint32_t *mask_row(const rpd_verify_args &a, int words, int b, int i) {
    return a.allowed + (static_cast<long long>(b) * (a.D + 1) + i) * words;
}

// A slice of a row: rows 0..D are the target's, D + 1 .. 2 D the draft model's.
template <typename T, bool kMask, int kWarps>
__device__ __forceinline__ void row_slice(const rpd_verify_args &a, const VerifyParams &p, int b, int i, int split, int splits,
                                          const void *base, long long offset, float temperature, float4 *out) {
    const Row<T> row(base, offset, a.V);
    const uint32_t *mask = kMask ? mask_row(a, p.words, b, i) : nullptr;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __shared__ float4 part[kWarps];
    if (temperature > 0.f) {
        const float c = exponent_scale(temperature);
        Stat st;
        walk_slice<T, kMask, kWarps * 32>(
            row, mask, p.words, split, splits, [&](const auto &z, int) { st.add(z, c); },
            [&](float z, int) {
                const float one[1] = {z};
                st.add(one, c);
            });
#pragma unroll
        for (int o = 16; o; o >>= 1)
            st.join(__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.sum(), o), c);
        if (lane == 0) part[warp] = make_float4(st.m, st.sum(), 0.f, 0.f);
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kWarps; ++w) st.join(part[w].x, part[w].y, c);
            *out = make_float4(st.m, st.sum(), 0.f, 0.f);
        }
    } else {
        Best best;
        walk_slice<T, kMask, kWarps * 32>(
            row, mask, p.words, split, splits,
            [&](const auto &z, int first) {
#pragma unroll
                for (int k = 0; k < Row<T>::kVec; ++k) best.add(z[k], first + k);
            },
            [&](float z, int at) { best.join(z, at); best.bad |= z != z; });
        best.bad = __any_sync(0xffffffffu, best.bad);
#pragma unroll
        for (int o = 16; o; o >>= 1)
            best.join(__shfl_xor_sync(0xffffffffu, best.m, o), __shfl_xor_sync(0xffffffffu, best.at, o));
        if (lane == 0) part[warp] = make_float4(best.m, best.bad ? 1.f : 0.f, __int_as_float(best.at), 0.f);
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kWarps; ++w) {
                best.join(part[w].x, __float_as_int(part[w].z));
                best.bad |= part[w].y != 0.f;
            }
            *out = make_float4(best.m, best.bad ? 1.f : 0.f, __int_as_float(best.at), 0.f);
        }
    }
}

template <typename T, bool kMask>
__global__ void __launch_bounds__(kVerifyThreads) k_verify_rows(const VerifyParams p) {
    const rpd_verify_args &a = p.a;
    const int kinds = a.draft ? 2 * a.D + 1 : a.D + 1;
    const int split = blockIdx.x % p.splits, r = blockIdx.x / p.splits % kinds, b = blockIdx.x / p.splits / kinds;
    const bool is_draft = r > a.D;
    const int i = is_draft ? r - a.D - 1 : r;
    pdl_wait();
    pdl_trigger();  // not before: k_verify_decide reads the call's inputs ahead of its own wait
    const int n = draft_count(a, b);
    const float temperature = temperature_of(a, b);
    // rows behind a sequence's last one are never read, nor a draft model's where the choice is greedy
    if (n < 0 || n > a.D || !(temperature >= 0.f) || (is_draft ? i >= n || temperature == 0.f : i > n)) return;
    float4 *out = p.partials + (static_cast<long long>(b) * (2 * a.D + 1) + r) * p.splits + split;
    if (is_draft)
        row_slice<T, false, kVerifyWarps>(a, p, b, i, split, p.splits, a.draft, draft_offset(a, b, i), temperature, out);
    else
        row_slice<T, kMask, kVerifyWarps>(a, p, b, i, split, p.splits, a.target, target_offset(a, b, i), temperature, out);
}

// ------------------------------------------------------------------------------ decision

// The race's leader: the largest w / e so far, the lowest index on a tie.  Quotients are w times the reciprocal
// (both right to a last place or two): a variate of 0 wins against any other, one that is negative or no number,
// and a weight that is not positive, never.
struct Race {
    float best = 0.f;
    int at = 0x7FFFFFFF;
    __device__ __forceinline__ void add(float score, int i) {  // a thread's indices rise
        if (score > best) {
            best = score;
            at = i;
        }
    }
    template <int N>
    __device__ __forceinline__ void add(const float (&score)[N], int first) {
        float top = score[0];
#pragma unroll
        for (int k = 1; k < N; ++k) top = fmaxf(top, score[k]);
        if (top > best) {
#pragma unroll
            for (int k = 0; k < N; ++k) add(score[k], first + k);
        }
    }
    __device__ __forceinline__ void join(float score, int i) {
        if (score > best || (score == best && i < at)) {
            best = score;
            at = i;
        }
    }
    __device__ __forceinline__ void join_warp() {
#pragma unroll
        for (int o = 16; o; o >>= 1)
            join(__shfl_xor_sync(0xffffffffu, best, o), __shfl_xor_sync(0xffffffffu, at, o));
    }
};

// Shared memory: for rows 0..D of the target largest logit, sum and argmax, for those of the draft model largest
// logit and sum; for every draft its logit in both.
struct DecideRows {
    float *tm, *ts, *dm, *ds, *zx, *zq;
    int *arg;
};
constexpr int kDecideRowBytes = 28;

// The CTA's part of a row of variates on its way to L2, while the statistics are still being made.
__device__ __forceinline__ void prefetch_slice(const float *row, int V, int split, int splits) {
    const uintptr_t first = (reinterpret_cast<uintptr_t>(row + static_cast<long long>(V) * split / splits) + 15) & ~uintptr_t(15);
    const uintptr_t last = reinterpret_cast<uintptr_t>(row + static_cast<long long>(V) * (split + 1) / splits) & ~uintptr_t(15);
    if (last > first)
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(first), "r"(static_cast<uint32_t>(last - first))
                     : "memory");
}

__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}

// What the race is run over: p (all drafts accepted), p without the rejected token, or max(p - q, 0).
enum Residual { kAll, kOthers, kExcess };

// The row that the next token is drawn from, at the place in it where a vector begins.
template <typename T>
struct Contest {
    const T *p, *q;
    const float *noise;
    const uint32_t *mask;
    int words, V, rejected;             // rejected: the token, for kOthers
    float c, tm, t_inv, dm, d_inv;      // exponent scale; largest logits and 1 / sums
    __device__ __forceinline__ float weight(float z) const { return ex2((z - tm) * c); }  // p times the sum
    __device__ __forceinline__ float other(float z) const { return ex2((z - dm) * c) * d_inv; }
};

// A token's score in the race (r: 1 / its variate) and, for kExcess, in the one over p itself (should no excess be
// positive: p = q but for roundings).  An excess below 0 is none: with its sign, and that of a negative variate, it
// would win.
template <int kKind, typename T>
__device__ __forceinline__ void contend(const Contest<T> &s, float z, float zq, float r, int at, float &score, float &plain) {
    const float w = s.weight(z);
    score = (kKind == kExcess ? fmaxf(fmaf(w, s.t_inv, -s.other(zq)), 0.f) : w) * r;
    if (kKind == kOthers && at == s.rejected) score = 0.f;
    if (kKind == kExcess) plain = w * r;
}

// This CTA's slice of the race.  Where variates and draft logits have the target's alignment, they are read in vectors
// too; otherwise a thread takes single tokens, neighbours side by side.
template <int kKind, bool kMask, int kThreads, typename T>
__device__ __forceinline__ void run_race(const Contest<T> &s, int split, int splits, Race &race, Race &plain) {
    constexpr int N = Row<T>::kVec, kUnroll = N == 4 ? 4 : 2;
    const Row<T> row(s.p, 0, s.V);
    const bool vectors = (reinterpret_cast<uintptr_t>(s.noise + row.peel) & 15) == 0 &&
                         (kKind != kExcess || (reinterpret_cast<uintptr_t>(s.q + row.peel) & 15) == 0);
    if (!vectors) {
        const int i0 = static_cast<int>(static_cast<long long>(s.V) * split / splits);
        const int i1 = static_cast<int>(static_cast<long long>(s.V) * (split + 1) / splits);
#pragma unroll 4
        for (int i = i0 + threadIdx.x; i < i1; i += kThreads) {
            float z = value(s.p[i]);
            if (kMask && !((s.mask[i >> 5] >> (i & 31)) & 1u)) z = kNoLogit;
            float score, other = 0.f;
            contend<kKind>(s, z, kKind == kExcess ? value(s.q[i]) : 0.f, inverse_variate(s.noise[i]), i, score, other);
            race.add(score, i);
            if (kKind == kExcess) plain.add(other, i);
        }
        return;
    }
    const int v0 = static_cast<int>(static_cast<long long>(row.vecs) * split / splits);
    const int v1 = static_cast<int>(static_cast<long long>(row.vecs) * (split + 1) / splits);
    const uint4 *pv = reinterpret_cast<const uint4 *>(s.p + row.peel);
    const uint4 *qv = reinterpret_cast<const uint4 *>(s.q + row.peel);
    const float4 *ev = reinterpret_cast<const float4 *>(s.noise + row.peel);
    for (int v = v0 + threadIdx.x; v < v1; v += kThreads * kUnroll) {
        uint4 raw[kUnroll], raw_q[kUnroll];
        float4 e[kUnroll][N / 4];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int at = min(v + u * kThreads, v1 - 1);
            raw[u] = pv[at];
            if (kKind == kExcess) raw_q[u] = qv[at];
#pragma unroll
            for (int k = 0; k < N / 4; ++k) e[u][k] = ev[at * (N / 4) + k];
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (v + u * kThreads < v1) {
                const int first = row.peel + (v + u * kThreads) * N;
                float z[N], zq[N];
                unpack(raw[u], z, T());
                if (kKind == kExcess) unpack(raw_q[u], zq, T());
                const uint32_t bits = kMask ? allowed_bits(s.mask, first, s.words) : 0u;
                float score[N], other[N], r[N];
#pragma unroll
                for (int k = 0; k < N / 4; ++k) {
                    inverse_variates(e[u][k].x, e[u][k].y, r[4 * k], r[4 * k + 1]);
                    inverse_variates(e[u][k].z, e[u][k].w, r[4 * k + 2], r[4 * k + 3]);
                }
#pragma unroll
                for (int k = 0; k < N; ++k)
                    contend<kKind>(s, kMask && !((bits >> k) & 1u) ? kNoLogit : z[k], kKind == kExcess ? zq[k] : 0.f, r[k],
                                   first + k, score[k], other[k]);
                race.add(score, first);
                if (kKind == kExcess) plain.add(other, first);
            }
        }
    }
    const int loose = split == 0 ? row.peel : 0, behind = row.peel + row.vecs * N;
    const int count = loose + (split == splits - 1 ? s.V - behind : 0);
    if (static_cast<int>(threadIdx.x) < count) {
        const int i = static_cast<int>(threadIdx.x) < loose ? threadIdx.x : behind + threadIdx.x - loose;
        float z = value(s.p[i]);
        if (kMask && !((s.mask[i >> 5] >> (i & 31)) & 1u)) z = kNoLogit;
        float score, other = 0.f;
        contend<kKind>(s, z, kKind == kExcess ? value(s.q[i]) : 0.f, inverse_variate(s.noise[i]), i, score, other);
        race.join(score, i);
        if (kKind == kExcess) plain.join(other, i);
    }
}

// ------------------------------------------------------------------------------ nothing drafted

// The row and its variates, for a score that has to be made anew.
template <typename T>
struct DrawRow {
    const T *p;
    const float *noise;
    float c;
    __device__ __forceinline__ float score(int at, float m) const {
        const float r = inverse_variate(noise[at]);
        return r < -kNoLogit ? ex2((value(p[at]) - m) * c) * r : r;
    }
};

// Statistics of a slice and the race over it in one pass, both relative to the running maximum.  A leader's score that has
// been multiplied on depends, in its last places, on the maxima that it has met; where another comes within 2^-10 of
// it, it is made anew from its logit and variate, so that of equal tokens the first one wins.  (To keep both with
// every leader made 128 rows 1 us slower.)
constexpr float kDrawNear = 0x1p-10f;

struct Draw {
    Stat st;
    Race race;
    template <int N, typename T>
    __device__ __forceinline__ void add(const float (&z)[N], const float (&e)[N], int first, const DrawRow<T> &row,
                                        int step = 1) {
        const float c = row.c;
        float top = st.m;
#pragma unroll
        for (int i = 0; i < N; ++i) top = fmaxf(top, z[i]);
        if (top > st.m) {
            const float f = ex2((st.m - top) * c);
            st.s = mul2(st.s, pack2(f, f));
            race.best = f > 0.f ? race.best * f : 0.f;
            st.m = top;
        }
        if (top == kNoLogit) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (z[i] != z[i]) st.s = pack2(z[i], z[i]);
            return;
        }
        const f32x2 minus_m = pack2(-st.m, -st.m), c2 = pack2(c, c);
        float score[N];
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            float x, y;
            unpack2(mul2(add2(pack2(z[i], i + 1 < N ? z[(i + 1) % N] : kNoLogit), minus_m), c2), x, y);
            x = ex2(x);
            y = ex2(y);
            st.s = add2(st.s, pack2(x, y));
            if (i + 1 < N) {
                float r0, r1;
                inverse_variates(e[i], e[(i + 1) % N], r0, r1);
                score[i] = x * r0;
                score[(i + 1) % N] = y * r1;
            } else {
                score[i] = x * inverse_variate(e[i]);
            }
        }
        float best = score[0];
#pragma unroll
        for (int i = 1; i < N; ++i) best = fmaxf(best, score[i]);
        if (best > race.best * (1.f - kDrawNear)) {
            if (best < race.best * (1.f + kDrawNear)) race.best = row.score(race.at, st.m);
#pragma unroll
            for (int i = 0; i < N; ++i) race.add(score[i], first + i * step);
        }
    }
    // Of all lanes of a warp, for all of them.
    template <typename T>
    __device__ __forceinline__ void join_warp(const DrawRow<T> &row) {
        float top = st.m, sum = st.sum();
#pragma unroll
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float f = top > kNoLogit ? ex2((st.m - top) * row.c) : 1.f;
        sum *= f;
        race.best = f > 0.f ? race.best * f : 0.f;
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        float most = most_of_warp(race.best);
        const bool near = race.best > 0.f && race.best >= most * (1.f - kDrawNear);
        if (__popc(__ballot_sync(0xffffffffu, near)) > 1) {
            if (near) race.best = row.score(race.at, top);
            most = most_of_warp(race.best);
        }
        race.at = __reduce_min_sync(0xffffffffu, race.best == most ? race.at : 0x7FFFFFFF);
        race.best = most;
        st.m = top;
        st.s = pack2(sum, 0.f);
    }
    static __device__ __forceinline__ float most_of_warp(float score) {  // scores are at least 0: ordered as their bits are
        return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(score)));
    }
    __device__ __forceinline__ float4 part() const { return make_float4(st.m, st.sum(), race.best, __int_as_float(race.at)); }
    __device__ __forceinline__ void set(const float4 &part) {
        st.m = part.x;
        st.s = pack2(part.y, 0.f);
        race.best = part.z;
        race.at = __float_as_int(part.w);
    }
};

template <typename T, bool kMask, int kThreads>
__device__ __forceinline__ void draw_slice(const DrawRow<T> &source, const uint32_t *mask, int words, int V, int split,
                                           int splits, Draw &draw) {
    const T *p = source.p;
    const float *noise = source.noise;
    constexpr int N = Row<T>::kVec, kUnroll = N == 4 ? 4 : 2;
    // single tokens that a thread asks for at a time, and the next ones before it scores these (39 rows of 136321 with a
    // stride that the variates do not have, from HBM: 14.1 us, the next ones only then 16.3)
    constexpr int kBatch = 8;
    const Row<T> row(p, 0, V);
    if (reinterpret_cast<uintptr_t>(noise + row.peel) & 15) {  // single tokens, neighbours side by side
        const int i0 = static_cast<int>(static_cast<long long>(V) * split / splits);
        const int i1 = static_cast<int>(static_cast<long long>(V) * (split + 1) / splits);
        float z[kBatch], e[kBatch], z_next[kBatch], e_next[kBatch];
        auto load = [&](int i, float (&zs)[kBatch], float (&es)[kBatch]) {
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int at = i + k * kThreads, from = min(at, i1 - 1);
                zs[k] = value(p[from]);
                es[k] = noise[from];
                if (at >= i1 || (kMask && !((mask[from >> 5] >> (from & 31)) & 1u))) zs[k] = kNoLogit;
            }
        };
        int i = i0 + threadIdx.x;
        if (i < i1) load(i, z, e);
        for (; i < i1; i += kThreads * kBatch) {
            if (i + kThreads * kBatch < i1) load(i + kThreads * kBatch, z_next, e_next);
            draw.add(z, e, i, source, kThreads);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                z[k] = z_next[k];
                e[k] = e_next[k];
            }
        }
        return;
    }
    const int v0 = static_cast<int>(static_cast<long long>(row.vecs) * split / splits);
    const int v1 = static_cast<int>(static_cast<long long>(row.vecs) * (split + 1) / splits);
    const int loose = split == 0 ? row.peel : 0, behind = row.peel + row.vecs * N;
    const int count = loose + (split == splits - 1 ? V - behind : 0);
    if (static_cast<int>(threadIdx.x) < loose) {  // (a thread's indices rise)
        const int i = threadIdx.x;
        const float z[1] = {kMask && !((mask[i >> 5] >> (i & 31)) & 1u) ? kNoLogit : value(p[i])}, e[1] = {noise[i]};
        draw.add(z, e, i, source);
    }
    const uint4 *pv = reinterpret_cast<const uint4 *>(p + row.peel);
    const float4 *ev = reinterpret_cast<const float4 *>(noise + row.peel);
    for (int v = v0 + threadIdx.x; v < v1; v += kThreads * kUnroll) {
        uint4 raw[kUnroll];
        float4 f[kUnroll][N / 4];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int at = min(v + u * kThreads, v1 - 1);
            raw[u] = pv[at];
#pragma unroll
            for (int k = 0; k < N / 4; ++k) f[u][k] = ev[at * (N / 4) + k];
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (v + u * kThreads < v1) {
                const int first = row.peel + (v + u * kThreads) * N;
                float z[N], e[N];
                unpack(raw[u], z, T());
                const uint32_t bits = kMask ? allowed_bits(mask, first, words) : 0u;
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    if (kMask) z[k] = (bits >> k) & 1u ? z[k] : kNoLogit;
                    const float4 &g = f[u][k / 4];
                    e[k] = k % 4 == 0 ? g.x : k % 4 == 1 ? g.y : k % 4 == 2 ? g.z : g.w;
                }
                draw.add(z, e, first, source);
            }
        }
    }
    if (static_cast<int>(threadIdx.x) >= loose && static_cast<int>(threadIdx.x) < count) {
        const int i = behind + threadIdx.x - loose;
        const float z[1] = {kMask && !((mask[i >> 5] >> (i & 31)) & 1u) ? kNoLogit : value(p[i])}, e[1] = {noise[i]};
        draw.add(z, e, i, source);
    }
}

// One cluster a sequence draws from its only row: every CTA a slice, joined in the first one.
template <typename T, bool kMask, int kThreads>
__global__ void __launch_bounds__(kThreads, kDecideResident / kThreads) k_sample(const VerifyParams p) {
    const rpd_verify_args &a = p.a;
    __shared__ float4 warp_part[kThreads / 32];
    __shared__ float4 cta_part[kVerifyMaxCluster];  // of the whole cluster, in its first CTA
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int ranks = static_cast<int>(cluster_size()), b = blockIdx.x / ranks;
    const int rank = static_cast<int>(cluster_ctarank());
    pdl_trigger();
    cluster_sync();  // every CTA of the cluster runs: their shared memory may be written
    pdl_wait();
    const int n = draft_count(a, b);
    const float temperature = temperature_of(a, b);
    const bool greedy = temperature == 0.f, usable = n == 0 && temperature >= 0.f && (greedy || a.noise);
    const float c = greedy ? 1.f : exponent_scale(temperature);
    const DrawRow<T> row{static_cast<const T *>(a.target) + target_offset(a, b, 0), a.noise + b * a.noise_stride, c};
    if (usable) {
        if (greedy) {
            row_slice<T, kMask, kThreads / 32>(a, p, b, 0, rank, ranks, a.target, target_offset(a, b, 0), 0.f, warp_part);
        } else {
            Draw draw;
            draw_slice<T, kMask, kThreads>(row, kMask ? mask_row(a, p.words, b, 0) : nullptr, p.words, a.V, rank, ranks, draw);
            draw.join_warp(row);
            if (lane == 0) warp_part[warp] = draw.part();
            __syncthreads();
            if (warp == 0) {
                draw = Draw();
                if (lane < kThreads / 32) draw.set(warp_part[lane]);
                draw.join_warp(row);
                if (lane == 0) warp_part[0] = draw.part();
            }
        }
        if (threadIdx.x == 0) {
            const uint32_t to = mapa_shared(smem_u32(&cta_part[rank]), 0);
            st_shared_cluster(to, __float_as_int(warp_part[0].x));
            st_shared_cluster(to + 4, __float_as_int(warp_part[0].y));
            st_shared_cluster(to + 8, __float_as_int(warp_part[0].z));
            st_shared_cluster(to + 12, __float_as_int(warp_part[0].w));
        }
    }
    cluster_sync();
    if (rank != 0 || warp != 0) return;
    int next = -1;
    if (usable && greedy) {
        Best best;
        bool nan = false;
        for (int r = 0; r < ranks; ++r) {
            best.join(cta_part[r].x, __float_as_int(cta_part[r].z));
            nan = nan || cta_part[r].y != 0.f;
        }
        if (!nan && best.m > kNoLogit && best.m < -kNoLogit) next = best.at;
    } else if (usable) {
        Draw draw;
        if (lane < ranks) draw.set(cta_part[lane]);
        draw.join_warp(row);
        if (draw.st.ok() && draw.race.best > 0.f) next = draw.race.at;
    }
    if (lane != 0) return;
    a.out_accepted[b] = 0;
    a.out_token[b] = next;
    a.out_status[b] = next < 0 ? RPD_ERR_INVALID_ARGUMENT : RPD_OK;
}

template <typename T, bool kMask, int kThreads>
__global__ void __launch_bounds__(kThreads, kDecideResident / kThreads) k_verify_decide(const VerifyParams p) {
    const rpd_verify_args &a = p.a;
    extern __shared__ float rows_smem[];
    __shared__ int first_stop;
    __shared__ Race warp_race[2][kThreads / 32];
    __shared__ Race cta_race[2][kVerifyMaxCluster];  // of the whole cluster, in its first CTA
    const int rows = a.D + 1;
    const DecideRows s{rows_smem,            rows_smem + rows,     rows_smem + 2 * rows, rows_smem + 3 * rows,
                       rows_smem + 4 * rows, rows_smem + 5 * rows, reinterpret_cast<int *>(rows_smem + 6 * rows)};
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int ranks = static_cast<int>(cluster_size()), b = blockIdx.x / ranks;
    const int rank = static_cast<int>(cluster_ctarank());
    pdl_trigger();
    // The rows kernel has seen its predecessors done before this one could start: the inputs may be read while it runs.
    const int n = draft_count(a, b);
    const float T_seq = temperature_of(a, b);
    const bool greedy = T_seq == 0.f;
    const bool usable = n >= 0 && n <= a.D && T_seq >= 0.f && (greedy || (a.noise && (n == 0 || a.uniform)));
    const float c = greedy ? 1.f : exponent_scale(T_seq);
    const bool drafts = a.draft && !greedy;
    const int32_t *tokens = a.tokens + static_cast<long long>(b) * a.D;
    if (threadIdx.x == 0) first_stop = usable ? n : 0;
    if (threadIdx.x == 32 && usable && !greedy) prefetch_slice(a.noise + b * a.noise_stride, a.V, rank, ranks);
    if (usable)
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const int x = tokens[i];
            const bool in = x >= 0 && x < a.V;
            float zx = kNoLogit, zq = kNoLogit;
            if (in && (!kMask || ((mask_row(a, p.words, b, i)[x >> 5] >> (x & 31)) & 1u)))
                zx = value(static_cast<const T *>(a.target)[target_offset(a, b, i) + x]);
            if (in && drafts) zq = value(static_cast<const T *>(a.draft)[draft_offset(a, b, i) + x]);
            s.zx[i] = zx;
            s.zq[i] = zq;
        }
    cluster_sync();  // every CTA of the cluster runs: their shared memory may be written
    pdl_wait();
    int stop = 0, next = -1;
    bool bad = true;
    if (usable) {
        // the slices of every row joined, a warp a row
        const float4 *partials = p.partials + static_cast<long long>(b) * (2 * a.D + 1) * p.splits;
        const int count = n + 1 + (drafts ? n : 0);
        for (int k = warp; k < count; k += kThreads / 32) {
            const int r = k <= n ? k : a.D + 1 + (k - n - 1);
            const float4 v = lane < p.splits ? partials[static_cast<long long>(r) * p.splits + lane]
                                             : make_float4(kNoLogit, 0.f, __int_as_float(0x7FFFFFFF), 0.f);
            if (greedy) {
                Best best;
                best.m = v.x;
                best.at = __float_as_int(v.z);
                const bool nan = __any_sync(0xffffffffu, v.y != 0.f);
#pragma unroll
                for (int o = 16; o; o >>= 1)
                    best.join(__shfl_xor_sync(0xffffffffu, best.m, o), __shfl_xor_sync(0xffffffffu, best.at, o));
                if (lane == 0) {
                    s.tm[k] = best.m;
                    s.ts[k] = !nan && best.m > kNoLogit && best.m < -kNoLogit ? 1.f : 0.f;
                    s.arg[k] = best.at;
                }
            } else {
                Stat st;
                st.m = v.x;
                st.s = pack2(v.y, 0.f);
#pragma unroll
                for (int o = 16; o; o >>= 1)
                    st.join(__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.sum(), o), c);
                if (lane == 0) {
                    (k <= n ? s.tm[k] : s.dm[k - n - 1]) = st.m;
                    (k <= n ? s.ts[k] : s.ds[k - n - 1]) = st.ok() ? st.sum() : 0.f;
                }
            }
        }
        __syncthreads();
        // every draft's verdict; the first rejection counts
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const int x = tokens[i];
            bool sound = s.ts[i] > 0.f;
            const float px = !sound ? 0.f : greedy ? (x == s.arg[i] ? 1.f : 0.f) : probability(s.zx[i], s.tm[i], c, s.ts[i]);
            float qx = 1.f;
            if (drafts) {
                sound = sound && s.ds[i] > 0.f;
                qx = sound ? probability(s.zq[i], s.dm[i], c, s.ds[i]) : 0.f;
            }
            const bool accept =
                sound && (greedy ? px > 0.f : a.uniform[static_cast<long long>(b) * a.D + i] * qx < px);
            if (!accept) atomicMin(&first_stop, i);
            if (rank == 0 && a.out_prob) a.out_prob[static_cast<long long>(b) * a.D + i] = px;
        }
        __syncthreads();
        stop = first_stop;
        const bool rejected = stop < n;
        bad = !(s.ts[stop] > 0.f) || (rejected && drafts && !(s.ds[stop] > 0.f));
        if (!bad && greedy) {
            next = s.arg[stop];
        } else if (!bad) {
            Race race, plain;
            const Contest<T> contest{static_cast<const T *>(a.target) + target_offset(a, b, stop),
                                     rejected && drafts ? static_cast<const T *>(a.draft) + draft_offset(a, b, stop) : nullptr,
                                     a.noise + b * a.noise_stride, kMask ? mask_row(a, p.words, b, stop) : nullptr, p.words, a.V,
                                     rejected ? tokens[stop] : -1, c, s.tm[stop],
                                     1.f / s.ts[stop], rejected && drafts ? s.dm[stop] : 0.f,
                                     rejected && drafts ? 1.f / s.ds[stop] : 0.f};
            if (!rejected)
                run_race<kAll, kMask, kThreads>(contest, rank, ranks, race, plain);
            else if (drafts)
                run_race<kExcess, kMask, kThreads>(contest, rank, ranks, race, plain);
            else
                run_race<kOthers, kMask, kThreads>(contest, rank, ranks, race, plain);
            race.join_warp();
            plain.join_warp();
            if (lane == 0) {
                warp_race[0][warp] = race;
                warp_race[1][warp] = plain;
            }
            __syncthreads();
            if (threadIdx.x < 2) {
                Race r = warp_race[threadIdx.x][0];
                for (int w = 1; w < kThreads / 32; ++w) {
                    const Race &o = warp_race[threadIdx.x][w];
                    r.join(o.best, o.at);
                }
                const uint32_t to = mapa_shared(smem_u32(&cta_race[threadIdx.x][rank]), 0);
                st_shared_cluster(to, __float_as_int(r.best));
                st_shared_cluster(to + 4, r.at);
            }
        }
    }
    cluster_sync();
    if (rank != 0) return;
    if (usable && !bad && !greedy) {
        Race r;
        for (int kind = 0; kind < 2 && r.best == 0.f; ++kind)
            for (int k = 0; k < ranks; ++k) r.join(cta_race[kind][k].best, cta_race[kind][k].at);
        next = r.best > 0.f ? r.at : -1;
        bad = next < 0;
    }
    for (int i = threadIdx.x; i <= a.D; i += kThreads) {
        const long long row = static_cast<long long>(b) * (a.D + 1);
        a.out_token[row + i] = i < stop ? tokens[i] : i == stop ? next : -1;
        if (a.out_prob && i < a.D && i >= (usable ? n : 0)) a.out_prob[static_cast<long long>(b) * a.D + i] = 0.f;
    }
    if (threadIdx.x == 0) {
        a.out_accepted[b] = stop;
        a.out_status[b] = bad ? RPD_ERR_INVALID_ARGUMENT : RPD_OK;
    }
}

// Slices of a row: eight CTAs an SM, none with less than a vector a thread.  (64 sequences of up to five drafts: 30.1 us
// with 2 slices, as chosen, 38.7 with 1, 32.1 with 4; 16 sequences of 32: 59.9 with 3, as chosen, 69.4 with 2, 61.3
// with 5.)
int verify_splits(long long rows, long long row_bytes, int num_sms) {
    const long long wanted = (8ll * num_sms + rows - 1) / rows;
    const long long most = std::max(1ll, row_bytes / (16 * kVerifyThreads));
    return static_cast<int>(std::max(1ll, std::min({wanted, most, static_cast<long long>(kVerifyMaxSplits)})));
}

// CTAs that share a sequence: up to eight, as long as all of them run at once.
int verify_cluster(int B, int threads, int num_sms) {
    int ranks = kVerifyMaxCluster;
    while (ranks > 1 && static_cast<long long>(B) * ranks > static_cast<long long>(kDecideResident / threads) * num_sms)
        ranks >>= 1;
    return ranks;
}

template <typename T, bool kMask, int kThreads>
cudaError_t launch_clusters(const VerifyParams &p, int num_sms, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    const int ranks = verify_cluster(p.a.B, kThreads, num_sms);
    cfg.gridDim = dim3(static_cast<unsigned>(p.a.B) * ranks);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = p.a.D > 0 ? static_cast<size_t>(p.a.D + 1) * kDecideRowBytes : 0;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ranks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return p.a.D > 0 ? cudaLaunchKernelEx(&cfg, k_verify_decide<T, kMask, kThreads>, p)
                     : cudaLaunchKernelEx(&cfg, k_sample<T, kMask, kThreads>, p);
}

template <typename T, bool kMask>
cudaError_t launch_verify(const VerifyParams &p, long long rows, int num_sms, cudaStream_t s) {
    if (p.a.D > 0) {
        const cudaError_t e = launch_pdl(k_verify_rows<T, kMask>, dim3(static_cast<unsigned>(rows * p.splits)),
                                         dim3(kVerifyThreads), 0, s, p);
        if (e != cudaSuccess) return e;
    }
    // few sequences: twice the threads a CTA (16 sequences: 59.9 us against 65.7; 64 sequences 32.7 against 30.1)
    return static_cast<long long>(p.a.B) * kVerifyMaxCluster * 512 <= static_cast<long long>(kDecideResident) * num_sms
               ? launch_clusters<T, kMask, 512>(p, num_sms, s)
               : launch_clusters<T, kMask, 256>(p, num_sms, s);
}

template <typename T>
cudaError_t launch_verify_type(const VerifyParams &p, long long rows, int num_sms, cudaStream_t s) {
    return p.a.allowed ? launch_verify<T, true>(p, rows, num_sms, s) : launch_verify<T, false>(p, rows, num_sms, s);
}

const char *verify_shape_error(int B, int D, int V) {
    if (B < 0 || D < 0 || V < 1) return "B and D must be >= 0, V >= 1";
    return nullptr;
}

}  // namespace
}  // namespace rpd

using namespace rpd;

extern "C" {

int64_t rpd_verify_workspace(int B, int D) {
    if (const char *m = verify_shape_error(B, D, 1)) {
        op_fail(RPD_ERR_INVALID_ARGUMENT, "%s", m);
        return -1;
    }
    return D == 0 ? 0 : static_cast<int64_t>(B) * (2 * static_cast<int64_t>(D) + 1) * kVerifyMaxSplits * 16;
}

int rpd_verify(const rpd_verify_args *args, void *workspace, int64_t workspace_bytes, void *stream_ptr) {
    if (!args) return op_fail(RPD_ERR_INVALID_ARGUMENT, "null argument");
    const rpd_verify_args &a = *args;
    if (const char *m = verify_shape_error(a.B, a.D, a.V)) return op_fail(RPD_ERR_INVALID_ARGUMENT, "%s", m);
    if (!type_size(a.type)) return op_fail(RPD_ERR_INVALID_ARGUMENT, "logits must be bf16, fp16 or fp32");
    if (a.D > kVerifyMaxDrafts || a.V > (1 << 24))
        return op_fail(RPD_ERR_UNSUPPORTED, "D must be <= %d and V <= %d", kVerifyMaxDrafts, 1 << 24);
    const long long rows = static_cast<long long>(a.B) * (a.draft ? 2 * a.D + 1 : a.D + 1);
    if (rows > kVerifyMaxRows)
        return op_fail(RPD_ERR_UNSUPPORTED, "too many rows (%lld)", rows);
    if (a.B == 0) return RPD_OK;
    if (!a.target || !a.out_accepted || !a.out_token || !a.out_status || (a.D > 0 && !a.tokens))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "null buffer");
    if (!a.temperature && (!a.noise || (a.D > 0 && !a.uniform)))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "uniform and noise are needed unless every temperature is 0");
    const int64_t need = rpd_verify_workspace(a.B, a.D);
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned16(workspace)))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "workspace: %lld bytes at a 16-byte boundary needed",
                       static_cast<long long>(need));
    if (a.target_seq_stride < 0 || a.target_row_stride < 0 || a.draft_seq_stride < 0 || a.draft_row_stride < 0 ||
        a.noise_stride < 0)
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "strides must be >= 0");
    const int size = type_size(a.type);
    const void *words[] = {a.tokens, a.lengths, a.temperature, a.allowed, a.uniform, a.noise,
                           a.out_accepted, a.out_token, a.out_status, a.out_prob};
    bool aligned = aligned_to(a.target, size) && aligned_to(a.draft, size);
    for (const void *w : words) aligned = aligned && aligned_to(w, 4);
    if (!aligned) return op_fail(RPD_ERR_INVALID_ARGUMENT, "buffers must be aligned to their elements");

    // the device that holds the target's logits runs the call, whichever is current
    cudaPointerAttributes at{};
    cudaError_t e = cudaPointerGetAttributes(&at, a.target);
    if (e != cudaSuccess || (at.type != cudaMemoryTypeDevice && at.type != cudaMemoryTypeManaged)) {
        cudaGetLastError();
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "target must be device memory");
    }
    DeviceGuard dg(at.device);
    if (dg.err != cudaSuccess) return op_cuda_fail(dg.err, "cudaSetDevice");
    if (const int rc = check_device(at.device)) return rc;
    const void *device[] = {a.draft, a.tokens, a.lengths, a.temperature, a.allowed, a.uniform, a.noise,
                            a.out_accepted, a.out_token, a.out_status, a.out_prob, need > 0 ? workspace : nullptr};
    for (const void *d : device)
        if (d && !pointer_usable(d, at.device, false))
            return op_fail(RPD_ERR_INVALID_ARGUMENT, "every buffer must be device memory on the device of the target");
    int num_sms = 0;
    e = cudaDeviceGetAttribute(&num_sms, cudaDevAttrMultiProcessorCount, at.device);
    if (e != cudaSuccess) return op_cuda_fail(e, "device query");

    VerifyParams p{};
    p.a = a;
    if (a.D == 0) p.a.draft = nullptr;
    p.partials = static_cast<float4 *>(workspace);
    p.splits = verify_splits(rows, static_cast<long long>(a.V) * size, num_sms);
    p.words = (a.V + 31) / 32;
    cudaStream_t s = static_cast<cudaStream_t>(stream_ptr);
    e = a.type == RPD_TYPE_F32    ? launch_verify_type<float>(p, rows, num_sms, s)
        : a.type == RPD_TYPE_BF16 ? launch_verify_type<__nv_bfloat16>(p, rows, num_sms, s)
                                  : launch_verify_type<__half>(p, rows, num_sms, s);
    if (e != cudaSuccess) return op_cuda_fail(e, "verification launch");
    return RPD_OK;
}

}  // extern "C"
