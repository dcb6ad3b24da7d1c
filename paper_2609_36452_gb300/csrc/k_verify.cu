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
// k_verify_rows reads every row of logits once and leaves its largest logit and the sum of the exponentials
// above it, a few slices of a row at a time: bound by HBM.  k_verify_decide, a cluster of CTAs a sequence,
// joins the slices, finds j, and scans the one row (or two) that the next token is drawn from: most of it is
// still in L2.  Statistics and probabilities are fp32, differences z - m come before the multiplication by
// 1 / T (with bf16 and fp16 logits they are exact or nearly so).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "op_host.h"
#include "ptx.cuh"

namespace rpd {
namespace {

constexpr int kVerifyThreads = 256;
constexpr int kVerifyWarps = kVerifyThreads / 32;
constexpr int kVerifyCluster = 8;     // CTAs that scan one sequence's row
constexpr int kVerifyMaxDrafts = 1024;
constexpr int kVerifyMaxSplits = 32;

struct VerifyParams {
    rpd_verify_args a;
    float4 *partials;  // [B][2 D + 1][splits]: largest logit, sum, lowest index of the largest logit
    int splits;
    int words;         // 32-bit words of a row of `allowed`
};

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

constexpr float kNoLogit = -__builtin_huge_valf();

// 1 / T in units of log2, so that e^(x / T) = 2^(x c).  Within bounds where infinite logits give 0 and the
// largest one's 0 stays 0.
__device__ __forceinline__ float exponent_scale(float T) {
    return fminf(fmaxf(1.4426950408889634f / T, 1e-37f), 1e30f);
}

// ------------------------------------------------------------------------------ statistics of the rows

// Running maximum and sum.  A sum that is not finite and positive marks a row without a distribution: a
// NaN or an infinite logit makes it NaN, and a row without any finite logit leaves it 0.
struct Stat {
    float m = kNoLogit, s = 0.f;
    template <int N>
    __device__ __forceinline__ void add(const float (&z)[N], float c) {
        float top = m;
#pragma unroll
        for (int i = 0; i < N; ++i) top = fmaxf(top, z[i]);
        if (top == kNoLogit) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (z[i] != z[i]) s = z[i];
            return;
        }
        if (top > m) {
            s *= ex2((m - top) * c);
            m = top;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) s += ex2((z[i] - m) * c);
    }
    __device__ __forceinline__ void join(float m2, float s2, float c) {
        const float top = fmaxf(m, m2);
        if (top == kNoLogit) {
            s += s2;
        } else {
            s = s * ex2((m - top) * c) + s2 * ex2((m2 - top) * c);
            m = top;
        }
    }
    __device__ __forceinline__ bool ok() const { return s > 0.f && s < -kNoLogit; }
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
template <typename T, bool kMask, typename F, typename G>
__device__ __forceinline__ void walk_slice(const Row<T> &row, const uint32_t *mask, int words, int split, int splits,
                                           const F &f, const G &g) {
    constexpr int N = Row<T>::kVec;
    constexpr int kUnroll = 4;
    const int v0 = static_cast<int>(static_cast<long long>(row.vecs) * split / splits);
    const int v1 = static_cast<int>(static_cast<long long>(row.vecs) * (split + 1) / splits);
    const uint4 *body = reinterpret_cast<const uint4 *>(row.p + row.peel);
    for (int v = v0 + threadIdx.x; v < v1; v += kVerifyThreads * kUnroll) {
        uint4 raw[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (v + u * kVerifyThreads < v1) raw[u] = body[v + u * kVerifyThreads];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int at = v + u * kVerifyThreads;
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
template <typename T, bool kMask>
__device__ __forceinline__ void row_slice(const rpd_verify_args &a, const VerifyParams &p, int b, int i, int split,
                                          const void *base, long long offset, float temperature, float4 *out) {
    const Row<T> row(base, offset, a.V);
    const uint32_t *mask = kMask ? mask_row(a, p.words, b, i) : nullptr;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __shared__ float4 part[kVerifyWarps];
    if (temperature > 0.f) {
        const float c = exponent_scale(temperature);
        Stat st;
        walk_slice<T, kMask>(
            row, mask, p.words, split, p.splits, [&](const auto &z, int) { st.add(z, c); },
            [&](float z, int) {
                const float one[1] = {z};
                st.add(one, c);
            });
#pragma unroll
        for (int o = 16; o; o >>= 1)
            st.join(__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o), c);
        if (lane == 0) part[warp] = make_float4(st.m, st.s, 0.f, 0.f);
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kVerifyWarps; ++w) st.join(part[w].x, part[w].y, c);
            *out = make_float4(st.m, st.s, 0.f, 0.f);
        }
    } else {
        Best best;
        walk_slice<T, kMask>(
            row, mask, p.words, split, p.splits,
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
            for (int w = 1; w < kVerifyWarps; ++w) {
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
    pdl_trigger();
    const int kinds = a.draft ? 2 * a.D + 1 : a.D + 1;
    const int split = blockIdx.x % p.splits, r = blockIdx.x / p.splits % kinds, b = blockIdx.x / p.splits / kinds;
    const bool is_draft = r > a.D;
    const int i = is_draft ? r - a.D - 1 : r;
    pdl_wait();
    const int n = draft_count(a, b);
    const float temperature = temperature_of(a, b);
    // rows behind a sequence's last one are never read, nor a draft model's where the choice is greedy
    if (n < 0 || n > a.D || !(temperature >= 0.f) || (is_draft ? i >= n || temperature == 0.f : i > n)) return;
    float4 *out = p.partials + (static_cast<long long>(b) * (2 * a.D + 1) + r) * p.splits + split;
    if (is_draft)
        row_slice<T, false>(a, p, b, i, split, a.draft, draft_offset(a, b, i), temperature, out);
    else
        row_slice<T, kMask>(a, p, b, i, split, a.target, target_offset(a, b, i), temperature, out);
}

// ------------------------------------------------------------------------------ decision

// Weight and variate of the race's leader: w / e is the largest so far, the lowest index on a tie.
// Compared by cross products, so that a variate of 0 wins against any other.
struct Race {
    float w = 0.f, e = 1.f;
    int at = 0x7FFFFFFF;
    __device__ __forceinline__ void add(float w2, float e2, int at2) {  // a thread's indices rise
        if (w2 > 0.f && e2 >= 0.f && w2 * e > w * e2) {
            w = w2;
            e = e2;
            at = at2;
        }
    }
    __device__ __forceinline__ void join(float w2, float e2, int at2) {
        const float x = w2 * e, y = w * e2;
        if (w2 > 0.f && (x > y || (x == y && at2 < at) || w == 0.f)) {
            w = w2;
            e = e2;
            at = at2;
        }
    }
    __device__ __forceinline__ void join_warp() {
#pragma unroll
        for (int o = 16; o; o >>= 1)
            join(__shfl_xor_sync(0xffffffffu, w, o), __shfl_xor_sync(0xffffffffu, e, o),
                 __shfl_xor_sync(0xffffffffu, at, o));
    }
};

// Shared memory: for rows 0..D of the target largest logit, sum and argmax, for those of the draft
// model largest logit and sum.
struct DecideRows {
    float *tm, *ts, *dm, *ds;
    int *arg;
};

template <typename T, bool kMask>
__global__ void __cluster_dims__(kVerifyCluster) __launch_bounds__(kVerifyThreads)
    k_verify_decide(const VerifyParams p) {
    const rpd_verify_args &a = p.a;
    extern __shared__ float rows_smem[];
    __shared__ int first_stop;
    __shared__ Race warp_race[2][kVerifyWarps];
    __shared__ Race cta_race[2][kVerifyCluster];  // of the whole cluster, in its first CTA
    const DecideRows s{rows_smem, rows_smem + (a.D + 1), rows_smem + 2 * (a.D + 1), rows_smem + 3 * (a.D + 1),
                       reinterpret_cast<int *>(rows_smem + 4 * (a.D + 1))};
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int b = blockIdx.x / kVerifyCluster, rank = cluster_ctarank();
    pdl_trigger();
    cluster_sync();  // every CTA of the cluster runs: their shared memory may be written
    pdl_wait();
    const int n = draft_count(a, b);
    const float T_seq = temperature_of(a, b);
    const bool greedy = T_seq == 0.f;
    const bool usable = n >= 0 && n <= a.D && T_seq >= 0.f && (greedy || (a.noise && (n == 0 || a.uniform)));
    const float c = greedy ? 1.f : exponent_scale(T_seq);
    const bool drafts = a.draft && !greedy;
    int stop = 0, next = -1;
    bool bad = true;
    if (threadIdx.x == 0) first_stop = usable ? n : 0;
    if (usable) {
        // the slices of every row joined, a warp a row
        const float4 *partials = p.partials + static_cast<long long>(b) * (2 * a.D + 1) * p.splits;
        const int count = n + 1 + (drafts ? n : 0);
        for (int k = warp; k < count; k += kVerifyWarps) {
            const int r = k <= n ? k : a.D + 1 + (k - n - 1);
            float4 v = lane < p.splits ? partials[static_cast<long long>(r) * p.splits + lane]
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
                st.s = v.y;
#pragma unroll
                for (int o = 16; o; o >>= 1)
                    st.join(__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o), c);
                if (lane == 0) {
                    const float sum = st.ok() ? st.s : 0.f;
                    if (k <= n) {
                        s.tm[k] = st.m;
                        s.ts[k] = sum;
                    } else {
                        s.dm[k - n - 1] = st.m;
                        s.ds[k - n - 1] = sum;
                    }
                }
            }
        }
        __syncthreads();
        // every draft's verdict; the first rejection counts
        for (int i = threadIdx.x; i < n; i += kVerifyThreads) {
            const int x = a.tokens[static_cast<long long>(b) * a.D + i];
            const bool in = x >= 0 && x < a.V;
            bool sound = s.ts[i] > 0.f;
            float px = 0.f, qx = 1.f;
            if (in && sound) {
                if (greedy) {
                    px = x == s.arg[i] ? 1.f : 0.f;
                } else if (!kMask || ((mask_row(a, p.words, b, i)[x >> 5] >> (x & 31)) & 1u)) {
                    const float z = value(static_cast<const T *>(a.target)[target_offset(a, b, i) + x]);
                    px = ex2((z - s.tm[i]) * c) / s.ts[i];
                }
            }
            if (drafts) {
                sound = sound && s.ds[i] > 0.f;
                qx = 0.f;
                if (in && sound) {
                    const float z = value(static_cast<const T *>(a.draft)[draft_offset(a, b, i) + x]);
                    qx = ex2((z - s.dm[i]) * c) / s.ds[i];
                }
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
            // the race: its weights, and - should no residual be positive (p = q but for roundings) -
            // the target's own probabilities
            Race race, plain;
            const Row<T> row(a.target, target_offset(a, b, stop), a.V);
            const uint32_t *mask = kMask ? mask_row(a, p.words, b, stop) : nullptr;
            const float *noise = a.noise + b * a.noise_stride;
            const T *q = rejected && drafts ? static_cast<const T *>(a.draft) + draft_offset(a, b, stop) : nullptr;
            const int x = rejected && !drafts ? a.tokens[static_cast<long long>(b) * a.D + stop] : -1;
            const float tm = s.tm[stop], t_inv = 1.f / s.ts[stop];
            const float dm = q ? s.dm[stop] : 0.f, d_inv = q ? 1.f / s.ds[stop] : 0.f;
            auto one = [&](float z, int at) {
                const float w = ex2((z - tm) * c) * t_inv, e = noise[at];
                float left = at == x ? 0.f : w;
                if (q) left = w - ex2((value(q[at]) - dm) * c) * d_inv;
                race.add(left, e, at);
                if (rejected) plain.add(w, e, at);
            };
            walk_slice<T, kMask>(
                row, mask, p.words, rank, kVerifyCluster,
                [&](const auto &z, int first) {
#pragma unroll
                    for (int k = 0; k < Row<T>::kVec; ++k) one(z[k], first + k);
                },
                one);
            race.join_warp();
            plain.join_warp();
            if (lane == 0) {
                warp_race[0][warp] = race;
                warp_race[1][warp] = plain;
            }
            __syncthreads();
            if (threadIdx.x < 2) {
                Race r = warp_race[threadIdx.x][0];
                for (int w = 1; w < kVerifyWarps; ++w) {
                    const Race &o = warp_race[threadIdx.x][w];
                    r.join(o.w, o.e, o.at);
                }
                const uint32_t to = mapa_shared(smem_u32(&cta_race[threadIdx.x][rank]), 0);
                st_shared_cluster(to, __float_as_int(r.w));
                st_shared_cluster(to + 4, __float_as_int(r.e));
                st_shared_cluster(to + 8, r.at);
            }
        }
    }
    cluster_sync();
    if (rank != 0) return;
    if (usable && !bad && !greedy) {
        Race r;
        for (int kind = 0; kind < 2 && r.w == 0.f; ++kind)
            for (int k = 0; k < kVerifyCluster; ++k)
                r.join(cta_race[kind][k].w, cta_race[kind][k].e, cta_race[kind][k].at);
        next = r.w > 0.f ? r.at : -1;
        bad = next < 0;
    }
    for (int i = threadIdx.x; i <= a.D; i += kVerifyThreads) {
        const long long row = static_cast<long long>(b) * (a.D + 1);
        a.out_token[row + i] = i < stop ? a.tokens[static_cast<long long>(b) * a.D + i] : i == stop ? next : -1;
        if (a.out_prob && i < a.D && i >= (usable ? n : 0)) a.out_prob[static_cast<long long>(b) * a.D + i] = 0.f;
    }
    if (threadIdx.x == 0) {
        a.out_accepted[b] = stop;
        a.out_status[b] = bad ? RPD_ERR_INVALID_ARGUMENT : RPD_OK;
    }
}

// Slices of a row: enough CTAs for every SM to hold eight, none with less than a vector a thread.
int verify_splits(long long rows, long long row_bytes, int num_sms) {
    const long long wanted = (8ll * num_sms + rows - 1) / rows;
    const long long most = std::max(1ll, row_bytes / (16 * kVerifyThreads));
    return static_cast<int>(std::max(1ll, std::min({wanted, most, static_cast<long long>(kVerifyMaxSplits)})));
}

template <typename T, bool kMask>
cudaError_t launch_verify(const VerifyParams &p, long long rows, cudaStream_t s) {
    cudaError_t e = launch_pdl(k_verify_rows<T, kMask>, dim3(static_cast<unsigned>(rows * p.splits)),
                               dim3(kVerifyThreads), 0, s, p);
    if (e != cudaSuccess) return e;
    return launch_pdl(k_verify_decide<T, kMask>, dim3(static_cast<unsigned>(p.a.B) * kVerifyCluster),
                      dim3(kVerifyThreads), static_cast<size_t>(p.a.D + 1) * 20, s, p);
}

template <typename T>
cudaError_t launch_verify_type(const VerifyParams &p, long long rows, cudaStream_t s) {
    return p.a.allowed ? launch_verify<T, true>(p, rows, s) : launch_verify<T, false>(p, rows, s);
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
    return static_cast<int64_t>(B) * (2 * static_cast<int64_t>(D) + 1) * kVerifyMaxSplits * 16;
}

int rpd_verify(const rpd_verify_args *args, void *workspace, int64_t workspace_bytes, void *stream_ptr) {
    if (!args) return op_fail(RPD_ERR_INVALID_ARGUMENT, "null argument");
    const rpd_verify_args &a = *args;
    if (const char *m = verify_shape_error(a.B, a.D, a.V)) return op_fail(RPD_ERR_INVALID_ARGUMENT, "%s", m);
    if (!type_size(a.type)) return op_fail(RPD_ERR_INVALID_ARGUMENT, "logits must be bf16, fp16 or fp32");
    if (a.D > kVerifyMaxDrafts || a.V > (1 << 24))
        return op_fail(RPD_ERR_UNSUPPORTED, "D must be <= %d and V <= %d", kVerifyMaxDrafts, 1 << 24);
    const long long rows = static_cast<long long>(a.B) * (a.draft ? 2 * a.D + 1 : a.D + 1);
    if (rows * kVerifyMaxSplits > 0x7FFFFFFFll || a.B > (0x7FFFFFFF / kVerifyCluster))
        return op_fail(RPD_ERR_UNSUPPORTED, "too many rows (%lld)", rows);
    if (a.B == 0) return RPD_OK;
    if (!a.target || !a.out_accepted || !a.out_token || !a.out_status || !workspace || (a.D > 0 && !a.tokens))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "null buffer");
    if (!a.temperature && (!a.noise || (a.D > 0 && !a.uniform)))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "uniform and noise are needed unless every temperature is 0");
    if (workspace_bytes < rpd_verify_workspace(a.B, a.D) || !aligned16(workspace))
        return op_fail(RPD_ERR_INVALID_ARGUMENT, "workspace: %lld bytes at a 16-byte boundary needed",
                       static_cast<long long>(rpd_verify_workspace(a.B, a.D)));
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
                            a.out_accepted, a.out_token, a.out_status, a.out_prob, workspace};
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
    e = a.type == RPD_TYPE_F32    ? launch_verify_type<float>(p, rows, s)
        : a.type == RPD_TYPE_BF16 ? launch_verify_type<__nv_bfloat16>(p, rows, s)
                                  : launch_verify_type<__half>(p, rows, s);
    if (e != cudaSuccess) return op_cuda_fail(e, "verification launch");
    return RPD_OK;
}

}  // extern "C"
