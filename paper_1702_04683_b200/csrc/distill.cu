// Distillation from a teacher's top logits: the k largest logits of a row with the row's normaliser, and the student's loss
// and gradient from such pairs.
//
//   lse = log sum exp(l_j / T)
//   q = softmax(t / T) over the list   or   q = exp(t / T - lse), r = max(0, 1 - sum q)
//   L = sum q (log q - log p) + r (log r - log p_rest),      p = softmax(s / T), p_rest = sum of p not listed
//   dL/ds_j = (W p_j - q_j) / T listed, (W - r / p_rest) p_j / T not listed,      W = sum q + r
//
// All of it is bound by HBM: every logit is read once and, with a gradient, one entry written for it; one exponential
// (two with a gradient) per logit.
#include <cooperative_groups.h>
#include <math.h>
#include <new>

#include "rows.cuh"

using namespace adacomp;

struct adacomp_distill {
    int device;
    uint32_t vocab;
    int n_sms;
    int* d_status;
};

namespace {

constexpr int kThreads = 512;
constexpr uint32_t kMaxPairs = 1024;
constexpr uint32_t kMaxVocab = 1u << 20;
constexpr uint32_t kStats = 8;
constexpr uint32_t kNone = 0xFFFFFFFFu;
constexpr double kLog2e = 1.4426950408889634;

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 16 bytes that nobody else's loads of the call have to see (no .nc: the gradient may take their place).
__device__ __forceinline__ uint4 load16_once(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// Two operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{ .reg .b64 a, b, c, d; mov.b64 a, {%2, %3}; mov.b64 b, {%4, %5}; mov.b64 c, {%6, %7}; fma.rn.f32x2 d, a, b, c; mov.b64 {%0, %1}, d; }"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{ .reg .b64 a, b, d; mov.b64 a, {%2, %3}; mov.b64 b, {%4, %5}; add.rn.f32x2 d, a, b; mov.b64 {%0, %1}, d; }"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

// The largest of two, NaN if one is.
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
template <typename T> __device__ __forceinline__ uint32_t max_nan_halves(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t max_nan_halves<__nv_bfloat16>(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
template <> __device__ __forceinline__ uint32_t max_nan_halves<__half>(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// The largest entry of a vector, NaN if it holds one.
template <typename T> __device__ __forceinline__ float vec_max(const uint4& v) {
    if constexpr (sizeof(T) == 4) {
        return max_nan(max_nan(__uint_as_float(v.x), __uint_as_float(v.y)), max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
    } else {
        const float2 f = halves<T>(max_nan_halves<T>(max_nan_halves<T>(v.x, v.y), max_nan_halves<T>(v.z, v.w)));
        return max_nan(f.x, f.y);
    }
}

template <typename T> constexpr int kVec = 16 / sizeof(T);

// A row on the 16-byte grid: `lead` entries before it, n_vecs vectors on it, the rest behind it.
struct Cut {
    uint32_t lead, n_vecs, loose;
    template <typename T> __device__ __forceinline__ static Cut of(const T* p, uint32_t n) {
        Cut c;
        const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p) % 16 / sizeof(T));
        c.lead = min(n, (kVec<T> - off) % kVec<T>);
        c.n_vecs = (n - c.lead) / kVec<T>;
        c.loose = n - c.n_vecs * kVec<T>;
        return c;
    }
    // The place of loose entry i, lead and rest counted through.
    template <typename T> __device__ __forceinline__ uint32_t loose_at(uint32_t i) const { return i < lead ? i : i + n_vecs * kVec<T>; }
};

// A running softmax sum: m the largest so far, s = sum exp((x - m) c) with c = log2(e) / T in base 2.
struct Running {
    float m, s;
    __device__ __forceinline__ void raise(float to, float c) {
        if (to > m) {
            s *= ex2((m - to) * c);
            m = to;
        }
    }
    // What stands for m in differences: an infinitely small largest one would make NaN of them.
    __device__ __forceinline__ float base() const { return m == -INFINITY ? 0.0f : m; }
    __device__ __forceinline__ void join(float m2, float s2, float c) {
        const float most = fmaxf(m, m2);
        const float a = m == most ? s : s * ex2((m - most) * c), b = m2 == most ? s2 : s2 * ex2((m2 - most) * c);
        m = most;
        s = a + b;
    }
};

__device__ __forceinline__ Running warp_join(Running r, float c) {
#pragma unroll
    for (int d = 16; d; d >>= 1) r.join(__shfl_xor_sync(~0u, r.m, d), __shfl_xor_sync(~0u, r.s, d), c);
    return r;
}

template <typename V> __device__ __forceinline__ V warp_sum(V x) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    return x;
}

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x = fmaxf(x, __shfl_xor_sync(~0u, x, d));
    return x;
}

struct Job {
    Rows logits, out, idx, val;
    const float* lse;
    const float* weight;
    float* loss;
    float* stats;
    int* status;
    uint32_t n_rows, vocab, k;
    float c;                        // log2(e) / T
    double inv_t;
};

__device__ __forceinline__ float load_value(const Rows& v, uint64_t at) {
    if (v.type == ADACOMP_F32) return reinterpret_cast<const float*>(v.data)[at];
    if (v.type == ADACOMP_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(v.data)[at]);
    return __half2float(reinterpret_cast<const __half*>(v.data)[at]);
}

// What a row's gradient is made of, next to its weight: e_j rest for a token that is not listed, e_j listed - q_j for one that is, with
// e_j = exp((s_j - m) / T) and q_j = exp((t_j - t_base) / T) q_scale, or exp(t_j / T - t_base) with the teacher's normaliser.
struct Shares {
    float m, rest, listed, t_base, q_scale, live;
};

enum Mode { kLoss = 0, kGrad = 1, kBoth = 2 };

// One block per row, two passes over it; the second finds much of it in L2.
template <typename T, int MODE>
__global__ void __launch_bounds__(kThreads) k_distill(const Job j) {
    constexpr int N = kVec<T>;
    extern __shared__ uint32_t s_bits[];            // one bit per token: whether it is listed
    __shared__ uint32_t s_idx[kMaxPairs];
    __shared__ float s_val[kMaxPairs];
    __shared__ float s_m[kThreads / 32], s_s[kThreads / 32], s_x[kThreads / 32];
    __shared__ double s_d[3][kThreads / 32];
    __shared__ Shares s_share;
    const uint32_t row = blockIdx.x, tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    const T* in = reinterpret_cast<const T*>(j.logits.data) + j.logits.offset(row);
    T* out = MODE == kLoss ? nullptr : reinterpret_cast<T*>(j.out.data) + j.out.offset(row);
    const float weight = j.weight ? j.weight[row] : 1.0f;
    Shares share = {};
    if (weight != 0.0f) {
        for (uint32_t i = tid; i < (j.vocab + 31) / 32; i += kThreads) s_bits[i] = 0;
        __syncthreads();
        bool again = false;
        for (uint32_t i = tid; i < j.k; i += kThreads) {
            const uint64_t at = j.idx.offset(row) + i;
            const int64_t v = j.idx.type == ADACOMP_I64 ? reinterpret_cast<const int64_t*>(j.idx.data)[at]
                                                        : reinterpret_cast<const int32_t*>(j.idx.data)[at];
            uint32_t token = kNone;
            if (v >= j.vocab) record_error(j.status, ADACOMP_ERR_INVALID);
            else if (v >= 0) token = static_cast<uint32_t>(v);
            s_idx[i] = token;
            s_val[i] = load_value(j.val, j.val.offset(row) + i);
            if (token != kNone) again |= (atomicOr(&s_bits[token / 32], 1u << token % 32) >> token % 32) & 1;
        }
        if (__syncthreads_or(again)) {              // a token twice: the first one counts
            bool drop[kMaxPairs / kThreads] = {};
#pragma unroll
            for (int r = 0; r < static_cast<int>(kMaxPairs / kThreads); ++r)
                for (uint32_t i = tid + r * kThreads, e = 0; i < j.k && e < i; ++e) drop[r] |= s_idx[e] == s_idx[i];
            __syncthreads();
#pragma unroll
            for (int r = 0; r < static_cast<int>(kMaxPairs / kThreads); ++r)
                if (drop[r]) s_idx[tid + r * kThreads] = kNone;
            __syncthreads();
        }
        if (MODE == kGrad) {
            const float* st = j.stats + static_cast<uint64_t>(row) * kStats;
            share = {st[0], st[1], st[2], st[3], st[4], st[5]};
        } else {
            // the row's largest logit, and the sum over what is not listed
            Running r = {-INFINITY, 0.0f};
            float listed_max = -INFINITY;
            const Cut cut = Cut::of(in, j.vocab);
            if (tid < cut.loose) {
                const uint32_t at = cut.loose_at<T>(tid);
                const float x = to_float(in[at]);
                if (s_bits[at / 32] >> at % 32 & 1) {
                    listed_max = fmaxf(listed_max, x);
                } else {
                    r.raise(x, j.c);
                    r.s += ex2((x - r.base()) * j.c);
                }
            }
            for (uint32_t v = tid; v < cut.n_vecs; v += kThreads) {
                Packed<T, N> p;
                p.v[0] = load16_once(in + cut.lead + v * N);
                float f[N];
                p.unpack(f);
                const uint32_t at = cut.lead + v * N;
                const uint32_t bits = __funnelshift_r(s_bits[at / 32], at / 32 + 1 < (j.vocab + 31) / 32 ? s_bits[at / 32 + 1] : 0, at);
                float most = f[0];
#pragma unroll
                for (int e = 1; e < N; ++e) most = fmaxf(most, f[e]);
                r.raise(most, j.c);
                const float base = r.base();
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float y = ex2((f[e] - base) * j.c);
                    r.s += bits >> e & 1 ? 0.0f : y;
                }
            }
            r.raise(listed_max, j.c);               // the listed ones' sum is taken from the list
            r = warp_join(r, j.c);
            if (lane == 0) s_m[warp] = r.m, s_s[warp] = r.s;
            __syncthreads();
            r = warp_join({s_m[lane % (kThreads / 32)], lane < kThreads / 32 ? s_s[lane] : 0.0f}, j.c);
            // the teacher's list
            float top = -INFINITY;
            for (uint32_t i = tid; i < j.k; i += kThreads)
                if (s_idx[i] != kNone) top = fmaxf(top, s_val[i]);
            top = warp_max(top);
            if (lane == 0) s_x[warp] = top;
            __syncthreads();
            top = warp_max(s_x[lane % (kThreads / 32)]);
            const float base = r.base(), t_base = top == -INFINITY ? 0.0f : top;
            const double lse = j.lse ? static_cast<double>(j.lse[row]) : 0.0;
            double q_sum = 0.0, cross = 0.0, listed = 0.0;
            for (uint32_t i = tid; i < j.k; i += kThreads) {
                if (s_idx[i] == kNone) continue;
                const float s = to_float(in[s_idx[i]]);
                listed += ex2((s - base) * j.c);
                const double t = j.lse ? s_val[i] * j.inv_t - lse : (static_cast<double>(s_val[i]) - t_base) * j.inv_t;
                // with the teacher's normaliser 1 - sum q is left over: small where the list says almost everything, so in 64 bits
                double q = j.lse ? exp(t) : expf(static_cast<float>(t));
                if (q > 1e300) q = NAN;
                q_sum += q;
                if (q != 0.0) cross += q * (t - (static_cast<double>(s) - base) * j.inv_t);
            }
            q_sum = warp_sum(q_sum), cross = warp_sum(cross), listed = warp_sum(listed);
            if (lane == 0) s_d[0][warp] = q_sum, s_d[1][warp] = cross, s_d[2][warp] = listed;
            const bool any = __syncthreads_or(top != -INFINITY);
            bool present = false;
            for (uint32_t i = tid; i < j.k; i += kThreads) present |= s_idx[i] != kNone;
            present = __syncthreads_or(present);
            if (tid == 0) {
                q_sum = cross = listed = 0.0;
                for (int w = 0; w < kThreads / 32; ++w) q_sum += s_d[0][w], cross += s_d[1][w], listed += s_d[2][w];
                const double rest = r.s, total = rest + listed;
                const bool live = present && (j.lse ? lse != -INFINITY : any || q_sum != q_sum) && total != 0.0;
                double loss = 0.0;
                if (live) {
                    const double log_total = log(total);
                    if (!j.lse) {
                        loss = cross / q_sum + log_total - log(q_sum);
                        share = {base, static_cast<float>(1.0 / total), static_cast<float>(1.0 / total), t_base, static_cast<float>(1.0 / q_sum), 1.0f};
                    } else {
                        const double left = rest > 0.0 && q_sum < 1.0 ? 1.0 - q_sum : 0.0, mass = q_sum + left;
                        loss = cross + q_sum * log_total + (left > 0.0 ? left * (log(left) - log(rest) + log_total) : 0.0);
                        share = {base, static_cast<float>(mass / total - (left > 0.0 ? left / rest : 0.0)), static_cast<float>(mass / total),
                                 static_cast<float>(lse), 1.0f, 1.0f};
                    }
                }
                if (q_sum != q_sum) share.rest = share.listed = NAN;
                if (j.loss) j.loss[row] = static_cast<float>(loss);
                s_share = share;
                if (j.stats) {
                    float4* st = reinterpret_cast<float4*>(j.stats + static_cast<uint64_t>(row) * kStats);
                    st[0] = make_float4(share.m, share.rest, share.listed, share.t_base);
                    st[1] = make_float4(share.q_scale, share.live, 0.0f, 0.0f);
                }
            }
            __syncthreads();
            share = s_share;
        }
    } else if (MODE != kGrad && tid == 0) {
        if (j.loss) j.loss[row] = 0.0f;
        if (j.stats) {
            float4* st = reinterpret_cast<float4*>(j.stats + static_cast<uint64_t>(row) * kStats);
            st[0] = st[1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
    }
    if (MODE == kLoss) return;

    // the gradient: windows on the output's grid
    const Cut cut = Cut::of(out, j.vocab);
    if (share.live == 0.0f) {
        for (uint32_t v = tid; v < cut.n_vecs; v += kThreads) *reinterpret_cast<uint4*>(out + cut.lead + v * N) = make_uint4(0, 0, 0, 0);
        if (tid < cut.loose) out[cut.loose_at<T>(tid)] = from_float<T>(0.0f);
        return;
    }
    const float g = static_cast<float>(weight * j.inv_t), rest = share.rest * g;
    const bool on_grid = (reinterpret_cast<uintptr_t>(in) - reinterpret_cast<uintptr_t>(out)) % 16 == 0;
    uint32_t token[kMaxPairs / kThreads];
    float listed[kMaxPairs / kThreads];
#pragma unroll
    for (int r = 0; r < static_cast<int>(kMaxPairs / kThreads); ++r) {
        const uint32_t i = tid + r * kThreads;
        token[r] = i < j.k ? s_idx[i] : kNone;
        if (token[r] == kNone) continue;
        const double t = j.lse ? s_val[i] * j.inv_t - share.t_base : (static_cast<double>(s_val[i]) - share.t_base) * j.inv_t;
        const float q = expf(static_cast<float>(t)) * share.q_scale;
        listed[r] = (ex2((to_float(in[token[r]]) - share.m) * j.c) * share.listed - q) * g;
    }
    __syncthreads();                                // before the gradient may take the place of a logit that is read here
    for (uint32_t v = tid; v < cut.n_vecs; v += kThreads) {
        Packed<T, N> p;
        if (on_grid) p.v[0] = load16_once(in + cut.lead + v * N);
        else p = load_shifted<T, N>(in, cut.lead + static_cast<int64_t>(v) * N, j.vocab);
        float f[N];
        p.unpack(f);
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = ex2((f[e] - share.m) * j.c) * rest;
        p.pack(f);
        *reinterpret_cast<uint4*>(out + cut.lead + v * N) = p.v[0];
    }
    if (tid < cut.loose) {
        const uint32_t at = cut.loose_at<T>(tid);
        out[at] = from_float<T>(ex2((to_float(in[at]) - share.m) * j.c) * rest);
    }
    __syncthreads();                                // the listed ones replace what has just been written
#pragma unroll
    for (int r = 0; r < static_cast<int>(kMaxPairs / kThreads); ++r)
        if (token[r] != kNone) out[token[r]] = from_float<T>(listed[r]);
}

// ---------------------------------------------------------------------------------------------- top logits

constexpr int kTopThreads = 256;
constexpr int kTopVecs = 4;                         // vectors of a thread in one step
constexpr uint32_t kTopStep = kTopThreads * kTopVecs;
constexpr uint32_t kCandidates = 2048;
constexpr int kBoundBits = 16;
constexpr uint32_t kTopCluster = 8;

struct TopJob {
    Rows logits;
    int32_t* idx;
    void* val;
    float* lse;
    uint32_t vocab, k;
    float c;
    double inv_t;
};

// Order of logits as whole numbers: NaN above all, +0 and -0 equal; below it the token, the lowest first.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);
    return x != x ? 0xFFFFFFFFu : u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ uint64_t composite(float x, uint32_t token) {
    return static_cast<uint64_t>(order_of(x)) << 32 | (0xFFFFFFFFu - token);
}
// A float that every entry above `bound` in order exceeds, other than by its token (NaN, which nothing fails to exceed, where there is none).
__device__ __forceinline__ float floor_of(uint64_t bound) {
    const uint32_t u = static_cast<uint32_t>(bound >> 32), bits = u >> 31 ? u ^ 0x80000000u : ~u;
    return __uint_as_float(bits == 0x80000000u ? 0x80000001u : bits);      // +0 does not exceed -0
}

// Sorts s_list[0 .. n) in falling order, n a power of two.  Up to one entry a thread, distances within a warp are exchanged by
// shuffles (256 entries: 12 barriers instead of 36).
__device__ void sort_list(uint64_t* s_list, uint32_t n) {
    if (n <= kTopThreads) {
        const uint32_t i = threadIdx.x;
        __syncthreads();
        uint64_t x = i < n ? s_list[i] : 0;
        for (uint32_t k = 2; k <= n; k *= 2)
            for (uint32_t d = k / 2; d; d /= 2) {
                uint64_t y;
                if (d >= 32) {
                    if (i < n) s_list[i] = x;
                    __syncthreads();
                    y = i < n ? s_list[i ^ d] : 0;
                    __syncthreads();
                } else {
                    y = __shfl_xor_sync(~0u, x, d);
                }
                const bool larger = ((i & k) == 0) == ((i & d) == 0);       // of the two, the one that this place keeps
                x = (x > y) == larger ? x : y;
            }
        if (i < n) s_list[i] = x;
    } else {
        for (uint32_t k = 2; k <= n; k *= 2)
            for (uint32_t d = k / 2; d; d /= 2) {
                __syncthreads();
                for (uint32_t i = threadIdx.x; i < n / 2; i += kTopThreads) {
                    const uint32_t a = 2 * i - (i & (d - 1)), b = a + d;
                    const uint64_t x = s_list[a], y = s_list[b];
                    if ((x < y) == ((a & k) == 0)) s_list[a] = y, s_list[b] = x;
                }
            }
    }
    __syncthreads();
}

// The entries above the k-th largest of those seen so far are collected in a list, which is cut back to its k largest when it
// has grown to twice that (or is full).  The first step's bound: with k of the threads' (or vectors') largest entries at or above a
// number, k entries are.  From there on about k ln(vocab / entries of a step) entries make it to the list, so most vectors cost a
// maximum, their exponentials and one comparison.
//
// A row is one block's work, or a cluster's where there are few rows: the first block then takes the others' lists through
// their shared memory.
template <typename T>
__global__ void __launch_bounds__(kTopThreads, 4) k_top_logits(const TopJob j) {
    constexpr int N = kVec<T>;
    __shared__ uint64_t s_list[kCandidates];
    __shared__ uint32_t s_count, s_above[kBoundBits];
    __shared__ float s_m[kTopThreads / 32], s_s[kTopThreads / 32];
    __shared__ Running s_run;
    namespace cg = cooperative_groups;
    const cg::cluster_group cluster = cg::this_cluster();
    const uint32_t ranks = cluster.num_blocks(), rank = cluster.block_rank();
    const uint32_t row = blockIdx.x / ranks, tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    const T* in = reinterpret_cast<const T*>(j.logits.data) + j.logits.offset(row);
    const Cut cut = Cut::of(in, j.vocab);
    const uint32_t per = (cut.n_vecs + ranks - 1) / ranks, from = min(rank * per, cut.n_vecs), to = min(from + per, cut.n_vecs);
    const uint32_t trigger = min(2 * j.k + 64, kCandidates);
    uint64_t bound = 0;                             // an entry must be above it
    float floor = NAN;
    Running r = {-INFINITY, 0.0f};
    if (tid == 0) s_count = 0;
    if (tid < kBoundBits) s_above[tid] = 0;
    __syncthreads();

    auto cut_back = [&]() {                         // the list sorted, and its k largest kept
        const uint32_t n = min(s_count, kCandidates);
        uint32_t size = 2;
        while (size < n) size *= 2;
        for (uint32_t i = n + tid; i < size; i += kTopThreads) s_list[i] = 0;
        sort_list(s_list, size);
        if (tid == 0) s_count = min(n, j.k);
        if (n >= j.k) bound = s_list[j.k - 1], floor = floor_of(bound);
        __syncthreads();
    };
    bool grown = false;
    auto taken = [&](uint64_t x) {                  // whether x needs no more care
        if (x <= bound) return true;
        const uint32_t place = atomicAdd(&s_count, 1);
        grown |= place >= trigger - 1;
        if (place >= kCandidates) return false;
        s_list[place] = x;
        return true;
    };

    // entries off the grid
    if (rank == 0) {
        const uint32_t at = tid < cut.loose ? cut.loose_at<T>(tid) : 0;
        if (tid < cut.loose) {
            const float x = to_float(in[at]);
            r.raise(x, j.c);
            r.s += ex2((x - r.base()) * j.c);
            taken(composite(x, at));                // fewer than the list has room for
        }
    }

    uint4 next[kTopVecs];
#pragma unroll
    for (int i = 0; i < kTopVecs; ++i) {
        const uint32_t v = from + i * kTopThreads + tid;
        next[i] = v < to ? load16(in + cut.lead + v * N) : make_uint4(0, 0, 0, 0);
    }
    for (uint32_t v0 = from; v0 < to; v0 += kTopStep) {
        uint4 p[kTopVecs];
        float most[kTopVecs];
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < kTopVecs; ++i) {
            p[i] = next[i];
            const bool here = v0 + i * kTopThreads + tid < to;
            most[i] = here ? vec_max<T>(p[i]) : -INFINITY;
            top = fmaxf(top, most[i]);
            const uint32_t v = v0 + kTopStep + i * kTopThreads + tid;
            if (v < to) next[i] = load16(in + cut.lead + v * N);
        }
        if (v0 == from) {
            // bit by bit the largest number that k of the largest entries reach; its lower bits do not matter
            uint32_t key[kTopVecs];
            const bool fine = j.k > kTopThreads / 2;
#pragma unroll
            for (int i = 0; i < kTopVecs; ++i) key[i] = v0 + i * kTopThreads + tid < to ? order_of(most[i]) : 0;
            if (!fine) {
                key[0] = max(max(key[0], key[1]), max(key[2], key[3]));
                key[1] = key[2] = key[3] = 0;
            }
            uint32_t reach = 0;
            for (int b = 0; b < kBoundBits; ++b) {
                const uint32_t t = reach | 0x80000000u >> b;
                uint32_t n = __popc(__ballot_sync(~0u, key[0] >= t));
                if (fine)
#pragma unroll
                    for (int i = 1; i < kTopVecs; ++i) n += __popc(__ballot_sync(~0u, key[i] >= t));
                if (lane == 0 && n) atomicAdd(&s_above[b], n);
                __syncthreads();
                if (s_above[b] >= j.k) reach = t;
            }
            if (reach) bound = (static_cast<uint64_t>(reach) << 32) - 1, floor = floor_of(bound);
        }
        // the sum
        r.raise(top, j.c);
        const float base = r.base();
        if (fabsf(base) < 1e30f) {
            const float2 c2 = make_float2(j.c, j.c), shift = make_float2(-base * j.c, -base * j.c);
            float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < kTopVecs; ++i) {
                if (v0 + i * kTopThreads + tid >= to) continue;
                Packed<T, N> q;
                q.v[0] = p[i];
                float f[N];
                q.unpack(f);
#pragma unroll
                for (int e = 0; e < N; e += 2) {
                    const float2 y = fma2(make_float2(f[e], f[e + 1]), c2, shift);
                    sum = add2(sum, make_float2(ex2(y.x), ex2(y.y)));
                }
            }
            r.s += sum.x + sum.y;
        } else {                                    // products with c may be too large
#pragma unroll
            for (int i = 0; i < kTopVecs; ++i) {
                if (v0 + i * kTopThreads + tid >= to) continue;
                Packed<T, N> q;
                q.v[0] = p[i];
                float f[N];
                q.unpack(f);
#pragma unroll
                for (int e = 0; e < N; ++e) r.s += ex2((f[e] - base) * j.c);
            }
        }
        // the list
        uint32_t waiting = 0;
#pragma unroll
        for (int i = 0; i < kTopVecs; ++i) {
            const uint32_t v = v0 + i * kTopThreads + tid;
            if (v >= to || most[i] <= floor) continue;
            Packed<T, N> q;
            q.v[0] = p[i];
            float f[N];
            q.unpack(f);
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (!(f[e] <= floor) && !taken(composite(f[e], cut.lead + v * N + e))) waiting |= 1u << (i * N + e);
        }
        while (__syncthreads_or(grown || waiting)) {
            cut_back();
            grown = false;
            // what found no room, once more: rows in an unlucky order
            for (uint32_t left = waiting; left; left &= left - 1) {
                const uint32_t b = __ffs(left) - 1, at = cut.lead + (v0 + b / N * kTopThreads + tid) * N + b % N;
                if (taken(composite(to_float(in[at]), at))) waiting &= ~(1u << b);
            }
        }
    }
    __syncthreads();
    cut_back();

    r = warp_join(r, j.c);
    if (lane == 0) s_m[warp] = r.m, s_s[warp] = r.s;
    __syncthreads();
    if (tid == 0) {
        r = {-INFINITY, 0.0f};
        for (int w = 0; w < kTopThreads / 32; ++w) r.join(s_m[w], s_s[w], j.c);
        s_run = r;
    }
    if (ranks > 1) {
        cluster.sync();
        if (rank == 0) {
            for (uint32_t i0 = 0; i0 < (ranks - 1) * j.k; i0 += kTopThreads) {
                const uint32_t i = i0 + tid, other = 1 + i / j.k;
                uint64_t x = 0;
                if (i < (ranks - 1) * j.k && i % j.k < *cluster.map_shared_rank(&s_count, other)) x = cluster.map_shared_rank(s_list, other)[i % j.k];
                for (;;) {
                    if (x && taken(x)) x = 0;
                    if (!__syncthreads_or(x != 0)) break;
                    cut_back();
                }
            }
            cut_back();
            if (tid == 0)
                for (uint32_t o = 1; o < ranks; ++o) {
                    const Running other = *cluster.map_shared_rank(&s_run, o);
                    r.join(other.m, other.s, j.c);
                }
        }
        cluster.sync();                             // nobody leaves while the first block reads here
        if (rank != 0) return;
    }
    T* val = reinterpret_cast<T*>(j.val) + static_cast<uint64_t>(row) * j.k;
    int32_t* idx = j.idx + static_cast<uint64_t>(row) * j.k;
    for (uint32_t i = tid; i < j.k; i += kTopThreads) {
        const uint32_t token = 0xFFFFFFFFu - static_cast<uint32_t>(s_list[i]);
        idx[i] = static_cast<int32_t>(token);
        val[i] = in[token];
    }
    if (j.lse && tid == 0)
        j.lse[row] = static_cast<float>(r.s != r.s ? static_cast<double>(r.s) : r.m == -INFINITY ? -INFINITY : r.m * j.inv_t + log(static_cast<double>(r.s)));
}

// ---------------------------------------------------------------------------------------------- host side

bool good_temperature(float t) { return t >= 0x1p-20f && t <= 0x1p20f; }

template <typename T, int MODE> int launch_distill(const Job& j, cudaStream_t stream) {
    const size_t smem = (j.vocab + 31) / 32 * 4;
    ADACOMP_CUDA(cudaFuncSetAttribute(k_distill<T, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kMaxVocab / 8)));
    k_distill<T, MODE><<<j.n_rows, kThreads, smem, stream>>>(j);
    ADACOMP_LAUNCH_CHECK();
    return ADACOMP_OK;
}

template <int MODE>
int distill(adacomp_distill_t* h, const adacomp_rows_t* logits, uint32_t n_rows, const adacomp_pairs_t* pairs, float temperature,
            const float* d_weight, float* d_loss, float* d_stats, const adacomp_rows_t* out, void* cuda_stream) {
    if (!h || !pairs || !good_temperature(temperature) || n_rows >= (1u << 31)) return ADACOMP_ERR_INVALID;
    if (pairs->k == 0 || pairs->k > kMaxPairs) return ADACOMP_ERR_INVALID;
    Job j = {};
    int rc = rows_view(logits, n_rows, false, &j.logits);
    if (rc == ADACOMP_OK) rc = rows_view(&pairs->idx, n_rows, true, &j.idx);
    if (rc == ADACOMP_OK) rc = rows_view(&pairs->val, n_rows, false, &j.val);
    if (rc == ADACOMP_OK && MODE != kLoss) rc = rows_view(out, n_rows, false, &j.out);
    if (rc != ADACOMP_OK) return rc;
    if (MODE != kLoss && (j.out.type != j.logits.type || !rows_apart(j.out, n_rows, h->vocab))) return ADACOMP_ERR_INVALID;
    if (!aligned(pairs->d_lse, 4) || !aligned(d_weight, 4) || !aligned(d_loss, 4) || !aligned(d_stats, 16)) return ADACOMP_ERR_INVALID;
    if (MODE == kGrad && n_rows && !d_stats) return ADACOMP_ERR_INVALID;
    if (n_rows == 0) return ADACOMP_OK;
    j.lse = pairs->d_lse;
    j.weight = d_weight;
    j.loss = d_loss;
    j.stats = d_stats;
    j.status = h->d_status;
    j.n_rows = n_rows;
    j.vocab = h->vocab;
    j.k = pairs->k;
    j.c = static_cast<float>(kLog2e / temperature);
    j.inv_t = 1.0 / temperature;
    DeviceGuard guard(h->device);
    ADACOMP_CUDA(guard.err);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (j.logits.type == ADACOMP_F32) return launch_distill<float, MODE>(j, stream);
    if (j.logits.type == ADACOMP_BF16) return launch_distill<__nv_bfloat16, MODE>(j, stream);
    return launch_distill<__half, MODE>(j, stream);
}

template <typename T> int launch_top(const TopJob& j, uint32_t n_rows, int n_sms, cudaStream_t stream) {
    // several blocks a row as long as all of them are on the SMs at once and each has some steps to do
    uint32_t ranks = 1;
    while (ranks < kTopCluster && static_cast<uint64_t>(n_rows) * ranks * 2 <= 4ull * n_sms &&
           j.vocab * sizeof(T) / 16 >= static_cast<uint64_t>(ranks) * 2 * kTopStep)
        ranks *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(n_rows * ranks);
    cfg.blockDim = dim3(kTopThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ranks;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = ranks > 1 ? 1 : 0;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k_top_logits<T>, j);
    if (e != cudaSuccess) return cuda_fail(e);
    ADACOMP_LAUNCH_CHECK();
    return ADACOMP_OK;
}

}  // namespace

extern "C" {

int adacomp_distill_workspace_bytes(uint32_t vocab, size_t* bytes_out) {
    if (!bytes_out || vocab == 0 || vocab > kMaxVocab) return ADACOMP_ERR_INVALID;
    *bytes_out = kAlign;
    return ADACOMP_OK;
}

int adacomp_distill_create(adacomp_distill_t** h, uint32_t vocab, void* d_workspace, size_t workspace_bytes, int device) {
    if (!h) return ADACOMP_ERR_INVALID;
    *h = nullptr;
    size_t need = 0;
    const int rc = adacomp_distill_workspace_bytes(vocab, &need);
    if (rc != ADACOMP_OK) return rc;
    if (!d_workspace || !aligned(d_workspace, kAlign)) return ADACOMP_ERR_INVALID;
    if (need > workspace_bytes) return ADACOMP_ERR_ALLOC;
    adacomp_distill_t* d = new (std::nothrow) adacomp_distill_t;
    if (!d) return ADACOMP_ERR_ALLOC;
    d->device = device;
    d->vocab = vocab;
    d->d_status = static_cast<int*>(d_workspace);
    DeviceGuard guard(device);
    cudaError_t err = guard.err;
    if (err == cudaSuccess) err = cudaDeviceGetAttribute(&d->n_sms, cudaDevAttrMultiProcessorCount, device);
    if (err == cudaSuccess) err = cudaMemset(d->d_status, 0, sizeof(int));
    if (err == cudaSuccess) err = cudaStreamSynchronize(nullptr);
    if (err != cudaSuccess) {
        delete d;
        return cuda_fail(err);
    }
    *h = d;
    return ADACOMP_OK;
}

int adacomp_top_logits(adacomp_distill_t* h, const adacomp_rows_t* logits, uint32_t n_rows, uint32_t k, float temperature,
                       int32_t* d_idx_out, void* d_val_out, float* d_lse_out, void* cuda_stream) {
    if (!h || n_rows >= (1u << 31) || !good_temperature(temperature)) return ADACOMP_ERR_INVALID;
    if (k == 0 || k > kMaxPairs || k > h->vocab) return ADACOMP_ERR_INVALID;
    TopJob j = {};
    const int rc = rows_view(logits, n_rows, false, &j.logits);
    if (rc != ADACOMP_OK) return rc;
    if (n_rows && (!d_idx_out || !d_val_out)) return ADACOMP_ERR_INVALID;
    if (!aligned(d_idx_out, 4) || !aligned(d_val_out, type_size(j.logits.type)) || !aligned(d_lse_out, 4)) return ADACOMP_ERR_INVALID;
    if (n_rows == 0) return ADACOMP_OK;
    j.idx = d_idx_out;
    j.val = d_val_out;
    j.lse = d_lse_out;
    j.vocab = h->vocab;
    j.k = k;
    j.c = static_cast<float>(kLog2e / temperature);
    j.inv_t = 1.0 / temperature;
    DeviceGuard guard(h->device);
    ADACOMP_CUDA(guard.err);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (j.logits.type == ADACOMP_F32) return launch_top<float>(j, n_rows, h->n_sms, stream);
    if (j.logits.type == ADACOMP_BF16) return launch_top<__nv_bfloat16>(j, n_rows, h->n_sms, stream);
    return launch_top<__half>(j, n_rows, h->n_sms, stream);
}

int adacomp_distill_loss(adacomp_distill_t* h, const adacomp_rows_t* logits, uint32_t n_rows, const adacomp_pairs_t* pairs,
                         float temperature, const float* d_weight, float* d_loss_out, float* d_stats_out, void* cuda_stream) {
    return distill<kLoss>(h, logits, n_rows, pairs, temperature, d_weight, d_loss_out, d_stats_out, nullptr, cuda_stream);
}

int adacomp_distill_grad(adacomp_distill_t* h, const adacomp_rows_t* logits, uint32_t n_rows, const adacomp_pairs_t* pairs,
                         float temperature, const float* d_weight, const float* d_stats, const adacomp_rows_t* out, void* cuda_stream) {
    return distill<kGrad>(h, logits, n_rows, pairs, temperature, d_weight, nullptr, const_cast<float*>(d_stats), out, cuda_stream);
}

int adacomp_distill_loss_grad(adacomp_distill_t* h, const adacomp_rows_t* logits, uint32_t n_rows, const adacomp_pairs_t* pairs,
                              float temperature, const float* d_weight, float* d_loss_out, const adacomp_rows_t* out, void* cuda_stream) {
    return distill<kBoth>(h, logits, n_rows, pairs, temperature, d_weight, d_loss_out, nullptr, out, cuda_stream);
}

int adacomp_distill_last_error(adacomp_distill_t* h, void* cuda_stream) {
    if (!h) return ADACOMP_ERR_INVALID;
    DeviceGuard guard(h->device);
    ADACOMP_CUDA(guard.err);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    int status = 0;
    ADACOMP_CUDA(cudaMemcpyAsync(&status, h->d_status, sizeof(int), cudaMemcpyDeviceToHost, stream));
    ADACOMP_CUDA(cudaMemsetAsync(h->d_status, 0, sizeof(int), stream));
    ADACOMP_CUDA(cudaStreamSynchronize(stream));
    return status;
}

int adacomp_distill_destroy(adacomp_distill_t* h) {
    delete h;
    return ADACOMP_OK;
}

}  // extern "C"
