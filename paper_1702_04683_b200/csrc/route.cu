// Routing of tokens to experts, and the gradient of the router's logits.
//
//   s = softmax(l) or 1 / (1 + exp(-l)); chosen by s + b: the best groups, then the top_k largest values in them
//   w_i = scale s_i, or scale s_i / (sum of the chosen s)
//
// The gradient, with d_i = scale dw_i and S the sum of the chosen scores:
//   ds_i = d_i, or (d_i - (sum d s) / S) / S;      dl_i = ds_i s_i (1 - s_i)  (sigmoid)
//   softmax: dl_e = s_e (ds_e - sum ds s); renormalised this vanishes outside of the chosen ones and is a softmax's over those
//
// A row is a warp's work.  Rows are short: large calls are bound by instruction issue (the rounds of the choice), small ones
// by the launch.
#include <math.h>
#include <new>

#include "rows.cuh"

using namespace adacomp;

struct adacomp_route {
    int device;
    adacomp_route_config_t config;
    int n_sms;
    int* d_status;
    uint32_t* d_ticket;             // blocks of a call that are through
    uint32_t* d_counts;             // [experts], zero between calls
};

namespace {

constexpr int kWarps = 4;
constexpr uint32_t kMaxExperts = 1024;
constexpr uint32_t kMaxChosen = 32;
constexpr uint32_t kMaxGroups = 32;

struct Job {
    Rows logits, out;
    adacomp_route_config_t cfg;
    const float* bias;
    const uint8_t* live;
    int32_t* experts;
    float* weights;                 // or their gradient
    uint32_t* counts_out;
    uint32_t* counts;
    uint32_t* ticket;
    int* status;
    uint32_t n_rows;
};

template <typename V> __device__ __forceinline__ V warp_sum(V x) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    return x;
}

template <typename V> __device__ __forceinline__ V warp_max(V x) {
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        const V y = __shfl_xor_sync(~0u, x, d);
        x = y > x ? y : x;
    }
    return x;
}

// The choice among a row's values s_v[0 .. experts) (-Inf: cannot be chosen), which are used up.  Lane i < top_k returns its place's
// expert, or -1.  The result tells whether two candidates that a decision hung on lie within `tol` of each other, other than by having
// the same logit and bias, which makes the decision one for a finer computation.
template <typename V, typename T>
__device__ bool choose(V* s_v, const T* logits, const float* bias, const adacomp_route_config_t& cfg, V tol, int* expert) {
    const uint32_t lane = threadIdx.x % 32, size = cfg.experts / cfg.groups;
    const V none = -INFINITY;
    uint32_t kept = ~0u;
    bool close = false;
    if (cfg.top_groups < cfg.groups) {
        V rating = none;
        if (lane < cfg.groups) {
            V first = none, second = none;
            for (uint32_t e = lane * size; e < (lane + 1) * size; ++e) {
                const V v = s_v[e];
                if (v > first) second = first, first = v;
                else if (v > second) second = v;
            }
            rating = cfg.group_terms == 2 && second != none ? first + second : first;
        }
        uint32_t better = 0;
        for (uint32_t g = 0; g < cfg.groups; ++g) {
            const V other = __shfl_sync(~0u, rating, g);
            better += other > rating || (other == rating && g < lane);
        }
        const bool in = lane < cfg.groups && better < cfg.top_groups;
        kept = __ballot_sync(~0u, in);
        const V least = -warp_max(in ? -rating : none), most = warp_max(lane < cfg.groups && !in ? rating : none);
        close = least - most <= 2 * tol;
    }
    V mine = none, last = none;
    int id = -1, last_id = -1;
    const uint32_t rounds = min(cfg.top_k + (tol > 0), cfg.experts);
    for (uint32_t r = 0; r < rounds; ++r) {
        V best = none;
        int at = INT_MAX;
        for (uint32_t e = lane; e < cfg.experts; e += 32)
            if (kept >> (e / size) & 1 && s_v[e] > best) best = s_v[e], at = static_cast<int>(e);
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            const V v = __shfl_xor_sync(~0u, best, d);
            const int a = __shfl_xor_sync(~0u, at, d);
            if (v > best || (v == best && a < at)) best = v, at = a;
        }
        if (best == none) break;
        // candidates come in falling order: close ones are neighbours
        if (r > 0 && last - best <= tol)
            close |= !(to_float(logits[at]) == to_float(logits[last_id]) && (!bias || bias[at] == bias[last_id]));
        last = best, last_id = at;
        if (lane == r) mine = best, id = at;
        __syncwarp();
        if (lane == 0) s_v[at] = none;
        __syncwarp();
    }
    *expert = lane < cfg.top_k && mine != none ? id : -1;
    return close;
}

// A chosen expert's score s (logit x; -Inf in lanes without one) divided by the sum over the warp.  Sigmoids that fp32 has no
// numbers for, or few bits, are exp(x) to all of its bits: their quotients are those of exp(x - the largest x).
__device__ __forceinline__ float quotient(float s, float x, bool soft) {
    float sum = warp_sum(s);
    if (!soft && sum < 0x1p-90f) {
        const float top = warp_max(x);
        s = x == -INFINITY ? 0.0f : expf(x - top);
        sum = warp_sum(s);
    }
    return sum > 0.0f ? s / sum : 0.0f;
}

template <typename T>
__global__ void __launch_bounds__(kWarps * 32) k_route(const Job j) {
    extern __shared__ double s_rows[];                      // a row of values per warp, then the counts
    __shared__ bool s_last;
    const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, E = j.cfg.experts, K = j.cfg.top_k;
    double* s_wide = s_rows + warp * E;
    float* s_v = reinterpret_cast<float*>(s_wide);
    uint32_t* s_counts = reinterpret_cast<uint32_t*>(s_rows + kWarps * E);
    for (uint32_t e = threadIdx.x; e < E; e += kWarps * 32) s_counts[e] = 0;
    __syncthreads();
    const bool soft = j.cfg.score == ADACOMP_SOFTMAX;
    for (uint32_t row = blockIdx.x * kWarps + warp; row < j.n_rows; row += gridDim.x * kWarps) {
        int id = -1;
        float w = 0.0f;
        if (!j.live || j.live[row]) {
            const T* l = reinterpret_cast<const T*>(j.logits.data) + j.logits.offset(row);
            float most = -INFINITY, bias_most = 0.0f, total = 0.0f;
            bool bad = false;
            for (uint32_t e = lane; e < E; e += 32) {
                const float x = to_float(l[e]), b = j.bias ? j.bias[e] : 0.0f;
                bad |= x != x || b != b || (soft && x == INFINITY);
                most = fmaxf(most, x);
                if (b != -INFINITY) bias_most = fmaxf(bias_most, fabsf(b));
                s_v[e] = x;
            }
            bad = __any_sync(~0u, bad);
            if (!bad) {
                most = warp_max(most);
                bias_most = warp_max(bias_most);
                const float base = most == -INFINITY ? 0.0f : most;
                for (uint32_t e = lane; e < E; e += 32) {
                    const float x = s_v[e], y = soft ? expf(x - base) : 1.0f / (1.0f + expf(-x));
                    total += y;
                    s_v[e] = x == -INFINITY ? -INFINITY : y;
                }
                total = warp_sum(total);
                const float unit = soft ? 1.0f / total : 1.0f;
                for (uint32_t e = lane; e < E; e += 32) s_v[e] = s_v[e] * unit + (j.bias ? j.bias[e] : 0.0f);
                __syncwarp();
                // scores are off by some rounding steps of the largest: 16 of them are allowed for
                const float tol = (unit + bias_most) * 0x1p-20f;
                if (choose<float, T>(s_v, l, j.bias, j.cfg, tol, &id)) {
                    double sum = 0.0;
                    __syncwarp();
                    for (uint32_t e = lane; e < E; e += 32) {
                        const double x = to_float(l[e]), y = soft ? exp(x - base) : 1.0 / (1.0 + exp(-x));
                        sum += y;
                        s_wide[e] = x == -INFINITY ? -INFINITY : y;
                    }
                    sum = warp_sum(sum);
                    for (uint32_t e = lane; e < E; e += 32)
                        s_wide[e] = (soft ? s_wide[e] / sum : s_wide[e]) + (j.bias ? static_cast<double>(j.bias[e]) : 0.0);
                    __syncwarp();
                    choose<double, T>(s_wide, l, j.bias, j.cfg, 0.0, &id);
                }
                const float x = id >= 0 ? to_float(l[id]) : -INFINITY;
                float s;
                if (!soft) s = 1.0f / (1.0f + expf(-x));
                else if (j.cfg.renormalize) s = expf(x - warp_max(x));           // relative to the largest chosen one
                else s = expf(x - base) / total;
                if (id < 0) s = 0.0f;
                if (j.cfg.renormalize) s = quotient(s, x, soft);
                w = s * j.cfg.scale;
            } else {
                w = NAN;
            }
            __syncwarp();
        }
        if (lane < K) {
            j.experts[static_cast<uint64_t>(row) * K + lane] = id;
            j.weights[static_cast<uint64_t>(row) * K + lane] = w;
            if (id >= 0) atomicAdd(&s_counts[id], 1u);
        }
    }
    if (!j.counts_out) return;
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < E; e += kWarps * 32)
        if (s_counts[e]) atomicAdd(&j.counts[e], s_counts[e]);
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) s_last = atomicAdd(j.ticket, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    for (uint32_t e = threadIdx.x; e < E; e += kWarps * 32) {
        j.counts_out[e] = __ldcg(&j.counts[e]);
        j.counts[e] = 0;
    }
    if (threadIdx.x == 0) *j.ticket = 0;
}

template <typename T>
__global__ void __launch_bounds__(kWarps * 32) k_route_grad(const Job j) {
    extern __shared__ float s_grads[];
    const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, E = j.cfg.experts, K = j.cfg.top_k;
    float* s_g = s_grads + warp * E;
    const bool soft = j.cfg.score == ADACOMP_SOFTMAX;
    for (uint32_t row = blockIdx.x * kWarps + warp; row < j.n_rows; row += gridDim.x * kWarps) {
        const T* l = reinterpret_cast<const T*>(j.logits.data) + j.logits.offset(row);
        T* out = reinterpret_cast<T*>(j.out.data) + j.out.offset(row);
        int id = lane < K ? j.experts[static_cast<uint64_t>(row) * K + lane] : -1;
        if (id >= static_cast<int>(E)) record_error(j.status, ADACOMP_ERR_INVALID), id = -1;
        __syncwarp();
        const uint32_t same = __match_any_sync(~0u, id >= 0 ? id : -1 - static_cast<int>(lane));
        if (id < 0 || lane != static_cast<uint32_t>(__ffs(same)) - 1) id = -1;
        const float x = id >= 0 ? to_float(l[id]) : -INFINITY;
        const float d = id >= 0 ? j.weights[static_cast<uint64_t>(row) * K + lane] * j.cfg.scale : 0.0f;
        const bool any = __any_sync(~0u, id >= 0), dense = any && soft && !j.cfg.renormalize;
        float total = 1.0f, base = 0.0f, common = 0.0f;
        if (dense) {
            float most = -INFINITY;
            for (uint32_t e = lane; e < E; e += 32) most = fmaxf(most, to_float(l[e]));
            most = warp_max(most);
            base = most == -INFINITY ? 0.0f : most;
            total = 0.0f;
            for (uint32_t e = lane; e < E; e += 32) total += expf(to_float(l[e]) - base);
            total = warp_sum(total);
        }
        float g = 0.0f;
        if (!soft) {
            float s = id >= 0 ? 1.0f / (1.0f + expf(-x)) : 0.0f;
            const float rest = 1.0f / (1.0f + expf(x));
            if (j.cfg.renormalize) {
                s = quotient(s, x, false);
                g = (d - warp_sum(d * s)) * s * rest;
            } else {
                g = d * s * rest;
            }
        } else if (j.cfg.renormalize) {
            const float top = warp_max(x), s = quotient(id >= 0 ? expf(x - top) : 0.0f, x, true);
            g = s * (d - warp_sum(d * s));
        } else {
            const float s = id >= 0 ? expf(x - base) / total : 0.0f;
            common = warp_sum(d * s);
            g = s * (d - common);
        }
        for (uint32_t e = lane; e < E; e += 32) s_g[e] = dense ? -(expf(to_float(l[e]) - base) / total) * common : 0.0f;
        __syncwarp();
        if (id >= 0) s_g[id] = g;
        __syncwarp();
        for (uint32_t e = lane; e < E; e += 32) out[e] = from_float<T>(s_g[e]);
        __syncwarp();
    }
}

// ---------------------------------------------------------------------------------------------- host side

int check_config(const adacomp_route_config_t* c) {
    if (!c || c->experts == 0 || c->experts > kMaxExperts || c->groups == 0 || c->groups > kMaxGroups || c->experts % c->groups != 0)
        return ADACOMP_ERR_INVALID;
    if (c->top_groups == 0 || c->top_groups > c->groups || c->group_terms == 0 || c->group_terms > 2) return ADACOMP_ERR_INVALID;
    if (c->top_k == 0 || c->top_k > kMaxChosen || c->top_k > c->experts / c->groups * c->top_groups) return ADACOMP_ERR_INVALID;
    if ((c->score != ADACOMP_SOFTMAX && c->score != ADACOMP_SIGMOID) || (c->renormalize != 0 && c->renormalize != 1) || !isfinite(c->scale))
        return ADACOMP_ERR_INVALID;
    return ADACOMP_OK;
}

size_t carve(adacomp_route_t* h, void* base, uint32_t experts) {
    Carver c(base);
    int* status = c.take<int>(1);
    uint32_t* ticket = c.take<uint32_t>(1);
    uint32_t* counts = c.take<uint32_t>(experts);
    if (h) h->d_status = status, h->d_ticket = ticket, h->d_counts = counts;
    return c.used;
}

uint32_t grid_of(const adacomp_route_t* h, uint32_t n_rows) {
    const uint32_t most = static_cast<uint32_t>(h->n_sms) * 8, need = (n_rows + kWarps - 1) / kWarps;
    return need < most ? need : most;
}

template <typename T> int launch_route(const Job& j, uint32_t blocks, cudaStream_t stream) {
    const size_t smem = kWarps * j.cfg.experts * sizeof(double) + j.cfg.experts * sizeof(uint32_t);
    k_route<T><<<blocks, kWarps * 32, smem, stream>>>(j);
    ADACOMP_LAUNCH_CHECK();
    return ADACOMP_OK;
}

template <typename T> int launch_grad(const Job& j, uint32_t blocks, cudaStream_t stream) {
    k_route_grad<T><<<blocks, kWarps * 32, kWarps * j.cfg.experts * sizeof(float), stream>>>(j);
    ADACOMP_LAUNCH_CHECK();
    return ADACOMP_OK;
}

}  // namespace

extern "C" {

int adacomp_route_workspace_bytes(const adacomp_route_config_t* config, size_t* bytes_out) {
    if (!bytes_out) return ADACOMP_ERR_INVALID;
    const int rc = check_config(config);
    if (rc != ADACOMP_OK) return rc;
    *bytes_out = carve(nullptr, nullptr, config->experts);
    return ADACOMP_OK;
}

int adacomp_route_create(adacomp_route_t** h, const adacomp_route_config_t* config, void* d_workspace, size_t workspace_bytes, int device) {
    if (!h) return ADACOMP_ERR_INVALID;
    *h = nullptr;
    size_t need = 0;
    const int rc = adacomp_route_workspace_bytes(config, &need);
    if (rc != ADACOMP_OK) return rc;
    if (!d_workspace || !aligned(d_workspace, kAlign)) return ADACOMP_ERR_INVALID;
    if (need > workspace_bytes) return ADACOMP_ERR_ALLOC;
    adacomp_route_t* r = new (std::nothrow) adacomp_route_t;
    if (!r) return ADACOMP_ERR_ALLOC;
    r->device = device;
    r->config = *config;
    carve(r, d_workspace, config->experts);
    DeviceGuard guard(device);
    cudaError_t err = guard.err;
    if (err == cudaSuccess) err = cudaDeviceGetAttribute(&r->n_sms, cudaDevAttrMultiProcessorCount, device);
    if (err == cudaSuccess) err = cudaMemset(d_workspace, 0, need);
    if (err == cudaSuccess) err = cudaStreamSynchronize(nullptr);
    if (err != cudaSuccess) {
        delete r;
        return cuda_fail(err);
    }
    *h = r;
    return ADACOMP_OK;
}

int adacomp_route(adacomp_route_t* h, const adacomp_rows_t* logits, uint32_t n_rows, const float* d_bias, const uint8_t* d_live,
                  int32_t* d_experts_out, float* d_weights_out, uint32_t* d_counts_out, void* cuda_stream) {
    if (!h || n_rows >= (1u << 31)) return ADACOMP_ERR_INVALID;
    Job j = {};
    const int rc = rows_view(logits, n_rows, false, &j.logits);
    if (rc != ADACOMP_OK) return rc;
    if (n_rows && (!d_experts_out || !d_weights_out)) return ADACOMP_ERR_INVALID;
    if (!aligned(d_bias, 4) || !aligned(d_experts_out, 4) || !aligned(d_weights_out, 4) || !aligned(d_counts_out, 4)) return ADACOMP_ERR_INVALID;
    DeviceGuard guard(h->device);
    ADACOMP_CUDA(guard.err);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (n_rows == 0) {
        if (d_counts_out) ADACOMP_CUDA(cudaMemsetAsync(d_counts_out, 0, h->config.experts * sizeof(uint32_t), stream));
        return ADACOMP_OK;
    }
    j.cfg = h->config;
    j.bias = d_bias;
    j.live = d_live;
    j.experts = d_experts_out;
    j.weights = d_weights_out;
    j.counts_out = d_counts_out;
    j.counts = h->d_counts;
    j.ticket = h->d_ticket;
    j.status = h->d_status;
    j.n_rows = n_rows;
    const uint32_t blocks = grid_of(h, n_rows);
    if (j.logits.type == ADACOMP_F32) return launch_route<float>(j, blocks, stream);
    if (j.logits.type == ADACOMP_BF16) return launch_route<__nv_bfloat16>(j, blocks, stream);
    return launch_route<__half>(j, blocks, stream);
}

int adacomp_route_grad(adacomp_route_t* h, const adacomp_rows_t* logits, uint32_t n_rows, const int32_t* d_experts,
                       const float* d_grad_weights, const adacomp_rows_t* out, void* cuda_stream) {
    if (!h || n_rows >= (1u << 31)) return ADACOMP_ERR_INVALID;
    Job j = {};
    int rc = rows_view(logits, n_rows, false, &j.logits);
    if (rc == ADACOMP_OK) rc = rows_view(out, n_rows, false, &j.out);
    if (rc != ADACOMP_OK) return rc;
    if (j.out.type != j.logits.type || !rows_apart(j.out, n_rows, h->config.experts)) return ADACOMP_ERR_INVALID;
    if (n_rows && (!d_experts || !d_grad_weights)) return ADACOMP_ERR_INVALID;
    if (!aligned(d_experts, 4) || !aligned(d_grad_weights, 4)) return ADACOMP_ERR_INVALID;
    if (n_rows == 0) return ADACOMP_OK;
    j.cfg = h->config;
    j.experts = const_cast<int32_t*>(d_experts);
    j.weights = const_cast<float*>(d_grad_weights);
    j.status = h->d_status;
    j.n_rows = n_rows;
    DeviceGuard guard(h->device);
    ADACOMP_CUDA(guard.err);
    const uint32_t blocks = grid_of(h, n_rows);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (j.logits.type == ADACOMP_F32) return launch_grad<float>(j, blocks, stream);
    if (j.logits.type == ADACOMP_BF16) return launch_grad<__nv_bfloat16>(j, blocks, stream);
    return launch_grad<__half>(j, blocks, stream);
}

int adacomp_route_last_error(adacomp_route_t* h, void* cuda_stream) {
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

int adacomp_route_destroy(adacomp_route_t* h) {
    delete h;
    return ADACOMP_OK;
}

}  // extern "C"
