// Embedding tables: lookup with scaling, and the gradient by sorted tokens.
//
//   lookup    out_t = round(s E[token_t])
//   gradient  dE[w][v] = s sum of the gradient rows of worker w's tokens that equal v
//
// The gradient sorts the pairs (worker * vocab + token, position), stable, so a row's summands stand together and in
// order; every row is then summed by whoever owns it, without atomics.  All of it is bound by HBM (one fp32 addition per
// entry read).
#include <math.h>
#include <new>

#include "numeric.cuh"

using namespace adacomp;

struct adacomp_embed {
    int device;
    uint32_t vocab, dim, max_tokens, max_workers, padding;
    int n_sms;
    int* d_status;
    uint32_t* d_key[2];             // [max_tokens] worker * vocab + token, before and after a pass of the sort
    uint32_t* d_pos[2];             // [max_tokens] which token it is
    uint32_t* d_table;              // [tiles][256] digit counts per tile, then their places
    uint32_t* d_seg_begin;          // [max_tokens + 1] first sorted token of every distinct one
    uint32_t* d_seg_key;            // [max_tokens]
    uint32_t* d_n_segs;
};

namespace {

constexpr int kThreads = 256;
constexpr int kSortItems = 8;
constexpr uint32_t kTile = kThreads * kSortItems;           // tokens per block of the sort
constexpr int kBins = 256;

// Device view of adacomp_rows_t.
struct Rows {
    char* data;
    int type;
    uint32_t group;
    uint64_t row_stride, group_stride;
    __device__ __forceinline__ uint64_t offset(uint32_t r) const {
        return group == 0 ? r * row_stride : (r / group) * group_stride + (r % group) * row_stride;
    }
};

// A token as it is stored; what does not fit `vocab` comes out as UINT32_MAX.
__device__ __forceinline__ uint32_t load_token(const Rows& tokens, uint32_t t, uint32_t vocab) {
    const uint64_t at = tokens.offset(t);
    uint64_t v;
    if (tokens.type == ADACOMP_I64) v = reinterpret_cast<const uint64_t*>(tokens.data)[at];
    else v = reinterpret_cast<const uint32_t*>(tokens.data)[at];
    return v < vocab ? static_cast<uint32_t>(v) : 0xFFFFFFFFu;      // negative numbers are large ones here
}

// ---------------------------------------------------------------------------------------------- lookup

// Threads of a block: x along a row, y over rows.
template <typename A, typename B, int N>
__global__ void __launch_bounds__(kThreads) k_embed_lookup(Rows table, Rows tokens, Rows out, uint32_t n_tokens, uint32_t vocab,
                                                            uint32_t dim, float scale, int* status) {
    const uint32_t t = blockIdx.x * blockDim.y + threadIdx.y;
    if (t >= n_tokens) return;
    const uint32_t v = load_token(tokens, t, vocab);
    B* dst = reinterpret_cast<B*>(out.data) + out.offset(t);
    const A* src = reinterpret_cast<const A*>(table.data) + static_cast<uint64_t>(v) * table.row_stride;
    if (v == 0xFFFFFFFFu && threadIdx.x == 0) record_error(status, ADACOMP_ERR_INVALID);
    for (uint32_t c = (blockIdx.y * blockDim.x + threadIdx.x) * N; c < dim; c += gridDim.y * blockDim.x * N) {
        float f[N];
#pragma unroll
        for (int j = 0; j < N; ++j) f[j] = 0.f;
        if (v != 0xFFFFFFFFu) {
            if constexpr (N > 1) {
                Packed<A, N> p;
                p.load(src + c);
                p.unpack(f);
            } else {
                f[0] = to_float(src[c]);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] = __fmul_rn(f[j], scale);
        }
        if constexpr (N > 1) {
            Packed<B, N> q;
            q.pack(f);
            q.store(dst + c);
        } else {
            dst[c] = from_float<B>(f[0]);
        }
    }
}

// ---------------------------------------------------------------------------------------------- sort

__global__ void __launch_bounds__(kThreads) k_embed_keys(Rows tokens, uint32_t n, uint32_t n_tokens, uint32_t vocab, uint32_t padding,
                                                          uint32_t none, uint32_t* key, uint32_t* pos, int* status) {
    const uint32_t t = blockIdx.x * kThreads + threadIdx.x;
    if (t >= n) return;
    const uint32_t v = load_token(tokens, t, vocab);
    if (v == 0xFFFFFFFFu) record_error(status, ADACOMP_ERR_INVALID);
    key[t] = v == 0xFFFFFFFFu || v == padding ? none : (t / n_tokens) * vocab + v;
    pos[t] = t;
}

__global__ void __launch_bounds__(kThreads) k_radix_count(const uint32_t* key, uint32_t n, int shift, uint32_t* table) {
    __shared__ uint32_t s_count[kBins];
    s_count[threadIdx.x] = 0;
    __syncthreads();
    for (int i = 0; i < kSortItems; ++i) {
        const uint32_t t = blockIdx.x * kTile + i * kThreads + threadIdx.x;
        if (t < n) atomicAdd(&s_count[(key[t] >> shift) & (kBins - 1)], 1u);
    }
    __syncthreads();
    table[threadIdx.x * gridDim.x + blockIdx.x] = s_count[threadIdx.x];     // digit-major: one running total over it gives the places
}

// Inclusive sum over the block's 1024 threads.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* s_warp) {
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, v, d);
        if (lane >= static_cast<uint32_t>(d)) v += y;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = v;
    __syncthreads();
    uint32_t before = 0;
    for (uint32_t k = 0; k < warp; ++k) before += s_warp[k];
    return v + before;
}

// In place: counts become the totals before them; *total (if any) their sum.
__global__ void __launch_bounds__(1024) k_running_total(uint32_t* a, uint32_t n, uint32_t* total) {
    __shared__ uint32_t s_warp[32];
    __shared__ uint32_t s_carry;
    if (threadIdx.x == 0) s_carry = 0;
    __syncthreads();
    for (uint32_t base = 0; base < n; base += 1024) {
        const uint32_t i = base + threadIdx.x;
        const uint32_t v = i < n ? a[i] : 0;
        const uint32_t upto = block_scan(v, s_warp) + s_carry;
        if (i < n) a[i] = upto - v;
        __syncthreads();
        if (threadIdx.x == 1023) s_carry = upto;
        __syncthreads();
    }
    if (total && threadIdx.x == 0) *total = s_carry;
}

__global__ void __launch_bounds__(kThreads) k_radix_scatter(const uint32_t* key, const uint32_t* pos, uint32_t n, int shift,
                                                             const uint32_t* table, uint32_t* key_out, uint32_t* pos_out) {
    __shared__ uint32_t s_place[kThreads / 32][kBins];      // how many of a digit the warps before have, then places
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (uint32_t d = lane; d < kBins; d += 32) s_place[warp][d] = 0;
    __syncwarp();
    uint32_t k[kSortItems], rank[kSortItems];
    const uint32_t base = blockIdx.x * kTile + warp * (32 * kSortItems) + lane;
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
        const uint32_t t = base + i * 32;
        k[i] = t < n ? key[t] : 0xFFFFFFFFu;
        const uint32_t d = (k[i] >> shift) & (kBins - 1);
        uint32_t same = __ballot_sync(0xFFFFFFFFu, t < n);
        if (t >= n) same = ~same;
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const uint32_t vote = __ballot_sync(0xFFFFFFFFu, (d >> b) & 1);
            same &= (d >> b) & 1 ? vote : ~vote;
        }
        const uint32_t before = __popc(same & ((1u << lane) - 1));
        rank[i] = s_place[warp][d] + before;
        __syncwarp();
        if (t < n && before == 0) s_place[warp][d] += __popc(same);
        __syncwarp();
    }
    __syncthreads();
    uint32_t at = table[threadIdx.x * gridDim.x + blockIdx.x];
    for (int w = 0; w < kThreads / 32; ++w) {
        const uint32_t c = s_place[w][threadIdx.x];
        s_place[w][threadIdx.x] = at;
        at += c;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSortItems; ++i) {
        const uint32_t t = base + i * 32;
        if (t >= n) continue;
        const uint32_t to = s_place[warp][(k[i] >> shift) & (kBins - 1)] + rank[i];
        key_out[to] = k[i];
        pos_out[to] = pos[t];
    }
}

// ---------------------------------------------------------------------------------------------- segments

__device__ __forceinline__ bool is_head(const uint32_t* key, uint32_t i, uint32_t none) {
    return key[i] != none && (i == 0 || key[i - 1] != key[i]);
}

__global__ void __launch_bounds__(kThreads) k_heads_count(const uint32_t* key, uint32_t n, uint32_t none, uint32_t* count) {
    int c = 0;
    for (int i = 0; i < kSortItems; ++i) {
        const uint32_t t = blockIdx.x * kTile + i * kThreads + threadIdx.x;
        c += __syncthreads_count(t < n && is_head(key, t, none));
    }
    if (threadIdx.x == 0) count[blockIdx.x] = c;
}

__global__ void __launch_bounds__(1024) k_heads_emit(const uint32_t* key, uint32_t n, uint32_t none, const uint32_t* place, uint32_t* seg_begin,
                                                      uint32_t* seg_key, uint32_t* n_segs) {
    __shared__ uint32_t s_warp[32];
    uint32_t carry = place[blockIdx.x];
    for (uint32_t base = blockIdx.x * kTile; base < n && base < (blockIdx.x + 1) * kTile; base += 1024) {
        const uint32_t t = base + threadIdx.x;
        const bool head = t < n && is_head(key, t, none);
        const uint32_t upto = carry + block_scan(head, s_warp);
        if (head) {
            seg_begin[upto - 1] = t;
            seg_key[upto - 1] = key[t];
        }
        // the last segment ends where the tokens without a gradient begin, or with the list
        if (t < n && key[t] != none && (t + 1 == n || key[t + 1] == none)) seg_begin[upto] = t + 1;
        carry += __syncthreads_count(head);
    }
    (void)n_segs;
}

__global__ void k_row_begin(const uint32_t* seg_key, const uint32_t* n_segs, uint32_t n_workers, uint32_t vocab, uint64_t* row_begin) {
    const uint32_t w = blockIdx.x * blockDim.x + threadIdx.x;
    if (w > n_workers) return;
    const uint64_t bound = static_cast<uint64_t>(w) * vocab;
    uint32_t lo = 0, hi = *n_segs;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (seg_key[mid] < bound) lo = mid + 1; else hi = mid;
    }
    row_begin[w] = lo;
}

// ---------------------------------------------------------------------------------------------- sums

struct Sums {
    const uint32_t *pos, *seg_begin, *seg_key, *n_segs;
    Rows grad;
    uint32_t dim, vocab;
    float scale;
    // rows form
    uint32_t* rows_out;
    char* values;
    uint32_t* idx_out;
    uint32_t idx_offset;
    // dense form
    int dense, accumulate;
    Rows out;
};

template <typename A, typename B, int N>
__global__ void __launch_bounds__(kThreads) k_embed_sums(const Sums p) {
    const uint32_t n_segs = *p.n_segs;
    for (uint32_t u = blockIdx.x * blockDim.y + threadIdx.y; u < n_segs; u += gridDim.x * blockDim.y) {
        const uint32_t from = p.seg_begin[u], to = p.seg_begin[u + 1], key = p.seg_key[u];
        if (p.rows_out && threadIdx.x == 0) p.rows_out[u] = key % p.vocab;
        B* dst = p.dense ? reinterpret_cast<B*>(p.out.data) + p.out.offset(key)
                         : reinterpret_cast<B*>(p.values) + static_cast<uint64_t>(u) * p.dim;
        for (uint32_t c = threadIdx.x * N; c < p.dim; c += blockDim.x * N) {
            float sum[N];
#pragma unroll
            for (int j = 0; j < N; ++j) sum[j] = 0.f;
            for (uint32_t i = from; i < to; ++i) {
                const A* src = reinterpret_cast<const A*>(p.grad.data) + p.grad.offset(p.pos[i]) + c;
                float f[N];
                if constexpr (N > 1) {
                    Packed<A, N> v;
                    v.load(src);
                    v.unpack(f);
                } else {
                    f[0] = to_float(*src);
                }
#pragma unroll
                for (int j = 0; j < N; ++j) sum[j] = __fadd_rn(sum[j], f[j]);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                sum[j] = __fmul_rn(sum[j], p.scale);
                if (p.accumulate) sum[j] = __fadd_rn(sum[j], to_float(dst[c + j]));
                dst[c + j] = from_float<B>(sum[j]);
                if (p.idx_out) p.idx_out[static_cast<uint64_t>(u) * p.dim + c + j] = p.idx_offset + (key % p.vocab) * p.dim + c + j;
            }
        }
    }
}

template <typename B>
__global__ void __launch_bounds__(kThreads) k_embed_zero(Rows out, uint32_t n_rows, uint32_t dim) {
    for (uint32_t r = blockIdx.x; r < n_rows; r += gridDim.x)
        for (uint32_t c = threadIdx.x; c < dim; c += kThreads)
            reinterpret_cast<B*>(out.data)[out.offset(r) + c] = from_float<B>(0.f);
}

// ---------------------------------------------------------------------------------------------- host

size_t carve(adacomp_embed_t* h, void* ws, uint32_t max_tokens) {
    Carver c(ws);
    const size_t n = max_tokens, tiles = (n + kTile - 1) / kTile;
    int* status = c.take<int>(1);
    uint32_t* n_segs = c.take<uint32_t>(1);
    uint32_t* list[6] = {};
    if (n) {
        for (int i = 0; i < 4; ++i) list[i] = c.take<uint32_t>(n);
        list[4] = c.take<uint32_t>(n + 1);
        list[5] = c.take<uint32_t>(n);
    }
    uint32_t* table = n ? c.take<uint32_t>(tiles * kBins) : nullptr;
    if (h) {
        h->d_status = status;
        h->d_n_segs = n_segs;
        h->d_key[0] = list[0]; h->d_key[1] = list[1];
        h->d_pos[0] = list[2]; h->d_pos[1] = list[3];
        h->d_seg_begin = list[4];
        h->d_seg_key = list[5];
        h->d_table = table;
    }
    return c.used;
}

int check_limits(uint32_t vocab, uint32_t dim, uint32_t max_tokens, uint32_t max_workers) {
    if (vocab == 0 || dim == 0 || max_workers == 0 || max_tokens >= (1u << 31) || dim >= (1u << 31)) return ADACOMP_ERR_INVALID;
    if (static_cast<uint64_t>(vocab) * max_workers > 0xFFFFFFFEull) return ADACOMP_ERR_INVALID;
    return ADACOMP_OK;
}

// Checks `r` and turns it into its device view.  Distances that make the groups one plain run lose the group.
int rows_view(const adacomp_rows_t* r, uint64_t n_rows, bool tokens, Rows* out) {
    if (!r) return ADACOMP_ERR_INVALID;
    if (tokens ? (r->type != ADACOMP_I32 && r->type != ADACOMP_I64) : !known_type(r->type)) return ADACOMP_ERR_INVALID;
    const uint32_t size = tokens ? (r->type == ADACOMP_I64 ? 8u : 4u) : type_size(r->type);
    if (n_rows && (!r->d_data || reinterpret_cast<uintptr_t>(r->d_data) % size)) return ADACOMP_ERR_INVALID;
    out->data = static_cast<char*>(r->d_data);
    out->type = r->type;
    out->group = r->group;
    out->row_stride = r->row_stride;
    out->group_stride = r->group_stride;
    if (r->group && (r->group >= n_rows || r->group_stride == r->group * r->row_stride)) out->group = 0;
    return ADACOMP_OK;
}

// Whether rows that are written keep clear of each other.
bool rows_apart(const Rows& r, uint64_t n_rows, uint64_t dim) {
    if (n_rows < 2) return true;
    if (r.group == 0) return r.row_stride >= dim;
    const uint64_t groups = (n_rows + r.group - 1) / r.group;
    const uint64_t in_group = r.group > 1 ? (r.group - 1) * r.row_stride + dim : dim;
    if ((r.group == 1 || r.row_stride >= dim) && r.group_stride >= in_group) return true;
    return r.group_stride >= dim && r.row_stride >= (groups - 1) * r.group_stride + dim;
}

// Whether every row starts on a 16-byte boundary.
bool on_grid(const Rows& r) {
    const uint32_t size = type_size(r.type);
    return reinterpret_cast<uintptr_t>(r.data) % 16 == 0 && r.row_stride * size % 16 == 0 &&
           (r.group == 0 || r.group_stride * size % 16 == 0);
}

uint32_t threads_along(uint32_t dim, uint32_t n) {
    uint32_t x = 32;
    while (x < kThreads && x * n < dim) x *= 2;
    return x;
}

template <typename A, typename B>
int launch_lookup(const Rows& table, const Rows& tokens, const Rows& out, uint32_t n_tokens, const adacomp_embed_t* h,
                  float scale, cudaStream_t stream) {
    constexpr int N = kItemElems<A, B>;
    const bool vec = h->dim % N == 0 && on_grid(table) && on_grid(out);
    const uint32_t x = threads_along(h->dim, vec ? N : 1), y = kThreads / x;
    const dim3 grid((n_tokens + y - 1) / y), block(x, y);
    if (vec) k_embed_lookup<A, B, N><<<grid, block, 0, stream>>>(table, tokens, out, n_tokens, h->vocab, h->dim, scale, h->d_status);
    else k_embed_lookup<A, B, 1><<<grid, block, 0, stream>>>(table, tokens, out, n_tokens, h->vocab, h->dim, scale, h->d_status);
    ADACOMP_LAUNCH_CHECK();
    return ADACOMP_OK;
}

template <typename A, typename B>
int launch_sums(const Sums& p, uint32_t n, bool out_vec, uint32_t n_out_rows, cudaStream_t stream) {
    constexpr int N = kItemElems<A, B>;
    if (p.dense && !p.accumulate) {
        k_embed_zero<B><<<n_out_rows < 2048 ? n_out_rows : 2048, kThreads, 0, stream>>>(p.out, n_out_rows, p.dim);
        ADACOMP_LAUNCH_CHECK();
    }
    if (n == 0) return ADACOMP_OK;
    const bool vec = p.dim % N == 0 && on_grid(p.grad) && out_vec;
    const uint32_t x = threads_along(p.dim, vec ? N : 1), y = kThreads / x;
    const dim3 grid((n + y - 1) / y), block(x, y);
    if (vec) k_embed_sums<A, B, N><<<grid, block, 0, stream>>>(p);
    else k_embed_sums<A, B, 1><<<grid, block, 0, stream>>>(p);
    ADACOMP_LAUNCH_CHECK();
    return ADACOMP_OK;
}

// Calls f<A, B>() for the types' numbers.
#define ADACOMP_BY_TYPE(fn, ta, tb, ...)                                                                        \
    [&]() -> int {                                                                                              \
        switch ((ta) * 3 + (tb)) {                                                                              \
            case 0: return fn<float, float>(__VA_ARGS__);                                                       \
            case 1: return fn<float, __nv_bfloat16>(__VA_ARGS__);                                               \
            case 2: return fn<float, __half>(__VA_ARGS__);                                                      \
            case 3: return fn<__nv_bfloat16, float>(__VA_ARGS__);                                               \
            case 4: return fn<__nv_bfloat16, __nv_bfloat16>(__VA_ARGS__);                                       \
            case 5: return fn<__nv_bfloat16, __half>(__VA_ARGS__);                                              \
            case 6: return fn<__half, float>(__VA_ARGS__);                                                      \
            case 7: return fn<__half, __nv_bfloat16>(__VA_ARGS__);                                              \
            default: return fn<__half, __half>(__VA_ARGS__);                                                    \
        }                                                                                                       \
    }()

// Sorts the call's tokens and finds the segments; returns which of the two buffers holds the sorted list.
int sort_tokens(const adacomp_embed_t* h, const Rows& tokens, uint32_t n_tokens, uint32_t n_workers, cudaStream_t stream, int* in) {
    const uint32_t n = n_tokens * n_workers, none = n_workers * h->vocab, tiles = (n + kTile - 1) / kTile;
    *in = 0;
    if (n == 0) {
        ADACOMP_CUDA(cudaMemsetAsync(h->d_n_segs, 0, sizeof(uint32_t), stream));
        return ADACOMP_OK;
    }
    k_embed_keys<<<(n + kThreads - 1) / kThreads, kThreads, 0, stream>>>(tokens, n, n_tokens, h->vocab, h->padding, none, h->d_key[0],
                                                                         h->d_pos[0], h->d_status);
    ADACOMP_LAUNCH_CHECK();
    for (int shift = 0; shift < 32 && (none >> shift) != 0; shift += 8) {
        k_radix_count<<<tiles, kThreads, 0, stream>>>(h->d_key[*in], n, shift, h->d_table);
        ADACOMP_LAUNCH_CHECK();
        k_running_total<<<1, 1024, 0, stream>>>(h->d_table, tiles * kBins, nullptr);
        ADACOMP_LAUNCH_CHECK();
        k_radix_scatter<<<tiles, kThreads, 0, stream>>>(h->d_key[*in], h->d_pos[*in], n, shift, h->d_table, h->d_key[*in ^ 1],
                                                        h->d_pos[*in ^ 1]);
        ADACOMP_LAUNCH_CHECK();
        *in ^= 1;
    }
    k_heads_count<<<tiles, kThreads, 0, stream>>>(h->d_key[*in], n, none, h->d_table);
    ADACOMP_LAUNCH_CHECK();
    k_running_total<<<1, 1024, 0, stream>>>(h->d_table, tiles, h->d_n_segs);
    ADACOMP_LAUNCH_CHECK();
    k_heads_emit<<<tiles, 1024, 0, stream>>>(h->d_key[*in], n, none, h->d_table, h->d_seg_begin, h->d_seg_key, h->d_n_segs);
    ADACOMP_LAUNCH_CHECK();
    return ADACOMP_OK;
}

int check_grad(const adacomp_embed_t* h, uint32_t n_tokens, uint32_t n_workers, float scale) {
    if (!h || n_workers == 0 || n_workers > h->max_workers || !isfinite(scale)) return ADACOMP_ERR_INVALID;
    if (static_cast<uint64_t>(n_tokens) * n_workers > h->max_tokens) return ADACOMP_ERR_CAPACITY;
    return ADACOMP_OK;
}

}  // namespace

extern "C" {

int adacomp_embed_workspace_bytes(uint32_t vocab, uint32_t dim, uint32_t max_tokens, uint32_t max_workers, size_t* bytes_out) {
    if (!bytes_out) return ADACOMP_ERR_INVALID;
    const int rc = check_limits(vocab, dim, max_tokens, max_workers);
    if (rc != ADACOMP_OK) return rc;
    *bytes_out = carve(nullptr, nullptr, max_tokens);
    return ADACOMP_OK;
}

int adacomp_embed_create(adacomp_embed_t** h, uint32_t vocab, uint32_t dim, uint32_t max_tokens, uint32_t max_workers,
                         uint32_t padding_token, void* d_workspace, size_t workspace_bytes, int device) {
    if (!h) return ADACOMP_ERR_INVALID;
    *h = nullptr;
    size_t need = 0;
    const int rc = adacomp_embed_workspace_bytes(vocab, dim, max_tokens, max_workers, &need);
    if (rc != ADACOMP_OK) return rc;
    if (!d_workspace || (reinterpret_cast<uintptr_t>(d_workspace) % kAlign) != 0) return ADACOMP_ERR_INVALID;
    if (need > workspace_bytes) return ADACOMP_ERR_ALLOC;
    adacomp_embed_t* e = new (std::nothrow) adacomp_embed_t;
    if (!e) return ADACOMP_ERR_ALLOC;
    e->device = device;
    e->vocab = vocab;
    e->dim = dim;
    e->max_tokens = max_tokens;
    e->max_workers = max_workers;
    e->padding = padding_token;
    carve(e, d_workspace, max_tokens);
    DeviceGuard guard(device);
    cudaError_t err = guard.err;
    if (err == cudaSuccess) err = cudaDeviceGetAttribute(&e->n_sms, cudaDevAttrMultiProcessorCount, device);
    if (err == cudaSuccess) err = cudaMemset(e->d_status, 0, sizeof(int));
    if (err == cudaSuccess) err = cudaStreamSynchronize(nullptr);
    if (err != cudaSuccess) {
        delete e;
        return cuda_fail(err);
    }
    *h = e;
    return ADACOMP_OK;
}

int adacomp_embed_lookup(adacomp_embed_t* h, const adacomp_rows_t* table, const adacomp_rows_t* tokens, uint32_t n_tokens,
                         float scale, const adacomp_rows_t* out, void* cuda_stream) {
    if (!h || !isfinite(scale) || n_tokens >= (1u << 31)) return ADACOMP_ERR_INVALID;
    Rows t, k, o;
    int rc = rows_view(table, h->vocab, false, &t);
    if (rc == ADACOMP_OK) rc = rows_view(tokens, n_tokens, true, &k);
    if (rc == ADACOMP_OK) rc = rows_view(out, n_tokens, false, &o);
    if (rc != ADACOMP_OK) return rc;
    if (t.group || !rows_apart(o, n_tokens, h->dim)) return ADACOMP_ERR_INVALID;
    if (n_tokens == 0) return ADACOMP_OK;
    DeviceGuard guard(h->device);
    ADACOMP_CUDA(guard.err);
    return ADACOMP_BY_TYPE(launch_lookup, t.type, o.type, t, k, o, n_tokens, h, scale, static_cast<cudaStream_t>(cuda_stream));
}

int adacomp_embed_grad_rows(adacomp_embed_t* h, const adacomp_rows_t* tokens, uint32_t n_tokens, uint32_t n_workers,
                            const adacomp_rows_t* grad, float scale, uint32_t* d_rows_out, uint64_t* d_row_begin_out,
                            void* d_values_out, int values_type, uint32_t* d_idx_out, uint64_t idx_offset, void* cuda_stream) {
    int rc = check_grad(h, n_tokens, n_workers, scale);
    if (rc != ADACOMP_OK) return rc;
    const uint32_t n = n_tokens * n_workers;
    if (!d_row_begin_out || !known_type(values_type) || (n && !d_values_out)) return ADACOMP_ERR_INVALID;
    if (reinterpret_cast<uintptr_t>(d_values_out) % type_size(values_type)) return ADACOMP_ERR_INVALID;
    if (d_idx_out && (idx_offset >= (1ull << 32) || idx_offset + static_cast<uint64_t>(h->vocab) * h->dim > (1ull << 32))) return ADACOMP_ERR_INVALID;
    Rows k;
    Sums p = {};
    rc = rows_view(tokens, n, true, &k);
    if (rc == ADACOMP_OK) rc = rows_view(grad, n, false, &p.grad);
    if (rc != ADACOMP_OK) return rc;
    DeviceGuard guard(h->device);
    ADACOMP_CUDA(guard.err);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    int in = 0;
    rc = sort_tokens(h, k, n_tokens, n_workers, stream, &in);
    if (rc != ADACOMP_OK) return rc;
    k_row_begin<<<(n_workers + 128) / 128, 128, 0, stream>>>(h->d_seg_key, h->d_n_segs, n_workers, h->vocab, d_row_begin_out);
    ADACOMP_LAUNCH_CHECK();
    p.pos = h->d_pos[in];
    p.seg_begin = h->d_seg_begin;
    p.seg_key = h->d_seg_key;
    p.n_segs = h->d_n_segs;
    p.dim = h->dim;
    p.vocab = h->vocab;
    p.scale = scale;
    p.rows_out = d_rows_out;
    p.values = static_cast<char*>(d_values_out);
    p.idx_out = d_idx_out;
    p.idx_offset = static_cast<uint32_t>(idx_offset);
    const bool vec = reinterpret_cast<uintptr_t>(d_values_out) % 16 == 0 && static_cast<uint64_t>(h->dim) * type_size(values_type) % 16 == 0 &&
                     (!d_idx_out || (reinterpret_cast<uintptr_t>(d_idx_out) % 16 == 0 && h->dim % 4 == 0));
    return ADACOMP_BY_TYPE(launch_sums, p.grad.type, values_type, p, n, vec, 0, stream);
}

int adacomp_embed_grad_dense(adacomp_embed_t* h, const adacomp_rows_t* tokens, uint32_t n_tokens, uint32_t n_workers,
                             const adacomp_rows_t* grad, float scale, const adacomp_rows_t* out, int accumulate, void* cuda_stream) {
    int rc = check_grad(h, n_tokens, n_workers, scale);
    if (rc != ADACOMP_OK) return rc;
    const uint32_t n = n_tokens * n_workers;
    Rows k;
    Sums p = {};
    rc = rows_view(tokens, n, true, &k);
    if (rc == ADACOMP_OK) rc = rows_view(grad, n, false, &p.grad);
    if (rc == ADACOMP_OK) rc = rows_view(out, static_cast<uint64_t>(n_workers) * h->vocab, false, &p.out);
    if (rc != ADACOMP_OK) return rc;
    if (!rows_apart(p.out, static_cast<uint64_t>(n_workers) * h->vocab, h->dim)) return ADACOMP_ERR_INVALID;
    DeviceGuard guard(h->device);
    ADACOMP_CUDA(guard.err);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    int in = 0;
    rc = sort_tokens(h, k, n_tokens, n_workers, stream, &in);
    if (rc != ADACOMP_OK) return rc;
    p.pos = h->d_pos[in];
    p.seg_begin = h->d_seg_begin;
    p.seg_key = h->d_seg_key;
    p.n_segs = h->d_n_segs;
    p.dim = h->dim;
    p.vocab = h->vocab;
    p.scale = scale;
    p.dense = 1;
    p.accumulate = accumulate != 0;
    return ADACOMP_BY_TYPE(launch_sums, p.grad.type, p.out.type, p, n, on_grid(p.out), n_workers * h->vocab, stream);
}

int adacomp_embed_last_error(adacomp_embed_t* h, void* cuda_stream) {
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

int adacomp_embed_destroy(adacomp_embed_t* h) {
    delete h;
    return ADACOMP_OK;
}

}  // extern "C"
