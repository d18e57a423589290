// Global gradient norm over many tensors, and clipping.
//
//   norm_w = |s| sqrt(sum_i g_i^2),   c_w = s min(1, max_norm / (norm_w + 1e-6)),   out_i = round(g_i c_w)
//
// Both kernels are one pass over the data (2 and 1 operations an entry): HBM bounds them.  The tensors of a call are cut
// into units of 32 KB of the input (first pass) or 8192 entries (second); blocks take units in turn, so short tensors next to
// each other in the list go to different blocks.  The second pass walks the units from the back, where some of what the first
// pass read last is still in L2 (38 of 102 MB; 64 MB come from HBM once more).  Of 161 tensors, 102 MB of fp32, the second pass
// reaches 57 % of the HBM rate: a block has some five units, and nothing of the next is under way while it writes one.
#include <cooperative_groups.h>
#include <math.h>
#include <new>

#include "numeric.cuh"

using namespace adacomp;

struct adacomp_clip {
    int device;
    uint32_t max_workers;
    int n_sms;
    double* d_partial;              // [workers][slots_of(blocks)] of a call
    uint32_t* d_done;               // [max_workers] blocks that have delivered their sum
    float* d_coef;                  // [max_workers]
};

namespace {

constexpr int kThreads = 256;
constexpr int kVecsPerThread = 8;
constexpr uint32_t kUnit = kThreads * kVecsPerThread;       // vectors of 16 bytes per unit of the first pass
// Blocks resident per SM.  Loads in flight count: 8 vectors a thread and 3 blocks read 6.4 GB in 866 us (7.4 TB/s), 4 and 6 in
// 884, 4 and 8 in 937.
constexpr int kNormBlocks = 3, kWriteBlocks = 4;
constexpr uint32_t kMaxBlocks = 1024;                       // blocks of a call with fewer workers; with more a worker has one
// A worker's partial sums fill whole lines of 128 bytes, so the workers of a call need kMaxBlocks + 16 of them each at most.
constexpr uint32_t kSlotLine = 16;
__host__ __device__ constexpr uint32_t slots_of(uint32_t n_blocks) { return (n_blocks + kSlotLine - 1) / kSlotLine * kSlotLine; }
// Gradients up to this many bytes: what the second pass reads and writes is given up first by L2, so that what the first pass
// read stays until it is read again.  Measured, both passes: 102 MB of fp32 57.2 -> 53.3 us, 52 MB of fp16 44.5 -> 40.2 us;
// but 683 MB of bf16 464 -> 471 us, where little of it can stay anyway.
constexpr uint64_t kKeepInL2 = 160ull << 20;
// Gradients of so many bytes a worker, and all workers together, are clipped in one launch.  The call with two launches and with
// one: 64 KB 10.3 and 8.8 us, 16 workers of 256 KB 11.2 and 9.1, of 512 KB 11.2 and 11.4; 64 workers of 64 KB 11.4 and
// 10.5, of 256 KB 12.4 and 14.6.
constexpr uint64_t kSmallBytes = 256 << 10, kSmallTotal = 4 << 20;
constexpr double kEps = 1e-6;

struct Tensor {
    const char* in;
    char* out;
    uint64_t n : 48, in_type : 8, out_type : 8;
    uint32_t first[2];              // its first unit among the launch's, of the first and of the second pass
};
static_assert(sizeof(Tensor) == 32, "table entries are packed");

// The tensors travel as kernel parameters: no upload, no buffer that a later call could overwrite, and the call can
// be captured.  Parameters may take 32764 bytes; longer lists take several launches.
template <int MAX> struct Table { Tensor t[MAX]; };
constexpr int kFew = 64, kMany = 960;

struct Job {
    uint32_t n_tensors, n_units[2];
    uint64_t in_stride, out_stride;
    float scale;
    float max_norm;
    int first, last;                // of the call's launches
    int give_up_first;              // the second pass's lines in L2
    uint32_t n_blocks;
    double* partial;
    uint32_t* done;
    float* norm_out;
    float* coef;
    float* coef_out;
};

// The table's copy in shared memory, and the tensor of a unit: the last one whose first unit is not behind it.  A warp looks
// it up in two steps of 32 entries each (a list has at most 960).
struct Lookup {
    const Tensor* t;
    uint32_t n, stride;
    template <int MAX> __device__ __forceinline__ Lookup(const Table<MAX>& tab, uint32_t count, Tensor* s_tab)
        : t(s_tab), n(count), stride((count + 31) / 32) {
        const uint4* src = reinterpret_cast<const uint4*>(tab.t);
        // read through a generic address, a thread an entry: as constant loads with an index they would go one by one (161
        // tensors: 25.4 -> 20.4 us for 102 MB)
        asm volatile("" : "+l"(src));
        for (uint32_t k = threadIdx.x; k < 2 * n; k += kThreads) reinterpret_cast<uint4*>(s_tab)[k] = src[k];
        __syncthreads();
    }
    __device__ __forceinline__ const Tensor& of(uint32_t unit, int pass) const {
        const uint32_t lane = threadIdx.x & 31;
        const uint32_t a = lane * stride;
        const uint32_t run = __popc(__ballot_sync(0xFFFFFFFFu, a < n && t[a].first[pass] <= unit)) - 1;
        const uint32_t b = run * stride + lane;
        const uint32_t in = __popc(__ballot_sync(0xFFFFFFFFu, lane < stride && b < n && t[b].first[pass] <= unit)) - 1;
        return t[run * stride + in];
    }
};

__device__ __forceinline__ uint32_t or4(const uint4& v) { return v.x | v.y | v.z | v.w; }

// Sum of the squares of what kVecsPerThread vectors hold.  In fp32 where that is safe (between 2^-100 and 2^100 no square
// overflowed, and what underflowed is below 2^-20 of one unit in the last place), otherwise in 64 bits.
template <typename T> __device__ __forceinline__ double sum_squares(const uint4 (&v)[kVecsPerThread]) {
    constexpr int N = 16 / sizeof(T);
    float s[2] = {0.f, 0.f};
    uint32_t any = 0;
#pragma unroll
    for (int k = 0; k < kVecsPerThread; ++k) {
        Packed<T, N> p;
        p.v[0] = v[k];
        float f[N];
        p.unpack(f);
#pragma unroll
        for (int j = 0; j < N; ++j) s[j & 1] = __fmaf_rn(f[j], f[j], s[j & 1]);
        any |= or4(v[k]);
    }
    const float sum = s[0] + s[1];
    if (sum >= 0x1p-100f && sum <= 0x1p100f) return static_cast<double>(sum);
    if ((any & (sizeof(T) == 4 ? 0x7FFFFFFFu : 0x7FFF7FFFu)) == 0) return 0.0;
    double d = 0.0;
#pragma unroll
    for (int k = 0; k < kVecsPerThread; ++k) {
        Packed<T, N> p;
        p.v[0] = v[k];
        float f[N];
        p.unpack(f);
#pragma unroll
        for (int j = 0; j < N; ++j) d = __fma_rn(static_cast<double>(f[j]), static_cast<double>(f[j]), d);
    }
    return d;
}

// The vector at address a (16-byte aligned) of a tensor that occupies [p, end): elements outside read as zeros.
template <typename T> __device__ __forceinline__ uint4 load_clamped(uintptr_t a, uintptr_t p, uintptr_t end) {
    if (a >= p && a + 16 <= end) return load16(reinterpret_cast<const void*>(a));
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    if (a + 16 > p && a < end) {
#pragma unroll
        for (int j = 0; j < 16 / static_cast<int>(sizeof(T)); ++j) {
            const uintptr_t e = a + j * sizeof(T);
            if (e < p || e >= end) continue;
            if constexpr (sizeof(T) == 4) w[j] = *reinterpret_cast<const uint32_t*>(e);
            else w[j / 2] |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(e)) << (16 * (j & 1));
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T>
__device__ __forceinline__ double unit_squares(const char* base, uint64_t n, uint32_t unit) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(base), end = p + n * sizeof(T);
    const uintptr_t first = (p & ~static_cast<uintptr_t>(15)) + static_cast<uint64_t>(unit) * kUnit * 16;
    const uintptr_t a = first + threadIdx.x * 16;
    uint4 v[kVecsPerThread];
    if (first >= p && first + kUnit * 16 <= end) {
#pragma unroll
        for (int k = 0; k < kVecsPerThread; ++k) v[k] = load16(reinterpret_cast<const void*>(a + k * kThreads * 16));
    } else {
#pragma unroll
        for (int k = 0; k < kVecsPerThread; ++k) v[k] = load_clamped<T>(a + k * kThreads * 16, p, end);
    }
    return sum_squares<T>(v);
}

__device__ __forceinline__ double block_sum(double x, double* s_warp) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
    if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = x;
    __syncthreads();
    double total = 0.0;
    if (threadIdx.x == 0)
        for (int i = 0; i < kThreads / 32; ++i) total += s_warp[i];
    __syncthreads();
    return total;                   // of thread 0
}

// This thread's share of the squares of worker w: units b, b + n_blocks, ...
__device__ __forceinline__ double worker_squares(const Lookup& tensors, const Job& job, uint32_t w, uint32_t b, uint32_t n_blocks) {
    double sum = 0.0;
    for (uint32_t u = b; u < job.n_units[0]; u += n_blocks) {
        const Tensor& t = tensors.of(u, 0);
        const char* base = t.in + w * job.in_stride * type_size(t.in_type);
        const uint32_t at = u - t.first[0];
        if (t.in_type == ADACOMP_F32) sum += unit_squares<float>(base, t.n, at);
        else if (t.in_type == ADACOMP_BF16) sum += unit_squares<__nv_bfloat16>(base, t.n, at);
        else sum += unit_squares<__half>(base, t.n, at);
    }
    return sum;
}

// A worker's norm from its sum of squares, and the factor for its entries.
__device__ __forceinline__ float norm_and_factor(const Job& job, double total, float* norm_out) {
    const double norm = fabs(static_cast<double>(job.scale)) * sqrt(total);
    *norm_out = static_cast<float>(norm);
    double c = static_cast<double>(job.max_norm) / (norm + kEps);
    if (c > 1.0 || isinf(job.max_norm)) c = 1.0;                // a NaN stays one
    return static_cast<float>(c * static_cast<double>(job.scale));
}

template <int MAX>
__global__ void __launch_bounds__(kThreads, kNormBlocks) k_grad_norm(const __grid_constant__ Table<MAX> tab, const Job job) {
    __shared__ double s_warp[kThreads / 32];
    __shared__ bool s_last;
    extern __shared__ Tensor s_tab[];
    const uint32_t w = blockIdx.y, b = blockIdx.x;
    const Lookup tensors(tab, job.n_tensors, s_tab);
    const double sum = block_sum(worker_squares(tensors, job, w, b, job.n_blocks), s_warp);
    if (threadIdx.x == 0) {
        double* slot = job.partial + static_cast<uint64_t>(w) * slots_of(job.n_blocks) + b;
        *slot = job.first ? sum : *slot + sum;
        s_last = false;
        if (job.last) {
            __threadfence();
            s_last = atomicAdd(job.done + w, 1u) == job.n_blocks - 1;
        }
    }
    __syncthreads();
    if (!s_last) return;
    // the worker's last block adds the partial sums, in their order
    __threadfence();
    double total = 0.0;
    for (uint32_t k = threadIdx.x; k < job.n_blocks; k += kThreads)
        total += __ldcg(job.partial + static_cast<uint64_t>(w) * slots_of(job.n_blocks) + k);
    total = block_sum(total, s_warp);
    if (threadIdx.x == 0) {
        job.done[w] = 0;
        const float f = norm_and_factor(job, total, job.norm_out + w);
        if (job.coef) job.coef[w] = f;
        if (job.coef_out) job.coef_out[w] = f;
    }
}

template <typename A, typename B, int N>
__device__ __forceinline__ void scale_store(const Packed<A, N>& p, B* out, float c, uint64_t policy) {
    float f[N];
    p.unpack(f);
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = __fmul_rn(f[j], c);
    Packed<B, N> q;
    q.pack(f);
    q.store_whole(out, policy);
}

// Entries per item of the second pass: 16 bytes of a 16-bit type, 32 of fp32.
constexpr int kItem = 8;
constexpr int kItemsPerThread = 4;
constexpr uint32_t kWriteUnit = kThreads * kItemsPerThread;

template <typename A, typename B>
__device__ __forceinline__ void write_unit(const Tensor& t, uint32_t w, const Job& job, uint32_t unit, float c, uint64_t policy) {
    constexpr int N = kItem;
    const A* in = reinterpret_cast<const A*>(t.in) + w * job.in_stride;
    B* out = reinterpret_cast<B*>(t.out) + w * job.out_stride;
    const int64_t n = static_cast<int64_t>(t.n);
    // items start on the output's own grid: item j holds entries [j N - skew, j N - skew + N)
    const int64_t skew = static_cast<int64_t>((reinterpret_cast<uintptr_t>(out) & (N * sizeof(B) - 1)) / sizeof(B));
    const int64_t unit_at = static_cast<int64_t>(unit) * kWriteUnit * N - skew, e0 = unit_at + threadIdx.x * N;
    const bool on_grid = (reinterpret_cast<uintptr_t>(in + e0) & (N * sizeof(A) - 1)) == 0;
    if (on_grid && unit_at >= 0 && unit_at + static_cast<int64_t>(kWriteUnit) * N <= n) {
        Packed<A, N> p[kItemsPerThread];
#pragma unroll
        for (int k = 0; k < kItemsPerThread; ++k) p[k].load_whole(in + e0 + k * (kThreads * N), policy);
#pragma unroll
        for (int k = 0; k < kItemsPerThread; ++k) scale_store<A, B, N>(p[k], out + e0 + k * (kThreads * N), c, policy);
        return;
    }
#pragma unroll 1
    for (int k = 0; k < kItemsPerThread; ++k) {
        const int64_t e = e0 + k * (kThreads * N);
        if (e >= 0 && e + N <= n) {
            Packed<A, N> p;
            if (on_grid) p.load_whole(in + e, policy);
            else p = load_shifted<A, N>(in, e, t.n);
            scale_store<A, B, N>(p, out + e, c, policy);
        } else {
#pragma unroll 1
            for (int j = 0; j < N; ++j)
                if (e + j >= 0 && e + j < n) out[e + j] = from_float<B>(__fmul_rn(to_float(in[e + j]), c));
        }
    }
}

template <typename A>
__device__ __forceinline__ void write_unit_from(const Tensor& t, uint32_t w, const Job& job, uint32_t unit, float c, uint64_t policy) {
    if (t.out_type == ADACOMP_F32) write_unit<A, float>(t, w, job, unit, c, policy);
    else if (t.out_type == ADACOMP_BF16) write_unit<A, __nv_bfloat16>(t, w, job, unit, c, policy);
    else write_unit<A, __half>(t, w, job, unit, c, policy);
}

// The second pass of worker w: units from the back.
__device__ __forceinline__ void worker_write(const Lookup& tensors, const Job& job, uint32_t w, uint32_t b, uint32_t n_blocks, float c) {
    const uint64_t policy = l2_policy(job.give_up_first != 0);
    for (uint32_t k = b; k < job.n_units[1]; k += n_blocks) {
        const uint32_t u = job.n_units[1] - 1 - k;
        const Tensor& t = tensors.of(u, 1);
        if (c == 1.0f && t.out == t.in) continue;           // in place, nothing to change
        const uint32_t at = u - t.first[1];
        if (t.in_type == ADACOMP_F32) write_unit_from<float>(t, w, job, at, c, policy);
        else if (t.in_type == ADACOMP_BF16) write_unit_from<__nv_bfloat16>(t, w, job, at, c, policy);
        else write_unit_from<__half>(t, w, job, at, c, policy);
    }
}

template <int MAX>
__global__ void __launch_bounds__(kThreads, kWriteBlocks) k_clip_write(const __grid_constant__ Table<MAX> tab, const Job job) {
    extern __shared__ Tensor s_tab[];
    const Lookup tensors(tab, job.n_tensors, s_tab);
    cudaGridDependencySynchronize();
    worker_write(tensors, job, blockIdx.y, blockIdx.x, job.n_blocks, job.coef[blockIdx.y]);
}

// Both passes of a small gradient in one launch: a cluster of kCluster blocks per worker, which tell each other their sums through
// shared memory.  The second read comes from L2.
constexpr uint32_t kCluster = 8;
template <int MAX>
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads, kNormBlocks)
    k_clip_small(const __grid_constant__ Table<MAX> tab, const Job job) {
    __shared__ double s_warp[kThreads / 32];
    __shared__ double s_sums[kCluster];
    __shared__ float s_factor;
    extern __shared__ Tensor s_tab[];
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    const uint32_t w = blockIdx.y, b = blockIdx.x;
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    const Lookup tensors(tab, job.n_tensors, s_tab);
    const double sum = block_sum(worker_squares(tensors, job, w, b, kCluster), s_warp);
    if (threadIdx.x == 0) s_warp[0] = sum;
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");        // every block has started: its shared memory may be written
    __syncthreads();
    if (threadIdx.x < kCluster) *cluster.map_shared_rank(s_sums + b, threadIdx.x) = s_warp[0];
    cluster.sync();
    if (threadIdx.x == 0) {
        double total = 0.0;
        for (uint32_t k = 0; k < kCluster; ++k) total += s_sums[k];
        float norm;
        s_factor = norm_and_factor(job, total, &norm);
        if (b == 0) {
            job.norm_out[w] = norm;
            if (job.coef_out) job.coef_out[w] = s_factor;
        }
    }
    __syncthreads();
    worker_write(tensors, job, w, b, kCluster, s_factor);
}

// Units of a tensor: by its input's vectors (norm) or by its items on the output's grid (write), counted so that they
// suffice wherever a worker's copy sits on the 16-byte grid.
uint64_t units_of(const adacomp_grad_tensor_t& t, bool write) {
    if (write) return (t.n + kItem - 1 + static_cast<uint64_t>(kWriteUnit) * kItem - 1) / (static_cast<uint64_t>(kWriteUnit) * kItem);
    return (t.n * type_size(t.grad_type) + 14 + kUnit * 16 - 1) / (kUnit * 16);
}

enum Pass { kNorm = 0, kWrite = 1, kBoth = 2 };

template <int MAX>
int launch(const Table<MAX>& tab, const Job& job, uint32_t n_workers, Pass pass, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(pass == kBoth ? kCluster : job.n_blocks, n_workers);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = job.n_tensors * sizeof(Tensor);
    cfg.stream = stream;
    // a write launch may start while the norm's last blocks finish: it waits for them itself
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pass == kWrite ? 1 : 0;
    const cudaError_t e = pass == kWrite ? cudaLaunchKernelEx(&cfg, k_clip_write<MAX>, tab, job)
                        : pass == kNorm ? cudaLaunchKernelEx(&cfg, k_grad_norm<MAX>, tab, job)
                                        : cudaLaunchKernelEx(&cfg, k_clip_small<MAX>, tab, job);
    if (e != cudaSuccess) return cuda_fail(e);
    ADACOMP_LAUNCH_CHECK();
    return ADACOMP_OK;
}

int check_tensors(const adacomp_grad_tensor_t* ts, uint32_t n_tensors, uint64_t in_stride, uint64_t out_stride, uint32_t n_workers,
                  bool write) {
    if (!ts && n_tensors) return ADACOMP_ERR_INVALID;
    for (uint32_t i = 0; i < n_tensors; ++i) {
        const adacomp_grad_tensor_t& t = ts[i];
        if (!known_type(t.grad_type) || t.n >= (1ull << 40)) return ADACOMP_ERR_INVALID;
        if (t.n && (!t.d_grad || !aligned(t.d_grad, type_size(t.grad_type)))) return ADACOMP_ERR_INVALID;
        if (!write) continue;
        if (!known_type(t.out_type)) return ADACOMP_ERR_INVALID;
        if (t.n == 0) continue;             // its pointers and strides mean nothing
        if (!t.d_out || !aligned(t.d_out, type_size(t.out_type))) return ADACOMP_ERR_INVALID;
        if (t.d_out == t.d_grad && t.out_type != t.grad_type) return ADACOMP_ERR_INVALID;
        // the workers' outputs keep clear of each other, and in place they lie where the gradients do
        if (n_workers > 1 && (out_stride < t.n || (t.d_out == t.d_grad && out_stride != in_stride))) return ADACOMP_ERR_INVALID;
    }
    return ADACOMP_OK;
}

// Fills the table from tensor *at on; false if a tensor alone has too many units.
bool fill_table(const adacomp_grad_tensor_t* ts, uint32_t n_tensors, uint32_t* at, bool write, Table<kMany>* tab, Job* job) {
    uint32_t n = 0;
    uint64_t units[2] = {0, 0};
    for (; *at < n_tensors && n < kMany; ++*at) {
        const adacomp_grad_tensor_t& t = ts[*at];
        if (t.n == 0) continue;
        const uint64_t u[2] = {units_of(t, false), write ? units_of(t, true) : 0};
        if (units[0] + u[0] >= (1ull << 32) || units[1] + u[1] >= (1ull << 32)) {
            if (n == 0) return false;
            break;
        }
        Tensor& e = tab->t[n++];
        e.in = static_cast<const char*>(t.d_grad);
        e.out = static_cast<char*>(t.d_out);
        e.n = t.n;
        e.in_type = static_cast<uint8_t>(t.grad_type);
        e.out_type = static_cast<uint8_t>(t.out_type);
        for (int p = 0; p < 2; ++p) {
            e.first[p] = static_cast<uint32_t>(units[p]);
            units[p] += u[p];
        }
    }
    job->n_tensors = n;
    job->n_units[0] = static_cast<uint32_t>(units[0]);
    job->n_units[1] = static_cast<uint32_t>(units[1]);
    return true;
}

int launch_table(const Table<kMany>& tab, const Job& job, uint32_t n_workers, Pass pass, cudaStream_t stream) {
    if (job.n_tensors > kFew) return launch(tab, job, n_workers, pass, stream);
    Table<kFew> few;
    for (uint32_t k = 0; k < job.n_tensors; ++k) few.t[k] = tab.t[k];
    return launch(few, job, n_workers, pass, stream);
}

// Blocks of one worker: all of a call's are resident at once where there are not more workers than that, and none is
// without work.
uint32_t blocks_per_worker(const adacomp_clip_t* h, uint64_t units, uint32_t n_workers, bool write) {
    uint64_t blocks = static_cast<uint64_t>(write ? kWriteBlocks : kNormBlocks) * h->n_sms;
    if (blocks > kMaxBlocks) blocks = kMaxBlocks;
    blocks /= n_workers;
    if (blocks > units) blocks = units;
    return blocks < 1 ? 1 : static_cast<uint32_t>(blocks);
}

size_t carve(adacomp_clip_t* h, void* ws, uint32_t max_workers) {
    Carver c(ws);
    double* partial = c.take<double>(kMaxBlocks + static_cast<size_t>(kSlotLine) * max_workers);
    uint32_t* done = c.take<uint32_t>(max_workers);
    float* coef = c.take<float>(max_workers);
    if (h) {
        h->d_partial = partial;
        h->d_done = done;
        h->d_coef = coef;
    }
    return c.used;
}

int run(adacomp_clip_t* h, const adacomp_grad_tensor_t* ts, uint32_t n_tensors, uint64_t in_stride, uint64_t out_stride,
        uint32_t n_workers, float scale, float max_norm, float* d_norm, float* d_coef_out, bool write, void* cuda_stream) {
    if (!h || !d_norm || n_workers == 0 || n_workers > h->max_workers || !isfinite(scale)) return ADACOMP_ERR_INVALID;
    if (write && !(max_norm > 0.f)) return ADACOMP_ERR_INVALID;
    if (!aligned(d_norm, sizeof(float)) || !aligned(d_coef_out, sizeof(float))) return ADACOMP_ERR_INVALID;
    int rc = check_tensors(ts, n_tensors, in_stride, out_stride, n_workers, write);
    if (rc != ADACOMP_OK) return rc;
    DeviceGuard guard(h->device);
    ADACOMP_CUDA(guard.err);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    Job job = {};
    job.in_stride = in_stride;
    job.out_stride = out_stride;
    job.scale = scale;
    job.max_norm = max_norm;
    job.partial = h->d_partial;
    job.done = h->d_done;
    job.norm_out = d_norm;
    job.coef = write ? h->d_coef : nullptr;
    job.coef_out = d_coef_out;
    uint64_t bytes = 0, units[2] = {0, 0};
    for (uint32_t i = 0; i < n_tensors; ++i) {
        if (ts[i].n == 0) continue;
        bytes += ts[i].n * type_size(ts[i].grad_type);
        units[0] += units_of(ts[i], false);
        if (write) units[1] += units_of(ts[i], true);
    }
    job.give_up_first = bytes * n_workers <= kKeepInL2;
    static thread_local Table<kMany> tab;
    bool whole = false;                                     // whether one table holds the call
    for (int pass = 0; pass < (write ? 2 : 1); ++pass) {
        job.n_blocks = blocks_per_worker(h, units[pass], n_workers, pass == 1);
        uint32_t at = 0;
        job.first = 1;
        do {
            if (!whole) {
                if (!fill_table(ts, n_tensors, &at, write, &tab, &job)) return ADACOMP_ERR_INVALID;
                whole = job.first && at == n_tensors;
            } else {
                at = n_tensors;
            }
            job.last = at == n_tensors;
            if (write && whole && bytes <= kSmallBytes && bytes * n_workers <= kSmallTotal)
                return launch_table(tab, job, n_workers, kBoth, stream);
            if (pass == 0 || job.n_tensors) rc = launch_table(tab, job, n_workers, pass == 0 ? kNorm : kWrite, stream);
            if (rc != ADACOMP_OK) return rc;
            job.first = 0;
        } while (at < n_tensors);
    }
    return ADACOMP_OK;
}

}  // namespace

extern "C" {

int adacomp_clip_workspace_bytes(uint32_t max_workers, size_t* bytes_out) {
    if (!bytes_out || max_workers == 0 || max_workers > 65535) return ADACOMP_ERR_INVALID;
    *bytes_out = carve(nullptr, nullptr, max_workers);
    return ADACOMP_OK;
}

int adacomp_clip_create(adacomp_clip_t** h, uint32_t max_workers, void* d_workspace, size_t workspace_bytes, int device) {
    if (!h) return ADACOMP_ERR_INVALID;
    *h = nullptr;
    size_t need = 0;
    const int rc = adacomp_clip_workspace_bytes(max_workers, &need);
    if (rc != ADACOMP_OK) return rc;
    if (!d_workspace || (reinterpret_cast<uintptr_t>(d_workspace) % kAlign) != 0) return ADACOMP_ERR_INVALID;
    if (need > workspace_bytes) return ADACOMP_ERR_ALLOC;
    adacomp_clip_t* c = new (std::nothrow) adacomp_clip_t;
    if (!c) return ADACOMP_ERR_ALLOC;
    c->device = device;
    c->max_workers = max_workers;
    carve(c, d_workspace, max_workers);
    DeviceGuard guard(device);
    cudaError_t e = guard.err;
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&c->n_sms, cudaDevAttrMultiProcessorCount, device);
    if (e == cudaSuccess) e = cudaMemset(c->d_done, 0, max_workers * sizeof(uint32_t));
    if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);
    if (e != cudaSuccess) {
        delete c;
        return cuda_fail(e);
    }
    *h = c;
    return ADACOMP_OK;
}

int adacomp_grad_norm(adacomp_clip_t* h, const adacomp_grad_tensor_t* h_tensors, uint32_t n_tensors, uint64_t grad_stride,
                      uint32_t n_workers, float scale, float* d_norm_out, void* cuda_stream) {
    return run(h, h_tensors, n_tensors, grad_stride, 0, n_workers, scale, 1.f, d_norm_out, nullptr, false, cuda_stream);
}

int adacomp_clip(adacomp_clip_t* h, const adacomp_grad_tensor_t* h_tensors, uint32_t n_tensors, uint64_t grad_stride,
                 uint64_t out_stride, uint32_t n_workers, float scale, float max_norm, float* d_norm_out,
                 float* d_coef_out, void* cuda_stream) {
    return run(h, h_tensors, n_tensors, grad_stride, out_stride, n_workers, scale, max_norm, d_norm_out, d_coef_out, true,
               cuda_stream);
}

int adacomp_clip_destroy(adacomp_clip_t* h) {
    delete h;
    return ADACOMP_OK;
}

}  // extern "C"
