// Embedding tables: lookup with scaling, and the gradient by sorted tokens.
//
//   lookup    out_t = round(s E[token_t])
//   gradient  dE[w][v] = s sum of the gradient rows of worker w's tokens that equal v
//
// The gradient sorts the pairs (worker * vocab + token, position), stable, so a row's summands stand together and in
// order; every row is then summed by whoever owns it, without floating-point atomics.  The sums and the lookup are bound by
// HBM (one fp32 operation per entry read), the sort by latency, small calls by the launch.
#include <cooperative_groups.h>
#include <math.h>
#include <new>

#include "rows.cuh"

using namespace adacomp;

struct adacomp_embed {
    int device;
    uint32_t vocab, dim, max_tokens, max_workers, padding;
    int n_sms;
    int* d_status;
    uint32_t* d_barrier;            // [3] arrivals, blocks that are through, and whether a wait ever ran out
    uint64_t* d_tok[2];             // [max_tokens] worker * vocab + token and which token it is, between the passes of a large sort
    uint32_t* d_table;              // [kSortBlocks][kMaxBins] digit counts per block
    uint32_t* d_seg_begin;          // [max_tokens + 1] first sorted token of every distinct one, and their end
    uint32_t* d_seg_key;            // [max_tokens]
    uint32_t* d_chunk_seg;          // [chunks + 1] how many segments begin before the chunk
    uint32_t* d_n_segs;             // [2] distinct tokens, and how many tokens of the sorted list have a gradient
    uint32_t* d_order;              // [max_tokens] positions in the order of the sort
    uint32_t wait_limit;            // polls of a barrier
    uint32_t cluster;               // blocks of the largest cluster that the device takes
    uint32_t* d_tickets;            // [levels][chunks][2][blocks along a row], all zero between calls
    uint32_t chunks;                // the most that a call has
    float* d_partial;               // [chunks][2][dim] sums of pieces of those
};

namespace {

constexpr int kThreads = 256;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kItems = 8;                                   // tokens per thread and step of the sort
constexpr uint32_t kStep = kSortThreads * kItems;
// Tokens per block of a cluster.  The whole call at 32768, 65536 and 131072 tokens of 64 columns: 25, 33 and 53 us with a
// cluster, 33, 35 and 43 without.
constexpr int kClusterItems = 4;
constexpr uint32_t kClusterStep = kSortThreads * kClusterItems;
constexpr uint32_t kSortBlocks = 128;
constexpr int kDigitBits = 9;
constexpr int kMaxBins = 1 << kDigitBits;
constexpr uint32_t kClusterSmem = kClusterStep * 8 + 16 * kMaxBins * 2 + kSortWarps * kMaxBins * 2;
constexpr uint32_t kWaitLimit = 1u << 22;                   // polls of a barrier, some seconds

// A token as it is stored; what does not fit `vocab` comes out as UINT32_MAX.
__device__ __forceinline__ uint32_t load_token(const Rows& tokens, uint32_t t, uint32_t vocab) {
    const uint64_t at = tokens.offset(t);
    uint64_t v;
    if (tokens.type == ADACOMP_I64) v = reinterpret_cast<const uint64_t*>(tokens.data)[at];
    else v = static_cast<uint64_t>(static_cast<int64_t>(reinterpret_cast<const int32_t*>(tokens.data)[at]));
    return v < vocab ? static_cast<uint32_t>(v) : 0xFFFFFFFFu;      // negative numbers are large ones here, above any vocabulary
}

// ---------------------------------------------------------------------------------------------- lookup

// Threads of a block: x along a row (in `tiles` blocks), y over rows.  A thread copies the same columns of R tokens (K groups
// of N columns, as the sums below), all of them on their way before the first is stored.
template <typename A, typename B, int N, int K, int R>
__global__ void __launch_bounds__(512) k_embed_lookup(Rows table, Rows tokens, Rows out, uint32_t n_tokens, uint32_t vocab, uint32_t dim,
                                                       uint32_t tiles, int wide, int passing, float scale, int* status) {
    const uint32_t t0 = blockIdx.x / tiles * (blockDim.y * R) + threadIdx.y, tile = blockIdx.x % tiles;
    const uint32_t step = blockDim.x * N, c = tile * K * step + threadIdx.x * N;
    const bool same = table.type == out.type && scale == 1.0f;
    uint32_t v[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t t = t0 + r * blockDim.y;
        v[r] = t < n_tokens ? load_token(tokens, t, vocab) : 0xFFFFFFFFu;
    }
    Packed<A, N> row[R][K];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int g = 0; g < K; ++g)
            if (v[r] != 0xFFFFFFFFu && c + g * step < dim)
                row[r][g].load(reinterpret_cast<const A*>(table.data) + v[r] * table.row_stride + c + g * step);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t t = t0 + r * blockDim.y;
        if (t >= n_tokens) continue;
        if (v[r] == 0xFFFFFFFFu && c == 0) record_error(status, ADACOMP_ERR_INVALID);
        B* dst = reinterpret_cast<B*>(out.data) + out.offset(t) + c;
#pragma unroll
        for (int g = 0; g < K; ++g) {
            if (c + g * step >= dim) continue;
            Packed<B, N> q;
            if (sizeof(A) == sizeof(B) && same && v[r] != 0xFFFFFFFFu) {
                q = *reinterpret_cast<const Packed<B, N>*>(&row[r][g]);         // nothing to convert and nothing to multiply
            } else {
                float f[N];
                if (v[r] != 0xFFFFFFFFu) {
                    row[r][g].unpack(f);
#pragma unroll
                    for (int k = 0; k < N; ++k) f[k] = __fmul_rn(f[k], scale);
                } else {
#pragma unroll
                    for (int k = 0; k < N; ++k) f[k] = 0.f;
                }
                q.pack(f);
            }
            if (Packed<B, N>::kVecs == 2 && wide) store32(dst, q.v[0], q.v[Packed<B, N>::kVecs - 1], l2_policy(passing != 0));
            else if (N > 1 && Packed<B, N>::kVecs == 1 && passing) __stcs(reinterpret_cast<uint4*>(dst + g * step), q.v[0]);
            else q.store(dst + g * step);
        }
    }
}

// The same where rows do not sit on the 16-byte grid and 16-bit entries make single ones too small a load: items of eight
// entries on the grid of each output row, taken from the two vectors of the table around them.  `total` entries lie between the
// table's first and its last.  Both ends of a row go entry by entry, and the warps that hold them wait for it: 32768 bf16 rows of
// 1001 take 37 us, of 1024 on the grid 21.
template <typename A, typename B, int R>
__global__ void __launch_bounds__(512) k_embed_lookup_off(Rows table, Rows tokens, Rows out, uint32_t n_tokens, uint32_t vocab, uint32_t dim,
                                                           uint32_t tiles, uint64_t total, float scale, int* status) {
    constexpr int N = 8;
    const uint32_t t0 = blockIdx.x / tiles * (blockDim.y * R) + threadIdx.y, tile = blockIdx.x % tiles;
    const int64_t item = static_cast<int64_t>(tile) * blockDim.x + threadIdx.x;
    const A* in = reinterpret_cast<const A*>(table.data);
    uint32_t v[R];
    int64_t e[R];
    Packed<A, N> row[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t t = t0 + r * blockDim.y;
        v[r] = t < n_tokens ? load_token(tokens, t, vocab) : 0xFFFFFFFFu;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t t = t0 + r * blockDim.y;
        const uintptr_t dst = reinterpret_cast<uintptr_t>(reinterpret_cast<B*>(out.data) + (t < n_tokens ? out.offset(t) : 0));
        e[r] = item * N - static_cast<int64_t>((dst & 15) / sizeof(B));
        if (v[r] == 0xFFFFFFFFu || e[r] >= dim) continue;
        const A* src = in + v[r] * table.row_stride;
        if (e[r] >= 0 && e[r] + N <= dim) {
            row[r] = load_shifted<A, N>(in, (src - in) + e[r], total);
        } else {                                            // a row's first and last entries
            float f[N];
#pragma unroll
            for (int k = 0; k < N; ++k) f[k] = e[r] + k >= 0 && e[r] + k < dim ? to_float(src[e[r] + k]) : 0.f;
            row[r].pack(f);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t t = t0 + r * blockDim.y;
        if (t >= n_tokens || e[r] >= dim) continue;
        if (v[r] == 0xFFFFFFFFu && item == 0) record_error(status, ADACOMP_ERR_INVALID);
        B* dst = reinterpret_cast<B*>(out.data) + out.offset(t);
        float f[N];
        if (v[r] != 0xFFFFFFFFu) {
            row[r].unpack(f);
#pragma unroll
            for (int k = 0; k < N; ++k) f[k] = __fmul_rn(f[k], scale);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) f[k] = 0.f;
        }
        if (e[r] >= 0 && e[r] + N <= dim) {
            Packed<B, N> q;
            q.pack(f);
            q.store(dst + e[r]);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (e[r] + k >= 0 && e[r] + k < dim) dst[e[r] + k] = from_float<B>(f[k]);
        }
    }
}

// ---------------------------------------------------------------------------------------------- sort

struct SortJob {
    Rows tokens;
    uint32_t n, n_tokens, n_workers, vocab, padding, none;  // none = n_workers * vocab: the key of tokens without a gradient
    uint32_t n_blocks, per_block;                           // blocks that sort, tokens of each (a multiple of kSortThreads)
    int passes, bits;
    uint64_t* tok[2];                                       // key and position, between the passes (the form without a cluster)
    uint32_t* table;
    uint32_t *order;                                        // the sorted tokens' positions, kLast set where a segment ends
    uint32_t *seg_begin, *seg_key, *n_segs, *chunk_seg;
    uint32_t chunk_shift;
    uint32_t share_shift;                                   // cluster form: log2 of the tokens of a block
    uint64_t* row_begin;                                    // or null
    uint32_t* barrier;
    uint32_t wait_limit;
    int* status;
};
constexpr uint32_t kLast = 1u << 31;

// Token t's key.
__device__ __forceinline__ uint32_t load_key(const SortJob& j, uint32_t t, bool report) {
    const uint32_t v = load_token(j.tokens, t, j.vocab);
    if (v == 0xFFFFFFFFu && report) record_error(j.status, ADACOMP_ERR_INVALID);
    return v == 0xFFFFFFFFu || v == j.padding ? j.none : (j.n_workers == 1 ? 0u : t / j.n_tokens * j.vocab) + v;
}

// Waits until all sorting blocks are here.  They are resident together (cooperative launch), so the wait ends; if it ever
// does not, the block says so and gives up: the sums then leave its lists alone.  From then on no block passes, in this call or
// a later one, until the host clears the words, whatever the count says: with the arrivals that were left behind it says so
// before all have delivered their counts, and places made of such counts lie anywhere.
__device__ __forceinline__ bool meet(const SortJob& j) {
    __shared__ int s_ok;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        const uint32_t target = (atomicAdd(j.barrier, 1u) / j.n_blocks + 1) * j.n_blocks;
        const uint32_t gave_up = __ldcg(j.barrier + 2);
        uint32_t seen = 0, polls = gave_up ? j.wait_limit : 0;
        do {
            asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(j.barrier) : "memory");
        } while (seen < target && polls++ < j.wait_limit);
        s_ok = seen >= target && gave_up == 0;
        if (seen < target) j.barrier[2] = 1;
    }
    __syncthreads();
    return s_ok != 0;
}

// Sum over the block's threads before this one, and over all of them.
template <int WARPS = kSortWarps>
__device__ __forceinline__ uint32_t block_before(uint32_t v, uint32_t* s_warp, uint32_t* total) {
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t upto = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, upto, d);
        if (lane >= static_cast<uint32_t>(d)) upto += y;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = upto;
    __syncthreads();
    const uint32_t w = WARPS == 32 || lane < WARPS ? s_warp[lane] : 0u;
    *total = __reduce_add_sync(0xFFFFFFFFu, w);
    return __reduce_add_sync(0xFFFFFFFFu, lane < warp ? w : 0u) + upto - v;
}

// Rows [r, stop) become zeros; where the table's rows follow each other without gaps, as one stretch of memory.
__device__ __forceinline__ void clear_rows(const Rows& out, uint64_t r, uint64_t stop, uint32_t dim, bool vec, uint32_t tid, uint32_t n_threads) {
    const uint32_t size = type_size(out.type);
    while (r < stop) {
        uint64_t end = r + 1;
        if (out.row_stride == dim) {
            end = stop;
            if (out.group && (r / out.group + 1) * out.group < end) end = (r / out.group + 1) * out.group;
        }
        char* dst = out.data + out.offset(static_cast<uint32_t>(r)) * size;
        const uint64_t bytes = (end - r) * dim * size;
        if (vec) {
            for (uint64_t c = tid * 16; c < bytes; c += n_threads * 16) *reinterpret_cast<uint4*>(dst + c) = make_uint4(0u, 0u, 0u, 0u);
        } else if (size == 4) {
            for (uint64_t c = tid * 4; c < bytes; c += n_threads * 4) *reinterpret_cast<uint32_t*>(dst + c) = 0u;
        } else {
            for (uint64_t c = tid * 2; c < bytes; c += n_threads * 2) *reinterpret_cast<uint16_t*>(dst + c) = 0;
        }
        r = end;
    }
}

// Clears rows while the tokens are being sorted on other SMs.  It needs nothing of the sort, but the sums wait for this
// kernel alone, so it ends after the sort.
__global__ void __launch_bounds__(kThreads) k_embed_clear(Rows out, uint64_t n_rows, uint32_t dim, int vec) {
    clear_rows(out, n_rows * blockIdx.x / gridDim.x, n_rows * (blockIdx.x + 1) / gridDim.x, dim, vec != 0, threadIdx.x, kThreads);
    cudaGridDependencySynchronize();
}

// Lanes of the warp that hold the same digit (of at most kDigitBits bits), among the real ones or among the others.  (The
// hardware's match instruction is no faster: 19.5 against 19.1 us for the sort of 32768 tokens.)
__device__ __forceinline__ uint32_t same_digit(uint32_t d, bool real) {
    const uint32_t all = __ballot_sync(0xFFFFFFFFu, real);
    uint32_t same = real ? all : ~all;
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
        const uint32_t vote = __ballot_sync(0xFFFFFFFFu, (d >> b) & 1);
        same &= (d >> b) & 1 ? vote : ~vote;
    }
    return same;
}

// Counts of digit `d` in the block's warps become the counts before each warp; returns their sum.
template <int WARPS = kSortWarps>
__device__ __forceinline__ uint32_t counts_to_places(uint16_t* s_count, uint32_t bins, uint32_t d) {
    uint32_t c[WARPS];
#pragma unroll
    for (int w = 0; w < WARPS; ++w) c[w] = s_count[w * bins + d];
    uint32_t sum = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
        s_count[w * bins + d] = static_cast<uint16_t>(sum);
        sum += c[w];
    }
    return sum;
}

// The same for digits 2 d and 2 d + 1 at once, in the halves of a word.
__device__ __forceinline__ uint32_t pair_counts_to_places(uint32_t* s_count, uint32_t pairs, uint32_t d) {
    uint32_t c[kSortWarps];
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) c[w] = s_count[w * pairs + d];
    uint32_t sum = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
        s_count[w * pairs + d] = sum;
        sum += c[w];
    }
    return sum;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// Sorted token i with key k between `last` and `next`, and its place in the lists that the sums read; `u` segments begin
// before it.
__device__ __forceinline__ void put_segment(const SortJob& j, uint64_t i, uint32_t k, uint32_t last, uint32_t next, uint32_t pos, bool head,
                                            uint32_t u) {
    if ((i & ((1u << j.chunk_shift) - 1)) == 0) j.chunk_seg[i >> j.chunk_shift] = u;
    j.order[i] = pos | (next != k ? kLast : 0u);
    if (head) {
        j.seg_begin[u] = static_cast<uint32_t>(i);
        j.seg_key[u] = k;
    }
    const bool end = k != j.none && next == j.none;                        // the last token with a gradient
    const uint32_t n_segs = u + head;
    if (end) {
        j.seg_begin[n_segs] = static_cast<uint32_t>(i) + 1;
        j.n_segs[0] = n_segs;
        j.n_segs[1] = static_cast<uint32_t>(i) + 1;
    }
    if (!j.row_begin || !(head || end)) return;
    if (j.n_workers == 1) {
        if (i == 0) j.row_begin[0] = 0;
        if (end) j.row_begin[1] = n_segs;
        return;
    }
    // only a worker's first token finds a worker before it that is not its own
    const uint32_t w = k / j.vocab;
    if (head && (i == 0 || last < w * j.vocab))
        for (uint32_t v = i == 0 ? 0u : last / j.vocab + 1; v <= w; ++v) j.row_begin[v] = u;
    if (end)
        for (uint32_t v = w + 1; v <= j.n_workers; ++v) j.row_begin[v] = n_segs;
}

// Block 0: the lists of a call without a token that has a gradient.
__device__ __forceinline__ void put_empty(const SortJob& j, bool nothing) {
    if (!nothing) return;
    if (threadIdx.x < 2) j.n_segs[threadIdx.x] = 0;
    if (j.row_begin)
        for (uint32_t v = threadIdx.x; v <= j.n_workers; v += kSortThreads) j.row_begin[v] = 0;
}

// Stable sort of the tokens by worker and token, and what the sums need to know about the sorted list.  Least significant
// digit first; a block ranks its tokens with ballots (a warp's rows of 32 in turn, one counter per warp and digit),
// the blocks tell each other their counts through a table in global memory.
__global__ void __launch_bounds__(kSortThreads, 1) k_embed_sort(const SortJob j) {
    cudaTriggerProgrammaticLaunchCompletion();              // the sums' blocks may line up: they wait for this kernel's end
    __shared__ uint16_t s_count[kSortWarps * kMaxBins];     // [warps][bins] of a digit in the warps before
    __shared__ uint32_t s_base[kMaxBins];
    __shared__ uint32_t s_all[kSortThreads], s_before[kSortThreads];
    __shared__ uint32_t s_warp[32];
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint64_t from = static_cast<uint64_t>(blockIdx.x) * j.per_block;
    const uint64_t to = from + j.per_block < j.n ? from + j.per_block : j.n;
    const uint32_t bins = 1u << j.bits, mask = bins - 1;
    uint16_t* mine = s_count + warp * bins;
    const uint32_t items = j.per_block < kStep ? j.per_block / kSortThreads : kItems;     // rows of 32 per warp and step
    const bool one_step = j.per_block <= kStep;
    uint64_t tok[kItems];
    uint32_t rank[kItems];
    for (int pass = 0; pass < j.passes; ++pass) {
        const uint64_t* in = j.tok[(pass & 1) ^ 1];
        const int shift = 32 + pass * j.bits;
        // Loads step `at`, ranks it and leaves s_count as places within the step; returns the step's count of digit tid.
        auto rank_step = [&](uint64_t at, bool report) -> uint32_t {
            for (uint32_t d = lane; d < bins / 2; d += 32) reinterpret_cast<uint32_t*>(mine)[d] = 0;
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
                const uint64_t t = at + (warp * items + i) * 32 + lane;
                if (i >= items || t >= to) continue;
                if (pass == 0) tok[i] = static_cast<uint64_t>(load_key(j, static_cast<uint32_t>(t), report)) << 32 | t;
                else tok[i] = __ldcg(in + t);
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
                if (i >= items) break;
                const bool real = at + (warp * items + i) * 32 + lane < to;
                const uint32_t d = static_cast<uint32_t>(tok[i] >> shift) & mask;
                const uint32_t same = same_digit(d, real);
                const uint32_t before = __popc(same & ((1u << lane) - 1));
                const uint32_t had = mine[d];
                rank[i] = had + before;
                __syncwarp();
                if (real && before == 0) mine[d] = static_cast<uint16_t>(had + __popc(same));
                __syncwarp();
            }
            __syncthreads();
            return tid < bins ? counts_to_places(s_count, bins, tid) : 0u;
        };
        uint32_t count = 0;
        for (uint64_t at = from; at < to || at == from; at += kStep) {
            if (at != from) __syncthreads();
            count += rank_step(at, true);
        }
        if (tid < bins) __stcg(j.table + blockIdx.x * bins + tid, count);
        if (!meet(j)) return;
        // the blocks' counts of a digit: kSortThreads / bins threads share them
        uint32_t all = 0, before = 0, total;
#pragma unroll 16
        for (uint32_t b = tid >> j.bits; b < j.n_blocks; b += kSortThreads >> j.bits) {
            const uint32_t c = __ldcg(j.table + b * bins + (tid & mask));
            all += c;
            if (b < blockIdx.x) before += c;
        }
        s_all[tid] = all;
        s_before[tid] = before;
        __syncthreads();
        if (tid < bins) {
            for (uint32_t k = tid + bins; k < kSortThreads; k += bins) {
                all += s_all[k];
                before += s_before[k];
            }
        }
        const uint32_t base = block_before(tid < bins ? all : 0u, s_warp, &total) + before;
        if (tid < bins) s_base[tid] = base;
        for (uint64_t at = from; at < to; at += kStep) {
            uint32_t step_count = 0;
            if (!one_step) {
                __syncthreads();
                step_count = rank_step(at, false);
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
                if (i >= items || at + (warp * items + i) * 32 + lane >= to) continue;
                const uint32_t d = static_cast<uint32_t>(tok[i] >> shift) & mask;
                __stcg(j.tok[pass & 1] + s_base[d] + mine[d] + rank[i], tok[i]);
            }
            if (!one_step) {
                __syncthreads();
                if (tid < bins) s_base[tid] += step_count;
            }
        }
        if (!meet(j)) return;
    }

    // Segments: where each begins, how many begin before every chunk, where each worker's begin.  A warp's tokens are
    // consecutive: neighbours come by shuffle, heads are counted by ballots, the warps' counts by one scan per step.
    const uint64_t* sorted = j.tok[(j.passes - 1) & 1];
    const uint64_t none = static_cast<uint64_t>(j.none) << 32;
    uint32_t heads[kItems], segs = 0, total;
    auto head_step = [&](uint64_t at) -> uint32_t {
        const uint64_t span = at + warp * items * 32 + lane;
        uint32_t before = j.none, in_warp = 0;                          // key in front of a row
#pragma unroll
        for (int i = 0; i < kItems; ++i)
            tok[i] = i < items && span + i * 32 < to ? __ldcg(sorted + span + i * 32) : none;
        if (span - lane > 0 && span - lane < j.n) before = static_cast<uint32_t>(__ldcg(sorted + (span - lane) - 1) >> 32);
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const uint32_t k = static_cast<uint32_t>(tok[i] >> 32);
            uint32_t last = __shfl_up_sync(0xFFFFFFFFu, k, 1);
            if (lane == 0) last = before;
            heads[i] = i < items ? __ballot_sync(0xFFFFFFFFu, k != j.none && (last != k || span + i * 32 == 0)) : 0u;
            in_warp += __popc(heads[i]);
            before = __shfl_sync(0xFFFFFFFFu, k, 31);
        }
        return in_warp;
    };
    uint32_t in_warp = 0;
    for (uint64_t at = from; at < to; at += kStep) {
        in_warp = head_step(at);
        block_before(lane == 0 ? in_warp : 0u, s_warp, &total);
        segs += total;
    }
    if (tid == 0) __stcg(j.table + blockIdx.x, segs);
    if (!meet(j)) return;
    block_before(tid < blockIdx.x ? __ldcg(j.table + tid) : 0u, s_warp, &total);
    segs = total;
    for (uint64_t at = from; at < to; at += kStep) {
        const uint64_t span = at + warp * items * 32 + lane;
        if (!one_step) in_warp = head_step(at);
        uint32_t u = segs + __shfl_sync(0xFFFFFFFFu, block_before(lane == 0 ? in_warp : 0u, s_warp, &total), 0);
        segs += total;
        uint32_t before = j.none, behind = j.none;
        const uint64_t first = span - lane, end = first + items * 32;
        if (first > 0 && first < j.n) before = static_cast<uint32_t>(__ldcg(sorted + first - 1) >> 32);
        if (end < j.n) behind = static_cast<uint32_t>(__ldcg(sorted + end) >> 32);
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            if (i >= items) break;
            const uint64_t t = span + i * 32;
            const uint32_t k = static_cast<uint32_t>(tok[i] >> 32);
            uint32_t last = __shfl_up_sync(0xFFFFFFFFu, k, 1), next = __shfl_down_sync(0xFFFFFFFFu, k, 1);
            const uint32_t behind_row = static_cast<uint32_t>(tok[i + 1 < kItems ? i + 1 : i] >> 32);
            const uint32_t after = i + 1 < items ? __shfl_sync(0xFFFFFFFFu, behind_row, 0) : behind;
            if (lane == 0) last = before;
            if (lane == 31) next = after;
            if (t < to)
                put_segment(j, t, k, last, t + 1 < j.n ? next : j.none, static_cast<uint32_t>(tok[i]), heads[i] >> lane & 1,
                            u + __popc(heads[i] & ((1u << lane) - 1)));
            u += __popc(heads[i]);
            before = __shfl_sync(0xFFFFFFFFu, k, 31);
        }
    }
    if (blockIdx.x == 0) put_empty(j, __ldcg(sorted) >> 32 == j.none);
    // the last block through leaves the barrier as it was
    if (tid == 0 && atomicAdd(j.barrier + 1, 1u) == j.n_blocks - 1) {
        j.barrier[0] = 0;
        j.barrier[1] = 0;
    }
}

// The same sort for up to kClusterStep tokens per block in one thread-block cluster: the tokens stay in registers and shared
// memory, a block's counts and the tokens themselves go straight to the shared memory of the block they belong to, and the
// cluster's barrier takes the place of the one in global memory.
__global__ void __launch_bounds__(kSortThreads, 1) k_embed_sort_cluster(const SortJob j) {
    extern __shared__ uint64_t s_mem64[];
    __shared__ uint32_t s_base[kMaxBins];
    __shared__ uint32_t s_warp[32];
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    cudaTriggerProgrammaticLaunchCompletion();
    cluster_arrive();
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t n_ranks = gridDim.x, me = blockIdx.x;    // one cluster
    const uint32_t share = 1u << j.share_shift, items = share / kSortThreads;
    uint64_t* s_tok = s_mem64;                                                  // [share] key and position
    const uint32_t bins = 1u << j.bits, mask = bins - 1;
    const uint32_t pairs = bins / 2;                                            // digits are counted in 16 bits, two to a word
    uint32_t* s_all = reinterpret_cast<uint32_t*>(s_tok + share);               // [n_ranks][pairs] the blocks' counts
    uint16_t* s_count = reinterpret_cast<uint16_t*>(s_all + n_ranks * pairs);   // [kSortWarps][bins]
    uint16_t* mine = s_count + warp * bins;
    const uint32_t from = me << j.share_shift;
    const uint32_t n_here = j.n > from ? (j.n - from < share ? j.n - from : share) : 0;
    const uint32_t span = warp * items * 32 + lane;                             // the warp's tokens: rows of 32, one after the other
    uint64_t tok[kClusterItems];
    uint32_t rank[kClusterItems];
#pragma unroll
    for (int i = 0; i < kClusterItems; ++i) {
        const uint32_t t = span + i * 32;
        tok[i] = static_cast<uint64_t>(j.none) << 32;
        if (i >= items || t >= n_here) continue;
        tok[i] = static_cast<uint64_t>(load_key(j, from + t, true)) << 32 | (from + t);
    }
    cluster_wait();                             // every block has started: its shared memory may be written from here on
    for (int pass = 0; pass < j.passes; ++pass) {
        const int shift = 32 + pass * j.bits;
        for (uint32_t d = lane; d < pairs; d += 32) reinterpret_cast<uint32_t*>(mine)[d] = 0;
        if (pass > 0) {
#pragma unroll
            for (int i = 0; i < kClusterItems; ++i)
                if (i < items && span + i * 32 < n_here) tok[i] = s_tok[span + i * 32];
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kClusterItems; ++i) {
            if (i >= items) break;
            const bool real = span + i * 32 < n_here;
            const uint32_t d = static_cast<uint32_t>(tok[i] >> shift) & mask;
            const uint32_t same = same_digit(d, real);
            const uint32_t before = __popc(same & ((1u << lane) - 1));
            const uint32_t had = mine[d];
            rank[i] = had + before;
            __syncwarp();
            if (real && before == 0) mine[d] = static_cast<uint16_t>(had + __popc(same));
            __syncwarp();
        }
        __syncthreads();
        if (tid < pairs) {
            const uint32_t both = pair_counts_to_places(reinterpret_cast<uint32_t*>(s_count), pairs, tid);
            for (uint32_t r = 0; r < n_ranks; ++r) cluster.map_shared_rank(s_all, r)[me * pairs + tid] = both;
        }
        cluster.sync();                         // the counts have arrived, and every block has its tokens in registers
        uint32_t all[2] = {0, 0}, before[2] = {0, 0}, total;
        if (tid < pairs) {
            for (uint32_t r = 0; r < n_ranks; ++r) {
                const uint32_t c = s_all[r * pairs + tid];
                all[0] += c & 0xFFFFu;
                all[1] += c >> 16;
                if (r < me) {
                    before[0] += c & 0xFFFFu;
                    before[1] += c >> 16;
                }
            }
        }
        const uint32_t base = block_before(all[0] + all[1], s_warp, &total);
        if (tid < pairs) {
            s_base[2 * tid] = base + before[0];
            s_base[2 * tid + 1] = base + all[0] + before[1];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kClusterItems; ++i) {
            if (i >= items) break;
            if (span + i * 32 >= n_here) continue;
            const uint32_t d = static_cast<uint32_t>(tok[i] >> shift) & mask;
            const uint32_t place = s_base[d] + mine[d] + rank[i];
            cluster.map_shared_rank(s_tok, place >> j.share_shift)[place & (share - 1)] = tok[i];
        }
        cluster.sync();
    }
    // Segments.  A warp's tokens are consecutive: its heads are counted by ballots, the warps' counts by one scan.
    const uint32_t* s_key = reinterpret_cast<const uint32_t*>(s_tok) + 1;       // [2 t] is token t's key
    uint32_t before_me = j.none, behind_me = j.none;
    if (me > 0) before_me = cluster.map_shared_rank(s_key, me - 1)[2 * (share - 1)];
    if (n_here == share && from + share < j.n) behind_me = cluster.map_shared_rank(s_key, me + 1)[0];
    uint32_t heads[kClusterItems], in_warp = 0;
#pragma unroll
    for (int i = 0; i < kClusterItems; ++i) {
        heads[i] = 0;
        if (i >= items) break;
        const uint32_t t = span + i * 32;
        bool head = false;
        if (t < n_here && s_key[2 * t] != j.none) head = t == 0 ? me == 0 || before_me != s_key[0] : s_key[2 * t - 2] != s_key[2 * t];
        heads[i] = __ballot_sync(0xFFFFFFFFu, head);
        in_warp += __popc(heads[i]);
    }
    uint32_t segs_here;
    uint32_t u = __shfl_sync(0xFFFFFFFFu, block_before(lane == 0 ? in_warp : 0u, s_warp, &segs_here), 0);
    if (tid < n_ranks) cluster.map_shared_rank(s_all, tid)[me] = segs_here;
    cluster.sync();
    cluster_arrive();                           // no more reads of the neighbours' shared memory
    for (uint32_t r = 0; r < me; ++r) u += s_all[r];
#pragma unroll
    for (int i = 0; i < kClusterItems; ++i) {
        if (i >= items) break;
        const uint32_t t = span + i * 32;
        if (t < n_here) {
            const uint64_t x = s_tok[t];
            const uint32_t last = t == 0 ? before_me : s_key[2 * t - 2];
            const uint32_t next = t + 1 < n_here ? s_key[2 * t + 2] : t + 1 == share ? behind_me : j.none;
            put_segment(j, from + t, static_cast<uint32_t>(x >> 32), last, next, static_cast<uint32_t>(x), heads[i] >> lane & 1,
                        u + __popc(heads[i] & ((1u << lane) - 1)));
        }
        u += __popc(heads[i]);
    }
    if (me == 0) put_empty(j, j.n == 0 || s_key[0] == j.none);
    cluster_wait();                             // nobody leaves while a neighbour may still read here
}

// ---------------------------------------------------------------------------------------------- sums

struct Sums {
    const uint32_t *order, *seg_begin, *seg_key, *chunk_seg, *n_segs;
    uint32_t n_chunks, chunk_shift;
    uint32_t tiles;                 // blocks along a row
    uint32_t sum_blocks;            // the blocks behind them write zeros
    float* partial;
    uint32_t* tickets;              // [levels][max_chunks][2][tiles]
    uint32_t max_chunks;
    const uint32_t* gave_up;
    Rows grad;
    uint32_t dim, vocab;
    float scale;
    // rows form
    uint32_t* rows_out;
    uint64_t* row_begin;
    uint32_t n_workers;
    char* values;
    uint32_t* idx_out;
    uint32_t idx_offset;
    // dense form
    int dense, accumulate;
    Rows out;
    uint64_t zero_first, zero_rows; // rows that become zeros where they have no token: zero_first .. zero_rows - 1
    int zero_vec;
    int wide;                       // rows of the results start on 32-byte boundaries
};

constexpr int kSumThreads = 288;               // a warp more than 256: rows of 257 .. 288 threads' width stay in one block
constexpr uint32_t kFanBits = 4, kFan = 1u << kFanBits;      // pieces that one block adds up
constexpr uint64_t kEnds = 1ull << 63;          // flag of a token that is its segment's last

// A finished sum goes to its row: `slot` counts segments, `at` is where the row starts in the dense table.
template <typename B, int N>
__device__ __forceinline__ void put_row(const Sums& p, uint32_t slot, uint64_t at, uint32_t row, uint32_t c, float (&sum)[N]) {
    B* dst = p.dense ? reinterpret_cast<B*>(p.out.data) + at + c : reinterpret_cast<B*>(p.values) + static_cast<uint64_t>(slot) * p.dim + c;
#pragma unroll
    for (int k = 0; k < N; ++k) sum[k] = __fmul_rn(sum[k], p.scale);
    if constexpr (N > 1) {
        Packed<B, N> q;
        if (p.accumulate) {
            float old[N];
#pragma unroll
            for (int i = 0; i < Packed<B, N>::kVecs; ++i) q.v[i] = reinterpret_cast<const uint4*>(dst)[i];
            q.unpack(old);
#pragma unroll
            for (int k = 0; k < N; ++k) sum[k] = __fadd_rn(sum[k], old[k]);
        }
        q.pack(sum);
        if (Packed<B, N>::kVecs == 2 && p.wide) store32(dst, q.v[0], q.v[Packed<B, N>::kVecs - 1]);
        else q.store(dst);
    } else {
        if (p.accumulate) sum[0] = __fadd_rn(sum[0], to_float(*dst));
        *dst = from_float<B>(sum[0]);
    }
    if (p.idx_out) {
        uint32_t* idx = p.idx_out + static_cast<uint64_t>(slot) * p.dim + c;
        const uint32_t first = p.idx_offset + row * p.dim + c;
        if constexpr (N == 8) {
            const uint4 a = make_uint4(first, first + 1, first + 2, first + 3), b = make_uint4(first + 4, first + 5, first + 6, first + 7);
            if (p.wide) {
                store32(idx, a, b);
            } else {
                reinterpret_cast<uint4*>(idx)[0] = a;
                reinterpret_cast<uint4*>(idx)[1] = b;
            }
        } else if constexpr (N == 4) {
            *reinterpret_cast<uint4*>(idx) = make_uint4(first, first + 1, first + 2, first + 3);
        } else {
            *idx = first;
        }
    }
}

// First of the n ascending keys that is not below `bound`, by whole warps (the block has no other): 32 probes a step (one at a
// time, 17 steps to the L2 and back took longer than the clearing they were for).
__device__ __forceinline__ uint32_t warp_lower_bound(const uint32_t* keys, uint32_t n, uint64_t bound) {
    const uint32_t lane = threadIdx.x + threadIdx.y * blockDim.x & 31;
    uint32_t lo = 0, hi = n;
    while (lo < hi) {
        const uint32_t step = (hi - lo + 31) / 32, at = lo + lane * step;
        const uint32_t below = __popc(__ballot_sync(0xFFFFFFFFu, at < hi && keys[at] < bound));
        if (below == 0) return lo;
        lo += (below - 1) * step + 1;
        if (lo + step - 1 < hi) hi = lo + step - 1;
    }
    return lo;
}

// A block's share of the rows without a token: the stretches between the keys of the sorted list.
__device__ void zero_gaps(const Sums& p, uint32_t block, uint32_t n_blocks) {
    constexpr uint32_t kKeys = 64;
    __shared__ uint32_t s_key[kKeys];
    const uint32_t n_segs = p.n_segs[0], tid = threadIdx.y * blockDim.x + threadIdx.x, n_threads = blockDim.x * blockDim.y;
    const uint64_t rows = p.zero_rows - p.zero_first;
    const uint64_t from = p.zero_first + rows * block / n_blocks, to = p.zero_first + rows * (block + 1) / n_blocks;
    uint32_t base = warp_lower_bound(p.seg_key, n_segs, from), k = kKeys;
    for (uint64_t r = from; r < to;) {
        if (k == kKeys) {
            __syncthreads();
            for (uint32_t i = tid; i < kKeys; i += n_threads) s_key[i] = base + i < n_segs ? p.seg_key[base + i] : 0xFFFFFFFFu;
            __syncthreads();
            base += kKeys;
            k = 0;
        }
        const uint64_t next = s_key[k] < to ? s_key[k] : to;
        clear_rows(p.out, r, next, p.dim, p.zero_vec != 0, tid, n_threads);
        r = next + 1;
        ++k;
    }
}

// Piece of a long segment that chunk `chunk` has summed: the one that begins in front of the chunk (0), or in it (1).
__device__ __forceinline__ float* piece_at(const Sums& p, uint32_t chunk, uint32_t which, uint32_t c) {
    return p.partial + (static_cast<uint64_t>(chunk) * 2 + which) * p.dim + c;
}
template <int N> __device__ __forceinline__ void put_piece(float* dst, const float (&sum)[N]) {
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int q = 0; q < N; q += 4) *reinterpret_cast<float4*>(dst + q) = make_float4(sum[q], sum[q + 1], sum[q + 2], sum[q + 3]);
    } else {
#pragma unroll
        for (int q = 0; q < N; ++q) dst[q] = sum[q];
    }
}

// Sums of one chunk's tokens: s_src says where their rows start and which of them end a segment, s_dst where the segments'
// results go.  `slot` is the first token's segment, u0 the first one that begins in the chunk.  A thread keeps K groups of N
// columns, `step` apart: N > 1 and K = 1 where rows sit on the 16-byte grid, N = 1 and K > 1 where they do not (one column at
// a time would leave too little in flight).
template <typename A, typename B, int N, int K, int BATCH>
__device__ __forceinline__ void sum_chunk(const Sums& p, const uint64_t* s_src, const uint64_t* s_dst, uint32_t len, uint32_t slot, uint32_t u0,
                                          uint32_t chunk, uint32_t c, uint32_t step) {
    float sum[K][N];
#pragma unroll
    for (int g = 0; g < K; ++g)
#pragma unroll
        for (int q = 0; q < N; ++q) sum[g][q] = 0.f;
    const A* grad = reinterpret_cast<const A*>(p.grad.data) + c;
    bool open = false;
    constexpr int kBatch = N * sizeof(A) == 32 ? BATCH / 2 : BATCH;         // rows in flight
    for (uint32_t i = 0; i < len; i += kBatch) {
        Packed<A, N> v[kBatch][K];
        uint64_t at[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) at[k] = s_src[i + k < len ? i + k : len - 1];
        // no branch between the loads, the last rows of a chunk repeat its last: 524288 tokens x 2048 455 -> 448 us for the call,
        // rows of 1001 bf16 entries 109 -> 81
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
#pragma unroll
            for (int g = 0; g < K; ++g) v[k][g].load(grad + (at[k] & ~kEnds) + (c + g * step < p.dim ? g * step : 0));
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (i + k >= len) break;
#pragma unroll
            for (int g = 0; g < K; ++g) {
                float f[N];
                v[k][g].unpack(f);
#pragma unroll
                for (int q = 0; q < N; ++q) sum[g][q] = __fadd_rn(sum[g][q], f[q]);
            }
            open = true;
            if (!(at[k] & kEnds)) continue;
            const bool piece = slot + 1 == u0;          // the last piece of a long segment
            const uint64_t at = piece ? 0 : s_dst[slot - u0];
#pragma unroll
            for (int g = 0; g < K; ++g) {
                if (g == 0 || c + g * step < p.dim) {
                    if (piece) put_piece<N>(piece_at(p, chunk, 0, c + g * step), sum[g]);
                    else put_row<B, N>(p, slot, at, static_cast<uint32_t>(at), c + g * step, sum[g]);
                }
#pragma unroll
                for (int q = 0; q < N; ++q) sum[g][q] = 0.f;
            }
            ++slot;
            open = false;
        }
    }
    if (!open) return;
#pragma unroll
    for (int g = 0; g < K; ++g)                         // a piece that goes on in the next chunk
        if (g == 0 || c + g * step < p.dim) put_piece<N>(piece_at(p, chunk, slot + 1 == u0 ? 0 : 1, c + g * step), sum[g]);
}

// What a chunk has to do.
struct Share {
    uint32_t a, b;                  // its tokens
    uint32_t u0, u1;                // the segments that begin in it
    bool lead, trail;               // whether it begins, ends with a piece of a long segment
};
template <typename Begin>
__device__ __forceinline__ Share share_of(uint64_t i0, uint32_t size, uint32_t live, uint32_t u0, uint32_t u1, const Begin& seg_begin) {
    Share s = {0, 0, u0, u1, false, false};
    const uint32_t i1 = static_cast<uint32_t>(i0 + size < live ? i0 + size : live);
    const uint32_t first = seg_begin[u0];                   // of the segments that begin here (or the end of the list)
    if (first > i0) s.lead = first - seg_begin[u0 - 1] > size;
    s.a = s.lead ? static_cast<uint32_t>(i0) : first;
    if (u1 > u0) {
        const uint32_t end = seg_begin[u1];
        s.trail = end - seg_begin[u1 - 1] > size;
        s.b = s.trail ? i1 : end;
    } else {
        s.b = !s.lead ? s.a : first < i1 ? first : i1;
    }
    return s;
}

// The pieces of long segments that a chunk has just delivered: the one it begins with (0) and the one it ends with (1).  The block
// that delivers the last of kFan consecutive pieces adds them up, in order, in the place of the first, and delivers that sum
// as a piece of the next level, until the segment is one.  So nobody waits, the tree of additions is fixed, and a segment of
// any length costs a few turns.  The whole block takes part.
struct Pieces {
    uint32_t head[2], count[2], seg[2];     // chunk in which the segment begins, its chunks (0: no piece), its number
};
template <typename Begin>
__device__ __forceinline__ Pieces pieces_of(const Share& s, uint32_t chunk, uint32_t shift, const Begin& seg_begin) {
    Pieces x = {{0, chunk}, {0, 0}, {s.u0 - 1, s.u1 - 1}};
    if (s.lead) {
        x.head[0] = seg_begin[s.u0 - 1] >> shift;
        x.count[0] = ((seg_begin[s.u0] - 1) >> shift) - x.head[0] + 1;
    }
    if (s.trail) x.count[1] = ((seg_begin[s.u1] - 1) >> shift) - chunk + 1;
    return x;
}
template <typename B, int N, int K, typename KeyOf>
__device__ __forceinline__ void finish_long(const Sums& p, const Pieces& x, uint32_t chunk, uint32_t tile, uint32_t c, uint32_t step, bool leader,
                                            const KeyOf& key_of, uint32_t* s_last) {
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        const uint32_t head = x.head[which];
        uint32_t count = x.count[which], node = chunk - head, level = 0;
        bool active = count > 0;
        while (__syncthreads_or(active)) {
            const uint32_t parent = node >> kFanBits, width = kFanBits * level;
            const uint32_t first = head + (parent << (width + kFanBits));                   // chunk of the group's first piece
            const uint32_t n = active ? (count - parent * kFan < kFan ? count - parent * kFan : kFan) : 0;
            if (active) __threadfence();
            __syncthreads();
            if (leader) {
                *s_last = 0;
                if (active) {
                    uint32_t* ticket = p.tickets + ((static_cast<uint64_t>(level) * p.max_chunks + first) * 2 + (first == head)) * p.tiles + tile;
                    if (atomicAdd(ticket, 1u) == n - 1) {
                        *ticket = 0;
                        *s_last = 1;
                    }
                }
            }
            __syncthreads();
            active = active && *s_last;
            if (!active) continue;
            __threadfence();
            const bool whole = count <= kFan;
#pragma unroll 1
            for (uint32_t g = 0, col = c; g < K && col < p.dim; ++g, col += step) {
                float sum[N];
#pragma unroll
                for (int k = 0; k < N; ++k) sum[k] = 0.f;
                for (uint32_t q = 0; q < n; q += 4) {
                    float f[4][N];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const uint32_t at = first + ((q + r) << width);
                        const float* src = piece_at(p, at, at == head ? 1 : 0, col);
                        if constexpr (N % 4 == 0) {
#pragma unroll
                            for (int k = 0; k < N; k += 4) {
                                const float4 v = q + r < n ? __ldcg(reinterpret_cast<const float4*>(src + k)) : make_float4(0.f, 0.f, 0.f, 0.f);
                                f[r][k] = v.x; f[r][k + 1] = v.y; f[r][k + 2] = v.z; f[r][k + 3] = v.w;
                            }
                        } else {
                            f[r][0] = q + r < n ? __ldcg(src) : 0.f;
                        }
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (q + r < n)
#pragma unroll
                            for (int k = 0; k < N; ++k) sum[k] = __fadd_rn(sum[k], f[r][k]);
                }
                if (whole) {
                    const uint32_t key = key_of(x.seg[which]);
                    put_row<B, N>(p, x.seg[which], p.dense ? p.out.offset(key) : 0, key % p.vocab, col, sum);
                } else {
                    put_piece<N>(piece_at(p, first, first == head ? 1 : 0, col), sum);
                }
            }
            if (whole) active = false;
            node = parent;
            count = (count + kFan - 1) >> kFanBits;
            ++level;
        }
    }
}

// A call whose sort gave up, or that sorts in this way after one that did: its lists read as empty.
__device__ __forceinline__ void put_no_rows(const Sums& p) {
    if (blockIdx.x != 0 || !p.row_begin) return;
    for (uint32_t w = threadIdx.y * blockDim.x + threadIdx.x; w <= p.n_workers; w += blockDim.x * blockDim.y) p.row_begin[w] = 0;
}

// Sums over the sorted list, cut into chunks of 2^chunk_shift tokens.  A chunk owns the segments that begin in it, to their
// end even if that lies in the next chunk; a segment longer than a chunk is cut at the chunks' borders, its pieces are
// added up by finish_long.  So the work per chunk is bounded, short segments need no second pass and the tree of additions
// depends on the tokens alone.  A thread keeps N columns; x runs along the row, y over chunks.
template <typename A, typename B, int N, int K>
__global__ void __launch_bounds__(kSumThreads, K == 1 ? 4 : 3) k_embed_sums(const Sums p) {
    extern __shared__ uint64_t s_mem[];
    cudaGridDependencySynchronize();
    if (*p.gave_up) {                                       // the sort did not get through: its lists are not to be followed
        put_no_rows(p);
        return;
    }
    if (blockIdx.x >= p.sum_blocks) {
        zero_gaps(p, blockIdx.x - p.sum_blocks, gridDim.x - p.sum_blocks);
        return;
    }
    const uint32_t size = 1u << p.chunk_shift;
    uint64_t* s_src = s_mem + static_cast<size_t>(threadIdx.y) * (3 * size);    // [2 size] where the rows of the chunk's tokens start
    uint64_t* s_dst = s_src + 2 * size;                                         // [size] where its segments' rows start
    const uint32_t chunk = blockIdx.x / p.tiles * blockDim.y + threadIdx.y, tile = blockIdx.x % p.tiles;
    const uint32_t n_segs = p.n_segs[0], live = p.n_segs[1];
    const uint32_t c = (tile * K * blockDim.x + threadIdx.x) * N;
    const uint64_t i0 = static_cast<uint64_t>(chunk) << p.chunk_shift;
    Share s = {};
    if (i0 < live) s = share_of(i0, size, live, p.chunk_seg[chunk], i0 + size < live ? p.chunk_seg[chunk + 1] : n_segs, p.seg_begin);
    for (uint32_t k = threadIdx.x; k < s.b - s.a; k += blockDim.x) {
        const uint32_t at = p.order[s.a + k];
        s_src[k] = p.grad.offset(at & ~kLast) | (at & kLast ? kEnds : 0ull);
    }
    for (uint32_t k = threadIdx.x; k < s.u1 - s.u0; k += blockDim.x) {
        const uint32_t key = p.seg_key[s.u0 + k];
        s_dst[k] = p.dense ? p.out.offset(key) : key % p.vocab;
        if (p.rows_out && tile == 0) p.rows_out[s.u0 + k] = key % p.vocab;
    }
    __syncthreads();
    // Four rows in flight per thread, 56 registers (four blocks of 256 per SM; from 16-bit rows to fp32 8 bytes spill, between
    // other types none): 524288 tokens x 2048 bf16 in 404 us, 6.3 TB/s with the pieces of long segments counted.  Measured against
    // it: the next four rows fetched before the last are added (80 registers) 430 us; rings of asynchronous copies to shared
    // memory, eight rows deep, 410; five blocks per SM, which spill more, +12 %.  An ordinary update (4 x 8192 tokens x 1024) has
    // 1024 blocks for 592 places and four dependent reads before a block's first sum: 167 MB in 38 us, 4.4 TB/s.
    if (c < p.dim) sum_chunk<A, B, N, K, 4>(p, s_src, s_dst, s.b - s.a, s.lead ? s.u0 - 1 : s.u0, s.u0, chunk, c, blockDim.x * N);
    if (!__syncthreads_or(s.lead || s.trail)) return;
    finish_long<B, N, K>(p, pieces_of(s, chunk, p.chunk_shift, p.seg_begin), chunk, tile, c, blockDim.x * N, threadIdx.x == 0,
                         [&](uint32_t u) { return p.seg_key[u]; }, reinterpret_cast<uint32_t*>(s_src));
}

// ---------------------------------------------------------------------------------------------- few tokens

// Few tokens: one launch does everything.  Every block sorts all tokens for itself in shared memory, which
// takes less than a second kernel's start, and then sums its chunks; the block that delivers the last piece of a long segment
// adds the pieces up.  Two blocks per SM leave 64 registers a thread: 16 to 92
// bytes spill, most with 16-bit rows.
constexpr int kSmallThreads = 512, kSmallWarps = kSmallThreads / 32, kSmallItems = 4;
constexpr uint32_t kSmallTokens = kSmallThreads * kSmallItems;
constexpr uint32_t kSmallShift = 3, kSmallChunk = 1u << kSmallShift, kSmallChunks = kSmallTokens / kSmallChunk;
constexpr uint32_t kSmallLanes = 64;                        // chunks a block takes at a time, at most

struct SmallMem {
    __device__ __forceinline__ uint32_t key(uint32_t t) const { return static_cast<uint32_t>(tok[t] >> 32); }
    __device__ __forceinline__ uint32_t seg_key(uint32_t u) const { return key(seg_begin[u]); }
    uint64_t tok[kSmallTokens];                             // key and position
    union {
        uint16_t count[kSmallWarps * kMaxBins];
        uint64_t rows[kSmallLanes][3 * kSmallChunk];        // s_src and s_dst of sum_chunk
    };
    uint32_t base[kMaxBins];
    uint32_t warp[32];
    uint16_t seg_begin[kSmallTokens + 1];
    uint16_t chunk_seg[kSmallChunks + 1];
    uint32_t n_segs, live, any_long;
    uint32_t last[kSmallLanes + 1];                         // whether a chunk's piece was the last one of its group
};

__device__ __forceinline__ void sort_small(const SortJob& j, SmallMem& m) {
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t bins = 1u << j.bits, mask = bins - 1;
    const uint32_t items = (j.n + kSmallThreads - 1) / kSmallThreads;
    const uint32_t span = warp * items * 32 + lane;
    uint16_t* mine = m.count + warp * bins;
    uint64_t tok[kSmallItems];
    uint32_t rank[kSmallItems], total;
    if (tid == 0) m.n_segs = m.live = m.any_long = 0;
#pragma unroll
    for (int i = 0; i < kSmallItems; ++i) {
        const uint32_t t = span + i * 32;
        tok[i] = static_cast<uint64_t>(j.none) << 32;
        if (i < items && t < j.n) tok[i] = static_cast<uint64_t>(load_key(j, t, blockIdx.x == 0)) << 32 | t;
    }
    for (int pass = 0; pass < j.passes; ++pass) {
        const int shift = 32 + pass * j.bits;
        for (uint32_t d = lane; d < bins / 2; d += 32) reinterpret_cast<uint32_t*>(mine)[d] = 0;
        if (pass > 0) {
#pragma unroll
            for (int i = 0; i < kSmallItems; ++i)
                if (i < items && span + i * 32 < j.n) tok[i] = m.tok[span + i * 32];
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kSmallItems; ++i) {
            if (i >= items || span - lane + i * 32 >= j.n) break;
            const bool real = span + i * 32 < j.n;
            const uint32_t d = static_cast<uint32_t>(tok[i] >> shift) & mask;
            const uint32_t same = same_digit(d, real);
            const uint32_t before = __popc(same & ((1u << lane) - 1));
            const uint32_t had = mine[d];
            rank[i] = had + before;
            __syncwarp();
            if (real && before == 0) mine[d] = static_cast<uint16_t>(had + __popc(same));
            __syncwarp();
        }
        __syncthreads();
        const uint32_t all = tid < bins ? counts_to_places<kSmallWarps>(m.count, bins, tid) : 0u;
        const uint32_t base = block_before<kSmallWarps>(all, m.warp, &total);
        if (tid < bins) m.base[tid] = base;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kSmallItems; ++i) {
            if (i >= items || span + i * 32 >= j.n) continue;
            const uint32_t d = static_cast<uint32_t>(tok[i] >> shift) & mask;
            m.tok[m.base[d] + mine[d] + rank[i]] = tok[i];
        }
        __syncthreads();
    }
    uint32_t heads[kSmallItems], in_warp = 0;
#pragma unroll
    for (int i = 0; i < kSmallItems; ++i) {
        const uint32_t t = span + i * 32;
        bool head = false;
        if (i < items && t < j.n) {
            const uint32_t k = m.key(t);
            head = k != j.none && (t == 0 || m.key(t - 1) != k);
        }
        heads[i] = __ballot_sync(0xFFFFFFFFu, head);
        in_warp += __popc(heads[i]);
    }
    uint32_t u = __shfl_sync(0xFFFFFFFFu, block_before<kSmallWarps>(lane == 0 ? in_warp : 0u, m.warp, &total), 0);
#pragma unroll
    for (int i = 0; i < kSmallItems; ++i) {
        const uint32_t t = span + i * 32;
        if (i < items && t < j.n) {
            const uint32_t k = m.key(t);
            const uint32_t at = u + __popc(heads[i] & ((1u << lane) - 1));
            const bool head = heads[i] >> lane & 1;
            if (t % kSmallChunk == 0) m.chunk_seg[t / kSmallChunk] = static_cast<uint16_t>(at);
            if (head) m.seg_begin[at] = static_cast<uint16_t>(t);
            if (k != j.none) {
                if (t + kSmallChunk < j.n && m.key(t + kSmallChunk) == k) m.any_long = 1;
                if (t + 1 == j.n || m.key(t + 1) == j.none) {
                    m.n_segs = at + head;
                    m.live = t + 1;
                    m.seg_begin[at + head] = static_cast<uint16_t>(t + 1);
                }
            }
        }
        u += __popc(heads[i]);
    }
    __syncthreads();
}

// Rows without a token in this block's share of the table: the stretches between two rows that have one.
__device__ __forceinline__ void clear_small(const Sums& p, const SmallMem& m) {
    const uint64_t from = p.zero_rows * blockIdx.x / gridDim.x, to = p.zero_rows * (blockIdx.x + 1) / gridDim.x;
    uint32_t lo = 0, hi = m.n_segs;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (m.seg_key(mid) < from) lo = mid + 1; else hi = mid;
    }
    for (uint64_t r = from; r < to; ++lo) {
        const uint64_t next = lo < m.n_segs && m.seg_key(lo) < to ? m.seg_key(lo) : to;
        clear_rows(p.out, r, next, p.dim, p.zero_vec != 0, threadIdx.x, kSmallThreads);
        r = next + 1;
    }
}

template <typename A, typename B, int N>
__global__ void __launch_bounds__(kSmallThreads, 2) k_embed_small(const SortJob j, const Sums p, uint32_t x, uint32_t y) {
    __shared__ SmallMem m;
    sort_small(j, m);
    if (blockIdx.x == 0 && j.row_begin && j.n_workers == 1) {
        if (threadIdx.x < 2) j.row_begin[threadIdx.x] = threadIdx.x ? m.n_segs : 0;
    } else if (blockIdx.x == 0 && j.row_begin) {
        for (uint32_t w = threadIdx.x; w <= j.n_workers; w += kSmallThreads) {
            uint32_t lo = 0, hi = m.n_segs;
            while (lo < hi) {
                const uint32_t mid = (lo + hi) / 2;
                if (m.seg_key(mid) < static_cast<uint64_t>(w) * j.vocab) lo = mid + 1; else hi = mid;
            }
            j.row_begin[w] = lo;
        }
    }
    const uint32_t tx = threadIdx.x % x, ty = threadIdx.x / x;
    const uint32_t jobs = (p.n_chunks + y - 1) / y * p.tiles;
    for (uint32_t job = blockIdx.x; job < jobs; job += gridDim.x) {
        const uint32_t chunk = job / p.tiles * y + ty, tile = job % p.tiles, c = (tile * x + tx) * N;
        const uint32_t i0 = chunk * kSmallChunk;
        uint64_t* s_src = m.rows[ty < y ? ty : 0];
        uint64_t* s_dst = s_src + 2 * kSmallChunk;
        Share s = {};
        if (ty < y && i0 < m.live) {
            s = share_of(i0, kSmallChunk, m.live, m.chunk_seg[chunk], i0 + kSmallChunk < m.live ? m.chunk_seg[chunk + 1] : m.n_segs,
                         m.seg_begin);
            for (uint32_t k = tx; k < s.b - s.a; k += x) {
                const uint32_t t = s.a + k;
                const bool ends = t + 1 == m.live || m.key(t + 1) != m.key(t);
                s_src[k] = p.grad.offset(static_cast<uint32_t>(m.tok[t])) | (ends ? kEnds : 0ull);
            }
            for (uint32_t k = tx; k < s.u1 - s.u0; k += x) {
                const uint32_t key = m.seg_key(s.u0 + k);
                s_dst[k] = p.dense ? p.out.offset(key) : key % p.vocab;
                if (p.rows_out && tile == 0) p.rows_out[s.u0 + k] = key % p.vocab;
            }
        }
        __syncthreads();
        if (c < p.dim) sum_chunk<A, B, N, 1, 8>(p, s_src, s_dst, s.b - s.a, s.lead ? s.u0 - 1 : s.u0, s.u0, chunk, c, x * N);
        __syncthreads();
        if (!m.any_long) continue;
        finish_long<B, N, 1>(p, pieces_of(s, chunk, kSmallShift, m.seg_begin), chunk, tile, c, 0, tx == 0 && ty < y,
                             [&](uint32_t u) { return m.seg_key(u); }, &m.last[ty < y ? ty : kSmallLanes]);
        __syncthreads();
    }
    if (p.zero_rows) clear_small(p, m);
}

// ---------------------------------------------------------------------------------------------- host

// Tokens per chunk: long enough to keep the pieces of long segments rare, short enough that all SMs have work.  With kChunkBits 21,
// 22 and 23 an update of 32768 tokens x 1024 took 73, 64 and 67 us when this was set; later versions differ by 3 %.
constexpr uint32_t kMinShift = 3, kMaxShift = 6;
constexpr uint32_t kChunkBits = 22;
uint32_t chunk_shift_of(uint64_t n, uint32_t dim) {
    uint32_t shift = kMinShift;
    while (shift < kMaxShift && (n * dim >> (kChunkBits + shift)) > 0) ++shift;
    return shift;
}

// Chunks of the largest call: calls of fewer tokens may have shorter, and so more, chunks.
uint64_t max_chunks(uint64_t max_tokens, uint32_t dim) {
    uint64_t most = max_tokens < kSmallTokens ? (max_tokens >> kSmallShift) + 1 : kSmallChunks;
    for (uint32_t shift = kMinShift; shift <= kMaxShift; ++shift) {
        uint64_t n = shift < kMaxShift ? ((1ull << (kChunkBits + shift)) - 1) / dim : max_tokens;  // the most tokens with such chunks
        if (n > max_tokens) n = max_tokens;
        if (chunk_shift_of(n, dim) == shift && (n >> shift) + 1 > most) most = (n >> shift) + 1;
    }
    return most;
}

size_t ticket_count(uint64_t chunks, uint32_t dim) {
    uint32_t levels = 1;
    while ((chunks >> (kFanBits * levels)) > 0) ++levels;
    return static_cast<size_t>(levels) * chunks * 2 * ((dim + 511) / 512);
}

size_t carve(adacomp_embed_t* h, void* ws, uint32_t max_tokens, uint32_t dim) {
    Carver c(ws);
    const size_t n = max_tokens ? max_tokens : 1, chunks = max_chunks(n, dim);
    adacomp_embed_t e = {};
    e.d_status = c.take<int>(1);
    e.d_n_segs = c.take<uint32_t>(2);
    e.d_barrier = c.take<uint32_t>(3);
    for (int i = 0; i < 2; ++i) e.d_tok[i] = c.take<uint64_t>(n);
    e.d_table = c.take<uint32_t>(static_cast<size_t>(kSortBlocks) * kMaxBins);
    e.d_seg_begin = c.take<uint32_t>(n + 1);
    e.d_seg_key = c.take<uint32_t>(n);
    e.d_chunk_seg = c.take<uint32_t>(chunks + 1);
    e.d_order = c.take<uint32_t>(n);
    e.d_tickets = c.take<uint32_t>(ticket_count(chunks, dim));
    e.d_partial = c.take<float>(chunks * 2 * dim);
    if (h) {
        h->d_status = e.d_status;
        h->d_n_segs = e.d_n_segs;
        h->d_barrier = e.d_barrier;
        for (int i = 0; i < 2; ++i) h->d_tok[i] = e.d_tok[i];
        h->d_table = e.d_table;
        h->d_seg_begin = e.d_seg_begin;
        h->d_seg_key = e.d_seg_key;
        h->d_chunk_seg = e.d_chunk_seg;
        h->d_order = e.d_order;
        h->d_tickets = e.d_tickets;
        h->chunks = static_cast<uint32_t>(chunks);
        h->d_partial = e.d_partial;
    }
    return c.used;
}

int check_limits(uint32_t vocab, uint32_t dim, uint32_t max_tokens, uint32_t max_workers) {
    if (vocab == 0 || dim == 0 || max_workers == 0 || max_tokens >= (1u << 31) || dim >= (1u << 31)) return ADACOMP_ERR_INVALID;
    if (static_cast<uint64_t>(vocab) * max_workers > 0xFFFFFFFEull) return ADACOMP_ERR_INVALID;
    return ADACOMP_OK;
}

// Threads of a block along a row of `cols` threads' worth of work (at most `most`), rows of a block, and blocks along the row.
void along_row(uint32_t cols, uint32_t most, uint32_t* x, uint32_t* y, uint32_t* tiles) {
    if (cols <= 16) {
        *x = 1;
        while (*x < cols) *x *= 2;
        *tiles = 1;
    } else {
        *tiles = (cols + most - 1) / most;
        *x = ((cols + *tiles - 1) / *tiles + 31) / 32 * 32;
    }
    *y = *x >= 256 ? 1 : 256 / *x;
}

template <typename A, typename B, int N, int K>
int launch_lookup_vec(const Rows& table, const Rows& tokens, const Rows& out, uint32_t n_tokens, const adacomp_embed_t* h, float scale,
                      cudaStream_t stream) {
    uint32_t x, y, tiles;
    const uint32_t cols = (h->dim + N * K - 1) / (N * K);
    along_row(cols, 512, &x, &y, &tiles);
    const dim3 block(x, y);
    const int wide = on_grid(out, 32);
    // An output that L2 cannot hold is written past it: 32768 x 2048 bf16, 134 MB, 41.4 -> 36.4 us (a plain copy of as much: 44).
    const int passing = static_cast<uint64_t>(n_tokens) * h->dim * sizeof(B) > (96ull << 20);
    // four tokens per thread once that still leaves every SM two thousand threads
    if (static_cast<uint64_t>(n_tokens) * cols >= 4ull * 2048 * h->n_sms) {
        const uint64_t grid = (static_cast<uint64_t>(n_tokens) + 4 * y - 1) / (4 * y) * tiles;
        if (grid > 0x7FFFFFFFull) return ADACOMP_ERR_INVALID;
        k_embed_lookup<A, B, N, K, 4><<<static_cast<uint32_t>(grid), block, 0, stream>>>(table, tokens, out, n_tokens, h->vocab, h->dim, tiles,
                                                                                         wide, passing, scale, h->d_status);
    } else {
        const uint32_t grid = (n_tokens + y - 1) / y * tiles;
        k_embed_lookup<A, B, N, K, 1><<<grid, block, 0, stream>>>(table, tokens, out, n_tokens, h->vocab, h->dim, tiles, wide, passing, scale,
                                                                  h->d_status);
    }
    ADACOMP_LAUNCH_CHECK();
    return ADACOMP_OK;
}

template <typename A, typename B>
int launch_lookup(const Rows& table, const Rows& tokens, const Rows& out, uint32_t n_tokens, const adacomp_embed_t* h,
                  float scale, cudaStream_t stream) {
    constexpr int N = kItemElems<A, B>;
    if (h->dim % N == 0 && on_grid(table, 16) && on_grid(out, 16))
        return launch_lookup_vec<A, B, N, 1>(table, tokens, out, n_tokens, h, scale, stream);
    // Off the grid: single entries, or for long rows of 16-bit entries items of eight.  32768 bf16 rows one way and the other: of
    // 250 entries 15.4 and 17.2 us, of 1001 52 and 37; fp32 rows of 1001 take 49 one entry at a time, of 1024 on the grid 43.
    if ((sizeof(A) == 4 && sizeof(B) == 4) || h->dim < 512)
        return launch_lookup_vec<A, B, 1, 4>(table, tokens, out, n_tokens, h, scale, stream);
    uint32_t x, y, tiles;
    const uint64_t cols = (static_cast<uint64_t>(h->dim) + 7 + 7) / 8;      // wherever a row starts
    along_row(static_cast<uint32_t>(cols), 512, &x, &y, &tiles);
    const uint64_t total = static_cast<uint64_t>(h->vocab - 1) * table.row_stride + h->dim;
    const dim3 block(x, y);
    if (n_tokens * cols >= 2ull * 2048 * h->n_sms) {
        const uint32_t grid = static_cast<uint32_t>((static_cast<uint64_t>(n_tokens) + 2 * y - 1) / (2 * y) * tiles);
        k_embed_lookup_off<A, B, 2><<<grid, block, 0, stream>>>(table, tokens, out, n_tokens, h->vocab, h->dim, tiles, total, scale,
                                                                h->d_status);
    } else {
        const uint32_t grid = (n_tokens + y - 1) / y * tiles;
        k_embed_lookup_off<A, B, 1><<<grid, block, 0, stream>>>(table, tokens, out, n_tokens, h->vocab, h->dim, tiles, total, scale,
                                                                h->d_status);
    }
    ADACOMP_LAUNCH_CHECK();
    return ADACOMP_OK;
}

// A launch whose blocks may line up while the kernel before it ends; they wait for it themselves.
template <typename... Args>
int launch_after(void (*kernel)(Args...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
    if (e != cudaSuccess) return cuda_fail(e);
    ADACOMP_LAUNCH_CHECK();
    return ADACOMP_OK;
}

// What the sort has to do, and what the sums read of it.
SortJob describe(const adacomp_embed_t* h, const Rows& tokens, uint32_t n_tokens, uint32_t n_workers, uint64_t* d_row_begin, float scale, Sums* p) {
    SortJob j = {};
    j.tokens = tokens;
    j.n = n_tokens * n_workers;
    j.n_tokens = n_tokens;
    j.n_workers = n_workers;
    j.vocab = h->vocab;
    j.padding = h->padding;
    j.none = n_workers * h->vocab;
    int bits = 0;
    while (bits < 32 && (j.none >> bits) != 0) ++bits;
    j.passes = (bits + kDigitBits - 1) / kDigitBits;
    j.bits = (bits + j.passes - 1) / j.passes;
    for (int i = 0; i < 2; ++i) j.tok[i] = h->d_tok[i];
    j.table = h->d_table;
    j.seg_begin = h->d_seg_begin;
    j.seg_key = h->d_seg_key;
    j.n_segs = h->d_n_segs;
    j.chunk_seg = h->d_chunk_seg;
    j.order = h->d_order;
    j.chunk_shift = chunk_shift_of(j.n, h->dim);
    j.row_begin = d_row_begin;
    j.barrier = h->d_barrier;
    j.wait_limit = h->wait_limit;
    j.status = h->d_status;
    p->order = j.order;
    p->seg_begin = j.seg_begin;
    p->seg_key = j.seg_key;
    p->chunk_seg = j.chunk_seg;
    p->n_segs = j.n_segs;
    p->chunk_shift = j.chunk_shift;
    p->n_chunks = static_cast<uint32_t>((static_cast<uint64_t>(j.n) + (1u << j.chunk_shift) - 1) >> j.chunk_shift);
    p->partial = h->d_partial;
    p->gave_up = h->d_barrier + 2;
    p->row_begin = d_row_begin;
    p->n_workers = n_workers;
    p->dim = h->dim;
    p->vocab = h->vocab;
    p->tickets = h->d_tickets;
    p->max_chunks = h->chunks;
    p->scale = scale;
    return j;
}

// Sorts the call's tokens and finds the segments.  zero: rows to clear on the side, or null.
int sort_tokens(const adacomp_embed_t* h, SortJob j, const Rows* zero, uint64_t zero_rows, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kSortThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t e;
    if (j.n <= h->cluster * kClusterStep) {
        // as many blocks as have a token per thread, then more tokens per thread
        uint32_t blocks = 1;
        while (blocks < h->cluster && blocks * kSortThreads < j.n) blocks *= 2;
        j.share_shift = 10;
        while ((blocks << j.share_shift) < j.n) ++j.share_shift;
        cfg.gridDim = dim3(blocks);
        cfg.dynamicSmemBytes = (2u << j.share_shift) * 4 + (blocks << j.bits) * 2 + (kSortWarps << j.bits) * 2;
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = blocks;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        e = cudaLaunchKernelEx(&cfg, k_embed_sort_cluster, j);
    } else {
        j.n_blocks = (j.n + 2047) / 2048;
        if (j.n_blocks > kSortBlocks) j.n_blocks = kSortBlocks;
        const uint32_t unit = (j.n + j.n_blocks - 1) / j.n_blocks > kStep ? kStep : kSortThreads;
        j.per_block = ((j.n + j.n_blocks - 1) / j.n_blocks + unit - 1) / unit * unit;
        cfg.gridDim = dim3(j.n_blocks);
        attr[0].id = cudaLaunchAttributeCooperative;
        attr[0].val.cooperative = 1;
        e = cudaLaunchKernelEx(&cfg, k_embed_sort, j);
    }
    if (e != cudaSuccess) return cuda_fail(e);
    ADACOMP_LAUNCH_CHECK();
    if (zero) {
        const int vec = on_grid(*zero, 16) && static_cast<uint64_t>(h->dim) * type_size(zero->type) % 16 == 0;
        const uint32_t most = 8 * static_cast<uint32_t>(h->n_sms);
        const int rc = launch_after(k_embed_clear, dim3(zero_rows < most ? static_cast<uint32_t>(zero_rows) : most), dim3(kThreads), 0, stream,
                                    *zero, zero_rows, h->dim, vec);
        if (rc != ADACOMP_OK) return rc;
    }
    return ADACOMP_OK;
}

constexpr uint64_t kSortMicros = 16, kTokensPerMicro = 8192, kClearPerMicro = 5 << 20;     // what sorting takes, and clearing meanwhile

template <typename A, typename B>
int launch_sums(const SortJob& j, Sums p, uint32_t out_grid, bool clear, const adacomp_embed_t* h, cudaStream_t stream) {
    constexpr int N = kItemElems<A, B>;
    const bool vec = p.dim % N == 0 && on_grid(p.grad, 16) && out_grid >= 16;
    p.wide = out_grid >= 32;
    constexpr int K = sizeof(A) == 4 ? 4 : 8;               // columns per thread off the grid, where there is work enough
    const uint32_t size = type_size(p.out.type);
    uint32_t x, y;
    along_row((p.dim + (vec ? N : 1) - 1) / (vec ? N : 1), 512, &x, &y, &p.tiles);
    y = kSmallThreads / x < kSmallLanes ? kSmallThreads / x : kSmallLanes;
    // One launch as long as its blocks run at once: with more of them every SM sorts more than once (2048 tokens: 15 us for the
    // call at 1024 columns, where two launches take 19, but 25 at 4096, where they take 21).
    const uint64_t small_blocks = static_cast<uint64_t>((j.n + kSmallChunk * y - 1) / (kSmallChunk * y)) * p.tiles;
    const bool small = j.n <= kSmallTokens / 2 || (j.n <= kSmallTokens && small_blocks <= static_cast<uint64_t>(h->n_sms));
    p.zero_vec = clear && on_grid(p.out, 16) && static_cast<uint64_t>(p.dim) * size % 16 == 0;
    if (!clear) p.zero_rows = 0;
    if (small) {
        p.chunk_shift = kSmallShift;
        p.n_chunks = (j.n + kSmallChunk - 1) / kSmallChunk;
        uint64_t blocks = small_blocks;
        const uint64_t most = 2 * static_cast<uint64_t>(h->n_sms);
        if (clear && blocks < p.zero_rows * p.dim * size / 32768) blocks = p.zero_rows * p.dim * size / 32768;     // 32 KB each
        if (blocks < 1) blocks = 1;
        if (blocks > most) blocks = most;
        if (vec) k_embed_small<A, B, N><<<static_cast<uint32_t>(blocks), kSmallThreads, 0, stream>>>(j, p, x, y);
        else k_embed_small<A, B, 1><<<static_cast<uint32_t>(blocks), kSmallThreads, 0, stream>>>(j, p, x, y);
        ADACOMP_LAUNCH_CHECK();
        return ADACOMP_OK;
    }
    // Rows without a token become zeros.  Where most have none, as many rows are cleared while the tokens are sorted as the
    // other SMs manage in that time (the sums write some of them once more); the others next to the sums, as they need it.
    p.zero_first = 0;
    if (clear && j.n <= p.zero_rows / 4) {
        const uint64_t row = static_cast<uint64_t>(p.dim) * size, in_time = (kSortMicros + j.n / kTokensPerMicro) * kClearPerMicro / row;
        if (in_time < p.zero_rows / 2) p.zero_first = in_time;      // for less the launch is not worth it
    }
    int rc = sort_tokens(h, j, p.zero_first ? &p.out : nullptr, p.zero_first, stream);
    if (rc != ADACOMP_OK) return rc;
    const uint32_t chunk_bytes = (3u << p.chunk_shift) * sizeof(uint64_t);
    const uint32_t per_thread = vec ? N : K;
    along_row((p.dim + per_thread - 1) / per_thread, kSumThreads, &x, &y, &p.tiles);
    while (y > 1 && y * chunk_bytes > 32 * 1024) y /= 2;
    while (x * y < 32) x *= 2;                              // narrow rows, long chunks: a whole warp, some of it without columns
    p.sum_blocks = (p.n_chunks + y - 1) / y * p.tiles;
    uint32_t zero_blocks = 0;
    if (clear && p.zero_first < p.zero_rows) {
        // some 64 KB per block: with 512 KB the last blocks run alone (131072 x 1024 fp32, 16384 tokens: 110 -> 129 us)
        const uint64_t left = p.zero_rows - p.zero_first, blocks = left * p.dim * size / 65536 + 1;
        zero_blocks = static_cast<uint32_t>(left < blocks ? left : blocks);
    }
    const dim3 block(x, y);
    return launch_after(vec ? k_embed_sums<A, B, N, 1> : k_embed_sums<A, B, 1, K>, dim3(p.sum_blocks + zero_blocks), block, y * chunk_bytes,
                        stream, p);
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

// The largest cluster that fits the device, with the shared memory that the sort's blocks may need.
cudaError_t prepare_cluster(uint32_t* blocks_out) {
    cudaError_t e = cudaFuncSetAttribute(k_embed_sort_cluster, cudaFuncAttributeMaxDynamicSharedMemorySize, kClusterSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_embed_sort_cluster, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    for (uint32_t blocks = 16; e == cudaSuccess; blocks /= 2) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(blocks);
        cfg.blockDim = dim3(kSortThreads);
        cfg.dynamicSmemBytes = kClusterSmem;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = blocks;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        int n = 0;
        e = cudaOccupancyMaxActiveClusters(&n, k_embed_sort_cluster, &cfg);
        *blocks_out = blocks;
        if (n > 0 || blocks == 1) break;
    }
    return e;
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
    *bytes_out = carve(nullptr, nullptr, max_tokens, dim);
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
    e->wait_limit = kWaitLimit;
    carve(e, d_workspace, max_tokens, dim);
    DeviceGuard guard(device);
    cudaError_t err = guard.err;
    if (err == cudaSuccess) err = cudaDeviceGetAttribute(&e->n_sms, cudaDevAttrMultiProcessorCount, device);
    if (err == cudaSuccess) err = prepare_cluster(&e->cluster);
    if (err == cudaSuccess) err = cudaMemset(e->d_status, 0, sizeof(int));
    if (err == cudaSuccess) err = cudaMemset(e->d_barrier, 0, 3 * sizeof(uint32_t));
    if (err == cudaSuccess) err = cudaMemset(e->d_tickets, 0, ticket_count(e->chunks, dim) * sizeof(uint32_t));
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
    if (!aligned(d_values_out, type_size(values_type)) || !aligned(d_rows_out, sizeof(uint32_t)) || !aligned(d_idx_out, sizeof(uint32_t)) ||
        !aligned(d_row_begin_out, sizeof(uint64_t)))
        return ADACOMP_ERR_INVALID;
    if (d_idx_out && (idx_offset >= (1ull << 32) || idx_offset + static_cast<uint64_t>(h->vocab) * h->dim > (1ull << 32)))
        return ADACOMP_ERR_INVALID;
    Rows k;
    Sums p = {};
    rc = rows_view(tokens, n, true, &k);
    if (rc == ADACOMP_OK) rc = rows_view(grad, n, false, &p.grad);
    if (rc != ADACOMP_OK) return rc;
    DeviceGuard guard(h->device);
    ADACOMP_CUDA(guard.err);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const SortJob j = describe(h, k, n_tokens, n_workers, d_row_begin_out, scale, &p);
    p.rows_out = d_rows_out;
    p.values = static_cast<char*>(d_values_out);
    p.idx_out = d_idx_out;
    p.idx_offset = static_cast<uint32_t>(idx_offset);
    uint64_t grid = reinterpret_cast<uintptr_t>(d_values_out) | static_cast<uint64_t>(h->dim) * type_size(values_type);
    if (d_idx_out) grid |= reinterpret_cast<uintptr_t>(d_idx_out) | static_cast<uint64_t>(h->dim) * 4;
    const uint32_t out_grid = grid % 32 == 0 ? 32 : grid % 16 == 0 ? 16 : 1;
    return ADACOMP_BY_TYPE(launch_sums, p.grad.type, values_type, j, p, out_grid, false, h, stream);
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
    const SortJob j = describe(h, k, n_tokens, n_workers, nullptr, scale, &p);
    p.dense = 1;
    p.accumulate = accumulate != 0;
    p.zero_rows = static_cast<uint64_t>(n_workers) * h->vocab;
    const uint32_t out_grid = on_grid(p.out, 32) ? 32 : on_grid(p.out, 16) ? 16 : 1;
    return ADACOMP_BY_TYPE(launch_sums, p.grad.type, p.out.type, j, p, out_grid, !accumulate, h, stream);
}

int adacomp_embed_set_wait_limit(adacomp_embed_t* h, uint32_t polls) {
    if (!h) return ADACOMP_ERR_INVALID;
    h->wait_limit = polls;
    return ADACOMP_OK;
}

int adacomp_embed_last_error(adacomp_embed_t* h, void* cuda_stream) {
    if (!h) return ADACOMP_ERR_INVALID;
    DeviceGuard guard(h->device);
    ADACOMP_CUDA(guard.err);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    int status = 0;
    uint32_t gave_up = 0;
    ADACOMP_CUDA(cudaMemcpyAsync(&status, h->d_status, sizeof(int), cudaMemcpyDeviceToHost, stream));
    ADACOMP_CUDA(cudaMemcpyAsync(&gave_up, h->d_barrier + 2, sizeof(uint32_t), cudaMemcpyDeviceToHost, stream));
    ADACOMP_CUDA(cudaMemsetAsync(h->d_status, 0, sizeof(int), stream));
    ADACOMP_CUDA(cudaStreamSynchronize(stream));
    if (gave_up) {                                                  // blocks that gave up left the barrier anywhere
        ADACOMP_CUDA(cudaMemsetAsync(h->d_barrier, 0, 3 * sizeof(uint32_t), stream));
        ADACOMP_CUDA(cudaStreamSynchronize(stream));
        return ADACOMP_ERR_TIMEOUT;
    }
    return status;
}

int adacomp_embed_destroy(adacomp_embed_t* h) {
    delete h;
    return ADACOMP_OK;
}

}  // extern "C"
