// Embedding tables: lookup with scaling, and the gradient by sorted tokens.
//
//   lookup    out_t = round(s E[token_t])
//   gradient  dE[w][v] = s sum of the gradient rows of worker w's tokens that equal v
//
// The gradient sorts the pairs (worker * vocab + token, position), stable, so a row's summands stand together and in
// order; every row is then summed by whoever owns it, without atomics.  All of it is bound by HBM (one fp32 addition per
// entry read).
#include <cooperative_groups.h>
#include <math.h>
#include <new>

#include "numeric.cuh"

using namespace adacomp;

struct adacomp_embed {
    int device;
    uint32_t vocab, dim, max_tokens, max_workers, padding;
    int n_sms;
    int* d_status;
    uint32_t* d_barrier;            // arrivals, and blocks that are through
    uint32_t* d_key[2];             // [max_tokens] worker * vocab + token, between the passes of the sort
    uint32_t* d_pos[2];             // [max_tokens] which token it is
    uint32_t* d_table;              // [kSortBlocks][kMaxBins] digit counts per block
    uint32_t* d_seg_begin;          // [max_tokens + 1] first sorted token of every distinct one, and their end
    uint32_t* d_seg_key;            // [max_tokens]
    uint32_t* d_chunk_seg;          // [chunks + 1] how many segments begin before the chunk
    uint32_t* d_n_segs;             // [2] distinct tokens, and how many tokens of the sorted list have a gradient
    uint32_t* d_n_long;             // [2] how many segments are longer than a chunk
    uint4* d_long;                  // [chunks] those
    uint32_t* d_order;              // [max_tokens] positions in the order of the sort
    uint32_t cluster;               // blocks of the largest cluster that the device takes
    uint32_t* d_tickets;            // [kSmallChunks][blocks along a row]
    float* d_partial;               // [chunks][2][dim] sums of pieces of those
};

namespace {

constexpr int kThreads = 256;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kItems = 8;                                   // tokens per thread and step of the sort
constexpr uint32_t kStep = kSortThreads * kItems;
constexpr uint32_t kSortBlocks = 64;
constexpr int kDigitBits = 9;
constexpr int kMaxBins = 1 << kDigitBits;
constexpr uint32_t kClusterSmem = 2 * kStep * 4 + 16 * kMaxBins * 4 + kSortWarps * kMaxBins * 2;
constexpr uint32_t kSpinLimit = 1u << 22;                   // polls of a barrier, some seconds

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

// Threads of a block: x along a row (in `tiles` blocks), y over rows; a thread copies the same columns of R tokens, all of them
// on their way before the first is stored.
template <typename A, typename B, int N, int R>
__global__ void __launch_bounds__(512) k_embed_lookup(Rows table, Rows tokens, Rows out, uint32_t n_tokens, uint32_t vocab, uint32_t dim,
                                                       uint32_t tiles, int wide, float scale, int* status) {
    const uint32_t t0 = blockIdx.x / tiles * (blockDim.y * R) + threadIdx.y, tile = blockIdx.x % tiles;
    const uint32_t c = (tile * blockDim.x + threadIdx.x) * N;
    uint32_t v[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t t = t0 + r * blockDim.y;
        v[r] = t < n_tokens ? load_token(tokens, t, vocab) : 0xFFFFFFFFu;
    }
    Packed<A, N> row[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (v[r] != 0xFFFFFFFFu && c < dim) row[r].load(reinterpret_cast<const A*>(table.data) + v[r] * table.row_stride + c);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t t = t0 + r * blockDim.y;
        if (t >= n_tokens || c >= dim) continue;
        float f[N];
        if (v[r] != 0xFFFFFFFFu) {
            row[r].unpack(f);
#pragma unroll
            for (int k = 0; k < N; ++k) f[k] = __fmul_rn(f[k], scale);
        } else {
            if (c == 0) record_error(status, ADACOMP_ERR_INVALID);
#pragma unroll
            for (int k = 0; k < N; ++k) f[k] = 0.f;
        }
        Packed<B, N> q;
        q.pack(f);
        B* dst = reinterpret_cast<B*>(out.data) + out.offset(t) + c;
        if (Packed<B, N>::kVecs == 2 && wide) store32(dst, q.v[0], q.v[Packed<B, N>::kVecs - 1]);
        else q.store(dst);
    }
}

// ---------------------------------------------------------------------------------------------- sort

struct SortJob {
    Rows tokens;
    uint32_t n, n_tokens, n_workers, vocab, padding, none;  // none = n_workers * vocab: the key of tokens without a gradient
    uint32_t n_blocks, per_block;                           // blocks that sort, tokens of each (a multiple of kSortThreads)
    int passes, bits;
    uint32_t* key[2];
    uint32_t* pos[2];
    uint32_t* table;
    uint32_t *order;                                        // the sorted tokens' positions, kLast set where a segment ends
    uint32_t *seg_begin, *seg_key, *n_segs, *chunk_seg, *n_long;
    uint32_t chunk_shift;
    uint32_t share_shift;                                   // cluster form: log2 of the tokens of a block
    uint64_t* row_begin;                                    // or null
    uint32_t* barrier;
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
// does not, the block says so and the caller gives up.
__device__ __forceinline__ bool meet(const SortJob& j) {
    __shared__ int s_ok;
    if (j.n_blocks == 1) {
        __syncthreads();
        return true;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        const uint32_t target = (atomicAdd(j.barrier, 1u) / j.n_blocks + 1) * j.n_blocks;
        uint32_t seen = 0, polls = 0;
        do {
            asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(j.barrier) : "memory");
        } while (seen < target && ++polls < kSpinLimit);
        s_ok = seen >= target;
        if (seen < target) record_error(j.status, ADACOMP_ERR_TIMEOUT);
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

__device__ __forceinline__ void zero_row(const Rows& out, uint64_t row, uint32_t dim, bool vec, uint32_t tid, uint32_t n_threads) {
    const uint32_t size = type_size(out.type);
    char* dst = out.data + out.offset(static_cast<uint32_t>(row)) * size;
    if (vec) {
        for (uint32_t c = tid; c < dim * size / 16; c += n_threads) reinterpret_cast<uint4*>(dst)[c] = make_uint4(0u, 0u, 0u, 0u);
    } else if (size == 4) {
        for (uint32_t c = tid; c < dim; c += n_threads) reinterpret_cast<uint32_t*>(dst)[c] = 0u;
    } else {
        for (uint32_t c = tid; c < dim; c += n_threads) reinterpret_cast<uint16_t*>(dst)[c] = 0;
    }
}

// Clears a table while the tokens are being sorted on other SMs.  It needs nothing of the sort, but the sums wait for this
// kernel alone, so it ends after the sort.
__global__ void __launch_bounds__(kThreads) k_embed_clear(Rows out, uint64_t n_rows, uint32_t dim, int vec) {
    for (uint64_t r = blockIdx.x; r < n_rows; r += gridDim.x) zero_row(out, r, dim, vec != 0, threadIdx.x, kThreads);
    cudaGridDependencySynchronize();
}

// Lanes of the warp that hold the same digit (of at most kDigitBits bits), among the real ones or among the others.
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

// Sorted token i with key k between `last` and `next`, and its place in the lists that the sums read; `u` segments begin
// before it.
__device__ __forceinline__ void put_segment(const SortJob& j, uint64_t i, uint32_t k, uint32_t last, uint32_t next, uint32_t pos, bool head, uint32_t u) {
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

// Block 0: the lists of a call without a token that has a gradient, and what the sums count up from zero.
__device__ __forceinline__ void put_empty(const SortJob& j, bool nothing) {
    if (threadIdx.x < 2) j.n_long[threadIdx.x] = 0;
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
    __shared__ uint32_t s_warp[32];
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint64_t from = static_cast<uint64_t>(blockIdx.x) * j.per_block;
    const uint64_t to = from + j.per_block < j.n ? from + j.per_block : j.n;
    const uint32_t bins = 1u << j.bits, mask = bins - 1;
    uint16_t* mine = s_count + warp * bins;
    const uint32_t items = j.per_block < kStep ? j.per_block / kSortThreads : kItems;     // rows of 32 per warp and step
    const bool one_step = j.per_block <= kStep;
    uint32_t key[kItems], pos[kItems], rank[kItems];
    for (int pass = 0; pass < j.passes; ++pass) {
        const uint32_t* key_in = j.key[(pass & 1) ^ 1];
        const uint32_t* pos_in = j.pos[(pass & 1) ^ 1];
        const int shift = pass * j.bits;
        // Loads step `at`, ranks it and leaves s_count as places within the step; returns the step's count of digit tid.
        auto rank_step = [&](uint64_t at, bool report) -> uint32_t {
            for (uint32_t d = lane; d < bins / 2; d += 32) reinterpret_cast<uint32_t*>(mine)[d] = 0;
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
                const uint64_t t = at + (warp * items + i) * 32 + lane;
                key[i] = j.none;
                pos[i] = 0;
                if (i >= items || t >= to) continue;
                if (pass == 0) {
                    key[i] = load_key(j, static_cast<uint32_t>(t), report);
                    pos[i] = static_cast<uint32_t>(t);
                } else {
                    key[i] = __ldcg(key_in + t);
                    pos[i] = __ldcg(pos_in + t);
                }
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
                if (i >= items) break;
                const bool real = at + (warp * items + i) * 32 + lane < to;
                const uint32_t d = (key[i] >> shift) & mask;
                const uint32_t same = same_digit(d, real);
                const uint32_t before = __popc(same & ((1u << lane) - 1));
                rank[i] = mine[d] + before;
                __syncwarp();
                if (real && before == 0) mine[d] += static_cast<uint16_t>(__popc(same));
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
        uint32_t all = count, before = 0;
        if (j.n_blocks > 1) {
            if (tid < bins) __stcg(j.table + blockIdx.x * bins + tid, count);
            if (!meet(j)) return;
            if (tid < bins) {
                all = 0;
#pragma unroll 8
                for (uint32_t b = 0; b < j.n_blocks; ++b) {
                    const uint32_t c = __ldcg(j.table + b * bins + tid);
                    all += c;
                    if (b < blockIdx.x) before += c;
                }
            }
        }
        uint32_t total;
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
                const uint32_t d = (key[i] >> shift) & mask;
                const uint32_t place = s_base[d] + mine[d] + rank[i];
                __stcg(j.key[pass & 1] + place, key[i]);
                __stcg(j.pos[pass & 1] + place, pos[i]);
            }
            if (!one_step) {
                __syncthreads();
                if (tid < bins) s_base[tid] += step_count;
            }
        }
        if (!meet(j)) return;
    }

    // Segments: where each begins, how many begin before every chunk, where each worker's begin.
    const uint32_t* sorted = j.key[(j.passes - 1) & 1];
    const uint32_t* sorted_pos = j.pos[(j.passes - 1) & 1];
    uint32_t segs = 0, total;
    if (j.n_blocks > 1) {
        for (uint64_t at = from; at < to; at += kSortThreads) {
            const uint64_t i = at + tid;
            bool head = false;
            if (i < to) {
                const uint32_t k = __ldcg(sorted + i);
                head = k != j.none && (i == 0 || __ldcg(sorted + i - 1) != k);
            }
            segs += __syncthreads_count(head);
        }
        if (tid == 0) __stcg(j.table + blockIdx.x, segs);
        if (!meet(j)) return;
        const uint32_t c = tid < j.n_blocks ? __ldcg(j.table + tid) : 0u;
        block_before(tid < blockIdx.x ? c : 0u, s_warp, &total);
        segs = total;
    }
    for (uint64_t at = from; at < to; at += kSortThreads) {
        const uint64_t i = at + tid;
        uint32_t k = j.none, last = j.none, next = j.none, pos_i = 0;
        if (i < to) {
            k = __ldcg(sorted + i);
            pos_i = __ldcg(sorted_pos + i);
            if (i > 0) last = __ldcg(sorted + i - 1);
            if (i + 1 < j.n) next = __ldcg(sorted + i + 1);
        }
        const bool head = k != j.none && (i == 0 || last != k);
        const uint32_t u = segs + block_before(head, s_warp, &total);
        segs += total;
        if (i < to) put_segment(j, i, k, last, next, pos_i, head, u);
    }
    if (blockIdx.x == 0) put_empty(j, j.n == 0 || __ldcg(sorted) == j.none);
    // the last block through leaves the barrier as it was
    if (j.n_blocks > 1 && tid == 0 && atomicAdd(j.barrier + 1, 1u) == j.n_blocks - 1) {
        j.barrier[0] = 0;
        j.barrier[1] = 0;
    }
}

// The same sort for up to kStep tokens per block in one thread-block cluster: the tokens stay in registers and shared memory, a block's counts and the tokens themselves go straight to the shared memory of the block they
// belong to, and the cluster's barrier takes the place of the one in global memory.
__global__ void __launch_bounds__(kSortThreads, 1) k_embed_sort_cluster(const SortJob j) {
    extern __shared__ uint64_t s_mem64[];
    __shared__ uint32_t s_base[kMaxBins];
    __shared__ uint32_t s_warp[32];
    cooperative_groups::cluster_group cluster = cooperative_groups::this_cluster();
    cudaTriggerProgrammaticLaunchCompletion();
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t n_ranks = gridDim.x, me = blockIdx.x;    // one cluster
    const uint32_t share = 1u << j.share_shift, items = share / kSortThreads;
    uint64_t* s_tok = s_mem64;                                                  // [share] key and position
    const uint32_t bins = 1u << j.bits, mask = bins - 1;
    uint32_t* s_all = reinterpret_cast<uint32_t*>(s_tok + share);               // [n_ranks][bins] the blocks' counts
    uint16_t* s_count = reinterpret_cast<uint16_t*>(s_all + n_ranks * bins);    // [kSortWarps][bins]
    uint16_t* mine = s_count + warp * bins;
    const uint32_t from = me << j.share_shift;
    const uint32_t n_here = j.n > from ? (j.n - from < share ? j.n - from : share) : 0;
    const uint32_t span = warp * items * 32 + lane;                             // the warp's tokens: rows of 32, one after the other
    uint64_t tok[kItems];
    uint32_t rank[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const uint32_t t = span + i * 32;
        tok[i] = static_cast<uint64_t>(j.none) << 32;
        if (i >= items || t >= n_here) continue;
        tok[i] = static_cast<uint64_t>(load_key(j, from + t, true)) << 32 | (from + t);
    }
    cluster.sync();                             // every block has started: its shared memory may be written from here on
    for (int pass = 0; pass < j.passes; ++pass) {
        const int shift = 32 + pass * j.bits;
        for (uint32_t d = lane; d < bins / 2; d += 32) reinterpret_cast<uint32_t*>(mine)[d] = 0;
        if (pass > 0) {
#pragma unroll
            for (int i = 0; i < kItems; ++i)
                if (i < items && span + i * 32 < n_here) tok[i] = s_tok[span + i * 32];
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
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
        uint32_t all = 0, before = 0, total;
        if (tid < bins) {
            all = counts_to_places(s_count, bins, tid);
            for (uint32_t r = 0; r < n_ranks; ++r) cluster.map_shared_rank(s_all, r)[me * bins + tid] = all;
        }
        cluster.sync();                         // the counts have arrived, and every block has its tokens in registers
        if (tid < bins) {
            all = 0;
            for (uint32_t r = 0; r < n_ranks; ++r) {
                const uint32_t c = s_all[r * bins + tid];
                all += c;
                if (r < me) before += c;
            }
        }
        const uint32_t base = block_before(all, s_warp, &total) + before;
        if (tid < bins) s_base[tid] = base;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
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
    uint32_t heads[kItems], in_warp = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
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
    for (uint32_t r = 0; r < me; ++r) u += s_all[r];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
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
    cluster.sync();                             // nobody leaves while a neighbour may still read here
}

// ---------------------------------------------------------------------------------------------- sums

struct Sums {
    const uint32_t *order, *seg_begin, *seg_key, *chunk_seg, *n_segs;
    uint32_t n, n_chunks, chunk_shift;
    uint32_t tiles;                 // blocks along a row
    uint32_t sum_blocks;            // the blocks behind them write zeros
    uint32_t* n_long;               // [2] segments of a few pieces, and of many
    uint4* long_list;               // first chunk, segment, pieces
    float* partial;
    uint32_t* tickets;              // [kSmallChunks][tiles], all zero between calls
    const int* status;
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
    uint64_t zero_rows;             // rows to look at for zeros, zero_run of them per block
    uint32_t zero_run;
    int zero_vec;
    int wide;                       // rows of the results start on 32-byte boundaries
};

constexpr uint32_t kMaxChunk = 64;
constexpr uint32_t kFewPieces = 16;             // a warp adds them alone
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

// Rows without a token, a run of them per block: which of them have one is looked up in the sorted list.
__device__ void zero_gaps(const Sums& p, uint32_t block) {
    __shared__ uint32_t s_has[kMaxChunk / 32];
    const uint32_t n_segs = *p.n_segs;
    const uint64_t from = static_cast<uint64_t>(block) * p.zero_run;
    const uint64_t to = from + p.zero_run < p.zero_rows ? from + p.zero_run : p.zero_rows;
    const uint32_t tid = threadIdx.y * blockDim.x + threadIdx.x, n_threads = blockDim.x * blockDim.y;
    if (tid < kMaxChunk / 32) s_has[tid] = 0;
    uint32_t lo = 0, hi = n_segs;               // first segment whose key is not below `from`
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (p.seg_key[mid] < from) lo = mid + 1; else hi = mid;
    }
    __syncthreads();
    for (uint32_t k = tid; k < p.zero_run && lo + k < n_segs; k += n_threads) {
        const uint64_t r = p.seg_key[lo + k];
        if (r < to) atomicOr(&s_has[(r - from) / 32], 1u << ((r - from) & 31));
    }
    __syncthreads();
    for (uint64_t r = from; r < to; ++r)
        if (!(s_has[(r - from) / 32] >> ((r - from) & 31) & 1)) zero_row(p.out, r, p.dim, p.zero_vec != 0, tid, n_threads);
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
// results go.  `slot` is the first token's segment, u0 the first one that begins in the chunk.
template <typename A, typename B, int N, int BATCH>
__device__ __forceinline__ void sum_chunk(const Sums& p, const uint64_t* s_src, const uint64_t* s_dst, uint32_t len, uint32_t slot, uint32_t u0,
                                          uint32_t chunk, uint32_t c) {
    float sum[N];
#pragma unroll
    for (int k = 0; k < N; ++k) sum[k] = 0.f;
    const A* grad = reinterpret_cast<const A*>(p.grad.data) + c;
    bool open = false;
    constexpr int kBatch = N * sizeof(A) == 32 ? BATCH / 2 : BATCH;         // rows in flight
    for (uint32_t i = 0; i < len; i += kBatch) {
        Packed<A, N> v[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (i + k < len) v[k].load(grad + (s_src[i + k] & ~kEnds));
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (i + k >= len) break;
            float f[N];
            v[k].unpack(f);
#pragma unroll
            for (int q = 0; q < N; ++q) sum[q] = __fadd_rn(sum[q], f[q]);
            open = true;
            if (s_src[i + k] & kEnds) {
                if (slot + 1 == u0) {           // the last piece of a long segment
                    put_piece<N>(piece_at(p, chunk, 0, c), sum);
                } else {
                    const uint64_t at = s_dst[slot - u0];
                    put_row<B, N>(p, slot, at, static_cast<uint32_t>(at), c, sum);
                }
#pragma unroll
                for (int q = 0; q < N; ++q) sum[q] = 0.f;
                ++slot;
                open = false;
            }
        }
    }
    if (open) put_piece<N>(piece_at(p, chunk, slot + 1 == u0 ? 0 : 1, c), sum);     // a piece that goes on in the next chunk
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

// Sums over the sorted list, cut into chunks of 2^chunk_shift tokens.  A chunk owns the segments that begin in it, to their
// end even if that lies in the next chunk; a segment longer than a chunk is cut at the chunks' borders, its pieces are
// added up by k_embed_join.  So the work per chunk is bounded, short segments need no second pass and the tree of additions
// depends on the tokens alone.  A thread keeps N columns; x runs along the row, y over chunks.
template <typename A, typename B, int N>
#ifdef V_MR
__global__ void __maxnreg__(V_MR) k_embed_sums
#else
__global__ void __launch_bounds__(512) k_embed_sums
#endif
(const Sums p) {
    extern __shared__ uint64_t s_mem[];
    cudaGridDependencySynchronize();
    if (*p.status == ADACOMP_ERR_TIMEOUT) return;           // the sort gave up: its lists are not to be followed
    if (blockIdx.x >= p.sum_blocks) {
        zero_gaps(p, blockIdx.x - p.sum_blocks);
        return;
    }
    const uint32_t size = 1u << p.chunk_shift;
    uint64_t* s_src = s_mem + static_cast<size_t>(threadIdx.y) * (3 * size);    // [2 size] where the rows of the chunk's tokens start
    uint64_t* s_dst = s_src + 2 * size;                                         // [size] where its segments' rows start
    const uint32_t chunk = blockIdx.x / p.tiles * blockDim.y + threadIdx.y, tile = blockIdx.x % p.tiles;
    const uint32_t n_segs = p.n_segs[0], live = p.n_segs[1];
    const uint32_t c = (tile * blockDim.x + threadIdx.x) * N;
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
    if (s.trail && tile == 0 && threadIdx.x == 0) {        // for k_embed_join: short lists from the front, long ones from the back
        const uint32_t pieces = ((p.seg_begin[s.u1] - 1) >> p.chunk_shift) - chunk + 1;
        const bool many = pieces > kFewPieces;
        const uint32_t e = atomicAdd(p.n_long + many, 1u);
        p.long_list[many ? p.n_chunks - 1 - e : e] = make_uint4(chunk, s.u1 - 1, pieces, 0u);
    }
    __syncthreads();
    // Four rows in flight per thread.  Fetching the next four before the last are added costs the registers of a block per SM
    // and gains nothing (524288 tokens: 512 -> 529 us for the whole call).
    if (c < p.dim) sum_chunk<A, B, N, 4>(p, s_src, s_dst, s.b - s.a, s.lead ? s.u0 - 1 : s.u0, s.u0, chunk, c);
}

// The long segments: their pieces, in order.  32 N columns of a segment are one job; with few pieces a warp does it, with many
// the block's eight warps take every eighth piece each.  Four pieces are in flight either way.
constexpr int kJoinLanes = 8;
template <int N>
__device__ __forceinline__ void add_pieces(const Sums& p, uint32_t chunk, uint32_t pieces, uint32_t first, uint32_t step, uint32_t c, float (&sum)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) sum[k] = 0.f;
    if (c >= p.dim) return;
    for (uint32_t q0 = first; q0 < pieces; q0 += 4 * step) {
        float f[4][N];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint32_t q = q0 + r * step;
            const float* src = piece_at(p, chunk + q, q == 0 ? 1 : 0, c);
            if constexpr (N % 4 == 0) {
#pragma unroll
                for (int k = 0; k < N; k += 4) {
                    const float4 v = q < pieces ? __ldcg(reinterpret_cast<const float4*>(src + k)) : make_float4(0.f, 0.f, 0.f, 0.f);
                    f[r][k] = v.x; f[r][k + 1] = v.y; f[r][k + 2] = v.z; f[r][k + 3] = v.w;
                }
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k) f[r][k] = q < pieces ? __ldcg(src + k) : 0.f;
            }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (q0 + r * step < pieces)
#pragma unroll
                for (int k = 0; k < N; ++k) sum[k] = __fadd_rn(sum[k], f[r][k]);
    }
}

template <typename B, int N>
__global__ void __launch_bounds__(32 * kJoinLanes) k_embed_join(const Sums p) {
    __shared__ float s_sum[kJoinLanes][32 * N];
    cudaGridDependencySynchronize();
    if (*p.status == ADACOMP_ERR_TIMEOUT) return;
    const uint32_t few = p.n_long[0], many = p.n_long[1];
    const uint32_t tiles = (p.dim + 32 * N - 1) / (32 * N);
    float sum[N];
    for (uint64_t job = blockIdx.x; job < static_cast<uint64_t>(many) * tiles; job += gridDim.x) {
        const uint4 seg = p.long_list[p.n_chunks - 1 - job / tiles];
        const uint32_t c = (static_cast<uint32_t>(job % tiles) * 32 + threadIdx.x) * N, key = p.seg_key[seg.y];
        add_pieces<N>(p, seg.x, seg.z, threadIdx.y, kJoinLanes, c, sum);
#pragma unroll
        for (int k = 0; k < N; ++k) s_sum[threadIdx.y][threadIdx.x * N + k] = sum[k];
        __syncthreads();
        if (threadIdx.y == 0 && c < p.dim) {
            for (int y = 1; y < kJoinLanes; ++y)
#pragma unroll
                for (int k = 0; k < N; ++k) sum[k] = __fadd_rn(sum[k], s_sum[y][threadIdx.x * N + k]);
            put_row<B, N>(p, seg.y, p.dense ? p.out.offset(key) : 0, key % p.vocab, c, sum);
        }
        __syncthreads();
    }
    for (uint64_t job = static_cast<uint64_t>(blockIdx.x) * kJoinLanes + threadIdx.y; job < static_cast<uint64_t>(few) * tiles;
         job += static_cast<uint64_t>(gridDim.x) * kJoinLanes) {
        const uint4 seg = p.long_list[job / tiles];
        const uint32_t c = (static_cast<uint32_t>(job % tiles) * 32 + threadIdx.x) * N, key = p.seg_key[seg.y];
        add_pieces<N>(p, seg.x, seg.z, 0, 1, c, sum);
        if (c < p.dim) put_row<B, N>(p, seg.y, p.dense ? p.out.offset(key) : 0, key % p.vocab, c, sum);
    }
}

// ---------------------------------------------------------------------------------------------- few tokens

// Up to kSmallTokens tokens: one launch does everything.  Every block sorts all tokens for itself in shared memory, which
// takes less than a second kernel's start, and then sums its chunks; the block that delivers the last piece of a long segment
// adds the pieces up.
constexpr int kSmallThreads = 512, kSmallWarps = kSmallThreads / 32, kSmallItems = 2;
constexpr uint32_t kSmallTokens = kSmallThreads * kSmallItems;
constexpr uint32_t kSmallShift = 3, kSmallChunk = 1u << kSmallShift, kSmallChunks = kSmallTokens / kSmallChunk;
constexpr uint32_t kSmallLanes = 64;                        // chunks a block takes at a time, at most

struct SmallMem {
    uint64_t tok[kSmallTokens];                             // key and position
    union {
        uint16_t count[kSmallWarps * kMaxBins];
        uint64_t rows[kSmallLanes][3 * kSmallChunk];        // s_src and s_dst of sum_chunk
    };
    uint32_t base[kMaxBins];
    uint32_t warp[32];
    uint32_t seg_begin[kSmallTokens + 1], seg_key[kSmallTokens];
    uint32_t chunk_seg[kSmallChunks + 1];
    uint32_t n_segs, live, any_long;
    uint32_t done[2 * kSmallLanes];                         // whether a chunk's piece was the last one
};

__device__ __forceinline__ void sort_small(const SortJob& j, SmallMem& m) {
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t bins = 1u << j.bits, mask = bins - 1;
    const uint32_t items = j.n <= kSmallThreads ? 1 : kSmallItems;
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
            const uint32_t k = static_cast<uint32_t>(m.tok[t] >> 32);
            head = k != j.none && (t == 0 || static_cast<uint32_t>(m.tok[t - 1] >> 32) != k);
        }
        heads[i] = __ballot_sync(0xFFFFFFFFu, head);
        in_warp += __popc(heads[i]);
    }
    uint32_t u = __shfl_sync(0xFFFFFFFFu, block_before<kSmallWarps>(lane == 0 ? in_warp : 0u, m.warp, &total), 0);
#pragma unroll
    for (int i = 0; i < kSmallItems; ++i) {
        const uint32_t t = span + i * 32;
        if (i < items && t < j.n) {
            const uint32_t k = static_cast<uint32_t>(m.tok[t] >> 32);
            const uint32_t at = u + __popc(heads[i] & ((1u << lane) - 1));
            const bool head = heads[i] >> lane & 1;
            if (t % kSmallChunk == 0) m.chunk_seg[t / kSmallChunk] = at;
            if (head) {
                m.seg_begin[at] = t;
                m.seg_key[at] = k;
            }
            if (k != j.none) {
                if (t + kSmallChunk < j.n && static_cast<uint32_t>(m.tok[t + kSmallChunk] >> 32) == k) m.any_long = 1;
                if (t + 1 == j.n || static_cast<uint32_t>(m.tok[t + 1] >> 32) == j.none) {
                    m.n_segs = at + head;
                    m.live = t + 1;
                    m.seg_begin[at + head] = t + 1;
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
    const uint32_t size = type_size(p.out.type);
    const bool flat = p.out.row_stride == p.dim;
    uint32_t lo = 0, hi = m.n_segs;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (m.seg_key[mid] < from) lo = mid + 1; else hi = mid;
    }
    for (uint64_t r = from; r < to;) {
        uint64_t stop = lo < m.n_segs && m.seg_key[lo] < to ? m.seg_key[lo] : to;
        if (stop == r) {
            ++lo;
            ++r;
            continue;
        }
        if (!flat) stop = r + 1;
        else if (p.out.group && (r / p.out.group + 1) * p.out.group < stop) stop = (r / p.out.group + 1) * p.out.group;
        char* dst = p.out.data + p.out.offset(static_cast<uint32_t>(r)) * size;
        const uint64_t bytes = (stop - r) * p.dim * size;
        if (p.zero_vec) {
            for (uint64_t c = threadIdx.x * 16; c < bytes; c += kSmallThreads * 16) *reinterpret_cast<uint4*>(dst + c) = make_uint4(0u, 0u, 0u, 0u);
        } else if (size == 4) {
            for (uint64_t c = threadIdx.x * 4; c < bytes; c += kSmallThreads * 4) *reinterpret_cast<uint32_t*>(dst + c) = 0u;
        } else {
            for (uint64_t c = threadIdx.x * 2; c < bytes; c += kSmallThreads * 2) *reinterpret_cast<uint16_t*>(dst + c) = 0;
        }
        r = stop;
    }
}

template <typename A, typename B, int N>
__global__ void __launch_bounds__(kSmallThreads) k_embed_small(const SortJob j, const Sums p, uint32_t x, uint32_t y) {
    __shared__ SmallMem m;
    sort_small(j, m);
    if (blockIdx.x == 0 && j.row_begin && j.n_workers == 1) {
        if (threadIdx.x < 2) j.row_begin[threadIdx.x] = threadIdx.x ? m.n_segs : 0;
    } else if (blockIdx.x == 0 && j.row_begin) {
        for (uint32_t w = threadIdx.x; w <= j.n_workers; w += kSmallThreads) {
            uint32_t lo = 0, hi = m.n_segs;
            while (lo < hi) {
                const uint32_t mid = (lo + hi) / 2;
                if (m.seg_key[mid] < static_cast<uint64_t>(w) * j.vocab) lo = mid + 1; else hi = mid;
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
            s = share_of(i0, kSmallChunk, m.live, m.chunk_seg[chunk], i0 + kSmallChunk < m.live ? m.chunk_seg[chunk + 1] : m.n_segs, m.seg_begin);
            for (uint32_t k = tx; k < s.b - s.a; k += x) {
                const uint32_t t = s.a + k, key = static_cast<uint32_t>(m.tok[t] >> 32);
                const bool ends = t + 1 == m.live || static_cast<uint32_t>(m.tok[t + 1] >> 32) != key;
                s_src[k] = p.grad.offset(static_cast<uint32_t>(m.tok[t])) | (ends ? kEnds : 0ull);
            }
            for (uint32_t k = tx; k < s.u1 - s.u0; k += x) {
                const uint32_t key = m.seg_key[s.u0 + k];
                s_dst[k] = p.dense ? p.out.offset(key) : key % p.vocab;
                if (p.rows_out && tile == 0) p.rows_out[s.u0 + k] = key % p.vocab;
            }
        }
        __syncthreads();
        if (c < p.dim) sum_chunk<A, B, N, 8>(p, s_src, s_dst, s.b - s.a, s.lead ? s.u0 - 1 : s.u0, s.u0, chunk, c);
        __syncthreads();
        if (!m.any_long) continue;
        // whose piece was the last of its segment
        __threadfence();
        __syncthreads();
        if (threadIdx.x < 2 * kSmallLanes) m.done[threadIdx.x] = 0;
        __syncthreads();
        uint32_t head[2] = {0, chunk}, pieces[2] = {0, 0};
        if (s.lead) head[0] = m.seg_begin[s.u0 - 1] / kSmallChunk, pieces[0] = (m.seg_begin[s.u0] - 1) / kSmallChunk - head[0] + 1;
        if (s.trail) pieces[1] = (m.seg_begin[s.u1] - 1) / kSmallChunk - chunk + 1;
        if (tx == 0) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                if (pieces[q] == 0) continue;
                uint32_t* ticket = p.tickets + head[q] * p.tiles + tile;
                if (atomicAdd(ticket, 1u) == pieces[q] - 1) {
                    *ticket = 0;
                    m.done[2 * ty + q] = 1;
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if (pieces[q] == 0 || !m.done[2 * ty + q] || c >= p.dim) continue;
            __threadfence();
            const uint32_t u = q == 0 ? s.u0 - 1 : s.u1 - 1, key = m.seg_key[u];
            float sum[N];
            add_pieces<N>(p, head[q], pieces[q], 0, 1, c, sum);
            put_row<B, N>(p, u, p.dense ? p.out.offset(key) : 0, key % p.vocab, c, sum);
        }
        __syncthreads();
    }
    if (p.zero_rows) clear_small(p, m);
}

// ---------------------------------------------------------------------------------------------- host

// Tokens per chunk: long enough to keep the pieces of long segments rare, short enough that all SMs have work.
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

size_t ticket_count(uint32_t dim) { return static_cast<size_t>(kSmallChunks) * ((dim + 511) / 512); }

size_t carve(adacomp_embed_t* h, void* ws, uint32_t max_tokens, uint32_t dim) {
    Carver c(ws);
    const size_t n = max_tokens ? max_tokens : 1, chunks = max_chunks(n, dim);
    adacomp_embed_t e = {};
    e.d_status = c.take<int>(1);
    e.d_n_segs = c.take<uint32_t>(2);
    e.d_barrier = c.take<uint32_t>(2);
    for (int i = 0; i < 2; ++i) {
        e.d_key[i] = c.take<uint32_t>(n);
        e.d_pos[i] = c.take<uint32_t>(n);
    }
    e.d_table = c.take<uint32_t>(static_cast<size_t>(kSortBlocks) * kMaxBins);
    e.d_seg_begin = c.take<uint32_t>(n + 1);
    e.d_seg_key = c.take<uint32_t>(n);
    e.d_chunk_seg = c.take<uint32_t>(chunks + 1);
    e.d_n_long = c.take<uint32_t>(2);
    e.d_long = c.take<uint4>(chunks);
    e.d_order = c.take<uint32_t>(n);
    e.d_tickets = c.take<uint32_t>(ticket_count(dim));
    e.d_partial = c.take<float>(chunks * 2 * dim);
    if (h) {
        h->d_status = e.d_status;
        h->d_n_segs = e.d_n_segs;
        h->d_barrier = e.d_barrier;
        for (int i = 0; i < 2; ++i) {
            h->d_key[i] = e.d_key[i];
            h->d_pos[i] = e.d_pos[i];
        }
        h->d_table = e.d_table;
        h->d_seg_begin = e.d_seg_begin;
        h->d_seg_key = e.d_seg_key;
        h->d_chunk_seg = e.d_chunk_seg;
        h->d_n_long = e.d_n_long;
        h->d_long = e.d_long;
        h->d_order = e.d_order;
        h->d_tickets = e.d_tickets;
        h->d_partial = e.d_partial;
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

// Whether every row starts on a boundary of so many bytes.
bool on_grid(const Rows& r, uint32_t bytes) {
    const uint32_t size = type_size(r.type);
    return reinterpret_cast<uintptr_t>(r.data) % bytes == 0 && r.row_stride * size % bytes == 0 &&
           (r.group == 0 || r.group_stride * size % bytes == 0);
}

// Threads of a sum's block along a row of `cols` threads' worth of work, chunks of a block, and blocks along the row.
void along_row(uint32_t cols, uint32_t chunk_bytes, uint32_t* x, uint32_t* y, uint32_t* tiles) {
    if (cols <= 16) {
        *x = 1;
        while (*x < cols) *x *= 2;
        *tiles = 1;
    } else {
        *tiles = (cols + 511) / 512;
        *x = ((cols + *tiles - 1) / *tiles + 31) / 32 * 32;
    }
    *y = *x >= 256 ? 1 : 256 / *x;
    while (*y > 1 && *y * chunk_bytes > 32 * 1024) *y /= 2;
}

template <typename A, typename B, int N>
int launch_lookup_vec(const Rows& table, const Rows& tokens, const Rows& out, uint32_t n_tokens, const adacomp_embed_t* h, float scale,
                      cudaStream_t stream) {
    uint32_t x, y, tiles;
    const uint32_t cols = (h->dim + N - 1) / N;
    along_row(cols, 1, &x, &y, &tiles);
    const dim3 block(x, y);
    const int wide = on_grid(out, 32);
    // four tokens per thread once that still leaves every SM two thousand threads
    if (static_cast<uint64_t>(n_tokens) * cols >= 4ull * 2048 * h->n_sms) {
        const uint64_t grid = (static_cast<uint64_t>(n_tokens) + 4 * y - 1) / (4 * y) * tiles;
        if (grid > 0x7FFFFFFFull) return ADACOMP_ERR_INVALID;
        k_embed_lookup<A, B, N, 4><<<static_cast<uint32_t>(grid), block, 0, stream>>>(table, tokens, out, n_tokens, h->vocab, h->dim, tiles, wide, scale, h->d_status);
    } else {
        const uint32_t grid = (n_tokens + y - 1) / y * tiles;
        k_embed_lookup<A, B, N, 1><<<grid, block, 0, stream>>>(table, tokens, out, n_tokens, h->vocab, h->dim, tiles, wide, scale, h->d_status);
    }
    ADACOMP_LAUNCH_CHECK();
    return ADACOMP_OK;
}

template <typename A, typename B>
int launch_lookup(const Rows& table, const Rows& tokens, const Rows& out, uint32_t n_tokens, const adacomp_embed_t* h,
                  float scale, cudaStream_t stream) {
    constexpr int N = kItemElems<A, B>;
    if (h->dim % N == 0 && on_grid(table, 16) && on_grid(out, 16)) return launch_lookup_vec<A, B, N>(table, tokens, out, n_tokens, h, scale, stream);
    return launch_lookup_vec<A, B, 1>(table, tokens, out, n_tokens, h, scale, stream);
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
    for (int i = 0; i < 2; ++i) {
        j.key[i] = h->d_key[i];
        j.pos[i] = h->d_pos[i];
    }
    j.table = h->d_table;
    j.seg_begin = h->d_seg_begin;
    j.seg_key = h->d_seg_key;
    j.n_segs = h->d_n_segs;
    j.chunk_seg = h->d_chunk_seg;
    j.n_long = h->d_n_long;
    j.order = h->d_order;
    j.chunk_shift = chunk_shift_of(j.n, h->dim);
    j.row_begin = d_row_begin;
    j.barrier = h->d_barrier;
    j.status = h->d_status;
    p->order = j.order;
    p->seg_begin = j.seg_begin;
    p->seg_key = j.seg_key;
    p->chunk_seg = j.chunk_seg;
    p->n_segs = j.n_segs;
    p->n = j.n;
    p->chunk_shift = j.chunk_shift;
    p->n_chunks = static_cast<uint32_t>((static_cast<uint64_t>(j.n) + (1u << j.chunk_shift) - 1) >> j.chunk_shift);
    p->n_long = h->d_n_long;
    p->long_list = h->d_long;
    p->partial = h->d_partial;
    p->status = h->d_status;
    p->dim = h->dim;
    p->vocab = h->vocab;
    p->tickets = h->d_tickets;
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
    if (j.n <= h->cluster * kStep) {
        // as many blocks as have a token per thread, then more tokens per thread
        uint32_t blocks = 1;
        while (blocks < h->cluster && blocks * kSortThreads < j.n) blocks *= 2;
        j.share_shift = 10;
        while ((blocks << j.share_shift) < j.n) ++j.share_shift;
        cfg.gridDim = dim3(blocks);
        cfg.dynamicSmemBytes = (2u << j.share_shift) * 4 + (blocks << j.bits) * 4 + (kSortWarps << j.bits) * 2;
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

template <typename A, typename B>
int launch_sums(const SortJob& j, Sums p, uint32_t out_grid, bool clear, const adacomp_embed_t* h, cudaStream_t stream) {
    constexpr int N = kItemElems<A, B>;
    const bool vec = p.dim % N == 0 && on_grid(p.grad, 16) && out_grid >= 16;
    p.wide = out_grid >= 32;
    const uint32_t cols = (p.dim + (vec ? N : 1) - 1) / (vec ? N : 1), size = type_size(p.out.type);
    p.zero_vec = clear && on_grid(p.out, 16) && static_cast<uint64_t>(p.dim) * size % 16 == 0;
    if (!clear) p.zero_rows = 0;
    uint32_t x, y;
    if (j.n <= kSmallTokens) {
        along_row(cols, 1, &x, &y, &p.tiles);
        y = kSmallThreads / x < kSmallLanes ? kSmallThreads / x : kSmallLanes;
        p.chunk_shift = kSmallShift;
        p.n_chunks = (j.n + kSmallChunk - 1) / kSmallChunk;
        uint64_t blocks = static_cast<uint64_t>((p.n_chunks + y - 1) / y) * p.tiles;
        const uint64_t most = 2 * static_cast<uint64_t>(h->n_sms);
        if (blocks < 1) blocks = 1;
        if (blocks > most || (clear && p.zero_rows * p.dim >= most * 4096)) blocks = most;
        if (vec) k_embed_small<A, B, N><<<static_cast<uint32_t>(blocks), kSmallThreads, 0, stream>>>(j, p, x, y);
        else k_embed_small<A, B, 1><<<static_cast<uint32_t>(blocks), kSmallThreads, 0, stream>>>(j, p, x, y);
        ADACOMP_LAUNCH_CHECK();
        return ADACOMP_OK;
    }
    // Rows without a token become zeros.  Few tokens: everything is cleared while they are sorted, and some rows are written
    // twice; many: the rows that need it are cleared next to the sums.
    const bool early = clear && j.n <= p.zero_rows / 4, gaps = clear && !early;
    int rc = sort_tokens(h, j, early ? &p.out : nullptr, p.zero_rows, stream);
    if (rc != ADACOMP_OK) return rc;
    const uint32_t chunk_bytes = (3u << p.chunk_shift) * sizeof(uint64_t);
    along_row(cols, chunk_bytes, &x, &y, &p.tiles);
    p.sum_blocks = (p.n_chunks + y - 1) / y * p.tiles;
    uint32_t zero_blocks = 0;
    if (gaps) {
        p.zero_run = 1;
        while (p.zero_run < kMaxChunk && static_cast<uint64_t>(p.zero_run) * p.dim * size < 32768) p.zero_run *= 2;
        zero_blocks = static_cast<uint32_t>((p.zero_rows + p.zero_run - 1) / p.zero_run);
    }
    const dim3 block(x, y);
    rc = launch_after(vec ? k_embed_sums<A, B, N> : k_embed_sums<A, B, 1>, dim3(p.sum_blocks + zero_blocks), block, y * chunk_bytes, stream, p);
    if (rc != ADACOMP_OK || p.n_chunks < 2) return rc;              // one chunk: no segment is longer
    constexpr int kWide = 16 / sizeof(B);
    const bool join_vec = out_grid >= 16 && p.dim % kWide == 0;
    return launch_after(join_vec ? k_embed_join<B, kWide> : k_embed_join<B, 1>, dim3(4 * static_cast<uint32_t>(h->n_sms)), dim3(32, kJoinLanes), 0, stream, p);
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
    carve(e, d_workspace, max_tokens, dim);
    DeviceGuard guard(device);
    cudaError_t err = guard.err;
    if (err == cudaSuccess) err = cudaDeviceGetAttribute(&e->n_sms, cudaDevAttrMultiProcessorCount, device);
    if (err == cudaSuccess) err = prepare_cluster(&e->cluster);
    if (err == cudaSuccess) err = cudaMemset(e->d_status, 0, sizeof(int));
    if (err == cudaSuccess) err = cudaMemset(e->d_barrier, 0, 2 * sizeof(uint32_t));
    if (err == cudaSuccess) err = cudaMemset(e->d_tickets, 0, ticket_count(dim) * sizeof(uint32_t));
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

int adacomp_embed_last_error(adacomp_embed_t* h, void* cuda_stream) {
    if (!h) return ADACOMP_ERR_INVALID;
    DeviceGuard guard(h->device);
    ADACOMP_CUDA(guard.err);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    int status = 0;
    ADACOMP_CUDA(cudaMemcpyAsync(&status, h->d_status, sizeof(int), cudaMemcpyDeviceToHost, stream));
    ADACOMP_CUDA(cudaMemsetAsync(h->d_status, 0, sizeof(int), stream));
    ADACOMP_CUDA(cudaStreamSynchronize(stream));
    if (status == ADACOMP_ERR_TIMEOUT) {                            // blocks that gave up left the barrier anywhere
        ADACOMP_CUDA(cudaMemsetAsync(h->d_barrier, 0, 2 * sizeof(uint32_t), stream));
        ADACOMP_CUDA(cudaStreamSynchronize(stream));
    }
    return status;
}

int adacomp_embed_destroy(adacomp_embed_t* h) {
    delete h;
    return ADACOMP_OK;
}

}  // extern "C"
