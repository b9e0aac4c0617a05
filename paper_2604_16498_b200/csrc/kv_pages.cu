// The tables of a KV cache in pages: pages to the requests that need some, and each token's slot; pages back.
//
// With have = ceil(len / P) and need = ceil((len + count) / P), a request's first new page is the sum of need - have over the requests before it, and
// its first token the sum of counts: two running sums over the requests, 1024 of them at a time.  Everything else follows from them for each page and
// each token alone, which finds its request by bisection of the sums in shared memory.
//
// Nothing here is bound by bytes (8192 tokens: 100 KB): the time is the launch and a chain of dependent reads (64 requests with a token each 2.5 us in a
// chain of calls, 3.6 with 1024 threads; 300 requests with 8192 tokens 4.5).  So one CTA does it all for a decode
// step, and a cluster of eight for many tokens, each of which makes the sums for itself.  Tables, counts and the stack of free pages are read from L2:
// the kernel before this one may have had older ones in L1.
#include "kv_cache.cuh"

namespace forge {
namespace {

constexpr int kPagesThreads = 1024, kFewThreads = 128;  // of a CTA; that of a small step
constexpr int kFewTokens = 512;                         // ... which has no more requests than threads, and tokens than this
constexpr int kManyTokens = 2048, kManyCtas = 8;        // from how many tokens on a cluster does it

struct PagesArgs {
    const int32_t *lens, *counts, *done;
    int32_t *table, *free_pages;
    const int32_t* free_count;
    int32_t *new_lens, *starts, *slots, *positions, *requests, *free_left;
    int B, max_pages, page_shift, num_pages, T;
};

// The sum of v over the threads up to this one; *all: over all threads.  `warps`: room for one of each warp.
template <int THREADS, typename V>
__device__ __forceinline__ V block_scan(V v, V* warps, V* all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    __syncthreads();  // `warps` of the sum before has been read
    if (lane == 31) warps[warp] = v;
    __syncthreads();
    static_assert(THREADS <= 1024, "a lane for each warp");
    V w = lane < THREADS / 32 ? warps[lane] : V(0);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V t = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += t;
    }
    *all = __shfl_sync(0xffffffffu, w, 31);
    const V before = __shfl_sync(0xffffffffu, w, max(warp - 1, 0));
    return warp > 0 ? v + before : v;
}
// The first of THREADS ascending sums that is above x; the last one if none is.
template <int THREADS>
__device__ __forceinline__ int first_above(const int* sums, int x) {
    int at = 0;
#pragma unroll
    for (int step = THREADS / 2; step > 0; step >>= 1)
        if (sums[at + step - 1] <= x) at += step;
    return at;
}
__device__ __forceinline__ int free_pages_of(const PagesArgs& a) { return min(max(__ldcg(a.free_count), 0), a.num_pages); }
__device__ __forceinline__ int clamped_len(const PagesArgs& a, int b) { return min(max(__ldcg(a.lens + b), 0), a.max_pages << a.page_shift); }

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

template <int CTAS, int THREADS>
__global__ void __launch_bounds__(THREADS) assign_pages_kernel(const PagesArgs a) {
    __shared__ int64_t warp_tokens[THREADS / 32];
    __shared__ int warp_pages[THREADS / 32];
    // of the requests of this turn: where their tokens and new pages end, how many rows they have (-1 - rows: refused)
    __shared__ int token_end[THREADS], page_end[THREADS], rows_of[THREADS];
    __shared__ int taken;
    pdl_launch_dependents();
    pdl_wait();
    const int rank = CTAS > 1 ? (int)blockIdx.x : 0, tid = threadIdx.x;  // the grid is one cluster
    const int room = free_pages_of(a), P1 = (1 << a.page_shift) - 1;
    if (tid == 0) taken = 0;
    int64_t tokens = 0;  // of the requests before this turn's
    int pages = 0;       // and new pages that they want (no more than T / P + B, those that T has no room for left out)
    for (int b0 = 0; b0 < a.B; b0 += THREADS) {
        const int b = b0 + tid;
        const int len = b < a.B ? clamped_len(a, b) : 0;
        const int64_t count = b >= a.B ? 0 : a.counts ? max(__ldcg(a.counts + b), 0) : 1;
        if (CTAS > 1) cluster_arrive();  // all have read lens, which new_lens may be
        int64_t all_tokens;
        int all_pages;
        const int64_t end = tokens + block_scan<THREADS>(count, warp_tokens, &all_tokens);
        const int have = (len + P1) >> a.page_shift;
        const int64_t need = (len + count + P1) >> a.page_shift;
        bool fits = need <= a.max_pages && end <= a.T;
        const int want = fits ? (int)need - have : 0;
        const int wanted = pages + block_scan<THREADS>(want, warp_pages, &all_pages);
        fits = fits && (want == 0 || wanted <= room);
        token_end[tid] = (int)min(end, (int64_t)a.T);
        page_end[tid] = wanted;
        rows_of[tid] = fits ? len : -1 - len;
        if (fits && want > 0) atomicMax(&taken, wanted);
        if (CTAS > 1) cluster_wait();
        if (rank == 0 && b < a.B) {
            a.new_lens[b] = fits ? (int)(len + count) : len;
            if (a.starts) {
                a.starts[b + 1] = token_end[tid];
                if (b == 0) a.starts[0] = 0;
            }
        }
        __syncthreads();
        const int page_to = min(pages + all_pages, taken);
        for (int i = pages + rank * THREADS + tid; i < page_to; i += CTAS * THREADS) {  // new pages into the table
            const int at = first_above<THREADS>(page_end, i), first = at > 0 ? page_end[at - 1] : pages;  // up to `taken` none is refused
            a.table[(int64_t)(b0 + at) * a.max_pages + ((rows_of[at] + P1) >> a.page_shift) + i - first] = __ldcg(a.free_pages + room - 1 - i);
        }
        const int token0 = (int)min(tokens, (int64_t)a.T), token1 = (int)min(tokens + all_tokens, (int64_t)a.T);
        for (int t = token0 + rank * THREADS + tid; t < token1; t += CTAS * THREADS) {
            const int at = first_above<THREADS>(token_end, t), has = rows_of[at], rows = has >= 0 ? has : -1 - has;
            const int pos = rows + t - (at > 0 ? token_end[at - 1] : token0);
            int slot = -1;
            if (has >= 0) {
                const int page = pos >> a.page_shift, old = (rows + P1) >> a.page_shift;
                const int entry = page < old ? __ldcg(a.table + (int64_t)(b0 + at) * a.max_pages + page)
                                             : __ldcg(a.free_pages + room - 1 - ((at > 0 ? page_end[at - 1] : pages) + page - old));
                if ((unsigned)entry < (unsigned)a.num_pages) slot = (entry << a.page_shift) + (pos & P1);
            }
            a.slots[t] = slot;
            if (a.positions) a.positions[t] = pos;
            if (a.requests) a.requests[t] = b0 + at;
        }
        tokens += all_tokens;
        pages += all_pages;
        __syncthreads();  // this turn's sums have been read
    }
    for (int64_t t = min(tokens, (int64_t)a.T) + rank * THREADS + tid; t < a.T; t += CTAS * THREADS) {  // behind the last token
        a.slots[t] = -1;
        if (a.positions) a.positions[t] = 0;
        if (a.requests) a.requests[t] = -1;
    }
    if (rank == 0 && tid == 0) a.free_left[0] = room - taken;  // all CTAs have read free_count: they have passed a barrier since
}

__global__ void __launch_bounds__(kPagesThreads) release_pages_kernel(const PagesArgs a) {
    __shared__ int64_t warp_pages[kPagesThreads / 32];
    __shared__ int64_t page_end[kPagesThreads];
    __shared__ int warp_good[kPagesThreads / 32];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, P1 = (1 << a.page_shift) - 1;
    int free = free_pages_of(a);
    for (int b0 = 0; b0 < a.B; b0 += kPagesThreads) {
        const int b = b0 + tid;
        const int64_t n = b < a.B && __ldcg(a.done + b) != 0 ? (clamped_len(a, b) + P1) >> a.page_shift : 0;
        int64_t all;
        page_end[tid] = block_scan<kPagesThreads>(n, warp_pages, &all);
        __syncthreads();
        for (int64_t i0 = 0; i0 < all; i0 += kPagesThreads) {
            const int64_t i = i0 + tid;
            int entry = -1;
            if (i < all) {
                int at = 0;
#pragma unroll
                for (int step = kPagesThreads / 2; step > 0; step >>= 1)
                    if (page_end[at + step - 1] <= i) at += step;
                entry = __ldcg(a.table + (int64_t)(b0 + at) * a.max_pages + (i - (at > 0 ? page_end[at - 1] : 0)));
            }
            const bool good = (unsigned)entry < (unsigned)a.num_pages;
            int all_good;
            const int to = free + block_scan<kPagesThreads>((int)good, warp_good, &all_good) - 1;
            if (good && to < a.num_pages) a.free_pages[to] = entry;
            free = min(free + all_good, a.num_pages);
        }
        __syncthreads();
    }
    if (tid == 0) a.free_left[0] = free;
}

bool odd4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

int tables_args(const forge_kv_page_tables* t, const int32_t* lens, int32_t* free_left, PagesArgs* a) {
    if (!t || !t->free_pages || !t->free_count || !lens || t->num_pages <= 0 || t->page_size <= 0) return FORGE_ERR_INVALID_ARG;
    if (odd4(t->free_pages) || odd4(t->free_count) || odd4(lens) || odd4(free_left)) return FORGE_ERR_INVALID_ARG;
    if (!page_size_ok(t->page_size)) return FORGE_ERR_UNSUPPORTED;
    int rows;
    const int st = check_table(t->table, t->B, t->max_pages, t->page_size, &rows);
    if (st != FORGE_OK) return st;
    if ((long long)t->num_pages * t->page_size >= (1LL << 31)) return FORGE_ERR_UNSUPPORTED;  // slots are counted in 32 bits
    *a = {};
    a->lens = lens;
    a->table = t->table;
    a->free_pages = t->free_pages;
    a->free_count = t->free_count;
    a->free_left = free_left ? free_left : t->free_count;
    a->B = t->B;
    a->max_pages = t->max_pages;
    a->page_shift = log2_of(t->page_size);
    a->num_pages = t->num_pages;
    return FORGE_OK;
}

}  // namespace
}  // namespace forge

extern "C" int forge_kv_assign_pages(const forge_kv_page_tables* tables, const int32_t* lens, const int32_t* counts,
                                     const forge_kv_page_slots* out, int32_t* free_left, void* stream) {
    using namespace forge;
    PagesArgs a;
    const int st = tables_args(tables, lens, free_left, &a);
    if (st != FORGE_OK) return st;
    if (!out || !out->new_lens || !out->slots || out->T <= 0 || odd4(counts) || odd4(out->new_lens) || odd4(out->starts) || odd4(out->slots) ||
        odd4(out->positions) || odd4(out->requests))
        return FORGE_ERR_INVALID_ARG;
    if (out->T > 1 << 30) return FORGE_ERR_UNSUPPORTED;
    a.counts = counts;
    a.new_lens = out->new_lens;
    a.starts = out->starts;
    a.slots = out->slots;
    a.positions = out->positions;
    a.requests = out->requests;
    a.T = out->T;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (a.B <= kFewThreads && a.T <= kFewTokens)
        FORGE_CUDA_TRY(launch_pdl(assign_pages_kernel<1, kFewThreads>, dim3(1), dim3(kFewThreads), 0, s, a));
    else if (a.T < kManyTokens)
        FORGE_CUDA_TRY(launch_pdl(assign_pages_kernel<1, kPagesThreads>, dim3(1), dim3(kPagesThreads), 0, s, a));
    else
        FORGE_CUDA_TRY(launch_pdl_cluster(assign_pages_kernel<kManyCtas, kPagesThreads>, dim3(kManyCtas), dim3(kPagesThreads), 0, kManyCtas, s, a));
    return finish_launch(1);
}

extern "C" int forge_kv_release_pages(const forge_kv_page_tables* tables, const int32_t* lens, const int32_t* done, int32_t* free_left,
                                      void* stream) {
    using namespace forge;
    PagesArgs a;
    const int st = tables_args(tables, lens, free_left, &a);
    if (st != FORGE_OK) return st;
    if (!done || odd4(done)) return FORGE_ERR_INVALID_ARG;
    a.done = done;
    FORGE_CUDA_TRY(launch_pdl(release_pages_kernel, dim3(1), dim3(kPagesThreads), 0, static_cast<cudaStream_t>(stream), a));
    return finish_launch(1);
}
