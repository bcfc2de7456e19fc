// Page tables and slot maps of a paged cache, made on the device from request lengths (mpq_pages_extend), and the
// way back (mpq_pages_trim).
//
// A batch's first tokens and first new pages are running sums over its entries, n_b and need_b.  A few hundred entries
// are summed in the time of one memory round trip, so every CTA makes the sums for itself, keeps them in shared memory and
// fills its share of the outputs from them: one launch, no second kernel that waits for the sums.  A slot's entry is
// found by bisection in shared memory.  The state that all CTAs read (lengths and the number of free pages) is changed by
// whichever CTA draws the last ticket, when all have read it; nobody waits.
// Bound by latency: four dependent loads (sequence, length, page, store) around the sums.  64 entries of one token take 4.5 us
// of the device, 512 entries with 200,000 new tokens 14, a trim 4 to 6.
#include "mpq_common.cuh"

namespace mpq {

constexpr int kPageThreads = 512;
constexpr int kPageBatch = 8192;                          // entries that shared memory holds

struct PageArgs {
    int32_t* table; int64_t per;
    int32_t* lens; int sequences;
    int32_t* free; int64_t pages;
    int32_t* count;                                       // [0] free pages, [1] tickets drawn in this call
    int page_size;
    const int32_t* seqs; const int32_t* amount; int batch;
    int64_t* slots; int64_t tokens;
    int32_t *starts, *kv_lens, *rows, *missing;
};

// What a CTA knows of an entry: its sequence (-1: none), tokens in the cache, first token and first page in the batch.
struct PageEntries {
    int32_t *seq, *len, *start, *first;                   // start and first have batch + 1 elements
    __device__ PageEntries(int32_t* s, int batch) : seq(s), len(s + batch), start(s + 2 * batch), first(s + 3 * batch + 1) {}
    static size_t bytes(int batch) { return (size_t)(4 * batch + 2) * sizeof(int32_t); }
};

__device__ __forceinline__ int pages_of(int64_t tokens, int page_size) { return (int)((tokens + page_size - 1) / page_size); }

// Running sums of two numbers over the CTA's threads, on top of `carry`; returns the sums before this thread's numbers.
__device__ __forceinline__ void block_scan(int64_t (&v)[2], int64_t (&carry)[2], int64_t (*sh)[2]) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int64_t s[2] = {v[0], v[1]};
    for (int o = 1; o < 32; o <<= 1)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t below = __shfl_up_sync(0xffffffffu, s[i], o);
            if (lane >= o) s[i] += below;
        }
    if (lane == 31) { sh[warp][0] = s[0]; sh[warp][1] = s[1]; }
    __syncthreads();
    int64_t before[2] = {carry[0], carry[1]};
#pragma unroll
    for (int w = 0; w < kPageThreads / 32; ++w)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (w < warp) before[i] += sh[w][i];
            carry[i] += sh[w][i];
        }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) v[i] = before[i] + s[i] - v[i];
}

// Index of the last entry whose first element is not behind x: starts ascend, entries without elements share theirs.
__device__ __forceinline__ int entry_of(const int32_t* starts, int batch, int32_t x) {
    int lo = 0, hi = batch;                               // starts[lo] <= x < starts[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// True in the CTA that is last to have read the state.
__device__ __forceinline__ bool last_reader(const PageArgs& g) {
    __shared__ int last;
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(g.count + 1, 1) == (int)gridDim.x - 1;
    }
    __syncthreads();
    return last != 0;
}

__global__ void __launch_bounds__(kPageThreads) pages_extend_kernel(const PageArgs g) {
    extern __shared__ int32_t held[];
    __shared__ int64_t sums[kPageThreads / 32][2];
    __shared__ int too_long;
    const PageEntries e(held, g.batch);
    chain_entry();
    const int count = g.count[0];
    if (threadIdx.x == 0) too_long = 0;
    __syncthreads();
    int64_t carry[2] = {0, 0};
    for (int b0 = 0; b0 < g.batch; b0 += kPageThreads) {
        const int b = b0 + threadIdx.x;
        int q = -1, n = 0, len = 0;
        if (b < g.batch) {
            q = g.seqs ? g.seqs[b] : b;
            n = g.amount[b];
            if (q < 0 || q >= g.sequences || n < 0) { q = -1; n = 0; }
            else len = max(0, g.lens[q]);
        }
        int64_t v[2] = {n, 0};
        if (b < g.batch) {
            const int64_t want = ((int64_t)len + n + g.page_size - 1) / g.page_size;
            if (want > g.per) too_long = 1;
            v[1] = want - pages_of(len, g.page_size);
        }
        block_scan(v, carry, sums);
        if (b < g.batch) { e.seq[b] = q; e.len[b] = len; e.start[b] = (int32_t)min(v[0], (int64_t)0x7fffffff); e.first[b] = (int32_t)min(v[1], (int64_t)0x7fffffff); }
    }
    const int total = (int)min(carry[0], (int64_t)0x7fffffff);
    if (threadIdx.x == 0) { e.start[g.batch] = total; e.first[g.batch] = (int32_t)min(carry[1], (int64_t)0x7fffffff); }
    const bool last = last_reader(g);                     // (its barriers also end the writes above)
    const int64_t lacking = carry[1] - count;
    const int missing = too_long ? -1 : carry[0] > g.tokens ? -2 : (int)min(max(lacking, (int64_t)0), (int64_t)0x7fffffff);
    const bool fine = missing == 0;
    if (last) {
        for (int b = threadIdx.x; fine && b < g.batch; b += kPageThreads)
            if (e.seq[b] >= 0) g.lens[e.seq[b]] = e.len[b] + (e.start[b + 1] - e.start[b]);
        if (threadIdx.x == 0) {
            if (fine) g.count[0] = count - (int)carry[1];
            g.count[1] = 0;
            *g.missing = missing;
        }
    }
    // page `i` of the new ones of an entry; in bounds whatever the state holds
    auto popped = [&](int64_t i) {
        const int64_t at = (int64_t)count - 1 - i;
        return at >= 0 && at < g.pages ? g.free[at] : 0;
    };
    const int64_t threads = (int64_t)gridDim.x * kPageThreads, thread = (int64_t)blockIdx.x * kPageThreads + threadIdx.x;
    for (int64_t b = thread; b <= g.batch; b += threads) {
        g.starts[b] = fine ? e.start[b] : 0;
        if (b < g.batch) g.kv_lens[b] = fine && e.seq[b] >= 0 ? e.len[b] + (e.start[b + 1] - e.start[b]) : 0;
    }
    for (int64_t t = thread; t < g.tokens; t += threads) {
        int64_t slot = -1;
        if (fine && t < total) {
            const int b = entry_of(e.start, g.batch, (int32_t)t);
            const int j = e.len[b] + (int)t - e.start[b], have = pages_of(e.len[b], g.page_size), i = j / g.page_size;
            const int page = i < have ? g.table[e.seq[b] * g.per + i] : (int)popped((int64_t)e.first[b] + i - have);
            slot = (int64_t)page * g.page_size + (j - i * g.page_size);
        }
        g.slots[t] = slot;
    }
    // rows of the batch's table in pieces of 128 entries, one to a warp
    const int lane = threadIdx.x & 31;
    const int64_t pieces = (g.per + 127) / 128;
    for (int64_t w = thread >> 5; w < pieces * g.batch; w += threads >> 5) {
        const int b = (int)(w / pieces);
        const int64_t i0 = w % pieces * 128;
        const int q = e.seq[b], have = q < 0 || !fine ? 0 : pages_of(e.len[b], g.page_size);
        const int want = q < 0 || !fine ? 0 : have + e.first[b + 1] - e.first[b];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t i = i0 + 32 * j + lane;
            if (i >= g.per) break;
            int page = 0;
            if (i < have) page = g.table[q * g.per + i];
            else if (i < want) {
                page = popped((int64_t)e.first[b] + i - have);
                g.table[q * g.per + i] = page;            // nobody reads the entries behind the sequence's old pages
            }
            g.rows[b * g.per + i] = page;
        }
    }
}

__global__ void __launch_bounds__(kPageThreads) pages_trim_kernel(const PageArgs g) {
    extern __shared__ int32_t held[];
    __shared__ int64_t sums[kPageThreads / 32][2];
    const PageEntries e(held, g.batch);                   // start: first page given back; first: the page's place in the sequence
    chain_entry();
    const int64_t count = min(max((int64_t)g.count[0], (int64_t)0), g.pages);
    int64_t carry[2] = {0, 0};
    for (int b0 = 0; b0 < g.batch; b0 += kPageThreads) {
        const int b = b0 + threadIdx.x;
        int q = -1, len = 0, keep = 0, first = 0;
        int64_t v[2] = {0, 0};
        if (b < g.batch) {
            q = g.seqs ? g.seqs[b] : b;
            keep = g.amount[b];
            if (q < 0 || q >= g.sequences || keep < 0) q = -1;
            else len = max(0, g.lens[q]);
            keep = min(keep, len);
            if (q >= 0) {
                first = pages_of(keep, g.page_size);
                v[0] = max((int64_t)0, min((int64_t)pages_of(len, g.page_size), g.per) - first);
            }
        }
        block_scan(v, carry, sums);
        if (b < g.batch) { e.seq[b] = q; e.len[b] = keep; e.start[b] = (int32_t)min(v[0], (int64_t)0x7fffffff); e.first[b] = first; }
    }
    const int64_t total = min(carry[0], g.pages - count); // no more than the list holds
    if (threadIdx.x == 0) e.start[g.batch] = (int32_t)min(carry[0], (int64_t)0x7fffffff);
    if (last_reader(g)) {
        for (int b = threadIdx.x; b < g.batch; b += kPageThreads)
            if (e.seq[b] >= 0) g.lens[e.seq[b]] = e.len[b];
        if (threadIdx.x == 0) { g.count[0] = (int)(count + total); g.count[1] = 0; }
    }
    // the first page given back lies deepest under the pages pushed after it: in the order in which mpq_pages_extend takes them
    for (int64_t i = (int64_t)blockIdx.x * kPageThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kPageThreads) {
        const int b = entry_of(e.start, g.batch, (int32_t)i);
        g.free[count + total - 1 - i] = g.table[e.seq[b] * g.per + e.first[b] + (i - e.start[b])];
    }
}

int pages_call(bool extend, const PageArgs& g, cudaStream_t st) {
    if (!g.table || !g.lens || !g.free || !g.count || (g.batch != 0 && !g.amount)) return MPQ_ERR_NULL;
    if (extend && (!g.starts || !g.missing || (g.tokens != 0 && !g.slots) || (g.batch != 0 && (!g.kv_lens || !g.rows)))) return MPQ_ERR_NULL;
    if (g.per <= 0 || g.sequences <= 0 || g.pages <= 0 || g.pages > 0x7fffffff || g.page_size <= 0 || g.per > 0x7fffffff / g.page_size || g.batch < 0 ||
        g.tokens < 0 || g.tokens > 0x7fffffff || (!g.seqs && g.batch > g.sequences)) return MPQ_ERR_BAD_SHAPE;
    if (g.batch > kPageBatch) return MPQ_ERR_UNSUPPORTED;
    for (const void* p : {(const void*)g.table, (const void*)g.lens, (const void*)g.free, (const void*)g.count, (const void*)g.seqs, (const void*)g.amount,
                          (const void*)g.starts, (const void*)g.kv_lens, (const void*)g.rows, (const void*)g.missing})
        if (reinterpret_cast<uintptr_t>(p) & 3u) return MPQ_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(g.slots) & 7u) return MPQ_ERR_ALIGN;
    static PerDeviceOnce once[2];
    auto* kernel = extend ? pages_extend_kernel : pages_trim_kernel;
    const int rc = once[extend].raise_smem_limit(kernel, PageEntries::bytes(kPageBatch));
    if (rc != MPQ_OK) return rc;
    const int sms = sm_count();
    if (sms == 0) return MPQ_ERR_CUDA;
    // four outputs a thread; a trim gives a small part of the table back
    const int64_t work = extend ? g.tokens + g.batch * g.per : g.batch * g.per / 8;
    const int64_t blocks = ceil_div(work, 4 * kPageThreads);
    return launch_chained_as(true, kernel, (unsigned)(blocks < 1 ? 1 : blocks < sms ? blocks : sms), kPageThreads, PageEntries::bytes(g.batch), st, g);
}

}  // namespace mpq

using namespace mpq;

extern "C" int mpq_pages_extend(int32_t* table, int64_t per_sequence, int32_t* lens, int sequences, int32_t* free_pages, int64_t pages,
                                int32_t* count, int page_size, const int32_t* seqs, const int32_t* new_tokens, int batch, int64_t tokens,
                                int64_t* slots, int32_t* q_starts, int32_t* kv_lens, int32_t* batch_table, int32_t* missing, void* stream) {
    const PageArgs g = {table, per_sequence, lens, sequences, free_pages, pages, count, page_size, seqs, new_tokens, batch,
                        slots, tokens, q_starts, kv_lens, batch_table, missing};
    return pages_call(true, g, (cudaStream_t)stream);
}

extern "C" int mpq_pages_trim(int32_t* table, int64_t per_sequence, int32_t* lens, int sequences, int32_t* free_pages, int64_t pages,
                              int32_t* count, int page_size, const int32_t* seqs, const int32_t* keep, int batch, void* stream) {
    const PageArgs g = {table, per_sequence, lens, sequences, free_pages, pages, count, page_size, seqs, keep, batch,
                        nullptr, 0, nullptr, nullptr, nullptr, nullptr};
    return pages_call(false, g, (cudaStream_t)stream);
}
