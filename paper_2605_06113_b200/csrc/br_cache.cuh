// The paged caches of the decode workers, kept in line with the request lengths that the routing step leaves on the GPU.
// A worker stores its requests' keys and values in P blocks of t tokens.  Row b of its block table names the blocks of the
// request in slot b, in token order; the blocks that no request holds are on a free list.  With n_b tokens in slot b:
//
//   br_block_tables   need_b = ceil(n_b / t).  Rows that hold more give their tails back, rows that hold less grow.
//   br_slot_map       token p of the request in slot b lives in cache slot table[b][p / t] t + p mod t.
//   br_page_lists     the running requests packed in slot order, with their blocks one after another.
//
// Prefix sums over a worker's slots turn each of them into independent copies: every moved block, token or page knows its
// source and its place from the sums alone, so nothing is ordered by atomics and results do not depend on timing.
#pragma once
#include "br_device.cuh"
#include "../../include/br.h"

namespace br {

constexpr int kCacheThreads = 256;          // at least BR_MAX_B: one slot a thread

struct CacheArgs {
    int32_t G, B, t, T, P;
    int32_t first_row;                      // first worker: first_instance * G
    const int32_t *len, *step;              // [N][G][B] and [N] or NULL
    int32_t *table, *n_blocks, *free_list, *n_free;
};

struct TableArgs {
    CacheArgs c;
    int32_t *n_blocks_out, *n_free_out, *short_out;
};

struct SlotArgs {
    CacheArgs c;
    const int32_t *n_new;
    int32_t room;
    int32_t *cu;
    int64_t *slots;
};

struct PageArgs {
    CacheArgs c;
    int32_t *n_seq, *seq_slot, *indptr, *indices, *last;
};

// tokens of the request in a slot: len + step, at least 0 and at most 2^31 - 1; 0 for a free slot
__device__ __forceinline__ int cache_tokens(int len, int step)
{
    if (len == BR_EMPTY_SLOT) return 0;
    const long long n = (long long)len + step;
    return n < 0 ? 0 : n > 0x7FFFFFFF ? 0x7FFFFFFF : (int)n;
}

__device__ __forceinline__ int blocks_of(int tokens, int t) { return tokens > 0 ? (tokens - 1) / t + 1 : 0; }

// Inclusive sum over the block's threads, in thread order; *total: the sum of all.
template <typename V>
__device__ __forceinline__ V block_scan(V v, V *part, V *total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    for (int o = 1; o < 32; o <<= 1) {
        const V u = __shfl_up_sync(kFull, v, o);
        if (lane >= o) v += u;
    }
    __syncthreads();                        // `part` may hold an earlier scan's sums
    if (lane == 31) part[warp] = v;
    __syncthreads();
    V before = 0, all = 0;
    for (int w = 0; w < warps; ++w) {
        if (w < warp) before += part[w];
        all += part[w];
    }
    *total = all;
    return v + before;
}

// the slot whose items contain item e: the first b with upto[b] > e (upto: inclusive sums of the items)
__device__ __forceinline__ int slot_of(const int *upto, int B, int e)
{
    int lo = 0, hi = B - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (upto[mid] > e) hi = mid; else lo = mid + 1;
    }
    return lo;
}

// One block a worker.  Block a of the growth (in slot and table order) is block a of those taken back (same order) while
// there are any, then the free list from its end; the rest of those taken back joins the free list, the first on top.
__global__ void __launch_bounds__(kCacheThreads) br_block_tables_kernel(const TableArgs a)
{
    __shared__ int back_upto[kCacheThreads], grow_upto[kCacheThreads], need_s[kCacheThreads], have_s[kCacheThreads];
    __shared__ long long part[kCacheThreads / 32];
    const CacheArgs &c = a.c;
    const size_t row = (size_t)c.first_row + blockIdx.x;
    const int b = threadIdx.x;
    const int step = c.step ? c.step[row / c.G] : 0;
    const int n_free = c.n_free[row];
    int need = 0, have = 0;
    if (b < c.B) {
        need = blocks_of(cache_tokens(c.len[row * c.B + b], step), c.t);
        have = c.n_blocks[row * c.B + b];
    }
    long long held, R, asked, missing;
    block_scan<long long>(have, part, &held);
    const bool bad = __syncthreads_or(have < 0 || have > c.T) || n_free < 0 || n_free + held > c.P;
    if (bad) {                              // counts that no sequence of updates leaves behind: the worker is left as it was
        if (b < c.B) a.n_blocks_out[row * c.B + b] = have;
        if (b == 0) {
            a.n_free_out[row] = n_free;
            if (a.short_out) a.short_out[row] = -1;
        }
        return;
    }
    const int back = max(have - need, 0), want = max(need - have, 0);
    const int back_in = (int)block_scan<long long>(back, part, &R);
    const int ask = need <= c.T ? want : 0;
    const long long ask_in = block_scan<long long>(ask, part, &asked);
    const int give = ask_in <= n_free + R ? ask : 0;
    long long A;
    const int grow_in = (int)block_scan<long long>(give, part, &A);
    block_scan<long long>(want - give, part, &missing);
    back_upto[b] = back_in; grow_upto[b] = grow_in; need_s[b] = need; have_s[b] = have;
    __syncthreads();
    if (b < c.B) a.n_blocks_out[row * c.B + b] = have + give - back;
    if (b == 0) {
        a.n_free_out[row] = n_free + (int)R - (int)A;
        if (a.short_out) a.short_out[row] = (int)min(missing, 0x7FFFFFFFll);
    }
    int32_t *table = c.table + row * c.B * c.T;
    int32_t *list = c.free_list + row * c.P;
    const int most = (int)max(R, A);
    for (int e = threadIdx.x; e < most; e += blockDim.x) {
        int id;
        if (e < (int)R) {
            const int s = slot_of(back_upto, c.B, e);
            id = table[(size_t)s * c.T + have_s[s] - (back_upto[s] - e)];
        } else {
            id = list[n_free - 1 - (e - (int)R)];
        }
        if (e < (int)A) {
            const int s = slot_of(grow_upto, c.B, e);
            table[(size_t)s * c.T + need_s[s] - (grow_upto[s] - e)] = id;
        } else {
            list[n_free + (int)R - 1 - e] = id;
        }
    }
}

// One block a worker: a token's place in the map is the sum of the new tokens ahead of it.
__global__ void __launch_bounds__(kCacheThreads) br_slot_map_kernel(const SlotArgs a)
{
    __shared__ int upto[kCacheThreads], tokens_s[kCacheThreads], held_s[kCacheThreads];
    __shared__ long long part[kCacheThreads / 32];
    const CacheArgs &c = a.c;
    const size_t row = (size_t)c.first_row + blockIdx.x;
    const int b = threadIdx.x;
    const int step = c.step ? c.step[row / c.G] : 0;
    int n = 0, q = 0, held = 0;
    if (b < c.B) {
        n = cache_tokens(c.len[row * c.B + b], step);
        q = a.n_new ? min(max(a.n_new[row * c.B + b], 0), n) : n > 0;
        held = min(max(c.n_blocks[row * c.B + b], 0), c.T);
    }
    long long all;
    const long long in = block_scan<long long>(q, part, &all);
    int32_t *cu = a.cu + row * (c.B + 1);
    upto[b] = (int)min(in, 0x7FFFFFFFll); tokens_s[b] = n; held_s[b] = held;
    __syncthreads();
    if (b < c.B) cu[b + 1] = upto[b];
    if (b == 0) cu[0] = 0;
    const int32_t *table = c.table + row * c.B * c.T;
    int64_t *out = a.slots + row * a.room;
    const int count = (int)min(all, (long long)a.room);
    for (int e = threadIdx.x; e < count; e += blockDim.x) {
        const int s = slot_of(upto, c.B, e);
        const int p = tokens_s[s] - (upto[s] - e), column = p / c.t;
        out[e] = column < held_s[s] ? (long long)table[(size_t)s * c.T + column] * c.t + (p - column * c.t) : -1;
    }
}

// One block a worker: the running slots move up, their blocks follow one another.
__global__ void __launch_bounds__(kCacheThreads) br_page_lists_kernel(const PageArgs a)
{
    __shared__ int upto[kCacheThreads];
    __shared__ int part[kCacheThreads / 32];
    const CacheArgs &c = a.c;
    const size_t row = (size_t)c.first_row + blockIdx.x;
    const int b = threadIdx.x;
    const int step = c.step ? c.step[row / c.G] : 0;
    int n = 0, need = 0, held = 0;
    if (b < c.B) {
        n = cache_tokens(c.len[row * c.B + b], step);
        need = blocks_of(n, c.t);
        held = min(max(c.n_blocks[row * c.B + b], 0), c.T);
    }
    const int pages = min(need, held);
    int count, all;
    const int rank = block_scan<int>(n > 0, part, &count) - (n > 0);
    const int in = block_scan<int>(pages, part, &all);
    upto[b] = in;
    int32_t *indptr = a.indptr + row * (c.B + 1);
    if (n > 0) {
        a.seq_slot[row * c.B + rank] = b;
        indptr[rank] = in - pages;
        a.last[row * c.B + rank] = pages == 0 ? 0 : need <= held ? n - (need - 1) * c.t : c.t;
    }
    if (b >= count && b < c.B) {
        a.seq_slot[row * c.B + b] = -1;
        a.last[row * c.B + b] = 0;
        indptr[b] = all;
    }
    if (b == 0) { indptr[c.B] = all; a.n_seq[row] = count; }
    __syncthreads();
    const int32_t *table = c.table + row * c.B * c.T;
    int32_t *out = a.indices + row * c.P;
    const int most = min(all, c.P);
    for (int e = threadIdx.x; e < most; e += blockDim.x) {
        const int s = slot_of(upto, c.B, e);
        out[e] = table[(size_t)s * c.T + (e - (s ? upto[s - 1] : 0))];
    }
}

}  // namespace br
