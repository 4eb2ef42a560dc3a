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
//
// A warp takes one worker, or one of `parts` equal pieces of what a worker has to move.  Each warp sums its worker's slots
// for itself (a few loads a lane, from L2 but for the first), which costs less than passing the sums between warps.  The
// pieces are cut from the items, not from the slots, so one long request is spread like many short ones.
#pragma once
#include "br_device.cuh"
#include "../../include/br.h"

namespace br {

constexpr int kCacheThreads = 256;

struct CacheArgs {
    int32_t G, B, t, T, P;
    int32_t first_row, workers;             // rows first_row .. first_row + workers of the arrays by worker
    int32_t parts;                          // warps a worker
    uint32_t t_magic; int32_t t_shift;      // p / t = umulhi(2 p, t_magic) >> t_shift for 0 <= p < 2^31
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

// The multiplier of a division by t, 1 <= t <= 2^20: with s = ceil(log2 t) and m = ceil(2^(31 + s) / t) < 2^32 the error
// m t - 2^(31 + s) is below t <= 2^s, so floor(p m / 2^(31 + s)) = floor(p / t) for p < 2^31 (Granlund and Montgomery).
inline void cache_divisor(int t, uint32_t *magic, int32_t *shift)
{
    int s = 0;
    while ((1 << s) < t) ++s;
    *magic = (uint32_t)(((1ull << (31 + s)) + t - 1) / t);
    *shift = s;
}

// Warps a worker.  Tables: a power of two, so that the warps of a worker make up a block.  Copies: pieces of 512 items or more.
constexpr int kCacheWarps = 148 * 64;       // the warps that the GPU holds at once
inline int cache_table_parts(int workers)
{
    int parts = 32;
    while (parts > 1 && (long long)parts * workers > kCacheWarps) parts /= 2;
    return parts;
}
inline int cache_copy_parts(int workers, int most_items)
{
    const int fill = 2 * kCacheWarps / workers + 1, cut = (most_items + 511) / 512;
    return fill < cut ? fill : cut;
}

__device__ __forceinline__ int over_t(const CacheArgs &c, int p) { return (int)(__umulhi(2u * (unsigned)p, c.t_magic) >> c.t_shift); }

// tokens of the request in a slot: len + step, at least 0 and at most 2^31 - 1; 0 for a free slot
__device__ __forceinline__ int cache_tokens(int len, int step)
{
    if (len == BR_EMPTY_SLOT) return 0;
    const long long n = (long long)len + step;
    return n < 0 ? 0 : n > 0x7FFFFFFF ? 0x7FFFFFFF : (int)n;
}

__device__ __forceinline__ int cache_blocks(const CacheArgs &c, int tokens) { return tokens > 0 ? over_t(c, tokens - 1) + 1 : 0; }

// a + b for 0 <= a, b < 2^31, at most 2^31 - 1
__device__ __forceinline__ int add_to_most(int a, int b) { return (int)min((unsigned)a + (unsigned)b, 0x7FFFFFFFu); }

// Sum of v over the lanes below this one (each sum at most 2^31 - 1).
__device__ __forceinline__ int sum_below(int v, int lane)
{
    int in = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(kFull, in, o);
        if (lane >= o) in = add_to_most(in, u);
    }
    const int below = __shfl_up_sync(kFull, in, 1);
    return lane ? below : 0;
}

// A slot's run of items in the sequence of all items of its worker: item e of the run, e < upto, is at e + shift in the slot.
struct Run { int upto, shift; };

// Position in the runs of a worker's B slots.
struct Walk {
    const Run *runs;
    int B, slot;
    Run at;
    // the slot of item e: the first whose run ends behind it
    __device__ __forceinline__ void seek(const Run *r, int B_, int e)
    {
        runs = r; B = B_;
        int lo = 0, hi = B - 1;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (runs[mid].upto > e) hi = mid; else lo = mid + 1;
        }
        slot = lo; at = runs[lo];
    }
    // on to item e, not before the present one
    __device__ __forceinline__ void to(int e)
    {
        while (at.upto <= e && slot < B - 1) at = runs[++slot];
    }
};

// Warp of the launch -> worker and piece; false behind the last worker.
__device__ __forceinline__ bool cache_place(const CacheArgs &c, size_t *row, int *part)
{
    const unsigned w = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const unsigned worker = w / (unsigned)c.parts;
    *part = (int)(w - worker * (unsigned)c.parts);
    *row = (size_t)c.first_row + worker;
    return worker < (unsigned)c.workers;
}

// Items [lo, hi) of `count` for this piece: equal numbers of units of 128, counted from `skew` items ahead of the first.
__device__ __forceinline__ void cache_piece(const CacheArgs &c, int part, int count, int skew, int *lo, int *hi)
{
    const int units = (count + skew + 127) / 128, each = (units + c.parts - 1) / c.parts;
    // (count is at most 2^30, so are the units before the last piece; the pieces behind them would pass 2^31 only as items)
    *lo = max(0, (int)min((long long)count, (long long)each * part * 128 - skew));
    *hi = (int)min((long long)count, (long long)each * (part + 1) * 128 - skew);
}

// Block a of the growth (in slot and table order) is block a of those taken back (same order) while there are any, then the
// free list from its end; the rest of those taken back joins the free list, the first on top.  What is read (the tails of
// rows that shrink, the list below n_free) is never written by the same call, so the pieces need no order; only the counts
// do, which are written where they may be read (one worker's warps share a block, and it meets before they are written).
template <int SPL>
__global__ void __launch_bounds__(1024) br_block_tables_kernel(const TableArgs a)
{
    extern __shared__ Run run_mem[];
    stream_order_gate();
    const CacheArgs &c = a.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Run *back_run = run_mem + (c.parts > 1 ? 0 : warp * 2 * c.B), *grow_run = back_run + c.B;
    size_t row; int part;
    const bool mine = cache_place(c, &row, &part);
    int n_free = 0, R = 0, A = 0;
    bool bad = false;
    if (mine) {
        const int step = c.step ? c.step[row / (unsigned)c.G] : 0;
        n_free = c.n_free[row];
        int need[SPL], have[SPL], held = 0, back = 0, ask = 0;
#pragma unroll
        for (int i = 0; i < SPL; ++i) {
            const int b = lane * SPL + i;
            need[i] = have[i] = 0;
            if (b < c.B) {
                need[i] = c.len[row * c.B + b];
                have[i] = c.n_blocks[row * c.B + b];
            }
        }
#pragma unroll
        for (int i = 0; i < SPL; ++i) {
            need[i] = lane * SPL + i < c.B ? cache_blocks(c, cache_tokens(need[i], step)) : 0;
            if ((unsigned)have[i] > (unsigned)c.T) { bad = true; continue; }
            held += have[i];
            back += max(have[i] - need[i], 0);
            ask += need[i] <= c.T ? max(need[i] - have[i], 0) : 0;
        }
        bad = __any_sync(kFull, bad) || (unsigned)n_free > (unsigned)c.P;
        // (with counts in range all sums stay below 2^30)
        bad = bad || n_free + (int)__reduce_add_sync(kFull, (unsigned)held) > c.P;
        if (!bad) {
            R = (int)__reduce_add_sync(kFull, (unsigned)back);
            int back_at = sum_below(back, lane), grow_at = sum_below(ask, lane);
            long long lacking = 0;
#pragma unroll
            for (int i = 0; i < SPL; ++i) {
                const int b = lane * SPL + i, less = max(have[i] - need[i], 0), more = max(need[i] - have[i], 0);
                if (b >= c.B) break;
                const Run taken = {back_at + less, need[i] - back_at};
                back_at += less;
                // a sum over all demands up to this one: the first that does not fit keeps out the ones behind it
                const int upto = grow_at + (need[i] <= c.T ? more : 0);
                const bool fits = need[i] <= c.T && upto <= n_free + R;
                const Run given = {fits ? upto : grow_at, have[i] - grow_at};
                if (part == 0) { back_run[b] = taken; grow_run[b] = given; }
                grow_at = upto;
                if (fits) A = upto; else lacking += more;
                have[i] += (fits ? more : 0) - less;
            }
            A = (int)__reduce_max_sync(kFull, (unsigned)A);
            if (part == 0 && a.short_out) {
                const bool some = __any_sync(kFull, lacking != 0);
                if (some)
                    for (int o = 16; o > 0; o >>= 1) lacking += __shfl_xor_sync(kFull, lacking, o);
                if (lane == 0) a.short_out[row] = (int)min(lacking, 0x7FFFFFFFll);
            }
        } else if (part == 0 && a.short_out && lane == 0) {
            a.short_out[row] = -1;
        }
        if (c.parts > 1) __syncthreads(); else __syncwarp();      // (with several warps a worker, a block holds one worker)
        if (part == 0) {
#pragma unroll
            for (int i = 0; i < SPL; ++i)
                if (lane * SPL + i < c.B) a.n_blocks_out[row * c.B + lane * SPL + i] = have[i];
            if (lane == 0) a.n_free_out[row] = n_free + R - A;
        }
        int lo, hi;
        cache_piece(c, part, max(R, A), 0, &lo, &hi);
        if (lo + lane < hi) {
            const auto table = mk_span(c.table + row * c.B * c.T, (long long)c.B * c.T);
            const auto list = mk_span(c.free_list + row * c.P, c.P);
            Walk from, to;
            if (lo + lane < R) from.seek(back_run, c.B, lo + lane);
            if (lo + lane < A) to.seek(grow_run, c.B, lo + lane);
            for (int e = lo + lane; e < hi; e += 32) {
                int id;
                if (e < R) {
                    from.to(e);
                    id = table[(long long)from.slot * c.T + e + from.at.shift];
                } else {
                    id = list[n_free + R - 1 - e];
                }
                if (e < A) {
                    to.to(e);
                    table[(long long)to.slot * c.T + e + to.at.shift] = id;
                } else {
                    list[n_free + R - 1 - e] = id;
                }
            }
        }
    }
}

// One new token a request: a lane's slots in a row, their places from the sums of the lanes below.
template <int SPL>
__global__ void __launch_bounds__(kCacheThreads) br_slot_newest_kernel(const SlotArgs a)
{
    stream_order_gate();
    const CacheArgs &c = a.c;
    const int lane = threadIdx.x & 31;
    size_t row; int part;
    if (!cache_place(c, &row, &part)) return;
    const int step = c.step ? c.step[row / (unsigned)c.G] : 0;
    int n[SPL], held[SPL], count = 0;
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        const int b = lane * SPL + i;
        n[i] = held[i] = 0;
        if (b < c.B) { n[i] = c.len[row * c.B + b]; held[i] = c.n_blocks[row * c.B + b]; }
    }
    const auto table = mk_span(c.table + row * c.B * c.T, (long long)c.B * c.T);
    const auto out = mk_span(a.slots + row * a.room, a.room);
    int32_t *cu = a.cu + row * (c.B + 1);
    long long slot[SPL];
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        const int b = lane * SPL + i;
        n[i] = b < c.B ? cache_tokens(n[i], step) : 0;
        slot[i] = -1;
        if (n[i] > 0) {
            const int column = over_t(c, n[i] - 1);
            if (column < min(held[i], c.T)) slot[i] = (long long)table[(long long)b * c.T + column] * c.t + (n[i] - 1 - column * c.t);
            ++count;
        }
    }
    int place = sum_below(count, lane);
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        const int b = lane * SPL + i;
        if (b >= c.B) break;
        cu[b] = place;
        if (n[i] > 0) {
            if (place < a.room) out[place] = slot[i];
            ++place;
        }
        if (b == c.B - 1) cu[c.B] = place;
    }
}

// Any number of new tokens: four in a row a lane, stored as 32 aligned bytes.
template <int SPL>
__global__ void __launch_bounds__(kCacheThreads) br_slot_map_kernel(const SlotArgs a)
{
    extern __shared__ Run run_mem[];
    stream_order_gate();
    const CacheArgs &c = a.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Run *run = run_mem + (size_t)warp * c.B;
    int *held_of = reinterpret_cast<int *>(run_mem + (size_t)(blockDim.x >> 5) * c.B) + (size_t)warp * c.B;
    size_t row; int part;
    if (!cache_place(c, &row, &part)) return;
    const int step = c.step ? c.step[row / (unsigned)c.G] : 0;
    int n[SPL], q[SPL], sum = 0;
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        const int b = lane * SPL + i;
        n[i] = q[i] = 0;
        if (b < c.B) {
            n[i] = c.len[row * c.B + b];
            q[i] = a.n_new[row * c.B + b];
            held_of[b] = min(max(c.n_blocks[row * c.B + b], 0), c.T);
        }
    }
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        n[i] = lane * SPL + i < c.B ? cache_tokens(n[i], step) : 0;
        q[i] = min(max(q[i], 0), n[i]);
        sum = add_to_most(sum, q[i]);
    }
    int place = sum_below(sum, lane);
    int32_t *cu = a.cu + row * (c.B + 1);
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        const int b = lane * SPL + i;
        if (b >= c.B) break;
        if (part == 0) cu[b] = place;
        run[b].shift = n[i] - q[i] - place;            // (a run that starts at 2^31 - 1 has no item below `room`)
        run[b].upto = place = add_to_most(place, q[i]);
        if (part == 0 && b == c.B - 1) cu[c.B] = place;
    }
    const int total = __shfl_sync(kFull, place, (c.B - 1) / SPL);
    __syncwarp();
    const auto table = mk_span(c.table + row * c.B * c.T, (long long)c.B * c.T);
    const auto out = mk_span(a.slots + row * a.room, a.room);
    const int count = min(total, a.room);
    // items are counted from the 32-byte boundary at or ahead of the row's first one (room is at most 2^30)
    const int skew = (int)(reinterpret_cast<uintptr_t>(a.slots + row * a.room) >> 3) & 3;
    int lo, hi;
    cache_piece(c, part, count, skew, &lo, &hi);
    int e = (lo + skew) / 128 * 128 + 4 * lane - skew;             // (lo is at a unit's start, or the row's)
    if (max(e, lo) >= hi) return;
    Walk w;
    w.seek(run, c.B, max(e, lo));
    for (; e < hi; e += 128) {
        const int first = max(e, lo);
        w.to(first);
        if (e >= lo && e + 4 <= hi && e + 4 <= w.at.upto && c.t >= 4) {
            const int p = e + w.at.shift, column = over_t(c, p), off = p - column * c.t, held = held_of[w.slot];
            const long long at = (long long)w.slot * c.T + column;
            const bool next = off + 3 >= c.t;
            const long long id0 = column < held ? table[at] : -1, id1 = next && column + 1 < held ? table[at + 1] : -1;
            const long long s0 = id0 * c.t + off, s1 = id1 * c.t + off - c.t;
            long long v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool in0 = off + j < c.t;
                v[j] = (in0 ? column : column + 1) < held ? (in0 ? s0 : s1) + j : -1;
            }
            longlong2 *o = vec_at<longlong2>(out, e);
            o[0] = make_longlong2(v[0], v[1]);
            o[1] = make_longlong2(v[2], v[3]);
        } else {
            const int last = min(e + 4, hi);
            for (int x = first; x < last; ++x) {
                w.to(x);
                const int p = x + w.at.shift, column = over_t(c, p);
                out[x] = column < held_of[w.slot]
                             ? (long long)table[(long long)w.slot * c.T + column] * c.t + (p - column * c.t) : -1;
            }
        }
    }
}

// Four pages in a row a lane, stored as 16 aligned bytes.
template <int SPL>
__global__ void __launch_bounds__(kCacheThreads) br_page_lists_kernel(const PageArgs a)
{
    extern __shared__ Run run_mem[];
    stream_order_gate();
    const CacheArgs &c = a.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Run *run = run_mem + (size_t)warp * c.B;
    size_t row; int part;
    if (!cache_place(c, &row, &part)) return;
    const int step = c.step ? c.step[row / (unsigned)c.G] : 0;
    int n[SPL], held[SPL], sum = 0, running = 0;
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        const int b = lane * SPL + i;
        n[i] = held[i] = 0;
        if (b < c.B) { n[i] = c.len[row * c.B + b]; held[i] = c.n_blocks[row * c.B + b]; }
    }
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        n[i] = lane * SPL + i < c.B ? cache_tokens(n[i], step) : 0;
        held[i] = min(max(held[i], 0), c.T);
        sum += min(cache_blocks(c, n[i]), held[i]);
        running += n[i] > 0;
    }
    int place = sum_below(sum, lane), rank = sum_below(running, lane);
    const int all = (int)__reduce_add_sync(kFull, (unsigned)sum), count = (int)__reduce_add_sync(kFull, (unsigned)running);
    const auto seq_slot = mk_span(a.seq_slot + row * c.B, c.B), last = mk_span(a.last + row * c.B, c.B);
    const auto indptr = mk_span(a.indptr + row * (c.B + 1), c.B + 1);
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        const int b = lane * SPL + i;
        if (b >= c.B) break;
        const int need = cache_blocks(c, n[i]), pages = min(need, held[i]);
        if (part == 0 && n[i] > 0) {
            seq_slot[rank] = b;
            indptr[rank] = place;
            last[rank] = pages == 0 ? 0 : need <= held[i] ? n[i] - (need - 1) * c.t : c.t;
            ++rank;
        }
        run[b].shift = -place;
        run[b].upto = place += pages;
        if (part == 0 && b >= count) { seq_slot[b] = -1; last[b] = 0; indptr[b] = all; }
    }
    if (part == 0 && lane == 0) { indptr[c.B] = all; a.n_seq[row] = count; }
    __syncwarp();
    const auto table = mk_span(c.table + row * c.B * c.T, (long long)c.B * c.T);
    const auto out = mk_span(a.indices + row * c.P, c.P);
    const int total = min(all, c.P);
    const int skew = (int)(reinterpret_cast<uintptr_t>(a.indices + row * c.P) >> 2) & 3;
    int lo, hi;
    cache_piece(c, part, total, skew, &lo, &hi);
    int e = (lo + skew) / 128 * 128 + 4 * lane - skew;
    if (max(e, lo) >= hi) return;
    Walk w;
    w.seek(run, c.B, max(e, lo));
    for (; e < hi; e += 128) {
        const int first = max(e, lo);
        w.to(first);
        if (e >= lo && e + 4 <= min(hi, w.at.upto)) {
            const long long at = (long long)w.slot * c.T + e + w.at.shift;
            *vec_at<int4>(out, e) = make_int4(table[at], table[at + 1], table[at + 2], table[at + 3]);
        } else {
            const int end = min(e + 4, hi);
            for (int x = first; x < end; ++x) {
                w.to(x);
                out[x] = table[(long long)w.slot * c.T + x + w.at.shift];
            }
        }
    }
}

}  // namespace br
