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
// A team of warps takes one worker: a single warp where there are many workers (eight of them a block), a block otherwise.  Each
// thread owns one or two slots, and one exchange of the warps' sums gives every slot its place.  What is to be moved is then cut
// into equal pieces by items, not by slots, so one long request is spread like many short ones.
//
// Large calls are bound by memory: 16 of the largest fleets' page lists (37.8 million blocks) take 53.5 us, 0.82 of the
// measured copy bandwidth, 146 million prompt tokens 201 us, 0.90.  Calls between two decode steps move next to nothing: 2.0 us
// for four workers, the launch, 6.5 us for 8,192, a tenth of which take a prompt.  (Device times of captured calls, here and below.)
#pragma once
#include <algorithm>
#include "br_device.cuh"
#include "../../include/br.h"

namespace br {

constexpr int kCacheTeams = 8;              // single-warp teams of a block
constexpr int kMoves = 8;                   // items of a lane on their way at once
// The warps of a launch that the rules below count as one round: all that 148 SMs have room for, 64 each.  Registers allow that
// in the slot kernels of whole blocks only (27 to 31 a thread); single-warp teams of slot maps (39) and page lists (40) hold 48
// warps an SM, block tables (48) 40, so that a round is up to 1.6 waves of theirs.  Counting 40 instead does not pay: 1,024 empty
// caches 67.2 us with four warps a worker, all of them resident, 61.9 with eight; page lists of 37.8 million blocks 55.0, 53.4; a
// third of the requests of 2,013 workers replaced 10.1 us with two warps, 11.0 with four, but 12.9 and 11.1 if not captured.
constexpr int kCacheWarps = 148 * 64;

// x / d = umulhi(2 x, magic) >> shift for 0 <= x < 2^31, 1 <= d <= 2^31 - 1: with s = ceil(log2 d) and
// m = ceil(2^(31 + s) / d) <= 2^32 - 1 (d no power of two) the error m d - 2^(31 + s) is below d <= 2^s, so
// floor(x m / 2^(31 + s)) = floor(x / d) for x < 2^31 (Granlund and Montgomery); a power of two has m = 2^31.
struct Divisor { uint32_t magic; int32_t shift; };

inline Divisor divisor(int d)
{
    int s = 0;
    while ((1ll << s) < d) ++s;
    return {(uint32_t)(((1ull << (31 + s)) + d - 1) / d), s};
}

__device__ __forceinline__ int over(int x, const Divisor &d) { return (int)(__umulhi(2u * (unsigned)x, d.magic) >> d.shift); }

struct CacheArgs {
    int32_t G, B, t, T, P;
    int32_t first_row, workers;             // rows first_row .. first_row + workers of the arrays by worker
    int32_t slices;                         // blocks a worker (one with single-warp teams)
    Divisor over_G, over_t, over_slices;
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

// The team of a worker, how many slots a thread of it owns (one or two), and how many blocks share the worker.
struct CacheShape { int warps, spl, slices; };

// Warps a worker for calls that move up to `items` items of it, at most `limit`: more while they stay within a round and each
// has more than 256 items, or up to four rounds of them while each has 2,048 or more, which evens out workers that move
// different amounts.  (8,192 workers with pools of 10,240 blocks: page lists 49.5 us with one warp a worker, 48.0 with two, 46.2
// with four, the rule's choice, 54.8 with eight.  Chunks of their prompts, room for 12,345 tokens: 119, 85.1, 84.7, 86.5.)
inline CacheShape cache_shape(int B, int workers, long long items, int limit)
{
    CacheShape s = {1, 1, 1};
    while (s.warps * 64 < B) s.warps *= 2;
    const auto worth = [&](long long warps) {
        return (warps * workers <= kCacheWarps && items > 256 * warps) || (warps * workers <= 4 * kCacheWarps && items >= 2048 * warps);
    };
    while (s.warps < limit && worth(2 * s.warps)) s.warps *= 2;
    s.spl = 32 * s.warps >= B ? 1 : 2;
    return s;
}

// ... and blocks a worker, by the same rule with pieces of 256 and of 2,048 items a warp, for calls that only copy: 146 million
// prompt tokens of 256 workers 396 us with one block of eight warps each, 216 with 8, 201 with 18, the rule's choice; chunks of 264
// workers 9.7 with one, 8.2 with four, the rule's choice, 9.8 with 8.
inline CacheShape cache_copy_shape(int B, int workers, int items)
{
    CacheShape s = cache_shape(B, workers, items, 8);
    if (s.warps > 1) {
        const long long warps = (long long)workers * s.warps;
        const long long fill = std::min(kCacheWarps / warps, (long long)items / (256 * s.warps));
        const long long even = std::min(4 * kCacheWarps / warps, (long long)items / (2048 * s.warps));
        s.slices = (int)std::max(1ll, std::max(fill, even));
    }
    return s;
}

// a + b, at most 2^31 - 1 and at least -2^31
__device__ __forceinline__ int add_to_most(int a, int b)
{
    int s;
    asm("add.sat.s32 %0, %1, %2;" : "=r"(s) : "r"(a), "r"(b));
    return s;
}

// tokens of the request in a slot: len + step, at least 0 and at most 2^31 - 1; 0 for a free slot
__device__ __forceinline__ int cache_tokens(int len, int step) { return len == BR_EMPTY_SLOT ? 0 : max(add_to_most(len, step), 0); }

__device__ __forceinline__ int cache_blocks(const CacheArgs &c, int tokens) { return tokens > 0 ? over(tokens - 1, c.over_t) + 1 : 0; }

// One thread's place: its team's worker, its first slot, and the piece of the worker's items that its warp moves.
template <bool ONE, int SPL>
struct Seat {
    int lane, warp, slot, piece, pieces;
    size_t row;
    bool any;                               // false behind the last worker
    __device__ __forceinline__ explicit Seat(const CacheArgs &c)
    {
        lane = threadIdx.x & 31; warp = threadIdx.x >> 5;
        unsigned worker;
        if (ONE) {
            worker = blockIdx.x * kCacheTeams + warp;
            slot = lane * SPL; piece = 0; pieces = 1;
            any = worker < (unsigned)c.workers;
        } else {
            worker = c.slices == 1 ? blockIdx.x : (unsigned)over((int)blockIdx.x, c.over_slices);
            slot = threadIdx.x * SPL;
            piece = (int)(blockIdx.x - worker * c.slices) * (int)(blockDim.x >> 5) + warp;
            pieces = c.slices * (int)(blockDim.x >> 5);
            any = true;
        }
        row = (size_t)c.first_row + worker;
    }
    __device__ __forceinline__ bool first_block() const { return ONE || piece < (int)(blockDim.x >> 5); }   // of its worker's
    __device__ __forceinline__ int step(const CacheArgs &c) const { return c.step ? c.step[over((int)row, c.over_G)] : 0; }
};

template <bool ONE> __device__ __forceinline__ void team_sync() { if (ONE) __syncwarp(); else __syncthreads(); }

// Sums over the threads of the team below this one, and over all of them, of x (at most 2^31 - 1 each) and y; the sum of z; and
// of w, a warp's own, the sums over the warps below and over all.
struct TeamSums { int x, y, x_all, y_all, z_all, w, w_all; };

// sum over the lanes below; *all: over the warp
__device__ __forceinline__ int lanes_below(int v, int lane, int *all)
{
    int in = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
        // (the shuffle's predicate says whether the lane o below is there)
        asm volatile("{ .reg .pred p; .reg .b32 u; shfl.sync.up.b32 u|p, %0, %1, 0, 0xffffffff; @p add.sat.s32 %0, %0, u; }" : "+r"(in) : "r"(o));
    *all = __shfl_sync(kFull, in, 31);
    const int below = __shfl_up_sync(kFull, in, 1);
    return lane ? below : 0;
}

// MOST: sums of x may pass 2^31 - 1.
template <bool ONE, bool MOST>
__device__ __forceinline__ TeamSums team_sums(int x, int y, int z, int w, int4 *part, int lane, int warp)
{
    TeamSums s = {0, 0, 0, 0, 0, 0, w};
    if (__any_sync(kFull, x != 0)) s.x = lanes_below(x, lane, &s.x_all);
    if (__any_sync(kFull, y != 0)) s.y = lanes_below(y, lane, &s.y_all);
    s.z_all = (int)__reduce_add_sync(kFull, (unsigned)z);
    if (ONE) return s;
    if (lane == 0) part[warp] = make_int4(s.x_all, s.y_all, s.z_all, w);
    __syncthreads();
    // (at most eight warps; lane l takes the sums of warp l)
    const int4 p = lane < (int)(blockDim.x >> 5) ? part[lane] : make_int4(0, 0, 0, 0);
    const bool below = lane < warp;
    if (MOST) {                             // (the high and the low half apart, then at most 2^31 - 1)
        const unsigned hi = __reduce_add_sync(kFull, (unsigned)p.x >> 16), lo = __reduce_add_sync(kFull, p.x & 0xFFFFu);
        const unsigned hb = __reduce_add_sync(kFull, below ? (unsigned)p.x >> 16 : 0u), lb = __reduce_add_sync(kFull, below ? p.x & 0xFFFFu : 0u);
        s.x_all = (int)min(((unsigned long long)hi << 16) + lo, 0x7FFFFFFFull);
        s.x = add_to_most(s.x, (int)min(((unsigned long long)hb << 16) + lb, 0x7FFFFFFFull));
    } else {
        s.x_all = (int)__reduce_add_sync(kFull, (unsigned)p.x);
        s.x += (int)__reduce_add_sync(kFull, below ? (unsigned)p.x : 0u);
    }
    s.y_all = (int)__reduce_add_sync(kFull, (unsigned)p.y);
    s.y += (int)__reduce_add_sync(kFull, below ? (unsigned)p.y : 0u);
    s.z_all = (int)__reduce_add_sync(kFull, (unsigned)p.z);
    s.w_all = (int)__reduce_add_sync(kFull, (unsigned)p.w);
    s.w = (int)__reduce_add_sync(kFull, below ? (unsigned)p.w : 0u);
    return s;
}

// A slot's run of items in the sequence of all items of its worker: item e of the run, e < upto, is entry e + shift of the
// worker's table (at most 256 rows of 2^22: the sum fits 32 bits).
struct Run { int upto, shift; };
// ... or token e + shift of the slot whose row is at `base` and holds `held` blocks
struct alignas(16) TokenRun { int upto, shift, base, held; };

// Position in a worker's runs.
template <typename RunT>
struct Walk {
    const RunT *runs;
    int last, here;
    RunT at;
    // the run of item e: the first that ends behind it (e lies in one of them)
    __device__ __forceinline__ void seek(const RunT *r, int count, int e)
    {
        runs = r; last = count - 1;
        int lo = 0, hi = last;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (runs[mid].upto > e) hi = mid; else lo = mid + 1;
        }
        here = lo; at = runs[lo];
    }
    // on to item e, not before the present one
    __device__ __forceinline__ void to(int e)
    {
        while (at.upto <= e && here < last) at = runs[++here];
    }
};

// A list whose entry -x is out[x].
template <typename Out> struct UpList {
    Out out;
    __device__ __forceinline__ auto &operator[](int i) const { return out[-i]; }
};

// The runs of the items of one warp, window by window of kMoves rows of 32.  Where one run covers a window, the rule for long
// requests, its items are a constant apart; up to three starts are compared with every item; with more of them a bit for each
// item that starts a run turns into the run of every item by counting bits, which has no loop that lanes leave one by one.  No
// run is empty.  (Lanes that walk through the runs one by one: page lists of 2,107 workers with runs of 33 blocks 29.5 us, 24.7
// this way; windows of 128 items, four loads a lane: 29.5, and filling 1,024 caches 79.4 us, 61.9 with 256.)
struct Windows {
    const Run *runs;
    int n, run;                             // run: that of the window's first item
    __device__ __forceinline__ void seek(const Run *r, int count, int e, int lane)
    {
        runs = r; n = count; run = 0;
        for (int k = 0; k < n; k += 32) run += __popc(__ballot_sync(kFull, k + lane < n && runs[k + lane].upto <= e));
    }
    // shift[u] of item e0 + 32 u + lane; on to the next window.  True if one run covers the window.
    __device__ __forceinline__ bool next(int e0, int lane, int (&shift)[kMoves])
    {
        int d = run + lane < n - 1 ? runs[run + lane].upto - e0 : 1 << 30;      // run + lane + 1 starts d items into the window
        unsigned in = __ballot_sync(kFull, d <= 32 * kMoves);
        const int only = runs[run].shift;
#pragma unroll
        for (int u = 0; u < kMoves; ++u) shift[u] = only;
        if (in == 0) return true;
        int count = __popc(in);
        if (count <= 3) {                   // (counting bits costs as much as four runs one by one)
            for (int k = 0; k < count; ++k) {
                const int from = __shfl_sync(kFull, d, k) - lane, then = runs[++run].shift;
#pragma unroll
                for (int u = 0; u < kMoves; ++u) shift[u] = 32 * u >= from ? then : shift[u];
            }
            return false;
        }
        unsigned starts[kMoves];
#pragma unroll
        for (int u = 0; u < kMoves; ++u) starts[u] = 0;
        for (int k = run + lane;;) {
#pragma unroll
            for (int u = 0; u < kMoves; ++u) starts[u] |= __reduce_or_sync(kFull, (d >> 5) == u ? 1u << (d & 31) : 0u);
            if (in != kFull) break;
            k += 32;
            d = k < n - 1 ? runs[k].upto - e0 : 1 << 30;
            in = __ballot_sync(kFull, d <= 32 * kMoves);
            count += __popc(in);
        }
        int r = run;
#pragma unroll
        for (int u = 0; u < kMoves; ++u) {
            shift[u] = runs[r + __popc(starts[u] & (0xFFFFFFFFu >> (31 - lane)))].shift;
            r += __popc(starts[u]);
        }
        run += count;
        return false;
    }
};

// An entry with few others of interest near it: 64 bytes of memory are fetched for it, not the usual 128 (newest tokens of
// 32,768 workers' requests: 43.1 us with plain loads, 29.1 this way; 259 MB read from DRAM, 138).
__device__ __forceinline__ int lone_entry(const int32_t *p)
{
    int v;
    asm volatile("ld.global.L2::64B.b32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

// Moves items [lo, hi) of a warp, kMoves of a lane at a time: item x is entry x + shift of its run in `table`, or entry top - x
// of `list`.
template <bool FROM_TABLE, bool TO_TABLE, typename Table, typename List>
__device__ __forceinline__ void move_items(const Run *from_runs, int n_from, const Run *to_runs, int n_to, int lo, int hi, int lane,
                                           const Table &table, const List &list, int top)
{
    if (lo >= hi) return;
    Windows from, to;
    if (FROM_TABLE) from.seek(from_runs, n_from, lo, lane);
    if (TO_TABLE) to.seek(to_runs, n_to, lo, lane);
    for (int e0 = lo; e0 < hi; e0 += 32 * kMoves) {
        const int e = e0 + lane;
        const bool full = e0 + 32 * kMoves <= hi;
        int id[kMoves], shift[kMoves];
        const bool one = FROM_TABLE ? from.next(e0, lane, shift) : true;
        if (full && one) {
            const int entry = FROM_TABLE ? e + shift[0] : top - e;
#pragma unroll
            for (int u = 0; u < kMoves; ++u) id[u] = FROM_TABLE ? table[entry + 32 * u] : list[entry - 32 * u];
        } else {
#pragma unroll
            for (int u = 0; u < kMoves; ++u)
                if (e + 32 * u < hi) id[u] = FROM_TABLE ? lone_entry(&table[e + 32 * u + shift[u]]) : list[top - e - 32 * u];
        }
        const bool one_to = TO_TABLE ? to.next(e0, lane, shift) : true;
        if (full && one_to) {
            const int entry = TO_TABLE ? e + shift[0] : top - e;
#pragma unroll
            for (int u = 0; u < kMoves; ++u) (TO_TABLE ? table[entry + 32 * u] : list[entry - 32 * u]) = id[u];
        } else {
#pragma unroll
            for (int u = 0; u < kMoves; ++u)
                if (e + 32 * u < hi) (TO_TABLE ? table[e + 32 * u + shift[u]] : list[top - e - 32 * u]) = id[u];
        }
    }
}

// Items [lo, hi) of `count` for one of `pieces`: equal numbers of units, counted from `skew` items ahead of the first.
__device__ __forceinline__ void cache_piece(int piece, int pieces, int count, int skew, int unit, int *lo, int *hi)
{
    if (pieces == 1) { *lo = 0; *hi = count; return; }
    const int units = (count + skew + unit - 1) / unit, each = (units + pieces - 1) / pieces;
    *lo = max(0, (int)min((long long)count, (long long)each * piece * unit - skew));
    *hi = (int)min((long long)count, (long long)each * (piece + 1) * unit - skew);
}

// Block a of the growth (in slot and table order) is block a of those taken back (same order) while there are any, then the
// free list from its end; the rest of those taken back joins the free list, the first on top.  What is read (the tails of
// rows that shrink, the list below n_free) is never written by the same call, so the moves need no order.  The counts may be
// written where they are read: a slot's by the thread that read it, the worker's after the whole team has read them.
// 1,024 empty caches take 37.8 million blocks in 61.9 us, 0.70 of the measured copy bandwidth.  48 registers a thread leave 40
// warps an SM, with eight loads a lane in flight: the launch of 1,024 blocks is a full wave of 740 and a partial second one.
// (40 registers spill, 66.8 us; four loads a lane 79.4.)  A burst that replaces a third of the requests of 2,013 workers takes 11.0 us,
// in 1.36 waves, by instructions (0.6 of the issue slots) and two trips to memory.  A decode step of 8,192 workers takes 6.5 us, in
// 1.38 waves: 3.6 where nothing moves, 4.5 with a block a request at most.
template <bool ONE, int SPL>
__global__ void __launch_bounds__(256, 5) br_block_tables_kernel(const TableArgs a)
{
    constexpr int kSlots = ONE ? 32 * SPL : BR_MAX_B;
    __shared__ Run runs[ONE ? kCacheTeams : 1][2][kSlots];
    __shared__ int4 part[ONE ? 1 : 8];
    __shared__ int granted[ONE ? 1 : 8];
    __shared__ long long wanted[ONE ? 1 : 8];
    stream_order_gate();
    const CacheArgs &c = a.c;
    const Seat<ONE, SPL> at(c);
    if (!at.any) return;
    const size_t row = at.row, slots = row * c.B;
    const int step = at.step(c), n_free = c.n_free[row];
    int need[SPL], have[SPL], held = 0, back = 0, ask = 0;
    int flags = 0;                          // some slot's count is out of range, its request is too long, it grows by several blocks
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        need[i] = BR_EMPTY_SLOT; have[i] = 0;
        if (at.slot + i < c.B) { need[i] = c.len[slots + at.slot + i]; have[i] = c.n_blocks[slots + at.slot + i]; }
    }
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        need[i] = cache_blocks(c, cache_tokens(need[i], step));
        const bool in_range = (unsigned)have[i] <= (unsigned)c.T, fits_row = need[i] <= c.T;
        const int more = in_range ? need[i] - have[i] : 0;
        flags |= (in_range ? 0 : 1 << 20) | (fits_row ? 0 : 1 << 24) | (more > 1 ? 1 << 28 : 0);
        held += in_range ? have[i] : 0;
        back += max(-more, 0);
        ask += fits_row ? max(more, 0) : 0;
    }
    flags = (int)__reduce_or_sync(kFull, (unsigned)flags);
    // the slots that give blocks back, and those that ask for some, are counted: their runs are packed
    int back_rank = 0, grow_rank = 0, n_back = 0, n_grow = 0;
    const auto rank = [&] {
        const unsigned below = (1u << at.lane) - 1;
#pragma unroll
        for (int i = 0; i < SPL; ++i) {
            const unsigned backs = __ballot_sync(kFull, have[i] > need[i]), grows = __ballot_sync(kFull, need[i] > have[i] && need[i] <= c.T);
            back_rank += __popc(backs & below); grow_rank += __popc(grows & below);
            n_back += __popc(backs); n_grow += __popc(grows);
        }
    };
    if (!ONE) rank();
    // (with counts in range all sums stay below 2^30; counts and flags take ten and four bits, from eight warps)
    TeamSums sum = team_sums<ONE, false>(back, ask, held, n_back + (n_grow << 10) + flags, part, at.lane, at.warp);
    if (!ONE) { n_back = sum.w_all & 1023; n_grow = sum.w_all >> 10 & 1023; }
    const bool bad = (sum.w_all & 15 << 20) != 0 || (unsigned)n_free > (unsigned)c.P || n_free + sum.z_all > c.P;
    const bool too_long = (sum.w_all & 15 << 24) != 0, several = ((unsigned)sum.w_all >> 28) != 0;
    if (bad) {                              // counts that no sequence of updates leaves behind: the worker stays as it is
#pragma unroll
        for (int i = 0; i < SPL; ++i)
            if (at.slot + i < c.B) a.n_blocks_out[slots + at.slot + i] = have[i];
        if (at.slot == 0) {
            a.n_free_out[row] = n_free;
            if (a.short_out) a.short_out[row] = -1;
        }
        return;
    }
    const int R = sum.x_all;
    const auto table = mk_span(c.table + slots * c.T, (long long)c.B * c.T);
    const auto list = mk_span(c.free_list + row * c.P, c.P);
    const bool all_fit = !too_long && sum.y_all <= n_free + R;
    // between two decode steps most workers only grow, by a block a request at most, and all of it fits: each thread serves
    // its own slots (four workers 3.05 us by the way below, 2.0 by this one)
    if (R == 0 && all_fit && !several) {
        int id[SPL];
#pragma unroll
        for (int i = 0; i < SPL; ++i) id[i] = need[i] > have[i] ? list[n_free - 1 - sum.y++] : -1;
#pragma unroll
        for (int i = 0; i < SPL; ++i) {
            if (at.slot + i >= c.B) break;
            if (need[i] > have[i]) table[(at.slot + i) * c.T + have[i]] = id[i];
            a.n_blocks_out[slots + at.slot + i] = need[i];
        }
        if (ONE) __syncwarp();              // (every lane has read n_free, which may be n_free_out)
        if (at.slot == 0) {
            a.n_free_out[row] = n_free - sum.y_all;
            if (a.short_out) a.short_out[row] = 0;
        }
        return;
    }
    Run *back_run = runs[ONE ? at.warp : 0][0], *grow_run = runs[ONE ? at.warp : 0][1];
    if (ONE) rank(); else { back_rank += sum.w & 1023; grow_rank += sum.w >> 10 & 1023; }
    int A = 0;
    long long want = 0;
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        if (at.slot + i >= c.B) break;
        const int less = max(have[i] - need[i], 0), more = max(need[i] - have[i], 0);
        if (less > 0) back_run[back_rank++] = {sum.x + less, (at.slot + i) * c.T + need[i] - sum.x};
        sum.x += less;
        // a sum over all demands up to this one: the first that does not fit keeps out the ones behind it
        const bool fits_row = need[i] <= c.T;
        const int upto = sum.y + (fits_row ? more : 0);
        const bool served = fits_row && upto <= n_free + R;
        // (the runs of requests that are not served lie behind A, the end of what is moved)
        if (more > 0 && fits_row) grow_run[grow_rank++] = {upto, (at.slot + i) * c.T + have[i] - sum.y};
        sum.y = upto;
        if (served) A = upto;
        want += more;
        a.n_blocks_out[slots + at.slot + i] = have[i] + (served ? more : 0) - less;
    }
    if (all_fit) {
        A = sum.y_all; want = A;
        team_sync<ONE>();
    } else {
        A = (int)__reduce_max_sync(kFull, (unsigned)A);
        for (int o = 16; o > 0; o >>= 1) want += __shfl_xor_sync(kFull, want, o);
        if (!ONE && at.lane == 0) { granted[at.warp] = A; wanted[at.warp] = want; }
        team_sync<ONE>();
        if (!ONE) {
            want = 0;
            for (int w = 0; w < (int)(blockDim.x >> 5); ++w) { A = max(A, granted[w]); want += wanted[w]; }
        }
    }
    if (at.slot == 0) {
        a.n_free_out[row] = n_free + R - A;
        if (a.short_out) a.short_out[row] = (int)min(want - A, 0x7FFFFFFFll);
    }
    int lo, hi;
    cache_piece(at.piece, at.pieces, max(R, A), 0, 32 * kMoves, &lo, &hi);
    const int both = min(R, A), top = n_free + R - 1;
    move_items<true, true>(back_run, n_back, grow_run, n_grow, lo, min(hi, both), at.lane, table, list, top);
    lo = max(lo, both);
    if (R < A) move_items<false, true>(back_run, 0, grow_run, n_grow, lo, hi, at.lane, table, list, top);
    else move_items<true, false>(back_run, n_back, grow_run, 0, lo, hi, at.lane, table, list, top);
}

// One new token a request: a thread reads the entry of each of its slots, its place is the number of running requests ahead.
// Bound by memory, where an entry costs 64 bytes: 32,768 workers of 58 requests 29.1 us, 154 MB of DRAM at 0.82 of the measured copy
// bandwidth; by the launch for single fleets, 2.1 us.
template <bool ONE, int SPL>
__global__ void __launch_bounds__(256) br_slot_newest_kernel(const SlotArgs a)
{
    __shared__ int4 part[ONE ? 1 : 8];
    stream_order_gate();
    const CacheArgs &c = a.c;
    const Seat<ONE, SPL> at(c);
    if (!at.any) return;
    const size_t row = at.row, slots = row * c.B;
    const int step = at.step(c);
    int n[SPL], held[SPL], count = 0;
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        n[i] = BR_EMPTY_SLOT; held[i] = 0;
        if (at.slot + i < c.B) { n[i] = c.len[slots + at.slot + i]; held[i] = c.n_blocks[slots + at.slot + i]; }
    }
    const auto table = mk_span(c.table + slots * c.T, (long long)c.B * c.T);
    const auto out = mk_span(a.slots + row * a.room, a.room);
    const auto cu = mk_span(a.cu + row * (c.B + 1), c.B + 1);
    long long slot[SPL];
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        n[i] = cache_tokens(n[i], step);
        slot[i] = -1;
        if (n[i] > 0) {
            const int column = over(n[i] - 1, c.over_t);
            if (column < min(held[i], c.T))
                slot[i] = (long long)lone_entry(&table[(at.slot + i) * c.T + column]) * c.t + (n[i] - 1 - column * c.t);
            ++count;
        }
    }
    const TeamSums sum = team_sums<ONE, false>(count, 0, 0, 0, part, at.lane, at.warp);
    int place = sum.x;
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        const int b = at.slot + i;
        if (b >= c.B) break;
        cu[b] = place;
        if (n[i] > 0) {
            if (place < a.room) out[place] = slot[i];
            ++place;
        }
        if (b == c.B - 1) cu[c.B] = place;
    }
}

struct alignas(32) FourSlots { long long v[4]; };

// 32 bytes in one store, so that every sector is written whole and once (two of 16 bytes wrote each sector twice, 294 us for 146
// million tokens; 219 this way, both with fewer blocks a worker than now)
__device__ __forceinline__ void store_four(FourSlots *p, const FourSlots &s)
{
#ifdef BR_BOUNDS
    for (int j = 0; j < 4; ++j) p->v[j] = s.v[j];                  // (the sink of an index out of range is not that aligned)
#else
    asm volatile("st.global.v4.b64 [%0], {%1, %2, %3, %4};" :: "l"(p), "l"(s.v[0]), "l"(s.v[1]), "l"(s.v[2]), "l"(s.v[3]) : "memory");
#endif
}

// Any number of new tokens: four in a row a lane, which take one division and one or two entries, stored as 32 aligned bytes.
// Bound by memory: 146 million prompt tokens 201 us, 1.17 GB at 0.90 of the measured copy bandwidth.  (Two groups of a lane at
// once, warps that take the groups of a block in turn, and streaming stores all stay within 1 % of that.)  Chunks of 264 workers
// 8.2 us, by instructions: a warp moves two groups of 128 tokens, one or two table entries a lane each, after a prologue that every
// block of the worker repeats (469 instructions a warp in all, 0.59 of the issue slots).
template <bool ONE, int SPL>
__global__ void __launch_bounds__(256) br_slot_map_kernel(const SlotArgs a)
{
    constexpr int kSlots = ONE ? 32 * SPL : BR_MAX_B;
    __shared__ TokenRun runs[ONE ? kCacheTeams : 1][kSlots];
    __shared__ int4 part[ONE ? 1 : 8];
    stream_order_gate();
    const CacheArgs &c = a.c;
    const Seat<ONE, SPL> at(c);
    if (!at.any) return;
    TokenRun *run = runs[ONE ? at.warp : 0];
    const size_t row = at.row, slots = row * c.B;
    const int step = at.step(c);
    int n[SPL], q[SPL], held[SPL], mine = 0, some = 0;
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        n[i] = BR_EMPTY_SLOT; q[i] = held[i] = 0;
        if (at.slot + i < c.B) {
            n[i] = c.len[slots + at.slot + i];
            q[i] = a.n_new[slots + at.slot + i];
            held[i] = c.n_blocks[slots + at.slot + i];
        }
    }
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        n[i] = cache_tokens(n[i], step);
        q[i] = min(max(q[i], 0), n[i]);
        mine = add_to_most(mine, q[i]);
        some += q[i] > 0;
    }
    const TeamSums sum = team_sums<ONE, true>(mine, some, 0, 0, part, at.lane, at.warp);
    const auto cu = mk_span(a.cu + row * (c.B + 1), c.B + 1);
    const bool first_block = at.first_block();
    int place = sum.x, rank = sum.y;
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        const int b = at.slot + i;
        if (b >= c.B) break;
        const int from = place;
        place = add_to_most(place, q[i]);
        // (a run that starts at 2^31 - 1 has no item below `room`)
        if (q[i] > 0) run[rank++] = {place, n[i] - q[i] - from, b * c.T, min(max(held[i], 0), c.T)};
        if (first_block) {
            cu[b] = from;
            if (b == c.B - 1) cu[c.B] = place;
        }
    }
    team_sync<ONE>();
    const auto table = mk_span(c.table + slots * c.T, (long long)c.B * c.T);
    const auto out = mk_span(a.slots + row * a.room, a.room);
    const int count = min(sum.x_all, a.room);
    // items are counted from the 32-byte boundary at or ahead of the row's first one (room is at most 2^30)
    const int skew = (int)(reinterpret_cast<uintptr_t>(a.slots + row * a.room) >> 3) & 3;
    int lo, hi;
    cache_piece(at.piece, at.pieces, count, skew, 128, &lo, &hi);
    int e = (lo + skew) / 128 * 128 - skew + 4 * at.lane;     // (lo is at a unit's start, or the row's)
    if (max(e, lo) >= hi) return;
    Walk<TokenRun> w;
    w.seek(run, sum.y_all, max(e, lo));
    for (; e < hi; e += 128) {
        w.to(max(e, lo));
        const int p = e + w.at.shift, column = over(max(p, 0), c.over_t), offset = p - column * c.t;
        const bool next = offset + 3 >= c.t;
        if (e >= lo && e + 4 <= min(hi, w.at.upto) && c.t >= 4 && column + next < w.at.held) {
            // four tokens of one request, in one block or two
            const int entry = w.at.base + column, id0 = table[entry], id1 = next ? table[entry + 1] : 0;
            const long long s0 = (long long)id0 * c.t + offset, s1 = (long long)id1 * c.t + (offset - c.t);
            FourSlots v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v.v[j] = (offset + j < c.t ? s0 : s1) + j;
            store_four(vec_at<FourSlots>(out, e), v);
        } else {
            int id[4], off[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                id[j] = off[j] = -1;
                if (e + j < lo || e + j >= hi) continue;
                w.to(e + j);
                const int pj = e + j + w.at.shift, cj = over(pj, c.over_t);
                if (cj < w.at.held) { off[j] = pj - cj * c.t; id[j] = lone_entry(&table[w.at.base + cj]); }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (e + j >= lo && e + j < hi) out[e + j] = off[j] < 0 ? -1 : (long long)id[j] * c.t + off[j];
        }
    }
}

// The running slots move up, their blocks follow one another: item x of the worker is entry x of its list, and rows of 32 items are
// read and written a line at a time.  Bound by memory for long requests, 37.8 million blocks 53.5 us at 0.82 of the measured copy
// bandwidth, and by instructions for short ones, 2,107 workers with runs of 33 blocks 24.7 us in 1.19 waves (40 registers, 48 warps an
// SM; 248 slots need four warps, and eight take 25.0).  (A lane that takes four blocks in a
// row: 60 us and 26.6; a run at a time: 90 and 48.)
template <bool ONE, int SPL>
__global__ void __launch_bounds__(256, 6) br_page_lists_kernel(const PageArgs a)
{
    constexpr int kSlots = ONE ? 32 * SPL : BR_MAX_B;
    __shared__ Run runs[ONE ? kCacheTeams : 1][kSlots];
    __shared__ int4 part[ONE ? 1 : 8];
    stream_order_gate();
    const CacheArgs &c = a.c;
    const Seat<ONE, SPL> at(c);
    if (!at.any) return;
    Run *run = runs[ONE ? at.warp : 0];
    const size_t row = at.row, slots = row * c.B;
    const int step = at.step(c);
    int n[SPL], held[SPL], mine = 0, counts = 0;             // counts: running requests, and those with blocks 16 bits up
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        n[i] = BR_EMPTY_SLOT; held[i] = 0;
        if (at.slot + i < c.B) { n[i] = c.len[slots + at.slot + i]; held[i] = c.n_blocks[slots + at.slot + i]; }
    }
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        n[i] = cache_tokens(n[i], step);
        held[i] = min(max(held[i], 0), c.T);
        const int pages = min(cache_blocks(c, n[i]), held[i]);
        mine += pages;
        counts += (n[i] > 0) + ((pages > 0) << 16);
    }
    const TeamSums sum = team_sums<ONE, false>(mine, counts, 0, 0, part, at.lane, at.warp);
    const auto seq_slot = mk_span(a.seq_slot + slots, c.B), last = mk_span(a.last + slots, c.B);
    const auto indptr = mk_span(a.indptr + row * (c.B + 1), c.B + 1);
    const bool first_block = at.first_block();
    const int n_seq = sum.y_all & 0xFFFF, runs_all = sum.y_all >> 16;
    int place = sum.x, rank = sum.y & 0xFFFF, run_rank = sum.y >> 16;
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        const int b = at.slot + i;
        if (b >= c.B) break;
        const int need = cache_blocks(c, n[i]), pages = min(need, held[i]);
        if (first_block && n[i] > 0) {
            seq_slot[rank] = b;
            indptr[rank] = place;
            last[rank] = pages == 0 ? 0 : need <= held[i] ? n[i] - (need - 1) * c.t : c.t;
            ++rank;
        }
        if (pages > 0) run[run_rank++] = {place + pages, b * c.T - place};
        place += pages;
        if (first_block && b >= n_seq) { seq_slot[b] = -1; last[b] = 0; indptr[b] = sum.x_all; }
    }
    if (first_block && at.slot == 0) { indptr[c.B] = sum.x_all; a.n_seq[row] = n_seq; }
    team_sync<ONE>();
    const auto table = mk_span(c.table + slots * c.T, (long long)c.B * c.T);
    const auto out = mk_span(a.indices + row * c.P, c.P);
    int lo, hi;
    cache_piece(at.piece, at.pieces, min(sum.x_all, c.P), 0, 32 * kMoves, &lo, &hi);
    // (indices are a list that runs upwards: entry x of it is item x)
    move_items<true, false>(run, runs_all, run, 0, lo, hi, at.lane, table, UpList<decltype(out)>{out}, 0);
}

}  // namespace br
