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
// A team of warps takes one worker: a single warp where there are workers enough to fill the GPU (eight of them a block), a
// block otherwise.  Each thread owns one or two slots, and one exchange of the warps' sums gives every slot its place.  What
// is to be moved is then cut into equal pieces by items, not by slots, so one long request is spread like many short ones.
#pragma once
#include "br_device.cuh"
#include "../../include/br.h"

namespace br {

constexpr int kCacheTeams = 8;              // single-warp teams of a block
constexpr int kMoves = 8;                   // items of a lane on their way at once
constexpr int kCacheWarps = 148 * 64;       // the warps that the GPU holds at once

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

// The team of a worker, and how many slots a thread of it owns (one or two).
struct CacheShape { int warps, spl, slices; };

// pieces: the pieces that what a worker moves may be cut into at most; limit: warps a block at most
inline CacheShape cache_shape(int B, int workers, int pieces, int limit)
{
    CacheShape s = {1, 1, 1};
    while (s.warps * 64 < B) s.warps *= 2;
    while (s.warps < limit && s.warps < pieces && 2ll * s.warps * workers <= kCacheWarps) s.warps *= 2;
    s.spl = 32 * s.warps >= B ? 1 : 2;
    return s;
}

// a team for copies of up to `items` items a worker, in pieces of 512 or more; more than one block a worker where workers are few
inline CacheShape cache_copy_shape(int B, int workers, int items)
{
    const int pieces = (items + 511) / 512;
    CacheShape s = cache_shape(B, workers, pieces, 8);
    if (s.warps > 1) {
        const long long fill = 2ll * kCacheWarps / ((long long)workers * s.warps), cut = pieces / s.warps;
        s.slices = (int)(fill < cut ? fill : cut);
        if (s.slices < 1) s.slices = 1;
    }
    return s;
}

// tokens of the request in a slot: len + step, at least 0 and at most 2^31 - 1; 0 for a free slot
__device__ __forceinline__ int cache_tokens(int len, int step)
{
    if (len == BR_EMPTY_SLOT) return 0;
    const long long n = (long long)len + step;
    return n < 0 ? 0 : n > 0x7FFFFFFF ? 0x7FFFFFFF : (int)n;
}

__device__ __forceinline__ int cache_blocks(const CacheArgs &c, int tokens) { return tokens > 0 ? over(tokens - 1, c.over_t) + 1 : 0; }

// a + b for 0 <= a, b < 2^31, at most 2^31 - 1
__device__ __forceinline__ int add_to_most(int a, int b) { return (int)min((unsigned)a + (unsigned)b, 0x7FFFFFFFu); }

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
    __device__ __forceinline__ int step(const CacheArgs &c) const { return c.step ? c.step[over((int)row, c.over_G)] : 0; }
};

template <bool ONE> __device__ __forceinline__ void team_sync() { if (ONE) __syncwarp(); else __syncthreads(); }

// Sums over the threads of the team below this one, and over all: of x (at most 2^31 - 1 each) and y, and the sum of z.
struct TeamSums { int x, y, x_all, y_all, z_all; };

__device__ __forceinline__ int lanes_below(int v, int lane)
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

template <bool ONE>
__device__ __forceinline__ TeamSums team_sums(int x, int y, int z, int4 *part, int lane, int warp)
{
    TeamSums s;
    s.x = lanes_below(x, lane); s.y = lanes_below(y, lane);
    s.x_all = __shfl_sync(kFull, add_to_most(s.x, x), 31); s.y_all = __shfl_sync(kFull, s.y + y, 31);
    s.z_all = (int)__reduce_add_sync(kFull, (unsigned)z);
    if (ONE) return s;
    if (lane == 0) part[warp] = make_int4(s.x_all, s.y_all, s.z_all, 0);
    __syncthreads();
    // (slots end with the eighth warp: 256 of them, one a thread)
    s.x_all = s.y_all = s.z_all = 0;
    const int warps = min((int)(blockDim.x >> 5), 8);
    int xb = 0, yb = 0;
    for (int w = 0; w < warps; ++w) {
        const int4 p = part[w];
        if (w == warp) { xb = s.x_all; yb = s.y_all; }
        s.x_all = add_to_most(s.x_all, p.x); s.y_all += p.y; s.z_all += p.z;
    }
    s.x = add_to_most(s.x, xb); s.y += yb;
    return s;
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

// Items [lo, hi) of `count` for one of `pieces`: equal numbers of units of 128, counted from `skew` items ahead of the first.
__device__ __forceinline__ void cache_piece(int piece, int pieces, int count, int skew, int *lo, int *hi)
{
    if (pieces == 1) { *lo = 0; *hi = count; return; }
    const int units = (count + skew + 127) / 128, each = (units + pieces - 1) / pieces;
    *lo = max(0, (int)min((long long)count, (long long)each * piece * 128 - skew));
    *hi = (int)min((long long)count, (long long)each * (piece + 1) * 128 - skew);
}

// Block a of the growth (in slot and table order) is block a of those taken back (same order) while there are any, then the
// free list from its end; the rest of those taken back joins the free list, the first on top.  What is read (the tails of
// rows that shrink, the list below n_free) is never written by the same call, so the moves need no order.  The counts may be
// written where they are read: a slot's by the thread that read it, the worker's after the whole team has read them.
template <bool ONE, int SPL>
__global__ void __launch_bounds__(ONE ? 32 * kCacheTeams : 1024) br_block_tables_kernel(const TableArgs a)
{
    constexpr int kSlots = ONE ? 32 * SPL : BR_MAX_B;
    __shared__ Run runs[ONE ? kCacheTeams : 1][2][kSlots];
    __shared__ int4 part[ONE ? 1 : 32];
    __shared__ int granted[ONE ? 1 : 8];
    __shared__ long long lacks[ONE ? 1 : 8];
    stream_order_gate();
    const CacheArgs &c = a.c;
    const Seat<ONE, SPL> at(c);
    if (!at.any) return;
    Run *back_run = runs[ONE ? at.warp : 0][0], *grow_run = runs[ONE ? at.warp : 0][1];
    const size_t row = at.row, slots = row * c.B;
    const int step = at.step(c), n_free = c.n_free[row];
    int need[SPL], have[SPL], held = 0, back = 0, ask = 0;
    bool bad = (unsigned)n_free > (unsigned)c.P;
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        need[i] = BR_EMPTY_SLOT; have[i] = 0;
        if (at.slot + i < c.B) { need[i] = c.len[slots + at.slot + i]; have[i] = c.n_blocks[slots + at.slot + i]; }
    }
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        need[i] = cache_blocks(c, cache_tokens(need[i], step));
        if ((unsigned)have[i] > (unsigned)c.T) { bad = true; continue; }
        held += have[i];
        back += max(have[i] - need[i], 0);
        ask += need[i] <= c.T ? max(need[i] - have[i], 0) : 0;
    }
    // (with counts in range all sums stay below 2^30)
    bad = ONE ? __any_sync(kFull, bad) : __syncthreads_or(bad);
    TeamSums sum = {0, 0, 0, 0, 0};
    if (!bad) {
        sum = team_sums<ONE>(back, ask, held, part, at.lane, at.warp);
        bad = n_free + sum.z_all > c.P;
    }
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
    int A = 0;
    long long lacking = 0;
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        if (at.slot + i >= c.B) break;
        const int less = max(have[i] - need[i], 0), more = max(need[i] - have[i], 0);
        back_run[at.slot + i] = {sum.x + less, need[i] - sum.x};
        sum.x += less;
        // a sum over all demands up to this one: the first that does not fit keeps out the ones behind it
        const int upto = sum.y + (need[i] <= c.T ? more : 0);
        const bool fits = need[i] <= c.T && upto <= n_free + R;
        grow_run[at.slot + i] = {fits ? upto : sum.y, have[i] - sum.y};
        sum.y = upto;
        if (fits) A = upto; else lacking += more;
        a.n_blocks_out[slots + at.slot + i] = have[i] + (fits ? more : 0) - less;
    }
    A = (int)__reduce_max_sync(kFull, (unsigned)A);
    if (__any_sync(kFull, lacking != 0))
        for (int o = 16; o > 0; o >>= 1) lacking += __shfl_xor_sync(kFull, lacking, o);
    if (!ONE && at.lane == 0 && at.warp < 8) { granted[at.warp] = A; lacks[at.warp] = lacking; }
    team_sync<ONE>();
    if (!ONE) {
        lacking = 0;
        for (int w = 0; w < min((int)(blockDim.x >> 5), 8); ++w) { A = max(A, granted[w]); lacking += lacks[w]; }
    }
    if (at.slot == 0) {
        a.n_free_out[row] = n_free + R - A;
        if (a.short_out) a.short_out[row] = (int)min(lacking, 0x7FFFFFFFll);
    }
    int lo, hi;
    cache_piece(at.piece, at.pieces, max(R, A), 0, &lo, &hi);
    int e = lo + at.lane;
    if (e >= hi) return;
    const auto table = mk_span(c.table + slots * c.T, (long long)c.B * c.T);
    const auto list = mk_span(c.free_list + row * c.P, c.P);
    Walk from, to;
    if (e < R) from.seek(back_run, c.B, e);
    if (e < A) to.seek(grow_run, c.B, e);
    for (; e < hi; e += 32 * kMoves) {
        int id[kMoves];
#pragma unroll
        for (int u = 0; u < kMoves; ++u) {
            const int x = e + 32 * u;
            if (x >= hi) break;
            if (x < R) {
                from.to(x);
                id[u] = table[(long long)from.slot * c.T + x + from.at.shift];
            } else {
                id[u] = list[n_free + R - 1 - x];
            }
        }
#pragma unroll
        for (int u = 0; u < kMoves; ++u) {
            const int x = e + 32 * u;
            if (x >= hi) break;
            if (x < A) {
                to.to(x);
                table[(long long)to.slot * c.T + x + to.at.shift] = id[u];
            } else {
                list[n_free + R - 1 - x] = id[u];
            }
        }
    }
}

// One new token a request.
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
                slot[i] = (long long)table[(long long)(at.slot + i) * c.T + column] * c.t + (n[i] - 1 - column * c.t);
            ++count;
        }
    }
    const TeamSums sum = team_sums<ONE>(count, 0, 0, part, at.lane, at.warp);
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

// 32 bytes in one store, so that every sector is written whole and once (two of 16 bytes wrote each sector twice)
__device__ __forceinline__ void store_four(FourSlots *p, const FourSlots &s)
{
    asm volatile("st.global.v4.b64 [%0], {%1, %2, %3, %4};" :: "l"(p), "l"(s.v[0]), "l"(s.v[1]), "l"(s.v[2]), "l"(s.v[3]) : "memory");
}

// Any number of new tokens: four in a row a lane, stored as 32 aligned bytes.
template <bool ONE, int SPL>
__global__ void __launch_bounds__(256) br_slot_map_kernel(const SlotArgs a)
{
    constexpr int kSlots = ONE ? 32 * SPL : BR_MAX_B;
    __shared__ Run runs[ONE ? kCacheTeams : 1][kSlots];
    __shared__ int held_by[ONE ? kCacheTeams : 1][kSlots];
    __shared__ int4 part[ONE ? 1 : 8];
    stream_order_gate();
    const CacheArgs &c = a.c;
    const Seat<ONE, SPL> at(c);
    if (!at.any) return;
    Run *run = runs[ONE ? at.warp : 0];
    int *held_of = held_by[ONE ? at.warp : 0];
    const size_t row = at.row, slots = row * c.B;
    const int step = at.step(c);
    int n[SPL], q[SPL], held[SPL], mine = 0;
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
    }
    const TeamSums sum = team_sums<ONE>(mine, 0, 0, part, at.lane, at.warp);
    const auto cu = mk_span(a.cu + row * (c.B + 1), c.B + 1);
    const bool first_slice = at.piece < (ONE ? 1 : (int)(blockDim.x >> 5));
    int place = sum.x;
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        const int b = at.slot + i;
        if (b >= c.B) break;
        const int from = place;
        place = add_to_most(place, q[i]);
        run[b] = {place, n[i] - q[i] - from};         // (a run that starts at 2^31 - 1 has no item below `room`)
        held_of[b] = min(max(held[i], 0), c.T);
        if (first_slice) {
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
    cache_piece(at.piece, at.pieces, count, skew, &lo, &hi);
    int e = (lo + skew) / 128 * 128 + 4 * at.lane - skew;          // (lo is at a unit's start, or the row's)
    if (max(e, lo) >= hi) return;
    Walk w;
    w.seek(run, c.B, max(e, lo));
    for (; e < hi; e += 128) {
        const int first = max(e, lo);
        w.to(first);
        if (e >= lo && e + 4 <= min(hi, w.at.upto) && c.t >= 4) {
            const int p = e + w.at.shift, column = over(p, c.over_t), off = p - column * c.t, held_here = held_of[w.slot];
            const long long entry = (long long)w.slot * c.T + column;
            const bool next = off + 3 >= c.t;
            const long long id0 = column < held_here ? table[entry] : -1, id1 = next && column + 1 < held_here ? table[entry + 1] : -1;
            const long long s0 = id0 * c.t + off, s1 = id1 * c.t + off - c.t;
            FourSlots v;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool in0 = off + j < c.t;
                v.v[j] = (in0 ? column : column + 1) < held_here ? (in0 ? s0 : s1) + j : -1;
            }
            store_four(vec_at<FourSlots>(out, e), v);
        } else {
            const int last = min(e + 4, hi);
            for (int x = first; x < last; ++x) {
                w.to(x);
                const int p = x + w.at.shift, column = over(p, c.over_t);
                out[x] = column < held_of[w.slot]
                             ? (long long)table[(long long)w.slot * c.T + column] * c.t + (p - column * c.t) : -1;
            }
        }
    }
}

// The running slots move up, their blocks follow one another.
template <bool ONE, int SPL>
__global__ void __launch_bounds__(256) br_page_lists_kernel(const PageArgs a)
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
    int n[SPL], held[SPL], mine = 0, running = 0;
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        n[i] = BR_EMPTY_SLOT; held[i] = 0;
        if (at.slot + i < c.B) { n[i] = c.len[slots + at.slot + i]; held[i] = c.n_blocks[slots + at.slot + i]; }
    }
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        n[i] = cache_tokens(n[i], step);
        held[i] = min(max(held[i], 0), c.T);
        mine += min(cache_blocks(c, n[i]), held[i]);
        running += n[i] > 0;
    }
    const TeamSums sum = team_sums<ONE>(mine, running, 0, part, at.lane, at.warp);
    const auto seq_slot = mk_span(a.seq_slot + slots, c.B), last = mk_span(a.last + slots, c.B);
    const auto indptr = mk_span(a.indptr + row * (c.B + 1), c.B + 1);
    const bool first_slice = at.piece < (ONE ? 1 : (int)(blockDim.x >> 5));
    int place = sum.x, rank = sum.y;
#pragma unroll
    for (int i = 0; i < SPL; ++i) {
        const int b = at.slot + i;
        if (b >= c.B) break;
        const int need = cache_blocks(c, n[i]), pages = min(need, held[i]);
        if (first_slice && n[i] > 0) {
            seq_slot[rank] = b;
            indptr[rank] = place;
            last[rank] = pages == 0 ? 0 : need <= held[i] ? n[i] - (need - 1) * c.t : c.t;
            ++rank;
        }
        run[b] = {place + pages, -place};
        place += pages;
        if (first_slice && b >= sum.y_all) { seq_slot[b] = -1; last[b] = 0; indptr[b] = sum.x_all; }
    }
    if (first_slice && at.slot == 0) { indptr[c.B] = sum.x_all; a.n_seq[row] = sum.y_all; }
    team_sync<ONE>();
    const auto table = mk_span(c.table + slots * c.T, (long long)c.B * c.T);
    const auto out = mk_span(a.indices + row * c.P, c.P);
    int lo, hi;
    cache_piece(at.piece, at.pieces, min(sum.x_all, c.P), 0, &lo, &hi);
    int e = lo + at.lane;
    if (e >= hi) return;
    Walk w;
    w.seek(run, c.B, e);
    for (; e < hi; e += 32 * kMoves) {
        int id[kMoves];
#pragma unroll
        for (int u = 0; u < kMoves; ++u) {
            const int x = e + 32 * u;
            if (x >= hi) break;
            w.to(x);
            id[u] = table[(long long)w.slot * c.T + x + w.at.shift];
        }
#pragma unroll
        for (int u = 0; u < kMoves; ++u)
            if (e + 32 * u < hi) out[e + 32 * u] = id[u];
    }
}

}  // namespace br
