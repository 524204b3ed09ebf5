// A cache of keys or values in pages, in the operands' own type: its tables, lists of its slots, writing into it, and the choice of pages
// by a cheap score.  Attention over it is in paged_attention.cuh.
//
// Request r's position p lies in row p % page of page tables[r][p / page].  Everything that says how much there is to do (lengths, new tokens,
// tables) is on the device, so a launch is sized by what the host knows (requests, tokens, width of the tables) and the kernels find their
// work themselves: each CTA forms the prefix sums over the requests that it needs, which costs it a microsecond and spares a launch.  Every kernel may be
// launched before the one ahead of it has ended: its CTAs wait for that first of all, all of them, so that what comes behind can count on it.  One does a
// little before: paged_select_kernel behind paged_score_kernel, which lets it begin only when all of its own CTAs have waited, and neither writes what tells of
// the tokens nor reads the lists.
#pragma once
#include <limits.h>

#include "attention_rows.cuh"
#include "div.h"

namespace b2sp {
namespace paged {

using attn::Bf16;

constexpr int kThreads = 256;
constexpr int kMostRequests = 8192;   // prefix sums over requests lie in shared memory

template <typename T> struct Pages {
    T *data;
    long long ld, sh, sp;   // elements: rows, heads, pages
    int pages;
    __device__ T *row(int page, int h, int r) const { return data + page * sp + h * sh + r * ld; }
};

struct Tables {
    int *entries;
    long long ld;
    int requests, width;
};

// What token i sees: `seen` positions of the request `row`; nothing where row is not a request.
struct Tokens {
    const int *rows, *seen;   // rows: NULL = token i belongs to request i
};
__device__ __forceinline__ int row_of(const Tokens &t, int i) { return t.rows ? t.rows[i] : i; }
__device__ __forceinline__ int seen_of(const Tokens &t, const Tables &tab, int page, int i)
{
    const int r = row_of(t, i), s = t.seen[i];
    if ((unsigned)r >= (unsigned)tab.requests) return 0;
    return (int)min((long long)max(s, 0), (long long)tab.width * page);
}

__device__ __forceinline__ long long quotient(long long a, long long b)   // of numbers that are not negative
{
    return (a | b) >> 32 ? a / b : (long long)((unsigned)a / (unsigned)b);
}
__device__ __forceinline__ int saturated(long long x) { return (int)min(x, (long long)INT_MAX); }
// Sum over the block, for all threads (8 warps of shared memory).
__device__ __forceinline__ long long block_sum(long long x, long long *warps)
{
#pragma unroll
    for (int w = 16; w; w >>= 1) x += __shfl_xor_sync(~0u, x, w);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = x;
    __syncthreads();
    x = 0;
    for (int w = 0; w < (int)blockDim.x / 32; ++w) x += warps[w];
    return x;
}
// Sum over the threads before this one, and (total) over all.
__device__ __forceinline__ long long block_before(long long x, long long *warps, long long &total)
{
    const int lane = threadIdx.x & 31;
    long long up = x;
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {
        const long long y = __shfl_up_sync(~0u, up, w);
        if (lane >= w) up += y;
    }
    __syncthreads();
    if (lane == 31) warps[threadIdx.x >> 5] = up;
    __syncthreads();
    long long before = 0;
    total = 0;
    for (int w = 0; w < (int)blockDim.x / 32; ++w) {
        if (w < (int)threadIdx.x >> 5) before += warps[w];
        total += warps[w];
    }
    return before + up - x;
}
// The same for three sums (each becomes what is before this thread).
__device__ __forceinline__ void block_before3(long long &x, long long &y, long long &z, long long *warps, long long &all_x, long long &all_y, long long &all_z)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = blockDim.x / 32;
    long long a = x, b = y, c = z;
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {
        const long long u = __shfl_up_sync(~0u, a, w), v = __shfl_up_sync(~0u, b, w), t = __shfl_up_sync(~0u, c, w);
        if (lane >= w) { a += u; b += v; c += t; }
    }
    if (lane == 31) { warps[warp] = a; warps[n + warp] = b; warps[2 * n + warp] = c; }
    __syncthreads();
    x = a - x; y = b - y; z = c - z;
    all_x = all_y = all_z = 0;
    for (int w = 0; w < n; ++w) {
        if (w < warp) { x += warps[w]; y += warps[n + w]; z += warps[2 * n + w]; }
        all_x += warps[w]; all_y += warps[n + w]; all_z += warps[2 * n + w];
    }
}
// Tokens' costs in a line, dealt to `parts` warps in equal shares of at least `least`: what warp `me` has.
struct Share {
    long long lo, hi, share, rest;   // [lo, hi) of the line; every warp's share; lo is `rest` behind the begin of token `row`
    int row;
};
__device__ __forceinline__ long long lanes_up_to(int x)   // sum over the lanes up to this one
{
    const int lane = threadIdx.x & 31;
    if (!__any_sync(~0u, x >> 26)) {
#pragma unroll
        for (int w = 1; w < 32; w <<= 1) {
            const int y = __shfl_up_sync(~0u, x, w);
            if (lane >= w) x += y;
        }
        return x;
    }
    long long up = x;
#pragma unroll
    for (int w = 1; w < 32; w <<= 1) {
        const long long y = __shfl_up_sync(~0u, up, w);
        if (lane >= w) up += y;
    }
    return up;
}
// load(base): what cost() needs of the tokens from base (a multiple of 32) on, one in a lane; cost(window): what each of the `units` units of a lane's token
// costs, for all lanes of a warp (0 behind the last).  The last window that cost() gets is the one that `row` lies in.  False: nothing.  All threads call it.
template <int THREADS, typename Load, typename Cost>
__device__ __forceinline__ bool deal(int M, int units, Load load, Cost cost, int parts, int me, int least, Share &s)
{
    constexpr int WARPS = THREADS / 32, KEPT = 256;   // KEPT: windows of 32 tokens whose sums are kept (8192 tokens; beyond them they are formed again)
    __shared__ long long sums[KEPT], others[WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, windows = (M + 31) / 32;
    long long all, up = 0;
    int c = 0;
    if (windows == 1) {   // each warp for itself
        c = cost(load(0));
        up = lanes_up_to(c);
        all = __shfl_sync(~0u, up, 31);
    } else {
        all = 0;
        // (a loop, not copies of it: instructions that run once wait for their own way into the cache)
        auto next = load(warp * 32);
#pragma unroll 1
        for (int w = warp; w < windows; w += WARPS) {
            const auto now = next;
            next = load((w + WARPS) * 32);
            const int x = cost(now);
            long long n;
            if (!__any_sync(~0u, x >> 26)) {
                n = __reduce_add_sync(~0u, x);
            } else {
                n = x;
#pragma unroll
                for (int d = 16; d; d >>= 1) n += __shfl_xor_sync(~0u, n, d);
            }
            if (lane == 0 && w < KEPT) sums[w] = n;
            all += n;
        }
        if (lane == 0) others[warp] = all;
        __syncthreads();
        all = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) all += others[w];
    }
    all *= units;
    s.share = max((long long)least, quotient(all + parts - 1, parts));
    s.lo = me * s.share;
    s.hi = min(s.lo + s.share, all);
    if (s.lo >= s.hi) return false;
    s.rest = s.lo;
    s.row = 0;
    if (windows > 1) {
        for (int w0 = 0; w0 < min(windows, KEPT); w0 += 32) {   // 32 windows at a time
            long long n = w0 + lane < min(windows, KEPT) ? sums[w0 + lane] * units : 0, x = n;
#pragma unroll
            for (int w = 1; w < 32; w <<= 1) {
                const long long y = __shfl_up_sync(~0u, x, w);
                if (lane >= w) x += y;
            }
            const unsigned behind = __ballot_sync(~0u, x > s.rest);
            const int k = behind ? __ffs(behind) - 1 : 31;
            s.rest -= __shfl_sync(~0u, behind ? x - n : x, k);
            s.row = (w0 + k + !behind) * 32;
            if (behind) break;
        }
        for (;; s.row += 32) {   // (more than one round only behind the sums that are kept)
            if (s.row >= M) return false;   // (not with lengths that stay as they are)
            c = cost(load(s.row));
            up = lanes_up_to(c);
            const long long n = __shfl_sync(~0u, up, 31) * units;
            if (n > s.rest) break;
            s.rest -= n;
        }
    }
    const unsigned behind = __ballot_sync(~0u, up * units > s.rest);
    const int k = __ffs(behind) - 1;
    s.rest -= __shfl_sync(~0u, up - c, k) * units;
    s.row += k;
    return behind != 0;
}
// The last r in [0, n) with ptr[r] <= x < ptr[r + 1]; ptr[0] = 0 <= x < ptr[n].
__device__ __forceinline__ int segment_of(const int *ptr, int n, int x)
{
    int lo = 0, hi = n;   // ptr[lo] <= x < ptr[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (ptr[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// ---- tables ----------------------------------------------------------------------------------------------------------------------
struct TablesArgs {
    Tables t;
    int page, pages, tokens, free_room;
    const int *lengths, *added, *free_count;
    int *free_pages;
    int *lengths_out, *row_ptr, *rows, *seen, *slots, *counts;
};
struct Request { int length, owned, total, need, back, fresh; };   // positions before and after; pages it has, takes, gives back; new tokens
__device__ __forceinline__ Request request(const TablesArgs &a, int r)
{
    Request q;
    const long long most = min((long long)a.t.width * a.page, (long long)INT_MAX);
    const int more = a.added[r];
    q.length = (int)min((long long)max(a.lengths[r], 0), most);
    q.owned = (int)((q.length + (a.page - 1ll)) / a.page);
    q.fresh = max(more, 0);
    q.total = more < 0 ? 0 : (int)min((long long)q.length + more, most);
    q.need = more < 0 ? 0 : (int)((q.total + (a.page - 1ll)) / a.page) - q.owned;
    q.back = more < 0 ? q.owned : 0;
    return q;
}

// Pages given back are pushed on the stack of free ones in order of requests, then new ones are popped in order of requests.  No CTA waits for
// another: which page the k-th new one is follows from the prefix sums, and one that is given back in the same step is read from the table
// of the request that ends, so everything is a function of the inputs, and any number of CTAs take any part of it.
// A count below 0 is what a step leaves that found too few pages.  Its lengths count positions that no page holds, so a step on top of it would push entries
// that are no pages and lose tokens without a word: it does nothing instead, and what the short step read is still there for it to be made again.
// Bound by latency: lengths, then (tokens) a table entry or a free page.  64 requests with a token each 4.1 us, 512 with 16384 new tokens 7.2 us.
__global__ void __launch_bounds__(kThreads) paged_tables_kernel(const TablesArgs a)
{
    extern __shared__ int prefix[];
    __shared__ long long warps[3 * kThreads / 32];
    const int R = a.t.requests, each = (R + kThreads - 1) / kThreads, r0 = min(R, (int)threadIdx.x * each), r1 = min(R, r0 + each);
    int *take = prefix, *back = prefix + R + 1, *ptr = prefix + 2 * (R + 1);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    long long n_take = 0, n_back = 0, n_new = 0, all_take, all_back, all_new;
    for (int r = r0; r < r1; ++r) {
        const Request q = request(a, r);
        n_take += q.need; n_back += q.back; n_new += q.fresh;
    }
    const int given = *a.free_count, count = min(max(given, 0), a.free_room);
    block_before3(n_take, n_back, n_new, warps, all_take, all_back, all_new);
    const long long me = blockIdx.x * (long long)kThreads + threadIdx.x, all = gridDim.x * (long long)kThreads;
    if (given < 0) {
        for (long long r = me; r < R; r += all) { a.lengths_out[r] = request(a, (int)r).length; a.row_ptr[r] = 0; }
        for (long long t = me; t < a.tokens; t += all) { a.rows[t] = -1; a.seen[t] = 0; a.slots[t] = -1; }
        if (me == 0) {
            a.row_ptr[R] = 0;
            a.counts[0] = given; a.counts[1] = 0; a.counts[2] = saturated(all_new); a.counts[3] = 0;
        }
        return;
    }
    const long long top = min(count + all_back, (long long)a.free_room);   // free pages before any is taken
    long long fit = 0;                                                      // tokens that get a row
    for (int r = r0; r < r1; ++r) {
        const Request q = request(a, r);
        take[r] = saturated(n_take); back[r] = saturated(n_back); ptr[r] = saturated(n_new);
        if (blockIdx.x == 0) {
            a.lengths_out[r] = q.total;
            a.row_ptr[r] = saturated(n_new);
            const long long got = min(max(top - n_take, 0ll), (long long)q.need);
            const long long end = got == q.need ? q.total : min((long long)q.total, (q.owned + got) * a.page);
            if (q.fresh) fit += max(0ll, min(end - q.length, a.tokens - n_new));
        }
        n_take += q.need; n_back += q.back; n_new += q.fresh;
    }
    if (threadIdx.x == 0) { take[R] = saturated(all_take); back[R] = saturated(all_back); ptr[R] = saturated(all_new); }
    if (blockIdx.x == 0) {
        fit = block_sum(fit, warps);
        if (threadIdx.x == 0) {
            a.row_ptr[R] = saturated(all_new);
            a.counts[0] = (int)max(top - all_take, -(long long)INT_MAX);
            a.counts[1] = saturated(all_new);
            a.counts[2] = saturated(all_new - fit);
            a.counts[3] = saturated(all_take);
        }
    }
    __syncthreads();
    const auto valid = [&](int p) { return (unsigned)p < (unsigned)a.pages ? p : -1; };
    const auto popped = [&](long long k) {
        const long long at = top - 1 - k;
        if (at < 0) return -1;
        if (at < count) return valid(a.free_pages[at]);
        const int j = (int)(at - count), r = segment_of(back, R, j);
        return valid(a.t.entries[r * a.t.ld + (j - back[r])]);
    };
    for (long long t = me; t < a.tokens; t += all) {
        int r = -1, seen = 0, slot = -1;
        if (t < ptr[R]) {
            r = segment_of(ptr, R, (int)t);
            const Request q = request(a, r);
            const long long at = q.length + (t - ptr[r]);
            if (at < q.total) {
                const int c = (int)(at / a.page);
                const int p = c < q.owned ? valid(a.t.entries[r * a.t.ld + c]) : popped((long long)take[r] + (c - q.owned));
                if (p >= 0) { seen = (int)at + 1; slot = p * a.page + (int)(at - (long long)c * a.page); }
            }
        }
        a.rows[t] = r; a.seen[t] = seen; a.slots[t] = slot;
    }
    for (long long k = me; k < take[R]; k += all) {
        const int r = segment_of(take, R, (int)k);
        a.t.entries[r * a.t.ld + request(a, r).owned + ((int)k - take[r])] = popped(k);
    }
    for (long long j = me; j < back[R] && count + j < a.free_room; j += all) {
        const int r = segment_of(back, R, (int)j);
        a.free_pages[count + j] = a.t.entries[r * a.t.ld + ((int)j - back[r])];
    }
}

// ---- lists of slots --------------------------------------------------------------------------------------------------------------
struct ListsArgs {
    Tables t;
    Tokens tok;
    int M, page, pages;
    long long entries;
    int *row_ptr, *col_idx;
    Div by_page;
};
// More than kListTokens tokens: the ends of their lists in a launch of their own.
constexpr int kScanThreads = 1024, kListTokens = 8192;
__global__ void __launch_bounds__(kScanThreads) paged_list_ends_kernel(const ListsArgs a)
{
    __shared__ long long warps[kScanThreads / 32];
    const int each = (a.M + kScanThreads - 1) / kScanThreads, i0 = (int)min((long long)a.M, threadIdx.x * (long long)each), i1 = min(a.M, i0 + each);
    long long n = 0, all;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int i = i0; i < i1; ++i) n += seen_of(a.tok, a.t, a.page, i);
    n = block_before(n, warps, all);
    for (int i = i0; i < i1; ++i) {
        a.row_ptr[i] = (int)min(n, a.entries);
        n += seen_of(a.tok, a.t, a.page, i);
    }
    if (threadIdx.x == 0) a.row_ptr[a.M] = (int)min(all, a.entries);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
// A thread takes four neighbouring entries: their list by a binary search over the ends, which each CTA forms for itself in shared memory (KEPT), then
// a page of the table for all four unless a page or a list ends among them.  Bound by latency (lengths, table), then by the stores.  64 lists of 524288 slots in
// all: 3.9 us (ends and lists as two kernels, an entry a thread, a warp 512 of them: 10.0).
template <bool KEPT>
__global__ void __launch_bounds__(kThreads) paged_list_kernel(const ListsArgs a)
{
    extern __shared__ int kept[];
    __shared__ long long warps[kThreads / 32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int *ends = KEPT ? kept : a.row_ptr;
    if (KEPT) {
        const int each = (a.M + kThreads - 1) / kThreads, i0 = min(a.M, (int)threadIdx.x * each), i1 = min(a.M, i0 + each);
        long long n = 0, all;
        for (int i = i0; i < i1; ++i) n += seen_of(a.tok, a.t, a.page, i);
        n = block_before(n, warps, all);
        for (int i = i0; i < i1; ++i) {
            kept[i] = (int)min(n, a.entries);
            if (blockIdx.x == 0) a.row_ptr[i] = kept[i];
            n += seen_of(a.tok, a.t, a.page, i);
        }
        if (threadIdx.x == 0) {
            kept[a.M] = (int)min(all, a.entries);
            if (blockIdx.x == 0) a.row_ptr[a.M] = kept[a.M];
        }
        __syncthreads();
    }
    const int all = ends[a.M];
    const bool fours = (reinterpret_cast<uintptr_t>(a.col_idx) & 15) == 0;
    for (long long e0 = (blockIdx.x * (long long)kThreads + threadIdx.x) * 4; e0 < a.entries; e0 += gridDim.x * (long long)kThreads * 4) {
        int slots[4];
        int i = -1, end = 0, first = 0, base = 0, c_of = -1, held = -1;   // the list that the last entry was of; its page
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const long long e = e0 + k;
            slots[k] = -1;
            if (e >= all) continue;
            if (i < 0 || e >= end) {
                i = segment_of(ends, a.M, (int)e);
                first = ends[i];
                end = ends[i + 1];
                base = row_of(a.tok, i);
                c_of = -1;
            }
            const int p = (int)e - first, c = (int)a.by_page((unsigned)p);
            if (c != c_of) held = a.t.entries[base * a.t.ld + (c_of = c)];
            if ((unsigned)held < (unsigned)a.pages) slots[k] = held * a.page + (p - c * a.page);
        }
        if (fours && e0 + 3 < a.entries) {
            *reinterpret_cast<int4 *>(a.col_idx + e0) = make_int4(slots[0], slots[1], slots[2], slots[3]);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (e0 + k < a.entries) a.col_idx[e0 + k] = slots[k];
        }
    }
}

// ---- writing ---------------------------------------------------------------------------------------------------------------------
template <typename T> struct WriteArgs {
    Tables t;
    const T *k, *v;
    long long k_ld, k_sh, v_ld, v_sh;
    int heads, d, page, tokens;
    const int *row_ptr, *lengths;
    Pages<T> kp, vp, means;   // means: data NULL = none; ld unused
};
struct Added { int length, n, first; };   // positions there are, new ones (as far as the table reaches), their first token
template <typename T> __device__ __forceinline__ Added added(const WriteArgs<T> &a, int r)
{
    Added q;
    const long long most = min((long long)a.t.width * a.page, (long long)INT_MAX);
    q.length = (int)min((long long)max(a.lengths[r], 0), most);
    q.first = min(max(a.row_ptr[r], 0), a.tokens);
    q.n = (int)min((long long)max(min(a.row_ptr[r + 1], a.tokens) - q.first, 0), most - q.length);
    return q;
}
// Eight neighbours (fp32: four) of a row, 16 bytes.  WIDE: one load; else element by element, zeros behind d.
template <typename T> struct Chunk {
    static constexpr int N = 16 / sizeof(T);
    uint4 u;
    __device__ __forceinline__ void load(const T *row, int e, int d, bool wide)
    {
        if (wide) { u = *reinterpret_cast<const uint4 *>(row + e); return; }
        unsigned w[4] = {};
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (e + i < d) {
                if constexpr (sizeof(T) == 2) w[i / 2] |= (unsigned)row[e + i].bits << 16 * (i & 1);
                else w[i] = __float_as_uint(row[e + i]);
            }
        u = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void store(T *row, int e, int d) const   // (16-byte aligned rows; what lies behind d stays)
    {
        if (e + N <= d) { *reinterpret_cast<uint4 *>(row + e) = u; return; }
        const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (e + i < d) {
                if constexpr (sizeof(T) == 2) row[e + i].bits = (unsigned short)(w[i / 2] >> 16 * (i & 1));
                else row[e + i] = __uint_as_float(w[i]);
            }
    }
    __device__ __forceinline__ void add_to(float (&x)[N]) const
    {
        const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (sizeof(T) == 2) x[i] += __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
            else x[i] += __uint_as_float(w[i]);
        }
    }
};

// A CTA per touched page and head: the request's new rows that lie in it are copied, and the mean of K's rows is formed from them and those that were
// there.  So a page's rows are summed in one place and order (in fp32, rounded once to the cache's type), and no row is written twice.
// Bound by HBM once there are many rows: 16384 tokens of 8 heads, width 128, 136 MB, 25.4 us, of which the floor is 20.8.  Eight CTAs of 128 threads on an SM
// with two rows' loads each; five with four rows' 28.7, three with eight rows' 34.2, ten with two rows' (which spill) 35.8 us.
constexpr int kWriteThreads = 128, kWriteRows = 2, kWriteCTAs = 8;   // CTAs of an SM
template <typename T>
__global__ void __launch_bounds__(kWriteThreads, kWriteCTAs) paged_write_kernel(const WriteArgs<T> a)
{
    using C = Chunk<T>;
    extern __shared__ int prefix[];   // [R + 1] touched pages before request r
    __shared__ long long warps[kWriteThreads / 32];
    __shared__ float sums[kWriteThreads][C::N];
    const int R = a.t.requests, each = (R + kWriteThreads - 1) / kWriteThreads, r0 = min(R, (int)threadIdx.x * each), r1 = min(R, r0 + each);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const auto touched = [&](int r) {
        const Added q = added(a, r);
        return q.n ? (int)((q.length + (long long)q.n + a.page - 1) / a.page) - q.length / a.page : 0;
    };
    long long n = 0, all;
    for (int r = r0; r < r1; ++r) n += touched(r);
    n = block_before(n, warps, all);
    for (int r = r0; r < r1; ++r) { prefix[r] = saturated(n); n += touched(r); }
    if (threadIdx.x == 0) prefix[R] = saturated(all);
    __syncthreads();
    const int chunks = (a.d + C::N - 1) / C::N;
    const long long units = (long long)prefix[R] * a.heads;
    for (long long u = blockIdx.x; u < units; u += gridDim.x) {
        const int s = (int)(u / a.heads), h = (int)(u - (long long)s * a.heads), r = segment_of(prefix, R, s);
        const Added q = added(a, r);
        const int c = q.length / a.page + (s - prefix[r]), held = a.t.entries[r * a.t.ld + c];
        const long long p0 = (long long)c * a.page;                                  // the page's first position
        const int old = (int)max(q.length - p0, 0ll);                                // rows that were there
        const int end = (int)min((long long)a.page, (long long)q.length + q.n - p0); // rows that are now
        if ((unsigned)held >= (unsigned)a.kp.pages) continue;                        // (the same for all threads)
        const bool means = a.means.data != nullptr;
        const T *k = a.k + h * a.k_sh + (q.first + (p0 - q.length)) * a.k_ld, *v = a.v + h * a.v_sh + (q.first + (p0 - q.length)) * a.v_ld;   // of row 0
        const bool k_wide = ((reinterpret_cast<uintptr_t>(a.k) | (uintptr_t)(a.k_ld * sizeof(T)) | (uintptr_t)(a.k_sh * sizeof(T))) & 15) == 0;
        const bool v_wide = ((reinterpret_cast<uintptr_t>(a.v) | (uintptr_t)(a.v_ld * sizeof(T)) | (uintptr_t)(a.v_sh * sizeof(T))) & 15) == 0;
        for (int c0 = 0; c0 < chunks; c0 += kWriteThreads) {   // (once, but for very wide rows)
            const int lanes = min(chunks - c0, kWriteThreads), groups = kWriteThreads / lanes, group = threadIdx.x / lanes;
            float x[C::N] = {};
            if (group < groups) {
                const int e = (c0 + threadIdx.x % lanes) * C::N;
                const bool whole = e + C::N <= a.d;
                for (int i0 = (means ? 0 : old) + group; i0 < end; i0 += kWriteRows * groups) {   // kWriteRows rows' loads at once
                    C y[kWriteRows], z[kWriteRows];
#pragma unroll
                    for (int n = 0; n < kWriteRows; ++n) {
                        const int i = i0 + n * groups;
                        y[n].u = make_uint4(0, 0, 0, 0);
                        if (i >= end) continue;
                        if (i < old) {
                            y[n].load(a.kp.row(held, h, i), e, a.d, whole);
                        } else {
                            y[n].load(k + i * a.k_ld, e, a.d, k_wide && whole);
                            z[n].load(v + i * a.v_ld, e, a.d, v_wide && whole);
                        }
                    }
#pragma unroll
                    for (int n = 0; n < kWriteRows; ++n) {
                        const int i = i0 + n * groups;
                        if (i >= old && i < end) {
                            y[n].store(a.kp.row(held, h, i), e, a.d);
                            z[n].store(a.vp.row(held, h, i), e, a.d);
                        }
                        if (means) y[n].add_to(x);
                    }
                }
            }
            if (means) {
#pragma unroll
                for (int i = 0; i < C::N; ++i) sums[threadIdx.x][i] = x[i];
                __syncthreads();
                for (int e = threadIdx.x; e < lanes * C::N && c0 * C::N + e < a.d; e += kWriteThreads) {
                    float y = 0.f;
                    for (int g = 0; g < groups; ++g) y += sums[g * lanes + e / C::N][e % C::N];
                    attn::narrow(y / (float)end, a.means.row(held, h, 0)[c0 * C::N + e]);
                }
                __syncthreads();
            }
        }
    }
}

// ---- the choice of pages ---------------------------------------------------------------------------------------------------------
template <typename T> struct SelectArgs {
    Tables t;
    Tokens tok;
    const T *q;
    long long q_ld, q_sh;
    int M, heads, kv_heads, d, page, keep, first, last;
    bool q_wide;                // 16-byte loads of q
    Pages<T> means;
    float2 *scores;             // [M][kv_heads][width]: a score in 32 bits and how far it may be off
    int *lists;                 // [M][kv_heads][keep]
    int *status;
};
template <typename T> __device__ __forceinline__ int pages_seen(const SelectArgs<T> &a, int i)
{
    return (int)((seen_of(a.tok, a.t, a.page, i) + (a.page - 1ll)) / a.page);
}
// A whole number that grows with x; NaN below everything else, both zeros alike.
__device__ __forceinline__ unsigned long long ordered(double x)
{
    if (x != x) return 0;
    const unsigned long long u = (unsigned long long)__double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | 1ull << 63;
}

// The choice is defined by scores in 64 bits, since between two close ones sums of 32 bits would choose by their order.  Few scores are that close: they
// are formed in 32 bits with a bound of the error, and a token whose border lies between two scores that are further apart than that is done; only
// where others lie within reach of the border these are formed again in 64 bits.  (All of them in 64 bits: 2 us more of the 9 to 10 for a token that sees
// 2048 pages, 8 key heads.)
//
// Scores of the pages of tokens that see more than a list holds: all tokens' and key heads' blocks of pages are dealt to the warps in equal shares; the sum of the
// group's queries is spread over LANES lanes, 16 bytes (HALVES: twice) of the mean each, and 32 / LANES pages are read by an instruction, a block by eight.  The
// next blocks' means are on their way to shared memory while this one's are added up (in registers they left room for fewer: 50.6 instead of 39.4 us for 64 tokens
// that see up to 2048 pages, 8 key heads, both kernels; their 134 MB take 20).  Few pages: bound by latencies.  A lane adds up eight products (in pairs) and
// the lanes' sums come together in at most five steps, so a score is off
// by at most 14 half steps of the sum of the products' magnitudes (one of them the query's rounding), and by what underflows.  That sum is no more than the
// product of the query's and the mean's lengths (Cauchy and Schwarz), which costs as many instructions as the score; kTiny is what squares lose that underflow.
// kScoreOff leaves room for the roundings of the bound itself and of what the choice makes of it.
constexpr float kScoreOff = 24.f * 5.9604645e-8f, kUnderflow = 1e-42f, kTiny = 1e-42f;
constexpr int kScoreThreads = 128, kScoreCTAs = 4, kScoreAhead = 1;   // CTAs of an SM (six: 22.3 instead of 18.9 us); blocks on their way (two: 40.7 instead of 39.4)
template <typename T, int LANES, int HALVES>
__global__ void __launch_bounds__(kScoreThreads, HALVES == 1 ? kScoreCTAs : kScoreCTAs / 2) paged_score_kernel(const SelectArgs<T> a)
{
    constexpr int N = 16 / sizeof(T), AT_ONCE = 8, STEP = 32 / LANES, BATCH = AT_ONCE * STEP;   // pages of an instruction, of a batch
    const int lane = threadIdx.x & 31, me = blockIdx.x * (kScoreThreads / 32) + (threadIdx.x >> 5), group = a.heads / a.kv_heads;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const auto blocks_of = [&](int i) {
        const int n = pages_seen(a, i);
        return n > a.keep ? (n + BATCH - 1) / BATCH : 0;
    };
    Share w;
    const auto load = [&](int base) { return base + lane < a.M ? blocks_of(base + lane) : 0; };
    if (!deal<kScoreThreads>(a.M, a.kv_heads, load, [](int blocks) { return blocks; }, gridDim.x * (kScoreThreads / 32), me, 1, w)) return;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (behind the wait: the choice reads lengths and writes lists before its own)
    struct At {   // a block
        int i, g, b, n, blocks;
    } at, front;   // the one that is added up, the one that is asked for
    at.i = w.row;
    at.n = pages_seen(a, at.i);
    at.blocks = (at.n + BATCH - 1) / BATCH;
    at.g = (int)w.rest / at.blocks;
    at.b = (int)w.rest - at.g * at.blocks;
    front = at;
    const auto step = [&](At &x) {   // whether it is another token's or head's
        if (++x.b < x.blocks) return false;
        x.b = 0;
        if (++x.g == a.kv_heads) {
            x.g = 0;
            do
                if (++x.i >= a.M) return false;
            while (!(x.blocks = blocks_of(x.i)));
            x.n = pages_seen(a, x.i);
        }
        return true;
    };
    const int e0 = lane % LANES * N;   // this lane's first element
    const bool ragged = a.d % N != 0;
    const unsigned head = (unsigned)(a.means.sh * sizeof(T)), per_page = (unsigned)(a.means.sp * sizeof(T));   // (below 2^32)
    uint64_t q[HALVES][N / 2];
    float norm = 0.f;   // of the query
    // each lane asks for what it reads itself, kScoreAhead blocks ahead
    extern __shared__ uint4 score_room[];
    uint4 *room = score_room + (threadIdx.x >> 5) * (kScoreAhead + 1) * AT_ONCE * HALVES * 32 + lane;
    const auto look_up = [&] {
        const int p = front.b * BATCH + lane % BATCH;
        return p < front.n ? a.t.entries[row_of(a.tok, front.i) * a.t.ld + p] : -1;
    };
    int entry = look_up(), held[kScoreAhead + 1], left = (int)(w.hi - w.lo), to_ask = left, asked = 0, summed = 0;   // asked, summed: places in the room
    const auto ask = [&] {   // for means of a block whose pages the lanes hold; entries are one more block ahead
        const int had = entry;
        if (to_ask > 0) {
            const char *base = reinterpret_cast<const char *>(a.means.data + e0) + (unsigned long long)front.g * head;
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                const unsigned p = (unsigned)__shfl_sync(~0u, had, j * STEP + lane / LANES);
                const char *mean = base + (unsigned long long)p * per_page;
#pragma unroll
                for (int x = 0; x < HALVES; ++x) {
                    const bool there = p < (unsigned)a.means.pages && e0 + x * 32 * N < a.d;
                    const unsigned dst = (unsigned)__cvta_generic_to_shared(room + ((asked * AT_ONCE + j) * HALVES + x) * 32);
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(there ? mean + x * 32 * 16 : reinterpret_cast<const char *>(a.means.data)),
                                 "r"(there ? 16 : 0) : "memory");
                }
            }
            if (--to_ask > 0) {
                step(front);
                entry = look_up();
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        asked = asked == kScoreAhead ? 0 : asked + 1;
        return had;
    };
    const auto pair = [](const uint4 &u, int k) {   // elements 2 k and 2 k + 1 of sixteen bytes
        const unsigned w[4] = {u.x, u.y, u.z, u.w};
        if constexpr (sizeof(T) == 2) return attn::two(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xffff0000u));
        else return attn::two(__uint_as_float(w[2 * k]), __uint_as_float(w[2 * k + 1]));
    };
#pragma unroll
    for (int x = 0; x < kScoreAhead; ++x) held[x] = ask();
    for (bool fresh = true;;) {
        held[kScoreAhead] = ask();
        const int p0 = at.b * BATCH;
        float2 *scores = a.scores + ((long long)at.i * a.kv_heads + at.g) * a.t.width + p0;
        if (fresh) {   // the sum of the queries, four heads' loads at once
            double total[HALVES][N] = {};
            const T *from = a.q + at.i * a.q_ld + (long long)at.g * group * a.q_sh;
            for (int h = 0; h < group; h += 4) {
                Chunk<T> y[4][HALVES];
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int x = 0; x < HALVES; ++x) {
                        y[k][x].u = make_uint4(0, 0, 0, 0);
                        if (h + k < group) y[k][x].load(from + (h + k) * a.q_sh, e0 + x * 32 * N, a.d, a.q_wide && e0 + x * 32 * N + N <= a.d);
                    }
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int x = 0; x < HALVES; ++x) {
                        float f[N] = {};
                        y[k][x].add_to(f);
#pragma unroll
                        for (int m = 0; m < N; ++m) total[x][m] += f[m];
                    }
            }
            norm = 0.f;
#pragma unroll
            for (int x = 0; x < HALVES; ++x)
#pragma unroll
                for (int k = 0; k < N / 2; ++k) {
                    const float y = (float)total[x][2 * k], z = (float)total[x][2 * k + 1];
                    q[x][k] = attn::two(y, z);
                    norm = fmaf(y, y, fmaf(z, z, norm));
                }
#pragma unroll
            for (int x = 1; x < LANES; x <<= 1) norm += __shfl_xor_sync(~0u, norm, x);
            norm = sqrtf(fmaf(norm, 1.0001f, kTiny));
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(kScoreAhead) : "memory");
        const uint4 *mean = room + summed * AT_ONCE * HALVES * 32;
        float sum[AT_ONCE], size[AT_ONCE];   // of the products, and of the mean's squares
        bool nothing = false;
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            uint64_t s2 = 0, m2 = 0;
#pragma unroll
            for (int x = 0; x < HALVES; ++x) {
                uint4 c = mean[(j * HALVES + x) * 32];
                if (ragged && e0 + x * 32 * N + N > a.d) {   // what lies behind d may be anything
                    unsigned *u = &c.x;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int left_of = a.d - (e0 + x * 32 * N) - k * (N / 4);   // elements of this word
                        u[k] = left_of <= 0 ? 0u : N == 8 && left_of == 1 ? u[k] & 0xffffu : u[k];
                    }
                }
#pragma unroll
                for (int k = 0; k < N / 2; ++k) {
                    const uint64_t f = pair(c, k);
                    s2 = attn::fma2(q[x][k], f, s2);
                    m2 = attn::fma2(f, f, m2);
                }
            }
            float y, z;
            attn::split(s2, y, z);
            sum[j] = y + z;
            attn::split(m2, y, z);
            size[j] = y + z;
            nothing |= size[j] == 0.f;
        }
        if (__any_sync(~0u, nothing && e0 < a.d)) {   // squares that underflow are something; a mean of zeros alone has an exact score
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j)
#pragma unroll
                for (int x = 0; x < HALVES; ++x)
                {
                    const uint4 c = mean[(j * HALVES + x) * 32];   // (with what lies behind d: a bound may be larger)
                    if ((c.x | c.y | c.z | c.w) & (sizeof(T) == 2 ? 0x7fff7fffu : 0x7fffffffu)) size[j] += kTiny;
                }
        }
        // LANES lanes' sums of eight: halves of what is left are exchanged until each lane has one, which is then summed up
        int mine = 0;
#pragma unroll
        for (int x = LANES / 2, v = AT_ONCE; x; x >>= 1) {
            if (v > 1) {
                v >>= 1;
                const bool up = lane & x;
                mine += up ? v : 0;
#pragma unroll
                for (int j = 0; j < AT_ONCE / 2; ++j)
                    if (j < v) {
                        sum[j] = (up ? sum[j + v] : sum[j]) + __shfl_xor_sync(~0u, up ? sum[j] : sum[j + v], x);
                        size[j] = (up ? size[j + v] : size[j]) + __shfl_xor_sync(~0u, up ? size[j] : size[j + v], x);
                    }
            } else {
                sum[0] += __shfl_xor_sync(~0u, sum[0], x);
                size[0] += __shfl_xor_sync(~0u, size[0], x);
            }
        }
        const int k = mine * STEP + lane / LANES, page = __shfl_sync(~0u, held[0], k);
        if (lane % (LANES / AT_ONCE) == 0 && p0 + k < at.n) {
            // (a page that is none scores -inf)
            const bool none = (unsigned)page >= (unsigned)a.means.pages;
            const float off = size[0] == 0.f ? 0.f : fmaf(norm * sqrtf(fmaf(size[0], 1.0001f, kTiny)), kScoreOff, kUnderflow);
            scores[k] = none ? make_float2(-CUDART_INF_F, 0.f) : make_float2(sum[0], off);
        }
        if (--left == 0) return;
        fresh = step(at);
        summed = summed == kScoreAhead ? 0 : summed + 1;
#pragma unroll
        for (int x = 0; x < kScoreAhead; ++x) held[x] = held[x + 1];
    }
}

// The block's sum of c.  One barrier a count: two places take turns, so that a warp that is ahead writes where nobody still adds up.  So all counts between
// two barriers of other kinds go by one `turn`.
template <int WARPS> __device__ __forceinline__ int count_all(int c, int (&sums)[2][WARPS], int &turn)
{
    c = __reduce_add_sync(~0u, c);
    if (WARPS == 1) return c;
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) sums[turn][threadIdx.x >> 5] = c;
    __syncthreads();
    c = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) c += sums[turn][w];
    return c;
}
// The largest border with at least `want` of the numbers at or above it (in(j, to): whether this lane's j-th is), found bit by bit; at_least: how many are.  It
// ends early where that is `want`.
template <int WARPS, typename In>
__device__ __forceinline__ unsigned border_of(In in, int rounds, int want, int &at_least, int (&sums)[2][WARPS], int &turn)
{
    unsigned border = 0;
    for (int bit = 31; bit >= 0 && at_least != want; --bit) {
        const unsigned to = border | 1u << bit;
        int c = 0;
#pragma unroll
        for (int j = 0; j < rounds; ++j) c += in(j, to);
        c = count_all<WARPS>(c, sums, turn);
        if (c >= want) { border = to; at_least = c; }
    }
    return border;
}
// Enters those pages p0 + 32 j + lane of each warp in `list` that are over the border, and as many of those at it as there is room for, the lower ones
// first: `ties`, INT_MAX for all.
template <int WARPS, typename Over, typename Tie>
__device__ __forceinline__ void enter(Over over, Tie tie, int rounds, int p0, int p1, int ties, int *list, int (&sums)[2][WARPS])
{
    const int lane = threadIdx.x & 31, warp = WARPS == 1 ? 0 : threadIdx.x >> 5;
    int to = 0, tied = 0;
    if (WARPS > 1) {   // each warp first counts what the ones before it enter
        int mine = 0, mine_tied = 0;
#pragma unroll
        for (int j = 0; j < rounds; ++j) { mine += over(j); mine_tied += tie(j); }
        mine = __reduce_add_sync(~0u, mine);
        mine_tied = __reduce_add_sync(~0u, mine_tied);
        __syncthreads();
        if (lane == 0) { sums[0][warp] = mine; sums[1][warp] = mine_tied; }
        __syncthreads();
        for (int w = 0; w < warp; ++w) { to += sums[0][w]; tied += sums[1][w]; }
        to += min(tied, ties);
    }
#pragma unroll
    for (int j = 0; j < rounds; ++j) {
        if (p0 + j * 32 >= p1) break;
        const unsigned equal = __ballot_sync(~0u, tie(j)), below = (1u << lane) - 1;
        const bool take = tie(j) ? tied + __popc(equal & below) < ties : over(j);
        const unsigned taken = __ballot_sync(~0u, take);
        if (take) list[to + __popc(taken & below)] = p0 + j * 32 + lane;
        to += __popc(taken);
        tied += __popc(equal);
    }
}
// By keys of 64 bits in memory: first by their upper halves, then, among those that have that of the border, by their lower ones.  turn: of the caller's
// counts, which some warps may still be adding up.
template <int WARPS>
__device__ __noinline__ void select_exactly(const unsigned long long *keys, int n, int keep, int p0, int p1, int each, int *list, int (&sums)[2][WARPS], int turn)
{
    const int lane = threadIdx.x & 31, rounds = each / 32;
    const auto key = [&](int j) { const int p = p0 + j * 32 + lane; return p < p1 ? keys[p] : 0; };
    const auto high = [&](int j) { return (unsigned)(key(j) >> 32); };
    const auto low = [&](int j) { return (unsigned)key(j); };
    int at_least = n, ties = INT_MAX;
    unsigned lower = 0;
    const unsigned border = border_of<WARPS>([&](int j, unsigned to) { return high(j) >= to; }, rounds, keep, at_least, sums, turn);
    const auto count = [&](auto in) {
        int c = 0;
        for (int j = 0; j < rounds; ++j) c += in(j);
        return count_all<WARPS>(c, sums, turn);
    };
    if (at_least != keep) {
        const int above = count([&](int j) { return high(j) > border; }), want = keep - above;
        int same = at_least - above;
        // (keys that are not there are 0, which is below any `to`)
        lower = border_of<WARPS>([&](int j, unsigned to) { return high(j) == border && low(j) >= to; }, rounds, want, same, sums, turn);
        if (same != want) ties = want - count([&](int j) { return high(j) == border && low(j) > lower; });
    }
    const auto over = [&](int j) { return high(j) > border || (high(j) == border && low(j) > lower); };
    const auto tie = [&](int j) { return p0 + j * 32 + lane < p1 && high(j) == border && low(j) == lower; };
    enter<WARPS>(over, tie, rounds, p0, p1, ties, list, sums);
}

__device__ __forceinline__ unsigned ordered(float x)
{
    const unsigned u = __float_as_uint(x + 0.f);
    return u >> 31 ? ~u : u | 1u << 31;
}
__device__ __forceinline__ float from_ordered(unsigned u) { return __uint_as_float(u >> 31 ? u & 0x7fffffffu : ~u); }

// Pages next to the border, with their scores of 64 bits; in: whether those of 32 bits are at or above it.
constexpr int kNear = 32;
struct Few {
    unsigned long long key[kNear];
    int page[kNear], in[kNear], n;
};
// The best `keep` of a token's pages, WARPS warps per token and key head with up to KEYS pages a lane in registers (0: any number, read again each time).  Bound
// by latency: one for the scores, then about ten counts, each a few instructions a key and (several warps) a barrier: a border is looked for between the best
// score and one that `keep` reach surely, the least of the lanes' best where there are lanes enough.
template <typename T, int WARPS, int KEYS>
__device__ __forceinline__ void select_best(const SelectArgs<T> &a, int i, int g, int n, float2 *scores, int *list, int (&sums)[2][WARPS], unsigned (&ends)[6][WARPS], Few &few)
{
    const int lane = threadIdx.x & 31, warp = WARPS == 1 ? 0 : threadIdx.x >> 5, keep = a.keep;
    const int each = ((n + WARPS - 1) / WARPS + 31) & ~31, p0 = warp * each, p1 = min(n, p0 + each), rounds = KEYS ? KEYS : each / 32;   // this warp's pages
    const auto always = [&](int p) { return p < a.first || p >= n - a.last; };
    unsigned off = 0;   // the largest error's bits; those of a NaN or an infinity where a score or an error is one
    unsigned top = 0, bottom = ~0u;   // of this lane's scores
    const auto load = [&](int j) { return scores[min(p0 + j * 32 + lane, n - 1)]; };
    const auto key = [&](int j, float2 s) {
        const int p = p0 + j * 32 + lane;
        const bool scored = p < p1 && !always(p);
        const unsigned x = ordered(s.x);
        off = max(off, !scored ? 0u : s.x < CUDART_INF_F && (s.x > -CUDART_INF_F || s.y == 0.f) ? __float_as_uint(s.y) : 0x7f800000u);
        top = max(top, scored ? x : 0u);
        bottom = min(bottom, scored ? x : ~0u);
        return scored ? x : p < p1 ? ~0u : 0u;
    };
    unsigned held[KEYS ? KEYS : 1];
    if constexpr (KEYS > 0) {
#pragma unroll
        for (int j0 = 0; j0 < KEYS; j0 += 8) {   // (eight loads on their way)
            if (p0 + j0 * 32 >= p1) {
#pragma unroll
                for (int j = 0; j < 8; ++j) held[j0 + j] = 0;
                continue;
            }
            float2 s[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] = load(j0 + j);
#pragma unroll
            for (int j = 0; j < 8; ++j) held[j0 + j] = key(j0 + j, s[j]);
        }
    } else {
        for (int j = 0; j < rounds; ++j) key(j, load(j));
    }
    const auto at = [&](int j) { if constexpr (KEYS > 0) return held[j]; else return key(j, load(j)); };
    unsigned least = __reduce_min_sync(~0u, top);
    top = __reduce_max_sync(~0u, top);
    bottom = __reduce_min_sync(~0u, bottom);
    off = __reduce_max_sync(~0u, off);
    if (WARPS > 1) {
        if (lane == 0) { ends[0][warp] = least; ends[1][warp] = top; ends[2][warp] = bottom; ends[3][warp] = off; }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WARPS; ++w) { least = min(least, ends[0][w]); top = max(top, ends[1][w]); bottom = min(bottom, ends[2][w]); off = max(off, ends[3][w]); }
    }
    const bool all = off >= 0x7f800000u;   // nothing is known of the scores
    int turn = 0, at_least = a.first + a.last;
    unsigned border = ~0u;   // (of what is always taken)
    bool sure = at_least == keep && !all;
    float reach = 0.f, in = 0.f;
    if (!sure && !all) {
        const auto count = [&](unsigned to) {
            int c = 0;
#pragma unroll
            for (int j = 0; j < rounds; ++j) c += at(j) >= to;
            return count_all<WARPS>(c, sums, turn);
        };
        if (keep - at_least <= 32 * WARPS && least) {
            border = least;
            at_least = count(border);
        } else {
            border = bottom;
            at_least = n;
        }
        unsigned behind = top + 1;   // what is always taken is all that is left there
#pragma unroll 1
        for (int step = 0; at_least != keep && behind - border > 1; ++step) {
            // halves of the scores' range, then (a few far out) of the numbers'
            unsigned to = ordered(0.5f * from_ordered(border) + 0.5f * from_ordered(behind));
            if (step >= 12 || to <= border || to >= behind) to = border + (behind - border) / 2;
            const int c = count(to);
            if (c >= keep) { border = to; at_least = c; } else { behind = to; }
        }
        // the lowest score that is in, the highest that is not
        unsigned lowest = ~0u, highest = 0;
#pragma unroll
        for (int j = 0; j < rounds; ++j) {
            const unsigned x = at(j);
            if (x >= border) lowest = min(lowest, x); else highest = max(highest, x);
        }
        lowest = __reduce_min_sync(~0u, lowest);
        highest = __reduce_max_sync(~0u, highest);
        if (WARPS > 1) {
            if (lane == 0) { ends[4][warp] = lowest; ends[5][warp] = highest; }
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WARPS; ++w) { lowest = min(lowest, ends[4][w]); highest = max(highest, ends[5][w]); }
        }
        reach = 2.1f * __uint_as_float(off);
        in = from_ordered(lowest);
        sure = at_least == keep && in - from_ordered(highest) > reach;
    }
    unsigned long long flip = 0;   // bit j: this lane's j-th page is on the other side of the border than its score of 32 bits
    if (!sure) {
        // Pages within reach of the border get scores of 64 bits; those above are in, those below are out (keys that no score has).
        const float from = in - reach, to = in + reach;
        const auto close = [&](float s) { return s >= from && s <= to; };
        unsigned long long *keys = reinterpret_cast<unsigned long long *>(scores);
        const int group = a.heads / a.kv_heads;
        const int *table = a.t.entries + row_of(a.tok, i) * a.t.ld;
        const auto sync = [] { if (WARPS > 1) __syncthreads(); else __syncwarp(); };
        double q[8] = {};   // the sum of the group's queries, elements lane, lane + 32 ...
        if ((WARPS == 1 ? lane : threadIdx.x) == 0) few.n = 0;
        // (loops, not copies of them, here and below: hardly any token comes here, and what few do waits for each instruction)
        if constexpr (WARPS == 1) {
#pragma unroll 1
            for (int h = 0; h < group; ++h) {
                const T *from = a.q + i * a.q_ld + (g * group + h) * a.q_sh + lane;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (lane + 32 * e < a.d) q[e] += attn::widen(from[32 * e]);
            }
            __syncwarp();
        } else {
            __shared__ double sum[256];
#pragma unroll 1
            for (int e = threadIdx.x; e < a.d; e += WARPS * 32) {
                const T *from = a.q + i * a.q_ld + (long long)g * group * a.q_sh + e;
                double y = 0;
#pragma unroll 4
                for (int h = 0; h < group; ++h, from += a.q_sh) y += attn::widen(*from);
                sum[e] = y;
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (lane + 32 * e < a.d) q[e] = sum[lane + 32 * e];
        }
        // scores of 64 bits of those of a lane's pages that are to have one (all lanes call it; page p0 + 32 j + lane)
        const auto exact_of = [&](int j, bool again) {
            unsigned long long key = 0;
            for (unsigned left = __ballot_sync(~0u, again); left;) {
                int which[4];
                double x[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    which[k] = left ? __ffs(left) - 1 : -1;
                    left &= left - 1;
                    x[k] = 0;
                    const int held = which[k] < 0 ? -1 : table[p0 + j * 32 + which[k]];
                    if ((unsigned)held >= (unsigned)a.means.pages) { x[k] = lane ? 0 : -CUDART_INF; continue; }
                    const T *mean = a.means.row(held, g, 0);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (lane + 32 * e < a.d) x[k] += q[e] * attn::widen(mean[lane + 32 * e]);
                }
#pragma unroll
                for (int w = 16; w; w >>= 1)
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[k] += __shfl_xor_sync(~0u, x[k], w);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (which[k] == lane) key = ordered(x[k]);
            }
            return key;
        };
        int near = kNear + 1;
        if constexpr (KEYS > 0)
            if (!all) {
                unsigned long long next_to = 0;   // bit j: this lane's j-th page is next to the border
                const unsigned first = ordered(from), range = ordered(to) - first;   // (no other key lies between two scores)
#pragma unroll
                for (int j = 0; j < KEYS; ++j) next_to |= (unsigned long long)(held[j] - first <= range) << j;
                near = count_all<WARPS>(__popcll(next_to), sums, turn);
                if (near <= kNear) {   // the usual case: a few, each of which counts those that are before it
                    for (; next_to; next_to &= next_to - 1) few.page[atomicAdd(&few.n, 1)] = p0 + (__ffsll((long long)next_to) - 1) * 32 + lane;   // (in any order)
                    sync();
#pragma unroll 1
                    for (int x = 2 * warp; x < near; x += 2 * WARPS) {
                        double y[2] = {};
                        float2 s[2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const int p = few.page[min(x + k, near - 1)], held = table[p];
                            s[k] = scores[p];
                            const bool read = (unsigned)held < (unsigned)a.means.pages;
                            const T *mean = a.means.row(read ? held : 0, g, 0) + lane;
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (read && lane + 32 * e < a.d) y[k] += q[e] * attn::widen(mean[32 * e]);
                        }
#pragma unroll
                        for (int w = 16; w; w >>= 1) { y[0] += __shfl_xor_sync(~0u, y[0], w); y[1] += __shfl_xor_sync(~0u, y[1], w); }
                        if (lane < 2 && x + lane < near) {
                            const float2 z = lane ? s[1] : s[0];
                            few.key[x + lane] = ordered(z.y == 0.f ? (double)z.x : lane ? y[1] : y[0]);   // (exact, or no page)
                            few.in[x + lane] = ordered(z.x) >= border;
                        }
                    }
                    sync();
                    int above = at_least;
                    for (int x = 0; x < near; ++x) above -= few.in[x];
                    for (int x = 0; x < near; ++x) {
                        const int p = few.page[x];
                        if (p < p0 || p >= p1 || (p & 31) != lane) continue;
                        int before = above;
                        for (int y = 0; y < near; ++y) before += few.key[y] > few.key[x] || (few.key[y] == few.key[x] && few.page[y] < p);
                        if ((before < keep) != (bool)few.in[x]) flip |= 1ull << (p - p0) / 32;
                    }
                }
            }
        if (near > kNear) {
            for (int j = 0; j < each / 32; ++j) {
                const int p = p0 + j * 32 + lane;
                unsigned long long key = 0;
                bool again = false;
                if (p < p1) {
                    const float2 s = scores[p];
                    again = !always(p) && (all || close(s.x));
                    key = always(p) || (!all && s.x > to) ? ~0ull : 0;
                    if (again && !all && s.y == 0.f) { key = ordered((double)s.x); again = false; }   // (exact, or no page)
                }
                const unsigned long long exact = exact_of(j, again);
                if (again) key = exact;
                if (p < p1) keys[p] = key;
            }
            __syncwarp();   // (a warp's keys are read by itself alone)
            select_exactly<WARPS>(keys, n, keep, p0, p1, each, list, sums, turn);
            return;
        }
    }
    enter<WARPS>([&](int j) { bool in = at(j) >= border; if constexpr (KEYS > 0) in ^= flip >> j & 1; return in; }, [](int) { return false; }, rounds, p0, p1, INT_MAX, list, sums);
}

// WARPS = 1: a CTA has four tokens and key heads (CTAs of one warp take longer to come and go than the choice).  MOST: most pages of a lane in registers;
// early: the launch ahead is that of the scores, whose CTAs have all waited for what made the tokens' numbers and read the lists before they let this one begin.
template <typename T, int WARPS, int MOST>
__global__ void __launch_bounds__(WARPS == 1 ? 128 : WARPS * 32) paged_select_kernel(const SelectArgs<T> a, bool early)
{
    constexpr int UNITS = WARPS == 1 ? 4 : 1;
    __shared__ int sums[2][WARPS];
    __shared__ unsigned ends[6][WARPS];
    __shared__ Few few_of[UNITS];
    if (!early) asm volatile("griddepcontrol.wait;" ::: "memory");
    const int mine = UNITS == 1 ? 0 : threadIdx.x >> 5, thread = UNITS == 1 ? threadIdx.x : threadIdx.x & 31;
    const int unit = blockIdx.x * UNITS + mine, units = a.M * a.kv_heads;
    Few &few = few_of[mine];
    const int i = unit / a.kv_heads, g = unit - i * a.kv_heads, n = unit < units ? pages_seen(a, i) : 0;
    int *list = a.lists + (long long)unit * a.keep;
    if (unit < units)
        for (int p = thread; p < a.keep; p += WARPS * 32)
            if (p >= n) list[p] = -1; else if (n <= a.keep) list[p] = p;
    if (early) asm volatile("griddepcontrol.wait;" ::: "memory");
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.status = 0;
    if (n <= a.keep) return;
    float2 *scores = a.scores + (long long)unit * a.t.width;
    if (MOST == 8 || n <= 256 * WARPS) select_best<T, WARPS, 8>(a, i, g, n, scores, list, sums, ends, few);
    else if (n <= 1024 * WARPS) select_best<T, WARPS, 32>(a, i, g, n, scores, list, sums, ends, few);
    else if (n <= 2048 * WARPS) select_best<T, WARPS, 64>(a, i, g, n, scores, list, sums, ends, few);
    else select_best<T, WARPS, 0>(a, i, g, n, scores, list, sums, ends, few);
}
}  // namespace paged
}  // namespace b2sp
