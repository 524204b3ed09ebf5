// A cache of keys or values in pages, in the operands' own type: its tables, lists of its slots, writing into it, and the choice of pages
// by a cheap score.  Attention over it is in paged_attention.cuh.
//
// Request r's position p lies in row p % page of page tables[r][p / page].  Everything that says how much there is to do (lengths, new tokens,
// tables) is on the device, so a launch is sized by what the host knows (requests, tokens, width of the tables) and the kernels find their
// work themselves: each CTA forms the prefix sums over the requests that it needs, which costs it a microsecond and spares a launch.
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
// Bound by latency: lengths, then (tokens) a table entry or a free page; 64 requests and 512 with 16384 new tokens: see the launch.
__global__ void __launch_bounds__(kThreads) paged_tables_kernel(const TablesArgs a)
{
    extern __shared__ int prefix[];
    __shared__ long long warps[kThreads / 32];
    const int R = a.t.requests, each = (R + kThreads - 1) / kThreads, r0 = min(R, (int)threadIdx.x * each), r1 = min(R, r0 + each);
    int *take = prefix, *back = prefix + R + 1, *ptr = prefix + 2 * (R + 1);
    long long n_take = 0, n_back = 0, n_new = 0, all_take, all_back, all_new;
    for (int r = r0; r < r1; ++r) {
        const Request q = request(a, r);
        n_take += q.need; n_back += q.back; n_new += q.fresh;
    }
    n_take = block_before(n_take, warps, all_take);
    n_back = block_before(n_back, warps, all_back);
    n_new = block_before(n_new, warps, all_new);
    const int count = min(max(*a.free_count, 0), a.free_room);
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
    const long long me = blockIdx.x * (long long)kThreads + threadIdx.x, all = gridDim.x * (long long)kThreads;
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
constexpr int kScanThreads = 1024;
__global__ void __launch_bounds__(kScanThreads) paged_list_ends_kernel(const ListsArgs a)
{
    __shared__ long long warps[kScanThreads / 32];
    const int each = (a.M + kScanThreads - 1) / kScanThreads, i0 = (int)min((long long)a.M, threadIdx.x * (long long)each), i1 = min(a.M, i0 + each);
    long long n = 0, all;
    for (int i = i0; i < i1; ++i) n += seen_of(a.tok, a.t, a.page, i);
    n = block_before(n, warps, all);
    for (int i = i0; i < i1; ++i) {
        a.row_ptr[i] = (int)min(n, a.entries);
        n += seen_of(a.tok, a.t, a.page, i);
    }
    if (threadIdx.x == 0) a.row_ptr[a.M] = (int)min(all, a.entries);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
// A warp takes kListShare neighbouring entries.  32 ends of rows are in its lanes at a time; an entry's row is found among them by five shuffles, so
// rows of one entry cost what rows of many do.  Bound by the stores.
constexpr int kListShare = 512;
__global__ void __launch_bounds__(kThreads) paged_list_kernel(const ListsArgs a)
{
    const int lane = threadIdx.x & 31;
    const long long lo = (blockIdx.x * (long long)(kThreads / 32) + (threadIdx.x >> 5)) * kListShare, hi = min(lo + kListShare, a.entries);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (lo >= hi) return;
    const int all = a.row_ptr[a.M];
    // the first row that ends behind lo (M if none does), by 32 probes at a time
    int base = 0;
    for (int len = a.M; len > 0;) {   // it lies in [base, base + len]
        const int step = (len + 31) / 32, at = base + lane * step;
        const bool inside = lane * (long long)step < len;
        const unsigned behind = __ballot_sync(~0u, inside && a.row_ptr[at + 1] > lo), probes = __ballot_sync(~0u, inside);
        const int k = behind ? __ffs(behind) - 1 : __popc(probes);   // probes before k end at or before lo
        if (k == 0) break;
        const int past = (k - 1) * step + 1;
        len = (behind ? k * step : len) - past;
        base += past;
    }
    int end = 0, start = 0;
    const auto window = [&](int at) {   // lane: start and end of row at + lane
        const int i = min(at + lane, a.M);
        start = a.row_ptr[i];
        end = at + lane < a.M ? a.row_ptr[i + 1] : INT_MAX;
    };
    window(base);
    for (long long e0 = lo; e0 < hi; e0 += 32) {
        const int e = (int)min(e0 + lane, (long long)INT_MAX);
        int slot = -1;
        bool open = e0 + lane < hi && e < all;
        while (__any_sync(~0u, open)) {
            int k = 0;   // ends at or before e among the 32
#pragma unroll
            for (int s = 16; s; s >>= 1) {
                const int y = __shfl_sync(~0u, end, k + s - 1);
                if (y <= e) k += s;
            }
            const int last = __shfl_sync(~0u, end, 31), k1 = min(k, 31);
            if (k == 31 && last <= e) k = 32;
            const int first = __shfl_sync(~0u, start, k1);
            if (open && k < 32) {
                const int i = base + k, p = e - first;
                const int c = (int)a.by_page((unsigned)p), held = a.t.entries[(long long)row_of(a.tok, i) * a.t.ld + c];
                if ((unsigned)held < (unsigned)a.pages) slot = held * a.page + (p - c * a.page);
                open = false;
            }
            if (__any_sync(~0u, open)) { base += 32; window(base); }
        }
        if (e0 + lane < hi) a.col_idx[e0 + lane] = slot;
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
constexpr int kWriteThreads = 128;
template <typename T>
__global__ void __launch_bounds__(kWriteThreads) paged_write_kernel(const WriteArgs<T> a)
{
    using C = Chunk<T>;
    extern __shared__ int prefix[];   // [R + 1] touched pages before request r
    __shared__ long long warps[kWriteThreads / 32];
    __shared__ float sums[kWriteThreads][C::N];
    const int R = a.t.requests, each = (R + kWriteThreads - 1) / kWriteThreads, r0 = min(R, (int)threadIdx.x * each), r1 = min(R, r0 + each);
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
                for (int i = (means ? 0 : old) + group; i < end; i += groups) {
                    C y;
                    if (i < old) {
                        y.load(a.kp.row(held, h, i), e, a.d, whole);
                    } else {
                        y.load(k + i * a.k_ld, e, a.d, k_wide && whole);
                        y.store(a.kp.row(held, h, i), e, a.d);
                        C z;
                        z.load(v + i * a.v_ld, e, a.d, v_wide && whole);
                        z.store(a.vp.row(held, h, i), e, a.d);
                    }
                    if (means) y.add_to(x);
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
    Pages<T> means;
    unsigned long long *keys;   // [M][kv_heads][width]
    int *lists;                 // [M][kv_heads][keep]
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

// Scores: a warp per 32 pages of a token and key head, the sum of the group's queries in its lanes.  Sums are formed in 64 bits: the result is a
// choice, and between two close scores sums of 32 bits would choose by their order.
constexpr int kScorePages = 32;
template <typename T>
__global__ void __launch_bounds__(kThreads) paged_score_kernel(const SelectArgs<T> a)
{
    const int lane = threadIdx.x & 31, blocks = (a.t.width + kScorePages - 1) / kScorePages;
    const long long unit = blockIdx.x * (long long)(kThreads / 32) + (threadIdx.x >> 5);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (unit >= (long long)a.M * a.kv_heads * blocks) return;
    const int b = (int)(unit % blocks), g = (int)(unit / blocks % a.kv_heads), i = (int)(unit / blocks / a.kv_heads);
    const int n = pages_seen(a, i), p0 = b * kScorePages, p1 = min(n, p0 + kScorePages);
    if (n <= a.keep || p0 >= n) return;
    const int *table = a.t.entries + row_of(a.tok, i) * a.t.ld;
    const int group = a.heads / a.kv_heads;
    unsigned long long *keys = a.keys + ((long long)i * a.kv_heads + g) * a.t.width;
    for (int p = p0; p < p1; ++p) {
        const int held = table[p];
        double x = 0;
        if ((unsigned)held < (unsigned)a.means.pages) {
            const T *mean = a.means.row(held, g, 0);
            for (int e = lane; e < a.d; e += 32) {
                double q = 0;
                for (int h = 0; h < group; ++h) q += attn::widen(a.q[i * a.q_ld + (g * group + h) * a.q_sh + e]);
                x += q * attn::widen(mean[e]);
            }
#pragma unroll
            for (int w = 16; w; w >>= 1) x += __shfl_xor_sync(~0u, x, w);
        } else {
            x = -CUDART_INF;
        }
        if (lane == 0) keys[p] = ordered(x);
    }
}

// The best `keep` of a token's pages, a CTA per token and key head.  The keep-th largest key is found bit by bit from the first in which the keys differ,
// each time by counting the keys that are at least as large; it ends early where exactly `keep` are.  A thread holds neighbouring pages, so
// that ties and the ascending order of the list follow from prefix sums over the threads.
constexpr int kHeld = 8;   // keys of a thread in registers; those behind are read again for each bit
template <typename T>
__global__ void __launch_bounds__(kThreads) paged_select_kernel(const SelectArgs<T> a)
{
    constexpr int W = kThreads / 32;
    __shared__ unsigned long long ands[W], ors[W];
    __shared__ int counts[2][W];
    __shared__ long long warps[W];
    const int i = blockIdx.x / a.kv_heads, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n = pages_seen(a, i);
    int *list = a.lists + (long long)blockIdx.x * a.keep;
    for (int p = threadIdx.x; p < a.keep; p += kThreads)
        if (p >= n) list[p] = -1; else if (n <= a.keep) list[p] = p;
    asm volatile("griddepcontrol.wait;" ::: "memory");   // (by all CTAs: what comes behind this launch counts on the one ahead of it)
    if (n <= a.keep) return;
    const unsigned long long *keys = a.keys + (long long)blockIdx.x * a.t.width;
    const int each = (n + kThreads - 1) / kThreads, p0 = (int)min((long long)n, threadIdx.x * (long long)each), mine = min(n - p0, each);
    const auto key = [&](int p) { return p < a.first || p >= n - a.last ? ~0ull : keys[p]; };
    unsigned long long held[kHeld];
#pragma unroll
    for (int j = 0; j < kHeld; ++j) held[j] = j < mine ? key(p0 + j) : 0;
    unsigned long long all_and = ~0ull, all_or = 0;
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
        if (j < mine) { all_and &= held[j]; all_or |= held[j]; }
    for (int j = kHeld; j < mine; ++j) { all_and &= key(p0 + j); all_or |= key(p0 + j); }
#pragma unroll
    for (int w = 16; w; w >>= 1) { all_and &= __shfl_xor_sync(~0u, all_and, w); all_or |= __shfl_xor_sync(~0u, all_or, w); }
    if (lane == 0) { ands[warp] = all_and; ors[warp] = all_or; }
    __syncthreads();
    for (int w = 0; w < W; ++w) { all_and &= ands[w]; all_or |= ors[w]; }
    const auto count = [&](auto &&inside, int turn) {
        int c = 0;
#pragma unroll
        for (int j = 0; j < kHeld; ++j) c += j < mine && inside(held[j]);
        for (int j = kHeld; j < mine; ++j) c += inside(key(p0 + j));
        c = __reduce_add_sync(~0u, c);
        if (lane == 0) counts[turn & 1][warp] = c;
        __syncthreads();
        c = 0;
        for (int w = 0; w < W; ++w) c += counts[turn & 1][w];
        return c;
    };
    unsigned long long border = all_and;   // the bits above the first difference; then the largest border with at least keep keys above or at it
    int at_least = n, turn = 0;
    const unsigned long long differ = all_and ^ all_or;
    for (int bit = differ ? 63 - __clzll((long long)differ) : -1; bit >= 0 && at_least != a.keep; --bit, ++turn) {
        if (turn == 0) border = all_and >> bit << bit;   // (this bit is zero in it)
        const unsigned long long to = border | 1ull << bit;
        const int c = count([&](unsigned long long x) { return x >= to; }, turn);
        if (c >= a.keep) { border = to; at_least = c; }
    }
    // all above the border, and as many at it as there is room for, the lower pages first
    int above = 0, at = 0;
#pragma unroll
    for (int j = 0; j < kHeld; ++j) { above += j < mine && held[j] > border; at += j < mine && held[j] == border; }
    for (int j = kHeld; j < mine; ++j) { above += key(p0 + j) > border; at += key(p0 + j) == border; }
    long long total_above, total;
    block_before(above, warps, total_above);
    const long long at_before = block_before(at, warps, total);
    const int room = (int)min(max((long long)a.keep - total_above - at_before, 0ll), (long long)at);   // of this thread's
    int to = (int)block_before(above + room, warps, total), left = room;
    const auto enter = [&](int j, unsigned long long x) {
        if (x > border || (x == border && left-- > 0)) list[to++] = p0 + j;
    };
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
        if (j < mine) enter(j, held[j]);
    for (int j = kHeld; j < mine; ++j) enter(j, key(p0 + j));
}
}  // namespace paged
}  // namespace b2sp
