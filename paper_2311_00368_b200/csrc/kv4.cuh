// A cache of keys or values held in 4 bits: writing, reading, and attention over it.
//
// Format of one row (one token, one head) of d elements, G = ceil(d / 32) groups of 32 neighbours:
//   scale of group c     s_c = bf16(max |x| / 7), a bf16; the quotient in fp32, both roundings to nearest even
//   code of an element   clamp(rint(x / s_c), -7, 7) + 8, in 4 bits (8 where s_c = 0, and in the tail behind d)
//   codes in memory      8 G halfwords: halfword g G + c holds elements 32 c + 4 g + {0, 1, 2, 3}, the first in the lowest bits
// 18 bytes per group.  A group with a NaN or an infinity has the scale NaN: reading it gives NaN.
// The order of the halfwords is what the attention kernel loads: lane g of eight finds its four elements of every group in 2 G
// neighbouring bytes (as a column of V), and two such pieces make a lane of four's share of every group (as a row of K).
#pragma once
#include <math_constants.h>

#include <type_traits>

#include "attention_rows.cuh"

namespace b2sp {
namespace kv4 {

using attn::Bf16;

struct Cache {
    uint8_t *codes;      // row (h, slot): codes + h * code_head + slot * code_ld, bytes
    Bf16 *scales;        // scales + h * scale_head + slot * scale_ld, elements
    long long code_ld, code_head, scale_ld, scale_head;
    int slots;
};

// n / d for 0 <= n < 2^31 by one multiplication (Granlund and Montgomery's round-up method).
struct Div {
    unsigned d, m, s;
    Div() = default;
    explicit Div(unsigned d_) : d(d_), s(0)
    {
        while ((1ull << s) < d) ++s;
        m = (unsigned)(((1ull << 32) * ((1ull << s) - d)) / d + 1);
    }
    __device__ __forceinline__ unsigned operator()(unsigned n) const { return (__umulhi(n, m) + n) >> s; }
};

// Slots that several tokens name take the last one's row.  Up to kScanTokens tokens a CTA of the writing kernel compares its tokens' slots
// with those of all later tokens; more go through an owner per slot in the workspace (two small launches ahead of the writing one: the owners of
// the slots named become -1, then the largest token): 16384 tokens cost 4 us this way, and the comparisons would be 1.3e8.
constexpr int kScanTokens = 1024, kWriteThreads = 256;

__global__ void __launch_bounds__(256) kv4_disown_kernel(const int *slots, int tokens, int cache_slots, int *owner)
{
    const int t = blockIdx.x * 256 + threadIdx.x;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (t < tokens && (unsigned)slots[t] < (unsigned)cache_slots) owner[slots[t]] = -1;
}
__global__ void __launch_bounds__(256) kv4_own_kernel(const int *slots, int tokens, int cache_slots, int *owner)
{
    const int t = blockIdx.x * 256 + threadIdx.x, s = t < tokens ? slots[t] : -1;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if ((unsigned)s < (unsigned)cache_slots) atomicMax(owner + s, t);
}

// Eight neighbours of a row; V = 8: 16-byte loads (bf16: one, fp32: two), else element by element.
template <typename T, int V> __device__ __forceinline__ void load8(const T *row, int c, int d, float (&x)[8])
{
    if (V == 8) {
        if (c >= d) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.f;
        } else if constexpr (sizeof(T) == 2) {
            const uint4 u = *reinterpret_cast<const uint4 *>(row + c);
            const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        } else {
            const float4 a = *reinterpret_cast<const float4 *>(row + c), b = *reinterpret_cast<const float4 *>(row + c + 4);
            x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = c + i < d ? attn::widen(row[c + i]) : 0.f;
    }
}
template <typename T, int V> __device__ __forceinline__ void store8(T *row, int c, int d, const float (&x)[8])
{
    if (V == 8) {
        if (c >= d) return;
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint4 *>(row + c) = make_uint4(attn::bf16x2(x[0], x[1]), attn::bf16x2(x[2], x[3]), attn::bf16x2(x[4], x[5]), attn::bf16x2(x[6], x[7]));
        } else {
            *reinterpret_cast<float4 *>(row + c) = make_float4(x[0], x[1], x[2], x[3]);
            *reinterpret_cast<float4 *>(row + c + 4) = make_float4(x[4], x[5], x[6], x[7]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < d) attn::narrow(x[i], row[c + i]);
    }
}

struct RowsArgs {
    int tokens, heads, d, G;
    long long ld, sh;        // of the rows in 16 or 32 bits
    const int *slots;
    Cache c;
    Div by_head, by_piece;   // divisors: heads, and the pieces of a row that threads take (write: 4 G quarters of groups; read: ceil(d / 8))
    unsigned first;          // (token, head) rows of earlier launches
    int *owner;              // write: NULL with few tokens
};

// Four lanes per group, eight elements each.  What bounds it is memory: 2 d bytes in, 18 G out; one thread per 16 bytes in flight.
template <typename T, int V, bool SCAN>
__global__ void __launch_bounds__(kWriteThreads) kv4_write_kernel(const T *x, const RowsArgs a)
{
    __shared__ int gone[kWriteThreads / 4];   // SCAN: which of the CTA's tokens a later one replaces
    const unsigned u = blockIdx.x * (unsigned)kWriteThreads + threadIdx.x;
    const unsigned row = a.by_piece(u), piece = u - row * a.by_piece.d, t = a.by_head(row), h = row - t * a.by_head.d;
    const bool on = t < (unsigned)a.tokens;
    const int slot = on ? a.slots[t] : -1;
    const int grp = piece >> 2, j = piece & 3;
    const bool live = (unsigned)slot < (unsigned)a.c.slots;
    float v[8] = {};
    if (live) load8<T, V>(x + (long long)t * a.ld + (long long)h * a.sh, grp * 32 + j * 8, a.d, v);
    const unsigned t0 = a.by_head(a.by_piece(blockIdx.x * (unsigned)kWriteThreads));
    if (SCAN) {
        const unsigned t1 = min((unsigned)a.tokens - 1, a.by_head(a.by_piece(blockIdx.x * (unsigned)kWriteThreads + kWriteThreads - 1)));
        if (threadIdx.x < kWriteThreads / 4) gone[threadIdx.x] = 0;
        __syncthreads();
        for (unsigned k = t0 + 1 + threadIdx.x; k < (unsigned)a.tokens; k += kWriteThreads) {
            const int s = a.slots[k];
            for (unsigned i = t0; i <= t1 && i < k; ++i)
                if (a.slots[i] == s) gone[i - t0] = 1;
        }
        __syncthreads();
    }
    float top = 0.f;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        top = fmaxf(top, fabsf(v[i]));
        odd |= !(fabsf(v[i]) <= 3.402823466e38f);
    }
    top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
    top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
    odd = __ballot_sync(~0u, odd) >> (threadIdx.x & 28) & 15;
    Bf16 s;
    attn::narrow(__fdiv_rn(top, 7.f), s);
    if (odd) s.bits = 0x7fff;
    const float f = attn::widen(s);
    unsigned word[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = f > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(v[i], f)), -7.f), 7.f) : 0.f;
        word[i >> 2] |= (unsigned)((int)q + 8) << (4 * (i & 3));
    }
    bool keep = live;
    if (SCAN) {
        keep = live && !gone[t - t0];
    } else {
        asm volatile("griddepcontrol.wait;" ::: "memory");   // the owners
        if (live) keep = a.owner[slot] == (int)t;
    }
    if (!keep) return;
    unsigned short *codes = reinterpret_cast<unsigned short *>(a.c.codes + (long long)h * a.c.code_head + (long long)slot * a.c.code_ld);
    codes[(2 * j) * a.G + grp] = (unsigned short)word[0];
    codes[(2 * j + 1) * a.G + grp] = (unsigned short)word[1];
    if (j == 0) a.c.scales[(long long)h * a.c.scale_head + (long long)slot * a.c.scale_ld + grp] = s;
}

// A thread per eight elements of the output; rows of slots outside the cache read as zeros.
template <typename T, int V>
__global__ void __launch_bounds__(256) kv4_read_kernel(const RowsArgs a, T *out)
{
    const unsigned u = blockIdx.x * 256u + threadIdx.x;
    unsigned row = a.by_piece(u);
    const int e = (int)(u - row * a.by_piece.d), grp = e >> 2, j = e & 3;
    row += a.first;
    const unsigned t = a.by_head(row), h = row - t * a.by_head.d;
    if (t >= (unsigned)a.tokens) return;
    const int slot = a.slots[t];
    float v[8] = {};
    if ((unsigned)slot < (unsigned)a.c.slots) {
        const unsigned short *codes = reinterpret_cast<const unsigned short *>(a.c.codes + (long long)h * a.c.code_head + (long long)slot * a.c.code_ld);
        const unsigned w0 = codes[(2 * j) * a.G + grp], w1 = codes[(2 * j + 1) * a.G + grp];
        const float s = attn::widen(a.c.scales[(long long)h * a.c.scale_head + (long long)slot * a.c.scale_ld + grp]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = s * (float)((int)(w0 >> (4 * i) & 15) - 8);
            v[4 + i] = s * (float)((int)(w1 >> (4 * i) & 15) - 8);
        }
    }
    store8<T, V>(out + (long long)t * a.ld + (long long)h * a.sh, e * 8, a.d, v);
}

// ---- attention ------------------------------------------------------------------------------------------------------------------
struct AttnArgs {
    int M, heads, kv_heads, d, splits, head_blocks;   // head_blocks: eights (or sixteens, NB = 2) of query heads that share one K and V
    const int *row_ptr, *col_idx;
    const Bf16 *q;
    long long q_ld, q_sh;
    Cache k, v;
    float scale;
    attn::View<Bf16> out;
    float *lse, *part;
    float2 *part_ml;
};

__device__ __forceinline__ void mma_bf16(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 128 + code of nibble I of both halves, as two bf16 (exact: bf16 holds whole numbers up to 256)
template <int I> __device__ __forceinline__ unsigned nibble_pair(unsigned y)
{
    return ((y >> (4 * I)) & 0x000f000fu) | 0x43004300u;
}
__device__ __forceinline__ unsigned minus136(unsigned x)   // (128 + code) - 136, exact
{
    unsigned r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(0x43084308u));
    return r;
}
__device__ __forceinline__ void cp_async(unsigned dst, const void *src, int bytes, int keep)
{
    if (bytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(keep) : "memory");
    else if (bytes == 8) asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(keep) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(keep) : "memory");
}

__device__ __forceinline__ unsigned transpose8(unsigned x)   // an 8 x 8 matrix of 16-bit elements over a warp
{
    unsigned r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// O = softmax(scale Q K^T) V of one query token's heads over (a part of) the slots that its row names.
//
// A CTA takes one token, one key/value head with up to 8 NB query heads that share it, and one part of the row; its four warps take
// every fourth 16 slots each and join at the end.  What it has to read is 36 G bytes a slot, so everything is done to keep loads in
// flight and instructions few: a ring of kStages tiles per warp filled by cp.async; codes become bf16 by one mask each (128 + code);
// the tensor core's legacy form multiplies them (m16n8k16: 16 slots of K by 8 query heads, then 16 elements of V by 8 query heads), the weights
// pass from the one product's layout to the other's by movmatrix.
//   * K: the row scale of a group multiplies the products of its 32 elements, in fp32; the 136 that each code carries too much is
//     taken off there as 136 sum(q), instead of off each code.
//   * V: the scale of (slot, group) multiplies the slot's weight before that is rounded to bf16 (half a step, 2^-8 of each weight --
//     the one rounding of this kernel beside that of the output); codes are made whole numbers -7 .. 7 first, as the sum over slots
//     would lose the small result in 136 sum(p).
//   * the running maximum moves only when a logit exceeds it by 8 (to base 2), so that O is rarely rescaled: weights up to 2^8.
// Slot r of a tile is row r of the first product; V's rows lie in the order (r & 1) * 4 + r / 2 of each half tile, so that the four lanes of
// a column of V read different banks.
constexpr int kStages = 4, kSlots = 16;
template <int G, int NB> struct Smem {
    static constexpr int ROW = 16 * G;
    static constexpr int K = 0, V = kSlots * ROW, KS = 2 * kSlots * ROW, VS = KS + kSlots * 8, IDX = VS + kSlots * 8, STAGE = IDX + kSlots * 4;
    static constexpr int RING = attn::kWarps * kStages * STAGE;
    static constexpr int JOIN = attn::kWarps * (8 * NB * 32 * G + 16 * NB) * 4;
    static constexpr int BYTES = RING > JOIN ? RING : JOIN;
};

// N halfwords at p (aligned as they lie), two to a word.
template <int N, int ALIGN> __device__ __forceinline__ void lds_halves(const char *p, unsigned (&w)[(N + 1) / 2])
{
    if constexpr (N == 8) { const uint4 u = *reinterpret_cast<const uint4 *>(p); w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w; }
    else if constexpr (N == 4) { const uint2 u = *reinterpret_cast<const uint2 *>(p); w[0] = u.x; w[1] = u.y; }
    else if constexpr (ALIGN == 4) {
#pragma unroll
        for (int i = 0; i < (N + 1) / 2; ++i) w[i] = reinterpret_cast<const unsigned *>(p)[i];
    } else {
        const unsigned short *h = reinterpret_cast<const unsigned short *>(p);
#pragma unroll
        for (int i = 0; i < (N + 1) / 2; ++i) w[i] = h[2 * i] | (2 * i + 1 < N ? (unsigned)h[2 * i + 1] << 16 : 0u);
    }
}
// Halfword A of a below halfword B of b.
template <int A, int B, int N> __device__ __forceinline__ unsigned pick(const unsigned (&a)[N], const unsigned (&b)[N])
{
    constexpr unsigned lo = (A & 1) ? 0x32 : 0x10, hi = (B & 1) ? 0x76 : 0x54;
    return __byte_perm(a[A / 2], b[B / 2], hi << 8 | lo);
}
template <int G> __device__ __forceinline__ void lds_scales(const char *p, int odd, float (&s)[G])
{
    if constexpr (G == 4) {
        const uint2 u = *reinterpret_cast<const uint2 *>(p);
        s[0] = __uint_as_float(u.x << 16); s[1] = __uint_as_float(u.x & 0xffff0000u);
        s[2] = __uint_as_float(u.y << 16); s[3] = __uint_as_float(u.y & 0xffff0000u);
    } else if constexpr (G == 2) {
        const unsigned u = *reinterpret_cast<const unsigned *>(p);
        s[0] = __uint_as_float(u << 16); s[1] = __uint_as_float(u & 0xffff0000u);
    } else {
#pragma unroll
        for (int c = 0; c < G; ++c) s[c] = __uint_as_float((unsigned)reinterpret_cast<const unsigned short *>(p)[odd + c] << 16);
    }
}
// f(std::integral_constant<int, i>) for i = 0 .. N - 1
template <int N, int I = 0, class F> __device__ __forceinline__ void each(F &&f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<N, I + 1>(f);
    }
}

template <int G, int NB>
__global__ void __launch_bounds__(attn::kWarps * 32, NB == 1 ? 4 : 3) kv4_attention_kernel(const AttnArgs a)
{
    using S = Smem<G, NB>;
    __shared__ __align__(16) char smem[S::BYTES];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int group = a.heads / a.kv_heads;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (the joining kernel waits for this grid's end where it reads)
    long long u = blockIdx.x;
    const int part = (int)(u % a.splits); u /= a.splits;
    const int hb = (int)(u % a.head_blocks); u /= a.head_blocks;
    const int hkv = (int)(u % a.kv_heads), row = (int)(u / a.kv_heads);
    const int first = a.row_ptr[row], last = a.row_ptr[row + 1], per = attn::part_len(last - first, a.splits);
    const long long begin = first + (long long)part * per;
    if (part && begin >= last) return;
    const int n = (int)min((long long)per, last - begin);
    const int *idx = a.col_idx + begin;
    const int tiles = (n + kSlots - 1) / kSlots, mine = tiles > warp ? (tiles - warp + attn::kWarps - 1) / attn::kWarps : 0;
    char *ring = smem + warp * kStages * S::STAGE;
    const unsigned ring_s = (unsigned)__cvta_generic_to_shared(ring);
    const uint8_t *kc = a.k.codes + hkv * a.k.code_head, *vc = a.v.codes + hkv * a.v.code_head;
    const Bf16 *ksc = a.k.scales + hkv * a.k.scale_head, *vsc = a.v.scales + hkv * a.v.scale_head;
    const int slots = min(a.k.slots, a.v.slots);

    auto fetch_idx = [&](int i) {   // the slot of lane & 15 of this warp's tile i, or -1
        const int at = (warp + i * attn::kWarps) * kSlots + (lane & 15);
        const int s = i < mine && at < n ? idx[at] : -1;
        return (unsigned)s < (unsigned)slots ? s : -1;
    };
    auto issue = [&](int i, int slot) {
        if (i < mine) {
            const int st = (i % kStages) * S::STAGE;
#pragma unroll
            for (int c = 0; c < G; ++c) {
                const int id = c * 32 + lane;
                const bool is_v = id >= kSlots * G;
                const int in = is_v ? id - kSlots * G : id, r = in / G, ch = in % G;
                const int s = __shfl_sync(~0u, slot, r);
                const uint8_t *src = is_v ? vc + (long long)max(s, 0) * a.v.code_ld : kc + (long long)max(s, 0) * a.k.code_ld;
                const int vrow = (r & 8) | ((r & 1) << 2) | (r >> 1 & 3);
                const int dst = is_v ? S::V + vrow * S::ROW + (G == 4 ? ch ^ (vrow & 2) : ch) * 16 : S::K + r * S::ROW + ch * 16;
                cp_async(ring_s + st + dst, src + ch * 16, 16, s >= 0 ? 16 : 0);
            }
            {
                const int r = lane & 15;
                const bool is_v = lane >= 16;
                const long long at = (long long)max(slot, 0) * (is_v ? a.v.scale_ld : a.k.scale_ld);
                const Bf16 *src = (is_v ? vsc : ksc) + at;
                const unsigned dst = ring_s + st + (is_v ? S::VS : S::KS) + r * 8;
                if constexpr (G == 4) cp_async(dst, src, 8, slot >= 0 ? 8 : 0);
                else if constexpr (G == 2) cp_async(dst, src, 4, slot >= 0 ? 4 : 0);
                else {   // whole words around an odd number of halfwords; bytes behind the row are not read
                    const int off = (int)(reinterpret_cast<uintptr_t>(src) & 2);
                    const char *p = reinterpret_cast<const char *>(src) - off;
                    const int bytes = off + 2 * G;
                    cp_async(dst, p, 4, slot >= 0 ? min(bytes, 4) : 0);
                    if (G == 3) cp_async(dst + 4, p + 4, 4, slot >= 0 ? bytes - 4 : 0);
                }
                if (lane < 16) *reinterpret_cast<int *>(ring + st + S::IDX + r * 4) = slot;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };

    // The first tiles are on their way while Q is read.  Q: lane (g, t) has elements 8 t .. 8 t + 7 of each group of query head g (of each eight)
    int next = fetch_idx(0);
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) {
        const int now = next;
        next = fetch_idx(i + 1);
        issue(i, now);
    }
    unsigned qa[G][2][2][NB];   // [group][k step][half of k]
    float qsum[G][NB][2];       // 136 times the sum over the group, of query heads 2 t and 2 t + 1
#pragma unroll
    for (int c = 0; c < G; ++c)
#pragma unroll
        for (int m = 0; m < NB; ++m) {
            const int hq = hb * 8 * NB + m * 8 + g;
            unsigned short x[8];
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int e = 32 * c + 8 * t + i;
                x[i] = hq < group && e < a.d ? a.q[(long long)row * a.q_ld + (long long)(hkv * group + hq) * a.q_sh + e].bits : 0;
                sum += __uint_as_float((unsigned)x[i] << 16);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) qa[c][i >> 1][i & 1][m] = x[i] | (unsigned)x[i + 4] << 16;
            sum += __shfl_xor_sync(~0u, sum, 1);
            sum += __shfl_xor_sync(~0u, sum, 2);
            qsum[c][m][0] = 136.f * __shfl_sync(~0u, sum, 8 * t);
            qsum[c][m][1] = 136.f * __shfl_sync(~0u, sum, 8 * t + 4);
        }
    float o[G][2][NB][4] = {};   // [group][pair of elements]: rows g (the first of the pair) and g + 8 (the second), columns 2 t, 2 t + 1
    float top[NB][2], sum[NB][2];
#pragma unroll
    for (int m = 0; m < NB; ++m) { top[m][0] = top[m][1] = -CUDART_INF_F; sum[m][0] = sum[m][1] = 0.f; }
    const float c2 = a.scale * attn::kLog2e;

    for (int i = 0; i < mine; ++i) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        __syncwarp();
        {
            const int now = next;
            next = fetch_idx(i + kStages);
            issue(i + kStages - 1, now);   // into the stage that the last iteration read (all lanes are past it)
        }
        const char *st = ring + (i % kStages) * S::STAGE;
        const int sl0 = *reinterpret_cast<const int *>(st + S::IDX + 4 * g), sl1 = *reinterpret_cast<const int *>(st + S::IDX + 4 * g + 32);
        float x[NB][4];   // logits: slots g (two heads), g + 8 (two heads)
        {
            unsigned w0[G], w1[G];
            lds_halves<2 * G, 4>(st + S::K + g * S::ROW + 4 * G * t, w0);
            lds_halves<2 * G, 4>(st + S::K + (g + 8) * S::ROW + 4 * G * t, w1);
            float s0[G], s1[G];
            lds_scales<G>(st + S::KS + g * 8, (G & 1) ? (int)((reinterpret_cast<uintptr_t>(ksc + sl0 * a.k.scale_ld) >> 1) & 1) : 0, s0);
            lds_scales<G>(st + S::KS + g * 8 + 64, (G & 1) ? (int)((reinterpret_cast<uintptr_t>(ksc + sl1 * a.k.scale_ld) >> 1) & 1) : 0, s1);
#pragma unroll
            for (int m = 0; m < NB; ++m) x[m][0] = x[m][1] = x[m][2] = x[m][3] = 0.f;
            each<G>([&](auto cc) {
                constexpr int c = decltype(cc)::value;
                const unsigned y0 = pick<c, G + c>(w0, w0), y1 = pick<c, G + c>(w1, w1);
                const unsigned a0 = nibble_pair<0>(y0), a1 = nibble_pair<0>(y1), a2 = nibble_pair<1>(y0), a3 = nibble_pair<1>(y1);
                const unsigned b0 = nibble_pair<2>(y0), b1 = nibble_pair<2>(y1), b2 = nibble_pair<3>(y0), b3 = nibble_pair<3>(y1);
#pragma unroll
                for (int m = 0; m < NB; ++m) {
                    float f[4] = {};
                    mma_bf16(f, a0, a1, a2, a3, qa[c][0][0][m], qa[c][0][1][m]);
                    mma_bf16(f, b0, b1, b2, b3, qa[c][1][0][m], qa[c][1][1][m]);
                    x[m][0] = fmaf(s0[c], f[0] - qsum[c][m][0], x[m][0]);
                    x[m][1] = fmaf(s0[c], f[1] - qsum[c][m][1], x[m][1]);
                    x[m][2] = fmaf(s1[c], f[2] - qsum[c][m][0], x[m][2]);
                    x[m][3] = fmaf(s1[c], f[3] - qsum[c][m][1], x[m][3]);
                }
            });
        }
        bool move = false;
#pragma unroll
        for (int m = 0; m < NB; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[m][e] = (e < 2 ? sl0 : sl1) >= 0 ? x[m][e] * c2 : -CUDART_INF_F;
                move |= x[m][e] > top[m][e & 1] + 8.f;
            }
        if (__any_sync(~0u, move)) {
#pragma unroll
            for (int m = 0; m < NB; ++m)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float to = fmaxf(x[m][e], x[m][e + 2]);
#pragma unroll
                    for (int w = 4; w < 32; w <<= 1) to = fmaxf(to, __shfl_xor_sync(~0u, to, w));
                    to = fmaxf(to, top[m][e]);
                    const float fall = to == -CUDART_INF_F ? 1.f : exp2f(top[m][e] - to);
                    top[m][e] = to;
                    sum[m][e] *= fall;
#pragma unroll
                    for (int c = 0; c < G; ++c)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            o[c][k][m][e] *= fall;
                            o[c][k][m][e + 2] *= fall;
                        }
                }
        }
#pragma unroll
        for (int m = 0; m < NB; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[m][e] = exp2f(x[m][e] - (top[m][e & 1] == -CUDART_INF_F ? 0.f : top[m][e & 1]));
                sum[m][e & 1] += x[m][e];
            }
        {
            // V: slots 2 t, 2 t + 1 and those eight on, this lane's row g of every product
            constexpr int H = (G + 1) / 2;
            unsigned w[4][H];
            const int at = G == 4 ? ((((g >> 1) ^ (t & 2)) << 4) | ((g & 1) << 3)) : 2 * G * g;
#pragma unroll
            for (int k = 0; k < 4; ++k) lds_halves<G, (G & 1) ? 2 : 4>(st + S::V + ((k >> 1) * 8 + (k & 1) * 4 + t) * S::ROW + at, w[k]);
            float s0[G], s1[G];
            lds_scales<G>(st + S::VS + g * 8, (G & 1) ? (int)((reinterpret_cast<uintptr_t>(vsc + sl0 * a.v.scale_ld) >> 1) & 1) : 0, s0);
            lds_scales<G>(st + S::VS + g * 8 + 64, (G & 1) ? (int)((reinterpret_cast<uintptr_t>(vsc + sl1 * a.v.scale_ld) >> 1) & 1) : 0, s1);
            each<G>([&](auto cc) {
                constexpr int c = decltype(cc)::value;
                const unsigned y0 = pick<c, c>(w[0], w[1]), y1 = pick<c, c>(w[2], w[3]);
                const unsigned a0 = minus136(nibble_pair<0>(y0)), a1 = minus136(nibble_pair<1>(y0)), a2 = minus136(nibble_pair<0>(y1)), a3 = minus136(nibble_pair<1>(y1));
                const unsigned b0 = minus136(nibble_pair<2>(y0)), b1 = minus136(nibble_pair<3>(y0)), b2 = minus136(nibble_pair<2>(y1)), b3 = minus136(nibble_pair<3>(y1));
#pragma unroll
                for (int m = 0; m < NB; ++m) {
                    const unsigned p0 = transpose8(attn::bf16x2(x[m][0] * s0[c], x[m][1] * s0[c])), p1 = transpose8(attn::bf16x2(x[m][2] * s1[c], x[m][3] * s1[c]));
                    mma_bf16(o[c][0][m], a0, a1, a2, a3, p0, p1);
                    mma_bf16(o[c][1][m], b0, b1, b2, b3, p0, p1);
                }
            });
        }
        __syncwarp();
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();   // the ring is free: the warps join in it

    constexpr int W = 32 * G, HEADS = 8 * NB, PER = HEADS * W + 2 * HEADS;
    float *join = reinterpret_cast<float *>(smem) + warp * PER;
#pragma unroll
    for (int m = 0; m < NB; ++m)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float l = sum[m][e];
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) l += __shfl_xor_sync(~0u, l, w);
            const int head = m * 8 + 2 * t + e;
            if (g == 0) {
                join[HEADS * W + head] = top[m][e];
                join[HEADS * W + HEADS + head] = l;
            }
#pragma unroll
            for (int c = 0; c < G; ++c)
                *reinterpret_cast<float4 *>(join + head * W + 32 * c + 4 * g) = make_float4(o[c][0][m][e], o[c][0][m][e + 2], o[c][1][m][e], o[c][1][m][e + 2]);
        }
    __syncthreads();
    join = reinterpret_cast<float *>(smem);
    const int width = attn::part_width(attn::kForward, a.d);
    for (int i = threadIdx.x; i < HEADS * (W / 4); i += attn::kWarps * 32) {
        const int m = i / (W / 4), e = i % (W / 4) * 4, hq = hb * HEADS + m;
        if (hq >= group || e >= width) continue;
        float high = -CUDART_INF_F, l = 0.f, x[4] = {};
#pragma unroll
        for (int w = 0; w < attn::kWarps; ++w) high = fmaxf(high, join[w * PER + HEADS * W + m]);
        const float ref = high == -CUDART_INF_F ? 0.f : high;
#pragma unroll
        for (int w = 0; w < attn::kWarps; ++w) {
            const float f = exp2f(join[w * PER + HEADS * W + m] - ref);
            l = fmaf(f, join[w * PER + HEADS * W + HEADS + m], l);
            const float4 y = *reinterpret_cast<const float4 *>(join + w * PER + m * W + e);
            x[0] = fmaf(f, y.x, x[0]); x[1] = fmaf(f, y.y, x[1]); x[2] = fmaf(f, y.z, x[2]); x[3] = fmaf(f, y.w, x[3]);
        }
        const int h = hkv * group + hq;
        if (a.part) {
            const long long unit = ((long long)h * a.M + row) * a.splits + part;
            attn::store4<float, 4>(a.part + unit * width, e, width, x);
            if (e == 0) a.part_ml[unit] = make_float2(high, l);
        } else {
            const float f = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] *= f;
            attn::store4<Bf16, 1>(a.out.at(0, h, row), e, a.d, x);
            if (e == 0) a.lse[(long long)row * a.heads + h] = l == 0.f ? -CUDART_INF_F : (high + log2f(l)) * attn::kLn2;
        }
    }
}

}  // namespace kv4
}  // namespace b2sp
