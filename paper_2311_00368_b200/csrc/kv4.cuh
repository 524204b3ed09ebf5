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

// i * a + j * b
__device__ __forceinline__ unsigned long long offset(unsigned i, unsigned a, unsigned j, unsigned b)
{
    return (unsigned long long)i * a + (unsigned long long)j * b;
}

// Slots that several tokens name take the last one's row.  Up to kScanTokens tokens a CTA of the writing kernel compares its tokens' slots
// with those of all later tokens; more go through an owner per slot in the workspace (two small launches ahead of the writing one: the owners of
// the slots named become -1, then the largest token): 16384 tokens cost 4 us this way, and the comparisons would be 1.3e8.
constexpr int kScanTokens = 1024, kWriteThreads = 256, kWritePieces = 4;

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
            // (first out of L2, which leaves more of the cache's rows there: 65536 tokens of 8 heads, width 64: 21.9 -> 20.4 us)
            __stcs(reinterpret_cast<uint4 *>(row + c), make_uint4(attn::bf16x2(x[0], x[1]), attn::bf16x2(x[2], x[3]), attn::bf16x2(x[4], x[5]), attn::bf16x2(x[6], x[7])));
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
    unsigned ld, sh;         // of the rows in 16 or 32 bits (all strides below 2^32: a product with an index is one instruction)
    const int *slots;
    uint8_t *codes;          // as in Cache
    Bf16 *scales;
    unsigned code_ld, code_head, scale_ld, scale_head;
    int cache_slots;
    Div by_head, by_piece;   // divisors: heads, and the pieces of a row that threads take (write: 4 G quarters of groups; read: ceil(d / 8))
    unsigned first;          // read: (four tokens, head) rows of earlier launches
    int *owner;              // write: NULL with few tokens
};

__device__ __forceinline__ unsigned max_nan2(unsigned a, unsigned b)   // of two bf16; a NaN stays one
{
    unsigned r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Four lanes per group, eight elements each.  Bound by instructions next to memory (2 d bytes in, 18 G out), so bfloat16 rows have a way of
// their own: the largest element is found on pairs, and eight divisions become multiplications by 1 / s.  Rounding x (1 / s) to a whole number r
// by adding 1.5 * 2^23 gives what rounding x / s gives, unless x / s lies halfway between whole numbers: x and s have eight significant bits, so x / s
// is either exactly halfway or at least 2^-10 of itself away from there, far more than the error of x (1 / s).  Halfway, x - r s is
// exactly half of s, and r is made even.  Scales near the ends of the exponent range take the divisions.
// With many tokens a thread takes the same piece of four neighbouring tokens, so that the loads of all of them are in flight at once.
template <typename T, int V, bool SCAN>
__global__ void __launch_bounds__(kWriteThreads) kv4_write_kernel(const T *x, const RowsArgs a)
{
    constexpr int N = SCAN ? 1 : kWritePieces;
    __shared__ int gone[kWriteThreads / 4];   // SCAN: which of the CTA's tokens a later one replaces
    constexpr bool PAIRS = sizeof(T) == 2 && V == 8;
    const unsigned u0 = blockIdx.x * (unsigned)kWriteThreads, u = u0 + threadIdx.x, row = a.by_piece(u), piece = u - row * a.by_piece.d;
    const unsigned tn = a.by_head(row), h = row - tn * a.by_head.d, t = tn * N;
    const int e = (int)piece * 8, grp = piece >> 2, j = piece & 3;
    const T *from = x + (offset(t, a.ld, h, a.sh) + e);
    int slot[N], owner[N];
    uint4 raw[N];
    float v[8] = {};
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const bool on = t + k < (unsigned)a.tokens;
        slot[k] = on ? a.slots[t + k] : -1;
        raw[k] = make_uint4(0, 0, 0, 0);
        if constexpr (PAIRS) {
            if (on && e < a.d) raw[k] = *reinterpret_cast<const uint4 *>(from + (unsigned long long)k * a.ld);
        }
    }
    if (SCAN) {
        const unsigned t0 = a.by_head(a.by_piece(u0)), t1 = min((unsigned)a.tokens - 1, a.by_head(a.by_piece(u0 + kWriteThreads - 1)));
        if (threadIdx.x < kWriteThreads / 4) gone[threadIdx.x] = 0;
        __syncthreads();
        for (unsigned k = t0 + 1 + threadIdx.x; k < (unsigned)a.tokens; k += kWriteThreads) {
            const int s = a.slots[k];
            for (unsigned i = t0; i <= t1 && i < k; ++i)
                if (a.slots[i] == s) gone[i - t0] = 1;
        }
        __syncthreads();
        owner[0] = (unsigned)slot[0] < (unsigned)a.cache_slots && gone[t - t0] == 0 ? (int)t : -1;
    } else {
        asm volatile("griddepcontrol.wait;" ::: "memory");   // the owners
#pragma unroll
        for (int k = 0; k < N; ++k) owner[k] = (unsigned)slot[k] < (unsigned)a.cache_slots ? a.owner[slot[k]] : -1;
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const unsigned w[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
        float top = 0.f;
        bool odd = false;   // a NaN or an infinity in the group
        if constexpr (PAIRS) {
            unsigned m = max_nan2(max_nan2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), max_nan2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
            m = max_nan2(m, __shfl_xor_sync(~0u, m, 1));
            m = max_nan2(m, __shfl_xor_sync(~0u, m, 2));
            m = max_nan2(m, m >> 16);
            top = __uint_as_float(m << 16);
            odd = !(top <= 3.402823466e38f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        } else {
            if (t + k < (unsigned)a.tokens) load8<T, V>(from - e + (unsigned long long)k * a.ld, e, a.d, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                top = fmaxf(top, fabsf(v[i]));
                odd |= !(fabsf(v[i]) <= 3.402823466e38f);
            }
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
            odd = __ballot_sync(~0u, odd) >> (threadIdx.x & 28) & 15;
        }
        Bf16 s;
        attn::narrow(__fdiv_rn(top, 7.f), s);
        if (odd) s.bits = 0x7fff;
        const float f = attn::widen(s);
        unsigned word[2] = {0, 0};
        bool divide = true;
        if (PAIRS) {
            const float inv = __frcp_rn(f), half = 0.5f * f;
            divide = !(f > 1e-30f && f < 1e30f);
            // on pairs: y = x / s + 1.5 * 2^23 rounded, minus = -r, rest = x - r s
            const uint64_t magic = attn::two(12582912.f, 12582912.f), by = attn::two(inv, inv), s2 = attn::two(f, f), neg = attn::two(-1.f, -1.f);
            float y[8], rest[8];
            bool halfway = false;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const uint64_t x2 = attn::two(v[i], v[i + 1]), y2 = attn::fma2(x2, by, magic), minus = attn::fma2(y2, neg, magic);
                attn::split(y2, y[i], y[i + 1]);
                attn::split(attn::fma2(minus, s2, x2), rest[i], rest[i + 1]);
                halfway |= fabsf(rest[i]) == half || fabsf(rest[i + 1]) == half;
            }
            if (halfway) {   // (one thread in a hundred) r is made even
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (fabsf(rest[i]) == half && (__float_as_uint(y[i]) & 1)) y[i] += copysignf(1.f, rest[i]);
            }
#pragma unroll
            for (int i = 7; i >= 0; --i) word[i >> 2] = word[i >> 2] * 16 + (__float_as_uint(y[i]) & 15);
            word[0] ^= 0x8888u;   // two's complement to offset by 8
            word[1] ^= 0x8888u;
        }
        if (divide) {
            word[0] = word[1] = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float q = f > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(v[i], f)), -7.f), 7.f) : 0.f;
                word[i >> 2] |= (unsigned)((int)q + 8) << (4 * (i & 3));
            }
        }
        if (owner[k] >= 0 && owner[k] == (int)(t + k)) {
            unsigned short *codes = reinterpret_cast<unsigned short *>(a.codes + offset(h, a.code_head, slot[k], a.code_ld)) + (2 * j * a.G + grp);
            codes[0] = (unsigned short)word[0];
            codes[a.G] = (unsigned short)word[1];
            if (j == 0) a.scales[offset(h, a.scale_head, slot[k], a.scale_ld) + grp] = s;
        }
    }
}

// A thread takes the same eight elements of four neighbouring tokens, so that the loads of all of them are in flight (slots, then codes and
// scales); rows of slots outside the cache read as zeros.
constexpr int kReadTokens = 4;
template <typename T, int V>
__global__ void __launch_bounds__(256) kv4_read_kernel(const RowsArgs a, T *out)
{
    const unsigned u = blockIdx.x * 256u + threadIdx.x, row = a.by_piece(u);
    const unsigned tn = a.by_head(row + a.first), h = row + a.first - tn * a.by_head.d, t = tn * kReadTokens;
    const int e = (int)(u - row * a.by_piece.d), grp = e >> 2, j = e & 3, at = 2 * j * a.G + grp;
    unsigned w0[kReadTokens], w1[kReadTokens];
    int slot[kReadTokens];
    float s[kReadTokens];
#pragma unroll
    for (int k = 0; k < kReadTokens; ++k) slot[k] = t + k < (unsigned)a.tokens ? a.slots[t + k] : -1;
    const uint8_t *codes = a.codes + (unsigned long long)h * a.code_head;
    const Bf16 *scales = a.scales + ((unsigned long long)h * a.scale_head + grp);
#pragma unroll
    for (int k = 0; k < kReadTokens; ++k) {
        w0[k] = w1[k] = 0x8888u;
        s[k] = 0.f;
        if ((unsigned)slot[k] < (unsigned)a.cache_slots) {
            const unsigned short *c = reinterpret_cast<const unsigned short *>(codes + (unsigned long long)(unsigned)slot[k] * a.code_ld) + at;
            w0[k] = c[0];
            w1[k] = c[a.G];
            s[k] = attn::widen(scales[(unsigned long long)(unsigned)slot[k] * a.scale_ld]);
        }
    }
    T *to = out + offset(t, a.ld, h, a.sh);
#pragma unroll
    for (int k = 0; k < kReadTokens; ++k) {
        if (t + k >= (unsigned)a.tokens) break;
        // a nibble below the exponent of 2^23 is 2^23 + code
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = s[k] * (__uint_as_float((w0[k] >> (4 * i) & 15) | 0x4b000000u) - 8388616.f);
            v[4 + i] = s[k] * (__uint_as_float((w1[k] >> (4 * i) & 15) | 0x4b000000u) - 8388616.f);
        }
        store8<T, V>(to + (unsigned long long)k * a.ld, e * 8, a.d, v);
    }
}

// ---- attention ------------------------------------------------------------------------------------------------------------------
struct AttnArgs {
    int M, heads, kv_heads, d, head_blocks;   // head_blocks: eights (or sixteens, NB = 2) of query heads that share one K and V
    int ctas, share;     // of a key/value head and head block; entries of each
    long long nnz;
    const int *row_ptr, *col_idx;
    const Bf16 *q;
    long long q_ld, q_sh;
    int q_wide;          // 16-byte loads of q
    Cache k, v;
    float scale;
    attn::View<Bf16> out;
    float *lse, *part;   // part: two slots per CTA of `ctas` (see the kernel), [heads][part_width]
    float2 *part_ml;
};
__device__ __forceinline__ long long part_slot(const AttnArgs &a, int cta, int slot, int h) { return ((long long)cta * 2 + slot) * a.heads + h; }

__device__ __forceinline__ void mma_f16(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same onto zeros.
__device__ __forceinline__ void mma_f16_first(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ unsigned f16x2(float lo, float hi)   // round to nearest even
{
    unsigned r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// The codes of nibbles 0 and 1 of both halves of y, less 8, as two f16 each.  A nibble in the lowest bits of the f16 1024 makes 1024 + code, one
// in the next four bits 1024 + 16 code; both differences are exact.  `k1024` is two f16 of 1024 in a register whose value the compiler does not know:
// with two constants it takes two instructions for (y & mask) | k1024, with one of them in a register one (263 -> 135 logical instructions
// per 32 slots).
__device__ __forceinline__ unsigned two_1024()
{
    unsigned r;
    asm volatile("mov.b32 %0, 0x64006400;" : "=r"(r));
    return r;
}
template <unsigned MASK> __device__ __forceinline__ unsigned onto_1024(unsigned y, unsigned k1024)
{
    unsigned r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(y), "n"(MASK), "r"(k1024));   // (y & MASK) | k1024
    return r;
}
__device__ __forceinline__ unsigned codes_low(unsigned y, unsigned k1024)
{
    unsigned r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(onto_1024<0x000f000fu>(y, k1024)), "r"(0x64086408u));
    return r;
}
__device__ __forceinline__ unsigned codes_high(unsigned y, unsigned k1024)
{
    unsigned r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(onto_1024<0x00f000f0u>(y, k1024)), "r"(0x2c002c00u), "r"(0xd480d480u));   // / 16 - 72
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
// every fourth 32 slots each and join at the end.  What it has to read is 36 G bytes a slot; what bounds it beside that is the integer pipe, which
// makes numbers of the codes (64 lanes a clock), so instructions are kept few: cp.async brings the next 32 slots into the other half of
// a warp's ring; a code becomes an f16 by one mask and one f16 addition or multiply-add on the other pipe; the tensor core's legacy form
// multiplies (m16n8k16: 16 slots of K by 8 query heads, then 16 elements of V by 8 query heads); the weights pass from the one product's layout to
// the other's by movmatrix.
//   * Q goes to f16 exactly: divided by a power of two that brings each head's largest element below 2; what is more than 2^-14 smaller
//     than that loses at most 2^-25 of it, as much as fp32 sums would.  The scale of a group of K multiplies the products of its 32 elements.
//   * The scale of (slot, group) of V multiplies the slot's weight, divided by a power of two per group that keeps all scales met so far below
//     2^7, and that is rounded to f16: half a step is 2^-11 of the product, 2^-25 at least.  Scales are not below 1 then, so a weight is off by no
//     more than 2^-11 of itself or 2^-25 of the row's largest.  That holds while the scales of a group lie within 2^7 of each other; where they do not,
//     the slot with the largest may weigh nothing, and the others would vanish beside it.  From the first such slots of a row on, each head's and
//     group's largest product among 16 slots is brought to 2^8 of its own, and the products of the 16 are added up in fp32 (32 heads over 8, width 128:
//     one token of 32768 slots 19.1 us, with every eighth scale 2^20 times the others 22.8; 64 tokens 315 and 333).  It is the one rounding of
//     this kernel beside that of the output.
//   * The running maximum moves only when a logit exceeds it by 8 (to base 2): weights up to 2^8.
// Slot r of a half tile is row r of the first product; V's rows lie in the order (r & 1) * 4 + r / 2 of each eight, so that the four lanes of
// a column of V read different banks.
//
// The entries of all rows, one behind the other, are dealt in equal shares to as many CTAs as run at once, so that rows of any lengths
// keep all SMs busy to the end.  A row inside one share is finished there; of a row that goes on, each CTA leaves its part in the workspace: in slot 0
// if the row began in an earlier share, else in slot 1; kv4_join_kernel joins the parts in order, and writes the rows without entries.
constexpr int kStages = 2, kSlots = 32;
constexpr float kDownFirst = 1.2676506e30f;   // 2^100
template <int G, int NB> struct Smem {
    static constexpr int ROW = 16 * G;
    static constexpr int K = 0, V = kSlots * ROW, KS = 2 * kSlots * ROW, VS = KS + kSlots * 8, STAGE = VS + kSlots * 8;
    static constexpr int WIDE = attn::kWarps * kStages * STAGE;   // behind the rings: 32 rows of scales of K and of V in fp32 per warp, four apart
    static constexpr int RING = WIDE + attn::kWarps * 2 * kSlots * 16;
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
// The same halfwords, each shifted right by eight bits (their lower bytes are of no interest afterwards).
template <int A, int B, int N> __device__ __forceinline__ unsigned pick_high(const unsigned (&a)[N], const unsigned (&b)[N])
{
    constexpr unsigned lo = (A & 1) ? 0x33 : 0x11, hi = (B & 1) ? 0x77 : 0x55;
    return __byte_perm(a[A / 2], b[B / 2], hi << 8 | lo);
}
// Whether a row of an odd number of scales begins in the middle of a word (cp.async brings whole words).
template <int G> __device__ __forceinline__ int odd_row(const Bf16 *scales, int slot, int ld)
{
    return (G & 1) ? (int)((reinterpret_cast<uintptr_t>(scales + (long long)slot * ld) >> 1) & 1) : 0;
}
template <int G> __device__ __forceinline__ void lds_scales(const char *p, int odd, float (&s)[G])   // bf16
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
template <int G> __device__ __forceinline__ void sts_wide(char *p, const float (&s)[G])
{
    if constexpr (G >= 3) *reinterpret_cast<float4 *>(p) = make_float4(s[0], s[1], s[2], G == 4 ? s[G - 1] : 0.f);
    else if constexpr (G == 2) *reinterpret_cast<float2 *>(p) = make_float2(s[0], s[1]);
    else *reinterpret_cast<float *>(p) = s[0];
}
template <int G> __device__ __forceinline__ void lds_wide(const char *p, float (&s)[G])
{
    if constexpr (G >= 3) {
        const float4 v = *reinterpret_cast<const float4 *>(p);
        s[0] = v.x; s[1] = v.y; s[2] = v.z;
        if (G == 4) s[G - 1] = v.w;
    } else if constexpr (G == 2) {
        const float2 v = *reinterpret_cast<const float2 *>(p);
        s[0] = v.x; s[1] = v.y;
    } else {
        s[0] = *reinterpret_cast<const float *>(p);
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

// The row that entry `at` (< row_ptr[M]) lies in: 32 ends are looked at at a time.
__device__ __forceinline__ int row_of(const int *row_ptr, int M, long long at)
{
    int lo = 0, hi = M;   // row_ptr[lo] <= at < row_ptr[hi]
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, k = min(lo + step * ((int)(threadIdx.x & 31) + 1), hi);
        const int n = __popc(__ballot_sync(~0u, row_ptr[k] <= at));   // the first n of them are not beyond it
        hi = min(lo + step * (n + 1), hi);
        lo += step * n;
    }
    return lo;
}

template <int G, int NB>
__global__ void __launch_bounds__(attn::kWarps * 32, 3) kv4_attention_kernel(const AttnArgs a)
{
    using S = Smem<G, NB>;
    __shared__ __align__(16) char smem[S::BYTES];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int group = a.heads / a.kv_heads;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (the joining kernel waits for this grid's end where it reads)
    const int cta = blockIdx.x % a.ctas, of = blockIdx.x / a.ctas, hb = of % a.head_blocks, hkv = of / a.head_blocks;
    const long long from0 = (long long)cta * a.share, to0 = min(from0 + a.share, min(a.nnz, (long long)a.row_ptr[a.M]));
    if (from0 >= to0) return;
    char *ring = smem + warp * kStages * S::STAGE, *wide = smem + S::WIDE + warp * 2 * kSlots * 16;
    const unsigned ring_s = (unsigned)__cvta_generic_to_shared(ring);
    const uint8_t *kc = a.k.codes + hkv * a.k.code_head, *vc = a.v.codes + hkv * a.v.code_head;
    const Bf16 *ksc = a.k.scales + hkv * a.k.scale_head, *vsc = a.v.scales + hkv * a.v.scale_head;
    const int slots = min(a.k.slots, a.v.slots);
    // where this lane's pieces of a tile go: G pieces of 16 bytes of K's codes and of V's
    unsigned dst_k[G], dst_v[G];   // shared addresses in stage 0
#pragma unroll
    for (int c = 0; c < G; ++c) {
        const int id = c * 32 + lane, r = id / G, ch = id % G, vrow = (r & 24) | ((r & 1) << 2) | (r >> 1 & 3);
        dst_k[c] = ring_s + S::K + r * S::ROW + ch * 16;
        dst_v[c] = ring_s + S::V + vrow * S::ROW + (G == 4 ? ch ^ (vrow & 2) : ch) * 16;
    }
    const unsigned k1024 = two_1024();
    const int k_ld = (int)a.k.code_ld, v_ld = (int)a.v.code_ld, ks_ld = (int)a.k.scale_ld, vs_ld = (int)a.v.scale_ld;

    for (int row = row_of(a.row_ptr, a.M, from0); row < a.M; ++row) {
        const int first = a.row_ptr[row], last = (int)min((long long)a.row_ptr[row + 1], a.nnz);
        if (first >= to0) break;
        const long long begin = max((long long)first, from0), end = min((long long)last, to0);
        if (begin >= end) continue;
        const int n = (int)(end - begin);
        const int *idx = a.col_idx + begin;
        const int tiles = (n + kSlots - 1) / kSlots, mine = tiles > warp ? (tiles - warp + attn::kWarps - 1) / attn::kWarps : 0;

        auto fetch_idx = [&](int i) {   // this lane's slot of the warp's tile i, or -1
            const int at = (warp + i * attn::kWarps) * kSlots + lane;
            const int s = i < mine && at < n ? idx[at] : -1;
            return (unsigned)s < (unsigned)slots ? s : -1;
        };
        auto scale_row = [&](unsigned dst, const Bf16 *src, int slot) {
            if constexpr (G == 4) cp_async(dst, src, 8, slot >= 0 ? 8 : 0);
            else if constexpr (G == 2) cp_async(dst, src, 4, slot >= 0 ? 4 : 0);
            else {   // whole words around an odd number of halfwords; bytes behind the row are not read
                const int off = (int)(reinterpret_cast<uintptr_t>(src) & 2);
                const char *p = reinterpret_cast<const char *>(src) - off;
                const int bytes = off + 2 * G;
                cp_async(dst, p, 4, slot >= 0 ? min(bytes, 4) : 0);
                if (G == 3) cp_async(dst + 4, p + 4, 4, slot >= 0 ? bytes - 4 : 0);
            }
        };
        auto issue = [&](int i, int slot) {
            if (i < mine) {
                const unsigned st = (unsigned)(i % kStages) * S::STAGE;
                const int at = max(slot, 0);
#pragma unroll
                for (int c = 0; c < G; ++c) {
                    const int s = __shfl_sync(~0u, slot, (c * 32 + lane) / G), r = max(s, 0), keep = s >= 0 ? 16 : 0, ch = (c * 32 + lane) % G * 16;
                    cp_async(dst_k[c] + st, kc + ((long long)r * k_ld + ch), 16, keep);
                    cp_async(dst_v[c] + st, vc + ((long long)r * v_ld + ch), 16, keep);
                }
                scale_row(ring_s + st + S::KS + lane * 8, ksc + (long long)at * ks_ld, slot);
                scale_row(ring_s + st + S::VS + lane * 8, vsc + (long long)at * vs_ld, slot);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };

        // The first tile is on its way while Q is read.  Q: lane (g, t) has elements 8 t .. 8 t + 7 of each group of query head g (of each eight)
        int cur = -1, now = fetch_idx(0), next = fetch_idx(1);   // slots of the tile at hand, of the one being fetched, of the one behind it
        issue(0, now);
        unsigned qa[G][2][2][NB];   // [group][k step][half of k]
        float c2[NB][2];            // scale log2(e) and what Q is divided by, of query heads 2 t and 2 t + 1
#pragma unroll
        for (int m = 0; m < NB; ++m) {
            const int hq = hb * 8 * NB + m * 8 + g;
            const Bf16 *q = a.q + (long long)row * a.q_ld + (long long)(hkv * group + hq) * a.q_sh;
            uint4 x[G];
            float high = 0.f;
#pragma unroll
            for (int c = 0; c < G; ++c) {
                const int e = 32 * c + 8 * t;
                x[c] = make_uint4(0, 0, 0, 0);
                if (hq < group) {
                    if (a.q_wide) {
                        if (e < a.d) x[c] = __ldg(reinterpret_cast<const uint4 *>(q + e));
                    } else {
                        unsigned short y[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[i] = e + i < a.d ? q[e + i].bits : 0;
                        x[c] = make_uint4(y[0] | (unsigned)y[1] << 16, y[2] | (unsigned)y[3] << 16, y[4] | (unsigned)y[5] << 16, y[6] | (unsigned)y[7] << 16);
                    }
                }
                const unsigned w[4] = {x[c].x, x[c].y, x[c].z, x[c].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) high = fmaxf(high, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xffff0000u))));
            }
            high = fmaxf(high, __shfl_xor_sync(~0u, high, 1));
            high = fmaxf(high, __shfl_xor_sync(~0u, high, 2));
            const int e = min(max((int)(__float_as_uint(high) >> 23) - 127, -126), 126);   // (a NaN or an infinity stays one)
            const float by = __uint_as_float((unsigned)(127 - e) << 23), up = a.scale * attn::kLog2e * __uint_as_float((unsigned)(127 + e) << 23);
            c2[m][0] = __shfl_sync(~0u, up, 8 * t);
            c2[m][1] = __shfl_sync(~0u, up, 8 * t + 4);
#pragma unroll
            for (int c = 0; c < G; ++c) {
                const unsigned w[4] = {x[c].x, x[c].y, x[c].z, x[c].w};
                float f[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f[2 * i] = __uint_as_float(w[i] << 16) * by;
                    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u) * by;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) qa[c][i >> 1][i & 1][m] = f16x2(f[i], f[i + 4]);
            }
        }
        float o[G][2][NB][4] = {};   // [group][pair of elements]: rows g (the first of the pair) and g + 8 (the second), columns 2 t, 2 t + 1
        float top[NB][2], base[NB][2], sum[NB][2];   // base: top, or 0 as long as that is -inf
        float down[G];               // what V's scales are multiplied by (at first kDownFirst, which any scale above 2^-93 moves)
        int fallen = 0;              // by how many powers of two, in all; above 7: scales of a group more than 2^7 apart have been met
#pragma unroll
        for (int c = 0; c < G; ++c) down[c] = kDownFirst;
#pragma unroll
        for (int m = 0; m < NB; ++m) { top[m][0] = top[m][1] = -CUDART_INF_F; base[m][0] = base[m][1] = 0.f; sum[m][0] = sum[m][1] = 0.f; }

        for (int i = 0; i < mine; ++i) {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncwarp();
            cur = now;
            now = next;
            next = fetch_idx(i + 2);
            issue(i + 1, now);   // into the stage that the last iteration read (all lanes are past it)
            const char *st = ring + (i % kStages) * S::STAGE;
            const unsigned valid = __ballot_sync(~0u, cur >= 0);
            bool small = false;
            {
                // a slot's scales per lane, to fp32
                float ks[G], vs[G], high = 0.f;
                lds_scales<G>(st + S::KS + lane * 8, odd_row<G>(ksc, max(cur, 0), ks_ld), ks);
                lds_scales<G>(st + S::VS + lane * 8, odd_row<G>(vsc, max(cur, 0), vs_ld), vs);
#pragma unroll
                for (int c = 0; c < G; ++c) high = fmaxf(high, vs[c] * down[c]);
                if (__any_sync(~0u, high > 128.f)) {   // a power of two that brings the largest of the group to 64 .. 128
#pragma unroll
                    for (int c = 0; c < G; ++c) {
                        float x = vs[c] * down[c] > 128.f ? vs[c] : 0.f;
#pragma unroll
                        for (int w = 1; w < 32; w <<= 1) x = fmaxf(x, __shfl_xor_sync(~0u, x, w));
                        if (x > 0.f) {   // (the same for all lanes)
                            const float to = __uint_as_float((unsigned)min(max(254 + 6 - (int)(__float_as_uint(x) >> 23), 1), 253) << 23);
                            const float f = to * __uint_as_float((254u << 23) - __float_as_uint(down[c]));
                            if (down[c] != kDownFirst) fallen += (int)((__float_as_uint(down[c]) - __float_as_uint(to)) >> 23);
                            down[c] = to;
#pragma unroll
                            for (int m = 0; m < NB; ++m)
#pragma unroll
                                for (int e = 0; e < 4; ++e) { o[c][0][m][e] *= f; o[c][1][m][e] *= f; }
                        }
                    }
                }
#pragma unroll
                for (int c = 0; c < G; ++c) {
                    vs[c] *= down[c];
                    small |= __float_as_uint(vs[c]) - 1u < 0x3f7fffffu;   // (above 0 and below 1)
                }
                sts_wide<G>(wide + lane * 16, ks);
                sts_wide<G>(wide + kSlots * 16 + lane * 16, vs);
            }
            if (__any_sync(~0u, small)) fallen = 8;
            __syncwarp();
            float x[2][NB][4];   // of each half tile: logits of slots g (two heads) and g + 8 (two heads)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r0 = 16 * j + g, r1 = r0 + 8;
                unsigned w0[G], w1[G];
                lds_halves<2 * G, 4>(st + S::K + r0 * S::ROW + 4 * G * t, w0);
                lds_halves<2 * G, 4>(st + S::K + r1 * S::ROW + 4 * G * t, w1);
                float s0[G], s1[G];
                lds_wide<G>(wide + r0 * 16, s0);
                lds_wide<G>(wide + r1 * 16, s1);
                each<G>([&](auto cc) {
                    constexpr int c = decltype(cc)::value;
                    const unsigned y0 = pick<c, G + c>(w0, w0), y1 = pick<c, G + c>(w1, w1), z0 = pick_high<c, G + c>(w0, w0), z1 = pick_high<c, G + c>(w1, w1);
                    const unsigned a0 = codes_low(y0, k1024), a1 = codes_low(y1, k1024), a2 = codes_high(y0, k1024), a3 = codes_high(y1, k1024);
                    const unsigned b0 = codes_low(z0, k1024), b1 = codes_low(z1, k1024), b2 = codes_high(z0, k1024), b3 = codes_high(z1, k1024);
#pragma unroll
                    for (int m = 0; m < NB; ++m) {
                        float f[4];
                        mma_f16_first(f, a0, a1, a2, a3, qa[c][0][0][m], qa[c][0][1][m]);
                        mma_f16(f, b0, b1, b2, b3, qa[c][1][0][m], qa[c][1][1][m]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[j][m][e] = c == 0 ? (e < 2 ? s0[0] : s1[0]) * f[e] : fmaf(e < 2 ? s0[c] : s1[c], f[e], x[j][m][e]);
                    }
                });
#pragma unroll
                for (int m = 0; m < NB; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[j][m][e] *= c2[m][e & 1];
                if (valid != ~0u) {
#pragma unroll
                    for (int m = 0; m < NB; ++m)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!(valid >> (e < 2 ? r0 : r1) & 1)) x[j][m][e] = -CUDART_INF_F;
                }
            }
            bool move = false;
#pragma unroll
            for (int m = 0; m < NB; ++m)
#pragma unroll
                for (int e = 0; e < 2; ++e) move |= fmaxf(fmaxf(x[0][m][e], x[0][m][e + 2]), fmaxf(x[1][m][e], x[1][m][e + 2])) > top[m][e] + 8.f;
            if (__any_sync(~0u, move)) {
#pragma unroll
                for (int m = 0; m < NB; ++m)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float to = fmaxf(fmaxf(x[0][m][e], x[0][m][e + 2]), fmaxf(x[1][m][e], x[1][m][e + 2]));
#pragma unroll
                        for (int w = 4; w < 32; w <<= 1) to = fmaxf(to, __shfl_xor_sync(~0u, to, w));
                        to = fmaxf(to, top[m][e]);
                        base[m][e] = to == -CUDART_INF_F ? 0.f : to;
                        const float fall = attn::ex2(top[m][e] - base[m][e]);
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
            auto half_tile = [&](auto jj, auto uneven) {   // 16 slots; uneven: scales too far apart for one power of two
                constexpr int j = decltype(jj)::value;
#pragma unroll
                for (int m = 0; m < NB; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[j][m][e] = attn::ex2(x[j][m][e] - base[m][e & 1]);
                        sum[m][e & 1] += x[j][m][e];
                    }
                // V: slots 2 t, 2 t + 1 and those eight on, this lane's row g of every product
                unsigned w[4][(G + 1) / 2];
                const int at = G == 4 ? ((((g >> 1) ^ (t & 2)) << 4) | ((g & 1) << 3)) : 2 * G * g;
#pragma unroll
                for (int k = 0; k < 4; ++k) lds_halves<G, (G & 1) ? 2 : 4>(st + S::V + (16 * j + (k >> 1) * 8 + (k & 1) * 4 + t) * S::ROW + at, w[k]);
                float s0[G], s1[G];
                lds_wide<G>(wide + kSlots * 16 + (16 * j + g) * 16, s0);
                lds_wide<G>(wide + kSlots * 16 + (16 * j + g + 8) * 16, s1);
                each<G>([&](auto cc) {
                    constexpr int c = decltype(cc)::value;
                    const unsigned y0 = pick<c, c>(w[0], w[1]), y1 = pick<c, c>(w[2], w[3]), z0 = pick_high<c, c>(w[0], w[1]), z1 = pick_high<c, c>(w[2], w[3]);
                    const unsigned a0 = codes_low(y0, k1024), a1 = codes_high(y0, k1024), a2 = codes_low(y1, k1024), a3 = codes_high(y1, k1024);
                    const unsigned b0 = codes_low(z0, k1024), b1 = codes_high(z0, k1024), b2 = codes_low(z1, k1024), b3 = codes_high(z1, k1024);
#pragma unroll
                    for (int m = 0; m < NB; ++m) {
                        float y[4];   // weights times scales: slot g, heads 2 t and 2 t + 1; slot g + 8
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[e] = x[j][m][e] * (e < 2 ? s0[c] : s1[c]);
                        if constexpr (!decltype(uneven)::value) {
                            const unsigned p0 = transpose8(f16x2(y[0], y[1])), p1 = transpose8(f16x2(y[2], y[3]));
                            mma_f16(o[c][0][m], a0, a1, a2, a3, p0, p1);
                            mma_f16(o[c][1][m], b0, b1, b2, b3, p0, p1);
                        } else {   // each head's largest product to 2^8 .. 2^9
                            float by[2], back[2], part0[4], part1[4];
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                float most = fmaxf(y[e], y[e + 2]);
#pragma unroll
                                for (int k = 4; k < 32; k <<= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, k));
                                const int to = min(max(262 - (int)(__float_as_uint(most) >> 23), 1), 253);
                                by[e] = __uint_as_float((unsigned)to << 23);
                                back[e] = __uint_as_float((unsigned)(254 - to) << 23);
                            }
                            const unsigned p0 = transpose8(f16x2(y[0] * by[0], y[1] * by[1])), p1 = transpose8(f16x2(y[2] * by[0], y[3] * by[1]));
                            mma_f16_first(part0, a0, a1, a2, a3, p0, p1);
                            mma_f16_first(part1, b0, b1, b2, b3, p0, p1);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                o[c][0][m][e] = fmaf(part0[e], back[e & 1], o[c][0][m][e]);
                                o[c][1][m][e] = fmaf(part1[e], back[e & 1], o[c][1][m][e]);
                            }
                        }
                    }
                });
            };
            if (fallen <= 7) {
                half_tile(std::integral_constant<int, 0>{}, std::false_type{});
                half_tile(std::integral_constant<int, 1>{}, std::false_type{});
            } else {
                half_tile(std::integral_constant<int, 0>{}, std::true_type{});
                half_tile(std::integral_constant<int, 1>{}, std::true_type{});
            }
            __syncwarp();
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();   // the ring is free: the warps join in it

        constexpr int W = 32 * G, HEADS = 8 * NB, PER = HEADS * W + 2 * HEADS;
#pragma unroll
        for (int c = 0; c < G; ++c) {
            const float up = __uint_as_float((254u << 23) - __float_as_uint(down[c]));   // 1 / a power of two
#pragma unroll
            for (int m = 0; m < NB; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) { o[c][0][m][e] *= up; o[c][1][m][e] *= up; }
        }
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
        const bool alone = begin == first && end == last;
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
            if (!alone) {
                const long long unit = part_slot(a, cta, first < from0 ? 0 : 1, h);
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
        __syncthreads();   // the next row's tiles go into the ring
    }
}

// A CTA per (row, query head): joins the parts of a row that several shares hold, each warp every eighth of them (all their loads at once) and the
// warps in order; zeros for a row without entries.
constexpr int kJoinWarps = 8;
__global__ void __launch_bounds__(kJoinWarps * 32) kv4_join_kernel(const AttnArgs a)
{
    __shared__ float sums[kJoinWarps][128], weight[kJoinWarps], highs[kJoinWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.x / a.heads, h = blockIdx.x % a.heads;
    const int first = a.row_ptr[row], last = (int)min((long long)a.row_ptr[row + 1], a.nnz);
    const int c0 = first / a.share, c1 = (last - 1) / a.share, width = attn::part_width(attn::kForward, a.d);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (last > first && c0 == c1) return;
    float x[4] = {}, high = -CUDART_INF_F, l = 0.f;
    if (last > first) {
        constexpr int AT = 8;
        for (int b = c0 + warp; b <= c1; b += kJoinWarps * AT) {   // (one round up to 64 parts)
            float y[AT][4];
            float2 ml[AT];
#pragma unroll
            for (int i = 0; i < AT; ++i) {
                const int c = b + i * kJoinWarps;
                ml[i] = make_float2(-CUDART_INF_F, 0.f);
                y[i][0] = y[i][1] = y[i][2] = y[i][3] = 0.f;
                if (c <= c1) {
                    const long long unit = part_slot(a, c, c == c0, h);
                    ml[i] = a.part_ml[unit];
                    attn::load_part(a.part + unit * width, lane * 4, width, y[i]);
                }
            }
            float to = high;
#pragma unroll
            for (int i = 0; i < AT; ++i) to = fmaxf(to, ml[i].x);
            const float ref = to == -CUDART_INF_F ? 0.f : to, fall = exp2f(high - ref);
            high = to;
            l *= fall;
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] *= fall;
#pragma unroll
            for (int i = 0; i < AT; ++i) {
                const float f = exp2f(ml[i].x - ref);
                l = fmaf(ml[i].y, f, l);
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = fmaf(f, y[i][k], x[k]);
            }
        }
    }
    *reinterpret_cast<float4 *>(&sums[warp][lane * 4]) = make_float4(x[0], x[1], x[2], x[3]);
    if (lane == 0) { weight[warp] = l; highs[warp] = high; }
    __syncthreads();
    if (warp) return;
    high = -CUDART_INF_F;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) high = fmaxf(high, highs[w]);
    const float ref = high == -CUDART_INF_F ? 0.f : high;
    l = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) {
        const float f = exp2f(highs[w] - ref);
        l = fmaf(f, weight[w], l);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = fmaf(f, sums[w][lane * 4 + k], x[k]);
    }
    const float f = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] *= f;
    attn::store4<Bf16, 1>(a.out.at(0, h, row), lane * 4, a.d, x);
    if (lane == 0) a.lse[(long long)row * a.heads + h] = l == 0.f ? -CUDART_INF_F : (high + log2f(l)) * attn::kLn2;
}

}  // namespace kv4
}  // namespace b2sp
