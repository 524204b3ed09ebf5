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

constexpr int kWriteChunk = 4096;   // tokens of one launch: among them a slot named twice is found by comparing
constexpr int kWriteTokens = 8;     // tokens of a CTA
constexpr int kWriteThreads = 256;

// Eight lanes per group, four elements each.  A slot that several tokens of a call name takes the last one's row: inside a launch the
// earlier tokens see the later one and leave the slot alone, and launches follow one another.  Slots outside the cache are skipped.
template <typename T, int V>
__global__ void __launch_bounds__(kWriteThreads) kv4_write_kernel(const T *x, long long ld, long long sh, int tokens, int heads, int d, int G, const int *slots, Cache c)
{
    __shared__ int slot_of[kWriteTokens];
    __shared__ int dead[kWriteTokens];
    const int t0 = blockIdx.x * kWriteTokens;
    if (threadIdx.x < kWriteTokens) {
        slot_of[threadIdx.x] = t0 + threadIdx.x < tokens ? slots[t0 + threadIdx.x] : -1;
        dead[threadIdx.x] = 0;
    }
    __syncthreads();
    int mine[kWriteTokens];
#pragma unroll
    for (int k = 0; k < kWriteTokens; ++k) mine[k] = slot_of[k];
    unsigned again = 0;
    for (int t = t0 + 1 + threadIdx.x; t < tokens; t += kWriteThreads) {
        const int s = slots[t];
#pragma unroll
        for (int k = 0; k < kWriteTokens; ++k)
            if (s == mine[k] && t > t0 + k) again |= 1u << k;
    }
    if (again) {
#pragma unroll
        for (int k = 0; k < kWriteTokens; ++k)
            if (again >> k & 1) dead[k] = 1;
    }
    __syncthreads();
    const int units = kWriteTokens * heads * G;   // groups; a multiple of eight, so octets of lanes are on or off together
    const int g = threadIdx.x & 7;
    for (int u0 = 0; u0 < units; u0 += kWriteThreads / 8) {
        const int u = u0 + (threadIdx.x >> 3);
        const bool on = u < units;
        const int grp = on ? u % G : 0, h = on ? u / G % heads : 0, k = on ? u / G / heads : 0;
        const int slot = slot_of[k];
        const bool live = on && !dead[k] && (unsigned)slot < (unsigned)c.slots;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (live) attn::load4<T, V>(x + (long long)(t0 + k) * ld + h * sh, grp * 32 + g * 4, d, v);
        float top = 0.f;
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            top = fmaxf(top, fabsf(v[i]));
            odd |= !(fabsf(v[i]) <= 3.402823466e38f);
        }
#pragma unroll
        for (int o = 4; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
        const unsigned vote = __ballot_sync(~0u, odd);
        odd = vote >> (threadIdx.x & 24) & 0xff;
        Bf16 s;
        attn::narrow(__fdiv_rn(top, 7.f), s);
        if (odd) s.bits = 0x7fff;
        const float f = attn::widen(s);
        unsigned word = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float q = f > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(v[i], f)), -7.f), 7.f) : 0.f;
            word |= (unsigned)((int)q + 8) << (4 * i);
        }
        if (!live) continue;
        reinterpret_cast<unsigned short *>(c.codes + h * c.code_head + slot * c.code_ld)[g * G + grp] = (unsigned short)word;
        if (g == 0) c.scales[h * c.scale_head + slot * c.scale_ld + grp] = s;
    }
}

// A thread per four elements of the output; rows of slots outside the cache read as zeros.
template <typename T, int V>
__global__ void __launch_bounds__(256) kv4_read_kernel(const int *slots, int tokens, int heads, int d, int G, Cache c, T *out, long long ld, long long sh)
{
    const int per = (d + 3) >> 2;
    const long long u = blockIdx.x * 256ll + threadIdx.x;
    const long long row = u / per;
    if (row >= (long long)tokens * heads) return;
    const int e = (int)(u - row * per), h = (int)(row % heads);
    const long long t = row / heads;
    const int slot = slots[t], grp = e >> 3, g = e & 7;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if ((unsigned)slot < (unsigned)c.slots) {
        const unsigned w = reinterpret_cast<const unsigned short *>(c.codes + h * c.code_head + slot * c.code_ld)[g * G + grp];
        const float s = attn::widen(c.scales[h * c.scale_head + slot * c.scale_ld + grp]);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = s * (float)((int)(w >> (4 * i) & 15) - 8);
    }
    attn::store4<T, V>(out + t * ld + h * sh, e * 4, d, v);
}

// ---- attention ------------------------------------------------------------------------------------------------------------------
struct AttnArgs {
    int M, heads, kv_heads, d, splits, head_blocks;   // head_blocks: groups of 8 * MH query heads that share one K and V
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

// O = softmax(scale Q K^T) V of one query token's heads over (a part of) the slots that its row names.
//
// A CTA takes one token, one key/value head with up to 8 MH query heads that share it, and one part of the row; its four warps take
// every fourth 16 slots each and join at the end.  What it has to read is 36 G bytes a slot, so everything is done to keep loads in
// flight and instructions few: a ring of kStages tiles per warp filled by cp.async; codes become bf16 by one mask each (128 + code);
// the tensor core's legacy form multiplies them (m16n8k16: query heads x elements of K, then query heads x slots of V).
//   * K: the row scale of a group multiplies the 8 products of its 32 elements, in fp32; the 136 that each code carries too much is
//     taken off there as 136 sum(q), instead of off each code.
//   * V: the scale of (slot, group) multiplies the slot's weight before that is rounded to bf16 (half a step, 2^-9 of each weight --
//     the one rounding of this kernel beside that of the output); codes are made whole numbers -7 .. 7 first, as the sum over slots
//     would lose the small result in 136 sum(p).
//   * the running maximum moves only when a logit exceeds it by 8 (to base 2), so that O is rarely rescaled: weights up to 2^8.
// Which slot is which column of the products is free: column n of a half tile is its slot (n & 1) * 4 + n / 2, so that a lane's two
// neighbouring columns are slots 4 apart and the four lanes of a column of V read different banks.
constexpr int kStages = 4, kSlots = 16;
template <int G> struct Smem {
    static constexpr int ROW = 16 * G;
    static constexpr int K = 0, V = kSlots * ROW, KS = 2 * kSlots * ROW, VS = KS + kSlots * 8, IDX = VS + kSlots * 8, STAGE = IDX + kSlots * 4;
    static constexpr int RING = attn::kWarps * kStages * STAGE;
    static constexpr int JOIN = attn::kWarps * (16 * 32 * G + 32) * 4;
    static constexpr int BYTES = RING > JOIN ? RING : JOIN;
};

// The G halfwords of a lane, two to a word.
template <int G> __device__ __forceinline__ void lds_pieces(const char *p, unsigned (&w)[(G + 1) / 2])
{
    if constexpr (G == 4) { const uint2 u = *reinterpret_cast<const uint2 *>(p); w[0] = u.x; w[1] = u.y; }
    else if constexpr (G == 2) { w[0] = *reinterpret_cast<const unsigned *>(p); }
    else if constexpr (G == 1) { w[0] = *reinterpret_cast<const unsigned short *>(p); }
    else {
        const unsigned short *h = reinterpret_cast<const unsigned short *>(p);
        w[0] = h[0] | (unsigned)h[1] << 16;
        w[1] = h[2];
    }
}
template <int C> __device__ __forceinline__ unsigned pick(unsigned a, unsigned b)   // halfword C & 1 of a below that of b
{
    return __byte_perm(a, b, (C & 1) ? 0x7632 : 0x5410);
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

template <int G, int MH>
__global__ void __launch_bounds__(attn::kWarps * 32) kv4_attention_kernel(const AttnArgs a)
{
    using S = Smem<G>;
    __shared__ __align__(16) char smem[S::BYTES];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int group = a.heads / a.kv_heads;
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

    auto fetch_idx = [&](int i) {   // the slot of lane & 15 of this warp's tile i, or -1
        const int at = (warp + i * attn::kWarps) * kSlots + (lane & 15);
        const int s = i < mine && at < n ? idx[at] : -1;
        return (unsigned)s < (unsigned)min(a.k.slots, a.v.slots) ? s : -1;
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
                const int krow = (r & 8) | ((r & 3) << 1) | (r >> 2 & 1);
                const int dst = is_v ? S::V + r * S::ROW + (G == 4 ? ch ^ (r & 2) : ch) * 16 : S::K + krow * S::ROW + ch * 16;
                cp_async(ring_s + st + dst, src + ch * 16, 16, s >= 0 ? 16 : 0);
            }
            {
                const int r = lane & 15;
                const bool is_v = lane >= 16;
                const long long at = is_v ? max(slot, 0) * a.v.scale_ld : max(slot, 0) * a.k.scale_ld;
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

    // Q: lane (g, t) has elements 8 t .. 8 t + 7 of each group of query heads g and (MH = 2) g + 8
    unsigned qa[G][2][2][MH];   // [group][k step][half of k][head]
    float qsum[G][MH];
#pragma unroll
    for (int c = 0; c < G; ++c)
#pragma unroll
        for (int m = 0; m < MH; ++m) {
            const int hq = hb * 8 * MH + m * 8 + g;
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
            qsum[c][m] = 136.f * sum;
        }
    float o[G][4][4] = {};   // [group][element of four][C fragment]
    float top[MH], sum[MH];
#pragma unroll
    for (int m = 0; m < MH; ++m) { top[m] = -CUDART_INF_F; sum[m] = 0.f; }
    const float c2 = a.scale * attn::kLog2e;

    int next = fetch_idx(0);
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) {
        const int now = next;
        next = fetch_idx(i + 1);
        issue(i, now);
    }
    for (int i = 0; i < mine; ++i) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        __syncwarp();
        {
            const int now = next;
            next = fetch_idx(i + kStages);
            issue(i + kStages - 1, now);   // into the stage that the last iteration read (all lanes are past it)
        }
        const char *st = ring + (i % kStages) * S::STAGE;
        const int *slot = reinterpret_cast<const int *>(st + S::IDX);
        float p[2][2][MH];   // [half tile][column 2 t + .][head]
        bool odd_v[2][2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            unsigned w0[(G + 1) / 2], w1[(G + 1) / 2];
            const char *kr = st + S::K + (8 * j + g) * S::ROW;
            lds_pieces<G>(kr + 4 * G * t, w0);
            lds_pieces<G>(kr + 4 * G * t + 2 * G, w1);
            float s[2][MH];
            const int sl0 = slot[8 * j + t], sl1 = slot[8 * j + 4 + t];
            float ks0[G], ks1[G];
            const int ok0 = (G & 1) ? (int)((reinterpret_cast<uintptr_t>(ksc + sl0 * a.k.scale_ld) >> 1) & 1) : 0;
            const int ok1 = (G & 1) ? (int)((reinterpret_cast<uintptr_t>(ksc + sl1 * a.k.scale_ld) >> 1) & 1) : 0;
            if (G & 1) {
                odd_v[j][0] = (reinterpret_cast<uintptr_t>(vsc + sl0 * a.v.scale_ld) >> 1) & 1;
                odd_v[j][1] = (reinterpret_cast<uintptr_t>(vsc + sl1 * a.v.scale_ld) >> 1) & 1;
            }
            lds_scales<G>(st + S::KS + (8 * j + t) * 8, ok0, ks0);
            lds_scales<G>(st + S::KS + (8 * j + 4 + t) * 8, ok1, ks1);
#pragma unroll
            for (int m = 0; m < MH; ++m) s[0][m] = s[1][m] = 0.f;
#pragma unroll
            for (int c = 0; c < G; ++c) {
                const unsigned y = (c & 1) ? pick<1>(w0[c / 2], w1[c / 2]) : pick<0>(w0[c / 2], w1[c / 2]);
                float f[4] = {};
                mma_bf16(f, qa[c][0][0][0], MH == 2 ? qa[c][0][0][MH - 1] : 0u, qa[c][0][1][0], MH == 2 ? qa[c][0][1][MH - 1] : 0u, nibble_pair<0>(y), nibble_pair<1>(y));
                mma_bf16(f, qa[c][1][0][0], MH == 2 ? qa[c][1][0][MH - 1] : 0u, qa[c][1][1][0], MH == 2 ? qa[c][1][1][MH - 1] : 0u, nibble_pair<2>(y), nibble_pair<3>(y));
#pragma unroll
                for (int m = 0; m < MH; ++m) {
                    s[0][m] = fmaf(ks0[c], f[2 * m] - qsum[c][m], s[0][m]);
                    s[1][m] = fmaf(ks1[c], f[2 * m + 1] - qsum[c][m], s[1][m]);
                }
            }
#pragma unroll
            for (int m = 0; m < MH; ++m) {
                p[j][0][m] = sl0 >= 0 ? s[0][m] * c2 : -CUDART_INF_F;
                p[j][1][m] = sl1 >= 0 ? s[1][m] * c2 : -CUDART_INF_F;
            }
        }
        bool move = false;
        float high[MH];
#pragma unroll
        for (int m = 0; m < MH; ++m) {
            float x = fmaxf(fmaxf(p[0][0][m], p[0][1][m]), fmaxf(p[1][0][m], p[1][1][m]));
            x = fmaxf(x, __shfl_xor_sync(~0u, x, 1));
            x = fmaxf(x, __shfl_xor_sync(~0u, x, 2));
            high[m] = x;
            move |= x > top[m] + 8.f;
        }
        if (__any_sync(~0u, move)) {
#pragma unroll
            for (int m = 0; m < MH; ++m) {
                const float to = fmaxf(top[m], high[m]), fall = to == -CUDART_INF_F ? 1.f : exp2f(top[m] - to);
                top[m] = to;
                sum[m] *= fall;
#pragma unroll
                for (int c = 0; c < G; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        o[c][e][2 * m] *= fall;
                        o[c][e][2 * m + 1] *= fall;
                    }
            }
        }
#pragma unroll
        for (int m = 0; m < MH; ++m) {
            const float ref = top[m] == -CUDART_INF_F ? 0.f : top[m];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    p[j][k][m] = exp2f(p[j][k][m] - ref);
                    sum[m] += p[j][k][m];
                }
        }
        // V: rows t and t + 4 of each half tile, this lane's column g of every product
        unsigned v0[2][(G + 1) / 2], v1[2][(G + 1) / 2];
        float s0[2][G], s1[2][G];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r0 = 8 * j + t, r1 = r0 + 4;
            const int at = G == 4 ? ((((g >> 1) ^ (r0 & 2)) << 4) | ((g & 1) << 3)) : 2 * G * g;   // (r1 & 2 = r0 & 2)
            lds_pieces<G>(st + S::V + r0 * S::ROW + at, v0[j]);
            lds_pieces<G>(st + S::V + r1 * S::ROW + at, v1[j]);
            lds_scales<G>(st + S::VS + r0 * 8, (G & 1) ? odd_v[j][0] : 0, s0[j]);
            lds_scales<G>(st + S::VS + r1 * 8, (G & 1) ? odd_v[j][1] : 0, s1[j]);
        }
#pragma unroll
        for (int c = 0; c < G; ++c) {
            unsigned pa[2][MH];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int m = 0; m < MH; ++m) pa[j][m] = attn::bf16x2(p[j][0][m] * s0[j][c], p[j][1][m] * s1[j][c]);
            const unsigned y0 = (c & 1) ? pick<1>(v0[0][c / 2], v1[0][c / 2]) : pick<0>(v0[0][c / 2], v1[0][c / 2]);
            const unsigned y1 = (c & 1) ? pick<1>(v0[1][c / 2], v1[1][c / 2]) : pick<0>(v0[1][c / 2], v1[1][c / 2]);
            const unsigned h0 = MH == 2 ? pa[0][MH - 1] : 0u, h1 = MH == 2 ? pa[1][MH - 1] : 0u;
            mma_bf16(o[c][0], pa[0][0], h0, pa[1][0], h1, minus136(nibble_pair<0>(y0)), minus136(nibble_pair<0>(y1)));
            mma_bf16(o[c][1], pa[0][0], h0, pa[1][0], h1, minus136(nibble_pair<1>(y0)), minus136(nibble_pair<1>(y1)));
            mma_bf16(o[c][2], pa[0][0], h0, pa[1][0], h1, minus136(nibble_pair<2>(y0)), minus136(nibble_pair<2>(y1)));
            mma_bf16(o[c][3], pa[0][0], h0, pa[1][0], h1, minus136(nibble_pair<3>(y0)), minus136(nibble_pair<3>(y1)));
        }
        __syncwarp();
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();   // the ring is free: the warps join in it

    constexpr int W = 32 * G, PER = 16 * W + 32;
    float *join = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int m = 0; m < MH; ++m) {
        float x = sum[m];
        x += __shfl_xor_sync(~0u, x, 1);
        x += __shfl_xor_sync(~0u, x, 2);
        if (t == 0) {
            join[warp * PER + 16 * W + m * 8 + g] = top[m];
            join[warp * PER + 16 * W + 16 + m * 8 + g] = x;
        }
#pragma unroll
        for (int c = 0; c < G; ++c)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                *reinterpret_cast<float4 *>(join + warp * PER + (m * 8 + g) * W + 32 * c + 4 * (2 * t + k)) =
                    make_float4(o[c][0][2 * m + k], o[c][1][2 * m + k], o[c][2][2 * m + k], o[c][3][2 * m + k]);
    }
    __syncthreads();
    const int width = attn::part_width(attn::kForward, a.d);
    for (int i = threadIdx.x; i < 8 * MH * (W / 4); i += attn::kWarps * 32) {
        const int m = i / (W / 4), e = i % (W / 4) * 4, hq = hb * 8 * MH + m;
        if (hq >= group || e >= width) continue;
        float high = -CUDART_INF_F, l = 0.f, x[4] = {};
#pragma unroll
        for (int w = 0; w < attn::kWarps; ++w) high = fmaxf(high, join[w * PER + 16 * W + m]);
        const float ref = high == -CUDART_INF_F ? 0.f : high;
#pragma unroll
        for (int w = 0; w < attn::kWarps; ++w) {
            const float f = exp2f(join[w * PER + 16 * W + m] - ref);
            l = fmaf(f, join[w * PER + 16 * W + 16 + m], l);
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
