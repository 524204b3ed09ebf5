// Launches of the tensor-core attention kernels: tensor maps, grids.
#include "attention_tiles.cuh"

#include <algorithm>
#include <atomic>
#include <climits>
#include <mutex>

namespace b2sp {
namespace attn {
namespace {

using EncodeTiledFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                   const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn()
{
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(p);
    });
    return fn;
}

// [batch][heads][rows][d] in boxes of `box` rows x 64 columns, 128-byte swizzle; what lies outside reads as zeros.  Dimensions that
// are shared (stride 0) or single become one, and their coordinate 0.
bool make_map(CUtensorMap *tm, const View<const Bf16> &v, int batch, int heads, int rows, int d, int box, Op *op)
{
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    const bool h1 = heads == 1 || v.sh == 0, b1 = batch == 1 || v.sb == 0, r1 = rows == 1;
    op->hm = h1 ? 0 : 1;
    op->bm = b1 ? 0 : 1;
    cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)rows, (cuuint64_t)(h1 ? 1 : heads), (cuuint64_t)(b1 ? 1 : batch)};
    cuuint64_t strides[3] = {(cuuint64_t)(r1 ? 256 : v.ld * 2), (cuuint64_t)(h1 ? 256 : v.sh * 2), (cuuint64_t)(b1 ? 256 : v.sb * 2)};
    cuuint32_t boxes[4] = {64, (cuuint32_t)box, 1, 1}, ones[4] = {1, 1, 1, 1};
    return enc(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<Bf16 *>(v.p), dims, strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Raises a kernel's limit of dynamic shared memory once per kernel and device.
template <class K> bool allow_smem(K *kernel, int bytes, std::atomic<unsigned long long> &done)
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    const unsigned long long bit = 1ull << (dev & 63);
    if (done.load(std::memory_order_acquire) & bit) return true;
    if (cudaFuncSetAttribute(reinterpret_cast<const void *>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
    done.fetch_or(bit, std::memory_order_release);
    return true;
}

TileArgs args(const TileCall &c)
{
    TileArgs a = {};
    a.g.s = c.s;
    a.g.ptr = c.row_ptr; a.g.idx = c.col_idx; a.g.ptr_stride = c.row_ptr_stride; a.g.idx_stride = c.nnz_stride;
    a.g.q = c.q; a.g.k = c.k; a.g.v = c.v; a.g.dout = c.dout;
    a.g.stat = c.stat; a.g.stat_stride = c.stat_stride;
    a.g.lse = c.lse; a.g.lse_head = c.s.M; a.g.lse_row = 1;
    a.g.splits = 1;
    a.plan = c.plan;
    a.col_ptr = c.plan.col_ptr; a.row_idx = c.plan.row_idx;
    a.status = c.status;
    return a;
}

template <int DP> b2sp_status forward(const TileCall &c, cudaStream_t st, int *launches)
{
    static std::atomic<unsigned long long> done{0};
    TileArgs a = args(c);
    a.g.out1 = c.out; a.g.rows = c.s.M;
    CUtensorMap q, k, v;
    if (!make_map(&q, c.q, c.s.batch, c.s.heads, c.s.M, c.s.d, 128, &a.q) || !make_map(&k, c.k, c.s.batch, c.s.kv_heads, c.s.K, c.s.d, 128, &a.k) ||
        !make_map(&v, c.v, c.s.batch, c.s.kv_heads, c.s.K, c.s.d, 128, &a.v) || !allow_smem(tile_forward_kernel<DP>, FwdCfg<DP>::BYTES, done))
        return B2SP_ERR_CUDA;
    const long long blocks = (long long)c.s.batch * c.s.heads * c.plan.RB;
    if (blocks > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    tile_forward_kernel<DP><<<(unsigned)blocks, kTileThreads, FwdCfg<DP>::BYTES, st>>>(q, k, v, a);
    ++*launches;
    return cudaGetLastError() == cudaSuccess ? B2SP_OK : B2SP_ERR_CUDA;
}

template <int DP> b2sp_status backward(const TileCall &c, cudaStream_t st, int *launches)
{
    static std::atomic<unsigned long long> done_q{0}, done_kv{0};
    TileArgs a = args(c);
    CUtensorMap q, o, k, v;
    const Shape &s = c.s;
    if (!allow_smem(tile_dq_kernel<DP>, DqCfg<DP>::BYTES, done_q) || !allow_smem(tile_dkv_kernel<DP>, DkvCfg<DP>::BYTES, done_kv)) return B2SP_ERR_CUDA;
    const long long qb = (long long)s.batch * s.heads * c.plan.RB, kb = (long long)s.batch * s.kv_heads * c.plan.CB;
    if (qb > INT_MAX || kb > INT_MAX) return B2SP_ERR_UNSUPPORTED;
    if (!make_map(&q, c.q, s.batch, s.heads, s.M, s.d, 128, &a.q) || !make_map(&o, c.dout, s.batch, s.heads, s.M, s.d, 128, &a.dout) ||
        !make_map(&k, c.k, s.batch, s.kv_heads, s.K, s.d, 64, &a.k) || !make_map(&v, c.v, s.batch, s.kv_heads, s.K, s.d, 64, &a.v))
        return B2SP_ERR_CUDA;
    a.g.out1 = c.dq; a.g.rows = s.M;
    tile_dq_kernel<DP><<<(unsigned)qb, kTileThreads, DqCfg<DP>::BYTES, st>>>(q, o, k, v, a);
    if (!make_map(&q, c.q, s.batch, s.heads, s.M, s.d, 64, &a.q) || !make_map(&o, c.dout, s.batch, s.heads, s.M, s.d, 64, &a.dout) ||
        !make_map(&k, c.k, s.batch, s.kv_heads, s.K, s.d, 128, &a.k) || !make_map(&v, c.v, s.batch, s.kv_heads, s.K, s.d, 128, &a.v))
        return B2SP_ERR_CUDA;
    a.g.out1 = c.dk; a.g.out2 = c.dv; a.g.rows = s.K;
    tile_dkv_kernel<DP><<<(unsigned)kb, DkvCfg<DP>::THREADS, DkvCfg<DP>::BYTES, st>>>(q, o, k, v, a);
    *launches += 2;
    return cudaGetLastError() == cudaSuccess ? B2SP_OK : B2SP_ERR_CUDA;
}

}  // namespace

// Widths up to 128 in whole 16-byte pieces, every address and stride a multiple of 16 bytes, and a factor that keeps the order of the
// products (the reference of the exponentials is the largest of them).
bool tiles_possible(const Shape &s, const View<const Bf16> *views, int n)
{
    if (s.d > kMaxTileHeadDim || (s.d & 7) || !(s.scale > 0.f) || !(s.scale <= 3.4e38f)) return false;
    for (int i = 0; i < n; ++i) {
        const View<const Bf16> &v = views[i];
        if ((reinterpret_cast<uintptr_t>(v.p) & 15) || ((v.ld | v.sh | v.sb) & 7) || v.ld < s.d) return false;
        if (v.ld >= (1ll << 38) || v.sh >= (1ll << 38) || v.sb >= (1ll << 38)) return false;
    }
    return true;
}

b2sp_status tiles_forward(const TileCall &c, cudaStream_t st, int *launches)
{
    return c.s.d <= 64 ? forward<64>(c, st, launches) : forward<128>(c, st, launches);
}
b2sp_status tiles_backward(const TileCall &c, cudaStream_t st, int *launches)
{
    return c.s.d <= 64 ? backward<64>(c, st, launches) : backward<128>(c, st, launches);
}

}  // namespace attn
}  // namespace b2sp
