// Host side of the tensor-core attention kernels: tensor maps, shared-memory limits, launches behind a running kernel.
#pragma once
#include <cuda.h>

#include <atomic>
#include <mutex>

#include "attention_tiles.cuh"

namespace b2sp {
namespace attn {

using EncodeTiledFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                   const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiledFn encode_fn()
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
inline bool make_map(CUtensorMap *tm, const View<const Bf16> &v, int batch, int heads, int rows, int d, int box, Op *op)
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

template <class... KArgs, class... Args>
inline void launch_behind_smem(void (*kern)(KArgs...), unsigned blocks, unsigned threads, size_t smem, cudaStream_t st, const Args &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaLaunchKernelEx(&cfg, kern, args...);
}

}  // namespace attn
}  // namespace b2sp
