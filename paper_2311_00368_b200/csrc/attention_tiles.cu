// Attention on the tensor cores: not there yet, every call takes the row kernels.
#include "attention_tiles.h"

namespace b2sp {
namespace attn {

bool tiles_possible(const Shape &, const View<const Bf16> *, int) { return false; }
b2sp_status tiles_forward(const TileCall &, cudaStream_t, int *) { return B2SP_ERR_UNSUPPORTED; }
b2sp_status tiles_backward(const TileCall &, cudaStream_t, int *) { return B2SP_ERR_UNSUPPORTED; }

}  // namespace attn
}  // namespace b2sp
