// Interface between the attention entry points and the tensor-core kernels.
#pragma once
#include "attention_rows.cuh"

namespace b2sp {
namespace attn {

struct TileCall {
    Shape s;
    Plan plan;
    long long tiles;                     // of all patterns
    const int *row_ptr, *col_idx;        // for rows that have to be taken one by one (see attention_tiles.cuh)
    long long row_ptr_stride, nnz_stride;
    View<const Bf16> q, k, v, dout;
    View<Bf16> out, dq, dk, dv;
    float *lse;
    const float2 *stat;
    long long stat_stride;
    int *status;
};

bool tiles_possible(const Shape &s, const View<const Bf16> *views, int n);
b2sp_status tiles_forward(const TileCall &c, cudaStream_t st, int *launches);
b2sp_status tiles_backward(const TileCall &c, cudaStream_t st, int *launches);

}  // namespace attn
}  // namespace b2sp
