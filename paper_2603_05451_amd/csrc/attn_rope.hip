// Rotary positions of queries and keys with the norms of their heads, forward and backward (gfx950): attn_rope_fwd and
// attn_rope_bwd of include/attn.h.  How: at the top of attn_rope_kernel.inc.
#include "common.h"
#include "launch.h"
#include "ops.h"

namespace attn {

template <int CTRL>
__device__ __forceinline__ float dpp_move(float x)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}

// Columns of the blocks' partial rows part[blocks of q, then of k][d], summed in a fixed order: 16 columns of one tensor a block, 64
// threads a column, four rows in flight in each.
__global__ void __launch_bounds__(1024)
attn_rope_sum_kernel(const float* __restrict__ part, int rows_q, int rows_k, int d, float* __restrict__ dwq, float* __restrict__ dwk)
{
    __shared__ float red[64][17];
    const int col = threadIdx.x & 15, first = threadIdx.x >> 4;
    const int k = blockIdx.x * 16 >= (unsigned)d, at = blockIdx.x * 16 - k * d + col;       // (d % 16 == 0)
    float* out = k ? dwk : dwq;
    if (!out) return;
    const float* p = part + (int64_t)(k ? rows_q : 0) * d + at;
    const int rows = k ? rows_k : rows_q;
    float x = 0.f;
    for (int r = first; r < rows; r += 256) {
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = r + 64 * i < rows ? p[(int64_t)(r + 64 * i) * d] : 0.f;
        x += (v[0] + v[1]) + (v[2] + v[3]);
    }
    red[first][col] = x;
    __syncthreads();
    if (first != 0) return;
    float y = 0.f;
#pragma unroll
    for (int i = 0; i < 64; ++i) y += red[i][col];
    out[at] = y;
}

#define ATTN_ELEM bf16
#define ATTN_ELEM8 bf16x8
#define ATTN_ELEM4 bf16x4
#include "elem.inc"
#undef ATTN_ELEM
#undef ATTN_ELEM8
#undef ATTN_ELEM4
#include "attn_rope_kernel.inc"

namespace f16k {
#define ATTN_ELEM f16
#define ATTN_ELEM8 f16x8
#define ATTN_ELEM4 f16x4
#include "elem.inc"
#undef ATTN_ELEM
#undef ATTN_ELEM8
#undef ATTN_ELEM4
#include "attn_rope_kernel.inc"
}  // namespace f16k

int launch_rope(RopeArgs a)
{
    rope_shapes(a.B * a.N, a.heads[0], a.heads[1], a.d, a.backward, a.shape);
    int rc = a.f16 ? f16k::launch_rope_dims(a) : (launch_rope_dims)(a);
    if (rc == 0 && a.part)
        rc = launch_kernel(attn_rope_sum_kernel, dim3(a.d / 8), dim3(1024), 0, a.stream, a.part, a.shape[0].blocks, a.shape[1].blocks, a.d, a.dw[0],
                           a.dw[1]) == hipSuccess ? 0 : -3;
    return rc;
}

}  // namespace attn
