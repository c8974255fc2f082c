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

// Columns of the blocks' partial rows part[rows][2][d], summed in a fixed order: 16 columns a block, 16 threads a column.
__global__ void __launch_bounds__(256)
attn_rope_sum_kernel(const float* __restrict__ part, int rows, int d, float* __restrict__ dwq, float* __restrict__ dwk)
{
    __shared__ float red[16][17];
    const int col = threadIdx.x & 15, first = threadIdx.x >> 4;
    const int at = blockIdx.x * 16 + col;                          // of 2 d (d % 16 == 0)
    float x = 0.f;
    for (int r = first; r < rows; r += 16) x += part[(int64_t)r * 2 * d + at];
    red[first][col] = x;
    __syncthreads();
    if (first != 0) return;
    float y = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) y += red[i][col];
    if (at < d) { if (dwq) dwq[at] = y; }
    else if (dwk) dwk[at - d] = y;
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
    const RopeShape r = rope_shape(a.B * a.N, a.heads[0] + a.heads[1], a.d, a.backward);
    a.hg_shift = r.hg_shift;
    a.shares = r.shares;
    a.units = 4 * (r.blocks / r.shares);
    int rc;
    if (a.f16) rc = a.interleaved ? f16k::launch_rope_l<true>(a, r.blocks) : f16k::launch_rope_l<false>(a, r.blocks);
    else rc = a.interleaved ? (launch_rope_l<true>)(a, r.blocks) : (launch_rope_l<false>)(a, r.blocks);
    if (rc == 0 && a.part)
        rc = launch_kernel(attn_rope_sum_kernel, dim3(a.d / 8), dim3(256), 0, a.stream, a.part, r.blocks, a.d, a.dw[0], a.dw[1]) == hipSuccess ? 0 : -3;
    return rc;
}

}  // namespace attn
