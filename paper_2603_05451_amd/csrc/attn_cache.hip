// Rows of a paged cache in 4 or 8 bits: quantising them as they are written, and reading them back (gfx950).
// attn_cache_write and attn_cache_read of include/attn.h; how, at the top of attn_cache_kernel.inc.
#include "cache_codes.h"
#include "common.h"
#include "launch.h"
#include "ops.h"

namespace attn {

typedef __attribute__((ext_vector_type(2))) uint32_t words2;       // 8 bytes

template <int CTRL>
__device__ __forceinline__ uint32_t quad_move(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true); }

#define ATTN_ELEM bf16
#define ATTN_ELEM8 bf16x8
#define ATTN_ELEM4 bf16x4
#include "elem.inc"
#undef ATTN_ELEM
#undef ATTN_ELEM8
#undef ATTN_ELEM4
#include "attn_cache_kernel.inc"

namespace f16k {
#define ATTN_ELEM f16
#define ATTN_ELEM8 f16x8
#define ATTN_ELEM4 f16x4
#include "elem.inc"
#undef ATTN_ELEM
#undef ATTN_ELEM8
#undef ATTN_ELEM4
#include "attn_cache_kernel.inc"
}  // namespace f16k

static int rows(const CacheRowsArgs& a, bool write)
{
    if (a.c.bits == 4) return a.f16 ? f16k::cache_rows<4>(a, write) : (cache_rows<4>)(a, write);
    return a.f16 ? f16k::cache_rows<8>(a, write) : (cache_rows<8>)(a, write);
}
int launch_cache_write(const CacheRowsArgs& a) { return rows(a, true); }
int launch_cache_read(const CacheRowsArgs& a) { return rows(a, false); }

}  // namespace attn
