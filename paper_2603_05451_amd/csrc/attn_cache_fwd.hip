// Attention of few queries per sequence over a paged cache in 4 or 8 bits (gfx950): attn_cache_fwd of include/attn.h.  How: at the
// top of attn_cache_fwd_kernel.inc.  ATTN_F16 names the element type of this object: one of the two per compilation.
#include "cache_codes.h"
#include "common.h"
#include "launch.h"
#include "ops.h"

namespace attn {
namespace {

// v_mfma_f32_16x16x32, D = A(16x32) * B(32x16) + C.  Lane l = 16 g + c:  A: row c, k = 8g..8g+7;  B: column c, the same k;
// C/D register r: row 4g + r, column c.
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// max / sum with the lane 16 apart (v_permlane16_swap exchanges odd rows of 16 lanes of the first operand with even rows of the second)
__device__ __forceinline__ float xquarter_max(float x)
{
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float xquarter_sum(float x)
{
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// ---- which keys a block takes, from the lengths in device memory
struct CachePlanArgs {
    int B, Hkv, page_shift, most;       // most: keys that a row of the table has room for
    int parts, min_tiles;               // cache_shape's
};
struct CachePlace {
    int b, len, chunk, chunks, chunk_tiles;     // of a sequence; chunks of chunk_tiles 32-key tiles
};

__device__ __forceinline__ int wave_sum(int x)
{
#pragma unroll
    for (int m = 1; m < 64; m *= 2) x += __shfl_xor(x, m);
    return x;
}
__device__ __forceinline__ int wave_prefix(int x)       // inclusive
{
    const int l = threadIdx.x & 63;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const int y = __shfl_up(x, m);
        x += l >= m ? y : 0;
    }
    return x;
}
// Keys of sequence b as the kernels take them: no more than its row of the table has room for, none if the length is negative.
__device__ __forceinline__ int cache_length(const CachePlanArgs& p, const int* __restrict__ lens, int b)
{
    return b < p.B ? min(max(lens[b], 0), p.most) : 0;
}
// Tiles of a chunk: all keys in about `parts` chunks, whole turns of the four waves, not below min_tiles.
__device__ __forceinline__ int cache_chunk_tiles(const CachePlanArgs& p, const int* __restrict__ lens)
{
    int total = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) total += (cache_length(p, lens, b0 + (threadIdx.x & 63)) + 31) >> 5;
    total = wave_sum(total);
    return __builtin_amdgcn_readfirstlane(max(((total + p.parts - 1) / p.parts + 3) & ~3, p.min_tiles));
}
__device__ __forceinline__ int cache_chunks(int len, int chunk_tiles) { return max(1, (((len + 31) >> 5) + chunk_tiles - 1) / chunk_tiles); }

// The sequence and chunk at place `slot` of all chunks, the sequences' in order; false behind the last one.
__device__ __forceinline__ bool cache_place(const CachePlanArgs& p, const int* __restrict__ lens, int slot, CachePlace& at)
{
    at.chunk_tiles = cache_chunk_tiles(p, lens);
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int b = b0 + (threadIdx.x & 63);
        const int len = cache_length(p, lens, b);
        const int n = b < p.B ? cache_chunks(len, at.chunk_tiles) : 0;
        const int upto = wave_prefix(n);
        const uint64_t past = __ballot(upto > slot);
        if (past) {
            const int l = __builtin_ctzll(past);
            at.b = b0 + l;
            at.len = __builtin_amdgcn_readlane(len, l);
            at.chunks = __builtin_amdgcn_readlane(n, l);
            at.chunk = slot - (__builtin_amdgcn_readlane(upto, l) - at.chunks);
            return true;
        }
        slot -= __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}
// The place of sequence b's first chunk.
__device__ __forceinline__ void cache_place_of(const CachePlanArgs& p, const int* __restrict__ lens, int b, CachePlace& at, int& slot0)
{
    at.b = b;
    at.chunk_tiles = cache_chunk_tiles(p, lens);
    at.len = cache_length(p, lens, b);
    at.chunks = __builtin_amdgcn_readfirstlane(cache_chunks(at.len, at.chunk_tiles));
    at.chunk = 0;
    int before = 0;
    for (int b0 = 0; b0 < b; b0 += 64) {
        const int i = b0 + (threadIdx.x & 63);
        if (i < b) before += cache_chunks(cache_length(p, lens, i), at.chunk_tiles);
    }
    slot0 = __builtin_amdgcn_readfirstlane(wave_sum(before));
}

#if ATTN_F16
#define ATTN_ELEM f16
#define ATTN_ELEM8 f16x8
#define ATTN_ELEM4 f16x4
#else
#define ATTN_ELEM bf16
#define ATTN_ELEM8 bf16x8
#define ATTN_ELEM4 bf16x4
#endif
#include "elem.inc"
#include "attn_cache_fwd_kernel.inc"

}  // namespace

#if ATTN_F16
int launch_cache_fwd_f16(const CacheFwdArgs& a) { return cache_fwd_dims(a); }
#else
int launch_cache_fwd_bf16(const CacheFwdArgs& a) { return cache_fwd_dims(a); }
#endif

}  // namespace attn
