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

// Inclusive prefix sums over the lanes of a wave: within 16 lanes, then the ends of rows 0 and 2 to rows 1 and 3, then that of row 1 to
// both upper rows.
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_moved(int x) { return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int wave_prefix(int x)
{
    x = add_moved<0x111, 0xf>(x);          // row_shr 1, 2, 4, 8
    x = add_moved<0x112, 0xf>(x);
    x = add_moved<0x114, 0xf>(x);
    x = add_moved<0x118, 0xf>(x);
    x = add_moved<0x142, 0xa>(x);          // row_bcast 15
    return add_moved<0x143, 0xc>(x);       // row_bcast 31
}
__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_prefix(x), 63); }

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
    return max(((total + p.parts - 1) / p.parts + 3) & ~3, p.min_tiles);
}
// The chunks of a sequence: whole ones, and one that is shorter (also if there are no keys, for its rows have results).
struct CacheSplit {
    int whole, rest;
};
__device__ __forceinline__ CacheSplit cache_split(int len, int chunk_tiles)
{
    const int tiles = (len + 31) >> 5, whole = tiles / chunk_tiles;
    return {whole, tiles > whole * chunk_tiles || tiles == 0};
}

// The sequence and chunk at place `slot` of all chunks: the whole ones of all sequences, in order, then the shorter ones, so that
// these fill up what the others leave.  False behind the last one.
__device__ __forceinline__ bool cache_place(const CachePlanArgs& p, const int* __restrict__ lens, int slot, CachePlace& at)
{
    at.chunk_tiles = cache_chunk_tiles(p, lens);
    for (int pass = 0; pass < 2; ++pass)
        for (int b0 = 0; b0 < p.B; b0 += 64) {
            const int b = b0 + (threadIdx.x & 63);
            const int len = cache_length(p, lens, b);
            const CacheSplit split = b < p.B ? cache_split(len, at.chunk_tiles) : CacheSplit{0, 0};
            const int n = pass ? split.rest : split.whole;
            const int upto = wave_prefix(n);
            const uint64_t past = __ballot(upto > slot);
            if (past) {
                const int l = __builtin_ctzll(past);
                auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
                at.b = b0 + l;
                at.len = of(len);
                at.chunks = of(split.whole + split.rest);
                at.chunk = pass ? of(split.whole) : slot - (of(upto) - of(n));
                return true;
            }
            slot -= __builtin_amdgcn_readlane(upto, 63);
        }
    return false;
}
// The places of sequence b's first whole chunk and of its shorter one (if there is one).
__device__ __forceinline__ void cache_place_of(const CachePlanArgs& p, const int* __restrict__ lens, int b, CachePlace& at, int& slot0, int& rest)
{
    at.b = b;
    at.chunk_tiles = cache_chunk_tiles(p, lens);
    at.chunk = 0;
    int whole = 0, before = 0, rests = 0, len = 0;      // whole chunks of all, those before b, shorter ones before b
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int i = b0 + (threadIdx.x & 63);
        const int n = cache_length(p, lens, i);
        const CacheSplit split = i < p.B ? cache_split(n, at.chunk_tiles) : CacheSplit{0, 0};
        whole += split.whole;
        if (i < b) { before += split.whole; rests += split.rest; }
        if (i == b) len = n;
    }
    at.len = wave_sum(len);
    const CacheSplit mine = cache_split(at.len, at.chunk_tiles);
    at.chunks = mine.whole + mine.rest;
    slot0 = wave_sum(before);
    rest = mine.rest ? wave_sum(whole) + wave_sum(rests) : -1;
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
