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
    int parts, min_tiles, waves;        // cache_shape's
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

// The chunks of a sequence: whole ones, and one that is shorter (also if there are no keys, for its rows have results), which is of class
// 1 ... 4 by its length in quarters, the longest first.
struct CacheSplit {
    int whole, rest;            // rest: its class, 0 if there is none
};

// What every wave of a launch finds out from the lengths, a sequence per lane; those of the first 64 HELD sequences are loaded at once and
// stay in registers (300 sequences of 500 keys, 8 heads, d = 128: 58 us with the loads of 64 sequences one after the other, three times).
// HELD = 1 is for up to 64 sequences: the code of the others, which a launch would have to fetch past, costs 0.3 ... 0.6 us.
template <int HELD>
struct CacheLengths {
    const CachePlanArgs& p;
    const int* __restrict__ lens;
    int held[HELD], chunk_tiles;
    float per_chunk;

    // Keys of sequence b as the kernels take them: no more than its row of the table has room for, none if the length is negative.
    __device__ __forceinline__ int fetch(int b) const { return b < p.B ? min(max(lens[b], 0), p.most) : 0; }
    // f(first of 64 sequences, length of the lane's), in order, until it says true
    template <typename F>
    __device__ __forceinline__ void each(F&& f) const
    {
        if (f(0, held[0]) || HELD == 1) return;
#pragma unroll
        for (int i = 1; i < HELD; ++i)
            if (64 * i >= p.B || f(64 * i, held[i])) return;
        for (int b0 = 64 * HELD; b0 < p.B; b0 += 64)
            if (f(b0, fetch(b0 + (threadIdx.x & 63)))) return;
    }
    __device__ __forceinline__ CacheLengths(const CachePlanArgs& plan, const int* __restrict__ l) : p(plan), lens(l)
    {
#pragma unroll
        for (int i = 0; i < HELD; ++i) held[i] = HELD == 1 || 64 * i < p.B ? fetch(64 * i + (threadIdx.x & 63)) : 0;
        // tiles of a chunk: all keys in about `parts` chunks, but the mean sequence in equal ones (of 1.2 chunks it would leave most of a
        // block's or wave's time unused); whole turns of its waves, not below min_tiles
        int total = 0, used = 0;
        each([&](int, int len) { total += (len + 31) >> 5; used += __popcll(__ballot(len > 0)); return false; });
        total = wave_sum(total);
        const uint32_t even = (uint32_t)(total + p.parts - 1) / p.parts, mean = (uint32_t)total / max(used, 1);
        const uint32_t n = (4 * mean + even) / max(4 * even, 1u);                      // mean / even, less a quarter, rounded
        chunk_tiles = max(((int)(n ? (mean + n - 1) / n : even) + p.waves - 1) & -p.waves, p.min_tiles);
        per_chunk = 1.0f / (float)chunk_tiles;
    }
    __device__ __forceinline__ CacheSplit split(int b, int len) const
    {
        if (b >= p.B) return {0, 0};
        const int tiles = (len + 31) >> 5;
        int whole = (int)((float)tiles * per_chunk), r = tiles - whole * chunk_tiles;      // (up to 2^26 / 8: off by one at most)
        if (r < 0) { --whole; r += chunk_tiles; }
        if (r >= chunk_tiles) { ++whole; r -= chunk_tiles; }
        r *= 4;
        return {whole, r == 0 && tiles > 0 ? 0 : 4 - (r >= chunk_tiles) - (r >= 2 * chunk_tiles) - (r >= 3 * chunk_tiles)};
    }
    // chunks of the five kinds: n[0] whole ones, n[1 ... 4] shorter ones
    __device__ __forceinline__ void count(int (&n)[5]) const
    {
#pragma unroll
        for (int c = 0; c < 5; ++c) n[c] = 0;
        each([&](int b0, int len) {
            const CacheSplit s = split(b0 + (threadIdx.x & 63), len);
            n[0] += s.whole;
#pragma unroll
            for (int c = 1; c < 5; ++c) n[c] += __popcll(__ballot(s.rest == c));
            return false;
        });
        n[0] = wave_sum(n[0]);
    }
};

// The sequence and chunk at place `slot` of all chunks: kind by kind, in the sequences' order within a kind.  The longest first, so that the
// shorter ones fill up what the others leave (48 sequences of 67 ... 7696 keys, 8 heads, d = 128, 4 bits: 24.8 us with the shorter chunks in
// the sequences' order, 21.5 so; 19.5 where all have the mean length).  False behind the last chunk.
template <int HELD>
__device__ __forceinline__ bool cache_place_among(const CachePlanArgs& p, const int* __restrict__ lens, int slot, CachePlace& at)
{
    const CacheLengths<HELD> all(p, lens);
    at.chunk_tiles = all.chunk_tiles;
    int n[5], kind = 0;
    all.count(n);
#pragma unroll
    for (int c = 0; c < 5; ++c)
        if (kind == c && slot >= n[c]) { slot -= n[c]; kind = c + 1; }
    if (kind == 5) return false;
    all.each([&](int b0, int len) {
        const CacheSplit split = all.split(b0 + (threadIdx.x & 63), len);
        const int mine = kind ? split.rest == kind : split.whole;
        const int upto = wave_prefix(mine);
        const uint64_t past = __ballot(upto > slot);
        if (past) {
            const int l = __builtin_ctzll(past);
            auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
            at.b = b0 + l;
            at.len = of(len);
            at.chunks = of(split.whole + (split.rest > 0));
            at.chunk = kind ? of(split.whole) : slot - (of(upto) - of(mine));
            return true;
        }
        slot -= __builtin_amdgcn_readlane(upto, 63);
        return false;
    });
    return true;
}
__device__ __forceinline__ bool cache_place(const CachePlanArgs& p, const int* __restrict__ lens, int slot, CachePlace& at)
{
    return p.B <= 64 ? cache_place_among<1>(p, lens, slot, at) : cache_place_among<8>(p, lens, slot, at);
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
