// Attention of chunks of new tokens over a paged cache in 4 or 8 bits (gfx950): attn_cache_chunk_fwd of include/attn.h.  How: at the top
// of attn_cache_chunk_kernel.inc.  ATTN_F16 names the element type of this object: one of the two per compilation.
#include "cache_codes.h"
#include "common.h"
#include "launch.h"
#include "ops.h"
#include "wave_sums.h"

namespace attn {
namespace {

// ---- which rows and keys a block takes, from the boundaries and lengths in device memory
struct ChunkPlanArgs {
    int B, T, G, Hkv, page_shift, most;     // most: keys that a row of the table has room for
    int few;                                // chunk_shape's
    int tile_shift, places;                 // keys of a step of the body for many rows, 2^tile_shift; blocks of a round per KV head (0: no keys are divided)
};
// A sequence: its first query, number of queries (0: there is nothing to do) and of keys.
struct ChunkSeq {
    int q0, nq, len;
};
struct ChunkPlace {
    ChunkSeq s;
    int b;                                  // its index
    int rt, part, parts, part_steps;        // row tile; which of the parts of its keys, of so many steps
    int first_tile, tile;                   // where results of parts go, in tiles of 32 rows per KV head: the sequence's first, the unit's first
};
// Sequences with few rows (queries times heads of a group) go by another body: 32 rows to a block, 128 keys to a step of it.
__device__ __forceinline__ bool chunk_few(const ChunkSeq& s, const ChunkPlanArgs& p) { return s.nq * p.G <= p.few; }
__device__ __forceinline__ int chunk_row_shift(const ChunkSeq& s, const ChunkPlanArgs& p) { return chunk_few(s, p) ? 5 : 7; }        // rows of a block, 2^...
static_assert(kChunkRows == 128);

// What every wave of a launch finds out, a sequence per lane (the first 64 stay in registers).
struct ChunkWork {
    const ChunkPlanArgs& p;
    const int* __restrict__ cu;
    const int* __restrict__ lens;
    ChunkSeq held;
    float per_cost;         // 1 / (the cost of a part, in quarters of a step)
    float per_unit;         // n0 steps of many rows take n0 / n + n / per_unit in n parts, which n^2 = n0 per_unit makes least

    __device__ __forceinline__ ChunkSeq fetch(int b) const { return fetch(p, cu, lens, b); }
    __device__ __forceinline__ static ChunkSeq fetch(const ChunkPlanArgs& p, const int* __restrict__ cu, const int* __restrict__ lens, int b)
    {
        if (b >= p.B) return {0, 0, 0};
        const int q0 = cu[b], q1 = cu[b + 1];
        const bool inside = q0 >= 0 && q1 > q0 && q1 <= p.T;               // others are not acted on
        return {q0, inside ? q1 - q0 : 0, min(max(lens[b], 0), p.most)};
    }
    // f(sequence of the lane, its index), 64 sequences after the other, until it says true
    template <typename F>
    __device__ __forceinline__ void each(F&& f) const
    {
        const int lane = threadIdx.x & 63;
        if (f(held, lane)) return;
        for (int b0 = 64; b0 < p.B; b0 += 64)
            if (f(fetch(b0 + lane), b0 + lane)) return;
    }
    __device__ __forceinline__ static int rounded(int x, int shift) { return (x + (1 << shift) - 1) >> shift; }
    __device__ __forceinline__ int row_tiles(const ChunkSeq& s) const { return rounded(s.nq * p.G, chunk_row_shift(s, p)); }
    __device__ __forceinline__ int step_shift(const ChunkSeq& s) const { return chunk_few(s, p) ? 7 : p.tile_shift; }
    __device__ __forceinline__ int steps(const ChunkSeq& s) const { return rounded(s.len, step_shift(s)); }
    __device__ __forceinline__ int step_cost(const ChunkSeq& s) const { return chunk_few(s, p) ? kChunkFewCost : 4; }
    // (by a product, not exactly rounded up: every wave that asks gets the same number, and the parts follow from it)
    __device__ __forceinline__ int parts(const ChunkSeq& s) const
    {
        if (p.places == 0) return 1;
        const bool few = chunk_few(s, p);
        const float n = (float)steps(s), of_cost = fminf(few ? kChunkFewCost * per_cost : 4 * per_cost, 0.25f);      // a part has four steps or more
        const int most = (int)ceilf(n * of_cost - 0.01f);
        return max(1, few ? most : min(most, (int)__builtin_amdgcn_sqrtf(n * per_unit)));
    }
    __device__ __forceinline__ int units(const ChunkSeq& s) const { return row_tiles(s) * parts(s); }
    __device__ __forceinline__ int unit_tiles(const ChunkSeq& s) const { return 1 << (chunk_row_shift(s, p) - 5); }      // tiles of 32 rows of a unit

    // What a part costs: all steps of all row tiles in about `places` parts (a round of blocks), longer if the sequences' last, shorter parts
    // would make it more.
    __device__ __forceinline__ ChunkWork(const ChunkPlanArgs& plan, const int* __restrict__ c, const int* __restrict__ l) : p(plan), cu(c), lens(l)
    {
        held = fetch(threadIdx.x & 63);
        per_cost = per_unit = 1.f;
        if (p.places == 0) return;
        float total = 0.f, many = 0.f;
        each([&](const ChunkSeq& s, int) {
            const float n = (float)row_tiles(s);
            total += n * (float)steps(s) * (float)step_cost(s);
            if (!chunk_few(s, p)) many += n;
            return false;
        });
        per_unit = kChunkPartCost / fmaxf(wave_sum(many) * (float)p.Hkv, 1.f);
        per_cost = (float)p.places / fmaxf(wave_sum(total), 1.f);
        for (int i = 0; i < 3; ++i) {
            int n = 0;
            each([&](const ChunkSeq& s, int) { n += units(s); return false; });
            n = wave_sum(n);
            if (n <= p.places) break;
            per_cost *= 0.8f;
        }
    }
    // The sequence and its part that unit u is; false behind the last one.
    __device__ __forceinline__ bool find(int u, ChunkPlace& at) const
    {
        bool found = false;
        int before = 0, tiles_before = 0;
        each([&](const ChunkSeq& s, int b) {
            const int mine = units(s), upto = before + wave_prefix(mine);
            const int tiles = p.places && parts(s) > 1 ? mine * unit_tiles(s) : 0;
            const int tiles_upto = p.places ? tiles_before + wave_prefix(tiles) : 0;
            const uint64_t past = __ballot(upto > u);
            if (past) {
                const int l = __builtin_ctzll(past);
                auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
                at.s = {of(s.q0), of(s.nq), of(s.len)};
                at.b = of(b);
                at.first_tile = of(tiles_upto) - of(tiles);
                place(at, u - (of(upto) - of(mine)));
                return found = true;
            }
            before = __builtin_amdgcn_readlane(upto, 63);
            tiles_before = __builtin_amdgcn_readlane(tiles_upto, 63);
            return false;
        });
        return found;
    }
    // Unit `local` of its sequence: part by part of the keys, in each the row tiles from the last, whose loops are the longest under the
    // mask, to the first.
    __device__ __forceinline__ void place(ChunkPlace& at, int local) const
    {
        const int rts = row_tiles(at.s), n = steps(at.s);
        at.parts = parts(at.s);
        at.part = local / rts;
        at.rt = rts - 1 - (local - at.part * rts);
        at.part_steps = (n + at.parts - 1) / at.parts;
        at.tile = at.first_tile + local * unit_tiles(at.s);
    }
    // The sequence of query t, as its lengths say (what its parts are, the attention kernel has left behind).
    __device__ __forceinline__ static bool of_query(const ChunkPlanArgs& p, const int* __restrict__ cu, const int* __restrict__ lens, int t, ChunkSeq& s, int& b)
    {
        for (int b0 = 0; b0 < p.B; b0 += 64) {
            const ChunkSeq x = fetch(p, cu, lens, b0 + (threadIdx.x & 63));
            const uint64_t here = __ballot(x.nq > 0 && t >= x.q0 && t < x.q0 + x.nq);
            if (here) {
                const int l = __builtin_ctzll(here);
                auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
                s = {of(x.q0), of(x.nq), of(x.len)};
                b = b0 + l;
                return true;
            }
        }
        return false;
    }
};

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
#include "attn_cache_chunk_kernel.inc"

}  // namespace

#if ATTN_F16
int launch_cache_chunk_f16(const CacheChunkArgs& a) { return cache_chunk_dims(a); }
#else
int launch_cache_chunk_bf16(const CacheChunkArgs& a) { return cache_chunk_dims(a); }
#endif

}  // namespace attn
