// Eviction from the paged cache by accumulated weight (gfx950): attn_cache_evict of include/attn.h.
//
// A block has a (sequence, KV head).  With `left` = min(len, keep) rows to stay, `recent` of them the last ones, the others (`stay`) are the
// candidates j < of = len - recent with the greatest weights, ties to the lowest j.  The weights are taken as whole numbers of the same order
// (least_first), and the stay-th greatest is found digit by digit (11, 11 and 10 bits) with a histogram in LDS.  Survivors below `stay` remain
// where they are.  There are as many other rows below (holes) as survivors from there on (movers): both are listed, holes first, in ascending
// order, by sums over the block, and the i-th mover goes into the i-th hole.  At most len - left + recent rows are moved at all, where closing
// the cache up in order would move nearly all of them.  The recent rows then go to the places from `stay` on, in order.
//
// The only atomics are counts of whole numbers: results do not depend on their order.
#include "common.h"
#include "launch.h"
#include "ops.h"
#include "wave_sums.h"

namespace attn {
namespace {

struct EvictPlan {
    int Hkv, page_shift, most, table_width, pages, recent;
    int kb, vb, ksb, vsb;       // bytes of a row: codes and scales of keys and values
    int64_t ints;
};

constexpr int kThreads = 1024;

// Weights in ascending order as whole numbers: 0 is a row that is not in the cache, NaN the greatest, -0 and 0 are equal.
__device__ __forceinline__ uint32_t least_first(float w)
{
    if (w != w) return 0xffffffffu;
    const uint32_t x = __float_as_uint(w + 0.0f);
    return x & 0x80000000u ? ~x : x | 0x80000000u;
}

// Exclusive sums over the block's threads, and the sum of all: to `before` and `all`.  `part`: 17 ints of LDS, free again behind the call's
// last barrier.
__device__ __forceinline__ void block_sums(int x, ATTN_LDS int* part, int& before, int& all)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int upto = wave_prefix(x);
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    const int p = lane < kThreads / 64 ? part[lane] : 0, q = wave_prefix(p);
    before = upto - x + (wave ? __builtin_amdgcn_readlane(q, wave - 1) : 0);
    all = __builtin_amdgcn_readlane(q, 63);
    __syncthreads();
}

__global__ void __launch_bounds__(kThreads)
attn_cache_evict_kernel(uint8_t* __restrict__ kc, uint8_t* __restrict__ ks, uint8_t* __restrict__ vc, uint8_t* __restrict__ vs,
                        float* __restrict__ weights, const int* __restrict__ table, const int* __restrict__ lens, const int* __restrict__ keep,
                        int* __restrict__ lens_out, EvictPlan plan, int* __restrict__ places_of_all)
{
    __shared__ int count[2048];
    __shared__ int part_[32];
    __shared__ int found[2];
    ATTN_LDS int* const part = (ATTN_LDS int*)part_;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = (int)blockIdx.x / plan.Hkv, kvh = (int)blockIdx.x - b * plan.Hkv;
    const int len = min(max(lens[b], 0), plan.most), left = min(len, max(keep[b], 0));
    if (kvh == 0 && tid == 0) lens_out[b] = left;
    if (left == len) return;
    const int recent = min(plan.recent, left), stay = left - recent, of = len - recent;
    const int* const pages_of = table + (int64_t)b * plan.table_width;
    const int in_page = (1 << plan.page_shift) - 1;
    // the row of key j among all rows [pages, Hkv, page], or -1
    auto row_of = [&](int j) __attribute__((always_inline)) -> int64_t {
        const int page = pages_of[j >> plan.page_shift];
        return (unsigned)page >= (unsigned)plan.pages ? -1 : (((int64_t)page * plan.Hkv + kvh) << plan.page_shift) + (j & in_page);
    };
    // four keys from j on, j a multiple of 4: they are in one page
    auto keys_at = [&](int j, uint32_t (&x)[4]) __attribute__((always_inline)) {
        const int64_t r = row_of(j);
        f32x4 w = {0.f, 0.f, 0.f, 0.f};
        if (r >= 0) w = *(const f32x4*)(weights + r);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = r >= 0 ? least_first(w[e]) : 0u;
    };
    int* const places = places_of_all + (int64_t)blockIdx.x * plan.ints;

    int moves = 0;
    if (stay > 0) {
        // ---- the stay-th greatest: its digits from the highest on
        uint32_t prefix = 0;                               // those found so far
        int wanted = stay;                                 // the greatest `wanted` of the keys that begin with them
#pragma unroll 1
        for (int digit = 0; digit < 3; ++digit) {
            const int low = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
            for (int i = tid; i < 2048; i += kThreads) count[i] = 0;
            __syncthreads();
            for (int j = 4 * tid; j < of; j += 4 * kThreads) {
                uint32_t x[4];
                keys_at(j, x);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool mine = j + e < of && (digit == 0 || x[e] >> (low + bits) == prefix);
                    if (mine) atomicAdd(&count[(x[e] >> low) & ((1 << bits) - 1)], 1);
                }
            }
            __syncthreads();
            // places 2 tid and 2 tid + 1, counted from the greatest
            const int hi = count[2047 - 2 * tid], lo = count[2046 - 2 * tid];
            int before, all;
            block_sums(hi + lo, part, before, all);
            if (before < wanted && wanted <= before + hi + lo) {
                const bool first = wanted <= before + hi;
                found[0] = 2047 - 2 * tid - (first ? 0 : 1);
                found[1] = wanted - before - (first ? 0 : hi);
            }
            __syncthreads();
            prefix = prefix << bits | (uint32_t)found[0];
            wanted = found[1];
            __syncthreads();
        }
        const uint32_t least = prefix;                     // of the survivors; `wanted` of those that are equal to it survive, the first ones

        // ---- holes and movers, in ascending order
        int equal = 0;
        for (int j0 = 0; j0 < of; j0 += 4 * kThreads) {
            const int j = j0 + 4 * tid;
            uint32_t x[4] = {0, 0, 0, 0};
            if (j < of) keys_at(j, x);
            int n = 0, before, all;
#pragma unroll
            for (int e = 0; e < 4; ++e) n += j + e < of && x[e] == least;
            block_sums(n, part, before, all);
            before += equal;
            equal += all;
            bool listed[4];
            n = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool same = x[e] == least;
                const bool stays = x[e] > least || (same && before < wanted);
                before += same;
                listed[e] = j + e < of && stays == (j + e >= stay);
                n += listed[e];
            }
            block_sums(n, part, before, all);
            before += moves;
            moves += all;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (listed[e]) places[before++] = j + e;
        }
        moves /= 2;
    }
    __syncthreads();

    // ---- rows from `from` to `to`, both of this sequence and head
    // a piece of `bytes` of a row: 16 codes' bytes, all scales, or the weight
    const int kp = plan.kb / 16, vp = plan.vb / 16, pieces = kp + vp + 1;
    struct Piece {
        u32x4 w;
        uint64_t k_scale, v_scale;
        float weight;
    };
    auto load = [&](Piece& x, int64_t r, int piece) __attribute__((always_inline)) {
        if (piece < kp) x.w = r < 0 ? u32x4{0, 0, 0, 0} : *(const u32x4*)(kc + r * plan.kb + 16 * piece);
        else if (piece < kp + vp) x.w = r < 0 ? u32x4{0, 0, 0, 0} : *(const u32x4*)(vc + r * plan.vb + 16 * (piece - kp));
        else {
            x.k_scale = x.v_scale = r < 0 ? ~0ull : 0ull;              // (a row of a page that is not there is NaN)
            for (int i = 0; r >= 0 && i < plan.ksb; ++i) x.k_scale |= (uint64_t)ks[r * plan.ksb + i] << (8 * i);
            for (int i = 0; r >= 0 && i < plan.vsb; ++i) x.v_scale |= (uint64_t)vs[r * plan.vsb + i] << (8 * i);
            x.weight = r < 0 ? 0.f : weights[r];
        }
    };
    auto store = [&](const Piece& x, int64_t r, int piece) __attribute__((always_inline)) {
        if (r < 0) return;
        if (piece < kp) *(u32x4*)(kc + r * plan.kb + 16 * piece) = x.w;
        else if (piece < kp + vp) *(u32x4*)(vc + r * plan.vb + 16 * (piece - kp)) = x.w;
        else {
            for (int i = 0; i < plan.ksb; ++i) ks[r * plan.ksb + i] = (uint8_t)(x.k_scale >> (8 * i));
            for (int i = 0; i < plan.vsb; ++i) vs[r * plan.vsb + i] = (uint8_t)(x.v_scale >> (8 * i));
            weights[r] = x.weight;
        }
    };
    // movers into holes: nothing that is written is read
    for (int64_t i = tid; i < (int64_t)moves * pieces; i += kThreads) {
        const int m = (int)(i / pieces), piece = (int)(i - (int64_t)m * pieces);
        Piece x;
        load(x, row_of(places[moves + m]), piece);
        store(x, row_of(places[m]), piece);
    }
    // the recent rows: what a turn writes may be what it and earlier ones have read, never what later ones will
    for (int64_t i0 = 0; i0 < (int64_t)recent * pieces; i0 += kThreads) {
        __syncthreads();
        const int64_t i = i0 + tid;
        const int m = (int)(i / pieces), piece = (int)(i - (int64_t)m * pieces);
        Piece x;
        if (m < recent) load(x, row_of(of + m), piece);
        __syncthreads();
        if (m < recent) store(x, row_of(stay + m), piece);
    }
}

}  // namespace

int launch_cache_evict(const CacheEvictArgs& a)
{
    const int most = a.table_width << a.c.page_shift;
    const EvictPlan plan{a.c.Hkv, a.c.page_shift, most, a.table_width, a.c.pages, a.recent, a.c.d_qk * a.c.bits / 8, a.c.d_v * a.c.bits / 8, a.c.d_qk / 32,
                         a.c.d_v / 32, evict_ints(most)};
    return launch_kernel(attn_cache_evict_kernel, dim3((unsigned)(a.B * a.c.Hkv)), dim3(kThreads), 0, a.stream, (uint8_t*)a.c.k, (uint8_t*)a.c.k_scale,
                         (uint8_t*)a.c.v, (uint8_t*)a.c.v_scale, a.weights, a.table, a.lens, a.keep, a.lens_out, plan, a.places) == hipSuccess ? 0 : -3;
}

}  // namespace attn
