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
    int64_t ints;
};

constexpr int kThreads = 1024;
constexpr int kHeld = 8;            // turns of 4 keys to a thread whose weights stay in registers: 32 768 keys
constexpr int kListed = 8192;       // holes and movers that LDS has room for (else they go to the workspace)
constexpr int kAtOnce = 4;          // pieces of rows that a thread moves in a turn

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

// The scale bytes of a row: BYTES of them, in words as large as their alignment is for certain.
template <int BYTES>
struct ScaleRow {
    using Word = std::conditional_t<BYTES % 8 == 0, uint64_t, std::conditional_t<BYTES % 4 == 0, uint32_t, std::conditional_t<BYTES % 2 == 0, uint16_t, uint8_t>>>;
    static constexpr int N = BYTES / sizeof(Word);
    Word w[N];
    __device__ __forceinline__ void fill(uint8_t byte)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = (Word)(0x0101010101010101ull * byte);
    }
    __device__ __forceinline__ void load(const uint8_t* all, int64_t row)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = ((const Word*)all)[row * N + i];
    }
    __device__ __forceinline__ void store(uint8_t* all, int64_t row) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) ((Word*)all)[row * N + i] = w[i];
    }
};

template <int DQK, int DV, int BITS>
__global__ void __launch_bounds__(kThreads)
attn_cache_evict_kernel(uint8_t* __restrict__ kc, uint8_t* __restrict__ ks, uint8_t* __restrict__ vc, uint8_t* __restrict__ vs,
                        float* __restrict__ weights, const int* __restrict__ table, const int* __restrict__ lens, const int* __restrict__ keep,
                        int* __restrict__ lens_out, EvictPlan plan, int* __restrict__ places_of_all)
{
    constexpr int KROW = DQK * BITS / 8, VROW = DV * BITS / 8;
    __shared__ int count[2048];
    __shared__ int part_[32];
    __shared__ int found[2];
    __shared__ int list[kListed];
    ATTN_LDS int* const part = (ATTN_LDS int*)part_;
    const int tid = threadIdx.x;
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
    const bool in_lds = 2 * min(stay, len - left) <= kListed;          // (there are no more holes than rows that leave, nor than that stay)

    int moves = 0;
    if (stay > 0) {
        uint32_t held[kHeld][4];
#pragma unroll
        for (int i = 0; i < kHeld; ++i)
            if (4 * kThreads * i < of) keys_at(min(4 * (kThreads * i + tid), of - 1) & ~3, held[i]);
        // f(first of 4 keys, their numbers) for every turn of the block
        auto each = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if (4 * kThreads * i < of) f(4 * (kThreads * i + tid), held[i]);
#pragma unroll 1
            for (int j0 = 4 * kThreads * kHeld; j0 < of; j0 += 4 * kThreads) {
                const int j = j0 + 4 * tid;
                uint32_t x[4] = {0, 0, 0, 0};
                if (j < of) keys_at(j, x);
                f(j, x);
            }
        };

        // ---- the stay-th greatest: its digits from the highest on
        uint32_t prefix = 0;                               // those found so far
        int wanted = stay;                                 // the greatest `wanted` of the keys that begin with them
#pragma unroll
        for (int digit = 0; digit < 3; ++digit) {
            constexpr int low_of[] = {21, 10, 0};
            const int low = low_of[digit], bits = digit == 2 ? 10 : 11;
            count[tid] = count[tid + kThreads] = 0;
            __syncthreads();
            each([&](int j, const uint32_t (&x)[4]) __attribute__((always_inline)) {
                int at[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) at[e] = j + e < of && (digit == 0 || x[e] >> (low + bits) == prefix) ? (int)((x[e] >> low) & ((1u << bits) - 1)) : -1;
                // (equal ones in one go: lanes that add to one place do so one after the other)
                int n = 1;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool more = e < 3 && at[e] == at[e < 3 ? e + 1 : 3];
                    if (!more && at[e] >= 0) atomicAdd(&count[at[e]], n);
                    n = more ? n + 1 : 1;
                }
            });
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
        }
        const uint32_t least = prefix;                     // of the survivors; `wanted` of those that are equal to it survive, the first ones

        // ---- holes and movers, in ascending order
        int equal = 0;
        each([&](int j, const uint32_t (&x)[4]) __attribute__((always_inline)) {
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
                if (listed[e]) {
                    if (in_lds) list[before] = j + e;
                    else places[before] = j + e;
                    ++before;
                }
        });
        moves /= 2;
        __syncthreads();
    }

    // ---- movers into holes, then the recent rows.  A turn reads all it moves before it writes.  What it writes is read by no later turn: holes are
    // read by none, and a recent row's new place lies below those that later ones come from.
    constexpr int KP = KROW / 16, VP = VROW / 16, PIECES = KP + VP + 1;            // of a row: 16 bytes of codes, and all scales and the weight
    struct Piece {
        union {
            u32x4 w;
            struct {
                ScaleRow<DQK / 32> k_scale;
                ScaleRow<DV / 32> v_scale;
                float weight;
            } s;
        };
        __device__ Piece() {}
    };
    const uint32_t items = (uint32_t)(moves + recent) * PIECES;        // (2^26 * 33 at most)
    for (uint32_t i0 = 0; i0 < items; i0 += kAtOnce * kThreads) {
        Piece x[kAtOnce];
        int64_t to[kAtOnce];
        int piece[kAtOnce];
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) {
            const uint32_t i = i0 + kThreads * e + tid;
            to[e] = -1;
            if (i >= items) continue;
            const int m = (int)(i / PIECES);
            piece[e] = (int)(i % PIECES);
            auto place = [&](int n) __attribute__((always_inline)) { return in_lds ? list[n] : places[n]; };
            const int64_t r = row_of(m < moves ? place(moves + m) : of + m - moves);
            to[e] = row_of(m < moves ? place(m) : stay + m - moves);
            // (a row of a page that is not there is NaN, its weight 0)
            if (piece[e] < KP) x[e].w = r < 0 ? u32x4{0, 0, 0, 0} : *(const u32x4*)(kc + r * KROW + 16 * piece[e]);
            else if (piece[e] < KP + VP) x[e].w = r < 0 ? u32x4{0, 0, 0, 0} : *(const u32x4*)(vc + r * VROW + 16 * (piece[e] - KP));
            else if (r < 0) {
                x[e].s.k_scale.fill(255);
                x[e].s.v_scale.fill(255);
                x[e].s.weight = 0.f;
            } else {
                x[e].s.k_scale.load(ks, r);
                x[e].s.v_scale.load(vs, r);
                x[e].s.weight = weights[r];
            }
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) {
            const int64_t r = to[e];
            if (r < 0) continue;
            if (piece[e] < KP) *(u32x4*)(kc + r * KROW + 16 * piece[e]) = x[e].w;
            else if (piece[e] < KP + VP) *(u32x4*)(vc + r * VROW + 16 * (piece[e] - KP)) = x[e].w;
            else {
                x[e].s.k_scale.store(ks, r);
                x[e].s.v_scale.store(vs, r);
                weights[r] = x[e].s.weight;
            }
        }
        __syncthreads();
    }
}

template <int DQK, int DV>
static int cache_evict_d(const CacheEvictArgs& a)
{
    const int most = a.table_width << a.c.page_shift;
    const EvictPlan plan{a.c.Hkv, a.c.page_shift, most, a.table_width, a.c.pages, a.recent, evict_ints(most)};
    auto run = [&](auto kern) {
        return launch_kernel(kern, dim3((unsigned)(a.B * a.c.Hkv)), dim3(kThreads), 0, a.stream, (uint8_t*)a.c.k, (uint8_t*)a.c.k_scale, (uint8_t*)a.c.v,
                             (uint8_t*)a.c.v_scale, a.weights, a.table, a.lens, a.keep, a.lens_out, plan, a.places) == hipSuccess ? 0 : -3;
    };
    return a.c.bits == 4 ? run(attn_cache_evict_kernel<DQK, DV, 4>) : run(attn_cache_evict_kernel<DQK, DV, 8>);
}

}  // namespace

int launch_cache_evict(const CacheEvictArgs& a)
{
    if (a.c.d_qk == 64 && a.c.d_v == 64) return cache_evict_d<64, 64>(a);
    if (a.c.d_qk == 96 && a.c.d_v == 96) return cache_evict_d<96, 96>(a);
    if (a.c.d_qk == 128 && a.c.d_v == 128) return cache_evict_d<128, 128>(a);
    if (a.c.d_qk == 192 && a.c.d_v == 128) return cache_evict_d<192, 128>(a);
    if (a.c.d_qk == 256 && a.c.d_v == 256) return cache_evict_d<256, 256>(a);
    return -2;
}

}  // namespace attn
