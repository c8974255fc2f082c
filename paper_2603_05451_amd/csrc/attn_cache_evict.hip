// Eviction from the paged cache by accumulated weight (gfx950): attn_cache_evict of include/attn.h.
//
// A block has a (sequence, KV head).  With `left` = min(len, keep) rows to stay, `recent` of them the last ones, the others (`stay`) are the
// candidates j < of = len - recent with the greatest weights, ties to the lowest j.  The weights are taken as whole numbers of the same order
// (least_first), and the stay-th greatest is found digit by digit (11, 11 and 10 bits) with a histogram in LDS.  Survivors below `stay` remain
// where they are.  There are as many other rows below (holes) as survivors from there on (movers): both are listed, holes first, in ascending
// order, by sums over the block, and the i-th mover goes into the i-th hole.  At most len - left + recent rows are moved at all, where closing
// the cache up in order would move nearly all of them.  The recent rows then go to the places from `stay` on, in order.
//
// What bounds it (8 heads, d = 128, 4 bits; states that were not evicted before, their memory not in the caches): for some thousand rows and many heads (32
// sequences of 4352 rows to 4096: 21.5 us, 5.1 for the bytes) a chain of fixed parts, each a latency of LDS or memory, and in a block of 16 waves the vector
// instructions' turns; for one long sequence (30 001 rows to 4096: 71 us) the eight blocks that there are: 26 us of selection, as a pass over the same state
// takes that finds nearly all survivors in place, and the moves of 3500 rows of each head through one CU.
//
// The only atomics are counts of whole numbers: results do not depend on their order.
#include "common.h"
#include "launch.h"
#include "ops.h"
#include "wave_sums.h"

namespace attn {
namespace {

struct EvictPlan {
    int Hkv, page_shift, most, table_width, pages, recent, held;
    int64_t ints;
};

// (512 are slower where blocks are few, 32 sequences of 4352 rows 25 us and 21.5, one of 30 001 94 and 71, and no faster for few rows; 256 sequences of 2112 rows,
// whose blocks are two to a CU then, take 39.5 with them and 54 so)
constexpr int NT = 1024;
// of the histogram, a lane's the even or the odd one (30 001 rows whose survivors are in place, selection that is: 30.8 us with one, 29.8 with two, at that time; of
// 71 us with moves it makes nothing that can be measured; four do not fit beside the weights)
constexpr int kCopies = 2;
constexpr int kAtOnce = 4;          // 16-byte pieces of rows that a thread moves in a turn

// Weights in ascending order as whole numbers: 0 is a row that is not in the cache, NaN the greatest, -0 and 0 are equal.
__device__ __forceinline__ uint32_t least_first(float w)
{
    if (w != w) return 0xffffffffu;
    const uint32_t x = __float_as_uint(w + 0.0f);
    return x & 0x80000000u ? ~x : x | 0x80000000u;
}

// Exclusive sums over the block's threads, and the sum of all: to `before` and `all`.  `part`: an int of LDS per wave, of this call's own.
__device__ __forceinline__ void block_sums(int x, ATTN_LDS int* part, int& before, int& all)
{
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int upto = wave_prefix(x);
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    const int q = wave_prefix(lane < NT / 64 ? part[lane] : 0);
    before = upto - x + (wave ? __builtin_amdgcn_readlane(q, wave - 1) : 0);
    all = __builtin_amdgcn_readlane(q, 63);
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

// The loops are not unrolled: most of a small call's time is fetching code that it runs once (4352 rows, passes over the same states, where 10.3 us are left
// now: 12.9 us with the weights in registers and every loop over them unrolled, 11.1 us so).
template <int DQK, int DV, int BITS>
__global__ void __launch_bounds__(NT)
attn_cache_evict_kernel(uint8_t* __restrict__ kc, uint8_t* __restrict__ ks, uint8_t* __restrict__ vc, uint8_t* __restrict__ vs,
                        float* __restrict__ weights, const int* __restrict__ table, const int* __restrict__ lens, const int* __restrict__ keep,
                        int* __restrict__ lens_out, EvictPlan plan, int* __restrict__ places_of_all)
{
    constexpr int KROW = DQK * BITS / 8, VROW = DV * BITS / 8;
    // weights of up to plan.held keys as whole numbers, and later the list of places: an entry lies no further than its key's number
    extern __shared__ __attribute__((aligned(16))) uint32_t held_[];
    __shared__ __attribute__((aligned(16))) int count[2048][kCopies];
    __shared__ int part_[4][NT / 64];
    __shared__ int found[3];
    ATTN_LDS uint32_t* const held = (ATTN_LDS uint32_t*)held_;
    auto part = [&](int i) __attribute__((always_inline)) { return (ATTN_LDS int*)part_[i]; };
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
    typedef __attribute__((ext_vector_type(4))) uint32_t keys4;
    // four keys from j on, j a multiple of 4: they are in one page; those past the end are not to be counted
    auto keys_at = [&](int j) __attribute__((always_inline)) {
        const int64_t r = row_of(j);
        f32x4 w = {0.f, 0.f, 0.f, 0.f};
        if (r >= 0) w = *(const f32x4*)(weights + r);
        keys4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = r >= 0 ? least_first(w[e]) : 0u;
        return x;
    };
    const bool in_lds = of <= plan.held;
    auto keys = [&](int j) __attribute__((always_inline)) { return in_lds ? *(const ATTN_LDS keys4*)(held + j) : keys_at(j); };
    int* const places = places_of_all + (int64_t)blockIdx.x * plan.ints;

    int moves = 0;
    if (stay > 0) {
        if (in_lds)
#pragma unroll 4
            for (int j = 4 * tid; j < of; j += 4 * NT) *(ATTN_LDS keys4*)(held + j) = keys_at(j);

        // ---- the stay-th greatest: its digits from the highest on, as far as it takes
        uint32_t prefix = 0;                               // those found so far
        int wanted = stay, same = 0;                       // the greatest `wanted` of the keys that begin with them, which are `same`
        int low = 32;                                      // bits of a number behind them
#pragma unroll 1
        while (low > 0) {
            const int bits = min(low, 11);
            low -= bits;
            for (int i = tid; i < 2048; i += NT)
#pragma unroll
                for (int c = 0; c < kCopies; ++c) count[i][c] = 0;
            __syncthreads();
#pragma unroll 1
            for (int j = 4 * tid; j < of; j += 4 * NT) {
                const keys4 x = keys(j);
                int at[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t begins = x[e] >> low;
                    at[e] = j + e < of && begins >> bits == prefix ? (int)(begins & ((1u << bits) - 1)) : -1;
                }
                // (equal ones in one go: lanes that add to one place do so one after the other)
                int n = 1;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool more = e < 3 && at[e] == at[e < 3 ? e + 1 : 3];
                    if (!more && at[e] >= 0) atomicAdd(&count[at[e]][tid % kCopies], n);
                    n = more ? n + 1 : 1;
                }
            }
            __syncthreads();
            // a thread's share of the places, counted from the greatest
            constexpr int PER = 2048 / NT;
            int here[PER], sum = 0, before, all;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                here[i] = 0;
#pragma unroll
                for (int c = 0; c < kCopies; ++c) here[i] += count[2047 - PER * tid - i][c];
                sum += here[i];
            }
            block_sums(sum, part(0), before, all);
            if (before < wanted && wanted <= before + sum) {
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    if (before < wanted && wanted <= before + here[i]) {
                        found[0] = 2047 - PER * tid - i;
                        found[1] = wanted - before;
                        found[2] = here[i];
                    }
                    before += here[i];
                }
            }
            __syncthreads();
            prefix = prefix << bits | (uint32_t)found[0];
            wanted = found[1];
            same = found[2];
            if (same == wanted) break;                     // all that begin so survive
        }
        const uint32_t least = prefix;                     // what survivors begin with at least; `wanted` of those that begin so survive, the first ones

        // ---- holes and movers, in ascending order
        // (8 keys of a thread in a turn where 4 would take more than one.  4 and 8, first passes over states: one sequence of 8000 rows 29.2 us and 28.9, 8 of
        // 30 001 92.9 and 92.1, one of 120 001 247 and 244, 32 of 1088 13.3 and 14.1, 256 of 2112 54.8 and 58.9; later ones: 30 001 rows 44.1 and 42.3)
        auto list = [&](auto of_thread) __attribute__((always_inline)) {
            constexpr int KT = decltype(of_thread)::value;
            int equal = 0;
#pragma unroll 1
            for (int j0 = 0, turn = 0; j0 < of; j0 += KT * NT, ++turn) {
                const int j = j0 + KT * tid;
                uint32_t x[KT];
#pragma unroll
                for (int i = 0; i < KT; i += 4) {
                    keys4 y = {0, 0, 0, 0};
                    if (j + i < of) y = keys(j + i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[i + e] = y[e];
                }
                int before = 0, all;
                if (same != wanted) {                          // ties: the first ones survive
                    int n = 0;
#pragma unroll
                    for (int e = 0; e < KT; ++e) n += j + e < of && x[e] >> low == least;
                    block_sums(n, part(turn & 1 ? 2 : 0), before, all);
                    before += equal;
                    equal += all;
                }
                int set = 0;                                   // a bit for each key that is listed
#pragma unroll
                for (int e = 0; e < KT; ++e) {
                    const bool is = x[e] >> low == least;
                    const bool stays = x[e] >> low > least || (is && (same == wanted || before < wanted));
                    before += is;
                    if (j + e < of && stays == (j + e >= stay)) set |= 1 << e;
                }
                block_sums(__popc(set), part(turn & 1 ? 3 : 1), before, all);
                before += moves;
                moves += all;
#pragma unroll
                for (int e = 0; e < KT; ++e)
                    if (set >> e & 1) {
                        if (in_lds) held[before] = j + e;
                        else places[before] = j + e;
                        ++before;
                    }
            }
        };
        if (of > 4 * NT) list(std::integral_constant<int, 8>());
        else list(std::integral_constant<int, 4>());
        moves /= 2;
        __syncthreads();
    }

    // ---- movers into holes, then the recent rows.  A turn reads all it moves before it writes.  What it writes is read by no later turn: holes are
    // read by none, and a recent row's new place lies below those that later ones come from.
    auto place = [&](int n) __attribute__((always_inline)) { return in_lds ? (int)held[n] : places[n]; };
    auto from_row = [&](int m) __attribute__((always_inline)) { return row_of(m < moves ? place(moves + m) : of + m - moves); };
    auto to_row = [&](int m) __attribute__((always_inline)) { return row_of(m < moves ? place(m) : stay + m - moves); };
    // (a row of a page that is not there is NaN, its weight 0)
    const int rows = moves + recent;
#pragma unroll 1
    for (int m0 = 0; m0 < rows; m0 += NT) {
        const int m = m0 + tid;
        ScaleRow<DQK / 32> k_scale;
        ScaleRow<DV / 32> v_scale;
        float weight = 0.f;
        int64_t from = -1, to = -1;
        if (m < rows) { from = from_row(m); to = to_row(m); }
        if (from >= 0) {
            k_scale.load(ks, from);
            v_scale.load(vs, from);
            weight = weights[from];
        } else {
            k_scale.fill(255);
            v_scale.fill(255);
        }
        __syncthreads();
        if (to >= 0) {
            k_scale.store(ks, to);
            v_scale.store(vs, to);
            weights[to] = weight;
        }
    }
    constexpr int KP = KROW / 16, VP = VROW / 16, PIECES = KP + VP;                // 16 bytes of codes each
    const uint32_t items = (uint32_t)rows * PIECES;        // (2^26 * 32 at most)
#pragma unroll 1
    for (uint32_t i0 = 0; i0 < items; i0 += kAtOnce * NT) {
        // (first where all of them are, then what is there: loads return in their order)
        const uint8_t* from[kAtOnce];
        uint8_t* to[kAtOnce];
        u32x4 x[kAtOnce];
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) {
            const uint32_t i = i0 + NT * e + tid;
            from[e] = to[e] = nullptr;
            if (i >= items) continue;
            const int m = (int)(i / PIECES), piece = (int)(i % PIECES);
            const int64_t f = from_row(m), t = to_row(m);
            uint8_t* const base = piece < KP ? kc + 16 * piece : vc + 16 * (piece - KP);
            const int row = piece < KP ? KROW : VROW;
            if (f >= 0) from[e] = base + f * row;
            if (t >= 0) to[e] = base + t * row;
        }
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e) x[e] = from[e] ? *(const u32x4*)from[e] : u32x4{0, 0, 0, 0};
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kAtOnce; ++e)
            if (to[e]) *(u32x4*)to[e] = x[e];
    }
}

template <int DQK, int DV, int BITS>
static int cache_evict_b(const CacheEvictArgs& a)
{
    const int most = a.table_width << a.c.page_shift, held = ((most < kEvictHeld ? most : kEvictHeld) + 3) & ~3;
    const EvictPlan plan{a.c.Hkv, a.c.page_shift, most, a.table_width, a.c.pages, a.recent, held, evict_ints(most)};
    auto kern = attn_cache_evict_kernel<DQK, DV, BITS>;
    static LdsOptIn lds;
    if (!lds.allow(kern, 4 * kEvictHeld)) return -3;
    return launch_kernel(kern, dim3((unsigned)(a.B * a.c.Hkv)), dim3(NT), (size_t)(4 * held), a.stream, (uint8_t*)a.c.k, (uint8_t*)a.c.k_scale, (uint8_t*)a.c.v,
                         (uint8_t*)a.c.v_scale, a.weights, a.table, a.lens, a.keep, a.lens_out, plan, a.places) == hipSuccess ? 0 : -3;
}
template <int DQK, int DV>
static int cache_evict_d(const CacheEvictArgs& a) { return a.c.bits == 4 ? cache_evict_b<DQK, DV, 4>(a) : cache_evict_b<DQK, DV, 8>(a); }

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
