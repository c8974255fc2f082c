// The attention weight that cached keys had from a call's queries (gfx950): attn_cache_weigh of include/attn.h.  How: at the top of
// attn_cache_weigh_kernel.inc.
#include "cache_codes.h"
#include "common.h"
#include "launch.h"
#include "ops.h"
#include "wave_sums.h"

namespace attn {

struct WeighPlan {
    int B, Nq, T, G, Hkv, page_shift, most, table_width, pages;
    uint32_t per_g;             // 2^32 / G, rounded up, to divide by G
    int causal, fresh, split;   // split: weigh_shape's
    float scale_log2e;
    Stride3 sq;
    long long lse_batch, lse_head;
};
struct WeighSeq {
    int q0, nq, len;            // first row of q; queries; keys (0: there is nothing to do)
};
struct WeighPlace {
    WeighSeq s;
    int b, group, groups;       // sequence, and which group of its keys
    int group_keys;
    int share, shares, share_tiles;     // which share of its tiles of rows
};

__device__ __forceinline__ WeighSeq weigh_seq(const WeighPlan& p, const int* __restrict__ cu, const int* __restrict__ lens, int b)
{
    if (b >= p.B) return {0, 0, 0};
    const int q0 = cu ? cu[b] : b * p.Nq, q1 = cu ? cu[b + 1] : q0 + p.Nq;
    if (q0 < 0 || q1 <= q0 || q1 > p.T) return {0, 0, 0};
    return {q0, q1 - q0, min(max(lens[b], 0), p.most)};
}

// How the sequences' work is shared out, from boundaries and lengths, the same in every wave of a launch (and of the one that adds up).
template <int KEYS, int RT>
struct WeighWork {
    const WeighPlan& p;
    const int* __restrict__ cu;
    const int* __restrict__ lens;
    int few_steps, share_tiles;         // few rows: KEYS keys of a group; many: tiles of rows of a share
    WeighSeq held;                      // the lane's of the first 64 sequences

    __device__ __forceinline__ WeighSeq seq(int b0) const { return b0 == 0 ? held : weigh_seq(p, cu, lens, b0 + (threadIdx.x & 63)); }

    __device__ __forceinline__ bool few(const WeighSeq& s) const { return s.nq * p.G <= kWeighFew; }
    __device__ __forceinline__ int steps(const WeighSeq& s) const { return (s.len + KEYS - 1) / KEYS; }
    __device__ __forceinline__ int tiles(const WeighSeq& s) const { return (s.nq * p.G + RT - 1) / RT; }
    // Of few rows as many keys to a group as make a round of groups, of many rows as many tiles to a share, two at least (256 queries, G = 4, d = 128,
    // over 2000 keys: 15.0 us, 18.6 with four at least, and the same with one).  Tiles that the mask leaves nothing of count in full: 4000 queries over
    // 4000 keys take 128 us, 122 if a triangle counts half, but 1024 over 1024 19.9 and 23.4.
    __device__ __forceinline__ WeighWork(const WeighPlan& plan, const int* __restrict__ c, const int* __restrict__ l) : p(plan), cu(c), lens(l)
    {
        held = weigh_seq(p, cu, lens, threadIdx.x & 63);
        float of_few = 0.f, of_many = 0.f;
        for (int b0 = 0; b0 < p.B; b0 += 64) {
            const WeighSeq s = seq(b0);
            const float n = (float)steps(s);
            if (few(s)) of_few += n;
            else of_many += n * (float)tiles(s);
        }
        const float of_round = (float)p.Hkv * (1.0f / kWeighRound);
        few_steps = max(1, (int)ceilf(wave_sum(of_few) * of_round));
        share_tiles = p.split ? max(2, (int)ceilf(fminf(wave_sum(of_many) * of_round, 1e9f))) : 1 << 30;
    }
    __device__ __forceinline__ int groups(const WeighSeq& s) const { const int n = few(s) ? few_steps : 1; return (steps(s) + n - 1) / n; }
    __device__ __forceinline__ int shares(const WeighSeq& s) const { return few(s) ? 1 : max(1, (int)(((int64_t)tiles(s) + share_tiles / 2) / share_tiles)); }
    // Group (ALL: and share) number u of all sequences'; false behind the last one.  Part: where the sums of its sequence's (share, group)s begin, if there
    // are more shares than one.
    template <bool ALL>
    __device__ __forceinline__ bool find(int u, WeighPlace& at, int& part) const
    {
        part = 0;
        for (int b0 = 0; b0 < p.B; b0 += 64) {
            const WeighSeq s = seq(b0);
            const int g = groups(s), n = shares(s), mine = ALL ? g * n : g, upto = wave_prefix(mine);
            const int divided = n > 1 ? g * n : 0, parts = p.split ? wave_prefix(divided) : 0;
            const uint64_t past = __ballot(upto > u);
            if (past) {
                const int l = __builtin_ctzll(past);
                auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
                at.s = {of(s.q0), of(s.nq), of(s.len)};
                at.b = b0 + l;
                at.groups = of(g);
                at.shares = of(n);
                const int local = u - (of(upto) - of(mine));
                at.share = ALL ? local / at.groups : 0;
                at.group = ALL ? local - at.share * at.groups : local;
                at.group_keys = KEYS * ((of(steps(s)) + at.groups - 1) / at.groups);
                at.share_tiles = (of(tiles(s)) + at.shares - 1) / at.shares;
                part += of(parts) - of(divided);
                return true;
            }
            u -= __builtin_amdgcn_readlane(upto, 63);
            part += __builtin_amdgcn_readlane(parts, 63);
        }
        return false;
    }
};

__device__ __forceinline__ int divide(uint32_t x, uint32_t per_g, int G)       // x / G, for any x
{
    const uint32_t q = __umulhi(x, per_g);
    return G == 1 ? (int)x : (int)(q - (q * (uint32_t)G > x));
}

#define ATTN_ELEM bf16
#define ATTN_ELEM8 bf16x8
#define ATTN_ELEM4 bf16x4
#include "elem.inc"
#undef ATTN_ELEM
#undef ATTN_ELEM8
#undef ATTN_ELEM4
#include "attn_cache_weigh_kernel.inc"

namespace f16k {
#define ATTN_ELEM f16
#define ATTN_ELEM8 f16x8
#define ATTN_ELEM4 f16x4
#include "elem.inc"
#undef ATTN_ELEM
#undef ATTN_ELEM8
#undef ATTN_ELEM4
#include "attn_cache_weigh_kernel.inc"
}  // namespace f16k

int launch_cache_weigh(const CacheWeighArgs& a)
{
    if (a.c.bits == 4) return a.f16 ? f16k::cache_weigh<4>(a) : (cache_weigh<4>)(a);
    return a.f16 ? f16k::cache_weigh<8>(a) : (cache_weigh<8>)(a);
}

}  // namespace attn
