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
    int causal, fresh;
    float scale_log2e;
    Stride3 sq;
    long long lse_batch, lse_head;
};
struct WeighSeq {
    int q0, nq, len;            // first row of q; queries; keys (0: there is nothing to do)
};
struct WeighPlace {
    WeighSeq s;
    int b, group;               // sequence, and which group of its keys
    int group_keys;
};

__device__ __forceinline__ WeighSeq weigh_seq(const WeighPlan& p, const int* __restrict__ cu, const int* __restrict__ lens, int b)
{
    if (b >= p.B) return {0, 0, 0};
    const int q0 = cu ? cu[b] : b * p.Nq, q1 = cu ? cu[b + 1] : q0 + p.Nq;
    if (q0 < 0 || q1 <= q0 || q1 > p.T) return {0, 0, 0};
    return {q0, q1 - q0, min(max(lens[b], 0), p.most)};
}
// Steps of KEYS keys in a group: one of many rows; of few rows as many as make about a round of groups of all such sequences.
template <int KEYS>
__device__ __forceinline__ int weigh_few_steps(const WeighPlan& p, const int* __restrict__ cu, const int* __restrict__ lens)
{
    float total = 0.f;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const WeighSeq s = weigh_seq(p, cu, lens, b0 + (threadIdx.x & 63));
        total += s.nq * p.G <= kWeighFew ? (float)((s.len + KEYS - 1) / KEYS) : 0.f;
    }
    return max(1, (int)ceilf(wave_sum(total) * (float)p.Hkv * (1.0f / kWeighRound)));
}
// Group `u` of all sequences' keys; false behind the last one.
template <int KEYS>
__device__ __forceinline__ bool weigh_find(const WeighPlan& p, const int* __restrict__ cu, const int* __restrict__ lens, int few_steps, int u, WeighPlace& at)
{
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const WeighSeq s = weigh_seq(p, cu, lens, b0 + (threadIdx.x & 63));
        const int n = s.nq * p.G <= kWeighFew ? few_steps : 1, steps = (s.len + KEYS - 1) / KEYS, mine = (steps + n - 1) / n, upto = wave_prefix(mine);
        const uint64_t past = __ballot(upto > u);
        if (past) {
            const int l = __builtin_ctzll(past);
            auto of = [&](int x) { return __builtin_amdgcn_readlane(x, l); };
            at.s = {of(s.q0), of(s.nq), of(s.len)};
            at.b = b0 + l;
            at.group = u - (of(upto) - of(mine));
            at.group_keys = KEYS * of((steps + max(mine, 1) - 1) / max(mine, 1));
            return true;
        }
        u -= __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

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
