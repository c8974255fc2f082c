// Host-side argument bundles of the rotary and cache calls, as launch.h has them for the attention calls, and the rules that
// share their work out (arithmetic on sizes alone, without HIP for a host compiler).
#pragma once
#include <stdint.h>

namespace attn {

// ---- rotary positions and head norms

// Lanes of a wave that hold one row: two chunks of 8 dims each, a power of two.
inline int rope_lanes(int d) { return d <= 64 ? 4 : d <= 128 ? 8 : 16; }

// Blocks of one launch at most, for a quarter of the 2^32 threads that it may have (the rotary calls have one for q and one for k).
constexpr int kMostBlocks = 1 << 22;

// Rows of a lane whose loads are in flight together.
constexpr int rope_rows(bool backward) { return backward ? 2 : 4; }

struct RopeShape {
    int blocks;         // of four waves
    int hg_shift;       // heads of a token side by side in a wave: 2^hg_shift
    int shares;         // blocks that divide the heads of a group of tokens
    int rows;           // rows of a lane in one turn
};
// How the rows of one tensor are shared out.  A lane goes through as many heads of its token as there are waves to spare for, for that
// many rows share their angles; but side by side in a wave are as many heads as make a KiB in a row (16384 tokens of 32 and 8 heads, d = 128:
// 77 us with every row slot at a token of its own, 71, 64 and 64 with 2, 4 and 8 heads a token), or half of that where it divides the
// heads and leaves no lane idle (32000 tokens of 12 + 12 heads, d = 64, norms: 48.3 us with 8 heads, 43.6 with 4).
inline RopeShape rope_shape(int tokens, int heads, int d, bool backward)
{
    const int slots = 64 / rope_lanes(d);
    RopeShape r{0, 0, 1, rope_rows(backward)};
    auto waves = [&] { return ((int64_t)tokens * (1 << r.hg_shift) + slots - 1) / slots; };
    while ((waves() < 1024 || (d << r.hg_shift) < 512) && (1 << r.hg_shift) < slots && (1 << r.hg_shift) < heads) ++r.hg_shift;
    const int part = heads & ((1 << r.hg_shift) - 1);
    if (part && part == 1 << r.hg_shift >> 1 && (d << r.hg_shift) >= 512 && waves() >= 2048) --r.hg_shift;
    // few tokens: a row per lane, its time is one row's (32 tokens, 32 + 8 heads, norms: 5.1 us with four rows, 4.1 so;
    // 256 tokens 5.4 and 4.8, 1024 6.9 and 8.0)
    const int singles = (heads + (1 << r.hg_shift) - 1) >> r.hg_shift;
    if (waves() * singles <= 1024) { r.rows = 1; r.shares = singles; }
    else if (waves() < 1024) r.shares = (singles + r.rows - 1) / r.rows;
    int64_t groups = (waves() + 3) / 4;
    if (r.shares > kMostBlocks) r.shares = kMostBlocks;
    if (groups * r.shares > kMostBlocks) groups = kMostBlocks / r.shares;
    if (backward && groups * r.shares > 512) groups = (512 + r.shares - 1) / r.shares;      // partial sums per block
    r.blocks = (int)(groups * r.shares);
    return r;
}
// q and k (heads_k = 0: there is none)
inline void rope_shapes(int tokens, int heads_q, int heads_k, int d, bool backward, RopeShape (&shape)[2])
{
    shape[0] = rope_shape(tokens, heads_q, d, backward);
    shape[1] = heads_k > 0 ? rope_shape(tokens, heads_k, d, backward) : RopeShape{0, 0, 1, 1};
}

// ---- attention over the cache

// Blocks of 16 rows that a wave takes together: two where there are more than 16 rows (queries times heads of a group), which read and
// convert the cache once and not twice (32 sequences of 4001 keys, 5 queries, H = 32/8, d = 128: 54.7 us with one, 40.9 with two).
inline int cache_row_blocks(int Nq, int H, int Hkv) { return (int64_t)Nq * (H / Hkv) > 16 ? 2 : 1; }

// Blocks of the attention kernel that a CU holds, which it is compiled for: what its registers allow without spilling more than a few.
// 32 sequences of 8000 keys, H = 32/8, us with one block fewer (where it is not one) / so / one more, with one and with two row blocks:
//   d = 64          4 bits 42 / 39 / 40, 58 / 53 / 51       8 bits 56 / 56 / 76, 66 / 62 / 93
//   d = 96                 66 / 56 / 77, 122 / 77 / 132            111 / 81 / 87, 128 / 89 / 257
//   d = 128                65 / 61 / 76, 113 / 81 / 197            138 / 102 / 132, 161 / 112 / 342
//   d = (192, 128)         112 / 75 / 75, 126 / 92 / 357           130 / 129 / 250, - / 162 / 216
//   d = 256                136 / 111 / 584, - / 188 / 632          - / 205 / 496, - / 231 / 1044
constexpr int cache_blocks_per_cu(int d_qk, int bits, int row_blocks)
{
    const bool lean = bits == 4 && row_blocks == 1;
    if (d_qk > 192) return lean ? 2 : 1;
    if (d_qk > 128) return bits == 8 && row_blocks == 2 ? 1 : 2;
    if (d_qk > 64) return lean ? 3 : 2;
    return row_blocks == 1 ? 4 : 3;
}

struct CacheShape {
    int waves;          // that share a chunk: the four of a block, or one
    int parts;          // chunks that the keys of all sequences are divided into, about: what one round of blocks takes
    int min_tiles;      // a chunk has at least so many 32-key tiles
    int slots;          // chunks at most: `parts` of three quarters of that length and one per sequence, or what the longest could have
};
// Where there are more (sequence, KV head, row group)s than the chip holds blocks, each is a wave's work: a block per one of them would take
// several rounds, whose first loads and merges all blocks go through at the same time (4 bits, 8 KV heads, one row block, us as blocks / as
// waves: d = 128 300 sequences of 500 keys 53.6 / 42.6, 192 of 1000 51.1 / 47.9, 128 of 2000 68.4 / 59.0; d = 96 100 of 1000 33.2 / 31.3; d = 256
// 200 of 500 70.3 / 58.9; 8 bits: d = 128 100 of 2000 97 / 90, d = 96 100 of 1000 46 / 41; below one round 32 of 4001 30.7 / 33.9).  The line
// could lie higher: units for just one round are the faster as blocks (d = 128 96 of 4001 83.7 / 84.4, 8 bits 64 of 4001 98.6 / 101.7; d = 64
// 128 of 2000 36.4 / 38; d = 192 64 of 2000 43.5 / 45.5), and with two row blocks those for 1.5 as well (32 sequences, 64 rows, 300 keys 15.1 / 22.2,
// 1000 26.5 / 33.7, 8000 134 / 140; 128 rows 236 / 242, 8 bits 317 / 315; 96 of 2000, 32 rows 74 / 83).
// A chunk has 8 tiles or more, two per wave (one sequence of 1000 keys 6.7 us with 8, 5.7 with 4, 8.4 with 16; of 8000 7.2, 7.6 and 8.8), but
// sequences that are short by the table's width are not divided: the merge, 3 us and a launch, costs more (with it / undivided, 16
// sequences of 500 keys 10.6 / 8.6, 760 12.8 / 11.3, 1020 13.3 / 13.5; d = 256: 500 14.5 / 13.1, 760 18.0 / 17.2, 1020 18.9 / 21.4).
inline CacheShape cache_shape(int B, int Nq, int H, int Hkv, int d_qk, int bits, int64_t most)
{
    const int rb = cache_row_blocks(Nq, H, Hkv);
    const int64_t rows = (int64_t)Nq * (H / Hkv);
    const int64_t side = Hkv * ((rows + 16 * rb - 1) / (16 * rb)), round = 256 * cache_blocks_per_cu(d_qk, bits, rb);
    const int64_t tiles = (most + 31) / 32;
    const int undivided = d_qk * bits <= 512 ? 24 : 16;
    CacheShape s;
    s.waves = B * side >= round ? 1 : 4;
    const int64_t places = round * (4 / s.waves);
    s.parts = (int)(side < places ? places / side : 1);
    s.min_tiles = tiles <= undivided ? undivided : 8;
    const int64_t each = (tiles + s.min_tiles - 1) / s.min_tiles, most_parts = ((int64_t)s.parts * 4 + 2) / 3 + B;
    s.slots = (int)(B * each < most_parts ? B * each : most_parts);
    return s;
}

// Rows (query, head) that a block of the merge takes: one per d_v / 4 of its threads where a sequence has few chunks, as far as sizes
// tell, one otherwise (48 sequences of 67 ... 7696 keys, H = 32, d = 128: 6.6 us with 1536 blocks of a row each, 5.7 with 192 of 8; 16 of 2000,
// d = 64, 64 rows: 6.2 and 4.7; with dozens of parts to a row these are dealt to the block's 8 groups of threads).
inline int cache_merge_rows(const CacheShape& s, int B, int d_v, int64_t most)
{
    const int64_t each = (most + 32 * s.min_tiles - 1) / (32 * s.min_tiles), likely = 2 * (s.parts / B) + 1;
    return (each < likely ? each : likely) <= 16 ? 1024 / d_v : 1;
}

// Blocks of the attention kernel, and of the merge.
inline int64_t cache_fwd_blocks(const CacheShape& s, int Nq, int H, int Hkv)
{
    const int rows = 16 * cache_row_blocks(Nq, H, Hkv);
    const int64_t units = (int64_t)s.slots * Hkv * (((int64_t)Nq * (H / Hkv) + rows - 1) / rows);
    return s.waves == 4 ? units : (units + 3) / 4;
}
inline int64_t cache_merge_blocks(const CacheShape& s, int B, int Nq, int H, int d_v, int64_t most)
{
    const int per = cache_merge_rows(s, B, d_v, most);
    return B * (((int64_t)Nq * H + per - 1) / per);
}

// ---- attention of chunks over the cache

constexpr int kChunkRows = 128;         // rows (query, head of a KV head's group) of a block: 32 per wave
// A step of the body for few rows (128 keys), in quarters of a step of the other (26 sequences, 22 of them with one query, 100 ... 4096 keys,
// G = 4, d = 128, 4 bits: 41.0, 36.3, 36.9 us with 2, 3, 4).
constexpr int kChunkFewCost = 3;
// So many parts of 128 rows cost what one step of the other does: each is 136 KB to memory and back (4 x 100 queries, 1000 keys, 8 heads:
// 35.3 us with as many parts as there are places for, 28.9 so; 8 x 100: 42.0 and 33.8; 4 x 100, 2000 keys: 40.8 and 43.4).
constexpr float kChunkPartCost = 53;

// Keys of a tile, and blocks that a CU holds: a tile of K and V in 16 bits, twice, is 64 KiB at d = 128 and at d = 256.
constexpr int chunk_tile_keys(int d_qk) { return d_qk <= 128 ? 64 : 32; }
constexpr int chunk_blocks_per_cu(int d_qk) { return d_qk <= 192 ? 2 : 1; }

struct ChunkShape {
    int few;            // a sequence with no more rows goes by the body for few: 32 rows of a block, whose waves share the keys
    int places;         // blocks of one round if the keys of a row tile may be divided over several, else 0
    int64_t units;      // blocks per KV head at most: (row tile, part)s
    int64_t part_tiles; // room for results of parts, per KV head: 32 rows (a part of a row tile of many rows has four)
};
inline int chunk_places(int places, int Hkv) { return places ? places / Hkv + 1 : 0; }        // per KV head
// Times below in us, G = 4, 8 KV heads, d = 128, 4 bits.
// Few rows: shared keys are unpacked once per 32 rows rather than 128, but four waves have them each to itself.  Up to 64 rows (batch of 32,
// 2000 keys: 48 rows 43.8 by the body for many, 36.0 by that for few; 64 rows 45.9, 37.2); up to 128 where row tiles leave most CUs idle (one
// sequence of 4000 keys: 96 rows 21.2, 16.6; 128 rows 22.3, 17.7) but not in batches (32 of 2000 keys: 96 rows 53.3, 57.4; 128 rows 61.8, 66.3).
// Keys are divided, which costs a merge, if the blocks that there are for sure without (T queries in full row tiles) do not fill a round
// and the table is wide.  Undivided and divided: few rows, 8 sequences of 700 keys 10.0, 10.6; of 1000 12.1, 11.5; of 1400 17.4, 13.5; 32 of
// 1400 keys 18.5, 19.6; of 2000 24.7, 23.0.  Many, 64 queries over 400 keys 17.2, 17.3; over 700 21.4, 19.2; 4 x 100 queries over 700 23.6,
// 27.0; over 1000 28.8, 28.9; over 2000 more than 50, 43.4.
inline ChunkShape chunk_shape(int B, int T, int H, int Hkv, int d_qk, int64_t most)
{
    const int64_t G = H / Hkv, round = 256 * chunk_blocks_per_cu(d_qk);
    const int64_t full = T * G / kChunkRows, seqs = B < T ? B : T;
    const bool idle = full * Hkv <= 64;
    ChunkShape s{idle ? 128 : 64, 0, idle ? T * G / 32 + seqs : full + 2 * seqs, 0};
    const int64_t wide = T * G > (int64_t)s.few * B ? (idle ? 512 : 960) : ((int64_t)B * Hkv < 128 ? 960 : 1536);
    if (full * Hkv < round && most > wide) {
        s.places = (int)round;
        s.units += round / Hkv + 3;
        // Only what is divided has results of parts.  n parts of 2 and more, rounded up from x > 1, are fewer than 2 x, and all x are the places.
        const int64_t divided = 2 * chunk_places(s.places, Hkv);
        s.part_tiles = (s.units < divided ? s.units : divided) * (T * G > s.few ? kChunkRows / 32 : 1);
    }
    return s;
}

// ---- weights of cached keys

// A sequence with no more rows goes by the body for few, which has all of them in registers (32 sequences of 4000 keys, G = 4, 8 KV heads, d = 128, 4 bits:
// one query 39.7 us by the body for many, 23.1 by that for few; 8 queries 45.1 and 24.2; one sequence with 8, 6.4 and 6.7).
constexpr int kWeighFew = 32;
constexpr int weigh_key_blocks(int d_qk) { return d_qk <= 128 ? 2 : 1; }        // of 32 keys that a wave takes together
constexpr int weigh_keys(int d_qk) { return 4 * 32 * weigh_key_blocks(d_qk); }  // of a block (of few rows: in one step)
// Rows of a tile of queries: 16 KiB of LDS at d = 64 and 128, twice (1024 queries over 16 001 keys: d = 64 108 us with 64 rows, 104 with 128; d = 256 351
// with 32 rows, 325 with 64).
constexpr int weigh_rows(int d_qk) { return d_qk <= 64 ? 128 : 64; }
constexpr int kWeighRound = 2 * 256;    // blocks that the chip holds

struct WeighShape {
    bool split;         // the rows of a sequence may be divided over several blocks, whose sums are added by a second kernel
    int64_t groups;     // of keys, at most
    int64_t units;      // blocks' work: (group, share of the rows)s, at most
    int64_t parts;      // those of sequences whose rows are divided, whose sums go by the workspace, at most
};
// Rows are divided where a call has 256 and more, unless every sequence has few (Nq: queries that one may have), as the sum's launch is 3 us then
// (32 x 4 queries over 4000 keys: 26.4 us with it, 23.6 without; 33 over 2000, 132 rows: 12.5, 11.1; 64 over 400 ... 2000: 12.3, 13.8; 128 over 2000: 13.2,
// 23.1; 512 over 2000: 19.6, 58.8).
inline WeighShape weigh_shape(int B, int64_t T, int64_t Nq, int H, int Hkv, int d_qk, int64_t most)
{
    WeighShape s;
    s.split = T * (H / Hkv) >= 256 && Nq * (H / Hkv) > kWeighFew;
    s.groups = (int64_t)B * Hkv * ((most + weigh_keys(d_qk) - 1) / weigh_keys(d_qk));
    // (shares are made for a round of units; rounding may make them one and a half)
    s.units = s.groups + (s.split ? 2 * (kWeighRound + Hkv) : 0);
    // (n of 2 and more that were rounded from x are 4/3 x at most, and all x are a round: 683)
    s.parts = !s.split ? 0 : s.units < kWeighRound * 3 / 2 ? s.units : kWeighRound * 3 / 2;
    return s;
}
inline int weigh_blocks(int64_t units) { return (int)(units < 2 * kWeighRound ? units : 2 * kWeighRound); }

// ---- eviction

constexpr int kEvictHeld = 32768;       // keys whose weights, and lists of places, a block has in LDS: 128 KiB
inline int64_t evict_ints(int64_t most) { return (most + 3) / 4 * 4; }     // of a (sequence, KV head)'s list of places
// Lists of wider tables go by the workspace.  Where no sequence can have one there it is not touched, and is what the lists would take only as long as that is little.
inline int64_t evict_bytes(int64_t heads, int64_t most)
{
    const int64_t lists = heads * evict_ints(most) * 4;
    return most <= kEvictHeld && lists > 65536 ? 65536 : lists;
}

}  // namespace attn

#if defined(__HIP__)
#include "launch.h"

namespace attn {

struct RopeArgs {
    const void* x[2];           // q, k (null where there is none, heads 0)
    const void* dy[2];          // backward pass: gradients of the outputs
    void* y[2];                 // outputs; backward pass: gradients of x
    Stride3 sx[2], sdy[2], sy[2];
    const void* w[2];           // weights of the norms, or null: ones
    float* dw[2];               // their gradients, or null
    float* part;                // partial sums of those: [blocks of q, then of k][d]
    int heads[2];
    const float* freqs;
    const int* positions;       // or null: 0, 1, ... in every sequence
    long long positions_batch;
    int B, N, d, rot, offset;
    float amplitude, sign, eps;
    bool interleaved, norm, backward, f16;
    void* stream;
    RopeShape shape[2];         // (launch_rope sets them)
};
int launch_rope(RopeArgs a);

// ---- the quantised cache

struct CacheArgs {
    void *k, *k_scale, *v, *v_scale;
    int pages, page_shift, Hkv, d_qk, d_v, bits;
};

struct CacheRowsArgs {          // writing (rows in x) and reading (rows in y, dense)
    CacheArgs c;
    const void *xk, *xv;
    long long k_row, k_head, v_row, v_head;
    void *yk, *yv;
    const int* slots;
    int T;
    bool f16;
    void* stream;
};
int launch_cache_write(const CacheRowsArgs& a);
int launch_cache_read(const CacheRowsArgs& a);

struct CacheFwdArgs {
    CacheArgs c;
    const void* q;
    void* o;
    float* lse;
    Stride3 sq, so;
    const int *table, *lens;
    int table_width;
    int B, Nq, H;
    float scale;
    int causal;
    float *part_o, *part_ml;    // unnormalised results of chunks: [slots][Hkv][Nq * H / Hkv][d_v], and {maximum, sum} of each row
    int* merge;                 // [B][4]: where a sequence's parts are
    bool f16;
    void* stream;
};
int launch_cache_fwd_bf16(const CacheFwdArgs& a);       // one object each
int launch_cache_fwd_f16(const CacheFwdArgs& a);
inline int launch_cache_fwd(const CacheFwdArgs& a) { return a.f16 ? launch_cache_fwd_f16(a) : launch_cache_fwd_bf16(a); }

struct CacheWeighArgs {
    CacheArgs c;
    const void* q;
    const float* lse;
    float* weights;
    Stride3 sq;
    long long lse_batch, lse_head;
    const int *table, *lens, *cu;       // cu null: sequence b has the queries b * Nq ... b * Nq + Nq - 1
    int table_width;
    int B, Nq, T, H;                    // T: rows of q in all
    float scale;
    int causal, fresh;
    float* parts;               // sums of shares of the rows: [weigh_shape's parts][weigh_keys]
    bool f16;
    void* stream;
};
int launch_cache_weigh(const CacheWeighArgs& a);

struct CacheEvictArgs {
    CacheArgs c;
    float* weights;
    const int *table, *lens, *keep;
    int* lens_out;
    int table_width, B, recent;
    int* places;                // [B][Hkv][evict_ints(most)], used where most is beyond kEvictHeld
    void* stream;
};
int launch_cache_evict(const CacheEvictArgs& a);

struct CacheChunkArgs {
    CacheArgs c;
    const void* q;              // packed [T, H, d_qk]
    void* o;
    float* lse;                 // [H, T]
    long long q_row, q_head, o_row, o_head;
    const int *table, *cu, *lens;
    int table_width;
    int B, T, H;
    float scale;
    int causal;
    float *part_o, *part_ml;    // unnormalised results of parts: [part_tiles * Hkv][32][d_v], and {maximum, sum} of each row
    int* merge;                 // [B][4]: where a sequence's parts are
    bool f16;
    void* stream;
};
int launch_cache_chunk_bf16(const CacheChunkArgs& a);     // one object each
int launch_cache_chunk_f16(const CacheChunkArgs& a);
inline int launch_cache_chunk(const CacheChunkArgs& a) { return a.f16 ? launch_cache_chunk_f16(a) : launch_cache_chunk_bf16(a); }

}  // namespace attn
#endif
