/*
 * C ABI of the MI355X (gfx950) fused attention library: exact scaled-dot-product
 * attention, forward and backward, bf16 storage, fp32 accumulation.
 *
 * What is computed (paper Sec. 2.1):
 *   forward   S = scale * Q K^T (+ causal mask), P = softmax_rows(S), O = P V,
 *             LSE_i = ln sum_j exp(S_ij)   (natural log, of the scaled, masked scores)
 *   backward  dV = P^T dO, dP = dO V^T, dS = P o (dP - D), D_i = sum_c dO_ic O_ic,
 *             dQ = scale * dS K, dK = scale * dS^T Q
 * The N x N matrices S, P, dP, dS never reach device memory; the forward pass keeps
 * tiled online-softmax statistics with thresholded rescaling (paper Sec. 3.1.4) and the
 * backward pass recomputes P from Q, K and LSE (paper Sec. 3.2).
 *
 * Conventions shared by every entry point
 *   - Every pointer is a DEVICE pointer owned by the caller.  The library never
 *     allocates, frees or keeps it.  `stream` is a hipStream_t passed as void*
 *     (NULL = the default stream).  Calls only enqueue work on `stream` and return.
 *   - Layouts are contiguous row-major ("token-major"):
 *       q, o, d_o, dq : [B, N, H,   d]   bf16      (d = d_qk for q/dq, d_v for o/d_o)
 *       k, dk         : [B, N, Hkv, d_qk] bf16
 *       v, dv         : [B, N, Hkv, d_v]  bf16
 *       lse           : [B, H, N]         fp32
 *     bf16 = upper 16 bits of an IEEE fp32; outputs are rounded to nearest even.
 *     All pointers must be 16-byte aligned.
 *   - Grouped-query attention: H % Hkv == 0; query head h reads KV head h / (H / Hkv);
 *     dk and dv are summed over the query heads of each group.
 *   - causal != 0: key j is visible to query i iff j <= i.
 *   - Supported shapes: (d_qk, d_v) in {(64,64), (96,96), (128,128), (192,128), (256,256)}; N a positive
 *     multiple of 128 (the attn_varlen_* entry points take any lengths).
 *   - Return value: ATTN_OK, or a negative code.  ATTN_EINVAL, ATTN_EUNSUPPORTED and
 *     ATTN_ETOOLARGE are found before anything is enqueued: no output has been touched.
 *     ATTN_ELAUNCH (the HIP runtime refused a launch or an attribute) can come from any of the
 *     launches of a call that has several (the backward pass, except where it is the one kernel described at attn_bwd: dQ kernel,
 *     then dK/dV, at d = 256 as a dV and a dK kernel; a call for its dK/dV pass that asks for ATTN_BWD_PREPARE: the
 *     prepare kernel in front; most variable-length calls: a small table kernel first; a variable-length
 *     or strided forward pass whose keys are divided: a merge kernel last, without which o and lse
 *     are untouched): the launches before the failed one stay enqueued and write their outputs (dq,
 *     dv, the workspace); the outputs of the failed and later launches are untouched.
 *   - A call's results depend on its arguments alone, bit for bit from run to run.  Kernels are
 *     chosen by all sizes, B and H among them, and differ in the order of fp32 sums (forward, dQ):
 *     the rows of one sequence agree to rounding, not to the bit, between calls with another number
 *     of sequences or heads beside it.
 *   - A NaN or an infinity in a row of v reaches o of the queries that see the row and, under the causal mask, may
 *     reach o of up to 94 queries before them (a masked probability of 0 times it), no others; in the
 *     backward pass it may reach every gradient of its sequence.
 *   - Re-entrant; no global state.  Calls on different streams may run concurrently
 *     as long as their outputs and workspaces do not overlap.
 */
#ifndef PAPER_2603_05451_AMD_ATTN_H
#define PAPER_2603_05451_AMD_ATTN_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    ATTN_OK = 0,
    ATTN_EINVAL = -1,       /* null pointer, non-positive size, H % Hkv != 0, misaligned pointer,
                               workspace too small */
    ATTN_EUNSUPPORTED = -2, /* head dims or N outside the supported set */
    ATTN_ELAUNCH = -3,      /* the HIP runtime refused a launch */
    ATTN_ETOOLARGE = -4     /* attn_bwd_noalloc only: B * H * N above ATTN_NOALLOC_MAX_ROWS */
};

/* Forward pass (paper Sec. 2.1 first display; tiled evaluation per Sec. 3.1.4).
 *   in : q [B,N,H,d_qk], k [B,N,Hkv,d_qk], v [B,N,Hkv,d_v]   bf16, device
 *   out: o [B,N,H,d_v] bf16, lse [B,H,N] fp32                 device
 * attn_fwd is attn_fwd_ex with d_qk = d_v = d. */
int attn_fwd(const void* q, const void* k, const void* v, void* o, float* lse,
             int B, int H, int Hkv, int N, int d, float scale, int causal, void* stream);
int attn_fwd_ex(const void* q, const void* k, const void* v, void* o, float* lse,
                int B, int H, int Hkv, int N, int d_qk, int d_v, float scale, int causal,
                void* stream);

/* Backward pass (paper Sec. 2.1 second display).
 *   in : q, k, v as above; o, d_o [B,N,H,d_v] bf16; lse [B,H,N] fp32 -- o and lse
 *        must be the outputs of the forward call with the same arguments
 *   out: dq [B,N,H,d_qk], dk [B,N,Hkv,d_qk], dv [B,N,Hkv,d_v]  bf16
 *   workspace: device scratch of at least attn_bwd_workspace_bytes(...) bytes,
 *        256-byte aligned; contents on entry are ignored, contents on exit are
 *        unspecified; may be reused by the next call on the same stream.
 * Two kernels are enqueued, in this order: the dQ kernel (one workgroup per query tile, dQ
 * accumulated on chip over all KV tiles; it also forms D = rowsum(dO o O) and the base-2 LSE of
 * its rows and leaves them in the workspace), then the dK/dV kernel (one workgroup per KV tile,
 * dK and dV accumulated on chip over all query tiles and all query heads of the group: the loop
 * structure of paper Sec. 3.2.2; at d = 256 a dV and a dK kernel).  The paper accumulates dQ with
 * global atomics inside the dK/dV loop (Sec. 3.2.2-3.2.3); on MI355X those atomics are memory-side
 * and cost more than recomputing S and dP, so dQ has its own pass -- except where one workgroup can hold all keys of a
 * sequence (up to 512 at d = 64, 256 at 96 and 128, of enough sequences and heads or few queries): one kernel then
 * makes S and dP once and sums dQ over the keys on chip, and the workspace is not used.  No atomics are used: results are bit-reproducible from run to run (the
 * property paper Sec. 3.2.4 obtains with semaphores). */
int attn_bwd(const void* q, const void* k, const void* v, const void* o, const void* d_o,
             const float* lse, void* dq, void* dk, void* dv,
             int B, int H, int Hkv, int N, int d, float scale, int causal,
             void* workspace, size_t workspace_bytes, void* stream);
int attn_bwd_ex(const void* q, const void* k, const void* v, const void* o, const void* d_o,
                const float* lse, void* dq, void* dk, void* dv,
                int B, int H, int Hkv, int N, int d_qk, int d_v, float scale, int causal,
                void* workspace, size_t workspace_bytes, void* stream);

/* attn_bwd_ex restricted to a subset of its passes, for per-kernel timing and profiling (the
 * backward of paper Sec. 3.2 is one logical step; this splits it at the kernel boundaries).
 * phases is a bit mask: ATTN_BWD_PREPARE (-D and base-2 LSE into the workspace), ATTN_BWD_DKDV
 * (writes dk, dv; reads -D and the base-2 LSE from the workspace), ATTN_BWD_DQ (writes dq).  All
 * arguments as attn_bwd_ex.  The dQ kernel computes -D and the base-2 LSE of its own rows
 * itself (the same values bit for bit as the prepare kernel) and writes them to the workspace,
 * so a call whose mask includes ATTN_BWD_DQ launches no prepare kernel: the dQ kernel runs first
 * and ATTN_BWD_DKDV, of the same or of a later call, reads what it left.  attn_bwd_ex is
 * therefore two kernels (three at d = 256, where ATTN_BWD_DKDV is two); ATTN_BWD_PREPARE has an
 * effect only in a mask without ATTN_BWD_DQ.  At sizes whose whole backward pass is one kernel, a call for
 * one pass is that kernel without the other pass's products: the same bits, in any order, and the workspace is
 * written by ATTN_BWD_PREPARE only and read by none. */
enum { ATTN_BWD_PREPARE = 1, ATTN_BWD_DKDV = 2, ATTN_BWD_DQ = 4, ATTN_BWD_ALL = 7 };
int attn_bwd_phases(const void* q, const void* k, const void* v, const void* o, const void* d_o,
                    const float* lse, void* dq, void* dk, void* dv,
                    int B, int H, int Hkv, int N, int d_qk, int d_v, float scale, int causal,
                    void* workspace, size_t workspace_bytes, void* stream, int phases);

/* attn_bwd_ex for callers that cannot allocate device memory at all: code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc (and with it torch's allocator).  The
 * workspace (-D and the base-2 LSE, 8 bytes per row of B * H * N) is an array inside the library's
 * own device image, 8 MiB per GPU the library runs on, held until the process ends; this call and
 * everything it reaches allocates and frees nothing.  Inputs, outputs, layouts and results are
 * those of attn_bwd_ex (bit for bit).
 *   - B * H * N must not exceed ATTN_NOALLOC_MAX_ROWS; beyond that the call returns
 *     ATTN_ETOOLARGE with nothing enqueued.
 *   - All calls on one GPU share that GPU's array: two calls that overlap in time on one GPU (on
 *     different streams, or from different host threads) race on it.  Calls on one stream, or
 *     ordered by events, are fine; nothing needs to be cleared between calls (every row that is
 *     read has been written earlier in the same call). */
#define ATTN_NOALLOC_MAX_ROWS (1 << 20)
int attn_bwd_noalloc(const void* q, const void* k, const void* v, const void* o, const void* d_o,
                     const float* lse, void* dq, void* dk, void* dv,
                     int B, int H, int Hkv, int N, int d_qk, int d_v, float scale, int causal,
                     void* stream);

/* Bytes of workspace attn_bwd(_ex) needs for these sizes (0 if they are invalid):
 * D and the base-2 LSE, [B,H,N] fp32 each (256-byte aligned sections). */
size_t attn_bwd_workspace_bytes(int B, int H, int Hkv, int N, int d_qk, int d_v);

/* Variable sequence lengths (paper Sec. 3.3: a list of query and key/value sequence lengths per
 * batch): B sequences packed back to back, attention inside each sequence only; a sequence's
 * number of queries and number of keys may differ (cross-attention, decoding against a cache).
 *   layouts  q, o, d_o, dq : [Tq, H, d]    k, dk : [Tk, Hkv, d_qk]    v, dv : [Tk, Hkv, d_v]   bf16
 *            lse           : [H, Tq] fp32
 *            cu_seqlens_q  : [B + 1] int32, DEVICE memory, cu[0] = 0, non-decreasing,
 *                            cu[B] = Tq = total_q; sequence b owns query rows cu[b] .. cu[b+1]-1.
 *            cu_seqlens_k  : the same for the key/value rows, cu[B] = Tk = total_k; may be the same
 *                            pointer as cu_seqlens_q (self-attention).
 *                            Any length >= 0 is allowed (no multiple-of-128 requirement), except that
 *                            a sequence with queries must have at least one key, and under a causal
 *                            mask at least as many keys as queries.
 *   causal != 0: the last query of a sequence is aligned with its last key: key j is visible to
 *   query i iff j <= i + (keys - queries) of that sequence; j <= i for self-attention.
 *   The host never reads the lengths: a small kernel turns them into tables of 128-row tiles (a decode
 *   step of at most 64 sequences -- no more queries than sequences, and H > Hkv, d_qk = 192 or more than
 *   128 keys per query -- does so in its attention kernel),
 *   sequences with the longest loop per tile first (the longest-processing-time-first order of
 *   Sec. 3.3), and the attention kernels are launched over upper bounds of total_q/128 + B query
 *   tiles per head and total_k/128 + B key tiles per key/value head.
 *   workspace: attn_varlen_workspace_bytes(..., backward) bytes, 256-byte aligned; the forward
 *   call needs the backward = 0 size, the backward call the backward = 1 size.  Contents on entry
 *   are ignored.  (Where few queries meet many keys the forward size includes room for partial results
 *   of a pass whose keys are divided over several blocks; with less room, down to the query-tile table
 *   alone, a call divides them less, and its results differ by the rounding of another summation
 *   order.)  All other conventions (device pointers, stream, alignment, head dims, error codes) are
 *   those of attn_fwd_ex / attn_bwd_ex.
 *   What makes the tables checks every sequence's boundaries on the device against total_q and total_k:
 *   a sequence whose rows do not lie inside the tensors (decreasing boundaries, boundaries past the
 *   totals) is left out, i.e. none of its rows is read or written, and the other sequences are
 *   served.  The remaining conditions (a key for every sequence with queries; keys >= queries under
 *   a causal mask) are not checked: rows that violate them hold unspecified values, nothing outside
 *   the tensors is touched. */
size_t attn_varlen_workspace_bytes(int B, int total_q, int total_k, int H, int Hkv, int d_qk, int d_v, int backward);
int attn_varlen_fwd(const void* q, const void* k, const void* v, void* o, float* lse,
                    const int* cu_seqlens_q, const int* cu_seqlens_k, int B, int total_q, int total_k,
                    int H, int Hkv, int d_qk, int d_v,
                    float scale, int causal, void* workspace, size_t workspace_bytes, void* stream);
/* The tile tables alone (paper Sec. 3.3: the sort's metadata can be cached).  Fills both tables
 * at the head of a workspace of the backward = 1 size.  A later attn_varlen_fwd / attn_varlen_bwd
 * (or _dtype) call on that workspace with the SAME B, total_q, total_k, H, Hkv and head dims may
 * then pass cu_seqlens_q = cu_seqlens_k = NULL: it skips the plan kernel and uses the tables as
 * they are (a backward call needs tables written by this function or by an earlier backward call;
 * a forward call with non-NULL cu_seqlens writes the query table only).  Calls never modify the
 * tables otherwise (what lies behind them is scratch: calls that share a planned workspace may not
 * overlap in time); results are bit-identical to those of calls that rebuild them in a workspace of
 * that size.  Table entries carry a mark and are checked against total_q: on a workspace that was
 * never planned the kernels find nothing to act on and leave the outputs untouched (tables planned
 * for OTHER lengths with the same totals cannot be told apart: that remains the caller's
 * responsibility). */
int attn_varlen_plan(const int* cu_seqlens_q, const int* cu_seqlens_k, int B, int total_q, int total_k,
                     int H, int Hkv, int d_qk, int d_v, void* workspace, size_t workspace_bytes, void* stream);
/* Backward of attn_varlen_fwd (paper Sec. 2.1 second display, per sequence): o and lse must be that
 * call's outputs for the same arguments; dk and dv are summed over the query heads of each group.
 * Every row of dq, dk, dv is written (dk = dv = 0 for the keys of a sequence without queries).
 * No atomics: bit-reproducible like attn_bwd. */
int attn_varlen_bwd(const void* q, const void* k, const void* v, const void* o, const void* d_o,
                    const float* lse, void* dq, void* dk, void* dv,
                    const int* cu_seqlens_q, const int* cu_seqlens_k, int B, int total_q, int total_k,
                    int H, int Hkv, int d_qk, int d_v,
                    float scale, int causal, void* workspace, size_t workspace_bytes, void* stream);

/* The same four operations on IEEE fp16 storage (the paper's benchmarks cover FP16 and BF16
 * inputs, Sec. 5): dtype = ATTN_BF16 is exactly the entry point without the suffix, dtype =
 * ATTN_F16 reads q, k, v, o, d_o and writes o, dq, dk, dv as fp16 (round to nearest even), with
 * fp16 MFMA operands (P and dS are rounded to fp16) and fp32 accumulation, statistics and LSE.
 * Any other dtype: ATTN_EUNSUPPORTED.  All remaining arguments and conventions as in
 * attn_fwd_ex, attn_bwd_ex, attn_varlen_fwd, attn_varlen_bwd. */
enum { ATTN_BF16 = 0, ATTN_F16 = 1 };
int attn_fwd_dtype(int dtype, const void* q, const void* k, const void* v, void* o, float* lse,
                   int B, int H, int Hkv, int N, int d_qk, int d_v, float scale, int causal, void* stream);
int attn_bwd_dtype(int dtype, const void* q, const void* k, const void* v, const void* o, const void* d_o,
                   const float* lse, void* dq, void* dk, void* dv,
                   int B, int H, int Hkv, int N, int d_qk, int d_v, float scale, int causal,
                   void* workspace, size_t workspace_bytes, void* stream);
int attn_varlen_fwd_dtype(int dtype, const void* q, const void* k, const void* v, void* o, float* lse,
                          const int* cu_seqlens_q, const int* cu_seqlens_k, int B, int total_q, int total_k,
                          int H, int Hkv, int d_qk, int d_v,
                          float scale, int causal, void* workspace, size_t workspace_bytes, void* stream);
int attn_varlen_bwd_dtype(int dtype, const void* q, const void* k, const void* v, const void* o, const void* d_o,
                          const float* lse, void* dq, void* dk, void* dv,
                          const int* cu_seqlens_q, const int* cu_seqlens_k, int B, int total_q, int total_k,
                          int H, int Hkv, int d_qk, int d_v,
                          float scale, int causal, void* workspace, size_t workspace_bytes, void* stream);

/* Strided layouts: the same attention on equal-length batches whose tensors are views with
 * arbitrary batch, token and head strides -- [B, H, N, d] tensors, slices of a fused QKV
 * projection, padded buffers -- with Nq >= 1 queries and Nk >= 1 keys per sequence (no
 * multiple-of-128 requirement; Nq != Nk is a prefix held in a cache, a decode step or
 * cross-attention).  The head dim is contiguous.  Element (b, n, h, c) of a tensor x with strides
 * sx (counted in ELEMENTS) is x[b * sx->batch + n * sx->row + h * sx->head + c]; q, o, d_o, dq
 * have Nq tokens and H heads, k, v, dk, dv Nk tokens and Hkv heads.
 * Every stride must be a non-negative multiple of 8 (16-byte vector accesses), non-zero
 * wherever the corresponding extent exceeds 1, and the token stride at most 2^23 elements;
 * outputs must not overlap themselves or any input.  lse is [B, H, Nq] fp32, contiguous.
 * causal != 0: the last query is aligned with the last key, key j is visible to query i iff
 * j <= i + Nk - Nq (the convention of the variable-length calls; the paper is silent on
 * Nq != Nk), and Nk >= Nq is required (ATTN_EINVAL otherwise).
 * Runs the variable-length kernels (the backward pass of few keys: attn_bwd's kernel for those) as on the sequence boundaries {0, Nq, 2 Nq, ...} and
 * {0, Nk, 2 Nk, ...}, whose tiles the kernels number themselves; on contiguous [B, N, H, d] tensors with
 * Nq = Nk = N a multiple of 128 the results are bit-identical to attn_fwd_dtype / attn_bwd_dtype (the
 * forward call then is that call).
 *   workspace: attn_strided_workspace_bytes(..., backward) bytes, 256-byte aligned, contents
 *   ignored on entry.  Other conventions as in attn_fwd_dtype / attn_bwd_dtype. */
typedef struct attn_strides {
    long long batch, row, head;
} attn_strides_t;
size_t attn_strided_workspace_bytes(int B, int H, int Hkv, int Nq, int Nk, int d_qk, int d_v, int backward);
int attn_fwd_strided(int dtype, const void* q, const attn_strides_t* sq, const void* k, const attn_strides_t* sk,
                     const void* v, const attn_strides_t* sv, void* o, const attn_strides_t* so, float* lse,
                     int B, int H, int Hkv, int Nq, int Nk, int d_qk, int d_v, float scale, int causal,
                     void* workspace, size_t workspace_bytes, void* stream);
int attn_bwd_strided(int dtype, const void* q, const attn_strides_t* sq, const void* k, const attn_strides_t* sk,
                     const void* v, const attn_strides_t* sv, const void* o, const attn_strides_t* so,
                     const void* d_o, const attn_strides_t* sdo, const float* lse,
                     void* dq, const attn_strides_t* sdq, void* dk, const attn_strides_t* sdk,
                     void* dv, const attn_strides_t* sdv,
                     int B, int H, int Hkv, int Nq, int Nk, int d_qk, int d_v, float scale, int causal,
                     void* workspace, size_t workspace_bytes, void* stream);

/* Rotary positions of queries and keys, with the norms of their heads in the same pass (the paper starts from the Q and K that
 * result).  For every row x of d numbers (a token of a head of q or of k):
 *     n   = x * w / sqrt(mean(x^2) + eps)       with norm != 0 (w: q_weight or k_weight [d], element type; null: ones), else n = x
 *     y_i = A (cos(a) n_i - sin(a) n_j),  y_j = A (sin(a) n_i + cos(a) n_j)        for the pairs (i, j) of the rotated dims
 *     y_c = n_c                                                                    for the others
 * The rotated dims are offset ... offset + rot - 1 of the head (rot and offset multiples of 16 and 8); pair p = 0 ... rot/2 - 1 is
 * dims (offset + p, offset + rot/2 + p), or, with interleaved != 0, (offset + 2p, offset + 2p + 1); a = position * freqs[p], as if
 * exact: far positions lose nothing; A = amplitude.  Contexts longer than trained ones are a matter of freqs and amplitude.
 * positions: int32, one per token, any value, token n of sequence b at positions[b * positions_batch + n] (positions_batch = 0: the
 * same for every sequence); null: n.  Sums and products are in fp32, with the power of two that a row takes whose squares would leave
 * its range; the result is rounded once, to the element type.  A row of zeros is NaN with eps = 0, zeros otherwise.
 *   tensors: views as in attn_fwd_strided, the token stride without its limit, q and q_out [B, N, H, d], k and k_out
 *   [B, N, Hkv, d] (B = 1 for packed tokens), d 64, 96, 128, 192 or 256; k and k_out may both be null.  An output may be
 *   its input (same address and strides); any other overlap is an error of the caller's. */
typedef struct attn_rope {
    const float* freqs;         /* [rot / 2], fp32, device */
    const int* positions;       /* device, or null */
    long long positions_batch;
    int rot, offset, interleaved;
    float amplitude;
    int norm;
    float eps;                  /* >= 0 */
    const void *q_weight, *k_weight;
} attn_rope_t;
int attn_rope_fwd(int dtype, const attn_rope_t* rope, const void* q, const attn_strides_t* sq, const void* k, const attn_strides_t* sk,
                  void* q_out, const attn_strides_t* sqo, void* k_out, const attn_strides_t* sko,
                  int B, int N, int H, int Hkv, int d, void* stream);
/* Its backward pass: dq and dk are the gradients of q_out and k_out, dq_in and dk_in receive those of q and k (an output may be
 * one of the pass's inputs of the same tensor), dq_weight and dk_weight (fp32 [d], each may be null) those of the weights, summed
 * over all rows in fp32 in an order that depends on the sizes alone.  q and k are the forward pass's inputs, needed with norm != 0
 * only (else they and their strides may be null).  workspace: attn_rope_workspace_bytes(...) bytes, 256-byte aligned, for the sums;
 * may be null where both dq_weight and dk_weight are.  Two kernels with the sums, one without. */
size_t attn_rope_workspace_bytes(int B, int N, int H, int Hkv, int d);
int attn_rope_bwd(int dtype, const attn_rope_t* rope, const void* dq, const attn_strides_t* sdq, const void* dk, const attn_strides_t* sdk,
                  const void* q, const attn_strides_t* sq, const void* k, const attn_strides_t* sk,
                  void* dq_in, const attn_strides_t* sdqi, void* dk_in, const attn_strides_t* sdki, float* dq_weight, float* dk_weight,
                  int B, int N, int H, int Hkv, int d, void* workspace, size_t workspace_bytes, void* stream);

/* A cache of keys and values in 4 or 8 bits, in pages: rows are quantised as they are written, read back, or attended to.
 *   k, v           : codes, [pages, Hkv, page, d_qk * bits / 8] and [pages, Hkv, page, d_v * bits / 8] bytes, 16-byte aligned
 *   k_scale, v_scale : [pages, Hkv, page, d_qk / 32] and [pages, Hkv, page, d_v / 32] bytes
 * all contiguous, in device memory.  A row (token, KV head) is in blocks of 32 channels with one scale byte s each, which stands
 * for 2^(s - 127) (255: the block is NaN); bits = 4: e2m1 codes (sign, 2 exponent bits, 1 mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6), the
 * even channel in the low half of the byte; bits = 8: e4m3 codes (largest value 448, 0x7f NaN).  (The block formats of the OCP
 * Microscaling specification v1.0, which gfx950 converts in hardware.)  The scale is the least power of two with which no element
 * of the block is cut off when it is rounded to nearest (ties to even); a block that holds an infinity or a NaN is NaN.  Rounding
 * is exact arithmetic: codes and scales depend on the row's values alone.
 *   page: tokens per page, a power of two, 16 ... 65536; pages * page <= 2^31 - 1; head dims as elsewhere.
 * Slot s is token s % page of page s / page.  Calls on rows take T of at least 1 and T * Hkv * d up to 2^34 - 2048. */
typedef struct attn_cache {
    void *k, *k_scale, *v, *v_scale;
    int pages, page, Hkv, d_qk, d_v, bits;
} attn_cache_t;
/* Quantises k [T, Hkv, d_qk] and v [T, Hkv, d_v] (views as in attn_rope_fwd; `batch` is not used) into the slots slots[0 ... T-1] (int32,
 * device).  A row whose slot is negative or past the cache is skipped (padding); the others must differ, or the bytes of a slot that is
 * given twice are unspecified.  No other byte of the cache is touched. */
int attn_cache_write(int dtype, const attn_cache_t* cache, const void* k, const attn_strides_t* sk, const void* v, const attn_strides_t* sv,
                     const int* slots, int T, void* stream);
/* The rows of these slots (any order, any number of times) as numbers of the element type: k [T, Hkv, d_qk], v [T, Hkv, d_v], contiguous;
 * zeros where a slot is negative or past the cache.  bf16 holds every value exactly but 2^128, which is infinite: what a number of at
 * least 7 * 2^125 (2.98e38; 4 bits) or 248 * 2^120 (3.30e38; 8 bits) was rounded to.  fp16 rounds, and is infinite from 2^16 on: of its own
 * numbers, those of at least 57344 (4 bits) or 63488 (8 bits). */
int attn_cache_read(int dtype, const attn_cache_t* cache, const int* slots, int T, void* k, void* v, void* stream);
/* Attention of Nq queries per sequence over that cache: sequence b has lens[b] keys (int32, device), key j in page
 * block_table[b * table_width + j / page] (int32, device) at j % page.  q and o are views [B, Nq, H, d] as in attn_rope_fwd, lse [B, H, Nq]
 * contiguous.  causal != 0: the last query is aligned with the last key (key j visible to query i iff j <= i + lens[b] - Nq).
 *   - A query without a visible key (an empty batch slot, lens[b] = 0, or causal with fewer keys than queries) has o = 0 and
 *     lse = -inf.  A negative length counts as 0, one beyond table_width * page as that.
 *   - Entries of the table behind a sequence's last key are not read.  A page number outside the cache makes the rows that see
 *     its keys NaN; nothing outside the tensors is touched.
 *   - Keys and values that are no finite numbers (a scale byte of 255; e4m3's own NaN, 0x7f, which attn_cache_write does not write;
 *     for fp16 queries, whose type the cache's numbers are taken in, what is beyond its range) reach the queries that see them and no
 *     others: a value makes its channel of their o infinite or NaN, a key all of it.  What the slots behind the last key hold (never
 *     written, another sequence's, NaN) reaches none.
 *   - Sums are in fp32, o's before their division by the row sum, with weights up to 2^8: finite values of 2^120 / lens[b] and more may
 *     make it infinite.
 *   - Lengths and pages are read on the device: a captured call may be replayed with others.  Any Nq works; it is meant for few
 *     (one token, a few drafted ones): chunks of prompts, and batches of both, go to attn_cache_chunk_fwd.
 *     B is 65536 at most, and meant to be up to some thousands: every block finds its keys from all lengths.  Sizes whose blocks (16 or
 *     32 rows of a KV head and a sequence, four of those where there are many) pass 2^22 are ATTN_EUNSUPPORTED.
 *   workspace: attn_cache_workspace_bytes(...) bytes, 256-byte aligned, contents ignored.  One kernel, and a merge where the table
 *   is wide enough for a sequence to be divided (without which the o and lse of divided sequences are untouched). */
size_t attn_cache_workspace_bytes(const attn_cache_t* cache, int B, int Nq, int H, int table_width);
int attn_cache_fwd(int dtype, const attn_cache_t* cache, const void* q, const attn_strides_t* sq, void* o, const attn_strides_t* so, float* lse,
                   const int* block_table, int table_width, const int* lens, int B, int Nq, int H, float scale, int causal,
                   void* workspace, size_t workspace_bytes, void* stream);

/* Attention of chunks of queries over that cache: sequence b has the queries cu_seqlens[b] ... cu_seqlens[b + 1] - 1 of q (packed [T, H, d_qk], int32
 * [B + 1], device) and lens[b] keys in the pages of its row of block_table, as in attn_cache_fwd; with a chunk of a prompt these are what was
 * cached before and the chunk itself, already written.  q and o are views [T, H, d] as in attn_rope_fwd (`batch` is not used), lse [H, T]
 * contiguous.  causal != 0: a sequence's last query is aligned with its last key (key j visible to its query i iff j <= i + lens[b] - queries).
 *   - Empty queries, lengths, pages and numbers that are not finite are dealt with as in attn_cache_fwd, whatever the chunk's length.
 *   - exp(score - maximum) is rounded to the element type for its product with V, as in the other attention calls (its sum, and lse, are of what was not
 *     rounded); all sums are in fp32, and o is rounded once.  The two roundings are of one size: of normal numbers o is off by 2.3e-3 relative in
 *     bf16, 2.8e-4 in fp16, where that of o alone makes 1.7e-3 and 2.1e-4.
 *   - A sequence whose boundaries do not ascend within 0 ... T has no queries.  Rows of q that belong to no sequence (padding behind the last
 *     one) are not touched in o and lse.  Two sequences must not share queries (the results of such rows are unspecified).
 *   - Boundaries, lengths and pages are read on the device: a captured call may be replayed with others.
 *     B is 65536 at most, T * H * d up to 2^34, T * H up to 2^28.
 *   workspace: attn_cache_chunk_workspace_bytes(...) bytes, 256-byte aligned, contents ignored.  One kernel, and a merge where there are so few rows
 *   that keys may be divided over blocks (without which the o and lse of divided sequences are untouched). */
size_t attn_cache_chunk_workspace_bytes(const attn_cache_t* cache, int B, int T, int H, int table_width);
int attn_cache_chunk_fwd(int dtype, const attn_cache_t* cache, const void* q, const attn_strides_t* sq, void* o, const attn_strides_t* so, float* lse,
                         const int* block_table, int table_width, const int* cu_seqlens, const int* lens, int B, int T, int H, float scale, int causal,
                         void* workspace, size_t workspace_bytes, void* stream);

/* The attention weight that every cached key had from the queries of one of these calls, added to its sum: weights is fp32 [pages, Hkv, page],
 * contiguous, 16-byte aligned, one per row of the cache, and
 *     weights(j) += sum over the sequence's queries i that see key j, and the heads h of the KV head's group, of exp(scale q_ih . k_j - lse_ih),
 * for every key j < lens[b] of every sequence that has queries.  q and lse are that call's: with cu_seqlens those of attn_cache_chunk_fwd (q packed,
 * Nq is T, lse [H, T]), with cu_seqlens null those of attn_cache_fwd (q [B, Nq, H, d_qk], lse [B, H, Nq]).
 *   - fresh != 0: the sequence's last keys, as many as it has queries, are the call's own: their weights are set, not added to, so that
 *     what a page held before does not matter.
 *   - A query with lse = -inf (it saw no key, or the caller leaves it out so) adds nothing to finite keys, whatever its row of q holds.  Entries of the
 *     table that are outside the cache are passed over.  Weights of other rows are not touched.
 *   - Numbers that are not finite go by the formula: a NaN key has the weight NaN, and so has every key that a query with lse = NaN sees; the queries
 *     that see a NaN key have that lse from the attention calls.  (attn_cache_evict takes NaN for the greatest.)  An infinite key (fp16: one beyond
 *     its range) gets 0 from a score of -inf, NaN from one of +inf or from a query left out.
 *   - Every row of the cache may belong to one sequence at most (a page that two sequences share has unspecified weights).
 *   - Sums are in fp32, in an order that depends on the sizes and lengths alone.  Limits as in the two calls.
 *   workspace: attn_cache_weigh_workspace_bytes(...) bytes (packed: whether there are cu_seqlens), 256-byte aligned, contents ignored.  One kernel, and
 *   one that adds up where there are rows enough for them to be divided over blocks (without which the weights of such sequences are untouched). */
size_t attn_cache_weigh_workspace_bytes(const attn_cache_t* cache, int B, int Nq, int H, int table_width, int packed);
int attn_cache_weigh(int dtype, const attn_cache_t* cache, const void* q, const attn_strides_t* sq, const float* lse, float* weights,
                     const int* block_table, int table_width, const int* cu_seqlens, const int* lens, int B, int Nq, int H, float scale, int causal,
                     int fresh, void* workspace, size_t workspace_bytes, void* stream);

/* Eviction by those weights: of every sequence with more than keep[b] rows (int32, device; a negative number counts as 0) that many stay, for each KV
 * head by itself: the last `recent` (no more than keep[b]), and of the others those with the greatest weights (ties: the first; NaN is the greatest,
 * -0 and 0 are equal).  The cache is closed up in place, rows with their weights: with n = keep[b] - recent, survivors below n remain where they
 * are, the others go, in ascending order, to the places below n that are free, the recent rows, in order, to n ... keep[b] - 1.  So rows change
 * their places, which attention does not mind (keys hold their positions), and few rows are moved; the last ones remain in order.  What lies behind
 * the first keep[b] rows is left as it is, and its pages are free.  lens_out[b] = min(lens[b], keep[b]); lens_out may not overlap lens or keep.
 *   - Lengths as in attn_cache_fwd.  A row of a page number outside the cache has the least weight; one that stays nevertheless is NaN, with weight 0, where
 *     it goes to a place in the cache.
 *   - Every row of the cache may belong to one sequence at most.
 *   - k_scale and v_scale are 8-byte aligned.  B * Hkv is 2^22 at most, table_width * page 2^26.
 *   workspace: attn_cache_evict_workspace_bytes(...) bytes (4 for every row that the table has room for, and head; 64 KiB at most for tables of up to
 *   32 768 rows), 256-byte aligned, contents ignored. */
size_t attn_cache_evict_workspace_bytes(const attn_cache_t* cache, int B, int table_width);
int attn_cache_evict(const attn_cache_t* cache, float* weights, const int* block_table, int table_width, const int* lens, const int* keep, int recent,
                     int B, int* lens_out, void* workspace, size_t workspace_bytes, void* stream);

/* Software 2^x of paper Sec. 3.1.3 (range reduction + degree-n minimax polynomial, p0 = 1, Horner
 * with FMAs, exponent splice), provided to measure its accuracy on this hardware; attn_fwd does not
 * use it (v_exp_f32 and the FMAs share one issue port on CDNA4, so emulation cannot add throughput:
 * the rate probes that show this live in a library of their own, include/attn_probes.h).
 *   attn_exp2_emulated: y[i] = 2^x[i] for n fp32 values; degree 3, 4 or 5, or 0 for the hardware
 *       instruction.  x, y: device pointers, 4-byte aligned, may not overlap partially. */
int attn_exp2_emulated(const float* x, float* y, size_t n, int degree, void* stream);

/* Human-readable text for a return code (static storage). */
const char* attn_strerror(int code);

/* Library version: major * 10000 + minor * 100 + patch. */
int attn_version(void);

#ifdef __cplusplus
}
#endif
#endif
