/*
 * flashmask.h -- C ABI of the MI355X (gfx950) FlashMask attention library.
 *
 * FlashMask (arXiv 2410.01359) describes an attention mask by four int32
 * vectors over the key columns: query row i may NOT attend to key column j iff
 *     LTS[j] <= i < LTE[j]   or   UTS[j] <= i < UTE[j]
 * (Section 4.1; rows and columns 0-based, intervals half-open, an interval with
 * start >= end is empty, any int32 value is accepted).  The library computes
 * exactly the dense-mask attention of Equations 1-2 and its gradients
 * (Algorithms 1 and 2, Section 4.4), skipping tiles that the per-block min/max
 * tables of Section 4.2 prove fully masked.
 *
 * Conventions shared by every entry point
 *   - All data pointers are DEVICE pointers owned by the caller and must stay
 *     valid until the stream has run past the call.  The library allocates and
 *     frees nothing, creates no streams and never synchronises the host: work
 *     is enqueued on `hip_stream` (a hipStream_t passed as void*; NULL is the
 *     default stream) and the call returns at once.
 *   - q, k, v, out, dout, dq, dk, dv: bf16, contiguous [B, H, N, d], d innermost.
 *   - lts, lte, uts, ute: int32, contiguous [B, N]; one mask per batch row,
 *     shared by all heads.
 *   - lse, and the library's own D vector: fp32 [B, H, N].
 *   - d must be 64 or 128; N is any positive length (one that is not a multiple
 *     of 128 runs at the next multiple, its extra columns masked); tensor
 *     pointers must be 16-byte aligned.
 *   - Outputs are overwritten in full.  The same call gives the same bits every time.  The order of its fp32 sums
 *     follows from how the work is cut (flashmask_work_cut), so the results of one (b, h) slice may differ in the
 *     last places with the B, H and N of the call that computes it and with the GPU's number of compute units.
 *   - Return value: FM_OK (0) or a negative FM_ERR_* code.  Only conditions the
 *     host can see are checked; bound VALUES live on the device and are not
 *     validated (the comparison above is defined for every int32).
 *   - Calls on different streams need different workspaces.
 *   - Calls may be recorded into a HIP graph (no allocation, no host synchronisation, and the only
 *     clears of global memory are kernels).  The first call of a kernel variant on a device raises
 *     that kernel's dynamic-LDS limit (hipFuncSetAttribute): issue one call of the same shape class
 *     (d, aligned or ragged N, contiguous or _ex; any sizes) outside the capture first.
 */
#ifndef FLASHMASK_H
#define FLASHMASK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  FM_OK = 0,
  FM_ERR_NULL = -1,      /* a required pointer is NULL */
  FM_ERR_SHAPE = -2,     /* B, H, N <= 0, d not in {64,128}, sizes beyond 32-bit indexing, bad block size */
  FM_ERR_ALIGN = -3,     /* a tensor pointer is not 16-byte aligned */
  FM_ERR_WORKSPACE = -4, /* workspace is NULL or smaller than flashmask_workspace_bytes() */
  FM_ERR_HIP = -5,       /* a kernel launch failed; see flashmask_last_hip_error() */
  FM_ERR_ARG = -6,       /* unknown pass id, type or layout, types that do not go together, scale <= 0 or not finite */
  FM_ERR_STATIC_LIMIT = -7 /* flashmask_fwd_noalloc: the problem does not fit the library's static scratch */
};

/* Pass ids for flashmask_workspace_bytes / flashmask_tile_shape. */
enum {
  FM_PASS_FWD = 0,      /* forward tile loop (Algorithm 1) */
  FM_PASS_BWD_DKDV = 1, /* backward, column-parallel dK/dV loop (Algorithm 2) */
  FM_PASS_BWD_DQ = 2,   /* backward, row-parallel dQ loop (Algorithm 2's dQ update, run per query block) */
  FM_PASS_BWD = 3       /* whole backward call (workspace query only) */
};

/* Tile-class byte written by flashmask_classify (Equation 4).
 * Low two bits: kind.  Bits 4 / 5: a partially masked tile needs the element
 * mask of the lower-triangle pair / of the upper-triangle pair. */
enum {
  FM_TILE_UNMASKED = 0,
  FM_TILE_PARTIAL = 1,
  FM_TILE_FULLY = 2,
  FM_TILE_NEED_LT = 1 << 4,
  FM_TILE_NEED_UT = 1 << 5
};

/*
 * Forward pass: Algorithm 1 (its outputs O and L), i.e. Equations 1-2 with
 * S = scale * Q K^T, masked scores = -inf, out = softmax(S) V and
 * lse_i = log sum_j exp(S_ij) (natural log, of the scaled scores).
 * A query row whose keys are all masked gets out = 0 and lse = -inf.
 *
 *   q, k, v        in   bf16 [B,H,N,d]
 *   lts..ute       in   int32 [B,N]
 *   scale          in   multiplies Q K^T (1/sqrt(d) in the paper's Equation 1); must be
 *                       positive and finite (FM_ERR_ARG otherwise)
 *   out            out  bf16 [B,H,N,d]
 *   lse            out  fp32 [B,H,N]
 *   workspace      scratch of at least flashmask_workspace_bytes(FM_PASS_FWD, ...)
 *                  bytes, 256-byte aligned; contents undefined afterwards.
 */
int flashmask_fwd(const void* q, const void* k, const void* v,
                  const int32_t* lts, const int32_t* lte, const int32_t* uts, const int32_t* ute,
                  float scale, void* out, float* lse,
                  int B, int H, int N, int d,
                  void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Backward pass: Algorithm 2.  Given the forward's out and lse and the upstream
 * gradient dout, writes dq, dk, dv (bf16 [B,H,N,d]):
 *   P = exp(S - lse), dV = P^T dO, dP = dO V^T, D_i = sum_c dO_ic O_ic,
 *   dS = P o (dP - D), dQ = scale dS K, dK = scale dS^T Q.
 * Rows with lse = -inf contribute nothing and get dq = 0.
 * The dQ accumulation runs per query block in a fixed order, so results are
 * bit-reproducible run to run (the paper's kernel needs a switch for that,
 * Section 5.2).
 *   workspace: at least flashmask_workspace_bytes(FM_PASS_BWD, ...) bytes.
 */
int flashmask_bwd(const void* q, const void* k, const void* v,
                  const void* out, const float* lse, const void* dout,
                  const int32_t* lts, const int32_t* lte, const int32_t* uts, const int32_t* ute,
                  float scale, void* dq, void* dk, void* dv,
                  int B, int H, int N, int d,
                  void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * flashmask_fwd for callers that cannot allocate device memory or pass a workspace: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, arithmetic,
 * kernels and results as flashmask_fwd, but the scratch (min/max tables, work counts, unit queues)
 * lives in a static device array inside the library instead of a caller's
 * workspace.  The call allocates and frees nothing.
 *   - Limit: flashmask_workspace_bytes(FM_PASS_FWD, B, H, N, d) must not exceed
 *     FLASHMASK_NOALLOC_SCRATCH_BYTES (4 MiB: about 250 000 row blocks of 128 queries over all batch
 *     rows and heads, e.g. B*H = 512 at N = 65536); larger problems return FM_ERR_STATIC_LIMIT and
 *     launch nothing.  Each GPU the library runs on holds its own copy of the array until the process
 *     ends.
 *   - The first call on a device looks the array's address up (hipGetSymbolAddress) and, like
 *     flashmask_fwd, raises the tile loop's dynamic-LDS limit: issue one call outside a capture first.
 *   - All calls on one GPU share that GPU's array: two calls that overlap in time on the same GPU
 *     (different streams or threads) race.  Calls on one stream, or otherwise ordered, are fine; the
 *     array's contents carry nothing from one call to the next.
 */
#define FLASHMASK_NOALLOC_SCRATCH_BYTES (4u << 20)
int flashmask_fwd_noalloc(const void* q, const void* k, const void* v,
                          const int32_t* lts, const int32_t* lte, const int32_t* uts, const int32_t* ute,
                          float scale, void* out, float* lse,
                          int B, int H, int N, int d, void* hip_stream);

/*
 * Layout of a bf16 tensor indexed [batch][head][row][d] for the *_ex entry points: distances, in
 * ELEMENTS, between consecutive batches, heads and rows; d itself is contiguous.  A tensor stored
 * [B,N,H,d] has {N*H*d, d, H*d}; a slice of a packed [B,N,3,H,d] projection has {N*3*H*d, d, 3*H*d}.
 * Every stride must be a multiple of 8 (16-byte vectors along d), row >= d and < 2^24
 * (FM_ERR_ALIGN / FM_ERR_SHAPE otherwise).
 */
typedef struct {
  int64_t batch, head, row;
} flashmask_strides;

/*
 * The forward and backward passes above for tensors that are not contiguous [B,H,N,d], and for
 * grouped K/V heads (the inference shape of the paper's Appendix, 32 query heads on 8 K/V heads):
 * k, v (and dk, dv) have H_kv heads, H % H_kv == 0, and query head h attends to K/V head
 * h / (H / H_kv); dk, dv are summed over the query heads of a group.  Same arithmetic, same
 * workspace size (flashmask_workspace_bytes with H), same error behaviour; lse stays fp32
 * contiguous [B,H,N].  Outputs must not overlap inputs or each other.
 *   forward : sq, sk, sv, so describe q, k, v, out
 *   backward: strides[8] describe q, k, v, out, dout, dq, dk, dv in this order
 */
int flashmask_fwd_ex(const void* q, const void* k, const void* v,
                     const int32_t* lts, const int32_t* lte, const int32_t* uts, const int32_t* ute,
                     float scale, void* out, float* lse,
                     int B, int H, int H_kv, int N, int d,
                     const flashmask_strides* sq, const flashmask_strides* sk,
                     const flashmask_strides* sv, const flashmask_strides* so,
                     void* workspace, size_t workspace_bytes, void* hip_stream);
int flashmask_bwd_ex(const void* q, const void* k, const void* v,
                     const void* out, const float* lse, const void* dout,
                     const int32_t* lts, const int32_t* lte, const int32_t* uts, const int32_t* ute,
                     float scale, void* dq, void* dk, void* dv,
                     int B, int H, int H_kv, int N, int d,
                     const flashmask_strides* strides,
                     void* workspace, size_t workspace_bytes, void* hip_stream);

/* Bytes of scratch a call of the given pass needs (FM_PASS_FWD or FM_PASS_BWD).
 * Returns 0 for an invalid shape or pass.  Host-only, no device work. */
size_t flashmask_workspace_bytes(int pass, int B, int H, int N, int d);

/*
 * Preprocessing step of Section 4.2 (Algorithm 1 "precompute the min and max
 * row index"): for every block of block_c key columns, the max and min of each
 * bound vector.
 *   minmax  out  int32 [B, 8, T_c], T_c = ceil(N / block_c), rows in the order
 *                LTStart^max, LTStart^min, LTEnd^max, LTEnd^min,
 *                UTStart^max, UTStart^min, UTEnd^max, UTEnd^min.
 * block_c must be a positive multiple of 32; any N > 0 is accepted here (a
 * ragged last block covers the columns that exist).
 */
int flashmask_preprocess(const int32_t* lts, const int32_t* lte, const int32_t* uts, const int32_t* ute,
                         int B, int N, int block_c, int32_t* minmax, void* hip_stream);

/*
 * Tile classification of Equation 4, as the skip tests and element-mask tests
 * of Algorithm 1 apply it, for every tile of block_r rows x block_c columns:
 * with r0 = i*block_r, r1 = min(r0 + block_r, N),
 *   fully(X)   = r0 >= XStart^max_j and r1 <= XEnd^min_j
 *   partial(X) = r1 >  XStart^min_j and r0 <  XEnd^max_j      X in {LT, UT}
 *   class = FULLY if fully(LT) or fully(UT); else PARTIAL | NEED_X bits if any
 *   partial(X); else UNMASKED.
 *   minmax  in   int32 [B, 8, T_c] as written by flashmask_preprocess
 *   cls     out  uint8 [B, T_r, T_c]
 * The attention kernels evaluate the same predicate on the fly; this entry
 * point exists so the tables can be checked bit for bit.
 */
int flashmask_classify(const int32_t* minmax, int B, int N, int block_r, int block_c,
                       uint8_t* cls, void* hip_stream);

/*
 * The tile scheduler's output for one pass (not in the paper; it is what balances skewed masks over
 * the chip), exported so that it can be checked like the tables above.  It is built here for any size; an
 * attention call builds and follows it where its loop is queued (flashmask_work_cut), the other cuts have
 * no queues.  Work units are row blocks
 * (FM_PASS_FWD, FM_PASS_BWD_DQ) or key blocks (FM_PASS_BWD_DKDV) of the pass's tile shape, numbered
 * (b * H + h) * T + block.  They are dealt to 8 queues; slot s belongs to queue s % 8 and holds the
 * (s / 8)-th unit that queue hands out:
 *   records  out  int32 [slots, 4] = {unit or -1 (no unit), first block of the unit's live range,
 *                 one past its last (0, 0 if every tile of the unit is fully masked), 0}
 *   slots    out  HOST int: number of slots (a multiple of 8, >= B * H * T); with records == NULL
 *                 the call only reports it.
 * Every unit appears exactly once; tiles outside a unit's live range are fully masked (Equation 4).
 * Slices (b, h) go to queues whole, slice b * H + h to queue (b * H + h) % 8, while they fill rounds
 * of 8; the slices left over are shared block by block between 2, 4 or 8 queues.  A queue holds its
 * whole slices in groups of two, one group after the other, then its part of the shared slices;
 * within a group the units holding at least an eighth of the largest possible work come first, by
 * falling work, then the lighter ones by falling octave of work.  workspace as for the pass
 * (FM_PASS_FWD for the forward, FM_PASS_BWD otherwise); the records are copied out of it on the
 * stream.  N here is rounded up to a multiple of 128 (T counts blocks of the padded length); the columns
 * past the end widen no live range (FM_PASS_FWD, FM_PASS_BWD_DQ: keys that both pairs mask for every row;
 * FM_PASS_BWD_DKDV: a ragged last key block has the keys that exist).
 */
int flashmask_unit_queues(int pass, const int32_t* lts, const int32_t* lte, const int32_t* uts, const int32_t* ute,
                          int B, int H, int N, int d, int32_t* records, int* slots,
                          void* workspace, size_t workspace_bytes, void* hip_stream);

/* Tile shape (rows x key columns) at which the given pass classifies and skips tiles where it is queued
 * (flashmask_work_cut), and of flashmask_unit_queues.  Of the other cuts, the halved one works on 64 x 64
 * tiles, and the dQ pass on tiles of 64 keys also at d = 64.  Host-only. */
int flashmask_tile_shape(int pass, int d, int* block_r, int* block_c);

/* How a tile loop's work is cut into workgroups. */
enum {
  FM_CUT_QUEUED = 0, /* units of 128 rows (dK/dV: 128 keys) off the unit queues */
  FM_CUT_DIRECT = 1, /* the same units without queues and their setup launches */
  FM_CUT_HALVED = 2, /* units of 64 rows (keys), their tiles shared by two groups of waves; no queues */
  FM_CUT_PAIRED = 3  /* units of 128 rows, their tiles shared by two groups of waves; no queues */
};
/* The cut that a call of this size takes in the given tile loop (FM_PASS_FWD, FM_PASS_BWD_DQ or
 * FM_PASS_BWD_DKDV) on a GPU of `compute_units` compute units (0: the current device).  Exported, like
 * the queues above, so that tests and benchmarks know what they run.  Host-only. */
int flashmask_work_cut(int pass, int B, int H, int H_kv, int N, int d, int compute_units, int* cut);
/* Launches that build the tables and queues of a forward (FM_PASS_FWD) or a whole backward (FM_PASS_BWD)
 * of this size before its tile loops: 0 where no loop is queued, else 1 or 3.  Host-only. */
int flashmask_setup_launches(int pass, int B, int H, int H_kv, int N, int d, int compute_units, int* launches);

/* Static, human-readable text for an FM_* code. */
const char* flashmask_strerror(int code);

/* Text of the last HIP error behind an FM_ERR_HIP on this thread ("" if none). */
const char* flashmask_last_hip_error(void);

/*
 * Measurement aid (not part of the paper's method): register `count` HOST
 * handles of already-created hipEvent_t objects.  While registered, every
 * flashmask_fwd / flashmask_bwd call records them on its stream between its
 * internal launches, so a benchmark can time one kernel inside the call:
 *   forward : [0] entry, [1] after preprocessing + unit queues, [2] after the tile loop
 *   backward: [0] entry, [1] after preprocessing + unit queues, [2] after the dQ loop (whose
 *             prologue is the D pre-pass), [3] after the dK/dV loop
 * The array must stay valid until cleared with (NULL, 0).  Process-global and
 * not thread-safe; entries that are NULL or beyond `count` are skipped.
 */
int flashmask_profile_events(void** events, int count);

/*
 * Measurement aid (not part of the paper's method): the matrix-core rate this chip reaches on its own.
 * Launches `workgroups` workgroups of 4 waves that do nothing but bf16 matrix-core instructions (the
 * 32x32x16 one the tile loops use, four independent accumulation chains per wave) on the operands given,
 * so a benchmark can time it with events on `hip_stream` and put the tile loops' rate next to what the
 * matrix cores deliver at the clock and power they hold by themselves (Section 5.4 of the paper quotes
 * its kernels against a theoretical peak; this is the measured counterpart).
 *   operands  in   device, 16 KiB of bf16 values, 16-byte aligned.  What they hold matters: the chip's
 *                  sustained clock depends on switching activity (zeros run at the nominal clock, random
 *                  values do not)
 *   sink      out  device, fp32 [workgroups * 256]
 *   iters     in   loop trips; each trip is 32 instruction slots per wave
 *   shape     in   0: the 32x32x16 instruction the tile loops use; 1: the 16x16x32 one (two per slot,
 *                  same floating-point operations), for comparison; 2: shape 0 with, per instruction,
 *                  the side work the forward loop has per matrix instruction (one 128-bit LDS operand
 *                  read, four fp32 multiply-adds, one exponential, all independent): the rate of the
 *                  loop's instruction mix under perfect scheduling
 *   flop      out  HOST double: floating-point operations of the launch
 */
int flashmask_mfma_ceiling(const void* operands, float* sink, int workgroups, int iters, int shape, double* flop,
                           void* hip_stream);

/*
 * Measurement aid (not part of the paper's method): the rate at which this chip takes the dQ update of
 * Algorithm 2 as the paper's column-parallel loop issues it -- every tile of the loop adds a 64 x 128
 * fp32 block into dQ in HBM.  `workgroups` workgroups each add `tiles` such blocks into
 *   acc  in/out  device fp32 [heads][n_tiles][64][128] (zero it first if the sums matter)
 * with no-return fp32 atomic adds, a head's adds all coming from one XCD.  A benchmark times the launch
 * with events; `bytes` (HOST double) receives the bytes of fp32 updates issued.  The backward here
 * computes dQ in a second, row-parallel loop instead, because this rate caps a fused loop far below
 * the matrix-core rate.
 */
int flashmask_atomic_ceiling(float* acc, int heads, int n_tiles, int tiles, int workgroups, double* bytes,
                              void* hip_stream);

/*
 * --- Around the attention call: rotary positions, a paged key-value cache, attention of new tokens over it ---------
 *
 * The conventions at the top of this file hold here too (device pointers, streams, no allocation, no synchronisation,
 * graph capture), with these differences: several element types, sequences of their own lengths, and index values (pages,
 * sequences, positions) that live on the device.  An index value out of its range is never followed: what each entry
 * point does then is said at it.  Sizes beyond the limits that are given here are refused with FM_ERR_SHAPE before anything is launched.
 */

/* Element types. */
enum {
  FM_TYPE_BF16 = 0,
  FM_TYPE_F16 = 1,
  FM_TYPE_F32 = 2,  /* flashmask_rope alone */
  FM_TYPE_E4M3 = 3  /* caches alone: 8 bits, sign, 4 exponent and 3 mantissa bits, largest value 448, no infinities */
};

/* Which elements of a head's first `rot` ones are turned together: i and i + rot / 2, or 2 i and 2 i + 1. */
enum { FM_ROPE_HALF = 0, FM_ROPE_INTERLEAVED = 1 };

/*
 * Rotary positions.  Pair i < rot / 2 of a row at position p is turned by the angle p * freqs[i]:
 *     a' = amp (a cos - b sin),   b' = amp (b cos + a sin),
 * elements from `rot` on are copied.  Scaled frequencies and `amp` are how contexts are stretched.  Angles are products in 64 bits, sines and
 * cosines of them within 1.2e-10 (up to angles of 2^45, where the product itself is off by more), what is multiplied by them in 32, with
 * one rounding to the type at the end.
 *   q, q_out       [B,H,N,d], k, k_out [B,H_kv,N,d], of `type` (BF16, F16, F32); strides[4] describe q, k, q_out, k_out in
 *                  elements (multiples of 16 bytes; see flashmask_strides).  An output may be its own input (same strides).
 *   freqs          double [rot / 2]
 *   positions      int32 [B,N], any values; NULL: 0 .. N - 1 in every batch row
 *   rot            a multiple of 16, 0 < rot <= d; d is 64 or 128
 *   H, H_kv        any, at most 16384 each;  B * N at most 2^27 - 256
 * flashmask_rope_bwd takes the gradients of q_out and k_out to those of q and k: the turn by the opposite angle.
 */
int flashmask_rope(const void* q, const void* k, void* q_out, void* k_out, const double* freqs, const int32_t* positions,
                   int type, int layout, double amp, int B, int H, int H_kv, int N, int d, int rot,
                   const flashmask_strides* strides, void* hip_stream);
int flashmask_rope_bwd(const void* dq_out, const void* dk_out, void* dq, void* dk, const double* freqs,
                       const int32_t* positions, int type, int layout, double amp, int B, int H, int H_kv, int N, int d,
                       int rot, const flashmask_strides* strides, void* hip_stream);

/*
 * A paged key-value cache.  Token j of sequence b lies in page table[b][j / page], slot j % page; the page's entry for
 * head h starts h * head elements further on, the slot's token * row.  Table values outside [0, num_pages) stand for
 * "no page" (-1 by custom).
 */
typedef struct {
  void* k;                  /* pages of `type`, 16-byte aligned; strides in elements, multiples of 16 bytes: .batch from page */
  void* v;                  /* to page, .head from head to head, .row from token to token (>= d, < 2^24); d contiguous */
  flashmask_strides sk, sv;
  const float* k_scale;     /* float [heads], both or neither; a cached value stands for value * scale[head]. */
  const float* v_scale;     /* required for E4M3, NULL otherwise */
  const int32_t* table;     /* int32 [sequences, columns] */
  int32_t type;             /* FM_TYPE_BF16, FM_TYPE_F16 or FM_TYPE_E4M3 */
  int32_t heads, d;         /* K/V heads, at most 16384; 64 or 128 */
  int32_t num_pages, page;  /* pages; tokens of a page, a multiple of 16, at most 2^20 */
  int32_t sequences, columns;  /* columns * page at most 2^30 */
} flashmask_cache;

/*
 * Writes `tokens` new tokens to the cache, their keys rotated (flashmask_rope), and rotates their queries.
 *   q, q_out    [tokens, H, d], k, v [tokens, heads, d] of `type` (BF16, F16; that of the cache, or the cache is E4M3);
 *               strides[4] describe q, k, v, q_out (.row from token to token, .batch unused).  q may be NULL (no queries).
 *   seqs        int32 [tokens]: the token's sequence; outside [0, sequences) it is padding and writes nothing
 *   positions   int32 [tokens]: its position, which is its place in the sequence and its angle.  Where the sequence's row has no
 *               page at that place nothing is written.
 *   freqs, layout, amp, rot   as for flashmask_rope; freqs == NULL: nothing is rotated (q must be NULL)
 * Keys go from the 32-bit result of the rotation to the cache's type in one rounding; an E4M3 cache takes value / scale,
 * held to +-448.  Two tokens of one call must not have the same place.  At most 2^27 tokens and 16384 query heads.
 */
int flashmask_cache_append(const flashmask_cache* cache, const void* q, const void* k, const void* v, void* q_out,
                           const int32_t* seqs, const int32_t* positions, const double* freqs, int type, int layout,
                           double amp, int tokens, int H, int rot, const flashmask_strides* strides, void* hip_stream);

/*
 * Attention of the last T (1 to 256) tokens of every sequence over the cache, which holds lens[b] tokens of it, the new ones among them:
 * query t is row i = lens[b] - T + t and sees key j iff
 *     j <= i,   j > i - window (window > 0),   and neither LTS[j] <= i < LTE[j] nor UTS[j] <= i < UTE[j].
 * out = softmax(scale * q K^T) V and lse as for flashmask_fwd; a row that sees nothing (a sequence shorter than T, an
 * empty one) gets 0 and -inf.  Keys that a row does not see have no influence on it, whatever they and their values hold; an
 * infinite value of a key that it sees makes the element infinite down to a weight of 2^-126 of the largest (below: NaN).
 *   q, out      [sequences, H, T, d] of `type` (BF16, F16; that of the cache, or the cache is E4M3); strides[2] describe q
 *               and out; H is a multiple of cache->heads, query head h reads K/V head h / (H / heads)
 *   lens        int32 [sequences], values below 0 count as 0.  A key whose place has no page is not seen.
 *   lts..ute    int32 [sequences, bound_columns], all or none (NULL); keys from bound_columns on have no interval
 *   window      0: none; else the row and window - 1 keys before it
 *   lse         float [sequences, H, T]
 *   workspace   at least flashmask_decode_workspace_bytes(), 256-byte aligned
 * Long sequences are split over workgroups and joined by a second launch; how follows from lens on the device.  The same
 * call gives the same bits every time.
 * Limits: 65535 sequences, H * T * sequences <= 2^30, sequences * columns * page <= 2^34, and sequences * heads * blocks (of 32 query
 * rows that share a K/V head) below about 2^25.  Where flashmask_decode_workspace_bytes is not 0 its arguments are within them.
 */
int flashmask_decode(const flashmask_cache* cache, const void* q, const int32_t* lens, const int32_t* lts,
                     const int32_t* lte, const int32_t* uts, const int32_t* ute, int bound_columns, int window, float scale,
                     void* out, float* lse, int type, int H, int T, const flashmask_strides* strides, void* workspace,
                     size_t workspace_bytes, void* hip_stream);
/* Bytes of scratch of a call on `sequences` sequences, 0 for an invalid shape.  Host-only. */
size_t flashmask_decode_workspace_bytes(int sequences, int H, int H_kv, int T, int d);

/*
 * Forks sequences: child r goes on from sequence parents[r], sharing its full pages.
 *   table_out   int32 [children, columns]: the parent's row.  A child with a page of its own (new_pages[r] >= 0) keeps the full
 *               pages lens / page; of a last page that is partly filled it gets a copy, in new_pages[r], in every pool.  Without one
 *               (-1) it goes on in the parent's last page.
 *   lens_out    int32 [children]: the parent's length
 *   pools       HOST array of num_pools device pointers, each to num_pages pages of page_bytes contiguous bytes (a
 *               multiple of 16): all layers' keys and values
 * A parent outside [0, sequences) gives an empty child; no page is copied from or to a place outside the pools.  The pages of
 * new_pages must differ from each other and from those in use; table_out, lens_out must not overlap table, lens.  At most 65535 children,
 * page_bytes at most 2^30.  Where a child gets a page of its own and its parent has none there, the page keeps what it holds.
 */
int flashmask_cache_fork(void* const* pools, int num_pools, size_t page_bytes, int num_pages, const int32_t* table,
                         const int32_t* lens, const int32_t* parents, const int32_t* new_pages, int32_t* table_out,
                         int32_t* lens_out, int sequences, int columns, int page, int children, void* hip_stream);

/*
 * The pages that no entry of the table names, in ascending order, -1 behind them, and their number.
 *   free_pages  int32 [num_pages], count int32 [1];  workspace: flashmask_cache_plan_bytes(num_pages), 256-byte aligned
 *   entries, num_pages   at most 2^30 each, here and below
 */
int flashmask_cache_free_list(const int32_t* table, int entries, int num_pages, int32_t* free_pages, int32_t* count,
                              void* workspace, size_t workspace_bytes, void* hip_stream);
/*
 * Moves the used pages to the front: with `used` pages named by the table, the used pages from there on go, in ascending
 * order, to the unused ones before it, in every pool; the table's entries follow.
 *   table_out   int32 [entries] (values outside [0, num_pages) stay as they are), used int32 [1]; neither overlaps table
 */
int flashmask_cache_compact(void* const* pools, int num_pools, size_t page_bytes, int num_pages, const int32_t* table,
                            int entries, int32_t* table_out, int32_t* used, void* workspace, size_t workspace_bytes,
                            void* hip_stream);
/* Bytes of scratch of the two calls above, 0 for an invalid number.  Host-only. */
size_t flashmask_cache_plan_bytes(int num_pages);

#ifdef __cplusplus
}
#endif
#endif /* FLASHMASK_H */
