/*
 * wise.h — C ABI of libwise, the gfx950 (MI355X) hot path of WISE
 * (Working-set Inference with Support Exploitation) for recurrent-depth
 * language models.
 *
 * The method (paper, Section 5): during the first t_d recurrent steps run
 * full causal attention and pool its probabilities into per
 * (query-block, key-block) masses (Section 5.1, eq. "block_attention_mass");
 * pick, per query block, the smallest set of key blocks whose pooled mass
 * reaches a threshold (Section 5.1, eq. "block_working_set"); for every later
 * step restrict attention to that fixed block support while Q/K/V are
 * recomputed (Section 5.2, eq. "wise_attention").  The support is kept as a
 * device-resident CSR schedule (Appendix B, "Sparse-kernel implementation").
 *
 * Conventions shared by every call
 * --------------------------------
 *  - Every tensor argument is a DEVICE pointer owned by the caller,
 *    contiguous, row-major.  The library allocates nothing: scratch space
 *    comes in as caller-owned workspaces sized by the *_workspace_bytes
 *    queries, except for wise_select_support_noalloc, which uses a fixed
 *    device array of its own (WISE_NOALLOC_SCRATCH_BYTES per GPU).
 *  - bf16 tensors are raw IEEE bfloat16 storage (uint16, round-to-nearest-even
 *    when produced by the library).
 *  - Shapes: q, o are [batch][heads][seq_len][head_dim]; k, v are
 *    [batch][kv_heads][seq_len][head_dim] (kv_heads = heads without
 *    grouped-query attention); lse is [batch][heads][seq_len]; acc is
 *    [batch][heads][nb][nb] with nb = seq_len / block.  CSR row
 *    r = (b * heads + h) * nb + qb: masses, supports and rows stay per query
 *    head, and query head h reads key-value head h / (heads / kv_heads).
 *  - Every call validates its arguments on the host BEFORE touching the
 *    device and returns a status; on any error nothing is launched and no
 *    output is written.  On success the work is only enqueued on
 *    `hip_stream` (a hipStream_t, NULL = default stream) and the call
 *    returns; device-side faults surface at the caller's next
 *    synchronisation.  WISE_ERR_HIP carries a failed launch.
 *  - Calls are stateless and re-entrant; calls on different streams with
 *    disjoint outputs may run concurrently.  No C++ exception crosses the ABI.
 *  - A successful call enqueues kernels only: no allocation, memset, copy or
 *    synchronisation, so calls may be captured in a HIP graph (the graph
 *    then reads whatever the captured buffers hold at replay time).
 *  - Supported: head_dim in {64, 96, 128}; block in {16, 32, 64, 128} (the
 *    block sizes of the paper's block-size sweep, Appendix "Block-Size
 *    Tradeoff"); seq_len % block == 0, and seq_len % 64 == 0 for blocks 16
 *    and 32 (the dense kernel's key tiles); nb <= 1024 for wise_select_support,
 *    wise_select_step and wise_support_from_masks.
 *  - Support bitmasks (the union mode and the diagnostics): uint64
 *    [rows][words], words = wise_mask_words(s) = ceil(nb / 64); bit
 *    (kb & 63) of word kb >> 6 of row r is set iff key block kb belongs to
 *    that row's set.  Several masks "back to back" means mask i starts at
 *    element i * rows * words.
 *  - Alignment: q, k, v, o and pools 16 bytes; workspace 256 bytes; masks, the
 *    counts of wise_mask_overlap and fp64 arrays 8 bytes; every other pointer 4 bytes.  A misaligned
 *    pointer is WISE_ERR_SHAPE.
 */
#ifndef WISE_H
#define WISE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define WISE_ABI_VERSION 6

typedef enum {
  WISE_OK = 0,
  WISE_ERR_NULL = 1,        /* a required pointer is NULL                    */
  WISE_ERR_SHAPE = 2,       /* non-positive dimension, seq_len % block != 0
                               (% 64 for blocks 16, 32), heads % kv_heads != 0,
                               a size that overflows int32 indexing, or a
                               misaligned pointer                            */
  WISE_ERR_UNSUPPORTED = 3, /* head_dim or block outside the supported set   */
  WISE_ERR_RANGE = 4,       /* tau outside (0, 1] / NaN, non-finite scale,
                               or unknown flag bit                           */
  WISE_ERR_WORKSPACE = 5,   /* workspace smaller than the size query returns */
  WISE_ERR_HIP = 6          /* a HIP launch reported an error                */
} wise_status;

/* Problem geometry shared by all calls.  scale <= 0 selects 1/sqrt(head_dim),
 * the softmax temperature of the paper's attention (Section 3, eq.
 * "recurrent_attention").  kv_heads: key-value heads for grouped-query
 * attention (the paper's second backbone shares 8 key-value heads among 32
 * query heads, Appendix B); 0 means kv_heads = heads; heads must be a
 * multiple of it. */
typedef struct {
  int32_t batch;
  int32_t heads;
  int32_t seq_len;
  int32_t head_dim;
  int32_t block;
  float scale;
  int32_t kv_heads;
} wise_shape;

/* Selection flags: blocks forced into every support after the cumulative-mass
 * cut.  The paper's own selection is flags = 0; the default used by this
 * library's callers is WISE_FORCE_SINK | WISE_FORCE_DIAG. */
enum {
  WISE_FORCE_SINK = 1u, /* key block 0 (the attention-sink block)     */
  WISE_FORCE_DIAG = 2u  /* key block qb (the causal diagonal block)   */
};

/*
 * wise_dense_attn_accum — full causal attention of one recurrent step,
 * optionally pooling its probabilities into block masses.
 *
 *   O = softmax(Q K^T * scale + M) V,  M the causal mask (key j <= query i)
 *       (Section 3, eq. "recurrent_attention")
 *   lse_i = log sum_{j<=i} exp(scale * q_i . k_j)      (natural log)
 *   if acc != NULL, for every kb <= qb:
 *     acc[b][h][qb][kb] += (1/block) * sum_{i in I_qb} sum_{j in I_kb, j<=i} A_ij
 *       (Section 5.1, eq. "block_attention_mass"); entries kb > qb untouched.
 *
 *   q       : bf16 [batch][heads][seq_len][head_dim], read-only.
 *   k, v    : bf16 [batch][kv_heads][seq_len][head_dim], read-only.
 *   o       : bf16, same shape as q, written.
 *   lse     : fp32 [batch][heads][seq_len] or NULL.
 *   acc     : fp32 [batch][heads][nb][nb] or NULL (plain dense attention).
 *             Read-modify-written in the same pass as the attention: the
 *             caller zeroes it before the first step it should sum.  Each
 *             acc row is owned by one work-group: no float atomics, bitwise
 *             deterministic.
 *   workspace, workspace_bytes : device scratch, 256-byte aligned, used
 *             only when acc != NULL (then required); contents on entry are
 *             ignored.  wise_mass_workspace_bytes(s) bytes let one launch
 *             cover every head; any smaller size down to
 *             wise_mass_workspace_min_bytes(s) (one key-value group of
 *             heads) runs the heads in consecutive launches of as many
 *             whole groups as fit, with the same results bit for bit.  It holds one fp32 per (query, 64-key span, or
 *             block-sized span for blocks 16 and 32, up to the query's tile)
 *             between the attention and its epilogue.
 * Errors: WISE_ERR_NULL (q, k, v, o NULL, or acc set with workspace NULL),
 *         WISE_ERR_SHAPE, WISE_ERR_UNSUPPORTED, WISE_ERR_WORKSPACE, WISE_ERR_HIP.
 */
wise_status wise_dense_attn_accum(const wise_shape* s, const void* q,
                                  const void* k, const void* v, void* o,
                                  float* lse, float* acc, void* workspace,
                                  size_t workspace_bytes, void* hip_stream);

/*
 * wise_select_support — per query block, the smallest set of key blocks whose
 * accumulated mass reaches tau of the row total (Section 5.1, eq.
 * "block_working_set", the arg-min over admissible blocks), plus the blocks
 * named in `flags`, emitted as CSR.
 *
 * Per row (b, h, qb), with v_kb = acc[b][h][qb][kb] for kb = 0..qb:
 *   1. order the candidates by (v descending, kb ascending);
 *   2. c_k = sum of the first k ordered masses, summed in that order in
 *      fp64 (c_0 = 0), total = c_{qb+1};
 *   3. k* = min{ k >= 0 : c_k >= tau * total }   (fp64);
 *   4. S = first k* ordered blocks  U  {0 if SINK}  U  {qb if DIAG};
 *      S empty (total == 0 and flags == 0) -> S = {qb};
 *   5. col_idx[row_ptr[r] .. row_ptr[r+1]) = S in ascending order.
 *
 *   acc       : fp32 [batch][heads][nb][nb], read-only (entries kb > qb ignored).
 *   tau       : 0 < tau <= 1.
 *   flags     : OR of WISE_FORCE_* bits.
 *   row_ptr   : int32 [rows + 1], rows = batch*heads*nb; row_ptr[0] = 0,
 *               row_ptr[rows] = nnz.
 *   col_idx   : int32 [wise_support_capacity(s)]; the first nnz are written.
 *   row_order : int32 [rows] or NULL: the schedule for wise_sparse_attn
 *               (Appendix B, "execution-metadata preparation"): rows grouped
 *               by (batch, head) in ascending order, and within a head by
 *               support size descending, ties by row id ascending.
 *   workspace : device scratch of at least wise_select_workspace_bytes(s)
 *               bytes; contents on entry are ignored.
 * Errors: WISE_ERR_NULL, WISE_ERR_SHAPE, WISE_ERR_UNSUPPORTED, WISE_ERR_RANGE,
 *         WISE_ERR_WORKSPACE, WISE_ERR_HIP.
 */
wise_status wise_select_support(const wise_shape* s, const float* acc,
                                float tau, uint32_t flags, int32_t* row_ptr,
                                int32_t* col_idx, int32_t* row_order,
                                void* workspace, size_t workspace_bytes,
                                void* hip_stream);

/* Bytes of the library's own per-device selection scratch (see
 * wise_select_support_noalloc). */
#define WISE_NOALLOC_SCRATCH_BYTES ((size_t)4 << 20)

/*
 * wise_select_support_noalloc — wise_select_support without a caller
 * workspace, for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc).
 *
 * Same selection, CSR, row order, arguments and errors as
 * wise_select_support, minus the workspace.  The per-row counts and
 * bitmasks live instead in a device array of WISE_NOALLOC_SCRATCH_BYTES
 * inside the library: every GPU the library runs on holds its own copy
 * until the process ends, and its address is looked up on the first call on
 * each device (the current device at the call).  The call performs no
 * allocation, free, memset or copy: it only enqueues the selection kernels.
 * Every row's scratch entries are written before they are read, so the
 * array's contents from earlier calls do not matter; but all calls on one
 * GPU share the array, so calls that overlap on one GPU (different streams
 * without ordering, different host threads) race and must not be issued.
 * Limit: wise_select_workspace_bytes(s) <= WISE_NOALLOC_SCRATCH_BYTES
 * (4 MiB: e.g. 28,160 rows of 128 blocks need 0.56 MiB), else
 * WISE_ERR_WORKSPACE and nothing is launched.
 * Errors: WISE_ERR_NULL, WISE_ERR_SHAPE, WISE_ERR_UNSUPPORTED, WISE_ERR_RANGE,
 *         WISE_ERR_WORKSPACE, WISE_ERR_HIP (also a failed address lookup).
 */
wise_status wise_select_support_noalloc(const wise_shape* s, const float* acc,
                                        float tau, uint32_t flags,
                                        int32_t* row_ptr, int32_t* col_idx,
                                        int32_t* row_order, void* hip_stream);

/*
 * wise_sparse_attn — attention of one late recurrent step restricted to a
 * block support (Section 5.2, eq. "wise_attention"):
 *   O = softmax(Q K^T * scale + M + R) V,  R_ij = 0 if kb(j) in S_{qb(i)},
 *   -inf otherwise.  Q/K/V are this step's; only the support is reused.
 *
 *   q         : bf16 [batch][heads][seq_len][head_dim], read-only.
 *   k, v      : bf16 [batch][kv_heads][seq_len][head_dim], read-only.
 *   row_ptr   : int32 [rows + 1], col_idx : int32 [nnz] — a CSR whose rows
 *               list key-block ids in strictly ascending order with every id
 *               <= qb (as written by wise_select_support).  Ids outside
 *               0..qb are skipped on the device (never read out of bounds);
 *               ordering and uniqueness are trusted, not re-checked.
 *   row_order : int32 [rows], a permutation of 0..rows-1, or NULL for the
 *               identity.  Schedule slot s runs row row_order[s].  The slots of
 *               a head (s / nb) run on as few of the 8 XCDs as even shares
 *               allow, earlier ones first, so rows of one head placed together
 *               share an L2.
 *   o         : bf16, same shape as q, written.  A row with an empty support
 *               writes zeros (and lse = -inf).
 *   lse       : fp32 [batch][heads][seq_len] or NULL.
 * Errors: WISE_ERR_NULL, WISE_ERR_SHAPE, WISE_ERR_UNSUPPORTED, WISE_ERR_HIP.
 */
wise_status wise_sparse_attn(const wise_shape* s, const void* q, const void* k,
                             const void* v, const int32_t* row_ptr,
                             const int32_t* col_idx, const int32_t* row_order,
                             void* o, float* lse, void* hip_stream);

/*
 * wise_sparse_attn_grouped — the same late step (Section 5.2, eq.
 * "wise_attention"), bit for bit the same outputs as wise_sparse_attn, run
 * by work-groups of wise_sparse_group_rows(s) consecutive query blocks of a
 * head (block 64: 4 at head_dim 128, 2 otherwise; block 128: 2 at head_dim
 * 128) over the union of their supports: each staged key tile serves all of
 * the group's rows that hold it, and every row attends only its own blocks.
 * Faster than wise_sparse_attn when consecutive rows' supports nearly
 * coincide and there are groups enough for every CU (dense supports: measured
 * 5% at density 0.90 with 4 rows of 64 keys, 4 to 8% above 0.92 with 2 rows at
 * head_dim 64), slower when they differ (35% slower at density 0.43 with 4
 * rows) and for 128-key blocks; the caller picks, e.g. by the support's
 * density against the break-even of the group shape.  Where grouping is unavailable (block 16
 * or 32, block 128 below head_dim 128, more than 1024 key blocks, or
 * seq_len not a multiple of the group's queries: 256 at head_dim 128, else
 * 128; wise_sparse_group_rows(s) == 0) the call runs wise_sparse_attn's
 * kernel.  Arguments as wise_sparse_attn, without
 * row_order (groups are issued heaviest first, per head).
 * Errors: WISE_ERR_NULL, WISE_ERR_SHAPE, WISE_ERR_UNSUPPORTED, WISE_ERR_HIP.
 */
wise_status wise_sparse_attn_grouped(const wise_shape* s, const void* q,
                                     const void* k, const void* v,
                                     const int32_t* row_ptr,
                                     const int32_t* col_idx, void* o,
                                     float* lse, void* hip_stream);

/* Query blocks per work-group of wise_sparse_attn_grouped: 4 or 2, or 0
 * where it runs wise_sparse_attn's kernel (-1 for an invalid shape). */
int32_t wise_sparse_group_rows(const wise_shape* s);

/*
 * wise_select_step — one discovery step's own support B_q^(t, eta), the set
 * that the paper's temporal union collects (Section 5.1, eq.
 * "block_working_set"), as a bitmask.
 *
 * Per row, steps 1-4 of wise_select_support on that step's masses with no
 * forced blocks (flags = 0): the heaviest k* blocks, k* the first prefix of
 * the (mass desc, block asc) order whose fp64 sum reaches tau of the row
 * total; an empty set (row total 0) becomes {qb}.
 *
 *   r     : fp32 [batch][heads][nb][nb], read-only: ONE step's block masses
 *           (wise_dense_attn_accum pooling into a zeroed buffer gives them).
 *   tau   : 0 < tau <= 1.
 *   mask  : uint64 [rows][words], every word written.
 * Errors: WISE_ERR_NULL, WISE_ERR_SHAPE, WISE_ERR_UNSUPPORTED, WISE_ERR_RANGE,
 *         WISE_ERR_HIP.
 */
wise_status wise_select_step(const wise_shape* s, const float* r, float tau,
                             uint64_t* mask, void* hip_stream);

/*
 * wise_support_from_masks — the paper's working set of Section 5.1, eq.
 * "block_working_set": per row, the union of n_masks per-step sets (masks
 * back to back, e.g. the window steps t_d-3..t_d from wise_select_step),
 * plus the blocks named in `flags`, emitted as CSR and row order exactly as
 * wise_select_support emits them.  Bits of key blocks past the diagonal are
 * ignored; an empty union with flags = 0 becomes {qb}.
 *
 *   masks     : uint64 [n_masks][rows][words], read-only.  n_masks >= 1.
 *   flags, row_ptr, col_idx, row_order, workspace, workspace_bytes: as for
 *               wise_select_support (same workspace size).
 * Errors: WISE_ERR_NULL, WISE_ERR_SHAPE (also n_masks < 1),
 *         WISE_ERR_UNSUPPORTED, WISE_ERR_RANGE, WISE_ERR_WORKSPACE, WISE_ERR_HIP.
 */
wise_status wise_support_from_masks(const wise_shape* s, const uint64_t* masks,
                                    int32_t n_masks, uint32_t flags,
                                    int32_t* row_ptr, int32_t* col_idx,
                                    int32_t* row_order, void* workspace,
                                    size_t workspace_bytes, void* hip_stream);

/*
 * wise_mask_union — out = bitwise OR of n_masks masks stored back to back:
 * the rolling working set W_q^(t) of Appendix C ("Stability of the Deployed
 * Working Set") when the masks are the per-step sets of steps
 * max(1, t-3)..t.
 *
 *   masks : uint64 [n_masks][rows][words], read-only.  n_masks >= 1.
 *   out   : uint64 [rows][words], written; it may coincide with one of the
 *           masks (each word is read before it is written), any other
 *           overlap is undefined.
 * Errors: WISE_ERR_NULL, WISE_ERR_SHAPE (also n_masks < 1), WISE_ERR_HIP.
 */
wise_status wise_mask_union(const wise_shape* s, const uint64_t* masks,
                            int32_t n_masks, uint64_t* out, void* hip_stream);

/*
 * wise_mask_overlap — sizes of the intersection and union of two masks read
 * as sets of (row, key block): counts[0] = |A & B|, counts[1] = |A | B|.
 * Their ratio is the adjacent rolling-set Jaccard J_roll of Appendix C
 * ("Stability of the Deployed Working Set") for A = W^(t-1), B = W^(t).
 *
 *   a, b   : uint64 [rows][words], read-only.
 *   counts : int64 [2], device, written.
 * Errors: WISE_ERR_NULL, WISE_ERR_SHAPE, WISE_ERR_HIP.
 */
wise_status wise_mask_overlap(const wise_shape* s, const uint64_t* a,
                              const uint64_t* b, int64_t* counts,
                              void* hip_stream);

/*
 * wise_support_mass — attention mass a block support retains from one step
 * of unrestricted attention: the retained future full-attention mass of
 * Section 7.1 and Appendix B (evaluation metrics), computed from that step's
 * block masses r (eq. "block_attention_mass").  Since each query's
 * probabilities sum to 1, sum_rows inside / sum_rows total is the fraction
 * of all causal attention mass that falls inside the support.
 *
 *   r        : fp32 [batch][heads][nb][nb], read-only: one step's masses.
 *   row_ptr, col_idx : a CSR support as for wise_sparse_attn (ids outside
 *              0..qb are skipped).
 *   row_mass : fp64 [rows][2], written: (sum of r[row][kb] over the row's
 *              blocks, sum of r[row][kb] over kb <= qb), each summed in fp64
 *              in a fixed order (bitwise reproducible).
 *   totals   : fp64 [2] or NULL, written: the two columns of row_mass summed
 *              over all rows, in a fixed order.
 * Errors: WISE_ERR_NULL, WISE_ERR_SHAPE, WISE_ERR_HIP.
 */
wise_status wise_support_mass(const wise_shape* s, const float* r,
                              const int32_t* row_ptr, const int32_t* col_idx,
                              double* row_mass, double* totals,
                              void* hip_stream);

/* Bytes of device workspace wise_dense_attn_accum needs when it pools block
 * masses: one fp32 per (query, E-key span up to the end of its tile of T
 * queries), E = block for blocks 16 and 32 and 64 otherwise, T = 256 for head_dim 128
 * when it divides seq_len, else 128 when it divides seq_len, else 64:
 * batch * heads * T * (T / E) * m (m + 1) / 2 * 4 with m = seq_len / T
 * (about half of seq_len^2 / E floats per head; 0 for an invalid shape). */
size_t wise_mass_workspace_bytes(const wise_shape* s);

/* The smallest workspace wise_dense_attn_accum accepts with acc != NULL:
 * wise_mass_workspace_bytes(s) / (batch * heads) * (heads / kv_heads), the
 * share of one key-value group of query heads (0 for an invalid shape). */
size_t wise_mass_workspace_min_bytes(const wise_shape* s);

/* 64-bit words per row of a support bitmask: ceil(nb / 64)
 * (-1 for an invalid shape). */
int32_t wise_mask_words(const wise_shape* s);

/* Bytes of device workspace wise_select_support needs for shape s
 * (0 for an invalid shape). */
size_t wise_select_workspace_bytes(const wise_shape* s);

/* Upper bound on nnz: batch * heads * nb * (nb + 1) / 2, the number of
 * causally admissible block pairs (-1 for an invalid shape). */
int64_t wise_support_capacity(const wise_shape* s);

/*
 * The paged key-value cache
 * -------------------------
 * What follows a prompt: single tokens (or a few drafted ones) whose
 * keys and values are kept.  They live in pages of a pool,
 *
 *   pool   : bf16 [planes][pages][kv_heads][page][head_dim].  Plane 2 l holds
 *            the keys and plane 2 l + 1 the values of layer l by convention;
 *            the calls that move pages move them in every plane.
 *   tables : int32 [seqs][max_pages], the page of tokens page*j .. page*j +
 *            page - 1 of a sequence in column j, -1 in columns past its last.
 *   lens   : int32 [seqs], tokens of a sequence (0: empty).
 *   refs   : int32 [pages], how many table entries name the page (free: <= 0).
 *
 * all on the device and owned by the caller, who starts with tables -1 and
 * lens and refs 0.  Sequences share a page by naming it; whoever is to write
 * into a shared page gets a copy first (wise_cache_reserve).  Ids of
 * sequences come in device arrays of n <= 1024 entries (n = 0 does nothing),
 * what each entry got goes to device arrays, and no call waits for the
 * device: a step of a serving loop (trim, fork, reserve, append, attend)
 * can be captured in one HIP graph.  Calls that share tables, lens, refs, pool or
 * a workspace must be ordered, by one stream or by events.  An entry whose
 * id lies outside 0..seqs-1 does nothing, and so does one whose id an earlier
 * entry of the same call already names (in wise_cache_append and
 * wise_prefix_attn an id may repeat, see there).  Page ids
 * outside 0..pages-1 are never followed.
 */
typedef struct {
  int32_t pages;     /* pages of the pool                                    */
  int32_t page;      /* tokens of a page: 16, 32, 64 or 128                  */
  int32_t kv_heads;
  int32_t head_dim;  /* 64, 96 or 128                                        */
  int32_t planes;    /* planes of the pool: 2 x layers                       */
  int32_t seqs;      /* rows of tables and lens                              */
  int32_t max_pages; /* columns of tables; max_pages * page <= 2^30          */
} wise_cache;

/*
 * wise_cache_fork — sequence dst[i] becomes a copy of src[i]: it names the
 * same pages (refs + 1 each) and has the same length.  No keys or values move.
 *
 * Every entry reads the state before the call.  It is refused, and leaves
 * everything as it is, when dst[i] is not empty, when src[i] is also a
 * destination of the call, or by the rules above (an earlier entry with the
 * same dst wins; a source may be named any number of times).
 *
 *   src, dst : int32 [n], device, read-only.
 *   done     : int32 [n] or NULL, written: 1, or 0 for a refused entry.
 * Errors: WISE_ERR_NULL, WISE_ERR_SHAPE (also n < 0), WISE_ERR_UNSUPPORTED
 *         (also n > 1024), WISE_ERR_HIP.
 */
wise_status wise_cache_fork(const wise_cache* c, int32_t n, const int32_t* src,
                            const int32_t* dst, int32_t* tables, int32_t* lens,
                            int32_t* refs, int32_t* done, void* hip_stream);

/*
 * wise_cache_trim — drops the tokens of sequence seq_ids[i] from new_lens[i]
 * on (drafts that were not accepted, a finished request): its length becomes
 * min(length, max(new_lens[i], 0)), pages wholly past it lose a reference, their
 * table entries become -1.
 *
 *   seq_ids  : int32 [n], device, read-only.
 *   new_lens : int32 [n], device, read-only, or NULL: 0 for every entry (the
 *              sequences are freed).
 * Errors: as wise_cache_fork.
 */
wise_status wise_cache_trim(const wise_cache* c, int32_t n,
                            const int32_t* seq_ids, const int32_t* new_lens,
                            int32_t* tables, int32_t* lens, int32_t* refs,
                            void* hip_stream);

/*
 * wise_cache_reserve — makes sequence seq_ids[i] counts[i] tokens longer and
 * gives it the pages that these need, so that wise_cache_append can write
 * them.  A last page that is partly filled and that other table entries name
 * too (refs > 1 before the call) is first replaced by a copy of its own: the
 * tokens it holds, in every plane.
 *
 * Pages are handed out in ascending order of id, to the entries in order and to each
 * in ascending order of its columns.  An entry is refused (granted 0,
 * nothing changed) by the rules above, when counts[i] <= 0, when the sequence would
 * outgrow max_pages * page tokens, or when it needs pages and
 * these and those that the entries before it need (but for entries refused for the
 * other reasons) are more than were free before the call.  Pages
 * that lose their last reference here are free from the next call on.
 *
 *   seq_ids, counts : int32 [n], device, read-only.
 *   granted   : int32 [n], written: counts[i], or 0 for a refused entry.
 *   pool      : all planes.
 *   workspace : device scratch of wise_cache_workspace_bytes(c) bytes, 256-byte
 *               aligned; contents on entry are ignored.
 * Errors: as wise_cache_fork, and WISE_ERR_WORKSPACE.
 */
wise_status wise_cache_reserve(const wise_cache* c, int32_t n,
                               const int32_t* seq_ids, const int32_t* counts,
                               int32_t* tables, int32_t* lens, int32_t* refs,
                               int32_t* granted, void* pool, void* workspace,
                               size_t workspace_bytes, void* hip_stream);

/*
 * wise_cache_append — writes the newest counts[i] tokens of sequence
 * seq_ids[i] (positions lens - counts[i] .. lens - 1, after wise_cache_reserve)
 * in one layer.  Tokens that fall on positions below 0, or on columns without
 * a page, are skipped.  Every id should occur once: an id that repeats
 * has its tokens written by each entry, in no order.
 *
 *   tokens  : token rows of k and v per entry, 1 or more.
 *   seq_ids : int32 [n], counts : int32 [n], device, read-only; counts[i] is
 *             taken as min(max(counts[i], 0), tokens).  wise_cache_reserve's
 *             `granted` is what to pass.
 *   k, v    : bf16 [n][kv_heads][tokens][head_dim], read-only; rows from
 *             counts[i] on are not read.
 *   k_pool, v_pool : the layer's two planes, [pages][kv_heads][page][head_dim].
 * Errors: as wise_cache_fork (WISE_ERR_SHAPE also for tokens < 1 and for
 *         n * kv_heads * tokens > 2^28 - 16).
 */
wise_status wise_cache_append(const wise_cache* c, int32_t n, int32_t tokens,
                              const int32_t* seq_ids, const int32_t* counts,
                              const void* k, const void* v,
                              const int32_t* tables, const int32_t* lens,
                              void* k_pool, void* v_pool, void* hip_stream);

/*
 * wise_cache_compact — moves the pages in use to the front of the pool: with
 * L of them, the k-th one of id >= L (ascending) moves to the k-th free page
 * of id < L, in every plane, and takes its references along; table entries
 * follow.  Afterwards pages 0..L-1 are in use and the others free.
 *
 *   live      : int32 [1] or NULL, device, written: L.
 *   workspace : as for wise_cache_reserve.
 * Errors: as wise_cache_reserve.
 */
wise_status wise_cache_compact(const wise_cache* c, int32_t* tables,
                               int32_t* refs, void* pool, int32_t* live,
                               void* workspace, size_t workspace_bytes,
                               void* hip_stream);

/*
 * wise_cache_shared — what neighbours of a batch have in common: shared[b] is
 * the number of leading pages that sequence b and sequence b - 1 both name and
 * both fill, or 0 if that is less than min_pages; shared[0] = 0.  The argument of
 * wise_prefix_attn.
 *
 *   batch   : 1 .. 1024 sequences, in the order of the attention call.
 *   seq_ids : int32 [batch], device, read-only, or NULL: sequence b is table row b.
 * Errors: as wise_cache_fork (WISE_ERR_SHAPE also for batch > seqs without
 *         seq_ids).
 */
wise_status wise_cache_shared(const wise_cache* c, int32_t batch,
                              int32_t min_pages, const int32_t* seq_ids,
                              const int32_t* tables, const int32_t* lens,
                              int32_t* shared, void* hip_stream);

/* Bytes of device workspace wise_cache_reserve and wise_cache_compact need
 * (0 for an invalid cache). */
size_t wise_cache_workspace_bytes(const wise_cache* c);

/* The newest q_len tokens of `batch` sequences.  heads must be a multiple of
 * the cache's kv_heads (query head h reads key-value head h / (heads /
 * kv_heads)), heads / kv_heads * q_len <= 128, batch <= 1024.  scale <= 0
 * selects 1/sqrt(head_dim). */
typedef struct {
  int32_t batch;
  int32_t heads;
  int32_t q_len;
  float scale;
} wise_queries;

/*
 * wise_prefix_attn — attention of the newest q_len tokens of every sequence
 * of a batch over its pages (Section 3, eq. "recurrent_attention", with keys
 * and values of the earlier positions kept): token t of sequence b sits at
 * position i = lens - q_len + t and attends the positions j <= i.
 *
 * Runs of sequences that begin with the same pages have these read once for
 * all: shared[b] is the number of leading pages that sequence b shares
 * with sequence b - 1 (wise_cache_shared counts them).  shared[b] <= 0 starts a
 * run, and what a run reads once is the least shared[b] of its other sequences, at
 * most the whole pages that all queries of the run see, in whole tiles of 64
 * tokens, through the table of its first sequence.  Where neighbours share unlike
 * numbers of pages (several prompts with a common header, a short request among
 * users of a long prompt), runs are cut so that fewer keys are read in all.  shared
 * changes which pages are read together, and the last bits, not what is computed.
 *
 *   q         : bf16 [batch][heads][q_len][head_dim], read-only.
 *   k_pool, v_pool : the layer's two planes, read-only.
 *   tables, lens : read-only.  A length is taken as at most max_pages * page.
 *               Positions from a sequence's length on, and positions on a page id outside
 *               0..pages-1, are not attended, whatever the pool holds there.
 *   seq_ids   : int32 [batch], device, or NULL: sequence b is table row b.  An
 *               id may repeat; one outside 0..seqs-1 is an empty sequence.
 *   shared    : int32 [batch], device, or NULL: nothing is shared.
 *   o         : bf16 [batch][heads][q_len][head_dim], written.  A row that sees
 *               no position is zero (and its lse -inf).
 *               An infinite value is what its dim of a row that sees it gets, whatever its
 *               weight (NaN beside NaN or the other infinity), and no other row or dim.
 *   lse       : fp32 [batch][heads][q_len] or NULL: natural log of the sum.
 *   workspace : device scratch of wise_prefix_workspace_bytes(c, a) bytes, 256-byte
 *               aligned; contents on entry are ignored.
 * Bitwise deterministic: the sums of a row run in an order that lens and shared
 * fix.
 * Errors: WISE_ERR_NULL, WISE_ERR_SHAPE, WISE_ERR_UNSUPPORTED, WISE_ERR_RANGE
 *         (scale), WISE_ERR_WORKSPACE, WISE_ERR_HIP.
 */
wise_status wise_prefix_attn(const wise_cache* c, const wise_queries* a,
                             const void* q, const void* k_pool,
                             const void* v_pool, const int32_t* tables,
                             const int32_t* lens, const int32_t* seq_ids,
                             const int32_t* shared, void* o, float* lse,
                             void* workspace, size_t workspace_bytes,
                             void* hip_stream);

/* Bytes of device workspace wise_prefix_attn needs (0 for invalid
 * arguments). */
size_t wise_prefix_workspace_bytes(const wise_cache* c, const wise_queries* a);

/* Static, NUL-terminated description of a status code. */
const char* wise_status_string(wise_status st);

/* WISE_ABI_VERSION of the loaded library. */
int32_t wise_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* WISE_H */
