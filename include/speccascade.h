/*
 * speccascade.h -- C interface of libspeccascade, the verify/defer step of
 * speculative cascades on AMD Instinct MI355X (gfx950).
 *
 * One call performs, for a block of gamma drafted positions in each of B
 * sequences, the verification half of GenSpecSample (Alg. 4) with the
 * cascade target T_delta (eq. (6), Alg. 5) of "Faster Cascades via
 * Speculative Decoding" (Narasimhan et al., arXiv 2405.19261):
 *
 *   q_{t+j} = softmax(z^q_{t+j} / T),  p_{t+j} = softmax(z^p_{t+j} / T)   (j = 0..gamma)
 *   delta_j  by the deferral rule of Table 1 (Chow eq. (2), Diff eq. (5),
 *            OPT eq. (11) with D_TV of Lemma 3)
 *   pi_j     = (1 - delta_j) q_j + delta_j p_j                            (eq. (6))
 *   a_j      = 1(u_j < min(1, pi_j(x_j) / q_j(x_j))), j < gamma; a_gamma = 0
 *   j*       = min{ j : a_j = 0 }
 *   token    ~ norm(max(0, pi_{j*} - q_{j*}))  if j* < gamma,  else ~ pi_gamma
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Pointers are DEVICE pointers on the current HIP device, allocated and
 *   owned by the caller.  The library reads inputs, writes outputs, and keeps
 *   no reference to either after the call returns.
 * - Work is enqueued on `stream` (NULL = the default stream) and is
 *   asynchronous: outputs are valid once the caller synchronises the stream.
 *   No call synchronises the host with the device.
 * - Logit tensors are row-major [B][gamma+1][V] (row stride V elements), in
 *   float32 or bfloat16.  Row gamma of the drafter tensor is the drafter's
 *   distribution at the bonus position t+gamma, which the extra-token target
 *   pi_{t+gamma} of Alg. 4 needs.
 * - Every argument is checked before any HIP call; a failed check returns
 *   its status and enqueues nothing.  spc_last_error() then describes it.
 * - Preconditions that are NOT checked: logits are finite or -inf, with at
 *   least one finite entry per row; uniforms lie in [0, 1).
 * - Defined behaviour: a draft token outside [0, V) rejects its position
 *   (no out-of-bounds read).  out_defer_mask is filled for all gamma+1
 *   positions, including those past j*.  Sequence b emits
 *   draft_tokens[b][0 .. accept_len[b]-1] followed by next_token[b].
 * - The internal workspace (used when no caller workspace is passed) is one
 *   buffer per device: calls that use it must not overlap in time on one
 *   device (issue them on one stream).  Calls with distinct caller
 *   workspaces may run concurrently.
 */
#ifndef SPECCASCADE_H
#define SPECCASCADE_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of the logit tensors.  Entry points take it as an int32_t
 * `dtype` holding one of these values (any other value is rejected), so that
 * an out-of-range value never reaches the library as an enum. */
typedef enum { SPC_F32 = 0, SPC_BF16 = 1 } spc_dtype;

/* The further element type of a paged cache's keys and values (spc_kv_cache):
 * 8-bit floats e4m3 (largest value 448, no infinities) with a float32 scale
 * per token and head. */
#define SPC_E4M3 2

/* Deferral rules of Table 1, two constant rules, and the token-specific rules
 * of Section 4.4.  A token rule r(v) marks token v as not acceptable and uses
 * the target of Alg. 6 (TokenSpecCascade) in place of T_delta:
 *   pi(v) = q(v) (1 - r(v)) + p(v) eta,   eta = sum_v r(v) q(v).
 * For a token rule, out_defer_mask[b][j] reports r(x_j), the rule's verdict
 * on the draft token (0 at the bonus position j = gamma), and row statistic
 * column 6 holds eta.  At temperature 0 r is read at the drafter's argmax
 * with temperature-1 probabilities; the one-hot target then sits at argmax p
 * when r = 1 and at argmax q otherwise.
 *
 * The other targets of Tables 1 and 3: LOSSY is lossy speculative decoding
 * with beta = 1, whose target (Lemma 2) needs no deferral decision (the mask
 * reports 0): a draft is kept with probability min(1, p(x) / ((1 - alpha)
 * q(x))), a rejection draws from max(0, p - q), and the extra token comes
 * from p (the target is not a normalised distribution).  BILD and the
 * log-loss rules defer with the mixture target T_delta of eq. (6); their
 * statistic (D, H(q), or H(q) - H(p), in nats) is row statistic column 7.
 * At temperature 0 the log-loss rules read the entropies of the
 * temperature-1 softmax, BILD reads D = lse_p - z_p(argmax q) (temperature
 * 1), and LOSSY's one-hot target sits at argmax p. */
typedef enum {
  SPC_RULE_CHOW = 0,     /* delta = 1(max_v q(v) < 1 - alpha)                 eq. (2)  */
  SPC_RULE_DIFF = 1,     /* delta = 1(max_v q(v) < max_v p(v) - alpha)        eq. (5)  */
  SPC_RULE_OPT = 2,      /* delta = 1(max_v q(v) < max_v p(v) - alpha D_TV)   eq. (11) */
  SPC_RULE_ALWAYS = 3,   /* delta = 1: standard speculative decoding (Alg. 1)          */
  SPC_RULE_NEVER = 4,    /* delta = 0: the drafter's own distribution                  */
  SPC_RULE_TOKEN_V1 = 5, /* r(v) = 1(q(v) < max_v p(v) - alpha)          TokenV1, 4.4  */
  SPC_RULE_TOKEN_V2 = 6, /* r(v) = 1(p(v) < max_v p(v) - alpha)          TokenV2, 4.4  */
  SPC_RULE_TOKEN_V3 = 7, /* r(v) = 1(p(v) < max_v p(v) (1 - alpha))      TokenV3, 4.4  */
  SPC_RULE_LOSSY = 8,    /* lossy speculative decoding with beta = 1 (Lemma 2):
                            pi = max{min{q, p / (1 - alpha)}, p}; alpha < 1            */
  SPC_RULE_BILD = 9,     /* BiLD*: delta = 1(D(q, p) > alpha), D = -sum_v q(v) log p(v)
                            (temperature 0: -log p(argmax q))          Table 1, Sec. 6 */
  SPC_RULE_CHOWLOG = 10, /* delta = 1(H(q) > alpha)                     Table 3, App. B */
  SPC_RULE_DIFFLOG = 11, /* delta = 1(H(p) < H(q) - alpha)              Table 3, App. D */
  SPC_RULE_OPTLOG = 12   /* delta = 1(H(p) < H(q) - alpha D_TV(p, q))   Table 3, App. D */
} spc_rule;

typedef enum {
  SPC_OK = 0,
  SPC_E_NULL = -1,      /* a required pointer is NULL                                 */
  SPC_E_SHAPE = -2,     /* B < 1, gamma < 1, gamma > SPC_MAX_GAMMA or V < 2 (any B:
                           large batches run as several launches), or a cache's,
                           stride's or chunk's size out of its range                  */
  SPC_E_RULE = -3,      /* a rule id outside spc_rule                                 */
  SPC_E_PARAM = -4,     /* alpha not finite, temperature not > 0 and finite, a
                           truncation setting out of its range, or an unknown dtype   */
  SPC_E_ALIGN = -5,     /* a pointer not aligned as its function asks (logits of the
                           verify and drafter calls: 16 bytes)                        */
  SPC_E_WORKSPACE = -6, /* caller workspace too small or misaligned                   */
  SPC_E_HIP = -7        /* a HIP call failed; spc_last_error() holds its message      */
} spc_status;

/* Largest block size: the first-rejection search runs in one 64-lane wavefront. */
#define SPC_MAX_GAMMA 63

/*
 * spc_verify -- one verify step at temperature `temperature` > 0 with the same
 * rule, alpha and temperature for all B sequences.  A temperature below
 * 2^-107 (any float32 down to the smallest subnormal) is computed as 2^-107:
 * z / T stays finite for logits up to ~10^6 and the softmax is then already
 * its T -> 0 limit over logits that differ by more than ~10^-30.
 *
 *   q_logits, p_logits  [B][gamma+1][V] drafter / verifier logits, `dtype`
 *   draft_tokens        [B][gamma] int32: x_t .. x_{t+gamma-1}
 *   uniforms            [B][gamma+1] float32 in [0,1): u[b][j], j < gamma, is
 *                       the draw of a_j (Alg. 4); u[b][gamma] drives the one
 *                       replacement or extra-token sample (inverse CDF in
 *                       vocabulary order: the smallest k whose cumulative mass
 *                       exceeds u times the total)
 *   rule, alpha         deferral rule (spc_rule) and its parameter
 *   out_accept_len      [B] int32: j* in [0, gamma]
 *   out_next_token      [B] int32: the token emitted at position t + j*
 *   out_defer_mask      [B][gamma+1] uint8: delta_j at every position
 */
spc_status spc_verify(const void* q_logits, const void* p_logits, int32_t dtype,
                      const int32_t* draft_tokens, const float* uniforms, int32_t B,
                      int32_t gamma, int32_t V, int32_t rule, float alpha, float temperature,
                      int32_t* out_accept_len, int32_t* out_next_token,
                      uint8_t* out_defer_mask, hipStream_t stream);

/*
 * spc_greedy_verify -- the temperature-0 step (Lemma 6, greedy case).
 * q~ and p~ are one-hot at the argmax of the raw logits (lowest index on a
 * tie); the rule's max-probabilities come from the temperature-1 softmax and
 * D_TV(p~, q~) = 1(argmax q != argmax p).  A draft is kept exactly when it
 * equals the argmax of pi~_j = (1 - delta_j) q~_j + delta_j p~_j, and the
 * emitted token is that argmax at position j*.  No uniforms are used; the
 * result is a deterministic function of the inputs.
 */
spc_status spc_greedy_verify(const void* q_logits, const void* p_logits, int32_t dtype,
                             const int32_t* draft_tokens, int32_t B, int32_t gamma, int32_t V,
                             int32_t rule, float alpha, int32_t* out_accept_len,
                             int32_t* out_next_token, uint8_t* out_defer_mask,
                             hipStream_t stream);

/*
 * Extended arguments.  Every field may be NULL / 0.
 *   rule_per_seq, alpha_per_seq, temp_per_seq  [B] device arrays overriding
 *       the scalar rule / alpha / temperature per sequence.  A per-sequence
 *       temperature of 0 selects the greedy step for that sequence.  Values
 *       are checked by the kernels: an invalid one makes that sequence emit
 *       accept_len = -1 and next_token = -1.
 *   out_row_stats  [B][gamma+1][8] float32: {m_q, lse_q, maxprob_q, m_p,
 *       lse_p, maxprob_p, tv, s} with m = max_v z_v / T and lse = log sum_v
 *       exp(z_v / T); greedy rows hold the temperature-1 values and the
 *       one-hot TV (for a token rule, r at argmax q).  tv is computed for OPT
 *       and OPTLOG rows only (0 elsewhere); token-rule rows hold eta there.
 *       s is the statistic of BILD and the log-loss rules (0 elsewhere).
 *   out_argmax     [B][gamma+1][2] int32: argmax of raw q and p logits
 *       (filled for greedy rows; -1 elsewhere).
 *   out_sample_norm [B] float32: the total mass W of the distribution
 *       sampled at j* (for a replacement, sum_v max(0, p - q) = D_TV).
 *   workspace, workspace_bytes  caller-owned device buffer of at least
 *       spc_workspace_bytes(B, gamma, V, dtype) bytes, 256-byte aligned,
 *       whose first spc_workspace_zero_bytes(B, gamma, V, dtype) bytes are
 *       zero before its first use (the kernels leave them zero again).
 *       NULL selects the internal per-device workspace, allocated on first
 *       use and grown as needed.
 *   rules_present  with rule_per_seq: a bitmask (bit i = rule i) of the
 *       rules the array may hold, 0 = any.  It lets the library skip the
 *       passes no sequence needs (the second pass of OPT, OPTLOG and the
 *       token rules; the first moments of BiLD* and the log-loss rules).  A
 *       sequence whose rule lies outside a nonzero mask is invalid (it
 *       reports accept_len = -1 and next_token = -1).
 *   ev_tiles_begin, ev_tiles_end  for profiling: events (owned by the
 *       caller) recorded on `stream` right before and right after the
 *       statistics kernel of the call's first launch, so that their elapsed
 *       time is that kernel's duration; NULL records nothing.  A record
 *       that fails makes the call return SPC_E_HIP before any kernel of
 *       that launch.
 */
typedef struct {
  const int32_t* rule_per_seq;
  const float* alpha_per_seq;
  const float* temp_per_seq;
  float* out_row_stats;
  int32_t* out_argmax;
  float* out_sample_norm;
  void* workspace;
  size_t workspace_bytes;
  uint32_t rules_present;
  hipEvent_t ev_tiles_begin;
  hipEvent_t ev_tiles_end;
} spc_verify_ex_args;

/* spc_verify with extended arguments; `ex` may be NULL.  `temperature`
 * applies where temp_per_seq is NULL.  There it must be > 0, or exactly 0 for
 * the batch-wide greedy step of spc_greedy_verify (uniforms may then be
 * NULL), which this entry point then runs with its optional outputs. */
spc_status spc_verify_ex(const void* q_logits, const void* p_logits, int32_t dtype,
                         const int32_t* draft_tokens, const float* uniforms, int32_t B,
                         int32_t gamma, int32_t V, int32_t rule, float alpha, float temperature,
                         int32_t* out_accept_len, int32_t* out_next_token,
                         uint8_t* out_defer_mask, const spc_verify_ex_args* ex,
                         hipStream_t stream);

/*
 * spc_verify_noalloc -- spc_verify_ex for callers that cannot allocate
 * device memory: code being recorded into a HIP graph, serving loops that
 * must not call hipMalloc, harnesses that forbid allocation.  It computes
 * exactly what spc_verify_ex computes (same kernels), but its workspace is a
 * static device array of spc_noalloc_scratch_bytes() bytes (32 MiB) that
 * every device running it holds until the process ends; it calls no
 * hipMalloc, hipFree or allocating library routine.
 *   ex            as for spc_verify_ex, except that ex->workspace must be
 *                 NULL (SPC_E_WORKSPACE otherwise)
 * A batch whose layout exceeds the scratch is run in launches of as many
 * whole sequences as fit; a shape of which not even one sequence fits
 * (gamma and V large: the layout grows with (gamma + 1) * V) returns
 * SPC_E_WORKSPACE.  The first call on a device clears the array's counter
 * region with a fill kernel on `stream`; every call leaves it cleared.
 * All calls on one device share the array: calls that overlap on one device
 * (other streams, other host threads) race and must be serialised by the
 * caller.  Other errors as spc_verify_ex.
 */
spc_status spc_verify_noalloc(const void* q_logits, const void* p_logits, int32_t dtype,
                              const int32_t* draft_tokens, const float* uniforms, int32_t B,
                              int32_t gamma, int32_t V, int32_t rule, float alpha,
                              float temperature, int32_t* out_accept_len,
                              int32_t* out_next_token, uint8_t* out_defer_mask,
                              const spc_verify_ex_args* ex, hipStream_t stream);

/* Size in bytes of spc_verify_noalloc's static scratch. */
size_t spc_noalloc_scratch_bytes(void);

/*
 * spc_draft_sample -- the drafter's sampling step of GenSpecSample (Alg. 4):
 * x_{t+j} ~ q_{t+j} = softmax(z / T) for one position of each of B sequences.
 *
 *   logits        [B][V] drafter logits, `dtype`, rows contiguous
 *   temperature   T for every sequence (T = 0: the argmax of the raw logits,
 *                 lowest index on a tie), unless temp_per_seq is given
 *   temp_per_seq  [B] float32 per-sequence temperatures, or NULL; a row
 *                 whose temperature is negative or not finite gets
 *                 out_token = -1
 *   uniforms      [B] float32 in [0,1): the token is the smallest k whose
 *                 cumulative mass (vocabulary order) exceeds u times the
 *                 total; may be NULL only for the batch-wide argmax
                 (temperature 0 and temp_per_seq NULL): with temp_per_seq
                 it is required even if every entry is 0
 *   out_token     [B] int32
 * Uses the statistics tiles and the tile-mass draw of spc_verify (one pass
 * over the logits) and the internal workspace.  Errors as spc_verify; a
 * negative or non-finite temperature is SPC_E_PARAM, an invalid per-sequence
 * one gives out_token = -1.
 */
spc_status spc_draft_sample(const void* logits, int32_t dtype, int32_t B, int32_t V,
                            float temperature, const float* temp_per_seq,
                            const float* uniforms, int32_t* out_token, hipStream_t stream);

/*
 * spc_draft_sample_ws -- spc_draft_sample with a caller workspace of
 * workspace_bytes >= spc_draft_workspace_bytes(B, V, dtype) bytes, 256-byte
 * aligned, whose first spc_workspace_zero_bytes(1, 1, 2, dtype) bytes are zero
 * before its first use (the kernels leave them zero).  NULL selects the
 * internal workspace.  A too-small or misaligned workspace is SPC_E_WORKSPACE.
 * Calls with distinct workspaces may run concurrently.
 */
spc_status spc_draft_sample_ws(const void* logits, int32_t dtype, int32_t B, int32_t V,
                               float temperature, const float* temp_per_seq,
                               const float* uniforms, int32_t* out_token, void* workspace,
                               size_t workspace_bytes, hipStream_t stream);

/* Bytes of device workspace one spc_draft_sample_ws call of this shape needs. */
size_t spc_draft_workspace_bytes(int32_t B, int32_t V, int32_t dtype);

/*
 * Truncated distributions: softmax(z / T) cut by top-k, top-p and min-p.
 *
 * A row's entries are taken in the order of their logits, the largest first
 * (the lowest index first on a tie).  Each setting keeps a prefix of that
 * order, and the shortest of the three is kept:
 *   top_k  the first k entries (0: all)
 *   top_p  the fewest entries whose mass reaches top_p times the mass of the
 *          first k (1: all); 0 < top_p <= 1
 *   min_p  the entries with z >= max z + T ln(min_p), i.e. of at least min_p
 *          times the largest probability (0: all); 0 <= min_p <= 1
 * Masked entries (-inf) are never kept.  A NaN counts as -inf, +inf as the
 * largest finite value.  Masses, their sums and the comparisons are in 64 bits.
 *
 * A field of spc_truncation applies to every sequence unless its [B] device
 * array is given.  An invalid scalar is SPC_E_PARAM; a sequence with an invalid
 * entry in an array keeps nothing.  Temperature 0 is the greedy step: see the
 * two functions.
 */
typedef struct {
  float temperature;
  int32_t top_k;
  float top_p;
  float min_p;
  const float* temp_per_seq;
  const int32_t* top_k_per_seq;
  const float* top_p_per_seq;
  const float* min_p_per_seq;
} spc_truncation;

/*
 * spc_sample -- one token for each of B rows from its truncated distribution,
 * renormalised: the smallest kept v (vocabulary order) whose cumulative mass
 * exceeds u times the kept total.  Temperature 0: the argmax (lowest index).
 *
 *   logits      [B][V], `dtype`, row b at element b * row_stride (>= V); any
 *               element alignment
 *   uniforms    [B] float32 in [0, 1); may be NULL only for the batch-wide
 *               greedy step (temperature 0 and temp_per_seq NULL)
 *   out_token   [B] int32; -1 for a row that keeps nothing (all entries
 *               masked, or invalid settings)
 *   out_logprob [B] float32 or NULL: ln of the token's probability under the
 *               renormalised kept distribution (0 at temperature 0, -inf
 *               with token -1)
 *   out_kept    [B] int32 or NULL: entries kept (1 at temperature 0, 0 with
 *               token -1)
 *   workspace   a 256-byte aligned buffer of at least
 *               spc_truncation_workspace_bytes(B, V, dtype) bytes (its contents
 *               need no preparation), or NULL for the internal workspace
 */
spc_status spc_sample(const void* logits, int32_t dtype, int32_t B, int32_t V,
                      int64_t row_stride, const spc_truncation* truncation,
                      const float* uniforms, int32_t* out_token, float* out_logprob,
                      int32_t* out_kept, void* workspace, size_t workspace_bytes,
                      hipStream_t stream);

/*
 * spc_truncate -- the truncated distributions as logits, for spc_verify: drafts
 * drawn by spc_sample follow the target exactly when the drafter's rows are
 * truncated as the drafts were, and the verifier's as the target asks.
 *
 *   logits      [B][rows_per_seq][V], `dtype`, contiguous; any element alignment
 *   out_logits  the same shape and type: kept entries as they are, the others
 *               -inf.  May be `logits` itself, but not overlap it otherwise.
 * Rows of a sequence at temperature 0 are left as they are (the greedy step
 * reads whole rows); rows of invalid settings become -inf.  The workspace is
 * that of spc_sample for B * rows_per_seq rows.
 */
spc_status spc_truncate(const void* logits, int32_t dtype, int32_t B, int32_t rows_per_seq,
                        int32_t V, const spc_truncation* truncation, void* out_logits,
                        void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Bytes of device workspace one spc_sample or spc_truncate call of this many
 * rows needs (0: none, a workspace is then not looked at). */
size_t spc_truncation_workspace_bytes(int64_t rows, int32_t V, int32_t dtype);

/*
 * A paged key/value cache, and the sequences in it.  A page holds page_size
 * consecutive tokens of one sequence for every key/value head; position t of
 * sequence b lies in page page_table[b][t / page_size], slot t % page_size.
 *   k_pages   [num_pages][kv_heads][page_size][head_dim]
 *   v_pages   [num_pages][kv_heads][head_dim][page_size] (transposed)
 *   k_scale, v_scale  [num_pages][kv_heads][page_size] float32, for SPC_E4M3
 *             only: a value is its code times its token's and head's scale
 *   dtype     SPC_BF16 or SPC_E4M3
 *   page_size a multiple of 16 (16 .. 1024); head_dim 64, 128 or 256; kv_heads
 *             and B at most 65535
 *   page_table [B][table_width] int32 device array; table_width * page_size
 *             is at most 2^30
 *   kv_len    [B] int32 device array: the tokens of a sequence, its new tokens
 *             included
 * Page and scale pointers are 16-byte aligned.
 *
 * New tokens come as rows.  Without row_start there are rows / B of them for
 * every sequence, sequence after sequence; with it (a [B+1] int32 device
 * array, not decreasing) sequence b has rows row_start[b] .. row_start[b+1]-1.
 * The last of a sequence's n new rows is at position kv_len[b] - 1, the first
 * at kv_len[b] - n.  A call takes at most 2^24 rows.  Rows before row_start[0]
 * and from row_start[B] on belong to no sequence: they are not read, and outputs
 * for them are left as they are.
 *
 * Rolling back is a smaller kv_len: nothing at or past it is read.  A token
 * whose page id lies outside [0, num_pages), or whose position lies outside
 * [0, table_width * page_size), is not in the cache: it is not written, not
 * read back, and not attended to.
 */
typedef struct {
  void* k_pages;
  void* v_pages;
  float* k_scale;
  float* v_scale;
  int32_t dtype;
  int32_t num_pages;
  int32_t page_size;
  int32_t kv_heads;
  int32_t head_dim;
  const int32_t* page_table;
  int32_t table_width;
  const int32_t* kv_len;
  int32_t B;
} spc_kv_cache;

/*
 * spc_kv_write -- the keys and values of new tokens into their pages.
 *
 *   k, v        [rows][kv_heads][head_dim], `dtype` (SPC_F32 or SPC_BF16), row r
 *               at element r * k_stride (v_stride), at least
 *               kv_heads * head_dim; element-aligned
 * SPC_BF16 caches round once (to nearest even).  SPC_E4M3 caches hold, for a
 * token and head, scale = max(amax / 448, 2^-126) with amax the largest
 * magnitude, and the codes of x / scale rounded to nearest even.  Inputs are
 * finite (not checked).  Two rows must not share a slot: sequences that share
 * pages may not write to them in one call.
 */
spc_status spc_kv_write(const spc_kv_cache* cache, const void* k, const void* v, int32_t dtype,
                        int64_t k_stride, int64_t v_stride, int64_t rows,
                        const int32_t* row_start, hipStream_t stream);

/*
 * spc_kv_read -- positions 0 .. length - 1 of every sequence as dense rows.
 *
 *   out_k, out_v  [B][length][kv_heads][head_dim], `dtype` (SPC_F32 or
 *               SPC_BF16), 16-byte aligned; length at most 2^26.  Positions at or
 *               past kv_len, or not in the cache, are left as they are.
 */
spc_status spc_kv_read(const spc_kv_cache* cache, void* out_k, void* out_v, int32_t dtype,
                       int32_t length, hipStream_t stream);

/*
 * spc_kv_attend -- attention of the new tokens over the cache, which holds
 * them already (spc_kv_write first):
 *   out = sum_t softmax_t(scale q.k_t) v_t,  t from max(0, s - window + 1) to s
 * for the new token at position s (window 0: from 0).  A row that sees no
 * cached token is zero, as are rows before position 0 (a chunk longer than kv_len).
 *
 *   q           [rows][heads][head_dim] bfloat16, row r at element r * q_stride;
 *               heads a multiple of kv_heads, head i reading key/value head
 *               i / (heads / kv_heads); element-aligned
 *   out         the same, row r at element r * out_stride, 8-byte aligned, the
 *               stride a multiple of 4
 *   max_rows    with row_start, the most rows of one sequence (rows of a
 *               longer one past it are left as they are); else ignored.  It
 *               sizes the launch and the workspace for every sequence: where
 *               they would be too large for one call, SPC_E_SHAPE
 * Scores, softmax statistics and sums are in 32 bits; probabilities enter the
 * second product in bfloat16.  Cached tokens below kv_len are finite (not
 * checked: a NaN in one makes the rows that see it NaN, and may make rows NaN
 * that do not); what lies at or past kv_len may be anything.
 *   workspace   a 256-byte aligned buffer of at least
 *               spc_kv_workspace_bytes(...) bytes, or NULL for the internal
 *               per-device workspace (see the conventions above)
 */
spc_status spc_kv_attend(const spc_kv_cache* cache, const void* q, int32_t dtype,
                         int64_t q_stride, int32_t heads, int64_t rows,
                         const int32_t* row_start, int32_t max_rows, float scale,
                         int32_t window, void* out, int64_t out_stride, void* workspace,
                         size_t workspace_bytes, hipStream_t stream);

/* Bytes of device workspace one spc_kv_attend call of these sizes needs (its
 * contents need no preparation; 0: none, or sizes that no call takes); max_rows
 * as there, 0 without row_start.  Of the cache only its sizes and type are read. */
size_t spc_kv_workspace_bytes(const spc_kv_cache* cache, int32_t heads, int64_t rows,
                              int32_t max_rows);

/* Bytes of device workspace one call of this shape needs. */
size_t spc_workspace_bytes(int32_t B, int32_t gamma, int32_t V, int32_t dtype);

/* Leading bytes of a workspace that must be zero before its first use
 * (completion counters at fixed offsets: the same for every shape, so one
 * zeroed workspace serves calls of any shape it is large enough for). */
size_t spc_workspace_zero_bytes(int32_t B, int32_t gamma, int32_t V, int32_t dtype);

/* Thread-local description of the last non-OK status ("" if none). */
const char* spc_last_error(void);

/* Frees the internal workspace of every device.  Not safe while a call that
 * uses it may still be running: synchronise first. */
void spc_release(void);

/* Library version string. */
const char* spc_version(void);

#ifdef __cplusplus
}
#endif

#endif /* SPECCASCADE_H */
