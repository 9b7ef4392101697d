// spc_internal.h -- structures shared by the C interface (spc_api.cpp) and the
// gfx950 kernels (spc_kernels.hip, spc_sample.hip, spc_kv.hip).  Not part of the
// public interface.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "speccascade.h"

namespace spc {

constexpr int kThreads = 256;  // four 64-lane wavefronts per workgroup

// Sampling distribution at j* (Alg. 4): the residual max(0, p - q), or the
// extra-token target pi_{t+gamma}, which is q or p; for a token rule the
// residual max(0, pi - q) or pi_{t+gamma} of the target of Alg. 6.
enum SampleKind : int32_t { kNone = -1, kResidual = 0, kQ = 1, kP = 2, kTokRes = 3, kTokPi = 4 };

// Partial statistics of one (row, stats tile), both tensors.  With c the
// per-sequence log2(e)/T:  s = sum over the tile of 2^(z*c - r),  r the
// reference zmax * c_hi of the tile (-inf for an all -inf tile).
struct TilePart {
  double s_q, s_p;
  float r_q, r_p;
  float zmax_q, zmax_p;   // largest raw logit of the tile
  int32_t amax_q, amax_p; // statistics tiles of greedy rows: the first entry of the
                          // first lane load attaining it; drafter tiles: the lowest
                          // index attaining it; else -1
};

// First moments of one (row, stats tile) for the log-loss rules and BiLD*,
// against the same references as its TilePart:  with a = z c - r,
//   hq = sum 2^a_q a_q,  hp = sum 2^a_p a_p,  x = sum 2^a_q a_p.
struct TileMom {
  double hq, hp, x;
};

// First moments (TileMom) a statistics pass may sum: x for BiLD*'s
// cross-entropy, hq for H(q), hp for H(p).
constexpr int kMomX = 1, kMomHQ = 2, kMomHP = 4;

// Per-row statistics after merging the tiles of a row.
struct RowStat {
  double lz_q, lz_p;      // log2 sum_v 2^(z_v * c)  (= lse / ln 2)
  double tv;              // D_TV(p, q) for OPT / OPTLOG rows, eta for token-rule rows, else 0
  double slog;            // a log-loss rule's statistic (nats): D(q,p), H(q) or H(q) - H(p)
  float zmax_q, zmax_p;
  int32_t amax_q, amax_p;
};

struct Params {
  const void* q;
  const void* p;
  const int32_t* draft;
  const float* uniforms;
  int32_t B, gamma, V;
  int32_t nt;              // statistics tiles per row
  int32_t rule;
  float alpha, temp;
  int32_t force_greedy;    // spc_greedy_verify: every sequence at temperature 0
  uint32_t rule_mask;      // rules per-sequence arrays may hold (0: any)
  int32_t mom_set;         // first moments the statistics tiles sum (kMom* bits; 0: none)
  const int32_t* rule_ps;
  const float* alpha_ps;
  const float* temp_ps;
  int32_t* out_accept;
  int32_t* out_token;
  uint8_t* out_defer;
  float* out_stats;
  int32_t* out_argmax;
  float* out_norm;
  // launch layout
  int64_t single_slots;    // jobs the job pass may hold: R nt kSlices (as ws_layout)
  int32_t nsub;            // sub-chunks of a row: nt * tile_subchunks
  int32_t tv_self;         // TV rows get their TV pass from their own tiles' registers
  int32_t pair;            // statistics workgroups take two tiles each (large batches)
  int32_t tv_jobs;         // TV rows' slices are job-pass items (else the TV pass kernel)
  int32_t may_greedy;      // some sequence may be at temperature 0
  uint32_t wait_ticks;     // bound of a wait inside a kernel (100 MHz clock ticks)
  // workspace: zero region (counters; every launch leaves it as it found it)
  uint32_t* hdr;           // [kHdrLines][kLineWords] job counters
  uint32_t* rowline;       // [kMaxRows][kLineWords] per-row and per-sequence counters
  uint32_t* samp_cnt;      // drafter kernel: per-row completion counters (kDraftCntStride)
  // workspace: data (written before it is read in every launch)
  uint64_t* jobs;          // [single_slots] job entries of the job pass
  TilePart* tiles;         // [R][nt] statistics partials
  double* tvpart;          // [R][nt][kSlices] TV partials (OPT) or eta partials (token rules)
  double* submass;         // [B][nsub] residual masses per sub-chunk of row j*
  TileMom* moms;           // [R][nt] first moments (log-loss rules and BiLD*)
  RowStat* rowstat;        // [R] merged row statistics
  int32_t* rowdec;         // [R] bit 0 a_j, bit 1 delta_j
  int32_t* etalist;        // [R][nt] tiles whose eta share needs a second look
  int32_t* etacnt;         // [R] tiles listed in etalist
};

// Entries per statistics tile and per drafter tile for a dtype.
int stat_tile_elems(int dtype);
// Sub-chunks (lane-load rows of a wavefront) per statistics tile.
int tile_subchunks(int dtype);
int draft_tile_elems(int dtype, bool long_tiles);

// Counters live on 128-byte lines of 32-bit words: arrivals on a shared line
// serialise.
constexpr int kLineWords = 32;
constexpr int64_t kMaxRows = 16384;    // rows (and sequences) per launch
// Job passes: workgroups of kJobThreads threads whose wavefronts take items
// independently; a row job has kSlices items per statistics tile.
constexpr int kJobThreads = 512;
// A statistics tile splits into kSlices slices, one per wavefront of its
// workgroup (the unit of second-pass partials and residual jobs).
constexpr int kSlices = kThreads / 64;
// Header lines: the count of jobs published for the job pass (line 1; lines
// 0, 2 and 3 are spare), then kExitLeaves + 1 lines counting the workgroups
// of the pass that have read it (a two-level tree; the last arrival clears
// the count).
constexpr int kExitLeaves = 16;
constexpr int kHdrExit = 4;
constexpr int kHdrLines = kHdrExit + kExitLeaves + 1;

// Words of a row line (counters and flags, zero between calls): the row's
// tile arrivals, the decided-row mask of the sequence with the same index (64
// bits), the row's "merged, TV pass open" flag and TV slice arrivals, the
// draw pass's arrivals for the sequence, the drafter kernel's per-row
// arrivals, and the sequence's outcome for the draw pass.
constexpr int kRowArrive = 0, kSeqMask = 2, kRowReady = 5, kRowTvArrive = 6, kSeqResArrive = 7,
              kDraftArrive = 8, kSeqInfo = 9, kRowGate = 10;
// A TV row's gate where its own tiles wait for its merge (64 bits): merged
// (take the TV pass), decided without one, and in the low bits the tiles whose
// workgroups gave up waiting, so at most kTvTiles tiles a row.
constexpr int kTvTiles = 62;
constexpr uint64_t kTvReady = 1ull << 63, kTvSkip = 1ull << 62, kTvLost = kTvSkip - 1;
// A sequence's outcome word (kSeqInfo): kSeqInfoSet | sample kind << 8 | j*.
constexpr uint32_t kSeqInfoSet = 0x80000000u;

// Words between the drafter kernel's per-row completion counters.
constexpr int kDraftCntStride = kLineWords;

// Workspace layout for a shape; offsets in bytes from the base.  The zero
// region (header lines, row lines) has the same size for every shape.
struct WsLayout {
  size_t hdr, rowline, zero_end;
  size_t jobs, tiles, tvpart, submass, moms, rowstat, rowdec, etalist, etacnt, total;
};
WsLayout ws_layout(int64_t B, int64_t gamma, int64_t V, int dtype);

// Enqueue the drafter sampling kernel (Params: q = the logits [B][V], nt,
// uniforms [B], temp_ps or temp, out_token, samp_cnt with kDraftCntStride,
// tiles).  argmax: some row may be at temperature 0.
// long_tiles: tiles of twice the statistics tile's lane loads (large
// batches) rather than the statistics tile's (small ones).
hipError_t launch_draft(const Params& P, int dtype, bool argmax, bool long_tiles,
                        hipStream_t stream);

// The short-sequence path (k_seq): a workgroup per sequence, rows of at most
// kSeqSubs sub-chunks of seq_sub_elems entries (a wavefront's lane load).  It
// uses no workspace but 16 readable bytes (hdr).
constexpr int kSeqSubs = 256;
int seq_sub_elems(int dtype);
hipError_t launch_seq(const Params& P, int dtype, hipEvent_t ev_begin, hipEvent_t ev_end,
                      hipStream_t stream);

// The small-problem path (k_small): a workgroup per row holding the row in
// registers; rows of at most small_row_elems entries, kSmallSub sub-chunks.
constexpr int kSmallSub = 64;
int small_row_elems(int dtype);
hipError_t launch_small(const Params& P, int dtype, hipEvent_t ev_begin,
                        hipEvent_t ev_end, hipStream_t stream);

// Enqueue one verify launch: the statistics tiles (k_tiles; with P.tv_self
// they also take their rows' TV passes), the TV pass kernel (k_tvpass) when
// `tv_pass`, the job pass (k_jobs, of `job_groups` workgroups) when
// `job_pass`, and last the draw pass (k_res) when `draw_pass`.
// ev_begin / ev_end (may be null): recorded right before and after k_tiles.
hipError_t launch_step(const Params& P, int dtype, bool draw_pass, bool tv_pass, bool job_pass, int job_groups, hipEvent_t ev_begin, hipEvent_t ev_end,
                       hipStream_t stream);

// Rows drawn from, or cut to, their truncated distributions (spc_sample,
// spc_truncate): R rows of V logits, row stride ld entries; row r has the
// settings of sequence r / rows_per_seq.  out: the cut logits (row stride
// out_ld; may be z), or NULL for a draw.
struct TruncParams {
  const void* z;
  void* out;
  int64_t ld, out_ld, R;
  int32_t rows_per_seq, V;
  float temp, top_p, min_p;
  int32_t top_k;
  const float* temp_ps;
  const int32_t* top_k_ps;
  const float* top_p_ps;
  const float* min_p_ps;
  const float* uniforms;
  int32_t* out_token;
  float* out_logprob;
  int32_t* out_kept;
  // rows of more than kTruncHeld entries: slices of a row (0: a workgroup holds
  // the row), and the workspace of a launch's R rows
  int32_t slices;
  int32_t items_max;         // entries of a row's list
  float* slice_max;          // [R][slices]
  uint64_t* slice_bins;      // [R][slices][kTruncBins]
  uint64_t* sub_weight;      // [R][slices][16]
  uint32_t* slice_kept;      // [R][slices]
  void* row_plan;            // [R] of trunc_plan_bytes()
  void* items;               // [R][items_max] of trunc_item_bytes()
};
constexpr int kTruncHeld = 32768, kTruncBins = 1024, kTruncItems = 8192;
int trunc_slice_elems(int dtype);  // entries of a slice
size_t trunc_plan_bytes();
size_t trunc_item_bytes();
hipError_t launch_truncated(const TruncParams& P, int dtype, hipStream_t stream);

// A call on a paged key/value cache (spc_kv_*): the cache's pages and the
// sequences' tables, and the chunk of new tokens.  Row r of the chunk is token
// r - start(b) of its sequence b: start given, or n rows a sequence.
struct KvParams {
  void* k;
  void* v;                  // keys [page][H][S][D], values [page][H][D][S]
  float* k_scale;
  float* v_scale;           // [page][H][S], 8-bit caches
  int32_t f8, pages, S, H, D;
  const int32_t* table;     // [B][width]
  const int32_t* len;       // [B] tokens of the sequence, its new ones included
  uint32_t s16_magic;       // t / S = (t / 16) s16_magic / 2^32 for t < 2^30 (0: S = 16)
  int32_t B, width;
  const int32_t* start;     // [B + 1] or NULL
  int64_t rows;
  int32_t n;                // rows per sequence (start: the most of one sequence)
  // spc_kv_write, spc_kv_read: dense keys and values
  const void* k_new;
  const void* v_new;
  int64_t k_stride, v_stride;
  void* k_out;
  void* v_out;
  int32_t L;                // positions read back
  // spc_kv_attend
  const void* q;
  void* out;
  int64_t q_stride, out_stride;
  int32_t heads, window;
  uint32_t g_magic;         // r / (heads / H) = r g_magic / 2^32 for every row r (0: not so)
  float scale;              // of q.k, times log2(e)
  int32_t from;             // positions before it are left out (another launch takes them)
  const uint8_t* mask;      // spc_cross_attend: [B] rows of mask_width, mask_stride apart, or NULL
  int64_t mask_stride;
  int32_t mask_width;
  int32_t shared;           // spc_kv_attend_shared: tokens that table's only row holds for all
  int32_t tile_rows;        // rows (new token, query head) a workgroup takes: 16, 32 or 128
  int32_t splits;           // most shares the keys are cut into
  float* part;              // [B * splits][H][row tiles][tile_rows][D + 2], splits > 1
  // spc_kv_weigh (length: L): part is [B * splits][H][row tiles][tile_rows][2]
  const float* weights;     // [B * H] rows, weights_stride apart, or NULL
  float* out_weights;
  int64_t weights_stride;
  float* scores;            // [B][H][n heads / H][width * S], or NULL
  int32_t parts;            // that the rows are cut into for their sums
  float* sums;              // [parts][B][H][min(width * S, L)], parts > 1
};
hipError_t launch_kv_write(const KvParams& P, int dtype, hipStream_t stream);
hipError_t launch_kv_read(const KvParams& P, int dtype, hipStream_t stream);
constexpr int kKvShares = 128;                // shares the keys of a row are cut into, at most
// Keys that a share of them has at least (shared: of any but a sequence's own).
int kv_share_keys(int tile_rows, bool f8, bool shared);
hipError_t launch_kv_attend(const KvParams& P, hipStream_t stream);
// What an attention's workgroups take, for how it is cut.
enum class AttendKind { kOwnTokens, kCrossTokens, kPrefix, kBehindPrefix };
hipError_t launch_cross_attend(const KvParams& P, hipStream_t stream);
// own: every sequence's tokens from pre.shared on (splits = 0: none has any); pre:
// the shared ones, with table their pages alone and the rows of all sequences as
// one's (tile_rows, splits, part of its own).
hipError_t launch_kv_attend_shared(const KvParams& own, const KvParams& pre, hipStream_t stream);
constexpr int kWeighRows = 32;     // rows of a key/value head whose scores a call may keep
// Keys that a share of more rows has at least.  (us by 512 / 256 / 128: 100 rows of 8
// sequences over up to 2048 keys, 16/4 heads of 64, 38 / 29 / 29; 64 of 1 over 8000, 8
// heads of 64, 22 / 21 / 24; 100 of 6 over up to 1500, 16/4 heads of 256, 60 / 50 / 47.)
constexpr int kWeighShare = 256;
constexpr int kWeighStats = 1024;  // rows whose statistics the second step holds
hipError_t launch_kv_weigh(const KvParams& P, hipStream_t stream);

// spc_kv_evict: of every sequence and head the tokens of the largest weights.
struct EvictParams {
  KvParams cache;
  const float* weights;     // [B * H] rows, weights_stride apart, of `length`
  int64_t weights_stride, out_stride;
  int32_t length, keep, first, recent;
  const int32_t* out_table;  // [B][out_width]
  int32_t out_width;
  int32_t* out_len;         // [B]
  int32_t* out_index;       // [B][H][keep]
  float* out_weights;       // rows of keep, out_stride apart, or NULL
};
hipError_t launch_kv_evict(const EvictParams& P, hipStream_t stream);

// Enqueue a kernel writing `bytes` zero bytes at `ptr` (a multiple of 4, ptr
// 4-byte aligned): a fill a graph capture may record.
hipError_t launch_fill_zero(void* ptr, size_t bytes, hipStream_t stream);

// The kernels a verify call runs, for tests of the dispatch: the first launch
// of a call of these sizes whose sequences may hold `rules` (a bitmask), on a
// device of `cus` compute units; 0 for sizes no call takes.
enum RouteBit : int32_t {
  kRouteSeq = 1,      // k_seq
  kRouteSmall = 2,    // k_small
  kRouteTiles = 4,    // k_tiles (and k_res)
  kRouteTvSelf = 8,   // TV passes from the row's own tiles
  kRouteTvPass = 16,  // k_tvpass
  kRouteTvJobs = 32,  // TV slices in the job pass
  kRouteJobs = 64,    // k_jobs
  kRoutePair = 128    // two tiles per workgroup
};

}  // namespace spc

extern "C" int32_t spc_debug_route(int32_t B, int32_t gamma, int32_t V, int32_t dtype,
                                   uint32_t rules, int32_t per_rule, int32_t greedy, int32_t cus);
