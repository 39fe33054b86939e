// Scored attention: what the host library hands the kernels of score_fwd.hip
// and score_bwd.hip.
//
// With S = scale q.k, f(x) = cap tanh(x / cap) (or x), positions p and a mask of
// key intervals, the attention weight of a visible pair is exp(A - LSE),
//   A_ij = f(S_ij) - slope_h |p_i - p_j|   or   f(S_ij) + bias[bucket(p_j - p_i), h].
#pragma once

#include <cstdint>

#include "zl_internal.h"

namespace zl {

// A run of consecutive K/V rows with consecutive positions.
struct ScoreRange {
  int32_t k_start, k_len, k_pos, reserved;
};
static_assert(sizeof(ScoreRange) == 16, "range record must stay 16 bytes");

// Forward, dQ: query rows [q_start, q_start + q_len) of one head against range_count key
// ranges: the first is here, the others follow at range_next in the table.  Row r stands
// at position q_pos + r.  slot: the partial slot it writes, or -1 for the final output.
// part: where a dQ item's sums for the bias table's gradient go; without one, 1 where two
// groups of waves share the item's keys.
struct ScoreItem {
  int32_t q_start, q_len, q_pos, head;
  ScoreRange range;
  int32_t range_next, range_count, slot, part;
};
// dK/dV: keys [k_start, k_start + k_len) of one K/V head against the rows of their segment,
// of the group's heads [g0, g0 + gn).  tile0: the segment's first 64-row tile.  part: the
// partial that the item leaves, or -1 where it has all of the group's heads.
struct ScoreKeyItem {
  int32_t k_start, k_len, k_pos, kv_head, q_start, q_len, q_pos, g0, gn, part, tile0, reserved;
};
// Rows of a 64-row query tile, for what they see together.
struct ScoreTile {
  int32_t row, rows, pos, reserved;
};
// Partials [part, part + parts) of the same keys.
struct ScoreSum {
  int32_t k_start, k_len, kv_head, part, parts, reserved[3];
};
static_assert(sizeof(ScoreItem) == 48 && sizeof(ScoreKeyItem) == 48 && sizeof(ScoreTile) == 16 && sizeof(ScoreSum) == 32,
              "table records must keep their size");

constexpr int kScoreMaxReach = ZL_SCORE_MAX_DISTANCE;
constexpr int kScoreMaxBuckets = ZL_SCORE_MAX_BUCKETS;
// Bins of relative positions reach so far beyond the table's: a block of 32 rows and 32
// keys within reach holds pairs up to 62 beyond it, and where the sums of its diagonals
// are added (score_dq.hip), lanes without one touch bins up to 70 beyond it.  The
// outermost bins on both sides are spare.
constexpr int kScoreBinMargin = 73;
constexpr int kScoreBins = 2 * (kScoreMaxReach + kScoreBinMargin) + 1;
constexpr int kScoreTileM = 128;     // query rows of a forward or dQ item: 4 waves x 32
constexpr int kScoreSplitKeys = 512;  // a shard's keys from which on two groups of waves may share them
constexpr int kScoreKvTileN = 128;   // keys of a dK/dV item: 4 producer waves x 32
constexpr int kScoreKvTileM = 64;    // query rows of a tile of its loop
// The backward's LSE of a row that sees nothing: its weights underflow to zero.
constexpr float kScoreNoKey = 1.0e30f;
// And of a row that has no gradient (LSE or D is no number): its weights overflow where it sees a key
// and are zero where a mask's exponent of -inf stands, which NaN would not leave.
constexpr float kScoreNoGrad = -1.0e38f;

// What happens to a score between the product and the softmax.
struct ScoreFn {
  const float* slope;         // [H], or NULL
  const void* bias;           // [n_buckets, H] bf16 or fp32, or NULL
  const int16_t* bucket;      // bucket of relative position r - reach, r in [0, 2 reach]
  int32_t bias_bf16, n_buckets, reach;
  int32_t causal;             // keys behind a row's own position are not visible
  const int32_t* key_lo;      // [Tq] visible key positions [lo, hi), or NULL
  const int32_t* key_hi;
  const int32_t* q_pos;       // [Tq] positions of the query rows, or NULL (the items' own)
  float scale_log2;           // softmax scale * log2(e)
  float cap_log2;             // cap * log2(e); 0: no cap
  float cap_in;               // 2 * scale_log2 / cap
};

struct ScoreFwdParams {
  ScoreFn fn;
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* lse;
  float* o_part;
  float* lse_part;
  const ScoreItem* items;
  const ScoreRange* ranges;
  int32_t n_items, num_heads, group;   // group: query heads per K/V head
  int32_t n_split;                     // items at the start whose keys two groups of waves share
  int64_t slot_stride, lse_slot_stride;
};

// Few rows: rows [row0, row0 + rows) of one K/V head's query rows (row m: query token
// m / group, head m % group of the group) against the keys [k_start, k_start + k_len).
// part: where the rows' partials start, or -1 where the item is alone and writes the
// result (slot as in ScoreItem).
struct ScoreFewItem {
  int32_t q_start, q_pos, row0, rows, kv_head, k_start, k_len, k_pos, part, slot, reserved[2];
};
// The partials of the same rows: `parts` times `rows` of them from `part` on.
struct ScoreJoin {
  int32_t q_start, row0, rows, kv_head, part, parts, slot, reserved;
};
static_assert(sizeof(ScoreFewItem) == 48 && sizeof(ScoreJoin) == 32, "table records must keep their size");

struct ScoreFewParams {
  ScoreFn fn;
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* lse;
  float* o_part;
  float* lse_part;
  const ScoreFewItem* items;
  const ScoreJoin* joins;
  float* part_o;               // workspace: [part rows, d]
  float* part_lse;             // [part rows]
  int32_t n_items, n_joins, num_heads, group;
  int64_t slot_stride, lse_slot_stride;
};

struct ScoreBwdParams {
  ScoreFn fn;
  const void* q;
  const void* k;
  const void* v;
  const void* out;
  const float* lse;
  const void* dout;
  void* dq;
  void* dk;
  void* dv;
  float* dsum;                 // [Tq, H] workspace: -D = -rowsum(dO * O)
  float* lse2;                 // [Tq, H] workspace: LSE * log2(e) - cap_log2, kScoreNoKey for rows that see nothing, kScoreNoGrad
  const ScoreItem* q_items;
  const ScoreKeyItem* kv_items;
  const ScoreRange* ranges;
  int32_t n_q_items, n_kv_items, num_heads, group;
  int32_t n_split;             // dQ: as in the forward
  int64_t total_q;
  float scale;
  // workspace: what each row sees, [row_lo, row_lo + row_len), and each 64-row tile's rows
  // together, [lo, hi)
  int32_t* row_lo;             // [Tq]
  int32_t* row_len;
  const ScoreTile* tiles;
  int2* tile_see;              // workspace [n_tiles]
  int32_t n_tiles;
  // partial dK, dV of items of some of a group's heads, [part][2][128][d], and their sums
  float* kv_part;
  const ScoreSum* sums;
  int32_t n_sums;
  // gradient of the bias table: each dQ item's sums per relative position, then per head and bucket
  void* dbias;                 // [n_buckets, H] in the table's type, or NULL
  float* dbias_part;           // [n_q_items, 2 reach + 1], the items of one head together
  const int32_t* head_first;   // first of each head there, [H + 1]
};

// Entries of a call's table in LDS.
static inline size_t score_bins(const ScoreFn& f) { return 2 * (size_t)(f.reach + kScoreBinMargin) + 1; }

// One workgroup of `threads` per item: `launch(first, count)` for runs of the n items, as many in each
// as keep a grid below 2^32 threads.
template <class F>
hipError_t in_grids(int64_t n, int threads, F&& launch) {
  const int64_t most = ((int64_t)1 << 32) / threads - 1;
  for (int64_t at = 0; at < n; at += most) launch(at, dim3((unsigned)(n - at < most ? n - at : most)));
  return hipGetLastError();
}

hipError_t launch_score_fwd(const ScoreFwdParams& p, int head_dim, hipStream_t s);
hipError_t launch_score_few(const ScoreFewParams& p, int head_dim, hipStream_t s);
hipError_t launch_score_pre(const ScoreBwdParams& p, int head_dim, hipStream_t s);
hipError_t launch_score_dkdv(const ScoreBwdParams& p, int head_dim, hipStream_t s);
hipError_t launch_score_dq(const ScoreBwdParams& p, int head_dim, hipStream_t s);
// Both in one launch, where their LDS allows (not with the widest tables).
bool score_both_fits(const ScoreBwdParams& p, int head_dim);
hipError_t launch_score_both(const ScoreBwdParams& p, int head_dim, hipStream_t s);
// Partial dK, dV added.
hipError_t launch_score_sum(const ScoreBwdParams& p, int head_dim, hipStream_t s);
// The bias table's gradient from the dQ items' sums.
hipError_t launch_score_dbias(const ScoreBwdParams& p, hipStream_t s);

}  // namespace zl
