// Attention over packed sequences and over caches: what the host plans and the
// kernels read (varlen.cpp, varlen_fwd.hip, varlen_bwd.hip).
//
// Rows are packed by key/value group: row r of a sequence and a key/value head is
// query token r / G under the group's head r % G (G = Hq / Hkv).  The rows of a
// group share their keys, so a workgroup's tile of rows covers few tokens: a
// single token fills G rows, a short sequence wastes less of a tile, and the
// diagonal is cut finer.
#pragma once
#include <stdint.h>

#include "common.h"
#include "kernels.h"

namespace upipe {

// One workgroup's rows of the forward (or of dQ): tile `tile` of a sequence, part
// `part` of its keys.  Parts leave fp32 results at rows p0 + part * Lq * Hq + ...
struct RowItem {
  int64_t q0, k0, p0;      // first query row, key row, partial row
  int32_t Lq, Lk;
  int32_t tile, part, parts, pad;
};
// 16 rows of a sequence whose parts are merged, or, with many_parts, one.
constexpr int kSomeParts = 64, kMostParts = 2048;
// Whether a workgroup merges one row (else 16): with many parts, or few rows of some.  us,
// two events among them, 16 rows | one: 8 rows of 16 parts 6.9 | 7.0, of 32 8.7 | 6.9; 768
// rows of 16 8.7 | 8.6, of 32 11.7 | 9.4; 2048 rows of 32 13.0 | 16.5, of 64 20.5 | 20.8.
inline bool many_parts(int parts, int64_t rows) {
  return parts > kSomeParts || (parts > 16 && rows < 1024);
}
struct MergeItem {
  int64_t q0, p0;
  int32_t Lq, parts, block, pad;
};
// A key block's walk over the query tiles from the last one down, or a segment of
// it: `count` tiles from tile `first` down; fp32 sums to slot `slot` unless < 0.
struct KeyItem {
  int64_t q0, k0, r0;      // r0: first row of the sequence among the row terms
  int32_t Lq, Lk;
  int32_t kb, first, count, slot;
};
// A key block whose segments' sums are added: slots slot .. slot + n - 1.
struct FoldItem {
  int64_t k0;
  int32_t Lk, kb, slot, n;
};
// Tile `tile` of a sequence's packed rows for dQ.
struct TileItem {
  int64_t q0, k0, r0;
  int32_t Lq, Lk, tile, pad;
};

enum Half { kHalfFwd = 1, kHalfDq = 2 };
struct PlanHeader {
  uint64_t magic;
  int64_t bytes;                       // of the whole plan
  int64_t total_q, total_k;            // rows up to the end of the last sequence
  int64_t part_rows;                   // fp32 partial rows of the forward
  int64_t term_rows;                   // row terms of one key/value head
  int64_t slots;                       // segment sums of one key/value head
  int32_t Hq, Hkv, causal;
  int32_t fwd_ks, dq_ks;               // 256 / rows of a workgroup: its key parts, unless half
  int32_t one_row;                     // of a merging workgroup
  int32_t n_fwd, n_merge, n_key, n_fold, n_dq;
  int32_t half;                        // kHalfFwd | kHalfDq: workgroups of four waves
  int64_t at_fwd, at_merge, at_key, at_fold, at_dq;     // byte offsets
};

// Query tokens of a 128-row tile of the backward.
__host__ __device__ inline int tile_tokens(int G) { return 128 / G; }

// ---- forward (varlen_fwd.hip) ----------------------------------------------
struct RowFwdArgs {
  HeadView q, k, v, o;       // k, v: batch = elements from one cache to the next
  float* lse;
  int64_t lse_head;          // elements from one head's log-sum-exps to the next
  float *part_o, *part_lse;  // fp32 rows of 128, and their log-sum-exps
  const RowItem* items;      // planned sequences
  const int32_t* lens;       // caches: valid rows of each
  int64_t cap;
  RowItem one;               // a single sequence (the shared prefix)
  int Hkv, G, causal;
  int B, nq, splits, part0;  // caches: their first part among those of a row
  bool ranked;               // caches: the longest first
};
enum RowMode { kRowsPlanned = 0, kRowsCache = 1, kRowsOne = 2 };
// Planned sequences: `blocks` items (of every key/value head).
hipError_t launch_rows_fwd(int ks, bool half, const RowFwdArgs& a, int64_t blocks, hipStream_t st);

// Caches, by tiles of 64 packed rows: `blocks` tiles of every key/value head, parts first.
hipError_t launch_cache_rows_fwd(const RowFwdArgs& a, int64_t blocks, hipStream_t st);

// The same caches behind a prefix (p, its rows in so many tiles of 128 / ks), both in one
// launch.
hipError_t launch_rows_prefix(int ks, const RowFwdArgs& p, const RowFwdArgs& c, int64_t tiles,
                              int64_t cache_blocks, hipStream_t st);

struct RowMergeArgs {
  const float *part_o, *part_lse;
  HeadView o;
  float* lse;
  int64_t lse_head;
  const MergeItem* items;    // planned sequences; else all rows of B caches
  int64_t rows;              // B * nq * Hq
  int Hq, nq;
  int parts;                 // not planned
  bool one_row;              // many_parts
};
hipError_t launch_rows_merge(const RowMergeArgs& a, int64_t items, hipStream_t st);

// ---- backward (varlen_bwd.hip) ---------------------------------------------
struct RowBwdArgs {
  HeadView q, k, v, o, dO, dq, dk, dv;
  const float* lse;
  int64_t lse_head;
  // Row terms [Hkv][term_rows]: D = dO.o and -sqrt(d) lse of the packed rows, in tiles
  // of 128 rows, tile_tokens(G) G of them used.  dQ leaves them for dK/dV.
  float *D, *lse_c;
  int64_t term_rows;
  float* sums;               // [Hkv][slots][2][128][128] sums of segments
  int64_t slots;
  const KeyItem* keys;
  const FoldItem* folds;
  const TileItem* dqs;
  int Hkv, G, causal;
};
// n items of every key/value head.
hipError_t launch_rows_dkdv(const RowBwdArgs& a, int64_t n, hipStream_t st);
hipError_t launch_rows_dkdv_fold(const RowBwdArgs& a, int64_t n, hipStream_t st);
hipError_t launch_rows_dq(int ks, bool half, const RowBwdArgs& a, int64_t n, hipStream_t st);

}  // namespace upipe
