// Entry points of attention over packed sequences and caches (declared in
// include/upipe.h), and the host's plan of their work.
//
// A plan lists every workgroup's work for one batch of lengths, longest first: the
// sequences differ in length, so a grid over the longest one would mostly be empty,
// and which tiles are long is not where the device can sort them for free.  A
// training step's layers, forward and backward, share one plan.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "../../include/upipe.h"
#include "api_internal.h"
#include "kernels.h"
#include "varlen.h"

namespace upipe {

namespace {

constexpr uint64_t kPlanMagic = 0x31306e6c70727670ull;
constexpr int kMaxSequences = 1 << 20;
constexpr int64_t kMaxTokens = int64_t(1) << 40;
// Elements from one token's row to the next: a stage of 128 rows is addressed with
// 32-bit byte offsets.
constexpr int64_t kMaxRowStride = int64_t(1) << 22;
// A launch counts its threads in 32 bits.
bool grid_fits(int64_t blocks, int threads) { return blocks < (int64_t(1) << 32) / threads; }
constexpr int kCUs = 256;

// Calls f(i) for the items in the order of their keys (>= 0), the largest first, of one key
// in the order they came.
template <class F>
void descending(const std::vector<int>& keys, F&& f) {
  int most = 0;
  for (int k : keys) most = std::max(most, k);
  std::vector<int> order(keys.size());
  if ((size_t)most < 4 * keys.size() + 1024) {      // counted: an eighth of the sort's time
    std::vector<int> at(most + 2);
    for (int k : keys) ++at[most - k + 1];
    for (int k = 0; k < most; ++k) at[k + 1] += at[k];
    for (size_t i = 0; i < keys.size(); ++i) order[at[most - keys[i]]++] = (int)i;
  } else {
    for (size_t i = 0; i < keys.size(); ++i) order[i] = (int)i;
    std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return keys[a] > keys[b]; });
  }
  for (int i : order) f(i);
}

// Time at which the last of these workgroups ends, `copies` of each: longest first,
// each to the first place that is free, `per_cu` (1 or 2) of them a CU, taking fixed +
// units * unit.  Where even an even spread would end after `limit` that is enough:
// infinity.
double makespan(const std::vector<int>& units, int copies, int per_cu, double fixed, double unit,
                double limit) {
  const int places = per_cu * kCUs;
  double all = 0.0, longest = 0.0;
  for (int u : units) {
    all += fixed + u * unit;
    longest = std::max(longest, fixed + u * unit);
  }
  if (std::max(all * copies / places, longest) >= limit) return INFINITY;
  // The copies of a workgroup go to places that are free together: one of them counts.
  const int heap = places % copies == 0 ? places / copies : places;
  if (heap < places) copies = 1;
  float free[2 * kCUs] = {};       // the first free one on top
  float end = 0.f;
  descending(units, [&](int n) {
    const float time = (float)(fixed + units[n] * unit);
    for (int i = 0; i < copies; ++i) {
      const float t = free[0] + time;
      end = std::max(end, t);
      int at = 0;
      for (int c; (c = 2 * at + 1) < heap; at = c) {
        if (c + 1 < heap && free[c + 1] < free[c]) ++c;
        if (free[c] >= t) break;
        free[at] = free[c];
      }
      free[at] = t;
    }
  });
  return end;
}

struct Lengths {
  int64_t q0, k0;
  int32_t Lq, Lk;
};

// A workgroup of the forward or of dQ: eight waves over 256 rows, or over 128 or 64 with a
// stage's keys in 2 or 4 parts, one a CU; or, half, four waves over 128 rows, two a CU, so
// that one's loads and stores hide behind the other's products.  us of a stage, and besides
// them of one alone and where they fill the chip and share its memory.
struct Shape {
  int ks;                // 256 / rows
  bool half;
  int keys, per_cu;      // of a stage
  double stage, fixed, full;
};
// What they lead to, us with 1 | 2 | 4 | half (* the chosen one): 16 documents of 256 tokens,
// 32 heads on 8, 51 | 51 | 73 | 40*; 100 of up to 700, 8 on 1, 90 | 116 | 182 | 80*; 8
// of 2048, 8 on 1, 78* | 92 | 131 | 78; 8192 tokens, 4 on 1, 91 (its keys in parts, merged) |
// 104 | 89* | 136; 32768 tokens, 4 on 1, 903* | 976 | 1173 | 1015; 512 tokens, 4 on 1, 22 |
// 16 | 14* | 16.
constexpr Shape kFwdShapes[4] = {{1, false, 128, 1, 3.5, 3.0, 10.0},
                                 {2, false, 128, 1, 2.0, 3.0, 7.0},
                                 {4, false, 128, 1, 1.2, 3.0, 6.5},
                                 {2, true, 64, 2, 1.9, 3.0, 6.5}};
// us that a merge launch takes, and that it takes for one part of 64 rows.  16 queries of 8
// heads on 50000 keys: in parts of 4 stages 18 + 5 us, of 16 26 + 5, whole 402; 500
// queries on 16000 keys: parts of 8 stages 43 + 6, whole 134.
constexpr double kMergeFixed = 4.0, kMergePart = 0.01;

struct FwdChoice {
  const Shape* shape = kFwdShapes;
  int most = 1 << 30;      // stages of a part
  double est = 0.0;
};

int row_tiles(int32_t Lq, int G, int rows) { return (int)(((int64_t)Lq * G + rows - 1) / rows); }

// Stages of tile `tile` of a sequence's packed rows.
int tile_stages(const Lengths& s, int G, const Shape& shape, int tile, int causal) {
  const int64_t rows = 256 / shape.ks;
  const int64_t last = (std::min((tile + 1) * rows, (int64_t)s.Lq * G) - 1) / G;
  const int64_t seen = causal ? std::min<int64_t>(s.Lk, last + 1 + s.Lk - s.Lq) : s.Lk;
  return seen <= 0 ? 0 : (int)((seen + shape.keys - 1) / shape.keys);
}

// Parts into which the keys of a sequence's tiles are cut so that none has more
// than `most` stages (if kMostParts suffice).
int seq_parts(const Lengths& s, int most) {
  const int stages = (s.Lk + 127) / 128;
  return std::max(1, std::min(kMostParts, (stages + most - 1) / most));
}

// Calls f(sequence, tile, part, parts, stages) for every workgroup of the forward.
template <class F>
void each_fwd(const std::vector<Lengths>& seqs, int G, int causal, const FwdChoice& c, F&& f) {
  for (size_t i = 0; i < seqs.size(); ++i) {
    const Lengths& s = seqs[i];
    const int np = seq_parts(s, c.most);
    for (int t = row_tiles(s.Lq, G, 256 / c.shape->ks) - 1; t >= 0; --t) {
      const int st = tile_stages(s, G, *c.shape, t, causal), per = (st + np - 1) / np;
      for (int p = 0; p < np; ++p)
        f((int)i, t, p, np, std::max(0, std::min(st, per * (p + 1)) - per * p));
    }
  }
}

// The time that a list of workgroups of a shape is expected to take.
double shape_time(const std::vector<int>& units, int Hkv, const Shape& shape, double limit) {
  const double share = std::min(1.0, (double)units.size() * Hkv / kCUs);
  return makespan(units, Hkv, shape.per_cu, shape.fixed + share * (shape.full - shape.fixed),
                  shape.stage, limit);
}

// The workgroups' shape, and the keys' split over them, whose list is expected to end
// first.
FwdChoice choose_fwd(const std::vector<Lengths>& seqs, int G, int Hkv, int causal) {
  FwdChoice best;
  std::vector<int> units;
  bool first = true;
  // Stages of all workgroups.
  auto look = [&](FwdChoice c) {
    units.clear();
    int64_t parts = 0, stages = 0;
    each_fwd(seqs, G, causal, c, [&](int, int, int, int np, int st) {
      units.push_back(st);
      parts += np > 1;
      stages += st;
    });
    const double merge =
        parts > 0 ? kMergeFixed + kMergePart * parts * Hkv * (4.0 / c.shape->ks) : 0.0;
    // parts take workspace: only for a gain
    const double limit = first ? INFINITY : (parts > 0 ? 0.95 : 1.0) * best.est;
    c.est = merge + shape_time(units, Hkv, *c.shape, limit - merge);
    if (c.est < limit) best = c;
    first = false;
    return stages * Hkv;
  };
  for (const Shape& shape : kFwdShapes) {
    FwdChoice c;
    c.shape = &shape;
    const int64_t stages = look(c), mean = (stages + kCUs - 1) / kCUs;      // of a CU
    // Near the whole chip's rate of the largest tiles: nothing to gain.
    if (shape.ks == 1 && best.est <= 1.1 * stages * shape.stage / kCUs) break;
    // no long ones to cut
    if (shape.half || units.empty()) continue;
    if (*std::max_element(units.begin(), units.end()) <= 2 * mean) continue;
    for (int64_t m : {mean, 2 * mean}) {
      c.most = (int)std::max<int64_t>(4, m);
      look(c);
    }
  }
  return best;
}

// us of a dK/dV tile of 128 rows, of a workgroup besides its tiles, of the fold's
// launch and of a segment's sums in it.  65536 tokens in documents of up to 32768, 8
// heads on 1: segments of 512 tiles 4.91 ms, of 128 or 256 the same, 1024 5.07, whole
// walks 7.22; 2048 tokens in documents of up to 700, 4 heads: 2 tiles 17 + 4 us, 1 tile
// 14 + 6, 4 tiles 23 + 4, whole walks 75.
constexpr double kKeyTile = 4.0, kKeyFixed = 8.0, kFoldFixed = 5.0, kFoldSum = 0.065;
constexpr int64_t kMaxSums = 2048;     // segment sums of all heads: 256 MB of workspace

// Tiles of packed rows that see a key block: first .. last (none: first > last).
void key_walk(const Lengths& s, int tpt, int kb, int causal, int* first, int* last) {
  *last = (s.Lq + tpt - 1) / tpt - 1;
  const int64_t tok = causal ? std::max<int64_t>(0, (int64_t)kb * 128 - (s.Lk - s.Lq)) : 0;
  *first = (int)std::min<int64_t>(tok / tpt, *last + 1);
}

// Calls f(sequence, r0, key block, segment, segments, first tile, tiles) for every
// workgroup of dK/dV, those of a segment side by side.  The walks of a sequence's key
// blocks are prefixes of one list,
// its tiles from the last one down.  That list is cut at every `most`-th tile, so that
// the workgroups of a segment walk the same tiles side by side and share their lines
// in L2 (walks cut each into even segments: 32768 rows of 8 heads on 1, 4330 | 4207 us).
template <class F>
void each_key(const std::vector<Lengths>& seqs, int G, int causal, int most, F&& f) {
  const int tpt = tile_tokens(G);
  int64_t r0 = 0;
  for (size_t s = 0; s < seqs.size(); ++s) {
    const int kbs = (seqs[s].Lk + 127) / 128;
    // Walks get shorter from key block to key block: `left` of them have a segment i.
    for (int i = 0, left = kbs; left > 0; ++i) {
      const int done = i > 0 ? i * most : 0;
      for (int kb = 0; kb < left; ++kb) {
        int first, last;
        key_walk(seqs[s], tpt, kb, causal, &first, &last);
        const int n = last - first + 1, segs = n <= most ? 1 : (n - 1) / most + 1;
        if (i >= segs) left = kb;
        else f((int)s, r0, kb, i, segs, last - done, segs > 1 ? std::min(n - done, most) : n);
      }
    }
    r0 += (int64_t)((seqs[s].Lq + tpt - 1) / tpt) * 128;
  }
}

// The longest segment with which all of them are expected to end first: the longest
// walk in n / 8 parts.
int choose_segment(const std::vector<Lengths>& seqs, int G, int Hkv, int causal) {
  const int tpt = tile_tokens(G), whole = 1 << 30;
  int longest = 1;
  for (const Lengths& s : seqs)
    if (s.Lk > 0) longest = std::max(longest, (s.Lq + tpt - 1) / tpt);
  std::vector<int> units;
  int best = whole, tried = 0;
  double best_est = 0.0;
  for (int n : {8, 10, 12, 14, 16, 18, 20, 24, 28, 32, 36, 40, 48, 56, 64, 80, 96, 128}) {
    const int most = (int)(((int64_t)longest * 8 + n - 1) / n);
    if (most == tried) continue;
    tried = most;
    int64_t slots = 0, tiles = 0;
    units.clear();
    each_key(seqs, G, causal, most, [&](int, int64_t, int, int, int segs, int, int count) {
      units.push_back(count);
      slots += segs > 1;
      tiles += count;
    });
    if (n > 8 && slots * Hkv > kMaxSums) continue;
    const double fold = slots > 0 ? kFoldFixed + kFoldSum * slots * Hkv : 0.0;
    const double limit = n == 8 ? INFINITY : best_est;
    const double est = fold + makespan(units, Hkv, 1, kKeyFixed, kKeyTile, limit - fold);
    if (est < limit) {
      best = most;
      best_est = est;
    }
    // Near the whole chip's rate, or segments of next to nothing.
    if (best_est <= 1.03 * tiles * Hkv * kKeyTile / kCUs || most <= 2) break;
  }
  return best;
}

// Of dQ, as the forward's: 59* in halves against 66 (1) for 16 documents of 256 tokens, 118*
// and 124 for 100 of up to 700, 111 and 109* for 8 of 2048; 8192 tokens, 4 heads on 1, 240 |
// 141 | 111* | 183; 512 tokens 28 | 21 | 17* | 21.
constexpr Shape kDqShapes[4] = {{1, false, 64, 1, 2.5, 4.0, 16.0},
                                {2, false, 128, 1, 2.8, 4.0, 11.0},
                                {4, false, 128, 1, 1.6, 4.0, 9.0},
                                {2, true, 64, 2, 2.7, 4.0, 12.0}};

// Calls f(sequence, r0, tile, stages) for every workgroup of dQ.
template <class F>
void each_dq(const std::vector<Lengths>& seqs, int G, int causal, const Shape& shape, F&& f) {
  const int tpt = tile_tokens(G);
  int64_t r0 = 0;
  for (size_t s = 0; s < seqs.size(); ++s) {
    for (int t = row_tiles(seqs[s].Lq, G, 256 / shape.ks) - 1; t >= 0; --t)
      f((int)s, r0, t, tile_stages(seqs[s], G, shape, t, causal));
    r0 += (int64_t)((seqs[s].Lq + tpt - 1) / tpt) * 128;
  }
}

const Shape& choose_dq(const std::vector<Lengths>& seqs, int G, int Hkv, int causal) {
  std::vector<int> units;
  const Shape* best = kDqShapes;
  double best_est = INFINITY;
  for (const Shape& shape : kDqShapes) {
    int64_t stages = 0;
    units.clear();
    each_dq(seqs, G, causal, shape, [&](int, int64_t, int, int st) {
      units.push_back(st);
      stages += st;
    });
    const double est = shape_time(units, Hkv, shape, best_est);
    if (est < best_est) {
      best = &shape;
      best_est = est;
    }
    if (shape.ks == 1 && est <= 1.1 * stages * Hkv * shape.stage / kCUs) break;
  }
  return *best;
}

// Longest first, in the order they came.
template <class T>
void longest_first(const std::vector<int>& units, const std::vector<T>& work, std::vector<T>* out) {
  out->reserve(work.size());
  descending(units, [&](int i) { out->push_back(work[i]); });
}

int check_lengths(const int64_t* cu_q, const int64_t* cu_k, int n, int Hq, int Hkv, int d, int causal,
                  std::vector<Lengths>* seqs) {
  if (n < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || !cu_q || !cu_k || (causal != 0 && causal != 1))
    return UPIPE_ERR_INVALID_ARG;
  if (d != HEAD_DIM || Hq > kMaxHeads || n > kMaxSequences) return UPIPE_ERR_UNSUPPORTED;
  if (cu_q[0] != 0 || cu_k[0] != 0) return UPIPE_ERR_INVALID_ARG;
  seqs->resize(n);
  int64_t tiles = 0, keys = 0;      // the least that the forward and dK/dV launch
  for (int i = 0; i < n; ++i) {
    if (cu_q[i + 1] < cu_q[i] || cu_k[i + 1] < cu_k[i]) return UPIPE_ERR_INVALID_ARG;
    const int64_t Lq = cu_q[i + 1] - cu_q[i], Lk = cu_k[i + 1] - cu_k[i];
    if (Lq > kMaxSeq || Lk > kMaxSeq || cu_q[i + 1] >= kMaxTokens || cu_k[i + 1] >= kMaxTokens)
      return UPIPE_ERR_UNSUPPORTED;
    (*seqs)[i] = {cu_q[i], cu_k[i], (int32_t)Lq, (int32_t)Lk};
    tiles += row_tiles((int32_t)Lq, Hq / Hkv, 256);
    keys += (Lk + 127) / 128;
  }
  // Before their lists are made, which may be more than the host's memory holds.
  return grid_fits(tiles * Hkv, 512) && grid_fits(keys * Hkv, 256) ? UPIPE_OK
                                                                   : UPIPE_ERR_UNSUPPORTED;
}

struct Plan {
  PlanHeader h{};
  std::vector<RowItem> fwd;
  std::vector<MergeItem> merge;
  std::vector<KeyItem> keys;
  std::vector<FoldItem> folds;
  std::vector<TileItem> dqs;
};

template <class T>
int64_t place(int64_t* end, const std::vector<T>& v) {
  const int64_t at = *end;
  *end = round_up(at + (int64_t)(v.size() * sizeof(T)), 64);
  return at;
}

int make_plan(const int64_t* cu_q, const int64_t* cu_k, int n, int Hq, int Hkv, int d, int causal,
              Plan* p) {
  std::vector<Lengths> seqs;
  const int rc = check_lengths(cu_q, cu_k, n, Hq, Hkv, d, causal, &seqs);
  if (rc != UPIPE_OK) return rc;
  const int G = Hq / Hkv;
  PlanHeader& h = p->h;
  h.magic = kPlanMagic;
  h.Hq = Hq;
  h.Hkv = Hkv;
  h.causal = causal;
  h.total_q = cu_q[n];
  h.total_k = cu_k[n];

  const FwdChoice c = choose_fwd(seqs, G, Hkv, causal);
  h.fwd_ks = c.shape->ks;
  h.half = c.shape->half ? kHalfFwd : 0;
  // Partial rows: [parts][Lq][Hq] of every sequence that is cut.
  std::vector<int64_t> p0;
  int parts = 1;
  int64_t merged = 0;
  for (const Lengths& s : seqs) {
    const int np = seq_parts(s, c.most);
    if (np > 1) merged += (int64_t)s.Lq * Hq;
    if (s.Lq > 0) parts = std::max(parts, np);
  }
  h.one_row = many_parts(parts, merged);
  const int per_block = h.one_row ? 1 : 16;
  for (const Lengths& s : seqs) {
    const int np = seq_parts(s, c.most);
    p0.push_back(h.part_rows);
    if (np < 2 || s.Lq < 1) continue;
    const int64_t rows = (int64_t)s.Lq * Hq;
    for (int64_t b = 0; b < (rows + per_block - 1) / per_block; ++b)
      p->merge.push_back({s.q0, h.part_rows, s.Lq, np, (int32_t)b, 0});
    h.part_rows += np * rows;
  }
  std::vector<int> units;
  std::vector<RowItem> fwd;
  each_fwd(seqs, G, causal, c, [&](int i, int tile, int part, int np, int stages) {
    const Lengths& s = seqs[i];
    units.push_back(stages);
    fwd.push_back({s.q0, s.k0, p0[i], s.Lq, s.Lk, tile, part, np, 0});
  });
  longest_first(units, fwd, &p->fwd);

  const int tpt = tile_tokens(G);
  for (const Lengths& s : seqs) h.term_rows += (int64_t)((s.Lq + tpt - 1) / tpt) * 128;
  units.clear();
  std::vector<KeyItem> keys;
  std::vector<int32_t> slot0;      // of the sequence's key blocks
  each_key(seqs, G, causal, choose_segment(seqs, G, Hkv, causal),
           [&](int i, int64_t r0, int kb, int seg, int segs, int first, int count) {
             const Lengths& s = seqs[i];
             if (seg == 0) {
               if (kb == 0) slot0.clear();
               slot0.push_back((int32_t)h.slots);
               if (segs > 1) {
                 p->folds.push_back({s.k0, s.Lk, kb, (int32_t)h.slots, segs});
                 h.slots += segs;
               }
             }
             units.push_back(count);
             keys.push_back({s.q0, s.k0, r0, s.Lq, s.Lk, kb, first, count,
                             segs > 1 ? slot0[kb] + seg : -1});
           });
  longest_first(units, keys, &p->keys);
  const Shape& dq = choose_dq(seqs, G, Hkv, causal);
  h.dq_ks = dq.ks;
  if (dq.half) h.half |= kHalfDq;
  units.clear();
  std::vector<TileItem> dqs;
  each_dq(seqs, G, causal, dq, [&](int i, int64_t r0, int tile, int stages) {
    const Lengths& s = seqs[i];
    units.push_back(stages);
    dqs.push_back({s.q0, s.k0, r0, s.Lq, s.Lk, tile, 0});
  });
  longest_first(units, dqs, &p->dqs);

  auto fits = [&](size_t items, int threads) { return grid_fits((int64_t)items * Hkv, threads); };
  if (!fits(p->fwd.size(), 512) || !fits(p->merge.size(), 256) ||
      !fits(p->keys.size(), 256) || !fits(p->folds.size() * 16, 256) || !fits(p->dqs.size(), 512))
    return UPIPE_ERR_UNSUPPORTED;
  h.n_fwd = (int32_t)p->fwd.size();
  h.n_merge = (int32_t)p->merge.size();
  h.n_key = (int32_t)p->keys.size();
  h.n_fold = (int32_t)p->folds.size();
  h.n_dq = (int32_t)p->dqs.size();
  int64_t end = round_up(sizeof(PlanHeader), 64);
  h.at_key = place(&end, p->keys);
  h.at_fold = place(&end, p->folds);
  h.at_dq = place(&end, p->dqs);
  h.at_fwd = place(&end, p->fwd);
  h.at_merge = place(&end, p->merge);
  h.bytes = end;
  return UPIPE_OK;
}

template <class T>
void put(char* to, int64_t at, const std::vector<T>& v) {
  if (!v.empty()) memcpy(to + at, v.data(), v.size() * sizeof(T));
}

const PlanHeader* header_of(const void* plan) {
  const PlanHeader* h = (const PlanHeader*)plan;
  return plan && ((uintptr_t)plan & 7) == 0 && h->magic == kPlanMagic ? h : nullptr;
}

size_t parts_bytes(int64_t rows) { return (size_t)rows * (HEAD_DIM + 1) * 4; }

size_t fwd_ws(const PlanHeader& h) { return parts_bytes(h.part_rows) + 16; }

size_t sums_at(const PlanHeader& h) {        // D and lse_c before them
  return (size_t)round_up(2 * h.Hkv * h.term_rows * 4, 256);
}

size_t bwd_ws(const PlanHeader& h) {
  return sums_at(h) + (size_t)h.Hkv * h.slots * 2 * 128 * HEAD_DIM * 4 + 16;
}

// Rows of q or dO whose tiles of 128 packed rows are addressed with 32-bit offsets.
bool tile_rows(const upipe_heads& v, int G) {
  const int64_t most = int64_t(1) << 30;
  return v.row <= most / 256 && v.head <= most / (2 * G) &&
         2 * (tile_tokens(G) * v.row + G * v.head) < most;
}

bool stage_rows(const upipe_heads& v) { return v.row <= kMaxRowStride; }

// Rows that a call writes, apart from those that it reads (T rows each).
bool apart(const upipe_heads& out, int64_t To, int Ho, const upipe_heads& in, int64_t Ti, int Hi) {
  return heads_apart(out, To, Ho, in, Ti, Hi);
}

}  // namespace

}  // namespace upipe

using namespace upipe;

extern "C" {

size_t upipe_varlen_plan_size(const int64_t* cu_q, const int64_t* cu_k, int n_seq, int Hq, int Hkv,
                              int d, int causal) {
  try {
    Plan p;
    return make_plan(cu_q, cu_k, n_seq, Hq, Hkv, d, causal, &p) == UPIPE_OK ? (size_t)p.h.bytes : 0;
  } catch (...) {
    return 0;
  }
}

int upipe_varlen_plan(const int64_t* cu_q, const int64_t* cu_k, int n_seq, int Hq, int Hkv, int d,
                      int causal, void* plan, size_t plan_bytes) {
  try {
    if (!plan || ((uintptr_t)plan & 7) != 0) return UPIPE_ERR_INVALID_ARG;
    Plan p;
    const int rc = make_plan(cu_q, cu_k, n_seq, Hq, Hkv, d, causal, &p);
    if (rc != UPIPE_OK) return rc;
    if (plan_bytes < (size_t)p.h.bytes) return UPIPE_ERR_WORKSPACE;
    char* to = (char*)plan;
    memset(to, 0, p.h.bytes);
    memcpy(to, &p.h, sizeof(p.h));
    put(to, p.h.at_fwd, p.fwd);
    put(to, p.h.at_merge, p.merge);
    put(to, p.h.at_key, p.keys);
    put(to, p.h.at_fold, p.folds);
    put(to, p.h.at_dq, p.dqs);
    return UPIPE_OK;
  } catch (...) {
    return UPIPE_ERR_HIP;
  }
}

size_t upipe_attn_fwd_varlen_workspace_size(const void* plan) {
  const PlanHeader* h = header_of(plan);
  return h ? fwd_ws(*h) : 0;
}

int upipe_attn_fwd_varlen(upipe_heads q, upipe_heads k, upipe_heads v, upipe_heads o, float* lse,
                          int64_t lse_head, const void* plan, const void* plan_dev, void* ws,
                          size_t ws_bytes, hipStream_t stream) {
  try {
    const PlanHeader* h = header_of(plan);
    if (!h || !aligned16(plan_dev)) return UPIPE_ERR_INVALID_ARG;
    const int64_t Tq = h->total_q, Tk = h->total_k;
    const int Hq = h->Hq, Hkv = h->Hkv;
    if (Tq == 0) return UPIPE_OK;
    if (!aligned16(lse) || !aligned16(ws)) return UPIPE_ERR_INVALID_ARG;
    if (lse_head < Tq || lse_head > kMaxTokens) return UPIPE_ERR_INVALID_ARG;
    if (!heads_ok(q, Tq, Hq) || !heads_ok(o, Tq, Hq) || !heads_distinct(o, Tq, Hq) ||
        (Tk > 0 && (!heads_ok(k, Tk, Hkv) || !heads_ok(v, Tk, Hkv))))
      return UPIPE_ERR_INVALID_ARG;
    // o may be q: a workgroup reads its rows before it writes them.
    if ((!heads_same(o, q) && !apart(o, Tq, Hq, q, Tq, Hq)) ||
        !apart(o, Tq, Hq, k, Tk, Hkv) ||
        !apart(o, Tq, Hq, v, Tk, Hkv))
      return UPIPE_ERR_INVALID_ARG;
    if (!stage_rows(k) || !stage_rows(v)) return UPIPE_ERR_UNSUPPORTED;
    if (ws_bytes < fwd_ws(*h)) return UPIPE_ERR_WORKSPACE;
    RowFwdArgs a{};
    a.q = view_of(q);
    a.k = view_of(k);
    a.v = view_of(v);
    a.o = view_of(o);
    a.lse = lse;
    a.lse_head = lse_head;
    a.part_o = (float*)ws;
    a.part_lse = a.part_o + h->part_rows * HEAD_DIM;
    a.items = (const RowItem*)((const char*)plan_dev + h->at_fwd);
    a.Hkv = Hkv;
    a.G = Hq / Hkv;
    a.causal = h->causal;
    UPIPE_LAUNCH(kRowsFwd, stream,
                 launch_rows_fwd(h->fwd_ks, (h->half & kHalfFwd) != 0, a, h->n_fwd, stream));
    if (h->n_merge > 0) {
      RowMergeArgs m{};
      m.part_o = a.part_o;
      m.part_lse = a.part_lse;
      m.o = a.o;
      m.lse = lse;
      m.lse_head = lse_head;
      m.items = (const MergeItem*)((const char*)plan_dev + h->at_merge);
      m.Hq = Hq;
      m.one_row = h->one_row;
      UPIPE_LAUNCH(kRowsMerge, stream, launch_rows_merge(m, h->n_merge, stream));
    }
    return UPIPE_OK;
  } catch (...) {
    return UPIPE_ERR_HIP;
  }
}

size_t upipe_attn_bwd_varlen_workspace_size(const void* plan) {
  const PlanHeader* h = header_of(plan);
  return h ? bwd_ws(*h) : 0;
}

int upipe_attn_bwd_varlen(upipe_heads q, upipe_heads k, upipe_heads v, upipe_heads o,
                          const float* lse, int64_t lse_head, upipe_heads dout, upipe_heads dq,
                          upipe_heads dk, upipe_heads dv, const void* plan, const void* plan_dev,
                          void* ws, size_t ws_bytes, hipStream_t stream) {
  try {
    const PlanHeader* h = header_of(plan);
    if (!h || !aligned16(plan_dev)) return UPIPE_ERR_INVALID_ARG;
    const int64_t Tq = h->total_q, Tk = h->total_k;
    const int Hq = h->Hq, Hkv = h->Hkv, G = Hq / Hkv;
    if (Tq == 0 && Tk == 0) return UPIPE_OK;
    if (!aligned16(ws) || (Tq > 0 && (!aligned16(lse) || lse_head < Tq || lse_head > kMaxTokens)))
      return UPIPE_ERR_INVALID_ARG;
    const upipe_heads *rq[4] = {&q, &o, &dout, &dq}, *rk[4] = {&k, &v, &dk, &dv};
    for (int i = 0; i < 4; ++i)
      if ((Tq > 0 && !heads_ok(*rq[i], Tq, Hq)) || (Tk > 0 && !heads_ok(*rk[i], Tk, Hkv)))
        return UPIPE_ERR_INVALID_ARG;
    if ((Tq > 0 && !heads_distinct(dq, Tq, Hq)) ||
        (Tk > 0 && (!heads_distinct(dk, Tk, Hkv) || !heads_distinct(dv, Tk, Hkv))))
      return UPIPE_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i)
      if (!apart(dq, Tq, Hq, *rq[i], Tq, Hq) ||
          !apart(dk, Tk, Hkv, *rq[i], Tq, Hq) || !apart(dv, Tk, Hkv, *rq[i], Tq, Hq))
        return UPIPE_ERR_INVALID_ARG;
    for (int i = 0; i < 2; ++i)
      if (!apart(dq, Tq, Hq, *rk[i], Tk, Hkv) || !apart(dk, Tk, Hkv, *rk[i], Tk, Hkv) ||
          !apart(dv, Tk, Hkv, *rk[i], Tk, Hkv))
        return UPIPE_ERR_INVALID_ARG;
    if (!apart(dq, Tq, Hq, dk, Tk, Hkv) || !apart(dq, Tq, Hq, dv, Tk, Hkv) ||
        !apart(dk, Tk, Hkv, dv, Tk, Hkv))
      return UPIPE_ERR_INVALID_ARG;
    if ((Tk > 0 && (!stage_rows(k) || !stage_rows(v))) ||
        (Tq > 0 && (!tile_rows(q, G) || !tile_rows(dout, G))))
      return UPIPE_ERR_UNSUPPORTED;
    if (ws_bytes < bwd_ws(*h)) return UPIPE_ERR_WORKSPACE;
    const char* dev = (const char*)plan_dev;
    RowBwdArgs a{};
    a.q = view_of(q);
    a.k = view_of(k);
    a.v = view_of(v);
    a.o = view_of(o);
    a.dO = view_of(dout);
    a.dq = view_of(dq);
    a.dk = view_of(dk);
    a.dv = view_of(dv);
    a.lse = lse;
    a.lse_head = lse_head;
    a.term_rows = h->term_rows;
    a.D = (float*)ws;
    a.lse_c = a.D + Hkv * h->term_rows;
    a.sums = (float*)((char*)ws + sums_at(*h));
    a.slots = h->slots;
    a.keys = (const KeyItem*)(dev + h->at_key);
    a.folds = (const FoldItem*)(dev + h->at_fold);
    a.dqs = (const TileItem*)(dev + h->at_dq);
    a.Hkv = Hkv;
    a.G = G;
    a.causal = h->causal;
    if (h->n_dq > 0)
      UPIPE_LAUNCH(kRowsDq, stream,
                   launch_rows_dq(h->dq_ks, (h->half & kHalfDq) != 0, a, h->n_dq, stream));
    if (h->n_key > 0) UPIPE_LAUNCH(kRowsDkdv, stream, launch_rows_dkdv(a, h->n_key, stream));
    if (h->n_fold > 0)
      UPIPE_LAUNCH(kRowsDkdvFold, stream, launch_rows_dkdv_fold(a, h->n_fold, stream));
    return UPIPE_OK;
  } catch (...) {
    return UPIPE_ERR_HIP;
  }
}

}  // extern "C"

// ---------------------------------------------------------------- caches
namespace upipe {

namespace {

// How a call over caches is cut: key parts of every row, and of the prefix.
struct CachePlan {
  int splits = 1;
  int prefix_ks = 1, prefix_parts = 0;
  int64_t rows = 0;        // B * nq * Hq
};

int check_cache(int64_t B, int nq, int64_t cap, int64_t P, int Hq, int Hkv, int d) {
  if (B < 1 || nq < 1 || cap < 1 || P < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0)
    return UPIPE_ERR_INVALID_ARG;
  if (d != HEAD_DIM || Hq > kMaxHeads || cap > kMaxSeq || P > kMaxSeq || nq > 128 || B > 65536)
    return UPIPE_ERR_UNSUPPORTED;
  // A row's sixteen lanes, or workgroups of 64 packed rows, a few parts each; behind a
  // prefix the workgroups of both.
  const int64_t rows = B * nq * Hq;
  return grid_fits(P > 0 ? 2 * rows + 8192 : rows, 512) ? UPIPE_OK : UPIPE_ERR_UNSUPPORTED;
}

// us of a cache's workgroup besides its stages, and of 128 keys of 64 rows with two
// workgroups a CU.
constexpr double kCacheFixed = 8.0, kCacheStage = 2.8;
// Workgroups of so many rounds of the chip are not cut further: parts take workspace.
constexpr int64_t kManyRounds = 8;

// Parts of caches of more than 32 packed rows, 4 stages at least, expected to end first:
// rounds of the chip, two workgroups a CU, and the merge's us of a part.  us with the merge:
// 4 caches of 15000 rows, 4 heads, 256 packed rows each, in 4 | 8 | 16 84 | 63 | 76; 24 of
// 8192, 8 heads, 36 rows, in 2 | 5 | 8 170 | 170 | 179, of 1 to 16384 in 4 | 8 | 12 139 |
// 124 | 132.
int tile_parts(int64_t groups, int64_t cap) {
  const int64_t places = 2 * kCUs, stages = (cap + 127) / 128;
  double best = 0.0;
  int parts = 1;
  for (int64_t p = 1; p <= std::max<int64_t>(1, std::min<int64_t>(stages / 4, places)); ++p) {
    if (p > 1 && groups * p > kManyRounds * places) break;
    const double t = (groups * p + places - 1) / places *
                         (kCacheFixed + (stages + p - 1) / p * kCacheStage) +
                     kMergePart * groups * p;
    if (p == 1 || t < best) {
      best = t;
      parts = (int)p;
    }
  }
  return parts;
}

// The prefix's workgroups: 128 or 64 packed rows (1 or 2 key parts inside) against one of
// some parts of it.  us of 64 keys of the only one on a CU and of one of two, and of a
// workgroup besides; a merge reads every part.  Up to one a CU leaves room for the
// caches' (`caches` us, half full), more of them push those behind.  us with the merge
// (in brackets by eight waves of 256 rows and caches first): 64 caches of 1 to 1024 rows, 64
// heads on 8, behind 16384, 128 rows in 4 | 8 | 16 parts 108 | 75 | 91 (91), 64 rows in 8 94;
// 64 of 200 behind 4096 in 4 | 8 | 16 39 | 38 | 47 (50), 64 rows in 4 36; 200 of 900 behind
// 32768 in 2 | 4 | 8 381 | 334 | 361 (405).
constexpr double kPrefixAlone[2] = {1.4, 1.1}, kPrefixBoth[2] = {2.3, 1.7};

void plan_prefix(int64_t rows, int64_t P, int Hkv, double caches, CachePlan* p) {
  const int64_t stages = (P + 63) / 64;
  double best = INFINITY;
  for (int ks = 1; ks <= 2; ++ks) {
    const double alone = kPrefixAlone[ks - 1], both = kPrefixBoth[ks - 1];
    const int64_t n = (rows * ks + 127) / 128 * Hkv;
    for (int64_t parts = 1; parts <= std::min<int64_t>(stages, 2 * kCUs); ++parts) {
      const int64_t w = n * parts, rest = w % (2 * kCUs), st = (stages + parts - 1) / parts;
      if (parts > 1 && w > kManyRounds * 2 * kCUs) break;
      const double more = std::max(0.0, (double)(rest - kCUs) / kCUs);
      double t = w / (2 * kCUs) * (kCacheFixed + st * both) + kMergePart * (2.0 / ks) * w;
      if (rest > 0) t += kCacheFixed + st * (alone + more * (both - alone));
      if (w > kCUs) t += caches;
      if (t < best) {
        best = t;
        p->prefix_ks = ks;
        p->prefix_parts = (int)parts;
      }
    }
  }
}

// Parts of caches of up to 32 packed rows, which wait for memory alone: of 1024 rows, unless
// they are more than four a CU, or of 2048, unless they are more than sixteen; or up to
// twice as many (512 rows each at least) where that fills the chip, two workgroups a
// CU, or whole rounds of it, better.  us with the merge (* the chosen one; the best is within
// 8 %): 24 caches of 8192 rows, 8 heads, in 2 | 5 | 6 | 8* | 16 parts 167 | 153 | 167 | 158 |
// 163, of 1 to 16384 in 4 | 6 | 8* | 12 | 16 121 | 107 | 105 | 110 | 115; 64 of 1 to 16384 in
// 2 | 4 | 8* | 16 414 | 393 | 394 | 406, 8 in 4 | 8 | 16* | 32 73 | 59 | 59 | 63; 40 of
// 8000, 2 heads, in 4 | 6 | 8 | 12* 67 | 60 | 76 | 65; 8 of 131000, one head, in 32 | 64 |
// 128* | 256 101 | 99 | 103 | 111; one of 131072 in 64 | 128 | 256* | 512 34 | 24 | 22 | 24.
int few_parts(int64_t groups, int64_t cap) {
  const int64_t slots = 2 * kCUs;
  const int64_t most = std::min((cap + 511) / 512, kMostParts - slots);     // and a prefix's
  const int64_t least =
      std::min(most, std::max({int64_t(1), std::min((cap + 1023) / 1024, 2 * slots / groups),
                               std::min((cap + 2047) / 2048, 8 * slots / groups)}));
  int64_t best = least;
  auto rounds = [&](int64_t p) { return (groups * p + slots - 1) / slots; };
  for (int64_t p = least + 1; p <= std::min(most, std::max(2 * least, slots / groups)); ++p)
    if (rounds(p) * best < rounds(best) * p) best = p;
  return (int)best;
}

// The lengths are on the device: the cut goes by the capacity, and a part is the same
// share of whatever a cache holds.
CachePlan plan_cache(int64_t B, int nq, int64_t cap, int64_t P, int Hq, int Hkv) {
  CachePlan p;
  p.rows = B * nq * Hq;
  const int64_t G = Hq / Hkv, groups = B * Hkv * ((nq * G + 63) / 64);
  p.splits = nq * G > 32 ? tile_parts(groups, cap) : few_parts(groups, cap);
  // half of the caches' bytes at 5.3 TB/s
  if (P > 0) plan_prefix(B * nq * G, P, Hkv, B * Hkv * (cap / 2) * 512 / 5.3e6, &p);
  return p;
}

// The rows of o outside the range of all caches.
bool apart_cache(const upipe_heads& o, int64_t T, int Hq, const upipe_heads& k, int64_t batch,
                 int64_t B, int64_t cap, int Hkv) {
  const int64_t so = (T - 1) * o.row + (Hq - 1) * o.head + HEAD_DIM;
  const int64_t sk = (B - 1) * batch + (cap - 1) * k.row + (Hkv - 1) * k.head + HEAD_DIM;
  return !overlap(o.p, 2 * so, k.p, 2 * sk);
}

int64_t cache_parts(const CachePlan& p) { return p.splits + p.prefix_parts; }

size_t cache_ws(const CachePlan& p) { return parts_bytes(cache_parts(p) * p.rows) + 16; }

}  // namespace

}  // namespace upipe

extern "C" {

size_t upipe_attn_decode_workspace_size(int64_t B, int nq, int64_t cap, int64_t P, int Hq, int Hkv,
                                        int d) {
  if (check_cache(B, nq, cap, P, Hq, Hkv, d) != UPIPE_OK) return 0;
  return cache_ws(plan_cache(B, nq, cap, P, Hq, Hkv));
}

int upipe_attn_decode(upipe_heads q, upipe_heads k, int64_t k_cache, upipe_heads v, int64_t v_cache,
                      const int32_t* lens, upipe_heads k_prefix, upipe_heads v_prefix, upipe_heads o,
                      float* lse, int64_t B, int nq, int64_t cap, int64_t P, int Hq, int Hkv, int d,
                      void* ws, size_t ws_bytes, hipStream_t stream) {
  try {
    const int rc = check_cache(B, nq, cap, P, Hq, Hkv, d);
    if (rc != UPIPE_OK) return rc;
    const int64_t T = B * nq, most = int64_t(1) << 60;
    if (!heads_ok(q, T, Hq) || !heads_ok(o, T, Hq) || !heads_distinct(o, T, Hq) ||
        !heads_ok(k, cap, Hkv) || !heads_ok(v, cap, Hkv) || !lens || ((uintptr_t)lens & 3) != 0 ||
        !aligned16(lse) || !aligned16(ws) || k_cache < 0 || v_cache < 0 || k_cache % 8 != 0 ||
        v_cache % 8 != 0 || k_cache > most / B || v_cache > most / B)
      return UPIPE_ERR_INVALID_ARG;
    if (P > 0 && (!heads_ok(k_prefix, P, Hkv) || !heads_ok(v_prefix, P, Hkv)))
      return UPIPE_ERR_INVALID_ARG;
    if ((!heads_same(o, q) && !apart(o, T, Hq, q, T, Hq)) ||
        !apart_cache(o, T, Hq, k, k_cache, B, cap, Hkv) ||
        !apart_cache(o, T, Hq, v, v_cache, B, cap, Hkv) ||
        (P > 0 && (!apart(o, T, Hq, k_prefix, P, Hkv) || !apart(o, T, Hq, v_prefix, P, Hkv))))
      return UPIPE_ERR_INVALID_ARG;
    if (!stage_rows(k) || !stage_rows(v) ||
        (P > 0 && (!stage_rows(k_prefix) || !stage_rows(v_prefix))))
      return UPIPE_ERR_UNSUPPORTED;
    const CachePlan p = plan_cache(B, nq, cap, P, Hq, Hkv);
    if (ws_bytes < cache_ws(p)) return UPIPE_ERR_WORKSPACE;
    const int G = Hq / Hkv;
    RowFwdArgs a{};
    a.q = view_of(q);
    a.o = view_of(o);
    a.lse = lse;
    a.part_o = (float*)ws;
    a.part_lse = a.part_o + cache_parts(p) * p.rows * HEAD_DIM;
    a.Hkv = Hkv;
    a.G = G;
    RowFwdArgs one = a;
    a.k = view_of(k);
    a.v = view_of(v);
    a.k.batch = k_cache;
    a.v.batch = v_cache;
    a.lens = lens;
    a.cap = cap;
    a.causal = 1;
    a.B = (int)B;
    a.nq = nq;
    a.splits = p.splits;
    a.part0 = p.prefix_parts;
    a.lse_head = nq;
    const int64_t blocks = ((int64_t)nq * G + 63) / 64 * B * p.splits;
    // The longest first, for some time of every workgroup, where they do not all start at once
    // and are not so many that they even each other out.  us in an order of chance | the
    // longest last, as they come and ranked: 24 caches of 1 to 16384 rows, 8 heads 110 | 114
    // and 102, with 9 new tokens 138 | 135 and 118; 64 of them 130 | 146 and 139.
    a.ranked = B <= 64 && B * Hkv <= kCUs && blocks * Hkv > 2 * kCUs;
    if (P > 0) {
      one.k = view_of(k_prefix);
      one.v = view_of(v_prefix);
      one.one.Lq = (int32_t)T;
      one.one.Lk = (int32_t)P;
      one.one.parts = p.prefix_parts;
      const int64_t tiles = (T * G * p.prefix_ks + 127) / 128;
      UPIPE_LAUNCH(kRowsFwd, stream,
                   launch_rows_prefix(p.prefix_ks, one, a, tiles, blocks,
                                      stream));
    } else {
      UPIPE_LAUNCH(kRowsFwd, stream, launch_cache_rows_fwd(a, blocks, stream));
    }
    if (cache_parts(p) == 1) return UPIPE_OK;
    RowMergeArgs m{};
    m.part_o = a.part_o;
    m.part_lse = a.part_lse;
    m.o = a.o;
    m.lse = lse;
    m.rows = p.rows;
    m.Hq = Hq;
    m.parts = (int)cache_parts(p);
    m.one_row = many_parts(m.parts, m.rows);
    m.nq = nq;
    UPIPE_LAUNCH(kRowsMerge, stream, launch_rows_merge(m, 0, stream));
    return UPIPE_OK;
  } catch (...) {
    return UPIPE_ERR_HIP;
  }
}

}  // extern "C"
