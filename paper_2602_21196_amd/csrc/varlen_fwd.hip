// Attention forward over packed sequences of different lengths, over caches with
// lengths on the device, and over a prefix that a batch shares, for gfx950.
//
//   o_i = sum_j softmax_j(q_i.k_j / sqrt d) v_j,   lse_i = log sum_j exp(q_i.k_j / sqrt d)
// over the keys that row i sees: with causal, j <= i + Lk - Lq of its own sequence.
//
// Work decomposition: as in the forward over equal lengths (128-key stages of K and
// V rows in LDS, double-buffered; S^T = K Q^T by MFMA, a row's scores in one lane
// pair, P in registers as the operand of O^T += V^T P^T; one pass with a running
// reference maximum), with
//   - rows packed by key/value group (varlen.h), KS parts of every stage's keys by a
//     workgroup's waves: 256, 128 or 64 rows; or, where many sequences are short,
//     workgroups of four waves over 128 rows and stages of 64 keys, two a CU: one's loads
//     of Q and stores of O hide behind the other's products;
//   - one launch over a host-made list of tiles, longest first;
//   - a tile's keys cut into parts where tiles are few: fp32 results, merged.
// Caches go by workgroups of four waves too, two a CU, 64 rows each; a prefix and the caches
// behind it share a launch, so that the products of the one hide the other's loads.
// What bounds it: MFMA issue where tiles fill the chip (131072 tokens, 4 heads on 1: 14.2
// ms, 1240 TFLOP/s, as the forward over equal lengths; 65536 tokens in documents of up to
// 32768, 8 heads: 2.29 ms, 1200), HBM in caches (24 of 1 to 16384 rows, 8 heads: 97 - 100
// us, 5.1 - 5.3 TB/s, as 24 of 8192; a plain read of as much 5.4), launches and one chain of
// stages in short calls.
#include "varlen.h"

namespace upipe {

namespace {

// A workgroup of NW waves: 16 NW keys per LDS stage, so that every wave copies four rows
// four times of K and of V.
template <int NW>
struct Stage {
  static constexpr int KEYS = 16 * NW;
  static constexpr int K_TILE = KEYS * HEAD_DIM * 2;      // 32 KB with 8 waves, and V as much
  static constexpr int BYTES = 2 * K_TILE;
};
constexpr float kSumMax = 256.f;   // lazy-rescale bound on a lane's stage sum (2^8)
// Reference max of a row before its first key (log2 domain): a finite stand-in for
// -inf, below every finite score times log2(e) / sqrt(d), so that a stage whose keys are
// all masked leaves the row at p = 0 rather than producing 0 * inf.
constexpr float kNoMax = -3e38f;

// P of a stage as the bf16 operand of P . V (one rounding of 2^-9 a weight, as the
// matrix instructions take it), and this lane's sum of it in fp32, before that
// rounding: lse is good to fp32.
template <int NT>
__device__ __forceinline__ float tile_probs(const f32x16 (&st)[NT], bf16x8 (&pf)[NT][2],
                                            float m_ref, float sl2) {
  float ls = 0.f;
#pragma unroll
  for (int tt = 0; tt < NT; ++tt)
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float p0 = fast_exp2(fmaf(st[tt][i], sl2, -m_ref));
      const float p1 = fast_exp2(fmaf(st[tt][i + 1], sl2, -m_ref));
      pf[tt][i >> 3][i & 7] = (bf16)p0;
      pf[tt][i >> 3][(i & 7) + 1] = (bf16)p1;
      ls += p0 + p1;
    }
  return ls;
}

// One stage for one wave: the 32 NT keys from key kb on.  k_at and v_at: this lane's
// place of the first key's chunk g and of its transposing reads of V (common.h); the
// others are exclusive-ors of them (a register for each would spill).  This lane's row
// sees the keys up to `lim`, the wave's first row those up to lim_w.  copy_k and copy_v
// issue the next stage's copies.
template <int NT, class CopyK, class CopyV>
__device__ __forceinline__ void fwd_stage(const char* smem, uint32_t k_at, uint32_t v_at, int kb,
                                          int lane, const bf16x8 (&qf)[8], int lim, int lim_w,
                                          f32x16 (&oacc)[4], float& m_ref, float& l_run,
                                          const CopyK& copy_k, const CopyV& copy_v) {
  const float sl2 = 1.4426950408889634f * 0.08838834764831845f;  // log2(e)/sqrt(128)
  const int g = lane >> 5;
  f32x16 st[NT];
#pragma unroll
  for (int tt = 0; tt < NT; ++tt)
#pragma unroll
    for (int i = 0; i < 16; ++i) st[tt][i] = 0.f;
#pragma unroll
  for (int s = 0; s < 8; ++s)
#pragma unroll
    for (int tt = 0; tt < NT; ++tt)
      st[tt] = mfma32x32x16(lds_read_b128(smem, (k_at ^ (32 * s)) + 8192 * tt), qf[s], st[tt]);
  // Keep six K fragment reads in flight ahead of the MFMAs: left alone,
  // the scheduler reads two, waits for them and multiplies, exposing the
  // LDS latency every two MFMAs.
  __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
  for (int i = 0; i < 8 * NT - 6; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, 6, 0);
  // The next stage's copies follow the two blocks of products they can hide
  // behind: a wave stands still while the CU takes them, and at the top of
  // the stage nothing of it is under way.  Against there, in the forward over equal
  // lengths: one head over 4096 keys 43 -> 39 us, 4 over 8192 90 -> 86, long calls,
  // where other waves fill the gap, within 0.5 %.
  copy_k();
  // Mask keys past the row's last visible key (wave-uniform test first).
  if (kb + 32 * NT - 1 > lim_w) {
#pragma unroll
    for (int tt = 0; tt < NT; ++tt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = kb + 32 * tt + 8 * (i >> 2) + 4 * g + (i & 3);
        if (key > lim) st[tt][i] = -INFINITY;
      }
  }
  bf16x8 pf[NT][2];
  float ls = tile_probs<NT>(st, pf, m_ref, sl2);
  if (__builtin_amdgcn_ballot_w64(!(ls <= kSumMax)) != 0) {
    float mx = st[0][0];
#pragma unroll
    for (int tt = 0; tt < NT; ++tt)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, st[tt][i]);
    mx = fmaxf(mx, __shfl_xor(mx, 32)) * sl2;
    const float m_new = fmaxf(m_ref, mx);
    const float alpha = fast_exp2(m_ref - m_new);
    m_ref = m_new;
    l_run *= alpha;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) oacc[dt][i] *= alpha;
    ls = tile_probs<NT>(st, pf, m_ref, sl2);
  }
  copy_v();
  l_run += ls;
#pragma unroll
  for (int c = 0; c < 2 * NT; ++c)
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
      oacc[dt] = mfma32x32x16(tr_operand_at(smem, v_at, 16 * c, dt), pf[c >> 1][c & 1], oacc[dt]);
  // Stream the V^T fragments: four (eight transposing reads) ahead, then
  // two reads per MFMA (the default schedule issued bursts of eight
  // reads and waited between them).
  __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
  for (int i = 0; i < 8 * NT - 4; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
}

// The KS parts of every row folded in fp32, in ascending key order: parts 1..
// pass (m_ref, l, acc) through the stage buffers (16 KB per wave, and behind all of these
// 512 bytes per wave) with fold_out, part 0 takes them with fold_in; a barrier before each.
template <int KS, int NW>
struct Fold {
  static constexpr int NQW = NW / KS;      // waves along the rows
  static_assert((KS - 1) * NQW * (4096 + 128) * (int)sizeof(float) <= 2 * Stage<NW>::BYTES,
                "the parts fit into the stage buffers");
};
template <int KS, int NW>
__device__ __forceinline__ void fold_out(char* smem, int ks, int wq, int lane,
                                         const f32x16 (&oacc)[4], float m_ref, float l_tot) {
  constexpr int NQW = Fold<KS, NW>::NQW;
  float* fold = reinterpret_cast<float*>(smem);
  float* fold_ml = fold + (KS - 1) * NQW * 4096;
  const int slot = (ks - 1) * NQW + wq;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      f32x4 v;
#pragma unroll
      for (int b = 0; b < 4; ++b) v[b] = oacc[dt][4 * a + b];
      *reinterpret_cast<f32x4*>(fold + slot * 4096 + (4 * dt + a) * 256 + lane * 4) = v;
    }
  fold_ml[slot * 128 + lane] = m_ref;
  fold_ml[slot * 128 + 64 + lane] = l_tot;
}

template <int KS, int NW>
__device__ __forceinline__ void fold_in(const char* smem, int wq, int lane, f32x16 (&oacc)[4],
                                        float& m_ref, float& l_tot) {
  constexpr int NQW = Fold<KS, NW>::NQW;
  const float* fold = reinterpret_cast<const float*>(smem);
  const float* fold_ml = fold + (KS - 1) * NQW * 4096;
#pragma unroll
  for (int p = 1; p < KS; ++p) {
    const int slot = (p - 1) * NQW + wq;
    const float m_p = fold_ml[slot * 128 + lane], l_p = fold_ml[slot * 128 + 64 + lane];
    const float m_new = fmaxf(m_ref, m_p);
    const float a0 = fast_exp2(m_ref - m_new), a1 = fast_exp2(m_p - m_new);
    m_ref = m_new;
    l_tot = l_tot * a0 + l_p * a1;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const f32x4 v =
            *reinterpret_cast<const f32x4*>(fold + slot * 4096 + (4 * dt + a) * 256 + lane * 4);
#pragma unroll
        for (int b = 0; b < 4; ++b) oacc[dt][4 * a + b] = oacc[dt][4 * a + b] * a0 + v[b] * a1;
      }
  }
}

// A row against its keys by plain arithmetic.  The lane pair of a row has its query and
// output elements as the tile has them.  Ends early once a visible score is not a number, or
// no element of the output is one: so they stay (an infinite one may still meet its
// opposite).  Then m_ref and l are the tile's again, all keys' sums, which no value enters;
// with large_scores they are not to be had from there, and every key is taken.
__device__ __forceinline__ void careful_row(const bf16* k, int64_t k_row, const bf16* v,
                                            int64_t v_row, int64_t key0, int64_t key1,
                                            const bf16x8 (&qf)[8], int g, bool large_scores,
                                            f32x16 (&oacc)[4], float& m_ref, float& l) {
  const float sl2 = 1.4426950408889634f * 0.08838834764831845f;
  const float m_tile = m_ref, l_tile = l;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[dt][i] = 0.f;
  m_ref = kNoMax;
  l = 0.f;
  for (int64_t j = key0; j < key1; ++j) {
    const bf16* kp = k + j * k_row + 8 * g;
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const bf16x8 kk = *reinterpret_cast<const bf16x8*>(kp + 16 * c);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf((float)kk[e], (float)qf[c][e], s);
    }
    s = (s + __shfl_xor(s, 32)) * sl2;
    asm volatile("" : "+v"(s));      // rounded, as the maximum is: not fused with it
    const float m_new = fmaxf(m_ref, s), alpha = fast_exp2(m_ref - m_new);
    const float p = fast_exp2(s - m_new);
    m_ref = m_new;
    l = l * alpha + p;
    const bf16* vp = v + j * v_row + 4 * g;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const bf16x4 vv = *reinterpret_cast<const bf16x4*>(vp + 32 * dt + 8 * a);
#pragma unroll
        for (int b = 0; b < 4; ++b)
          oacc[dt][4 * a + b] = fmaf(p, (float)vv[b], oacc[dt][4 * a + b] * alpha);
      }
    if (!(l == l)) break;
    bool some = large_scores;      // element that is a number
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) some |= oacc[dt][i] == oacc[dt][i];
    if (!(some | (bool)__shfl_xor((int)some, 32))) {
      m_ref = m_tile;
      l = l_tile;
      break;
    }
  }
}

// Infinite or not a number.
__device__ __forceinline__ bool odd(float x) { return !(fabsf(x) < INFINITY); }

// The odd elements of the rows with `mine`: what the odd visible values of their column add
// up to, +-inf or not a number; that is the result, whatever the weights and the finite
// values.  The wave goes through the keys that all of its rows see, key0 .. common - 1, two
// columns a lane, a row through its rest, to key1.  Returns whether an element is left
// whose visible values are all finite.
__device__ __forceinline__ int settle_columns(const bf16* v, int64_t v_row, int key0, int common,
                                              int key1, bool mine, f32x16 (&oacc)[4]) {
  const int lane = threadIdx.x & 63, g = lane >> 5;
  float sum[2] = {0.f, 0.f};
  const bf16* p = v + key0 * v_row + 2 * lane;
  auto take = [&](uint32_t x) {
    const float lo = __uint_as_float(x << 16), hi = __uint_as_float(x & 0xffff0000u);
    sum[0] += odd(lo) ? lo : 0.f;
    sum[1] += odd(hi) ? hi : 0.f;
  };
  constexpr int U = 8;      // loads under way
  const int rest = max(common, key0);
  int j0 = key0;
  for (; j0 + U <= common; j0 += U) {
    uint32_t x[U];
#pragma unroll
    for (int u = 0; u < U; ++u, p += v_row) x[u] = *reinterpret_cast<const uint32_t*>(p);
#pragma unroll
    for (int u = 0; u < U; ++u) take(x[u]);
    if (__builtin_amdgcn_ballot_w64(sum[0] == sum[0] || sum[1] == sum[1]) == 0) common = j0;
  }
#pragma unroll 1
  for (; j0 < common; ++j0, p += v_row) take(*reinterpret_cast<const uint32_t*>(p));
  constexpr float OPEN = 3.4028235e38f;      // an odd element whose visible values are not, so far
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      // of column 32 dt + 8 (i / 4) + 4 g + i % 4
      const float c = __shfl(sum[i & 1], 16 * dt + 4 * (i >> 2) + 2 * g + ((i & 3) >> 1));
      oacc[dt][i] = mine && odd(oacc[dt][i]) ? odd(c) ? c : OPEN : oacc[dt][i];
      // (a condition is a pair of scalar registers: those of 64 elements would spill)
      if (i % 8 == 7) __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll 1
  for (int j = rest; j < key1 && mine; ++j) {
    const bf16* vp = v + j * v_row + 4 * g;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const bf16x4 x = *reinterpret_cast<const bf16x4*>(vp + 32 * dt + 8 * a);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const float o = oacc[dt][4 * a + b], y = (float)x[b];
          oacc[dt][4 * a + b] = odd(y) ? o == OPEN ? y : o + y : o;
        }
        if (a % 2 == 1) __builtin_amdgcn_sched_barrier(0);
      }
  }
  float least = 1.f;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) least = fminf(least, fabsf(oacc[dt][i] - OPEN));
  return mine && least == 0.f;
}

// A masked key's weight is 0, but the matrix instructions also multiply that 0 by the
// key's value, which may be infinite or not a number: then the rows of its stage come
// out as NaN.  Where a row's visible values are odd in the same columns that settles it;
// else it is formed again without the masked ones.  (All rows again, where one column of every
// value is odd: 32768 tokens of 8 heads 123 ms, settled 5.3, clean 2.0.)  `lim`: the row's
// last key, lim_w: the first row's of the wave, key1: the end of the row's keys of this part,
// `end`: the end of the keys that its tile multiplied.  So is a row of scores beyond 2^30
// formed again: there the rounding of their maximum, which the stages' fused multiply-adds
// see, is more than exp2 spans.
__device__ __forceinline__ void mend_row(bool row_ok, const bf16* k, int64_t k_row, const bf16* v,
                                         int64_t v_row, int key0, int key1, int lim, int lim_w,
                                         int end, const bf16x8 (&qf)[8], int g, f32x16 (&oacc)[4],
                                         float& m_ref, float& l) {
  float z = 0.f;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) z = fmaf(oacc[dt][i], 0.f, z);
  z += __shfl_xor(z, 32);
  const bool far = m_ref != kNoMax && fabsf(m_ref) > 1073741824.f;
  const bool bad = row_ok && (far || !(z == z));      // both lanes of a row alike
  if (__builtin_amdgcn_ballot_w64(bad) == 0) return;
  bool again = bad && far, mine = bad && !far;
  z = 0.f;
  for (int j = max(lim + 1, key0); j < end && mine; ++j) {
    const bf16* p = v + j * v_row + 64 * g;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const bf16x8 x = *reinterpret_cast<const bf16x8*>(p + 8 * c);
#pragma unroll
      for (int e = 0; e < 8; ++e) z = fmaf((float)x[e], 0.f, z);
    }
  }
  z += __shfl_xor(z, 32);
  mine = mine && !(z == z);      // a masked value is to blame
  if (__builtin_amdgcn_ballot_w64(mine) != 0) {
    const int left = settle_columns(v, v_row, key0, min(lim_w + 1, end), key1, mine, oacc);
    again |= (left | __shfl_xor(left, 32)) != 0;
  }
  if (again) careful_row(k, k_row, v, v_row, key0, key1, qf, g, far, oacc, m_ref, l);
}

// A row's result, by the lane pair that holds it: the part's, in fp32, or the row's own.
__device__ __forceinline__ void write_row(const RowFwdArgs& a, bool part, const RowItem& it,
                                          int64_t part_rows, int64_t lse_at, int tok, int h, int Hq,
                                          int g, const f32x16 (&oacc)[4], float m_ref,
                                          float l_tot) {
  const bool some = !(l_tot <= 0.f);
  const float inv = some ? 1.f / l_tot : 0.f;   // no visible key: O = 0
  const float row_lse = some ? (m_ref + __log2f(l_tot)) * 0.6931471805599453f : -INFINITY;
  if (part) {
    const int64_t at = it.p0 + it.part * part_rows + (int64_t)tok * Hq + h;
    if (g == 0) a.part_lse[at] = row_lse;
    if (!some) return;           // the merge does not use the row of an empty part
    float* pp = a.part_o + at * HEAD_DIM + 4 * g;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 ov;
#pragma unroll
        for (int b = 0; b < 4; ++b) ov[b] = oacc[dt][4 * i + b] * inv;
        *reinterpret_cast<f32x4*>(pp + 32 * dt + 8 * i) = ov;
      }
    return;
  }
  bf16* op = a.o.p + (it.q0 + tok) * a.o.row + h * a.o.head + 4 * g;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bf16x4 ov;
#pragma unroll
      for (int b = 0; b < 4; ++b) ov[b] = (bf16)(oacc[dt][4 * i + b] * inv);
      *reinterpret_cast<bf16x4*>(op + 32 * dt + 8 * i) = ov;
    }
  if (g == 0) a.lse[lse_at + h * a.lse_head + tok] = row_lse;
}

// The n-th cache to be worked on and its valid rows: where a.ranked (up to 64 caches) the
// longest first, since workgroups start in their order.  Lane i has cache i's length above
// its place from the end, so that no two are alike; the n-th of these numbers bit by bit is
// the largest that more than n of them reach (counting the larger ones of every lane
// takes twice as long).
__device__ __forceinline__ int nth_cache(const RowFwdArgs& a, int n, int& Lk) {
  auto valid = [&](int i) { return (int)min(max((int64_t)a.lens[i], (int64_t)0), a.cap); };
  if (!a.ranked) {
    Lk = valid(n);
    return n;
  }
  const int lane = threadIdx.x & 63;
  const int len = lane < a.B ? valid(lane) : 0;
  const uint32_t key = lane < a.B ? (uint32_t)len * 64 + (63 - lane) : 0;
  uint32_t nth = 0;
  for (uint32_t bit = 1u << (37 - __builtin_clz((uint32_t)a.cap)); bit != 0; bit >>= 1)
    if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(key >= (nth | bit))) > n) nth |= bit;
  const int b = __builtin_ctzll(__builtin_amdgcn_ballot_w64(lane < a.B && key == nth));
  Lk = __builtin_amdgcn_readlane(len, b);
  return b;
}

// A workgroup: BQ packed rows of one key/value head against a range of its keys; number
// `block` of a launch's.
template <int KS, int MODE, int NW>
__device__ __forceinline__ void rows_fwd(const RowFwdArgs& a, char* smem, int block) {
  constexpr int BKS = Stage<NW>::KEYS, K_TILE = Stage<NW>::K_TILE, STAGE = Stage<NW>::BYTES;
  constexpr int NQW = NW / KS;           // waves along the rows
  constexpr int NT = BKS / 32 / KS;      // 32-key tiles of a stage per wave
  constexpr int BQ = 32 * NQW;           // rows per workgroup
  const int t = threadIdx.x;
  const int lane = t & 63;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wq = KS == 1 ? w : w % NQW, ks = KS == 1 ? 0 : w / NQW;
  const int r32 = lane & 31, g = lane >> 5;
  const int G = a.G, Hq = a.Hkv * G;
  int kvh = block % a.Hkv;
  const int idx = block / a.Hkv;

  RowItem it;
  int64_t cache = 0, lse_at, part_rows;
  if (MODE == kRowsPlanned) {
    it = a.items[idx];
    lse_at = it.q0;
    part_rows = (int64_t)it.Lq * Hq;
  } else if (MODE == kRowsOne) {
    // The tiles that share a part of a head's keys on one XCD (blocks go round the eight)
    // one after another; parts that there are not end at once.
    it = a.one;
    const int tiles = (it.Lq * G + BQ - 1) / BQ, u = block / (8 * tiles) * 8 + (block & 7);
    if (u >= a.Hkv * it.parts) return;
    it.tile = block / 8 % tiles;
    kvh = u / it.parts;
    it.part = u % it.parts;
    lse_at = 0;                  // always parts
    part_rows = (int64_t)it.Lq * Hq;
  } else {
    const int tiles = (a.nq * G + BQ - 1) / BQ;
    const int b = nth_cache(a, idx / a.splits % a.B, it.Lk);
    it.tile = idx / a.splits / a.B % tiles;
    it.part = idx % a.splits + a.part0;
    it.parts = a.splits;
    it.q0 = (int64_t)b * a.nq;
    it.k0 = 0;
    it.p0 = it.q0 * Hq;
    it.Lq = a.nq;
    cache = b;
    lse_at = it.q0 * Hq;
    part_rows = (int64_t)a.B * a.nq * Hq;
  }
  const int n_rows = it.Lq * G, delta = it.Lk - it.Lq;
  const int r0 = it.tile * BQ, rw = r0 + 32 * wq, row = rw + r32;
  const bool row_ok = row < n_rows;
  int tok = row / G, hg = row - tok * G;

  const uint32_t kb_row = (uint32_t)(a.k.row * 2), vb_row = (uint32_t)(a.v.row * 2);
  const bf16* kp = a.k.p + cache * a.k.batch + it.k0 * a.k.row + kvh * a.k.head;
  const bf16* vp = a.v.p + cache * a.v.batch + it.k0 * a.v.row + kvh * a.v.head;
  uint32_t offk[4], offv[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 4 * (4 * w + i) + (lane >> 4);       // stage row, 16 lanes per row
    offk[i] = r * kb_row + ((uint32_t)((lane & 15) ^ (r & 15)) << 4);
    offv[i] = r * vb_row + (((lane & 15) ^ tsw(r)) << 4);
  }

  // Keys that the workgroup's and this wave's last row, this lane's row and the
  // wave's first row see; -1: none.
  auto last_key = [&](int tk) { return a.causal ? min(tk + delta, it.Lk - 1) : it.Lk - 1; };
  const int seen = last_key((min(r0 + BQ, n_rows) - 1) / G) + 1;
  const int nst = max(0, (seen + BKS - 1) / BKS);
  int j0 = 0, j1 = nst;
  if (MODE != kRowsPlanned || it.parts > 1) {
    const int per = (nst + it.parts - 1) / it.parts;
    j0 = min(nst, per * (MODE == kRowsCache ? it.part - a.part0 : it.part));
    j1 = min(nst, j0 + per);
  }
  const int k_part = 32 * NT * ks;          // first key of this wave's part of a stage
  const int seen_w = last_key((min(rw + 32, n_rows) - 1) / G) + 1;
  const int nw = rw >= n_rows ? 0 : max(0, min(j1, (seen_w - k_part + BKS - 1) / BKS));
  const int lim = last_key(tok), lim_w = last_key(rw / G);
  const uint32_t lds0 = lds_address(smem);
  // A stage's rows: 64-bit bases, so a cache may be of any length; rows past the
  // last key, and those of no stage, read as zero.
  auto source = [&](const bf16* p, int64_t row_elems, int j) {
    const int n = j < j1 ? min(BKS, it.Lk - j * BKS) : 0;
    return rsrc_words(p + (int64_t)j * BKS * row_elems,
                      n > 0 ? (uint32_t)((n - 1) * (int)row_elems + HEAD_DIM) * 2 : 0);
  };
  if (j0 < j1) {
    copy4_b128(source(kp, a.k.row, j0), offk, 0, lds0 + (j0 & 1) * STAGE + 4096 * w);
    copy4_b128(source(vp, a.v.row, j0), offv, 0, lds0 + (j0 & 1) * STAGE + K_TILE + 4096 * w);
  }

  // Q^T B-operand fragments for the whole key loop: lane = row, k-group g covers
  // head-dim [16s + 8g, 16s + 8g + 8).
  bf16x8 qf[8];
#pragma unroll
  for (int s = 0; s < 8; ++s)
#pragma unroll
    for (int e = 0; e < 8; ++e) qf[s][e] = (bf16)0.f;
  if (row_ok) {
    const bf16* qp = a.q.p + (it.q0 + tok) * a.q.row + (kvh * G + hg) * a.q.head + 8 * g;
#pragma unroll
    for (int s = 0; s < 8; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(qp + 16 * s);
  }

  f32x16 oacc[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) oacc[dt][i] = 0.f;
  float m_ref = kNoMax;      // reference max of the scaled scores
  float l_run = 0.f;         // this lane's partial row sum

  const uint32_t k_lane = swz256(k_part + r32, g), v_lane = K_TILE + k_part * 256 + tr_base(lane);
  for (int j = j0; j < j1; ++j) {
    const uint32_t boff = (j & 1) * STAGE;
    wait_vmem();
    __syncthreads();   // stage j landed for all waves; stage j-1's buffer is free
    const uint32_t nlds = lds0 + ((j + 1) & 1) * STAGE + 4096 * w;
    const i32x4 nk = source(kp, a.k.row, j + 1), nv = source(vp, a.v.row, j + 1);
    if (j >= nw) {                          // whole stage masked for this wave
      copy4_b128(nk, offk, 0, nlds);
      copy4_b128(nv, offv, 0, nlds + K_TILE);
      continue;
    }
    fwd_stage<NT>(smem, k_lane + boff, v_lane + boff, j * BKS + k_part, lane, qf, lim, lim_w, oacc,
                  m_ref, l_run, [&]() { copy4_b128(nk, offk, 0, nlds); },
                  [&]() { copy4_b128(nv, offv, 0, nlds + K_TILE); });
  }

  wait_vmem();       // the last stage's empty copies (to LDS) have ended
  {
    // The row's place again: kept through the loop it would spill.
    int rr = rw;
    asm volatile("" : "+s"(rr));
    rr += threadIdx.x & 31;
    tok = rr / G;
    hg = rr - tok * G;
  }
  float l_tot = l_run + __shfl_xor(l_run, 32);
  if (KS > 1) {
    __syncthreads();   // every wave is done reading the last stage, and copying
    if (ks > 0) fold_out<KS, NW>(smem, ks, wq, lane, oacc, m_ref, l_tot);
    __syncthreads();
    if (ks > 0) return;
    fold_in<KS, NW>(smem, wq, lane, oacc, m_ref, l_tot);
  }
  mend_row(row_ok, kp, a.k.row, vp, a.v.row, j0 * BKS, min(lim + 1, j1 * BKS), lim,
           lim_w, min(it.Lk, min(j1, (seen_w + BKS - 1) / BKS) * BKS), qf, g, oacc, m_ref, l_tot);
  if (!row_ok) return;
  const bool part =
      MODE == kRowsOne || (MODE == kRowsCache ? a.splits + a.part0 : it.parts) > 1;
  write_row(a, part, it, part_rows, lse_at, tok, kvh * G + hg, Hq, g, oacc, m_ref, l_tot);
}

template <int KS, int MODE, int NW>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 1 : 2) void rows_fwd_kernel(RowFwdArgs a) {
  __shared__ __attribute__((aligned(1024))) char smem[2 * Stage<NW>::BYTES];
  rows_fwd<KS, MODE, NW>(a, smem, blockIdx.x);
}

// A shared prefix and the caches behind it in one launch, the prefix's workgroups first: of
// the two on a CU one may wait for memory while the other multiplies.
template <int KS>
__global__ __launch_bounds__(256, 2) void rows_prefix_kernel(RowFwdArgs p, RowFwdArgs c,
                                                             int n_prefix) {
  __shared__ __attribute__((aligned(1024))) char smem[2 * Stage<4>::BYTES];
  const int b = blockIdx.x;
  if (b < n_prefix) rows_fwd<KS, kRowsOne, 4>(p, smem, b);
  else rows_fwd<2, kRowsCache, 4>(c, smem, b - n_prefix);
}

// The parts of every row to o and lse: weights e^(lse_i - max), the sums in fp32, one
// rounding.  Sixteen lanes a row, GP groups of them to share many parts: first the
// weights of all parts, then their outputs, several loads under way at a time (one
// after the other 256 parts of 8 rows took 17 us, twice what forming them did).  An empty
// part has the weight -1: its row is not written, where a part whose weight is 0 in fp32
// may hold a visible value that is infinite or not a number.
template <int GP, bool PLANNED>
__global__ __launch_bounds__(256) void rows_merge_kernel(RowMergeArgs a) {
  constexpr int ROWS = 16 / GP;                       // of a workgroup
  __shared__ float weights[ROWS][GP > 1 ? kMostParts : kSomeParts];
  __shared__ float sh[GP][HEAD_DIM], red[8];
  const int c = threadIdx.x & 15, grp = threadIdx.x >> 4;
  const int gp = GP > 1 ? grp : 0, lr = GP > 1 ? 0 : grp;
  int64_t r, q0 = 0, p0 = 0, rows = a.rows;
  int parts = a.parts;
  if (PLANNED) {
    const MergeItem it = a.items[blockIdx.x];
    q0 = it.q0;
    p0 = it.p0;
    rows = (int64_t)it.Lq * a.Hq;
    parts = it.parts;
    r = (int64_t)it.block * ROWS + lr;
  } else {
    r = (int64_t)blockIdx.x * ROWS + lr;
  }
  if (r >= rows) return;         // GP > 1: none or all of a workgroup
  const float* pl = a.part_lse + p0 + r;
  float m = -INFINITY, l = 0.f;
  if (GP == 1) {
    float v[kSomeParts / 16];
#pragma unroll
    for (int u = 0; u < kSomeParts / 16; ++u) {
      v[u] = c + 16 * u < parts ? pl[(c + 16 * u) * rows] : -INFINITY;
      m = fmaxf(m, v[u]);
    }
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
    // (a NaN is passed over by fmaxf and comes in with its weight)
#pragma unroll
    for (int u = 0; u < kSomeParts / 16; ++u) {
      const float wt = v[u] == -INFINITY ? -1.f : v[u] == m ? 1.f : __expf(v[u] - m);
      weights[lr][c + 16 * u] = wt;
      l += wt < 0.f ? 0.f : wt;
    }
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) l += __shfl_xor(l, off);
    __builtin_amdgcn_wave_barrier();
  } else {
    for (int i = threadIdx.x; i < parts; i += 256) {
      const float v = pl[i * rows];
      weights[0][i] = v;
      m = fmaxf(m, v);
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    for (int i = threadIdx.x; i < parts; i += 256) {
      const float v = weights[0][i];
      const float wt = v == -INFINITY ? -1.f : v == m ? 1.f : __expf(v - m);
      weights[0][i] = wt;
      l += wt < 0.f ? 0.f : wt;
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) l += __shfl_xor(l, off);
    if ((threadIdx.x & 63) == 0) red[4 + (threadIdx.x >> 6)] = l;
    __syncthreads();
    l = (red[4] + red[5]) + (red[6] + red[7]);
  }
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  const float* po = a.part_o + (p0 + r) * HEAD_DIM + 8 * c;
  constexpr int U = 4;
  for (int i0 = gp; i0 < parts; i0 += U * GP) {
    f32x4 lo[U], hi[U];
    float wt[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(i0 + u * GP, parts - 1);
      const float* p = po + i * rows * HEAD_DIM;
      lo[u] = *reinterpret_cast<const f32x4*>(p);
      hi[u] = *reinterpret_cast<const f32x4*>(p + 4);
      wt[u] = i0 + u * GP < parts ? weights[lr][i] : -1.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool empty = wt[u] < 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[e] = fmaf(wt[u], empty ? 0.f : lo[u][e], acc[e]);
        acc[4 + e] = fmaf(wt[u], empty ? 0.f : hi[u][e], acc[4 + e]);
      }
    }
  }
  if (GP > 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sh[gp][8 * c + e] = acc[e];
    __syncthreads();
    if (gp > 0) return;
    for (int i = 1; i < GP; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += sh[i][8 * c + e];
  }
  const bool some = !(l <= 0.f);
  const int64_t tok = r / a.Hq;
  const int h = (int)(r - tok * a.Hq);
  bf16x8 out;
#pragma unroll
  for (int e = 0; e < 8; ++e) out[e] = (bf16)(some ? acc[e] / l : 0.f);
  *reinterpret_cast<bf16x8*>(a.o.p + (q0 + tok) * a.o.row + h * a.o.head + 8 * c) = out;
  if (c == 0) {
    const float v = some ? fmaf(__log2f(l), 0.6931471805599453f, m) : -INFINITY;
    if (PLANNED) a.lse[q0 + tok + h * a.lse_head] = v;
    else a.lse[((tok / a.nq) * a.Hq + h) * a.nq + tok % a.nq] = v;
  }
}

}  // namespace

hipError_t launch_rows_fwd(int ks, bool half, const RowFwdArgs& a, int64_t blocks, hipStream_t st) {
  const dim3 grid((unsigned)(blocks * a.Hkv));
  if (half) return enqueue(rows_fwd_kernel<1, kRowsPlanned, 4>, grid, 256, st, a);
  return enqueue(ks == 1   ? rows_fwd_kernel<1, kRowsPlanned, 8>
                 : ks == 2 ? rows_fwd_kernel<2, kRowsPlanned, 8>
                           : rows_fwd_kernel<4, kRowsPlanned, 8>,
                 grid, 512, st, a);
}

hipError_t launch_cache_rows_fwd(const RowFwdArgs& a, int64_t blocks, hipStream_t st) {
  return enqueue(rows_fwd_kernel<2, kRowsCache, 4>, dim3((unsigned)(blocks * a.Hkv)), 256, st, a);
}

hipError_t launch_rows_prefix(int ks, const RowFwdArgs& p, const RowFwdArgs& c, int64_t tiles,
                              int64_t cache_blocks, hipStream_t st) {
  const int n_prefix = (int)((p.Hkv * p.one.parts + 7) / 8 * 8 * tiles);
  return enqueue(ks == 1 ? rows_prefix_kernel<1> : rows_prefix_kernel<2>,
                 dim3((unsigned)(n_prefix + cache_blocks * c.Hkv)), 256, st, p, c, n_prefix);
}

hipError_t launch_rows_merge(const RowMergeArgs& a, int64_t items, hipStream_t st) {
  const bool planned = a.items != nullptr;
  const int64_t blocks = planned ? items : a.one_row ? a.rows : (a.rows + 15) / 16;
  return enqueue(planned ? (a.one_row ? rows_merge_kernel<16, true> : rows_merge_kernel<1, true>)
                         : (a.one_row ? rows_merge_kernel<16, false> : rows_merge_kernel<1, false>),
                 dim3((unsigned)blocks), 256, st, a);
}

}  // namespace upipe
