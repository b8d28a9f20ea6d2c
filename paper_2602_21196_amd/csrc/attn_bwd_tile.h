// The dK/dV work on one tile of query rows, shared by the backward's kernels: the
// LDS stage, the operand fragments, and the products and gradients of a pair of
// 32-row subtiles by one wave.  Rows are counted as the caller packs them: `mykey`
// and `kw` stand for the first rows that see the lane's key and the wave's first.
#pragma once
#include "common.h"

namespace upipe {

namespace {

constexpr float kSl2 = 1.4426950408889634f * 0.08838834764831845f;  // log2(e)/sqrt(128)
constexpr float kScale = 0.08838834764831845f;                      // 1/sqrt(128)

// ------------------------------------------------------------------ dK / dV
// LDS stage for one tile of QT query rows of one head: Q and dO rows
// [QT][128] (256-B rows, transposing-read swizzle), then lse and D [QT].  The
// B operands of dV += P^T dO and dK += dS^T Q are read out of the rows with
// transposing LDS reads, so no [d][S] copies of Q and dO are needed.  A tile
// is consumed as pairs of 32-row subtiles, the upper 64 rows first.
constexpr int QT = 128;
constexpr int ROWT = QT * HEAD_DIM * 2;
constexpr int OFF_Q = 0, OFF_DO = ROWT, OFF_LSE = 2 * ROWT, OFF_D = OFF_LSE + QT * 4;
constexpr int KV_STAGE = 2 * ROWT + QT * 8;
constexpr int KV_BLK = ROWT / 1024 / 4;     // 1 KB blocks per wave per array

// Operand fragments of one block of 16 MFMAs.
struct Frags {
  bf16x8 f[16];
};

// S^T / dP^T block of one 32-row subtile (rows `sub`..+31 of the tile):
// fragment 2 s + 0 is Q, 2 s + 1 is dO, both for head-dim 16 s..
__device__ __forceinline__ void read_sdp(const char* buf, int sub, int r32, int g, Frags& fr) {
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    fr.f[2 * s] = lds_read_b128(buf + OFF_Q, swzt(sub + r32, 2 * s + g));
    fr.f[2 * s + 1] = lds_read_b128(buf + OFF_DO, swzt(sub + r32, 2 * s + g));
  }
}

// dV / dK block of one subtile: fragment 4 dt + 2 kt + 0 is dO, + 1 is Q, as
// B operands with head-dim columns 32 dt.. and the 16 query rows sub + 16 kt..
__device__ __forceinline__ void read_dvdk(const char* buf, int sub, int lane, Frags& fr) {
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      fr.f[4 * dt + 2 * kt] = tr_operand(buf + OFF_DO, sub + 16 * kt, 32 * dt, lane);
      fr.f[4 * dt + 2 * kt + 1] = tr_operand(buf + OFF_Q, sub + 16 * kt, 32 * dt, lane);
    }
}

// A staged tile as pair_step reads it.
struct TileRows {
  const char* buf;
  const char* dbuf;      // where the dV / dK products read their rows
  int r32, g, lane;
  __device__ __forceinline__ void sdp(int sub, Frags& fr) const { read_sdp(buf, sub, r32, g, fr); }
  __device__ __forceinline__ void dvdk(int sub, Frags& fr) const { read_dvdk(dbuf, sub, lane, fr); }
};

// Accumulator seeds of the 32-row subtile at rows `sub`.. of the tile, in the
// MFMA C layout (element 4a + b is row sub + 8a + 4g + b), loaded from the
// staged rows straight into the accumulators: the score accumulator starts at
// -sqrt(d) lse of its row, so that it ends at q.k - sqrt(d) lse and
// P = exp2(acc log2(e) / sqrt(d)) needs no lse term; the dP accumulator
// starts at D, and the value fragments come negated, so that chain ends at
// D - dP and dS needs no subtraction: P (D - dP) = -dS.  A pair's seeds are
// read before its fragments: LDS reads complete in order, and a seed read
// behind a burst of fragment reads would wait for the whole burst.
__device__ __forceinline__ void subtile_seed(const char* buf, int sub, int g, f32x16& sacc,
                                             f32x16& pacc) {
  const float* Dl = reinterpret_cast<const float*>(buf + OFF_D) + sub;
  const float* Ll = reinterpret_cast<const float*>(buf + OFF_LSE) + sub;
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const f32x4 d4 = *reinterpret_cast<const f32x4*>(Dl + 8 * a + 4 * g);
    const f32x4 l4 = *reinterpret_cast<const f32x4*>(Ll + 8 * a + 4 * g);
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      pacc[4 * a + b] = d4[b];
      sacc[4 * a + b] = l4[b];
    }
  }
}

// S^T and D - dP^T of one subtile from its fragments (16 MFMAs), on top of
// the seeds.
__device__ __forceinline__ void subtile_sdp(const Frags& fr, const bf16x8 (&kf)[8],
                                            const bf16x8 (&nvf)[8], f32x16& sacc, f32x16& pacc) {
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    sacc = mfma32x32x16(fr.f[2 * s], kf[s], sacc);
    pacc = mfma32x32x16(fr.f[2 * s + 1], nvf[s], pacc);
  }
}

// P and -dS of one subtile as bf16 A operands, from its lse-seeded scores
// and D - dP.  Negation is exact and commutes with rounding, so the dK
// accumulators carry exactly -dK (the final scale is -1/sqrt d).  No masking
// here (subtile_mask).
__device__ __forceinline__ void subtile_pds(const f32x16& sacc, const f32x16& pacc,
                                            bf16x8 (&pf)[2], bf16x8 (&sf)[2]) {
  float p[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) p[i] = fast_exp2(sacc[i] * kSl2);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    pf[i >> 3][i & 7] = (bf16)p[i];
    sf[i >> 3][i & 7] = (bf16)(p[i] * pacc[i]);
  }
}

// Subtiles across the diagonal (wave-uniform `diag`; first row qs): zero the
// P and dS entries of keys after the row, by selection (unmasked they may be
// inf or NaN).  This runs after the conversions and between two regions: a
// branch ends the compiler's scheduling block, and inside a region it would
// split the MFMA / VALU interleave in two.
template <bool CAUSAL>
__device__ __forceinline__ void subtile_mask(uint32_t qs, uint32_t mykey, bool diag, int g,
                                             bf16x8 (&pf)[2], bf16x8 (&sf)[2]) {
  if (CAUSAL && diag) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (mykey > qs + 8 * (i >> 2) + 4 * g + (i & 3)) {
        pf[i >> 3][i & 7] = (bf16)0.f;
        sf[i >> 3][i & 7] = (bf16)0.f;
      }
  }
}

__device__ __forceinline__ void dvdk_products(const Frags& fr, const bf16x8 (&pf)[2],
                                              const bf16x8 (&sf)[2], f32x16 (&dva)[4],
                                              f32x16 (&dka)[4]) {
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      dva[dt] = mfma32x32x16(pf[kt], fr.f[4 * dt + 2 * kt], dva[dt]);
      dka[dt] = mfma32x32x16(sf[kt], fr.f[4 * dt + 2 * kt + 1], dka[dt]);
    }
}

// Scheduling request for a region of 16 MFMAs and the VALU work of one
// subtile's P and dS: one MFMA after every few VALU instructions, so the
// matrix unit and the vector ALU of the one wave on the SIMD work side by
// side (the region's LDS reads are left to the scheduler: asking for them
// first bunched the first MFMAs behind them).
constexpr int KV_NV = 5;   // VALU instructions requested between two MFMAs
// Region A (no VALU): its 16 MFMAs with the 32 transposing reads of the
// next block's fragments, two per MFMA; region D with the next pair's
// fragment reads, one per MFMA.
template <int NDS>
__device__ __forceinline__ void interleave_mfma_lds() {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, NDS, 0);
  }
}
__device__ __forceinline__ void interleave_mfma_valu() {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x002, KV_NV, 0);
  }
}

// One pair of subtiles (rows base..base+63 of the tile), in four fenced
// regions so that each block of 16 MFMAs shares its region with VALU work it
// does not depend on:
//   A: S/dP products of the upper subtile
//   B: S/dP products of the lower subtile   | P, dS of the upper subtile
//   C: dV/dK products of the upper subtile  | P, dS of the lower subtile
//   D: dV/dK products of the lower subtile
// The LDS fragments of each block are read one region ahead; fa holds the
// upper subtile's S / dP fragments on entry, and with PF it is refilled
// during region D (which has no other LDS reads) with those of the next
// pair of the tile.  Regions A and D each begin with 2 NB blocks of the next
// tile's copies, from `blk` on.  The lower subtile is computed even where only
// the upper one is needed: the diagonal mask then zeroes all of its P and dS.
// So is a pair that this wave's keys do not see at all; its dV / dK products then
// read the tile's upper pair (Tile::dvdk), which the wave computes anyway:
// what a zero P or dS does to those rows is done already, where a row of the
// masked pair that holds an infinity or NaN would give 0 x NaN.
template <bool CAUSAL, bool PF, int NB, class Copy, class Tile>
__device__ __forceinline__ void pair_step(const Copy& next, int blk, const Tile& tile, int base,
                                          uint32_t qb, uint32_t kw, uint32_t mykey, int g,
                                          const bf16x8 (&kf)[8], const bf16x8 (&vf)[8],
                                          f32x16 (&dva)[4], f32x16 (&dka)[4], Frags& fa) {
  Frags fb;
  f32x16 s1, p1, s0, p0;
  bf16x8 pf1[2], sf1[2], pf0[2], sf0[2];
  const uint32_t q1 = qb + base + 32, q0 = qb + base;
  subtile_seed(tile.buf, base + 32, g, s1, p1);
  subtile_seed(tile.buf, base, g, s0, p0);
  __builtin_amdgcn_sched_barrier(0);
  tile.sdp(base, fb);
  __builtin_amdgcn_sched_barrier(0);
  next.blocks(blk, 2 * NB);
  subtile_sdp(fa, kf, vf, s1, p1);                                            // A
  tile.dvdk(base + 32, fa);
  interleave_mfma_lds<2>();
  __builtin_amdgcn_sched_barrier(0);
  subtile_sdp(fb, kf, vf, s0, p0);                                            // B
  subtile_pds(s1, p1, pf1, sf1);
  interleave_mfma_valu();
  __builtin_amdgcn_sched_barrier(0);
  subtile_mask<CAUSAL>(q1, mykey, q1 < kw + 31, g, pf1, sf1);
  dvdk_products(fa, pf1, sf1, dva, dka);                                      // C
  tile.dvdk(base, fb);
  subtile_pds(s0, p0, pf0, sf0);
  interleave_mfma_valu();
  __builtin_amdgcn_sched_barrier(0);
  subtile_mask<CAUSAL>(q0, mykey, q0 < kw + 31, g, pf0, sf0);
  next.blocks(blk + 2 * NB, 2 * NB);
  dvdk_products(fb, pf0, sf0, dva, dka);                                      // D
  if (PF) {   // the next pair's upper subtile
    tile.sdp(base - 32, fa);
    interleave_mfma_lds<1>();
  }
}

}  // namespace

}  // namespace upipe
