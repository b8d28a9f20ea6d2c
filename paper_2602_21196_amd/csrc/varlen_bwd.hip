// Attention backward over packed sequences of different lengths, for gfx950.
//
//   P_ij  = exp(q_i.k_j / sqrt d - lse_i),   D_i = dO_i . o_i,
//   dS_ij = P_ij (dO_i . v_j - D_i),         dV_j = sum_i P_ij dO_i,
//   dK_j  = sum_i dS_ij q_i / sqrt d,        dQ_i = sum_j dS_ij k_j / sqrt d
// over the visible pairs of each sequence; P and dS are rounded to bf16 for their
// products (as the matrix instructions take them), all sums are fp32.  The rows of
// a key/value group are packed (varlen.h), so dK and dV sum over the group's heads by
// walking its rows.  No atomics: every sum has a fixed order.
//   dq:    a workgroup owns 256, 128 or 64 packed rows (or 128 with four waves, two of them
//          a CU: the forward's reasons), forms their terms, D and
//          -sqrt(d) lse, which it leaves for dkdv, and walks stages of keys
//   dkdv:  a workgroup owns 128 keys of one key/value head and walks the tiles of
//          rows that see them, from the last one down; long walks are cut into
//          segments side by side, whose sums are added in their order
// The products of a tile are those of the backward over equal lengths
// (attn_bwd_tile.h).  MFMA-bound: 131072 tokens, 4 heads on 1: dQ 20.9, dK/dV 30.0 - 31.1
// ms (20.4 and 30.8 there); 65536 tokens in documents of up to 32768, 8 heads on 1: 3.3
// and 4.8 ms.  Short batches: a chain of tiles and launches (2048 tokens in documents of
// up to 700, 4 heads: 15 and 17 us).
#include "attn_bwd_tile.h"
#include "varlen.h"

namespace upipe {

namespace {

// ------------------------------------------------------------------ dK / dV
// The copies of one tile by one wave, as the products' kernel wants them
// (attn_bwd_tile.h): KV_BLK blocks of four rows of Q and of dO, and the row terms.  A
// lane's places in a tile are the same for all tiles and kept.  INSIDE: the rows of a
// token do not reach into the next token's, so what lies behind the last token is cut off
// by the sources' sizes; else (head-major rows) every lane asks (65536 tokens in documents,
// 8 heads: 4.91 | 5.02 ms).
template <bool INSIDE>
struct RowCopy {
  i32x4 q, dO, lse, D;       // of the tile
  uint32_t at_q[KV_BLK], at_d[KV_BLK];     // this lane's 16 bytes of every block
  uint32_t per_g;            // ceil(2^16 / G)
  int tokens;                // valid tokens of the tile
  uint32_t lds;
  int w;

  __device__ __forceinline__ void init(int wave, int lane, int G, const HeadView& Q,
                                       const HeadView& dOv) {
    w = wave;
    per_g = (65536 + G - 1) / G;
#pragma unroll
    for (int i = 0; i < KV_BLK; ++i) {
      const uint32_t r = 4 * (KV_BLK * w + i) + (lane >> 4);
      const uint32_t t = (r * per_g) >> 16, h = r - t * G;      // r / G for r < 128
      const uint32_t c = ((lane & 15) ^ tsw(r)) << 4;
      at_q[i] = (t * (uint32_t)Q.row + h * (uint32_t)Q.head) * 2 + c;
      at_d[i] = (t * (uint32_t)dOv.row + h * (uint32_t)dOv.head) * 2 + c;
    }
  }
  // Blocks i0 .. i0 + n - 1 of this wave's (both even).
  __device__ __forceinline__ void blocks(int i0, int n) const {
    auto ok = [&](int i) {
      const uint32_t r = 4 * (KV_BLK * w + i) + ((threadIdx.x & 63) >> 4);
      return INSIDE || (int)((r * per_g) >> 16) < tokens;      // else no row: zeros
    };
#pragma unroll
    for (int i = i0; i < i0 + n; i += 2) {
      const bool ok0 = ok(i), ok1 = ok(i + 1);
      copy2x2_b128<OFF_DO - OFF_Q>(q, dO, ok0 ? at_q[i] : 0x80000000u,
                                   ok1 ? at_q[i + 1] : 0x80000000u, ok0 ? at_d[i] : 0x80000000u,
                                   ok1 ? at_d[i + 1] : 0x80000000u,
                                   lds + OFF_Q + (KV_BLK * w + i) * 1024);
    }
  }
  __device__ __forceinline__ void rows(int lane) const {
    if (lane < QT / 4) {
      if (w == 0) copy_b128(lse, lane * 16u, 0, lds + OFF_LSE);
      else if (w == 1) copy_b128(D, lane * 16u, 0, lds + OFF_D);
    }
  }
};

// A staged tile by two per-lane places and exclusive-ors (common.h): a register for
// every address would spill.
struct PlacedTile {
  const char *buf, *smem;
  uint32_t sdp_at, tr;       // of this lane's chunk of row r32, of its transposing reads
  __device__ __forceinline__ void sdp(int sub, Frags& fr) const {
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      fr.f[2 * s] = lds_read_b128(smem, (sdp_at ^ (32 * s)) + OFF_Q + sub * 256);
      fr.f[2 * s + 1] = lds_read_b128(smem, (sdp_at ^ (32 * s)) + OFF_DO + sub * 256);
    }
  }
  __device__ __forceinline__ void dvdk(int sub, Frags& fr) const {
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        fr.f[4 * dt + 2 * kt] = tr_operand_at(smem, tr, sub + 16 * kt + OFF_DO / 256, dt);
        fr.f[4 * dt + 2 * kt + 1] = tr_operand_at(smem, tr, sub + 16 * kt + OFF_Q / 256, dt);
      }
  }
};

template <bool INSIDE>
__global__ __launch_bounds__(256, 1) void rows_dkdv_kernel(RowBwdArgs a) {
  __shared__ __attribute__((aligned(1024))) char smem[2 * KV_STAGE];
  const int t = threadIdx.x;
  const int lane = t & 63;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int r32 = lane & 31, g = lane >> 5;
  const int kvh = blockIdx.x % a.Hkv, G = a.G, tpt = tile_tokens(G);
  const KeyItem it = a.keys[blockIdx.x / a.Hkv];
  const int kw = 128 * it.kb + 32 * w, mykey = kw + r32;
  // First packed row that sees a key: the diagonal, within the sequence's rows.
  auto first_row = [&](int key) {
    return (uint32_t)(a.causal ? min(max(key - (it.Lk - it.Lq), 0), it.Lq) * G : 0);
  };
  const uint32_t sees_w0 = first_row(kw), sees_w31 = first_row(kw + 31), sees = first_row(mykey);

  const uint32_t lds0 = lds_address(smem);
  RowCopy<INSIDE> next;
  next.init(w, lane, G, a.q, a.dO);
  const bf16* qh = a.q.p + it.q0 * a.q.row + kvh * G * a.q.head;
  const bf16* dh = a.dO.p + it.q0 * a.dO.row + kvh * G * a.dO.head;
  const float* lh = a.lse_c + kvh * a.term_rows + it.r0;
  const float* Dh = a.D + kvh * a.term_rows + it.r0;
  // Tile qt to the stage at `lds`; past the walk's end tile 0 with sizes of none (zeros).
  // INSIDE: sizes up to the end of the last token's rows.
  const uint32_t q_row = (uint32_t)a.q.row * 2, d_row = (uint32_t)a.dO.row * 2;
  const uint32_t q_in = (uint32_t)((G - 1) * a.q.head + HEAD_DIM) * 2;
  const uint32_t d_in = (uint32_t)((G - 1) * a.dO.head + HEAD_DIM) * 2;
  auto aim = [&](int qt, bool some, uint32_t lds) {
    const uint32_t on = some ? 0xffffffffu : 0u;
    const int tile = qt & (int)on;
    const int64_t tok = (int64_t)tile * tpt;
    next.tokens = min(tpt, it.Lq - (int)tok);
    next.q = rsrc_words(qh + tok * a.q.row,
                        (INSIDE ? (next.tokens - 1) * q_row + q_in : 0x7fffffffu) & on);
    next.dO = rsrc_words(dh + tok * a.dO.row,
                         (INSIDE ? (next.tokens - 1) * d_row + d_in : 0x7fffffffu) & on);
    // rows without a token have no terms: zeros
    next.lse = rsrc_words(lh + (int64_t)tile * QT, (uint32_t)(next.tokens * G * 4) & on);
    next.D = rsrc_words(Dh + (int64_t)tile * QT, (uint32_t)(next.tokens * G * 4) & on);
    next.lds = lds;
  };
  aim(it.first, it.count > 0, lds0);
  next.rows(lane);
  next.blocks(0, KV_BLK);

  // K and -V B-operand fragments (lane = key column, k = head dim); -V makes
  // the dP products count down from D.  Keys past the last repeat it; their sums
  // are not used.
  bf16x8 kf[8], vf[8];
  {
    const int64_t key = it.k0 + min(mykey, it.Lk - 1);
    const bf16* kp = a.k.p + key * a.k.row + kvh * a.k.head + 8 * g;
    const bf16* vp = a.v.p + key * a.v.row + kvh * a.v.head + 8 * g;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      kf[s] = *reinterpret_cast<const bf16x8*>(kp + 16 * s);
      vf[s] = -*reinterpret_cast<const bf16x8*>(vp + 16 * s);
    }
    // Only ever MFMA operands, which may come from AGPRs: the VGPRs are left to
    // the score accumulators and the P / dS arithmetic.
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      asm volatile("" : "+a"(kf[s]));
      asm volatile("" : "+a"(vf[s]));
    }
  }
  // C layout: lane = head-dim column 32*dt + r32, element i = key row
  // kw + 8*(i/4) + 4*g + (i%4).
  f32x16 dka[4], dva[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      dka[dt][i] = 0.f;
      dva[dt][i] = 0.f;
    }
  // Zeros that the compiler does not know for zeros: knowing them it keeps half of the
  // sums in VGPRs, swaps them with AGPRs in every tile and spills addresses (dK/dV of
  // 131072 rows of 4 heads 37.8 ms).
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) asm volatile("" : "+a"(dka[dt]), "+a"(dva[dt]));

  const uint32_t sdp_lane = swzt(r32, g), tr_lane = tr_base(lane);
  for (int n = 0; n < it.count; ++n) {
    const char* buf = smem + (n & 1) * KV_STAGE;
    const uint32_t qb = (uint32_t)(it.first - n) * (tpt * G);    // first row of the tile
    wait_vmem();
    __syncthreads();   // this tile landed for all waves; the other buffer is free
    aim(it.first - n - 1, n + 1 < it.count, lds0 + ((n + 1) & 1) * KV_STAGE);
    next.rows(lane);
    // Pairs of 32-row subtiles, upper rows first.  A pair that this wave's keys do not
    // see is computed too, masked whole, on the rows of the other pair.
    const uint32_t boff = (n & 1) * KV_STAGE;
    PlacedTile upper{buf, smem, sdp_lane + boff, tr_lane + boff}, lower = upper;
    if (qb + 63 < sees_w0) lower.tr += 64 * HEAD_DIM * 2;
    Frags fa;
    upper.sdp(96, fa);
    pair_step<true, true, 1>(next, 0, upper, 64, qb, sees_w31 - 31, sees, g, kf, vf, dva, dka, fa);
    pair_step<true, false, 1>(next, 4, lower, 0, qb, sees_w31 - 31, sees, g, kf, vf, dva, dka, fa);
  }

  wait_vmem();      // the last tile's empty copies (to LDS) have ended
  if (it.slot >= 0) {
    float* pk = a.sums + (kvh * a.slots + it.slot) * (2 * 128 * HEAD_DIM) + 32 * w * HEAD_DIM;
    float* pv = pk + 128 * HEAD_DIM;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t off = (8 * (i >> 2) + 4 * g + (i & 3)) * HEAD_DIM + 32 * dt + r32;
        pk[off] = dka[dt][i];
        pv[off] = dva[dt][i];
      }
    return;
  }
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int key = kw + 8 * (i >> 2) + 4 * g + (i & 3);
      if (key < it.Lk) {
        const int64_t at = it.k0 + key;
        a.dk.p[at * a.dk.row + kvh * a.dk.head + 32 * dt + r32] = (bf16)(dka[dt][i] * -kScale);
        a.dv.p[at * a.dv.row + kvh * a.dv.head + 32 * dt + r32] = (bf16)dva[dt][i];
      }
    }
}

// The segments' sums of a key block, added in the order of its walk: 16 workgroups a
// block, a thread has eight consecutive elements of one key's dK or dV.
__global__ __launch_bounds__(256) void rows_dkdv_fold_kernel(RowBwdArgs a) {
  const int kvh = blockIdx.y;
  const FoldItem it = a.folds[blockIdx.x / 16];
  const int e8 = ((blockIdx.x % 16) * 256 + threadIdx.x) * 8;      // in [2][128][128]
  const float* p = a.sums + (kvh * a.slots + it.slot) * (2 * 128 * HEAD_DIM) + e8;
  f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
#pragma unroll 4
  for (int i = 0; i < it.n; ++i, p += 2 * 128 * HEAD_DIM) {
    lo += *reinterpret_cast<const f32x4*>(p);
    hi += *reinterpret_cast<const f32x4*>(p + 4);
  }
  const bool is_v = e8 >= 128 * HEAD_DIM;
  const int key = 128 * it.kb + (e8 / HEAD_DIM) % 128, e = e8 % HEAD_DIM;
  if (key >= it.Lk) return;
  const float f = is_v ? 1.f : -kScale;
  bf16x8 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    out[i] = (bf16)(lo[i] * f);
    out[4 + i] = (bf16)(hi[i] * f);
  }
  const HeadView& d = is_v ? a.dv : a.dk;
  *reinterpret_cast<bf16x8*>(d.p + (it.k0 + key) * d.row + kvh * d.head + e) = out;
}

// ---------------------------------------------------------------------- dQ
// Eight waves of 32 packed rows x a part of every stage's keys: 256 rows x 64-key
// stages, or, with the keys of 128-key stages in 2 or 4 parts, 128 or 64 rows, whose
// sums are added in fp32 through LDS.  Four waves: 128 rows x 64-key stages.
template <int KS, int NW>
struct DqTile {
  static constexpr int NQW = NW / KS;               // waves along the rows
  static constexpr int BQ = 32 * NQW;               // rows per workgroup
  static constexpr int BK = KS == 1 ? 64 : 128;     // keys per stage
  static constexpr int NH = BK / 32 / KS;           // 32-key blocks of a stage per wave
  static constexpr int T = BK * HEAD_DIM * 2;
  static constexpr int OFF_K = 0, OFF_V = T;
  static constexpr int STAGE = 2 * T;
  static constexpr int BLK = T / 1024 / NW;         // 1 KB blocks per wave per tensor
};
constexpr int DQ_LA = 4;     // K/V fragment reads kept in flight
// D of the rows that see no more keys than these, one block of products, comes from
// the weights themselves, and dK/dV after this kernel uses it: o carries half a step of
// bf16 and the steps of the weights that formed it, and where few keys share the weight
// dP - D cancels to little more than that.  Documents of 1 to 700 tokens: dQ and dK
// 2.4e-3 off instead of 2.6e-3 (2.3e-3 are the roundings of dS and of the result).
constexpr int kFewKeys = 32;

template <int KS, int NW>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 1 : 2) void rows_dq_kernel(RowBwdArgs a) {
  using T = DqTile<KS, NW>;
  __shared__ __attribute__((aligned(1024))) char smem[2 * T::STAGE];
  const int t = threadIdx.x;
  const int lane = t & 63;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wq = KS == 1 ? w : w % T::NQW, ks = KS == 1 ? 0 : w / T::NQW;
  const int r32 = lane & 31, g = lane >> 5;
  const int kvh = blockIdx.x % a.Hkv, G = a.G;
  const TileItem it = a.dqs[blockIdx.x / a.Hkv];
  const int n_rows = it.Lq * G, delta = it.Lk - it.Lq;
  const int r0 = it.tile * T::BQ, rw = r0 + 32 * wq;
  const int row = min(rw + r32, n_rows - 1);     // rows past the last compute on it
  const int tok = row / G, hg = row - tok * G;

  const uint32_t kb_row = (uint32_t)(a.k.row * 2), vb_row = (uint32_t)(a.v.row * 2);
  const bf16* kp = a.k.p + it.k0 * a.k.row + kvh * a.k.head;
  const bf16* vp = a.v.p + it.k0 * a.v.row + kvh * a.v.head;
  const uint32_t lds0 = lds_address(smem);
  uint32_t offk[T::BLK], offv[T::BLK];
#pragma unroll
  for (int i = 0; i < T::BLK; ++i) {
    const int r = 4 * (T::BLK * w + i) + (lane >> 4);      // row of the tile, 16 lanes per row
    const uint32_t c = ((lane & 15) ^ tsw(r)) << 4;
    offk[i] = r * kb_row + c;
    offv[i] = r * vb_row + c;
  }
  auto last_key = [&](int tk) { return a.causal ? min(tk + delta, it.Lk - 1) : it.Lk - 1; };
  const int seen = last_key((min(r0 + T::BQ, n_rows) - 1) / G) + 1;
  const int nst = max(0, (seen + T::BK - 1) / T::BK);
  auto source = [&](const bf16* p, int64_t row_elems, int j) {
    const int n = j < nst ? min(T::BK, it.Lk - j * T::BK) : 0;
    return rsrc_words(p + (int64_t)j * T::BK * row_elems,
                      n > 0 ? (uint32_t)((n - 1) * (int)row_elems + HEAD_DIM) * 2 : 0);
  };
  auto issue = [&](i32x4 rk, i32x4 rv, int i, uint32_t lds) {
    copy2x2_b128<T::OFF_V - T::OFF_K>(rk, rv, offk[i], offk[i + 1], offv[i], offv[i + 1],
                                      lds + T::OFF_K + (T::BLK * w + i) * 1024);
  };
  {
    const i32x4 rk = source(kp, a.k.row, 0), rv = source(vp, a.v.row, 0);
#pragma unroll
    for (int i = 0; i < T::BLK; i += 2) issue(rk, rv, i, lds0);
  }

  // The row's terms: for dkdv too, in tiles of 128 rows.  A row that sees no key has zeros:
  // every pair of its is masked, and zeros keep what is masked finite.
  auto put_term = [&](float* to, float x) {
    const int tpt = tile_tokens(G);
    if (ks == 0 && g == 0 && rw + r32 < n_rows)
      to[kvh * a.term_rows + it.r0 + (int64_t)(tok / tpt) * 128 + (tok % tpt) * G + hg] = x;
  };
  const int lim = last_key(tok), lim_w = last_key(rw / G);
  bf16x8 qf[8], df[8];
  float nlse, Dq = 0.f;   // nlse = -sqrt(d) lse: the score accumulator's seed
  {
    const int h = kvh * G + hg;
    const bf16* qp = a.q.p + (it.q0 + tok) * a.q.row + h * a.q.head + 8 * g;
    const bf16* dp = a.dO.p + (it.q0 + tok) * a.dO.row + h * a.dO.head + 8 * g;
    const bf16* op = a.o.p + (it.q0 + tok) * a.o.row + h * a.o.head + 8 * g;
    const float l = a.lse[h * a.lse_head + it.q0 + tok];
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      qf[s] = *reinterpret_cast<const bf16x8*>(qp + 16 * s);
      df[s] = *reinterpret_cast<const bf16x8*>(dp + 16 * s);
      const bf16x8 of = *reinterpret_cast<const bf16x8*>(op + 16 * s);
#pragma unroll
      for (int e = 0; e < 8; ++e) Dq = fmaf((float)df[s][e], (float)of[e], Dq);
    }
    Dq += __shfl_xor(Dq, 32);
    const bool none = l == -INFINITY;
    nlse = none ? 0.f : l * -11.313708498984761f;     // -sqrt(128) lse
    if (none) Dq = 0.f;
    put_term(a.lse_c, nlse);
    if (lim < 0 || lim >= kFewKeys) put_term(a.D, Dq);
  }

  f32x16 qacc[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) qacc[dt][i] = 0.f;

  const int k_part = 32 * T::NH * ks;        // first key of this wave's part of a stage
  const uint32_t k_lane = T::OFF_K + k_part * 256 + swzt(r32, g);
  const uint32_t v_lane = T::OFF_V + k_part * 256 + swzt(r32, g);
  const uint32_t t_lane = T::OFF_K + k_part * 256 + tr_base(lane);
  // Stages with a key of this wave's part that a row of it may see come first.
  const int seen_w = last_key((min(rw + 32, n_rows) - 1) / G) + 1;
  const int nw = rw >= n_rows ? 0 : max(0, min(nst, (seen_w - k_part + T::BK - 1) / T::BK));
  int j = 0;
  for (; j < nw; ++j) {
    const uint32_t boff = (j & 1) * T::STAGE;
    wait_vmem();
    __syncthreads();   // tile j landed for all waves; tile j-1's buffer is free
    const uint32_t nlds = lds0 + ((j + 1) & 1) * T::STAGE;
    const i32x4 nk = source(kp, a.k.row, j + 1), nv = source(vp, a.v.row, j + 1);
    const int kb = j * T::BK + k_part;
    const bool diag = kb + 32 * T::NH - 1 > lim_w;
    // 32 keys at a time: one score and one dP accumulator live at a time, which leaves
    // registers for DQ_LA fragment reads in flight ahead of the S / dP MFMAs.  The
    // fragment addresses are exclusive-ors of three bases.
    const uint32_t ka = k_lane + boff, va = v_lane + boff, ta = t_lane + boff;
#pragma unroll
    for (int hh = 0; hh < T::NH; ++hh) {
      f32x16 sacc, pacc;
#pragma unroll
      for (int i = 0; i < 16; ++i) { sacc[i] = nlse; pacc[i] = 0.f; }
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        sacc = mfma32x32x16(lds_read_b128(smem, (ka ^ (32 * s)) + 8192 * hh), qf[s], sacc);
        pacc = mfma32x32x16(lds_read_b128(smem, (va ^ (32 * s)) + 8192 * hh), df[s], pacc);
      }
      __builtin_amdgcn_sched_group_barrier(0x100, DQ_LA, 0);
#pragma unroll
      for (int i = 0; i < 16 - DQ_LA; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, DQ_LA, 0);
      // The next tile's copies go out behind the products they can hide behind.
      if (hh == 0) issue(nk, nv, 0, nlds);
      if (T::BLK > 2 && hh == T::NH - 1) issue(nk, nv, 2, nlds);
      if (hh == 0 && kb == 0 && lim_w < kFewKeys) {
        // All that the first rows see are these keys: D = sum_j P_ij dP_ij.
        float d = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (8 * (i >> 2) + 4 * g + (i & 3) <= lim)
            d = fmaf(fast_exp2(sacc[i] * kSl2), pacc[i], d);
        d += __shfl_xor(d, 32);
        if (lim >= 0 && lim < kFewKeys) {
          Dq = d;
          put_term(a.D, d);
        }
      }
      float ds[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) ds[i] = fast_exp2(sacc[i] * kSl2) * (pacc[i] - Dq);
      if (diag) {   // wave-uniform; by selection: masked, they may be inf or NaN
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (kb + 32 * hh + 8 * (i >> 2) + 4 * g + (i & 3) > lim) ds[i] = 0.f;
      }
      bf16x8 sf[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) sf[i >> 3][i & 7] = (bf16)ds[i];
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
          qacc[dt] =
              mfma32x32x16(tr_operand_at(smem, ta, 32 * hh + 16 * c, dt), sf[c], qacc[dt]);
    }
  }
  // The others: only this wave's share of the copies.
  for (; j < nst; ++j) {
    wait_vmem();
    __syncthreads();
    const i32x4 nk = source(kp, a.k.row, j + 1), nv = source(vp, a.v.row, j + 1);
#pragma unroll
    for (int i = 0; i < T::BLK; i += 2) issue(nk, nv, i, lds0 + ((j + 1) & 1) * T::STAGE);
  }
  wait_vmem();       // the last stage's empty copies (to LDS) have ended
  if (KS > 1) {
    // Add the KS parts' sums in ascending key order: parts 1.. pass theirs through
    // the stage buffers (16 KB per wave).
    float* fold = reinterpret_cast<float*>(smem);
    __syncthreads();   // every wave is done reading the last stage
    if (ks > 0) {
      float* mine = fold + ((ks - 1) * T::NQW + wq) * 4096 + lane * 4;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f32x4 v;
#pragma unroll
          for (int b = 0; b < 4; ++b) v[b] = qacc[dt][4 * i + b];
          *reinterpret_cast<f32x4*>(mine + (4 * dt + i) * 256) = v;
        }
    }
    __syncthreads();
    if (ks > 0) return;
#pragma unroll
    for (int p = 1; p < KS; ++p) {
      const float* part = fold + ((p - 1) * T::NQW + wq) * 4096 + lane * 4;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(part + (4 * dt + i) * 256);
#pragma unroll
          for (int b = 0; b < 4; ++b) qacc[dt][4 * i + b] += v[b];
        }
    }
  }
  if (rw + r32 >= n_rows) return;
  bf16* op = a.dq.p + (it.q0 + tok) * a.dq.row + (kvh * G + hg) * a.dq.head + 4 * g;
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bf16x4 ov;
#pragma unroll
      for (int b = 0; b < 4; ++b) ov[b] = (bf16)(qacc[dt][4 * i + b] * kScale);
      *reinterpret_cast<bf16x4*>(op + 32 * dt + 8 * i) = ov;
    }
}

}  // namespace

hipError_t launch_rows_dkdv(const RowBwdArgs& a, int64_t n, hipStream_t st) {
  auto inside = [&](const HeadView& v) { return v.row >= (a.G - 1) * v.head + HEAD_DIM; };
  return enqueue(inside(a.q) && inside(a.dO) ? rows_dkdv_kernel<true> : rows_dkdv_kernel<false>,
                 dim3((unsigned)(n * a.Hkv)), 256, st, a);
}

hipError_t launch_rows_dkdv_fold(const RowBwdArgs& a, int64_t n, hipStream_t st) {
  return enqueue(rows_dkdv_fold_kernel, dim3((unsigned)(n * 16), (unsigned)a.Hkv), 256, st, a);
}

hipError_t launch_rows_dq(int ks, bool half, const RowBwdArgs& a, int64_t n, hipStream_t st) {
  const dim3 grid((unsigned)(n * a.Hkv));
  if (half) return enqueue(rows_dq_kernel<1, 4>, grid, 256, st, a);
  return enqueue(ks == 1   ? rows_dq_kernel<1, 8>
                 : ks == 2 ? rows_dq_kernel<2, 8>
                           : rows_dq_kernel<4, 8>,
                 grid, 512, st, a);
}

}  // namespace upipe
