// RMS norm of every query and key head with the rotary embedding behind it, in
// one pass, and its gradients.
//
// A row x of 128 elements (one head of one token) at position p, with weights w:
//   r = (mean x^2 + eps)^(-1/2),   y = R(p) (r x w)
// where R(p) turns the pairs (e, e + 64) as in upipe_rope.  Backward, from dy:
//   g = R(p)^T dy,   a = g w,   dw += g n (over all rows),
//   dx = r (a - n mean(a n)) with n = r x
// r is formed again in the backward: it comes out of the row that is read anyway.
//
// HBM-bound: x is read once and y written (backward: x and dy read, dx written).  Eight
// lanes hold a row, lane j the elements 8j.. and 64 + 8j.., so a pair lies in one lane
// and a wave reads whole 128-byte lines.  The pairs of heads of all tokens of q, then
// those of k, are dealt out to workgroups, one tensor to each, so a thread holds one
// tensor's 16 weights (and its 16 sums of dw).  The angles are formed once per token and
// pair of heads, in fp64 turns (positions to 2^32) with the frequencies from the
// kernel's arguments.  The norm's sums, r, the rotation and the sums of dw are fp32; y,
// dx and a bf16 dw are rounded once.  65536 tokens: 40 heads forward 247 - 252 us (5.3 - 5.4
// TB/s, a large copy 5.1), 72 heads backward 690 - 708 us (5.1 - 5.2 TB/s; a head at a time
// 742); 4000 tokens, 40 heads 17 and 27 us (before the weights came by wide loads and
// without 64-bit divisions 22 and 31).
#include "common.h"
#include "kernels.h"

namespace upipe {

namespace {

constexpr int kPairsPerBlock = 32;    // 256 threads, 8 lanes a row, a pair of heads at a time

__device__ __forceinline__ float sum8(float v) {
#pragma unroll
  for (int off = 4; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

// A lane's 16 of a row's 128 elements.
struct Row16 {
  bf16x8 lo, hi;
};
__device__ __forceinline__ Row16 load_row(const bf16* p) {
  return {*reinterpret_cast<const bf16x8*>(p), *reinterpret_cast<const bf16x8*>(p + 64)};
}

// This lane's 16 weights.
template <bool W32>
__device__ __forceinline__ void load_weights(const void* w, int j, float (&out)[16]) {
  if (W32) {
    const f32x4* p = static_cast<const f32x4*>(w) + 2 * j;
    const f32x4 v[4] = {p[0], p[1], p[16], p[17]};
#pragma unroll
    for (int e = 0; e < 16; ++e) out[e] = v[e >> 2][e & 3];
  } else {
    const Row16 v = load_row(static_cast<const bf16*>(w) + 8 * j);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      out[e] = (float)v.lo[e];
      out[8 + e] = (float)v.hi[e];
    }
  }
}

// The pairs of heads of one tensor that this lane group takes: pair first, first +
// step, ... (both in 32 bits), as token t < T and pair p of it.
struct PairWalk {
  int64_t t;
  int p, pairs, t_step, p_step;
  __device__ __forceinline__ PairWalk(uint32_t first, uint32_t step, int H) {
    pairs = (H + 1) / 2;
    t = first / (uint32_t)pairs;
    p = first - (uint32_t)t * pairs;
    t_step = step / (uint32_t)pairs;
    p_step = step - t_step * pairs;
  }
  __device__ __forceinline__ void next() {
    t += t_step;
    p += p_step;
    if (p >= pairs) {
      p -= pairs;
      ++t;
    }
  }
};

// This lane's angles at a position: cos and sin of its eight pairs.
__device__ __forceinline__ void angles(double pos, const double (&f)[8], float (&c)[8],
                                       float (&s)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const double turns = pos * f[e];
    cos_sin_turns((float)(turns - rint(turns)), c[e], s[e]);
  }
}

// The workgroup's tensor, its number among that tensor's and their count.
__device__ __forceinline__ const NormRopeSide& side_of(const NormRopeArgs& a, int& block,
                                                       int& blocks) {
  const bool is_q = (int)blockIdx.x < a.blocks_q;
  block = is_q ? blockIdx.x : blockIdx.x - a.blocks_q;
  blocks = is_q ? a.blocks_q : gridDim.x - a.blocks_q;
  return is_q ? a.q : a.k;
}

template <bool W32>
__global__ __launch_bounds__(256) void norm_rope_kernel(NormRopeArgs a) {
  int block, blocks;
  const NormRopeSide& s = side_of(a, block, blocks);
  const int j = threadIdx.x & 7;
  PairWalk it(block * kPairsPerBlock + (threadIdx.x >> 3), blocks * kPairsPerBlock, s.H);
  if (it.t >= a.T) return;
  const bf16* x0 = s.x.p + 8 * j;
  bf16* y0 = s.y.p + 8 * j;
  // The rows of the walk's pair (an odd last head twice), past its end those of the last
  // token, which go unused; a pair ahead (16000 tokens, 40 heads 62 -> 60.5 us; the
  // backward's registers do not hold it: 708 -> 727).
  auto load = [&](Row16 (&x)[2], int64_t& pos) {
    const int64_t t = min(it.t, a.T - 1);
    const bf16* xp = x0 + t * s.x.row;
    x[0] = load_row(xp + 2 * it.p * s.x.head);
    x[1] = load_row(xp + min(2 * it.p + 1, s.H - 1) * s.x.head);
    pos = a.positions[t];
  };
  Row16 next[2];
  int64_t next_pos;
  load(next, next_pos);
  float w[16];
  load_weights<W32>(s.w, j, w);
  double f[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = a.freq.turns[8 * j + e];
  while (it.t < a.T) {
    const int64_t t = it.t;
    const int h = 2 * it.p, n = min(2, s.H - h);
    const Row16 x[2] = {next[0], next[1]};
    const double pos = (double)next_pos;
    it.next();
    load(next, next_pos);
    float c[8], sn[8];
    angles(pos, f, c, sn);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (u >= n) break;
      float v[16], ss = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = (float)x[u].lo[e];
        v[8 + e] = (float)x[u].hi[e];
        ss = fmaf(v[e], v[e], ss);
        ss = fmaf(v[8 + e], v[8 + e], ss);
      }
      const float r = __frsqrt_rn(fmaf(sum8(ss), 1.f / HEAD_DIM, a.eps));
      Row16 y;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float p = v[e] * r * w[e], q = v[8 + e] * r * w[8 + e];
        rope_pair(p, q, c[e], sn[e], false);
        y.lo[e] = (bf16)p;
        y.hi[e] = (bf16)q;
      }
      bf16* yp = y0 + t * s.y.row + (h + u) * s.y.head;
      *reinterpret_cast<bf16x8*>(yp) = y.lo;
      *reinterpret_cast<bf16x8*>(yp + 64) = y.hi;
    }
  }
}

// dx of every row, and each workgroup's sums of dw to partial[block][128].
template <bool W32>
__global__ __launch_bounds__(256) void norm_rope_bwd_kernel(NormRopeArgs a,
                                                            float* __restrict__ partial) {
  __shared__ float sums[4][HEAD_DIM];
  int block, blocks;
  const NormRopeSide& s = side_of(a, block, blocks);
  const int j = threadIdx.x & 7;
  PairWalk it(block * kPairsPerBlock + (threadIdx.x >> 3), blocks * kPairsPerBlock, s.H);
  const bf16* x0 = s.x.p + 8 * j;
  const bf16* d0 = s.dy.p + 8 * j;
  bf16* y0 = s.y.p + 8 * j;
  float w[16], dw[16];
  load_weights<W32>(s.w, j, w);
  double f[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = a.freq.turns[8 * j + e];
#pragma unroll
  for (int e = 0; e < 16; ++e) dw[e] = 0.f;
  for (; it.t < a.T; it.next()) {
    const int h = 2 * it.p, n = min(2, s.H - h);
    const bf16* xp = x0 + it.t * s.x.row + h * s.x.head;
    const bf16* dp = d0 + it.t * s.dy.row + h * s.dy.head;
    Row16 x[2], d[2];
    x[0] = load_row(xp);
    d[0] = load_row(dp);
    if (n > 1) {
      x[1] = load_row(xp + s.x.head);
      d[1] = load_row(dp + s.dy.head);
    }
    float c[8], sn[8];
    angles((double)a.positions[it.t], f, c, sn);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (u >= n) break;
      float v[16], g[16], ss = 0.f, ax = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = (float)x[u].lo[e];
        v[8 + e] = (float)x[u].hi[e];
        g[e] = (float)d[u].lo[e];
        g[8 + e] = (float)d[u].hi[e];
        rope_pair(g[e], g[8 + e], c[e], sn[e], true);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        ss = fmaf(v[e], v[e], ss);
        ax = fmaf(g[e] * w[e], v[e], ax);
      }
      const float r = __frsqrt_rn(fmaf(sum8(ss), 1.f / HEAD_DIM, a.eps));
      const float m = sum8(ax) * r * (1.f / HEAD_DIM);      // mean(a r x)
      Row16 y;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float nx = v[e] * r;
        dw[e] = fmaf(g[e], nx, dw[e]);
        const bf16 dx = (bf16)(r * fmaf(g[e], w[e], -nx * m));
        if (e < 8) y.lo[e] = dx;
        else y.hi[e - 8] = dx;
      }
      bf16* yp = y0 + it.t * s.y.row + (h + u) * s.y.head;
      *reinterpret_cast<bf16x8*>(yp) = y.lo;
      *reinterpret_cast<bf16x8*>(yp + 64) = y.hi;
    }
  }
  // The eight row groups of a wave, then the four waves, always in this order.
#pragma unroll
  for (int e = 0; e < 16; ++e) {
#pragma unroll
    for (int off = 8; off <= 32; off <<= 1) dw[e] += __shfl_xor(dw[e], off);
    if ((threadIdx.x & 56) == 0) sums[threadIdx.x >> 6][8 * j + (e & 7) + 64 * (e >> 3)] = dw[e];
  }
  __syncthreads();
  const int e = threadIdx.x;
  if (e < HEAD_DIM)
    partial[(int64_t)blockIdx.x * HEAD_DIM + e] =
        (sums[0][e] + sums[1][e]) + (sums[2][e] + sums[3][e]);
}

// dwq (blockIdx.y = 0) and dwk (1): the workgroups' sums added in fp64, in an order
// that the sizes alone fix, and rounded once.  A workgroup takes 16 elements, 64
// threads each, eight loads under way at a time (16 threads, one load: 19 us for 1001
// sums).
__global__ __launch_bounds__(1024) void norm_dw_fold_kernel(const float* __restrict__ partial,
                                                            int blocks_q, int blocks_k, void* dwq,
                                                            void* dwk, int w_fp32) {
  __shared__ double sums[64][17];
  const int e = threadIdx.x & 15, p = threadIdx.x >> 4, at = blockIdx.x * 16 + e;
  const bool is_q = blockIdx.y == 0;
  const float* from = partial + (is_q ? 0 : (int64_t)blocks_q * HEAD_DIM) + at;
  const int n = is_q ? blocks_q : blocks_k;
  double sum = 0.0;
  for (int b0 = p; b0 < n; b0 += 8 * 64) {
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int b = b0 + 64 * u;
      v[u] = from[(int64_t)min(b, n - 1) * HEAD_DIM];
      if (b >= n) v[u] = 0.f;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) sum += (double)v[u];
  }
  sums[p][e] = sum;
  __syncthreads();
  for (int half = 32; half >= 1; half >>= 1) {
    if (p < half) sums[p][e] += sums[p + half][e];
    __syncthreads();
  }
  if (p > 0) return;
  sum = sums[0][e];
  void* dw = is_q ? dwq : dwk;
  if (w_fp32) static_cast<float*>(dw)[at] = (float)sum;
  else static_cast<bf16*>(dw)[at] = (bf16)(float)sum;
}

}  // namespace

// Workgroups of one tensor's rows: every lane group has one pair of heads while that
// needs no more than `most` workgroups, and 2048 pairs at most: dw's fp32 sums are of up
// to 4096 rows each, whose rounding stays below 2^-12 of their terms.
static int norm_blocks(int64_t T, int H, int most) {
  const int64_t n = (T * ((H + 1) / 2) + kPairsPerBlock - 1) / kPairsPerBlock;
  const int64_t least = (n + 2047) / 2048;
  return (int)(n < most ? n : least > most ? least : most);
}

constexpr int kNormFwdBlocks = 4096, kNormBwdBlocks = 1024;

hipError_t launch_norm_rope(NormRopeArgs a, hipStream_t st) {
  a.blocks_q = norm_blocks(a.T, a.q.H, kNormFwdBlocks);
  const int blocks_k = norm_blocks(a.T, a.k.H, kNormFwdBlocks);
  return enqueue(a.w_fp32 ? norm_rope_kernel<true> : norm_rope_kernel<false>,
                 dim3((unsigned)(a.blocks_q + blocks_k)), 256, st, a);
}

int64_t norm_rope_bwd_partials(int64_t T, int Hq, int Hkv) {
  return norm_blocks(T, Hq, kNormBwdBlocks) + norm_blocks(T, Hkv, kNormBwdBlocks);
}

hipError_t launch_norm_rope_bwd(NormRopeArgs a, float* partial, hipStream_t st) {
  a.blocks_q = norm_blocks(a.T, a.q.H, kNormBwdBlocks);
  const int blocks_k = norm_blocks(a.T, a.k.H, kNormBwdBlocks);
  return enqueue(a.w_fp32 ? norm_rope_bwd_kernel<true> : norm_rope_bwd_kernel<false>,
                 dim3((unsigned)(a.blocks_q + blocks_k)), 256, st, a, partial);
}

hipError_t launch_norm_dw_fold(const float* partial, int64_t T, int Hq, int Hkv, void* dwq,
                               void* dwk, int w_fp32, hipStream_t st) {
  return enqueue(norm_dw_fold_kernel, dim3(HEAD_DIM / 16, 2), 1024, st, partial,
                 norm_blocks(T, Hq, kNormBwdBlocks), norm_blocks(T, Hkv, kNormBwdBlocks), dwq, dwk,
                 w_fp32);
}

}  // namespace upipe
