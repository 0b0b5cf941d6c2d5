// Per-head RMSNorm of queries and keys with the position rotation in the same pass:
//
//   x^ = x * gain / sqrt(mean(x^2) + eps)       over the D values of one head, FP32
//   (a, b) -> (a cos - b sin, b cos + a sin)    for each pair of the first 2 * half dimensions, angle 2 pi frac(p * turns[j])
//
// rounded to the storage type once.  Pairs are neighbours (2j, 2j + 1), as in the framework's projections, or the two
// halves (j, j + half).  Bound by memory: every value is read and written once, 4 bytes of traffic per value against
// about ten FP32 operations, so a row of D values belongs to D / 8 lanes, with both members of every pair in one lane:
// neighbours come with one 16-byte access, halves with two of 8 bytes.  Nothing goes through shared memory.  The angle
// is reduced in FP64 (position times turns keeps 2^-22 of a turn at position 2^31) and only its fraction goes to FP32;
// sine and cosine are computed once per token and lane and reused for all the heads that a lane group walks, two rows in
// flight at a time.  How many groups share the heads of a token is set so that the device is full once: one group per head
// for a few tokens, one or two for a long prompt (16384 tokens of 80 heads: 402 us with one group per head, where the
// sines cost more than the memory, 128 us with two).
#pragma once
#include "common.cuh"

namespace thinfer {

struct QkNormRopeArgs {
  const half_t *q, *k;
  half_t *q_out, *k_out;
  long long q_stride, k_stride, q_out_stride, k_out_stride;  // elements between tokens
  const half_t *q_gain, *k_gain;
  const double* turns;       // [half]
  const int32_t* positions;  // [tokens]
  int tokens, n_q, n_kv;
  int half;                  // pairs that are rotated (a multiple of 8)
  int chunks;                // lane groups that share the heads of one token
  float eps;
  float least;               // a smaller sum of squares is too small for FP32 beside eps
};

constexpr int kQkRowsInFlight = 2;

// The rows of one lane group from head `from` on.  In the BF16 build it stops at the first row whose sum of squares leaves FP32
// and returns that head; -1: all done.  SCALED: such rows are scaled by a power of two (and eps by its square) instead.
template <int D, bool HALVES, bool SCALED>
__device__ __forceinline__ int qk_norm_rope_rows(const QkNormRopeArgs& a, int from) {
  constexpr int LPR = D / 8;        // lanes per row
  constexpr int U = SCALED ? 1 : kQkRowsInFlight;
  const int lane = threadIdx.x & 31, sub = lane % LPR;
  const unsigned group_mask = (LPR == 16 ? 0xffffu : 0xffu) << (lane & ~(LPR - 1));
  const long long group = (static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x) / LPR;
  const long long token = group / a.chunks;
  const int chunk = static_cast<int>(group - token * a.chunks);
  if (!SCALED) pdl_wait();             // behind what needs no memory
  const int pos = token < a.tokens ? a.positions[token] : -1;
  if (pos < 0) return -1;              // the same for the group, and shuffles stay inside it
  // this lane's values: two runs of four.  Halves: values j .. j + 3 of both halves, or eight behind the rotated ones
  const int j0 = 4 * sub;
  const bool rotated = j0 < a.half;
  const int e0 = HALVES ? (rotated ? j0 : 2 * j0) : 8 * sub, e1 = HALVES && rotated ? a.half + j0 : e0 + 4;
  float cs[4], sn[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    cs[i] = 1.f;
    sn[i] = 0.f;
    if (rotated) {
      const double t = static_cast<double>(pos) * a.turns[j0 + i];
      sincospif(2.f * static_cast<float>(t - rint(t)), &sn[i], &cs[i]);
    }
  }
  auto load8 = [&](const half_t* p) {
    if (!HALVES) return *reinterpret_cast<const uint4*>(p + e0);
    const uint2 x = *reinterpret_cast<const uint2*>(p + e0), y = *reinterpret_cast<const uint2*>(p + e1);
    return make_uint4(x.x, x.y, y.x, y.y);
  };
  // heads first, first + chunks, ... of q or of k; the head it stopped at
  auto walk = [&](const half_t* src, half_t* dst, const half_t* gain, int first, int n) {
    float g[8];
    unpack8(load8(gain), g);
    for (int h0 = first; h0 < n; h0 += U * a.chunks) {
      uint4 raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (h0 + u * a.chunks < n) raw[u] = load8(src + static_cast<long long>(h0 + u * a.chunks) * D);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + u * a.chunks;
        if (h >= n) break;
        float x[8];
        unpack8(raw[u], x);
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(group_mask, ss, o);
        float eps = a.eps;
        if (kStorageType == 1 && !(ss >= a.least && ss <= 0x1p120f)) {   // the same for the group
          if (!SCALED) return h;
          const float by = ss < a.least ? 0x1p96f : 0x1p-72f;
          eps = eps * by * by;
          ss = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            x[i] *= by;
            ss = fmaf(x[i], x[i], ss);
          }
#pragma unroll
          for (int o = LPR / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(group_mask, ss, o);
        }
        const float rstd = rsqrtf(ss / static_cast<float>(D) + eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] * rstd * g[i];
        float y[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // lanes behind the rotated values turn by nothing
          const int p = HALVES ? i : 2 * i, q = HALVES ? i + 4 : 2 * i + 1;
          y[p] = x[p] * cs[i] - x[q] * sn[i];
          y[q] = x[q] * cs[i] + x[p] * sn[i];
        }
        half_t* out = dst + static_cast<long long>(h) * D;
        const uint4 v = make_uint4(pack2(y[0], y[1]), pack2(y[2], y[3]), pack2(y[4], y[5]), pack2(y[6], y[7]));
        if (HALVES) {
          *reinterpret_cast<uint2*>(out + e0) = make_uint2(v.x, v.y);
          *reinterpret_cast<uint2*>(out + e1) = make_uint2(v.z, v.w);
        } else {
          *reinterpret_cast<uint4*>(out + e0) = v;
        }
      }
    }
    return n;
  };
  // chunk, chunk + chunks, ... of the queries, and the same sequence of heads goes on behind them
  if (from < a.n_q) {
    const int h = walk(a.q + token * a.q_stride, a.q_out + token * a.q_out_stride, a.q_gain, SCALED ? from : chunk, a.n_q);
    if (kStorageType == 1 && !SCALED && h < a.n_q) return h;
  }
  const int first = SCALED && from >= a.n_q ? from : chunk >= a.n_q ? chunk : chunk + (a.n_q - chunk + a.chunks - 1) / a.chunks * a.chunks;
  if (first < a.n_q + a.n_kv) {
    const int h = walk(a.k + token * a.k_stride, a.k_out + token * a.k_out_stride, a.k_gain, first - a.n_q, a.n_kv);
    if (kStorageType == 1 && !SCALED && h < a.n_kv) return a.n_q + h;
  }
  return -1;
}

// Apart, so that little is kept in registers for it: BF16 prompts take 128 us instead of 125 for looking out for such rows,
// 129.5 with the scaling in the walk over all rows, 131 with one look at two rows.
template <int D, bool HALVES>
__device__ __noinline__ void qk_norm_rope_far_rows(const QkNormRopeArgs& a, int from) {
  qk_norm_rope_rows<D, HALVES, true>(a, from);
}

template <int D, bool HALVES>
__global__ void __launch_bounds__(256, 4) qk_norm_rope_kernel(const __grid_constant__ QkNormRopeArgs a) {
  pdl_launch_dependents();
  const int from = qk_norm_rope_rows<D, HALVES, false>(a, 0);
  if (kStorageType == 1 && from >= 0) qk_norm_rope_far_rows<D, HALVES>(a, from);
}

}  // namespace thinfer
