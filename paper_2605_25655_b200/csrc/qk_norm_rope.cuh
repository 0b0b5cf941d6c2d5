// Per-head RMSNorm of queries and keys with the position rotation in the same pass:
//
//   x^ = x * gain / sqrt(mean(x^2) + eps)       over the D values of one head, FP32
//   (a, b) -> (a cos - b sin, b cos + a sin)    for each pair of the first 2 * half dimensions, angle 2 pi frac(p * turns[j])
//
// rounded to the storage type once.  Pairs are neighbours (2j, 2j + 1), as in the framework's projections, or the two
// halves (j, j + half).  Bound by memory: every value is read and written once, 4 bytes of traffic per value against
// about ten FP32 operations, so a row of D values belongs to D / 8 lanes with one 16-byte access each; nothing goes
// through shared memory.  The angle is reduced in FP64 (position times turns keeps 2^-22 of a turn at position 2^31)
// and only its fraction goes to FP32; sine and cosine are computed once per token and lane and reused for all the
// heads that a lane group walks, four rows in flight at a time.  How many groups share the heads of a token is set so
// that the device is full about twice: one group per head for a few tokens, a few for a long prompt (16384 tokens of 80
// heads: 404 us with one group per head, where the sines cost more than the memory).
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
};

template <int D, bool HALVES>
__global__ void __launch_bounds__(256) qk_norm_rope_kernel(const QkNormRopeArgs a) {
  constexpr int LPR = D / 8;        // lanes per row
  constexpr int NCS = HALVES ? 8 : 4;
  const int lane = threadIdx.x & 31, sub = lane % LPR;
  const long long group = (static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x) / LPR;
  const long long token = group / a.chunks;
  const int chunk = static_cast<int>(group - token * a.chunks);
  const int heads = a.n_q + a.n_kv;
  const int e0 = sub * 8;
  // every lane walks the same number of heads: the shuffles below need the whole warp
  const int pos = token < a.tokens ? __ldg(a.positions + token) : -1;
  const bool live = pos >= 0;
  float cs[NCS], sn[NCS];
  const int j0 = HALVES ? (e0 < a.half ? e0 : e0 - a.half) : e0 / 2;
  const bool rotated = e0 < 2 * a.half;
#pragma unroll
  for (int i = 0; i < NCS; ++i) {
    cs[i] = 1.f;
    sn[i] = 0.f;
    if (rotated && live) {
      const double t = static_cast<double>(pos) * __ldg(a.turns + j0 + i);
      sincospif(2.f * static_cast<float>(t - rint(t)), &sn[i], &cs[i]);
    }
  }
  const int step = HALVES ? a.half / 8 : 0;                       // lanes between the two halves of a pair
  const int partner = HALVES && rotated ? (e0 < a.half ? lane + step : lane - step) : lane;
  const float sign = e0 < a.half ? -1.f : 1.f;
  const uint4 gq = ldg_cached(a.q_gain + e0), gk = ldg_cached(a.k_gain + e0);
  const half_t* const q = a.q + token * a.q_stride + e0;
  const half_t* const k = a.k + token * a.k_stride + e0;
  half_t* const q_out = a.q_out + token * a.q_out_stride + e0;
  half_t* const k_out = a.k_out + token * a.k_out_stride + e0;
  constexpr int U = 4;
  for (int h0 = 0; h0 < heads; h0 += U * a.chunks) {
    uint4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * a.chunks + chunk;
      raw[u] = make_uint4(0, 0, 0, 0);
      if (live && h < heads)
        raw[u] = *reinterpret_cast<const uint4*>(h < a.n_q ? q + static_cast<long long>(h) * D : k + static_cast<long long>(h - a.n_q) * D);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (h0 + u * a.chunks >= heads) break;                       // the same for the whole warp: the shuffles need all of it
      const int h = h0 + u * a.chunks + chunk;
      float x[8], g[8];
      unpack8(raw[u], x);
      unpack8(h < a.n_q ? gq : gk, g);
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      const float rstd = rsqrtf(ss / static_cast<float>(D) + a.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = x[i] * rstd * g[i];
      float y[8];
      if (HALVES) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float other = __shfl_sync(0xffffffffu, x[i], partner);
          y[i] = rotated ? x[i] * cs[i % NCS] + sign * other * sn[i % NCS] : x[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[2 * i] = rotated ? x[2 * i] * cs[i] - x[2 * i + 1] * sn[i] : x[2 * i];
          y[2 * i + 1] = rotated ? x[2 * i + 1] * cs[i] + x[2 * i] * sn[i] : x[2 * i + 1];
        }
      }
      if (live && h < heads)
        *reinterpret_cast<uint4*>(h < a.n_q ? q_out + static_cast<long long>(h) * D : k_out + static_cast<long long>(h - a.n_q) * D) =
            make_uint4(pack2(y[0], y[1]), pack2(y[2], y[3]), pack2(y[4], y[5]), pack2(y[6], y[7]));
    }
  }
}

}  // namespace thinfer
