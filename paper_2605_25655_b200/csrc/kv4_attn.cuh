// Attention of the newest `queries` tokens of every request over its 4-bit paged cache:
//
//   S[i, t] = q_i . k_t / sqrt(D),  t < len - (queries - 1 - i)        (the query tokens are the last of the len keys)
//   out_i   = sum_t softmax_t(S[i, t]) v_t,   k_t, v_t = offset + scale * code;   0 where a query sees no key
//
// One CTA per (request, query token, query head): D / 8 lanes per key, an online softmax per lane group, merged at
// the end.  FP32 throughout.
#pragma once
#include "kv4_layout.cuh"

namespace thinfer {

struct Kv4AttnArgs {
  Kv4Cache c;
  const int32_t* lens;   // [batch]
  const half_t* q;       // [batch * queries] tokens, q_stride elements apart
  half_t* out;           // [batch * queries][n_q][D]
  long long q_stride;
  int batch, queries, n_q, group;
  float scale;           // 1 / sqrt(D)
};

constexpr int kKv4SimpleThreads = 128;

template <int D>
__global__ void __launch_bounds__(kKv4SimpleThreads) kv4_attn_simple_kernel(const Kv4AttnArgs a) {
  constexpr int LPR = D / 8;
  constexpr int NG = kKv4SimpleThreads / LPR;
  __shared__ float sm[NG], sl[NG], so[NG][D];
  const int g = threadIdx.x / LPR, sub = threadIdx.x % LPR;
  const int token = blockIdx.x, b = token / a.queries, i = token - b * a.queries;
  const int h = blockIdx.y, hk = h / a.group;
  const int page = 1 << a.c.page_shift;
  const long long cap = static_cast<long long>(a.c.max_pages) << a.c.page_shift;
  long long lim = static_cast<long long>(__ldg(a.lens + b)) - (a.queries - 1 - i);
  if (lim > cap) lim = cap;
  const int limit = static_cast<int>(lim);
  float q[8], o[8];
  unpack8(*reinterpret_cast<const uint4*>(a.q + token * a.q_stride + static_cast<long long>(h) * D + sub * 8), q);
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = 0.f;
  for (int t0 = 0; t0 < limit; t0 += NG) {   // uniform trip count: the shuffles need the whole warp
    const int t = t0 + g;
    const uint8_t* block = t < limit ? kv4_block(a.c, b, t, hk) : nullptr;
    uint32_t kw = 0, vw = 0;
    float2 kp = make_float2(__int_as_float(0x7fffffff), 0.f), vp = kp;
    if (block != nullptr) {
      const int slot = t & (page - 1);
      kw = *reinterpret_cast<const uint32_t*>(block + slot * (D / 2) + sub * 4);
      const uint16_t* vs = reinterpret_cast<const uint16_t*>(block + page * (D / 2) + (slot >> 1) * D + sub * 8) + (slot & 1);
      vw = vs[0] | (static_cast<uint32_t>(vs[2]) << 16);
      kp = kv4_unpack_params(*reinterpret_cast<const uint32_t*>(block + page * D + slot * 4));
      vp = kv4_unpack_params(*reinterpret_cast<const uint32_t*>(block + page * D + page * 4 + slot * 4));
    }
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(q[j], fmaf(kp.x, static_cast<float>((kw >> (4 * j)) & 15u), kp.y), s);
#pragma unroll
    for (int off = LPR / 2; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    if (t < limit) {
      s *= a.scale;
      const float mn = fmaxf(m, s), ms = mn == -INFINITY ? 0.f : mn;
      const float al = __expf(m - ms), p = __expf(s - ms);
      m = mn;
      l = l * al + p;
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = o[j] * al + p * fmaf(vp.x, static_cast<float>((vw >> (4 * j)) & 15u), vp.y);
    }
  }
  if (sub == 0) {
    sm[g] = m;
    sl[g] = l;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) so[g][sub * 8 + j] = o[j];
  __syncthreads();
  for (int e = threadIdx.x; e < D; e += kKv4SimpleThreads) {
    float mx = -INFINITY;
    for (int w = 0; w < NG; ++w) mx = fmaxf(mx, sm[w]);
    const float ms = mx == -INFINITY ? 0.f : mx;
    float L = 0.f, O = 0.f;
    for (int w = 0; w < NG; ++w) {
      const float al = __expf(sm[w] - ms);
      L += sl[w] * al;
      O += so[w][e] * al;
    }
    a.out[(static_cast<size_t>(token) * a.n_q + h) * D + e] = f_to_h(limit > 0 ? O / L : 0.f);
  }
}

}  // namespace thinfer
