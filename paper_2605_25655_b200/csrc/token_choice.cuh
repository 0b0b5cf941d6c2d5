// From logits to probabilities, and from two models' probabilities to the drafted tokens that stay.
#pragma once
#include "common.cuh"

namespace thinfer {

// ------------------------------------------------------------------ probabilities
struct TokenProbsArgs {
  const float* logits;
  float* out;
  const float* temperature;         // [rows], nullptr: 1
  long long stride, out_stride;     // elements between rows
  int vocab;
};

// The largest logit so far, the lowest index that has it, and whether there was a NaN.
struct TopLogit {
  float value;
  int index;
  bool nan;
};
__device__ __forceinline__ TopLogit top_of(const TopLogit& a, const TopLogit& b) {
  const bool second = b.value > a.value || (b.value == a.value && b.index < a.index);
  return {second ? b.value : a.value, second ? b.index : a.index, a.nan || b.nan};
}

// exp(d / T) for d <= 0, with log2(e) / T = high + low: what the product loses comes back as a factor, so that the exponent
// of a far logit is as exact as d itself.
__device__ __forceinline__ float token_weight(float d, float high, float low) {
  const float a = d * high;
  if (!(a >= -160.f)) return 0.f;   // and -inf, whatever the temperature
  const float rest = fmaf(d, high, -a) + d * low;
  return exp2f(a) * fmaf(rest, 0.693147180559945f, 1.f);
}

__global__ void __launch_bounds__(512) token_probs_kernel(const __grid_constant__ TokenProbsArgs a) {
  __shared__ float s_value[16], s_sum[16];
  __shared__ int s_index[16];
  __shared__ bool s_nan[16];
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float* x = a.logits + blockIdx.x * a.stride;
  float* out = a.out + blockIdx.x * a.out_stride;
  const float temp = a.temperature ? a.temperature[blockIdx.x] : 1.f;
  TopLogit top{-INFINITY, a.vocab, false};
  for (int i = tid; i < a.vocab; i += 512) top = top_of(top, {x[i], i, x[i] != x[i]});
  for (int o = 16; o > 0; o >>= 1)
    top = top_of(top, {__shfl_xor_sync(~0u, top.value, o), __shfl_xor_sync(~0u, top.index, o), __shfl_xor_sync(~0u, top.nan, o) != 0});
  if (lane == 0) s_value[warp] = top.value, s_index[warp] = top.index, s_nan[warp] = top.nan;
  __syncthreads();
  for (int w = 0; w < 16; ++w) top = top_of(top, {s_value[w], s_index[w], s_nan[w]});
  const bool bad = top.nan || (top.value == INFINITY && temp > 0.f);
  const bool none = top.value == -INFINITY;
  const double by = 1.4426950408889634 / temp;
  const float high = fminf(static_cast<float>(by), 3e38f), low = by < 3e38 ? static_cast<float>(by - high) : 0.f;
  float sum = 0.f;
  if (temp > 0.f && !bad && !none)
    for (int i = tid; i < a.vocab; i += 512) sum += token_weight(x[i] - top.value, high, low);
  sum = warp_sum(sum);
  if (lane == 0) s_sum[warp] = sum;
  __syncthreads();
  sum = 0.f;
  for (int w = 0; w < 16; ++w) sum += s_sum[w];
  const float scale = 1.f / sum;
  for (int i = tid; i < a.vocab; i += 512) {
    float p;
    if (bad)
      p = __int_as_float(0x7fffffff);
    else if (none)
      p = 0.f;
    else if (temp > 0.f)
      p = token_weight(x[i] - top.value, high, low) * scale;
    else
      p = i == top.index ? 1.f : 0.f;
    out[i] = p;
  }
}

// ------------------------------------------------------------------ verification
struct VerifyDraftsArgs {
  const float *p, *q;               // [batch][drafts + 1][vocab], [batch][drafts][vocab] or nullptr
  long long p_batch, p_row, q_batch, q_row;
  const int32_t *tokens, *counts;   // [batch][drafts], [batch] or nullptr
  const float* uniforms;            // [batch][drafts + 1]
  int32_t *out, *accepted;          // [batch][drafts + 1], [batch]
  int drafts, vocab;
};

// One request: how many of its drafts stay, then the token behind them by inverse CDF.
__global__ void __launch_bounds__(512) verify_drafts_kernel(const __grid_constant__ VerifyDraftsArgs a) {
  __shared__ int s_kept, s_token, s_last;
  __shared__ double s_sum[512];
  pdl_launch_dependents();
  pdl_wait();
  const int b = blockIdx.x, tid = threadIdx.x, n = a.drafts;
  int count = a.counts ? a.counts[b] : n;
  if (count < 0) return;            // padding
  count = min(count, n);
  if (tid == 0) s_kept = count, s_token = a.vocab, s_last = -1;
  __syncthreads();
  const float *p = a.p + b * a.p_batch, *q = a.q ? a.q + b * a.q_batch : nullptr, *u = a.uniforms + static_cast<long long>(b) * (n + 1);
  const int32_t* drafted = a.tokens + static_cast<long long>(b) * n;
  for (int i = tid; i < count; i += 512) {
    const int t = drafted[i];
    bool stays = t >= 0 && t < a.vocab;
    if (stays) stays = static_cast<double>(u[i]) * (q ? q[i * a.q_row + t] : 1.f) < static_cast<double>(p[i * a.p_row + t]);
    if (!stays) atomicMin(&s_kept, i);
  }
  __syncthreads();
  const int kept = s_kept;
  const float* row = p + kept * a.p_row;
  const float* off = q && kept < count ? q + kept * a.q_row : nullptr;
  int gone = !q && kept < count ? drafted[kept] : -1;
  const int per = (a.vocab + 511) / 512, from = min(a.vocab, tid * per), to = min(a.vocab, from + per);
  double total = 0;
  for (int again = 0; again < 2; ++again) {
    auto left = [&](int v) {
      const double r = v == gone ? 0.0 : static_cast<double>(row[v]) - (off ? static_cast<double>(off[v]) : 0.0);
      return r > 0 ? r : 0.0;
    };
    double mine = 0;
    int last = -1;
    for (int v = from; v < to; ++v) {
      const double r = left(v);
      mine += r;
      if (r > 0) last = v;
    }
    s_sum[tid] = mine;
    if (last >= 0) atomicMax(&s_last, last);
    __syncthreads();
    double before = 0;
    total = 0;
    for (int w = 0; w < 512; ++w) {
      if (w == tid) before = total;
      total += s_sum[w];
    }
    const double target = static_cast<double>(u[n]) * total;
    if (total > 0) {
      for (int v = from; v < to; ++v) {
        before += left(v);
        if (before > target) {
          atomicMin(&s_token, v);
          break;
        }
      }
    }
    __syncthreads();
    if (total > 0 || (off == nullptr && gone < 0)) break;
    off = nullptr;                  // the target has nothing that the draft has less of
    gone = -1;
  }
  if (tid == 0) {
    a.accepted[b] = kept;
    s_token = total > 0 ? min(s_token, s_last) : -1;
  }
  __syncthreads();
  for (int i = tid; i <= n; i += 512) a.out[static_cast<long long>(b) * (n + 1) + i] = i < kept ? drafted[i] : i == kept ? s_token : -1;
}

}  // namespace thinfer
