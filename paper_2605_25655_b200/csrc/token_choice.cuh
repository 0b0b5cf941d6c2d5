// From logits to probabilities, and from two models' probabilities to the drafted tokens that stay.
#pragma once
#include <limits.h>

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

// exp(d / T) for the distance d <= 0 from the largest logit, with log2(e) / T = high + low: what the product loses comes back as a
// factor, so that the exponent of a far logit is as exact as d itself.  Weights below 2^-126 are 0, those of -inf and NaN too.
// Beyond T = 2^64 logits and T are taken 2^-80 times, so that no distance leaves FP32 that T would bring back; there an infinite T
// may stand for 10^30, which makes every weight of a finite logit 1.  Temperatures below 2^-126 count as that.
struct TokenHeat {
  float by, high, rest, least;   // by: what logits are multiplied by; rest = low * ln 2; least: where the exponent is -200
};
__device__ __forceinline__ TokenHeat token_heat(float temperature) {
  constexpr float kLog = 1.44269504088896f, kRest = 1.92596299e-8f;   // log2(e) and what FP32 leaves of it
  const float by = temperature > 0x1p64f ? 0x1p-80f : 1.f, t = fminf(fmaxf(temperature, 0x1p-126f) * by, 1e30f);
  const float high = kLog / t, low = (fmaf(-high, t, kLog) + kRest) / t;
  return {by, high, low * 0.693147180559945f, -200.f / high};
}
// The weight of logit x; top: the largest one times by.
__device__ __forceinline__ float token_weight(float x, float top, const TokenHeat& h) {
  const float d = fmaxf(fmaf(x, h.by, -top), h.least);
  const float a = d * h.high, rest = fmaf(fmaf(d, h.high, -a), 0.693147180559945f, d * h.rest), w = ex2_approx(a);
  return fmaf(w, rest, w);
}
// Two at a time.
__device__ __forceinline__ uint64_t token_weights(float x, float y, float top, const TokenHeat& h) {
  const uint64_t d = f32x2(fmaxf(fmaf(x, h.by, -top), h.least), fmaxf(fmaf(y, h.by, -top), h.least)), high = f32x2(h.high, h.high), a = mul_f32x2(d, high);
  const float2 e = f32x2_unpack(a);
  const uint64_t less = fma_f32x2(d, high, f32x2(-e.x, -e.y));
  const uint64_t rest = fma_f32x2(less, f32x2(0.693147180559945f, 0.693147180559945f), mul_f32x2(d, f32x2(h.rest, h.rest)));
  const uint64_t w = f32x2(ex2_approx(e.x), ex2_approx(e.y));
  return fma_f32x2(w, rest, w);
}
// The larger one; NaN where there is one.
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

__device__ __forceinline__ uint32_t token_cluster(uint32_t* rank) {   // size of this CTA's cluster
  uint32_t n;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(*rank));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
  return n;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint4 cluster_read(const void* shared, uint32_t rank) {   // the same 16 bytes of another CTA
  uint32_t at;
  uint4 v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(shared)), "r"(rank));
  asm volatile("ld.shared::cluster.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}

// A row as 16-byte slots of memory, whatever its alignment: slot s holds elements 4 s - before .. + 3; those outside the row
// are not touched.
struct TokenRow {
  const float* at;             // of slot 0
  int before, count, slots;
  int first_whole, wholes;     // slots that lie inside the row
  __device__ __forceinline__ TokenRow(const float* row, int n) {
    before = static_cast<int>(reinterpret_cast<uintptr_t>(row) >> 2) & 3;
    at = row - before;
    count = n;
    slots = static_cast<int>((static_cast<unsigned>(n) + before + 3) / 4);
    first_whole = before > 0 ? 1 : 0;
    wholes = static_cast<int>((static_cast<unsigned>(n) + before) / 4) - first_whole;
  }
  __device__ __forceinline__ bool whole(int s) const { return s - first_whole >= 0 && s - first_whole < wholes; }
};

// The ends of a row, apart from the code that every slot takes.
__device__ __noinline__ float4 token_load_end(const float* from, int s, int before, int count, float fill) {
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long long place = 4ll * s + i - before;
    f[i] = place >= 0 && place < count ? from[4ll * s + i] : fill;
  }
  return make_float4(f[0], f[1], f[2], f[3]);
}
__device__ __noinline__ void token_store_end(float* to, int s, int before, int count, float4 v) {
  const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long long place = 4ll * s + i - before;
    if (place >= 0 && place < count) to[4ll * s + i] = f[i];
  }
}
// Slot s of a row with the places of `row`; aligned: its memory has their alignment too.
__device__ __forceinline__ float4 token_load(const TokenRow& row, const float* from, bool aligned, int s, float fill) {
  if (!row.whole(s)) return token_load_end(from, s, row.before, row.count, fill);
  if (!aligned) return make_float4(from[4ll * s], from[4ll * s + 1], from[4ll * s + 2], from[4ll * s + 3]);
  const uint4 v = ld_stream(from + 4ll * s);
  return make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
}

// A cluster holds one row in shared memory: `steps` slots of four logits a thread, which nobody else touches.  Every CTA brings its
// slice down to weights against its own largest logit, then the CTAs exchange (largest, sum) once, and the weights leave
// with one factor.  Bound by memory: each logit is read once and each probability written once.  A slice of 64 KB leaves
// room for three CTAs on an SM, one of which reads while another computes and a third one writes (two with the slice in registers: 84 us
// instead of 74 for 320 x 128000, 4.4 TB/s of reads and writes; 1 x 32000: 4.2 us, a chain of one load, two reductions and
// the exchange).
__global__ void __launch_bounds__(512, 3) token_probs_kernel(const __grid_constant__ TokenProbsArgs a) {
  extern __shared__ float4 s_x[];   // [steps][threads]
  __shared__ float s_top[16], s_sum[16];
  __shared__ int s_index;
  __shared__ uint4 s_mine;          // largest (NaN where there is one), sum, its lowest index
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads >> 5;
  uint32_t rank;
  const uint32_t ctas = token_cluster(&rank);
  const long long which = blockIdx.x / ctas;
  const TokenRow row(a.logits + which * a.stride, a.vocab);
  const int slice = (row.slots + static_cast<int>(ctas) - 1) / static_cast<int>(ctas), from = slice * static_cast<int>(rank) + tid, to = min(row.slots, from - tid + slice);
  const int mine = to > from ? (to - from + threads - 1) / threads : 0;   // this thread's slots
  float4* x = s_x + tid;
  if (tid == 0) s_index = INT_MAX;
  pdl_wait();
  for (int e = 0, s = from; e < mine; ++e, s += threads) {
    if (row.whole(s))
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(x + e * threads)), "l"(row.at + 4ll * s) : "memory");
    else
      x[e * threads] = token_load_end(row.at, s, row.before, row.count, -INFINITY);
  }
  const float temp = a.temperature ? a.temperature[which] : 1.f;
  const bool greedy = !(temp > 0.f);
  const TokenHeat heat = token_heat(greedy ? 1.f : temp);
  asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory");
  float top = -INFINITY;
#pragma unroll 4
  for (int e = 0; e < mine; ++e) {
    const float4 v = x[e * threads];
    top = max_nan(max_nan(top, v.x, v.y), v.z, v.w);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) s_top[warp] = top;
  __syncthreads();
  top = lane < warps ? s_top[lane] : -INFINITY;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
  top = __shfl_sync(0xffffffffu, top, 0);
  float sum = 0.f;
  if (greedy) {
    int index = INT_MAX;
    for (int e = mine - 1; e >= 0; --e) {
      const float4 v = x[e * threads];
      const int i = 4 * (from + e * threads) - row.before;
      index = v.x == top ? i : v.y == top ? i + 1 : v.z == top ? i + 2 : v.w == top ? i + 3 : index;
    }
    index = __reduce_min_sync(0xffffffffu, index);
    if (lane == 0 && index != INT_MAX) atomicMin(&s_index, index);
  } else {
    uint64_t sums = f32x2(0.f, 0.f);
    const float its_top = top * heat.by;
#pragma unroll 2
    for (int e = 0; e < mine; ++e) {
      float4 v = x[e * threads];
      const uint64_t lo = token_weights(v.x, v.y, its_top, heat), hi = token_weights(v.z, v.w, its_top, heat);
      sums = add_f32x2(sums, add_f32x2(lo, hi));
      *reinterpret_cast<ulonglong2*>(x + e * threads) = make_ulonglong2(lo, hi);
    }
    const float2 both = f32x2_unpack(sums);
    sum = both.x + both.y;
    sum = warp_sum(sum);
    if (lane == 0) s_sum[warp] = sum;
  }
  __syncthreads();
  if (!greedy) {
    sum = lane < warps ? s_sum[lane] : 0.f;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    sum = __shfl_sync(0xffffffffu, sum, 0);
  }
  float all_top = top, all_sum = sum;
  int first = s_index;
  if (ctas > 1) {                   // lane c: what CTA c has
    if (tid == 0) s_mine = make_uint4(__float_as_uint(top), __float_as_uint(sum), static_cast<uint32_t>(s_index), 0u);
    cluster_arrive();
    cluster_wait();
    uint4 other = make_uint4(__float_as_uint(-INFINITY), 0u, INT_MAX, 0u);
    if (lane < static_cast<int>(ctas)) other = cluster_read(&s_mine, lane);
    __syncwarp();
    cluster_arrive();               // this warp has read; the CTA leaves when all have
    const float its = __uint_as_float(other.x);
    all_top = its;
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) all_top = max_nan(all_top, __shfl_xor_sync(0xffffffffu, all_top, o));
    all_top = __shfl_sync(0xffffffffu, all_top, 0);
    if (greedy) {
      first = __reduce_min_sync(0xffffffffu, its == all_top ? static_cast<int>(other.z) : INT_MAX);
    } else {
      all_sum = __uint_as_float(other.y) * token_weight(its, all_top * heat.by, heat);
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) all_sum += __shfl_xor_sync(0xffffffffu, all_sum, o);
      all_sum = __shfl_sync(0xffffffffu, all_sum, 0);
    }
  }
  const bool bad = all_top != all_top || (!greedy && all_top == INFINITY);
  const float by = bad ? __int_as_float(0x7fffffff) : all_top == -INFINITY ? 0.f : token_weight(top, all_top * heat.by, heat) / all_sum;
  if (all_top == -INFINITY) first = INT_MAX;
  float* out = a.out + which * a.out_stride - row.before;
  const bool aligned = (reinterpret_cast<uintptr_t>(out) & 15) == 0;
#pragma unroll 2
  for (int e = 0; e < mine; ++e) {
    const int s = from + e * threads;
    float4 v = x[e * threads];
    if (greedy) {
      const int i = first - (4 * s - row.before);
      v = make_float4(i == 0 ? 1.f : 0.f, i == 1 ? 1.f : 0.f, i == 2 ? 1.f : 0.f, i == 3 ? 1.f : 0.f);
      if (bad) v.x = v.y = v.z = v.w = by;
    } else {
      v.x *= by, v.y *= by, v.z *= by, v.w *= by;   // NaN where by is
    }
    if (!row.whole(s)) {
      token_store_end(out, s, row.before, row.count, v);
    } else if (aligned) {
      *reinterpret_cast<float4*>(out + 4ll * s) = v;
    } else {
      out[4ll * s] = v.x, out[4ll * s + 1] = v.y, out[4ll * s + 2] = v.z, out[4ll * s + 3] = v.w;
    }
  }
  if (ctas > 1) cluster_wait();
}

// Rows that no cluster holds: one CTA a row, which reads it three times, the second and third time from L2.  A thread has more than 800
// weights there: eight at a time are added up in FP32, what comes of them in FP64 (a running sum in FP32 would drift by
// 2^-24 for every second weight of one size).
__global__ void __launch_bounds__(512) token_probs_long_kernel(const __grid_constant__ TokenProbsArgs a) {
  __shared__ float s_top[16];
  __shared__ double s_sum[16];
  __shared__ int s_nan, s_index;
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float* x = a.logits + blockIdx.x * a.stride;
  float* out = a.out + blockIdx.x * a.out_stride;
  if (tid == 0) s_nan = 0, s_index = INT_MAX;
  pdl_wait();
  const float temp = a.temperature ? a.temperature[blockIdx.x] : 1.f;
  float top = -INFINITY;
  bool nan = false;
#pragma unroll 8
  for (long long i = tid; i < a.vocab; i += 512) {
    const float v = x[i];
    top = fmaxf(top, v);
    nan |= v != v;
  }
  top = warp_max(top);
  if (lane == 0) s_top[warp] = top;
  __syncthreads();
  if (nan) s_nan = 1;
  for (int w = 0; w < 16; ++w) top = fmaxf(top, s_top[w]);
  const bool greedy = !(temp > 0.f);
  const TokenHeat heat = token_heat(greedy ? 1.f : temp);
  const float its_top = top * heat.by;
  double sum = 0;
  if (greedy) {
    int index = INT_MAX;
#pragma unroll 8
    for (long long i = tid; i < a.vocab; i += 512)
      if (x[i] == top) index = min(index, static_cast<int>(i));
    if (index != INT_MAX) atomicMin(&s_index, index);
  } else {
    for (long long i = tid; i < a.vocab; i += 8 * 512) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = i + 512 * e < a.vocab ? token_weight(x[i + 512 * e], its_top, heat) : 0.f;
      sum += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) s_sum[warp] = sum;
  __syncthreads();
  sum = 0;
  for (int w = 0; w < 16; ++w) sum += s_sum[w];
  const bool bad = s_nan != 0 || (!greedy && top == INFINITY), none = top == -INFINITY;
  const float by = static_cast<float>(1.0 / sum);
#pragma unroll 8
  for (long long i = tid; i < a.vocab; i += 512)
    out[i] = bad ? __int_as_float(0x7fffffff) : none ? 0.f : greedy ? (i == s_index ? 1.f : 0.f) : token_weight(x[i], its_top, heat) * by;
}

// ------------------------------------------------------------------ verification
struct VerifyDraftsArgs {
  const float *p, *q;               // [batch][drafts + 1][vocab], [batch][drafts][vocab] or nullptr
  long long p_batch, p_row, q_batch, q_row;
  const int32_t *tokens, *counts;   // [batch][drafts], [batch] or nullptr
  const float* uniforms;            // [batch][drafts + 1]
  int32_t *out, *accepted;          // [batch][drafts + 1], [batch]
  int drafts, vocab;
  int steps;                        // of four values a thread in one round
};

// The sums of a block's threads, in every thread; order: lanes, then warps.
__device__ __forceinline__ double block_sum(double v, double* s_warp, int warps) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  const int lane = threadIdx.x & 31;
  __syncthreads();                  // the last sums have been read
  if (lane == 0) s_warp[threadIdx.x >> 5] = v;
  __syncthreads();
  v = lane < warps ? s_warp[lane] : 0.0;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return __shfl_sync(0xffffffffu, v, 0);
}

// The first part whose sum, with those before it, exceeds the target - or, where rounding or the target leave none, the last one that
// has something.  -1: there is nothing.  before: what comes before it.
struct Pick {
  double before = 0, picked_before = 0;
  int picked = -1;
  bool found = false;
  __device__ __forceinline__ void part(int i, double sum, double target) {
    if (!found && sum > 0) {
      picked = i;
      picked_before = before;
      found = before + sum > target;
    }
    before += sum;
  }
};

// The same among the lanes of a warp, one part each; *upto: what comes before this lane's.
__device__ __forceinline__ int pick_lane(double sum, double before, double target, double* upto) {
  double all = sum;
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double v = __shfl_up_sync(0xffffffffu, all, o);
    if (lane >= o) all += v;
  }
  const unsigned over = __ballot_sync(0xffffffffu, sum > 0 && before + all > target), some = __ballot_sync(0xffffffffu, sum > 0);
  const double left = __shfl_up_sync(0xffffffffu, all, 1);
  *upto = before + (lane > 0 ? left : 0.0);
  return over ? __ffs(over) - 1 : some ? 31 - __clz(some) : 0;
}

// A cluster per request.  Every CTA works out by itself how many drafts stay; then it sums up its slice of what is drawn from in
// FP64, so that the order of the sums moves the borders between tokens by some 2^-53 of the whole only, and leaves every thread's sum
// of each step of four values in shared memory (of a long vocabulary: of one round of 16 steps).  The CTAs exchange their
// sums, and the one that holds the target looks for the token among its steps and warps, then lanes, and reads the last four
// values again.  (64 registers, 40 bytes spilled: two CTAs an SM.)
constexpr int kVerifySteps = 16;
__global__ void __launch_bounds__(512, 2) verify_drafts_kernel(const __grid_constant__ VerifyDraftsArgs a) {
  extern __shared__ double s_step[];   // [steps][threads]
  __shared__ int s_token;
  __shared__ double s_warp[16], s_part[kVerifySteps];
  __shared__ __align__(16) double s_mine[2];
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads >> 5, n = a.drafts, steps = a.steps;
  uint32_t rank;
  const uint32_t ctas = token_cluster(&rank);
  const long long b = blockIdx.x / ctas;
  const float *p = a.p + b * a.p_batch, *q = a.q ? a.q + b * a.q_batch : nullptr, *u = a.uniforms + b * (n + 1);
  const int32_t* drafted = a.tokens + b * n;
  pdl_wait();
  // every warp by itself: the first of its drafts that does not stay, 32 at a time
  int count = a.counts ? a.counts[b] : n;
  const float draw = u[n];
  int kept = n;
  for (int at = 0; at < n && kept == n; at += 32) {
    const int i = at + lane, t = i < n ? drafted[i] : 0;
    const float chance = i < n ? u[i] : 0.f;
    bool goes = i >= count;
    if (i < n && (t < 0 || t >= a.vocab))
      goes = true;
    else if (i < n)
      goes = goes || !(static_cast<double>(chance) * (q ? q[i * a.q_row + t] : 1.f) < static_cast<double>(p[i * a.p_row + t]));
    const unsigned gone = __ballot_sync(0xffffffffu, i < n && goes);
    if (gone) kept = at + __ffs(gone) - 1;
  }
  if (count < 0) return;            // padding, for the whole cluster
  count = min(count, n);
  const TokenRow row(p + kept * a.p_row, a.vocab);
  // what is taken off: the draft's probabilities, in slots as those of the target, or all of a certain draft
  const float* off = kept < count && q ? q + kept * a.q_row - row.before : nullptr;
  int gone = -1, gone_slot = -1;    // of the certain draft: its place in its slot
  if (kept < count && !q && drafted[kept] >= 0 && drafted[kept] < a.vocab) {
    const long long place = static_cast<long long>(drafted[kept]) + row.before;
    gone_slot = static_cast<int>(place / 4);
    gone = static_cast<int>(place % 4);
  }
  const bool off_aligned = (reinterpret_cast<uintptr_t>(off) & 15) == 0;
  const int slice = (row.slots + static_cast<int>(ctas) - 1) / static_cast<int>(ctas), from = min(static_cast<long long>(row.slots), static_cast<long long>(slice) * rank);
  const int to = min(static_cast<long long>(row.slots), static_cast<long long>(from) + slice), step = steps * threads;
  // the four values of slot s, and what is taken off them
  auto load = [&](int s, float4& x, float4& y) {
    x = y = make_float4(0.f, 0.f, 0.f, 0.f);
    if (s >= to) return;
    x = token_load(row, row.at, true, s, 0.f);
    if (off) y = token_load(row, off, off_aligned, s, 0.f);
    if (s == gone_slot) {
      x.x = gone == 0 ? 0.f : x.x;
      x.y = gone == 1 ? 0.f : x.y;
      x.z = gone == 2 ? 0.f : x.z;
      x.w = gone == 3 ? 0.f : x.w;
    }
  };
  // max(have - less, 0), 0 where one is NaN: an exact difference of FP32 numbers, unless their sizes are 2^29 apart
  auto rest = [](float have, float less) {
    const bool more = have > less;
    return static_cast<double>(more ? have : 0.f) - static_cast<double>(more ? less : 0.f);
  };
  // the steps of one round: this thread's sum.  One walk over short code: every CTA fetches its instructions anew.
  auto sum_round = [&](int at) {
    double mine = 0;
#pragma unroll 1
    for (int e0 = 0; e0 < steps; e0 += 4) {
      float4 x[4], y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) load(e0 + e < steps ? at + (e0 + e) * threads + tid : to, x[e], y[e]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (e0 + e >= steps) break;
        const double v = (rest(x[e].x, y[e].x) + rest(x[e].y, y[e].y)) + (rest(x[e].z, y[e].z) + rest(x[e].w, y[e].w));
        s_step[(e0 + e) * threads + tid] = v;
        mine += v;
      }
    }
    return mine;
  };
  int token = -1;
  bool have = false;                // this CTA draws the token
  for (int again = 0; again < 2; ++again) {
    double mine = 0;
    for (int at = from; at < to; at += step) mine += sum_round(at);
    mine = block_sum(mine, s_warp, warps);
    Pick cta;
    double total = mine;
    if (ctas > 1) {
      if (tid == 0) s_mine[0] = mine;
      cluster_arrive();
      cluster_wait();
      double its = 0;               // lane c: of CTA c
      if (lane < static_cast<int>(ctas)) {
        const uint4 v = cluster_read(s_mine, lane);
        its = __hiloint2double(static_cast<int>(v.y), static_cast<int>(v.x));
      }
      __syncwarp();
      cluster_arrive();             // this warp has read; the CTA goes on when all have
      total = its;
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
      total = __shfl_sync(0xffffffffu, total, 0);
      double upto = 0;
      const int who = pick_lane(its, 0.0, static_cast<double>(draw) * total, &upto);
      cta.picked = who;
      cta.picked_before = __shfl_sync(0xffffffffu, upto, who);
    } else {
      cta.part(0, mine, static_cast<double>(draw) * total);
    }
    if (total > 0) {
      have = cta.picked == static_cast<int>(rank);
      if (have) {
        const double target = static_cast<double>(draw) * total;
        double before = cta.picked_before;
        int at = from;
        if (from + step < to) {     // the round, read again
          Pick round;
          round.before = before;
          for (int r = from; r < to; r += step) round.part((r - from) / step, block_sum(sum_round(r), s_warp, warps), target);
          at = from + round.picked * step;
          before = round.picked_before;
          sum_round(at);
          __syncthreads();
        }
        // the step: warp w sums up steps w, w + warps, ...
        if (tid == 0) s_token = -1;
        for (int e = warp; e < steps; e += warps) {
          double v = 0;
#pragma unroll 4
          for (int i = lane; i < threads; i += 32) v += s_step[e * threads + i];
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
          if (lane == 0) s_part[e] = v;
        }
        __syncthreads();
        if (warp == 0) {            // the step, the warp's worth of threads, the thread, its value
          double upto = 0;
          const int e = pick_lane(lane < steps ? s_part[lane] : 0.0, before, target, &upto);
          before = __shfl_sync(0xffffffffu, upto, e);
          double v = 0;
#pragma unroll 4
          for (int i = 0; i < warps; ++i) v += s_step[e * threads + lane * warps + i];
          const int part = pick_lane(v, before, target, &upto);
          before = __shfl_sync(0xffffffffu, upto, part);
          const int place = pick_lane(lane < warps ? s_step[e * threads + part * warps + lane] : 0.0, before, target, &upto);
          if (lane == place) {
            const int s = at + e * threads + part * warps + place;
            float4 x, y;
            load(s, x, y);
            Pick value;
            value.before = upto;
            value.part(0, rest(x.x, y.x), target);
            value.part(1, rest(x.y, y.y), target);
            value.part(2, rest(x.z, y.z), target);
            value.part(3, rest(x.w, y.w), target);
            s_token = static_cast<int>(4ll * s + value.picked - row.before);
          }
        }
        __syncthreads();
        token = s_token;
      }
    } else {
      have = rank == 0;             // nothing to draw from
    }
    if (ctas > 1) cluster_wait();
    if (total > 0 || (off == nullptr && gone_slot < 0)) break;
    off = nullptr;                  // the target has nothing that the draft has less of: drawn from the target
    gone_slot = -1;
  }
  if (!have) return;
  if (tid == 0) a.accepted[b] = kept;
  for (int i = tid; i <= n; i += threads) a.out[b * (n + 1) + i] = i < kept ? drafted[i] : i == kept ? token : -1;
}

}  // namespace thinfer
