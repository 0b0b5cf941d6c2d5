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

// exp(d / T) for d <= 0, with log2(e) / T = high + low: what the product loses comes back as a factor, so that the exponent
// of a far logit is as exact as d itself.
struct TokenHeat {
  float high, low;
};
__device__ __forceinline__ TokenHeat token_heat(float temperature) {
  const double by = 1.4426950408889634 / temperature;
  const float high = fminf(static_cast<float>(by), 3e38f);
  return {high, by < 3e38 ? static_cast<float>(by - high) : 0.f};
}
__device__ __forceinline__ float token_weight(float d, const TokenHeat& h) {
  const float a = d * h.high;
  if (!(a >= -160.f)) return 0.f;   // and -inf, whatever the temperature
  const float rest = fmaf(d, h.high, -a) + d * h.low;
  return exp2f(a) * fmaf(rest, 0.693147180559945f, 1.f);
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
  const float* at;    // of slot 0
  int before, count;
  long long slots;
  __device__ __forceinline__ TokenRow(const float* row, int n) {
    before = static_cast<int>(reinterpret_cast<uintptr_t>(row) >> 2) & 3;
    at = row - before;
    count = n;
    slots = (static_cast<long long>(n) + before + 3) / 4;
  }
  __device__ __forceinline__ bool whole(long long s) const { return 4 * s >= before && 4 * s + 4 - before <= count; }
  __device__ __forceinline__ bool has(long long s, int i) const { return 4 * s + i >= before && 4 * s + i - before < count; }
  __device__ __forceinline__ float4 load(long long s, float fill) const {
    if (whole(s)) {
      const uint4 v = ld_stream(at + 4 * s);
      return make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
    }
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = has(s, i) ? at[4 * s + i] : fill;
    return make_float4(f[0], f[1], f[2], f[3]);
  }
};

// A cluster holds one row in registers: E slots of four logits a thread.  Every CTA brings its slice down to weights against its
// own largest logit, then the CTAs exchange (largest, sum) once, and the weights leave with one factor.  Bound by memory: each
// logit is read once and each probability written once.
template <int E>
__global__ void __launch_bounds__(512) token_probs_kernel(const __grid_constant__ TokenProbsArgs a) {
  __shared__ float s_top[16], s_sum[16];
  __shared__ int s_nan, s_index;
  __shared__ uint4 s_mine;          // largest, sum, its lowest index, whether there was a NaN
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  uint32_t rank;
  const uint32_t ctas = token_cluster(&rank);
  const long long which = blockIdx.x / ctas;
  const TokenRow row(a.logits + which * a.stride, a.vocab);
  const long long slice = (row.slots + ctas - 1) / ctas, from = slice * rank, to = min(row.slots, from + slice);
  if (tid == 0) s_nan = 0, s_index = INT_MAX;
  pdl_wait();
  const float temp = a.temperature ? a.temperature[which] : 1.f;
  const bool greedy = !(temp > 0.f);
  float4 x[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const long long s = from + e * blockDim.x + tid;
    x[e] = s < to ? row.load(s, -INFINITY) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
  }
  float top = -INFINITY;
  bool nan = false;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    top = fmaxf(top, fmaxf(fmaxf(x[e].x, x[e].y), fmaxf(x[e].z, x[e].w)));
    nan |= x[e].x != x[e].x || x[e].y != x[e].y || x[e].z != x[e].z || x[e].w != x[e].w;
  }
  top = warp_max(top);
  if (lane == 0) s_top[warp] = top;
  __syncthreads();
  if (nan) s_nan = 1;
  for (int w = 0; w < warps; ++w) top = fmaxf(top, s_top[w]);
  float sum = 0.f;
  const TokenHeat heat = token_heat(greedy ? 1.f : temp);
  if (greedy) {
    int index = INT_MAX;
#pragma unroll
    for (int e = E - 1; e >= 0; --e) {
      const int i = static_cast<int>(4 * (from + e * blockDim.x + tid)) - row.before;
      index = x[e].x == top ? i : x[e].y == top ? i + 1 : x[e].z == top ? i + 2 : x[e].w == top ? i + 3 : index;
    }
    index = __reduce_min_sync(0xffffffffu, index);
    if (lane == 0 && index != INT_MAX) atomicMin(&s_index, index);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      x[e].x = token_weight(x[e].x - top, heat);
      x[e].y = token_weight(x[e].y - top, heat);
      x[e].z = token_weight(x[e].z - top, heat);
      x[e].w = token_weight(x[e].w - top, heat);
      sum += (x[e].x + x[e].y) + (x[e].z + x[e].w);
    }
    sum = warp_sum(sum);
    if (lane == 0) s_sum[warp] = sum;
  }
  __syncthreads();
  if (!greedy) {
    sum = 0.f;
    for (int w = 0; w < warps; ++w) sum += s_sum[w];
  }
  // all CTAs' (largest, sum)
  float all_top = top, all_sum = sum;
  int first = s_index;
  bool bad = s_nan != 0;
  if (ctas > 1) {
    if (tid == 0) s_mine = make_uint4(__float_as_uint(top), __float_as_uint(sum), static_cast<uint32_t>(s_index), static_cast<uint32_t>(s_nan));
    cluster_arrive();
    cluster_wait();
    uint4 other[8];
#pragma unroll
    for (uint32_t c = 0; c < 8; ++c)
      if (c < ctas) other[c] = cluster_read(&s_mine, c);
    cluster_arrive();               // this CTA has read; it leaves when all have
    all_top = -INFINITY;
#pragma unroll
    for (uint32_t c = 0; c < 8; ++c)
      if (c < ctas) {
        all_top = fmaxf(all_top, __uint_as_float(other[c].x));
        bad |= other[c].w != 0;
      }
    all_sum = 0.f;
    first = INT_MAX;
#pragma unroll
    for (uint32_t c = 0; c < 8; ++c)
      if (c < ctas) {
        const float its = __uint_as_float(other[c].x);
        all_sum += __uint_as_float(other[c].y) * token_weight(its - all_top, heat);
        if (its == all_top) first = min(first, static_cast<int>(other[c].z));
      }
  }
  bad |= !greedy && all_top == INFINITY;
  const float by = bad ? __int_as_float(0x7fffffff) : all_top == -INFINITY ? 0.f : token_weight(top - all_top, heat) / all_sum;
  if (all_top == -INFINITY) first = INT_MAX;
  float* out = a.out + which * a.out_stride - row.before;
  const bool aligned = (reinterpret_cast<uintptr_t>(out) & 15) == 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const long long s = from + e * blockDim.x + tid;
    if (s >= to) continue;
    float p[4] = {x[e].x * by, x[e].y * by, x[e].z * by, x[e].w * by};
    if (greedy) {
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = bad ? by : 4 * s + i - row.before == first ? 1.f : 0.f;
    } else if (bad) {
      p[0] = p[1] = p[2] = p[3] = by;
    }
    if (aligned && row.whole(s)) {
      *reinterpret_cast<float4*>(out + 4 * s) = make_float4(p[0], p[1], p[2], p[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (row.has(s, i)) out[4 * s + i] = p[i];
    }
  }
  if (ctas > 1) cluster_wait();
}

// Rows that no cluster holds: one CTA a row, which reads it three times, the second and third time from L2.
__global__ void __launch_bounds__(512) token_probs_long_kernel(const __grid_constant__ TokenProbsArgs a) {
  __shared__ float s_top[16], s_sum[16];
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
  float sum = 0.f;
  if (greedy) {
    int index = INT_MAX;
#pragma unroll 8
    for (long long i = tid; i < a.vocab; i += 512)
      if (x[i] == top) index = min(index, static_cast<int>(i));
    if (index != INT_MAX) atomicMin(&s_index, index);
  } else {
#pragma unroll 8
    for (long long i = tid; i < a.vocab; i += 512) sum += token_weight(x[i] - top, heat);
  }
  sum = warp_sum(sum);
  if (lane == 0) s_sum[warp] = sum;
  __syncthreads();
  sum = 0.f;
  for (int w = 0; w < 16; ++w) sum += s_sum[w];
  const bool bad = s_nan != 0 || (!greedy && top == INFINITY), none = top == -INFINITY;
  const float by = 1.f / sum;
#pragma unroll 8
  for (long long i = tid; i < a.vocab; i += 512)
    out[i] = bad ? __int_as_float(0x7fffffff) : none ? 0.f : greedy ? (i == s_index ? 1.f : 0.f) : token_weight(x[i] - top, heat) * by;
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

// The sums of a block's threads, in every thread; order: lanes, then warps.
__device__ __forceinline__ double block_sum(double v, double* s_warp, int warps) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();                  // the last sums have been read
  if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0;
  for (int w = 0; w < warps; ++w) v += s_warp[w];
  return v;
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

// A cluster per request.  Every CTA works out by itself how many drafts stay; then it holds a slice of what is drawn from in
// registers, E slots of four values a thread (of a long vocabulary: round by round), and sums it up in FP64, so that
// the drawn token does not depend on the order of the sums.  The CTAs exchange their sums, and the one that holds the target
// looks for the token among its steps, warps, lanes and values.
template <int E>
__global__ void __launch_bounds__(512, 1) verify_drafts_kernel(const __grid_constant__ VerifyDraftsArgs a) {
  __shared__ int s_kept, s_token;
  __shared__ double s_warp[16], s_part[E * 16];
  __shared__ __align__(16) double s_mine[2];
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5, n = a.drafts;
  uint32_t rank;
  const uint32_t ctas = token_cluster(&rank);
  const long long b = blockIdx.x / ctas;
  pdl_wait();
  int count = a.counts ? a.counts[b] : n;
  if (count < 0) return;            // padding, for the whole cluster
  count = min(count, n);
  if (tid == 0) s_kept = count;
  __syncthreads();
  const float *p = a.p + b * a.p_batch, *q = a.q ? a.q + b * a.q_batch : nullptr, *u = a.uniforms + b * (n + 1);
  const int32_t* drafted = a.tokens + b * n;
  const float draw = u[n];
  for (int i = tid; i < count; i += blockDim.x) {
    const int t = drafted[i];
    bool stays = t >= 0 && t < a.vocab;
    if (stays) stays = static_cast<double>(u[i]) * (q ? q[i * a.q_row + t] : 1.f) < static_cast<double>(p[i * a.p_row + t]);
    if (!stays) atomicMin(&s_kept, i);
  }
  __syncthreads();
  const int kept = s_kept;
  const TokenRow row(p + kept * a.p_row, a.vocab);
  bool less = kept < count;         // the draft's probabilities are taken off
  const int gone = less && !q ? drafted[kept] : -1;
  const float* off = less && q ? q + kept * a.q_row - row.before : nullptr;   // slots as those of the target
  const bool off_aligned = (reinterpret_cast<uintptr_t>(off) & 15) == 0;
  const long long slice = (row.slots + ctas - 1) / ctas, from = min(row.slots, slice * rank), to = min(row.slots, from + slice);
  const long long step = static_cast<long long>(E) * blockDim.x;
  float4 x[E], y[E];
  auto load = [&](long long at) {   // slots at + e * blockDim.x + tid
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const long long s = at + e * blockDim.x + tid;
      x[e] = s < to ? row.load(s, 0.f) : make_float4(0.f, 0.f, 0.f, 0.f);
      y[e] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (s >= to || !less) continue;
      if (off && off_aligned && row.whole(s)) {
        const uint4 v = ld_stream(off + 4 * s);
        y[e] = make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
      } else if (off) {
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = row.has(s, i) ? off[4 * s + i] : 0.f;
        y[e] = make_float4(f[0], f[1], f[2], f[3]);
      } else {                      // a certain draft: all of it goes
        const long long i = static_cast<long long>(gone) + row.before - 4 * s;
        if (i >= 0 && i < 4) (i == 0 ? x[e].x : i == 1 ? x[e].y : i == 2 ? x[e].z : x[e].w) = 0.f;
      }
    }
  };
  auto rest = [](float have, float off) {
    const double r = static_cast<double>(have) - static_cast<double>(off);
    return r > 0 ? r : 0.0;
  };
  auto sum_of = [&](int e) { return (rest(x[e].x, y[e].x) + rest(x[e].y, y[e].y)) + (rest(x[e].z, y[e].z) + rest(x[e].w, y[e].w)); };
  int token = -1;
  bool have = false;                // this CTA draws the token
  for (int again = 0; again < 2; ++again) {
    double mine = 0;
    for (long long at = from; at < to; at += step) {
      load(at);
#pragma unroll
      for (int e = 0; e < E; ++e) mine += sum_of(e);
    }
    mine = block_sum(mine, s_warp, warps);
    Pick cta;
    double total = mine;
    if (ctas > 1) {
      if (tid == 0) s_mine[0] = mine;
      cluster_arrive();
      cluster_wait();
      double sums[8];
#pragma unroll
      for (uint32_t c = 0; c < 8; ++c)
        if (c < ctas) {
          const uint4 v = cluster_read(s_mine, c);
          sums[c] = __hiloint2double(static_cast<int>(v.y), static_cast<int>(v.x));
        }
      cluster_arrive();
      total = 0;
#pragma unroll
      for (uint32_t c = 0; c < 8; ++c)
        if (c < ctas) total += sums[c];
#pragma unroll
      for (uint32_t c = 0; c < 8; ++c)
        if (c < ctas) cta.part(static_cast<int>(c), sums[c], static_cast<double>(draw) * total);
    } else {
      cta.part(0, mine, static_cast<double>(draw) * total);
    }
    if (total > 0) {
      have = cta.picked == static_cast<int>(rank);
      if (have) {
        const double target = static_cast<double>(draw) * total;
        double before = cta.picked_before;
        long long at = from;
        if (from + step < to) {     // the round, read again
          Pick round;
          round.before = before;
          for (long long r = from; r < to; r += step) {
            load(r);
            double s = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) s += sum_of(e);
            round.part(static_cast<int>((r - from) / step), block_sum(s, s_warp, warps), target);
          }
          at = from + round.picked * step;
          before = round.picked_before;
          load(at);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
          double s = sum_of(e);
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
          if (lane == 0) s_part[e * warps + warp] = s;
        }
        if (tid == 0) s_token = -1;
        __syncthreads();
        // the step and warp, by every warp: E / 2 (or 1) of the E * 16 sums a lane
        constexpr int kEach = (E * 16 + 31) / 32;
        double some_of[kEach], sum = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
          some_of[i] = lane * kEach + i < E * warps ? s_part[lane * kEach + i] : 0.0;
          sum += some_of[i];
        }
        double upto = 0;
        const int who = pick_lane(sum, before, target, &upto);
        Pick part;
        part.before = upto;
#pragma unroll
        for (int i = 0; i < kEach; ++i) part.part(lane * kEach + i, some_of[i], target);
        const int picked = __shfl_sync(0xffffffffu, part.picked, who);
        before = __shfl_sync(0xffffffffu, part.picked_before, who);
        if (picked % warps == warp) {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            if (e != picked / warps) continue;
            if (lane == pick_lane(sum_of(e), before, target, &upto)) {
              Pick value;
              value.before = upto;
              value.part(0, rest(x[e].x, y[e].x), target);
              value.part(1, rest(x[e].y, y[e].y), target);
              value.part(2, rest(x[e].z, y[e].z), target);
              value.part(3, rest(x[e].w, y[e].w), target);
              s_token = static_cast<int>(4 * (at + e * static_cast<long long>(blockDim.x) + tid)) + value.picked - row.before;
            }
          }
        }
        __syncthreads();
        token = s_token;
      }
    } else {
      have = rank == 0;             // nothing to draw from
    }
    if (ctas > 1) cluster_wait();
    if (total > 0 || !less) break;
    less = false;                   // the target has nothing that the draft has less of: drawn from the target
  }
  if (!have) return;
  if (tid == 0) a.accepted[b] = kept;
  for (int i = tid; i <= n; i += blockDim.x) a.out[b * (n + 1) + i] = i < kept ? drafted[i] : i == kept ? token : -1;
}

}  // namespace thinfer
