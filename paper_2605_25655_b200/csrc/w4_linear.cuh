// y[r][o] = sum over the groups of scale[o][group] * sum over its columns of x[r][k] * (code[o][k] - zero[o][group])
// for few token rows r and weights in 4 bits (w4_weights.cuh).
//
// The differences code - zero are whole numbers of five bits, exact in the storage type, so mma.m16n8k16 (16 weight rows,
// 8 tokens, 16 columns) multiplies them with the tokens without any rounding; its FP32 sums are scaled group by group.
#pragma once
#include "w4_weights.cuh"

namespace thinfer {

struct W4LinearArgs {
  W4View v;
  const half_t* x;
  void* y;
  long long x_stride, y_stride;   // elements between token rows
  int rows, n, k;
};

// d += a * b, one m16n8k16 step: a 16 weight rows, b 8 tokens.
__device__ __forceinline__ void w4_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32." THINFER_MMA_SYNC_TYPES ".f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <bool F32>
__device__ __forceinline__ void w4_store(const W4LinearArgs& a, long long row, long long out, float v) {
  if (row >= a.rows || out >= a.n) return;
  if (F32)
    static_cast<float*>(a.y)[row * a.y_stride + out] = v;
  else
    static_cast<half_t*>(a.y)[row * a.y_stride + out] = f_to_h(v);
}

// One warp per tile of 16 weight rows and 8 tokens.
template <int G, bool F32>
__global__ void __launch_bounds__(128) w4_linear_kernel(const __grid_constant__ W4LinearArgs a) {
  constexpr int P = 128 / G;
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const long long tile = static_cast<long long>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  if (tile >= a.v.tiles) return;
  const int row = static_cast<int>(blockIdx.y) * 8 + g;   // of this lane's fragment of the tokens
  const half_t* x = a.x + row * a.x_stride + 8 * t;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  for (long long block = 0; block < a.v.blocks; ++block) {
    const long long u = tile * a.v.blocks + block;
    const uint4* in = reinterpret_cast<const uint4*>(a.v.codes + u * 1024) + lane;
    const uint4 c0 = ld_stream(in), c1 = ld_stream(in + 32);
    const uint32_t words[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
    uint4 token[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int col = static_cast<int>(block) * 128 + 32 * q;
      token[q] = row < a.rows && col + 8 * t < a.k ? ld_stream(x + col) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const float2 scale = h2_to_f2(reinterpret_cast<const half2_t*>(a.v.scales)[(u * 8 + g) * P + p]);
      const W4Zero z = w4_zero<true>(a.v.zeros[(u * 8 + g) * P + p]);
      float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int q = p * 4 / P; q < (p + 1) * 4 / P; ++q) {
        uint32_t r[4];
        w4_unpack<true>(words[2 * q], z, r);
        w4_mma(d, r, token[q].x, token[q].y);
        w4_unpack<true>(words[2 * q + 1], z, r);
        w4_mma(d, r, token[q].z, token[q].w);
      }
      sum[0] = fmaf(scale.x, d[0], sum[0]);
      sum[1] = fmaf(scale.x, d[1], sum[1]);
      sum[2] = fmaf(scale.y, d[2], sum[2]);
      sum[3] = fmaf(scale.y, d[3], sum[3]);
    }
  }
  // rows g and 8 + g of the tile, tokens 2 t and 2 t + 1
  const long long token = static_cast<long long>(blockIdx.y) * 8 + 2 * t;
#pragma unroll
  for (int i = 0; i < 4; ++i) w4_store<F32>(a, token + i % 2, tile * 16 + g + 8 * (i / 2), sum[i] * kW4SumsBy);
}

}  // namespace thinfer
