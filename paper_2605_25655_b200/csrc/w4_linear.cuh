// y[r][o] = sum over the groups of scale[o][group] * sum over its columns of x[r][k] * (code[o][k] - zero[o][group])
// for few token rows r and weights in 4 bits (w4_weights.cuh).
//
// The differences code - zero are whole numbers of five bits, exact in the storage type, so mma.m16n8k16 (16 weight rows,
// 8 tokens, 16 columns) multiplies them with the tokens without any rounding; its FP32 sums are scaled group by group.
//
// Bound by the weights' bytes: they go from memory straight into the registers of the lane that multiplies them, several
// blocks ahead, 64 KB in flight per SM.  The device is divided into clusters of 1 to 8 CTAs, one CTA of 16 warps per SM.  A cluster
// owns a run of weight rows, and each of its CTAs a slice of the columns, whose tokens it keeps in shared memory in the order
// of the lanes that read them.  Inside a CTA the (rows, block of 128 columns) units are dealt out to the warps in equal
// contiguous runs; what a warp has summed up for its rows goes to a slot of shared memory, and at the end the cluster adds
// up the slots in a fixed order, so that equal calls give equal bits, without a workspace and without a second launch.
#pragma once
#include "w4_weights.cuh"

namespace thinfer {

constexpr int kW4Warps = 16;

struct W4LinearArgs {
  W4View v;
  const half_t* x;
  void* y;
  long long x_stride, y_stride;   // elements between token rows
  int rows, n, k, fp32;
  int blocks_at_once;             // blocks of a CTA's slice that shared memory holds
  int groups_at_once;             // row groups (of 16 R rows) whose slots it holds
};

__device__ __forceinline__ uint32_t w4_cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t w4_cluster_size() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void w4_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float4 w4_cluster_load(uint32_t addr, uint32_t rank) {
  uint32_t at;
  float4 v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}

// d += a * b, one m16n8k16 step: a 16 weight rows, b 8 tokens.
__device__ __forceinline__ void w4_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32." THINFER_MMA_SYNC_TYPES ".f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void w4_store(const W4LinearArgs& a, long long row, long long out, float v) {
  if (row >= a.rows || out >= a.n) return;
  v *= kW4SumsBy;
  if (a.fp32)
    static_cast<float*>(a.y)[row * a.y_stride + out] = v;
  else
    static_cast<half_t*>(a.y)[row * a.y_stride + out] = f_to_h(v);
}

// The codes and parameters of one block of R tiles, as lane 4 g + t holds them: scale and zero of group t % P.
template <int R>
struct W4Unit {
  uint4 codes[R][2];
  uint32_t scale[R], zero[R];
};

template <int NT, int R, int P>
__device__ __forceinline__ void w4_multiply(const W4Unit<R>& unit, const uint4* x, float (&sum)[R][NT][4]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    W4Zero z[R];
    float2 scale[R];
    float d[R][NT][4];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const uint32_t s = P == 1 ? unit.scale[i] : __shfl_sync(0xffffffffu, unit.scale[i], (lane & 28) + p);
      z[i] = w4_zero<true>(P == 1 ? unit.zero[i] : __shfl_sync(0xffffffffu, unit.zero[i], (lane & 28) + p));
      scale[i] = h2_to_f2(*reinterpret_cast<const half2_t*>(&s));
#pragma unroll
      for (int j = 0; j < NT; ++j) d[i][j][0] = d[i][j][1] = d[i][j][2] = d[i][j][3] = 0.f;
    }
#pragma unroll
    for (int q = p * 4 / P; q < (p + 1) * 4 / P; ++q) {
      uint4 token[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) token[j] = x[(q * NT + j) * 32 + lane];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        uint32_t r[4];
        w4_unpack<true>(q % 2 ? unit.codes[i][q / 2].z : unit.codes[i][q / 2].x, z[i], r);
#pragma unroll
        for (int j = 0; j < NT; ++j) w4_mma(d[i][j], r, token[j].x, token[j].y);
        w4_unpack<true>(q % 2 ? unit.codes[i][q / 2].w : unit.codes[i][q / 2].y, z[i], r);
#pragma unroll
        for (int j = 0; j < NT; ++j) w4_mma(d[i][j], r, token[j].z, token[j].w);
      }
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        sum[i][j][0] = fmaf(scale[i].x, d[i][j][0], sum[i][j][0]);
        sum[i][j][1] = fmaf(scale[i].x, d[i][j][1], sum[i][j][1]);
        sum[i][j][2] = fmaf(scale[i].y, d[i][j][2], sum[i][j][2]);
        sum[i][j][3] = fmaf(scale[i].y, d[i][j][3], sum[i][j][3]);
      }
  }
}

// NT: tiles of 8 tokens; R: tiles of 16 weight rows that a warp multiplies with what it reads of the tokens; G: columns of a group.
template <int NT, int R, int G>
__global__ void __launch_bounds__(kW4Warps * 32, 1) w4_linear_kernel(const __grid_constant__ W4LinearArgs a) {
  constexpr int P = 128 / G, kAhead = R == 1 ? 4 : 2;
  extern __shared__ uint4 smem[];
  pdl_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ctas = static_cast<int>(w4_cluster_size()), rank = static_cast<int>(w4_cluster_rank());
  const int cluster = static_cast<int>(blockIdx.x) / ctas, clusters = static_cast<int>(gridDim.x) / ctas;
  const int first_token = static_cast<int>(blockIdx.y) * (8 * NT);
  const int blocks = static_cast<int>(a.v.blocks), tiles = static_cast<int>(a.v.tiles);
  // this CTA's blocks and this cluster's row groups
  const int block0 = static_cast<int>(static_cast<long long>(blocks) * rank / ctas);
  const int slice = static_cast<int>(static_cast<long long>(blocks) * (rank + 1) / ctas) - block0;
  const long long groups = (tiles + R - 1) / R;
  const int group0 = static_cast<int>(groups * cluster / clusters), group1 = static_cast<int>(groups * (cluster + 1) / clusters);
  uint4* x_s = smem;                                        // [block][q][token tile][lane]
  uint4* slots = smem + a.blocks_at_once * (4 * NT * 32);   // [row group + warp][tile][token tile][lane]
  const int held = a.blocks_at_once;
  const int at_p = lane / 4 * P + lane % P;                 // this lane's parameters of a block
  pdl_wait();

  for (int from = group0; from < group1; from += a.groups_at_once) {
    const int batch = min(a.groups_at_once, group1 - from);
    // a run of the (row group, block) units, block by block
    const int units = batch * held, u0 = static_cast<int>(static_cast<long long>(units) * warp / kW4Warps), u1 = static_cast<int>(static_cast<long long>(units) * (warp + 1) / kW4Warps);
    for (int phase = 0; phase * held < slice || phase == 0; ++phase) {
      const int here = min(held, slice - phase * held);     // blocks of this phase; the rest of `held` is skipped
      W4Unit<R> ring[kAhead];
      int next_group = u0 / held, next_block = u0 - next_group * held, next = u0;
      auto load = [&](W4Unit<R>& unit) {
        if (next >= u1) return;
        if (next_block < here) {
#pragma unroll
          for (int i = 0; i < R; ++i) {
            const int tile = (from + next_group) * R + i;
            if (R > 1 && tile >= tiles) {
              unit.codes[i][0] = unit.codes[i][1] = make_uint4(0, 0, 0, 0);
              unit.scale[i] = unit.zero[i] = 0;
              continue;
            }
            const long long at = static_cast<long long>(tile) * blocks + block0 + phase * held + next_block;
            const uint4* codes = reinterpret_cast<const uint4*>(a.v.codes) + at * 64 + lane;
            unit.codes[i][0] = ld_stream(codes);
            unit.codes[i][1] = ld_stream(codes + 32);
            unit.scale[i] = reinterpret_cast<const uint32_t*>(a.v.scales)[at * (8 * P) + at_p];
            unit.zero[i] = a.v.zeros[at * (8 * P) + at_p];
          }
        }
        ++next;
        if (++next_block == held) {
          next_block = 0;
          ++next_group;
        }
      };
#pragma unroll
      for (int d = 0; d < kAhead; ++d) load(ring[d]);
      // the tokens of this slice's blocks
      if (from == group0 || held < slice) {
        __syncthreads();                                    // nobody reads those of the phase before any more
        for (int i = tid; i < 8 * NT * 16 * here; i += kW4Warps * 32) {
          const int row = i / (16 * here), piece = i - row * (16 * here), col = (block0 + phase * held) * 128 + piece * 8;
          const bool there = first_token + row < a.rows && col < a.k;
          const half_t* src = there ? a.x + (first_token + row) * a.x_stride + col : a.x;
          uint4* dst = x_s + ((piece >> 2) * NT + (row >> 3)) * 32 + (row & 7) * 4 + (piece & 3);
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
        }
        asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory");
        __syncthreads();
      }
      float sum[R][NT][4] = {};
      int group = u0 / held, block = u0 - group * held;
      for (int u = u0; u < u1; u += kAhead) {
#pragma unroll
        for (int d = 0; d < kAhead; ++d) {
          if (u + d < u1) {
            if (block < here) w4_multiply<NT, R, P>(ring[d], x_s + block * (4 * NT * 32), sum);
            load(ring[d]);
            if (++block == held || u + d + 1 == u1) {       // the last unit of a row group, or of this warp
              float4* slot = reinterpret_cast<float4*>(slots) + (group + warp) * (R * NT * 32) + lane;
#pragma unroll
              for (int i = 0; i < R; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                  float4& to = slot[(i * NT + j) * 32];
                  float4 v = make_float4(sum[i][j][0], sum[i][j][1], sum[i][j][2], sum[i][j][3]);
                  if (phase > 0) v.x += to.x, v.y += to.y, v.z += to.z, v.w += to.w;
                  to = v;
                  sum[i][j][0] = sum[i][j][1] = sum[i][j][2] = sum[i][j][3] = 0.f;
                }
              if (block == held) {
                block = 0;
                ++group;
              }
            }
          }
        }
      }
    }
    // the cluster adds up what its CTAs' warps have for each row group
    w4_cluster_sync();
    const uint32_t slots_at = smem_u32(slots);
    for (int i = rank * (kW4Warps * 32) + tid; i < batch * (R * NT * 32); i += ctas * (kW4Warps * 32)) {
      const int group = i / (R * NT * 32), part = i - group * (R * NT * 32);
      // warp w begins at unit w * units / 16: the ones that hold the group's first and last unit
      const int w0 = (kW4Warps * (group * held + 1) - 1) / units, w1 = (kW4Warps * ((group + 1) * held) - 1) / units;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int c = 0; c < ctas; ++c)
        for (int w = w0; w <= w1; ++w) {
          if (w * units / kW4Warps == (w + 1) * units / kW4Warps) continue;   // it had none
          const float4 p = w4_cluster_load(slots_at + static_cast<uint32_t>((group + w) * (R * NT * 32) + part) * 16, c);
          v.x += p.x, v.y += p.y, v.z += p.z, v.w += p.w;
        }
      const long long out = (static_cast<long long>(from + group) * R + part / (NT * 32)) * 16 + part % 32 / 4;
      const long long token = first_token + part / 32 % NT * 8 + part % 4 * 2;
      w4_store(a, token, out, v.x);
      w4_store(a, token + 1, out, v.y);
      w4_store(a, token, out + 8, v.z);
      w4_store(a, token + 1, out + 8, v.w);
    }
    w4_cluster_sync();                                      // the slots are read, by the other CTAs too
  }
}

}  // namespace thinfer
