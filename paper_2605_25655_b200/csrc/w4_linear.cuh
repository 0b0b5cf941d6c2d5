// y[r][o] = sum over the groups of scale[o][group] * sum over its columns of x[r][k] * (code[o][k] - zero[o][group])
// for few token rows r and weights in 4 bits (w4_weights.cuh).
//
// The differences code - zero are whole numbers of five bits, exact in the storage type, so mma.m16n8k16 (16 weight rows,
// 8 tokens, 16 columns) multiplies them with the tokens without any rounding; its FP32 sums are scaled group by group.
//
// Bound by the weights' bytes: every warp brings its own into a ring of shared memory, two units of 2 KB ahead of the one that it
// multiplies, 64 KB (with two token tiles 48) under way per SM (loads into registers instead stopped each warp at its newest load, 42 us
// against 29 for 4 x 28672 x 8192).  The device is divided into clusters of 1 to 8 CTAs, one CTA of 16 (12) warps per SM.  A cluster owns a
// run of weight rows, and each of its CTAs a slice of the columns, whose tokens it keeps in shared memory in the order of
// the lanes that read them.  Inside a CTA the (32 rows, 128 columns) units are dealt out to the warps in equal contiguous
// runs; what a warp has summed up for its rows goes to a slot of shared memory, and at the end the cluster adds up the
// slots in a fixed order, so that equal calls give equal bits, without a workspace and without a second launch.
//
// 4 x 28672 x 8192 in groups of 128 (122 MB): 29 us alone in a graph, 65 % of a copy's rate; the stream itself takes 20 us (6.0
// TB/s), the rest is the launch, the tokens (1.2 us), the sums in the CTA and the cluster (2.5 us).  1 x 4096 x 4096: 5.9 us.
// 16 x 28672 x 8192: 39 us; the matrix instructions take 28 of 68 cycles a unit, dependences between few warps the rest.  BF16, whose
// scales take the factor of the differences off: 44 us.  In groups of 32 up to 12 bytes a thread are spilled.
// Tried: FP16 codes as subnormal numbers with the zero points taken off sums of the tokens (half of the unpacking: no
// change for 8 tokens, 46 instead of 41 us for 16); four tiles a warp and 8 warps (32 and 47 us); one tile and 16 warps.
#pragma once
#include "w4_weights.cuh"

namespace thinfer {

constexpr int kW4Ahead = 2;   // units that are on their way while one is multiplied

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
// Release: what this warp has read of other CTAs' memory has been read, so that they may leave.
__device__ __forceinline__ void w4_cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void w4_cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ float4 w4_cluster_load(uint32_t addr, uint32_t rank) {
  uint32_t at;
  float4 v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at));
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
  if (a.fp32)
    static_cast<float*>(a.y)[row * a.y_stride + out] = v;
  else
    static_cast<half_t*>(a.y)[row * a.y_stride + out] = f_to_h(v);
}

__device__ __forceinline__ void w4_mma_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {   // d = a * b
  asm("mma.sync.aligned.m16n8k16.row.col.f32." THINFER_MMA_SYNC_TYPES ".f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

// What lane 4 g + t has summed up: weight rows out + g and out + 8 + g, tokens token + 2 t, + 1.
__device__ __forceinline__ void w4_output(const W4LinearArgs& a, long long out, int token, const float4& v) {
  const int lane = threadIdx.x & 31;
  out += lane >> 2;
  token += 2 * (lane & 3);
  w4_store(a, token, out, v.x);
  w4_store(a, token + 1, out, v.y);
  w4_store(a, token, out + 8, v.z);
  w4_store(a, token + 1, out + 8, v.w);
}

// What a warp multiplies at a time: one block of R tiles, with their scales and zeros behind the codes.
template <int R, int P>
struct W4Stage {
  static constexpr int kScales = R * 1024, kZeros = kScales + R * P * 32, kBytes = (kZeros + R * P * 8 + 15) / 16 * 16;
};

__device__ __forceinline__ void w4_copy16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void w4_copy8(uint32_t dst, const void* src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void w4_copies_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void w4_copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// sum += scale * (a block of R tiles times its tokens).  x[j]: where this lane finds its columns of token tile j; `quarter`
// from one 32 columns to the next.
template <int NT, int R, int P, bool FAR>
__device__ __forceinline__ void w4_multiply(const uint8_t* stage, const uint32_t (&scales)[R][P], const uint4* const (&x)[NT], int quarter, float (&sum)[R][NT][4]) {
  const int lane = threadIdx.x & 31;
  uint4 codes[R][2];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) codes[i][h] = reinterpret_cast<const uint4*>(stage)[i * 64 + h * 32 + lane];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    W4Zero z[R];
    float2 scale[R];
    float d[R][NT][4];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int at = (i * 8 + (lane >> 2)) * P + p;
      z[i] = w4_zero<true>(stage[W4Stage<R, P>::kZeros + at]);
      scale[i] = h2_to_f2(*reinterpret_cast<const half2_t*>(&scales[i][p]));
      if (!FAR && kW4SumsBy != 1.f) scale[i].x *= kW4SumsBy, scale[i].y *= kW4SumsBy;
    }
#pragma unroll
    for (int q = p * 4 / P; q < (p + 1) * 4 / P; ++q) {
      uint4 token[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) token[j] = x[j][q * quarter];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        uint32_t r[4];
        w4_unpack<true>(q % 2 ? codes[i][q / 2].z : codes[i][q / 2].x, z[i], r);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          if (q == p * 4 / P)
            w4_mma_first(d[i][j], r, token[j].x, token[j].y);
          else
            w4_mma(d[i][j], r, token[j].x, token[j].y);
        }
        w4_unpack<true>(q % 2 ? codes[i][q / 2].w : codes[i][q / 2].y, z[i], r);
#pragma unroll
        for (int j = 0; j < NT; ++j) w4_mma(d[i][j], r, token[j].z, token[j].w);
      }
    }
    if (FAR)
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const bool x_far = w4_far(scale[i].x), y_far = w4_far(scale[i].y);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          d[i][j][0] *= x_far ? kW4SumsBy : 1.f, d[i][j][1] *= x_far ? kW4SumsBy : 1.f;
          d[i][j][2] *= y_far ? kW4SumsBy : 1.f, d[i][j][3] *= y_far ? kW4SumsBy : 1.f;
        }
        scale[i].x *= x_far ? 1.f : kW4SumsBy;
        scale[i].y *= y_far ? 1.f : kW4SumsBy;
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

template <int NT, int R, int P>
__device__ __forceinline__ void w4_multiply(const uint8_t* stage, const uint4* const (&x)[NT], int quarter, float (&sum)[R][NT][4]) {
  uint32_t scales[R][P];
  bool far = false;
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int p = 0; p < P; ++p) {
      scales[i][p] = reinterpret_cast<const uint32_t*>(stage + W4Stage<R, P>::kScales)[(i * 8 + (threadIdx.x & 31) / 4) * P + p];
      far |= w4_far(scales[i][p]);
    }
  if (kW4SumsBy != 1.f && __any_sync(0xffffffffu, far))   // one way for the whole block: in between, a branch would keep the instructions of two groups apart
    w4_multiply<NT, R, P, true>(stage, scales, x, quarter, sum);
  else
    w4_multiply<NT, R, P, false>(stage, scales, x, quarter, sum);
}

// The units of one warp on their way into its ring: one block of R tiles after the other along a row group, then the next
// group's.  Every lane keeps the address of what it copies itself, so that a unit costs a few additions.
template <int R, int P>
struct W4Feed {
  static constexpr int kPieces = 5 * P * R;       // of 8 bytes: 4 P of scales and P of zeros for each tile
  const W4LinearArgs& a;
  uint32_t ring, to;
  int left, step, steps, here, block, tile;       // units, step of the group, steps of a group and how many of them exist, the first one's block
  const uint8_t* codes;
  const uint8_t* params[(kPieces + 31) / 32];
  long long apart[R];                             // from the first tile's codes to the others'

  __device__ __forceinline__ void begin_group() {
    const int lane = threadIdx.x & 31;
    const long long blocks = a.v.blocks;
    // behind the last tile the last one is read again; what comes of it is not kept
    const int last = static_cast<int>(a.v.tiles) - 1, first = min(tile, last);
    const long long at = first * blocks + block;
    codes = a.v.codes + at * 1024 + lane * 16;
#pragma unroll
    for (int i = 0; i < R; ++i) apart[i] = (min(tile + i, last) - first) * blocks * 1024;
#pragma unroll
    for (int h = 0; h < (kPieces + 31) / 32; ++h) {
      const int piece = lane + 32 * h, i = piece / (5 * P), j = piece - i * 5 * P;
      const long long mine = at + (min(tile + i, last) - first) * blocks;
      params[h] = j < 4 * P ? a.v.scales + mine * (32 * P) + j * 8 : a.v.zeros + mine * (8 * P) + (j - 4 * P) * 8;
    }
  }
  __device__ __forceinline__ W4Feed(const W4LinearArgs& args, uint32_t ring_, int u0, int u1, int steps_, int here_, int block_, int first_tile)
      : a(args), ring(ring_), to(ring_), left(u1 - u0), step(u0 % steps_), steps(steps_), here(here_), block(block_), tile(first_tile + u0 / steps_ * R) {
    begin_group();
    codes += step * 1024;
#pragma unroll
    for (int h = 0; h < (kPieces + 31) / 32; ++h) params[h] += step * stride(h);
  }
  __device__ __forceinline__ static int stride(int h) {
    const int piece = (threadIdx.x & 31) + 32 * h;
    return piece % (5 * P) < 4 * P ? 32 * P : 8 * P;
  }
  __device__ __forceinline__ void next() {
    const int lane = threadIdx.x & 31;
    if (left > 0) {
      if (step < here) {
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) w4_copy16(to + i * 1024 + h * 512 + lane * 16, codes + apart[i] + h * 512);
#pragma unroll
        for (int h = 0; h < (kPieces + 31) / 32; ++h) {
          const int piece = lane + 32 * h, i = piece / (5 * P), j = piece - i * 5 * P;
          const int dst = j < 4 * P ? W4Stage<R, P>::kScales + i * P * 32 + j * 8 : W4Stage<R, P>::kZeros + i * P * 8 + (j - 4 * P) * 8;
          if (piece < kPieces) w4_copy8(to + dst, params[h]);
        }
      }
      --left;
      if (++step == steps) {
        step = 0;
        tile += R;
        if (left > 0) begin_group();
      } else {
        codes += 1024;
#pragma unroll
        for (int h = 0; h < (kPieces + 31) / 32; ++h) params[h] += stride(h);
      }
      to = to == ring + kW4Ahead * W4Stage<R, P>::kBytes ? ring : to + W4Stage<R, P>::kBytes;
    }
    w4_copies_done();
  }
};

// NT: tiles of 8 tokens; R: tiles of 16 weight rows that a warp multiplies with what it reads of the tokens; G: columns of a group.
// Warps: a CTA's.
template <int NT, int R, int G, int Warps>
__global__ void __launch_bounds__(Warps * 32, 1) w4_linear_kernel(const __grid_constant__ W4LinearArgs a) {
  constexpr int P = 128 / G, kStage = W4Stage<R, P>::kBytes, kGroup = R * NT * 32;
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
  const int held = a.blocks_at_once;
  const int rows = min(8 * NT, a.rows - first_token);       // of the tokens
  uint4* x_s = smem;                                        // [block][q][token][t]
  uint4* slots = smem + held * (16 * rows);                 // [row group + warp][tile][token tile][lane]
  const uint8_t* ring = reinterpret_cast<const uint8_t*>(slots + (a.groups_at_once + Warps - 1) * kGroup) + warp * (kW4Ahead + 1) * kStage;
  bool waited = false;

  for (int from = group0; from < group1; from += a.groups_at_once) {
    const int batch = min(a.groups_at_once, group1 - from);
    // a run of the (row group, block) units
    const int units = batch * held, u0 = units * warp / Warps, u1 = units * (warp + 1) / Warps;
    for (int phase = 0; phase * held < slice || phase == 0; ++phase) {
      const int here = min(held, slice - phase * held);     // blocks of this phase; the rest of `held` is skipped
      const bool tokens = from == group0 || held < slice;   // to be fetched for this phase
      W4Feed<R, P> feed(a, smem_u32(ring), u0, u1, held, here, block0 + phase * held, from * R);
      if (!waited) pdl_wait();                              // behind the index arithmetic, which takes as long as a load
      waited = true;
      if (tokens) {
        __syncthreads();                                    // nobody reads those of the phase before any more
        // the products of a token that is not there go nowhere: only what lies behind the last column has to be 0
        const int col0 = (block0 + phase * held) * 128;
        for (int piece = tid; piece < 16 * here; piece += Warps * 32) {
          const int col = col0 + piece * 8;
          const half_t* src = a.x + first_token * a.x_stride + col;
          uint32_t dst = smem_u32(x_s + (piece >> 2) * rows * 4 + (piece & 3));
#pragma unroll 4
          for (int row = 0; row < rows; ++row, dst += 64)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(col < a.k ? src + row * a.x_stride : a.x), "r"(col < a.k ? 16 : 0) : "memory");
        }
        w4_copies_done();
      }
#pragma unroll
      for (int d = 0; d < kW4Ahead; ++d) feed.next();
      if (tokens) {
        w4_copies_wait<kW4Ahead>();
        __syncthreads();
      }
      float sum[R][NT][4] = {};
      int group = u0 / held, step = u0 - group * held;
      const uint8_t* stage = ring;
      const uint4* x[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) x[j] = x_s + step * (16 * rows) + min(8 * j + (lane >> 2), rows - 1) * 4 + (lane & 3);
      for (int u = u0; u < u1; ++u) {
        w4_copies_wait<kW4Ahead - 1>();
        __syncwarp();                                       // all lanes' copies of this unit are there, and all have read the last one
        feed.next();
        if (step < here) w4_multiply<NT, R, P>(stage, x, 4 * rows, sum);
#pragma unroll
        for (int j = 0; j < NT; ++j) x[j] += 16 * rows;
        stage = stage == ring + kW4Ahead * kStage ? ring : stage + kStage;
        if (++step == held || u + 1 == u1) {                // the last unit of a row group, or of this warp
          float4* slot = reinterpret_cast<float4*>(slots) + (group + warp) * kGroup + lane;
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
#pragma unroll
          for (int j = 0; j < NT; ++j) x[j] -= step * (16 * rows);
          step = 0;
          ++group;
        }
      }
    }
    __syncthreads();
    // What the warps of this CTA have for each row group, in the order of the warps: w0 holds the group's first unit, w1 its
    // last; the sum goes to w0's slot.  Warp w begins at unit w * units / Warps.
    auto warp_of = [&](int unit) { return __popc(__ballot_sync(0xffffffffu, lane < Warps && units * lane / Warps <= unit)) - 1; };
    float4* slot = reinterpret_cast<float4*>(slots) + lane;
    for (int g = warp; g < batch; g += Warps) {
      const int w0 = warp_of(g * held), w1 = warp_of((g + 1) * held - 1);
      float4* to = slot + (g + w0) * kGroup;
#pragma unroll
      for (int i = 0; i < R * NT; ++i) {
        float4 v = to[i * 32];
        for (int w = w0 + 1; w <= w1; ++w) {
          if (w * units / Warps == (w + 1) * units / Warps) continue;   // it had none
          const float4 p = to[(w - w0) * kGroup + i * 32];
          v.x += p.x, v.y += p.y, v.z += p.z, v.w += p.w;
        }
        if (ctas == 1)
          w4_output(a, ((from + g) * R + i / NT) * 16ll, first_token + i % NT * 8, v);
        else
          to[i * 32] = v;
      }
    }
    if (ctas > 1) {
      w4_cluster_sync();
      for (int g = rank * Warps + warp; g < batch; g += ctas * Warps) {
        const int w0 = warp_of(g * held);
        const uint32_t at = smem_u32(slot + (g + w0) * kGroup);
        float4 v[R * NT];
#pragma unroll
        for (int i = 0; i < R * NT; ++i) {
          float4 p[8];
#pragma unroll
          for (int c = 0; c < 8; ++c)
            if (c < ctas) p[c] = w4_cluster_load(at + i * 512, c);
          v[i] = p[0];
#pragma unroll
          for (int c = 1; c < 8; ++c)
            if (c < ctas) v[i].x += p[c].x, v[i].y += p[c].y, v[i].z += p[c].z, v[i].w += p[c].w;
        }
        if (g + ctas * Warps >= batch) w4_cluster_arrive();   // this warp's last read, ahead of its last stores
#pragma unroll
        for (int i = 0; i < R * NT; ++i) w4_output(a, ((from + g) * R + i / NT) * 16ll, first_token + i % NT * 8, v[i]);
      }
      if (rank * Warps + warp >= batch) w4_cluster_arrive();  // it had nothing to read
      w4_cluster_wait();                                    // the slots are read, by the other CTAs too
    } else {
      __syncthreads();
    }
  }
}

}  // namespace thinfer
