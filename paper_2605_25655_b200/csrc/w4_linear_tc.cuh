// The products of w4_linear.cuh for more tokens, on the 5th-generation tensor cores: with 17 rows and more, mma.sync would take
// longer than the weights' bytes (16 weight rows by 8 tokens by 16 columns take two cycles of an SM; 64 rows 273 us as a
// simple kernel, 117 us as in w4_linear.cuh, for 19 us of bytes).
//
// Weights are the A operand, in tensor memory: 128 rows by a block of 128 columns per warpgroup, each warp turning the codes of
// its two tiles into the storage type (exact differences code - zero) and storing them with the 16 x 256 bit shape, whose lanes are
// those of the layout in w4_weights.cuh.  Tokens are the B operand, in shared memory with 128-byte swizzle, copied in pieces of 4
// columns, in the order that the layout has the columns in.  The products of a group of columns
// go to columns of tensor memory of their own, from which every thread scales and adds up one weight row by N tokens in FP32.
//
// A CTA holds W warpgroups, each with its own 128 rows, so that what is read of the tokens serves 128 W rows.  The (rows,
// block) units of the whole matrix are dealt out to one CTA per SM in equal contiguous runs; rows that belong to one CTA are stored, the
// others' partial sums go to the workspace and are added up by a second kernel in the order of the CTAs.
#pragma once
#include "w4_linear.cuh"

namespace thinfer {

constexpr int kW4TcAhead = 3, kW4TokenStages = 6;   // units on their way; blocks of tokens, which come one unit earlier

struct W4TcArgs {
  W4LinearArgs a;
  float* parts;          // [CTA][first segment of its run, last one][token][row of the CTA's tile]
  long long row_tiles;   // of 128 W rows
};

template <int N>
constexpr int w4_tc_groups() { return N == 64 ? 3 : 4; }   // warpgroups, by the registers and tensor memory that N tokens take
template <int N, int P>
constexpr int w4_tc_round() {   // groups of columns whose sums tensor memory holds at a time
  constexpr int room = (512 / w4_tc_groups<N>() / 32 * 32 - 64) / N;
  return P < room ? P : room;
}
template <int N, int P>
constexpr int w4_tc_smem() { return 1024 + kW4TokenStages * N * 256 + w4_tc_groups<N>() * 4 * (kW4TcAhead + 1) * W4Stage<2, P>::kBytes; }

// A run of units: CTA c of `ctas` begins at unit c * units / ctas.
__host__ __device__ __forceinline__ long long w4_run(long long c, long long units, long long ctas) { return c * units / ctas; }
__device__ __forceinline__ long long w4_run_of(long long unit, long long units, long long ctas) { return (ctas * (unit + 1) - 1) / units; }

// 16 lanes by 64 columns of tensor memory: r[4 i ..] of lane 4 g + t are columns 8 i + 2 t, + 1 of lane g, then of lane 8 + g.
__device__ __forceinline__ void tmem_st_16x64(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x8.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
      "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}

template <int N, int P>
__global__ void __launch_bounds__(w4_tc_groups<N>() * 128, 1) w4_linear_tc_kernel(const __grid_constant__ W4TcArgs args) {
  constexpr int W = w4_tc_groups<N>(), kRound = w4_tc_round<N, P>(), kRounds = P / kRound, kColumns = 512 / W / 32 * 32;
  constexpr int kStage = W4Stage<2, P>::kBytes, kTokens = N * 256, kTile = W * 128;
  constexpr uint32_t kIdesc = idesc_f16(128, N, 0, 0);
  static_assert(P % kRound == 0 && 64 + kRound * N <= kColumns, "groups per round");
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t token_full[kW4TokenStages], token_empty[kW4TokenStages], done[W];
  __shared__ uint32_t tmem_holder;
  __shared__ volatile int dead;    // a wait has run out: nothing is waited for any more, and the results are NaN
  const W4LinearArgs& a = args.a;
  uint8_t* tokens = smem_raw + (1024 - (smem_u32(smem_raw) & 1023)) % 1024;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    for (int i = 0; i < kW4TokenStages; ++i) {
      mbar_init(&token_full[i], 4 * W);
      mbar_init(&token_empty[i], W);
    }
    for (int i = 0; i < W; ++i) mbar_init(&done[i], 1);
    dead = 0;
    fence_barrier_init();
  }
  if (warp == 1) tmem_alloc(&tmem_holder, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&tmem_holder);
  pdl_launch_dependents();   // behind the allocation: a successor must not take the tensor memory first and then wait for this kernel
  pdl_wait();
  const int blocks = static_cast<int>(a.v.blocks);
  const long long units = args.row_tiles * blocks, ctas = gridDim.x, cta = blockIdx.x;
  const long long u0 = w4_run(cta, units, ctas);
  const int count = static_cast<int>(w4_run(cta + 1, units, ctas) - u0);
  const int first_block = static_cast<int>(u0 % blocks);
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (dead) return false;
    if (mbar_wait(bar, parity, nullptr)) return true;
    dead = 1;
    return false;
  };

  const int wg = warp >> 2;
  const uint8_t* ring = tokens + kW4TokenStages * kTokens + warp * (kW4TcAhead + 1) * kStage;
  const uint32_t mine = tmem + wg * kColumns + (static_cast<uint32_t>((warp & 3) * 32) << 16);   // this warp's lanes
  W4Feed<2, P, kW4TcAhead, 8 * W> feed(a, smem_u32(ring), 0, count, blocks, blocks, 0, 0);
  feed.at(u0, blocks, 2 * warp);
  // tokens warp, warp + 4 W, ...: 32 pieces of 4 columns
  const int token_unit = (((lane >> 3) & 1) * 2 + (lane & 1)) * 2 + ((lane >> 2) & 1);
  const uint32_t token_to = smem_u32(tokens) + (lane >> 4) * (N * 128) + ((lane >> 1) & 1) * 8;
  int token_block = first_block;
  auto copy_tokens = [&](int i) {
    if (i >= count) return;
    const int at = i % kW4TokenStages;
    if (i >= kW4TokenStages) wait(&token_empty[at], (i / kW4TokenStages - 1) & 1);
    const int col = token_block * 128 + 4 * lane;
#pragma unroll
    for (int row = warp; row < N; row += 4 * W) {
      const bool there = row < a.rows && col < a.k;
      asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(token_to + at * kTokens + row * 128 + ((token_unit ^ (row & 7)) << 4)),
                   "l"(there ? a.x + row * a.x_stride + col : a.x), "r"(there ? 8 : 0)
                   : "memory");
    }
    if (++token_block == blocks) token_block = 0;
  };
  copy_tokens(0);
#pragma unroll
  for (int d = 0; d < kW4TcAhead; ++d) {
    copy_tokens(d + 1);
    feed.next();
  }
  float acc[N];
#pragma unroll
  for (int j = 0; j < N; ++j) acc[j] = 0.f;
  float scale[P] = {};
  uint32_t rounds = 0;            // of this warpgroup so far
  long long row_tile = u0 / blocks;
  int block = first_block, begun = first_block;
  const uint8_t* stage = ring;
  // adds the sums of the groups of the last round to this thread's row
  auto collect = [&](int first) {
    const bool ok = __all_sync(0xffffffffu, wait(&done[wg], (rounds - 1) & 1));
    tc_fence_after();
    if (ok) {
#pragma unroll
      for (int p = 0; p < kRound; ++p)
#pragma unroll
        for (int j = 0; j < N; j += 16) {
          uint32_t d[16];
          tmem_ld16(mine + 64 + p * N + j, d);
          tmem_ld_wait();
#pragma unroll
          for (int c = 0; c < 16; ++c) acc[j + c] = fmaf(scale[first + p], __uint_as_float(d[c]), acc[j + c]);
        }
    }
    tc_fence_before();
  };
  // what this CTA has of a row tile, from block `begun` to block `last`
  auto flush = [&](int last) {
    const int row = wg * 128 + (warp & 3) * 32 + lane;
    if (begun == 0 && last == blocks - 1) {
#pragma unroll
      for (int j = 0; j < N; ++j) w4_store(a, j, row_tile * kTile + row, dead ? __int_as_float(0x7fffffff) : acc[j]);
    } else {
      const bool first = row_tile * blocks + begun == u0;
      float* part = args.parts + ((cta * 2 + (first ? 0 : 1)) * N) * kTile + row;
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j < a.rows) part[j * kTile] = dead ? __int_as_float(0x7fffffff) : acc[j];
    }
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = 0.f;
  };
  for (int i = 0; i < count; ++i) {
    w4_copies_wait<kW4TcAhead - 1>();
    fence_proxy_async_smem();                             // the tokens are read by the tensor cores
    __syncwarp();
    if (lane == 0) {
      if (i == 0) mbar_arrive(&token_full[0]);
      mbar_arrive(&token_full[(i + 1) % kW4TokenStages]);
    }
    uint4 codes[2][2];
    uint32_t zeros[2][P];
    float next_scale[P];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int h = 0; h < 2; ++h) codes[c][h] = reinterpret_cast<const uint4*>(stage)[c * 64 + h * 32 + lane];
#pragma unroll
      for (int p = 0; p < P; ++p) zeros[c][p] = stage[W4Stage<2, P>::kZeros + (c * 8 + (lane >> 2)) * P + p];
    }
#pragma unroll
    for (int p = 0; p < P; ++p)   // of this thread's row: tile lane / 16, row lane % 16
      next_scale[p] = h_to_f(reinterpret_cast<const half_t*>(stage + W4Stage<2, P>::kScales)[(((lane >> 4) * 8 + (lane & 7)) * P + p) * 2 + ((lane >> 3) & 1)]);
    stage = stage == ring + kW4TcAhead * kStage ? ring : stage + kStage;
    copy_tokens(i + kW4TcAhead + 1);
    feed.next();
    uint32_t r[32];
    auto unpack = [&](int c) {
#pragma unroll
      for (int w = 0; w < 8; ++w) {   // step w: columns 16 w .. of the block as they lie
        const uint4& from = codes[c][w / 4];
        uint32_t v[4];
        w4_unpack<true>(w % 4 == 0 ? from.x : w % 4 == 1 ? from.y : w % 4 == 2 ? from.z : from.w, w4_zero<true>(zeros[c][w * P / 8]), v);
        r[4 * w] = v[0];
        r[4 * w + 1] = v[2];
        r[4 * w + 2] = v[1];
        r[4 * w + 3] = v[3];
      }
    };
    unpack(0);
    if (i > 0) {
      collect(P - kRound);
      if (block == 0) {
        flush(blocks - 1);
        ++row_tile;
        begun = 0;
      }
    }
    tmem_st_16x64(mine, r);
    unpack(1);
    tmem_st_16x64(mine + (16u << 16), r);
    tmem_st_wait();
    tc_fence_before();
#pragma unroll
    for (int p = 0; p < P; ++p) scale[p] = next_scale[p];
#pragma unroll
    for (int round = 0; round < kRounds; ++round) {
      asm volatile("bar.sync %0, 128;" ::"r"(wg + 1) : "memory");
      if ((warp & 3) == 0 && lane == 0) {
        const int at = i % kW4TokenStages;
        bool ok = round > 0 || wait(&token_full[at], (i / kW4TokenStages) & 1);
        tc_fence_after();
        if (ok && !dead) {
          const uint64_t b = smem_desc_sw128(smem_u32(tokens + at * kTokens), 16, 1024);
#pragma unroll
          for (int p = 0; p < kRound; ++p)
#pragma unroll
            for (int w = 0; w < 8 / P; ++w) {
              const int s = (round * kRound + p) * (8 / P) + w;
              tc_mma_f16_ts(tmem + wg * kColumns + 64 + p * N, tmem + wg * kColumns + s * 8, b + (s / 4) * (N * 128 >> 4) + (s % 4) * 2, kIdesc, w > 0);
            }
          tc_commit(&done[wg]);
          if (round == kRounds - 1) tc_commit(&token_empty[at]);
        }
      }
      __syncwarp();
      ++rounds;
      if (round < kRounds - 1) collect(round * kRound);
    }
    if (++block == blocks) block = 0;
  }
  if (count > 0) {
    collect(P - kRound);
    flush(block == 0 ? blocks - 1 : block - 1);
  }
  w4_copies_wait<0>();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, 512);
}

// Adds up the partial sums of row tiles that several CTAs have: one thread per weight row and token.
template <int N>
__global__ void __launch_bounds__(256) w4_linear_join_kernel(const __grid_constant__ W4TcArgs args, int ctas) {
  constexpr int kTile = w4_tc_groups<N>() * 128;
  pdl_launch_dependents();
  const W4LinearArgs& a = args.a;
  const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x, row_tile = i / kTile;
  const int row = static_cast<int>(i % kTile), token = blockIdx.y;
  const long long blocks = a.v.blocks, units = args.row_tiles * blocks;
  pdl_wait();
  if (row_tile >= args.row_tiles) return;
  const long long c0 = w4_run_of(row_tile * blocks, units, ctas), c1 = w4_run_of(row_tile * blocks + blocks - 1, units, ctas);
  if (c0 == c1) return;
  const long long slot = w4_run(c0, units, ctas) >= row_tile * blocks ? 0 : 1;
  float v = args.parts[((c0 * 2 + slot) * N + token) * kTile + row];
  for (long long c = c0 + 1; c <= c1; ++c) v += args.parts[(c * 2 * N + token) * kTile + row];
  w4_store(a, token, row_tile * kTile + row, v);
}

}  // namespace thinfer
