// The products of w4_linear.cuh for more tokens, on the 5th-generation tensor cores: with mma.sync, 16 weight rows by 8 tokens by 16
// columns take two cycles of an SM, which is more than their bytes take from 24 tokens on, and the fragments of the tokens
// cost registers and issue slots before that.
//
// Weights are the A operand, in tensor memory: 128 rows by a block of 128 columns per warpgroup, each warp turning the codes of
// its two tiles into the storage type (exact differences code - zero) and storing them with the 16 x 256 bit shape, whose lanes are
// those of the layout in w4_weights.cuh.  Tokens are the B operand, in shared memory with 128-byte swizzle.  A first, small kernel lays
// them out block by block as they stand there, their columns in the order that the weights have.  The products of a group
// of columns go to columns of tensor memory of their own, from which every thread scales and adds up one weight row by N
// tokens in FP32.
//
// A CTA per SM: W warpgroups that unpack, each with its own 128 rows; a warp that feeds codes, scales and tokens of one block
// after the other to a ring (three copies a block, and the zeros by its lanes: loaded by those who unpack, two blocks ahead, they
// cost 5 % more); and a warp for each warpgroup that issues its tensor instructions (as a
// part of the unpacking warps that took a third of their time).  While the tensor cores multiply a block, its warpgroup unpacks
// the next.  The (rows, block) units of the whole matrix are dealt out to the CTAs in equal contiguous runs; their partial
// sums go to the workspace, and a last kernel adds them up in the order of the CTAs.
//
// 64 x 28672 x 8192 in groups of 128 (127 MB): 45 us in FP16, 47 in BF16, of which 7 are the two small kernels; 32 rows 34 and 37.  A
// copy would take 19, the products 18.  Bound by the unpacking: two or three warps for each of a SM's quarters do not cover its
// dependences, and their registers (tokens' sums, codes, 64 unpacked words) leave room for no more.
#pragma once
#include "w4_linear.cuh"

namespace thinfer {

// W: two warpgroups with 168 registers a thread, or three with 128 - where those are enough and the sums of 128 rows have room beside
// the weights.  28672 x 8192 in FP16, us, two / three: 64 rows 44.7 / 45.0 in groups of 128, 54.6 / 64.2 of 64, 77.8 / 84.1 of 32; 32 rows
// 38.7 / 34.3 in groups of 128, 41.2 / 41.0 of 64, 48.1 / 57.0 of 32 (BF16 the same way).
constexpr int w4_tc_groups(int n, int group) { return n == 64 || group < 128 ? 2 : 3; }

struct W4TcArgs {
  W4LinearArgs a;
  uint8_t* tokens;       // [block][N * 256 bytes]
  float* parts;          // [row tile + CTA][token][row of the tile]: every piece of a row tile that a CTA has, each in a place of its own
  long long row_tiles;
};

template <int N, int P>
struct W4Tc {
  static constexpr int W = w4_tc_groups(N, 128 / P), kTile = W * 128, kThreads = (4 * W + 1 + W) * 32;   // kTile: weight rows of a CTA
  static constexpr int kColumns = 512 / W / 32 * 32;                                          // of tensor memory, for a warpgroup
  // Tensor memory of a warpgroup: the weights of one or two blocks, and the sums of one or two blocks, or of as many groups of
  // a block as fit (the others follow in further rounds).
  static constexpr int kA = P * N <= kColumns - 128 ? 2 : 1, kSums = kA * 64, kRoom = (kColumns - kSums) / N;
  static constexpr int kRound = P <= kRoom ? P : kRoom >= 2 ? 2 : 1, kRounds = P / kRound;
  static constexpr int kD = kRounds == 1 && kA == 2 && 2 * P * N <= kColumns - kSums ? 2 : 1;
  static constexpr int kCodes = W * 8192, kScales = W * 8 * 32 * P, kTokens = N * 256;
  static constexpr int kBytes = kCodes + kTokens + kScales, kZeros = W * 8 * 8 * P, kStage = (kBytes + kZeros + 1023) / 1024 * 1024;
  static constexpr int kFit = 224 * 1024 / kStage, kStages = kFit < 8 ? kFit : 8;
  static constexpr int kSmem = 1024 + kStages * kStage;
  static_assert(P % kRound == 0 && kSums + kD * kRound * N <= kColumns, "the sums of a round");
};

// A run of units: CTA c of `ctas` begins at unit c * units / ctas.
__host__ __device__ __forceinline__ long long w4_run(long long c, long long units, long long ctas) { return c * units / ctas; }
__device__ __forceinline__ int w4_run_of(long long unit, long long units, long long ctas) {
  const long long n = ctas * (unit + 1) - 1;
  if (n < 1ll << 32) return static_cast<int>(static_cast<uint32_t>(n) / static_cast<uint32_t>(units));
  return static_cast<int>(n / units);
}

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
// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(one));
  return one != 0;
}
__device__ __forceinline__ void w4_bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}

// The tokens, block by block as shared memory holds them: 64 columns in 128 bytes of a row of N, twice, the 16-byte units of
// row r at unit ^ (r % 8).  Position 16 s' + 4 t + 2 b + e of half c is column 64 c + 32 (s' / 2) + 8 t + 4 (s' % 2) + 2 b + e of the block.
template <int N>
__global__ void __launch_bounds__(256) w4_tokens_kernel(const __grid_constant__ W4TcArgs args) {
  pdl_wait();
  // Behind the wait: the next kernel takes an SM's shared and tensor memory for itself, and its warps wait for the feeder's copies for a
  // limited time, which must not pass behind a long predecessor of this one.
  pdl_launch_dependents();
  const W4LinearArgs& a = args.a;
  const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
  const long long block = i / (N * 16);
  if (block < a.v.blocks) {
    const int at = static_cast<int>(i % (N * 16)), half = at / (N * 8), row = at / 8 % N, unit = at % 8, from = unit ^ (row & 7);
    const long long col = block * 128 + half * 64 + from / 4 * 32 + (from & 1) * 16 + (from / 2 & 1) * 4;
    uint2 lo = make_uint2(0, 0), hi = lo;
    if (row < a.rows) {
      const half_t* x = a.x + row * a.x_stride + col;
      if (col < a.k) lo = *reinterpret_cast<const uint2*>(x);
      if (col + 8 < a.k) hi = *reinterpret_cast<const uint2*>(x + 8);
    }
    reinterpret_cast<uint4*>(args.tokens)[i] = make_uint4(lo.x, lo.y, hi.x, hi.y);
  }
  fence_proxy_async_all();
}

template <int N, int P>
__global__ void __launch_bounds__(W4Tc<N, P>::kThreads, 1)
w4_linear_tc_kernel(const __grid_constant__ W4TcArgs args, const __grid_constant__ CUtensorMap codes_map, const __grid_constant__ CUtensorMap scales_map) {
  using T = W4Tc<N, P>;
  constexpr int W = T::W;
  constexpr uint32_t kIdesc = idesc_f16(128, N, 0, 0);
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t full[T::kStages], empty[T::kStages], a_full[W][2], d_free[W], done[W][2];
  __shared__ uint32_t tmem_holder;
  __shared__ volatile int dead;    // a wait has run out: whom it happened to waits no more, and the results are NaN
  const W4LinearArgs& a = args.a;
  uint8_t* ring = smem_raw + (1024 - (smem_u32(smem_raw) & 1023)) % 1024;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  if (tid == 0) {
    for (int i = 0; i < T::kStages; ++i) {
      mbar_init(&full[i], 1 + 32);       // the copies, and what each lane of the feeder has copied itself
      mbar_init(&empty[i], 4 * W + W);   // the warps that unpack, and the products that read the tokens
    }
    for (int i = 0; i < W; ++i) {
      mbar_init(&d_free[i], 4);
      for (int j = 0; j < 2; ++j) {      // of even and odd units: with two sums the warps may be a unit ahead of who waits
        mbar_init(&a_full[i][j], 4);
        mbar_init(&done[i][j], 1);
      }
    }
    dead = 0;
    fence_barrier_init();
  }
  if (warp == 1) tmem_alloc(&tmem_holder, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&tmem_holder);
  pdl_launch_dependents();   // behind the allocation: a successor must not take the tensor memory first and then wait for this kernel
  const int blocks = static_cast<int>(a.v.blocks);
  const long long units = args.row_tiles * blocks, ctas = gridDim.x, cta = blockIdx.x;
  const long long u0 = w4_run(cta, units, ctas);
  const int count = static_cast<int>(w4_run(cta + 1, units, ctas) - u0);
  const int first_tile = static_cast<int>(u0 / blocks), first_block = static_cast<int>(u0 % blocks);
  bool alive = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (alive && !mbar_wait(bar, parity, nullptr)) {
      alive = false;
      dead = 1;
    }
    return alive;
  };

  if (warp == 4 * W) {
    // The feeder.  Nothing is read ahead of this wait: the packed weights may have been written by the kernel in front of the call.
    pdl_wait();
    fence_proxy_async_all();
    int tile = first_tile, block = first_block;
    int issued = count;
    for (int i = 0; i < count; ++i) {
      const int s = i % T::kStages;
      if (i >= T::kStages && !__all_sync(0xffffffffu, wait(&empty[s], (i / T::kStages - 1) & 1))) {
        issued = i;
        break;
      }
      uint8_t* stage = ring + s * T::kStage;
      if (lane == 0) {
        mbar_expect_tx(&full[s], T::kBytes);
        tma_load_3d(stage, &codes_map, &full[s], 0, block, tile * 8 * W);
        tma_load_3d(stage + T::kCodes + T::kTokens, &scales_map, &full[s], 0, block, tile * 8 * W);
        w4_bulk_load(stage + T::kCodes, args.tokens + static_cast<long long>(block) * T::kTokens, T::kTokens, &full[s]);
      }
      if (lane < 8 * W) {          // the zeros of a tile: up to 32 bytes, which need not be a tensor copy's 16
        const uint8_t* from = a.v.zeros + (min(tile * 8 * W + lane, static_cast<int>(a.v.tiles) - 1) * static_cast<long long>(blocks) + block) * (8 * P);
        const uint32_t to = smem_u32(stage + T::kBytes + lane * (8 * P));
        if (P == 1) w4_copy8(to, from);
        if (P >= 2) w4_copy16(to, from);
        if (P == 4) w4_copy16(to + 16, from + 16);
      }
      asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&full[s])) : "memory");
      if (++block == blocks) {
        block = 0;
        ++tile;
      }
    }
    // nothing of its own is under way when it leaves
    for (int i = issued > T::kStages ? issued - T::kStages : 0; i < issued; ++i) mbar_wait(&full[i % T::kStages], (i / T::kStages) & 1, nullptr);
  } else if (warp > 4 * W) {
    // the products of warpgroup wg
    const int wg = warp - 4 * W - 1;
    const uint32_t columns = tmem + wg * T::kColumns;
    const uint64_t first = smem_desc_sw128(smem_u32(ring + T::kCodes), 16, 1024);
    uint32_t frees = 0;
    for (int i = 0; i < count; ++i) {
      const int s = i % T::kStages;
      bool ok = wait(&full[s], (i / T::kStages) & 1);
      ok = wait(&a_full[wg][i & 1], (i >> 1) & 1) && ok;
      const uint64_t b = first + static_cast<uint64_t>(s * (T::kStage >> 4));
#pragma unroll
      for (int round = 0; round < T::kRounds; ++round) {
        if (round > 0) ok = wait(&d_free[wg], frees++ & 1) && ok;
        ok = __all_sync(0xffffffffu, ok);
        tc_fence_after();
        if (ok && elect_one()) {
#pragma unroll
          for (int p = 0; p < T::kRound; ++p)
#pragma unroll
            for (int w = 0; w < 8 / P; ++w) {
              const int st = (round * T::kRound + p) * (8 / P) + w;
              tc_mma_f16_ts(columns + T::kSums + (T::kD == 2 ? (i & 1) * (P * N) : 0) + p * N, columns + (T::kA == 2 ? (i & 1) * 64 : 0) + st * 8, b + (st / 4) * (N * 128 >> 4) + (st % 4) * 2, kIdesc, w > 0);
            }
          tc_commit(&done[wg][T::kRounds == 1 ? i & 1 : 0]);
          if (round == T::kRounds - 1) tc_commit(&empty[s]);
        }
        __syncwarp();
      }
    }
  } else {
    const int wg = warp >> 2;
    const uint32_t mine = tmem + wg * T::kColumns + (static_cast<uint32_t>((warp & 3) * 32) << 16);   // this warp's lanes
    float acc[N];
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = 0.f;
    float scale[P] = {};
    uint32_t rounds = 0;            // of this warpgroup so far
    int row_tile = first_tile, block = first_block;
    // adds the sums of the groups of the last round to this thread's row
    auto collect = [&](int first, int i) {   // i: the unit, counted from the run's beginning
      const bool ok = __all_sync(0xffffffffu, T::kRounds == 1 ? wait(&done[wg][i & 1], (i >> 1) & 1) : wait(&done[wg][0], rounds++ & 1));
      tc_fence_after();
      if (ok) {
#pragma unroll
        for (int p = 0; p < T::kRound; ++p) {
          const uint32_t from = mine + T::kSums + (T::kD == 2 ? (i & 1) * (P * N) : 0) + p * N;
          const bool far = w4_far(scale[first + p]);
          const float by = scale[first + p] * (far ? 1.f : kW4SumsBy);
          if (kW4SumsBy != 1.f && __any_sync(0xffffffffu, far)) {   // few sums at a time: registers are short, and hardly any weights are that large
            const float other = far ? kW4SumsBy : 1.f;
#pragma unroll
            for (int j = 0; j < N; j += 16) {
              uint32_t d[16];
              tmem_ld16(from + j, d);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 16; ++e) acc[j + e] = fmaf(by, __uint_as_float(d[e]) * other, acc[j + e]);
            }
            continue;
          }
          uint32_t d[N / 16][16];
#pragma unroll
          for (int j = 0; j < N / 16; ++j) tmem_ld16(from + 16 * j, d[j]);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < N; j += 2) {
            const float x = __uint_as_float(d[j / 16][j % 16]), y = __uint_as_float(d[j / 16][j % 16 + 1]);
            if (N == 32) {   // two at a time: 54 instead of 56 us for 24 x 32000 x 8192 in groups of 32; with 64 tokens' registers 84 instead of 80
              const float2 v = f32x2_unpack(fma_f32x2(f32x2(by, by), f32x2(x, y), f32x2(acc[j], acc[j + 1])));
              acc[j] = v.x;
              acc[j + 1] = v.y;
            } else {
              acc[j] = fmaf(by, x, acc[j]);
              acc[j + 1] = fmaf(by, y, acc[j + 1]);
            }
          }
        }
      }
      tc_fence_before();
    };
    // What this CTA has of a row tile, to a place of its own: nobody else's piece is read or waited for here.
    auto flush = [&] {
      const bool lost = dead;
      float* part = args.parts + (row_tile + cta) * (N * T::kTile) + wg * 128 + (warp & 3) * 32 + lane;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if (j < a.rows) part[j * T::kTile] = lost ? __int_as_float(0x7fffffff) : acc[j];
        acc[j] = 0.f;
      }
    };
    for (int i = 0; i < count; ++i) {
      const int s = i % T::kStages;
      const uint8_t* stage = ring + s * T::kStage;
      wait(&full[s], (i / T::kStages) & 1);
      uint4 codes[2][2];
      float next_scale[P];
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h) codes[c][h] = reinterpret_cast<const uint4*>(stage)[(2 * warp + c) * 64 + h * 32 + lane];
#pragma unroll
      for (int p = 0; p < P; ++p)   // of this thread's row: tile lane / 16, row lane % 16
        next_scale[p] = h_to_f(reinterpret_cast<const half_t*>(stage + T::kCodes + T::kTokens)[(((2 * warp + (lane >> 4)) * 8 + (lane & 7)) * P + p) * 2 + ((lane >> 3) & 1)]);
      uint32_t zero[2];             // the bytes of P groups of row g of both tiles
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint8_t* z = stage + T::kBytes + ((2 * warp + c) * 8 + (lane >> 2)) * P;
        zero[c] = P == 4 ? *reinterpret_cast<const uint32_t*>(z) : P == 2 ? *reinterpret_cast<const uint16_t*>(z) : *z;
      }
      uint32_t r[2][32];
      auto unpack = [&](int c) {
#pragma unroll
        for (int w = 0; w < 8; ++w) {   // step w: columns 16 w .. of the block as they lie
          const uint4& from = codes[c][w / 4];
          uint32_t v[4];
          w4_unpack<true>(w % 4 == 0 ? from.x : w % 4 == 1 ? from.y : w % 4 == 2 ? from.z : from.w, w4_zero<true>(zero[c] >> (8 * (w * P / 8)) & 255u), v);
          r[c][4 * w] = v[0];
          r[c][4 * w + 1] = v[2];
          r[c][4 * w + 2] = v[1];
          r[c][4 * w + 3] = v[3];
        }
      };
      auto collect_last = [&] {
        if (i == 0) return;
        collect(P - T::kRound, i - 1);
        if (block == 0) {
          flush();
          ++row_tile;
        }
      };
      // Into the weights that the products of the last block do not read, while they are under way; or, where there is room for
      // one block only, behind them.  With room for the sums of two blocks those of the last one are read when the products of this
      // one are on their way.
      const uint32_t to = mine + (T::kA == 2 ? (i & 1) * 64 : 0);
      unpack(0);
      if (T::kA == 1) collect_last();
      tmem_st_16x64(to, r[0]);
      unpack(1);
      tmem_st_16x64(to + (16u << 16), r[1]);
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty[s]);
      if (T::kA == 2 && T::kD == 1) collect_last();
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&a_full[wg][i & 1]);
      if (T::kD == 2) collect_last();
#pragma unroll
      for (int p = 0; p < P; ++p) scale[p] = next_scale[p];
#pragma unroll
      for (int round = 0; round < T::kRounds - 1; ++round) {
        collect(round * T::kRound, i);
        __syncwarp();
        if (lane == 0) mbar_arrive(&d_free[wg]);
      }
      if (++block == blocks) block = 0;
    }
    if (count > 0) {
      collect(P - T::kRound, count - 1);
      flush();
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, 512);
}

// Adds up the partial sums: 128 weight rows and N / 2 tokens a CTA, a fourth of those a thread: one wave of CTAs for 28672 rows (16
// tokens a CTA also where N is 64: two waves, 0.4 us more).
template <int N, int W>
__global__ void __launch_bounds__(512) w4_linear_join_kernel(const __grid_constant__ W4TcArgs args, int ctas) {
  pdl_launch_dependents();
  constexpr int kTile = W * 128, kEach = N / 8;
  const W4LinearArgs& a = args.a;
  const int row_tile = blockIdx.x / W, row = blockIdx.x % W * 128 + threadIdx.x % 128, token = (blockIdx.y * 4 + threadIdx.x / 128) * kEach;
  const long long blocks = a.v.blocks, units = args.row_tiles * blocks, first = row_tile * blocks, segment = static_cast<long long>(N) * kTile;
  const int c0 = w4_run_of(first, units, ctas), c1 = w4_run_of(first + blocks - 1, units, ctas);
  const float* from = args.parts + (row_tile + c0) * segment + token * kTile + row;   // the CTAs' pieces follow each other
  const int here = min(kEach, a.rows - token);
  pdl_wait();
  float v[kEach];
#pragma unroll
  for (int j = 0; j < kEach; ++j) v[j] = j < here ? from[j * kTile] : 0.f;
#pragma unroll 2
  for (int c = 1; c <= c1 - c0; ++c) {
    from += segment;
#pragma unroll
    for (int j = 0; j < kEach; ++j) v[j] += j < here ? from[j * kTile] : 0.f;
  }
#pragma unroll
  for (int j = 0; j < kEach; ++j) w4_store(a, token + j, static_cast<long long>(row_tile) * kTile + row, v[j]);
}

}  // namespace thinfer
