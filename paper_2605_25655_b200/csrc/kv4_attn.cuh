// Attention of the newest `queries` tokens of every request over its 4-bit paged cache:
//
//   S[i, t] = q_i . k_t / sqrt(D),  t < len - (queries - 1 - i)        (the query tokens are the last of the len keys)
//   out_i   = sum_t softmax_t(S[i, t]) v_t,   k_t, v_t = offset + scale * code;   0 where a query sees no key
//
// Scale and offset of a row belong to all its D values, so neither has to touch the codes:
//
//   S[i, t]  = scale_t (q_i . code_t) + offset_t (sum of q_i)
//   out_i    = ( sum_t w_t (code_t - 8) + sum_t p_t (offset_t + 8 scale_t) ) / sum_t p_t,   w_t = p_t scale_t
//
// and the matrix instructions multiply by the codes themselves.  A code in the low mantissa bits of an FP16 number is
// the subnormal code * 2^-24 (bits 0-3) or code * 2^-20 (bits 4-7), which the tensor cores take at face value: one AND
// turns two codes into two operands, one shift per eight codes reaches the other byte of a half, and the powers of two
// are put back in FP32.  All products q * code and weight * code are then exact in FP32.  Both builds use FP16
// operands: a query row is scaled by the power of two that brings its largest value to [2^12, 2^13), which loses
// nothing within 2^-22 of that value.
//
// Cache rows are the A operand (16 tokens, or 16 dimensions, per instruction) and up to 8 query columns - the query
// heads of one KV head times the query tokens - are the B operand, so that each instruction consumes 256 codes:
//
//   S^T[token, column] = K[token, :] Q^T        A = K codes, B = Q (registers, once per segment)
//   O^T[dim, column]  += V^T[dim, token] P^T    A = V codes (the layout keeps token pairs together), B = weights
//
// The weights w go to FP16 relative to a running reference per column; sums of p and of p times the middle of the row
// stay in FP32.  The 8 is taken off the codes by one more instruction per 16 tokens (a matrix of ones gives the sum of
// the rounded weights) and a packed FP32 multiply-add per pair of accumulators and 32 tokens: a rounding of w then
// counts with the distance from the middle of the row, not with the whole code, and the accumulators stay as small as
// the result, so that the truncation of the matrix unit's additions does not add up (over 16384 keys the FP16 error
// against 64 bits was 3.2e-4 with the 8 taken off at the end and 2.9e-4 now; 2.1e-4 is the rounding of the result).  The
// running maximum and that reference move only when a weight would exceed 2^8 (one vote per 16 tokens): the shuffles and
// the rescaling of the output are then off the usual path.
//
// Bound: HBM, D + 8 bytes per key and KV head; at 6.4 TB/s an SM has to consume 48 codes a cycle, which leaves 2.7
// issue slots per code and half as many for the ANDs and shifts (half rate).  Work: all (request, KV head, column tile)
// pairs are cut into units of 32 tokens, laid end to end and dealt out in equal runs, first to the CTAs (one per SM),
// then to the warps of a CTA; the lengths are only known on the device, so each CTA sums them up itself.  Each warp
// streams its units through a private ring in shared memory with 16-byte asynchronous copies, and needs no other warp
// until its range is done.  (Bulk copies took fewer instructions to write but more to issue: four of them per 32 tokens
// cost 150 issue cycles where nine 16-byte copies by all lanes cost 30: 209 against 185 us for 64 requests of up to 16384
// keys, 8 KV heads.)  What a warp cannot finish is merged in shared memory; what a CTA cannot finish goes to the workspace
// and a second kernel, chained to this one, merges it in CTA order: the result does not depend on timing, and the
// workspace needs no initial state.
//
// Measured: those 64 requests, 845 MB, in 189 us a call when calls follow one another (4.5 TB/s, 70 % of a copy: the kernel meets the
// 1000 W limit), and in 161 us (BF16 173) in short replayed runs, before it does.  About 510 instructions per 32 tokens and warp, 54 % of the cycles of the half-rate integer
// pipe, the rest latency that three warps per scheduler do not cover; without any arithmetic the copies alone take 129 us.
// 16 requests of up to 1279 keys, 40 KV heads: 26 us, of which 3 pass before the first key arrives and 5 behind the last.
#pragma once
#include "kv4_layout.cuh"

namespace thinfer {

constexpr int kKv4Unit = 32;         // tokens of one ring stage
constexpr int kKv4Stages = 2;        // more made no difference: 12 warps keep 50 to 100 KB of an SM in flight
// Warps of a CTA, one CTA per SM: what the registers allow (168 and 255 a thread).
template <int NT>
__host__ __device__ constexpr int kv4_warps() {
  return NT == 1 ? 12 : 8;
}
constexpr float kKv4Low = -3.402823466e38f;   // running maximum before the first key: no finite score lies below it
// Scores are put together without a factor of 2^12 in the BF16 build and multiplied by it last: with the 2^24 of the codes in
// one factor, a query of 2^116 and more made that factor infinite however small the keys were.  FP16 has no such numbers.
constexpr float kKv4Last = kStorageType == 1 ? 0x1p12f : 1.f;

// What a CTA leaves for the second kernel about the pair that begins in it and ends in a later one.
struct Kv4Split {
  int b, hk, col0, last;   // last: the CTA it ends in, -1: there is no such pair
};

struct Kv4AttnArgs {
  Kv4Cache c;
  const int32_t* lens;   // [batch]
  const half_t* q;       // [batch * queries] tokens, q_stride elements apart
  half_t* out;           // [batch * queries][n_q][D]
  long long q_stride;
  int batch, queries, n_q, group;
  int cols;              // group * queries: query columns of one KV head
  int col_tiles;
  Kv4Split* splits;      // [grid]
  float* parts;          // [grid][2] unfinished pieces of CTAs: [columns][D] outputs, then [columns][2] maximum and sum;
                         // piece 0 began in an earlier CTA, piece 1 begins here
  float scale_log2;      // log2(e) / sqrt(D)
  float inv_group;       // 1 / group
};

template <int D>
__host__ __device__ constexpr int kv4_stage_bytes() {
  return kKv4Unit * (D + 8);
}
template <int D, int NT>
__host__ __device__ constexpr int kv4_partial_floats() {  // one unfinished piece: outputs, then maximum and sum
  return NT * 8 * (D + 2);
}
// Memory of one warp: its ring, which takes the piece that ends its range once it has drained; the query columns of the
// pairs that begin in each ring stage; room for the piece that begins its range.
template <int D, int NT>
__host__ __device__ constexpr int kv4_query_bytes() {
  return NT * 8 * D * 2;
}
template <int D, int NT>
__host__ __device__ constexpr int kv4_ring_bytes() {
  return kKv4Stages * kv4_stage_bytes<D>();
}
template <int D, int NT>
__host__ __device__ constexpr int kv4_warp_bytes() {
  return kv4_ring_bytes<D, NT>() + kKv4Stages * kv4_query_bytes<D, NT>() + kv4_partial_floats<D, NT>() * 4;
}

// ------------------------------------------------------------------ schedule
// Units of request b times (KV heads x column tiles), summed over the requests: pref[b] is the first unit of b.
// A length beyond what the table can name gives NaN whatever it is: it counts as one unit more than the table holds,
// behind the last key of every query.
__device__ __forceinline__ int kv4_len(const Kv4AttnArgs& a, int b) {
  const long long cap = min((static_cast<long long>(a.c.max_pages) << a.c.page_shift) + kKv4Unit + a.queries, 0x7fffffc0ll);
  const int n = a.lens[b];
  return n < 0 ? 0 : static_cast<int>(min(static_cast<long long>(n), cap));
}
// a / b of numbers that are not negative; nearly always both fit 32 bits, where a division costs a fifth
__device__ __forceinline__ long long div_pos(long long a, long long b) {
  return ((a | b) >> 32) == 0 ? static_cast<long long>(static_cast<uint32_t>(a) / static_cast<uint32_t>(b)) : a / b;
}
__device__ __forceinline__ int kv4_units(int len) { return (len + kKv4Unit - 1) / kKv4Unit; }

// Shared memory of the schedule: pref[0 .. batch] first units of the requests, then their lengths.
__host__ __device__ constexpr size_t kv4_plan_bytes(int batch) { return (static_cast<size_t>(batch) + 1) * 8 + static_cast<size_t>(batch) * 4; }
struct Kv4Plan {
  const long long* pref;
  const int* len;
};

__device__ __forceinline__ Kv4Plan kv4_plan(const Kv4AttnArgs& a, uint8_t* mem, long long* warp_sums) {
  long long* pref = reinterpret_cast<long long*>(mem);
  int* lens = reinterpret_cast<int*>(pref + a.batch + 1);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int per_unit = a.c.n_kv * a.col_tiles;
  long long carry = 0;
  for (int b0 = 0; b0 < a.batch; b0 += blockDim.x) {
    const int b = b0 + threadIdx.x;
    const int len = b < a.batch ? kv4_len(a, b) : 0;
    const long long v = static_cast<long long>(kv4_units(len)) * per_unit;
    long long s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += u;
    }
    if (lane == 31) warp_sums[warp] = s;
    __syncthreads();
    long long before = carry, all = 0;
    for (int w = 0; w < warps && b0 + w * 32 < a.batch; ++w) {
      if (w < warp) before += warp_sums[w];
      all += warp_sums[w];
    }
    if (b < a.batch) {
      pref[b] = before + s - v;
      lens[b] = len;
    }
    carry += all;
    if (b0 + static_cast<int>(blockDim.x) < a.batch) __syncthreads();
  }
  if (threadIdx.x == 0) pref[a.batch] = carry;
  __syncthreads();
  return Kv4Plan{pref, lens};
}

// A pair and a unit in it.
struct Kv4Place {
  int b, hk, ct, unit, units, len;
  long long pair_first;  // first unit of the pair
};
// Where unit u lies.  Requests without keys have no units.
__device__ __forceinline__ Kv4Place kv4_place(const Kv4AttnArgs& a, const Kv4Plan& plan, long long u) {
  int lo = 0, hi = a.batch - 1;
  while (lo < hi) {      // the last request that begins at or before u
    const int mid = (lo + hi + 1) >> 1;
    if (plan.pref[mid] <= u) lo = mid;
    else hi = mid - 1;
  }
  Kv4Place p;
  p.b = lo;
  p.len = plan.len[lo];
  p.units = kv4_units(p.len);
  const long long in_b = u - plan.pref[lo];
  const int pair = static_cast<int>(div_pos(in_b, p.units));
  p.unit = static_cast<int>(in_b - static_cast<long long>(pair) * p.units);
  p.pair_first = u - p.unit;
  p.hk = a.col_tiles == 1 ? pair : pair / a.col_tiles;
  p.ct = pair - p.hk * a.col_tiles;
  return p;
}
// The pair behind p's; there has to be one.
__device__ __forceinline__ void kv4_next_pair(const Kv4AttnArgs& a, const Kv4Plan& plan, Kv4Place& p) {
  p.pair_first += p.units;
  p.unit = 0;
  if (++p.ct == a.col_tiles) {
    p.ct = 0;
    if (++p.hk == a.c.n_kv) {
      p.hk = 0;
      do {
        p.len = plan.len[++p.b];
      } while (p.len == 0);
      p.units = kv4_units(p.len);
    }
  }
}
// col / group of a query column (below 2^18, where a rounded product is exact enough)
__device__ __forceinline__ int kv4_query_of(const Kv4AttnArgs& a, int col) {
  return a.queries == 1 ? 0 : static_cast<int>((static_cast<float>(col) + 0.5f) * a.inv_group);
}
// CTAs that take part: with few units some stay idle rather than split pairs further.
__device__ __forceinline__ long long kv4_ctas(long long total, int grid, int warps) {
  return total < static_cast<long long>(grid) * warps ? (static_cast<int>(total) + warps - 1) / warps : grid;
}
__device__ __forceinline__ long long kv4_cta_first(long long total, long long ctas, long long i) { return div_pos(i * total, ctas); }
__device__ __forceinline__ long long kv4_cta_of(long long total, long long ctas, long long u) { return div_pos((u + 1) * ctas - 1, total); }

// ------------------------------------------------------------------ instructions
__device__ __forceinline__ void mma_f16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
  return d;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void async_copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
template <int W>
__device__ __forceinline__ void lds_words(uint32_t (&r)[W], const uint8_t* p) {
  if constexpr (W == 4) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    r[0] = v.x;
    r[1] = v.y;
    r[2] = v.z;
    r[3] = v.w;
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    r[0] = v.x;
    r[1] = v.y;
  }
}
__device__ __forceinline__ float2 lds_params(const uint8_t* p) { return kv4_unpack_params(*reinterpret_cast<const uint32_t*>(p)); }

// Where lane (r, c) = (lane / 4, lane % 4) finds things in a block of 16 tokens.  Row r of the score tile is token
// 4 (r / 2) + r % 2 and row r + 8 the token two further: after the 8 x 8 transposes lane c then holds the weights of
// tokens 4c .. 4c + 3, two neighbouring pairs of the V layout.
__device__ __forceinline__ int kv4_row_token(int r) { return 4 * (r >> 1) + (r & 1); }

// A ring stage: K codes and V codes of 32 tokens as in a page, then the params.  Within each 128 bytes of codes the
// 16-byte pieces are permuted so that the lanes that read together (four token pairs of V, or tokens 0, 1, 4, 5 of K
// where two rows share 64 bytes) meet different banks: piece p of line n is at p ^ kv4_key(n).
template <int D, bool V>
__host__ __device__ constexpr int kv4_key(int line) {
  return V ? 2 * ((D == 128 ? line >> 1 : line) & 3) : (D == 128 ? 0 : 4 * (line & 1));
}
// Byte offset of byte `at` of a code part.
template <int D, bool V>
__device__ __forceinline__ int kv4_at(int at) {
  return at ^ (kv4_key<D, V>(at >> 7) << 4);
}

// State of one warp's current pair: columns 2c and 2c + 1 of every column tile.
template <int D, int NT>
struct Kv4Acc {
  float o[NT][D / 16][4];
  float m[NT][2], l[NT][2], z[NT][2], ref[NT][2];  // maximum, sum of p, sum of p times row middle, reference of w
  float qf[NT][2], qs[NT][2];                      // scale of the code product, scaled sum of the query; over kKv4Last
  int lim[NT][2];                                  // keys a column sees
  uint32_t q[NT][D / 16][2];                       // B operand

  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        m[n][j] = kKv4Low;
        l[n][j] = z[n][j] = 0.f;
        ref[n][j] = __int_as_float(245 << 23);  // 2^118: the first weight sets it
      }
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][i][e] = 0.f;
    }
  }
};

__device__ __forceinline__ float exact_inverse(float pow2) { return __int_as_float((254 << 23) - __float_as_int(pow2)); }

// Requests the query columns of a pair: 16-byte pieces, piece k of column i at k ^ (i & 7).  Columns behind the last one
// are not written.
template <int D, int NT>
__device__ __forceinline__ void kv4_request_queries(const Kv4AttnArgs& a, uint32_t dst, int b, int hk, int col0) {
  constexpr int PER = D / 8;           // pieces of a column
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int n = 0; n < NT * 8 * PER / 32; ++n) {
    const int i = (n * 32 + lane) / PER, k = lane % PER, col = col0 + i;
    if (col < a.cols) {
      const int qi = kv4_query_of(a, col), h = hk * a.group + (col - qi * a.group);
      const half_t* src = a.q + (static_cast<long long>(b) * a.queries + qi) * a.q_stride + static_cast<long long>(h) * D + k * 8;
      async_copy16(dst + i * (2 * D) + ((k ^ (i & 7)) << 4), src);
    }
  }
}

// The query columns of a pair as B operand: lane (r, c) converts the D / 4 values of column r that start at c D / 4.
template <int D, int NT>
__device__ __forceinline__ void kv4_load_queries(const Kv4AttnArgs& a, Kv4Acc<D, NT>& s, const uint8_t* from, int len, int col0) {
  constexpr int W = D / 32;
  const int lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const bool there = col0 + 8 * n + r < a.cols;
    float x[8 * W];
#pragma unroll
    for (int w = 0; w < W; ++w) {
      float f[8];
      unpack8(*reinterpret_cast<const uint4*>(from + (8 * n + r) * (2 * D) + (((c * W + w) ^ r) << 4)), f);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[8 * w + e] = there ? f[e] : 0.f;
    }
    float top = 0.f, sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8 * W; ++e) {
      top = fmaxf(top, fabsf(x[e]));
      sum = fmaf(x[e], 1.f / kKv4Last, sum);   // the sum of large values of one sign may pass FP32
    }
#pragma unroll
    for (int off = 1; off < 4; off <<= 1) {
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
      sum += __shfl_xor_sync(0xffffffffu, sum, off);
    }
    const int ex = min(max(__float_as_int(top) >> 23, 13), 253);
    const float up = __int_as_float((266 - ex) << 23), down = __int_as_float((ex - 12) << 23);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float* y = x + 8 * w;
      s.q[n][2 * w][0] = pack_f16(y[0] * up, y[4] * up);
      s.q[n][2 * w][1] = pack_f16(y[1] * up * 0.0625f, y[5] * up * 0.0625f);   // codes in bits 4-7 weigh 16 times more
      s.q[n][2 * w + 1][0] = pack_f16(y[2] * up, y[6] * up);
      s.q[n][2 * w + 1][1] = pack_f16(y[3] * up * 0.0625f, y[7] * up * 0.0625f);
    }
    const float qf = (16777216.f / kKv4Last) * down * a.scale_log2, qs = sum * a.scale_log2;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      s.qf[n][j] = __shfl_sync(0xffffffffu, qf, 8 * c + 4 * j);
      s.qs[n][j] = __shfl_sync(0xffffffffu, qs, 8 * c + 4 * j);
      const int cj = col0 + 8 * n + 2 * c + j;
      s.lim[n][j] = cj < a.cols ? len - (a.queries - 1 - kv4_query_of(a, cj)) : 0;
    }
  }
}

// 32 tokens of a ring stage, 16 at a time.  MASKED: some of them are behind the end for some column, or on no page (bit
// b of `bad`: the tokens 16 b .. 16 b + 15).
template <int D, int NT, bool MASKED>
__device__ __forceinline__ void kv4_stage(Kv4Acc<D, NT>& s, const uint8_t* stage, int t0, uint32_t bad) {
  constexpr int W = D / 32, MT = D / 16;
  constexpr uint32_t LO = 0x000f000fu, HI = 0x00f000f0u, ONE = 0x3c003c00u;
  constexpr int KP = kKv4Unit * D, VP = KP + kKv4Unit * 4;
  const int lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3;
  const int tr = kv4_row_token(r);
  float ones[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) ones[n][e] = 0.f;
  // ---- scores of all 32 tokens: their latency lies beside the weights of the first 16
  float scores[2][NT][4];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    float (&sc)[NT][4] = scores[b];
    float sd[NT][4];   // a second chain of instructions
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) sc[n][e] = sd[n][e] = 0.f;
    {
      uint32_t ka[W], kb[W];
      lds_words<W>(ka, stage + 16 * b * (D / 2) + kv4_at<D, false>(tr * (D / 2) + c * (D / 8)));
      lds_words<W>(kb, stage + 16 * b * (D / 2) + kv4_at<D, false>((tr + 2) * (D / 2) + c * (D / 8)));
#pragma unroll
      for (int w = 0; w < W; ++w)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const uint32_t x = hf ? ka[w] >> 8 : ka[w], y = hf ? kb[w] >> 8 : kb[w];
#pragma unroll
          for (int n = 0; n < NT; ++n)
            mma_f16_16816(hf ? sd[n] : sc[n], x & LO, y & LO, x & HI, y & HI, s.q[n][2 * w + hf][0], s.q[n][2 * w + hf][1]);
        }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[n][e] += sd[n][e];
    }
  }
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const float (&sc)[NT][4] = scores[b];
    // ---- weights
    float2 kp[2], vp[2];   // [row r | row r + 8] scale, offset; for V scale, middle of the row
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int t = 16 * b + tr + 2 * e;
      kp[e] = lds_params(stage + KP + t * 4);
      vp[e] = lds_params(stage + VP + t * 4);
      vp[e].y = fmaf(8.f, vp[e].x, vp[e].y);
    }
    auto seen = [&](int e, int n, int j) { return !MASKED || t0 + 16 * b + tr + 2 * e < s.lim[n][j]; };
    auto raw = [&](int e, int n, int j, float minus) {   // score - minus, log2 units
      float x = kStorageType == 1 ? fmaf(fmaf(kp[e].x * s.qf[n][j], sc[n][2 * e + j], kp[e].y * s.qs[n][j]), kKv4Last, -minus)
                                  : fmaf(kp[e].x, sc[n][2 * e + j] * s.qf[n][j], fmaf(kp[e].y, s.qs[n][j], -minus));
      if (MASKED) {
        if ((bad >> b) & 1u) x = __int_as_float(0x7fffffff);
        if (!seen(e, n, j)) x = -INFINITY;
      }
      return x;
    };
    // value params of a masked token may be anything: they must not meet a weight of zero
    auto vscale = [&](int e, int n, int j) { return !MASKED || seen(e, n, j) ? vp[e].x : 0.f; };
    auto vmid = [&](int e, int n, int j) { return !MASKED || seen(e, n, j) ? vp[e].y : 0.f; };
    float p[NT][4], w[NT][4];
    float top = 0.f;
    auto weights = [&]() {
      top = 0.f;
      if constexpr (!MASKED) {   // both columns at once in packed FP32: 4 of 168 us
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint64_t qf = f32x2(s.qf[n][0], s.qf[n][1]), qs = f32x2(s.qs[n][0], s.qs[n][1]);
          const uint64_t less = f32x2(-s.m[n][0], -s.m[n][1]), ref = f32x2(s.ref[n][0], s.ref[n][1]);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint64_t kx = f32x2(kp[e].x, kp[e].x), ky = f32x2(kp[e].y, kp[e].y), vx = f32x2(vp[e].x, vp[e].x);
            const uint64_t codes = f32x2(sc[n][2 * e], sc[n][2 * e + 1]);
            const float2 x = f32x2_unpack(kStorageType == 1 ? fma_f32x2(fma_f32x2(mul_f32x2(kx, qf), codes, mul_f32x2(ky, qs)), f32x2(kKv4Last, kKv4Last), less)
                                                            : fma_f32x2(kx, mul_f32x2(codes, qf), fma_f32x2(ky, qs, less)));
            const float x0 = ex2_approx(x.x), x1 = ex2_approx(x.y);
            const float2 y = f32x2_unpack(mul_f32x2(mul_f32x2(f32x2(x0, x1), ref), vx));
            p[n][2 * e] = x0;
            p[n][2 * e + 1] = x1;
            w[n][2 * e] = y.x;
            w[n][2 * e + 1] = y.y;
            top = fmax3(top, x0, y.x);
            top = fmax3(top, x1, y.y);
          }
        }
      } else {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float x = ex2_approx(raw(e, n, j, s.m[n][j]));
              const float y = x * s.ref[n][j] * vscale(e, n, j);
              p[n][2 * e + j] = x;
              w[n][2 * e + j] = y;
              top = fmax3(top, x, y);
            }
      }
    };
    weights();
    if (__any_sync(0xffffffffu, top > 256.f)) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float mx = fmax3(s.m[n][j], raw(0, n, j, 0.f), raw(1, n, j, 0.f));
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
          const float al = ex2_approx(s.m[n][j] - mx);
          float big = exact_inverse(s.ref[n][j]) * al;
#pragma unroll
          for (int e = 0; e < 2; ++e) big = fmaxf(big, ex2_approx(raw(e, n, j, mx)) * vscale(e, n, j));
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, off));
          // at most 2^118: scales down to BF16's smallest leave weights inside FP16, and p * ref (p <= 2^8) inside FP32
          const int ex = min(max(__float_as_int(big) >> 23, 9), 252);
          const float ref = __int_as_float((254 - ex) << 23);
          const float move = (al * ref) * exact_inverse(s.ref[n][j]);
          s.m[n][j] = mx;
          s.ref[n][j] = ref;
          s.l[n][j] *= al;
          s.z[n][j] *= al;
          ones[n][j] *= move;
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            s.o[n][i][j] *= move;
            s.o[n][i][2 + j] *= move;
          }
        }
      weights();
    }
    uint32_t pb[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          s.l[n][j] += p[n][2 * e + j];
          s.z[n][j] = fmaf(p[n][2 * e + j], vmid(e, n, j), s.z[n][j]);
        }
        pb[n][e] = transpose_8x8(pack_f16(w[n][2 * e], w[n][2 * e + 1]));
      }
      mma_f16_16816(ones[n], ONE, ONE, ONE, ONE, pb[n][0], pb[n][1]);
    }
    // ---- output
    uint32_t va[W], vb[W];
    const uint8_t* v = stage + kKv4Unit * (D / 2) + 8 * b * D;   // 8 pairs: a multiple of the lines the keys repeat after
    lds_words<W>(va, v + kv4_at<D, true>(2 * c * D + r * (D / 8)));
    lds_words<W>(vb, v + kv4_at<D, true>((2 * c + 1) * D + r * (D / 8)));
#pragma unroll
    for (int i = 0; i < W; ++i)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const uint32_t x = hf ? va[i] >> 8 : va[i], y = hf ? vb[i] >> 8 : vb[i];
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_f16_16816(s.o[n][2 * i + hf], x & LO, x & HI, y & LO, y & HI, pb[n][0], pb[n][1]);
      }
  }
  // ---- 8 off every code
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const uint64_t sum = f32x2(ones[n][0], ones[n][1]);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const float2 x = f32x2_unpack(fma_f32x2(sum, f32x2(-0x1p-21f, -0x1p-21f), f32x2(s.o[n][i][0], s.o[n][i][1])));
      const float2 y = f32x2_unpack(fma_f32x2(sum, f32x2(-0x1p-17f, -0x1p-17f), f32x2(s.o[n][i][2], s.o[n][i][3])));
      s.o[n][i][0] = x.x;
      s.o[n][i][1] = x.y;
      s.o[n][i][2] = y.x;
      s.o[n][i][3] = y.y;
    }
  }
}

// Values of column (n, j), dimensions r D / 8 + 4 i + {0, 1, 2, 3}, i < D / 32.
template <int D, int NT>
__device__ __forceinline__ float4 kv4_value4(const Kv4Acc<D, NT>& s, int n, int j, int i, float z, float back) {
  constexpr float F0 = 16777216.f, F1 = 1048576.f;  // 2^24 and 2^20: the place of the code in its operand
  const float(&x)[4] = s.o[n][2 * i], (&y)[4] = s.o[n][2 * i + 1];
  return make_float4(fmaf(x[j] * F0, back, z), fmaf(x[2 + j] * F1, back, z), fmaf(y[j] * F0, back, z), fmaf(y[2 + j] * F1, back, z));
}
__device__ __forceinline__ void kv4_store4(half_t* dst, float4 v) {
  *reinterpret_cast<uint2*>(dst) = make_uint2(pack2(v.x, v.y), pack2(v.z, v.w));
}
// Where 16 bytes of a column of an unfinished piece lie in shared memory: permuted so that the 8 lanes (two rows r, four
// column pairs) that store together meet different banks.
template <int D>
__device__ __forceinline__ int kv4_piece_at(int col, int p) {  // p: 16-byte part of the column's D floats
  const int c = (col >> 1) & 3;
  return col * D + ((p ^ (D == 128 ? c : (c & 1) | (c & 2) << 1)) << 2);
}
// First output element of a column.
template <int D>
__device__ __forceinline__ half_t* kv4_out(const Kv4AttnArgs& a, int b, int hk, int col) {
  const int i = kv4_query_of(a, col), h = hk * a.group + (col - i * a.group);
  return a.out + ((static_cast<size_t>(b) * a.queries + i) * a.n_q + h) * D;
}

struct Kv4Piece {
  long long pair;          // first unit of the pair, -1: no piece
  int units, b, hk, col0;
};

template <int D, int NT>
__global__ void __launch_bounds__(kv4_warps<NT>() * 32, 1) kv4_attn_kernel(const Kv4AttnArgs a) {
  constexpr int W = D / 32, NC = NT * 8, NS = kKv4Stages, STAGE = kv4_stage_bytes<D>(), CW = kv4_warps<NT>();
  constexpr int PART = kv4_partial_floats<D, NT>(), WARP_BYTES = kv4_warp_bytes<D, NT>();
  extern __shared__ __align__(128) uint8_t kv4_mem[];
  __shared__ long long warp_sums[CW];
  __shared__ Kv4Piece pieces[2 * CW];       // unfinished pieces, 2 w: head, 2 w + 1: tail of warp w
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x < 2 * CW) pieces[threadIdx.x].pair = -1;
  pdl_wait();
  if (threadIdx.x == 0) a.splits[blockIdx.x].last = -1;
  const Kv4Plan plan = kv4_plan(a, kv4_mem + CW * WARP_BYTES, warp_sums);
  // requests without keys: zeros, dealt out over the CTAs
  for (int b = blockIdx.x; b < a.batch; b += gridDim.x)
    if (plan.len[b] == 0) {
      uint4* dst = reinterpret_cast<uint4*>(a.out + static_cast<size_t>(b) * a.queries * a.n_q * D);
      const int n = a.queries * a.n_q * (D / 8);
      for (int i = threadIdx.x; i < n; i += CW * 32) dst[i] = make_uint4(0, 0, 0, 0);
    }
  const long long total = plan.pref[a.batch], ctas = kv4_ctas(total, gridDim.x, CW);
  if (blockIdx.x >= ctas) return;
  const long long c_beg = kv4_cta_first(total, ctas, blockIdx.x), c_units = kv4_cta_first(total, ctas, blockIdx.x + 1) - c_beg;
  const long long w_beg = c_beg + div_pos(warp * c_units, CW);
  const int w_units = static_cast<int>(c_beg + div_pos((warp + 1) * c_units, CW) - w_beg);
  uint8_t* const mine = kv4_mem + warp * WARP_BYTES;
  const uint32_t ring = smem_u32(mine);
  const int shift = a.c.page_shift, P = 1 << shift;

  // ---- requests: walk the warp's units ahead of the arithmetic, across segments
  int f_u = 0, f_end = 0;              // next unit to request and end of the segment it is in, from w_beg
  int f_t = 0, f_base = 0;             // its first token, table column of `ids`
  const uint8_t* f_blocks = nullptr;   // pool + head offset
  const int32_t* f_row = nullptr;
  Kv4Place pl{}, f_pl;                 // of the arithmetic and of the requests
  if (w_units > 0) pl = kv4_place(a, plan, w_beg);
  f_pl = pl;
  int ids = -1, ids_next = -1;         // page numbers of 32 table columns from f_base, and of the next 32
  int f_slot = 0;
  uint32_t bad_of = 0;                 // two bits for each ring stage: tokens 0 .. 15 or 16 .. 31 are on no page
  // this lane's place in a copy of 512 bytes of codes (line lane / 8), in an even and an odd one, and in the params
  const uint32_t k_to = kv4_at<D, false>(lane * 16);
  const uint32_t v_to[2] = {static_cast<uint32_t>(kv4_at<D, true>(lane * 16)), static_cast<uint32_t>(kv4_at<D, true>(512 + lane * 16) - 512)};
  const int par_from = P * D + (lane & 8 ? P * 4 : 0) + (lane & 3) * 16;
  auto load_ids = [&](int base) {
    const int col = base + lane;
    return col < a.c.max_pages && (static_cast<long long>(col) << shift) < f_pl.len ? f_row[col] : -1;
  };
  auto request = [&]() {               // one stage, if there is one left
    if (f_u < w_units) {
      if (f_u >= f_end) {              // enter the next segment
        if (f_u != 0) kv4_next_pair(a, plan, f_pl);
        f_end = f_u + min(w_units - f_u, f_pl.units - f_pl.unit);
        f_t = f_pl.unit * kKv4Unit;
        f_blocks = a.c.pool + static_cast<size_t>(f_pl.hk) * a.c.block_bytes;
        f_row = a.c.table + static_cast<size_t>(f_pl.b) * a.c.max_pages;
        f_base = (f_t >> shift) & ~31;
        ids = load_ids(f_base);
        ids_next = load_ids(f_base + 32);
        kv4_request_queries<D, NT>(a, ring + kv4_ring_bytes<D, NT>() + f_slot * kv4_query_bytes<D, NT>(), f_pl.b, f_pl.hk, f_pl.ct * NC);
      }
      ++f_u;
      const int t = f_t;
      f_t += kKv4Unit;
      int col = (t >> shift) - f_base;
      if (col >= 32) {
        f_base += 32;
        col -= 32;
        ids = ids_next;
        ids_next = load_ids(f_base + 32);
      }
      // the two halves of 16 tokens: on one page, or on two of 16 tokens; no request for what lies behind the end
      const int at0 = t & (P - 1), at1 = (t + 16) & (P - 1);
      const int page0 = __shfl_sync(0xffffffffu, ids, col), page1 = shift == 4 ? __shfl_sync(0xffffffffu, ids, (col + 1) & 31) : page0;
      const bool there1 = t + 16 < f_pl.len;
      const bool ok0 = static_cast<unsigned>(page0) < static_cast<unsigned>(a.c.n_pages);
      const bool ok1 = static_cast<unsigned>(page1) < static_cast<unsigned>(a.c.n_pages);
      const uint32_t bad = (ok0 ? 0u : 1u) | (ok1 || !there1 ? 0u : 2u);
      bad_of = (bad_of & ~(3u << (2 * f_slot))) | bad << (2 * f_slot);
      const uint32_t dst = ring + f_slot * STAGE;
      const uint8_t* from0 = f_blocks + static_cast<size_t>(page0) * a.c.page_bytes;
      const uint8_t* from1 = shift == 4 ? f_blocks + static_cast<size_t>(page1) * a.c.page_bytes : from0;
      constexpr int HALF = 8 * D;      // code bytes of 16 tokens
      if (ok0) {
        const uint8_t* k = from0 + at0 * (D / 2) + lane * 16;
        const uint8_t* v = k + P * (D / 2);
#pragma unroll
        for (int i = 0; i < HALF / 512; ++i) {
          async_copy16(dst + i * 512 + k_to, k + i * 512);
          async_copy16(dst + 2 * HALF + i * 512 + v_to[i & 1], v + i * 512);
        }
      }
      if (ok1 && there1) {
        const uint8_t* k = from1 + at1 * (D / 2) + lane * 16;
        const uint8_t* v = k + P * (D / 2);
#pragma unroll
        for (int i = 0; i < HALF / 512; ++i) {
          const int j = HALF / 512 + i;
          async_copy16(dst + HALF + i * 512 + k_to, k + i * 512);
          async_copy16(dst + 3 * HALF + i * 512 + v_to[j & 1], v + i * 512);
        }
      }
      // params: lanes 0-3, 4-7 K of the halves, 8-11, 12-15 V of the halves
      const bool second = (lane & 4) != 0;
      if (lane < 16 && (second ? ok1 && there1 : ok0))
        async_copy16(dst + 4 * HALF + lane * 16, (second ? from1 + at1 * 4 : from0 + at0 * 4) + par_from);
      f_slot = f_slot + 1 == NS ? 0 : f_slot + 1;
    }
  };
#pragma unroll
  for (int i = 0; i < NS - 1; ++i) {
    request();
    async_commit();
  }

  Kv4Acc<D, NT> s;
  int slot = 0;
  for (int u = 0; u < w_units;) {
    const int n_units = min(w_units - u, pl.units - pl.unit), col0 = pl.ct * NC;
    s.reset();
    const int t_end = min(pl.len, (pl.unit + n_units) * kKv4Unit), t_all = pl.len - (a.queries - 1) - kKv4Unit;
    const int t_beg = pl.unit * kKv4Unit;
    for (int t0 = t_beg; t0 < t_end; t0 += kKv4Unit) {
      async_wait<NS - 2>();              // this lane's copies of the stage have landed
      const uint32_t bad = (bad_of >> (2 * slot)) & 3u;
      __syncwarp();                      // everybody's have, and everybody has read the stage before it, which is filled next
      request();
      async_commit();
      const uint8_t* stage = mine + slot * STAGE;
      if (t0 == t_beg) kv4_load_queries<D, NT>(a, s, mine + kv4_ring_bytes<D, NT>() + slot * kv4_query_bytes<D, NT>(), pl.len, col0);
      if (bad == 0 && t0 <= t_all) kv4_stage<D, NT, false>(s, stage, t0, 0);
      else kv4_stage<D, NT, true>(s, stage, t0, bad);
      slot = slot + 1 == NS ? 0 : slot + 1;
    }
    // ---- the segment's result: sums over the lanes that hold other tokens of the same columns
    int here;
    asm volatile("mov.u32 %0, %%laneid;" : "=r"(here));   // opaque: addresses kept for this in the loop above cost it 5 of 162 us
    const int r = here >> 2, c = here & 3;
    const bool head = pl.unit > 0, whole = !head && n_units == pl.units;
    // the piece that ends the range takes the ring, which nobody fills any more
    float* part = reinterpret_cast<float*>(mine + (head ? WARP_BYTES - PART * 4 : 0));
    if (!whole && lane == 0) pieces[2 * warp + (head ? 0 : 1)] = Kv4Piece{pl.pair_first, pl.units, pl.b, pl.hk, col0};
    __syncwarp();
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float l = s.l[n][j], z = s.z[n][j];
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) {
          l += __shfl_xor_sync(0xffffffffu, l, off);
          z += __shfl_xor_sync(0xffffffffu, z, off);
        }
        const float back = exact_inverse(s.ref[n][j]);
        const int col = 8 * n + 2 * c + j;
        if (whole) {
          if (col0 + col < a.cols) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            half_t* dst = kv4_out<D>(a, pl.b, pl.hk, col0 + col) + r * (D / 8);
#pragma unroll
            for (int i = 0; i < W; ++i) {
              const float4 v = kv4_value4<D, NT>(s, n, j, i, z, back);
              kv4_store4(dst + 4 * i, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < W; ++i)
            *reinterpret_cast<float4*>(part + kv4_piece_at<D>(col, r * W + i)) = kv4_value4<D, NT>(s, n, j, i, z, back);
          if (r == 0) *reinterpret_cast<float2*>(part + NC * D + 2 * col) = make_float2(s.m[n][j], l);
        }
      }
    u += n_units;
    if (u < w_units) kv4_next_pair(a, plan, pl);
  }
  __syncthreads();

  // ---- unfinished pieces.  Lane i knows piece i; a task is GROUP columns of one pair, dealt over the warps.  A warp adds up
  // CHAINS columns beside each other (each of them two where 16 lanes cover one): a task is all latency.
  constexpr int CHAINS = 2, PASS = 128 / D, GROUP = CHAINS * PASS;
  static_assert(2 * CW <= 32, "a lane for every piece");
  static_assert(NC % GROUP == 0, "whole tasks");
  const int tasks = (min(NC, a.cols) + GROUP - 1) / GROUP;   // only the last tile of several has fewer columns
  const long long my_pair = lane < 2 * CW ? pieces[lane].pair : -1;
  const unsigned my_members = __match_any_sync(0xffffffffu, my_pair);
  const bool leads = my_pair >= 0 && __ffs(my_members) - 1 == lane;
  const unsigned leaders = __ballot_sync(0xffffffffu, leads);
  const int my_rank = __popc(leaders & ((1u << lane) - 1));
  const float* const my_part = reinterpret_cast<const float*>(kv4_mem + (lane >> 1) * WARP_BYTES + ((lane & 1) ? 0 : WARP_BYTES - PART * 4));
  for (int task = warp; task < __popc(leaders) * tasks; task += CW) {
    const int rank = task / tasks, col0 = (task - rank * tasks) * GROUP;
    const int k = __ffs(__ballot_sync(0xffffffffu, leads && my_rank == rank)) - 1;   // the pair's first piece
    const unsigned members = __shfl_sync(0xffffffffu, my_members, k);
    const Kv4Piece pc = pieces[k];
    const bool member = (members >> lane) & 1u;
    float top[GROUP], l[GROUP], f[GROUP];   // of the task's columns; f: this lane's piece
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
      const float2 ml = member ? *reinterpret_cast<const float2*>(my_part + NC * D + 2 * (col0 + i)) : make_float2(kKv4Low, 0.f);
      top[i] = ml.x;
      l[i] = ml.y;
    }
#pragma unroll
    for (int i = 0; i < GROUP; ++i) {
      const float m = top[i];
      top[i] = warp_max(m);
      f[i] = ex2_approx(m - top[i]);
      l[i] = warp_sum(l[i] * f[i]);
    }
    const int mine_col = PASS == 1 ? 0 : lane >> 4, d = (lane * 4) % D;
    float4 v[CHAINS];
#pragma unroll
    for (int h = 0; h < CHAINS; ++h) v[h] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (unsigned rest = members; rest != 0;) {   // four pieces at a time
      float g[4][CHAINS];
      float4 x[4][CHAINS];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const bool more = rest != 0;
        const int i = more ? __ffs(rest) - 1 : k;  // behind the last piece: a piece of the pair again, with weight 0
        rest &= rest - 1;
        const float* part = reinterpret_cast<const float*>(kv4_mem + (i >> 1) * WARP_BYTES + ((i & 1) ? 0 : WARP_BYTES - PART * 4));
#pragma unroll
        for (int h = 0; h < CHAINS; ++h) {
          g[q][h] = __shfl_sync(0xffffffffu, f[h * PASS], i);
          if (PASS == 2) {
            const float g1 = __shfl_sync(0xffffffffu, f[h * PASS + PASS - 1], i);
            g[q][h] = mine_col ? g1 : g[q][h];
          }
          if (!more) g[q][h] = 0.f;
          x[q][h] = *reinterpret_cast<const float4*>(part + kv4_piece_at<D>(col0 + h * PASS + mine_col, d >> 2));
        }
      }
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int h = 0; h < CHAINS; ++h)
          v[h] = make_float4(fmaf(x[q][h].x, g[q][h], v[h].x), fmaf(x[q][h].y, g[q][h], v[h].y), fmaf(x[q][h].z, g[q][h], v[h].z),
                             fmaf(x[q][h].w, g[q][h], v[h].w));
    }
    const bool done = pc.pair >= c_beg && pc.pair + pc.units <= c_beg + c_units;
    float* ws = a.parts + (static_cast<size_t>(blockIdx.x) * 2 + (pc.pair < c_beg ? 0 : 1)) * PART;
#pragma unroll
    for (int h = 0; h < CHAINS; ++h) {
      const int col = col0 + h * PASS + mine_col;
      const float sum = PASS == 2 && mine_col ? l[h * PASS + PASS - 1] : l[h * PASS];
      const float largest = PASS == 2 && mine_col ? top[h * PASS + PASS - 1] : top[h * PASS];
      if (done) {
        if (pc.col0 + col < a.cols) {
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
          kv4_store4(kv4_out<D>(a, pc.b, pc.hk, pc.col0 + col) + d, make_float4(v[h].x * inv, v[h].y * inv, v[h].z * inv, v[h].w * inv));
        }
      } else {
        *reinterpret_cast<float4*>(ws + col * D + d) = v[h];
        if (d == 0) *reinterpret_cast<float2*>(ws + NC * D + 2 * col) = make_float2(largest, sum);
      }
    }
    if (!done && pc.pair >= c_beg && col0 == 0 && lane == 0)
      a.splits[blockIdx.x] = Kv4Split{pc.b, pc.hk, pc.col0, static_cast<int>(kv4_cta_of(total, ctas, pc.pair + pc.units - 1))};
  }
}

// Merges the pieces of the pair that begins in CTA blockIdx.x of the kernel above and ends in a later one, one warp per
// column.
template <int D, int NT>
__global__ void __launch_bounds__(NT * 256) kv4_attn_join_kernel(const Kv4AttnArgs a) {
  constexpr int NC = NT * 8, PART = kv4_partial_floats<D, NT>(), V = D / 32;
  pdl_launch_dependents();
  pdl_wait();
  const int first = blockIdx.x, col = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // 32 pieces at a time: lane i reads the maximum and sum of piece i, then all lanes add up the outputs, whose loads do not
  // wait for one another.  Piece 1 of the first CTA, piece 0 of the others.
  auto piece = [&](int i) { return a.parts + (static_cast<size_t>(i) * 2 + (i == first ? 1 : 0)) * PART; };
  struct alignas(4 * V) Wide {
    float v[V];
  };
  auto values = [&](int i) { return reinterpret_cast<const Wide*>(piece(i) + col * D)[lane]; };
  auto max_and_sum = [&](int i0) {
    return i0 + lane < static_cast<int>(gridDim.x) ? *reinterpret_cast<const float2*>(piece(i0 + lane) + NC * D + 2 * col) : make_float2(0.f, 0.f);
  };
  // most pairs end in the next CTA: the first pieces are read along with the word that says whether there is a pair at all
  constexpr int EARLY = 2;
  Wide early[EARLY];
  float2 ml = max_and_sum(first);
#pragma unroll
  for (int i = 0; i < EARLY; ++i) early[i] = first + i < static_cast<int>(gridDim.x) ? values(first + i) : Wide{};
  const Kv4Split sp = a.splits[first];
  if (sp.last < 0) return;
  const int out_col = sp.col0 + col;
  if (out_col >= a.cols) return;
  float m = kKv4Low, l = 0.f, o[V];
#pragma unroll
  for (int e = 0; e < V; ++e) o[e] = 0.f;
  for (int i0 = first; i0 <= sp.last; i0 += 32) {
    const int n = min(32, sp.last - i0 + 1);
    if (i0 != first) ml = max_and_sum(i0);
    if (lane >= n) ml = make_float2(kKv4Low, 0.f);
    const float mn = fmaxf(m, warp_max(ml.x)), f0 = ex2_approx(m - mn), f = ex2_approx(ml.x - mn);
    m = mn;
    l = fmaf(l, f0, warp_sum(ml.y * f));
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] *= f0;
    int i = 0;
    if (i0 == first) {                 // the pair ends in a later CTA: there are at least two pieces
      static_assert(EARLY == 2, "pieces that every pair here has");
#pragma unroll
      for (; i < EARLY; ++i) {
        const float g = __shfl_sync(0xffffffffu, f, i);
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = fmaf(early[i].v[e], g, o[e]);
      }
    }
#pragma unroll 16
    for (; i < n; ++i) {
      const float g = __shfl_sync(0xffffffffu, f, i);
      const Wide x = values(i0 + i);
#pragma unroll
      for (int e = 0; e < V; ++e) o[e] = fmaf(x.v[e], g, o[e]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint32_t* dst = reinterpret_cast<uint32_t*>(kv4_out<D>(a, sp.b, sp.hk, out_col)) + lane * (V / 2);
  if constexpr (V == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv));
  else *dst = pack2(o[0] * inv, o[1] * inv);
}

}  // namespace thinfer
