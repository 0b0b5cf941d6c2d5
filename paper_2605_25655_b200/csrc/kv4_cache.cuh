// Writing tokens into the 4-bit paged cache and reading them back.  D / 16 lanes hold one row (token, head, K or V), 16
// values each: with 8 values a lane the work that a row needs whatever its length took as long as the memory (52 against
// 41 us to write, 32 against 28 us to read 6800 tokens of 32 heads).  The row's extremes come from shuffles of packed 16-bit
// pairs, and the codes leave as 32-bit words (K) or as the halves that belong to the token (V).  A lane group looks its
// token's page up once, walks rows of that token, several in flight at a time, and goes on to further tokens.
//
// Measured at those tokens: writing 39 us (145 MB, 3.7 TB/s; the SMs are busy in some 60 % of their issue slots, and more loads in
// flight cost warps: 73 us against 69 for reserve, append and read with rows requested one ahead, 76 two ahead), reading 28
// us (145 MB, 5.2 TB/s, waits for its loads).  At one token per request both are one chain of three loads: 2 us.
#pragma once
#include "kv4_layout.cuh"

namespace thinfer {

struct Kv4TokensArgs {
  Kv4Cache c;
  const int32_t *rows, *positions;       // [tokens] table row and position of each token; negative: skipped
  long long tokens;
  const half_t *k, *v;                   // append: [tokens][n_kv][D], k_stride / v_stride elements between tokens
  half_t *k_out, *v_out;                 // read
  long long k_stride, v_stride;          // elements between tokens
  long long k_head, v_head;              // elements between heads
  int chunks;                            // lane groups that share the rows of one token
};

// Where a lane group's token lives.
struct Kv4Spot {
  uint8_t* page;   // first block of its page, nullptr: no page there
  int slot;
  bool skip;       // the token is padding
};

// The tokens of a lane group: first, first + step, ...  Row and position are read two tokens ahead and the page number
// one token ahead, so that only the first token waits for the chain of three loads.
struct Kv4Walk {
  const Kv4TokensArgs& a;
  long long token, step;
  int row1, pos1, row2, pos2, page1;   // of the next token, of the one after it; page of the next
  __device__ __forceinline__ void look(long long t, int& row, int& pos) const {
    row = t < a.tokens ? a.rows[t] : -1;
    pos = t < a.tokens ? a.positions[t] : -1;
  }
  __device__ __forceinline__ int page_of(int row, int pos) const {
    if (row < 0 || pos < 0 || row >= a.c.n_rows || (pos >> a.c.page_shift) >= a.c.max_pages) return -1;
    return a.c.table[static_cast<size_t>(row) * a.c.max_pages + (pos >> a.c.page_shift)];
  }
  __device__ __forceinline__ Kv4Walk(const Kv4TokensArgs& args, long long first, long long step_) : a(args), token(first - step_), step(step_) {
    look(first, row1, pos1);
    look(first + step, row2, pos2);
    page1 = page_of(row1, pos1);
  }
  // Moves to the next token; false behind the last one.
  __device__ __forceinline__ bool next(Kv4Spot& s) {
    token += step;
    if (token >= a.tokens) return false;
    const bool there = page1 >= 0 && page1 < a.c.n_pages;
    s.skip = row1 < 0 || pos1 < 0;
    s.slot = pos1 & ((1 << a.c.page_shift) - 1);
    s.page = there ? a.c.pool + static_cast<size_t>(page1) * a.c.page_bytes : nullptr;
    row1 = row2;
    pos1 = pos2;
    page1 = page_of(row1, pos1);
    look(token + 2 * step, row2, pos2);
    return true;
  }
};

constexpr int kKv4CtasPerSm = 3;        // of 256 threads
constexpr int kKv4RowsInFlight = 2;     // of an append; a read's rows are a quarter as large

__device__ __forceinline__ half2_t max2_nan(half2_t a, half2_t b) { return __hmax2_nan(a, b); }
__device__ __forceinline__ half2_t min2_nan(half2_t a, half2_t b) { return __hmin2_nan(a, b); }

// x / 15, correctly rounded: a product with the rounded reciprocal and one correction by the exact residual (Markstein's
// division theorem).
__device__ __forceinline__ float by_15(float x) {
  const float q = x * (1.f / 15.f);
  return fmaf(fmaf(-15.f, q, x), 1.f / 15.f, q);
}

// a + b, not negative: exact, or the neighbour of the exact sum with an odd last bit.
__device__ __forceinline__ float odd_sum(float a, float b) {
  return __int_as_float(__float_as_int(__fadd_rz(a, b)) | (__float_as_int(__fadd_ru(a, b)) & 1));
}
// x + less, not negative, two at a time: exact, or the neighbour of the exact sum with an odd last bit.
__device__ __forceinline__ uint64_t kv4_less(uint64_t x, uint64_t less) {
  return add_rz_f32x2(x, less) | (add_rp_f32x2(x, less) & 0x0000000100000001ull);
}

// Codes of eight values of a row with the given offset and scale, four bits each.  The quotient (x - offset) / scale is a
// product with a reciprocal and one correction by the residual, so that a quotient half way between two codes (common:
// 16-bit values lie on a grid) comes out as exactly that and the addition of 1.5 * 2^23 rounds it to the even code.  A
// quotient beside such a point must not land on it: where x - offset takes more than 24 bits (a value far smaller than the
// offset, or the other way round), the difference is rounded to the neighbour with an odd last bit.  A half step is a
// multiple of scale / 2 with at most 16 bits, so neither an odd difference of 24 bits nor its quotient, rounded once more,
// is one, and both lie on the side of it on which the exact difference lies: the codes are the exact quotient's.  (That is
// three instructions more for two values, 39 instead of 36 us; done only in rows that have such values, which takes their
// smallest size, 41.)  Two values at a time in packed FP32 (38 instead of 40 us).  A scale too small or too large for a
// reciprocal is left to a division, of halves (exact for 16-bit values), whose difference is inside FP32.
__device__ __forceinline__ uint32_t kv4_codes(const float (&x)[8], float lo, float scale) {
  uint32_t word = 0;
  const uint64_t less = f32x2(-lo, -lo);
  // a normal scale is within 2^-8 of (max - min) / 15, so that no code can pass 15
  const float smallest = kStorageType == 1 ? 0x1p-100f : 0x1p-14f;
  if (scale >= smallest && scale < 0x1p100f) {
    constexpr float M = 12582912.f;
    const float r = __fdividef(1.f, scale);
    const uint64_t inv = f32x2(r, r), neg = f32x2(-scale, -scale), magic = f32x2(M, M), back = f32x2(-M, -M);
    auto whole = [&](float a, float b) {   // M + code of two values
      const uint64_t d = kv4_less(f32x2(a, b), less), q = mul_f32x2(d, inv);
      return add_f32x2(fma_f32x2(fma_f32x2(q, neg, d), inv, q), magic);
    };
    // pairs of values 4 apart, so that the codes of two neighbours meet in the low byte of M + code + 16 * next code
    uint32_t byte[4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint64_t next = add_f32x2(whole(x[2 * j + 1], x[2 * j + 5]), back);
      const float2 both = f32x2_unpack(fma_f32x2(next, f32x2(16.f, 16.f), whole(x[2 * j], x[2 * j + 4])));
      byte[j] = __float_as_int(both.x);
      byte[j + 2] = __float_as_int(both.y);
    }
    return __byte_perm(__byte_perm(byte[0], byte[1], 0x0040), __byte_perm(byte[2], byte[3], 0x0040), 0x5410);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float d = __int_as_float(__float_as_int(__fmaf_rz(0.5f, x[j], -0.5f * lo)) | (__float_as_int(__fmaf_ru(0.5f, x[j], -0.5f * lo)) & 1));
    const float q = scale > 0.f ? fminf(rintf(__fdiv_rn(d, 0.5f * scale)), 15.f) : 0.f;
    word |= static_cast<uint32_t>(q) << (4 * j);
  }
  return word;
}

// Heads chunk, chunk + chunks, ... of K and then of V, as one sequence of 2 n_kv rows: the first head of V.
__device__ __forceinline__ int kv4_first_v(int chunk, int chunks, int n_kv) {
  return chunk >= n_kv ? chunk - n_kv : (chunks - (n_kv - chunk) % chunks) % chunks;
}

template <int D, bool V>
__device__ __forceinline__ void kv4_append_rows(const Kv4TokensArgs& a, const Kv4Spot& s, const half_t* src, int first, unsigned mask, int sub) {
  constexpr int LPR = D / 16, U = kKv4RowsInFlight;
  const int n = a.c.n_kv, page = 1 << a.c.page_shift, step = a.chunks;
  uint8_t* const params = s.page + page * D + (V ? page * 4 : 0) + s.slot * 4;
  uint8_t* const codes = s.page + (V ? page * (D / 2) + (s.slot >> 1) * D + sub * 8 + (s.slot & 1) * 2 : s.slot * (D / 2) + sub * 4);
  src += sub * 8;                      // values 8 sub .. 8 sub + 7 of each half of the row: accesses of a group lie side by side
  for (int h0 = first; h0 < n; h0 += U * step) {
    uint4 raw[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (h0 + u * step < n) {
        const half_t* p = src + (h0 + u * step) * D;
        raw[u][0] = *reinterpret_cast<const uint4*>(p);
        raw[u][1] = *reinterpret_cast<const uint4*>(p + D / 2);
      }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * step;
      if (h >= n) break;
      // extremes of the row, exact in 16 bits: largest value and largest negated value as one pair
      const half2_t* x2 = reinterpret_cast<const half2_t*>(raw[u]);
      half2_t up = x2[0], down = x2[0];
#pragma unroll
      for (int j = 1; j < 8; ++j) {
        up = max2_nan(up, x2[j]);
        down = min2_nan(down, x2[j]);
      }
      half2_t ends;
      ends.x = __hmax_nan(up.x, up.y);
      ends.y = __hneg(__hmin_nan(down.x, down.y));
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) {
        const uint32_t other = __shfl_xor_sync(mask, *reinterpret_cast<const uint32_t*>(&ends), o);
        ends = max2_nan(ends, *reinterpret_cast<const half2_t*>(&other));
      }
      const float2 hl = h2_to_f2(ends);
      // The span has to keep on which side of a tie of its fifteenth it lies: where FP16 ends take more than 24 bits, with an odd
      // last bit, as above (BF16 ends so far apart are too far from any tie).  A BF16 row may span more than FP32's largest value,
      // though not more than twice that: halves there.
      constexpr float H = kStorageType == 1 ? 0.5f : 1.f;
      const float hi = hl.x, lo = -hl.y;
      const float span = kStorageType == 1 ? H * hi - H * lo : odd_sum(hi, -lo), probe = span * 0.f;   // probe: NaN as soon as one value is NaN or infinite
      const float scale = h_to_f(f_to_h(by_15(span) * (1.f / H)));
      uint32_t word[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float x[8];
        unpack8(raw[u][j], x);
        word[j] = kv4_codes(x, lo, scale);
      }
      const int at = h * a.c.block_bytes;
      if (sub == 0) *reinterpret_cast<uint32_t*>(params + at) = kv4_pack_params(scale + probe, lo + probe);
      if (!V) {
        *reinterpret_cast<uint32_t*>(codes + at) = word[0];
        *reinterpret_cast<uint32_t*>(codes + at + D / 4) = word[1];
      } else {  // groups of four dimensions, 16 bits each, in the halves that belong to this token of the pair
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          *reinterpret_cast<uint16_t*>(codes + at + j * (D / 2)) = static_cast<uint16_t>(word[j]);
          *reinterpret_cast<uint16_t*>(codes + at + j * (D / 2) + 4) = static_cast<uint16_t>(word[j] >> 16);
        }
      }
    }
  }
}

template <int D>
__global__ void __launch_bounds__(256, kKv4CtasPerSm) kv4_append_kernel(const Kv4TokensArgs a) {
  constexpr int LPR = D / 16;
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, sub = lane % LPR;
  const unsigned mask = ((1u << LPR) - 1u) << (lane & ~(LPR - 1));
  const long long group = (static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x) / LPR;
  const long long first = group / a.chunks, step = static_cast<long long>(gridDim.x) * blockDim.x / LPR / a.chunks;
  const int chunk = static_cast<int>(group - first * a.chunks), first_v = kv4_first_v(chunk, a.chunks, a.c.n_kv);
  if (first >= step) return;
  pdl_wait();
  Kv4Walk walk(a, first, step);
  for (Kv4Spot s; walk.next(s);) {
    if (s.page == nullptr) continue;  // the same for the group, and shuffles stay inside it
    kv4_append_rows<D, false>(a, s, a.k + walk.token * a.k_stride, chunk, mask, sub);
    kv4_append_rows<D, true>(a, s, a.v + walk.token * a.v_stride, first_v, mask, sub);
  }
}

template <int D, bool V>
__device__ __forceinline__ void kv4_read_rows(const Kv4TokensArgs& a, const Kv4Spot& s, half_t* dst, long long head_stride, int first, int sub) {
  constexpr int U = 4 * kKv4RowsInFlight;
  const int n = a.c.n_kv, page = 1 << a.c.page_shift, step = a.chunks;
  const uint8_t* const params = s.page + page * D + (V ? page * 4 : 0) + s.slot * 4;
  const uint8_t* const codes = s.page + (V ? page * (D / 2) + (s.slot >> 1) * D + sub * 8 : s.slot * (D / 2) + sub * 4);
  dst += sub * 8;
  for (int h0 = first; h0 < n; h0 += U * step) {
    uint2 word[U];
    uint32_t par[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = (h0 + u * step) * a.c.block_bytes;
      word[u] = make_uint2(0, 0);
      par[u] = 0x7fff7fffu;                            // no page there: NaN
      if (s.page != nullptr && h0 + u * step < n) {
        par[u] = *reinterpret_cast<const uint32_t*>(params + at);
        if (!V) {
          word[u] = make_uint2(*reinterpret_cast<const uint32_t*>(codes + at), *reinterpret_cast<const uint32_t*>(codes + at + D / 4));
        } else {  // both tokens of the pair, this token's halves
          const uint2 x = *reinterpret_cast<const uint2*>(codes + at), y = *reinterpret_cast<const uint2*>(codes + at + D / 2);
          const int halves = s.slot & 1 ? 0x7632 : 0x5410;
          word[u] = make_uint2(__byte_perm(x.x, x.y, halves), __byte_perm(y.x, y.y, halves));
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * step;
      if (h >= n) break;
      const float2 p = kv4_unpack_params(par[u]);
      // two codes at a time as the low mantissa bits of FP16 numbers: code * 2^-24, or 2^-20 from the high nibbles.  The power
      // of two goes to the code, where it is exact: 2^24 times the scale of a BF16 row may be beyond FP32
      const uint64_t scale = f32x2(p.x, p.x), offset = f32x2(p.y, p.y);
      half_t* out = dst + h * head_stride;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const uint32_t w = g ? word[u].y : word[u].x;
        float x[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t b = (j & 2 ? w >> 8 : w) & (j & 1 ? 0x00f000f0u : 0x000f000fu);
          const float2 c = __half22float2(*reinterpret_cast<const __half2*>(&b));
          const uint64_t up = j & 1 ? f32x2(0x1p20f, 0x1p20f) : f32x2(0x1p24f, 0x1p24f);
          const float2 y = f32x2_unpack(fma_f32x2(scale, mul_f32x2(f32x2(c.x, c.y), up), offset));
          x[j] = y.x;
          x[j + 4] = y.y;
        }
        *reinterpret_cast<uint4*>(out + g * (D / 2)) = make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
      }
    }
  }
}

template <int D>
__global__ void __launch_bounds__(256, kKv4CtasPerSm) kv4_read_kernel(const Kv4TokensArgs a) {
  constexpr int LPR = D / 16;
  pdl_launch_dependents();
  const int sub = (threadIdx.x & 31) % LPR;
  const long long group = (static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x) / LPR;
  const long long first = group / a.chunks, step = static_cast<long long>(gridDim.x) * blockDim.x / LPR / a.chunks;
  const int chunk = static_cast<int>(group - first * a.chunks), first_v = kv4_first_v(chunk, a.chunks, a.c.n_kv);
  if (first >= step) return;
  pdl_wait();
  Kv4Walk walk(a, first, step);
  for (Kv4Spot s; walk.next(s);) {
    if (s.skip) continue;
    kv4_read_rows<D, false>(a, s, a.k_out + walk.token * a.k_stride, a.k_head, chunk, sub);
    kv4_read_rows<D, true>(a, s, a.v_out + walk.token * a.v_stride, a.v_head, first_v, sub);
  }
}

}  // namespace thinfer
