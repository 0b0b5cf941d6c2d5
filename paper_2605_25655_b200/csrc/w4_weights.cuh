// Weights in 4 bits with a scale and a zero point per row and group of G columns (32, 64 or 128): layout, quantising, reading
// back.  A code c stands for scale * (c - zero); per group lo = min(0, min w), hi = max(0, max w), scale = (hi - lo) / 15
// rounded to the storage type, zero = clamp(rint(-lo / scale), 0, 15), code = clamp(rint(w / scale) + zero, 0, 15).
//
// Layout: rows in tiles of 16, columns in blocks of 128, both padded with zero bytes; a tile's blocks follow each other.
// Row 8 i + g of a tile, column 32 q + 8 t + 4 s + 2 b + e of a block, P = 128 / G groups in a block:
//   codes   [tile][block][q / 2][g][t][q % 2][s][e][b]   byte: row g in the low, row 8 + g in the high four bits
//   scales  [tile][block][g][P][i]                       16-bit
//   zeros   [tile][block][g][P]                          byte as for the codes
// so that lane 4 g + t of a warp finds the 64 codes of a block that it feeds to mma.m16n8k16 (rows g and 8 + g) in two
// 16-byte words, one after the other for the 32 lanes, and the 8 columns 32 q + 8 t .. of a token in one.
#pragma once
#include "common.cuh"

namespace thinfer {

struct W4View {
  uint8_t *codes, *scales, *zeros;
  long long tiles, blocks;
};

__host__ __device__ __forceinline__ long long w4_tiles(long long n) { return (n + 15) / 16; }
__host__ __device__ __forceinline__ long long w4_blocks(long long k) { return (k + 127) / 128; }
inline W4View w4_view(void* packed, int n, int k, int group) {
  W4View v{};
  v.tiles = w4_tiles(n);
  v.blocks = w4_blocks(k);
  v.codes = static_cast<uint8_t*>(packed);
  v.scales = v.codes + v.tiles * v.blocks * 1024;
  v.zeros = v.scales + v.tiles * v.blocks * (128 / group) * 32;
  return v;
}
inline size_t w4_packed_bytes(int n, int k, int group) {
  return static_cast<size_t>(w4_tiles(n)) * static_cast<size_t>(w4_blocks(k)) * (1024 + static_cast<size_t>(128 / group) * 40);
}

// ------------------------------------------------------------------ codes to numbers
// c - zero of the 8 codes of one word as pairs of the storage type, exactly: r[0], r[2] of row g, r[1], r[3] of row 8 + g.
// FP16: 0x6400 | c is 1024 + c; 0x6400 | 16 c is 1024 + 16 c, of which one multiply-add makes c - zero, so that only every
// other pair needs a shift.  BF16 has seven bits behind the point: 0x4300 | c is 128 + c.  For sums (SUMS) the BF16 build makes
// 2^-12 of that, at no cost: a token value times up to 15, 128 of them added up, could leave FP32, which a 4096th cannot.  At the
// other end nothing is lost: the smallest token, 2^-133, times 2^-12 is a multiple of FP32's smallest number.
struct W4Zero {
  uint32_t lo, hi;   // of row g and of row 8 + g
};
__device__ __forceinline__ uint32_t w4_and_or(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t w4_sub(uint32_t a, uint32_t b) {
  const half2_t d = __hsub2(*reinterpret_cast<half2_t*>(&a), *reinterpret_cast<half2_t*>(&b));
  return *reinterpret_cast<const uint32_t*>(&d);
}
#ifdef THINFER_BF16
constexpr float kW4SumsBy = 4096.f;   // what sums of the differences are multiplied by as the scale is applied
template <bool SUMS>
__device__ __forceinline__ W4Zero w4_zero(uint32_t both) {   // the byte of two zeros
  constexpr uint32_t kOne = SUMS ? 0x3d003d00u : 0x43004300u;
  return {(both & 15u) * 0x00010001u + kOne, (both >> 4) * 0x00010001u + kOne};
}
template <bool SUMS>
__device__ __forceinline__ void w4_unpack(uint32_t w, const W4Zero& z, uint32_t (&r)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = w4_sub(w4_and_or(w >> (4 * i), 0x000f000fu, SUMS ? 0x3d003d00u : 0x43004300u), i % 2 ? z.hi : z.lo);
}
#else
constexpr float kW4SumsBy = 1.f;
template <bool SUMS>
__device__ __forceinline__ W4Zero w4_zero(uint32_t both) {
  return {(both & 15u) * 0x00010001u + 0x64006400u, (both >> 4) * 0x00100010u + 0xd400d400u};
}
template <bool SUMS>
__device__ __forceinline__ void w4_unpack(uint32_t w, const W4Zero& z, uint32_t (&r)[4]) {
  const __half2 sixteenth = __floats2half2_rn(0.0625f, 0.0625f);
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    const uint32_t v = w >> (4 * i), b = w4_and_or(v, 0x00f000f0u, 0x64006400u);
    r[i] = w4_sub(w4_and_or(v, 0x000f000fu, 0x64006400u), z.lo);
    const __half2 d = __hfma2(*reinterpret_cast<const __half2*>(&b), sixteenth, *reinterpret_cast<const __half2*>(&z.hi));
    r[i + 1] = *reinterpret_cast<const uint32_t*>(&d);
  }
}
#endif

// Whether a scale times kW4SumsBy could leave FP32 (from 2^97; of a pair of 16-bit scales: one of them).  Then the group's sums are
// multiplied instead: where that leaves FP32 so does their product with the scale.
__device__ __forceinline__ bool w4_far(float scale) { return kW4SumsBy != 1.f && fabsf(scale) >= 0x1p97f; }
__device__ __forceinline__ bool w4_far(uint32_t scales) { return kW4SumsBy != 1.f && (((scales & 0x70007000u) + 0x10001000u) & 0x80008000u) != 0; }

// Two 16-bit numbers out of two pairs, chosen as __byte_perm chooses bytes.
template <int Which>
__device__ __forceinline__ half2_t w4_pair(half2_t a, half2_t b) {
  const uint32_t d = __byte_perm(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b), Which);
  return *reinterpret_cast<const half2_t*>(&d);
}

// ------------------------------------------------------------------ quantising
struct W4QuantizeArgs {
  W4View v;
  const half_t* w;
  long long stride;   // elements between rows
  int n, k;
};

__device__ __forceinline__ half_t w4_round(double x) {
#ifdef THINFER_BF16
  return __double2bfloat16(x);
#else
  return __double2half(x);
#endif
}

// Scale and zero point of a group with these extremes (high >= 0, low = -min >= 0, NaN if one of its values is).
struct W4Scale {
  half_t scale;
  float scaled, inverse, zero;   // scale * by; what a weight * by is multiplied by; the zero point
  float by;                      // 2^100 for BF16 scales whose inverse leaves FP32
  bool plain;                    // by is 1, and no weight comes out below -zero
};

// (high + low) / 15 in the storage type, rounded once: sum and quotient are rounded to odd in FP32, which keeps on which side
// of the middle of two 16-bit numbers the exact quotient is.  What FP32 cannot hold on the way goes through FP64, where
// the sum of two FP16 numbers is exact and what is rounded away of BF16 numbers is far smaller than the distance to a middle.
__device__ __forceinline__ half_t w4_fifteenth(float high, float low) {
  const float range = high + low;
  if (kStorageType == 1 && !(range >= 0x1p-90f && range <= 0x1p120f)) return w4_round((static_cast<double>(high) + static_cast<double>(low)) / 15.0);
  float sum = __fadd_rz(high, low);
  if (sum != __fadd_ru(high, low)) sum = __uint_as_float(__float_as_uint(sum) | 1u);
  constexpr float kInverse = 1.f / 15.f;
  float q = sum * kInverse;
  q = fmaf(fmaf(-15.f, q, sum), kInverse, q);
  const float left = fmaf(-15.f, q, sum);   // exact
  uint32_t bits = __float_as_uint(q);
  if (left < 0.f) --bits;
  if (left != 0.f) bits |= 1u;
  return f_to_h(__uint_as_float(bits));
}

__device__ __forceinline__ W4Scale w4_scale(float high, float low) {
  W4Scale s{};
  s.by = 1.f;
  s.plain = true;
  s.scale = f_to_h(0.f);
  if (!(high <= 3.4e38f && low <= 3.4e38f)) {   // a NaN or an infinity: the group reads as NaN
    s.scale = f_to_h(__int_as_float(0x7fffffff));
    s.plain = false;
    return s;
  }
  if (high == 0.f && low == 0.f) return s;
  s.scale = w4_fifteenth(high, low);
  s.scaled = h_to_f(s.scale);
  if (s.scaled == 0.f) {
    s.plain = false;
    return s;
  }
  if (kStorageType == 1 && s.scaled < 0x1p-100f) {
    s.by = 0x1p100f;
    s.plain = false;
  }
  s.scaled *= s.by;
  s.inverse = __frcp_rn(s.scaled);
  const float w = low * s.by, q = w * s.inverse, zero = rintf(fmaf(fmaf(-s.scaled, q, w), s.inverse, q));
  s.zero = fminf(zero, 15.f);
  s.plain = s.plain && zero <= 15.f;
  return s;
}

// rint(w / scale) between -zero and 15 - zero (whole numbers: cutting before the rounding is cutting after it), in the low
// bits of 1.5 * 2^23 + it.  The product with the inverse is corrected by its residual, after which a quotient that is the
// middle of two whole numbers comes out as that; no other comes within 2^-16 of one.
__device__ __forceinline__ uint32_t w4_code(float w, const W4Scale& s) {
  w *= s.by;
  const float q = w * s.inverse, r = fmaf(fmaf(-s.scaled, q, w), s.inverse, q);
  return __float_as_uint(fminf(fmaxf(r, -s.zero), 15.f - s.zero) + 12582912.f);
}
// The same for two weights of a plain group: with zero = rint(low / scale) none comes out below -zero.
struct W4Plain {
  uint64_t inverse, scaled;   // twice; -scaled
  float most;
};
__device__ __forceinline__ uint2 w4_codes(half2_t w, const W4Plain& s) {
  const float2 f = h2_to_f2(w);
  const uint64_t x = f32x2(f.x, f.y), q = mul_f32x2(x, s.inverse);
  const float2 r = f32x2_unpack(fma_f32x2(fma_f32x2(s.scaled, q, x), s.inverse, q));
  const float2 c = f32x2_unpack(add_f32x2(f32x2(fminf(r.x, s.most), fminf(r.y, s.most)), f32x2(12582912.f, 12582912.f)));
  return make_uint2(__float_as_uint(c.x), __float_as_uint(c.y));
}

// One warp per tile and block, 8 loads of 16 bytes in flight per lane: rows g and 8 + g, columns 32 q + 8 t ..  Bound by memory
// with groups of 128 columns.  A word's eight codes are summed up as they come (the word so far times 16 plus the next),
// and what 1.5 * 2^23 and the zero points add comes off once a word.
template <int G>
__global__ void __launch_bounds__(256, 3) w4_quantize_kernel(const __grid_constant__ W4QuantizeArgs a) {
  constexpr int P = 128 / G;
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const long long units = a.v.tiles * a.v.blocks, step = static_cast<long long>(gridDim.x) * 8;
  for (long long u = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5); u < units; u += step) {
    const long long tile = u / a.v.blocks, block = u - tile * a.v.blocks;
    const int col = static_cast<int>(block) * 128 + 8 * t;
    uint4 raw[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const long long row = tile * 16 + 8 * i + g;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        raw[i][q] = row < a.n && col + 32 * q < a.k ? ld_stream(a.w + row * a.stride + col + 32 * q) : make_uint4(0, 0, 0, 0);
    }
    // (largest, largest negated) of every group, in all four lanes of its rows
    half2_t ends[2][P];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int p = 0; p < P; ++p) {
        half2_t high = f2_to_h2(0.f, 0.f), low = high;
#pragma unroll
        for (int q = p * 4 / P; q < (p + 1) * 4 / P; ++q) {
          const half2_t* h = reinterpret_cast<const half2_t*>(&raw[i][q]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            high = __hmax2_nan(high, h[j]);
            low = __hmin2_nan(low, h[j]);
          }
        }
        low = __hneg2(low);
        half2_t both = __hmax2_nan(w4_pair<0x5410>(high, low), w4_pair<0x7632>(high, low));
#pragma unroll
        for (int o = 1; o <= 2; o <<= 1) {
          const uint32_t other = __shfl_xor_sync(0xffffffffu, *reinterpret_cast<uint32_t*>(&both), o);
          both = __hmax2_nan(both, *reinterpret_cast<const half2_t*>(&other));
        }
        ends[i][p] = both;
      }
    // lane t works out the parameters of group t % P of both rows
    W4Scale own[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      half2_t mine = ends[i][0];
#pragma unroll
      for (int p = 1; p < P; ++p) mine = t % P == p ? ends[i][p] : mine;
      const float2 e = h2_to_f2(mine);
      own[i] = w4_scale(e.x, e.y);
    }
    const long long at = (u * 8 + g) * P + t;
    if (t < P) {
      reinterpret_cast<half2_t*>(a.v.scales)[at] = half2_t(own[0].scale, own[1].scale);
      a.v.zeros[at] = static_cast<uint8_t>(static_cast<uint32_t>(own[0].zero) | static_cast<uint32_t>(own[1].zero) << 4);
    }
    const bool plain = __all_sync(0xffffffffu, own[0].plain && own[1].plain);
    auto of = [&](float v, int p) { return P == 1 ? v : __shfl_sync(0xffffffffu, v, (lane & 28) + p); };
    constexpr uint32_t kMagic = 0x4b400000u * 0x11111111u;
    uint32_t words[8];
    if (plain) {
#pragma unroll
      for (int p = 0; p < P; ++p) {
        W4Plain s[2];
        float zero[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float scaled = of(own[i].scaled, p), inverse = of(own[i].inverse, p);
          zero[i] = of(own[i].zero, p);
          s[i] = {f32x2(inverse, inverse), f32x2(-scaled, -scaled), 15.f - zero[i]};
        }
        const uint32_t less = static_cast<uint32_t>(zero[0]) * 0x01010101u + static_cast<uint32_t>(zero[1]) * 0x10101010u - kMagic;
#pragma unroll
        for (int q = p * 4 / P; q < (p + 1) * 4 / P; ++q)
#pragma unroll
          for (int st = 0; st < 2; ++st) {
            uint2 c[2][2];           // [b][i]
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int i = 0; i < 2; ++i) c[b][i] = w4_codes(reinterpret_cast<const half2_t*>(&raw[i][q])[2 * st + b], s[i]);
            uint32_t w = c[1][1].y;   // nibble 4 e + 2 b + i, highest first
            w = w * 16u + c[1][0].y;
            w = w * 16u + c[0][1].y;
            w = w * 16u + c[0][0].y;
            w = w * 16u + c[1][1].x;
            w = w * 16u + c[1][0].x;
            w = w * 16u + c[0][1].x;
            w = w * 16u + c[0][0].x;
            words[2 * q + st] = w + less;
          }
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        W4Scale s[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          s[i].scaled = of(own[i].scaled, q * P / 4);
          s[i].inverse = of(own[i].inverse, q * P / 4);
          s[i].zero = of(own[i].zero, q * P / 4);
          s[i].by = of(own[i].by, q * P / 4);
        }
#pragma unroll 1
        for (int st = 0; st < 2; ++st) {
          uint32_t w = 0;
#pragma unroll
          for (int n = 7; n >= 0; --n) {   // nibble 4 e + 2 b + i
            const uint4& from = raw[n & 1][q];
            const uint32_t pair = st == 0 ? (n & 2 ? from.y : from.x) : (n & 2 ? from.w : from.z);
            const float2 f = h2_to_f2(*reinterpret_cast<const half2_t*>(&pair));
            w = w * 16u + w4_code(n & 4 ? f.y : f.x, s[n & 1]) - 0x4b400000u + static_cast<uint32_t>(s[n & 1].zero);
          }
          if (st == 0)
            words[2 * q] = w;
          else
            words[2 * q + 1] = w;
        }
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (col + 32 * q >= a.k) words[2 * q] = words[2 * q + 1] = 0;
    uint4* out = reinterpret_cast<uint4*>(a.v.codes + u * 1024) + lane;
    out[0] = make_uint4(words[0], words[1], words[2], words[3]);
    out[32] = make_uint4(words[4], words[5], words[6], words[7]);
  }
}

// ------------------------------------------------------------------ reading back
struct W4ReadArgs {
  W4View v;
  half_t* w;
  long long stride;
  int n, k;
};

__device__ __forceinline__ half2_t w4_times(uint32_t x, half2_t s) { return __hmul2(*reinterpret_cast<half2_t*>(&x), s); }

// Lets no later kernel start before it has ended: what it writes may be the weights of a model, and the kernels of a decode step read
// those ahead of their wait.
template <int G>
__global__ void __launch_bounds__(256) w4_read_kernel(const __grid_constant__ W4ReadArgs a) {
  constexpr int P = 128 / G;
  pdl_wait();
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const long long units = a.v.tiles * a.v.blocks, step = static_cast<long long>(gridDim.x) * 8;
  for (long long u = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5); u < units; u += step) {
    const long long tile = u / a.v.blocks, block = u - tile * a.v.blocks;
    const uint4* in = reinterpret_cast<const uint4*>(a.v.codes + u * 1024) + lane;
    const uint4 c0 = ld_stream(in), c1 = ld_stream(in + 32);
    const uint32_t words[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
    half2_t scale[P];
    uint32_t zero[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
      scale[p] = reinterpret_cast<const half2_t*>(a.v.scales)[(u * 8 + g) * P + p];
      zero[p] = a.v.zeros[(u * 8 + g) * P + p];
    }
    const int col = static_cast<int>(block) * 128 + 8 * t;
    half_t* out = a.w + (tile * 16 + g) * a.stride + col;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int p = q * P / 4;
      const W4Zero z = w4_zero<false>(zero[p]);
      half2_t v[2][4];
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        uint32_t r[4];
        w4_unpack<false>(words[2 * q + st], z, r);
        // an exact difference times the scale, rounded once
        v[0][2 * st] = w4_times(r[0], w4_pair<0x1010>(scale[p], scale[p]));
        v[0][2 * st + 1] = w4_times(r[2], w4_pair<0x1010>(scale[p], scale[p]));
        v[1][2 * st] = w4_times(r[1], w4_pair<0x3232>(scale[p], scale[p]));
        v[1][2 * st + 1] = w4_times(r[3], w4_pair<0x3232>(scale[p], scale[p]));
      }
      if (col + 32 * q >= a.k) continue;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (tile * 16 + 8 * i + g < a.n) *reinterpret_cast<uint4*>(out + 8 * i * a.stride + 32 * q) = *reinterpret_cast<const uint4*>(v[i]);
    }
  }
}

}  // namespace thinfer
