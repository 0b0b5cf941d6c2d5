// Writing tokens into the 4-bit paged cache and reading them back.  Both are bound by memory: D / 8 lanes hold one
// row (token, head, K or V) with one 16-byte access each, the row's extremes come from shuffles, and the codes leave
// as one 32-bit word per lane.
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
};

// A row index in the order (token, head, K | V).
struct Kv4RowIndex {
  long long token;
  int head, which;
};
__device__ __forceinline__ Kv4RowIndex kv4_row_index(long long i, int n_kv) {
  Kv4RowIndex r;
  r.token = i / (2 * n_kv);
  const int rest = static_cast<int>(i - r.token * (2 * n_kv));
  r.which = rest / n_kv;
  r.head = rest - r.which * n_kv;
  return r;
}

template <int D>
__global__ void __launch_bounds__(256) kv4_append_kernel(const Kv4TokensArgs a) {
  constexpr int LPR = D / 8;
  const int lane = threadIdx.x & 31, sub = lane % LPR;
  const long long i = (static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x) / LPR;
  const Kv4RowIndex r = kv4_row_index(i, a.c.n_kv);
  uint8_t* block = nullptr;
  int slot = 0;
  if (r.token < a.tokens) {
    const int row = __ldg(a.rows + r.token), pos = __ldg(a.positions + r.token);
    if (row >= 0 && pos >= 0) block = kv4_block(a.c, row, pos, r.head);
    slot = pos & ((1 << a.c.page_shift) - 1);
  }
  uint4 raw = make_uint4(0, 0, 0, 0);
  if (block != nullptr) {
    const half_t* src = (r.which ? a.v + r.token * a.v_stride : a.k + r.token * a.k_stride) + static_cast<long long>(r.head) * D;
    raw = *reinterpret_cast<const uint4*>(src + sub * 8);
  }
  float x[8];
  unpack8(raw, x);
  float lo = x[0], hi = x[0], probe = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    lo = fminf(lo, x[j]);
    hi = fmaxf(hi, x[j]);
    probe += x[j] * 0.f;  // NaN as soon as one value is NaN or infinite
  }
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    probe += __shfl_xor_sync(0xffffffffu, probe, o);
  }
  if (block == nullptr) return;
  const float scale = h_to_f(f_to_h(__fdiv_rn(hi - lo, 15.f)));
  uint32_t word = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float c = scale > 0.f ? fminf(rintf(__fdiv_rn(x[j] - lo, scale)), 15.f) : 0.f;
    word |= static_cast<uint32_t>(c) << (4 * j);
  }
  const int page = 1 << a.c.page_shift;
  uint8_t* par = block + page * D + (r.which ? page * 4 : 0) + slot * 4;
  if (sub == 0) *reinterpret_cast<uint32_t*>(par) = kv4_pack_params(scale + probe, lo + probe);
  if (r.which == 0) {
    *reinterpret_cast<uint32_t*>(block + slot * (D / 2) + sub * 4) = word;
  } else {  // two groups of four dimensions, 16 bits each, in the halves that belong to this token of the pair
    uint16_t* dst = reinterpret_cast<uint16_t*>(block + page * (D / 2) + (slot >> 1) * D + sub * 8) + (slot & 1);
    dst[0] = static_cast<uint16_t>(word);
    dst[2] = static_cast<uint16_t>(word >> 16);
  }
}

template <int D>
__global__ void __launch_bounds__(256) kv4_read_kernel(const Kv4TokensArgs a) {
  constexpr int LPR = D / 8;
  const int sub = (threadIdx.x & 31) % LPR;
  const long long i = (static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x) / LPR;
  const Kv4RowIndex r = kv4_row_index(i, a.c.n_kv);
  if (r.token >= a.tokens) return;
  const int row = __ldg(a.rows + r.token), pos = __ldg(a.positions + r.token);
  if (row < 0 || pos < 0) return;
  const uint8_t* block = kv4_block(a.c, row, pos, r.head);
  const int page = 1 << a.c.page_shift, slot = pos & (page - 1);
  float scale = __int_as_float(0x7fffffff), off = scale;  // no page there: NaN
  uint32_t word = 0;
  if (block != nullptr) {
    const float2 p = kv4_unpack_params(*reinterpret_cast<const uint32_t*>(block + page * D + (r.which ? page * 4 : 0) + slot * 4));
    scale = p.x;
    off = p.y;
    if (r.which == 0) {
      word = *reinterpret_cast<const uint32_t*>(block + slot * (D / 2) + sub * 4);
    } else {
      const uint16_t* src = reinterpret_cast<const uint16_t*>(block + page * (D / 2) + (slot >> 1) * D + sub * 8) + (slot & 1);
      word = src[0] | (static_cast<uint32_t>(src[2]) << 16);
    }
  }
  float x[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = fmaf(scale, static_cast<float>((word >> (4 * j)) & 15u), off);
  half_t* dst = (r.which ? a.v_out + r.token * a.v_stride + r.head * a.v_head : a.k_out + r.token * a.k_stride + r.head * a.k_head);
  *reinterpret_cast<uint4*>(dst + sub * 8) = make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
}

}  // namespace thinfer
