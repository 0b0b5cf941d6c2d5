// Layout of the 4-bit paged key / value cache and the arithmetic of one quantised row.
//
// A page holds P tokens (16, 32, 64 or 128) of one layer: for every KV head one block of P * (D + 8) bytes,
//   K codes   [P][D/2]           byte i of a token: code 2i in the low four bits, code 2i + 1 in the high ones
//   V codes   [P/2][D/4][2][2]   token pair, group of four dimensions, token of the pair, two bytes as for K
//   K params  [P][2] 16-bit      scale, offset of the token's row
//   V params  [P][2] 16-bit
// and a code c stands for offset + scale * c.  V puts the two tokens of a pair side by side in every 32-bit word: the
// matrix instructions of the output product contract over tokens and want two neighbouring tokens of one dimension in
// a register, which a mask and a shift then give without any permutation.
//
// Quantisation of a row x of D values: offset = min x (exact in 16 bits), scale = (max x - min x) / 15 rounded to the
// storage type, code = (x - offset) / scale rounded to nearest, ties to even, at most 15; scale 0 gives code 0.  A row
// that holds a NaN or an infinity gets NaN params, so that everything that reads it sees NaN; a finite row is stored as it
// is, over the whole range of the type (at whose end a value read back may round to infinity).  The rounding of the
// scale to 16 bits costs at most half a unit of its last place times 15 at the top of the row: 15 * 2^-12 of a step in
// FP16 and 15 * 2^-9 in BF16, small against the half step of the code itself.
#pragma once
#include "common.cuh"

namespace thinfer {

struct Kv4Cache {
  uint8_t* pool;         // pages of one layer
  const int32_t* table;  // [n_rows][max_pages] page ids
  int n_rows, max_pages, n_pages;
  int page_shift;        // log2 of the page size
  int n_kv;
  int block_bytes;       // P * (D + 8)
  size_t page_bytes;     // n_kv * block_bytes
};

__device__ __forceinline__ uint32_t kv4_pack_params(float scale, float offset) { return pack2(scale, offset); }
__device__ __forceinline__ float2 kv4_unpack_params(uint32_t p) { return h2_to_f2(*reinterpret_cast<const half2_t*>(&p)); }

}  // namespace thinfer
