// C entry points (include/thinfer.h) of the per-head norm with rotation and of the 4-bit paged cache.  Every call
// checks its arguments on the host, enqueues its kernels on the given stream and returns; no call allocates, waits or
// keeps anything for the next.
#include <cmath>

#include "kv4_attn.cuh"
#include "kv4_cache.cuh"
#include "kv4_pages.cuh"
#include "op_host.cuh"
#include "qk_norm_rope.cuh"

using namespace thinfer;

namespace {

int page_shift_of(int page) { return page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : page == 128 ? 7 : -1; }

int check_layout(int32_t n_kv, int32_t head_dim, int32_t page_size) {
  if (n_kv <= 0 || head_dim <= 0 || page_size <= 0) return op_fail(THINFER_EINVAL, "n_kv_heads, head_dim and page_size must be positive");
  if (head_dim != 64 && head_dim != 128) return op_fail(THINFER_EUNSUPPORTED, "head_dim %d: 64 and 128 are supported", head_dim);
  if (page_shift_of(page_size) < 0) return op_fail(THINFER_EUNSUPPORTED, "page_size %d: 16, 32, 64 and 128 are supported", page_size);
  if (n_kv > 1024) return op_fail(THINFER_EUNSUPPORTED, "n_kv_heads %d > 1024", n_kv);
  return THINFER_OK;
}

int check_tables(const void* table, int32_t rows, int32_t max_pages, int32_t n_pages) {
  if (table == nullptr || !aligned4(table)) return op_fail(THINFER_EINVAL, "the page table is NULL or not 4-byte aligned");
  if (rows <= 0 || max_pages <= 0 || n_pages <= 0) return op_fail(THINFER_EINVAL, "rows, max_pages and n_pages must be positive");
  return THINFER_OK;
}

int check_cache(const void* pool, const void* table, int32_t rows, int32_t max_pages, int32_t n_pages, int32_t n_kv,
                int32_t head_dim, int32_t page_size) {
  if (pool == nullptr || !aligned16(pool)) return op_fail(THINFER_EINVAL, "the pool is NULL or not 16-byte aligned");
  int rc = check_layout(n_kv, head_dim, page_size);
  if (rc == THINFER_OK) rc = check_tables(table, rows, max_pages, n_pages);
  if (rc != THINFER_OK) return rc;
  if ((static_cast<int64_t>(max_pages) << page_shift_of(page_size)) > 0x7fffffff)
    return op_fail(THINFER_EUNSUPPORTED, "max_pages %d: a row holds fewer than 2^31 tokens", max_pages);
  return THINFER_OK;
}

Kv4Cache make_cache(const void* pool, const int32_t* table, int32_t rows, int32_t max_pages, int32_t n_pages, int32_t n_kv,
                    int32_t head_dim, int32_t page_size) {
  Kv4Cache c{};
  c.pool = static_cast<uint8_t*>(const_cast<void*>(pool));
  c.table = table;
  c.n_rows = rows;
  c.max_pages = max_pages;
  c.n_pages = n_pages;
  c.page_shift = page_shift_of(page_size);
  c.n_kv = n_kv;
  c.block_bytes = page_size * (head_dim + 8);
  c.page_bytes = static_cast<size_t>(n_kv) * c.block_bytes;
  return c;
}

// n rows `stride` elements apart: in order, aligned, and within 2^50 elements, so that no product here leaves 64 bits.
bool stride_ok(int64_t stride, int64_t least, int64_t n) {
  return stride >= least && stride % 8 == 0 && (n <= 1 || stride <= (int64_t{1} << 50) / n);
}

// Lane groups of `lanes` lanes that share the rows of one token: as many as fill the device once (2048 threads an
// SM), one row each at most.  Twice as many cost 5 to 15 % for long prompts, sixteen times 50 to 70 %.
int share(int64_t tokens, int64_t rows, int lanes) {
  const int64_t want = static_cast<int64_t>(op_sm_count()) * 2048 / lanes;
  const int64_t n = (want + tokens - 1) / tokens;
  return static_cast<int>(n < 1 ? 1 : n > rows ? rows : n);
}

// The same for an append or a read, whose lane groups go on to further tokens.  While one group per row fits the device
// `at_once` times, that; otherwise a power of two, so that the groups of a warp are on neighbouring heads of one token: at
// most 8 rows each (append of 7000 tokens of 32 heads, 32 / 16 / 8 / 4 rows: 21, 15, 11, 12 us), and more groups while the
// device is not full.  Against as many groups as 2048 threads an SM hold: appends of 6800 tokens of 32 heads 36 instead of
// 38 us, of 17000 from L2 20 instead of 39 (before their codes were made exact, which adds 7 % on either side); reads of 5000
// tokens of 8 heads 7 instead of 9, of 6800 of 32 heads 28 against 27.
int share_rows(int64_t tokens, int64_t rows, int lanes, int at_once) {
  const int64_t slots = static_cast<int64_t>(op_sm_count()) * (kKv4CtasPerSm * 256 / lanes);
  if (tokens * rows <= slots * at_once) return static_cast<int>(rows);
  int64_t n = rows < 4 ? rows : 4;
  while (2 * n <= rows && (rows > 8 * n || tokens * n * 4 <= slots * 3)) n *= 2;
  return static_cast<int>(n);
}

// CTAs of 256 threads for that many groups per token: `waves` resident waves at most, and at least one token's.  An append
// takes two: the second evens out the first, 20 instead of 26 us for 17000 tokens of 32 heads whose rows lie in L2 (36
// instead of 35 for 6800 from memory); a read gains nothing.
int token_ctas(int64_t tokens, int chunks, int lanes, int waves) {
  const int64_t per_cta = 256 / lanes, most = static_cast<int64_t>(kKv4CtasPerSm) * waves * op_sm_count();
  const int64_t ctas = (tokens * chunks + per_cta - 1) / per_cta, least = (chunks + per_cta - 1) / per_cta;
  return static_cast<int>(ctas < most ? ctas : most > least ? most : least);
}

size_t pool_bytes(int32_t n_pages, int32_t n_kv, int32_t head_dim, int32_t page_size) {   // of one layer
  return static_cast<size_t>(n_pages) * n_kv * page_size * (head_dim + 8);
}
size_t rows_bytes(int64_t n, int64_t stride, int64_t row) { return static_cast<size_t>((n - 1) * stride + row) * 2; }   // from first to last element
size_t table_bytes(int32_t rows, int32_t max_pages) { return static_cast<size_t>(rows) * max_pages * 4; }

// Blocks of d elements at i * ts + h * hs (i < n, h < heads; ts >= d): whether one of them shares an element with one of the
// same blocks `apart` elements further on; own: the same ones, each against the others.
bool blocks_meet(bool own, int64_t apart, int64_t ts, int64_t hs, int64_t n, int64_t heads, int64_t d) {
  for (int64_t dh = 1 - heads; dh < heads; ++dh) {
    const int64_t base = apart + dh * hs;
    // the smallest di with base + di * ts >= 0: only for that one and the one before it can the sum lie within d of 0
    const int64_t low = base >= 0 ? -(base / ts) : (-base + ts - 1) / ts;
    for (int64_t di = low - 1; di <= low; ++di) {
      const int64_t at = base + di * ts;
      if (di > -n && di < n && at > -d && at < d && !(own && dh == 0 && di == 0)) return true;
    }
  }
  return false;
}

int check_plan(int32_t rows, int32_t n_pages) {
  if (rows > kPlanMaxRows) return op_fail(THINFER_EUNSUPPORTED, "%d rows > %d", rows, kPlanMaxRows);
  if (n_pages > kPlanMaxPages) return op_fail(THINFER_EUNSUPPORTED, "%d pages > %d", n_pages, kPlanMaxPages);
  return THINFER_OK;
}

// Threads of the one CTA that plans: with little to look at its barriers are what takes the time.
int plan_threads(int32_t rows, int32_t max_pages, int32_t n_pages) {
  const int64_t entries = static_cast<int64_t>(rows) * max_pages;
  if (n_pages > 16384 || entries > 8192) return kPlanThreads;
  return entries <= 1024 ? 256 : 512;
}

size_t moves_bytes(int32_t most) { return 16 + static_cast<size_t>(most) * sizeof(PageMove); }

int copy_pages(void* pool, const int* count, const PageMove* moves, int most_moves, int layers, int n_kv, int d, int page,
               int n_pages, cudaStream_t st) {
  const size_t page_bytes = static_cast<size_t>(n_kv) * page * (d + 8);
  const long long units = static_cast<long long>(most_moves) * layers * n_kv * (page / 16);
  const long long ctas = (units + 15) / 16, room = static_cast<long long>(op_sm_count()) * 32;   // 8 warps, two units each; a resident wave (8 an SM) took 3 % longer
  return op_launch(d == 128 ? kv4_copy_pages_kernel<128> : kv4_copy_pages_kernel<64>,
                   dim3(static_cast<unsigned>(ctas < room ? ctas : room)), dim3(256), 0, st, static_cast<uint8_t*>(pool),
                   count, moves, layers, n_kv, page_shift_of(page), page_bytes, page_bytes * static_cast<size_t>(n_pages));
}

// Column tiles of 8 (16 where a KV head has more query columns than 8, so that its keys are unpacked half as often) and
// one CTA per SM.
struct AttnPlan {
  int tiles, col_tiles, grid;
  size_t split_bytes, part_bytes;
};
int plan_attention(int32_t batch, int32_t queries, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, AttnPlan* p) {
  if (head_dim != 64 && head_dim != 128) return op_fail(THINFER_EUNSUPPORTED, "head_dim %d: 64 and 128 are supported", head_dim);
  if (n_q_heads % n_kv_heads != 0) return op_fail(THINFER_EUNSUPPORTED, "n_q_heads must be a multiple of n_kv_heads");
  const int64_t cols = static_cast<int64_t>(n_q_heads / n_kv_heads) * queries;
  p->tiles = cols > 8 ? 2 : 1;
  const int64_t col_tiles = (cols + 8 * p->tiles - 1) / (8 * p->tiles);
  if (batch > 2048 || col_tiles * n_kv_heads > 16384)
    return op_fail(THINFER_EUNSUPPORTED, "kv4_attention: batch %d > 2048, or more than 262144 query columns per request", batch);
  p->col_tiles = static_cast<int>(col_tiles);
  p->grid = op_sm_count();
  p->split_bytes = (static_cast<size_t>(p->grid) * sizeof(Kv4Split) + 255) / 256 * 256;
  p->part_bytes = static_cast<size_t>(p->grid) * 2 * p->tiles * 8 * (head_dim + 2) * 4;
  return THINFER_OK;
}

template <int D, int NT>
int launch_attention(const Kv4AttnArgs& a, int grid, cudaStream_t st) {
  const size_t smem = kv4_warps<NT>() * kv4_warp_bytes<D, NT>() + kv4_plan_bytes(a.batch);
  int rc = opt_in<kv4_attn_kernel<D, NT>>(smem);
  if (rc == THINFER_OK) rc = op_launch(kv4_attn_kernel<D, NT>, dim3(grid), dim3(kv4_warps<NT>() * 32), smem, st, a);
  if (rc == THINFER_OK) rc = op_launch(kv4_attn_join_kernel<D, NT>, dim3(grid), dim3(NT * 256), 0, st, a);
  return rc;
}

}  // namespace

extern "C" {

int thinfer_rope_turns(float base, int32_t rotary_dim, double* host_out) {
  if (host_out == nullptr || !(base > 0.f) || rotary_dim <= 0 || rotary_dim % 2 != 0)
    return op_fail(THINFER_EINVAL, "rope_turns: base must be positive, rotary_dim positive and even");
  for (int j = 0; j < rotary_dim / 2; ++j)
    host_out[j] = std::pow(static_cast<double>(base), -2.0 * j / rotary_dim) / 6.283185307179586476925286766559;
  return THINFER_OK;
}

int thinfer_op_qk_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride, void* q_out,
                            int64_t q_out_stride, void* k_out, int64_t k_out_stride, const void* q_gain,
                            const void* k_gain, const double* turns, const int32_t* positions, int32_t tokens,
                            int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t rotary_dim, int32_t halves,
                            float eps, void* cuda_stream) {
  if (q == nullptr || k == nullptr || q_out == nullptr || k_out == nullptr || q_gain == nullptr || k_gain == nullptr ||
      (turns == nullptr && rotary_dim > 0) || positions == nullptr)
    return op_fail(THINFER_EINVAL, "qk_norm_rope: NULL pointer");
  if (tokens <= 0 || n_q_heads <= 0 || n_kv_heads <= 0 || head_dim <= 0 || rotary_dim < 0 || !(eps >= 0.f))
    return op_fail(THINFER_EINVAL, "qk_norm_rope: a size is not positive, or eps is negative");
  if (head_dim != 64 && head_dim != 128) return op_fail(THINFER_EUNSUPPORTED, "head_dim %d: 64 and 128 are supported", head_dim);
  if (rotary_dim > head_dim || rotary_dim % 16 != 0)
    return op_fail(THINFER_EUNSUPPORTED, "rotary_dim %d: a multiple of 16 up to head_dim", rotary_dim);
  if (halves != 0 && halves != 1) return op_fail(THINFER_EINVAL, "halves must be 0 or 1");
  if (n_q_heads > 65536 || n_kv_heads > 65536) return op_fail(THINFER_EUNSUPPORTED, "more than 65536 heads");
  const int64_t q_row = static_cast<int64_t>(n_q_heads) * head_dim, k_row = static_cast<int64_t>(n_kv_heads) * head_dim;
  if (!stride_ok(q_stride, q_row, tokens) || !stride_ok(q_out_stride, q_row, tokens) || !stride_ok(k_stride, k_row, tokens) ||
      !stride_ok(k_out_stride, k_row, tokens))
    return op_fail(THINFER_EINVAL, "qk_norm_rope: a token stride is below heads * head_dim or no multiple of 8");
  if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out) || !aligned16(q_gain) || !aligned16(k_gain) ||
      !aligned4(positions) || (reinterpret_cast<uintptr_t>(turns) & 7u) != 0)
    return op_fail(THINFER_EINVAL, "qk_norm_rope: a pointer is not aligned");
  auto meet = [&](const void* x, int64_t sx, int64_t wx, const void* y, int64_t sy, int64_t wy) {
    return rows_overlap(x, sx * 2, wx * 2, y, sy * 2, wy * 2, tokens);
  };
  if (((q_out != q || q_out_stride != q_stride) && meet(q_out, q_out_stride, q_row, q, q_stride, q_row)) ||
      ((k_out != k || k_out_stride != k_stride) && meet(k_out, k_out_stride, k_row, k, k_stride, k_row)) ||
      meet(q_out, q_out_stride, q_row, k, k_stride, k_row) || meet(k_out, k_out_stride, k_row, q, q_stride, q_row) ||
      meet(q_out, q_out_stride, q_row, k_out, k_out_stride, k_row))
    return op_fail(THINFER_EINVAL, "qk_norm_rope: an output overlaps an input that it does not replace, or the other output");
  const size_t gain_bytes = static_cast<size_t>(head_dim) * 2;
  for (const Span& in : {Span{q_gain, gain_bytes}, Span{k_gain, gain_bytes}, Span{turns, static_cast<size_t>(rotary_dim) * 4}, Span{positions, static_cast<size_t>(tokens) * 4}})
    if (rows_meet(q_out, q_out_stride * 2, q_row * 2, tokens, in) || rows_meet(k_out, k_out_stride * 2, k_row * 2, tokens, in))
      return op_fail(THINFER_EINVAL, "qk_norm_rope: an output overlaps gains, turns or positions");
  QkNormRopeArgs a{};
  a.q = static_cast<const half_t*>(q);
  a.k = static_cast<const half_t*>(k);
  a.q_out = static_cast<half_t*>(q_out);
  a.k_out = static_cast<half_t*>(k_out);
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.q_out_stride = q_out_stride;
  a.k_out_stride = k_out_stride;
  a.q_gain = static_cast<const half_t*>(q_gain);
  a.k_gain = static_cast<const half_t*>(k_gain);
  a.turns = turns;
  a.positions = positions;
  a.tokens = tokens;
  a.n_q = n_q_heads;
  a.n_kv = n_kv_heads;
  a.half = rotary_dim / 2;
  a.eps = eps;
  a.least = eps < 0x1p-80f ? 0x1p-100f : 0.f;   // beside a larger eps nothing is lost below 2^-100
  a.chunks = share(tokens, static_cast<int64_t>(n_q_heads) + n_kv_heads, head_dim / 8);
  const int64_t groups = static_cast<int64_t>(tokens) * a.chunks, per_cta = 256 / (head_dim / 8);
  const int64_t ctas = (groups + per_cta - 1) / per_cta;
  if (ctas > 0x7fffffff) return op_fail(THINFER_EUNSUPPORTED, "qk_norm_rope: too many tokens");
  auto kernel = head_dim == 128 ? (halves ? qk_norm_rope_kernel<128, true> : qk_norm_rope_kernel<128, false>)
                                : (halves ? qk_norm_rope_kernel<64, true> : qk_norm_rope_kernel<64, false>);
  return op_launch(kernel, dim3(static_cast<unsigned>(ctas)), dim3(256), 0, static_cast<cudaStream_t>(cuda_stream), a);
}

int thinfer_kv4_page_bytes(int32_t n_kv_heads, int32_t head_dim, int32_t page_size, size_t* bytes) {
  if (bytes == nullptr) return op_fail(THINFER_EINVAL, "bytes is NULL");
  const int rc = check_layout(n_kv_heads, head_dim, page_size);
  if (rc != THINFER_OK) return rc;
  *bytes = static_cast<size_t>(n_kv_heads) * page_size * (head_dim + 8);
  return THINFER_OK;
}

int thinfer_op_kv4_append(void* pool, int32_t n_pages, const int32_t* table, int32_t n_rows, int32_t max_pages,
                          const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* rows,
                          const int32_t* positions, int32_t tokens, int32_t n_kv_heads, int32_t head_dim,
                          int32_t page_size, void* cuda_stream) {
  const int rc = check_cache(pool, table, n_rows, max_pages, n_pages, n_kv_heads, head_dim, page_size);
  if (rc != THINFER_OK) return rc;
  if (k == nullptr || v == nullptr || rows == nullptr || positions == nullptr || tokens <= 0)
    return op_fail(THINFER_EINVAL, "kv4_append: NULL pointer or no tokens");
  const int64_t row = static_cast<int64_t>(n_kv_heads) * head_dim;
  if (!stride_ok(k_stride, row, tokens) || !stride_ok(v_stride, row, tokens) || !aligned16(k) || !aligned16(v) || !aligned4(rows) || !aligned4(positions))
    return op_fail(THINFER_EINVAL, "kv4_append: a pointer or a token stride is not aligned, or a stride is below heads * head_dim");
  const size_t list_bytes = static_cast<size_t>(tokens) * 4;
  if (meet({{pool, pool_bytes(n_pages, n_kv_heads, head_dim, page_size)}},
           {{k, rows_bytes(tokens, k_stride, row)}, {v, rows_bytes(tokens, v_stride, row)}, {table, table_bytes(n_rows, max_pages)}, {rows, list_bytes}, {positions, list_bytes}}))
    return op_fail(THINFER_EINVAL, "kv4_append: the pool overlaps what is written into it, the table, rows or positions");
  Kv4TokensArgs a{};
  a.c = make_cache(pool, table, n_rows, max_pages, n_pages, n_kv_heads, head_dim, page_size);
  a.rows = rows;
  a.positions = positions;
  a.tokens = tokens;
  a.chunks = share_rows(tokens, 2 * static_cast<int64_t>(n_kv_heads), head_dim / 16, 2);
  a.k = static_cast<const half_t*>(k);
  a.v = static_cast<const half_t*>(v);
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  const int ctas = token_ctas(tokens, a.chunks, head_dim / 16, 2);
  return op_launch(head_dim == 128 ? kv4_append_kernel<128> : kv4_append_kernel<64>, dim3(static_cast<unsigned>(ctas)),
                   dim3(256), 0, static_cast<cudaStream_t>(cuda_stream), a);
}

int thinfer_op_kv4_read(const void* pool, int32_t n_pages, const int32_t* table, int32_t n_rows, int32_t max_pages,
                        void* k_out, void* v_out, int64_t token_stride, int64_t head_stride, const int32_t* rows,
                        const int32_t* positions, int32_t tokens, int32_t n_kv_heads, int32_t head_dim,
                        int32_t page_size, void* cuda_stream) {
  const int rc = check_cache(pool, table, n_rows, max_pages, n_pages, n_kv_heads, head_dim, page_size);
  if (rc != THINFER_OK) return rc;
  if (k_out == nullptr || v_out == nullptr || rows == nullptr || positions == nullptr || tokens <= 0)
    return op_fail(THINFER_EINVAL, "kv4_read: NULL pointer or no tokens");
  if (!stride_ok(token_stride, head_dim, tokens) || !stride_ok(head_stride, head_dim, n_kv_heads) || !aligned16(k_out) || !aligned16(v_out) ||
      !aligned4(rows) || !aligned4(positions))
    return op_fail(THINFER_EINVAL, "kv4_read: a pointer or a stride is not aligned, or a stride is below head_dim");
  const int64_t d = head_dim, across = (n_kv_heads - 1) * head_stride + d, along = (tokens - 1) * token_stride + d;
  const size_t out_bytes = static_cast<size_t>(along + across - d) * 2, list_bytes = static_cast<size_t>(tokens) * 4;
  // one of the two usual orders, or looked at block by block
  if (token_stride < across && head_stride < along && blocks_meet(true, 0, token_stride, head_stride, tokens, n_kv_heads, d))
    return op_fail(THINFER_EINVAL, "kv4_read: with these strides rows of an output overlap each other");
  const int64_t apart = (reinterpret_cast<intptr_t>(v_out) - reinterpret_cast<intptr_t>(k_out)) / 2;
  if (overlap(k_out, out_bytes, v_out, out_bytes) && blocks_meet(false, apart, token_stride, head_stride, tokens, n_kv_heads, d))
    return op_fail(THINFER_EINVAL, "kv4_read: k_out and v_out overlap");
  if (meet({{k_out, out_bytes}, {v_out, out_bytes}}, {{pool, pool_bytes(n_pages, n_kv_heads, head_dim, page_size)}, {table, table_bytes(n_rows, max_pages)},
                                                      {rows, list_bytes}, {positions, list_bytes}}))
    return op_fail(THINFER_EINVAL, "kv4_read: an output overlaps the pool, the table, rows or positions");
  Kv4TokensArgs a{};
  a.c = make_cache(pool, table, n_rows, max_pages, n_pages, n_kv_heads, head_dim, page_size);
  a.rows = rows;
  a.positions = positions;
  a.tokens = tokens;
  a.chunks = share_rows(tokens, 2 * static_cast<int64_t>(n_kv_heads), head_dim / 16, 1);
  a.k_out = static_cast<half_t*>(k_out);
  a.v_out = static_cast<half_t*>(v_out);
  a.k_stride = a.v_stride = token_stride;
  a.k_head = a.v_head = head_stride;
  const int ctas = token_ctas(tokens, a.chunks, head_dim / 16, 1);
  return op_launch(head_dim == 128 ? kv4_read_kernel<128> : kv4_read_kernel<64>, dim3(static_cast<unsigned>(ctas)),
                   dim3(256), 0, static_cast<cudaStream_t>(cuda_stream), a);
}

int thinfer_kv4_attention_workspace(int32_t batch, int32_t queries, int32_t n_q_heads, int32_t n_kv_heads,
                                    int32_t head_dim, size_t* bytes) {
  if (bytes == nullptr || batch <= 0 || queries <= 0 || n_q_heads <= 0 || n_kv_heads <= 0)
    return op_fail(THINFER_EINVAL, "kv4_attention: a size is not positive, or bytes is NULL");
  AttnPlan p;
  const int rc = plan_attention(batch, queries, n_q_heads, n_kv_heads, head_dim, &p);
  if (rc != THINFER_OK) return rc;
  *bytes = p.split_bytes + p.part_bytes;
  return THINFER_OK;
}

int thinfer_op_kv4_attention(const void* q, int64_t q_stride, const void* pool, int32_t n_pages, const int32_t* table,
                             int32_t max_pages, const int32_t* lens, void* out, int32_t batch, int32_t queries,
                             int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t page_size, void* workspace,
                             size_t workspace_bytes, void* cuda_stream) {
  int rc = check_cache(pool, table, batch, max_pages, n_pages, n_kv_heads, head_dim, page_size);
  if (rc != THINFER_OK) return rc;
  if (q == nullptr || lens == nullptr || out == nullptr || workspace == nullptr || queries <= 0 || n_q_heads <= 0)
    return op_fail(THINFER_EINVAL, "kv4_attention: NULL pointer, or a size that is not positive");
  AttnPlan p;
  rc = plan_attention(batch, queries, n_q_heads, n_kv_heads, head_dim, &p);
  if (rc != THINFER_OK) return rc;
  if (!stride_ok(q_stride, static_cast<int64_t>(n_q_heads) * head_dim, static_cast<int64_t>(batch) * queries) || !aligned16(q) || !aligned16(out) || !aligned4(lens) || !aligned16(workspace))
    return op_fail(THINFER_EINVAL, "kv4_attention: a pointer or the token stride is not aligned, or the stride is below heads * head_dim");
  if (workspace_bytes < p.split_bytes + p.part_bytes)
    return op_fail(THINFER_ECAPACITY, "kv4_attention: the workspace has %zu bytes of %zu", workspace_bytes, p.split_bytes + p.part_bytes);
  const size_t out_bytes = static_cast<size_t>(batch) * queries * n_q_heads * head_dim * 2, ws_bytes = p.split_bytes + p.part_bytes;
  const size_t q_bytes = ((static_cast<size_t>(batch) * queries - 1) * q_stride + static_cast<size_t>(n_q_heads) * head_dim) * 2;
  const size_t tab_bytes = static_cast<size_t>(batch) * max_pages * 4, len_bytes = static_cast<size_t>(batch) * 4;
  if (overlap(out, out_bytes, workspace, ws_bytes) || overlap(out, out_bytes, q, q_bytes) || overlap(out, out_bytes, table, tab_bytes) ||
      overlap(out, out_bytes, lens, len_bytes) || overlap(workspace, ws_bytes, q, q_bytes) || overlap(workspace, ws_bytes, table, tab_bytes) ||
      overlap(workspace, ws_bytes, lens, len_bytes) ||
      meet({{pool, pool_bytes(n_pages, n_kv_heads, head_dim, page_size)}}, {{out, out_bytes}, {workspace, ws_bytes}}))
    return op_fail(THINFER_EINVAL, "kv4_attention: the output or the workspace overlaps an input, or they overlap each other");
  Kv4AttnArgs a{};
  a.c = make_cache(pool, table, batch, max_pages, n_pages, n_kv_heads, head_dim, page_size);
  a.lens = lens;
  a.q = static_cast<const half_t*>(q);
  a.out = static_cast<half_t*>(out);
  a.q_stride = q_stride;
  a.batch = batch;
  a.queries = queries;
  a.n_q = n_q_heads;
  a.group = n_q_heads / n_kv_heads;
  a.cols = a.group * queries;
  a.col_tiles = p.col_tiles;
  a.splits = static_cast<Kv4Split*>(workspace);
  a.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.split_bytes);
  a.inv_group = 1.f / static_cast<float>(a.group);
  a.scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(head_dim));
  // no more CTAs than the table's capacity could give a unit per warp
  const int64_t units = static_cast<int64_t>(batch) * n_kv_heads * p.col_tiles *
                        ((static_cast<int64_t>(max_pages) * page_size + kKv4Unit - 1) / kKv4Unit);
  const int warps = p.tiles == 1 ? kv4_warps<1>() : kv4_warps<2>();
  const int64_t most = (units + warps - 1) / warps;
  const int grid = most < p.grid ? static_cast<int>(most) : p.grid;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (head_dim == 128) return p.tiles == 1 ? launch_attention<128, 1>(a, grid, st) : launch_attention<128, 2>(a, grid, st);
  return p.tiles == 1 ? launch_attention<64, 1>(a, grid, st) : launch_attention<64, 2>(a, grid, st);
}

int thinfer_op_kv4_reserve(int32_t* table, const int32_t* lens, const int32_t* add, int32_t* lens_out, int64_t* refused,
                           int32_t n_rows, int32_t max_pages, int32_t n_pages, int32_t page_size, void* cuda_stream) {
  int rc = check_tables(table, n_rows, max_pages, n_pages);
  if (rc == THINFER_OK) rc = check_layout(1, 64, page_size);
  if (rc == THINFER_OK) rc = check_plan(n_rows, n_pages);
  if (rc != THINFER_OK) return rc;
  if (lens == nullptr || add == nullptr || lens_out == nullptr || refused == nullptr || !aligned4(lens) || !aligned4(add) ||
      !aligned4(lens_out) || !aligned8(refused))
    return op_fail(THINFER_EINVAL, "kv4_reserve: a pointer is NULL or not 4-byte aligned");
  const size_t nb = static_cast<size_t>(n_rows) * 4, tb = nb * max_pages;
  if (overlap(table, tb, lens, nb) || overlap(table, tb, add, nb) || overlap(table, tb, lens_out, nb) || overlap(table, tb, refused, 8))
    return op_fail(THINFER_EINVAL, "kv4_reserve: the table overlaps another tensor");
  if ((lens_out != lens && overlap(lens_out, nb, lens, nb)) || overlap(lens_out, nb, add, nb) || overlap(refused, 8, lens, nb) ||
      overlap(refused, 8, add, nb) || overlap(refused, 8, lens_out, nb))
    return op_fail(THINFER_EINVAL, "kv4_reserve: lens_out may be lens itself; other outputs must not overlap inputs");
  if ((static_cast<int64_t>(max_pages) * page_size) > 0x7fffffff)
    return op_fail(THINFER_EUNSUPPORTED, "max_pages %d: a row holds fewer than 2^31 tokens", max_pages);
  const PageTables t{table, lens, n_rows, max_pages, n_pages, page_shift_of(page_size)};
  const size_t smem = static_cast<size_t>(plan_words(n_pages)) * 8;
  rc = opt_in<kv4_reserve_kernel>(smem);
  if (rc != THINFER_OK) return rc;
  return op_launch(kv4_reserve_kernel, dim3(1), dim3(plan_threads(n_rows, max_pages, n_pages)), smem, static_cast<cudaStream_t>(cuda_stream), t,
                   table, add, lens_out, refused);
}

int thinfer_kv4_pages_workspace(int32_t n_rows, int32_t n_pages, size_t* bytes) {
  if (bytes == nullptr || n_rows <= 0 || n_pages <= 0) return op_fail(THINFER_EINVAL, "kv4_pages_workspace: a size is not positive, or bytes is NULL");
  const int rc = check_plan(n_rows, n_pages);
  if (rc != THINFER_OK) return rc;
  *bytes = moves_bytes(n_rows > n_pages / 2 ? n_rows : n_pages / 2);  // a compaction moves at most half of the pages
  return THINFER_OK;
}

int thinfer_op_kv4_fork(void* pool, int32_t n_layers, int32_t n_pages, const int32_t* table, const int32_t* lens,
                        const int32_t* source, int32_t* table_out, int32_t* lens_out, int64_t* refused, int32_t n_rows,
                        int32_t max_pages, int32_t n_kv_heads, int32_t head_dim, int32_t page_size, void* workspace,
                        size_t workspace_bytes, void* cuda_stream) {
  int rc = check_cache(pool, table, n_rows, max_pages, n_pages, n_kv_heads, head_dim, page_size);
  if (rc == THINFER_OK) rc = check_plan(n_rows, n_pages);
  if (rc != THINFER_OK) return rc;
  if (n_layers <= 0 || lens == nullptr || source == nullptr || table_out == nullptr || lens_out == nullptr || refused == nullptr ||
      workspace == nullptr || !aligned4(lens) || !aligned4(source) || !aligned4(table_out) || !aligned4(lens_out) ||
      !aligned8(refused) || !aligned16(workspace))
    return op_fail(THINFER_EINVAL, "kv4_fork: a pointer is NULL or not aligned, or n_layers is not positive");
  const size_t nb = static_cast<size_t>(n_rows) * 4, tb = nb * max_pages;
  const void* ins[3] = {table, lens, source};
  const size_t in_b[3] = {tb, nb, nb};
  void* outs[3] = {table_out, lens_out, refused};
  const size_t out_b[3] = {tb, nb, 8};
  for (int o = 0; o < 3; ++o) {
    for (int i = 0; i < 3; ++i)
      if (overlap(outs[o], out_b[o], ins[i], in_b[i])) return op_fail(THINFER_EINVAL, "kv4_fork: an output overlaps an input");
    for (int p = 0; p < o; ++p)
      if (overlap(outs[o], out_b[o], outs[p], out_b[p])) return op_fail(THINFER_EINVAL, "kv4_fork: two outputs overlap");
  }
  if (workspace_bytes < moves_bytes(n_rows)) return op_fail(THINFER_ECAPACITY, "kv4_fork: the workspace is too small");
  const Span all_pages{pool, pool_bytes(n_pages, n_kv_heads, head_dim, page_size) * n_layers}, ws{workspace, moves_bytes(n_rows)};
  if (meet({all_pages, ws}, {{table, tb}, {lens, nb}, {source, nb}, {table_out, tb}, {lens_out, nb}, {refused, 8}}) || meet({all_pages}, {ws}))
    return op_fail(THINFER_EINVAL, "kv4_fork: the pool or the workspace overlaps another tensor");
  const PageTables t{table, lens, n_rows, max_pages, n_pages, page_shift_of(page_size)};
  const size_t smem = static_cast<size_t>(plan_words(n_pages)) * 8 + nb * 4;
  rc = opt_in<kv4_fork_kernel>(smem);
  if (rc != THINFER_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  int* count = static_cast<int*>(workspace);
  PageMove* moves = reinterpret_cast<PageMove*>(static_cast<char*>(workspace) + 16);
  rc = op_launch(kv4_fork_kernel, dim3(1), dim3(plan_threads(n_rows, max_pages, n_pages)), smem, st, t, source, table_out, lens_out, refused, count, moves);
  if (rc != THINFER_OK) return rc;
  return copy_pages(pool, count, moves, n_rows, n_layers, n_kv_heads, head_dim, page_size, n_pages, st);
}

int thinfer_op_kv4_compact(void* pool, int32_t n_layers, int32_t n_pages, const int32_t* table, const int32_t* lens,
                           int32_t* table_out, int64_t* live_pages, int32_t n_rows, int32_t max_pages,
                           int32_t n_kv_heads, int32_t head_dim, int32_t page_size, void* workspace,
                           size_t workspace_bytes, void* cuda_stream) {
  int rc = check_cache(pool, table, n_rows, max_pages, n_pages, n_kv_heads, head_dim, page_size);
  if (rc == THINFER_OK) rc = check_plan(n_rows, n_pages);
  if (rc != THINFER_OK) return rc;
  if (n_layers <= 0 || lens == nullptr || table_out == nullptr || live_pages == nullptr || workspace == nullptr || !aligned4(lens) ||
      !aligned4(table_out) || !aligned8(live_pages) || !aligned16(workspace))
    return op_fail(THINFER_EINVAL, "kv4_compact: a pointer is NULL or not aligned, or n_layers is not positive");
  const size_t nb = static_cast<size_t>(n_rows) * 4, tb = nb * max_pages;
  if (overlap(table_out, tb, table, tb) || overlap(table_out, tb, lens, nb) || overlap(live_pages, 8, table, tb) ||
      overlap(live_pages, 8, lens, nb) || overlap(live_pages, 8, table_out, tb))
    return op_fail(THINFER_EINVAL, "kv4_compact: an output overlaps another tensor");
  const int most = n_pages / 2 > 0 ? n_pages / 2 : 1;
  if (workspace_bytes < moves_bytes(n_pages / 2)) return op_fail(THINFER_ECAPACITY, "kv4_compact: the workspace is too small");
  const Span all_pages{pool, pool_bytes(n_pages, n_kv_heads, head_dim, page_size) * n_layers}, ws{workspace, moves_bytes(n_pages / 2)};
  if (meet({all_pages, ws}, {{table, tb}, {lens, nb}, {table_out, tb}, {live_pages, 8}}) || meet({all_pages}, {ws}))
    return op_fail(THINFER_EINVAL, "kv4_compact: the pool or the workspace overlaps another tensor");
  const PageTables t{table, lens, n_rows, max_pages, n_pages, page_shift_of(page_size)};
  const size_t smem = static_cast<size_t>(plan_words(n_pages)) * 8;
  rc = opt_in<kv4_compact_kernel>(smem);
  if (rc != THINFER_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  int* count = static_cast<int*>(workspace);
  PageMove* moves = reinterpret_cast<PageMove*>(static_cast<char*>(workspace) + 16);
  rc = op_launch(kv4_compact_kernel, dim3(1), dim3(plan_threads(n_rows, max_pages, n_pages)), smem, st, t, table_out, live_pages, count, moves);
  if (rc != THINFER_OK) return rc;
  return copy_pages(pool, count, moves, most, n_layers, n_kv_heads, head_dim, page_size, n_pages, st);
}

}  // extern "C"
