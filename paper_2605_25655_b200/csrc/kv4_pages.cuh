// Page tables of the 4-bit cache on the device: reserving pages for new tokens, forking rows, compacting the pool.
//
// A page is in use when a row's table names it among its first ceil(len / P) entries; nothing else records ownership,
// so no reference counts can go wrong and no host state has to follow the device.  One CTA marks the pages in use in
// a shared-memory bitmap (one bit per page of the pool), takes prefix counts of it, and answers "the k-th free page"
// by a binary search: all choices go to the lowest page number first and depend on nothing but the tables.
// The pages that have to move are written to a list that a second kernel, chained to the first, copies with all SMs.
#pragma once
#include "kv4_layout.cuh"

namespace thinfer {

constexpr int kPlanThreads = 1024;
constexpr int kPlanMaxPages = 1 << 18;
constexpr int kPlanMaxRows = 4096;

struct PageMove {
  int src, dst, tokens;  // tokens: the filled ones, rounded up to 16 by the copy
};

struct PageTables {
  const int32_t* table;
  const int32_t* lens;
  int rows, max_pages, n_pages, page_shift;
};

__device__ __forceinline__ int tables_clamp(const PageTables& t, int n) {  // tokens of a row, within what its table can name
  const long long cap = static_cast<long long>(t.max_pages) << t.page_shift;
  return n < 0 ? 0 : (n > cap ? static_cast<int>(cap) : n);
}
__device__ __forceinline__ int tables_len(const PageTables& t, int r) { return tables_clamp(t, t.lens[r]); }
__device__ __forceinline__ int pages_for(int tokens, int shift) {
  return static_cast<int>((static_cast<long long>(tokens) + (1 << shift) - 1) >> shift);
}

// Calls f(row, column, tokens of the row, entry) for every entry of the tables, used or not, with live = false for those
// behind a row's pages.  Small tables are taken as one run of entries, four per thread in flight, whose lengths and
// numbers are read at the same time; of large ones only the live spans of each row are read, a warp per span (ALL: the
// others are visited as well, without being read).
constexpr int kPlanSpan = 256;           // table columns of one warp task
constexpr int kPlanFlat = 1 << 16;       // entries up to which a table counts as small
template <bool ALL, typename F>
__device__ __forceinline__ void for_entries(const PageTables& t, F f) {
  const long long entries = static_cast<long long>(t.rows) * t.max_pages;
  if (entries <= kPlanFlat) {
    constexpr int U = 4;
    const int e = static_cast<int>(entries);
    for (int i0 = threadIdx.x; i0 < e; i0 += U * blockDim.x) {
      int p[U], n[U], r[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * blockDim.x;
        if (i < e) {
          r[u] = static_cast<int>(static_cast<unsigned>(i) / static_cast<unsigned>(t.max_pages));
          p[u] = t.table[i];
          n[u] = t.lens[r[u]];
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * blockDim.x;
        if (i >= e) break;
        const int c = i - r[u] * t.max_pages, len = tables_clamp(t, n[u]);
        const bool live = c < pages_for(len, t.page_shift);
        if (ALL || live) f(r[u], c, len, p[u], live);
      }
    }
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int spans = (t.max_pages + kPlanSpan - 1) / kPlanSpan;
  const long long tasks = static_cast<long long>(t.rows) * spans;
  for (long long k = warp; k < tasks; k += warps) {
    const int r = static_cast<int>(k / spans), c0 = static_cast<int>(k - static_cast<long long>(r) * spans) * kPlanSpan;
    const int len = tables_len(t, r), n = pages_for(len, t.page_shift);
    const int c1 = min(ALL ? t.max_pages : n, c0 + kPlanSpan);
    const int32_t* row = t.table + static_cast<size_t>(r) * t.max_pages;
    for (int c = c0 + lane; c < c1; c += 32) f(r, c, len, c < n ? row[c] : -1, c < n);
  }
}

// Exclusive sum over the CTA of one value per thread; total for everybody.  buf: 33 ints of shared memory.
__device__ __forceinline__ int block_exclusive(int v, int* buf, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  int s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += u;
  }
  __syncthreads();
  if (lane == 31) buf[warp] = s;
  __syncthreads();
  if (warp == 0) {
    int w = lane < warps ? buf[lane] : 0, ws = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, ws, o);
      if (lane >= o) ws += u;
    }
    buf[lane] = ws - w;
    if (lane == 31) buf[32] = ws;
  }
  __syncthreads();
  *total = buf[32];
  return buf[warp] + s - v;
}

// Bitmap of the pages in use and, per 32-page word, the number of pages in use in the words before it.
struct PageMap {
  uint32_t* bits;
  int* before;
  int words, live;
  __device__ int live_below(int p) const {
    const int w = p >> 5;
    if (w >= words) return live;
    return before[w] + __popc(bits[w] & ((1u << (p & 31)) - 1u));
  }
  __device__ bool used(int p) const { return (bits[p >> 5] >> (p & 31)) & 1u; }
  // the k-th free page (from 0), k < n_pages - live: the bits behind the last page count as free and come last
  __device__ int free_page(int k) const {
    int lo = 0, hi = words - 1;
    while (lo < hi) {  // the last word with at most k free pages before it
      const int mid = (lo + hi + 1) >> 1;
      if (32 * mid - before[mid] <= k) lo = mid;
      else hi = mid - 1;
    }
    // the (k+1)-th set bit of the word, by halves
    uint32_t z = ~bits[lo];
    int left = k - (32 * lo - before[lo]), at = 0;
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) {
      const int n = __popc(z & ((1u << w) - 1u));
      if (left >= n) {
        left -= n;
        at += w;
        z >>= w;
      }
    }
    return 32 * lo + at;
  }
};

__host__ __device__ constexpr int plan_words(int n_pages) { return (n_pages + 31) / 32; }

// Whole CTA.  mem: 2 * plan_words ints of shared memory.
__device__ __forceinline__ PageMap map_pages(const PageTables& t, int* mem, int* buf) {
  PageMap m;
  m.words = plan_words(t.n_pages);
  m.bits = reinterpret_cast<uint32_t*>(mem);
  m.before = mem + m.words;
  for (int w = threadIdx.x; w < m.words; w += blockDim.x) m.bits[w] = 0;
  __syncthreads();
  for_entries<false>(t, [&](int, int, int, int p, bool) {
    if (p >= 0 && p < t.n_pages) atomicOr(&m.bits[p >> 5], 1u << (p & 31));
  });
  __syncthreads();
  const int per = (m.words + blockDim.x - 1) / blockDim.x;
  const int w0 = min(m.words, static_cast<int>(threadIdx.x) * per), w1 = min(m.words, w0 + per);
  int mine = 0;
  for (int w = w0; w < w1; ++w) mine += __popc(m.bits[w]);
  int run = block_exclusive(mine, buf, &m.live);
  for (int w = w0; w < w1; ++w) {
    m.before[w] = run;
    run += __popc(m.bits[w]);
  }
  __syncthreads();
  return m;
}

// ---------------------------------------------------------------- reserve
// Rows in ascending order take the lowest free pages for `add` more tokens each; a row whose pages, with those of the
// rows before it, do not fit the pool or its table keeps its length and is counted in *refused.
// Bounded by the latency of one CTA's dependent steps (1.8 us when no row opens a page, 3.6 us for the 8 rows of a prompt
// batch).  The new pages are dealt over all threads: with a warp per row, 8 rows of 256 new pages took 26 us, now 7.
__global__ void __launch_bounds__(kPlanThreads) kv4_reserve_kernel(const PageTables t, int32_t* table, const int32_t* add,
                                                                   int32_t* lens_out, int64_t* refused) {
  extern __shared__ int plan_mem[];
  __shared__ int buf[33];
  __shared__ int wanted, bad;
  __shared__ int row_begin[kPlanThreads], row_need[kPlanThreads], row_first[kPlanThreads];
  pdl_launch_dependents();
  pdl_wait();
  if (threadIdx.x == 0) wanted = bad = 0;
  __syncthreads();
  auto need_of = [&](int r, int* first, long long* after) {
    const int n = max(t.lens[r], 0), a = max(add[r], 0);   // a length beyond the table asks for what it says, and is refused
    *first = pages_for(n, t.page_shift);
    *after = static_cast<long long>(n) + a;
    return static_cast<int>(((*after + (1 << t.page_shift) - 1) >> t.page_shift) - *first);
  };
  int first = 0;
  long long after = 0;
  for (int r = threadIdx.x; r < t.rows; r += blockDim.x)
    if (need_of(r, &first, &after) > 0) wanted = 1;
  __syncthreads();
  PageMap m{};
  if (wanted) m = map_pages(t, plan_mem, buf);  // most decode steps stay inside their pages and need no map
  const int free_pages = t.n_pages - m.live;
  long long carry = 0;
  for (int r0 = 0; r0 < t.rows; r0 += blockDim.x) {
    const int r = r0 + threadIdx.x;
    int need = 0;
    if (r < t.rows) need = need_of(r, &first, &after);
    // a need beyond the pool refuses its row and those behind it whatever its size: clamped so that the sum stays small
    const int asked = min(need, t.n_pages + 1);
    int total;
    const int local = block_exclusive(asked, buf, &total);
    const long long begin = carry + local;
    if (r < t.rows) {
      // a row that claims more tokens than its table can name is refused as well
      const bool fits = t.lens[r] <= (static_cast<long long>(t.max_pages) << t.page_shift) &&
                        (need == 0 || (begin + need <= free_pages && first + need <= t.max_pages));
      if (!fits) atomicAdd(&bad, 1);
      lens_out[r] = fits ? static_cast<int>(after) : t.lens[r];
      need = fits ? need : 0;
    }
    row_begin[threadIdx.x] = local;
    row_need[threadIdx.x] = need;
    row_first[threadIdx.x] = first;
    __syncthreads();
    // the new pages of these rows, one per thread and step: page g belongs to the last row that begins at or before it
    const int n = static_cast<int>(min(static_cast<long long>(total), free_pages - carry));
    for (int g = threadIdx.x; g < n; g += blockDim.x) {
      int lo = 0, hi = min(static_cast<int>(blockDim.x), t.rows - r0) - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (row_begin[mid] <= g) lo = mid;
        else hi = mid - 1;
      }
      const int j = g - row_begin[lo];
      if (j < row_need[lo])
        table[static_cast<size_t>(r0 + lo) * t.max_pages + row_first[lo] + j] = m.free_page(static_cast<int>(carry) + g);
    }
    carry += total;
    __syncthreads();
  }
  if (threadIdx.x == 0) *refused = bad;
}

// ---------------------------------------------------------------- fork
__global__ void __launch_bounds__(kPlanThreads) kv4_fork_kernel(const PageTables t, const int32_t* source, int32_t* table_out,
                                                                int32_t* lens_out, int64_t* refused, int* move_count,
                                                                PageMove* moves) {
  extern __shared__ int plan_mem[];
  __shared__ int buf[33];
  __shared__ int bad;
  pdl_launch_dependents();
  int* owner = plan_mem;                  // [rows] who keeps the partly filled last page of a source
  int* fresh = plan_mem + t.rows;         // [rows] page of a row's own copy, or -1
  int* from = plan_mem + 2 * t.rows;      // [rows] the source
  int* tokens = plan_mem + 3 * t.rows;    // [rows] the new length
  pdl_wait();
  for (int r = threadIdx.x; r < t.rows; r += blockDim.x) owner[r] = 0x7fffffff;
  if (threadIdx.x == 0) bad = 0;
  const PageMap m = map_pages(t, plan_mem + 4 * t.rows, buf);
  for (int r = threadIdx.x; r < t.rows; r += blockDim.x) {
    const int s = source[r];
    if (s >= 0 && s < t.rows) atomicMin(&owner[s], s == r ? -1 : r);
  }
  __syncthreads();
  const int free_pages = t.n_pages - m.live, page = 1 << t.page_shift;
  int carry = 0;
  for (int r0 = 0; r0 < t.rows; r0 += blockDim.x) {
    const int r = r0 + threadIdx.x;
    int s = -1, n = 0, old = -1;
    bool ok = true;
    if (r < t.rows) {
      s = source[r];
      if (s >= t.rows) {
        ok = false;
        s = -1;
      }
      if (s >= 0) n = tables_len(t, s);
      if ((n & (page - 1)) != 0 && owner[s] != r && !(owner[s] == -1 && s == r)) {
        old = t.table[static_cast<size_t>(s) * t.max_pages + (n >> t.page_shift)];
        if (old >= t.n_pages) old = -1;  // no page of the pool: the entry is taken over as it is
      }
    }
    int total;
    const int k = carry + block_exclusive(old >= 0 ? 1 : 0, buf, &total);
    if (r < t.rows) {
      fresh[r] = -1;
      if (old >= 0) {
        if (k < free_pages) {
          fresh[r] = m.free_page(k);
          moves[k] = PageMove{old, fresh[r], n & (page - 1)};
        } else {
          ok = false;
        }
      }
      if (!ok) {
        n = 0;
        atomicAdd(&bad, 1);
      }
      lens_out[r] = n;
      from[r] = s;
      tokens[r] = n;
    }
    carry += total;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    *refused = bad;
    *move_count = min(carry, free_pages);
  }
  // the new tables, entry by entry, four per thread in flight
  const long long entries = static_cast<long long>(t.rows) * t.max_pages;
  constexpr int U = 4;
  for (long long i0 = threadIdx.x; i0 < entries; i0 += U * blockDim.x) {
    int p[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = i0 + static_cast<long long>(u) * blockDim.x;
      p[u] = -1;
      if (i < entries) {
        const int r = (i >> 32) == 0 ? static_cast<int>(static_cast<unsigned>(i) / static_cast<unsigned>(t.max_pages)) : static_cast<int>(i / t.max_pages);
        const int c = static_cast<int>(i - static_cast<long long>(r) * t.max_pages), pages = pages_for(tokens[r], t.page_shift);
        if (c < pages) p[u] = fresh[r] >= 0 && c == pages - 1 ? fresh[r] : t.table[static_cast<size_t>(from[r]) * t.max_pages + c];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = i0 + static_cast<long long>(u) * blockDim.x;
      if (i < entries) table_out[i] = p[u];
    }
  }
}

// ---------------------------------------------------------------- compact
// Live pages with a number >= the number of live pages move, in ascending order, into the free pages below it.
__global__ void __launch_bounds__(kPlanThreads) kv4_compact_kernel(const PageTables t, int32_t* table_out, int64_t* live_out,
                                                                   int* move_count, PageMove* moves) {
  extern __shared__ int plan_mem[];
  __shared__ int buf[33];
  pdl_launch_dependents();
  pdl_wait();
  const PageMap m = map_pages(t, plan_mem, buf);
  const int stay = m.live_below(m.live), n_moves = m.live - stay;
  // moves in the order of their sources
  for (int w = (m.live >> 5) + threadIdx.x; w < m.words; w += blockDim.x) {
    uint32_t z = m.bits[w];
    if (w == (m.live >> 5)) z &= ~((1u << (m.live & 31)) - 1u);
    for (; z != 0; z &= z - 1) {
      const int p = 32 * w + __ffs(z) - 1, k = m.live_below(p) - stay;
      moves[k] = PageMove{p, m.free_page(k), 0};
    }
  }
  if (threadIdx.x == 0) {
    *live_out = m.live;
    *move_count = n_moves;
  }
  __syncthreads();
  for_entries<true>(t, [&](int r, int c, int n, int p, bool live) {
    if (!live) {
      p = -1;
    } else if (p >= m.live && p < t.n_pages) {
      const int k = m.live_below(p) - stay;
      atomicMax(&moves[k].tokens, min(1 << t.page_shift, n - (c << t.page_shift)));
      p = moves[k].dst;
    }
    table_out[static_cast<size_t>(r) * t.max_pages + c] = p;
  });
}

// ---------------------------------------------------------------- the copies
// A warp takes 16 tokens of one (move, layer, head) block at a time: D / 4 pieces of 16 bytes of K codes, as many of V
// codes and four of each kind of params.  Two such units are in flight at a time.
template <int D>
__global__ void __launch_bounds__(256) kv4_copy_pages_kernel(uint8_t* pool, const int* move_count, const PageMove* moves,
                                                             int layers, int n_kv, int page_shift, size_t page_bytes,
                                                             size_t layer_bytes) {
  constexpr int R = D / 64, U = 2;     // rows of 32 pieces of each kind of codes
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x & 31, page = 1 << page_shift, group_shift = page_shift - 4;
  const long long warps = static_cast<long long>(gridDim.x) * (blockDim.x >> 5);
  const long long first = static_cast<long long>(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int blocks = layers * n_kv;    // of one move
  const long long units = (static_cast<long long>(*move_count) * blocks) << group_shift;
  for (long long i0 = first; i0 < units; i0 += U * warps) {
    uint4 v[U][2 * R + 1];
    uint8_t* dst[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long i = i0 + u * warps;
      dst[u] = nullptr;
      if (i >= units) continue;
      const long long b = i >> group_shift;
      const int g = static_cast<int>(i) & ((1 << group_shift) - 1);
      const int k = (b >> 32) == 0 ? static_cast<int>(static_cast<uint32_t>(b) / static_cast<uint32_t>(blocks)) : static_cast<int>(b / blocks);
      const int rest = static_cast<int>(b - static_cast<long long>(k) * blocks), layer = rest / n_kv, head = rest - layer * n_kv;
      const PageMove mv = moves[k];
      if (16 * g >= mv.tokens) continue;
      const size_t base = static_cast<size_t>(layer) * layer_bytes + static_cast<size_t>(head) * (page * (D + 8)) + g * (8 * D);
      const uint8_t* src = pool + base + static_cast<size_t>(mv.src) * page_bytes;
      dst[u] = pool + base + static_cast<size_t>(mv.dst) * page_bytes;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        v[u][r] = ld_stream(src + (r * 32 + lane) * 16);
        v[u][R + r] = ld_stream(src + page * (D / 2) + (r * 32 + lane) * 16);
      }
      // params: lanes 0-3 of K, 4-7 of V; 64 bytes for 16 tokens, 8 D back to the start of the block's codes
      const int par = page * D - g * (8 * D) + g * 64 + (lane & 4 ? page * 4 : 0) + (lane & 3) * 16;
      if (lane < 8) v[u][2 * R] = ld_stream(src + par);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (dst[u] == nullptr) continue;
      const int g = static_cast<int>(i0 + u * warps) & ((1 << group_shift) - 1);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        *reinterpret_cast<uint4*>(dst[u] + (r * 32 + lane) * 16) = v[u][r];
        *reinterpret_cast<uint4*>(dst[u] + page * (D / 2) + (r * 32 + lane) * 16) = v[u][R + r];
      }
      const int par = page * D - g * (8 * D) + g * 64 + (lane & 4 ? page * 4 : 0) + (lane & 3) * 16;
      if (lane < 8) *reinterpret_cast<uint4*>(dst[u] + par) = v[u][2 * R];
    }
  }
}

}  // namespace thinfer
