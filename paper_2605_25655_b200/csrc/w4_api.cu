// C entry points (include/thinfer.h) of the weights in 4 bits with group scales.  Every call checks its arguments on the
// host, enqueues its kernel on the given stream and returns; no call allocates, waits or keeps anything for the next.
#include <atomic>

#include "op_host.cuh"
#include "w4_linear.cuh"
#include "w4_linear_tc.cuh"
#include "w4_weights.cuh"

using namespace thinfer;

namespace {

constexpr int kMaxRows = 64;

int check_shape(int32_t n_out, int32_t k, int32_t group) {
  if (n_out <= 0 || k <= 0 || group <= 0) return op_fail(THINFER_EINVAL, "w4: n_out, k and group must be positive");
  if (group != 32 && group != 64 && group != 128) return op_fail(THINFER_EUNSUPPORTED, "w4: group %d: 32, 64 and 128 are supported", group);
  if (k % 8 != 0) return op_fail(THINFER_EUNSUPPORTED, "w4: k %d is no multiple of 8", k);
  return THINFER_OK;
}

// n rows of `least` elements `stride` elements apart: in order, aligned where `unit` elements are moved at once, and within 2^50
// elements, so that no product here leaves 64 bits.
bool rows_ok(int64_t stride, int64_t least, int64_t n, int64_t unit) {
  return stride >= least && stride % unit == 0 && (n <= 1 || stride <= (int64_t{1} << 50) / n);
}

// CTAs of 8 warps, a tile and block per warp, at most `waves` times 8 CTAs per SM.
unsigned unit_ctas(const W4View& v, int waves) {
  const int64_t ctas = (v.tiles * v.blocks + 7) / 8, most = static_cast<int64_t>(op_sm_count()) * 8 * waves;
  return static_cast<unsigned>(ctas < most ? ctas : most);
}

constexpr int64_t kLinearSmem = 226 * 1024, kLinearTokens = 96 * 1024;   // of a CTA; of that for the tokens, at most

// How many clusters of 2^log2 CTAs, one CTA per SM, the current device runs at once (asked once per device).
int active_clusters(int log2, int* count) {
  static std::atomic<int> known[SmemOptIn::kMaxDevices][4];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return op_fail(THINFER_ECUDA, "no current device");
  const bool keep = dev >= 0 && dev < SmemOptIn::kMaxDevices;
  *count = keep ? known[dev][log2].load(std::memory_order_relaxed) : 0;
  if (*count > 0) return THINFER_OK;
  const int rc = opt_in<w4_linear_kernel<1, 2, 128, 16>>(kLinearSmem);
  if (rc != THINFER_OK) return rc;
  cudaLaunchConfig_t lc{};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 1u << log2;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  lc.gridDim = dim3(static_cast<unsigned>(op_sm_count()) << log2);
  lc.blockDim = dim3(512);
  lc.dynamicSmemBytes = kLinearSmem;
  lc.attrs = attr;
  lc.numAttrs = 1;
  const cudaError_t e = cudaOccupancyMaxActiveClusters(count, w4_linear_kernel<1, 2, 128, 16>, &lc);
  if (e != cudaSuccess) return op_fail(THINFER_ECUDA, "cannot ask for the number of clusters: %s", cudaGetErrorString(e));
  if (*count < 1) *count = 1;
  if (keep) known[dev][log2].store(*count, std::memory_order_relaxed);
  return THINFER_OK;
}

struct LinearPlan {
  int cluster, clusters, blocks_at_once, groups_at_once;
  size_t smem;
};

// Cluster size by the bytes that the busiest CTA moves: weights, its share of the tokens (from L2, at half price), and what a
// round of sums at the end costs in bytes that could have been read meanwhile.
int plan_linear(int tiles, int blocks, int rows, int nt, int r, int warps, int stage, int token_tiles, LinearPlan* best) {
  const int64_t tokens = rows < 8 * nt ? rows : 8 * nt, groups = (tiles + r - 1) / r, per_block = tokens * 256, per_group = static_cast<int64_t>(r) * nt * 512;
  const int64_t ring = static_cast<int64_t>(warps) * (kW4Ahead + 1) * stage, left = kLinearSmem - ring - (warps + 7) * per_group;
  const int64_t most = (left < kLinearTokens ? left : kLinearTokens) / per_block;   // blocks, beside slots for 8 row groups
  int64_t least = INT64_MAX;
  for (int log2 = 0; log2 <= 3; ++log2) {
    const int64_t ctas = 1 << log2;
    if (ctas > blocks) break;
    int active = 0;
    const int rc = active_clusters(log2, &active);
    if (rc != THINFER_OK) return rc;
    int64_t clusters = active / token_tiles;
    clusters = clusters < 1 ? 1 : clusters > groups ? groups : clusters;
    const int64_t slice = (blocks + ctas - 1) / ctas, phases = (slice + most - 1) / most, held = (slice + phases - 1) / phases;
    const int64_t per = (groups + clusters - 1) / clusters, room = (kLinearSmem - ring - held * per_block) / per_group - (warps - 1);
    const int64_t batches = (per + room - 1) / room, batch = (per + batches - 1) / batches;
    const int64_t cost = per * slice * r * 1064 + (phases > 1 ? batches : 1) * slice * tokens * 128 + (batches * phases - 1) * 25000 + log2 * 6000 + (log2 == 3 ? 12000 : 0);
    if (cost >= least) continue;
    least = cost;
    best->cluster = static_cast<int>(ctas);
    best->clusters = static_cast<int>(clusters);
    best->blocks_at_once = static_cast<int>(held);
    best->groups_at_once = static_cast<int>(batch);
    best->smem = static_cast<size_t>(ring + held * per_block + (batch + warps - 1) * per_group);
  }
  return THINFER_OK;
}

template <int NT, int R, int G, int Warps>
int launch_linear(W4LinearArgs& a, cudaStream_t st) {
  const int token_tiles = (a.rows + 8 * NT - 1) / (8 * NT);
  LinearPlan p{};
  int rc = plan_linear(static_cast<int>(a.v.tiles), static_cast<int>(a.v.blocks), a.rows, NT, R, Warps, W4Stage<R, 128 / G>::kBytes, token_tiles, &p);
  if (rc == THINFER_OK) rc = opt_in<w4_linear_kernel<NT, R, G, Warps>>(kLinearSmem);
  if (rc != THINFER_OK) return rc;
  a.blocks_at_once = p.blocks_at_once;
  a.groups_at_once = p.groups_at_once;
  return op_launch_clusters(w4_linear_kernel<NT, R, G, Warps>, static_cast<unsigned>(p.cluster), dim3(static_cast<unsigned>(p.cluster * p.clusters), static_cast<unsigned>(token_tiles)),
                            dim3(Warps * 32), p.smem, st, a);
}

// Whether the tensor-memory kernel takes over: in front of and behind its stream it has two small kernels (tokens laid out, partial
// sums added up, some 5 us), while the other one walks over the weights again for every 16 rows, and needs up to 16 rows
// for longer than the bytes only where there are many of them.  FP16, us, the other one / this one, by tiles x blocks (a call
// of these varies by up to 5 %):
//   groups of 128  8192: 24 rows 10.6 / 10.9, 33 rows 13.2 / 12.7, 64 rows 16.5 / 14.5;  22016: 16 rows 12.7 / 15.4, 24 rows 17.3 / 15.7;
//                  57344: 16 rows 22.4 / 21.6;  114688: 8 rows 29.8 / 32.2, 16 rows 39.0 / 33.3, 24 rows 66.5 / 34.4, 64 rows 131 / 46
//   groups of 64   8192: 24 rows 10.8 / 12.2, 33 rows 13.7 / 13.9;  22016: 16 rows 13.0 / 15.6, 24 rows 18.5 / 15.7;  114688: 16 rows 42.5 / 40.4
//   groups of 32   8192: 24 rows 11.6 / 11.7, 33 rows 14.6 / 15.4, 64 rows 18.7 / 17.2;  22016: 24 rows 20.1 / 17.0;  114688: 16 rows 46.6 / 46.0
bool on_tensor_memory(int64_t rows, int64_t tiles, int64_t blocks, int group) {
  const int64_t units = tiles * blocks;
  return rows > 16 ? units > (rows > 32 ? 7 : 10) * 1024 : rows > 8 && group > 32 && units > 80 * 1024;
}

struct TcPlan {
  long long row_tiles;
  int ctas;
  size_t token_bytes, part_bytes;
  size_t bytes() const { return token_bytes + part_bytes; }
};
int tc_tokens(int rows) { return rows <= 32 ? 32 : 64; }
TcPlan plan_tc(int n, int group, int64_t tiles, int64_t blocks) {
  const int64_t tile = w4_tc_groups(n, group) * 128;
  TcPlan p{};
  p.row_tiles = (tiles * 16 + tile - 1) / tile;
  // as many CTAs as the device has SMs, but no more than 8 a row tile, whose sums one thread adds up (runs do not begin with a tile:
  // up to 9 CTAs may have a piece of it)
  const int64_t most = blocks < 8 ? p.row_tiles * blocks : p.row_tiles * 8;
  const int sms = op_sm_count();
  p.ctas = most < sms ? static_cast<int>(most) : sms;
  p.token_bytes = static_cast<size_t>(blocks) * n * 256;
  p.part_bytes = static_cast<size_t>(p.row_tiles + p.ctas) * n * tile * 4;
  return p;
}
size_t linear_workspace(int32_t rows, int32_t n_out, int32_t k, int32_t group) {
  return on_tensor_memory(rows, w4_tiles(n_out), w4_blocks(k), group) ? plan_tc(tc_tokens(rows), group, w4_tiles(n_out), w4_blocks(k)).bytes() : 0;
}

template <int N, int G>
int launch_tc(const W4LinearArgs& a, void* workspace, cudaStream_t st) {
  constexpr int P = 128 / G, W = W4Tc<N, P>::W, kSmem = W4Tc<N, P>::kSmem;
  const TcPlan p = plan_tc(N, G, a.v.tiles, a.v.blocks);
  char* ws = static_cast<char*>(workspace);
  const W4TcArgs args{a, reinterpret_cast<uint8_t*>(ws), reinterpret_cast<float*>(ws + p.token_bytes), p.row_tiles};
  CUtensorMap codes, scales;
  if (!op_tensor_map(&codes, a.v.codes, 256, a.v.blocks, a.v.tiles, W * 8) || !op_tensor_map(&scales, a.v.scales, 8 * P, a.v.blocks, a.v.tiles, W * 8))
    return op_fail(THINFER_ECUDA, "cuTensorMapEncodeTiled failed for packed weights");
  int rc = opt_in<w4_linear_tc_kernel<N, P>>(kSmem);
  if (rc == THINFER_OK) rc = op_launch(w4_tokens_kernel<N>, dim3(static_cast<unsigned>((a.v.blocks * N * 16 + 255) / 256)), dim3(256), 0, st, args);
  if (rc == THINFER_OK) rc = op_launch(w4_linear_tc_kernel<N, P>, dim3(static_cast<unsigned>(p.ctas)), dim3(W4Tc<N, P>::kThreads), kSmem, st, args, codes, scales);
  if (rc == THINFER_OK)
    rc = op_launch(w4_linear_join_kernel<N, W>, dim3(static_cast<unsigned>(p.row_tiles * W), static_cast<unsigned>((a.rows + N / 2 - 1) / (N / 2))), dim3(512), 0, st, args, p.ctas);
  return rc;
}

template <int G>
int launch_linear(W4LinearArgs& a, void* workspace, cudaStream_t st) {
  if (!on_tensor_memory(a.rows, a.v.tiles, a.v.blocks, G)) return a.rows <= 8 ? launch_linear<1, 2, G, 16>(a, st) : launch_linear<2, 2, G, 12>(a, st);
  return a.rows <= 32 ? launch_tc<32, G>(a, workspace, st) : launch_tc<64, G>(a, workspace, st);
}

}  // namespace

extern "C" {

int thinfer_w4_bytes(int32_t n_out, int32_t k, int32_t group, size_t* bytes) {
  if (bytes == nullptr) return op_fail(THINFER_EINVAL, "bytes is NULL");
  const int rc = check_shape(n_out, k, group);
  if (rc != THINFER_OK) return rc;
  *bytes = w4_packed_bytes(n_out, k, group);
  return THINFER_OK;
}

int thinfer_op_w4_quantize(const void* w, int64_t w_stride, void* packed, int32_t n_out, int32_t k, int32_t group, void* cuda_stream) {
  const int rc = check_shape(n_out, k, group);
  if (rc != THINFER_OK) return rc;
  if (w == nullptr || packed == nullptr) return op_fail(THINFER_EINVAL, "w4_quantize: NULL pointer");
  if (!rows_ok(w_stride, k, n_out, 8) || !aligned16(w) || !aligned16(packed))
    return op_fail(THINFER_EINVAL, "w4_quantize: a pointer or the row stride is not aligned, or the stride is below k");
  if (rows_meet(w, w_stride * 2, static_cast<int64_t>(k) * 2, n_out, {packed, w4_packed_bytes(n_out, k, group)}))
    return op_fail(THINFER_EINVAL, "w4_quantize: the packed weights overlap the weights");
  W4QuantizeArgs a{};
  a.v = w4_view(packed, n_out, k, group);
  a.w = static_cast<const half_t*>(w);
  a.stride = w_stride;
  a.n = n_out;
  a.k = k;
  auto kernel = group == 128 ? w4_quantize_kernel<128> : group == 64 ? w4_quantize_kernel<64> : w4_quantize_kernel<32>;
  return op_launch(kernel, dim3(unit_ctas(a.v, 4)), dim3(256), 0, static_cast<cudaStream_t>(cuda_stream), a);
}

int thinfer_op_w4_read(const void* packed, void* w, int64_t w_stride, int32_t n_out, int32_t k, int32_t group, void* cuda_stream) {
  const int rc = check_shape(n_out, k, group);
  if (rc != THINFER_OK) return rc;
  if (w == nullptr || packed == nullptr) return op_fail(THINFER_EINVAL, "w4_read: NULL pointer");
  if (!rows_ok(w_stride, k, n_out, 8) || !aligned16(w) || !aligned16(packed))
    return op_fail(THINFER_EINVAL, "w4_read: a pointer or the row stride is not aligned, or the stride is below k");
  if (rows_meet(w, w_stride * 2, static_cast<int64_t>(k) * 2, n_out, {packed, w4_packed_bytes(n_out, k, group)}))
    return op_fail(THINFER_EINVAL, "w4_read: the output overlaps the packed weights");
  W4ReadArgs a{};
  a.v = w4_view(const_cast<void*>(packed), n_out, k, group);
  a.w = static_cast<half_t*>(w);
  a.stride = w_stride;
  a.n = n_out;
  a.k = k;
  auto kernel = group == 128 ? w4_read_kernel<128> : group == 64 ? w4_read_kernel<64> : w4_read_kernel<32>;
  return op_launch(kernel, dim3(unit_ctas(a.v, 4)), dim3(256), 0, static_cast<cudaStream_t>(cuda_stream), a);
}

int thinfer_w4_linear_workspace(int32_t rows, int32_t n_out, int32_t k, int32_t group, size_t* bytes) {
  const int rc = check_shape(n_out, k, group);
  if (rc != THINFER_OK) return rc;
  if (bytes == nullptr || rows <= 0) return op_fail(THINFER_EINVAL, "w4_linear: no rows, or bytes is NULL");
  if (rows > kMaxRows) return op_fail(THINFER_EUNSUPPORTED, "w4_linear: %d rows > %d: read the weights back and multiply those", rows, kMaxRows);
  *bytes = linear_workspace(rows, n_out, k, group);
  return THINFER_OK;
}

int thinfer_op_w4_linear(const void* x, int64_t x_stride, const void* packed, void* y, int64_t y_stride, int32_t rows, int32_t n_out,
                         int32_t k, int32_t group, int32_t out_fp32, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  const int rc = check_shape(n_out, k, group);
  if (rc != THINFER_OK) return rc;
  if (x == nullptr || packed == nullptr || y == nullptr || rows <= 0) return op_fail(THINFER_EINVAL, "w4_linear: NULL pointer, or no rows");
  if (out_fp32 != 0 && out_fp32 != 1) return op_fail(THINFER_EINVAL, "w4_linear: out_fp32 must be 0 or 1");
  if (rows > kMaxRows) return op_fail(THINFER_EUNSUPPORTED, "w4_linear: %d rows > %d: read the weights back and multiply those", rows, kMaxRows);
  const int64_t size = out_fp32 ? 4 : 2;
  if (!rows_ok(x_stride, k, rows, 8) || !rows_ok(y_stride, n_out, rows, 1) || !aligned16(x) || !aligned16(packed) ||
      reinterpret_cast<uintptr_t>(y) % size != 0)
    return op_fail(THINFER_EINVAL, "w4_linear: a pointer or a row stride is not aligned, or a stride is below the row's length");
  if (rows_overlap(y, y_stride * size, n_out * size, x, x_stride * 2, static_cast<int64_t>(k) * 2, rows) ||
      rows_meet(y, y_stride * size, n_out * size, rows, {packed, w4_packed_bytes(n_out, k, group)}))
    return op_fail(THINFER_EINVAL, "w4_linear: the output overlaps an input");
  const size_t need = linear_workspace(rows, n_out, k, group);
  if (need > 0) {
    if (workspace == nullptr || !aligned16(workspace)) return op_fail(THINFER_EINVAL, "w4_linear: the workspace is NULL or not 16-byte aligned");
    if (workspace_bytes < need) return op_fail(THINFER_ECAPACITY, "w4_linear: the workspace has %zu bytes of %zu", workspace_bytes, need);
    const Span ws{workspace, need};
    if (rows_meet(y, y_stride * size, n_out * size, rows, ws) || rows_meet(x, x_stride * 2, static_cast<int64_t>(k) * 2, rows, ws) ||
        meet({ws}, {{packed, w4_packed_bytes(n_out, k, group)}}))
      return op_fail(THINFER_EINVAL, "w4_linear: the workspace overlaps another tensor");
  }
  W4LinearArgs a{};
  a.v = w4_view(const_cast<void*>(packed), n_out, k, group);
  a.x = static_cast<const half_t*>(x);
  a.y = y;
  a.x_stride = x_stride;
  a.y_stride = y_stride;
  a.rows = rows;
  a.n = n_out;
  a.k = k;
  a.fp32 = out_fp32;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (group == 128) return launch_linear<128>(a, workspace, st);
  return group == 64 ? launch_linear<64>(a, workspace, st) : launch_linear<32>(a, workspace, st);
}

}  // extern "C"
