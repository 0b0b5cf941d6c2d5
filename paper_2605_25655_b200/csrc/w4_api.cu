// C entry points (include/thinfer.h) of the weights in 4 bits with group scales.  Every call checks its arguments on the
// host, enqueues its kernel on the given stream and returns; no call allocates, waits or keeps anything for the next.
#include "op_host.cuh"
#include "w4_linear.cuh"
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

template <int G>
int launch_linear(const W4LinearArgs& a, bool fp32, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>((a.v.tiles + 3) / 4), static_cast<unsigned>((a.rows + 7) / 8));
  return op_launch(fp32 ? w4_linear_kernel<G, true> : w4_linear_kernel<G, false>, grid, dim3(128), 0, st, a);
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

int thinfer_op_w4_linear(const void* x, int64_t x_stride, const void* packed, void* y, int64_t y_stride, int32_t rows, int32_t n_out,
                         int32_t k, int32_t group, int32_t out_fp32, void* cuda_stream) {
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
  W4LinearArgs a{};
  a.v = w4_view(const_cast<void*>(packed), n_out, k, group);
  a.x = static_cast<const half_t*>(x);
  a.y = y;
  a.x_stride = x_stride;
  a.y_stride = y_stride;
  a.rows = rows;
  a.n = n_out;
  a.k = k;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (group == 128) return launch_linear<128>(a, out_fp32 != 0, st);
  return group == 64 ? launch_linear<64>(a, out_fp32 != 0, st) : launch_linear<32>(a, out_fp32 != 0, st);
}

}  // extern "C"
