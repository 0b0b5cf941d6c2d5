// C entry points (include/thinfer.h) of what chooses tokens: probabilities of logits, verification of drafts.  Every call
// checks its arguments on the host, enqueues its kernel on the given stream and returns; no call allocates, waits or keeps
// anything for the next.
#include "op_host.cuh"
#include "token_choice.cuh"

using namespace thinfer;

namespace {

constexpr int64_t kFar = int64_t{1} << 50;   // elements: no product below leaves 64 bits

// Whether the device has room for n clusters at once: two CTAs on an SM, but for some SMs that no cluster of this size finds
// neighbours for (verification of 37 x 32000 in clusters of 4 instead of 8: 9.8 us instead of 13.1; 74 x 32000 logits in
// clusters of 2 instead of 4: 6.7 instead of 9.7).
bool clusters_fit(int64_t n, int64_t ctas) { return (n + 4) * ctas <= static_cast<int64_t>(op_sm_count()) * 2; }

// Clusters of up to 8 CTAs for rows of `slots` 16-byte slots, with up to `most` slots in a CTA's slice: as many CTAs as hold a row,
// and as many as the device has room for while a CTA has more than 256 slots.
struct RowPlan {
  unsigned ctas, threads;
  int each;   // slots of a thread
};
RowPlan plan_rows(int64_t rows, int64_t slots, int64_t most, int64_t threads) {
  RowPlan p{1, 0, 1};
  while (p.ctas < 8 && (slots > p.ctas * most || (clusters_fit(rows, p.ctas * 2) && slots > p.ctas * 256))) p.ctas *= 2;
  int64_t slice = (slots + p.ctas - 1) / p.ctas;
  if (slice > most) slice = most;
  p.each = static_cast<int>((slice + threads - 1) / threads);
  p.threads = static_cast<unsigned>(((slice + p.each - 1) / p.each + 31) / 32 * 32);
  return p;
}

bool stride_ok(int64_t stride, int64_t least, int64_t n) { return stride >= least && (n <= 1 || stride <= kFar / n); }

}  // namespace

extern "C" {

int thinfer_op_token_probs(const float* logits, int64_t logit_stride, const float* temperature, float* probs, int64_t prob_stride,
                           int32_t rows, int32_t vocab, void* cuda_stream) {
  if (logits == nullptr || probs == nullptr || rows <= 0 || vocab <= 0) return op_fail(THINFER_EINVAL, "token_probs: NULL pointer, or a size that is not positive");
  if (!stride_ok(logit_stride, vocab, rows) || !stride_ok(prob_stride, vocab, rows) || !aligned4(logits) || !aligned4(probs) || !aligned4(temperature))
    return op_fail(THINFER_EINVAL, "token_probs: a pointer is not aligned, or a row stride is below vocab");
  const int64_t wide = static_cast<int64_t>(vocab) * 4;
  if ((probs != logits || prob_stride != logit_stride) && rows_overlap(probs, prob_stride * 4, wide, logits, logit_stride * 4, wide, rows))
    return op_fail(THINFER_EINVAL, "token_probs: the output overlaps the logits without being them");
  if (temperature != nullptr && rows_meet(probs, prob_stride * 4, wide, rows, {temperature, static_cast<size_t>(rows) * 4}))
    return op_fail(THINFER_EINVAL, "token_probs: the output overlaps the temperatures");
  TokenProbsArgs a{};
  a.logits = logits;
  a.out = probs;
  a.temperature = temperature;
  a.stride = logit_stride;
  a.out_stride = prob_stride;
  a.vocab = vocab;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const int64_t slots = (static_cast<int64_t>(vocab) + 6) / 4;   // wherever a row begins
  constexpr int64_t kUsual = 4096, kMost = 27 * 512;             // of a slice: 64 and 216 KB
  if (slots > 8 * kMost) return op_launch(token_probs_long_kernel, dim3(static_cast<unsigned>(rows)), dim3(512), 0, st, a);
  // 256 threads where there is a lot to do: half of the threads to set up and reduce over (320 x 128000 77 -> 74 us with the
  // rest of that step), else 512 for latency
  const RowPlan plan = plan_rows(rows, slots, slots > 8 * kUsual ? kMost : kUsual, rows * slots > 1 << 19 ? 256 : 512);
  const int64_t ctas = static_cast<int64_t>(rows) * plan.ctas;
  if (ctas > 0x7fffffff) return op_fail(THINFER_EUNSUPPORTED, "token_probs: too many rows");
  const size_t smem = static_cast<size_t>(plan.each) * plan.threads * 16;
  const int rc = opt_in<token_probs_kernel>(smem);
  if (rc != THINFER_OK) return rc;
  return op_launch_clusters(token_probs_kernel, plan.ctas, dim3(static_cast<unsigned>(ctas)), dim3(plan.threads), smem, st, a);
}

int thinfer_op_verify_drafts(const float* p, int64_t p_batch_stride, int64_t p_row_stride, const float* q, int64_t q_batch_stride,
                             int64_t q_row_stride, const int32_t* drafts, const float* uniforms, const int32_t* counts, int32_t* tokens,
                             int32_t* accepted, int32_t batch, int32_t n_drafts, int32_t vocab, void* cuda_stream) {
  if (p == nullptr || uniforms == nullptr || tokens == nullptr || accepted == nullptr || (drafts == nullptr && n_drafts > 0))
    return op_fail(THINFER_EINVAL, "verify_drafts: NULL pointer");
  if (batch <= 0 || n_drafts < 0 || vocab <= 0) return op_fail(THINFER_EINVAL, "verify_drafts: batch or vocab is not positive, or n_drafts is negative");
  if (n_drafts > 65535) return op_fail(THINFER_EUNSUPPORTED, "verify_drafts: %d drafts > 65535", n_drafts);
  if (n_drafts == 0) q = nullptr;
  const int64_t n = n_drafts, b = batch;
  if (p_batch_stride < 0 || p_row_stride < 0 || p_batch_stride > kFar / b || p_row_stride > kFar / (n + 1) ||
      (q != nullptr && (q_batch_stride < 0 || q_row_stride < 0 || q_batch_stride > kFar / b || q_row_stride > kFar / n)))
    return op_fail(THINFER_EINVAL, "verify_drafts: a stride is negative, or beyond any memory");
  for (const void* x : {static_cast<const void*>(p), static_cast<const void*>(q), static_cast<const void*>(drafts), static_cast<const void*>(uniforms),
                        static_cast<const void*>(counts), static_cast<const void*>(tokens), static_cast<const void*>(accepted)})
    if (!aligned4(x)) return op_fail(THINFER_EINVAL, "verify_drafts: a pointer is not 4-byte aligned");
  auto all = [&](const void* x, int64_t sb, int64_t sr, int64_t r) { return Span{x, x ? static_cast<size_t>((b - 1) * sb + (r - 1) * sr + vocab) * 4 : 0}; };
  const Span out{tokens, static_cast<size_t>(b * (n + 1)) * 4}, kept{accepted, static_cast<size_t>(b) * 4};
  for (const Span& in : {all(p, p_batch_stride, p_row_stride, n + 1), all(q, q_batch_stride, q_row_stride, n), Span{drafts, static_cast<size_t>(b * n) * 4},
                         Span{uniforms, static_cast<size_t>(b * (n + 1)) * 4}, Span{counts, counts ? static_cast<size_t>(b) * 4 : 0}})
    if (in.bytes != 0 && meet({out, kept}, {in})) return op_fail(THINFER_EINVAL, "verify_drafts: an output overlaps an input");
  if (meet({out}, {kept})) return op_fail(THINFER_EINVAL, "verify_drafts: tokens and accepted overlap");
  VerifyDraftsArgs a{};
  a.p = p;
  a.q = q;
  a.p_batch = p_batch_stride;
  a.p_row = p_row_stride;
  a.q_batch = q_batch_stride;
  a.q_row = q_row_stride;
  a.tokens = drafts;
  a.counts = counts;
  a.uniforms = uniforms;
  a.out = tokens;
  a.accepted = accepted;
  a.drafts = n_drafts;
  a.vocab = vocab;
  const int64_t slots = (static_cast<int64_t>(vocab) + 6) / 4;
  // 256 threads for few requests where a full cluster of them has up to four steps: fewer warps to reduce over (1 x 32000 6.6 us
  // instead of 7.2, 8 x 32000 6.9 instead of 7.5; 100 x 32000 17.8 instead of 13.7)
  const int64_t threads = slots <= 8 * 4 * 256 && clusters_fit(batch, 8) ? 256 : 512;
  const RowPlan plan = plan_rows(batch, slots, kVerifySteps * threads, threads);
  const int64_t ctas = static_cast<int64_t>(batch) * plan.ctas;
  if (ctas > 0x7fffffff) return op_fail(THINFER_EUNSUPPORTED, "verify_drafts: too many requests");
  a.steps = plan.each;
  const size_t smem = static_cast<size_t>(plan.each) * plan.threads * 8;
  const int rc = opt_in<verify_drafts_kernel>(smem);
  if (rc != THINFER_OK) return rc;
  return op_launch_clusters(verify_drafts_kernel, plan.ctas, dim3(static_cast<unsigned>(ctas)), dim3(plan.threads), smem, static_cast<cudaStream_t>(cuda_stream), a);
}

}  // extern "C"
