// Host-only stand-ins for the kernel launchers of sdnn_serve.h, linked instead of the .hip files into the
// sanitizer build of the host code (see sdnn_launch_stubs.cpp).  They go through the arithmetic of a
// launch and refuse what no launch has threads for; everything else fails with hipErrorNotSupported.
#include "sdnn_serve_shape.h"

namespace sdnn {
namespace {
hipError_t launched(bool fits) { return fits ? hipErrorNotSupported : hipErrorInvalidConfiguration; }
}  // namespace

hipError_t launch_attend_shared(const sdnn_block_cache& c, const sdnn_tokens& t, const sdnn_heads& q, const sdnn_heads&,
                                int32_t shared, float, float*, float*, hipStream_t) {
  return launched(shared_shape(c, t.tokens, t.sequences, t.max_blocks, q.heads, shared).fits);
}
hipError_t launch_norm(const sdnn_heads& q, const sdnn_heads&, const sdnn_heads* k, const sdnn_heads*, int dtype,
                       int32_t tokens, int32_t head_dim, const int32_t*, const sdnn_head_norm&, const sdnn_rotation* r,
                       hipStream_t) {
  const int vec = row_pairs(dtype, r ? r->layout : SDNN_ROPE_HALF, r ? r->pairs : 0, head_dim);
  return launched(launchable(run_shape(tokens, head_dim / (2 * vec), {q.heads, k ? k->heads : 0, 0}).groups, kRowThreads));
}
hipError_t launch_q8_append(const sdnn_q8_cache& c, const sdnn_tokens& t, int dtype, const sdnn_heads&, const sdnn_heads&,
                            const sdnn_head_norm*, const sdnn_rotation* r, const sdnn_heads* q, const sdnn_heads*,
                            hipStream_t) {
  const int vec = row_pairs(dtype, r ? r->layout : SDNN_ROPE_HALF, r ? r->pairs : 0, c.head_dim);
  const bool windows = by_windows(t);
  const RunShape s = run_shape(t.tokens, c.head_dim / (2 * vec), {q ? q->heads : 0, c.kv_heads, windows ? 0 : c.kv_heads});
  return launched(launchable(s.groups + (windows ? window_groups(t, c.kv_heads) : 0), kRowThreads) &&
                  launchable(mean_groups(t, c.kv_heads), kRowThreads));
}
hipError_t launch_q8_read(const sdnn_q8_cache& c, const sdnn_tokens& t, int, const sdnn_heads* k, const sdnn_heads* v,
                          hipStream_t) {
  const RowShape s = row_shape(t.tokens, c.head_dim / 8, {k ? c.kv_heads : 0, v ? c.kv_heads : 0, 0});
  return launched(launchable(by_windows(t) ? window_groups(t, c.kv_heads) : s.groups, kRowThreads));
}
hipError_t launch_q8_attend(const sdnn_q8_cache& c, const sdnn_tokens& t, int, const sdnn_heads& q, const sdnn_heads&,
                            const int32_t* chosen, int32_t blocks, int32_t shared, float, float*, float*, hipStream_t) {
  const sdnn_block_cache as = as_blocks(c);
  if (shared > 0 && t.sequences > 1)
    return launched(shared_shape(as, t.tokens, t.sequences, t.max_blocks, q.heads, shared).fits);
  const AttendShape s = attend_shape(as, t, q.heads, chosen ? blocks : 0);
  return launched(launchable(s.groups, s.threads) && launchable(s.join_groups, 256));
}
hipError_t launch_sample(const void*, int64_t, int, int32_t rows, int32_t vocab, const float*, const sdnn_sampling&, int32_t*,
                         float*, float*, hipStream_t) {
  return launched(launchable(rows, kSampleThreads) && sample_floats(rows, vocab) >= 0);
}

}  // namespace sdnn
