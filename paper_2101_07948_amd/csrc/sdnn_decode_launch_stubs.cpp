// Host-only stand-ins for the kernel launchers of sdnn_decode.h, linked instead of the .hip files into the
// sanitizer build of the host code (see sdnn_launch_stubs.cpp).  They go through the arithmetic of a
// launch and refuse what no launch has threads for; everything else fails with hipErrorNotSupported.
#include "sdnn_decode_internal.h"
#include "sdnn_decode_shape.h"

namespace sdnn {
namespace {
hipError_t launched(bool fits) { return fits ? hipErrorNotSupported : hipErrorInvalidConfiguration; }
}  // namespace

hipError_t launch_rope(const sdnn_heads&, const sdnn_heads&, int, int32_t tokens, int32_t, const int32_t*,
                       const sdnn_rotation&, bool, hipStream_t) {
  return launched(launchable(rope_groups(tokens), kRopeThreads));
}
hipError_t launch_append(const sdnn_block_cache& c, const sdnn_tokens& t, const sdnn_heads&, const sdnn_heads&,
                         const sdnn_rotation*, const sdnn_heads* q, const sdnn_heads*, hipStream_t) {
  const AppendShape s = append_shape(c, t);
  return launched(launchable(s.windows * c.kv_heads + (q ? rope_groups(t.tokens) : 0), kRopeThreads));
}
hipError_t launch_select(const sdnn_block_cache& c, const sdnn_tokens& t, const sdnn_heads& q, int32_t, int32_t, int32_t,
                         int32_t*, hipStream_t) {
  const SelectShape s = select_shape(c, t, q.heads);
  return launched(launchable(s.groups, s.threads));
}
hipError_t launch_attend(const sdnn_block_cache& c, const sdnn_tokens& t, const sdnn_heads& q, const sdnn_heads&,
                         const int32_t* chosen, int32_t blocks, float, float*, float*, hipStream_t) {
  const AttendShape s = attend_shape(c, t, q.heads, chosen ? blocks : 0);
  return launched(launchable(s.groups, s.threads) && launchable(s.join_groups, 256));
}
hipError_t launch_qmat_pack(const sdnn_qmat_s& w, const uint8_t*, const void*, const uint8_t*, hipStream_t) {
  return launched(qmat_weight_bytes(w) >= 0 && qmat_meta_bytes(w) >= 0);
}
hipError_t launch_qmat(const sdnn_qmat_s&, const void*, int64_t, int64_t, void*, int64_t, int64_t, int32_t, int, const float*,
                       int, hipStream_t) {
  return hipErrorNotSupported;
}

}  // namespace sdnn
