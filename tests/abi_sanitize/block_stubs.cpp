// Stand-ins for the launchers of the operators around the attention (see launch_stubs.cpp): each aborts.
#include <cstdio>
#include <cstdlib>

#include "block_ops.h"
#include "cross.h"

namespace spa2 {
[[noreturn]] static void reached(const char* what) {
  std::fprintf(stderr, "a rejected call reached %s\n", what);
  std::abort();
}
size_t norm_rotate_partials_bytes(const spa2_norm_shape& s) { return (size_t)s.d * 8; }
hipError_t launch_norm_rotate(const void*, const void*, const float*, const float*, const NormTables&, const spa2_norm_shape&, float,
                              void*, void*, hipStream_t) { reached("launch_norm_rotate"); }
hipError_t launch_norm_rotate_bwd(const void*, const void*, const float*, const float*, const NormTables&, const void*, const void*,
                                  const spa2_norm_shape&, float, void*, void*, float*, float*, void*, hipStream_t) {
  reached("launch_norm_rotate_bwd");
}
hipError_t launch_dropout(const void*, int, const void*, int, int64_t, uint32_t, uint64_t, uint64_t, const int64_t*, void*, int,
                          hipStream_t) { reached("launch_dropout"); }
hipError_t launch_cross_few(const void*, const void*, const void*, const CrossDims&, const int32_t*, float, void*, void*, float*, void*,
                            hipStream_t) { reached("launch_cross_few"); }
hipError_t launch_cross_fwd(const void*, const void*, const void*, const CrossDims&, const int32_t*, float, void*, void*, float*, void*,
                            hipStream_t) { reached("launch_cross_fwd"); }
hipError_t launch_cross_dq(const void*, const void*, const void*, const void*, const void*, const void*, const float*, const CrossDims&,
                           const int32_t*, float, float*, float*, void*, int32_t*, int, const SplitPlan&, hipStream_t) {
  reached("launch_cross_dq");
}
hipError_t launch_cross_dkdv(const void*, const void*, const void*, const void*, const float*, const float*, const CrossDims&,
                             const int32_t*, float, void*, void*, const SplitPlan&, hipStream_t) { reached("launch_cross_dkdv"); }
size_t fwd_slot_bytes(const Dims& m) { return (size_t)(256 * (m.d / 2) + 512) * 4; }
size_t dq_slot_bytes(const Dims& m) { return (size_t)256 * (m.d / 2) * 4; }
size_t dkdv_slot_bytes(const Dims& m) { return (size_t)4 * (m.d / 32) * 16 * 64 * 4; }
}  // namespace spa2
