// Stand-ins for the launchers of the operators of a training step (see launch_stubs.cpp): each aborts.
#include <cstdio>
#include <cstdlib>

#include "step_ops.h"
#include "window.h"

namespace spa2 {
[[noreturn]] static void reached(const char* what) {
  std::fprintf(stderr, "a rejected call reached %s\n", what);
  std::abort();
}
int gate_per_sample(const spa2_gate_shape& s, bool) { return s.tokens < 256 ? (int)s.tokens : 256; }
size_t gate_partials_bytes(const spa2_gate_shape& s) { return (size_t)s.samples * gate_per_sample(s, true) * 3 * (size_t)s.width * 4; }
hipError_t launch_gate_norm(const void*, const void*, const spa2_gate_params&, const spa2_gate_shape&, float, void*, void*, float*,
                            hipStream_t) { reached("launch_gate_norm"); }
hipError_t launch_gate_norm_bwd(const void*, const spa2_gate_params&, const spa2_gate_shape&, float, const void*, const void*, const void*,
                                const float*, void*, void*, const spa2_gate_grads&, void*, hipStream_t) { reached("launch_gate_norm_bwd"); }
size_t clip_partials_bytes() { return 6144; }
hipError_t launch_clip(const spa2_gradient*, int, double, double, float*, void*, hipStream_t) { reached("launch_clip"); }
hipError_t launch_window_few(const void*, const void*, const void*, const CrossDims&, const int32_t*, const Window&, float, void*, void*,
                             float*, void*, hipStream_t) { reached("launch_window_few"); }
hipError_t launch_window_fwd(const void*, const void*, const void*, const CrossDims&, const int32_t*, const Window&, float, void*, void*,
                             float*, void*, hipStream_t) { reached("launch_window_fwd"); }
hipError_t launch_window_dq(const void*, const void*, const void*, const void*, const void*, const void*, const float*, const CrossDims&,
                            const int32_t*, const Window&, float, float*, float*, void*, int32_t*, int, const SplitPlan&, hipStream_t) {
  reached("launch_window_dq");
}
hipError_t launch_window_dkdv(const void*, const void*, const void*, const void*, const float*, const float*, const CrossDims&,
                              const int32_t*, const Window&, float, void*, void*, const WindowColumns&, void*, void*, hipStream_t) {
  reached("launch_window_dkdv");
}
size_t fwd_slot_bytes(const Dims& m) { return (size_t)(256 * (m.d / 2) + 512) * 4; }
size_t dq_slot_bytes(const Dims& m) { return (size_t)256 * (m.d / 2) * 4; }
size_t dkdv_slot_bytes(const Dims& m) { return (size_t)4 * (m.d / 32) * 16 * 64 * 4; }
}  // namespace spa2
