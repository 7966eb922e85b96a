// Host-side declarations of the operators of a training step around the attention (not part of the ABI): the gated sum with its
// norms, the norm over all gradients and their clipping.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "spa2.h"

namespace spa2 {

inline int gate_threads(int width) { return 64 * ((width + 511) / 512); }      // of a workgroup
int gate_per_sample(const spa2_gate_shape& s, bool backward);
size_t gate_partials_bytes(const spa2_gate_shape& s);
hipError_t launch_gate_norm(const void* x, const void* branch, const spa2_gate_params& p, const spa2_gate_shape& s, float eps,
                            void* y, void* n, float* stats, hipStream_t stream);
hipError_t launch_gate_norm_bwd(const void* branch, const spa2_gate_params& p, const spa2_gate_shape& s, float eps, const void* y,
                                const void* dy, const void* dn, const float* stats, void* dx, void* dbranch,
                                const spa2_gate_grads& grads, void* ws, hipStream_t stream);

size_t clip_partials_bytes();
hipError_t launch_clip(const spa2_gradient* gradients, int count, double max_norm, double eps, float* norm, void* ws,
                       hipStream_t stream);

}  // namespace spa2
