// Host-side declarations of the operators around the block-sparse attention (not part of the ABI): norm and rotation of
// q and k, dropout with the residual sum.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "spa2.h"

namespace spa2 {

constexpr int64_t CACHE_BYTES = 256ll << 20;         // memory-side cache of the card

struct NormTables { const float* cos; const float* sin; const void* positions; };

size_t norm_rotate_partials_bytes(const spa2_norm_shape& s);
hipError_t launch_norm_rotate(const void* q, const void* k, const float* q_weight, const float* k_weight, const NormTables& t,
                              const spa2_norm_shape& s, float eps, void* q_out, void* k_out, hipStream_t stream);
hipError_t launch_norm_rotate_bwd(const void* q, const void* k, const float* q_weight, const float* k_weight,
                                  const NormTables& t, const void* d_q_out, const void* d_k_out, const spa2_norm_shape& s,
                                  float eps, void* dq, void* dk, float* d_q_weight, float* d_k_weight, void* ws,
                                  hipStream_t stream);

// y = residual + x * keep / (1 - cut / 2^16); residual may be null.  Types: SPA2_DTYPE_*, out_dtype that of y.
hipError_t launch_dropout(const void* x, int x_dtype, const void* residual, int residual_dtype, int64_t n, uint32_t cut,
                          uint64_t seed, uint64_t offset, const int64_t* seed_offset, void* y, int out_dtype, hipStream_t stream);

}  // namespace spa2
