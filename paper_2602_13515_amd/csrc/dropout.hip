// Dropout of a branch and the sum with the residual stream, y = residual + x keep / (1 - p), and its backward pass, which is
// the same without a residual.  The mask is drawn from a counter-based generator and never stored: the backward pass draws it
// again.
//
// Generator: Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011); key = seed,
// counter = (element / 8, offset), 64 bits each.  Its 128 bits serve 8 elements of 16 bits: element e of the vector has the low
// (e even) or high (e odd) half of word e / 2 and is kept where that number is at least `cut` = round(2^16 p).
// 16 bits an element: p is then a multiple of 2^-16 (and the factor that of the rounded p, so that the expectation is exact),
// and the generator, 20 wide multiplications a draw, costs half of what 32 bits would.
//
// Bound: HBM.  75,600 x 5120 in bf16, forward with a residual 389 us (6.0 TB/s), backward 248 us (6.2 TB/s).
#include "block_ops.h"
#include "spa2_device.h"

namespace spa2 {

__device__ __forceinline__ u32x4 philox(uint64_t index, uint64_t offset, uint64_t seed) {
  uint32_t c0 = (uint32_t)index, c1 = (uint32_t)(index >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0; c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1; c3 = (uint32_t)a;
    k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
  }
  return u32x4{c0, c1, c2, c3};
}

struct DropArgs {
  const void* x; const void* residual; void* y;
  const int64_t* seed_offset;           // device: (seed, offset) instead of the two below, or null
  uint64_t seed, offset;
  int64_t n;
  uint32_t cut;
  float factor;
};

__device__ __forceinline__ void drop_load(const uint16_t* p, float (&x)[8]) {
  const u32x4 v = *(const u32x4*)p;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const uint32_t u = v[c];
    x[2 * c] = __builtin_bit_cast(float, u << 16);
    x[2 * c + 1] = __builtin_bit_cast(float, u & 0xffff0000u);
  }
}
__device__ __forceinline__ void drop_load(const float* p, float (&x)[8]) {
  const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
  for (int c = 0; c < 4; ++c) { x[c] = a[c]; x[4 + c] = b[c]; }
}
__device__ __forceinline__ void drop_store(uint16_t* p, const float (&x)[8]) {
  *(u32x4*)p = u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
}
__device__ __forceinline__ void drop_store(float* p, const float (&x)[8]) {
  *(f32x4*)p = f32x4{x[0], x[1], x[2], x[3]};
  *(f32x4*)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ float drop_one(const uint16_t* p) { return __builtin_bit_cast(float, (uint32_t)*p << 16); }
__device__ __forceinline__ float drop_one(const float* p) { return *p; }
__device__ __forceinline__ void drop_one_store(uint16_t* p, float x) { *p = (uint16_t)pack_bf16(x, x); }
__device__ __forceinline__ void drop_one_store(float* p, float x) { *p = x; }

template <typename X, typename R, bool RES, typename Y>
__global__ __launch_bounds__(256) void dropout_kernel(DropArgs a) {
  uint64_t seed = a.seed, offset = a.offset;
  if (a.seed_offset) { seed = (uint64_t)a.seed_offset[0]; offset = (uint64_t)a.seed_offset[1]; }
  const int64_t vectors = (a.n + 7) / 8;
  for (int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x; v < vectors; v += (int64_t)gridDim.x * 256) {
    const X* x = (const X*)a.x + 8 * v;
    const R* res = (const R*)a.residual + 8 * v;
    Y* y = (Y*)a.y + 8 * v;
    const u32x4 bits = philox((uint64_t)v, offset, seed);
    if (8 * v + 8 <= a.n) {
      float t[8], r[8];
      drop_load(x, t);
      if (RES) drop_load(res, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t word = bits[e >> 1], d = e & 1 ? word >> 16 : word & 0xffffu;
        // (a dropped infinity or NaN leaves the residual as it is)
        const float kept = d >= a.cut ? t[e] : 0.f;
        t[e] = RES ? fmaf(kept, a.factor, r[e]) : kept * a.factor;
      }
      drop_store(y, t);
    } else {
      const int left = (int)(a.n - 8 * v);               // the last vector, 1 to 7 elements
      for (int e = 0; e < left; ++e) {
        const uint32_t word = e < 2 ? bits[0] : e < 4 ? bits[1] : e < 6 ? bits[2] : bits[3], d = e & 1 ? word >> 16 : word & 0xffffu;
        const float kept = d >= a.cut ? drop_one(x + e) : 0.f;
        drop_one_store(y + e, RES ? fmaf(kept, a.factor, drop_one(res + e)) : kept * a.factor);
      }
    }
  }
}

// A vector a thread: the workgroups that run at a time then work on one stretch of memory.  (8192 of them that walk all of it, 2
// GB apart, took 833 instead of 636 us on 75,600 x 5120, both passes.)
constexpr int64_t MAX_WGS = 1 << 23;     // (2^32 threads are more than a launch may have)

hipError_t launch_dropout(const void* x, int x_dtype, const void* residual, int residual_dtype, int64_t n, uint32_t cut,
                          uint64_t seed, uint64_t offset, const int64_t* seed_offset, void* y, int out_dtype, hipStream_t stream) {
  DropArgs a;
  a.x = x; a.residual = residual; a.y = y; a.seed_offset = seed_offset; a.seed = seed; a.offset = offset; a.n = n; a.cut = cut;
  a.factor = cut == 65536u ? 0.f : (float)(65536.0 / (65536.0 - cut));
  const int64_t wgs = ((n + 7) / 8 + 255) / 256;
  const dim3 grid((unsigned)(wgs > MAX_WGS ? MAX_WGS : wgs)), block(256);
  const bool xb = x_dtype == SPA2_DTYPE_BF16, yb = out_dtype == SPA2_DTYPE_BF16, rb = residual_dtype == SPA2_DTYPE_BF16;
  if (!residual) {
    if (xb && yb)       hipLaunchKernelGGL((dropout_kernel<uint16_t, uint16_t, false, uint16_t>), grid, block, 0, stream, a);
    else if (!xb && yb) hipLaunchKernelGGL((dropout_kernel<float, float, false, uint16_t>), grid, block, 0, stream, a);
    else if (!xb)       hipLaunchKernelGGL((dropout_kernel<float, float, false, float>), grid, block, 0, stream, a);
    else                return hipErrorInvalidValue;
  } else if (xb && rb)  hipLaunchKernelGGL((dropout_kernel<uint16_t, uint16_t, true, uint16_t>), grid, block, 0, stream, a);
  else if (xb)          hipLaunchKernelGGL((dropout_kernel<uint16_t, float, true, float>), grid, block, 0, stream, a);
  else                  hipLaunchKernelGGL((dropout_kernel<float, float, true, float>), grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace spa2
