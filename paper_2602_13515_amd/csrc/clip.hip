// The norm over all gradients of a step, and the gradients scaled to a largest norm.
//
//   norm = (sum over all tensors of x^2)^1/2      out = x min(1, max_norm / (norm + eps))
//
// Two passes, each one launch for every CLIP_TABLE tensors, whose addresses and sizes travel in the launch's arguments (nothing
// is copied to the device, so that a captured call reads nothing of the host's later).  The first leaves a sum for each of its
// workgroups; every workgroup of the second adds up all of these, in the same order, and has the factor without a launch between.
// Squares are taken and summed in fp64, where those of fp32 numbers are exact and do not overflow, in a fixed order.  The second
// pass multiplies in fp64 and rounds once; where the factor is 1 and a result lies where its gradient does, nothing is touched.
#include "spa2_device.h"
#include "step_ops.h"

namespace spa2 {

constexpr int CLIP_TABLE = 120;          // tensors of a launch: their table fills most of the 4 KB that its arguments may have
constexpr int CLIP_CHUNK = 4096;         // elements that a workgroup takes at a time, 16 a thread
constexpr int CLIP_WGS = 2048;           // workgroups at most: all that run at a time

struct ClipItem { const void* x; void* out; int64_t n; };
struct ClipArgs {
  ClipItem item[CLIP_TABLE];
  int32_t first[CLIP_TABLE + 1];         // chunks of the tensors in front of each
  uint8_t types[CLIP_TABLE];             // bit 0: x is fp32, bit 1: out is
  int32_t count;
  double* part;
  int32_t parts;
  float* norm;                           // written by the launch that has it
  double max_norm, eps;
  bool again;                            // not the first launch of its pass: sums are added to those that are there
};
static_assert(sizeof(ClipArgs) <= 4096, "arguments of a launch");

// 16 bytes from any element on
typedef u32x4 __attribute__((aligned(2))) clip_u32x4;
typedef f32x4 __attribute__((aligned(4))) clip_f32x4;

template <bool F32>
__device__ __forceinline__ void clip_load8(const void* p, int64_t at, float (&x)[8]) {
  if constexpr (F32) {
    const f32x4 a = *(const clip_f32x4*)((const float*)p + at), b = *(const clip_f32x4*)((const float*)p + at + 4);
#pragma unroll
    for (int c = 0; c < 4; ++c) { x[c] = a[c]; x[4 + c] = b[c]; }
  } else {
    const u32x4 v = *(const clip_u32x4*)((const uint16_t*)p + at);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint32_t u = v[c];
      x[2 * c] = __builtin_bit_cast(float, u << 16);
      x[2 * c + 1] = __builtin_bit_cast(float, u & 0xffff0000u);
    }
  }
}
template <bool F32>
__device__ __forceinline__ void clip_store8(void* p, int64_t at, const float (&x)[8]) {
  if constexpr (F32) {
    *(clip_f32x4*)((float*)p + at) = f32x4{x[0], x[1], x[2], x[3]};
    *(clip_f32x4*)((float*)p + at + 4) = f32x4{x[4], x[5], x[6], x[7]};
  } else {
    *(clip_u32x4*)((uint16_t*)p + at) = u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
  }
}
template <bool F32>
__device__ __forceinline__ float clip_one(const void* p, int64_t at) {
  if constexpr (F32) return ((const float*)p)[at];
  else               return __builtin_bit_cast(float, (uint32_t)((const uint16_t*)p)[at] << 16);
}
template <bool F32>
__device__ __forceinline__ void clip_put(void* p, int64_t at, float x) {
  if constexpr (F32) ((float*)p)[at] = x;
  else               ((uint16_t*)p)[at] = (uint16_t)pack_bf16(x, x);
}

// sum over the workgroup, in every thread (lds: four numbers)
__device__ __forceinline__ double clip_block_sum(double x, double* lds) {
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) x += __shfl_xor(x, s, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  return ((lds[0] + lds[1]) + lds[2]) + lds[3];
}

template <bool F32>
__device__ __forceinline__ double clip_squares(const ClipItem& t, int64_t base, double sum) {
  const int tid = threadIdx.x;
  float x[2][8];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int64_t at = base + r * (CLIP_CHUNK / 2) + 8 * tid;
    if (at + 8 <= t.n) {
      clip_load8<F32>(t.x, at, x[r]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[r][e] = at + e < t.n ? clip_one<F32>(t.x, at + e) : 0.f;
    }
  }
#pragma unroll
  for (int r = 0; r < 2; ++r)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fma((double)x[r][e], (double)x[r][e], sum);
  return sum;
}

__global__ __launch_bounds__(256) void clip_norm_kernel(ClipArgs a) {
  __shared__ double lds[4];
  double sum = 0.0;
  int t = 0;
  for (int c = blockIdx.x; c < a.first[a.count]; c += gridDim.x) {
    while (c >= a.first[t + 1]) ++t;
    const ClipItem item = a.item[t];
    const int64_t base = (int64_t)(c - a.first[t]) * CLIP_CHUNK;
    sum = a.types[t] & 1 ? clip_squares<true>(item, base, sum) : clip_squares<false>(item, base, sum);
  }
  sum = clip_block_sum(sum, lds);
  if (threadIdx.x == 0) a.part[blockIdx.x] = a.again ? a.part[blockIdx.x] + sum : sum;
}

template <bool F32, bool OUT32>
__device__ __forceinline__ void clip_chunk(const ClipItem& t, int64_t base, double factor) {
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int64_t at = base + r * (CLIP_CHUNK / 2) + 8 * threadIdx.x;
    if (at + 8 <= t.n) {
      float x[8];
      clip_load8<F32>(t.x, at, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = (float)((double)x[e] * factor);
      clip_store8<OUT32>(t.out, at, x);
    } else {
      for (int e = 0; e < 8 && at + e < t.n; ++e)
        clip_put<OUT32>(t.out, at + e, (float)((double)clip_one<F32>(t.x, at + e) * factor));
    }
  }
}

__global__ __launch_bounds__(256) void clip_scale_kernel(ClipArgs a) {
  __shared__ double lds[4];
  double sum = 0.0;
  for (int p = threadIdx.x; p < a.parts; p += 256) sum += a.part[p];
  const double norm = sqrt(clip_block_sum(sum, lds)), size = norm + a.eps;
  if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
  // (a NaN stays one; no limit leaves everything as it is)
  double factor = 1.0;
  if (a.max_norm < (double)INFINITY && size != 0.0) factor = a.max_norm / size;
  if (factor >= 1.0) factor = 1.0;
  int t = 0;
  for (int c = blockIdx.x; c < a.first[a.count]; c += gridDim.x) {
    while (c >= a.first[t + 1]) ++t;
    const ClipItem item = a.item[t];
    if (factor == 1.0 && item.out == item.x) continue;
    const int64_t base = (int64_t)(c - a.first[t]) * CLIP_CHUNK;
    switch (a.types[t]) {
      case 0: clip_chunk<false, false>(item, base, factor); break;
      case 1: clip_chunk<true, false>(item, base, factor); break;
      case 2: clip_chunk<false, true>(item, base, factor); break;
      default: clip_chunk<true, true>(item, base, factor); break;
    }
  }
}

size_t clip_partials_bytes() { return CLIP_WGS * sizeof(double); }

hipError_t launch_clip(const spa2_gradient* gradients, int count, double max_norm, double eps, float* norm, void* ws,
                       hipStream_t stream) {
  ClipArgs a;
  a.part = (double*)ws;
  a.max_norm = max_norm; a.eps = eps;
  auto chunks_of = [](int64_t n) { return (int)((n + CLIP_CHUNK - 1) / CLIP_CHUNK); };
  // the next table from gradient g on; whether it is for the second pass (only what has a result)
  auto fill = [&](int& g, bool scale) {
    a.count = 0;
    a.first[0] = 0;
    for (; g < count && a.count < CLIP_TABLE; ++g) {
      const spa2_gradient& x = gradients[g];
      if (x.n == 0 || (scale && !x.out)) continue;
      a.item[a.count] = {x.x, x.out, x.n};
      a.types[a.count] = (uint8_t)((x.dtype == SPA2_DTYPE_F32) | (x.out_dtype == SPA2_DTYPE_F32) << 1);
      a.first[a.count + 1] = a.first[a.count] + chunks_of(x.n);
      ++a.count;
    }
  };
  a.parts = 1;
  for (int g = 0; g < count;) {
    fill(g, false);
    const int chunks = a.first[a.count];
    a.parts = a.parts > chunks ? a.parts : chunks < CLIP_WGS ? chunks : CLIP_WGS;
  }
  a.norm = nullptr;
  a.again = false;
  for (int g = 0; g < count;) {            // (every launch has all workgroups: each sum is written by the first one)
    fill(g, false);
    hipLaunchKernelGGL(clip_norm_kernel, dim3((unsigned)a.parts), dim3(256), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.again = true;
  }
  a.norm = norm;
  for (int g = 0; g < count;) {
    fill(g, true);
    const int chunks = a.first[a.count];
    if (!chunks && !a.norm) continue;
    hipLaunchKernelGGL(clip_scale_kernel, dim3((unsigned)(chunks < 1 ? 1 : chunks < CLIP_WGS ? chunks : CLIP_WGS)), dim3(256), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.norm = nullptr;
  }
  return hipSuccess;
}

}  // namespace spa2
