// Device parts that the forward and the backward pass of the gated sum with its norms share.
#pragma once
#include "spa2_device.h"
#include "step_ops.h"

namespace spa2 {

// A row's channels: thread t of a workgroup of `threads` owns chunks of eight, t, t + threads, ... (GATE_CHUNKS of them).
constexpr int GATE_WAVES = 8;                          // of a workgroup, at most

struct GateArgs {
  const void* x; const void* branch; const void* y_in; const void* dy; const void* dn;      // (y_in, dy, dn: backward)
  void* y; void* n; float* stats;                      // stats: [3][rows] mean and 1 / deviation of y, 1 / size of the branch
  void* dx; void* dbranch; float* part;                // part: [workgroup][3][width] sums over its rows
  spa2_gate_params p;
  int64_t gate_sb, scale_sb, shift_sb;
  int64_t tokens, rows;                                // of a sample, of all
  int width, per_sample, kind;                         // workgroups of a sample
  bool params32, post;
  float eps;
};

// 16 bytes from any element on: rows of odd width start anywhere
typedef u32x4 __attribute__((aligned(2))) gate_u32x4;
typedef f32x4 __attribute__((aligned(4))) gate_f32x4;

// left: channels from here to the row's end (ODD: fewer than eight maybe; the others are zero)
template <bool ODD>
__device__ __forceinline__ void gate_load(const uint16_t* p, int left, float (&x)[8]) {
  if (!ODD || left >= 8) {
    const u32x4 v = *(const gate_u32x4*)p;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint32_t u = v[c];
      x[2 * c] = __builtin_bit_cast(float, u << 16);
      x[2 * c + 1] = __builtin_bit_cast(float, u & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < left ? __builtin_bit_cast(float, (uint32_t)p[e] << 16) : 0.f;
  }
}
template <bool ODD>
__device__ __forceinline__ void gate_load(const float* p, int left, float (&x)[8]) {
  if (!ODD || left >= 8) {
    const f32x4 a = *(const gate_f32x4*)p, b = *(const gate_f32x4*)(p + 4);
#pragma unroll
    for (int c = 0; c < 4; ++c) { x[c] = a[c]; x[4 + c] = b[c]; }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < left ? p[e] : 0.f;
  }
}
template <bool ODD>
__device__ __forceinline__ void gate_store(uint16_t* p, int left, const float (&x)[8]) {
  const u32x4 v = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
  if (!ODD || left >= 8) {
    *(gate_u32x4*)p = v;
  } else {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < left) p[e] = (uint16_t)(e & 1 ? v[e / 2] >> 16 : v[e / 2]);
  }
}
template <bool ODD>
__device__ __forceinline__ void gate_store(float* p, int left, const float (&x)[8]) {
  if (!ODD || left >= 8) {
    *(gate_f32x4*)p = f32x4{x[0], x[1], x[2], x[3]};
    *(gate_f32x4*)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
  } else {
#pragma unroll
    for (int e = 0; e < 7; ++e)
      if (e < left) p[e] = x[e];
  }
}
// eight parameters, or `otherwise`
template <bool ODD>
__device__ __forceinline__ void gate_param(const void* p, bool fp32, int64_t at, int left, float otherwise, float (&x)[8]) {
  if (!p) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = otherwise;
  } else if (fp32) {
    gate_load<ODD>((const float*)p + at, left, x);
  } else {
    gate_load<ODD>((const uint16_t*)p + at, left, x);
  }
}
__device__ __forceinline__ float gate_one(const void* p, bool fp32, int64_t at, float otherwise) {
  if (!p) return otherwise;
  return fp32 ? ((const float*)p)[at] : __builtin_bit_cast(float, (uint32_t)((const uint16_t*)p)[at] << 16);
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) x += __shfl_xor(x, s, 64);
  return x;
}
// Sums over the workgroup of two numbers that every lane of a wave has, in every thread.  lds: one of two arrays in turn (a wave may
// still read the one before, none the one before that), so that one barrier is enough.
struct GatePair { float a, b; };
__device__ __forceinline__ GatePair block_sum(GatePair x, float (&lds)[GATE_WAVES][2], int waves, int w, int lane) {
  if (waves == 1) return x;
  if (lane == 0) { lds[w][0] = x.a; lds[w][1] = x.b; }
  __syncthreads();
  GatePair r = {lds[0][0], lds[0][1]};
  for (int i = 1; i < waves; ++i) { r.a += lds[i][0]; r.b += lds[i][1]; }
  return r;
}

}  // namespace spa2
