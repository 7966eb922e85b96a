// A branch, normed and gated, added to the residual stream, and the norm of the sum, modulated: what stands between two branches of
// a transformer block, in one pass.
//
//   u = b (mean b^2 + eps)^-1/2 w_b   (u = b without w_b)        y = x + gate u, rounded to x's type
//   h = (y - mean y) (var y + eps)^-1/2   (RMS: no mean)          n = (h w + c) (1 + scale) + shift, rounded once
//
// The norm is that of y as it is stored, which is also what the backward pass reads.  A workgroup takes rows of one sample, whose
// parameters it holds in registers, combined to three factors a channel: gate w_b, w (1 + scale), c (1 + scale) + shift.  The
// deviation is taken about each wave's own mean and the waves' are joined (no difference of large sums), with one barrier a row.
// Bound: HBM.
#include "gate_norm.h"

namespace spa2 {

template <typename X, typename B, typename N, int CHUNKS, bool ODD>
__global__ __launch_bounds__(64 * GATE_WAVES) void gate_norm_kernel(GateArgs a) {
  __shared__ float lds[2][GATE_WAVES][2];
  const int threads = blockDim.x, waves = threads / 64, t = threadIdx.x, lane = t & 63;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int64_t b = blockIdx.x / a.per_sample, first = blockIdx.x % a.per_sample;
  float gate[CHUNKS][8], mul[CHUNKS][8], add[CHUNKS][8];
  float own = 0.f;                                     // channels of this wave
#pragma unroll
  for (int k = 0; k < CHUNKS; ++k) {
    const int at = 8 * (t + threads * k), left = a.width - at;
    own += (float)min(max(a.width - 8 * (64 * w + threads * k), 0), 512);
    if (left <= 0) continue;
    float s[8], c[8];
    gate_param<ODD>(a.p.gate, a.params32, b * a.gate_sb + at, left, 1.f, gate[k]);
    gate_param<ODD>(a.p.branch_weight, a.params32, at, left, 1.f, s);
#pragma unroll
    for (int e = 0; e < 8; ++e) gate[k][e] *= s[e];
    gate_param<ODD>(a.p.weight, a.params32, at, left, 1.f, mul[k]);
    gate_param<ODD>(a.p.bias, a.params32, at, left, 0.f, c);
    gate_param<ODD>(a.p.scale, a.params32, b * a.scale_sb + at, left, 0.f, s);
    gate_param<ODD>(a.p.shift, a.params32, b * a.shift_sb + at, left, 0.f, add[k]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      mul[k][e] *= 1.f + s[e];
      add[k][e] = fmaf(c[e], 1.f + s[e], add[k][e]);
    }
  }
  const float per = 1.f / (float)a.width;
  int turn = 0;
  auto buffer = [&]() -> float (&)[GATE_WAVES][2] {
    turn ^= 1;
    return lds[turn];
  };
  for (int64_t token = first; token < a.tokens; token += a.per_sample) {
    const int64_t row = b * a.tokens + token, base = row * a.width;
    float y[CHUNKS][8], u[CHUNKS][8];
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
      const int at = 8 * (t + threads * k), left = a.width - at;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[k][e] = u[k][e] = 0.f;
      if (left <= 0) continue;
      gate_load<ODD>((const X*)a.x + base + at, left, y[k]);
      if (a.branch) gate_load<ODD>((const B*)a.branch + base + at, left, u[k]);
    }
    if (a.branch) {
      float rb = 1.f;
      if (a.post) {
        float sq = 0.f;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e) sq = fmaf(u[k][e], u[k][e], sq);
        sq = block_sum({wave_sum(sq), 0.f}, buffer(), waves, w, lane).a;
        rb = rsqrtf(fmaf(sq, per, a.eps));
        if (a.stats && t == 0) a.stats[2 * a.rows + row] = rb;
      }
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k) {
        const int at = 8 * (t + threads * k), left = a.width - at;
        if (left <= 0) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[k][e] = fmaf(u[k][e] * rb, gate[k][e], y[k][e]);
        gate_store<ODD>((X*)a.y + base + at, left, y[k]);
        if constexpr (sizeof(X) == 2) {
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const uint32_t p = pack_bf16(y[k][e], y[k][e + 1]);
            y[k][e] = __builtin_bit_cast(float, p << 16);
            y[k][e + 1] = __builtin_bit_cast(float, p & 0xffff0000u);
          }
        }
        if constexpr (ODD) {
#pragma unroll
          for (int e = 0; e < 8; ++e) y[k][e] = e < left ? y[k][e] : 0.f;
        }
      }
    }
    if (a.kind == SPA2_NORM_NONE) continue;
    float mean = 0.f, r;
    if (a.kind == SPA2_NORM_LAYER) {
      float s = 0.f, dev = 0.f;
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += y[k][e];
      s = wave_sum(s);
      const float here = s / own;
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k) {
        const int left = a.width - 8 * (t + threads * k);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float d = y[k][e] - here;
          dev = left > (ODD ? e : 0) ? fmaf(d, d, dev) : dev;
        }
      }
      dev = wave_sum(dev);
      if (waves == 1) {
        mean = here;
      } else {
        float (&x)[GATE_WAVES][2] = buffer();
        if (lane == 0) { x[w][0] = s; x[w][1] = dev; }
        __syncthreads();
        for (int i = 0; i < waves; ++i) mean += x[i][0];
        mean *= per;
        dev = 0.f;
        for (int i = 0; i < waves; ++i) {
          float n = 0.f;                               // channels of wave i
#pragma unroll
          for (int k = 0; k < CHUNKS; ++k) n += (float)min(max(a.width - 8 * (64 * i + threads * k), 0), 512);
          const float off = x[i][0] / n - mean;
          dev += fmaf(n * off, off, x[i][1]);
        }
      }
      r = rsqrtf(fmaf(dev, per, a.eps));
    } else {
      float sq = 0.f;
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) sq = fmaf(y[k][e], y[k][e], sq);
      sq = block_sum({wave_sum(sq), 0.f}, buffer(), waves, w, lane).a;
      r = rsqrtf(fmaf(sq, per, a.eps));
    }
    if (a.stats && t == 0) { a.stats[row] = mean; a.stats[a.rows + row] = r; }
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
      const int at = 8 * (t + threads * k), left = a.width - at;
      if (left <= 0) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[k][e] = fmaf((y[k][e] - mean) * r, mul[k][e], add[k][e]);
      gate_store<ODD>((N*)a.n + base + at, left, y[k]);
    }
  }
}

// Workgroups: as many as run at a time (16 waves a compute unit), each with the rows p, p + per_sample, ... of a sample, so that
// those that run at a time work on one stretch of memory.
constexpr int GATE_FWD_WAVES = 16, GATE_BWD_WAVES = 12, CUS = 256;
static int gate_chunks(int width) { return width <= 512 * 2 * GATE_WAVES ? 2 : 4; }
int gate_threads(int width) { const int each = 512 * gate_chunks(width); return 64 * ((width + each - 1) / each); }
int gate_per_sample(const spa2_gate_shape& s, bool backward) {
  const int64_t wgs = CUS * (backward ? GATE_BWD_WAVES : GATE_FWD_WAVES) / (gate_threads(s.width) / 64);
  int64_t per = (wgs + s.samples - 1) / s.samples;
  return (int)(per < s.tokens ? per : s.tokens);
}

GateArgs gate_args(const spa2_gate_shape& s, const spa2_gate_params& p, float eps, bool backward) {
  GateArgs a = {};
  a.p = p;
  a.gate_sb = s.gate_sb; a.scale_sb = s.scale_sb; a.shift_sb = s.shift_sb;
  a.tokens = s.tokens; a.rows = s.samples * s.tokens;
  a.width = s.width; a.kind = s.kind; a.params32 = s.param_dtype == SPA2_DTYPE_F32; a.post = s.post != 0;
  a.eps = eps;
  a.per_sample = gate_per_sample(s, backward);
  return a;
}

template <typename X, typename B, typename N>
static void launch_types(const GateArgs& a, const dim3& grid, const dim3& block, hipStream_t stream) {
  const bool odd = a.width % 8, wide = gate_chunks(a.width) == 4;
  if (wide && odd)      hipLaunchKernelGGL((gate_norm_kernel<X, B, N, 4, true>), grid, block, 0, stream, a);
  else if (wide)        hipLaunchKernelGGL((gate_norm_kernel<X, B, N, 4, false>), grid, block, 0, stream, a);
  else if (odd)         hipLaunchKernelGGL((gate_norm_kernel<X, B, N, 2, true>), grid, block, 0, stream, a);
  else                  hipLaunchKernelGGL((gate_norm_kernel<X, B, N, 2, false>), grid, block, 0, stream, a);
}

hipError_t launch_gate_norm(const void* x, const void* branch, const spa2_gate_params& p, const spa2_gate_shape& s, float eps,
                            void* y, void* n, float* stats, hipStream_t stream) {
  GateArgs a = gate_args(s, p, eps, false);
  a.x = x; a.branch = branch; a.y = y; a.n = n; a.stats = stats;
  const dim3 grid((unsigned)(a.per_sample * s.samples)), block((unsigned)gate_threads(s.width));
  const bool x32 = s.x_dtype == SPA2_DTYPE_F32, b32 = s.branch_dtype == SPA2_DTYPE_F32, n32 = s.out_dtype == SPA2_DTYPE_F32;
  if (!x32)             launch_types<uint16_t, uint16_t, uint16_t>(a, grid, block, stream);
  else if (b32 && n32)  launch_types<float, float, float>(a, grid, block, stream);
  else if (b32)         launch_types<float, float, uint16_t>(a, grid, block, stream);
  else if (n32)         launch_types<float, uint16_t, float>(a, grid, block, stream);
  else                  launch_types<float, uint16_t, uint16_t>(a, grid, block, stream);
  return hipGetLastError();
}

}  // namespace spa2
