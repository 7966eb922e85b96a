// Backward pass of the gated sum with its norms (formulas of the forward pass: gate_norm.hip).  With the upstream gradients dy and dn
// of the sum and of its norm, a = w (1 + scale), h and r the normed sum and 1 / deviation, u the normed branch and rb 1 / its size:
//
//   g = dn a      D = dy + r (g - mean g - h mean (g h))   (RMS: without mean g)
//   dx = D        du = D gate w_b      db = rb (du - u mean (du u))   (db = D gate without w_b)
//   S1 = sum dn h    S2 = sum dn    T = sum D u     over the tokens of each sample, a channel each, and from these
//   dscale = w S1 + c S2    dshift = S2    dgate = w_b T    dw = sum (1 + scale) S1    dc = sum (1 + scale) S2    dw_b = sum gate T
//
// h and u are made again from y and the branch and the statistics that the forward pass leaves.  A workgroup takes rows of one
// sample and keeps the three sums of its channels in registers; they are joined by a launch behind, in fp64 and a fixed order, and
// those of all samples by another one where a parameter is shared and there are several.
// Bound: HBM.
#include "gate_norm.h"

namespace spa2 {

int gate_threads(int width);
GateArgs gate_args(const spa2_gate_shape& s, const spa2_gate_params& p, float eps, bool backward);

template <typename X, typename B, typename N, int CHUNKS, bool ODD>
__global__ __launch_bounds__(64 * GATE_WAVES) void gate_norm_bwd_kernel(GateArgs a) {
  __shared__ float lds[2][GATE_WAVES][2];
  const int threads = blockDim.x, waves = threads / 64, t = threadIdx.x, lane = t & 63;
  const int w = __builtin_amdgcn_readfirstlane(t >> 6);
  const int64_t b = blockIdx.x / a.per_sample, first = blockIdx.x % a.per_sample;
  const bool normed = a.kind != SPA2_NORM_NONE, layer = a.kind == SPA2_NORM_LAYER;
  float gate[CHUNKS][8], mul[CHUNKS][8], s1[CHUNKS][8], s2[CHUNKS][8], sg[CHUNKS][8];
#pragma unroll
  for (int k = 0; k < CHUNKS; ++k) {
    const int at = 8 * (t + threads * k), left = a.width - at;
#pragma unroll
    for (int e = 0; e < 8; ++e) s1[k][e] = s2[k][e] = sg[k][e] = 0.f;
    if (left <= 0) continue;
    float s[8];
    gate_param<ODD>(a.p.gate, a.params32, b * a.gate_sb + at, left, 1.f, gate[k]);
    gate_param<ODD>(a.p.branch_weight, a.params32, at, left, 1.f, s);
#pragma unroll
    for (int e = 0; e < 8; ++e) gate[k][e] *= s[e];
    gate_param<ODD>(a.p.weight, a.params32, at, left, 1.f, mul[k]);
    gate_param<ODD>(a.p.scale, a.params32, b * a.scale_sb + at, left, 0.f, s);
#pragma unroll
    for (int e = 0; e < 8; ++e) mul[k][e] *= 1.f + s[e];
  }
  const float per = 1.f / (float)a.width;
  int turn = 0;
  auto buffer = [&]() -> float (&)[GATE_WAVES][2] {
    turn ^= 1;
    return lds[turn];
  };
  for (int64_t token = first; token < a.tokens; token += a.per_sample) {
    const int64_t row = b * a.tokens + token, base = row * a.width;
    // d: dy, then D;  h: y, then the normed sum;  g: dn, then dn a;  u: the branch, normed
    float d[CHUNKS][8], h[CHUNKS][8], g[CHUNKS][8], u[CHUNKS][8];
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
      const int at = 8 * (t + threads * k), left = a.width - at;
#pragma unroll
      for (int e = 0; e < 8; ++e) d[k][e] = h[k][e] = g[k][e] = u[k][e] = 0.f;
      if (left <= 0) continue;
      if (normed) {
        gate_load<ODD>((const N*)a.dn + base + at, left, g[k]);
        gate_load<ODD>((const X*)a.y_in + base + at, left, h[k]);
      }
      if (a.dy) gate_load<ODD>((const X*)a.dy + base + at, left, d[k]);
      if (a.branch) gate_load<ODD>((const B*)a.branch + base + at, left, u[k]);
    }
    if (normed) {
      const float mean = a.stats[row], r = a.stats[a.rows + row];
      float sum = 0.f, along = 0.f;
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k) {
        if (a.width - 8 * (t + threads * k) <= 0) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          h[k][e] = (h[k][e] - mean) * r;              // (behind the row's end: times a g of zero)
          s1[k][e] = fmaf(g[k][e], h[k][e], s1[k][e]);
          s2[k][e] += g[k][e];
          g[k][e] *= mul[k][e];
          sum += g[k][e];
          along = fmaf(g[k][e], h[k][e], along);
        }
      }
      const GatePair all = block_sum({layer ? wave_sum(sum) : 0.f, wave_sum(along)}, buffer(), waves, w, lane);
      const float m = all.a * per, c = all.b * per;
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) d[k][e] = fmaf(r, fmaf(-h[k][e], c, g[k][e] - m), d[k][e]);
    }
    if (a.dx) {
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k) {
        const int at = 8 * (t + threads * k), left = a.width - at;
        if (left > 0) gate_store<ODD>((X*)a.dx + base + at, left, d[k]);
      }
    }
    if (!a.branch) continue;
    float rb = 1.f, c = 0.f;
    if (a.post) {
      rb = a.stats[2 * a.rows + row];
      float along = 0.f;
#pragma unroll
      for (int k = 0; k < CHUNKS; ++k) {
        if (a.width - 8 * (t + threads * k) <= 0) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[k][e] *= rb;
          along = fmaf(d[k][e] * gate[k][e], u[k][e], along);
        }
      }
      c = block_sum({wave_sum(along), 0.f}, buffer(), waves, w, lane).a * per;
    }
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
      const int at = 8 * (t + threads * k), left = a.width - at;
      if (left <= 0) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sg[k][e] = fmaf(d[k][e], u[k][e], sg[k][e]);
        d[k][e] = a.post ? rb * fmaf(-u[k][e], c, d[k][e] * gate[k][e]) : d[k][e] * gate[k][e];
      }
      if (a.dbranch) gate_store<ODD>((B*)a.dbranch + base + at, left, d[k]);
    }
  }
  if (!a.part) return;
  float* part = a.part + (int64_t)blockIdx.x * 3 * a.width;
#pragma unroll
  for (int k = 0; k < CHUNKS; ++k) {
    const int at = 8 * (t + threads * k), left = a.width - at;
    if (left <= 0) continue;
    if (normed) {
      gate_store<ODD>(part + at, left, s1[k]);
      gate_store<ODD>(part + a.width + at, left, s2[k]);
    }
    if (a.branch) gate_store<ODD>(part + 2 * (int64_t)a.width + at, left, sg[k]);
  }
}

// ------------------------------------------------------------------ gradients of the parameters
struct GateSums {
  float* part;                           // [samples][per_sample][3][width]
  spa2_gate_params p;
  spa2_gate_grads d;
  int64_t gate_sb, scale_sb, shift_sb;
  int samples, per_sample, width, columns;               // columns: workgroups that share a sample's channels
  bool params32, normed, branch;
};
constexpr int SUM_GROUPS = 16;           // a workgroup: 64 channels, the summands in 16 groups

__device__ __forceinline__ void grad_put(const GateSums& a, void* p, int64_t at, double x) {
  if (!p) return;
  if (a.params32) ((float*)p)[at] = (float)x;
  else            ((uint16_t*)p)[at] = (uint16_t)pack_bf16((float)x, 0.f);
}

// Sums of a sample's workgroups; parameters of its own.  With one sample all gradients are written here, with several the sums
// take the place of the first workgroup's.
__global__ __launch_bounds__(64 * SUM_GROUPS) void gate_sums_kernel(GateSums a) {
  __shared__ double lds[3][SUM_GROUPS][64];
  const int lane = threadIdx.x & 63, g = threadIdx.x >> 6, b = blockIdx.x / a.columns, c = blockIdx.x % a.columns * 64 + lane;
  double s[3] = {0.0, 0.0, 0.0};
  float* part = a.part + (int64_t)b * a.per_sample * 3 * a.width + c;
  if (c < a.width) {
    for (int p = g; p < a.per_sample; p += 4 * SUM_GROUPS) {         // four in flight
      float x[4][3];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float* q = part + (int64_t)min(p + u * SUM_GROUPS, a.per_sample - 1) * 3 * a.width;
        x[u][0] = a.normed ? q[0] : 0.f;
        x[u][1] = a.normed ? q[a.width] : 0.f;
        x[u][2] = a.branch ? q[2 * (int64_t)a.width] : 0.f;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < 3; ++i) s[i] += p + u * SUM_GROUPS < a.per_sample ? (double)x[u][i] : 0.0;
    }
  }
#pragma unroll
  for (int i = 0; i < 3; ++i) lds[i][g][lane] = s[i];
  __syncthreads();
  if (g || c >= a.width) return;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    s[i] = 0.0;
    for (int k = 0; k < SUM_GROUPS; ++k) s[i] += lds[i][k][lane];
  }
  const double weight = gate_one(a.p.weight, a.params32, c, 1.f), bias = gate_one(a.p.bias, a.params32, c, 0.f);
  const double post = gate_one(a.p.branch_weight, a.params32, c, 1.f), gate = gate_one(a.p.gate, a.params32, b * a.gate_sb + c, 1.f);
  const double scale = 1.0 + gate_one(a.p.scale, a.params32, b * a.scale_sb + c, 0.f);
  const bool one = a.samples == 1;
  if (one || a.gate_sb) grad_put(a, a.d.gate, b * a.gate_sb + c, post * s[2]);
  if (one || a.scale_sb) grad_put(a, a.d.scale, b * a.scale_sb + c, weight * s[0] + bias * s[1]);
  if (one || a.shift_sb) grad_put(a, a.d.shift, b * a.shift_sb + c, s[1]);
  if (one) {
    grad_put(a, a.d.weight, c, scale * s[0]);
    grad_put(a, a.d.bias, c, scale * s[1]);
    grad_put(a, a.d.branch_weight, c, gate * s[2]);
    return;
  }
  part[0] = (float)s[0];
  part[a.width] = (float)s[1];
  part[2 * (int64_t)a.width] = (float)s[2];
}

// Gradients of what all samples share: sums over the samples.
__global__ __launch_bounds__(64 * SUM_GROUPS) void gate_shared_kernel(GateSums a) {
  __shared__ double lds[6][SUM_GROUPS][64];
  const int lane = threadIdx.x & 63, g = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  double s[6] = {0.0, 0.0, 0.0, 0.0, 0.0, 0.0};
  if (c < a.width) {
    const double weight = gate_one(a.p.weight, a.params32, c, 1.f), bias = gate_one(a.p.bias, a.params32, c, 0.f);
    const double post = gate_one(a.p.branch_weight, a.params32, c, 1.f);
#pragma unroll 1
    for (int64_t b = g; b < a.samples; b += SUM_GROUPS) {
      const float* q = a.part + b * a.per_sample * 3 * a.width + c;
      const double gate = gate_one(a.p.gate, a.params32, b * a.gate_sb + c, 1.f);
      const double scale = 1.0 + gate_one(a.p.scale, a.params32, b * a.scale_sb + c, 0.f);
      const double x = q[0], y = q[a.width], z = q[2 * (int64_t)a.width];
      s[0] += scale * x;
      s[1] += scale * y;
      s[2] += gate * z;
      s[3] += post * z;
      s[4] += weight * x + bias * y;
      s[5] += y;
    }
  }
#pragma unroll
  for (int i = 0; i < 6; ++i) lds[i][g][lane] = s[i];
  __syncthreads();
  if (g || c >= a.width) return;
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    s[i] = 0.0;
    for (int k = 0; k < SUM_GROUPS; ++k) s[i] += lds[i][k][lane];
  }
  grad_put(a, a.d.weight, c, s[0]);
  grad_put(a, a.d.bias, c, s[1]);
  grad_put(a, a.d.branch_weight, c, s[2]);
  if (!a.gate_sb) grad_put(a, a.d.gate, c, s[3]);
  if (!a.scale_sb) grad_put(a, a.d.scale, c, s[4]);
  if (!a.shift_sb) grad_put(a, a.d.shift, c, s[5]);
}

template <typename X, typename B, typename N>
static void launch_types(const GateArgs& a, const dim3& grid, const dim3& block, hipStream_t stream) {
  const bool odd = a.width % 8, wide = a.width > 512 * 2 * GATE_WAVES;
  if (wide && odd)      hipLaunchKernelGGL((gate_norm_bwd_kernel<X, B, N, 4, true>), grid, block, 0, stream, a);
  else if (wide)        hipLaunchKernelGGL((gate_norm_bwd_kernel<X, B, N, 4, false>), grid, block, 0, stream, a);
  else if (odd)         hipLaunchKernelGGL((gate_norm_bwd_kernel<X, B, N, 2, true>), grid, block, 0, stream, a);
  else                  hipLaunchKernelGGL((gate_norm_bwd_kernel<X, B, N, 2, false>), grid, block, 0, stream, a);
}

size_t gate_partials_bytes(const spa2_gate_shape& s) {
  return (size_t)s.samples * gate_per_sample(s, true) * 3 * (size_t)s.width * sizeof(float);
}

hipError_t launch_gate_norm_bwd(const void* branch, const spa2_gate_params& p, const spa2_gate_shape& s, float eps, const void* y,
                                const void* dy, const void* dn, const float* stats, void* dx, void* dbranch,
                                const spa2_gate_grads& grads, void* ws, hipStream_t stream) {
  GateArgs a = gate_args(s, p, eps, true);
  a.branch = branch; a.y_in = y; a.dy = dy; a.dn = dn; a.stats = (float*)stats; a.dx = dx; a.dbranch = dbranch;
  const bool any = grads.gate || grads.branch_weight || grads.weight || grads.bias || grads.scale || grads.shift;
  a.part = any ? (float*)ws : nullptr;
  const dim3 grid((unsigned)(a.per_sample * s.samples)), block((unsigned)gate_threads(s.width));
  const bool x32 = s.x_dtype == SPA2_DTYPE_F32, b32 = s.branch_dtype == SPA2_DTYPE_F32, n32 = s.out_dtype == SPA2_DTYPE_F32;
  if (!x32)             launch_types<uint16_t, uint16_t, uint16_t>(a, grid, block, stream);
  else if (b32 && n32)  launch_types<float, float, float>(a, grid, block, stream);
  else if (b32)         launch_types<float, float, uint16_t>(a, grid, block, stream);
  else if (n32)         launch_types<float, uint16_t, float>(a, grid, block, stream);
  else                  launch_types<float, uint16_t, uint16_t>(a, grid, block, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !any) return e;
  const int columns = (s.width + 63) / 64;
  GateSums q = {a.part, p, grads, s.gate_sb, s.scale_sb, s.shift_sb, (int)s.samples, a.per_sample, s.width, columns, a.params32,
                s.kind != SPA2_NORM_NONE, branch != nullptr};
  hipLaunchKernelGGL(gate_sums_kernel, dim3((unsigned)(columns * s.samples)), dim3(64 * SUM_GROUPS), 0, stream, q);
  e = hipGetLastError();
  const bool shared = grads.weight || grads.bias || grads.branch_weight || (grads.gate && !s.gate_sb) || (grads.scale && !s.scale_sb) ||
                      (grads.shift && !s.shift_sb);
  if (e != hipSuccess || s.samples == 1 || !shared) return e;
  hipLaunchKernelGGL(gate_shared_kernel, dim3((unsigned)columns), dim3(64 * SUM_GROUPS), 0, stream, q);
  return hipGetLastError();
}

}  // namespace spa2
