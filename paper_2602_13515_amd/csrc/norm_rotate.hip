// Norm of every head of q and k, and the rotation of its channels by position, in one pass; and its backward pass.
//
//   r = (mean_c x_c^2 + eps)^-1/2      n_c = x_c r w_c      y = R n
//   R turns the pairs (a, b) of the first `rot` channels by their token's angles: (a cos - b sin, b cos + a sin); a pair is
//   (c, c + rot / 2), or (2 c, 2 c + 1) where channels are interleaved.
// Backward, with dn = R^T dy:
//   dw_c = sum over rows of dn_c x_c r      dx = r (g - x r^2 mean_c(g x)),  g = dn w
//
// D / 16 lanes own a row, 16 channels each: two chunks of 8 that hold both halves of 8 pairs, so that a rotation needs no
// exchange between lanes and every access is 16 bytes.  Lanes behind the rotated channels turn theirs by an angle of zero.
// A lane stays with its token and walks over heads: the cosines and sines (4 bytes for each 2-byte channel of a head) are read
// once for all heads of the workgroup and held in registers.
#include "block_ops.h"
#include "spa2_device.h"

namespace spa2 {

struct NormArgs {
  const void* x[2]; const void* dy[2]; void* y[2];     // q and k: input, upstream gradient (backward), result
  const float* w[2];
  int64_t sb[2], sh[2], sn[2], osb[2], osh[2], osn[2];
  int heads[2], per_slice[2], slices_q;                // heads a workgroup walks; blockIdx.y < slices_q: q
  const float* cos; const float* sin; const void* positions;
  int64_t pos_sb;
  int pos_bits, table_rows, rot, B, N, tokens, tiles;  // tokens a workgroup takes at a time; tiles of them in all
  float eps;
  float* part;                                         // backward: [blockIdx.y][blockIdx.x][D] sums of dn x r, or null
};

__device__ __forceinline__ void norm_load(const uint16_t* p, float (&x)[8]) {
  const u32x4 v = *(const u32x4*)p;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const uint32_t u = v[c];
    x[2 * c] = __builtin_bit_cast(float, u << 16);
    x[2 * c + 1] = __builtin_bit_cast(float, u & 0xffff0000u);
  }
}
__device__ __forceinline__ void norm_load(const float* p, float (&x)[8]) {
  const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
  for (int c = 0; c < 4; ++c) { x[c] = a[c]; x[4 + c] = b[c]; }
}
__device__ __forceinline__ void norm_store(uint16_t* p, const float (&x)[8]) {
  *(u32x4*)p = u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
}
__device__ __forceinline__ void norm_store(float* p, const float (&x)[8]) {
  *(f32x4*)p = f32x4{x[0], x[1], x[2], x[3]};
  *(f32x4*)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}

// sum over the LANES lanes that own a row
template <int LANES>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
  for (int s = 1; s < LANES; s <<= 1) x += __shfl_xor(x, s, 64);
  return x;
}

// Both chunks of a lane turned by its angles (BACK: by minus the angles).
template <bool INTERLEAVED, bool BACK>
__device__ __forceinline__ void rotate(float (&a)[8], float (&b)[8], const float (&cs)[8], const float (&sn)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float& p = INTERLEAVED ? (i < 4 ? a[2 * i] : b[2 * i - 8]) : a[i];
    float& q = INTERLEAVED ? (i < 4 ? a[2 * i + 1] : b[2 * i - 7]) : b[i];
    const float s = BACK ? -sn[i] : sn[i], u = p, v = q;
    p = fmaf(u, cs[i], -(v * s));
    q = fmaf(v, cs[i], u * s);
  }
}

template <int D, typename T, bool INTERLEAVED, bool BACKWARD>
__global__ __launch_bounds__(256) void norm_rotate_kernel(NormArgs a) {
  constexpr int LANES = D / 16, GROUPS = 256 / LANES;
  const int tid = threadIdx.x, u = tid % LANES, group = tid / LANES;
  const int z = blockIdx.y >= a.slices_q, slice = blockIdx.y - (z ? a.slices_q : 0);
  const int head0 = slice * a.per_slice[z] + group / a.tokens, head1 = min((slice + 1) * a.per_slice[z], a.heads[z]);
  const int head_step = GROUPS / a.tokens;
  // chunks of this lane, in channels
  const bool turned = u < a.rot / 16;
  const int ca = 8 * (!INTERLEAVED && turned ? u : 2 * u), cb = 8 * (!INTERLEAVED && turned ? u + a.rot / 16 : 2 * u + 1);
  float wa[8], wb[8], sa[8], sb[8];
  if (a.w[z]) {
    norm_load(a.w[z] + ca, wa);
    norm_load(a.w[z] + cb, wb);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) wa[i] = wb[i] = 1.f;
  }
  if (BACKWARD) {
#pragma unroll
    for (int i = 0; i < 8; ++i) sa[i] = sb[i] = 0.f;
  }
  const int64_t all = (int64_t)a.B * a.N;
  for (int tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const int64_t token = (int64_t)tile * a.tokens + group % a.tokens;
    if (token >= all) break;                           // (later tiles are further on still)
    const int b = (int)(token / a.N), n = (int)(token - (int64_t)b * a.N);
    float cs[8], sn[8];
    if (turned) {
      int64_t row = n;
      if (a.pos_bits == 32) row = ((const int32_t*)a.positions)[b * a.pos_sb + n];
      if (a.pos_bits == 64) row = ((const int64_t*)a.positions)[b * a.pos_sb + n];
      row = min(max(row, (int64_t)0), (int64_t)a.table_rows - 1);        // (caller data)
      const int64_t at = row * (a.rot / 2) + 8 * u;
      norm_load(a.cos + at, cs);
      norm_load(a.sin + at, sn);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) { cs[i] = 1.f; sn[i] = 0.f; }
    }
    const T* x0 = (const T*)a.x[z] + b * a.sb[z] + n * a.sn[z];
    const int64_t out0 = b * a.osb[z] + n * a.osn[z];
    for (int h = head0; h < head1; h += head_step) {
      float xa[8], xb[8];
      norm_load(x0 + h * a.sh[z] + ca, xa);
      norm_load(x0 + h * a.sh[z] + cb, xb);
      const int64_t out = out0 + h * a.osh[z];
      float square = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) square = fmaf(xa[i], xa[i], fmaf(xb[i], xb[i], square));
      if constexpr (!BACKWARD) {
        const float r = 1.f / sqrtf(row_sum<LANES>(square) * (1.f / D) + a.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) { xa[i] = xa[i] * r * wa[i]; xb[i] = xb[i] * r * wb[i]; }
        rotate<INTERLEAVED, false>(xa, xb, cs, sn);
        norm_store((uint16_t*)a.y[z] + out + ca, xa);
        norm_store((uint16_t*)a.y[z] + out + cb, xb);
      } else {
        float ga[8], gb[8], inner = 0.f;
        norm_load((const uint16_t*)a.dy[z] + out + ca, ga);
        norm_load((const uint16_t*)a.dy[z] + out + cb, gb);
        rotate<INTERLEAVED, true>(ga, gb, cs, sn);
#pragma unroll
        for (int i = 0; i < 8; ++i) inner = fmaf(ga[i] * wa[i], xa[i], fmaf(gb[i] * wb[i], xb[i], inner));
        const float r = 1.f / sqrtf(row_sum<LANES>(square) * (1.f / D) + a.eps);
        inner = row_sum<LANES>(inner) * r * (1.f / D);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float na = xa[i] * r, nb = xb[i] * r;
          sa[i] = fmaf(ga[i], na, sa[i]);
          sb[i] = fmaf(gb[i], nb, sb[i]);
          xa[i] = r * fmaf(-na, inner, ga[i] * wa[i]);
          xb[i] = r * fmaf(-nb, inner, gb[i] * wb[i]);
        }
        norm_store((T*)a.y[z] + out + ca, xa);
        norm_store((T*)a.y[z] + out + cb, xb);
      }
    }
  }
  if constexpr (BACKWARD) {
    if (!a.part) return;
    // sums of the lanes that hold the same channels: over a wave by exchange, over the waves through LDS
    __shared__ float sums[4][D];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int s = LANES; s < 64; s <<= 1) {
        sa[i] += __shfl_xor(sa[i], s, 64);
        sb[i] += __shfl_xor(sb[i], s, 64);
      }
    }
    if ((tid & 63) < LANES) {
      norm_store(&sums[tid >> 6][ca], sa);
      norm_store(&sums[tid >> 6][cb], sb);
    }
    __syncthreads();
    if (tid < D)
      a.part[((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * D + tid] = (sums[0][tid] + sums[1][tid]) + (sums[2][tid] + sums[3][tid]);
  }
}

// Sums the workgroups' parts in a fixed order: 16 channels a workgroup, 16 lanes a channel.
__global__ __launch_bounds__(256) void norm_weight_finish(const float* part, int D, int rows_q, int rows_k, float* dwq, float* dwk) {
  __shared__ double sums[16][17];
  const int groups = D / 16, z = blockIdx.x >= groups, c = threadIdx.x & 15, l = threadIdx.x >> 4;
  const int channel = (blockIdx.x - (z ? groups : 0)) * 16 + c;
  const float* p = part + (z ? (int64_t)rows_q * D : 0) + channel;
  const int rows = z ? rows_k : rows_q;
  double s = 0.0;
  for (int r = l; r < rows; r += 16 * 8) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p[(int64_t)min(r + 16 * i, rows - 1) * D];
#pragma unroll
    for (int i = 0; i < 8; ++i) s += r + 16 * i < rows ? (double)x[i] : 0.0;
  }
  sums[l][c] = s;
  __syncthreads();
  if (l == 0) {
#pragma unroll
    for (int i = 1; i < 16; ++i) s += sums[i][c];
    float* out = z ? dwk : dwq;
    if (out) out[channel] = (float)s;
  }
}

namespace {

struct NormGrid { int tokens, tiles, x, slices[2], per_slice[2]; };

// Which rows a workgroup takes.
NormGrid norm_grid(const spa2_norm_shape& s, bool backward) {
  NormGrid g;
  const int groups = 256 / (s.d / 16);
  const int64_t all = (int64_t)s.B * s.N;
  g.tokens = groups;
  while (g.tokens > 1 && g.tokens / 2 >= all) g.tokens /= 2;
  g.tiles = (int)((all + g.tokens - 1) / g.tokens);
  const int heads[2] = {s.Hq, s.Hk}, at_once = groups / g.tokens;
  for (int z = 0; z < 2; ++z) {
    // heads of a token in slices where whole tokens would leave compute units idle
    int slices = 1;
    const int most = (heads[z] + at_once - 1) / at_once;
    while (slices < most && (int64_t)g.tiles * slices < 1024) ++slices;
    g.per_slice[z] = (heads[z] + slices - 1) / slices;
    g.slices[z] = (heads[z] + g.per_slice[z] - 1) / g.per_slice[z];
  }
  g.x = g.tiles < 1 << 20 ? g.tiles : 1 << 20;         // (workgroups walk the tiles)
  if (backward) {
    const int most = 2048 / (g.slices[0] + g.slices[1]);
    if (g.x > (most < 1 ? 1 : most)) g.x = most < 1 ? 1 : most;
  }
  return g;
}

NormArgs norm_args(const NormTables& t, const spa2_norm_shape& s, const NormGrid& g, const float* q_weight, const float* k_weight,
                   float eps) {
  NormArgs a = {};
  a.w[0] = q_weight; a.w[1] = k_weight;
  const int64_t in[2][3] = {{s.q_sb, s.q_sh, s.q_sn}, {s.k_sb, s.k_sh, s.k_sn}};
  const int64_t out[2][3] = {{s.qo_sb, s.qo_sh, s.qo_sn}, {s.ko_sb, s.ko_sh, s.ko_sn}};
  for (int z = 0; z < 2; ++z) {
    a.sb[z] = in[z][0]; a.sh[z] = in[z][1]; a.sn[z] = in[z][2];
    a.osb[z] = out[z][0]; a.osh[z] = out[z][1]; a.osn[z] = out[z][2];
    a.heads[z] = z ? s.Hk : s.Hq; a.per_slice[z] = g.per_slice[z];
  }
  a.slices_q = g.slices[0];
  a.cos = t.cos; a.sin = t.sin; a.positions = t.positions;
  a.pos_sb = s.pos_sb; a.pos_bits = s.pos_bits; a.table_rows = s.table_rows; a.rot = s.rot;
  a.B = s.B; a.N = s.N; a.tokens = g.tokens; a.tiles = g.tiles;
  a.eps = eps;
  return a;
}

template <int D, typename T, bool BACKWARD>
void launch_typed(const NormArgs& a, const NormGrid& g, bool interleaved, hipStream_t stream) {
  const dim3 grid((unsigned)g.x, (unsigned)(g.slices[0] + g.slices[1])), block(256);
  if (interleaved) hipLaunchKernelGGL((norm_rotate_kernel<D, T, true, BACKWARD>), grid, block, 0, stream, a);
  else             hipLaunchKernelGGL((norm_rotate_kernel<D, T, false, BACKWARD>), grid, block, 0, stream, a);
}

template <bool BACKWARD>
hipError_t launch_any(const NormArgs& a, const NormGrid& g, const spa2_norm_shape& s, hipStream_t stream) {
  const bool bf16 = s.dtype == SPA2_DTYPE_BF16, il = s.interleaved != 0;
  if (s.d == 128) bf16 ? launch_typed<128, uint16_t, BACKWARD>(a, g, il, stream) : launch_typed<128, float, BACKWARD>(a, g, il, stream);
  else            bf16 ? launch_typed<64, uint16_t, BACKWARD>(a, g, il, stream) : launch_typed<64, float, BACKWARD>(a, g, il, stream);
  return hipGetLastError();
}

}  // namespace

size_t norm_rotate_partials_bytes(const spa2_norm_shape& s) {
  const NormGrid g = norm_grid(s, true);
  return (size_t)g.x * (size_t)(g.slices[0] + g.slices[1]) * (size_t)s.d * sizeof(float);
}

hipError_t launch_norm_rotate(const void* q, const void* k, const float* q_weight, const float* k_weight, const NormTables& t,
                              const spa2_norm_shape& s, float eps, void* q_out, void* k_out, hipStream_t stream) {
  const NormGrid g = norm_grid(s, false);
  NormArgs a = norm_args(t, s, g, q_weight, k_weight, eps);
  a.x[0] = q; a.x[1] = k;
  a.y[0] = q_out; a.y[1] = k_out;
  return launch_any<false>(a, g, s, stream);
}

hipError_t launch_norm_rotate_bwd(const void* q, const void* k, const float* q_weight, const float* k_weight,
                                  const NormTables& t, const void* d_q_out, const void* d_k_out, const spa2_norm_shape& s,
                                  float eps, void* dq, void* dk, float* d_q_weight, float* d_k_weight, void* ws,
                                  hipStream_t stream) {
  const NormGrid g = norm_grid(s, true);
  NormArgs a = norm_args(t, s, g, q_weight, k_weight, eps);
  a.x[0] = q; a.x[1] = k;
  a.dy[0] = d_q_out; a.dy[1] = d_k_out;
  a.y[0] = dq; a.y[1] = dk;
  a.part = d_q_weight || d_k_weight ? (float*)ws : nullptr;
  const hipError_t e = launch_any<true>(a, g, s, stream);
  if (e != hipSuccess || !a.part) return e;
  hipLaunchKernelGGL(norm_weight_finish, dim3((unsigned)(2 * (s.d / 16))), dim3(256), 0, stream, (const float*)ws, s.d,
                     g.x * g.slices[0], g.x * g.slices[1], d_q_weight, d_k_weight);
  return hipGetLastError();
}

}  // namespace spa2
