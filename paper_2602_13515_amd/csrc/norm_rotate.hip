// Norm of every head of q and k, and the rotation of its channels by position, in one pass; and its backward pass.
//
//   r = (mean_c x_c^2 + eps)^-1/2      n_c = x_c r w_c      y = R n
//   R turns the pairs (a, b) of the first `rot` channels by their token's angles: (a cos - b sin, b cos + a sin); a pair is
//   (c, c + rot / 2), or (2 c, 2 c + 1) where channels are interleaved.
// Backward, with dn = R^T dy:
//   dw_c = sum over rows of dn_c x_c r      dx = r (g - x r^2 mean_c(g x)),  g = dn w
//
// A lane owns two vectors of V channels of a row, which lie next to those of the neighbouring lanes and hold both halves of the
// lane's V pairs: a rotation needs no exchange between lanes.  V is 8 in the forward pass of bf16 (16 bytes), else 4.  Lanes behind
// the rotated channels turn theirs by an angle of zero.  A lane stays with its token and walks over heads: the cosines and
// sines (4 bytes for each 2-byte channel of a head) are read once for its heads and held in registers.  A workgroup takes few
// tokens and many of their heads, which lie next to each other in what a projection leaves.
// Bound: HBM.  75,600 tokens, 40 heads, d = 128, bf16 567 us (5.5 TB/s); 32,760 tokens, 12 heads, fp32, forward 108, backward 183 us
// (5.6, 5.5 TB/s) and 8 for the weights (with vectors of 8 channels of fp32, 32 bytes apart, 123 and 239).
#include "block_ops.h"
#include "spa2_device.h"

namespace spa2 {

// of q (0) or k (1)
struct NormSide {
  const void* x; const void* dy; void* y;              // input, upstream gradient (backward), result
  const float* w;
  int64_t sb, sh, sn, osb, osh, osn;
  int heads, tokens, tiles, slices, per_slice, walkers;       // tokens a workgroup takes at a time, tiles of them in all; heads
};                                                            // in slices; workgroups that walk the tiles of a slice
struct NormArgs {
  NormSide side[2];
  const float* cos; const float* sin; const void* positions;
  int64_t pos_sb;
  int pos_bits, table_rows, rot, B, N;
  float eps;
  float* part;                                         // backward: [workgroup][D] sums of dn x r, or null
};

constexpr int norm_vector(size_t size, bool backward) { return size == 2 && !backward ? 8 : 4; }
constexpr int norm_lanes(int d, size_t size, bool backward) { return d / (2 * norm_vector(size, backward)); }

// V channels as fp32
template <int V> __device__ __forceinline__ void norm_load(const uint16_t* p, float* x) {
  if constexpr (V == 8) {
    const u32x4 v = *(const u32x4*)p;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint32_t u = v[c];
      x[2 * c] = __builtin_bit_cast(float, u << 16);
      x[2 * c + 1] = __builtin_bit_cast(float, u & 0xffff0000u);
    }
  } else {
    const u32x2 v = *(const u32x2*)p;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const uint32_t u = v[c];
      x[2 * c] = __builtin_bit_cast(float, u << 16);
      x[2 * c + 1] = __builtin_bit_cast(float, u & 0xffff0000u);
    }
  }
}
template <int V> __device__ __forceinline__ void norm_load(const float* p, float* x) {
  if constexpr (V == 2) {
    const f32x2 v = *(const f32x2*)p;
    x[0] = v[0]; x[1] = v[1];
  } else {
#pragma unroll
    for (int q = 0; q < V; q += 4) {
      const f32x4 v = *(const f32x4*)(p + q);
#pragma unroll
      for (int c = 0; c < 4; ++c) x[q + c] = v[c];
    }
  }
}
template <bool PAST, typename P>
__device__ __forceinline__ void norm_put(P* p, P x) {
  if constexpr (PAST) __builtin_nontemporal_store(x, p);
  else                *p = x;
}
// PAST: past the memory-side cache
template <int V, bool PAST> __device__ __forceinline__ void norm_store(uint16_t* p, const float* x) {
  if constexpr (V == 8) norm_put<PAST>((u32x4*)p, u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])});
  else                  norm_put<PAST>((u32x2*)p, u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])});
}
template <int V, bool PAST> __device__ __forceinline__ void norm_store(float* p, const float* x) {
  static_assert(V == 4, "16 bytes");
  norm_put<PAST>((f32x4*)p, f32x4{x[0], x[1], x[2], x[3]});
}

// sum over the LANES lanes that own a row
template <int LANES>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
  for (int s = 1; s < LANES; s <<= 1) x += __shfl_xor(x, s, 64);
  return x;
}

// A lane's 2 V channels turned by its angles (BACK: by minus the angles).  Pair i: channels 2 i and 2 i + 1 of the lane's where
// pairs are interleaved, else i and V + i (its first vector lies in the first half of the rotated channels, the second behind).
template <bool INTERLEAVED, bool BACK, int V>
__device__ __forceinline__ void rotate(float (&x)[2 * V], const float (&cs)[V], const float (&sn)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float& p = x[INTERLEAVED ? 2 * i : i];
    float& q = x[INTERLEAVED ? 2 * i + 1 : V + i];
    const float s = BACK ? -sn[i] : sn[i], u = p, v = q;
    p = fmaf(u, cs[i], -(v * s));
    q = fmaf(v, cs[i], u * s);
  }
}

template <int D, typename T, bool INTERLEAVED, bool BACKWARD, bool PAST>
__global__ __launch_bounds__(256) void norm_rotate_kernel(NormArgs a) {
  constexpr int V = norm_vector(sizeof(T), BACKWARD), LANES = norm_lanes(D, sizeof(T), BACKWARD), GROUPS = 256 / LANES;
  const int tid = threadIdx.x, u = tid % LANES, group = tid / LANES;
  const int wgs_q = a.side[0].slices * a.side[0].walkers;
  const bool is_k = (int)blockIdx.x >= wgs_q;
  const NormSide& z = a.side[is_k];
  const int wg = blockIdx.x - (is_k ? wgs_q : 0), slice = wg / z.walkers;
  const int head0 = slice * z.per_slice + group / z.tokens, head1 = min((slice + 1) * z.per_slice, z.heads);
  const int head_step = GROUPS / z.tokens;
  // channels of this lane's vectors
  const int turning = a.rot / (2 * V);                 // lanes of a row that turn theirs: the first
  const bool turned = u < turning;
  const int first = turned ? V * u : a.rot + V * (u - turning), second = first + V * (turned ? turning : LANES - turning);
  const int at[2] = {first, second};                   // (the turning lanes' first vectors are the first half of the rotated channels)
  float w[2 * V], sums[2 * V];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (z.w) norm_load<V>(z.w + at[k], w + V * k);
    else
#pragma unroll
      for (int i = 0; i < V; ++i) w[V * k + i] = 1.f;
  }
  if (BACKWARD) {
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) sums[i] = 0.f;
  }
  const int64_t all = (int64_t)a.B * a.N;
  for (int tile = wg % z.walkers; tile < z.tiles; tile += z.walkers) {
    const int64_t token = (int64_t)tile * z.tokens + group % z.tokens;
    if (token >= all) break;                           // (later tiles are further on still)
    const int b = (int)(token / a.N), n = (int)(token - (int64_t)b * a.N);
    float cs[V], sn[V];
    if (turned) {
      int64_t row = n;
      if (a.pos_bits == 32) row = ((const int32_t*)a.positions)[b * a.pos_sb + n];
      if (a.pos_bits == 64) row = ((const int64_t*)a.positions)[b * a.pos_sb + n];
      row = min(max(row, (int64_t)0), (int64_t)a.table_rows - 1);        // (caller data)
      const int64_t angles = row * (a.rot / 2);
      if constexpr (INTERLEAVED) {                     // half of a vector's channels are pairs
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          norm_load<V / 2>(a.cos + angles + at[k] / 2, cs + V / 2 * k);
          norm_load<V / 2>(a.sin + angles + at[k] / 2, sn + V / 2 * k);
        }
      } else {
        norm_load<V>(a.cos + angles + first, cs);
        norm_load<V>(a.sin + angles + first, sn);
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) { cs[i] = 1.f; sn[i] = 0.f; }
    }
    const T* x0 = (const T*)z.x + b * z.sb + n * z.sn;
    const int64_t out0 = b * z.osb + n * z.osn;
#pragma unroll 1
    for (int h = head0; h < head1; h += head_step) {
      float x[2 * V];
#pragma unroll
      for (int k = 0; k < 2; ++k) norm_load<V>(x0 + h * z.sh + at[k], x + V * k);
      const int64_t out = out0 + h * z.osh;
      float square = 0.f;
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) square = fmaf(x[i], x[i], square);
      if constexpr (!BACKWARD) {
        const float r = 1.f / sqrtf(row_sum<LANES>(square) * (1.f / D) + a.eps);
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) x[i] = x[i] * r * w[i];
        rotate<INTERLEAVED, false, V>(x, cs, sn);
#pragma unroll
        for (int k = 0; k < 2; ++k) norm_store<V, PAST>((uint16_t*)z.y + out + at[k], x + V * k);
      } else {
        float g[2 * V], inner = 0.f;
#pragma unroll
        for (int k = 0; k < 2; ++k) norm_load<V>((const uint16_t*)z.dy + out + at[k], g + V * k);
        rotate<INTERLEAVED, true, V>(g, cs, sn);
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) inner = fmaf(g[i] * w[i], x[i], inner);
        const float r = 1.f / sqrtf(row_sum<LANES>(square) * (1.f / D) + a.eps);
        inner = row_sum<LANES>(inner) * r * (1.f / D);
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) {
          const float hat = x[i] * r;
          sums[i] = fmaf(g[i], hat, sums[i]);
          x[i] = r * fmaf(-hat, inner, g[i] * w[i]);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) norm_store<V, PAST>((T*)z.y + out + at[k], x + V * k);
      }
    }
  }
  if constexpr (BACKWARD) {
    if (!a.part) return;
    // sums of the lanes that hold the same channels: over a wave by exchange, over the waves through LDS
    __shared__ float lds[4][D];
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) {
#pragma unroll
      for (int s = LANES; s < 64; s <<= 1) sums[i] += __shfl_xor(sums[i], s, 64);
    }
    if ((tid & 63) < LANES) {
#pragma unroll
      for (int k = 0; k < 2; ++k) norm_store<V, false>(&lds[tid >> 6][at[k]], sums + V * k);
    }
    __syncthreads();
    if (tid < D) a.part[(int64_t)blockIdx.x * D + tid] = (lds[0][tid] + lds[1][tid]) + (lds[2][tid] + lds[3][tid]);
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

// Which rows a workgroup takes: as many heads of a token as there are, up to half of its groups of lanes, so that a wave's accesses
// lie next to each other.  (75,600 tokens, 40 heads, heads at a time 1 / 2 / 4 / 8 / 16 / 32: 671 / 661 / 656 / 642 / 628 / 642 us.)
// Heads of a token go to several workgroups where whole tokens would leave compute units idle.
void norm_side(NormSide& z, const spa2_norm_shape& s, int heads, bool backward) {
  const int groups = 256 / norm_lanes(s.d, s.dtype == SPA2_DTYPE_BF16 ? 2 : 4, backward);
  const int64_t all = (int64_t)s.B * s.N;
  int at_once = 1;
  for (int x = 2; x <= heads && x <= groups / 2; x *= 2)
    if (4 * ((heads + x - 1) / x * x) <= 5 * heads) at_once = x;          // (an idle group in five at most)
  z.heads = heads;
  z.tokens = groups / at_once;
  z.tiles = (int)((all + z.tokens - 1) / z.tokens);
  int slices = 1;
  const int most = (heads + at_once - 1) / at_once;
  while (slices < most && (int64_t)z.tiles * slices < 1024) ++slices;
  z.per_slice = (most + slices - 1) / slices * at_once;
  z.slices = (heads + z.per_slice - 1) / z.per_slice;
  // (backward: the sums over tokens of as few workgroups as fill the chip are left to be added)
  const int limit = backward ? (int)((int64_t)2048 * heads / (s.Hq + s.Hk)) / z.slices : 1 << 20;
  z.walkers = z.tiles < limit ? z.tiles : (limit < 1 ? 1 : limit);
}
int norm_wgs(const NormSide& z) { return z.slices * z.walkers; }

NormArgs norm_args(const NormTables& t, const spa2_norm_shape& s, const float* q_weight, const float* k_weight, float eps,
                   bool backward) {
  NormArgs a = {};
  for (int i = 0; i < 2; ++i) norm_side(a.side[i], s, i ? s.Hk : s.Hq, backward);
  NormSide &q = a.side[0], &k = a.side[1];
  q.w = q_weight; k.w = k_weight;
  q.sb = s.q_sb; q.sh = s.q_sh; q.sn = s.q_sn; q.osb = s.qo_sb; q.osh = s.qo_sh; q.osn = s.qo_sn;
  k.sb = s.k_sb; k.sh = s.k_sh; k.sn = s.k_sn; k.osb = s.ko_sb; k.osh = s.ko_sh; k.osn = s.ko_sn;
  a.cos = t.cos; a.sin = t.sin; a.positions = t.positions;
  a.pos_sb = s.pos_sb; a.pos_bits = s.pos_bits; a.table_rows = s.table_rows; a.rot = s.rot;
  a.B = s.B; a.N = s.N;
  a.eps = eps;
  return a;
}

template <int D, typename T, bool BACKWARD>
void launch_typed(const NormArgs& a, bool interleaved, bool past, hipStream_t stream) {
  const dim3 grid((unsigned)(norm_wgs(a.side[0]) + norm_wgs(a.side[1]))), block(256);
  const auto kernel = interleaved ? (past ? norm_rotate_kernel<D, T, true, BACKWARD, true> : norm_rotate_kernel<D, T, true, BACKWARD, false>)
                                  : (past ? norm_rotate_kernel<D, T, false, BACKWARD, true> : norm_rotate_kernel<D, T, false, BACKWARD, false>);
  hipLaunchKernelGGL(kernel, grid, block, 0, stream, a);
}

template <bool BACKWARD>
hipError_t launch_any(const NormArgs& a, const spa2_norm_shape& s, hipStream_t stream) {
  const bool bf16 = s.dtype == SPA2_DTYPE_BF16, il = s.interleaved != 0;
  // Stored past the memory-side cache where what is read and written does not fit in it.  75,600 tokens, 40 heads 588 / 562 us,
  // 32,760 tokens, 12 heads, fp32, both passes 361 / 351.
  const int64_t size = bf16 ? 2 : 4;
  const bool past = (int64_t)s.B * s.N * (s.Hq + s.Hk) * s.d * (BACKWARD ? 2 * size + 2 : size + 2) > CACHE_BYTES;
  if (s.d == 128) bf16 ? launch_typed<128, uint16_t, BACKWARD>(a, il, past, stream) : launch_typed<128, float, BACKWARD>(a, il, past, stream);
  else            bf16 ? launch_typed<64, uint16_t, BACKWARD>(a, il, past, stream) : launch_typed<64, float, BACKWARD>(a, il, past, stream);
  return hipGetLastError();
}

}  // namespace

size_t norm_rotate_partials_bytes(const spa2_norm_shape& s) {
  NormSide q = {}, k = {};
  norm_side(q, s, s.Hq, true);
  norm_side(k, s, s.Hk, true);
  return (size_t)(norm_wgs(q) + norm_wgs(k)) * (size_t)s.d * sizeof(float);
}

hipError_t launch_norm_rotate(const void* q, const void* k, const float* q_weight, const float* k_weight, const NormTables& t,
                              const spa2_norm_shape& s, float eps, void* q_out, void* k_out, hipStream_t stream) {
  NormArgs a = norm_args(t, s, q_weight, k_weight, eps, false);
  a.side[0].x = q; a.side[1].x = k;
  a.side[0].y = q_out; a.side[1].y = k_out;
  return launch_any<false>(a, s, stream);
}

hipError_t launch_norm_rotate_bwd(const void* q, const void* k, const float* q_weight, const float* k_weight,
                                  const NormTables& t, const void* d_q_out, const void* d_k_out, const spa2_norm_shape& s,
                                  float eps, void* dq, void* dk, float* d_q_weight, float* d_k_weight, void* ws,
                                  hipStream_t stream) {
  NormArgs a = norm_args(t, s, q_weight, k_weight, eps, true);
  a.side[0].x = q; a.side[1].x = k;
  a.side[0].dy = d_q_out; a.side[1].dy = d_k_out;
  a.side[0].y = dq; a.side[1].y = dk;
  a.part = d_q_weight || d_k_weight ? (float*)ws : nullptr;
  const hipError_t e = launch_any<true>(a, s, stream);
  if (e != hipSuccess || !a.part) return e;
  hipLaunchKernelGGL(norm_weight_finish, dim3((unsigned)(2 * (s.d / 16))), dim3(256), 0, stream, (const float*)ws, s.d,
                     norm_wgs(a.side[0]), norm_wgs(a.side[1]), d_q_weight, d_k_weight);
  return hipGetLastError();
}

}  // namespace spa2
