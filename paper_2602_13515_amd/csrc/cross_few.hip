// Attention to another sequence for few query rows (up to 32 over the query heads of a key head: one token, or a few, against a
// cache).  Bound: HBM, every key and value is read once.
//
// A workgroup takes the rows of all query heads of a key head together (row r: head r / Nq, query r % Nq).  As in fwd.hip a
// lane owns one row and everything is computed transposed, S^T = K Q^T and O^T += V^T P^T; but here the waves share no tile:
// each walks tiles of 32 keys of its own, copied global -> LDS directly and two tiles ahead, without a barrier, so that a compute
// unit has 64 to 128 KB on the way.  The waves' results are joined through LDS, those of several workgroups by a launch behind
// (a workgroup a row; joined by the last part to arrive, which needed counters set to zero by a launch in front, 32 rows and one
// sample of 65,536 keys took 342 instead of 28 us).  Only the rows that are there are exchanged.
//
// Who takes which keys: where there are few (sample, key head) pairs, the key blocks of all samples stand in one line, sample after
// sample, and every workgroup of a head takes an equal stretch of it, whatever the lengths are: a sample that it shares with
// others leaves a partial result.  (Cut by size alone, in equal parts of the longest sample, 280 to 576 workgroups of unlike
// number on the compute units took 127 to 168 us on the first case below.)  Where there are many pairs, or short samples, a
// workgroup takes one pair.
// Measured, us: one query, seven samples of 8190 to 32,760 keys and an empty one, 40 heads sharing 8, d = 128 115 (5.1 TB/s); 8
// samples of 32,760 keys 188 (5.7 TB/s; the copies alone 182); 8 samples of 8192 keys, 8 heads 50, d = 64 30; 1 sample of 65,536, 2
// heads 26; 600 samples of 77, 4 heads, d = 64 16.
// P goes into its product in two bf16 parts, as in the backward pass of such rows (cross.h): the matrix cores wait for the copies
// anyway.  The error of O is then that of its own rounding, where one part left 1.07 to 1.29 times that; the price is 0 to 1 us of
// the above, and with 32 rows, one part / two, 55.3 / 55.7, d = 64 33.9 / 34.2, 28.0 / 28.9 and 20.1 / 20.6.  (Many rows: fwd.hip.)
#include "cross.h"
#include "row_map.h"
#include "spa2_device.h"

namespace spa2 {

struct FewArgs {
  const uint16_t* q; const uint16_t* k; const uint16_t* v;
  uint16_t* o; uint16_t* o_res; float* lse;
  CrossKeys kv;
  int B, Hk, Nq, rows;           // rows = group * Nq
  int workers;                   // workgroups of a key head that share the line of key blocks; 0: one a (sample, key head)
  int64_t sb, sh, sn;
  float scale_log2;
  float* pool; int slot_floats;  // partial results (few_slot)
};

constexpr int FEW_WAVES = 2;     // (two workgroups of 64 KB share a compute unit; of four waves and 128 KB one: 127 / 140 us)
// Blocks of a sample in the line: one at least, so that every sample is somebody's.
__device__ __forceinline__ int few_blocks(int keys) { return max((keys + BKV - 1) / BKV, 1); }

// The line: blocks of the samples lane, 64 + lane, ..., and how many a stretch has.
constexpr int FEW_CHUNKS = FEW_SAMPLES / 64;
struct FewLine { int n[FEW_CHUNKS], total, per; };
__device__ __forceinline__ FewLine few_line(const FewArgs& a, int lane) {
  FewLine r;
  r.total = 0;
#pragma unroll
  for (int c = 0; c < FEW_CHUNKS; ++c) {
    const int b = 64 * c + lane;
    r.n[c] = b < a.B ? few_blocks(a.kv.lengths ? min(max(a.kv.lengths[b], 0), a.kv.Nk) : a.kv.Nk) : 0;
  }
#pragma unroll
  for (int c = 0; c < FEW_CHUNKS; ++c) r.total += r.n[c];
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) r.total += __shfl_xor(r.total, s, 64);
  r.total = __builtin_amdgcn_readfirstlane(r.total);
  r.per = max((r.total + a.workers - 1) / a.workers, FEW_LEAST);
  return r;
}
// First place of sample b.
__device__ __forceinline__ int few_first(const FewLine& line, int b, int lane) {
  int before = 0;
#pragma unroll
  for (int c = 0; c < FEW_CHUNKS; ++c) before += 64 * c + lane < b ? line.n[c] : 0;
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) before += __shfl_xor(before, s, 64);
  return __builtin_amdgcn_readfirstlane(before);
}
// The sample that place `at` (inside the line) belongs to, and that sample's first place.
struct FewSample { int b, first; };
__device__ __forceinline__ FewSample few_sample(const FewArgs& a, const FewLine& line, int place, int lane) {
  FewSample r = {0, 0};
  int run = 0;
#pragma unroll
  for (int c = 0; c < FEW_CHUNKS; ++c) {
    if (64 * c >= a.B) break;
    int sum = line.n[c];                                 // of this sample and those before it
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int x = __shfl_up(sum, s, 64);
      sum += lane >= s ? x : 0;
    }
    const int at = run + sum - line.n[c];
    const uint64_t here = __builtin_amdgcn_ballot_w64(line.n[c] > 0 && at <= place && place < at + line.n[c]);
    if (here) {
      const int l = __builtin_ctzll(here);
      r.b = 64 * c + l;
      r.first = __shfl(at, l, 64);
    }
    run += __shfl(sum, 63, 64);
  }
  r.b = __builtin_amdgcn_readfirstlane(r.b); r.first = __builtin_amdgcn_readfirstlane(r.first);
  return r;
}
// Stretches that a sample lies in, and where part p of its result lies: a stretch has two slots, for the sample that it begins
// inside of or with and for the one that it ends inside of.
struct FewParts { int i0, parts, starts; };
__device__ __forceinline__ FewParts few_parts(int first, int n, int per) {
  const int i0 = first / per;
  return {i0, (first + n - 1) / per - i0 + 1, first == i0 * per};
}
__device__ __forceinline__ int few_slot(const FewArgs& a, const FewParts& s, int hk, int p) {
  return 2 * (hk * a.workers + s.i0 + p) + (p == 0 && !s.starts);
}

// Four channels (4 c ..) of a row's sum x with maximum m and sum of weights l: O = x / l, LSE.
__device__ __forceinline__ int64_t few_row(const FewArgs& a, int b, int hk, int r) {
  return b * a.sb + ((int64_t)hk * a.kv.group + r / a.Nq) * a.sh + (r % a.Nq) * a.sn;
}
__device__ __forceinline__ void few_finish(const FewArgs& a, int b, int hk, int row, int c, f32x4 x, float m, float l) {
  const float inv = 1.f / l;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] *= inv;
  const u32x2 out = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
  const int64_t off = few_row(a, b, hk, row) + 4 * c;
  *(u32x2*)(a.o + off) = out;
  if (a.o_res) {
    const u32x2 r = {pack_bf16(x[0] - __builtin_bit_cast(float, out[0] << 16), x[1] - __builtin_bit_cast(float, out[0] & 0xffff0000u)),
                     pack_bf16(x[2] - __builtin_bit_cast(float, out[1] << 16), x[3] - __builtin_bit_cast(float, out[1] & 0xffff0000u))};
    *(u32x2*)(a.o_res + off) = r;
  }
  if (c == 0) a.lse[((int64_t)b * a.Hk + hk) * a.rows + row] = m * LN2 + __logf(l);      // (heads and queries of a key head: consecutive)
}
// 2^(m_p - m) for a part whose maximum is m_p; a part that saw no score but minus infinity has no weight
__device__ __forceinline__ float few_weight(float m_p, float m) { return m_p == -INFINITY ? 0.f : fast_exp2(m_p - m); }

// LDS of a workgroup
template <int D>
struct FewLds {
  static constexpr int TK = 32, TILE_B = TK * D * 2, STAGE_B = 2 * TILE_B, WAVE_B = 2 * STAGE_B;      // a stage: K rows, then V rows
  unsigned char smem[FEW_WAVES * WAVE_B];
  float stat[FEW_WAVES][32][2];
};

// Keys [key0, key1) of sample b and key head hk; its result goes to a slot where others share the sample (slot >= 0).
struct FewPiece { int b, hk, key0, key1, slot; };
template <int D>
__device__ __forceinline__ void few_piece(const FewArgs& a, const FewPiece& pc, FewLds<D>& lds) {
  constexpr int TK = 32, NK = D / 16, NMB = D / 32, CPR = D / 8, RPI = 64 / CPR, NCP = TK / RPI, WAVES = FEW_WAVES, NT = 64 * WAVES;
  constexpr int TILE_B = FewLds<D>::TILE_B, STAGE_B = FewLds<D>::STAGE_B, WAVE_B = FewLds<D>::WAVE_B;
  constexpr int PITCH = D + 4;                                                        // floats a row in the exchange
  static_assert(32 * PITCH * 4 <= WAVE_B, "a wave's sums fit its stages");
  unsigned char* smem = lds.smem;
  auto& stat = lds.stat;
  const int b = pc.b, hk = pc.hk, key0 = pc.key0, key1 = pc.key1;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, hf = lane >> 5;
  if (key1 <= key0) {                        // a sample without keys: O = 0, LSE = -inf
    for (int x = tid; x < a.rows * CPR; x += NT) {
      const int64_t off = few_row(a, b, hk, x / CPR) + 8 * (x % CPR);
      *(u32x4*)(a.o + off) = u32x4{0, 0, 0, 0};
      if (a.o_res) *(u32x4*)(a.o_res + off) = u32x4{0, 0, 0, 0};
    }
    if (tid < a.rows) a.lse[((int64_t)b * a.Hk + hk) * a.rows + tid] = -INFINITY;
    return;
  }

  // copies of this wave's tile: as in dkdv_item, lane l fills chunk position l % CPR of row RPI r + l / CPR and fetches the
  // chunk that the swizzle puts there; rows past the part's end repeat its last key
  const char* k_head = (const char*)(a.k + b * a.kv.sb + hk * a.kv.sh);
  const char* v_head = (const char*)(a.v + b * a.kv.sb + hk * a.kv.sh);
  const uint64_t row_bytes = (uint64_t)a.kv.sn * 2;
  const uint32_t sm = lds_addr_of(smem) + w * WAVE_B;
  const int tiles_all = (key1 - key0 + TK - 1) / TK, tiles = (tiles_all - w + WAVES - 1) / WAVES;   // this wave's: w, w + WAVES, ...
  uint32_t voff[NCP];
  int rows_set = -1;
  auto copy_tile = [&](int t, uint32_t stage) {
    const int at = key0 + (w + WAVES * t) * TK, last = min(TK, key1 - at) - 1;
    if (last != rows_set) {
      rows_set = last;
#pragma unroll
      for (int r = 0; r < NCP; ++r) {
        const int row = RPI * r + lane / CPR;
        voff[r] = (uint32_t)((min(row, last) * a.kv.sn + (((lane % CPR) ^ swz<D>(row)) * 8)) * 2);
      }
    }
    const char* kp = k_head + (uint64_t)at * row_bytes;
    const char* vp = v_head + (uint64_t)at * row_bytes;
    static_for<0, NCP>([&](auto R) { raw_copy16_to_lds_at<decltype(R)::v * 1024>(kp, voff[decltype(R)::v], stage); });
    static_for<0, NCP>([&](auto R) { raw_copy16_to_lds_at<TILE_B + decltype(R)::v * 1024>(vp, voff[decltype(R)::v], stage); });
  };

  raw_copies_done();                                     // (what is counted from here on are the copies)
  bf16x8 qf[NK];
  {
    const uint16_t* qp = a.q + few_row(a, b, hk, min(r32, a.rows - 1)) + 8 * hf;
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) qf[kk] = *(const bf16x8*)(qp + 16 * kk);
  }
  f32x16 oacc[NMB];
#pragma unroll
  for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
    for (int v = 0; v < 16; ++v) oacc[mb][v] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  const int s16 = lane & 15, hb16 = (lane >> 4) & 1;
  const uint32_t k_off = 2 * swz_idx<D>(r32, 8 * hf);
  const uint32_t v_off0 = TILE_B + 2 * swz_idx<D>(4 * hf + (s16 >> 2), 16 * hb16 + 4 * (s16 & 3));
  const uint32_t v_off1 = TILE_B + 2 * swz_idx<D>(8 + 4 * hf + (s16 >> 2), 16 * hb16 + 4 * (s16 & 3));

  if (tiles > 0) {
    copy_tile(0, sm);
    copy_tile(min(1, tiles - 1), sm + STAGE_B);          // (past the end the last tile is requested again, into a stage nobody reads)
  }
  for (int t = 0; t < tiles; ++t) {
    const uint32_t stage = sm + (t & 1) * STAGE_B;
    const uint32_t ka = stage + k_off, v0 = stage + v_off0, v1 = stage + v_off1;
    raw_copies_left<3 * NCP>();                          // K of this tile has landed
    f32x16 s = zero;
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) s = mfma32(lds_ld16(ka ^ (kk << 5)), qf[kk], s);
    const int valid = key1 - (key0 + (w + WAVES * t) * TK) - 4 * hf;
    if (valid + 4 * hf < TK) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (8 * (v >> 2) + (v & 3) >= valid) s[v] = -INFINITY;
    }
    float mx = s[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) mx = fmaxf(mx, s[v]);
    const float m_new = fmaxf(m_run, max_halves(mx) * a.scale_log2);
    if (__builtin_amdgcn_ballot_w64(m_new != m_run) != 0) {
      // (nothing seen yet, or only scores of minus infinity: the sums are zero and stay so)
      const float alpha = m_run == m_new ? 1.f : fast_exp2(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
        for (int v = 0; v < 16; ++v) oacc[mb][v] *= alpha;
      m_run = m_new;
    }
    uint32_t pk[8], rest[8];                             // P in two bf16 parts
    const float shift = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float p0 = fast_exp2(fmaf(s[2 * u], a.scale_log2, -shift)), p1 = fast_exp2(fmaf(s[2 * u + 1], a.scale_log2, -shift));
      pk[u] = pack_bf16(p0, p1);
      rest[u] = pack_rest(p0, p1, pk[u]);
      l_run += p0 + p1;
    }
    raw_copies_left<2 * NCP>();                          // and V
#pragma unroll
    for (int cc = 0; cc < 2; ++cc) {
      const bf16x8 p = __builtin_bit_cast(bf16x8, u32x4{pk[4 * cc], pk[4 * cc + 1], pk[4 * cc + 2], pk[4 * cc + 3]});
      const bf16x8 p_rest = __builtin_bit_cast(bf16x8, u32x4{rest[4 * cc], rest[4 * cc + 1], rest[4 * cc + 2], rest[4 * cc + 3]});
#pragma unroll
      for (int mb = 0; mb < NMB; ++mb) {
        const int o = cc * 16 * D * 2;
        const bf16x8 x = join_tr(lds_tr4_at((v0 ^ (mb << 6)) + o), lds_tr4_at((v1 ^ (mb << 6)) + o));
        oacc[mb] = mfma32(x, p, oacc[mb]);
        oacc[mb] = mfma32(x, p_rest, oacc[mb]);
      }
    }
    copy_tile(min(t + 2, tiles - 1), stage);             // (the products above have read this stage)
  }
  raw_copies_done();                                     // nothing may land in the LDS from here on
  const float l_tot = sum_halves(l_run);

  // ---- the waves' results, joined: every wave leaves its sums in its own stages
  float* mine = (float*)(smem + w * WAVE_B);
#pragma unroll
  for (int mb = 0; mb < NMB; ++mb)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *(f32x4*)(mine + r32 * PITCH + 32 * mb + 8 * g + 4 * hf) = f32x4{oacc[mb][4 * g], oacc[mb][4 * g + 1], oacc[mb][4 * g + 2], oacc[mb][4 * g + 3]};
  if (hf == 0) { stat[w][r32][0] = m_run; stat[w][r32][1] = l_tot; }
  __syncthreads();
  constexpr int QUADS = D / 4;                           // a thread takes four channels of a row at a time
  float* slot = a.pool + (int64_t)max(pc.slot, 0) * a.slot_floats;
  for (int x = tid; x < a.rows * QUADS; x += NT) {
    const int row = x / QUADS, c = x % QUADS;
    float m = stat[0][row][0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) m = fmaxf(m, stat[i][row][0]);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      const float f = few_weight(stat[i][row][0], m);
      const f32x4 y = *(const f32x4*)((const float*)(smem + i * WAVE_B) + row * PITCH + 4 * c);
      l = fmaf(stat[i][row][1], f, l);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = fmaf(y[e], f, sum[e]);
    }
    if (pc.slot < 0) {
      few_finish(a, b, hk, row, c, sum, m, l);
    } else {
      *(f32x4*)(slot + row * D + 4 * c) = sum;
      if (c == 0) *(f32x2*)(slot + a.rows * D + 2 * row) = f32x2{m, l};
    }
  }
}

template <int D>
__global__ __launch_bounds__(64 * FEW_WAVES) void cross_few_kernel(FewArgs a) {
  __shared__ __align__(1024) FewLds<D> lds;
  if (a.workers == 0) {
    const int b = blockIdx.x / a.Hk, keys = cross_length(a.kv, b);
    few_piece<D>(a, FewPiece{b, (int)blockIdx.x % a.Hk, 0, keys, -1}, lds);
    return;
  }
  const int hk = blockIdx.x % a.Hk, i = blockIdx.x / a.Hk, lane = threadIdx.x & 63;
  const FewLine line = few_line(a, lane);
  const int begin = i * line.per, stop = min(begin + line.per, line.total);
  if (begin >= stop) return;
  const FewSample start = few_sample(a, line, begin, lane);
  int first = start.first;                               // of sample b
  for (int b = start.b, at = begin; at < stop; ++b) {
    const int keys = cross_length(a.kv, b), n = few_blocks(keys), end = min(first + n, stop);
    const FewParts s = few_parts(first, n, line.per);
    const FewPiece pc = {b, hk, (at - first) * BKV, min(keys, (end - first) * BKV), s.parts == 1 ? -1 : few_slot(a, s, hk, i - s.i0)};
    few_piece<D>(a, pc, lds);
    __syncthreads();                                     // (the next piece's tiles land where this one's results were)
    first += n;
    at = end;
  }
}

// Row `row` of a (sample, key head) whose keys several workgroups shared: their results, joined.  A thread takes four channels and
// every G-th part, in order; then the G are added in order.
template <int D>
__global__ __launch_bounds__(256) void cross_few_join_kernel(FewArgs a) {
  constexpr int QUADS = D / 4, G = 256 / QUADS;
  __shared__ __align__(16) float sums[G][D];
  __shared__ float stat[G][2];
  const int row = blockIdx.x % a.rows, unit = blockIdx.x / a.rows, b = unit / a.Hk, hk = unit % a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, c = tid % QUADS, g = tid / QUADS;
  const FewLine line = few_line(a, lane);
  const FewParts s = few_parts(few_first(line, b, lane), few_blocks(cross_length(a.kv, b)), line.per);
  if (s.parts == 1) return;
  float m = -INFINITY, l = 0.f;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  for (int p = g; p < s.parts; p += 4 * G) {             // four parts in flight
    f32x2 ml[4];
    f32x4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float* slot = a.pool + (int64_t)few_slot(a, s, hk, min(p + i * G, s.parts - 1)) * a.slot_floats;
      ml[i] = *(const f32x2*)(slot + a.rows * D + 2 * row);
      x[i] = *(const f32x4*)(slot + row * D + 4 * c);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (p + i * G >= s.parts) break;
      const float m_new = fmaxf(m, ml[i][0]), old = few_weight(m, m_new), f = few_weight(ml[i][0], m_new);
      l = fmaf(ml[i][1], f, l * old);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = fmaf(x[i][e], f, sum[e] * old);
      m = m_new;
    }
  }
  *(f32x4*)&sums[g][4 * c] = sum;
  if (c == 0) { stat[g][0] = m; stat[g][1] = l; }
  __syncthreads();
  if (g) return;
#pragma unroll
  for (int i = 1; i < G; ++i) m = fmaxf(m, stat[i][0]);
  l = 0.f;
  sum = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < G; ++i) {
    const float f = few_weight(stat[i][0], m);
    const f32x4 x = *(const f32x4*)&sums[i][4 * c];
    l = fmaf(stat[i][1], f, l);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] = fmaf(x[e], f, sum[e]);
  }
  few_finish(a, b, hk, row, c, sum, m, l);
}

hipError_t launch_cross_few(const void* q, const void* k, const void* v, const CrossDims& m, const int32_t* lengths, float scale,
                            void* o, void* o_res, float* lse, void* ws, hipStream_t stream) {
  FewArgs a = {};
  a.q = (const uint16_t*)q; a.k = (const uint16_t*)k; a.v = (const uint16_t*)v;
  a.o = (uint16_t*)o; a.o_res = (uint16_t*)o_res; a.lse = lse;
  a.kv = cross_keys(m, lengths);
  a.B = m.q.B; a.Hk = m.Hk; a.Nq = m.q.N; a.rows = m.group * m.q.N;
  a.sb = m.q.sb; a.sh = m.q.sh; a.sn = m.q.sn;
  a.scale_log2 = scale * LOG2E;
  a.workers = cross_few_ws(m).workers;
  a.pool = (float*)ws;
  a.slot_floats = (int)(few_slot_bytes(a.rows, m.q.d) / 4);
  const dim3 grid((unsigned)((a.workers ? a.workers : m.q.B) * m.Hk)), block(64 * FEW_WAVES);
  if (m.q.d == 128) hipLaunchKernelGGL(cross_few_kernel<128>, grid, block, 0, stream, a);
  else              hipLaunchKernelGGL(cross_few_kernel<64>, grid, block, 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.workers <= 1) return e;
  const dim3 rows((unsigned)(m.q.B * m.Hk * a.rows));
  if (m.q.d == 128) hipLaunchKernelGGL(cross_few_join_kernel<128>, rows, dim3(256), 0, stream, a);
  else              hipLaunchKernelGGL(cross_few_join_kernel<64>, rows, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace spa2
