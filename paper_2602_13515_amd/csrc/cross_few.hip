// Attention to another sequence for few query rows (up to 32 over the query heads of a key head: one token, or a few, against a
// cache).  Bound: HBM, every key and value is read once.
//
// A workgroup takes the rows of all query heads of a key head together (row r: head r / Nq, query r % Nq).  As in fwd.hip a
// lane owns one row and everything is computed transposed, S^T = K Q^T and O^T += V^T P^T; but here the waves share no tile:
// each walks tiles of 32 keys of its own, copied global -> LDS directly and two tiles ahead, without a barrier, so that a compute
// unit has 64 to 128 KB on the way.  The waves' results are joined through LDS, those of several workgroups by the last to arrive;
// only the rows that are there are exchanged.
//
// Who takes which keys: where there are few (sample, key head) pairs, the key blocks of all samples stand in one line, sample after
// sample, and every workgroup of a head takes an equal stretch of it, whatever the lengths are: a sample that it shares with
// others leaves a partial result.  (Cut by size alone, in equal parts of the longest sample, 280 to 576 workgroups of unlike
// number on the compute units took 127 to 168 us where an even 512 take EVEN.)  Where there are many pairs, a workgroup takes one.
// Measured: FEW.
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
  int32_t* arrive;               // [B][Hk] parts of a sample that have left their result
  float* pool; int slot_floats;  // [Hk][workers][2]: of the sample that a stretch begins inside of or with, of the one it ends inside of
};

constexpr int FEW_WAVES = 2;     // (two workgroups of 64 KB share a compute unit; of four waves and 128 KB one: 127 / 140 us)
constexpr int FEW_LEAST = 4;     // key blocks that a stretch has at least
constexpr int FEW_SAMPLES = 1024;       // samples that a line may have
inline int few_resident(int d) { return 512 * 128 / d; }

// A part's result: [row][D] unnormalised sums, then (maximum in log2 units, sum) of each row.
inline size_t few_slot_bytes(int rows, int d) { return (size_t)rows * (d + 2) * 4; }

// Blocks of a sample in the line: one at least, so that every sample is somebody's.
__device__ __forceinline__ int few_blocks(int keys) { return max((keys + BKV - 1) / BKV, 1); }

// Where stretch i of `workers` begins and ends in the line, and in which sample (that sample's first place in the line).
struct FewLine { int begin, end, per, b, first; };
__device__ __forceinline__ FewLine few_line(const FewArgs& a, int i, int lane) {
  constexpr int CHUNKS = FEW_SAMPLES / 64;
  int n[CHUNKS], total = 0;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int b = 64 * c + lane;
    n[c] = b < a.B ? few_blocks(a.kv.lengths ? min(max(a.kv.lengths[b], 0), a.kv.Nk) : a.kv.Nk) : 0;
  }
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) total += n[c];
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) total += __shfl_xor(total, s, 64);
  FewLine r;
  r.per = max((total + a.workers - 1) / a.workers, FEW_LEAST);
  r.begin = min(i * r.per, total);
  r.end = min(r.begin + r.per, total);
  r.b = 0; r.first = 0;
  int run = 0;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    if (64 * c >= a.B) break;
    int sum = n[c];                                      // of this sample and those before it
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int x = __shfl_up(sum, s, 64);
      sum += lane >= s ? x : 0;
    }
    const int at = run + sum - n[c];
    const uint64_t here = __builtin_amdgcn_ballot_w64(n[c] > 0 && at <= r.begin && r.begin < at + n[c]);
    if (here) {
      const int l = __builtin_ctzll(here);
      r.b = 64 * c + l;
      r.first = __shfl(at, l, 64);
    }
    run += __shfl(sum, 63, 64);
  }
  r.per = __builtin_amdgcn_readfirstlane(r.per);
  r.begin = __builtin_amdgcn_readfirstlane(r.begin); r.end = __builtin_amdgcn_readfirstlane(r.end);
  r.b = __builtin_amdgcn_readfirstlane(r.b); r.first = __builtin_amdgcn_readfirstlane(r.first);
  return r;
}

// LDS of a workgroup
template <int D>
struct FewLds {
  static constexpr int TK = 32, TILE_B = TK * D * 2, STAGE_B = 2 * TILE_B, WAVE_B = 2 * STAGE_B;      // a stage: K rows, then V rows
  unsigned char smem[FEW_WAVES * WAVE_B];
  float stat[FEW_WAVES][32][2];
  int word;
};

// Keys [key0, key1) of sample b and key head hk.  parts: workgroups that share the sample's keys; slots of the first and of the
// others lie first_slot and next_slots, next_slots + 2, ... (in slots).
struct FewPiece { int b, hk, key0, key1, parts, slot, first_slot, next_slots; };
template <int D>
__device__ __forceinline__ void few_piece(const FewArgs& a, const FewPiece& pc, FewLds<D>& lds) {
  constexpr int TK = 32, NK = D / 16, NMB = D / 32, CPR = D / 8, RPI = 64 / CPR, NCP = TK / RPI, WAVES = FEW_WAVES, NT = 64 * WAVES;
  constexpr int TILE_B = FewLds<D>::TILE_B, STAGE_B = FewLds<D>::STAGE_B, WAVE_B = FewLds<D>::WAVE_B;
  constexpr int PITCH = D + 4;                                                        // floats a row in the exchange
  static_assert(32 * PITCH * 4 <= WAVE_B, "a wave's sums fit its stages");
  unsigned char* smem = lds.smem;
  auto& stat = lds.stat;
  const int b = pc.b, hk = pc.hk, group = a.kv.group, key0 = pc.key0, key1 = pc.key1, parts = pc.parts, unit = b * a.Hk + hk;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, hf = lane >> 5;
  const int64_t q_base = b * a.sb + (int64_t)hk * group * a.sh;
  const int64_t stat_base = (int64_t)unit * a.rows;                                   // (heads and queries of a key head: consecutive)
  auto row_at = [&](int r) -> int64_t { return q_base + (r / a.Nq) * a.sh + (r % a.Nq) * a.sn; };

  if (key1 <= key0) {                        // a sample without keys: O = 0, LSE = -inf
    for (int x = tid; x < a.rows * CPR; x += NT) {
      const int64_t off = row_at(x / CPR) + 8 * (x % CPR);
      *(u32x4*)(a.o + off) = u32x4{0, 0, 0, 0};
      if (a.o_res) *(u32x4*)(a.o_res + off) = u32x4{0, 0, 0, 0};
    }
    if (tid < a.rows) a.lse[stat_base + tid] = -INFINITY;
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
    const uint16_t* qp = a.q + row_at(min(r32, a.rows - 1)) + 8 * hf;
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
    uint32_t pk[8];
    const float shift = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
    for (int u = 0; u < 8; ++u) {                        // (the sum is taken over the rounded values: see fwd.hip)
      pk[u] = pack_bf16(fast_exp2(fmaf(s[2 * u], a.scale_log2, -shift)), fast_exp2(fmaf(s[2 * u + 1], a.scale_log2, -shift)));
      l_run = dot2_ones(pk[u], l_run);
    }
    raw_copies_left<2 * NCP>();                          // and V
#pragma unroll
    for (int cc = 0; cc < 2; ++cc) {
      const bf16x8 p = __builtin_bit_cast(bf16x8, u32x4{pk[4 * cc], pk[4 * cc + 1], pk[4 * cc + 2], pk[4 * cc + 3]});
#pragma unroll
      for (int mb = 0; mb < NMB; ++mb) {
        const int o = cc * 16 * D * 2;
        oacc[mb] = mfma32(join_tr(lds_tr4_at((v0 ^ (mb << 6)) + o), lds_tr4_at((v1 ^ (mb << 6)) + o)), p, oacc[mb]);
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
  auto finish = [&](int row, int c, f32x4 x, float m, float l) {
    const float inv = 1.f / l;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] *= inv;
    const u32x2 out = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    const int64_t off = row_at(row) + 4 * c;
    *(u32x2*)(a.o + off) = out;
    if (a.o_res) {
      const u32x2 r = {pack_bf16(x[0] - __builtin_bit_cast(float, out[0] << 16), x[1] - __builtin_bit_cast(float, out[0] & 0xffff0000u)),
                       pack_bf16(x[2] - __builtin_bit_cast(float, out[1] << 16), x[3] - __builtin_bit_cast(float, out[1] & 0xffff0000u))};
      *(u32x2*)(a.o_res + off) = r;
    }
    if (c == 0) a.lse[stat_base + row] = m * LN2 + __logf(l);
  };
  auto weight = [](float m_p, float m) -> float { return m_p == -INFINITY ? 0.f : fast_exp2(m_p - m); };
  float* slot = a.pool + (int64_t)pc.slot * a.slot_floats;
  for (int x = tid; x < a.rows * QUADS; x += NT) {
    const int row = x / QUADS, c = x % QUADS;
    float m = stat[0][row][0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) m = fmaxf(m, stat[i][row][0]);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      const float f = weight(stat[i][row][0], m);
      const f32x4 y = *(const f32x4*)((const float*)(smem + i * WAVE_B) + row * PITCH + 4 * c);
      l = fmaf(stat[i][row][1], f, l);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = fmaf(y[e], f, sum[e]);
    }
    if (parts == 1) {
      finish(row, c, sum, m, l);
    } else {
      part_store2(slot + row * D + 4 * c, sum[0], sum[1]);
      part_store2(slot + row * D + 4 * c + 2, sum[2], sum[3]);
      if (c == 0) part_store2(slot + a.rows * D + 2 * row, m, l);
    }
  }
  if (parts == 1) return;
  if (!last_part(a.arrive + unit, parts, &lds.word)) return;
  // the last part joins all of them, in part order
  auto part_at = [&](int p) -> const float* {
    return a.pool + (int64_t)(p == 0 ? pc.first_slot : pc.next_slots + 2 * (min(p, parts - 1) - 1)) * a.slot_floats;
  };
  for (int x = tid; x < a.rows * QUADS; x += NT) {
    const int row = x / QUADS, c = x % QUADS;
    float m = -INFINITY, l = 0.f;
    for (int p = 0; p < parts; p += 4) {                 // four loads in flight
      float mp[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) mp[i] = part_load2(part_at(p + i) + a.rows * D + 2 * row)[0];
      m = fmaxf(fmaxf(m, fmaxf(mp[0], mp[1])), fmaxf(mp[2], mp[3]));
    }
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < parts; p += 4) {
      f32x2 ml[4], lo[4], hi[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float* ps = part_at(p + i);
        ml[i] = part_load2(ps + a.rows * D + 2 * row);
        lo[i] = part_load2(ps + row * D + 4 * c);
        hi[i] = part_load2(ps + row * D + 4 * c + 2);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float f = p + i < parts ? weight(ml[i][0], m) : 0.f;
        l = fmaf(ml[i][1], f, l);
        sum[0] = fmaf(lo[i][0], f, sum[0]); sum[1] = fmaf(lo[i][1], f, sum[1]);
        sum[2] = fmaf(hi[i][0], f, sum[2]); sum[3] = fmaf(hi[i][1], f, sum[3]);
      }
    }
    finish(row, c, sum, m, l);
  }
}

template <int D>
__global__ __launch_bounds__(64 * FEW_WAVES) void cross_few_kernel(FewArgs a) {
  __shared__ __align__(1024) FewLds<D> lds;
  if (a.workers == 0) {
    const int b = blockIdx.x / a.Hk, keys = cross_length(a.kv, b);
    few_piece<D>(a, FewPiece{b, (int)blockIdx.x % a.Hk, 0, keys, 1, 0, 0, 0}, lds);
    return;
  }
  const int hk = blockIdx.x % a.Hk, i = blockIdx.x / a.Hk;
  const FewLine line = few_line(a, i, threadIdx.x & 63);
  const int slots = 2 * (hk * a.workers);                // the slots of this head's stretches
  int first = line.first;                                // of sample b
  for (int b = line.b, at = line.begin; at < line.end; ++b) {
    const int keys = cross_length(a.kv, b), n = few_blocks(keys), end = min(first + n, line.end);
    FewPiece pc;
    pc.b = b; pc.hk = hk;
    pc.key0 = (at - first) * BKV; pc.key1 = min(keys, (end - first) * BKV);
    const int i0 = first / line.per, i1 = (first + n - 1) / line.per;      // stretches that the sample lies in
    pc.parts = i1 - i0 + 1;
    pc.first_slot = slots + 2 * i0 + (first != i0 * line.per);
    pc.next_slots = slots + 2 * (i0 + 1);
    pc.slot = slots + 2 * i + (at != line.begin);
    few_piece<D>(a, pc, lds);
    __syncthreads();                                     // (the next piece's tiles land where this one's results were)
    first += n;
    at = end;
  }
}

// Workgroups of a key head that share the line of its key blocks, or 0.
static int few_workers(const CrossDims& m) {
  const int64_t units = (int64_t)m.q.B * m.Hk;
  const int resident = few_resident(m.q.d);
  if (m.q.B > FEW_SAMPLES || units >= 2 * resident) return 0;
  const int64_t most = ((int64_t)m.q.B * m.q.Tn + FEW_LEAST - 1) / FEW_LEAST, want = (resident + m.Hk - 1) / m.Hk;
  return (int)(want < most ? want : most);
}

CrossFewWs cross_few_ws(const CrossDims& m) {
  CrossFewWs w;
  w.workers = few_workers(m);
  // (one stretch a head: nothing is shared)
  w.counters = w.workers > 1 ? round256((size_t)m.q.B * m.Hk * 4) : 0;
  w.pool = w.counters;
  w.total = w.counters + (w.workers > 1 ? round256((size_t)2 * w.workers * m.Hk * few_slot_bytes(m.group * m.q.N, m.q.d)) : 0);
  return w;
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
  const CrossFewWs w = cross_few_ws(m);
  a.workers = w.workers;
  a.slot_floats = (int)(few_slot_bytes(a.rows, m.q.d) / 4);
  if (w.total) {
    a.arrive = (int32_t*)ws;
    a.pool = (float*)((char*)ws + w.pool);
    const hipError_t e = launch_zero_ints(a.arrive, m.q.B * m.Hk, stream);
    if (e != hipSuccess) return e;
  }
  const dim3 grid((unsigned)((a.workers ? a.workers : m.q.B) * m.Hk)), block(64 * FEW_WAVES);
  if (m.q.d == 128) hipLaunchKernelGGL(cross_few_kernel<128>, grid, block, 0, stream, a);
  else              hipLaunchKernelGGL(cross_few_kernel<64>, grid, block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace spa2
