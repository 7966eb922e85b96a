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
#include "window.h"

namespace spa2 {

struct FewArgs {
  static constexpr bool WINDOW = false;
  const uint16_t* q; const uint16_t* k; const uint16_t* v;
  uint16_t* o; uint16_t* o_res; float* lse;
  CrossKeys kv;
  int B, Hk, Nq, rows;           // rows = group * Nq
  int workers, least;            // workgroups of a key head that share the line of key blocks, 0: one a (sample, key head); blocks of a stretch
  int64_t sb, sh, sn;
  float scale_log2;
  float* pool; int slot_floats;  // partial results (few_slot)
};
// Attention over a window (window.h): a sample's keys are those blocks that its queries see, first ones and window in one line.
// Measured: one query, the last 4096 of up to 32,760 keys and four first ones, 8 samples, 40 heads sharing 8, d = 128 28 to 32 us
// (134 MB, 4.2 to 4.7 TB/s), the join 4.4: a workgroup has eight or nine blocks, two of a wave's eight or nine tiles on their way before
// the first is worked on.  Lengths and places are read once, together (one after another, and again for every piece: 3 us more).
struct WindowFewArgs : FewArgs {
  static constexpr bool WINDOW = true;
  Window win;
  int aim;                       // parts of a key head's samples in all, about (workers: at most)
  int32_t* plan;                 // [sample][2]: its first part, its parts; for the join
};
// A sample's keys, and the place of its first query.
struct FewSeen { int keys, start; };
template <class Args>
__device__ __forceinline__ FewSeen few_seen(const Args& a, int b) {
  FewSeen s = {cross_length(a.kv, b), 0};
  if constexpr (Args::WINDOW) s.start = window_start(a.win, b);
  return s;
}
template <class Args>
__device__ __forceinline__ WindowSpan few_span(const Args& a, FewSeen s) { return window_span(a.win, s.keys, s.start, s.start + a.win.nq - 1); }

constexpr int FEW_WAVES = 2;     // (two workgroups of 64 KB share a compute unit; of four waves and 128 KB one: 127 / 140 us)
// Blocks of a sample in the line: one at least, so that every sample is somebody's.
template <class Args>
__device__ __forceinline__ int few_blocks(const Args& a, FewSeen s) {
  if constexpr (Args::WINDOW) return max(few_span(a, s).count(), 1);
  else                        return max((s.keys + BKV - 1) / BKV, 1);
}

// Sum over the lanes of a wave.
__device__ __forceinline__ int few_sum(int x) {
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) x += __shfl_xor(x, s, 64);
  return __builtin_amdgcn_readfirstlane(x);
}
// The line, 64 samples at a time: a lane holds sample 64 c + lane's blocks (0 past the last), keys and place.  Blocks in all, blocks
// of a stretch.
// WINDOW: windows are mostly of one length, and a workgroup that takes the end of one and the start of the next waits for its first
// copies twice.  A sample's blocks are therefore cut into parts, as even as can be, of at most `per` blocks, the least that makes no more
// parts than there are workgroups, and the parts stand in the line (total: parts); where they stand goes to the join by memory.  Measured, us,
// kernel and join, one query, stretches of one line / this: 4096 keys, 8 samples, 8 key heads 33.7 + 4.5 / 28.3 + 4.3, of unlike length 31.0 + 4.6 /
// 26.8 + 4.2; one long sample among short ones, no limit to the left 35.6 + 6.6 / 27.0 + 6.0; 2048 keys, 100 samples, one head 25.6 + 5.7 / 23.2 +
// 4.2; 600 samples of 20,000 keys, one head, d = 64 515 + 24 / 566 + 8.
struct FewLine { int c, n, keys, start, total, per; };
template <class Args>
__device__ __forceinline__ void few_chunk(const Args& a, FewLine& line, int c, int lane) {
  const int b = min(64 * c + lane, a.B - 1);             // (lengths and starts are requested together)
  int keys = a.kv.Nk, start = 0;
  if constexpr (Args::WINDOW) start = a.win.starts ? a.win.starts[b] : a.win.start;
  if (a.kv.lengths) keys = a.kv.lengths[b];
  line.c = c;
  line.keys = min(max(keys, 0), a.kv.Nk);
  line.start = 0;
  if constexpr (Args::WINDOW) line.start = window_clamp(start);
  line.n = 64 * c + lane < a.B ? few_blocks(a, FewSeen{line.keys, line.start}) : 0;
}
// What the lane's sample takes of the line: blocks; parts.
template <class Args>
__device__ __forceinline__ int few_units(const FewLine& line) { return Args::WINDOW ? (line.n + line.per - 1) / line.per : line.n; }
template <class Args>
__device__ __forceinline__ FewLine few_line(const Args& a, int lane) {
  FewLine r;
  int n = 0;
  for (int c = (a.B - 1) / 64; c >= 0; --c) {
    few_chunk(a, r, c, lane);
    n += r.n;
  }
  r.total = few_sum(n);
  if constexpr (Args::WINDOW) {
    for (r.per = max((r.total + a.aim - 1) / a.aim, a.least);; r.per += max(r.per / 16, 1)) {
      n = 0;
      for (int c = (a.B - 1) / 64; c >= 0; --c) {
        if (c != r.c) few_chunk(a, r, c, lane);
        n += few_units<Args>(r);
      }
      n = few_sum(n);
      if (n <= a.workers) break;             // (at the latest with the longest sample's blocks: there are no less workgroups than samples)
    }
    r.total = n;
  } else {
    r.per = max((r.total + a.workers - 1) / a.workers, a.least);
  }
  return r;
}
// What the line holds of sample b.
template <class Args>
__device__ __forceinline__ FewSeen few_seen(const Args& a, FewLine& line, int b, int lane) {
  if (b / 64 != line.c) few_chunk(a, line, b / 64, lane);
  return FewSeen{__builtin_amdgcn_readlane(line.keys, b & 63), __builtin_amdgcn_readlane(line.start, b & 63)};
}
// First place of sample b.
template <class Args>
__device__ __forceinline__ int few_first(const Args& a, FewLine& line, int b, int lane) {
  int before = 0;
  for (int c = 0; 64 * c < b; ++c) {
    if (c != line.c) few_chunk(a, line, c, lane);
    before += 64 * c + lane < b ? few_units<Args>(line) : 0;
  }
  return few_sum(before);
}
// The sample that place `place` (inside the line) belongs to, and that sample's first place.
struct FewSample { int b, first; };
template <class Args>
__device__ __forceinline__ FewSample few_sample(const Args& a, FewLine& line, int place, int lane) {
  int run = 0;
  for (int c = 0; 64 * c < a.B; ++c) {
    if (c != line.c) few_chunk(a, line, c, lane);
    const int n = few_units<Args>(line);
    int sum = n;                                         // of this sample and those before it
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int x = __shfl_up(sum, s, 64);
      sum += lane >= s ? x : 0;
    }
    const int at = run + sum - n;
    const uint64_t here = __builtin_amdgcn_ballot_w64(n > 0 && at <= place && place < at + n);
    if (here) {
      const int l = __builtin_ctzll(here);
      return FewSample{64 * c + l, __builtin_amdgcn_readlane(at, l)};
    }
    run += __builtin_amdgcn_readlane(sum, 63);
  }
  return FewSample{0, 0};
}
// Stretches that a sample lies in, and where part p of its result lies: a stretch has two slots, for the sample that it begins
// inside of or with and for the one that it ends inside of.
// (WINDOW: parts of the sample, each of which has a slot.)
struct FewParts { int i0, parts, starts; };
template <class Args>
__device__ __forceinline__ FewParts few_parts(int first, int n, int per) {
  if constexpr (Args::WINDOW) return {first, (n + per - 1) / per, 1};
  const int i0 = first / per;
  return {i0, (first + n - 1) / per - i0 + 1, first == i0 * per};
}
template <class Args>
__device__ __forceinline__ int few_slot(const Args& a, const FewParts& s, int hk, int p) {
  if constexpr (Args::WINDOW) return hk * a.workers + s.i0 + p;
  return 2 * (hk * a.workers + s.i0 + p) + (p == 0 && !s.starts);
}

// Four channels (4 c ..) of a row's sum x with maximum m and sum of weights l: O = x / l, LSE.
__device__ __forceinline__ int64_t few_row(const FewArgs& a, int b, int hk, int r) {
  return b * a.sb + ((int64_t)hk * a.kv.group + r / a.Nq) * a.sh + (r % a.Nq) * a.sn;
}
template <class Args>
__device__ __forceinline__ void few_finish(const Args& a, int b, FewSeen seen, int hk, int row, int c, f32x4 x, float m, float l) {
  float inv = 1.f / l;
  if constexpr (Args::WINDOW) {
    if (window_blind(a.win, seen.keys, seen.start + row % a.win.nq)) inv = 0.f;
  }
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
// (WINDOW: keys of the line of the sample's blocks, so many from its start)
struct FewPiece { int b, hk, key0, key1, slot; FewSeen seen; };
template <int D, class Args>
__device__ __forceinline__ void few_piece(const Args& a, const FewPiece& pc, FewLds<D>& lds) {
  constexpr bool WINDOW = Args::WINDOW;
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
  // (WINDOW) what the sample's queries see, and this lane's: first keys and from `near` to `last`
  WindowSpan span;
  int keys = 0, start = 0, last_seen = 0, near = 0;
  if constexpr (WINDOW) {
    keys = pc.seen.keys;
    start = pc.seen.start;
    span = few_span(a, pc.seen);
    const int p = start + min(r32, a.rows - 1) % a.win.nq;
    last_seen = min(p + a.win.right, keys - 1);
    near = p - a.win.left;
  }
  auto place = [&](int t) -> int {                       // first key of this wave's tile t
    const int at = key0 + (w + WAVES * t) * TK;
    if constexpr (WINDOW) return span.block(at / BKV) * BKV + at % BKV;
    else                  return at;
  };
  auto copy_tile = [&](int t, uint32_t stage) {
    // (WINDOW: keys that none of the queries sees are not read; offsets are then those from the block's start)
    const int at = place(t);
    const bool part_seen = WINDOW && !span.whole(at / BKV);
    const int last = WINDOW ? (part_seen ? TK + at : TK - 1) : min(TK, key1 - at) - 1, origin = part_seen ? at / BKV * BKV : at;
    if (last != rows_set) {
      rows_set = last;
#pragma unroll
      for (int r = 0; r < NCP; ++r) {
        const int row = RPI * r + lane / CPR, from = part_seen ? span.stand_in(at / BKV, at + row) - origin : min(row, last);
        voff[r] = (uint32_t)((from * a.kv.sn + (((lane % CPR) ^ swz<D>(row)) * 8)) * 2);
      }
    }
    const char* kp = k_head + (uint64_t)origin * row_bytes;
    const char* vp = v_head + (uint64_t)origin * row_bytes;
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
    const int at = place(t), valid = key1 - at - 4 * hf;
    if constexpr (WINDOW) {
      if (!window_full(a.win, keys, start, start + a.win.nq - 1, at, at + TK - 1)) {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int key = at + 8 * (v >> 2) + (v & 3) + 4 * hf;
          if (key > last_seen || (key < near && key >= a.win.sinks)) s[v] = -INFINITY;
        }
      }
    } else if (valid + 4 * hf < TK) {
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
      few_finish(a, b, pc.seen, hk, row, c, sum, m, l);
    } else {
      *(f32x4*)(slot + row * D + 4 * c) = sum;
      if (c == 0) *(f32x2*)(slot + a.rows * D + 2 * row) = f32x2{m, l};
    }
  }
}

// keys of a sample's line
template <class Args>
__device__ __forceinline__ int few_keys(const Args& a, FewSeen seen) {
  if constexpr (Args::WINDOW) {
    const WindowSpan s = few_span(a, seen);
    return s.count() ? (s.count() - 1) * BKV + min(BKV, s.hi - s.block(s.count() - 1) * BKV) : 0;
  }
  return seen.keys;
}
template <int D, class Args>
__global__ __launch_bounds__(64 * FEW_WAVES) void cross_few_kernel(Args a) {
  __shared__ __align__(1024) FewLds<D> lds;
  if (a.workers == 0) {
    const int b = blockIdx.x / a.Hk;
    const FewSeen seen = few_seen(a, b);
    few_piece<D>(a, FewPiece{b, (int)blockIdx.x % a.Hk, 0, few_keys(a, seen), -1, seen}, lds);
    return;
  }
  const int hk = blockIdx.x % a.Hk, i = blockIdx.x / a.Hk, lane = threadIdx.x & 63;
  FewLine line = few_line(a, lane);
  if constexpr (Args::WINDOW) {
    if (i >= line.total) return;
    const FewSample at = few_sample(a, line, i, lane);
    const FewSeen seen = few_seen(a, line, at.b, lane);
    const int n = few_blocks(a, seen), p = i - at.first;
    const FewParts s = few_parts<Args>(at.first, n, line.per);
    if (p == 0 && hk == 0 && threadIdx.x == 0) { a.plan[2 * at.b] = s.i0; a.plan[2 * at.b + 1] = s.parts; }
    const int even = n / s.parts, more = n % s.parts, k0 = p * even + min(p, more), k1 = k0 + even + (p < more);
    few_piece<D>(a, FewPiece{at.b, hk, k0 * BKV, min(few_keys(a, seen), k1 * BKV), s.parts == 1 ? -1 : few_slot(a, s, hk, p), seen}, lds);
    return;
  }
  const int begin = i * line.per, stop = min(begin + line.per, line.total);
  if (begin >= stop) return;
  const FewSample start = few_sample(a, line, begin, lane);
  int first = start.first;                               // of sample b
  for (int b = start.b, at = begin; at < stop; ++b) {
    const FewSeen seen = few_seen(a, line, b, lane);
    const int keys = few_keys(a, seen), n = few_blocks(a, seen), end = min(first + n, stop);
    const FewParts s = few_parts<Args>(first, n, line.per);
    const FewPiece pc = {b, hk, (at - first) * BKV, min(keys, (end - first) * BKV), s.parts == 1 ? -1 : few_slot(a, s, hk, i - s.i0), seen};
    few_piece<D>(a, pc, lds);
    __syncthreads();                                     // (the next piece's tiles land where this one's results were)
    first += n;
    at = end;
  }
}

// Row `row` of a (sample, key head) whose keys several workgroups shared: their results, joined.  A thread takes four channels and
// every G-th part, in order; then the G are added in order.
template <int D, class Args>
__global__ __launch_bounds__(256) void cross_few_join_kernel(Args a) {
  constexpr int QUADS = D / 4, G = 256 / QUADS;
  __shared__ __align__(16) float sums[G][D];
  __shared__ float stat[G][2];
  const int row = blockIdx.x % a.rows, unit = blockIdx.x / a.rows, b = unit / a.Hk, hk = unit % a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, c = tid % QUADS, g = tid / QUADS;
  FewSeen seen;
  FewParts s;
  if constexpr (Args::WINDOW) {
    seen = few_seen(a, b);
    s = FewParts{scalar_ld(a.plan + 2 * b), scalar_ld(a.plan + 2 * b + 1), 1};
  } else {
    FewLine line = few_line(a, lane);
    const int first = few_first(a, line, b, lane);
    seen = few_seen(a, line, b, lane);
    s = few_parts<Args>(first, few_blocks(a, seen), line.per);
  }
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
  few_finish(a, b, seen, hk, row, c, sum, m, l);
}

template <class Args>
static hipError_t launch_few(Args& a, const void* q, const void* k, const void* v, const CrossDims& m, const int32_t* lengths, float scale,
                             void* o, void* o_res, float* lse, const CrossFewWs& share, void* ws, hipStream_t stream) {
  a.q = (const uint16_t*)q; a.k = (const uint16_t*)k; a.v = (const uint16_t*)v;
  a.o = (uint16_t*)o; a.o_res = (uint16_t*)o_res; a.lse = lse;
  a.kv = cross_keys(m, lengths);
  a.B = m.q.B; a.Hk = m.Hk; a.Nq = m.q.N; a.rows = m.group * m.q.N;
  a.sb = m.q.sb; a.sh = m.q.sh; a.sn = m.q.sn;
  a.scale_log2 = scale * LOG2E;
  a.workers = share.workers; a.least = share.least;
  a.pool = (float*)ws;
  a.slot_floats = (int)(few_slot_bytes(a.rows, m.q.d) / 4);
  const dim3 grid((unsigned)((a.workers ? a.workers : m.q.B) * m.Hk)), block(64 * FEW_WAVES);
  if (m.q.d == 128) hipLaunchKernelGGL((cross_few_kernel<128, Args>), grid, block, 0, stream, a);
  else              hipLaunchKernelGGL((cross_few_kernel<64, Args>), grid, block, 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.workers <= 1) return e;
  const dim3 rows((unsigned)(m.q.B * m.Hk * a.rows));
  if (m.q.d == 128) hipLaunchKernelGGL((cross_few_join_kernel<128, Args>), rows, dim3(256), 0, stream, a);
  else              hipLaunchKernelGGL((cross_few_join_kernel<64, Args>), rows, dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_cross_few(const void* q, const void* k, const void* v, const CrossDims& m, const int32_t* lengths, float scale,
                            void* o, void* o_res, float* lse, void* ws, hipStream_t stream) {
  FewArgs a = {};
  return launch_few(a, q, k, v, m, lengths, scale, o, o_res, lse, cross_few_ws(m), ws, stream);
}
hipError_t launch_window_few(const void* q, const void* k, const void* v, const CrossDims& m, const int32_t* lengths, const Window& win,
                             float scale, void* o, void* o_res, float* lse, void* ws, hipStream_t stream) {
  WindowFewArgs a = {};
  a.win = win;
  const WindowFewWs share = window_few_ws(m, win);
  a.aim = share.aim;
  a.plan = (int32_t*)((char*)ws + share.plan);
  return launch_few(a, q, k, v, m, lengths, scale, o, o_res, lse, share, ws, stream);
}

}  // namespace spa2
