// Attention to another sequence: what its kernels, which are the block-sparse ones over whole rows and columns, have besides
// their arguments, and how a launch's lists are cut.
#pragma once
#include "spa2_check.h"
#include "spa2_internal.h"

namespace spa2 {

struct CrossDims {
  Dims q;                        // of q, o, dO, dQ: H query heads, N queries, T_m blocks of them; T_n blocks of keys
  int Hk, Nk, group;             // key heads, keys, query heads of a key head
  int64_t ksb, ksh, ksn;         // strides of k and v
  int64_t dsb, dsh, dsn;         // of dK and dV
};

// keys of a sample (lengths: device, [B], or null)
struct CrossKeys {
  const int32_t* lengths;
  int Nk, group;
  int64_t sb, sh, sn;
};
inline CrossKeys cross_keys(const CrossDims& m, const int32_t* lengths) { return {lengths, m.Nk, m.group, m.ksb, m.ksh, m.ksn}; }

// Every list of a launch has up to list_max entries; a unit's list is cut into parts of len entries where the units alone do
// not fill the chip.  The cut with the least estimated time, in entries: rounds of `resident` workgroups that each take `start`
// besides their entries, and a part's results joined, `join` each.  Lists of rows end with their sample's
// keys, which only the device knows: for these (`ragged`) the mean of that time and of the one where half of all entries are
// there, in lists of any length (the mean load, then the longest part).  Measured, dK/dV of 96 columns of 256 query blocks, d = 128:
// 5 parts a column 222 us; 16 parts, the fullest rounds, 265 (the last part to arrive adds up 16 times 64 KB).
struct CrossParts { int len, parts; };
struct CutCost { double start, join; int least; bool ragged; };
inline CrossParts cross_parts(int64_t units, int list_max, int resident, const CutCost& c) {
  CrossParts best = {list_max, 1};
  double least = 0.0;
  for (int want = 1; want <= (list_max + c.least - 1) / c.least && units * want <= 4 * (int64_t)resident && units * want <= SPLIT_POOL_MAX; ++want) {
    const int len = (list_max + want - 1) / want, made = (list_max + len - 1) / len;
    const int64_t wgs = units * made;
    const double joins = made > 1 ? made * c.join : 0.0;
    double t = (double)((wgs + resident - 1) / resident) * (len + c.start) + joins;
    if (c.ragged)
      t = 0.5 * (t + 0.5 * (double)units * list_max / resident + c.start * (double)((wgs / 2 + resident) / resident) + len + joins);
    if (want == 1 || t < 0.98 * least) { least = t; best = {len, made}; }
  }
  return best;
}

// What a kernel needs of a workspace: a partial result for each part, and arrival counters (dK/dV: the last part of a column to
// arrive adds up all of them; the counters are set to zero by the launch in front).
struct CrossSection { CrossParts cut; int slots; size_t counters, pool; };
inline CrossSection cross_section(int64_t units, int list_max, int resident, const CutCost& cost, size_t slot_bytes) {
  CrossSection s;
  s.cut = cross_parts(units, list_max, resident, cost);
  s.slots = s.cut.parts > 1 ? (int)(units * s.cut.parts) : 0;
  s.counters = round256((size_t)s.slots * 4);
  s.pool = round256((size_t)s.slots * slot_bytes);
  return s;
}
inline SplitPlan cross_plan(const CrossSection& s, void* counters, void* pool, size_t slot_bytes) {
  SplitPlan p = {};
  p.planned = true;
  p.fixed_len = s.cut.len;
  p.fixed_parts = s.cut.parts;
  if (!s.slots) return p;
  p.pool_slots = (int)s.slots;
  p.slot_floats = (int)(slot_bytes / 4);
  p.arrive = (int32_t*)counters;
  p.pool = (float*)pool;
  return p;
}

// (start and join in key blocks of 128 rows, or query blocks of 64 keys)
inline CrossSection cross_fwd_section(const CrossDims& m) {
  return cross_section((int64_t)m.q.B * m.q.H * m.q.Tm, m.q.Tn, RESIDENT_WGS, CutCost{3.5, 0.03, 8, true}, fwd_slot_bytes(m.q));
}
inline CrossSection cross_dq_section(const CrossDims& m) {
  return cross_section((int64_t)m.q.B * m.q.H * m.q.Tm, m.q.Tn, RESIDENT_WGS, CutCost{3.5, 0.03, 8, true}, dq_slot_bytes(m.q));
}
inline CrossSection cross_dkdv_section(const CrossDims& m) {
  return cross_section((int64_t)m.q.B * m.Hk * m.q.Tn, m.group * m.q.Tm, dkdv_resident(m.q), CutCost{1.3, 0.4, 4, false},
                       dkdv_slot_bytes(m.q));
}

// Workspace of the forward pass: the pool.  Of the backward pass: D, LSE, counters of dK/dV, pools.
constexpr int FEW_ROWS = 32;
// Whether the rows that read a key head are so few that the kernel for few rows takes them (a wave's 32).  With 32 rows, us, that
// kernel / the other: 8 samples of 8192 keys, 8 heads 56 / 74, d = 64 34 / 36; 64 samples of 512 27 / 27; 1 of 65,536, 2 heads 29 / 61;
// 600 of 77, 4 heads, d = 64 21 / 22; 2 of 77, 40 heads 8.1 / 6.6; with one row 50 / 76, 30 / 36, 24 / 25, 26 / 59, 16 / 22, 6.2 / 6.2.
// The backward pass of such rows takes P and dS into their products in two bf16 parts: nothing averages over so few rows, and one
// part leaves an error of dQ, dK and dV of sqrt(2), for single rows and keys up to 2.2, times that of their own rounding to bf16; two
// leave that alone.  Two parts / one, us: 8 samples of 8192 keys, 8 heads of 32 rows 285 / 270, d = 64 109 / 97; 64 samples of 512, one
// row 128 / 118; 1 of 65,536, 2 heads, one row 124 / 114; 600 of 77, 4 heads of 32 rows, d = 64 69 / 64; 2 of 77, 40 heads 19.4 / 18.2.
inline bool cross_few(const CrossDims& m) { return (int64_t)m.group * m.q.N <= FEW_ROWS; }
// The kernel for few rows: workgroups of a key head that share the line of its key blocks (cross_few.hip), or 0; a part's result:
// [row][D] unnormalised sums, then (maximum in log2 units, sum) of each row.
constexpr int FEW_LEAST = 8;            // key blocks that a stretch of the line has at least (without a window)
constexpr int FEW_SAMPLES = 1024;       // samples that a line may have
inline size_t few_slot_bytes(int rows, int d) { return ((size_t)rows * (d + 2) * 4 + 15) & ~(size_t)15; }
struct CrossFewWs { int workers, least; size_t total; };
inline CrossFewWs cross_few_ws(const CrossDims& m, int least = FEW_LEAST) {
  CrossFewWs w = {0, least, 0};
  const int64_t units = (int64_t)m.q.B * m.Hk, resident = 512 * 128 / m.q.d;        // (workgroups that run at a time)
  if (m.q.B > FEW_SAMPLES || units >= 2 * resident || m.q.Tn < 2 * least) return w;
  const int64_t most = ((int64_t)m.q.B * m.q.Tn + least - 1) / least, want = (resident + m.Hk - 1) / m.Hk;
  w.workers = (int)(want < most ? want : most);
  // (one stretch a head: nothing is shared)
  if (w.workers > 1) w.total = round256((size_t)2 * w.workers * m.Hk * few_slot_bytes(m.group * m.q.N, m.q.d));
  return w;
}
struct CrossFwdWs { CrossSection s; size_t total; };
inline CrossFwdWs cross_fwd_ws(const CrossDims& m) {
  CrossFwdWs w;
  w.s = cross_fwd_section(m);
  w.total = w.s.pool;
  return w;
}
struct CrossBwdWs { CrossSection dkdv, dq; size_t lse, dkdv_counters, dkdv_pool, dq_pool, total; };
inline CrossBwdWs cross_bwd_ws(const CrossDims& m) {
  CrossBwdWs w;
  w.dkdv = cross_dkdv_section(m);
  w.dq = cross_dq_section(m);
  w.lse = round256((size_t)m.q.B * m.q.H * m.q.N * sizeof(float));
  w.dkdv_counters = 2 * w.lse;
  w.dkdv_pool = w.dkdv_counters + w.dkdv.counters;
  w.dq_pool = w.dkdv_pool + w.dkdv.pool;
  w.total = w.dq_pool + w.dq.pool;
  return w;
}

hipError_t launch_cross_few(const void* q, const void* k, const void* v, const CrossDims& m, const int32_t* lengths, float scale,
                            void* o, void* o_res, float* lse, void* ws, hipStream_t stream);
hipError_t launch_cross_fwd(const void* q, const void* k, const void* v, const CrossDims& m, const int32_t* lengths, float scale,
                            void* o, void* o_res, float* lse, void* ws, hipStream_t stream);
// (delta, lse_out: D and LSE, written here for the dK/dV kernel; zero: integers that the launch sets to zero for it)
hipError_t launch_cross_dq(const void* q, const void* k, const void* v, const void* o, const void* o_res, const void* d_o,
                           const float* lse, const CrossDims& m, const int32_t* lengths, float scale, float* delta, float* lse_out,
                           void* dq, int32_t* zero, int zeros, const SplitPlan& plan, hipStream_t stream);
hipError_t launch_cross_dkdv(const void* q, const void* k, const void* v, const void* d_o, const float* lse, const float* delta,
                             const CrossDims& m, const int32_t* lengths, float scale, void* dk, void* dv, const SplitPlan& plan,
                             hipStream_t stream);

}  // namespace spa2
