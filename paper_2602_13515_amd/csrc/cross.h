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
// not fill the chip: as many parts as give the fullest rounds of `resident` workgroups, over one to four rounds, and no
// parts below `least` entries.
struct CrossParts { int len, parts; };
inline CrossParts cross_parts(int64_t units, int list_max, int resident, int least) {
  CrossParts best = {list_max, 1};
  double fill = 0.0;
  for (int rounds = 1; rounds <= 4; ++rounds) {
    int64_t parts = (int64_t)rounds * resident / units;
    if (parts > (list_max + least - 1) / least) parts = (list_max + least - 1) / least;
    if (parts < 1) continue;
    const int len = (int)((list_max + parts - 1) / parts);
    const int made = (list_max + len - 1) / len;
    const int64_t wgs = units * made;
    const double f = (double)units * list_max / ((double)((wgs + resident - 1) / resident) * resident * len);
    if (f > 1.02 * fill) { fill = f; best = {len, made}; }
  }
  return best;
}

// What a kernel needs of a workspace: arrival counters (zeroed before the launch) and partial results, one of each a part.
struct CrossSection { CrossParts cut; int slots; size_t counters, pool; };
inline CrossSection cross_section(int64_t units, int list_max, int resident, int least, size_t slot_bytes) {
  CrossSection s;
  s.cut = cross_parts(units, list_max, resident, least);
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

CrossSection cross_fwd_section(const CrossDims& m);
CrossSection cross_dq_section(const CrossDims& m);
CrossSection cross_dkdv_section(const CrossDims& m);

// Workspace of the forward pass: counters, pool.  Of the backward pass: D, counters of dK/dV and of dQ, pools.
struct CrossFwdWs { CrossSection s; size_t pool, total; };
inline CrossFwdWs cross_fwd_ws(const CrossDims& m) {
  CrossFwdWs w;
  w.s = cross_fwd_section(m);
  w.pool = w.s.counters;
  w.total = w.pool + w.s.pool;
  return w;
}
struct CrossBwdWs { CrossSection dkdv, dq; size_t dkdv_counters, dq_counters, dkdv_pool, dq_pool, total; };
inline CrossBwdWs cross_bwd_ws(const CrossDims& m) {
  CrossBwdWs w;
  w.dkdv = cross_dkdv_section(m);
  w.dq = cross_dq_section(m);
  w.dkdv_counters = round256((size_t)m.q.B * m.q.H * m.q.N * sizeof(float));
  w.dq_counters = w.dkdv_counters + w.dkdv.counters;
  w.dkdv_pool = w.dq_counters + w.dq.counters;
  w.dq_pool = w.dkdv_pool + w.dkdv.pool;
  w.total = w.dq_pool + w.dq.pool;
  return w;
}

hipError_t launch_cross_fwd(const void* q, const void* k, const void* v, const CrossDims& m, const int32_t* lengths, float scale,
                            void* o, void* o_res, float* lse, void* ws, hipStream_t stream);
hipError_t launch_cross_delta(const void* o, const void* o_res, const void* d_o, const CrossDims& m, float* delta, int32_t* zero,
                              int zeros, hipStream_t stream);
hipError_t launch_cross_dq(const void* q, const void* k, const void* v, const void* d_o, const float* lse, const float* delta,
                           const CrossDims& m, const int32_t* lengths, float scale, void* dq, const SplitPlan& plan,
                           hipStream_t stream);
hipError_t launch_cross_dkdv(const void* q, const void* k, const void* v, const void* d_o, const float* lse, const float* delta,
                             const CrossDims& m, const int32_t* lengths, float scale, void* dk, void* dv, const SplitPlan& plan,
                             hipStream_t stream);

}  // namespace spa2
