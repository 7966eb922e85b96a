// Argument checks and sizes that the entry points of attention to another sequence and of attention over a window share (host side).
#pragma once
#include "cross.h"
#include "spa2_check.h"

namespace spa2 {

constexpr int64_t CROSS_MAX_BLOCKS = 1 << 23;       // workgroups are numbered in 32 bits, also in threads

// a stride triple of bf16 heads
inline int check_strides(int64_t sb, int64_t sh, int64_t sn, int64_t least, int d) {
  if (sb < least || sh < least || sn < d || sn > SPA2_MAX_TOKEN_STRIDE) return SPA2_ERR_SHAPE;
  return sb % 8 || sh % 8 || sn % 8 ? SPA2_ERR_ALIGN : SPA2_OK;
}

inline int check_cross_shape(const spa2_cross_shape* s) {
  if (!s) return SPA2_ERR_NULL;
  if (s->B <= 0 || s->Hq <= 0 || s->Hk <= 0 || s->Nq <= 0 || s->Nk <= 0 || s->d <= 0 || s->Hq % s->Hk) return SPA2_ERR_SHAPE;
  if (s->d != 64 && s->d != 128) return SPA2_ERR_UNSUPPORTED;
  const int64_t tm = ((int64_t)s->Nq + SPA2_BQ - 1) / SPA2_BQ, tn = ((int64_t)s->Nk + SPA2_BKV - 1) / SPA2_BKV;
  if ((int64_t)s->B * s->Hq > CROSS_MAX_BLOCKS || (int64_t)s->B * s->Hq * tm > CROSS_MAX_BLOCKS ||
      (int64_t)s->B * s->Hk * tn > CROSS_MAX_BLOCKS)
    return SPA2_ERR_SHAPE;
  int rc = check_strides(s->q_sb, s->q_sh, s->q_sn, 1, s->d);
  if (rc == SPA2_OK) rc = check_strides(s->k_sb, s->k_sh, s->k_sn, 0, s->d);
  return rc;
}

// The query heads of a key head are taken as one head of more rows where a stride says so (one query a head, or heads whose
// queries follow each other in memory): their keys and values are then read once, not once a head.  One query, 8 samples of up
// to 32,760 keys, 40 heads sharing 8, d = 128, by the kernel for many rows: 554 us head by head, 168 together (by the one for few rows 113).
// `most`: queries of a head up to which this is done.
inline CrossDims cross_dims(const spa2_cross_shape& s, int most = 1 << 30) {
  CrossDims m;
  m.q.B = s.B; m.q.H = s.Hq; m.q.N = s.Nq; m.q.d = s.d;
  m.q.sb = s.q_sb; m.q.sh = s.q_sh; m.q.sn = s.q_sn;
  m.Hk = s.Hk; m.Nk = s.Nk; m.group = s.Hq / s.Hk;
  const int64_t step = s.Nq == 1 ? s.q_sh : s.q_sn;
  if (m.group > 1 && s.Nq <= most && (int64_t)m.group * s.Nq <= 1 << 30 && s.q_sh == s.Nq * step && step >= s.d && step <= SPA2_MAX_TOKEN_STRIDE) {
    m.q.H = s.Hk; m.q.N = m.group * s.Nq;
    m.q.sh = m.group * s.q_sh; m.q.sn = step;
    m.group = 1;
  }
  m.q.Tm = (m.q.N + SPA2_BQ - 1) / SPA2_BQ;
  m.q.Tn = (s.Nk + SPA2_BKV - 1) / SPA2_BKV;
  m.ksb = s.k_sb; m.ksh = s.k_sh; m.ksn = s.k_sn;
  m.dsb = s.d_sb; m.dsh = s.d_sh; m.dsn = s.d_sn;
  return m;
}

}  // namespace spa2
