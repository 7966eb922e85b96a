// Host-only check of which blocks attention over a window walks (csrc/window.h), against every pair written out: lists hold what is
// seen and nothing twice, copies read keys that some query sees, "all of them see all of it" holds, lists and parts fit the
// sizes that the host cuts by.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "window.h"

namespace spa2 {
size_t fwd_slot_bytes(const Dims& m) { return (size_t)(256 * (m.d / 2) + 512) * 4; }
size_t dq_slot_bytes(const Dims& m) { return (size_t)256 * (m.d / 2) * 4; }
size_t dkdv_slot_bytes(const Dims& m) { return (size_t)4 * (m.d / 32) * 16 * 64 * 4; }
}  // namespace spa2
using namespace spa2;

#define CHECK(x)                                                                                              \
  do {                                                                                                        \
    if (!(x)) {                                                                                               \
      std::printf("line %d: %s (Nq %d Nk %d keys %d start %d left %d right %d sinks %d rows %d)\n", __LINE__, #x, \
                  w.nq, Nk, keys, start, w.left, w.right, w.sinks, rows);                                      \
      return 1;                                                                                               \
    }                                                                                                         \
  } while (0)

int main() {
  std::mt19937 g(7);
  auto pick = [&](int lo, int hi) { return (int)(lo + g() % (uint32_t)(hi - lo + 1)); };
  for (int round = 0; round < 1500; ++round) {
    const int small = round % 3;
    const int Nk = pick(1, small ? 700 : 150), Nq = pick(1, small ? 700 : 150), group = pick(1, 3);
    int keys = pick(0, 4) ? pick(0, Nk) : Nk, start = pick(-900, 1200);
    if (round % 50 == 1) start = pick(0, 1) ? -2000000000 : 2000000000;
    start = window_clamp(start);
    Window w = {nullptr, start, pick(0, 5) ? pick(0, small == 1 ? 900 : 70) : WINDOW_NO_LIMIT, pick(0, 3) ? pick(0, small == 2 ? 300 : 0) : WINDOW_NO_LIMIT, 0, Nq};
    if (pick(0, 4) == 0) w.left = WINDOW_MOST;
    w.sinks = w.left == WINDOW_NO_LIMIT ? 0 : pick(0, 2) ? pick(0, Nk < 200 ? Nk : 200) : 0;
    const bool joined = Nq <= 64 && round % 2;
    const int rows = joined ? Nq * group : Nq;
    auto sees = [&](int p, int j) {
      return j >= 0 && j < keys && (long)j <= (long)p + w.right && ((long)j >= (long)p - w.left || j < w.sinks);
    };
    CrossDims m = {};
    m.q.B = pick(1, 3); m.q.H = joined ? 1 : group; m.Hk = 1; m.group = joined ? 1 : group; m.Nk = Nk;
    m.q.N = rows; m.q.d = 128; m.q.Tm = (rows + BQ - 1) / BQ; m.q.Tn = (Nk + BKV - 1) / BKV;
    const CrossSection fwd = window_fwd_section(m, w);
    for (int i = 0; i < m.q.Tm; ++i) {
      int p0, p1;
      const int r1 = i * BQ + BQ < rows ? i * BQ + BQ - 1 : rows - 1;
      window_places(w, start, rows, i * BQ, r1, p0, p1);
      const WindowSpan s = window_span(w, keys, p0, p1);
      std::vector<int> listed(Nk / BKV + 2, 0);
      CHECK(s.count() >= 0 && s.count() <= window_row_list(m, w));
      CHECK((s.count() + fwd.cut.len - 1) / fwd.cut.len <= fwd.cut.parts);
      for (int t = 0; t < s.count(); ++t) {
        CHECK(s.block(t) >= 0 && s.block(t) < m.q.Tn && (t == 0 || s.block(t) > s.block(t - 1)));
        listed[s.block(t)] = 1;
      }
      std::vector<char> any(Nk, 0);
      for (int r = i * BQ; r <= r1; ++r) {
        const int p = window_place(w, start, rows, r);
        CHECK(p >= p0 && p <= p1);
        bool blind = true;
        for (int j = 0; j < keys; ++j)
          if (sees(p, j)) { any[j] = 1; blind = false; }
        CHECK(blind == window_blind(w, keys, p));
      }
      for (int j = 0; j < Nk; ++j) CHECK(!any[j] || listed[j / BKV]);
      for (int t = 0; t < s.count(); ++t) {
        const int j = s.block(t);
        bool whole = true;
        for (int x = 0; x < BKV; ++x) {
          const int key = j * BKV + x, from = s.stand_in(j, key);
          const bool seen = key < Nk && any[key];
          whole = whole && seen;
          CHECK(from >= j * BKV && from < j * BKV + BKV && from < keys && any[from]);
          CHECK(!seen || from == key);
        }
        CHECK(!s.whole(j) || whole);
        CHECK(window_blocks(s.sinks, s.lo, s.hi).has(j) == s.whole(j));
        for (int wave = 0; wave < 4; ++wave) {
          int q0, q1;
          window_places(w, start, rows, i * BQ + 32 * wave, i * BQ + 32 * wave + 31, q0, q1);
          const bool full = window_full(w, keys, q0, q1, j * BKV, j * BKV + BKV - 1);
          CHECK(window_full_blocks(w, keys, q0, q1).has(j) == full);
          if (!full) continue;
          for (int r = i * BQ + 32 * wave; r < i * BQ + 32 * wave + 32 && r < rows; ++r)
            for (int x = 0; x < BKV; ++x) CHECK(sees(window_place(w, start, rows, r), j * BKV + x));
        }
      }
    }
    if (joined) continue;
    const WindowColumns cols = window_columns(m, w);
    CHECK(cols.blocks <= m.q.Tn && cols.blocks * BKV >= (w.sinks < Nk ? w.sinks : Nk));
    for (int j = 0; j < m.q.Tn; ++j) {
      const int last = (j * BKV + BKV < keys ? j * BKV + BKV : keys) - 1;
      const WindowRows r = window_rows(w, start, Nq, j * BKV, last);
      for (int i = 0; i < Nq; ++i) {
        bool seen = false;
        for (int key = j * BKV; key <= last; ++key) seen = seen || sees(start + i, key);
        CHECK(seen == (i >= r.r0 && i <= r.r1));
      }
      const int halves = r.r1 < r.r0 ? 0 : r.r1 / 64 - r.r0 / 64 + 1, all = group * halves;
      const CrossSection& cut = j < cols.blocks ? cols.first : cols.rest;
      CHECK(j < cols.blocks || halves <= window_column_list(m, w));
      CHECK((all + cut.cut.len - 1) / cut.cut.len <= cut.cut.parts);
      CHECK(cut.cut.parts == 1 || cut.slots == (int)(m.q.B * m.Hk * (j < cols.blocks ? cols.blocks : m.q.Tn - cols.blocks) * cut.cut.parts));
    }
    CHECK(cols.total >= cols.counters + (size_t)(cols.first.slots + cols.rest.slots) * dkdv_slot_bytes(m.q));
  }
  for (int heads : {1, 2, 3, 8, 12, 40, 300})
    for (int blocks : {0, 1, 7, 15, 16, 17, 33, 100, 256, 487, 512, 591})
      for (int turn = 0; turn < 6; ++turn) {
        const Window w = {nullptr, 0, turn % 3 == 1 ? WINDOW_NO_LIMIT : 5, turn % 3 == 2 ? WINDOW_NO_LIMIT : 7, 0, 100};
        CrossDims m = {};
        m.Nk = 1000; m.q.d = 128;
        const WindowDeal d = window_deal(w, m, heads, blocks, turn < 3);
        std::vector<int> seen((size_t)heads * blocks, 0);
        for (int wg = 0; wg < d.wgs; ++wg) {
          const HeadBlock hb = window_dealt(d, wg);
          if (!hb.valid) continue;
          if (hb.bh < 0 || hb.bh >= heads || hb.blk < 0 || hb.blk >= blocks) { std::printf("dealt outside\n"); return 1; }
          ++seen[(size_t)hb.bh * blocks + hb.blk];
        }
        for (int n : seen)
          if (n != 1) { std::printf("%d heads of %d blocks: one is dealt %d times\n", heads, blocks, n); return 1; }
      }
  std::printf("windows hold\n");
  return 0;
}
