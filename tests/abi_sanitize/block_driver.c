/* Host-only exerciser of the argument checks of the operators around the attention, built with AddressSanitizer and
 * UndefinedBehaviorSanitizer (see driver.c): sizes and strides at the ends of their types, every call rejected before a launch. */
#include <limits.h>
#include <math.h>
#include <stdio.h>

#include "spa2.h"

static int failures = 0;
#define EXPECT(call, code)                                                                  \
  do {                                                                                      \
    int rc_ = (call);                                                                       \
    if (rc_ != (code)) { printf("line %d: got %d, expected %d\n", __LINE__, rc_, (code)); ++failures; } \
  } while (0)

int main(void) {
  void* fake = (void*)0x1000;
  void* odd = (void*)0x1004;
  float* f = (float*)fake;
  const size_t big = (size_t)1 << 60;
  spa2_norm_shape n = {2, 4, 2, 10, 128, 0, 128, 0, 10, 0, 0, 5120, 128, 512, 2560, 128, 256, 5120, 128, 512, 2560, 128, 256}, x;
  spa2_cross_shape c = {2, 4, 2, 10, 20, 128, 5120, 128, 512, 5120, 128, 256, 5120, 128, 256}, y;
#define NORM(s) spa2_norm_rotate(fake, fake, f, f, f, f, 0, &s, 1e-6f, fake, fake, 0)
#define NORM_BWD(s, ws, bytes) spa2_norm_rotate_bwd(fake, fake, f, f, f, f, 0, fake, fake, &s, 1e-6f, fake, fake, f, f, ws, bytes, 0)
#define CROSS(s) spa2_cross_fwd(fake, fake, fake, 0, &s, 0.1f, fake, 0, f, fake, big, 0)
#define CROSS_BWD(s, ws, bytes) spa2_cross_bwd(fake, fake, fake, 0, fake, 0, fake, f, &s, 0.1f, fake, fake, fake, ws, bytes, 0)
  x = n; x.B = x.N = x.Hq = x.Hk = INT_MAX; x.table_rows = INT_MAX;
  EXPECT(NORM(x), SPA2_ERR_SHAPE); EXPECT(NORM_BWD(x, fake, big), SPA2_ERR_SHAPE);
  EXPECT(spa2_norm_rotate_bwd_workspace_bytes(&x) != 0, 0);
  x = n; x.B = INT_MIN; EXPECT(NORM(x), SPA2_ERR_SHAPE);
  x = n; x.rot = INT_MIN; EXPECT(NORM(x), SPA2_ERR_UNSUPPORTED);
  x = n; x.rot = INT_MAX; EXPECT(NORM(x), SPA2_ERR_UNSUPPORTED);
  x = n; x.q_sb = LLONG_MIN; EXPECT(NORM(x), SPA2_ERR_SHAPE);
  x = n; x.q_sb = LLONG_MAX; EXPECT(NORM(x), SPA2_ERR_ALIGN);
  x = n; x.pos_sb = -1; EXPECT(NORM(x), SPA2_ERR_SHAPE);
  x = n; x.pos_bits = 64; EXPECT(NORM(x), SPA2_ERR_NULL);
  EXPECT(NORM_BWD(n, 0, big), SPA2_ERR_WORKSPACE); EXPECT(NORM_BWD(n, fake, 1), SPA2_ERR_WORKSPACE);
  EXPECT(NORM_BWD(n, odd, big), SPA2_ERR_ALIGN);
  EXPECT(spa2_norm_rotate(fake, fake, f, f, f, f, 0, 0, 1e-6f, fake, fake, 0), SPA2_ERR_NULL);
  EXPECT(spa2_norm_rotate(fake, fake, f, f, f, f, 0, &n, NAN, fake, fake, 0), SPA2_ERR_RANGE);
  EXPECT(spa2_norm_rotate(fake, fake, f, (float*)odd, f, f, 0, &n, 1e-6f, fake, fake, 0), SPA2_ERR_ALIGN);

  y = c; y.B = y.Hq = y.Hk = y.Nq = y.Nk = INT_MAX;
  EXPECT(CROSS(y), SPA2_ERR_SHAPE); EXPECT(CROSS_BWD(y, fake, big), SPA2_ERR_SHAPE);
  EXPECT(spa2_cross_fwd_workspace_bytes(&y) != 0 || spa2_cross_bwd_workspace_bytes(&y) != 0, 0);
  y = c; y.Hq = INT_MIN; EXPECT(CROSS(y), SPA2_ERR_SHAPE);
  y = c; y.Nq = INT_MAX; EXPECT(CROSS(y), SPA2_ERR_SHAPE);
  y = c; y.Nk = INT_MAX; EXPECT(CROSS(y), SPA2_ERR_SHAPE);
  y = c; y.q_sh = LLONG_MAX - 7; y.Nq = 1; EXPECT(CROSS_BWD(y, fake, 1), SPA2_ERR_WORKSPACE);        /* (a stride too long to join heads by) */
  y = c; y.k_sn = LLONG_MAX; EXPECT(CROSS(y), SPA2_ERR_SHAPE);
  y = c; y.d_sn = LLONG_MIN; EXPECT(CROSS_BWD(y, fake, big), SPA2_ERR_SHAPE);
  EXPECT(CROSS_BWD(c, 0, big), SPA2_ERR_WORKSPACE); EXPECT(CROSS_BWD(c, fake, 64), SPA2_ERR_WORKSPACE);
  EXPECT(CROSS_BWD(c, odd, big), SPA2_ERR_ALIGN);
  EXPECT(spa2_cross_fwd(fake, fake, fake, (const int32_t*)0x1001, &c, 0.1f, fake, 0, f, fake, big, 0), SPA2_ERR_ALIGN);
  EXPECT(spa2_cross_fwd(fake, fake, fake, 0, &c, INFINITY, fake, 0, f, fake, big, 0), SPA2_ERR_RANGE);

  EXPECT(spa2_dropout_add(fake, 0, LLONG_MIN, 0, 0, 0.5, 1, 2, 0, fake, 0), SPA2_ERR_SHAPE);
  EXPECT(spa2_dropout_add(fake, 0, 8, INT_MAX, 0, 0.5, 1, 2, 0, fake, 0), SPA2_ERR_UNSUPPORTED);
  EXPECT(spa2_dropout_add(fake, 0, 8, 0, 0, HUGE_VAL, 1, 2, 0, fake, 0), SPA2_ERR_RANGE);
  EXPECT(spa2_dropout_add(fake, 0, 8, 0, 0, NAN, 1, 2, 0, fake, 0), SPA2_ERR_RANGE);
  EXPECT(spa2_dropout_bwd(fake, 8, 0, 0, -HUGE_VAL, 1, 2, 0, fake, 0), SPA2_ERR_RANGE);
  EXPECT(spa2_dropout_bwd(fake, 8, 0, 0, 0.5, 1, 2, (const int64_t*)odd, fake, 0), SPA2_ERR_ALIGN);
  if (!failures) printf("all rejected before launch\n");
  return failures != 0;
}
