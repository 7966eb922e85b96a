/* Host-only exerciser of the argument checks of the operators of a training step, built with AddressSanitizer and
 * UndefinedBehaviorSanitizer (see driver.c): sizes, strides and limits at the ends of their types, every call rejected before a launch. */
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
  void* odd = (void*)0x1001;
  float* f = (float*)fake;
  const size_t big = (size_t)1 << 60;
  const int limits[] = {INT_MIN, -1, 0, 1, 4096, 1 << 28};
  spa2_cross_shape c = {2, 4, 2, 10, 20, 128, 5120, 128, 512, 5120, 128, 256, 5120, 128, 256}, y;
  spa2_window w = {5, 0, 3}, z;
#define WINDOW(s, l) spa2_window_fwd(fake, fake, fake, 0, 0, &s, &l, 0.1f, fake, 0, f, fake, big, 0)
#define WINDOW_BWD(s, l, ws, bytes) spa2_window_bwd(fake, fake, fake, 0, 0, fake, 0, fake, f, &s, &l, 0.1f, fake, fake, fake, ws, bytes, 0)
  y = c; y.B = y.Hq = y.Hk = y.Nq = y.Nk = INT_MAX;
  EXPECT(WINDOW(y, w), SPA2_ERR_SHAPE); EXPECT(WINDOW_BWD(y, w, fake, big), SPA2_ERR_SHAPE);
  EXPECT(spa2_window_fwd_workspace_bytes(&y, &w) != 0 || spa2_window_bwd_workspace_bytes(&y, &w) != 0, 0);
  y = c; y.B = y.Hq = y.Hk = 1; y.Nq = (1 << 28) + 1; EXPECT(WINDOW(y, w), SPA2_ERR_SHAPE);
  y = c; y.B = y.Hq = y.Hk = 1; y.Nk = (1 << 28) + 1; EXPECT(WINDOW_BWD(y, w, fake, big), SPA2_ERR_SHAPE);
  z = w; z.left = (1 << 28) + 1; EXPECT(WINDOW(c, z), SPA2_ERR_RANGE);
  z = w; z.right = INT_MAX; EXPECT(WINDOW(c, z), SPA2_ERR_RANGE);
  z = w; z.sinks = INT_MAX; EXPECT(WINDOW_BWD(c, z, fake, big), SPA2_ERR_RANGE);
  z = w; z.sinks = -1; EXPECT(WINDOW(c, z), SPA2_ERR_RANGE);
  /* workspaces of the largest shapes and limits: no sum overflows, and none is accepted that is too small */
  for (int l = 0; l < 6; ++l)
    for (int r = 0; r < 6; ++r)
      for (int s = 2; s < 6; ++s) {
        z.left = limits[l]; z.right = limits[r]; z.sinks = limits[s];
        y = c; y.B = y.Hq = y.Hk = 1; y.Nq = y.Nk = 1 << 28; y.q_sb = y.k_sb = y.d_sb = LLONG_MAX / 8 * 8;
        if (spa2_window_bwd_workspace_bytes(&y, &z) < ((size_t)1 << 31)) { printf("a workspace too small\n"); ++failures; }
        EXPECT(WINDOW_BWD(y, z, fake, 1), SPA2_ERR_WORKSPACE);
        EXPECT(WINDOW_BWD(c, z, fake, 8), SPA2_ERR_WORKSPACE);
        y = c; y.Hq = 32; y.Nq = 1 << 15; y.Nk = 1 << 24;
        EXPECT(WINDOW_BWD(y, z, 0, big), SPA2_ERR_WORKSPACE);
        EXPECT(WINDOW_BWD(y, z, odd, big), SPA2_ERR_ALIGN);
      }
  EXPECT(spa2_window_fwd(fake, fake, fake, odd, 0, &c, &w, 0.1f, fake, 0, f, fake, big, 0), SPA2_ERR_ALIGN);
  EXPECT(spa2_window_fwd(fake, fake, fake, 0, odd, &c, &w, 0.1f, fake, 0, f, fake, big, 0), SPA2_ERR_ALIGN);
  EXPECT(spa2_window_fwd(fake, fake, fake, 0, 0, &c, 0, 0.1f, fake, 0, f, fake, big, 0), SPA2_ERR_NULL);
  EXPECT(spa2_window_fwd(fake, fake, fake, 0, 0, 0, &w, 0.1f, fake, 0, f, fake, big, 0), SPA2_ERR_NULL);
  EXPECT(spa2_window_fwd(fake, fake, fake, 0, 0, &c, &w, NAN, fake, 0, f, fake, big, 0), SPA2_ERR_RANGE);

  spa2_gate_shape g = {2, 10, 0, 64, 64, 64, SPA2_NORM_LAYER, 1, 1, 1, 1, 1}, h;
  spa2_gate_params p = {fake, fake, fake, fake, fake, fake}, q;
  spa2_gate_grads d = {fake, fake, fake, fake, fake, fake}, e;
#define GATE(s) spa2_gate_norm(fake, fake, &p, &s, 1e-6f, fake, fake, f, 0)
#define GATE_BWD(s, ws, bytes) spa2_gate_norm_bwd(fake, &p, &s, 1e-6f, fake, fake, fake, f, fake, fake, &d, ws, bytes, 0)
  h = g; h.samples = h.tokens = LLONG_MAX; EXPECT(GATE(h), SPA2_ERR_SHAPE); EXPECT(GATE_BWD(h, fake, big), SPA2_ERR_SHAPE);
  EXPECT(spa2_gate_norm_bwd_workspace_bytes(&h) != 0, 0);
  h = g; h.tokens = LLONG_MAX; EXPECT(GATE(h), SPA2_ERR_SHAPE);
  h = g; h.tokens = LLONG_MIN; EXPECT(GATE(h), SPA2_ERR_SHAPE);
  h = g; h.width = INT_MAX; EXPECT(GATE(h), SPA2_ERR_SHAPE);
  h = g; h.width = INT_MIN; EXPECT(GATE(h), SPA2_ERR_SHAPE);
  h = g; h.gate_sb = LLONG_MIN; EXPECT(GATE(h), SPA2_ERR_SHAPE);
  h = g; h.shift_sb = LLONG_MAX; EXPECT(GATE(h), SPA2_ERR_SHAPE);
  h = g; h.scale_sb = 63; EXPECT(GATE(h), SPA2_ERR_SHAPE);
  h = g; h.kind = INT_MAX; EXPECT(GATE(h), SPA2_ERR_UNSUPPORTED);
  h = g; h.x_dtype = INT_MIN; EXPECT(GATE(h), SPA2_ERR_UNSUPPORTED);
  h = g; h.x_dtype = 0; EXPECT(GATE(h), SPA2_ERR_UNSUPPORTED);             /* (fp32 branch into a bf16 stream) */
  h = g; h.param_dtype = 2; EXPECT(GATE_BWD(h, fake, big), SPA2_ERR_UNSUPPORTED);
  EXPECT(GATE_BWD(g, 0, big), SPA2_ERR_WORKSPACE); EXPECT(GATE_BWD(g, fake, 64), SPA2_ERR_WORKSPACE); EXPECT(GATE_BWD(g, odd, big), SPA2_ERR_ALIGN);
  h = g; h.samples = 1 << 22; h.width = 8192; EXPECT(GATE(h), SPA2_ERR_SHAPE);      /* (2^32 threads) */
  h = g; h.samples = 1 << 21; h.tokens = 1 << 18; h.width = 8192; h.gate_sb = h.scale_sb = h.shift_sb = 8192;
  EXPECT(GATE_BWD(h, fake, ((size_t)1 << 38)), SPA2_ERR_WORKSPACE);
  q = p; q.weight = odd; EXPECT(spa2_gate_norm(fake, fake, &q, &g, 1e-6f, fake, fake, f, 0), SPA2_ERR_ALIGN);
  e = d; e.bias = odd; EXPECT(spa2_gate_norm_bwd(fake, &p, &g, 1e-6f, fake, fake, fake, f, fake, fake, &e, fake, big, 0), SPA2_ERR_ALIGN);
  EXPECT(spa2_gate_norm(fake, fake, &p, &g, -INFINITY, fake, fake, f, 0), SPA2_ERR_RANGE);
  EXPECT(spa2_gate_norm(fake, fake, &p, &g, 0.f, fake, fake, f, 0), SPA2_ERR_RANGE);

  spa2_gradient t[3] = {{fake, fake, 10, 1, 1}, {0, 0, 0, 0, 0}, {fake, 0, 7, 0, 0}};
#define CLIP(n) spa2_clip_gradients(t, n, 1.0, 1e-6, f, fake, 16, 0)
  EXPECT(CLIP(INT_MIN), SPA2_ERR_SHAPE); EXPECT(CLIP(0), SPA2_ERR_SHAPE); EXPECT(CLIP(3), SPA2_ERR_WORKSPACE);
  t[0].n = LLONG_MAX; EXPECT(CLIP(3), SPA2_ERR_SHAPE);
  t[0].n = LLONG_MIN; EXPECT(CLIP(3), SPA2_ERR_SHAPE);
  t[0].n = (int64_t)1 << 42; EXPECT(CLIP(3), SPA2_ERR_SHAPE);              /* (with the third one's) */
  t[0].n = 10; t[0].dtype = INT_MAX; EXPECT(CLIP(3), SPA2_ERR_UNSUPPORTED);
  t[0].dtype = 0; EXPECT(CLIP(3), SPA2_ERR_UNSUPPORTED);                   /* (in place, of another type) */
  t[0].dtype = 1; t[0].x = odd; EXPECT(CLIP(3), SPA2_ERR_ALIGN);
  t[0].x = 0; EXPECT(CLIP(3), SPA2_ERR_NULL);
  t[0].x = fake;
  EXPECT(spa2_clip_gradients(t, 3, NAN, 1e-6, f, fake, big, 0), SPA2_ERR_RANGE);
  EXPECT(spa2_clip_gradients(t, 3, -1.0, 1e-6, f, fake, big, 0), SPA2_ERR_RANGE);
  EXPECT(spa2_clip_gradients(t, 3, 1.0, INFINITY, f, fake, big, 0), SPA2_ERR_RANGE);
  EXPECT(spa2_clip_gradients(t, 3, 1.0, 1e-6, 0, fake, big, 0), SPA2_ERR_NULL);
  EXPECT(spa2_clip_gradients(0, 3, 1.0, 1e-6, f, fake, big, 0), SPA2_ERR_NULL);
  EXPECT(spa2_clip_gradients(t, 3, 1.0, 1e-6, f, odd, big, 0), SPA2_ERR_ALIGN);
  if (!failures) printf("all rejected before launch\n");
  return failures != 0;
}
