// Internal declarations of the gated linear recurrence (glr.hip, mixers.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace linsimp {

struct GlrShape {
  int64_t B, H, n;
  int D, dtype;
  float scale;
  size_t esize() const { return dtype == 1 ? 2 : 4; }
  int64_t BH() const { return B * H; }
  int64_t nch() const { return (n + 31) / 32; }
};

struct GlrArgs {
  const void *q, *k, *v, *g, *dout;       // [BH][n][D]
  const float *s0, *ds1;                  // [BH][D][D] or null
  const int* lens;                        // [B] or null
  void *out, *dq, *dk, *dv, *dg;          // [BH][n][D]
  float *s1, *ds0;                        // [BH][D][D] or null
  // workspace: per segment the state it adds, then (after the scan) the state it
  // starts from, and the decay across it; forward and (backward) reverse
  float *part, *rpart;                    // [BH][G][D*D]
  float *fac, *rfac;                      // [BH][G][D]
  int* again;                             // [BH][G] whether a segment has a chunk for the exact way
  void* states;                           // backward: [BH][nch][D*D] operand type, fragment order
  float* pre;                             // backward, G > 1: [BH][nch][D] log decay from the segment's start to each
  int H, n, nch, G, cps;                  // chunks of 32 rows in all, segments, chunks per segment
  int exact;                              // keep the low half of the rounded keys (a float32 state is asked for)
  float scale;
};

// segments per (sequence, head) of a forward or a backward
int glr_segments(const GlrShape& s, bool backward);
int launch_glr_fwd(const GlrShape& s, GlrArgs a, hipStream_t st);
int launch_glr_bwd(const GlrShape& s, GlrArgs a, hipStream_t st);
int launch_glr_step(const GlrShape& s, const void* q, const void* k, const void* v, const void* g, float* state,
                    void* out, hipStream_t st);

}  // namespace linsimp
