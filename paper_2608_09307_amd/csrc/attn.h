// Internal declarations of the softmax attention (attn.hip, mixers.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace linsimp {

struct AttnShape {
  int64_t B, H, Hkv, nq, nk, window;
  int D, dtype, causal;
  float scale;
  size_t esize() const { return dtype == 1 ? 2 : 4; }
};

// Kernel arguments (device pointers; a null pos means forward or backward)
struct AttnArgs {
  const void *q, *k, *v;         // [B][H][nq][D], [B][Hkv][nk][D] (the step writes its token into k, v)
  const void *knew, *vnew;       // step: the new token's rows [B][Hkv][D]
  const int64_t* pos;            // step: [B] index of the new token (negative: none)
  const int *lens_q, *lens_k;    // [B] or null
  void* out;                     // [B][H][nq][D] (input of the backward)
  float* lse;                    // [B][H][nq] natural logarithm, or null
  const void* dout;
  void *dq, *dk, *dv;
  float *part, *pml;             // ns > 1: [ns][B][H][nq][D] unnormalised outputs, [..][2] maximum (log2) and sum;
                                 // backward, nsq or nsk > 1: the splits' gradients (dq's, then dk's and dv's)
  float* delta;                  // [B][H][nq]
  int B, H, Hkv, G, nq, nk, causal, window;
  int ntq, ntk, ns, nsq, nsk;    // query and key tiles of 128; splits of the forward, the query and the key sweep
  float scale, c;                // c = scale log2(e)
};

int attn_splits(const AttnShape& s);
void attn_bwd_splits(const AttnShape& s, int* nsq, int* nsk);
int launch_attn_fwd(const AttnShape& s, const AttnArgs& a, hipStream_t st);
int launch_attn_bwd(const AttnShape& s, const AttnArgs& a, hipStream_t st);

}  // namespace linsimp
