// C ABI of softmax attention and the gated linear recurrence: argument
// validation, workspace carving and dispatch.  Contracts: include/linsimp.h.
#include "../../include/linsimp.h"

#include <math.h>

#include "attn.h"
#include "glr.h"
#include "linsimp_internal.h"

using namespace linsimp;

namespace {

size_t al(size_t x) { return (x + 255) & ~(size_t)255; }

int check_width(const char* what, int D, int dtype) {
  if (dtype != LINSIMP_F32 && dtype != LINSIMP_BF16) {
    set_error("%s: dtype %d is not LINSIMP_F32 or LINSIMP_BF16", what, dtype);
    return LINSIMP_E_INVALID_ARG;
  }
  if (!(D == 32 || D == 64 || (D == 128 && dtype == LINSIMP_BF16))) {
    set_error("%s: D=%d is not 32, 64 or (bf16) 128", what, D);
    return LINSIMP_E_UNSUPPORTED;
  }
  return LINSIMP_OK;
}

// an optional pointer (NULL, or aligned)
int check_opt(const char* name, const void* p, uintptr_t mask) {
  if (((uintptr_t)p & mask) == 0) return LINSIMP_OK;
  set_error("%s is not %d-byte aligned", name, (int)mask + 1);
  return LINSIMP_E_INVALID_ARG;
}

int check_attn(const linsimp_attn_dims* d, AttnShape* s) {
  if (d == nullptr) { set_error("dims is NULL"); return LINSIMP_E_INVALID_ARG; }
  if (d->B < 1 || d->H < 1 || d->Hkv < 1 || d->nq < 1 || d->nk < 1) {
    set_error("attn: sizes must be positive (B=%lld H=%lld Hkv=%lld nq=%lld nk=%lld)", (long long)d->B,
              (long long)d->H, (long long)d->Hkv, (long long)d->nq, (long long)d->nk);
    return LINSIMP_E_INVALID_ARG;
  }
  if (int rc = check_width("attn", d->D, d->dtype)) return rc;
  if (d->H % d->Hkv != 0) {
    set_error("attn: H=%lld is not a multiple of Hkv=%lld", (long long)d->H, (long long)d->Hkv);
    return LINSIMP_E_INVALID_ARG;
  }
  if (d->causal != 0 && d->causal != 1) { set_error("attn: causal must be 0 or 1"); return LINSIMP_E_INVALID_ARG; }
  if (d->window < 0 || (d->window > 0 && d->causal == 0)) {
    set_error("attn: window must be >= 0, and 0 without causal");
    return LINSIMP_E_INVALID_ARG;
  }
  if (!(d->scale >= 1e-18f && d->scale <= 1e18f)) {
    set_error("attn: scale must be between 1e-18 and 1e18");
    return LINSIMP_E_INVALID_ARG;
  }
  // rows and slots are 32-bit within a head, and a grid has fewer than 2^32 threads
  const int64_t big = (int64_t)1 << 30;
  if (d->B > big || d->H > big || d->nq > big || d->nk > big || d->B * d->H > (int64_t)1 << 20 ||
      d->B * d->H * d->nq > (int64_t)1 << 30 || d->B * d->Hkv * d->nk > (int64_t)1 << 38) {
    set_error("attn: sizes too large: B*H=%lld (at most 2^20), B*H*nq (at most 2^30), nk (at most 2^30), "
              "B*Hkv*nk (at most 2^38)", (long long)(d->B > big || d->H > big ? -1 : d->B * d->H));
    return LINSIMP_E_UNSUPPORTED;
  }
  s->B = d->B; s->H = d->H; s->Hkv = d->Hkv; s->nq = d->nq; s->nk = d->nk;
  s->window = d->window >= d->nk ? 0 : d->window;      // (no query then loses a key to it)
  s->D = d->D; s->dtype = d->dtype; s->causal = d->causal; s->scale = d->scale;
  return LINSIMP_OK;
}

// the key sweep's grid: a workgroup for every 128 keys
int check_attn_bwd(const AttnShape& s) {
  if (s.B * s.Hkv * s.nk <= (int64_t)1 << 30) return LINSIMP_OK;
  set_error("attn backward: B*Hkv*nk=%lld is above 2^30", (long long)(s.B * s.Hkv * s.nk));
  return LINSIMP_E_UNSUPPORTED;
}

size_t attn_fwd_ws(const AttnShape& s, AttnArgs* a, void* base) {
  const size_t rows = (size_t)s.B * s.H * s.nq;
  const int ns = attn_splits(s);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    void* p = base ? (char*)base + off : nullptr;
    off += al(bytes);
    return (float*)p;
  };
  float* part = ns > 1 ? take((size_t)ns * rows * s.D * 4) : nullptr;
  float* pml = ns > 1 ? take((size_t)ns * rows * 2 * 4) : nullptr;
  if (a) { a->ns = ns; a->part = part; a->pml = pml; }
  return off > 256 ? off : 256;
}

// delta, then the splits' gradients: dq's are summed before the key sweep writes its own
size_t attn_bwd_ws(const AttnShape& s, AttnArgs* a, void* base) {
  const size_t qe = (size_t)s.B * s.H * s.nq * s.D * 4, ke = (size_t)s.B * s.Hkv * s.nk * s.D * 4;
  const size_t delta = al((size_t)s.B * s.H * s.nq * 4);
  int nsq, nsk;
  attn_bwd_splits(s, &nsq, &nsk);
  const size_t pq = nsq > 1 ? nsq * qe : 0, pk = nsk > 1 ? 2 * nsk * ke : 0;
  if (a) { a->nsq = nsq; a->nsk = nsk; a->delta = (float*)base; a->part = (float*)((char*)base + delta); }
  return delta + al(pq > pk ? pq : pk);
}

AttnArgs attn_args(const AttnShape& s) {
  AttnArgs a{};
  a.B = (int)s.B; a.H = (int)s.H; a.Hkv = (int)s.Hkv; a.G = (int)(s.H / s.Hkv);
  a.nq = (int)s.nq; a.nk = (int)s.nk; a.causal = s.causal; a.window = (int)s.window;
  a.ntq = (int)((s.nq + 127) / 128); a.ntk = (int)((s.nk + 127) / 128);
  a.ns = a.nsq = a.nsk = 1; a.scale = s.scale; a.c = s.scale * 1.4426950408889634f;
  return a;
}

int check_glr(const linsimp_glr_dims* d, GlrShape* s, bool step = false) {
  if (d == nullptr) { set_error("dims is NULL"); return LINSIMP_E_INVALID_ARG; }
  if (d->B < 1 || d->H < 1 || d->n < 1) {
    set_error("glr: sizes must be positive (B=%lld H=%lld n=%lld)", (long long)d->B, (long long)d->H, (long long)d->n);
    return LINSIMP_E_INVALID_ARG;
  }
  if (int rc = check_width("glr", d->D, d->dtype)) return rc;
  if (!isfinite(d->scale)) { set_error("glr: scale must be finite"); return LINSIMP_E_INVALID_ARG; }
  // (sequence, head) pairs index the scan's grid (the step's: a grid of fewer than 2^32 threads)
  const int64_t big = (int64_t)1 << 30, most = step ? ((int64_t)1 << 24) - 1 : 65535;
  if (d->B > big || d->H > big || d->n > big || d->B * d->H > most || d->B * d->H * d->n > (int64_t)1 << 31) {
    set_error("glr: sizes too large: B*H at most %lld, n at most 2^30, B*H*n at most 2^31", (long long)most);
    return LINSIMP_E_UNSUPPORTED;
  }
  s->B = d->B; s->H = d->H; s->n = d->n; s->D = d->D; s->dtype = d->dtype; s->scale = d->scale;
  return LINSIMP_OK;
}

// which segments need the exact way; G > 1: their states and decays (backward: both directions); backward: the chunk states
size_t glr_ws(const GlrShape& s, int G, bool backward, GlrArgs* a, void* base) {
  const size_t BH = (size_t)s.BH(), DD = (size_t)s.D * s.D;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    void* p = base ? (char*)base + off : nullptr;
    off += al(bytes);
    return p;
  };
  int* again = (int*)take(BH * G * 4);
  float* part = G > 1 ? (float*)take(BH * G * DD * 4) : nullptr;
  float* fac = G > 1 ? (float*)take(BH * G * s.D * 4) : nullptr;
  float* rpart = G > 1 && backward ? (float*)take(BH * G * DD * 4) : nullptr;
  float* rfac = G > 1 && backward ? (float*)take(BH * G * s.D * 4) : nullptr;
  void* states = backward ? take(BH * (size_t)s.nch() * DD * s.esize()) : nullptr;
  float* pre = G > 1 && backward ? (float*)take(BH * (size_t)s.nch() * s.D * 4) : nullptr;
  if (a) { a->pre = pre; a->again = again; a->part = part; a->fac = fac; a->rpart = rpart; a->rfac = rfac; a->states = states; }
  return off;
}

GlrArgs glr_args(const GlrShape& s, bool backward) {
  GlrArgs a{};
  a.H = (int)s.H; a.n = (int)s.n; a.nch = (int)s.nch();
  a.G = glr_segments(s, backward); a.cps = (a.nch + a.G - 1) / a.G;
  a.scale = s.scale;
  return a;
}

}  // namespace

extern "C" {

size_t linsimp_attn_workspace_size(const linsimp_attn_dims* dims, int for_backward) {
  AttnShape s;
  if (check_attn(dims, &s) != LINSIMP_OK || (for_backward && check_attn_bwd(s) != LINSIMP_OK)) return 0;
  const size_t fwd = attn_fwd_ws(s, nullptr, nullptr);
  const size_t bwd = for_backward ? attn_bwd_ws(s, nullptr, nullptr) : 0;
  return fwd > bwd ? fwd : bwd;
}

int linsimp_attn_fwd(const linsimp_attn_dims* dims, const void* q, const void* k, const void* v,
                     const int32_t* lens_q, const int32_t* lens_k, void* out, float* lse,
                     void* workspace, size_t workspace_bytes, void* stream) {
  AttnShape s;
  int rc = check_attn(dims, &s);
  if (rc) return rc;
  const void* ps[] = {q, k, v, out};
  if ((rc = check_ptrs("q,k,v,out", ps, 4))) return rc;
  if ((rc = check_opt("lens_q", lens_q, 3)) || (rc = check_opt("lens_k", lens_k, 3)) || (rc = check_opt("lse", lse, 15)))
    return rc;
  if ((rc = check_buf("workspace", workspace, workspace_bytes, attn_fwd_ws(s, nullptr, nullptr)))) return rc;
  AttnArgs a = attn_args(s);
  a.q = q; a.k = k; a.v = v; a.lens_q = lens_q; a.lens_k = lens_k; a.out = out; a.lse = lse;
  attn_fwd_ws(s, &a, workspace);
  return launch_attn_fwd(s, a, (hipStream_t)stream);
}

int linsimp_attn_bwd(const linsimp_attn_dims* dims, const void* q, const void* k, const void* v,
                     const int32_t* lens_q, const int32_t* lens_k, const void* out,
                     const float* lse, const void* dout, void* dq, void* dk, void* dv,
                     void* workspace, size_t workspace_bytes, void* stream) {
  AttnShape s;
  int rc = check_attn(dims, &s);
  if (!rc) rc = check_attn_bwd(s);
  if (rc) return rc;
  const void* ps[] = {q, k, v, out, lse, dout, dq, dk, dv};
  if ((rc = check_ptrs("q,k,v,out,lse,dout,dq,dk,dv", ps, 9))) return rc;
  if ((rc = check_opt("lens_q", lens_q, 3)) || (rc = check_opt("lens_k", lens_k, 3))) return rc;
  if ((rc = check_buf("workspace", workspace, workspace_bytes, attn_bwd_ws(s, nullptr, nullptr)))) return rc;
  AttnArgs a = attn_args(s);
  a.q = q; a.k = k; a.v = v; a.lens_q = lens_q; a.lens_k = lens_k;
  a.out = (void*)out; a.lse = (float*)lse; a.dout = dout; a.dq = dq; a.dk = dk; a.dv = dv;
  attn_bwd_ws(s, &a, workspace);
  return launch_attn_bwd(s, a, (hipStream_t)stream);
}

int linsimp_attn_step(const linsimp_attn_dims* dims, const void* q, const void* k, const void* v,
                      void* kcache, void* vcache, const int64_t* pos, void* out, void* workspace,
                      size_t workspace_bytes, void* stream) {
  AttnShape s;
  int rc = check_attn(dims, &s);
  if (rc) return rc;
  if (s.nq != 1 || dims->window != 0) {
    set_error("attn step: nq must be 1 and window 0 (the ring's slots are the window)");
    return LINSIMP_E_INVALID_ARG;
  }
  const void* ps[] = {q, k, v, kcache, vcache, pos, out};
  if ((rc = check_ptrs("q,k,v,kcache,vcache,pos,out", ps, 7))) return rc;
  if ((rc = check_buf("workspace", workspace, workspace_bytes, attn_fwd_ws(s, nullptr, nullptr)))) return rc;
  AttnArgs a = attn_args(s);
  a.q = q; a.k = kcache; a.v = vcache; a.knew = k; a.vnew = v; a.pos = pos; a.out = out;
  attn_fwd_ws(s, &a, workspace);
  return launch_attn_fwd(s, a, (hipStream_t)stream);
}

size_t linsimp_glr_workspace_size(const linsimp_glr_dims* dims, int for_backward) {
  GlrShape s;
  if (check_glr(dims, &s) != LINSIMP_OK) return 0;
  const size_t fwd = glr_ws(s, glr_segments(s, false), false, nullptr, nullptr);
  const size_t bwd = for_backward ? glr_ws(s, glr_segments(s, true), true, nullptr, nullptr) : 0;
  return fwd > bwd ? fwd : bwd;
}

int linsimp_glr_fwd(const linsimp_glr_dims* dims, const void* q, const void* k, const void* v,
                    const void* g, const float* s0, const int32_t* lens, void* out, float* s1,
                    void* workspace, size_t workspace_bytes, void* stream) {
  GlrShape s;
  int rc = check_glr(dims, &s);
  if (rc) return rc;
  const void* ps[] = {q, k, v, g, out};
  if ((rc = check_ptrs("q,k,v,g,out", ps, 5))) return rc;
  if ((rc = check_opt("s0", s0, 15)) || (rc = check_opt("lens", lens, 3)) || (rc = check_opt("s1", s1, 15))) return rc;
  GlrArgs a = glr_args(s, false);
  if ((rc = check_buf("workspace", workspace, workspace_bytes, glr_ws(s, a.G, false, nullptr, nullptr)))) return rc;
  a.q = q; a.k = k; a.v = v; a.g = g; a.s0 = s0; a.lens = lens; a.out = out; a.s1 = s1;
  a.exact = s1 != nullptr;
  glr_ws(s, a.G, false, &a, workspace);
  return launch_glr_fwd(s, a, (hipStream_t)stream);
}

int linsimp_glr_bwd(const linsimp_glr_dims* dims, const void* q, const void* k, const void* v,
                    const void* g, const float* s0, const int32_t* lens, const void* dout,
                    const float* ds1, void* dq, void* dk, void* dv, void* dg, float* ds0,
                    void* workspace, size_t workspace_bytes, void* stream) {
  GlrShape s;
  int rc = check_glr(dims, &s);
  if (rc) return rc;
  const void* ps[] = {q, k, v, g, dout, dq, dk, dv, dg};
  if ((rc = check_ptrs("q,k,v,g,dout,dq,dk,dv,dg", ps, 9))) return rc;
  if ((rc = check_opt("s0", s0, 15)) || (rc = check_opt("lens", lens, 3)) || (rc = check_opt("ds1", ds1, 15)) ||
      (rc = check_opt("ds0", ds0, 15)))
    return rc;
  GlrArgs a = glr_args(s, true);
  if ((rc = check_buf("workspace", workspace, workspace_bytes, glr_ws(s, a.G, true, nullptr, nullptr)))) return rc;
  a.q = q; a.k = k; a.v = v; a.g = g; a.s0 = s0; a.lens = lens; a.dout = dout; a.ds1 = ds1;
  a.dq = dq; a.dk = dk; a.dv = dv; a.dg = dg; a.ds0 = ds0;
  a.exact = ds0 != nullptr;
  glr_ws(s, a.G, true, &a, workspace);
  return launch_glr_bwd(s, a, (hipStream_t)stream);
}

int linsimp_glr_step(const linsimp_glr_dims* dims, const void* q, const void* k, const void* v,
                     const void* g, float* state, void* out, void* stream) {
  GlrShape s;
  int rc = check_glr(dims, &s, true);
  if (rc) return rc;
  if (s.n != 1) { set_error("glr step: n must be 1"); return LINSIMP_E_INVALID_ARG; }
  const void* ps[] = {q, k, v, g, state, out};
  if ((rc = check_ptrs("q,k,v,g,state,out", ps, 6))) return rc;
  return launch_glr_step(s, q, k, v, g, state, out, (hipStream_t)stream);
}

}  // extern "C"
