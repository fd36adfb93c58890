// Gated linear recurrence on gfx950: forward, backward and the single-token step.
//
//   S_t = diag(exp(g_t)) S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t
//   R_t = scale q_t do_t^T + diag(exp(g_{t+1})) R_{t+1}        (gradient of S_t)
//   dq_t = scale S_t do_t,  dk_t = R_t v_t,  dv_t = R_t^T k_t
//   dg_t = rowsum(R_t * diag(exp(g_t)) S_{t-1})
//
// Rows are taken in chunks of 32.  With G_t the sum of g over the chunk's rows
// up to t, a pair s <= t of one chunk has the weight (per channel d)
// exp(G_t - G_s) = e_t / e_s with e_t = exp(G_t - G_15), the decay from the
// middle of the chunk, so that
//   P_ts = sum_d (q_t e_t)_d (k_s / e_s)_d        (a matrix product of scaled rows)
//   o_t  = (q_t e_t) Z + sum_{s <= t} P_ts v_s,   Z = exp(G_15) S_start
//   S_end = exp(G_31 - G_15) (Z + sum_s (k_s / e_s) v_s^T)
// and the state is carried from middle to middle with one scaling per chunk.
// The same rows serve the backward, which runs from the last chunk to the first
// with Y = exp(G_31 - G_15) R_end in the place of Z:
//   dk_s = (Y v_s + sum_{t > s} dP_ts q_t e_t) / e_s + diagonal,  and so on.
//
// e_t and 1 / e_t are both representable while a channel decays by less than
// 2^60 across either half of the chunk.  A chunk in which one decays faster (a
// gate that clears its channel) takes the exact way instead: the pairs are
// split by the highest bit in which t and s differ, and both factors of a pair
// are decays to or from the border between the halves of its block, at most 1.
//
// The sums of g are matrix products with matrices of ones (g is exact in the
// operand type), transposed so that a lane holds one row t and 16 consecutive
// channels: rows are read and written in 16-byte pieces, and all of a row's
// elementwise work stays in its lane.  In bf16 the scaled rows, the pair
// weights and the state as an operand are rounded to bf16 (each 2^-8 relative
// at most); the state, all sums and the decays are float32.  Where a float32
// state is an output, the rows that it sums keep a second bf16 term, so that
// it is off by 2^-17 of its terms at most.
//
// Times beside the kernels are of a settled clock (it moves with the load for the
// first 10 to 50 ms of a run, and the times by up to 30% with it); two times with
// an arrow, or a list of variants, were taken in turn in one session each and
// compare with each other only.
#include "glr.h"

#include <type_traits>

#include "common.h"
#include "linsimp_internal.h"
#include "prof.h"

namespace linsimp {

static constexpr float kFast = 60.0f;        // log2 of the largest decay across half a chunk on the short way
static constexpr float kClear = -1e30f;      // g below this (-inf) clears the channel just the same

// ---- storage: 32 rows; a lane's 16 channels are two 16-byte pieces with the
// middle groups of four swapped, so that a 16-byte read of a row gives an
// operand fragment in accumulator row order (common.h, permuted storage) ----
template <typename T> struct Row16 {
  static constexpr int VE = 16 / (int)sizeof(T), NV = 16 / VE;
  typedef T V __attribute__((ext_vector_type(VE)));
  V p[NV];
  LS_DEV void load(const T* row) {
#pragma unroll
    for (int i = 0; i < NV; ++i) p[i] = *(const V*)(row + i * VE);
  }
  LS_DEV void keep(bool ok) {                                  // a row that does not exist is zero
    if (!__any(!ok)) return;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < VE; ++e) p[i][e] = ok ? p[i][e] : (T)0.0f;
  }
  // the same row, so that its conversion to float32 is made again rather than kept
  LS_DEV Row16 again() const {
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    Row16 r;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      i32x4 x = __builtin_bit_cast(i32x4, p[i]);
      asm("" : "+v"(x));
      r.p[i] = __builtin_bit_cast(V, x);
    }
    return r;
  }
  LS_DEV static Row16 either(bool first, const Row16& a, const Row16& b) {
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    Row16 r;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const i32x4 x = __builtin_bit_cast(i32x4, a.p[i]), y = __builtin_bit_cast(i32x4, b.p[i]);
      i32x4 z;
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] = first ? x[e] : y[e];
      r.p[i] = __builtin_bit_cast(V, z);
    }
    return r;
  }
  LS_DEV float at(int v) const { return (float)p[v / VE][v % VE]; }
  LS_DEV void set(int v, float x) { p[v / VE][v % VE] = (T)x; }
};
LS_DEV void put_row(bf16* dst, const Row16<bf16>& r) {         // dst: the row's 16-channel block
  bf16x8 a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i] = r.p[0][i]; a[4 + i] = r.p[1][i];
    b[i] = r.p[0][4 + i]; b[4 + i] = r.p[1][4 + i];
  }
  *(bf16x8*)dst = a;
  *(bf16x8*)(dst + 8) = b;
}
LS_DEV void put_row(float* dst, const Row16<float>& r) {
#pragma unroll
  for (int v = 0; v < 16; ++v) dst[v] = r.at(v);
}
LS_DEV void get_row(const bf16* src, float (&x)[16]) {
  const bf16x8 a = *(const bf16x8*)src, b = *(const bf16x8*)(src + 8);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = (float)a[i]; x[8 + i] = (float)a[4 + i];
    x[4 + i] = (float)b[i]; x[12 + i] = (float)b[4 + i];
  }
}
LS_DEV void get_row(const float* src, float (&x)[16]) {
#pragma unroll
  for (int v = 0; v < 16; ++v) x[v] = src[v];
}
template <typename T> LS_DEV void store_row(T* row, const float (&x)[16]) {
  Row16<T> r;
#pragma unroll
  for (int v = 0; v < 16; ++v) r.set(v, x[v]);
#pragma unroll
  for (int i = 0; i < Row16<T>::NV; ++i) *(typename Row16<T>::V*)(row + i * Row16<T>::VE) = r.p[i];
}

// accumulator column n of a 32-channel tile <-> channel: the register v of half
// h of a tile with these columns as rows is then channel 16 h + v
LS_DEV int chan_of(int n) { return 16 * ((n >> 2) & 1) + 4 * (n >> 3) + (n & 3); }

// ---- operand fragments along the rows of a stored matrix [row][channel] ----
// Lane column n <-> channel n0 + n (LANE = false) or n0 + chan_of(n) (true);
// contraction over rows, in natural or accumulator row order.
LS_DEV int swap4(int g) { return ((g & 1) << 1) | (g >> 1); }
template <bool LANE> LS_DEV bf16x4 tr4(int L, const bf16* mat, int ld, int k0, int n0) {
  const int s = L & 15, c = 4 * ((L >> 4) & 1) + (s & 3);
  const int at = LANE ? 16 * (c & 1) + 4 * swap4(c >> 1) : 16 * (c >> 2) + 4 * swap4(c & 3);
  return lds_tr4(mat + (k0 + (s >> 2)) * ld + n0 + at);
}
template <bool LANE> LS_DEV bf16x8 rows_nat(int L, const bf16* mat, int ld, int ks, int n0) {
  const int h = L >> 5;
  return cat44(tr4<LANE>(L, mat, ld, 16 * ks + 8 * h, n0), tr4<LANE>(L, mat, ld, 16 * ks + 8 * h + 4, n0));
}
template <bool LANE> LS_DEV bf16x8 rows_crow(int L, const bf16* mat, int ld, int sp, int n0) {
  const int h = L >> 5;
  return cat44(tr4<LANE>(L, mat, ld, 16 * sp + 4 * h, n0), tr4<LANE>(L, mat, ld, 16 * sp + 8 + 4 * h, n0));
}
template <bool LANE> LS_DEV float rows_nat(int L, const float* mat, int ld, int ks, int n0) {
  const int n = L & 31;
  return mat[(2 * ks + (L >> 5)) * ld + n0 + (LANE ? chan_of(n) : n)];
}
template <bool LANE> LS_DEV float rows_crow(int L, const float* mat, int ld, int sp, int n0) {
  const int n = L & 31;
  return mat[(8 * (sp >> 2) + 4 * (L >> 5) + (sp & 3)) * ld + n0 + (LANE ? chan_of(n) : n)];
}

template <typename T> LS_DEV typename MF<T>::frag frag_of(const float (&x)[MF<T>::KPL]);
template <> LS_DEV bf16x8 frag_of<bf16>(const float (&x)[8]) {
  bf16x8 f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = (bf16)x[e];
  return f;
}
template <> LS_DEV float frag_of<float>(const float (&x)[1]) { return x[0]; }

// 32 x 32 matrix of 0, 1, -1 as an operand: column = this lane's row t, contraction row r
template <typename T, class Fn> LS_DEV typename MF<T>::frag ones_where(int L, int ks, Fn f) {
  const int t = L & 31;
  float x[MF<T>::KPL];
#pragma unroll
  for (int e = 0; e < MF<T>::KPL; ++e) x[e] = f(t, ks * MF<T>::KS + (L >> 5) * MF<T>::KPL + e);
  return frag_of<T>(x);
}

template <typename T> struct GlrBase {
  static constexpr int NKS = 32 / MF<T>::KS;              // k-steps over 32 rows
  // row stride of a 32-channel matrix.  Here and in the kernels' 32-row matrices 16
  // bytes are added to a row: rows are written and read whole as often as transposed
  // (32 heads of 16384 tokens, D = 128, backward: 517 us at tr_pad's pitch, 494 here)
  static constexpr int WST = 32 + MF<T>::PAD;
};

// sums of this wave's 32 gates over rows picked by f(t, r): register v <-> channel 16 h + v, lane <-> t
template <typename T, class Fn> LS_DEV f32x16 gate_sum(int l, const T* sg, Fn f) {
  f32x16 acc = zero16();
#pragma unroll
  for (int ks = 0; ks < GlrBase<T>::NKS; ++ks)
    acc = MF<T>::mma(rows_nat<true>(l, sg, GlrBase<T>::WST, ks, 0), ones_where<T>(l, ks, f), acc);
  return acc;
}
// row selections
struct Middle { LS_DEV float operator()(int t, int r) const { return r > 15 ? (r <= t ? 1.f : 0.f) : (r > t ? -1.f : 0.f); } };
struct UpTo { LS_DEV float operator()(int t, int r) const { return r <= t ? 1.f : 0.f; } };
struct After { LS_DEV float operator()(int t, int r) const { return r > t ? 1.f : 0.f; } };
struct All { LS_DEV float operator()(int, int) const { return 1.f; } };
// halves of size L: to the end of the earlier half for its rows, from the start of the later half for its own
struct Border {
  int L;
  LS_DEV float operator()(int t, int r) const {
    const bool later = (t & L) != 0;
    const int from = later ? t & ~(L - 1) : t + 1, rows = later ? t - from + 1 : (t | (L - 1)) - t;
    return (unsigned)(r - from) < (unsigned)rows ? 1.f : 0.f;
  }
};
// rows that level L joins: in the two halves of one block of 2 L (the highest bit in which they differ is L)
LS_DEV bool joins(int L, int s, int t) { return ((s ^ t) & ~(L - 1)) == L; }
// a row that joins none unless `ok`
LS_DEV int row_if(bool ok, int t) { return ok ? t : t ^ 64; }

// The lane, as a value of chunk c: what is derived from it (addresses, masks, the
// matrices of ones) is then made anew in every chunk instead of being kept in
// registers across the loop, where it pushed parts of the state to memory (313
// spilled registers in the backward, 35 us per chunk).
LS_DEV int lane_in(int lane, int c) {
  asm("" : "+v"(lane) : "s"(c));
  return lane;
}

// A lane's 16 channels of a chunk's row: a base that is the same in all lanes and
// an offset in 32 bits, the same for all the chunk's matrices
template <typename T> LS_DEV const T* lane_ptr(const T* base, unsigned off) { return (const T*)((const char*)base + off); }
template <typename T> LS_DEV T* lane_ptr(T* base, unsigned off) { return (T*)((char*)base + off); }
// byte offset of row 32 c + col (or the last row that exists) from row 32 c
template <typename T, int D> LS_DEV unsigned lane_off(int l, int c, int n) {
  return (unsigned)((min(l & 31, n - 1 - 32 * c) * D + 16 * (l >> 5)) * (int)sizeof(T));
}

LS_DEV float dot_add(const bf16x8& a, const bf16x8& b, float acc) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) acc = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{a[e], a[e + 1]}, bf16x2{b[e], b[e + 1]}, acc, false);
  return acc;
}
LS_DEV float dot_add(float a, float b, float acc) { return __builtin_fmaf(a, b, acc); }

// a lane's 16 values, and back
LS_DEV void put_lane(float* dst, const float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) *(f32x4*)(dst + 4 * i) = f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
}
LS_DEV void get_lane(const float* src, float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x4 y = *(const f32x4*)(src + 4 * i);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[4 * i + e] = y[e];
  }
}

LS_DEV float ex(float x) { return fast_exp2(x * kLog2e); }

// 16 values per half, taken from the lanes of column `from`, to 32 consecutive floats
LS_DEV void put_vec(int l, int from, float* dst, const f32x16& x) {
  if ((l & 31) != from) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) *(f32x4*)(dst + 16 * (l >> 5) + 4 * i) = f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
}
LS_DEV void get_vec(int l, const float* src, float (&x)[16]) {
  const int h = l >> 5;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x4 y = *(const f32x4*)(src + 16 * h + 4 * i);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[4 * i + e] = y[e];
  }
}

// A chunk's gates, from the wave's 32 channels of g in LDS: E = log2 of e_t, and
// the scaling that brings the carried state to the middle of this chunk,
//   fz = exp(lack + sum over the first 16 rows),  lack' = sum over the last 16
// (REV: the last, then the first).  lo, lack, lack', fz: the wave's 32 floats each.
// Returns whether the channels allow the short way (a cleared channel's sums
// come out as NaN and do not).
template <typename T> struct Picks {                    // of every chunk: made once
  typename MF<T>::frag mid[GlrBase<T>::NKS], one;
  LS_DEV void init(int l) {
#pragma unroll
    for (int ks = 0; ks < GlrBase<T>::NKS; ++ks) mid[ks] = ones_where<T>(l, ks, Middle{});
    one = ones_where<T>(l, 0, All{});
  }
};
template <typename T, bool REV>
LS_DEV bool gate_chunk(int l, const Picks<T>& pick, const T* sg, f32x16& E, float* lo, const float* lack, float* next, float* fz) {
  using F = MF<T>;
  constexpr int NKS = GlrBase<T>::NKS, WST = GlrBase<T>::WST;
  f32x16 first = zero16();
  E = zero16();
#pragma unroll
  for (int ks = 0; ks < NKS; ++ks) {
    const typename F::frag x = rows_nat<true>(l, sg, WST, ks, 0);
    E = F::mma(x, pick.mid[ks], E);
    if (ks < NKS / 2) first = F::mma(x, pick.one, first);
  }
  put_vec(l, 0, REV ? next : lo, first);
  put_vec(l, 31, REV ? lo : next, E);                  // (row 31's sum from the middle: the last 16 rows)
  bool fast = true;
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    E[v] *= kLog2e;
    fast = fast && fabsf(E[v]) <= kFast;
  }
  wave_lds_sync();
  if (l < 32) fz[l] = ex(lack[l] + lo[l]);
  return !__any(!fast);
}
// The same for the exact way: g as it is used there, the state brought to the
// chunk's border, and the decay across the whole chunk.
template <typename T>
LS_DEV void gate_exact(int l, T* sg) {
  float x[16];
  T* row = sg + (l & 31) * GlrBase<T>::WST + 16 * (l >> 5);
  get_row(row, x);
  Row16<T> r;
#pragma unroll
  for (int v = 0; v < 16; ++v) r.set(v, x[v] < kClear ? kClear : x[v]);
  put_row(row, r);
  wave_lds_sync();
}
template <typename T>
LS_DEV void border_exact(int l, const T* sg, float* lo, const float* lack, float* next, float* fz, float* all) {
  put_vec(l, 0, lo, gate_sum(l, sg, All{}));
  wave_lds_sync();
  if (l < 32) {
    all[l] = ex(lo[l]);
    fz[l] = ex(lack[l]);
    next[l] = 0.0f;
  }
}

// rows t: x scaled per channel to the operand type, and what that rounding left
template <typename T>
LS_DEV void put_scaled(int l, T* hi, T* lo, int ld, const Row16<T>& x, const float (&f)[16], bool low) {
  Row16<T> a;
#pragma unroll
  for (int v = 0; v < 16; ++v) a.set(v, x.at(v) * f[v]);
  put_row(hi + (l & 31) * ld + 16 * (l >> 5), a);
  if (sizeof(T) == 2 && low) {
    Row16<T> b;
#pragma unroll
    for (int v = 0; v < 16; ++v) b.set(v, x.at(v) * f[v] - a.at(v));
    put_row(lo + (l & 31) * ld + 16 * (l >> 5), b);
  }
}
template <typename T> LS_DEV void put_decayed(int l, T* hi, T* lo, int ld, const Row16<T>& x, const f32x16& E, float sign, float sc, bool low) {
  float f[16];
#pragma unroll
  for (int v = 0; v < 16; ++v) f[v] = fast_exp2(E[v] * sign) * sc;
  put_scaled(l, hi, lo, ld, x, f, low);
}

// The rows of level L of the exact way: q of the rows in later halves, k of those in
// earlier ones, decayed from or to the border between the halves by f.  The product
// of this matrix with itself holds the level's pairs (against a matrix of each, with
// half of the rows zero: 48 heads of 2048 tokens, D = 64, resets in every chunk,
// forward and backward 364 -> 266 us).
template <typename T>
LS_DEV void put_level(int l, int L, const T* sg, T* dst, int ld, const Row16<T>& xq, const Row16<T>& xk, float (&f)[16]) {
  const f32x16 B = gate_sum(l, sg, Border{L});
#pragma unroll
  for (int v = 0; v < 16; ++v) f[v] = ex(B[v]);
  put_scaled(l, dst, dst, ld, Row16<T>::either((l & L) != 0, xq, xk).again(), f, false);
}

// a 32 x 32 tile as the next product's operand, all of it and with the elements (row, column) that f keeps
template <typename T> struct Tile {
  using F = MF<T>;
  typename F::frag f[F::CSTEPS];
  LS_DEV void set(const f32x16& x) {
#pragma unroll
    for (int sp = 0; sp < F::CSTEPS; ++sp) f[sp] = F::cfrag(x, sp);
  }
  // of `this` or of `other`, the rows that level L joins with the lane's column
  LS_DEV typename F::frag level(int l, int sp, int L, const Tile& other) const {
    const bool later = (l & L) != 0;
    if constexpr (sizeof(T) == 2) {
      typedef int i32x4 __attribute__((ext_vector_type(4)));
      const i32x4 a = __builtin_bit_cast(i32x4, f[sp]), b = __builtin_bit_cast(i32x4, other.f[sp]);
      i32x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool lo = joins(L, crow(8 * sp + 2 * e, l >> 5), l & 31), hi = joins(L, crow(8 * sp + 2 * e + 1, l >> 5), l & 31);
        y[e] = (later ? a[e] : b[e]) & ((lo ? 0xffff : 0) | (hi ? (int)0xffff0000 : 0));
      }
      return __builtin_bit_cast(typename F::frag, y);
    } else {
      return joins(L, crow(sp, l >> 5), l & 31) ? (later ? f[sp] : other.f[sp]) : 0.0f;
    }
  }
};

// rows (registers) of 32-row tiles times v[0 .. 32 NT - 1]
template <int NT> LS_DEV void scale_rows(int l, f32x16 (&S)[NT], const float* v) {
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 x = *(const f32x4*)(v + 32 * i + 8 * g + 4 * (l >> 5));
#pragma unroll
      for (int e = 0; e < 4; ++e) S[i][4 * g + e] *= x[e];
    }
}

// a state [D][D] (or zero): registers <-> its rows, lanes <-> column `at`
template <int NT> LS_DEV void load_state(int l, f32x16 (&S)[NT], const float* src, int D, int at) {
#pragma unroll
  for (int i = 0; i < NT; ++i) S[i] = zero16();
  if (src == nullptr) return;
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) S[i][v] = src[(size_t)(32 * i + crow(v, l >> 5)) * D + at];
}
// one of its rows per lane: registers <-> its columns
template <int NT> LS_DEV void load_state_t(int l, f32x16 (&S)[NT], const float* row) {
#pragma unroll
  for (int i = 0; i < NT; ++i) S[i] = zero16();
  if (row == nullptr) return;
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 x = *(const f32x4*)(row + 32 * i + 8 * g + 4 * (l >> 5));
#pragma unroll
      for (int e = 0; e < 4; ++e) S[i][4 * g + e] = x[e];
    }
}

LS_DEV int glr_len(const GlrArgs& a, int bh) {
  return a.lens ? min(max(a.lens[bh / a.H], 0), a.n) : a.n;
}

// product of stored rows with stored rows: rows a[lane], columns b[lane], over NT tiles of 32 channels
template <typename T, int NT> LS_DEV f32x16 rows_by_rows(int h, const T* arow, const T* brow) {
  using F = MF<T>;
  f32x16 acc = zero16();
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int sp = 0; sp < F::CSTEPS; ++sp) acc = F::mma(F::ldc(arow, 32 * i, sp, h), F::ldc(brow, 32 * i, sp, h), acc);
  return acc;
}

// ---------------------------------------------------------------------------
// Forward.  One wave per 32 value channels (columns of S, all key rows in
// registers); wave w also scales the 32 key channels w for all waves.  One
// barrier per chunk, two sets of scaled rows, the next chunk's rows in flight.
// 32 heads of 16384 tokens, D = 128, 16 segments a head: 164 us, 4.3 TB/s
// (more than half of a chunk is the wait for its rows), after 92 us for the
// segments' parts (4.5 TB/s) and 11 for their scan; whole heads at once instead
// leave seven eighths of the CUs idle: 1450 us.
// ---------------------------------------------------------------------------
template <typename T, int D> struct GlrFwd {
  static constexpr int NW = D / 32, NT = 64 * NW;
  static constexpr int ST = D + MF<T>::PAD, WST = GlrBase<T>::WST;
  static constexpr int NLO = sizeof(T) == 2 ? 1 : 0;
  static constexpr int MAT = 32 * ST, WM = 32 * WST;
  static constexpr int ELEMS = (4 + 2 * NLO) * MAT + 2 * NW * WM;
};

template <typename T, int D, bool EXACT>
__global__ __launch_bounds__(2 * D) __attribute__((amdgpu_waves_per_eu(2))) void k_glr_fwd(GlrArgs a) {
  using F = MF<T>;
  using C = GlrFwd<T, D>;
  constexpr int NW = C::NW, ST = C::ST, WST = C::WST;
  __shared__ __align__(16) T smem[C::ELEMS];
  __shared__ __align__(16) float sfz[2][D], spend[2][D], slo[D], sall[D];
  __shared__ int sslow[2][NW];
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
  int l = lane, col = l & 31, h = l >> 5;
  auto sQ = [&](int i) { return smem + i * C::MAT; };
  auto sK = [&](int i) { return smem + (2 + i) * C::MAT; };
  auto sL = [&](int i) { return smem + (4 + i * C::NLO) * C::MAT; };
  T* sg = smem + (4 + 2 * C::NLO) * C::MAT + w * C::WM;
  T* sv = sg + NW * C::WM;
  if (EXACT && a.again[blockIdx.x] == 0) return;
  const int bh = blockIdx.x / a.G, seg = blockIdx.x % a.G;
  const int len = glr_len(a, bh), c0 = seg * a.cps, c1 = min(a.nch, c0 + a.cps);
  const size_t base = (size_t)bh * a.n * D + 32 * w;

  f32x16 S[NW];                                      // rows: key channel; column n: value channel 32 w + chan_of(n)
  {
    const float* src = a.G > 1 ? a.part + ((size_t)bh * a.G + seg) * D * D : a.s0 ? a.s0 + (size_t)bh * D * D : nullptr;
    load_state<NW>(l, S, src, D, 32 * w + chan_of(col));
  }
  // spend[c & 1]: the log decay that S still lacks before chunk c
  if (tid < D) spend[c0 & 1][tid] = 0.0f;
  __syncthreads();
  Picks<T> pick;
  pick.init(l);
  Row16<T> rq, rk, rg, rv;
  auto load = [&](int c) {
    const size_t at = base + (size_t)32 * c * D;
    const unsigned off = lane_off<T, D>(l, c, a.n);
    rq.load(lane_ptr((const T*)a.q + at, off)); rk.load(lane_ptr((const T*)a.k + at, off));
    rg.load(lane_ptr((const T*)a.g + at, off)); rv.load(lane_ptr((const T*)a.v + at, off));
  };
  load(c0);
  const int cl = min(c1, (len + 31) / 32);           // chunks with rows that exist
  bool gave_up = false;
#pragma unroll 1
  for (int c = c0; c < cl; ++c) {
    l = lane_in(lane, c); col = l & 31; h = l >> 5;
    const int i = c & 1, t = 32 * c + col;
    const bool ok = t < len;
    rq.keep(ok); rk.keep(ok); rg.keep(ok); rv.keep(ok);
    put_row(sv + col * WST + 16 * h, rv);
    put_row(sg + col * WST + 16 * h, rg);
    wave_lds_sync();
    {
      f32x16 E;
      const bool fast = gate_chunk<T, false>(l, pick, sg, E, slo + 32 * w, spend[i] + 32 * w, spend[i ^ 1] + 32 * w, sfz[i] + 32 * w);
      put_decayed(l, sQ(i) + 32 * w, sQ(i), ST, rq, E, 1.0f, a.scale, false);
      put_decayed(l, sK(i) + 32 * w, sL(i) + 32 * w, ST, rk, E, -1.0f, 1.0f, a.exact);
      if (l == 0) sslow[i][w] = !fast;
    }
    if (c + 1 < cl) load(c + 1);
    __syncthreads();
    bool slow = false;
#pragma unroll
    for (int x = 0; x < NW; ++x) slow = slow || sslow[i][x];
    slow = uniform((int)slow);
    if (!EXACT && slow) {                            // the segment is left to the exact way
      gave_up = true;
      break;
    }
    const T *qrow = sQ(i) + col * ST, *krow = sK(i) + col * ST;
    f32x16 P = zero16(), O = zero16();               // P^T: rows s, columns t;  O^T: rows value channel
    auto readout = [&](auto with_p) {                // O = S q, and P of the same rows
#pragma unroll
      for (int dt = 0; dt < NW; ++dt)
#pragma unroll
        for (int sp = 0; sp < F::CSTEPS; ++sp) {
          const typename F::frag y = F::ldc(qrow, 32 * dt, sp, h);
          if constexpr (decltype(with_p)::value) P = F::mma(F::ldc(krow, 32 * dt, sp, h), y, P);
          O = F::mma(F::cfrag(S[dt], sp), y, O);
        }
    };
    if (!EXACT || !slow) {
      scale_rows<NW>(l, S, sfz[i]);
      readout(std::integral_constant<bool, true>{});
#pragma unroll
      for (int v = 0; v < 16; ++v) P[v] = crow(v, h) <= col ? P[v] : 0.0f;
    } else {
      // the exact way: level by level, then the decays from the start and to the end
      Row16<T> xq, xk;
      const unsigned off = lane_off<T, D>(l, c, a.n);
      xq.load(lane_ptr((const T*)a.q + base + (size_t)32 * c * D, off));
      xk.load(lane_ptr((const T*)a.k + base + (size_t)32 * c * D, off));
      xq.keep(ok); xk.keep(ok);
      gate_exact(l, sg);
      put_row(sQ(i) + col * ST + 32 * w + 16 * h, xq);
      put_row(sK(i) + col * ST + 32 * w + 16 * h, xk);
      __syncthreads();
      f32x16 M = rows_by_rows<T, NW>(h, krow, qrow);
#pragma unroll
      for (int v = 0; v < 16; ++v) P[v] = crow(v, h) == col ? M[v] : P[v];
      __syncthreads();
      float f[16];
      bool odd = true;                               // (two matrices in turn: one barrier for a level)
#pragma unroll 1
      for (int L = 1; L <= 16; L *= 2, odd = !odd) {
        T* X = odd ? sK(i) : sQ(i);
        put_level(l, L, sg, X + 32 * w, ST, xq, xk, f);
        __syncthreads();
        M = rows_by_rows<T, NW>(h, X + col * ST, X + col * ST);
        const int tc = row_if((col & L) != 0, col);
#pragma unroll
        for (int v = 0; v < 16; ++v) P[v] = joins(L, crow(v, h), tc) ? M[v] : P[v];
      }
#pragma unroll
      for (int v = 0; v < 16; ++v) P[v] *= a.scale;
      __syncthreads();
      border_exact(l, sg, slo + 32 * w, spend[i] + 32 * w, spend[i ^ 1] + 32 * w, sfz[i] + 32 * w, sall + 32 * w);
      f32x16 B = gate_sum(l, sg, UpTo{});
#pragma unroll
      for (int v = 0; v < 16; ++v) f[v] = ex(B[v]) * a.scale;
      put_scaled(l, sQ(i) + 32 * w, sQ(i), ST, xq.again(), f, false);
      B = gate_sum(l, sg, After{});
#pragma unroll
      for (int v = 0; v < 16; ++v) f[v] = ex(B[v]);
      put_scaled(l, sK(i) + 32 * w, sL(i) + 32 * w, ST, xk.again(), f, a.exact);
      __syncthreads();
      scale_rows<NW>(l, S, sfz[i]);
      readout(std::integral_constant<bool, false>{});
      scale_rows<NW>(l, S, sall);
      if (c + 1 < cl) load(c + 1);                   // (again, rather than kept through all this)
    }
#pragma unroll
    for (int sp = 0; sp < F::CSTEPS; ++sp) O = F::mma(rows_crow<true>(l, sv, WST, sp, 0), F::cfrag(P, sp), O);
#pragma unroll
    for (int ks = 0; ks < GlrBase<T>::NKS; ++ks) {
      const typename F::frag x = rows_nat<true>(l, sv, WST, ks, 0);
#pragma unroll
      for (int dt = 0; dt < NW; ++dt) S[dt] = F::mma(rows_nat<false>(l, sK(i), ST, ks, 32 * dt), x, S[dt]);
      if (C::NLO && a.exact) {
#pragma unroll
        for (int dt = 0; dt < NW; ++dt) S[dt] = F::mma(rows_nat<false>(l, sL(i), ST, ks, 32 * dt), x, S[dt]);
      }
    }
    float y[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) y[v] = ok ? O[v] : 0.0f;
    if (t < a.n) store_row(lane_ptr((T*)a.out + base + (size_t)32 * c * D, lane_off<T, D>(l, c, a.n)), y);
  }
  // rows that do not exist
  {
    float y[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) y[v] = 0.0f;
    for (int c = max(c0, cl); c < c1; ++c)
      if (32 * c + col < a.n) store_row(lane_ptr((T*)a.out + base + (size_t)32 * c * D, lane_off<T, D>(l, c, a.n)), y);
  }
  if (!EXACT && tid == 0) a.again[blockIdx.x] = gave_up;
  if (gave_up || a.s1 == nullptr || seg != a.G - 1) return;
  __syncthreads();
  if (tid < D) sall[tid] = ex(spend[max(c0, cl) & 1][tid]);
  __syncthreads();
  scale_rows<NW>(l, S, sall);
  float* dst = a.s1 + (size_t)bh * D * D;
#pragma unroll
  for (int dt = 0; dt < NW; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) dst[(size_t)(32 * dt + crow(v, h)) * D + 32 * w + chan_of(col)] = S[dt][v];
}

// ---------------------------------------------------------------------------
// State walk: wave w holds the state of key channels 32 w .. as S^T (rows: value
// channel, column n: key channel chan_of(n)), so a chunk's scaling is one
// register per lane and its scaled rows are the wave's own.
//   REV = false  S over a segment's rows, from k and v
//   REV = true   R backwards over a segment's rows, from q and do
// From zero, to the segment's own part and the decay across it.  STORE: also Z of
// every chunk (S_start on the exact way) as operand fragments for the backward,
// which adds what the segment's start state, decayed by `pre`, contributes; a
// single segment starts from s0 itself.  (The state is carried in float32; what is
// stored is rounded as the product that reads it would round it.)  Bound by memory: both walks of 32 heads
// of 16384 tokens, D = 128, with every chunk's 32 KB of Z written: 247 us, 5.4 TB/s.
// ---------------------------------------------------------------------------
template <typename T, int D> struct GlrWalk {
  static constexpr int NW = D / 32, NT = 64 * NW;
  static constexpr int ST = D + MF<T>::PAD, WST = GlrBase<T>::WST;
  static constexpr int NLO = sizeof(T) == 2 ? 1 : 0;
  static constexpr int ELEMS = 2 * 32 * ST + (2 + NLO) * NW * 32 * WST;
};

template <typename T, int D, bool REV, bool STORE>
LS_DEV void glr_walk(const GlrArgs& a, T* smem, float* svec, int (*sslow)[D / 32], int bh, int seg) {
  using F = MF<T>;
  using C = GlrWalk<T, D>;
  constexpr int NW = C::NW, ST = C::ST, WST = C::WST;
  const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6);
  int l = lane, col = l & 31, h = l >> 5;
  auto sV = [&](int i) { return smem + i * 32 * ST; };
  T* sg = smem + 2 * 32 * ST + w * (2 + C::NLO) * 32 * WST;
  T* sk = sg + 32 * WST;
  T* sl = sk + C::NLO * 32 * WST;
  const int len = glr_len(a, bh), c0 = seg * a.cps, c1 = min(a.nch, c0 + a.cps);
  const int cl = max(c0, min(c1, (len + 31) / 32));
  const size_t base = (size_t)bh * a.n * D + 32 * w;
  const float sc = REV ? a.scale : 1.0f;
  const int me = 32 * w + chan_of(col);                  // this lane's key channel

  f32x16 S[NW];
  {
    const float* src = STORE && a.G == 1 && a.s0 ? a.s0 + (size_t)bh * D * D : nullptr;
    load_state_t<NW>(l, S, src ? src + (size_t)me * D : nullptr);
  }
  // this wave's vectors: lack (two chunks), sums, scaling, decay across the chunk
  float *vec = svec + w * 160, *vlo = vec + 64, *vfz = vec + 96, *vall = vec + 128;
  if (l < 32) vec[l] = 0.0f;
  float total = 0.0f;                                    // log decay across the rows so far, of channel 32 w + l (l < 32)
  Picks<T> pick;
  pick.init(l);
  Row16<T> rk, rg, rv;
  auto load = [&](int c) {
    const size_t at = base + (size_t)32 * c * D;
    const unsigned off = lane_off<T, D>(l, c, a.n);
    rk.load(lane_ptr((const T*)(REV ? a.q : a.k) + at, off)); rg.load(lane_ptr((const T*)a.g + at, off));
    rv.load(lane_ptr((const T*)(REV ? a.dout : a.v) + at, off));
  };
  if (cl > c0) load(REV ? cl - 1 : c0);
#pragma unroll 1
  for (int u = 0; u < cl - c0; ++u) {
    l = lane_in(lane, u); col = l & 31; h = l >> 5;
    const int c = REV ? cl - 1 - u : c0 + u, i = u & 1, t = 32 * c + col;
    const bool ok = t < len;
    rk.keep(ok); rg.keep(ok); rv.keep(ok);
    put_row(sV(i) + col * ST + 32 * w + 16 * h, rv);
    put_row(sg + col * WST + 16 * h, rg);
    wave_lds_sync();
    const Row16<T> xk = rk;
    {
      f32x16 E;
      const bool fast = gate_chunk<T, REV>(l, pick, sg, E, vlo, vec + 32 * i, vec + 32 * (i ^ 1), vfz);
      put_decayed(l, sk, sl, WST, rk, E, REV ? 1.0f : -1.0f, sc, a.exact);
      if (l == 0) sslow[i][w] = !fast;
    }
    if (u + 1 < cl - c0) load(REV ? c - 1 : c + 1);
    __syncthreads();
    bool slow = false;
#pragma unroll
    for (int x = 0; x < NW; ++x) slow = slow || sslow[i][x];
    slow = uniform((int)slow);
    if (STORE && a.G > 1 && l < 32)                      // the decay from the segment's start to what is stored
      a.pre[((size_t)bh * a.nch + c) * D + 32 * w + l] = total + (slow ? 0.0f : vlo[l]);
    if (__builtin_expect(!slow, 1)) {
      if (l < 32) total += vlo[l] + vec[32 * (i ^ 1) + l];
    } else {
      gate_exact(l, sg);
      border_exact(l, sg, vlo, vec + 32 * i, vec + 32 * (i ^ 1), vfz, vall);
      if (l < 32) total += vlo[l];
      f32x16 B;
      if (REV) B = gate_sum(l, sg, UpTo{});
      else B = gate_sum(l, sg, After{});
      float f[16];
#pragma unroll
      for (int v = 0; v < 16; ++v) f[v] = ex(B[v]) * sc;
      put_scaled(l, sk, sl, WST, xk.again(), f, a.exact);
      wave_lds_sync();
    }
    const float zc = vfz[chan_of(col)];
#pragma unroll
    for (int et = 0; et < NW; ++et) S[et] *= zc;
    if constexpr (STORE) {
      typename F::frag* dst = (typename F::frag*)a.states + (((size_t)bh * a.nch + c) * NW + w) * NW * F::CSTEPS * 64 + (unsigned)l;
#pragma unroll
      for (int et = 0; et < NW; ++et)
#pragma unroll
        for (int sp = 0; sp < F::CSTEPS; ++sp) dst[(et * F::CSTEPS + sp) * 64] = F::cfrag(S[et], sp);
    }
    if (slow) {
      const float ac = vall[chan_of(col)];
#pragma unroll
      for (int et = 0; et < NW; ++et) S[et] *= ac;
    }
#pragma unroll
    for (int ks = 0; ks < GlrBase<T>::NKS; ++ks) {
      const typename F::frag x = rows_nat<true>(l, sk, WST, ks, 0);
      typename F::frag xl = F::zero();
      if (C::NLO && a.exact) xl = rows_nat<true>(l, sl, WST, ks, 0);
#pragma unroll
      for (int et = 0; et < NW; ++et) {
        const typename F::frag y = rows_nat<false>(l, sV(i), ST, ks, 32 * et);
        S[et] = F::mma(y, x, S[et]);
        if (C::NLO && a.exact) S[et] = F::mma(y, xl, S[et]);
      }
    }
  }
  if (!STORE || seg < a.G - 1) {
    wave_lds_sync();
    if (l < 32) (REV ? a.rfac : a.fac)[((size_t)bh * a.G + seg) * D + 32 * w + l] = ex(total);
    const float zc = ex(vec[32 * ((cl - c0) & 1) + chan_of(col)]);
    float* dst = (REV ? a.rpart : a.part) + ((size_t)bh * a.G + seg) * D * D + (size_t)me * D;
#pragma unroll
    for (int et = 0; et < NW; ++et)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(f32x4*)(dst + 32 * et + 8 * g + 4 * h) =
            f32x4{S[et][4 * g] * zc, S[et][4 * g + 1] * zc, S[et][4 * g + 2] * zc, S[et][4 * g + 3] * zc};
  }
}

// The segments' own parts (the last segment adds to no later one; reversed, the
// first to no earlier one), for the backward with every chunk's Z.
template <typename T, int D, bool BWD>
__global__ __launch_bounds__(2 * D) __attribute__((amdgpu_waves_per_eu(2))) void k_glr_walk(GlrArgs a) {
  using C = GlrWalk<T, D>;
  __shared__ __align__(16) T smem[C::ELEMS];
  __shared__ __align__(16) float svec[C::NW * 160];
  __shared__ int sslow[2][C::NW];
  const int segs = BWD ? a.G : a.G - 1, bh = blockIdx.x / segs, seg = blockIdx.x % segs;
  if (blockIdx.y == 0) glr_walk<T, D, false, BWD>(a, smem, svec, sslow, bh, seg);
  else if (BWD && seg > 0) glr_walk<T, D, true, false>(a, smem, svec, sslow, bh, seg);
}

// The state that every segment starts from, in the place of its part: four
// elements of one row per thread.  blockIdx.z: forward, reverse.
template <int D> __global__ __launch_bounds__(256) void k_glr_scan(GlrArgs a) {
  const int bh = blockIdx.y, i4 = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (i4 >= D * D) return;
  const bool rev = blockIdx.z != 0;
  float* p = (rev ? a.rpart : a.part) + (size_t)bh * a.G * D * D + i4;
  const float* f = (rev ? a.rfac : a.fac) + (size_t)bh * a.G * D + i4 / D;
  const float* init = rev ? a.ds1 : a.s0;
  f32x4 cur = init ? *(const f32x4*)(init + (size_t)bh * D * D + i4) : f32x4{0.f, 0.f, 0.f, 0.f};
  constexpr int NB = 8;                                   // parts in flight
  for (int j0 = 0; j0 < a.G; j0 += NB) {
    f32x4 x[NB];
    float y[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int u = min(j0 + j, a.G - 2), s = rev ? a.G - 1 - u : u;
      x[j] = *(const f32x4*)(p + (size_t)s * D * D);
      y[j] = f[(size_t)s * D];
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int u = j0 + j, s = rev ? a.G - 1 - u : u;
      if (u < a.G) {
        *(f32x4*)(p + (size_t)s * D * D) = cur;
        cur = cur * y[j] + x[j];
      }
    }
  }
}

// sum over this lane and the later lanes of its half (lane <-> row t of the chunk)
LS_DEV float rows_from(float x) {
  const int l = lane_id();
  x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x101, 0xF, 0xF, true));   // row_shl:1, 0 past the end
  x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x102, 0xF, 0xF, true));
  x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x104, 0xF, 0xF, true));
  x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x108, 0xF, 0xF, true));
  const float up0 = rlane(x, 16), up1 = rlane(x, 48);     // the later 16 rows' sum, for the earlier ones
  return x + ((l & 16) ? 0.0f : (l & 32) ? up1 : up0);
}

// ---------------------------------------------------------------------------
// Backward, from the last chunk of a segment to its first.  Waves 0 .. NW-1 own
// 32 key channels each (dq, dk, dg; R transposed, column n: key channel), waves
// NW .. 2 NW-1 own 32 value channels each (dv; R, column n: value channel).
// With c_r = (q_r e_r) * (dq part from s < r) - (k_r / e_r) * (dk part from t > r)
//   dg_t = W + sum_{r >= t} c_r,  W = rowsum(R_end * S_end):
// every pair adds to the rows it spans and cancels before them, with the same
// rounded factors on both sides, so nothing is left of it there; the pairs of a
// row with itself are left out of c and added to dq and dk apart.
// 32 heads of 16384 tokens, D = 128: 444 us, 4.0 TB/s (Z is a third of the bytes).
// Both kinds of wave work on one chunk between two barriers and hold 256
// registers, two waves on a SIMD; the vector pipe is 37% and the matrix pipe 16%
// busy, the rest is the chain from a chunk's gates to its gradients.  The exact
// instance at D = 128 keeps 260 to 288 of its registers in scratch memory, the
// forward's 161: with resets in every chunk the same case takes 2.0 ms backward
// and 0.56 forward.
// ---------------------------------------------------------------------------
template <typename T, int D, bool LOW> struct GlrBwd {
  static constexpr int NW = D / 32, NT = 128 * NW;
  static constexpr int ST = D + MF<T>::PAD, WST = GlrBase<T>::WST, EST = 36;
  static constexpr int MAT = 32 * ST;
  static constexpr int ELEMS = (LOW ? 10 : 8) * MAT + 2 * NW * 32 * WST;
};

template <typename T, int D, bool EXACT, bool LOW>
__global__ __launch_bounds__(4 * D) __attribute__((amdgpu_waves_per_eu(2))) void k_glr_bwd(GlrArgs a) {
  using F = MF<T>;
  using C = GlrBwd<T, D, LOW>;
  constexpr int NW = C::NW, ST = C::ST, NKS = GlrBase<T>::NKS;
  __shared__ __align__(16) T smem[C::ELEMS];
  __shared__ __align__(16) float sfz[2][D], spend[2][D], slo[D], sall[D], sw[D];
  __shared__ __align__(16) float se[2][NW][32 * C::EST];       // e_t of the key waves' rows
  __shared__ int sslow[2][NW];
  const int tid = threadIdx.x, lane = tid & 63, wv = uniform(tid >> 6);
  int l = lane, col = l & 31, h = l >> 5;
  const bool keys = wv < NW;
  const int w = keys ? wv : wv - NW;
  auto sQ = [&](int i) { return smem + i * C::MAT; };
  auto sK = [&](int i) { return smem + (2 + i) * C::MAT; };
  auto sV = [&](int i) { return smem + (4 + i) * C::MAT; };
  auto sO = [&](int i) { return smem + (6 + i) * C::MAT; };
  auto sL = [&](int i) { return smem + (LOW ? 8 + i : 0) * C::MAT; };
  auto sG = [&](int i) { return smem + (LOW ? 10 : 8) * C::MAT + (i * NW + w) * 32 * C::WST; };
  if (EXACT && a.again[blockIdx.x] == 0) return;
  const int bh = blockIdx.x / a.G, seg = blockIdx.x % a.G;
  const int len = glr_len(a, bh), c0 = seg * a.cps, c1 = min(a.nch, c0 + a.cps);
  const int cl = max(c0, min(c1, (len + 31) / 32));
  const size_t base = (size_t)bh * a.n * D + 32 * w;
  const float* src = a.G > 1 ? a.rpart + ((size_t)bh * a.G + seg) * D * D : a.ds1 ? a.ds1 + (size_t)bh * D * D : nullptr;

  // rows that do not exist
  {
    float y[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) y[v] = 0.0f;
    for (int c = cl; c < c1; ++c) {
      if (32 * c + col >= a.n) continue;
      const size_t at = base + (size_t)32 * c * D;
      const unsigned off = lane_off<T, D>(l, c, a.n);
      if (keys) {
        store_row(lane_ptr((T*)a.dq + at, off), y);
        store_row(lane_ptr((T*)a.dk + at, off), y);
        store_row(lane_ptr((T*)a.dg + at, off), y);
      } else {
        store_row(lane_ptr((T*)a.dv + at, off), y);
      }
    }
  }
  // spend[c & 1]: the log decay that R still lacks after chunk c
  if (tid < D) spend[0][tid] = spend[1][tid] = 0.0f;
  __syncthreads();

  auto any_slow = [&](int i) {
    bool slow = false;
#pragma unroll
    for (int x = 0; x < NW; ++x) slow = slow || sslow[i][x];
    return uniform((int)slow) != 0;
  };
  f32x16 R[NW];
  bool gave_up = false;                                  // a chunk needs the exact way: the segment is left to it

  if (keys) {
    const int me = 32 * w + chan_of(col);
    load_state_t<NW>(l, R, src ? src + (size_t)me * D : nullptr);
    // the segment's start state, which the stored Z lack
    const bool start = a.G > 1 && (seg > 0 || a.s0 != nullptr);
    Tile<T> z0[NW];
    {
      f32x16 x[NW];
      load_state_t<NW>(l, x, start ? a.part + (((size_t)bh * a.G + seg) * D + me) * D : nullptr);
#pragma unroll
      for (int et = 0; et < NW; ++et) z0[et].set(x[et]);
    }
#pragma unroll 1
    for (int c = cl - 1; c >= c0; --c) {
      l = lane_in(lane, c); col = l & 31; h = l >> 5;
      const int i = c & 1, t = 32 * c + col;
      const bool whole = 32 * c + 32 <= len, ok = t < len;
      T* sg = sG(i);
      // this chunk's rows where they are needed
      auto rows_of = [&](Row16<T>& xq, Row16<T>& xk) {
        const size_t at = base + (size_t)32 * c * D;
        const unsigned off = lane_off<T, D>(l, c, a.n);
        xq.load(lane_ptr((const T*)a.q + at, off)); xk.load(lane_ptr((const T*)a.k + at, off));
      };
      const typename F::frag* zs = (const typename F::frag*)a.states + (((size_t)bh * a.nch + c) * NW + w) * NW * F::CSTEPS * 64 + (unsigned)l;
      float decay = kNegInf;                             // of the start state, channel 32 w + (l & 31); log
      if (start) decay = a.pre[((size_t)bh * a.nch + c) * D + 32 * w + (unsigned)(l & 31)];
      typename F::frag z[NW][F::CSTEPS];                // Z of this chunk, on its way before the barrier
#pragma unroll
      for (int et = 0; et < NW; ++et)
#pragma unroll
        for (int sp = 0; sp < F::CSTEPS; ++sp) z[et][sp] = zs[(et * F::CSTEPS + sp) * 64];
      __syncthreads();
      const bool slow = any_slow(i);
      if (!EXACT && slow) {
        gave_up = true;
        break;
      }
      const T *vrow = sV(i) + col * ST, *orow = sO(i) + col * ST;
      T *qme = sQ(i) + col * ST + 32 * w + 16 * h, *kme = sK(i) + col * ST + 32 * w + 16 * h;

      // dP^T (rows s, columns t) and dP (rows t, columns s); the parts of dq, dk and W from outside the chunk
      Tile<T> dPt, dP;
      float diag = 0.0f, through = 0.0f;
      f32x16 aq = zero16(), ak = zero16();
      auto keep_pairs = [&](f32x16 pt, f32x16 p) {
#pragma unroll
        for (int v = 0; v < 16; ++v) diag += crow(v, h) == col ? pt[v] : 0.0f;
        diag = half_swap_add(diag);
        if (!EXACT || !slow) {                           // the strictly earlier pairs
          const int x = col - 4 * h;
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            pt[v] = crow(v, 0) < x ? pt[v] : 0.0f;
            p[v] = crow(v, 0) > x ? p[v] : 0.0f;
          }
        }
        dPt.set(pt);
        dP.set(p);
      };
      auto outside = [&](float zc, auto with_pairs) {
        f32x16 pt = zero16(), p = zero16(), a0 = zero16();
        float t0 = 0.0f;
#pragma unroll
        for (int et = 0; et < NW; ++et) {
          R[et] *= zc;
#pragma unroll
          for (int sp = 0; sp < F::CSTEPS; ++sp) {
            const typename F::frag vf = F::ldc(vrow, 32 * et, sp, h), of = F::ldc(orow, 32 * et, sp, h);
            if constexpr (decltype(with_pairs)::value) {
              pt = F::mma(vf, of, pt);
              p = F::mma(of, vf, p);
            }
            const typename F::frag r = F::cfrag(R[et], sp);
            through = dot_add(r, z[et][sp], through);
            t0 = dot_add(r, z0[et].f[sp], t0);
            aq = F::mma(z[et][sp], of, aq);
            ak = F::mma(r, vf, ak);
            a0 = F::mma(z0[et].f[sp], of, a0);
          }
          __builtin_amdgcn_sched_barrier(0);             // (one tile's operands in registers at a time)
        }
        if constexpr (decltype(with_pairs)::value) keep_pairs(pt, p);
        // what the segment's start state adds (without one: zeros)
        __builtin_amdgcn_sched_barrier(0);
        float y[16];
        if (h == 0) sw[32 * w + (l & 31)] = ex(decay);
        wave_lds_sync();
        get_vec(l, sw + 32 * w, y);
        through = __builtin_fmaf(sw[me], t0, through);
#pragma unroll
        for (int v = 0; v < 16; ++v) aq[v] = __builtin_fmaf(y[v], a0[v], aq[v]);
        wave_lds_sync();
        through = half_swap_add(through);
      };
      // W into sw: what passes through the chunk, and the pairs that start in it and end after it
      auto put_w = [&]() {
        float y[16];
        get_row(kme, y);
#pragma unroll
        for (int v = 0; v < 16; ++v) y[v] *= ak[v];
        const float ends = half_reduce16(y);
        if (h == 0) sw[me] = through;
        wave_lds_sync();
        if ((col & 1) == 0) sw[32 * w + 16 * h + (col >> 1)] += ends;
        wave_lds_sync();
      };
      // dg from the row sums
      auto put_dg = [&](float (&x)[16]) {
        float W[16];
        get_vec(l, sw + 32 * w, W);
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          x[v] = W[v] + rows_from(x[v]);
        }
        if (!whole) {
#pragma unroll
          for (int v = 0; v < 16; ++v) x[v] = ok ? x[v] : 0.0f;
        }
        if (t < a.n) store_row(lane_ptr((T*)a.dg + base + (size_t)32 * c * D, lane_off<T, D>(l, c, a.n)), x);
      };
      auto put_grad = [&](void* g, float (&x)[16]) {
        if (!whole) {
#pragma unroll
          for (int v = 0; v < 16; ++v) x[v] = ok ? x[v] : 0.0f;
        }
        if (t < a.n) store_row(lane_ptr((T*)g + base + (size_t)32 * c * D, lane_off<T, D>(l, c, a.n)), x);
      };
      if (!EXACT || !slow) {
        outside(sfz[i][me], std::integral_constant<bool, true>{});
        put_w();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int sp = 0; sp < F::CSTEPS; ++sp) {
          aq = F::mma(rows_crow<true>(l, sK(i), ST, sp, 32 * w), dPt.f[sp], aq);
          ak = F::mma(rows_crow<true>(l, sQ(i), ST, sp, 32 * w), dP.f[sp], ak);
        }
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) {
          const typename F::frag b = rows_nat<true>(l, sQ(i), ST, ks, 32 * w);
#pragma unroll
          for (int et = 0; et < NW; ++et) R[et] = F::mma(rows_nat<false>(l, sO(i), ST, ks, 32 * et), b, R[et]);
        }
        __builtin_amdgcn_sched_barrier(0);
        // (the pairs of a row with itself: dP_tt k_t = e_t dP_tt (k_t / e_t), and alike)
        float x[16], y[16];
        get_row(qme, x);
        get_row(kme, y);
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const float z = x[v] * aq[v] - y[v] * ak[v];
          aq[v] = __builtin_fmaf(diag, y[v], aq[v]);
          ak[v] = __builtin_fmaf(diag, x[v], ak[v]);
          x[v] = z;
        }
        put_dg(x);
        __builtin_amdgcn_sched_barrier(0);
        get_lane(se[i][w] + col * C::EST + 16 * h, y);
#pragma unroll
        for (int v = 0; v < 16; ++v) x[v] = y[v] * a.scale * aq[v];
        put_grad(a.dq, x);
#pragma unroll
        for (int v = 0; v < 16; ++v) x[v] = __builtin_amdgcn_rcpf(y[v]) * ak[v];
        put_grad(a.dk, x);
      } else {
        // the exact way: what comes from outside the chunk last, so that the rows are scaled for it then
        float dq[16], dk[16], x[16];
        Row16<T> xq, xk;
        rows_of(xq, xk);
        xq.keep(ok); xk.keep(ok);
        gate_exact(l, sg);
        keep_pairs(rows_by_rows<T, NW>(h, vrow, orow), rows_by_rows<T, NW>(h, orow, vrow));
#pragma unroll
        for (int v = 0; v < 16; ++v) dq[v] = dk[v] = x[v] = 0.0f;
        put_row(qme, xq);                                // (the diagonal, for the value waves)
        put_row(kme, xk);
        __syncthreads();
        __syncthreads();
        bool odd = true;                                 // (two matrices in turn: one barrier for a level)
#pragma unroll 1
        for (int L = 1; L <= 16; L *= 2, odd = !odd) {
          T* X = odd ? sK(i) : sQ(i);
          float f[16], y[16];
          put_level(l, L, sg, X + 32 * w, ST, xq, xk, f);
          __syncthreads();
          f32x16 b = zero16();
#pragma unroll
          for (int sp = 0; sp < F::CSTEPS; ++sp) b = F::mma(rows_crow<true>(l, X, ST, sp, 32 * w), dPt.level(l, sp, L, dP), b);
          get_row(X + col * ST + 32 * w + 16 * h, y);
          const bool later = (col & L) != 0;             // b is of dq in later halves, of dk in earlier ones
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const float z = b[v] * a.scale, e = f[v] * z;
            x[v] = __builtin_fmaf(later ? y[v] : -y[v], z, x[v]);
            dq[v] += later ? e : 0.0f;
            dk[v] += later ? 0.0f : e;
          }
        }
        {
          float f[16];
          __syncthreads();
          border_exact(l, sg, slo + 32 * w, spend[i] + 32 * w, spend[i ^ 1] + 32 * w, sfz[i] + 32 * w, sall + 32 * w);
          f32x16 B = gate_sum(l, sg, UpTo{});
#pragma unroll
          for (int v = 0; v < 16; ++v) f[v] = ex(B[v]) * a.scale;
          put_scaled(l, sQ(i) + 32 * w, sL(i) + 32 * w, ST, xq.again(), f, LOW);
          B = gate_sum(l, sg, After{});
#pragma unroll
          for (int v = 0; v < 16; ++v) f[v] = ex(B[v]);
          put_scaled(l, sK(i) + 32 * w, sK(i), ST, xk.again(), f, false);
          __syncthreads();
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int et = 0; et < NW; ++et)                  // (read again, rather than kept through the levels)
#pragma unroll
          for (int sp = 0; sp < F::CSTEPS; ++sp) z[et][sp] = zs[(et * F::CSTEPS + sp) * 64];
        outside(sfz[i][me], std::integral_constant<bool, false>{});
        through *= sall[me];
        put_w();
        float y[16];
        f32x16 B = gate_sum(l, sg, UpTo{});
        get_row(qme, y);
#pragma unroll
        for (int v = 0; v < 16; ++v) { x[v] += y[v] * aq[v]; dq[v] += ex(B[v]) * a.scale * aq[v]; }
        B = gate_sum(l, sg, After{});
        get_row(kme, y);
#pragma unroll
        for (int v = 0; v < 16; ++v) { x[v] -= y[v] * ak[v]; dk[v] += ex(B[v]) * ak[v]; }
        put_dg(x);
        __builtin_amdgcn_sched_barrier(0);
        rows_of(xq, xk);                                 // (again)
        xq.keep(ok); xk.keep(ok);
        diag *= a.scale;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          dq[v] = __builtin_fmaf(diag, xk.at(v), dq[v]);
          dk[v] = __builtin_fmaf(diag, xq.at(v), dk[v]);
        }
        put_grad(a.dq, dq);
        put_grad(a.dk, dk);
#pragma unroll
        for (int et = 0; et < NW; ++et) R[et] *= sall[me];
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) {
          const typename F::frag b = rows_nat<true>(l, sQ(i), ST, ks, 32 * w);
#pragma unroll
          for (int et = 0; et < NW; ++et) R[et] = F::mma(rows_nat<false>(l, sO(i), ST, ks, 32 * et), b, R[et]);
        }
      }
    }
  } else {
    load_state<NW>(l, R, src, D, 32 * w + chan_of(col));
    // They also scale the key rows: while the key waves work on chunk c, chunk c - 1
    // is staged, from rows loaded a chunk earlier.
    Picks<T> pick;
    pick.init(l);
    Row16<T> rq, rk, rg, rv, ro;
    auto load = [&](int c) {
      const size_t at = base + (size_t)32 * c * D;
      const unsigned off = lane_off<T, D>(l, c, a.n);
      rg.load(lane_ptr((const T*)a.g + at, off)); rq.load(lane_ptr((const T*)a.q + at, off));
      rk.load(lane_ptr((const T*)a.k + at, off)); rv.load(lane_ptr((const T*)a.v + at, off));
      ro.load(lane_ptr((const T*)a.dout + at, off));
    };
    auto stage = [&](int c) {
      const int i = c & 1;
      const bool ok = 32 * c + col < len;
      rq.keep(ok); rk.keep(ok); rg.keep(ok); rv.keep(ok); ro.keep(ok);
      put_row(sG(i) + col * C::WST + 16 * h, rg);
      put_row(sV(i) + col * ST + 32 * w + 16 * h, rv);
      put_row(sO(i) + col * ST + 32 * w + 16 * h, ro);
      wave_lds_sync();
      f32x16 E;
      const bool fast = gate_chunk<T, true>(l, pick, sG(i), E, slo + 32 * w, spend[i] + 32 * w, spend[i ^ 1] + 32 * w, sfz[i] + 32 * w);
      put_decayed(l, sK(i) + 32 * w, sK(i), ST, rk, E, -1.0f, 1.0f, false);
      float f[16];
#pragma unroll
      for (int v = 0; v < 16; ++v) f[v] = fast_exp2(E[v]);
      put_lane(se[i][w] + col * C::EST + 16 * h, f);
#pragma unroll
      for (int v = 0; v < 16; ++v) f[v] *= a.scale;
      put_scaled(l, sQ(i) + 32 * w, sL(i) + 32 * w, ST, rq, f, LOW);
      if (l == 0) sslow[i][w] = !fast;
      if (c > c0) load(c - 1);
    };
    if (cl > c0) {
      load(cl - 1);
      stage(cl - 1);
    }
#pragma unroll 1
    for (int c = cl - 1; c >= c0; --c) {
      l = lane_in(lane, c); col = l & 31; h = l >> 5;
      const int i = c & 1, t = 32 * c + col;
      __syncthreads();
      const bool slow = any_slow(i);
      if (!EXACT && slow) {
        gave_up = true;
        break;
      }
      const T *qrow = sQ(i) + col * ST, *krow = sK(i) + col * ST;
      f32x16 P = zero16(), A = zero16();                 // P: rows t, columns s;  A: dv^T
      auto outside = [&](auto with_p) {
#pragma unroll
        for (int dt = 0; dt < NW; ++dt)
#pragma unroll
          for (int sp = 0; sp < F::CSTEPS; ++sp) {
            const typename F::frag y = F::ldc(krow, 32 * dt, sp, h);
            if constexpr (decltype(with_p)::value) P = F::mma(F::ldc(qrow, 32 * dt, sp, h), y, P);
            A = F::mma(F::cfrag(R[dt], sp), y, A);
          }
      };
      if (!EXACT || !slow) {
        scale_rows<NW>(l, R, sfz[i]);
        outside(std::integral_constant<bool, true>{});
#pragma unroll
        for (int v = 0; v < 16; ++v) P[v] = crow(v, h) >= col ? P[v] : 0.0f;
      } else {
        __syncthreads();
        f32x16 M = rows_by_rows<T, NW>(h, qrow, krow);
#pragma unroll
        for (int v = 0; v < 16; ++v) P[v] = crow(v, h) == col ? M[v] : P[v];
        __syncthreads();
        bool odd = true;
#pragma unroll 1
        for (int L = 1; L <= 16; L *= 2, odd = !odd) {
          const T* X = (odd ? sK(i) : sQ(i)) + col * ST;
          __syncthreads();
          M = rows_by_rows<T, NW>(h, X, X);
          const int sc = row_if((col & L) == 0, col);
#pragma unroll
          for (int v = 0; v < 16; ++v) P[v] = joins(L, sc, crow(v, h)) ? M[v] : P[v];
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) P[v] *= a.scale;
        __syncthreads();
        __syncthreads();
        scale_rows<NW>(l, R, sfz[i]);
        outside(std::integral_constant<bool, false>{});
        scale_rows<NW>(l, R, sall);
      }
#pragma unroll
      for (int sp = 0; sp < F::CSTEPS; ++sp) A = F::mma(rows_crow<true>(l, sO(i), ST, sp, 32 * w), F::cfrag(P, sp), A);
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        const typename F::frag b = rows_nat<true>(l, sO(i), ST, ks, 32 * w);
#pragma unroll
        for (int dt = 0; dt < NW; ++dt) R[dt] = F::mma(rows_nat<false>(l, sQ(i), ST, ks, 32 * dt), b, R[dt]);
        if constexpr (LOW) {
#pragma unroll
          for (int dt = 0; dt < NW; ++dt) R[dt] = F::mma(rows_nat<false>(l, sL(i), ST, ks, 32 * dt), b, R[dt]);
        }
      }
      float y[16];
#pragma unroll
      for (int v = 0; v < 16; ++v) y[v] = t < len ? A[v] : 0.0f;
      if (t < a.n) store_row(lane_ptr((T*)a.dv + base + (size_t)32 * c * D, lane_off<T, D>(l, c, a.n)), y);
      if (c > c0) stage(c - 1);
    }
  }
  if (!EXACT && tid == 0) a.again[blockIdx.x] = gave_up;
  if (gave_up || a.ds0 == nullptr || seg != 0) return;
  // what R lacks before the first chunk (seg 0: c0 = 0, and chunk -1 has the other parity)
  __syncthreads();
  if (tid < D) sall[tid] = ex(cl > c0 ? spend[1][tid] : 0.0f);
  __syncthreads();
  if (keys) return;
  scale_rows<NW>(l, R, sall);
  float* dst = a.ds0 + (size_t)bh * D * D;
#pragma unroll
  for (int dt = 0; dt < NW; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) dst[(size_t)(32 * dt + crow(v, h)) * D + 32 * w + chan_of(col)] = R[dt][v];
}

// ---------------------------------------------------------------------------
// Single-token step: one workgroup per (sequence, head); the state is read and
// written once, 16 bytes per thread, all of a thread's rows in flight.  Bound by
// those bytes: 4096 states of 128 x 128: 84 us, 6.4 TB/s.
// ---------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__(256) void k_glr_step(const T* q, const T* k, const T* v, const T* g, float* state, T* out, float scale) {
  constexpr int TPR = D / 4, RP = 256 / TPR, IT = D / RP;      // threads per row, rows per pass
  __shared__ float sa[D], sk[D], sq[D];
  __shared__ __align__(16) float so[RP][D];
  const size_t bh = blockIdx.x;
  const int tid = threadIdx.x, e0 = (tid % TPR) * 4, r0 = tid / TPR;
  float* S = state + bh * D * D;
  f32x4 x[IT];
#pragma unroll
  for (int i = 0; i < IT; ++i) x[i] = *(const f32x4*)(S + (size_t)(r0 + i * RP) * D + e0);
  if (tid < D) {
    sa[tid] = ex((float)g[bh * D + tid]);
    sk[tid] = (float)k[bh * D + tid];
    sq[tid] = (float)q[bh * D + tid] * scale;
  }
  typedef T V4 __attribute__((ext_vector_type(4)));
  const V4 v4 = *(const V4*)(v + bh * D + e0);
  const f32x4 vv = {(float)v4[0], (float)v4[1], (float)v4[2], (float)v4[3]};
  __syncthreads();
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const int r = r0 + i * RP;
    x[i] = x[i] * sa[r] + vv * sk[r];
    o += x[i] * sq[r];
    *(f32x4*)(S + (size_t)r * D + e0) = x[i];
  }
  *(f32x4*)(so[r0] + e0) = o;
  __syncthreads();
  if (tid < D) {
    float y = 0.0f;
#pragma unroll
    for (int i = 0; i < RP; ++i) y += so[i][tid];
    out[bh * D + tid] = (T)y;
  }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
static int launch_status(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return 0;
  set_error("%s launch failed: %s", what, hipGetErrorString(e));
  return -4;
}

// Workgroups of the main kernel that a CU is counted with.  LDS lets it hold, forward
// at D = 32, 64, 128: 7, 4, 2 (float32 6, 3), backward: 4, 2, 1 (float32 3, 1), and these
// are taken except at two places in float32, where the measurements are against them.
// Microseconds of 32 heads of 16384, 256 of 1024 and 32 of 4096 tokens:
//   forward D = 32 bf16, counted 4: 66, 38, 28, 7: 61, 36, 29;  float32, 4: 130, 69, 45,
//   6: 143, 81, 53;  forward D = 64 float32, 4: 409, 191, 107, 3: 359, 183, 111;
//   backward D = 32 float32, 4: 376, 190, 103, 3: 339, 167, 97;  backward D = 64 float32,
//   2: 914, 450, 248, 1: 1000, 450, 265
static int counted_per_cu(const GlrShape& s, bool backward) {
  const bool half = s.dtype == 1;
  if (backward) return s.D == 128 ? 1 : s.D == 64 ? 2 : half ? 4 : 3;
  return s.D == 128 ? 2 : s.D == 64 ? (half ? 4 : 3) : half ? 7 : 4;
}

// Segments per (sequence, head): the count that minimises the time in units of
// one chunk of the main kernel, `slots` workgroups counted as running at once: rounds
// times (chunks per segment + its prologue and stores), and for more than one segment
// the walk that finds the segments' parts, the scan and two launches.  Forward
// and backward, D = 64, 48 heads of 2048 tokens: 427 us in one segment, 177 in 4,
// 137 in 8, 124 in 16, 151 in 32 (this rule: 16 forward, 10 backward, 121 us);
// D = 128, 32 heads of 16384: 5.7 ms in one, 1.84 in 4, 1.12 in 8 or 16, 1.38 in
// 64 (16 forward, 8 backward, 1.07 ms).
int glr_segments(const GlrShape& s, bool backward) {
  const int64_t slots = 256 * (int64_t)counted_per_cu(s, backward), BH = s.BH(), nch = s.nch();
  const double kEnds = 2.0, kWalk = backward ? 0.7 : 0.6, kLaunch = backward ? 4.0 : 6.0;
  int best = 1;
  double best_t = 1e300;
  for (int64_t G = 1; G <= 256 && G <= nch && (G == 1 || BH * G < 65536); ++G) {
    const int64_t cps = (nch + G - 1) / G;
    if ((nch + cps - 1) / cps != G) continue;                  // the last segment would be empty
    const double rounds = (double)((BH * G + slots - 1) / slots);
    double t = rounds * ((double)cps + kEnds);
    if (G > 1) t += kWalk * t + kLaunch + 0.3 * (double)(BH * G) / (double)slots;
    if (t < best_t) { best_t = t; best = (int)G; }
  }
  return best;
}

template <typename T, int D, bool BWD> static int run_parts(const GlrShape& s, const GlrArgs& a, hipStream_t st) {
  {
    const dim3 grid((unsigned)(s.BH() * (BWD ? a.G : a.G - 1)), BWD && a.G > 1 ? 2 : 1);
    ProfScope ps(BWD ? "glr_states" : "glr_parts", st);
    k_glr_walk<T, D, BWD><<<grid, 2 * D, 0, st>>>(a);
  }
  if (int rc = launch_status("glr parts")) return rc;
  if (a.G == 1) return 0;
  ProfScope ps("glr_scan", st);
  k_glr_scan<D><<<dim3((D * D / 4 + 255) / 256, (unsigned)s.BH(), BWD ? 2 : 1), 256, 0, st>>>(a);
  return launch_status("glr scan");
}

template <typename T, int D> static int run_fwd(const GlrShape& s, const GlrArgs& a, hipStream_t st) {
  (void)hipGetLastError();
  if (a.G > 1)
    if (int rc = run_parts<T, D, false>(s, a, st)) return rc;
  const unsigned grid = (unsigned)(s.BH() * a.G);
  {
    ProfScope ps("glr_fwd", st);
    k_glr_fwd<T, D, false><<<grid, 2 * D, 0, st>>>(a);
  }
  if (int rc = launch_status("glr forward")) return rc;
  ProfScope ps("glr_fwd_exact", st);
  k_glr_fwd<T, D, true><<<grid, 2 * D, 0, st>>>(a);
  return launch_status("glr forward, exact way");
}

// the short way's launch, then that of the segments that it left
template <typename T, int D, bool LOW> static int run_sweeps(const GlrShape& s, const GlrArgs& a, hipStream_t st) {
  const unsigned grid = (unsigned)(s.BH() * a.G);
  {
    ProfScope ps("glr_bwd", st);
    k_glr_bwd<T, D, false, LOW><<<grid, 4 * D, 0, st>>>(a);
  }
  if (int rc = launch_status("glr backward")) return rc;
  ProfScope ps("glr_bwd_exact", st);
  k_glr_bwd<T, D, true, LOW><<<grid, 4 * D, 0, st>>>(a);
  return launch_status("glr backward, exact way");
}

template <typename T, int D> static int run_bwd(const GlrShape& s, const GlrArgs& a, hipStream_t st) {
  (void)hipGetLastError();
  if (int rc = run_parts<T, D, true>(s, a, st)) return rc;
  return sizeof(T) == 2 && a.exact ? run_sweeps<T, D, sizeof(T) == 2>(s, a, st) : run_sweeps<T, D, false>(s, a, st);
}

#define GLR_DISPATCH(FN, ...)                                                    \
  if (s.dtype == 1 && s.D == 32) return FN<bf16, 32>(__VA_ARGS__);               \
  if (s.dtype == 1 && s.D == 64) return FN<bf16, 64>(__VA_ARGS__);               \
  if (s.dtype == 1 && s.D == 128) return FN<bf16, 128>(__VA_ARGS__);             \
  if (s.dtype == 0 && s.D == 32) return FN<float, 32>(__VA_ARGS__);              \
  if (s.dtype == 0 && s.D == 64) return FN<float, 64>(__VA_ARGS__);              \
  set_error("glr: unsupported dtype=%d D=%d", s.dtype, s.D);                     \
  return -2;

int launch_glr_fwd(const GlrShape& s, GlrArgs a, hipStream_t st) { GLR_DISPATCH(run_fwd, s, a, st) }
int launch_glr_bwd(const GlrShape& s, GlrArgs a, hipStream_t st) { GLR_DISPATCH(run_bwd, s, a, st) }

template <typename T, int D>
static int run_step(const GlrShape& s, const void* q, const void* k, const void* v, const void* g, float* state,
                    void* out, hipStream_t st) {
  (void)hipGetLastError();
  ProfScope ps("glr_step", st);
  k_glr_step<T, D><<<(unsigned)s.BH(), 256, 0, st>>>((const T*)q, (const T*)k, (const T*)v, (const T*)g, state, (T*)out, s.scale);
  return launch_status("glr step");
}
int launch_glr_step(const GlrShape& s, const void* q, const void* k, const void* v, const void* g, float* state,
                    void* out, hipStream_t st) {
  GLR_DISPATCH(run_step, s, q, k, v, g, state, out, st)
}

}  // namespace linsimp
