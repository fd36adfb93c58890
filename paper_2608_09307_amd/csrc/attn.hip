// Softmax attention on gfx950: forward, backward from recomputed probabilities,
// and the single-token step on a ring cache.
//
//   s_ij = scale q_i . k_j over the visible j,  lse_i = log sum_j exp s_ij
//   p_ij = exp(s_ij - lse_i),  o_i = sum_j p_ij v_j
//   delta_i = do_i . o_i,  ds_ij = p_ij (do_i . v_j - delta_i)
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i
//
// Every product runs on 32 x 32 matrix-core tiles (common.h): a tile of scores
// is formed with the contraction index of the next product on its rows, so the
// probabilities go from accumulator registers straight into that product's
// operand and never through LDS.  Probabilities and ds are rounded to the
// operand type there (bf16: 2^-8 relative at most, and the errors average out
// over the keys); scores, maxima, sums and outputs are float32 until the final
// store.
//
// Times beside the kernels are of a settled clock (it moves with the load for the
// first 10 to 50 ms of a run, and the times by up to 30% with it); two times with
// an arrow, or a list of variants, were taken in turn in one session each and
// compare with each other only.
#include "attn.h"

#include <math.h>

#include "common.h"
#include "linsimp_internal.h"
#include "prof.h"

namespace linsimp {

static constexpr int kMaxSplits = 64;
static constexpr float kLn2 = 0.6931471805599453f;

// A sequence's lengths and its mask: query i (position i + off) sees key j when
// lo(i) <= j <= hi(i).
struct Seq {
  int lq, lk, off, causal, window;
  LS_DEV int lo(int i) const { return window > 0 ? max(0, i + off - window + 1) : 0; }
  LS_DEV int hi(int i) const { return causal ? min(lk - 1, i + off) : lk - 1; }
  // the queries that see key j: first(j) <= i <= last(j)
  LS_DEV int first(int j) const { return j >= lk ? lq : causal ? j - off : 0; }
  LS_DEV int last(int j) const { return window > 0 ? min(lq - 1, j - off + window - 1) : lq - 1; }
};

LS_DEV Seq seq_of(const AttnArgs& a, int b) {
  Seq s;
  s.lq = a.lens_q ? min(max(a.lens_q[b], 0), a.nq) : a.nq;
  s.lk = a.lens_k ? min(max(a.lens_k[b], 0), a.nk) : a.nk;
  s.off = s.lk - s.lq;
  s.causal = a.causal;
  s.window = a.window;
  return s;
}

// Workgroup -> (tile, head).  Workgroups are dealt to the eight XCDs in turn, so
// with a multiple of eight heads every XCD keeps whole heads, whose tiles share
// its L2; the longest tiles of all of them come first (48 heads of 2048 tokens,
// D = 64: key sweep 139 -> 105 us against whole heads in turn, which left a CU
// with the long tiles of each).
LS_DEV void tile_and_head(int nt, int heads, bool late_first, int& tile, int& head) {
  const int lin = (int)blockIdx.x;
  int t;
  if (heads % 8 == 0) {
    const int hx = heads >> 3, slot = lin >> 3;
    head = (lin & 7) + 8 * (slot % hx);
    t = slot / hx;
  } else {
    head = lin % heads;
    t = lin / heads;
  }
  tile = late_first ? nt - 1 - t : t;
}

// Workgroup -> (32 columns, part of a key head's keys).  The `ncg` workgroups that read
// the same keys run one after the other, with a multiple of eight parts on one XCD, so
// that the keys come from its L2 (512 sequences, 16 heads on 4, 32 queries, 512 keys,
// D = 128: 423 -> 214 us against all parts of one set of columns after the other).
LS_DEV void cols_and_part(int ncg, int parts, int& cg, int& part) {
  const int lin = (int)blockIdx.x;
  if (parts % 8 == 0) {
    const int slot = lin >> 3;
    cg = slot % ncg;
    part = (slot / ncg) * 8 + (lin & 7);
  } else {
    cg = lin % ncg;
    part = lin / ncg;
  }
}

// Row padding of the backward's tiles, which are read by rows and transposed: a
// pitch of 80 or 208 bytes modulo 256 (16 heads of 16k tokens, D = 128: key sweep
// 2.38 -> 2.20 ms, query sweep 1.57 -> 1.51 against tr_pad's pitch, at which the
// row reads conflict; 16 or 48 bytes: 2.36 and 2.25; 32: 2.24).
template <typename T, int N> constexpr int both_pad() {
  if (sizeof(T) != 2) return 1;
  for (int p = 0; p < 128; p += 8) {
    const int b = (2 * (N + p)) % 256;
    if (b == 80 || b == 208) return p;
  }
  return 8;
}

// 16 bytes of a row to LDS, whole where the rows are laid out in 16-byte steps
template <typename T, typename V>
LS_DEV void put_piece(T* at, int lstride, V x) {
  if ((lstride * (int)sizeof(T)) % 16 == 0) {
    *(V*)at = x;
  } else {
#pragma unroll
    for (int e = 0; e < 16 / (int)sizeof(T); ++e) at[e] = x[e];
  }
}

// Staging of row tiles (common.h) with one address for the workgroup and an offset
// in 32 bits per lane: rows row0 .. of a dense [*, COLS] matrix of `rows` rows,
// those past its end read from its last one (and staged as zeros).
template <typename T, int ROWS, int COLS, int NT>
struct TileRows : StageRows<T, ROWS, COLS, NT> {
  using S = StageRows<T, ROWS, COLS, NT>;
  LS_DEV void load(const T* g, int row0, int rows, int tid) {
    const int at = min(row0, rows - 1), last = rows - 1 - at;
    const char* base = (const char*)(g + (size_t)at * COLS);
#pragma unroll
    for (int it = 0; it < S::IT; ++it) {
      const int idx = min(tid + NT * it, S::N - 1);
      const unsigned off = (unsigned)((min(idx / S::CPR, last) * COLS + (idx % S::CPR) * S::VE) * (int)sizeof(T));
      this->x[it] = *(const typename S::V*)(base + off);
    }
  }
  // rows from hi on become zeros, in the one tile that has them: a select for each
  // value of every tile was a quarter of the forward's instructions at D = 64
  LS_DEV void store(T* lds, int lstride, int row0, int hi, int tid) {
    if (row0 + ROWS > hi) {
#pragma unroll
      for (int it = 0; it < S::IT; ++it)
        if (row0 + (tid + NT * it) / S::CPR >= hi) this->x[it] = typename S::V{};
    }
#pragma unroll
    for (int it = 0; it < S::IT; ++it) {
      const int idx = tid + NT * it;
      if (S::N % NT != 0 && idx >= S::N) continue;
      put_piece(lds + (idx / S::CPR) * lstride + (idx % S::CPR) * S::VE, lstride, this->x[it]);
    }
  }
};

// operand fragments of one row of a dense [*, D] matrix (lane's row, its half's k)
template <typename T, int D>
LS_DEV void row_frags(typename MF<T>::frag (&f)[D / MF<T>::KS], const T* row) {
  const int h = lane_id() >> 5;
#pragma unroll
  for (int s = 0; s < D / MF<T>::KS; ++s) f[s] = MF<T>::ld(row, s * MF<T>::KS + h * MF<T>::KPL);
}

// an accumulator column (rows e = 32 et + crow(v, h)) to `row`, four values at a time
template <typename T, int D>
LS_DEV void store_col(T* row, const f32x16 (&acc)[D / 32], float f) {
  const int h = lane_id() >> 5;
  typedef T V4 __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int et = 0; et < D / 32; ++et)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      V4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = (T)(acc[et][4 * g + e] * f);
      *(V4*)(row + et * 32 + 8 * g + 4 * h) = y;
    }
}

// an accumulator whose rows start from row[0 .. 31]
LS_DEV f32x16 crow_acc(const float* row) {
  float x[16];
  crow_vals(row, x);
  f32x16 a;
#pragma unroll
  for (int v = 0; v < 16; ++v) a[v] = x[v];
  return a;
}

LS_DEV f32x16 splat16(float x) {
  f32x16 a;
#pragma unroll
  for (int v = 0; v < 16; ++v) a[v] = x;
  return a;
}

// Running maximum (in log2 units), sum and output of 32 query columns.
template <int D>
struct Online {
  f32x16 o[D / 32];      // O^T: rows e, columns query
  float m, l;            // this lane's column (both halves agree on m; l is this half's part)
  LS_DEV void clear() {
#pragma unroll
    for (int et = 0; et < D / 32; ++et) o[et] = zero16();
    m = kNegInf;
    l = 0.0f;
  }
  // scores (masked ones at -inf) to probabilities, in place; c = scale log2(e).
  // The frame m only follows the maximum when that outgrows it by 2^8: the
  // frame cancels in o / l, and most tiles then rescale nothing.
  template <int NT>
  LS_DEV void absorb(f32x16 (&s)[NT], float c) {
    float mx = kNegInf;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[t][v]);
    mx = half_swap_max(mx) * c;
    if (__any(mx > m + 8.0f)) {
      const float mn = fmaxf(m, mx);
      const float f = m == kNegInf ? 0.0f : fast_exp2(m - mn);
#pragma unroll
      for (int et = 0; et < D / 32; ++et) o[et] *= f;
      l *= f;
      m = mn;
    }
    const float ms = m == kNegInf ? 0.0f : m;          // nothing visible yet
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        s[t][v] = fast_exp2(__builtin_fmaf(s[t][v], c, -ms));
        l += s[t][v];
      }
  }
};

// ---------------------------------------------------------------------------
// Forward.  A workgroup of four waves owns 128 queries of one head, a wave 32 of
// them as matrix columns with their fragments in registers; keys come in tiles
// of 64, staged once for the four waves, two tiles in LDS and one on its way.
// With `ns` > 1 the keys are split over ns workgroups and joined afterwards.
// 16 heads of 16384 causal tokens, D = 128: 1.12 ms, 980 TFLOP/s (a square bf16
// matrix product of 8192: 1340), the matrix pipe 48% and the vector pipe 38% busy;
// 48 heads of 2048, D = 64: 42.5 us, 610 TFLOP/s, 28% and 43%.  Neither pipe is
// full: in a wave the scores' product, the maximum, the exps and the second product
// follow each other, and two or three waves of a SIMD do not fill the gaps.
// ---------------------------------------------------------------------------
template <typename T, int D>
struct FwdCfg {
  static constexpr int KT = 64, NW = 4, NT = 64 * NW, BQ = 32 * NW;
  static constexpr int KST = D + MF<T>::PAD, VST = D + tr_pad<T, D>();
  static constexpr int KB = KT * KST, VB = KT * VST;           // elements of one tile
  static constexpr int BYTES = 2 * (KB + VB) * (int)sizeof(T);
};

template <typename T, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void k_attn_fwd(AttnArgs a) {
  using F = MF<T>;
  using C = FwdCfg<T, D>;
  constexpr int KT = C::KT;
  static_assert(C::BYTES <= 80 * 1024, "two workgroups per CU");
  __shared__ __align__(16) T smem[2 * (C::KB + C::VB)];
  auto sK = [&](int i) { return smem + i * C::KB; };
  auto sV = [&](int i) { return smem + 2 * C::KB + i * C::VB; };
  const int tid = threadIdx.x, l = tid & 63, col = l & 31, h = l >> 5, wv = uniform(tid >> 6);
  int tile, bhs;
  tile_and_head(a.ntq, a.B * a.H * a.ns, a.causal, tile, bhs);
  const int bh = bhs / a.ns, sp = bhs % a.ns;
  const int b = bh / a.H, kh = (bh % a.H) / a.G;
  const Seq sq = seq_of(a, b);
  const int q0 = tile * C::BQ, qw = q0 + wv * 32, qi = qw + col;
  const T* ks = (const T*)a.k + ((size_t)b * a.Hkv + kh) * a.nk * D;
  const T* vs = (const T*)a.v + ((size_t)b * a.Hkv + kh) * a.nk * D;

  // key tiles of this workgroup (its share of them)
  int t0 = 0, t1 = 0;
  if (q0 < sq.lq) {
    const int qe = min(q0 + C::BQ, sq.lq) - 1;
    const int first = sq.lo(q0) / KT, last = sq.hi(qe) < 0 ? -1 : sq.hi(qe) / KT;
    const int per = (last - first + 1 + a.ns - 1) / a.ns;
    t0 = first + sp * per;
    t1 = min(last + 1, t0 + per);
  }
  typename F::frag qf[D / F::KS];
  row_frags<T, D>(qf, (const T*)a.q + ((size_t)bh * a.nq + min(qi, a.nq - 1)) * D);
  Online<D> st;
  st.clear();
  TileRows<T, KT, D, C::NT> rk, rv;
  if (t0 < t1) {
    rk.load(ks, t0 * KT, sq.lk, tid);
    rv.load(vs, t0 * KT, sq.lk, tid);
    rk.store(sK(0), C::KST, t0 * KT, sq.lk, tid);
    rv.store(sV(0), C::VST, t0 * KT, sq.lk, tid);
    rk.load(ks, (t0 + 1) * KT, sq.lk, tid);
    rv.load(vs, (t0 + 1) * KT, sq.lk, tid);
  }
  const int wlo = sq.lo(qw), whi = sq.hi(min(qw + 31, sq.lq - 1));      // keys any of the wave's queries sees
  const int alo = sq.lo(qw + 31), ahi = sq.hi(qw);                      // keys all of them see
#pragma unroll 1
  for (int t = t0; t < t1; ++t) {
    const int cur = (t - t0) & 1, k0 = t * KT;
    __syncthreads();                                    // tile t is staged; the other buffer is free
    if (t + 1 < t1) {
      rk.store(sK(cur ^ 1), C::KST, k0 + KT, sq.lk, tid);
      rv.store(sV(cur ^ 1), C::VST, k0 + KT, sq.lk, tid);
      rk.load(ks, k0 + 2 * KT, sq.lk, tid);
      rv.load(vs, k0 + 2 * KT, sq.lk, tid);
    }
    if (qw >= sq.lq || k0 > whi || k0 + KT <= wlo) continue;
    f32x16 s[KT / 32];
#pragma unroll
    for (int kt = 0; kt < KT / 32; ++kt) {
      const T* krow = sK(cur) + (kt * 32 + col) * C::KST;
      s[kt] = zero16();
#pragma unroll
      for (int i = 0; i < D / F::KS; ++i) s[kt] = F::mma(F::ld(krow, i * F::KS + h * F::KPL), qf[i], s[kt]);
    }
    if (k0 < alo || k0 + KT - 1 > ahi) {
      const int lo = sq.lo(qi), hi = sq.hi(qi);
#pragma unroll
      for (int kt = 0; kt < KT / 32; ++kt)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int j = k0 + kt * 32 + crow(v, h);
          s[kt][v] = j >= lo && j <= hi ? s[kt][v] : kNegInf;
        }
    }
    st.absorb(s, a.c);
#pragma unroll
    for (int kt = 0; kt < KT / 32; ++kt)
#pragma unroll
      for (int i = 0; i < F::CSTEPS; ++i) {
        const typename F::frag p = F::cfrag(s[kt], i);
#pragma unroll
        for (int et = 0; et < D / 32; ++et)
          st.o[et] = F::mma(F::tld_crow(sV(cur), C::VST, kt * 32, i, et * 32), p, st.o[et]);
      }
  }
  const float lt = half_swap_add(st.l);
  if (qi >= a.nq) return;
  if (a.ns > 1) {
    const size_t row = ((size_t)sp * a.B * a.H + bh) * a.nq + qi;
    store_col<float, D>(a.part + row * D, st.o, 1.0f);
    if (h == 0) *(float2*)(a.pml + row * 2) = float2{st.m, lt};
    return;
  }
  const bool none = qi >= sq.lq || lt == 0.0f;          // a padding row, or no visible key
  const size_t row = (size_t)bh * a.nq + qi;
  const float inv = 1.0f / lt;
  if (none) {
#pragma unroll
    for (int et = 0; et < D / 32; ++et) st.o[et] = zero16();
  }
  store_col<T, D>((T*)a.out + row * D, st.o, none ? 0.0f : inv);
  if (a.lse != nullptr && h == 0) a.lse[row] = none ? kNegInf : (st.m + __log2f(lt)) * kLn2;
}

// Joins the ns partial results of query rows, one row at a time in each group of
// D / 4 x P threads: P of them share the partial results of four columns.
template <typename T, int D, int P>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  constexpr int TPR = D / 4, RPB = 256 / (TPR * P);       // threads across a row, rows per workgroup
  __shared__ float sml[RPB][2 * kMaxSplits];
  __shared__ __align__(16) float so[RPB][P][D + 4];
  const size_t rows = (size_t)a.B * a.H * a.nq;
  const int tid = threadIdx.x, g = tid / (TPR * P), in = tid % (TPR * P), pr = in / TPR, e0 = (in % TPR) * 4;
  const size_t row = (size_t)blockIdx.x * RPB + g;
  const bool ok = row < rows;
  for (int s = in; ok && s < a.ns; s += TPR * P)
    *(float2*)&sml[g][2 * s] = *(const float2*)(a.pml + ((size_t)s * rows + row) * 2);
  __syncthreads();
  float m = kNegInf;
  for (int s = 0; ok && s < a.ns; ++s) m = fmaxf(m, sml[g][2 * s]);
  float l = 0.0f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = pr; ok && s < a.ns; s += P) {
    const float ms = sml[g][2 * s];
    const float f = ms == kNegInf ? 0.0f : fast_exp2(ms - m);
    o += *(const f32x4*)(a.part + ((size_t)s * rows + row) * D + e0) * f;
    l += sml[g][2 * s + 1] * f;
  }
  *(f32x4*)(so[g][pr] + e0) = o;
  if (e0 == 0) so[g][pr][D] = l;
  __syncthreads();
  if (!ok || pr != 0) return;
  l = so[g][0][D];
#pragma unroll
  for (int p = 1; p < P; ++p) {
    o += *(const f32x4*)(so[g][p] + e0);
    l += so[g][p][D];
  }
  const int b = (int)(row / ((size_t)a.H * a.nq)), i = (int)(row % a.nq);
  const bool none = i >= (a.lens_q ? a.lens_q[b] : a.nq) || l == 0.0f;
  typedef T V4 __attribute__((ext_vector_type(4)));
  V4 y;
  const float inv = 1.0f / l;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (T)(none ? 0.0f : o[e] * inv);
  *(V4*)((T*)a.out + row * D + e0) = y;
  if (a.lse != nullptr && e0 == 0) a.lse[row] = none ? kNegInf : (m + __log2f(l)) * kLn2;
}

// ---------------------------------------------------------------------------
// Few queries over a long axis (the single-token step, and forwards of at most
// 32 queries per head).  The queries of all heads that share a key head are the
// columns of a tile, so the keys are read once for 32 of them.  Each wave
// walks keys of its own in tiles of 32, through LDS of its own, without a
// barrier until the four waves (and then the ns workgroups) are joined.  Bound
// by the cache's bytes: one tile is in LDS and the next in flight in registers.
// 16 query heads on 4 key heads, 256 sequences in rings of 8192, D = 128: 0.55 ms,
// 6.0 TB/s (float32, D = 64: 0.63 ms, 5.3); 4 sequences of 64k tokens, 2 key heads:
// 30 us, 5.7 TB/s, and 5 to join.
// ---------------------------------------------------------------------------
template <typename T, int D>
struct FewCfg {
  static constexpr int NW = 4, NT = 64 * NW;
  static constexpr int KST = D + MF<T>::PAD, VST = D + tr_pad<T, D>();
  static constexpr int WAVE = 32 * (KST + VST) * (int)sizeof(T);
  static constexpr int JOIN = NW * 32 * (D + 4) * 4 + NW * 64 * 4;
  static constexpr int BYTES = NW * WAVE > JOIN ? NW * WAVE : JOIN;
};

// 32 rows of a cache of dense [*, D] rows, 16-byte pieces per lane, all in flight
template <typename T, int D>
struct WaveRows {
  static constexpr int VE = 16 / (int)sizeof(T), CPR = D / VE, IT = 32 * CPR / 64;
  typedef T V __attribute__((ext_vector_type(VE)));
  V x[IT];
  // row `slot` is read from `fresh` (the new token) instead
  LS_DEV void load(const T* g, int row0, int hi, int slot, const T* fresh) {
    const int l = lane_id();
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int idx = l + 64 * it, r = min(row0 + idx / CPR, hi - 1), c = (idx % CPR) * VE;
      const T* p = r == slot ? fresh : g + (size_t)r * D;
      x[it] = *(const V*)(p + c);
    }
  }
  LS_DEV void store(T* lds, int ld, int row0, int hi) {
    const int l = lane_id();
    if (row0 + 32 > hi) {
#pragma unroll
      for (int it = 0; it < IT; ++it)
        if (row0 + (l + 64 * it) / CPR >= hi) x[it] = V{};
    }
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int idx = l + 64 * it;
      put_piece(lds + (idx / CPR) * ld + (idx % CPR) * VE, ld, x[it]);
    }
  }
};

template <typename T, int D, bool STEP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void k_attn_few(AttnArgs a) {
  using F = MF<T>;
  using C = FewCfg<T, D>;
  static_assert(C::BYTES <= 80 * 1024, "two workgroups per CU");
  __shared__ __align__(16) char smem[C::BYTES];
  const int tid = threadIdx.x, l = tid & 63, col = l & 31, h = l >> 5, wv = uniform(tid >> 6);
  const int ncol = a.G * a.nq, ncg = (ncol + 31) / 32;
  int cg, part;
  cols_and_part(ncg, a.B * a.Hkv * a.ns, cg, part);
  const int sp = part % a.ns, bk = part / a.ns;
  const int b = bk / a.Hkv, kh = bk % a.Hkv;
  const int c = cg * 32 + col, cc = min(c, ncol - 1);
  const int qh = kh * a.G + cc / a.nq, qi = cc % a.nq;
  const size_t qrow = ((size_t)b * a.H + qh) * a.nq + qi;
  T* sK = (T*)(smem + wv * C::WAVE);
  T* sV = sK + 32 * C::KST;

  Seq sq;
  int slot = -1, lo, hi;
  if (STEP) {
    const int64_t p = a.pos[b];
    sq.lq = p < 0 ? 0 : 1;
    sq.lk = p < 0 ? 0 : p < (int64_t)a.nk ? (int)p + 1 : a.nk;
    slot = p < 0 ? -1 : (int)(p % a.nk);
    sq.off = sq.lk - sq.lq; sq.causal = 0; sq.window = 0;
    lo = 0; hi = sq.lk;
  } else {
    sq = seq_of(a, b);
    lo = sq.lq > 0 ? sq.lo(0) : 0;
    hi = sq.lq > 0 ? sq.hi(sq.lq - 1) + 1 : 0;
  }
  const size_t kv = ((size_t)b * a.Hkv + kh) * a.nk * D;
  const T *ks = (const T*)a.k + kv, *vs = (const T*)a.v + kv;
  const T *kn = STEP ? (const T*)a.knew + (size_t)bk * D : ks, *vn = STEP ? (const T*)a.vnew + (size_t)bk * D : vs;
  if (STEP && slot >= 0 && sp == 0 && cg == 0 && tid < D) {      // (no workgroup reads that slot from the cache)
    ((T*)a.k)[kv + (size_t)slot * D + tid] = kn[tid];
    ((T*)a.v)[kv + (size_t)slot * D + tid] = vn[tid];
  }
  const int first = lo / 32, ntile = hi > lo ? (hi - 1) / 32 - first + 1 : 0;
  const int per = (ntile + a.ns - 1) / a.ns;
  const int t0 = first + sp * per + wv, t1 = first + min(ntile, (sp + 1) * per);

  Online<D> st;
  st.clear();
  typename F::frag qf[D / F::KS];
  row_frags<T, D>(qf, (const T*)a.q + qrow * D);
  WaveRows<T, D> rk, rv;
  if (t0 < t1) {
    rk.load(ks, t0 * 32, hi, slot, kn);
    rv.load(vs, t0 * 32, hi, slot, vn);
  }
#pragma unroll 1
  for (int t = t0; t < t1; t += C::NW) {
    rk.store(sK, C::KST, t * 32, hi);
    rv.store(sV, C::VST, t * 32, hi);
    if (t + C::NW < t1) {
      rk.load(ks, (t + C::NW) * 32, hi, slot, kn);
      rv.load(vs, (t + C::NW) * 32, hi, slot, vn);
    }
    wave_lds_sync();
    f32x16 s[1];
    s[0] = zero16();
    const T* krow = sK + col * C::KST;
#pragma unroll
    for (int i = 0; i < D / F::KS; ++i) s[0] = F::mma(F::ld(krow, i * F::KS + h * F::KPL), qf[i], s[0]);
    const int jlo = sq.lo(qi), jhi = sq.hi(qi);
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const int j = t * 32 + crow(v, h);
      s[0][v] = j >= jlo && j <= jhi ? s[0][v] : kNegInf;
    }
    st.absorb(s, a.c);
#pragma unroll
    for (int i = 0; i < F::CSTEPS; ++i) {
      const typename F::frag p = F::cfrag(s[0], i);
#pragma unroll
      for (int et = 0; et < D / 32; ++et) st.o[et] = F::mma(F::tld_crow(sV, C::VST, 0, i, et * 32), p, st.o[et]);
    }
    wave_lds_sync();                                    // the reads above, before the next tile's writes
  }
  // join the waves
  const float lt = half_swap_add(st.l);
  float* sO = (float*)smem;                             // [NW][32 columns][D + 4]
  float* sM = sO + C::NW * 32 * (D + 4);                // [NW][32][2]
  __syncthreads();
  store_col<float, D>(sO + (wv * 32 + col) * (D + 4), st.o, 1.0f);
  if (h == 0) { sM[(wv * 32 + col) * 2] = st.m; sM[(wv * 32 + col) * 2 + 1] = lt; }
  __syncthreads();
  constexpr int TPR = D / 4;
  for (int r = tid / TPR; r < 32; r += C::NT / TPR) {
    const int rc = cg * 32 + r, e0 = (tid % TPR) * 4;
    if (rc >= ncol) break;
    float m = kNegInf, lsum = 0.0f;
#pragma unroll
    for (int w = 0; w < C::NW; ++w) m = fmaxf(m, sM[(w * 32 + r) * 2]);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < C::NW; ++w) {
      const float mw = sM[(w * 32 + r) * 2];
      const float f = mw == kNegInf ? 0.0f : fast_exp2(mw - m);
      lsum += sM[(w * 32 + r) * 2 + 1] * f;
      o += *(const f32x4*)(sO + (w * 32 + r) * (D + 4) + e0) * f;
    }
    const int i = rc % a.nq;
    const size_t row = ((size_t)b * a.H + kh * a.G + rc / a.nq) * a.nq + i;
    if (a.ns > 1) {
      const size_t prow = (size_t)sp * a.B * a.H * a.nq + row;
      *(f32x4*)(a.part + prow * D + e0) = o;
      if (e0 == 0) *(float2*)(a.pml + prow * 2) = float2{m, lsum};
      continue;
    }
    const bool none = i >= sq.lq || lsum == 0.0f;
    const float inv = 1.0f / lsum;
    typedef T V4 __attribute__((ext_vector_type(4)));
    V4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (T)(none ? 0.0f : o[e] * inv);
    *(V4*)((T*)a.out + row * D + e0) = y;
    if (a.lse != nullptr && e0 == 0) a.lse[row] = none ? kNegInf : (m + __log2f(lsum)) * kLn2;
  }
}

// ---------------------------------------------------------------------------
// Backward, query sweep: dq, and delta for the key sweep.  Layout of the
// forward: a wave owns 32 query columns with q and do in registers; per tile of
// 32 keys  S^T = K q,  dP^T = V do,  dS^T = P^T (dP^T - delta),  dq^T += K^T dS^T.
// Rows of up to 64 values take two such tiles at once, so that the exponentials
// of one run under the products of the other (48 heads of 2048 tokens, D = 64: 67
// -> 63 us, the key sweep 98 -> 88; at D = 128 there are no registers for it).
// delta is formed from the stored out, whose rounding to the operand type (bf16:
// 2^-8 of its terms) is all that dq holds in a row with a single key: the sum over
// p dP instead would need the whole row before its first ds.
// 16 heads of 16384 causal tokens, D = 128: 1.45 ms, 1130 TFLOP/s of its three
// products, the matrix pipe 59% busy, the LDS 50%.
// ---------------------------------------------------------------------------
template <typename T, int D>
struct DqCfg {
  static constexpr int KT = sizeof(T) == 2 && D < 128 ? 64 : 32, NW = 4, NT = 64 * NW, BQ = 32 * NW;
  static constexpr int KST = D + both_pad<T, D>(), VST = D + MF<T>::PAD;
  static constexpr int KB = KT * KST, VB = KT * VST;
  static constexpr int BYTES = 2 * (KB + VB) * (int)sizeof(T);
};

template <typename T, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void k_attn_dq(AttnArgs a) {
  using F = MF<T>;
  using C = DqCfg<T, D>;
  constexpr int KT = C::KT;
  __shared__ __align__(16) T smem[2 * (C::KB + C::VB)];
  auto sK = [&](int i) { return smem + i * C::KB; };
  auto sV = [&](int i) { return smem + 2 * C::KB + i * C::VB; };
  const int tid = threadIdx.x, l = tid & 63, col = l & 31, h = l >> 5, wv = uniform(tid >> 6);
  int tile, bhs;
  tile_and_head(a.ntq, a.B * a.H * a.nsq, a.causal, tile, bhs);
  const int bh = bhs / a.nsq, sp = bhs % a.nsq;
  const int b = bh / a.H, kh = (bh % a.H) / a.G;
  const Seq sq = seq_of(a, b);
  const int q0 = tile * C::BQ, qw = q0 + wv * 32, qi = qw + col;
  const T* ks = (const T*)a.k + ((size_t)b * a.Hkv + kh) * a.nk * D;
  const T* vs = (const T*)a.v + ((size_t)b * a.Hkv + kh) * a.nk * D;
  int t0 = 0, t1 = 0;
  if (q0 < sq.lq) {
    const int qe = min(q0 + C::BQ, sq.lq) - 1;
    const int first = sq.lo(q0) / KT, last = sq.hi(qe) < 0 ? -1 : sq.hi(qe) / KT;
    const int per = (last - first + a.nsq) / a.nsq;
    t0 = first + sp * per;
    t1 = min(last + 1, t0 + per);
  }
  const size_t row = (size_t)bh * a.nq + min(qi, a.nq - 1);
  typename F::frag qf[D / F::KS], of[D / F::KS];
  row_frags<T, D>(qf, (const T*)a.q + row * D);
  row_frags<T, D>(of, (const T*)a.dout + row * D);
  float delta = 0.0f;
  {
    const T* orow = (const T*)a.out + row * D;
#pragma unroll
    for (int s = 0; s < D / F::KS; ++s) {
      const typename F::frag x = F::ld(orow, s * F::KS + h * F::KPL);
#pragma unroll
      for (int e = 0; e < F::KPL; ++e) delta = __builtin_fmaf(fel(x, e), fel(of[s], e), delta);
    }
    delta = half_swap_add(delta);
  }
  const bool live = qi < sq.lq && a.lse[row] != kNegInf;
  // the products start from -lse / scale (-inf: a row without keys) and -delta
  const float s0 = live ? -a.lse[row] * kLog2e / a.c : kNegInf;
  if (!live) delta = 0.0f;
  if (qi < a.nq && h == 0 && sp == 0) a.delta[row] = delta;

  f32x16 acc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) acc[dt] = zero16();
  TileRows<T, KT, D, C::NT> rk, rv;
  if (t0 < t1) {
    rk.load(ks, t0 * KT, sq.lk, tid);
    rv.load(vs, t0 * KT, sq.lk, tid);
    rk.store(sK(0), C::KST, t0 * KT, sq.lk, tid);
    rv.store(sV(0), C::VST, t0 * KT, sq.lk, tid);
    rk.load(ks, (t0 + 1) * KT, sq.lk, tid);
    rv.load(vs, (t0 + 1) * KT, sq.lk, tid);
  }
  const int wlo = sq.lo(qw), whi = sq.hi(min(qw + 31, sq.lq - 1));
  const int alo = sq.lo(qw + 31), ahi = qw + 31 < sq.lq ? sq.hi(qw) : -1;
#pragma unroll 1
  for (int t = t0; t < t1; ++t) {
    const int cur = (t - t0) & 1, k0 = t * KT;
    __syncthreads();
    if (t + 1 < t1) {
      rk.store(sK(cur ^ 1), C::KST, k0 + KT, sq.lk, tid);
      rv.store(sV(cur ^ 1), C::VST, k0 + KT, sq.lk, tid);
      rk.load(ks, k0 + 2 * KT, sq.lk, tid);
      rv.load(vs, k0 + 2 * KT, sq.lk, tid);
    }
    if (qw >= sq.lq || k0 > whi || k0 + KT <= wlo) continue;
    f32x16 s[KT / 32], dp[KT / 32];
#pragma unroll
    for (int kt = 0; kt < KT / 32; ++kt) {
      const T* krow = sK(cur) + (kt * 32 + col) * C::KST;
      const T* vrow = sV(cur) + (kt * 32 + col) * C::VST;
      s[kt] = splat16(s0);
      dp[kt] = splat16(-delta);
#pragma unroll
      for (int i = 0; i < D / F::KS; ++i) {
        s[kt] = F::mma(F::ld(krow, i * F::KS + h * F::KPL), qf[i], s[kt]);
        dp[kt] = F::mma(F::ld(vrow, i * F::KS + h * F::KPL), of[i], dp[kt]);
      }
    }
    const bool part = k0 < alo || k0 + KT - 1 > ahi;
    const int lo = live ? sq.lo(qi) : 1, hi = live ? sq.hi(qi) : 0;
#pragma unroll
    for (int kt = 0; kt < KT / 32; ++kt) {
#pragma unroll
      for (int v = 0; v < 16; ++v) s[kt][v] = fast_exp2(s[kt][v] * a.c) * dp[kt][v];
    }
    if (part) {
#pragma unroll
      for (int kt = 0; kt < KT / 32; ++kt)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int j = k0 + kt * 32 + crow(v, h);
          s[kt][v] = j >= lo && j <= hi ? s[kt][v] : 0.0f;
        }
    }
#pragma unroll
    for (int kt = 0; kt < KT / 32; ++kt)
#pragma unroll
      for (int i = 0; i < F::CSTEPS; ++i) {
        const typename F::frag p = F::cfrag(s[kt], i);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
          acc[dt] = F::mma(F::tld_crow(sK(cur), C::KST, kt * 32, i, dt * 32), p, acc[dt]);
      }
  }
  if (qi >= a.nq) return;
  if (a.nsq > 1) store_col<float, D>(a.part + ((size_t)sp * a.B * a.H * a.nq + row) * D, acc, a.scale);
  else store_col<T, D>((T*)a.dq + row * D, acc, a.scale);
}

// The gradients of split sweeps: the ns partial sums of n elements, in order
// (blockIdx.y: of the first and of the second result).
template <typename T>
__global__ __launch_bounds__(256) void k_attn_sum(const float* part, T* out0, T* out1, size_t n, int ns) {
  typedef T V4 __attribute__((ext_vector_type(4)));
  const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  T* out = blockIdx.y ? out1 : out0;
  part += (size_t)blockIdx.y * ns * n;
  if (i >= n) return;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int s = 0; s < ns; ++s) x += *(const f32x4*)(part + (size_t)s * n + i);
  V4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = (T)x[e];
  *(V4*)(out + i) = y;
}

// ---------------------------------------------------------------------------
// Backward, key sweep: dk and dv.  A wave owns 32 key columns with k and v in
// registers; per tile of 32 query rows (of every head that shares the keys)
//   S = q K^T,  dP = do V^T,  dv^T += do^T P,  dk^T += q^T dS.
// Each gradient is summed by one wave in a fixed order: no atomics.
// 16 heads of 16384 causal tokens, D = 128: 2.14 ms, 1030 TFLOP/s of its four
// products, the matrix pipe 48% busy.  The LDS is the busiest unit, 55% with 22% of
// that bank conflicts: dk, dv and k take 192 of 256 registers, so v is read from it
// for every tile.
// ---------------------------------------------------------------------------
template <typename T, int D>
struct KvCfg {
  static constexpr int QT = sizeof(T) == 2 && D < 128 ? 64 : 32, NW = 4, NT = 64 * NW, BK = 32 * NW;
  static constexpr int ST = D + both_pad<T, D>();
  static constexpr int QB = QT * ST;
  static constexpr bool VLDS = sizeof(T) == 2 && D == 128;
  static constexpr int VST = D + MF<T>::PAD;
  static constexpr int BYTES = 2 * (2 * QB) * (int)sizeof(T) + 2 * 2 * QT * 4;
};

template <typename T, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void k_attn_dkv(AttnArgs a) {
  using F = MF<T>;
  using C = KvCfg<T, D>;
  constexpr int QT = C::QT;
  __shared__ __align__(16) T smem[4 * C::QB];
  __shared__ __align__(16) T sV[C::VLDS ? 128 * C::VST : 8];
  __shared__ __align__(16) float srow[2][2][QT];          // -lse / scale and -delta of the staged rows
  auto sQ = [&](int i) { return smem + i * C::QB; };
  auto sO = [&](int i) { return smem + (2 + i) * C::QB; };
  const int tid = threadIdx.x, l = tid & 63, col = l & 31, h = l >> 5, wv = uniform(tid >> 6);
  int tile, bks;
  tile_and_head(a.ntk, a.B * a.Hkv * a.nsk, false, tile, bks);
  const int bk = bks / a.nsk, sp = bks % a.nsk;
  const int b = bk / a.Hkv, kh = bk % a.Hkv;
  const Seq sq = seq_of(a, b);
  const int j0 = tile * C::BK, jw = j0 + wv * 32, kj = jw + col;
  const size_t first = ((size_t)bk * a.nk + min(kj, a.nk - 1)) * D;
  typename F::frag kf[D / F::KS], vf[D / F::KS];
  row_frags<T, D>(kf, (const T*)a.k + first);
  if constexpr (C::VLDS) {                                // (each half-wave row is read by its own lane only)
    row_frags<T, D>(vf, (const T*)a.v + first);
#pragma unroll
    for (int i = 0; i < D / F::KS; ++i) *(typename F::frag*)(sV + (wv * 32 + col) * C::VST + i * F::KS + h * F::KPL) = vf[i];
  } else {
    row_frags<T, D>(vf, (const T*)a.v + first);
  }

  // query rows that see any of the workgroup's keys
  int i0 = 0, i1 = 0;
  if (j0 < sq.lk) {
    i0 = a.causal ? max(0, j0 - sq.off) : 0;
    i1 = a.window > 0 ? min(sq.lq, min(j0 + C::BK, sq.lk) - 1 - sq.off + a.window) : sq.lq;
  }
  const int t0 = i0 / QT, per = i1 > i0 ? (i1 - 1) / QT - t0 + 1 : 0;      // tiles per head
  // tiles of all heads of the group in turn, this workgroup's share of them
  const int share = (per * a.G + a.nsk - 1) / a.nsk;
  const int u0 = min(sp * share, per * a.G), total = min(share, per * a.G - u0);

  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt) { dk[dt] = zero16(); dv[dt] = zero16(); }
  TileRows<T, QT, D, C::NT> rq, ro;
  float rs = 0.0f;
  const float rc = 1.0f / a.c;
  // the tile that is loaded next: head g of the group, rows r
  const int rlast = (t0 + per - 1) * QT;
  int lg = total > 0 ? u0 / per : 0, lr = (t0 + (total > 0 ? u0 % per : 0)) * QT;
  int r0 = lr;
  auto load = [&]() {
    const size_t base = ((size_t)b * a.H + kh * a.G + lg) * a.nq;
    rq.load((const T*)a.q + base * D, lr, sq.lq, tid);
    ro.load((const T*)a.dout + base * D, lr, sq.lq, tid);
    if (tid < 2 * QT) {
      const int r = min(lr + (tid & (QT - 1)), sq.lq - 1);
      const float x = tid < QT ? a.lse[base + r] : a.delta[base + r];
      rs = tid >= QT ? -x : x == kNegInf ? kNegInf : -x * kLog2e * rc;
    }
    const bool wrap = lr == rlast;
    lr = wrap ? t0 * QT : lr + QT;
    lg = wrap ? min(lg + 1, a.G - 1) : lg;
  };
  auto stage = [&](int r0, int i) {
    rq.store(sQ(i), C::ST, r0, sq.lq, tid);
    ro.store(sO(i), C::ST, r0, sq.lq, tid);
    if (tid < 2 * QT) srow[i][tid / QT][tid & (QT - 1)] = rs;
  };
  if (total > 0) {
    load();
    stage(r0, 0);
    load();
  }
#pragma unroll 1
  for (int u = 0; u < total; ++u) {
    const int cur = u & 1, rn = r0 == rlast ? t0 * QT : r0 + QT, rr = r0;
    __syncthreads();
    if (u + 1 < total) {
      stage(rn, cur ^ 1);
      load();
    }
    r0 = rn;
    // whether any (all) of the tile's rows see any (all) of the wave's keys
    const int re = min(rr + QT, sq.lq) - 1;
    if (jw >= sq.lk || sq.hi(re) < jw || sq.lo(rr) > jw + 31) continue;
    const bool all = rr + QT <= sq.lq && jw + 31 <= sq.hi(rr) && jw >= sq.lo(rr + QT - 1);
    const int ilo = sq.first(kj), ihi = sq.last(kj);
    // the products start from -lse / scale and -delta of their rows
    f32x16 s[QT / 32], dp[QT / 32];
#pragma unroll
    for (int qt = 0; qt < QT / 32; ++qt) {
      const T* qrow = sQ(cur) + (qt * 32 + col) * C::ST;
      s[qt] = crow_acc(srow[cur][0] + qt * 32);
#pragma unroll
      for (int i = 0; i < D / F::KS; ++i) s[qt] = F::mma(F::ld(qrow, i * F::KS + h * F::KPL), kf[i], s[qt]);
    }
#pragma unroll
    for (int qt = 0; qt < QT / 32; ++qt)
#pragma unroll
      for (int v = 0; v < 16; ++v) s[qt][v] = fast_exp2(s[qt][v] * a.c);
    if (!all) {
#pragma unroll
      for (int qt = 0; qt < QT / 32; ++qt)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int r = rr + qt * 32 + crow(v, h);
          s[qt][v] = r >= ilo && r <= ihi ? s[qt][v] : 0.0f;
        }
    }
#pragma unroll
    for (int qt = 0; qt < QT / 32; ++qt) {
      const T* orow = sO(cur) + (qt * 32 + col) * C::ST;
      dp[qt] = crow_acc(srow[cur][1] + qt * 32);
#pragma unroll
      for (int i = 0; i < D / F::KS; ++i)
        dp[qt] = F::mma(F::ld(orow, i * F::KS + h * F::KPL),
                        C::VLDS ? F::ld(sV + (wv * 32 + col) * C::VST, i * F::KS + h * F::KPL) : vf[i], dp[qt]);
#pragma unroll
      for (int i = 0; i < F::CSTEPS; ++i) {
        const typename F::frag p = F::cfrag(s[qt], i);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
          dv[dt] = F::mma(F::tld_crow(sO(cur), C::ST, qt * 32, i, dt * 32), p, dv[dt]);
      }
    }
#pragma unroll
    for (int qt = 0; qt < QT / 32; ++qt)
#pragma unroll
      for (int v = 0; v < 16; ++v) dp[qt][v] *= s[qt][v];
    if (!all) {                                          // (0 times whatever a key past the end holds)
#pragma unroll
      for (int qt = 0; qt < QT / 32; ++qt)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int r = rr + qt * 32 + crow(v, h);
          dp[qt][v] = r >= ilo && r <= ihi ? dp[qt][v] : 0.0f;
        }
    }
#pragma unroll
    for (int qt = 0; qt < QT / 32; ++qt)
#pragma unroll
      for (int i = 0; i < F::CSTEPS; ++i) {
        const typename F::frag ds = F::cfrag(dp[qt], i);
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
          dk[dt] = F::mma(F::tld_crow(sQ(cur), C::ST, qt * 32, i, dt * 32), ds, dk[dt]);
      }
  }
  if (kj >= a.nk) return;
  int j = jw + (lane_id() & 31);
  asm("" : "+v"(j));                                      // (the row's address made again, not kept through the loop)
  const size_t krow = (size_t)bk * a.nk + j;
  if (a.nsk > 1) {                                        // [2][ns][B][Hkv][nk][D]
    const size_t rows = (size_t)a.B * a.Hkv * a.nk;
    store_col<float, D>(a.part + ((size_t)sp * rows + krow) * D, dk, a.scale);
    store_col<float, D>(a.part + ((size_t)(a.nsk + sp) * rows + krow) * D, dv, 1.0f);
  } else {
    store_col<T, D>((T*)a.dk + krow * D, dk, a.scale);
    store_col<T, D>((T*)a.dv + krow * D, dv, 1.0f);
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

// Whether the few-row kernel runs (the step has no other), and so which time model
// the splits come from.  It reads a key head's keys once per 32 columns, the tiled
// kernel once per head and 128 queries: up to 32 queries of a head never more often.
// Microseconds, tiled / few-row, at G heads on a key head, D = 128:
//   256 sequences, 4 key heads, G = 4, 64, 512 and 2048 keys:  nq = 32: 44/44, 167/108,
//     575/339;  48: 49/61, 181/150, 593/457;  96: -, 204/283, 655/828
//   256 sequences, 16 heads, G = 1, the same:  nq = 32: 43/45, 217/207, 747/756;
//     40: 47/79, 228/235, 752/782
//   4 sequences, 2 key heads, G = 8, 65536 keys:  nq = 6: 307/56, 32: 312/145
// Above 32 it would still win where many heads share long keys and lose elsewhere.
bool attn_few(const AttnShape& s) { return s.nq <= 32; }

// Workgroups that share one query tile's (or key head's) keys, from the time in
// microseconds: the longest workgroup's key tiles and the whole load at the rate
// of a full chip, which add up in squares (neither is hidden behind the other
// when they are equal), and for more than one split the joining launch and the
// partial results.  The constants are measured: a tile of 64 keys takes
// 0.45 + 0.0075 D (float32: 0.3 + 0.05 D) on a CU, however many workgroups share
// the CU; a round of 128 keys of the few-row kernel 0.9 + 0.005 D, and all of
// them together the bytes of k and v at 5 TB/s.  A workgroup that has its CU to
// itself in the last round takes 1.36 times as long for a tile as one of two
// (32 heads of 1000 queries, 9000 keys, D = 128, where two fit: 246 us in one
// piece, 193 in two, 219 in three, 198 in four; D = 64, three: 99 in two, 102 in
// three, 112 in four, 107 in eight; D = 32, five: 74 in three, 70 in four, 76 in
// six; 64 heads, D = 32: 136 in two, 139 in three).  E.g. 16 heads of 2048 tokens,
// D = 128: 54 us in one piece, 46 in two; 4 heads' 64k keys for 16 heads and one
// token: 800 us in one piece, 40 in 32 to 64.  A step of 4 sequences, 64 heads on
// one key head, 64k slots, D = 128: 157 us in 4 pieces, 43 in the 38 taken; 8
// sequences, 128 heads on one, 32k slots: 297 in one piece, 49 in 16.
int attn_splits(const AttnShape& s) {
  const bool few = attn_few(s);
  const int64_t ntq = few ? 1 : (s.nq + 127) / 128;
  const double groups = (double)(few ? s.B * s.Hkv * ((s.H / s.Hkv * s.nq + 31) / 32) : s.B * s.H * ntq);
  double most = (double)s.nk, mean = (double)s.nk;        // keys of the longest and of the average workgroup
  if (s.causal && !few && s.nq <= s.nk) mean = (double)s.nk - 0.5 * (double)s.nq;
  if (s.window > 0) {
    const double w = (double)(s.window + 128);
    most = most < w ? most : w;
    mean = mean < w ? mean : w;
  }
  const double tile = few ? 128.0 : 64.0;
  const double us = few ? 0.9 + 0.005 * s.D : s.dtype == 1 ? 0.45 + 0.0075 * s.D : 0.3 + 0.05 * s.D;
  // workgroups of the tiled kernel that a CU holds (registers at D = 32, LDS above)
  const int fit = s.D == 32 ? (s.dtype == 1 ? 5 : 4) : s.D * s.esize() >= 256 ? 2 : 3;
  const double bytes = 2.0 * s.D * (double)s.esize();     // of one key and value
  const double partial = (double)(s.B * s.H * s.nq) * (s.D + 2) * 4.0;
  int best = 1;
  double best_t = 1e300;
  for (int n = 1; n <= kMaxSplits && (n == 1 || (n * tile < most + tile && groups * n < 65536)); ++n) {
    const double longest = (most / tile / n + (few ? 1.5 : 3.0)) * us;
    double load = few ? groups * mean * bytes / 5e6 + groups * n * 2.0 * us / 512
                      : groups * n * (mean / tile / n + 3.0) * us * 0.9 / 256;
    const int rounds = (int)ceil(groups * n / 256);
    if (!few && rounds > fit && rounds % fit == 1) load *= 1.0 + 0.36 / rounds;
    double t = sqrt(longest * longest + load * load);
    if (n > 1) t += 4.0 + n * partial / 4e6;
    if (t < 0.98 * best_t) { best_t = t; best = n; }
  }
  return best;
}

template <typename T, int D>
static int run_fwd(const AttnShape& s, AttnArgs a, hipStream_t st) {
  const char* what = a.pos != nullptr ? "attn step" : "attn forward";
  (void)hipGetLastError();
  if (attn_few(s)) {
    const unsigned grid = (unsigned)(s.B * s.Hkv * a.ns * ((a.G * a.nq + 31) / 32));
    ProfScope ps(a.pos != nullptr ? "attn_step" : "attn_few", st);
    if (a.pos != nullptr) k_attn_few<T, D, true><<<grid, 256, 0, st>>>(a);
    else k_attn_few<T, D, false><<<grid, 256, 0, st>>>(a);
  } else {
    ProfScope ps("attn_fwd", st);
    k_attn_fwd<T, D><<<(unsigned)(s.B * s.H * a.ns * a.ntq), 256, 0, st>>>(a);
  }
  if (int rc = launch_status(what)) return rc;
  if (a.ns > 1) {
    // many rows: one set of threads per row; few: all of a workgroup on one
    const int64_t rows = s.B * s.H * s.nq;
    ProfScope ps("attn_join", st);
    if (rows >= 4096) k_attn_join<T, D, 1><<<(unsigned)((rows + 1024 / D - 1) / (1024 / D)), 256, 0, st>>>(a);
    else k_attn_join<T, D, 1024 / D><<<(unsigned)rows, 256, 0, st>>>(a);
    return launch_status("attn join");
  }
  return 0;
}

// Splits of the backward sweeps, as above: `groups` workgroups of `most` (`mean`)
// tiles of 32 rows, `us` microseconds each; `bytes` of one partial result.
static int sweep_splits(double groups, double most, double mean, double us, double bytes) {
  int best = 1;
  double best_t = 1e300;
  for (int n = 1; n <= 32 && (n == 1 || (n <= most && groups * n < 65536)); ++n) {
    const double longest = (most / n + 4.0) * us, load = groups * n * (mean / n + 4.0) * us / 256;
    double t = sqrt(longest * longest + load * load);
    if (n > 1) t += 4.0 + 2.0 * n * bytes / 4e6;
    if (t < 0.98 * best_t) { best_t = t; best = n; }
  }
  return best;
}

// A tile of 32 keys takes the query sweep 0.35 + 0.0035 D us (float32: 0.4 +
// 0.065 D), a tile of 32 queries the key sweep 0.5 + 0.0053 D (0.4 + 0.09 D).
// 12 heads on 6 key heads, 777 tokens, D = 32, float32: key sweep 57 -> 22 us and 6 for the sum.
void attn_bwd_splits(const AttnShape& s, int* nsq, int* nsk) {
  const double G = (double)(s.H / s.Hkv), D = s.D;
  const bool half = s.dtype == 1;
  double most = (double)s.nk, mean = (double)s.nk, kmost = (double)s.nq, kmean = (double)s.nq;
  if (s.causal && s.nq <= s.nk) {
    mean = (double)s.nk - 0.5 * (double)s.nq;
    kmean = (double)s.nq * mean / (double)s.nk;
  }
  if (s.window > 0) {
    const double w = (double)(s.window + 128);
    most = most < w ? most : w; mean = mean < w ? mean : w;
    kmost = kmost < w ? kmost : w; kmean = kmean < w ? kmean : w;
  }
  *nsq = sweep_splits((double)(s.B * s.H * ((s.nq + 127) / 128)), most / 32, mean / 32,
                      half ? 0.35 + 0.0035 * D : 0.4 + 0.065 * D, (double)(s.B * s.H * s.nq) * D * 4);
  *nsk = sweep_splits((double)(s.B * s.Hkv * ((s.nk + 127) / 128)), G * kmost / 32, G * kmean / 32,
                      half ? 0.5 + 0.0053 * D : 0.4 + 0.09 * D, 2.0 * (double)(s.B * s.Hkv * s.nk) * D * 4);
}

template <typename T>
static int run_sum(const float* part, void* out0, void* out1, size_t n, int ns, hipStream_t st) {
  ProfScope ps("attn_sum", st);
  k_attn_sum<T><<<dim3((unsigned)((n / 4 + 255) / 256), out1 ? 2 : 1), 256, 0, st>>>(part, (T*)out0, (T*)out1, n, ns);
  return launch_status("attn sum");
}

template <typename T, int D>
static int run_bwd(const AttnShape& s, AttnArgs a, hipStream_t st) {
  const size_t nq = (size_t)s.B * s.H * s.nq * D, nk = (size_t)s.B * s.Hkv * s.nk * D;
  (void)hipGetLastError();
  {
    ProfScope ps("attn_dq", st);
    k_attn_dq<T, D><<<(unsigned)(s.B * s.H * a.nsq * a.ntq), 256, 0, st>>>(a);
  }
  if (int rc = launch_status("attn dq sweep")) return rc;
  if (a.nsq > 1)
    if (int rc = run_sum<T>(a.part, a.dq, nullptr, nq, a.nsq, st)) return rc;
  {
    ProfScope ps("attn_dkv", st);
    k_attn_dkv<T, D><<<(unsigned)(s.B * s.Hkv * a.nsk * a.ntk), 256, 0, st>>>(a);
  }
  if (int rc = launch_status("attn dk/dv sweep")) return rc;
  if (a.nsk == 1) return 0;
  return run_sum<T>(a.part, a.dk, a.dv, nk, a.nsk, st);
}

#define ATTN_DISPATCH(FN)                                                        \
  if (s.dtype == 1 && s.D == 32) return FN<bf16, 32>(s, a, st);                  \
  if (s.dtype == 1 && s.D == 64) return FN<bf16, 64>(s, a, st);                  \
  if (s.dtype == 1 && s.D == 128) return FN<bf16, 128>(s, a, st);                \
  if (s.dtype == 0 && s.D == 32) return FN<float, 32>(s, a, st);                 \
  if (s.dtype == 0 && s.D == 64) return FN<float, 64>(s, a, st);                 \
  set_error("attn: unsupported dtype=%d D=%d", s.dtype, s.D);                    \
  return -2;

int launch_attn_fwd(const AttnShape& s, const AttnArgs& a, hipStream_t st) { ATTN_DISPATCH(run_fwd) }
int launch_attn_bwd(const AttnShape& s, const AttnArgs& a, hipStream_t st) { ATTN_DISPATCH(run_bwd) }

}  // namespace linsimp
