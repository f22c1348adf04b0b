// Clipped policy loss with a KL term to a reference policy, forward and backward, from the trainer's logits z and the reference
// policy's logits y (or its log-probability of the token alone).
//
//   r = pi(a) / mu(a),  M = 0 where A > 0 and r > 1 + eps_high, or A < 0 and r < 1 - eps_low
//   loss = s sum_t [ -min(r A, clip(r) A) + beta KL_t ],   g = s M r A,   l_j = log pi_j - log rho_j
//   KL(pi || rho):  dz_j = pi_j (g + s beta (l_j - KL)) - g 1[j = a]
//   KL(rho || pi):  dz_j = pi_j (g + s beta) - s beta rho_j - g 1[j = a]
//   k3 = e^x - x - 1, x = log rho(a) - log pi(a):  dz_j = (pi_j - 1[j = a]) (g - s beta (1 - e^x))
//
// Each row is needed twice, for its sums and for its gradient, and is to cross HBM once: it is read a second time from L2, by the SM that read
// it first, before the rows that lie between the two reads push it out.
//
// policy_kl_ring_kernel, rows of all tensors on the same phase of 16 bytes: one persistent CTA per SM, a cluster of CTAs per row (each takes
// every n-th slot of it),
//   two producer lanes keep two rings of 16 KB slots filled by bulk asynchronous copies: the rows for their sums, and the same rows again for
//                      their gradient; the first runs ahead of the second by a row and a few slots, no more
//   8 sum warps        (16 for two tensors, taking slots in turn) add up a slot's exp and differences, and go on to the next row without waiting for anything
//   2 scalar warps     take the rows in turn: merge the sum warps' numbers, exchange them with the other CTAs of the cluster, work out the row's
//                      scalars in 64 bits and hand the gradient's coefficients to
//   8 gradient warps
// All waits are bounded.
// policy_kl_kernel, any layout: a CTA per row, one role after the other.
//
// 4096 x 151936 bf16, back to back: k3 443 us, 87 % of the measured copy rate over one read and one write of the logits; KL(pi || rho) 827 us, 70 % over two
// reads and a write, KL(rho || pi) 887 us.  The ring alone, without any arithmetic, takes 722 to 774 us of the latter; 62 % of the issue slots are busy.
// Rows held in registers of a cluster between the two uses (850 and 1976 us), or handed out by a queue to whichever SM is free, were slower.
//
// The token's own entry is left out of the sums and added in 64 bits, so that 1 - pi(a) keeps its relative accuracy.  Differences enter the
// sums as (z - max z) - (y - max y): the KL, a small difference of large sums, then does not depend on offsets between z and y.
#include <atomic>

#include "dppo_rowvec.cuh"

namespace dppo {
namespace {

constexpr int kTeam = 256, kTeamWarps = kTeam / 32;        // threads that work on a slot
constexpr int kScalarWarps = 2;
constexpr int kSlot = 16384;               // bytes of a slot, all tensors
constexpr int kSumSlots = 4, kGradSlots = 9, kSlots = kSumSlots + kGradSlots;
constexpr int kAhead = 11;                 // slots by which the sums may lead the gradient, beyond a row
constexpr int kHand = kScalarWarps;        // rows on their way from the sums to the gradient
constexpr int kMaxCluster = 8;
// teams that take the sums' slots in turn: the two exponentials an entry of two tensors keep one team busy too long (8 KB of each tensor,
// 4096 x 151936 bf16, KL(pi || rho): 909 us with one, 837 with two)
template <bool TWO> constexpr int kSumTeams = TWO ? 2 : 1;
template <bool TWO> constexpr int kRingThreads = (kSumTeams<TWO> + 1) * kTeam + 32 * kScalarWarps + 64;
template <bool TWO> constexpr int kChunk = TWO ? kSlot / 2 : kSlot;    // bytes of a tensor in a slot
constexpr int kMaxTeams = 2;

constexpr int kThreads = 512, kWarps = kThreads / 32;      // of the kernel for any layout
constexpr int kUnroll = 2;

// what a thread knows of its part of a row
struct Part { float mz, S, my, Sy, W; };   // reference and sum of exp of z, the same of y, sum of exp times the difference
// The same of a warp and of all of them.  From here on in 64 bits: the KL is what two large numbers leave, some 20 times smaller than they are.
struct Sums { float mz, my; double S, Sy, W; };

// Coefficients of the row's gradient: dz_j = e^(z_j - zr) (B ((z_j - zr) - (y_j - yr)) + A) for KL(pi || rho), e^(z_j - zr) A - B e^(y_j - yr) for
// KL(rho || pi), A e^(z_j - zr) for k3, and its value at the token.  zr and yr are the two log-sum-exp, rounded.
struct Coef { float zr, yr, A, B, fix; int some; };        // some: 0 for a row of zeros

// exp(z - m) of a vector's pairs; `arg` receives z - m
template <typename T> __device__ __forceinline__ void exp_pairs(const uint4& z, float m, float2* arg, float2* e) {
  const float2 l2 = make_float2(kLog2e, kLog2e);
  less_pairs<T>(z, m, arg);
#pragma unroll
  for (int i = 0; i < Vec<T>::N / 2; ++i) {
    const float2 x = __fmul2_rn(arg[i], l2);
    e[i] = make_float2(ex2_approx(x.x), ex2_approx(x.y));
  }
}

__device__ __forceinline__ void st_cluster_f64(uint32_t cluster_addr, double v) {
  asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(cluster_addr), "d"(v) : "memory");
}

__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint32_t min_nan_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// exp(d) without the rounding of d log2(e): what the product lost multiplies it by one plus that.  On average it is low by kExLow of itself (measured
// as the KL's mean error, with and without it, on logits of standard deviation 1 and 3 in both types).  (Far down the
// product would overflow, and what it lost be no number.)
__device__ __forceinline__ float exp_exact_arg(float d) {
  d = max_nan(d, -200.f);
  const float x = d * kLog2e, v = ex2_approx(x);
  return fmaf(v, fmaf(x, -(float)kLn2, d), v);
}

constexpr double kExLow = 1.5e-8;

struct PolicyParams {
  RowParams row;             // logits, ids, mu_logp, adv, token_mask, dlogits, outputs (divergence: the KL), workspace
  const void* y;             // reference logits, or null
  int64_t ld_y;
  const float* ref_logp;     // k3
  float beta, eps_low, eps_high;
  double scale;              // s, or 0: in the workspace's header
};

// What the scalar stage reads of a row besides its sums (loaded ahead of them).
struct RowIn { float z_a, y_a, mu, adv, ref; };
template <typename InT, int FORM>
__device__ __forceinline__ RowIn row_in(const PolicyParams& q, int64_t t, int a) {
  const RowParams& p = q.row;
  RowIn r;
  r.z_a = to_f32<InT>((reinterpret_cast<const InT*>(p.logits) + t * p.ld_in)[a]);
  r.y_a = FORM != DPPO_KL_K3 ? to_f32<InT>((reinterpret_cast<const InT*>(q.y) + t * q.ld_y)[a]) : 0.f;
  r.mu = p.mu_logp[t];
  r.adv = p.adv[t];
  r.ref = FORM == DPPO_KL_K3 ? q.ref_logp[t] : 0.f;
  return r;
}

// The row's scalars and coefficients from its sums over the entries other than the token's (against mz and my; W against mz - my), by one warp.
// 64-bit functions that do not depend on one another are evaluated side by side, a lane each (0: of pi, 1: of rho).
template <int FORM>
__device__ __forceinline__ Coef finish_row(const PolicyParams& q, int64_t t, const RowIn& in, const Sums& w, int lane, double s, bool write) {
  constexpr bool TWO = FORM != DPPO_KL_K3;
  const RowParams& p = q.row;
  const float mz = w.mz, my = w.my, z_a = in.z_a, y_a = in.y_a, mu = in.mu, adv = in.adv;
  const double S = w.S, Sy = w.Sy, W = w.W;
  const bool second = TWO && lane == 1;
  // maximum over the row, the weight of the others and of the token against it
  const float tok = second ? y_a : z_a, top = second ? my : mz;
  const double sum = second ? Sy : S;
  const bool have_tok = !(tok <= kLowest), have_others = !(top == kLowest);
  const double big = have_tok && (!have_others || tok > top) ? (double)tok : (double)top;
  const double d_tok = have_tok ? (double)tok - big : -INFINITY, d_top = have_others ? (double)top - big : -INFINITY;
  const double e_far = exp(fmin(d_tok, d_top));          // the larger of the two is the maximum itself
  const double w_tok = d_tok >= d_top ? (have_tok ? 1.0 : 0.0) : e_far;
  const double w_others = have_others ? (d_top >= d_tok ? sum : sum * e_far) : 0.0;
  const double total = w_tok + w_others;
  const double log_total = log(total);                   // -inf: no mass; NaN: a logit that is none
  const double p_tok = w_tok / total, p_others = w_others / total;
  const float lse_l = (float)(big + log_total);
  const bool fine = isfinite(big + log_total) && (!have_tok || isfinite(tok));
  // Log-probabilities, and what the rounded log-sum-exp is above the exact one, from differences with the maximum: logits may be far from zero.
  const double lp_l = d_tok - log_total, above_l = ((double)lse_l - big) - log_total;
  auto of = [&](double v, int l) { return __shfl_sync(0xffffffffu, v, l); };
  const double above = of(above_l, 0), above_y = TWO ? of(above_l, 1) : 0.0, pi_a = of(p_tok, 0), pi_o = of(p_others, 0);
  const double rho_a = TWO ? of(p_tok, 1) : 0.0, rho_o = TWO ? of(p_others, 1) : 0.0;
  bool ok = __shfl_sync(0xffffffffu, (int)fine, 0) && (!TWO || __shfl_sync(0xffffffffu, (int)fine, 1));
  double kl = 0.0, g = 0.0, r = 0.0, row_loss = 0.0, mu_a = 0.0;
  int M = 0;
  Coef co = {};
  if (ok) {
    const double lp = of(lp_l, 0), b = s * (double)q.beta;
    const double ref = FORM == DPPO_KL_K3 ? (double)in.ref - lp : 0.0;
    const double ex = FORM == DPPO_KL_K3 && lane == 1 ? expm1(ref) : exp(lane == 0 ? lp - (double)mu : (lane == 1 ? above_y : (lane == 2 ? above : (double)mu)));
    r = of(ex, 0);
    mu_a = of(ex, 3);
    const double fz = of(ex, 2);
    const double A = (double)adv, lo = 1.0 - (double)q.eps_low, hi = 1.0 + (double)q.eps_high;
    M = ((A > 0.0 && r > hi) || (A < 0.0 && r < lo)) ? 0 : 1;
    g = M ? s * r * A : 0.0;
    const double surrogate = M ? r * A : (A > 0.0 ? hi : lo) * A;
    co.zr = __shfl_sync(0xffffffffu, lse_l, 0);
    if (FORM == DPPO_KL_K3) {
      const double em = of(ex, 1), gk = g + b * em;
      kl = em - ref;
      co.A = (float)(gk * fz);
      co.fix = (float)(-gk * pi_o);
    } else {
      // KL: sum over the other entries of probability * difference of the log-probabilities, and the token's own term.  W is against mz - my;
      // shift is the difference of the log-probabilities that logits of mz and my would have.
      const double top_l = d_top - log_total, shift = of(top_l, 0) - of(top_l, 1), l_a = lp - of(lp_l, 1);
      co.yr = __shfl_sync(0xffffffffu, lse_l, 1);
      if (FORM == DPPO_KL_PI_REF) {
        kl = (pi_o > 0.0 ? pi_o * (W / S + shift) : 0.0) + (pi_a > 0.0 ? pi_a * l_a : 0.0);
        co.B = (float)(b * fz);
        co.A = (float)(fz * (g + b * (above - above_y - kl)));
        co.fix = (float)(-g * pi_o + (pi_a > 0.0 ? b * pi_a * (l_a - kl) : 0.0));
      } else {
        kl = (rho_o > 0.0 ? rho_o * (W / Sy - shift) : 0.0) - (rho_a > 0.0 ? rho_a * l_a : 0.0);
        co.A = (float)(fz * (g + b));
        co.B = (float)(b * of(ex, 1));
        co.fix = (float)(-g * pi_o + b * (pi_a - rho_a));
      }
    }
    row_loss = s * ((double)q.beta * kl - surrogate);
    // (in fp32, which is what the row's numbers are handed on in: an infinite coefficient times nothing would be no number)
    ok = fabs(kl) < 1e30 && isfinite((float)row_loss) && isfinite(co.A) && isfinite(co.B) && isfinite(co.fix);
  }
  if (!ok) { kl = r = row_loss = 0.0; M = 0; }
  if (write && lane == 0) {
    p.divergence[t] = (float)kl;
    p.mask[t] = (uint8_t)M;
    p.row_loss[t] = (float)row_loss;
    p.row_r[t] = (float)r;
    p.row_absdiff[t] = ok ? (float)fabs(mu_a - pi_a) : 0.f;
    if (!ok) atomicOr(p.status, DPPO_STATUS_NONFINITE_ROW);
  }
  co.some = ok;
  return co;
}

__device__ __forceinline__ void masked_row(const RowParams& p, int64_t t, int a) {
  p.divergence[t] = 0.f;
  p.mask[t] = 0;
  p.row_loss[t] = p.row_r[t] = p.row_absdiff[t] = 0.f;
  if (a == -2) atomicOr(p.status, DPPO_STATUS_BAD_SAMPLED_ID);
}

// Adds NV vectors of z (and y) to a thread's sums: any entries, the references moved up to the maxima.
template <typename InT, int FORM, int NV>
__device__ __forceinline__ void add_careful(Part& w, uint4* zv, uint4* yv) {
  constexpr bool TWO = FORM != DPPO_KL_K3;
  constexpr int N = Vec<InT>::N;
  RawMax<InT> mz, my;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    if (TWO) zv[k] = clamp_raw<InT>(zv[k]);      // (a difference of two must stay finite)
    mz.add(zv[k]);
    if (TWO) {
      yv[k] = clamp_raw<InT>(yv[k]);
      my.add(yv[k]);
    }
  }
  // the thread's sums so far, against the new maxima
  const float bz = max_nan(w.mz, mz.value()), by = TWO ? max_nan(w.my, my.value()) : 0.f;
  if (!(bz == w.mz) || (TWO && !(by == w.my))) {
    const float fz = ex2_approx((w.mz - bz) * kLog2e), fy = TWO ? ex2_approx((w.my - by) * kLog2e) : 0.f;
    // (where a sum vanishes against the new maximum its differences do too, however large they are)
    w.S *= fz;
    w.Sy *= fy;
    if (FORM == DPPO_KL_PI_REF) w.W = fz != 0.f && w.S != 0.f ? fmaf(w.S, (w.mz - bz) - (w.my - by), fz * w.W) : 0.f;
    if (FORM == DPPO_KL_REF_PI) w.W = fy != 0.f && w.Sy != 0.f ? fmaf(w.Sy, (w.my - by) - (w.mz - bz), fy * w.W) : 0.f;
    w.mz = bz;
    w.my = by;
  }
  float2 S = make_float2(0.f, 0.f), Sy = S, W = S;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    float2 az[N / 2], ez[N / 2];
    exp_pairs<InT>(zv[k], bz, az, ez);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) S = __fadd2_rn(S, ez[i]);
    if (TWO) {
      const float2 neg = make_float2(-1.f, -1.f);
      float2 ay[N / 2], ey[N / 2];
      exp_pairs<InT>(yv[k], by, ay, ey);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        Sy = __fadd2_rn(Sy, ey[i]);
        if (FORM == DPPO_KL_PI_REF) W = __ffma2_rn(ez[i], __ffma2_rn(ay[i], neg, az[i]), W);
        else W = __ffma2_rn(ey[i], __ffma2_rn(az[i], neg, ay[i]), W);
      }
    }
  }
  w.S += S.x + S.y;
  w.Sy += Sy.x + Sy.y;
  w.W += W.x + W.y;
  // A reference that is still the lowest: all its entries have probability zero.  (Against one another their exponentials are 1.)
  if (w.mz == kLowest) { w.S = 0.f; if (FORM == DPPO_KL_PI_REF) w.W = 0.f; }
  if (TWO && w.my == kLowest) { w.Sy = 0.f; if (FORM == DPPO_KL_REF_PI) w.W = 0.f; }
}

// smallest of raw entries, kept raw
template <typename T> struct RawMin;
template <> struct RawMin<__nv_bfloat16> {
  uint32_t m = 0x7F7F7F7Fu;
  __device__ __forceinline__ void add(const uint4& v) { m = min_nan_bf16x2(min_nan_bf16x2(m, v.x), min_nan_bf16x2(min_nan_bf16x2(v.y, v.z), v.w)); }
  __device__ __forceinline__ float value() const { return min_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u)); }
};
template <> struct RawMin<float> {
  float m = -kLowest;
  __device__ __forceinline__ void add(const uint4& v) {
    m = min_nan(min_nan(m, __uint_as_float(v.x)), min_nan(min_nan(__uint_as_float(v.y), __uint_as_float(v.z)), __uint_as_float(v.w)));
  }
  __device__ __forceinline__ float value() const { return m; }
};

// The same for ordinary entries: against references that stay where the thread's first vector put them.  Where that does not do (an entry far above
// its reference, -inf, NaN: the sums show it) the entries go the careful way.  exp(y_j - y_ref) is formed from exp(z_j - z_ref) and the exponential of the difference, which is near one: what the first is off by
// then stands in both sums alike and leaves the KL, where two exponentials on their own leave it 4e-8 off (relative to a KL of 0.045, logits of
// standard deviation 3 and 151936 entries: 1.8e-6 and now 6e-7).  For this z_j must not be so low that its exponential vanishes.
template <typename InT, int FORM, int NV>
__device__ __forceinline__ void add_vectors(Part& w, uint4* zv, uint4* yv) {
  constexpr bool TWO = FORM != DPPO_KL_K3;
  constexpr int N = Vec<InT>::N;
  if (w.mz == kLowest && (!TWO || w.my == kLowest)) {      // (nothing but probability zero so far, in either: no sums to move)
    RawMax<InT> mz, my;
    mz.add(zv[0]);
    w.mz = mz.value();
    if (TWO) { my.add(yv[0]); w.my = my.value(); }
  }
  float2 S = make_float2(0.f, 0.f), Sy = S, W = S;
  RawMin<InT> low;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    float2 az[N / 2], ez[N / 2];
    exp_pairs<InT>(zv[k], w.mz, az, ez);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) S = __fadd2_rn(S, ez[i]);
    if (TWO) {
      const float2 neg = make_float2(-1.f, -1.f), nl2 = make_float2(-kLog2e, -kLog2e);
      low.add(zv[k]);
      float2 ay[N / 2];
      less_pairs<InT>(yv[k], w.my, ay);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const float2 d = __ffma2_rn(ay[i], neg, az[i]), x = __fmul2_rn(d, nl2), ey = __fmul2_rn(ez[i], make_float2(ex2_approx(x.x), ex2_approx(x.y)));
        Sy = __fadd2_rn(Sy, ey);
        W = __ffma2_rn(FORM == DPPO_KL_PI_REF ? ez[i] : ey, d, W);
      }
    }
  }
  const float s = S.x + S.y, sy = Sy.x + Sy.y, d = FORM == DPPO_KL_REF_PI ? -(W.x + W.y) : W.x + W.y;
  constexpr float most = 7.3786976e19f;    // 2^66; false for NaN
  if (w.mz > kLowest && s <= most && (!TWO || (w.my > kLowest && sy <= most && fabsf(d) <= most && low.value() - w.mz >= -80.f))) {
    w.S += s;
    w.Sy += sy;
    w.W += d;
  } else {
    add_careful<InT, FORM, NV>(w, zv, yv);
  }
}

// The lanes' sums as one, against their maxima (a lane that saw nothing but probability zero counts nothing; NaN stays).
template <int FORM>
__device__ __forceinline__ Sums merge_lanes(const Sums& w) {
  constexpr bool TWO = FORM != DPPO_KL_K3;
  Sums r = {};
  r.mz = warp_max_nan(w.mz);
  r.my = TWO ? warp_max_nan(w.my) : 0.f;
  // The factor of y from that of z, as in add_vectors, where neither vanishes.  (64-bit exponentials cost 4096 rows of 32000 entries a quarter more time.)
  const float dz = w.mz - r.mz, off = dz - (w.my - r.my);
  const double fz = w.mz == kLowest ? 0.0 : (double)exp_exact_arg(dz);
  double fy = 0.0;
  if (TWO && w.my != kLowest) fy = fz != 0.0 && dz >= -80.f && off >= -80.f ? fz * (off == 0.f ? 1.0 : (double)exp_exact_arg(-off) * (1.0 + kExLow)) : (double)exp_exact_arg(w.my - r.my);
  r.S = warp_sum(fz != 0.0 ? fz * w.S : 0.0);
  if (TWO) {
    r.Sy = warp_sum(fy != 0.0 ? fy * w.Sy : 0.0);
    r.W = warp_sum(FORM == DPPO_KL_PI_REF ? (fz != 0.0 ? fz * fma(w.S, (double)off, w.W) : 0.0) : (fy != 0.0 ? fy * fma(-w.Sy, (double)off, w.W) : 0.0));
  }
  return r;
}
template <int FORM>
__device__ __forceinline__ Sums merge_lanes(const Part& w) {
  return merge_lanes<FORM>(Sums{w.mz, w.my, (double)w.S, (double)w.Sy, (double)w.W});
}

// The gradient of one vector.  (Two tensors: an entry of probability zero may lie infinitely far from its other logit; the token's own entry, which the
// sums leave out as such a one, makes no difference here.)
template <typename InT, int FORM>
__device__ __forceinline__ void grad_vector(const Coef& co, const uint4& zv, const uint4& yv, float* out) {
  constexpr bool TWO = FORM != DPPO_KL_K3;
  constexpr int N = Vec<InT>::N;
  const float2 A2 = make_float2(co.A, co.A), B2 = make_float2(co.B, co.B), nB = make_float2(-co.B, -co.B), neg = make_float2(-1.f, -1.f);
  float2 az[N / 2], ez[N / 2];
  exp_pairs<InT>(TWO ? clamp_raw<InT>(zv) : zv, co.zr, az, ez);
  if (TWO) {
    const uint4 yc = clamp_raw<InT>(yv);
    float2 ay[N / 2], ey[N / 2];
    if (FORM == DPPO_KL_REF_PI) exp_pairs<InT>(yc, co.yr, ay, ey); else less_pairs<InT>(yc, co.yr, ay);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      if (FORM == DPPO_KL_PI_REF) {
        const float2 d = __ffma2_rn(ay[i], neg, az[i]);
        // (e B) first, so that an entry of probability zero stays zero however large its difference is
        ez[i] = __ffma2_rn(__fmul2_rn(ez[i], B2), d, __fmul2_rn(ez[i], A2));
      } else {
        ez[i] = __ffma2_rn(ey[i], nB, __fmul2_rn(ez[i], A2));
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) ez[i] = __fmul2_rn(ez[i], A2);
  }
#pragma unroll
  for (int i = 0; i < N / 2; ++i) { out[2 * i] = ez[i].x; out[2 * i + 1] = ez[i].y; }
}

// ------------------------------------------------------------------------------------------------ ring of bulk copies
struct RingMisc {
  unsigned long long full[kSlots], empty[kSlots];          // of both rings: the sums' slots, then the gradient's
  unsigned long long part_full[kHand], part_empty[kHand];  // sums of a row: sum warps -> scalar warp
  unsigned long long coef_full[kHand], coef_empty[kHand];  // coefficients of a row: scalar warp -> gradient warps
  unsigned long long x_full[kHand], x_empty[kHand];        // sums of a row of every CTA of the cluster
  Sums part[kHand][kMaxTeams * kTeamWarps], x_part[kHand][kMaxCluster];
  Coef coef[kHand];
  int abort_flag;
  unsigned int grad_slots;                                 // slots the gradient warps have finished
};
constexpr int kMiscBytes = 4096;
static_assert(sizeof(RingMisc) <= kMiscBytes, "misc area");

// A row's image in the ring: from the 16-byte boundary at or below its first element (head elements early) on.
struct Geom { int head, lo, hi; };         // lo .. hi - 1: the vectors wholly in the row
template <typename InT> __device__ __forceinline__ Geom geom_of(const RowParams& p, int64_t t) {
  const int head = (int)head_of(reinterpret_cast<const InT*>(p.logits) + t * p.ld_in);
  return Geom{head, head ? 1 : 0, (head + (int)p.V) / Vec<InT>::N};
}

// One lane: the slots of this CTA's rows into a ring, in order, as slots come free.  follow: stay at most `lead` slots ahead of that count.
template <typename InT, int FORM>
__device__ __forceinline__ void produce(const PolicyParams& q, unsigned char* slots, uint32_t full, uint32_t empty, int nslots, int C, uint64_t policy,
                                        const WaitCtl& wc, volatile unsigned int* follow, unsigned int lead, int rank, int CL) {
  constexpr bool TWO = FORM != DPPO_KL_K3;
  constexpr int CHUNK = kChunk<TWO>;
  const RowParams& p = q.row;
  const int64_t t0 = blockIdx.x / CL, G = gridDim.x / CL;
  const uint32_t base = smem_u32(slots);
  RingPos pos{0, 0};
  bool first_lap = true;
  unsigned int issued = 0;
  int a = load_meta(p, t0);
  for (int64_t t = t0; t < p.T; t += G) {
    const int a_next = load_meta(p, t + G);
    if (a >= 0) {
      const InT* zrow = reinterpret_cast<const InT*>(p.logits) + t * p.ld_in;
      const InT* yrow = TWO ? reinterpret_cast<const InT*>(q.y) + t * q.ld_y : zrow;
      const int head = (int)head_of(zrow);
      const char* zi = reinterpret_cast<const char*>(zrow - head);
      const char* yi = reinterpret_cast<const char*>(yrow - head);
      const int64_t xend = (int64_t)(head + p.V) * (int64_t)sizeof(InT), xa = xend & ~(int64_t)15;      // end of the image, and of what bulk copies bring
      for (int c = rank; c < C; c += CL) {
        const int s = pos.slot;
        if (follow) {
          if (issued - *follow >= lead) {
            const unsigned long long w0 = globaltimer_ns();
            while (issued - *follow >= lead) {
              if (wc.aborted()) return;
              if (globaltimer_ns() - w0 > wc.limit_ns) { wc.abort(); return; }
              __nanosleep(64);
            }
          }
          ++issued;
        }
        if (!first_lap && !mbar_wait(empty + 8u * s, pos.phase ^ 1u, wc)) return;
        const int64_t off = (int64_t)c * CHUNK;
        const uint32_t bytes = off < xa ? (uint32_t)min((int64_t)CHUNK, xa - off) : 0u, dst = base + (uint32_t)s * kSlot;
        if (xend > xa && xa >= off && xa < off + CHUNK) {
          // the row's last elements, behind its last 16-byte boundary: plain loads, so that nothing behind the row is read
          unsigned char* sp = slots + (size_t)s * kSlot + (xa - off);
          for (int i = 0; i < (int)(xend - xa) / (int)sizeof(InT); ++i) {
            reinterpret_cast<InT*>(sp)[i] = reinterpret_cast<const InT*>(zi + xa)[i];
            if (TWO) reinterpret_cast<InT*>(sp + CHUNK)[i] = reinterpret_cast<const InT*>(yi + xa)[i];
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        if (bytes) {
          mbar_arrive_expect_tx(full + 8u * s, TWO ? 2u * bytes : bytes);
          bulk_load(dst, zi + off, bytes, full + 8u * s, policy);
          if (TWO) bulk_load(dst + CHUNK, yi + off, bytes, full + 8u * s, policy);
        } else {
          mbar_arrive(full + 8u * s);
        }
        pos.advance(nslots);
        if (pos.slot == 0) first_lap = false;
      }
    }
    a = a_next;
  }
}

template <typename InT, typename OutT, int FORM>
__global__ void __launch_bounds__(kRingThreads<FORM != DPPO_KL_K3>, 1) policy_kl_ring_kernel(const __grid_constant__ PolicyParams q, int C, int lead) {
  extern __shared__ __align__(128) unsigned char smem[];
  constexpr bool TWO = FORM != DPPO_KL_K3;
  constexpr int N = Vec<InT>::N, CHUNK = kChunk<TWO>, VECS = CHUNK / 16, TEAMS = kSumTeams<TWO>;
  constexpr int PER = VECS / kTeam;        // vectors of a tensor that a thread takes from a slot
  const RowParams& p = q.row;
  RingMisc* misc = reinterpret_cast<RingMisc*>(smem + (size_t)kSlots * kSlot);
  const uint32_t base = smem_u32(smem), full = smem_u32(&misc->full[0]), empty = smem_u32(&misc->empty[0]);
  const uint32_t part_full = smem_u32(&misc->part_full[0]), part_empty = smem_u32(&misc->part_empty[0]);
  const uint32_t coef_full = smem_u32(&misc->coef_full[0]), coef_empty = smem_u32(&misc->coef_empty[0]);
  const WaitCtl wc{&misc->abort_flag, p.wait_ns};
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int CL = (int)cluster_nctarank(), rank = CL > 1 ? (int)cluster_ctarank() : 0;
  if (tid == 0) {
    for (int i = 0; i < kSlots; ++i) { mbar_init(full + 8u * i, 1); mbar_init(empty + 8u * i, kTeamWarps); }
    for (int i = 0; i < kHand; ++i) {
      mbar_init(part_full + 8u * i, TEAMS * kTeamWarps);
      mbar_init(part_empty + 8u * i, 1);
      mbar_init(coef_full + 8u * i, 1);
      mbar_init(coef_empty + 8u * i, kTeamWarps);
      mbar_init(smem_u32(&misc->x_full[i]), (uint32_t)CL);
      mbar_init(smem_u32(&misc->x_empty[i]), (uint32_t)CL);
    }
    misc->abort_flag = 0;
    misc->grad_slots = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  if (CL > 1) cluster_sync_all();          // the peers' barriers exist before anything is sent to them
  const int64_t t0 = blockIdx.x / CL, G = gridDim.x / CL;

  if (warp >= (TEAMS + 1) * kTeamWarps + kScalarWarps) {
    // ------------------------------------------------------------------ producers
    // (test injection: they issue nothing, so that every wait for a slot runs out)
    if (lane == 0 && !(p.inject & DPPO_INJECT_NO_COPIES)) {
      uint64_t policy;
      if (warp == (TEAMS + 1) * kTeamWarps + kScalarWarps) {
        asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(policy));
        produce<InT, FORM>(q, smem, full, empty, kSumSlots, C, policy, wc, &misc->grad_slots, (unsigned int)lead, rank, CL);
      } else {
        asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
        produce<InT, FORM>(q, smem + (size_t)kSumSlots * kSlot, full + 8u * kSumSlots, empty + 8u * kSumSlots, kGradSlots, C, policy, wc, nullptr, 0u, rank, CL);
      }
    }
  } else if (warp < TEAMS * kTeamWarps) {
    // ------------------------------------------------------------------ sums
    const int team = warp / kTeamWarps, ttid = tid % kTeam;
    int turn = 0;                          // whose slot it is
    RingPos pos{0, 0};
    uint32_t n = 0;
    int a = load_meta(p, t0);
    for (int64_t t = t0; t < p.T; t += G) {
      const int a_next = load_meta(p, t + G);
      if (__shfl_sync(0xffffffffu, (int)wc.aborted(), 0)) break;
      if (a >= 0) {
        const Geom g = geom_of<InT>(p, t);
        const int av = (a + g.head) / N, ai = (a + g.head) % N;        // the token's vector, and its place there
        Part w{kLowest, 0.f, kLowest, 0.f, 0.f};
        for (int c = rank; c < C; c += CL) {
          const bool mine = TEAMS == 1 || turn == team;
          turn = turn + 1 == TEAMS ? 0 : turn + 1;
          if (!mine) { pos.advance(kSumSlots); continue; }
          const bool ok = mbar_wait_warp(full + 8u * pos.slot, pos.phase, wc);
          const uint32_t sz = base + (uint32_t)pos.slot * kSlot + 16u * (uint32_t)ttid;
          if (ok) {
            uint4 zv[PER], yv[TWO ? PER : 1];
#pragma unroll
            for (int k = 0; k < PER; ++k) {
              zv[k] = lds128(sz + (uint32_t)k * (16u * kTeam));
              if (TWO) yv[k] = lds128(sz + CHUNK + (uint32_t)k * (16u * kTeam));
            }
            const int v0 = c * VECS + ttid;
            if (c * VECS < g.lo || (c + 1) * VECS > g.hi) {            // a slot with an end of the row in it: what is not the row's counts as -inf
#pragma unroll
              for (int k = 0; k < PER; ++k) {
                const int v = v0 + k * kTeam;
                if (v < g.lo || v >= g.hi) {
#pragma unroll
                  for (int i = 0; i < N; ++i)
                    if (v * N + i < g.head || v * N + i >= g.head + (int)p.V) {
                      set_raw(zv[k], i, from_f32<InT>(-INFINITY));
                      if (TWO) set_raw(yv[k], i, from_f32<InT>(-INFINITY));
                    }
                }
              }
            }
            if (av >= c * VECS && av < (c + 1) * VECS) {               // the slot with the token's entry
#pragma unroll
              for (int k = 0; k < PER; ++k)
                if (v0 + k * kTeam == av) {
#pragma unroll
                  for (int i = 0; i < N; ++i)
                    if (i == ai) {
                      set_raw(zv[k], i, from_f32<InT>(-INFINITY));
                      if (TWO) set_raw(yv[k], i, from_f32<InT>(-INFINITY));
                    }
                }
            }
            add_vectors<InT, FORM, PER>(w, zv, yv);
          }
          // (a vote on the sums, which are never negative: the arrival is not to be moved up between the loads and their use)
          if (!__any_sync(0xffffffffu, w.S < 0.f || (TWO && w.Sy < 0.f)) && lane == 0) mbar_arrive(empty + 8u * pos.slot);
          pos.advance(kSumSlots);
        }
        const Sums sums = merge_lanes<FORM>(w);
        if (lane == 0) {
          const uint32_t b = n % kHand, u = n / kHand;
          if (u == 0 || mbar_wait(part_empty + 8u * b, (u & 1u) ^ 1u, wc)) {
            misc->part[b][warp] = sums;
            mbar_arrive(part_full + 8u * b);
          }
        }
        ++n;
      }
      a = a_next;
    }
  } else if (warp < (TEAMS + 1) * kTeamWarps) {
    // ------------------------------------------------------------------ gradient
    const int gtid = tid - TEAMS * kTeam;
    const uint32_t ring = base + kSumSlots * kSlot, gfull = full + 8u * kSumSlots, gempty = empty + 8u * kSumSlots;
    RingPos pos{0, 0};
    uint32_t n = 0;
    unsigned int done = 0;
    int a = load_meta(p, t0);
    for (int64_t t = t0; t < p.T; t += G) {
      const int a_next = load_meta(p, t + G);
      if (__shfl_sync(0xffffffffu, (int)wc.aborted(), 0)) break;
      const int head = geom_of<InT>(p, t).head;
      const RowRef<OutT, N> rd(reinterpret_cast<OutT*>(p.dlogits) + t * p.ld_out, head, p.V);
      if (a < 0) {
        const float zero[N] = {};
        for (int v = rank * kTeam + gtid; v < rd.nvec; v += CL * kTeam) store_vec<OutT, N>(rd, v, zero);
      } else {
        const uint32_t b = n % kHand, u = n / kHand;
        const bool have = mbar_wait_warp(coef_full + 8u * b, u & 1u, wc);
        Coef co = misc->coef[b];
        // (a vote on what was read, whatever its answer: the arrival is not to be moved up before the loads)
        if ((!__any_sync(0xffffffffu, co.zr + co.yr + co.A + co.B + co.fix == 1.f && co.some) || p.V > 0) && lane == 0 && have)
          mbar_arrive(coef_empty + 8u * b);
        if (!have) co.some = 0;
        ++n;
        const int av = (a + head) / N;
        OutT* image = rd.row - head;       // where vector 0 goes, whole or not
        for (int c = rank; c < C; c += CL) {
          const bool ok = mbar_wait_warp(gfull + 8u * pos.slot, pos.phase, wc);
          const uint32_t sz = ring + (uint32_t)pos.slot * kSlot + 16u * (uint32_t)gtid;
          const int v0 = c * VECS + gtid;
          if (ok) {
            uint4 zv[PER], yv[TWO ? PER : 1];
#pragma unroll
            for (int k = 0; k < PER; ++k) {
              zv[k] = lds128(sz + (uint32_t)k * (16u * kTeam));
              if (TWO) yv[k] = lds128(sz + CHUNK + (uint32_t)k * (16u * kTeam));
            }
            if (co.some && c * VECS >= rd.lo && (c + 1) * VECS <= rd.hi) {
#pragma unroll
              for (int k = 0; k < PER; ++k) {
                float out[N];
                grad_vector<InT, FORM>(co, zv[k], TWO ? yv[k] : zv[k], out);
                Store<OutT, N>::run(image + (int64_t)(v0 + k * kTeam) * N, 0u, out);
              }
            } else {
#pragma unroll
              for (int k = 0; k < PER; ++k) {
                float out[N] = {};
                if (co.some) grad_vector<InT, FORM>(co, zv[k], TWO ? yv[k] : zv[k], out);
                if (v0 + k * kTeam < rd.nvec) store_vec<OutT, N>(rd, v0 + k * kTeam, out);
              }
            }
            if (co.some && av >= c * VECS && av < (c + 1) * VECS && (av - v0) % kTeam == 0) rd.row[a] = from_f32<OutT>(co.fix);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(gempty + 8u * pos.slot);
          ++done;
          if (gtid == 0) *(volatile unsigned int*)&misc->grad_slots = done;
          pos.advance(kGradSlots);
        }
      }
      a = a_next;
    }
  } else {
    // ------------------------------------------------------------------ scalars
    const uint32_t sw = (uint32_t)(warp - (TEAMS + 1) * kTeamWarps);
    const double s = q.scale > 0.0 ? q.scale : p.hdr->scale;
    uint32_t n = 0;
    int a = load_meta(p, t0);
    for (int64_t t = t0; t < p.T; t += G) {
      const int a_next = load_meta(p, t + G);
      if (__shfl_sync(0xffffffffu, (int)wc.aborted(), 0)) break;
      if (a < 0) {
        if (sw == 0 && lane == 0 && rank == 0) masked_row(p, t, a);
      } else if (n++ % kScalarWarps == sw) {
        const uint32_t b = (n - 1) % kHand, u = (n - 1) / kHand;
        const RowIn in = row_in<InT, FORM>(q, t, a);
        bool have = mbar_wait_warp(part_full + 8u * b, u & 1u, wc);
        const Sums none{kLowest, kLowest, 0.0, 0.0, 0.0};
        Sums w = have && lane < TEAMS * kTeamWarps ? misc->part[b][lane] : none;
        w = merge_lanes<FORM>(w);
        if (lane == 0 && have) mbar_arrive(part_empty + 8u * b);           // (behind the exchange between the lanes: all have what they read)
        if (CL > 1) {
          // the CTAs of the cluster exchange their sums: lane r sends to CTA r once every CTA has read the buffer's last content
          const uint32_t xf = smem_u32(&misc->x_full[b]), xe = smem_u32(&misc->x_empty[b]);
          if (have && u > 0) have = __all_sync(0xffffffffu, mbar_wait_cluster(xe, (u & 1u) ^ 1u, wc));
          if (have && lane < CL) {
            const uint32_t dst = map_to_cta(smem_u32(&misc->x_part[b][rank]), (uint32_t)lane);
            st_cluster_f32x2(dst, w.mz, w.my);
            st_cluster_f64(dst + 8, w.S);
            st_cluster_f64(dst + 16, w.Sy);
            st_cluster_f64(dst + 24, w.W);
            bar_arrive_cluster(map_to_cta(xf, (uint32_t)lane));
          }
          if (have) have = __all_sync(0xffffffffu, mbar_wait_cluster(xf, u & 1u, wc));
          w = have && lane < CL ? misc->x_part[b][lane] : none;
          w = merge_lanes<FORM>(w);
          if (have && lane < CL) bar_arrive_cluster(map_to_cta(xe, (uint32_t)lane));
        }
        if (have) {
          const Coef co = finish_row<FORM>(q, t, in, w, lane, s, rank == 0);
          if (lane == 0 && (u == 0 || mbar_wait(coef_empty + 8u * b, (u & 1u) ^ 1u, wc))) {
            misc->coef[b] = co;
            mbar_arrive(coef_full + 8u * b);
          }
        }
      }
      a = a_next;
    }
  }
  __syncwarp();
  if (wc.aborted()) {
    if (lane == 0) atomicOr(p.status, DPPO_STATUS_WAIT_LIMIT);
    drain_after_abort();
  }
  if (CL > 1) cluster_sync_all();          // a peer may still be sending to this CTA's shared memory
}

// ----------------------------------------------------------------------------------------------------------- any layout
template <typename InT, typename OutT, int FORM>
__global__ void __launch_bounds__(kThreads) policy_kl_kernel(const __grid_constant__ PolicyParams q) {
  constexpr bool TWO = FORM != DPPO_KL_K3;
  constexpr int N = Vec<InT>::N;
  __shared__ Sums parts[kWarps];
  __shared__ Coef s_coef;
  const RowParams& p = q.row;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int64_t t = blockIdx.x; t < p.T; t += gridDim.x) {
    const int a = load_meta(p, t);
    const InT* zrow = reinterpret_cast<const InT*>(p.logits) + t * p.ld_in;
    const InT* yrow = TWO ? reinterpret_cast<const InT*>(q.y) + t * q.ld_y : zrow;
    const uint32_t head = head_of(zrow);
    const RowRef<const InT, N> rz(zrow, head, p.V), ry(yrow, head, p.V);
    const RowRef<OutT, N> rd(reinterpret_cast<OutT*>(p.dlogits) + t * p.ld_out, head, p.V);
    if (a < 0) {
      zero_row<OutT, N>(rd, 0, 1, kThreads);
      if (tid == 0) masked_row(p, t, a);
      continue;
    }
    const RowIn in = row_in<InT, FORM>(q, t, a);
    const int av = (int)(((uint32_t)a + head) / N), ai = (int)(((uint32_t)a + head) % N);
    uint4 zv[kUnroll], yv[TWO ? kUnroll : 1];
    Part w{kLowest, 0.f, kLowest, 0.f, 0.f};
    for (int v0 = tid; v0 - tid < rz.nvec; v0 += kUnroll * kThreads) {
      load_vecs<kUnroll>(zv, rz, v0, kThreads, rz.nvec);
      if (TWO) load_vecs<kUnroll>(yv, ry, v0, kThreads, rz.nvec);
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
        if (v0 + k * kThreads == av) {
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (i == ai) {
              set_raw(zv[k], i, from_f32<InT>(-INFINITY));
              if (TWO) set_raw(yv[k], i, from_f32<InT>(-INFINITY));
            }
        }
      add_careful<InT, FORM, kUnroll>(w, zv, yv);
    }
    Sums sums = merge_lanes<FORM>(w);
    if (lane == 0) parts[warp] = sums;
    __syncthreads();
    if (warp == 0) {
      sums = merge_lanes<FORM>(lane < kWarps ? parts[lane] : Sums{kLowest, kLowest, 0.0, 0.0, 0.0});
      const Coef co = finish_row<FORM>(q, t, in, sums, lane, q.scale > 0.0 ? q.scale : p.hdr->scale, true);
      if (lane == 0) s_coef = co;
    }
    __syncthreads();
    const Coef co = s_coef;
    if (!co.some) {
      zero_row<OutT, N>(rd, 0, 1, kThreads);
      continue;
    }
    for (int v0 = tid; v0 < rz.nvec; v0 += kUnroll * kThreads) {
      load_vecs<kUnroll>(zv, rz, v0, kThreads, rz.nvec);
      if (TWO) load_vecs<kUnroll>(yv, ry, v0, kThreads, rz.nvec);
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        const int v = v0 + k * kThreads;
        if (v >= rz.nvec) break;
        float out[N];
        grad_vector<InT, FORM>(co, zv[k], TWO ? yv[k] : zv[k], out);
        store_vec<OutT, N>(rd, v, out);
      }
    }
    if (av % kThreads == tid) rd.row[a] = from_f32<OutT>(co.fix);
  }
}

// CTAs that share a row: as many as keep the rows that lie between their two reads in L2 (320 KB of a row to a CTA at most), more where
// rows are few.
int cluster_of(int64_t T, int C, int slot, int sms) {
  int CL = 1;
  while (CL < kMaxCluster && (int64_t)C * slot > (int64_t)CL * 327680) CL *= 2;
  while (CL < kMaxCluster && T * CL * 2 <= sms && C >= 2 * CL) CL *= 2;
  return CL;
}

template <typename InT, typename OutT, int FORM>
cudaError_t launch_form(const PolicyParams& q, bool ring, cudaStream_t st) {
  int dev = 0, sms = 148;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  const int64_t T = q.row.T;
  if (!ring) {
    policy_kl_kernel<InT, OutT, FORM><<<(unsigned)(T < 4 * sms ? T : 4 * sms), kThreads, 0, st>>>(q);
    return cudaGetLastError();
  }
  constexpr int CHUNK = kChunk<FORM != DPPO_KL_K3>, THREADS = kRingThreads<FORM != DPPO_KL_K3>;
  const int64_t bytes = q.row.V * (int64_t)sizeof(InT) + 16 - (int64_t)sizeof(InT);        // of a row with the largest head
  const int C = (int)((bytes + CHUNK - 1) / CHUNK), smem = kSlots * kSlot + kMiscBytes;
  auto kernel = policy_kl_ring_kernel<InT, OutT, FORM>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  int CL = cluster_of(T, C, kSlot, sms);
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.blockDim = dim3(THREADS, 1, 1);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cfg.attrs = attr;
  int64_t clusters = sms;
  if (CL > 1) {
    // as many clusters as the device runs at a time (asked once per device and size)
    static std::atomic<int> known[64][4] = {};         // (calls may come from several threads)
    const int li = CL == 2 ? 1 : (CL == 4 ? 2 : 3);
    int nc = dev >= 0 && dev < 64 ? known[dev][li].load() : 0;
    if (nc <= 0) {
      attr[0].val.clusterDim.x = (unsigned)CL;
      cfg.numAttrs = 1;
      cfg.gridDim = dim3((unsigned)(sms / CL * CL), 1, 1);
      e = cudaOccupancyMaxActiveClusters(&nc, kernel, &cfg);
      if (e != cudaSuccess || nc <= 0) { (void)cudaGetLastError(); CL = 1; nc = sms; }      // no room for such clusters: one CTA per row
      else if (dev >= 0 && dev < 64) known[dev][li] = nc;
    }
    clusters = nc;
  }
  attr[0].val.clusterDim.x = (unsigned)CL;
  cfg.numAttrs = CL > 1 ? 1 : 0;
  cfg.gridDim = dim3((unsigned)((T < clusters ? T : clusters) * CL), 1, 1);
  return cudaLaunchKernelEx(&cfg, kernel, q, C, (C + CL - 1) / CL + kAhead);
}

template <typename InT, typename OutT>
cudaError_t launch_types(const PolicyParams& q, int form, bool ring, cudaStream_t st) {
  switch (form) {
    case DPPO_KL_K3: return launch_form<InT, OutT, DPPO_KL_K3>(q, ring, st);
    case DPPO_KL_PI_REF: return launch_form<InT, OutT, DPPO_KL_PI_REF>(q, ring, st);
    default: return launch_form<InT, OutT, DPPO_KL_REF_PI>(q, ring, st);
  }
}

size_t esize(int dt) { return dt == DPPO_BF16 ? 2 : 4; }
bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + nb && y < x + na;
}

}  // namespace
}  // namespace dppo

extern "C" int dppo_policy_kl_fwd_bwd(const void* logits, int64_t T, int64_t V, int64_t logits_row_stride, int logits_dtype,
                                      const void* ref_logits, int64_t ref_row_stride, const float* ref_logp,
                                      const int32_t* sampled_ids, const float* mu_logp, const float* advantages,
                                      const uint8_t* token_mask, int kl_form, float kl_coef, float eps_low, float eps_high,
                                      const dppo_opts* opts, float* loss, float* kl, uint8_t* mask, void* dlogits,
                                      int64_t dlogits_row_stride, float* stats, int32_t* status,
                                      void* workspace, size_t workspace_bytes, void* cuda_stream) {
  using namespace dppo;
  dppo_opts o = {};
  if (opts) o = *opts;
  if (T < 0 || V < 1 || V > ((int64_t)1 << 30) || T > ((int64_t)1 << 27)) return DPPO_ERR_SHAPE;
  if (logits_dtype != DPPO_F32 && logits_dtype != DPPO_BF16) return DPPO_ERR_DTYPE;
  if (o.dlogits_dtype != DPPO_DLOGITS_SAME && o.dlogits_dtype != DPPO_DLOGITS_F32) return DPPO_ERR_DTYPE;
  if (kl_form < DPPO_KL_PI_REF || kl_form > DPPO_KL_K3) return DPPO_ERR_VARIANT;
  if (!(kl_coef >= 0.f) || !isfinite(kl_coef) || !(eps_low >= 0.f) || !(eps_high >= 0.f) || o.wait_limit_us < 0) return DPPO_ERR_UNSUPPORTED;
  const bool two = kl_form != DPPO_KL_K3;
  if (!loss || !status) return DPPO_ERR_NULL;
  if (T > 0 && (!logits || !sampled_ids || !mu_logp || !advantages || !kl || !mask || !dlogits || (two ? !ref_logits : !ref_logp))) return DPPO_ERR_NULL;
  if (T > 1 && (logits_row_stride < V || dlogits_row_stride < V || (two && ref_row_stride < V))) return DPPO_ERR_STRIDE;
  const int out_dtype = o.dlogits_dtype == DPPO_DLOGITS_F32 ? DPPO_F32 : logits_dtype;
  if ((uintptr_t)logits % esize(logits_dtype) || (uintptr_t)dlogits % esize(out_dtype) || (two && (uintptr_t)ref_logits % esize(logits_dtype))) return DPPO_ERR_ALIGN;
  if ((uintptr_t)sampled_ids % 4 || (uintptr_t)mu_logp % 4 || (uintptr_t)advantages % 4 || (uintptr_t)ref_logp % 4 || (uintptr_t)loss % 4 ||
      (uintptr_t)kl % 4 || (uintptr_t)stats % 4 || (uintptr_t)status % 4) return DPPO_ERR_ALIGN;
  if (T > 0) {
    // The gradient in place of the logits is fine: a row's sums are complete before its coefficients are, a slot's gradient is written by the CTA that
    // has just read the slot for the second time, and of a 16-byte vector that two rows share each takes and writes its own entries.  Any other
    // overlap is not.
    const size_t nz = ((size_t)(T - 1) * logits_row_stride + V) * esize(logits_dtype), nd = ((size_t)(T - 1) * dlogits_row_stride + V) * esize(out_dtype);
    const bool in_place = dlogits == logits && out_dtype == logits_dtype && (T == 1 || dlogits_row_stride == logits_row_stride);
    if (!in_place && overlap(logits, nz, dlogits, nd)) return DPPO_ERR_ALIAS;
    if (two && overlap(ref_logits, ((size_t)(T - 1) * ref_row_stride + V) * esize(logits_dtype), dlogits, nd)) return DPPO_ERR_ALIAS;
  }
  if (!workspace || (uintptr_t)workspace % 256 || workspace_bytes < dppo_workspace_bytes(T, V, 0, 0)) return DPPO_ERR_WORKSPACE;
  PolicyParams q = {};
  RowParams& p = q.row;
  p.logits = logits; p.T = T; p.V = V; p.ld_in = logits_row_stride; p.sampled_ids = sampled_ids; p.mu_logp = mu_logp; p.adv = advantages;
  p.token_mask = token_mask; p.loss_scale = o.loss_scale; p.dlogits = dlogits; p.ld_out = dlogits_row_stride; p.divergence = kl; p.mask = mask;
  p.loss = loss; p.stats = stats; p.status = status;
  p.wait_ns = wait_limit_ns(o.wait_limit_us); p.inject = o.test_inject;
  const size_t es = esize(logits_dtype);
  // the ring: rows that start on one phase of 16 bytes in both tensors, at a base on a boundary (the bytes in front of a row's first element,
  // up to the boundary, are then the row before's)
  const bool ring = (uintptr_t)logits % 16 == 0 && (!two || ((uintptr_t)ref_logits % 16 == 0 && (T <= 1 || (logits_row_stride * es) % 16 == (ref_row_stride * es) % 16)));
  char* ws = reinterpret_cast<char*>(workspace);
  const size_t per = (dppo_workspace_bytes(T, V, 0, 0) - 256) / 3;
  p.hdr = reinterpret_cast<WsHeader*>(ws);
  p.row_loss = reinterpret_cast<float*>(ws + 256);
  p.row_r = reinterpret_cast<float*>(ws + 256 + per);
  p.row_absdiff = reinterpret_cast<float*>(ws + 256 + 2 * per);
  q.y = ref_logits; q.ld_y = ref_row_stride; q.ref_logp = ref_logp; q.beta = kl_coef; q.eps_low = eps_low; q.eps_high = eps_high;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  // without a mask the scale is known here, and the count of valid rows is only wanted for the statistics
  q.scale = o.loss_scale > 0.f ? (double)o.loss_scale : (!token_mask && T > 0 ? 1.0 / (double)T : 0.0);
  if ((q.scale == 0.0 || stats) && launch_prelude(p, st) != cudaSuccess) return DPPO_ERR_CUDA;
  if (T > 0) {
    cudaError_t e;
    if (logits_dtype == DPPO_BF16 && out_dtype == DPPO_BF16) e = launch_types<__nv_bfloat16, __nv_bfloat16>(q, kl_form, ring, st);
    else if (logits_dtype == DPPO_BF16) e = launch_types<__nv_bfloat16, float>(q, kl_form, ring, st);
    else e = launch_types<float, float>(q, kl_form, ring, st);
    if (e != cudaSuccess) return DPPO_ERR_CUDA;
  }
  return launch_finalize(p, st) == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
}
