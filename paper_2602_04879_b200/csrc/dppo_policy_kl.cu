// Clipped policy loss with a KL term to a reference policy, forward and backward, from the trainer's logits z and the reference
// policy's logits y (or its log-probability of the token alone).
//
//   r = pi(a) / mu(a),  M = 0 where A > 0 and r > 1 + eps_high, or A < 0 and r < 1 - eps_low
//   loss = s sum_t [ -min(r A, clip(r) A) + beta KL_t ],   g = s M r A,   l_j = log pi_j - log rho_j
//   KL(pi || rho):  dz_j = pi_j (g + s beta (l_j - KL)) - g 1[j = a]
//   KL(rho || pi):  dz_j = pi_j (g + s beta) - s beta rho_j - g 1[j = a]
//   k3 = e^x - x - 1, x = log rho(a) - log pi(a):  dz_j = (pi_j - 1[j = a]) (g - s beta (1 - e^x))
//
// A row (of both tensors) is held in the registers of a cluster of up to 8 CTAs from its one read to its gradient's write: each thread
// loads its vectors, all in flight at once, and keeps them packed; every warp works out its maxima and its sums of exp and of exp times
// the difference, hands them to all CTAs of the cluster through distributed shared memory, and behind the cluster's barrier each CTA
// works out the row's scalars (64 bits) and writes its part of the gradient.  Rows too long for that are read again from L2.
//
// The token's own entry is left out of the sums and added in 64 bits, so that 1 - pi(a) keeps its relative accuracy.  Differences enter the
// sums as (z - max z) - (y - max y): the KL, a small difference of large sums, then does not depend on offsets between z and y.
#include "dppo_rowvec.cuh"

namespace dppo {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;

struct PolicyParams {
  RowParams row;             // logits, ids, mu_logp, adv, token_mask, dlogits, outputs (divergence: the KL), workspace
  const void* y;             // reference logits, or null
  int64_t ld_y;
  const float* ref_logp;     // k3
  float beta, eps_low, eps_high;
  double scale;              // s, or 0: in the workspace's header
};

// what a warp knows of its part of a row
struct Part { float mz, S, my, Sy, W, pad; };

// exp(z - m) of a vector's pairs; `arg` receives z - m
template <int N> __device__ __forceinline__ void exp_pairs(const float2* z, float m, float2* arg, float2* e) {
  const float2 nm = make_float2(-m, -m), l2 = make_float2(kLog2e, kLog2e);
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    arg[i] = __fadd2_rn(z[i], nm);
    const float2 x = __fmul2_rn(arg[i], l2);
    e[i] = make_float2(ex2_approx(x.x), ex2_approx(x.y));
  }
}

// coefficients of the row's gradient: dz_j = e^(z_j - zr) (B (z_j - y_j - c) + A) - C e^(y_j - yr), and its value at the token
struct Coef { float zr, yr, A, B, c, C, fix; int zero; };

template <typename InT, typename OutT, int FORM, int NV, bool RESIDENT, int BLOCKS>
__global__ void __launch_bounds__(kThreads, BLOCKS) policy_kl_kernel(PolicyParams q) {
  constexpr bool TWO = FORM != DPPO_KL_K3;
  constexpr int N = Vec<InT>::N;
  constexpr uint32_t INF = RawOf<InT>::kNegInf;
  __shared__ Part parts[kMaxCluster * kWarps];
  __shared__ Coef s_coef;
  const RowParams& p = q.row;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int CL = (int)cluster_nctarank(), rank = CL > 1 ? (int)cluster_ctarank() : 0;
  const int64_t t = blockIdx.x / CL;
  const int a = load_meta(p, t);
  const InT* zrow = reinterpret_cast<const InT*>(p.logits) + t * p.ld_in;
  const InT* yrow = TWO ? reinterpret_cast<const InT*>(q.y) + t * q.ld_y : zrow;
  const uint32_t head = head_of(zrow);
  const RowRef<const InT> rz(zrow, head), ry(yrow, head);
  const RowRef<OutT> rd(reinterpret_cast<OutT*>(p.dlogits) + t * p.ld_out, head);
  if (a < 0) {
    zero_row<OutT, N>(rd, head, p.V, rank, CL, kThreads);
    if (rank == 0 && tid == 0) {
      p.divergence[t] = 0.f;
      p.mask[t] = 0;
      p.row_loss[t] = p.row_r[t] = p.row_absdiff[t] = 0.f;
      if (a == -2) atomicOr(p.status, DPPO_STATUS_BAD_SAMPLED_ID);
    }
    return;
  }
  if (CL > 1) cluster_arrive();            // (the peers have to run before anything is sent to them)
  const int64_t nvec = ((int64_t)head + p.V + N - 1) / N;
  const int64_t av = ((int64_t)a + head) / N;
  const int ai = (int)(((int64_t)a + head) % N);
  const int64_t step = (int64_t)kThreads * CL, v_first = (int64_t)rank * kThreads + tid;
  float z_a = 0.f, y_a = 0.f, mu = 0.f, adv = 0.f;
  if (warp == 0) {                         // in flight while the row is
    z_a = to_f32<InT>(zrow[a]);
    if (TWO) y_a = to_f32<InT>(yrow[a]);
    mu = p.mu_logp[t];
    adv = p.adv[t];
  }

  uint4 zv[NV], yv[TWO ? NV : 1];
  auto load = [&](int64_t v0) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int64_t v = v0 + k * step;
      zv[k] = make_uint4(INF, INF, INF, INF);
      if (TWO) yv[k] = zv[k];
      if (v < nvec) {
        zv[k] = load_vec<InT>(rz, v * N - head, p.V);
        if (TWO) yv[k] = load_vec<InT>(ry, v * N - head, p.V);
      }
    }
  };
  Part w{kLowest, 0.f, kLowest, 0.f, 0.f, 0.f};
  for (int64_t v0 = v_first; v0 - tid < nvec || v0 == v_first; v0 += NV * step) {      // once where the row is resident
    load(v0);
    RawMax<InT> mz, my;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      if (v0 + k * step == av) {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (i == ai) {
            set_raw(zv[k], i, from_f32<InT>(-INFINITY));
            if (TWO) set_raw(yv[k], i, from_f32<InT>(-INFINITY));
          }
      }
      zv[k] = clamp_raw<InT>(zv[k]);
      mz.add(zv[k]);
      if (TWO) {
        yv[k] = clamp_raw<InT>(yv[k]);
        my.add(yv[k]);
      }
    }
    const float bz = max_nan(w.mz, warp_max_nan(mz.value())), by = TWO ? max_nan(w.my, warp_max_nan(my.value())) : 0.f;
    if (!RESIDENT && v0 != v_first) {      // the sums so far, against the new maxima
      const float fz = ex2_approx((w.mz - bz) * kLog2e), fy = TWO ? ex2_approx((w.my - by) * kLog2e) : 0.f;
      if (FORM == DPPO_KL_PI_REF) w.W = (w.mz > kLowest) ? fz * fmaf(w.S, (w.mz - bz) - (w.my - by), w.W) : 0.f;
      if (FORM == DPPO_KL_REF_PI) w.W = (w.my > kLowest) ? fy * fmaf(w.Sy, (w.my - by) - (w.mz - bz), w.W) : 0.f;
      w.S *= fz;
      w.Sy *= fy;
    }
    w.mz = bz;
    w.my = by;
    float2 S = make_float2(0.f, 0.f), Sy = S, W = S;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float2 z[N / 2], az[N / 2], ez[N / 2];
      to_pairs<InT>(zv[k], z);
      exp_pairs<N>(z, bz, az, ez);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) S = __fadd2_rn(S, ez[i]);
      if (TWO) {
        const float2 neg = make_float2(-1.f, -1.f);
        float2 ay[N / 2], ey[N / 2];
        to_pairs<InT>(yv[k], z);
        exp_pairs<N>(z, by, ay, ey);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
          Sy = __fadd2_rn(Sy, ey[i]);
          if (FORM == DPPO_KL_PI_REF) W = __ffma2_rn(ez[i], __ffma2_rn(ay[i], neg, az[i]), W);
          else W = __ffma2_rn(ey[i], __ffma2_rn(az[i], neg, ay[i]), W);
        }
      }
    }
    w.S += warp_sum_f32(S.x + S.y);
    if (TWO) {
      w.Sy += warp_sum_f32(Sy.x + Sy.y);
      w.W += warp_sum_f32(W.x + W.y);
    }
    if (RESIDENT) break;
  }
  const int slot = rank * kWarps + warp;
  if (CL > 1) {
    cluster_wait();
    if (lane < CL) {
      const uint32_t dst = map_to_cta(smem_u32(&parts[slot]), (uint32_t)lane);
      st_cluster_f32x2(dst, w.mz, w.S);
      if (TWO) {
        st_cluster_f32x2(dst + 8, w.my, w.Sy);
        st_cluster_f32x2(dst + 16, w.W, 0.f);
      }
    }
    cluster_sync_all();
  } else {
    if (lane == 0) parts[slot] = w;
    __syncthreads();
  }

  if (warp == 0) {
    // ---- the row's scalars, by every CTA for itself
    constexpr int PER = kMaxCluster * kWarps / 32;
    Part x[PER];
    double Mz = -INFINITY, My = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int k = lane + 32 * i;
      x[i] = k < CL * kWarps ? parts[k] : Part{kLowest, 0.f, kLowest, 0.f, 0.f, 0.f};
      if (!(x[i].mz > kLowest) && x[i].S == x[i].S) x[i].S = 0.f;         // a warp that saw nothing but probability zero counts nothing
      if (!(x[i].my > kLowest) && x[i].Sy == x[i].Sy) x[i].Sy = 0.f;
      if (x[i].S != 0.f) Mz = fmax(Mz, (double)x[i].mz);
      if (TWO && x[i].Sy != 0.f) My = fmax(My, (double)x[i].my);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      Mz = fmax(Mz, __shfl_xor_sync(0xffffffffu, Mz, o));
      if (TWO) My = fmax(My, __shfl_xor_sync(0xffffffffu, My, o));
    }
    // sums over the other entries, against Mz and My; W against Mz - My
    double S = 0.0, Sy = 0.0, W = 0.0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const double fz = x[i].S != 0.f ? exp((double)x[i].mz - Mz) : 0.0, fy = (TWO && x[i].Sy != 0.f) ? exp((double)x[i].my - My) : 0.0;
      S += fz * (double)x[i].S;
      if (TWO) Sy += fy * (double)x[i].Sy;
      const double off = ((double)x[i].mz - (double)x[i].my) - (Mz - My);
      if (FORM == DPPO_KL_PI_REF && fz != 0.0) W += fz * ((double)x[i].W + (double)x[i].S * off);
      if (FORM == DPPO_KL_REF_PI && fy != 0.0) W += fy * ((double)x[i].W - (double)x[i].Sy * off);
    }
    S = warp_sum(S);
    if (TWO) { Sy = warp_sum(Sy); W = warp_sum(W); }
    if (z_a <= kLowest) z_a = -INFINITY;
    if (y_a <= kLowest) y_a = -INFINITY;
    double lse, other, lse_y = 0.0, other_y = 0.0;
    combine_lse(Mz, S, (double)z_a, lse, other);
    if (TWO) combine_lse(My, Sy, (double)y_a, lse_y, other_y);
    bool ok = isfinite(lse) && isfinite(lse_y);
    double kl = 0.0, g = 0.0, lp = 0.0, r = 0.0, row_loss = 0.0, pi_a = 0.0;
    int M = 0;
    Coef co = {};
    co.zero = 1;
    const double s = q.scale > 0.0 ? q.scale : p.hdr->scale;
    if (ok) {
      lp = (double)z_a - lse;
      pi_a = exp(lp);
      r = exp(lp - (double)mu);
      const double A = (double)adv, lo = 1.0 - (double)q.eps_low, hi = 1.0 + (double)q.eps_high;
      M = ((A > 0.0 && r > hi) || (A < 0.0 && r < lo)) ? 0 : 1;
      g = M ? s * r * A : 0.0;
      const double surrogate = M ? r * A : (A > 0.0 ? hi : lo) * A;
      const double b = s * (double)q.beta;
      double lr_a = 0.0;                   // log rho(a)
      if (FORM == DPPO_KL_K3) {
        const double d = (double)q.ref_logp[t] - lp;
        kl = expm1(d) - d;
        const double gk = g + b * expm1(d);
        const double near = (double)(float)lse;
        co.zr = (float)lse;
        co.A = (float)(gk * exp(near - lse));
        co.fix = (float)(gk * expm1(lp));
      } else {
        lr_a = (double)y_a - lse_y;
        const double c = lse - lse_y;      // sum over the other entries of probability * (difference of the log-probabilities)
        if (FORM == DPPO_KL_PI_REF) {
          kl = (S > 0.0 ? exp(Mz - lse) * (W + S * ((Mz - My) - c)) : 0.0) + (pi_a > 0.0 ? pi_a * (lp - lr_a) : 0.0);
        } else {
          const double rho_a = exp(lr_a);
          kl = (Sy > 0.0 ? exp(My - lse_y) * (W + Sy * (c - (Mz - My))) : 0.0) + (rho_a > 0.0 ? rho_a * (lr_a - lp) : 0.0);
        }
        const double nz = (double)(float)lse, ny = (double)(float)lse_y, fz = exp(nz - lse);
        co.zr = (float)lse;
        co.yr = (float)lse_y;
        if (FORM == DPPO_KL_PI_REF) {
          co.c = (float)c;
          co.B = (float)(b * fz);
          co.A = (float)(fz * (g - b * (c - (double)co.c + kl)));
          co.fix = (float)(g * expm1(lp) + (pi_a > 0.0 ? b * pi_a * (lp - lr_a - kl) : 0.0));
        } else {
          co.A = (float)(fz * (g + b));
          co.C = (float)(b * exp(ny - lse_y));
          co.fix = (float)(g * expm1(lp) + b * (pi_a - exp(lr_a)));
        }
      }
      row_loss = s * ((double)q.beta * kl - surrogate);
      ok = fabs(kl) < 1e30 && isfinite(row_loss) && isfinite(g);
      co.zero = 0;
    }
    if (!ok) { co.zero = 1; kl = r = row_loss = 0.0; M = 0; }
    if (lane == 0) {
      s_coef = co;
      if (rank == 0) {
        p.divergence[t] = (float)kl;
        p.mask[t] = (uint8_t)M;
        p.row_loss[t] = (float)row_loss;
        p.row_r[t] = (float)r;
        p.row_absdiff[t] = ok ? (float)fabs(exp((double)mu) - pi_a) : 0.f;
        if (!ok) atomicOr(p.status, DPPO_STATUS_NONFINITE_ROW);
      }
    }
  }
  __syncthreads();
  const Coef co = s_coef;
  if (co.zero) {
    zero_row<OutT, N>(rd, head, p.V, rank, CL, kThreads);
    return;
  }
  const float2 A2 = make_float2(co.A, co.A), B2 = make_float2(co.B, co.B), nc = make_float2(-co.c, -co.c), C2 = make_float2(-co.C, -co.C), neg = make_float2(-1.f, -1.f);
  for (int64_t v0 = v_first; v0 - tid < nvec || v0 == v_first; v0 += NV * step) {
    if (!RESIDENT) {
      load(v0);
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        zv[k] = clamp_raw<InT>(zv[k]);
        if (TWO) yv[k] = clamp_raw<InT>(yv[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int64_t v = v0 + k * step;
      if (v >= nvec) break;
      float2 z[N / 2], az[N / 2], ez[N / 2];
      float out[N];
      to_pairs<InT>(zv[k], z);
      exp_pairs<N>(z, co.zr, az, ez);
      if (TWO) {
        float2 y[N / 2], ay[N / 2], ey[N / 2];
        to_pairs<InT>(yv[k], y);
        if (FORM == DPPO_KL_REF_PI) exp_pairs<N>(y, co.yr, ay, ey);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
          // (e B) first: an entry of probability zero stays zero whatever its difference is
          if (FORM == DPPO_KL_PI_REF) ez[i] = __ffma2_rn(__fmul2_rn(ez[i], B2), __fadd2_rn(__ffma2_rn(y[i], neg, z[i]), nc), __fmul2_rn(ez[i], A2));
          else ez[i] = __ffma2_rn(ey[i], C2, __fmul2_rn(ez[i], A2));
        }
      } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) ez[i] = __fmul2_rn(ez[i], A2);
      }
#pragma unroll
      for (int i = 0; i < N / 2; ++i) { out[2 * i] = ez[i].x; out[2 * i + 1] = ez[i].y; }
      if (v == av) {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (i == ai) out[i] = co.fix;
      }
      store_vec<OutT, N>(rd, v * N - head, p.V, out);
    }
    if (RESIDENT) break;
  }
}

template <typename InT, typename OutT, int FORM, int NV, bool RESIDENT, int BLOCKS>
cudaError_t launch_one(const PolicyParams& q, int CL, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)CL; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(q.row.T * CL), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = CL > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, policy_kl_kernel<InT, OutT, FORM, NV, RESIDENT, BLOCKS>, q);
}

template <typename InT, typename OutT, int FORM>
cudaError_t launch_form(const PolicyParams& q, cudaStream_t st) {
  constexpr int N = Vec<InT>::N;
  constexpr int NV = (FORM == DPPO_KL_K3 && N == 4) ? 20 : 10;            // 80 registers of row at most
  constexpr int BLOCKS = FORM == DPPO_KL_K3 && N == 8 ? 3 : 2;
  const int64_t nvec = (q.row.V + 2 * N - 2) / N;
  int CL = 1;
  while (CL < kMaxCluster && (int64_t)CL * kThreads * NV < nvec) CL *= 2;
  while (CL < kMaxCluster && q.row.T * CL < 2 * 148 && (int64_t)CL * kThreads < nvec) CL *= 2;      // few rows: more SMs each
  if ((int64_t)CL * kThreads * NV >= nvec) return launch_one<InT, OutT, FORM, NV, true, BLOCKS>(q, CL, st);
  return launch_one<InT, OutT, FORM, NV, false, BLOCKS>(q, CL, st);
}

template <typename InT, typename OutT>
cudaError_t launch_types(const PolicyParams& q, int form, cudaStream_t st) {
  switch (form) {
    case DPPO_KL_K3: return launch_form<InT, OutT, DPPO_KL_K3>(q, st);
    case DPPO_KL_PI_REF: return launch_form<InT, OutT, DPPO_KL_PI_REF>(q, st);
    default: return launch_form<InT, OutT, DPPO_KL_REF_PI>(q, st);
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
  if (!(kl_coef >= 0.f) || !isfinite(kl_coef) || !(eps_low >= 0.f) || !(eps_high >= 0.f)) return DPPO_ERR_UNSUPPORTED;
  const bool two = kl_form != DPPO_KL_K3;
  if (!loss || !status) return DPPO_ERR_NULL;
  if (T > 0 && (!logits || !sampled_ids || !mu_logp || !advantages || !kl || !mask || !dlogits || (two ? !ref_logits : !ref_logp))) return DPPO_ERR_NULL;
  if (T > 1 && (logits_row_stride < V || dlogits_row_stride < V || (two && ref_row_stride < V))) return DPPO_ERR_STRIDE;
  const int out_dtype = o.dlogits_dtype == DPPO_DLOGITS_F32 ? DPPO_F32 : logits_dtype;
  if ((uintptr_t)logits % esize(logits_dtype) || (uintptr_t)dlogits % esize(out_dtype) || (two && (uintptr_t)ref_logits % esize(logits_dtype))) return DPPO_ERR_ALIGN;
  if ((uintptr_t)sampled_ids % 4 || (uintptr_t)mu_logp % 4 || (uintptr_t)advantages % 4 || (uintptr_t)ref_logp % 4 || (uintptr_t)loss % 4 ||
      (uintptr_t)kl % 4 || (uintptr_t)stats % 4 || (uintptr_t)status % 4) return DPPO_ERR_ALIGN;
  if (T > 0) {
    // the gradient in place of the logits is fine (a cluster holds its row before it writes); any other overlap is not
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
  char* ws = reinterpret_cast<char*>(workspace);
  const size_t per = (dppo_workspace_bytes(T, V, 0, 0) - 256) / 3;
  p.hdr = reinterpret_cast<WsHeader*>(ws);
  p.row_loss = reinterpret_cast<float*>(ws + 256);
  p.row_r = reinterpret_cast<float*>(ws + 256 + per);
  p.row_absdiff = reinterpret_cast<float*>(ws + 256 + 2 * per);
  q.y = ref_logits; q.ld_y = ref_row_stride; q.ref_logp = ref_logp; q.beta = kl_coef; q.eps_low = eps_low; q.eps_high = eps_high;
  // without a mask the scale is known here, and the count of valid rows is only wanted for the statistics
  q.scale = o.loss_scale > 0.f ? (double)o.loss_scale : (!token_mask && T > 0 ? 1.0 / (double)T : 0.0);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  if ((q.scale == 0.0 || stats) && launch_prelude(p, st) != cudaSuccess) return DPPO_ERR_CUDA;
  if (T > 0) {
    cudaError_t e;
    if (logits_dtype == DPPO_BF16 && out_dtype == DPPO_BF16) e = launch_types<__nv_bfloat16, __nv_bfloat16>(q, kl_form, st);
    else if (logits_dtype == DPPO_BF16) e = launch_types<__nv_bfloat16, float>(q, kl_form, st);
    else e = launch_types<float, float>(q, kl_form, st);
    if (e != cudaSuccess) return DPPO_ERR_CUDA;
  }
  return launch_finalize(p, st) == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
}
