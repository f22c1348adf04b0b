// Log-probabilities of given tokens and their gradient, and the loss over pairs of sequences that is built from the two.
//
//   logp_t = z_t[a_t] - lse_t,   dz_tj = c_t (1[j = a_t] - pi_tj),   c_t = d loss / d logp_t
//
// Both kernels stream the rows with plain 16-byte loads and no state between rows.  The forward pass gives a row to a cluster of up to
// 8 CTAs (few rows: more SMs per row), which add up exp(z - max) of the entries other than the token's own and merge their partial sums
// through distributed shared memory; the backward pass is cut into pieces of a row that know everything beforehand.
//
// Pairs of sequences: the coefficient c_t of a row needs the sums over all rows of its pair, so the logits are read twice (forward, a
// single CTA for the pairs, backward).  The backward pass walks the rows from the last to the first: those it starts with were
// read last and still lie in L2.
//
// All of it is bound by HBM: forward 8192 x 151936 bf16 388 us, 97 % of the measured copy rate; 16 pairs, 6000 x 151936 bf16, 845 us for three passes over
// 1.82 GB.  A CTA per row and four vectors in flight a thread: eight are slower (445 us for the 8192 rows; fewer CTAs an SM), and so are 2, 4 or 8 CTAs
// to a row where there are rows enough (422, 486, 661 us); for one row they are the faster ones (18.5, 12.4, 9.5 and 8.2 us).
#include "dppo_rowvec.cuh"

namespace dppo {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kUnroll = 4;                 // vectors a thread has in flight
constexpr int kMaxCluster = 8;

__device__ __forceinline__ void st_cluster_f64x2(uint32_t cluster_addr, double a, double b) {
  asm volatile("st.shared::cluster.v2.f64 [%0], {%1, %2};" ::"r"(cluster_addr), "d"(a), "d"(b) : "memory");
}

struct LogpParams {
  const void* z;
  int64_t T, V, ld;
  const int32_t* ids;
  const uint8_t* token_mask;
  float* logp;
  double* lse;                             // may be null
  int32_t* status;
  // pairs of sequences (null for dppo_token_logp)
  const int64_t* cu;
  int64_t P;
  const float* ref_logp;
  double* ratio;                           // logp - ref_logp; NaN: row dropped
  float* coef;                             // zero for rows outside the sequences
};

// valid row: its token; -1: masked out or outside the sequences; -2: token out of range
__device__ __forceinline__ int row_token(const int32_t* ids, const uint8_t* token_mask, int64_t t, int64_t V) {
  if (token_mask && token_mask[t] == 0) return -1;
  const int a = ids[t];
  return (a < 0 || (int64_t)a >= V) ? -2 : a;
}

// exp(z - m) of a vector's pairs, added up.  What is off on one side for all rows of a sequence would add up: log2(e) comes in two parts (rounded to fp32
// it is 1.3e-8 off, times the depth of a row's mass below its maximum), and the argument is raised by what ex2_approx is low by on average (measured
// 4.6e-8 of its value over flat rows; its value at zero is exact and stays so).
template <int N> __device__ __forceinline__ float2 exp_sum(const float2* z, float m) {
  constexpr float kRest = (float)(1.4426950408889634 - (double)kLog2e), kRaise = 6.6e-8f;
  const float2 nm = make_float2(-m, -m), l2 = make_float2(kLog2e, kLog2e), rest = make_float2(kRest, kRest), raise = make_float2(kRaise, kRaise);
  float2 s = make_float2(0.f, 0.f);
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const float2 d = __fadd2_rn(z[i], nm), x = __ffma2_rn(d, l2, __ffma2_rn(d, rest, raise));
    s = __fadd2_rn(s, make_float2(ex2_approx(x.x), ex2_approx(x.y)));
  }
  return s;
}

template <typename InT>
__global__ void __launch_bounds__(kThreads) token_logp_kernel(LogpParams p) {
  __shared__ double2 parts[kMaxCluster * kWarps];         // (maximum, sum of exp) of every warp of the cluster, in its first CTA
  constexpr int N = Vec<InT>::N;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int CL = (int)cluster_nctarank(), rank = CL > 1 ? (int)cluster_ctarank() : 0;
  const int64_t t = blockIdx.x / CL;
  int a = row_token(p.ids, p.token_mask, t, p.V);
  if (p.cu && (t < p.cu[0] || t >= p.cu[2 * p.P])) a = -1;
  if (a < 0) {
    if (rank == 0 && tid == 0) {
      p.logp[t] = 0.f;
      if (p.lse) p.lse[t] = a == -2 ? (double)NAN : 0.0;
      if (p.ratio) { p.ratio[t] = a == -2 ? (double)NAN : 0.0; p.coef[t] = 0.f; }
      if (a == -2) atomicOr(p.status, DPPO_STATUS_BAD_SAMPLED_ID);
    }
    return;
  }
  if (CL > 1) cluster_arrive();            // (the peers have to run before anything is sent to them)
  const InT* row = reinterpret_cast<const InT*>(p.z) + t * p.ld;
  const uint32_t head = head_of(row);
  const RowRef<const InT, N> r(row, head, p.V);
  const int step = kThreads * CL;
  // the token's entry is left out of the sums: 1 - pi(a) keeps its relative accuracy
  const int own = (int)(((uint32_t)a + head) / N) - (rank * kThreads + tid);       // vectors from this thread's first to the token's
  const int own_k = own >= 0 && own % step == 0 ? own / step : -1;
  float m = kLowest, s = 0.f;
  for (int v0 = rank * kThreads + tid, k0 = 0; v0 < r.nvec; v0 += kUnroll * step, k0 += kUnroll) {
    uint4 raw[kUnroll];
    RawMax<InT> mx;
    load_vecs<kUnroll>(raw, r, v0, step, r.nvec);
    if (own_k >= k0 && own_k < k0 + kUnroll) {
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (k0 + k == own_k && i == (int)(((uint32_t)a + head) % N)) set_raw(raw[k], i, from_f32<InT>(-INFINITY));
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      raw[k] = clamp_raw<InT>(raw[k]);
      mx.add(raw[k]);
    }
    const float vm = mx.value();
    if (!(vm <= m)) { s *= ex2_approx((m - vm) * kLog2e); m = vm; }
    float2 acc = make_float2(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      float2 z[N / 2];
      to_pairs<InT>(raw[k], z);
      acc = __fadd2_rn(acc, exp_sum<N>(z, m));
    }
    s += acc.x + acc.y;
  }
  const float wm = warp_max_nan(m);
  const double ws = warp_sum((double)s * exp((double)m - (double)wm));
  const int slot = rank * kWarps + warp;
  if (CL > 1) {
    cluster_wait();
    if (lane == 0) st_cluster_f64x2(map_to_cta(smem_u32(&parts[slot]), 0u), (double)wm, ws);
    cluster_sync_all();
  } else {
    if (lane == 0) parts[slot] = make_double2((double)wm, ws);
    __syncthreads();
  }
  if (rank != 0 || warp != 0) return;
  double pm[kMaxCluster * kWarps / 32], ps[kMaxCluster * kWarps / 32], M = -INFINITY, S = 0.0;
#pragma unroll
  for (int i = 0; i < kMaxCluster * kWarps / 32; ++i) {
    const int k = lane + 32 * i;
    const double2 x = k < CL * kWarps ? parts[k] : make_double2((double)kLowest, 0.0);
    const bool some = x.x > (double)kLowest || x.y != x.y;         // a warp that saw nothing but probability zero counts nothing
    pm[i] = x.x;
    ps[i] = some ? x.y : 0.0;
    if (some) M = fmax(M, pm[i]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmax(M, __shfl_xor_sync(0xffffffffu, M, o));
#pragma unroll
  for (int i = 0; i < kMaxCluster * kWarps / 32; ++i)
    if (ps[i] != 0.0) S += ps[i] * exp(pm[i] - M);
  S = warp_sum(S);
  if (lane == 0) {
    float z_a = to_f32<InT>(row[a]);
    if (z_a <= kLowest) z_a = -INFINITY;
    double lse, log_other;
    combine_lse(M, S, (double)z_a, lse, log_other);
    const bool ok = isfinite(lse);
    // -log(1 + sum over the others / the token's own): z_a - lse would round at the size of lse
    const double u = S > 0.0 ? S * exp(M - (double)z_a) : 0.0;
    const double lp = !ok ? 0.0 : (isfinite(u) ? -log1p(u) : (double)z_a - lse);
    p.logp[t] = (float)lp;
    if (p.lse) p.lse[t] = ok ? lse : (double)NAN;
    if (p.ratio) p.ratio[t] = ok ? lp - (p.ref_logp ? (double)p.ref_logp[t] : 0.0) : (double)NAN;
    if (!ok) atomicOr(p.status, DPPO_STATUS_NONFINITE_ROW);
  }
}

struct GradParams {
  const void* z;
  int64_t T, V, ld, ld_out, pieces;        // pieces: parts of a row, each a CTA's
  const int32_t* ids;
  const uint8_t* token_mask;
  const double* lse;
  const float* coef;                       // c_t
  void* dz;
  int32_t* status;
  int backwards;
};

template <typename InT, typename OutT>
__global__ void __launch_bounds__(kThreads) token_grad_kernel(GradParams p) {
  constexpr int N = Vec<InT>::N;
  for (int64_t item = blockIdx.x; item < p.T * p.pieces; item += gridDim.x) {
    const int64_t at = p.backwards ? p.T * p.pieces - 1 - item : item;
    const int64_t t = at / p.pieces;
    const int v0 = (int)(at - t * p.pieces) * (kUnroll * kThreads) + (int)threadIdx.x;
    const InT* row = reinterpret_cast<const InT*>(p.z) + t * p.ld;
    const uint32_t head = head_of(row);
    const RowRef<const InT, N> r(row, head, p.V);
    const RowRef<OutT, N> d(reinterpret_cast<OutT*>(p.dz) + t * p.ld_out, head, p.V);
    const int a = row_token(p.ids, p.token_mask, t, p.V);
    const float c = p.coef[t];
    const double lse = p.lse[t];
    if (c != 0.f && (a == -2 || (a >= 0 && !isfinite(lse))) && threadIdx.x == 0)
      atomicOr(p.status, a == -2 ? DPPO_STATUS_BAD_SAMPLED_ID : DPPO_STATUS_NONFINITE_ROW);
    if (a < 0 || c == 0.f || !isfinite(lse)) {
      const float zero[N] = {};
#pragma unroll
      for (int k = 0; k < kUnroll; ++k)
        if (v0 + k * kThreads < r.nvec) store_vec<OutT, N>(d, v0 + k * kThreads, zero);
      continue;
    }
    const int av = (int)(((uint32_t)a + head) / N);
    const bool own = av >= v0 && av < v0 + kUnroll * kThreads && (av - v0) % kThreads == 0;
    const float z_a = own ? to_f32<InT>(row[a]) : 0.f;     // (read before the gradient may overwrite it)
    uint4 raw[kUnroll];
    load_vecs<kUnroll>(raw, r, v0, kThreads, r.nvec);
    // pi = exp(z - lse): z - (float)lse is exact for the entries that count, what (float)lse lacks goes into the factor
    const float near = (float)lse;
    const double over = (double)near - lse;
    const float f = (float)(-(double)c * (fabs(over) < kNearZero ? exp_series(over) : (double)ex2_approx((float)over * kLog2e)));
    const float2 nr = make_float2(-near, -near), l2 = make_float2(kLog2e, kLog2e), f2 = make_float2(f, f);
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const int v = v0 + k * kThreads;
      if (v >= r.nvec) break;
      float2 z[N / 2];
      to_pairs<InT>(raw[k], z);
      float x[N];
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const float2 arg = __fmul2_rn(__fadd2_rn(z[i], nr), l2);
        const float2 e = __fmul2_rn(make_float2(ex2_approx(arg.x), ex2_approx(arg.y)), f2);
        x[2 * i] = e.x;
        x[2 * i + 1] = e.y;
      }
      store_vec<OutT, N>(d, v, x);
    }
    if (own) d.row[a] = from_f32<OutT>((float)(-(double)c * expm1((double)z_a - lse)));      // c (1 - pi(a)), without the cancellation
  }
}

// ------------------------------------------------------------------------------------------------- pairs of sequences
struct PairParams {
  int64_t T, P;
  const int64_t* cu;
  const uint8_t* token_mask;
  const double* ratio;
  double* seq;                             // [2 P] workspace: sums, then coefficients
  int64_t* seq_n;                          // [2 P] rows that count
  float* coef;                             // [T]
  int variant, average;
  double beta, smoothing, margin, loss_scale;
  float* loss;
  float* reward;
  int32_t* status;
};

constexpr int kPairThreads = 1024, kPairWarps = kPairThreads / 32;

__device__ __forceinline__ double softplus(double x) { return fmax(x, 0.0) + log1p(exp(-fabs(x))); }
__device__ __forceinline__ double sigmoid(double x) { return x >= 0.0 ? 1.0 / (1.0 + exp(-x)) : exp(x) / (1.0 + exp(x)); }

// One CTA: sums over the sequences (W warps each), the pairs, the rows' coefficients.  All sums in 64 bits and a fixed order.
__global__ void __launch_bounds__(kPairThreads) preference_pairs_kernel(PairParams p) {
  __shared__ int s_bad;
  __shared__ double s_sum[kPairWarps];
  __shared__ int64_t s_n[kPairWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t nseq = 2 * p.P;
  if (tid == 0) s_bad = 0;
  __syncthreads();
  int bad = 0;
  for (int64_t i = tid; i <= nseq; i += kPairThreads) {
    const int64_t c = p.cu[i];
    bad |= c < 0 || c > p.T || (i < nseq && p.cu[i + 1] < c);
  }
  if (bad) s_bad = 1;
  __syncthreads();
  if (s_bad) {                             // no sequence can be trusted: no loss, no gradient
    for (int64_t t = tid; t < p.T; t += kPairThreads) p.coef[t] = 0.f;
    for (int64_t i = tid; i < nseq; i += kPairThreads) p.reward[i] = 0.f;
    if (tid == 0) { *p.loss = 0.f; atomicOr(p.status, DPPO_STATUS_BAD_SEQUENCES); }
    return;
  }
  int W = 1;                               // warps of a sequence
  while (W < kPairWarps && W * nseq < kPairWarps) W *= 2;
  const int groups = kPairWarps / W;
  for (int64_t base = 0; base < nseq; base += groups) {
    const int64_t q = base + warp / W;
    double sum = 0.0;
    int64_t n = 0;
    if (q < nseq) {
      const int64_t end = p.cu[q + 1];
      for (int64_t t = p.cu[q] + (warp % W) * 32 + lane; t < end; t += 32 * W) {
        if (p.token_mask && p.token_mask[t] == 0) continue;
        sum += p.ratio[t];
        ++n;
      }
    }
    sum = warp_sum(sum);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
    if (lane == 0) { s_sum[warp] = sum; s_n[warp] = n; }
    __syncthreads();
    if (tid < groups && base + tid < nseq) {
      double all = 0.0;
      int64_t cnt = 0;
      for (int w = 0; w < W; ++w) { all += s_sum[tid * W + w]; cnt += s_n[tid * W + w]; }
      p.seq[base + tid] = all;
      p.seq_n[base + tid] = cnt;
    }
    __syncthreads();
  }
  double loss = 0.0;
  int64_t pairs = 0;
  for (int64_t i = tid; i < p.P; i += kPairThreads) {
    const int64_t nw = p.seq_n[2 * i], nl = p.seq_n[2 * i + 1];
    double cw = 0.0, cl = 0.0, Rw = 0.0, Rl = 0.0;
    if (nw > 0 && nl > 0) {                // a pair without rows on either side is none
      const double bw = p.beta / (p.average ? (double)nw : 1.0), bl = p.beta / (p.average ? (double)nl : 1.0);
      const double h = bw * p.seq[2 * i] - bl * p.seq[2 * i + 1] - p.margin;
      double L, dh;
      if (p.variant == DPPO_PREF_SIGMOID) {
        L = (1.0 - p.smoothing) * softplus(-h) + p.smoothing * softplus(h);
        dh = p.smoothing * sigmoid(h) - (1.0 - p.smoothing) * sigmoid(-h);
      } else if (p.variant == DPPO_PREF_IPO) {
        const double x = (h - 0.5) / p.beta;
        L = x * x;
        dh = 2.0 * x / p.beta;
      } else {
        L = fmax(0.0, 1.0 - h);
        dh = h < 1.0 ? -1.0 : 0.0;
      }
      if (isfinite(h) && isfinite(L)) {
        Rw = bw * p.seq[2 * i];
        Rl = bl * p.seq[2 * i + 1];
        cw = dh * bw;
        cl = -dh * bl;
        loss += L;
        ++pairs;
      } else {
        atomicOr(p.status, DPPO_STATUS_NONFINITE_ROW);
      }
    }
    p.reward[2 * i] = (float)Rw;
    p.reward[2 * i + 1] = (float)Rl;
    p.seq[2 * i] = cw;
    p.seq[2 * i + 1] = cl;
  }
  loss = warp_sum(loss);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) pairs += __shfl_xor_sync(0xffffffffu, pairs, o);
  if (lane == 0) { s_sum[warp] = loss; s_n[warp] = pairs; }
  __syncthreads();
  loss = 0.0;
  pairs = 0;
  for (int w = 0; w < kPairWarps; ++w) { loss += s_sum[w]; pairs += s_n[w]; }
  const double scale = p.loss_scale > 0.0 ? p.loss_scale : (pairs > 0 ? 1.0 / (double)pairs : 0.0);
  if (tid == 0) *p.loss = (float)(scale * loss);
  for (int64_t base = 0; base < nseq; base += groups) {
    const int64_t q = base + warp / W;
    if (q >= nseq) continue;
    const float c = (float)(scale * p.seq[q]);
    const int64_t end = p.cu[q + 1];
    for (int64_t t = p.cu[q] + (warp % W) * 32 + lane; t < end; t += 32 * W) p.coef[t] = (p.token_mask && p.token_mask[t] == 0) ? 0.f : c;
  }
}

// ---------------------------------------------------------------------------------------------------------- launchers
// CTAs that share a row of the forward pass: more where the rows are few
int logp_cluster(int64_t T, int64_t V, int elem) {
  const int64_t vecs = (V * elem + 15) / 16;
  int CL = 1;
  while (CL < kMaxCluster && T * CL < 148 * 8 && vecs > (int64_t)CL * kThreads * kUnroll) CL *= 2;
  return CL;
}

template <typename InT>
cudaError_t launch_logp_t(const LogpParams& p, cudaStream_t st) {
  const int CL = logp_cluster(p.T, p.V, (int)sizeof(InT));
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)CL; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(p.T * CL), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = CL > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, token_logp_kernel<InT>, p);
}

cudaError_t launch_logp(const LogpParams& p, int dtype, cudaStream_t st) {
  return dtype == DPPO_BF16 ? launch_logp_t<__nv_bfloat16>(p, st) : launch_logp_t<float>(p, st);
}

cudaError_t launch_grad(GradParams p, int in_dtype, int out_dtype, cudaStream_t st) {
  const int elem = in_dtype == DPPO_BF16 ? 2 : 4, N = 16 / elem;
  const int64_t nvec = (p.V + 2 * N - 2) / N;              // of a row with the largest head
  p.pieces = (nvec + kUnroll * kThreads - 1) / (kUnroll * kThreads);
  const int64_t items = p.T * p.pieces;
  const unsigned grid = (unsigned)(items < (1 << 30) ? items : (1 << 30));
  if (in_dtype == DPPO_BF16 && out_dtype == DPPO_BF16) token_grad_kernel<__nv_bfloat16, __nv_bfloat16><<<grid, kThreads, 0, st>>>(p);
  else if (in_dtype == DPPO_BF16) token_grad_kernel<__nv_bfloat16, float><<<grid, kThreads, 0, st>>>(p);
  else token_grad_kernel<float, float><<<grid, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}

size_t elem_size(int dt) { return dt == DPPO_BF16 ? 2 : 4; }
size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// shared argument checks of a call over logits (and its gradient, when dz is asked for)
int check_rows(const void* z, int64_t T, int64_t V, int64_t ld, int dtype, const int32_t* ids, const int32_t* status) {
  if (T < 0 || V < 1 || V > ((int64_t)1 << 30) || T > ((int64_t)1 << 27)) return DPPO_ERR_SHAPE;
  if (dtype != DPPO_F32 && dtype != DPPO_BF16) return DPPO_ERR_DTYPE;
  if (!status || (T > 0 && (!z || !ids))) return DPPO_ERR_NULL;
  if (T > 1 && ld < V) return DPPO_ERR_STRIDE;
  if ((uintptr_t)z % elem_size(dtype) || (uintptr_t)ids % 4 || (uintptr_t)status % 4) return DPPO_ERR_ALIGN;
  return DPPO_OK;
}
int check_gradient(const void* z, int64_t T, int64_t V, int64_t ld, int dtype, const void* dz, int64_t ld_out, int out_dtype) {
  if (T > 0 && !dz) return DPPO_ERR_NULL;
  if (T > 1 && ld_out < V) return DPPO_ERR_STRIDE;
  if ((uintptr_t)dz % elem_size(out_dtype)) return DPPO_ERR_ALIGN;
  if (T == 0) return DPPO_OK;
  const uintptr_t in0 = (uintptr_t)z, in1 = in0 + ((size_t)(T - 1) * ld + V) * elem_size(dtype);
  const uintptr_t out0 = (uintptr_t)dz, out1 = out0 + ((size_t)(T - 1) * ld_out + V) * elem_size(out_dtype);
  const bool in_place = dz == z && out_dtype == dtype && (T == 1 || ld == ld_out);
  return (!in_place && in0 < out1 && out0 < in1) ? DPPO_ERR_ALIAS : DPPO_OK;
}

}  // namespace
}  // namespace dppo

extern "C" int dppo_token_logp(const void* logits, int64_t T, int64_t V, int64_t logits_row_stride, int logits_dtype,
                               const int32_t* sampled_ids, const uint8_t* token_mask, float* logp, double* lse,
                               int32_t* status, void* cuda_stream) {
  using namespace dppo;
  const int rc = check_rows(logits, T, V, logits_row_stride, logits_dtype, sampled_ids, status);
  if (rc != DPPO_OK) return rc;
  if (T > 0 && !logp) return DPPO_ERR_NULL;
  if ((uintptr_t)logp % 4 || (uintptr_t)lse % 8) return DPPO_ERR_ALIGN;
  if (T == 0) return DPPO_OK;
  LogpParams p = {};
  p.z = logits; p.T = T; p.V = V; p.ld = logits_row_stride; p.ids = sampled_ids; p.token_mask = token_mask;
  p.logp = logp; p.lse = lse; p.status = status;
  return launch_logp(p, logits_dtype, reinterpret_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
}

extern "C" int dppo_token_logp_bwd(const void* logits, int64_t T, int64_t V, int64_t logits_row_stride, int logits_dtype,
                                   const int32_t* sampled_ids, const uint8_t* token_mask, const double* lse, const float* dlogp,
                                   int dlogits_dtype, void* dlogits, int64_t dlogits_row_stride, int32_t* status, void* cuda_stream) {
  using namespace dppo;
  int rc = check_rows(logits, T, V, logits_row_stride, logits_dtype, sampled_ids, status);
  if (rc != DPPO_OK) return rc;
  if (dlogits_dtype != DPPO_DLOGITS_SAME && dlogits_dtype != DPPO_DLOGITS_F32) return DPPO_ERR_DTYPE;
  if (T > 0 && (!lse || !dlogp)) return DPPO_ERR_NULL;
  if ((uintptr_t)dlogp % 4 || (uintptr_t)lse % 8) return DPPO_ERR_ALIGN;
  const int out_dtype = dlogits_dtype == DPPO_DLOGITS_F32 ? DPPO_F32 : logits_dtype;
  rc = check_gradient(logits, T, V, logits_row_stride, logits_dtype, dlogits, dlogits_row_stride, out_dtype);
  if (rc != DPPO_OK || T == 0) return rc;
  GradParams g = {};
  g.z = logits; g.T = T; g.V = V; g.ld = logits_row_stride; g.ld_out = dlogits_row_stride; g.ids = sampled_ids; g.token_mask = token_mask;
  g.lse = lse; g.coef = dlogp; g.dz = dlogits; g.status = status;
  return launch_grad(g, logits_dtype, out_dtype, reinterpret_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
}

extern "C" size_t dppo_preference_workspace_bytes(int64_t T, int64_t P) {
  using namespace dppo;
  if (T < 0) T = 0;
  if (P < 0) P = 0;
  // per row: log-sum-exp, log ratio, coefficient; per sequence: sum and number of rows
  return 2 * up256((size_t)T * 8) + up256((size_t)T * 4) + 2 * up256((size_t)P * 16) + 256;
}

extern "C" int dppo_preference_fwd_bwd(const void* logits, int64_t T, int64_t V, int64_t logits_row_stride, int logits_dtype,
                                       const int32_t* sampled_ids, const uint8_t* token_mask, const float* ref_logp,
                                       const int64_t* cu_seqlens, int64_t P, int variant, float beta, float label_smoothing,
                                       float margin, int average, const dppo_opts* opts, float* loss, float* reward, float* logp,
                                       void* dlogits, int64_t dlogits_row_stride, int32_t* status,
                                       void* workspace, size_t workspace_bytes, void* cuda_stream) {
  using namespace dppo;
  dppo_opts o = {};
  if (opts) o = *opts;
  int rc = check_rows(logits, T, V, logits_row_stride, logits_dtype, sampled_ids, status);
  if (rc != DPPO_OK) return rc;
  if (P < 0 || P > ((int64_t)1 << 24)) return DPPO_ERR_SHAPE;
  if (o.dlogits_dtype != DPPO_DLOGITS_SAME && o.dlogits_dtype != DPPO_DLOGITS_F32) return DPPO_ERR_DTYPE;
  if (variant < DPPO_PREF_SIGMOID || variant > DPPO_PREF_HINGE) return DPPO_ERR_VARIANT;
  if (!(beta > 0.f) || !isfinite(beta) || !isfinite(margin) || !(label_smoothing >= 0.f && label_smoothing <= 0.5f)) return DPPO_ERR_UNSUPPORTED;
  if (label_smoothing != 0.f && variant != DPPO_PREF_SIGMOID) return DPPO_ERR_UNSUPPORTED;
  if (!loss || !cu_seqlens || (P > 0 && !reward) || (T > 0 && !logp)) return DPPO_ERR_NULL;
  if ((uintptr_t)loss % 4 || (uintptr_t)reward % 4 || (uintptr_t)logp % 4 || (uintptr_t)ref_logp % 4 || (uintptr_t)cu_seqlens % 8) return DPPO_ERR_ALIGN;
  const int out_dtype = o.dlogits_dtype == DPPO_DLOGITS_F32 ? DPPO_F32 : logits_dtype;
  rc = check_gradient(logits, T, V, logits_row_stride, logits_dtype, dlogits, dlogits_row_stride, out_dtype);
  if (rc != DPPO_OK) return rc;
  if (!workspace || (uintptr_t)workspace % 256 || workspace_bytes < dppo_preference_workspace_bytes(T, P)) return DPPO_ERR_WORKSPACE;
  char* ws = reinterpret_cast<char*>(workspace);
  double* lse = reinterpret_cast<double*>(ws);
  double* ratio = reinterpret_cast<double*>(ws += up256((size_t)T * 8));
  float* coef = reinterpret_cast<float*>(ws += up256((size_t)T * 8));
  double* seq = reinterpret_cast<double*>(ws += up256((size_t)T * 4));
  int64_t* seq_n = reinterpret_cast<int64_t*>(ws += up256((size_t)P * 16));
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (T > 0) {
    LogpParams p = {};
    p.z = logits; p.T = T; p.V = V; p.ld = logits_row_stride; p.ids = sampled_ids; p.token_mask = token_mask;
    p.logp = logp; p.lse = lse; p.status = status; p.cu = cu_seqlens; p.P = P; p.ref_logp = ref_logp; p.ratio = ratio; p.coef = coef;
    if (launch_logp(p, logits_dtype, st) != cudaSuccess) return DPPO_ERR_CUDA;
  }
  PairParams q = {};
  q.T = T; q.P = P; q.cu = cu_seqlens; q.token_mask = token_mask; q.ratio = ratio; q.seq = seq; q.seq_n = seq_n; q.coef = coef;
  q.variant = variant; q.average = average; q.beta = beta; q.smoothing = label_smoothing; q.margin = margin; q.loss_scale = o.loss_scale;
  q.loss = loss; q.reward = reward; q.status = status;
  preference_pairs_kernel<<<1, kPairThreads, 0, st>>>(q);
  if (cudaGetLastError() != cudaSuccess) return DPPO_ERR_CUDA;
  if (T > 0) {
    GradParams g = {};
    g.z = logits; g.T = T; g.V = V; g.ld = logits_row_stride; g.ld_out = dlogits_row_stride; g.ids = sampled_ids; g.token_mask = token_mask;
    g.lse = lse; g.coef = coef; g.dz = dlogits; g.status = status; g.backwards = 1;
    if (launch_grad(g, logits_dtype, out_dtype, st) != cudaSuccess) return DPPO_ERR_CUDA;
  }
  return DPPO_OK;
}
