// Drawing tokens from rows of logits: temperature, top-k, top-p and min-p, from one given uniform number per row, with the
// record that the loss entry points read (sampled id, log mu of it, the top-K ids and probabilities).
//
// For a row z with temperature tau the weights are w_j = exp((z_j - max z) / tau).  In the order "logit descending, id
// ascending" the kept tokens are a prefix: the first top_k; of those the shortest prefix that holds top_p of their mass; of
// those the ones with w_j >= min_p.  The token drawn is the lowest id whose running sum of kept weights, taken in the order
// of the ids, exceeds u times their total.  Every choice is therefore a threshold in one order and a search in the other,
// and no row is ever sorted.
//
// Sums are kept in 64 bits and the exponentials are good to about 1e-12.  A drawn id differs from the exact one where u
// falls within the error d of the running sum of a boundary between two tokens, which happens in about 2 d V of the rows:
// at V = 151936 with fp32 (d near 1e-8) in one row of a few hundred, with this arithmetic in one of several millions.
//
// One cluster of CTAs (one CTA when there are many rows) per row.
//   pass A    every warp takes chunks of the row: maximum of each lane's elements (the lane's "group"), maximum and, where
//             the row needs its whole mass, sum of weights of the chunk, all left in the leader CTA's shared memory.
//   list      the kk-th largest group maximum bounds the kk-th largest element from below, and only the few groups whose
//             maximum reaches it can hold one of the kk largest: those groups alone are read again, and what passes the bound
//             is sorted in shared memory.  This is all that top-k and the top-K record need.
//   search    for cuts that lie below the list (top-p over a broad row, top_k > 1024): a histogram of the row over steps of 1/32
//             octave of weight tells where the cut should be; a second pass sums exactly what lies above that neighbourhood and
//             lists what lies in it.  Where that misses, or thousands of equal logits meet the cut, the cut is bracketed by passes
//             with three pivots at a time until it is found.
//   draw      inside the list, or, when the kept set is larger, in the one chunk that the running sum of the chunks' sums
//             points to.
//
// Bounded by issue slots in the passes that sum: 8 operations in 64 bits an element (t, its rounding, the remainder, four for the
// polynomial, the sum), each of which takes a scheduler two cycles, and about 16 others: some 35 cycles for 32 elements, 3.7
// elements a cycle and SM, where HBM delivers about 12 in bf16.  The leader's phases after pass A (list, sort, draw) are latency,
// hidden behind another row's pass where an SM has two rows.
//
// Measured on B200 (V = 151936): 2048 rows bf16 at tau = 1 with a record of 64: 449 us = 1.39 TB/s of logits (95 us would be HBM's
// time); 61 rows with all four settings mixed: 82 us; 256 fp32 rows of 50257 with top-p 0.9: 86 us; one row with top-k 50: 12 us.
// 2048 rows with top-k 50, which need no sums over the row: 203 us = 3.1 TB/s.
#include <cooperative_groups.h>
#include <float.h>
#include <limits.h>

#include "dppo_common.cuh"
#include "dppo_pipe.cuh"

namespace dppo {
namespace {

namespace cg = cooperative_groups;

constexpr int kSWarps = 16;             // most warps of a CTA
constexpr int kSMaxChunks = 256;       // chunks of a row; a longer row has longer chunks
constexpr int kSList = 4096;           // entries of the sorted list
constexpr int kSMaxTop = DPPO_SAMPLE_MAX_TOPK;      // largest list that is asked for
constexpr int kSProbe = 256;           // list length tried first for top-p / min-p alone
constexpr int kSMaxCluster = 8;
constexpr unsigned long long kFixOne = 1ull << 51;        // weight 1 in the fixed-point sums by chunk: all of a list may lie in one chunk
static_assert(kSList <= ~0ull / kFixOne, "the list's weights, 1 each at most, add up in 64 bits");
constexpr double kLog2eD = 1.4426950408889634074;

struct SampleParams {
  const void* logits;
  int64_t V, ld;
  const double* uniform;
  const float *temperature, *top_p, *min_p;
  const int32_t* top_k;
  const uint8_t* token_mask;
  int K;
  int vecs;              // 16-byte vectors per lane and chunk
  int32_t* ids;
  float* logp;
  int32_t* topk_ids;
  float* topk_p;
  int32_t* status;
};

enum { OP_DONE = 0, OP_PIVOTS, OP_COMPACT, OP_EQUAL, OP_CDF, OP_HIST, OP_SPLIT };
constexpr int kSBins = 2048;           // histogram: steps of 1/32 octave of weight below the maximum, 64 octaves
struct Cmd {
  int op;
  uint32_t lo, hi;       // OP_COMPACT: keys [lo, hi)
  float v[3];            // OP_PIVOTS: ascending; OP_EQUAL, OP_CDF: v[0]; OP_SPLIT: summed from v[0] up, listed from v[1] up to it; OP_HIST:
  int tie;               // counted below v[0] and tie (as in a Cut)
};

struct SampleSmem {
  double csum[kSMaxChunks];
  double cref[kSMaxChunks];               // pass A: log2 of what the chunk's sum is relative to; NaN: relative to its maximum
  double red[kSWarps];
  double mass[kSMaxCluster][3];           // OP_PIVOTS results of the cluster's CTAs
  unsigned long long cnt[kSMaxCluster][3];
  double wmass[kSWarps][3];
  unsigned wcnt[kSWarps][3];
  unsigned long long list[kSList];
  union {
    float gmax[kSMaxChunks * 32];         // until the list is made
    double pref[kSList];                  // then: running sums along the list
  };
  unsigned long long cfix[kSMaxChunks];   // kept weights of listed elements by chunk, in units of 1 / kFixOne
  alignas(16) unsigned bins[kSBins];
  float cmax[kSMaxChunks];
  float rec_z[kSMaxTop];
  int rec_id[kSMaxTop];
  Cmd cmd;
  int wsum[kSWarps];
  int n_list;
  int pick;
  double dval;
};

// order-preserving keys of floats (+0 and -0 the same)
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k); }
constexpr uint32_t kKeyNegInf = 0x007fffffu, kKeyInf = 0xff800000u;

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// warp maximum; a NaN anywhere gives a NaN (canonical NaNs are positive and lie above +inf in integer order)
__device__ __forceinline__ float warp_max_nan(float v) {
  const int b = __float_as_int(v);
  const int m = __reduce_max_sync(0xffffffffu, b >= 0 ? b : b ^ 0x7fffffff);
  return __int_as_float(m >= 0 ? m : m ^ 0x7fffffff);
}

// 2^(z c - R) for -1020 <= z c - R <= 1000: = 2^(n>>5) 2^((n & 31)/32) 2^f with n the nearest integer to 32 (z c - R) and |f| <= 1/64.
// R is a multiple of 1/32, so that the addition of a large constant that finds n can subtract R in the same step.  2^f by
// its Taylor polynomial of degree 4 (the next term is below 1.3e-12); 2^(i/32) is held by lane i of the warp (a table in shared
// memory would be read with bank conflicts).  All lanes of the warp have to take part.
struct Exp2 {
  static constexpr double kMagic = 6755399441055744.0 / 32.0;       // 1.5 2^52 / 32: adding it rounds to multiples of 1/32
  double c, K, off;          // K = kMagic - R; where |max c| reaches 2^30, R = 0 and z - off takes z's place;
                             // FAR = false leaves out the subtraction and is for off = 0 only
  __device__ __forceinline__ void set(double c_, double ref, bool& far, double& log2_ref) {
    c = c_;
    far = !(fabs(ref * c_) < 1073741824.0);
    off = far ? ref : 0.0;
    const double R = far ? 0.0 : (fma(ref, c_, kMagic) - kMagic);
    K = kMagic - R;
    log2_ref = R;
  }
  // The same for a group of G logits at once, weight = q * s: step by step for all of them, because one chain of dependent 64-bit
  // operations leaves the units idle most of the time.
  template <bool FAR, int G> __device__ __forceinline__ void group(const float* z, int tab_hi, int tab_lo, double* q, double* s) const {
    double f[G];
    int n[G];
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const double x = FAR ? (double)z[i] - off : (double)z[i];
      const double t = fma(x, c, K);
      f[i] = fma(x, c, -(t - K));
      n[i] = __double2loint(t);
    }
#pragma unroll
    for (int i = 0; i < G; ++i) q[i] = fma(f[i], 9.6181291076284772e-3, 5.5504108664821580e-2);     // ln2^4 / 24, ln2^3 / 6
#pragma unroll
    for (int i = 0; i < G; ++i) q[i] = fma(q[i], f[i], 2.4022650695910071e-1);                     // ln2^2 / 2
#pragma unroll
    for (int i = 0; i < G; ++i) q[i] = fma(q[i], f[i], 6.9314718055994531e-1);
#pragma unroll
    for (int i = 0; i < G; ++i) q[i] = fma(q[i], f[i], 1.0);
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const int hi = __shfl_sync(0xffffffffu, tab_hi, n[i]), lo = __shfl_sync(0xffffffffu, tab_lo, n[i]);
      s[i] = __hiloint2double(hi + ((n[i] & ~31) << 15), lo);
    }
  }
  template <bool FAR> __device__ __forceinline__ void parts(float z, int tab_hi, int tab_lo, double& q, double& s) const {
    group<FAR, 1>(&z, tab_hi, tab_lo, &q, &s);
  }
  // sum[i] += weight of z[i], add_group
  template <bool FAR, int G, typename F> __device__ __forceinline__ void add_group(const float* z, int tab_hi, int tab_lo, double* sum, F take) const {
    double q[G], s[G];
    group<FAR, G>(z, tab_hi, tab_lo, q, s);
#pragma unroll
    for (int i = 0; i < G; ++i) if (take(i)) sum[i] = fma(q[i], s[i], sum[i]);
  }
};

template <typename T> struct Row;
template <> struct Row<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& v, float* z) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { z[2 * i] = __uint_as_float(w[i] << 16); z[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  static __device__ __forceinline__ uint32_t bits(const void* p, int64_t j) { return reinterpret_cast<const unsigned short*>(p)[j]; }
  static __device__ __forceinline__ float at(const void* p, int64_t j) { return __uint_as_float(bits(p, j) << 16); }
  static __device__ __forceinline__ void put(uint4& v, int e, uint32_t b) {
    uint32_t* w = &v.x;
    w[e >> 1] = (e & 1) ? ((w[e >> 1] & 0xffffu) | (b << 16)) : ((w[e >> 1] & 0xffff0000u) | b);
  }
  static constexpr uint32_t kFill = 0xff80ff80u;      // -inf twice
  static __device__ __forceinline__ float max_of(const uint4& v) {
    auto h = [](uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); };
    const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(h(v.x), h(v.y)), __hmax2_nan(h(v.z), h(v.w)));
    return max_nan(__low2float(m), __high2float(m));
  }
};
template <> struct Row<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& v, float* z) {
    z[0] = __uint_as_float(v.x); z[1] = __uint_as_float(v.y); z[2] = __uint_as_float(v.z); z[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint32_t bits(const void* p, int64_t j) { return reinterpret_cast<const uint32_t*>(p)[j]; }
  static __device__ __forceinline__ float at(const void* p, int64_t j) { return __uint_as_float(bits(p, j)); }
  static __device__ __forceinline__ void put(uint4& v, int e, uint32_t b) { (&v.x)[e] = b; }
  static constexpr uint32_t kFill = 0xff800000u;
  static __device__ __forceinline__ float max_of(const uint4& v) {
    return max_nan(max_nan(__uint_as_float(v.x), __uint_as_float(v.y)), max_nan(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
};

// One row as 16-byte vectors: vector s holds the elements [s N - head, s N - head + N), head = elements between the 16-byte
// boundary below the row's first element and that element.  Whole vectors are loaded as such; the first and the last may
// be partial and are put together element by element, with -inf outside the row.
template <typename T> struct RowView {
  const T* row;
  int V, head, nvec;
  __device__ __forceinline__ uint4 load(int s) const {
    const int64_t j = (int64_t)s * Row<T>::N - head;
    if (j >= 0 && j + Row<T>::N <= V) return __ldg(reinterpret_cast<const uint4*>(row + j));
    uint4 v = make_uint4(Row<T>::kFill, Row<T>::kFill, Row<T>::kFill, Row<T>::kFill);
    if (s < nvec) {
#pragma unroll
      for (int e = 0; e < Row<T>::N; ++e)
        if (j + e >= 0 && j + e < V) Row<T>::put(v, e, Row<T>::bits(row, j + e));
    }
    return v;
  }
};

struct Cut { float z; int tie; };         // keeps z_j > z, and z_j == z with j <= tie
__device__ __forceinline__ bool kept(const Cut& c, float z, int j) { return z > c.z || (z == c.z && j <= c.tie); }
__device__ __forceinline__ Cut tighter(const Cut& a, const Cut& b) {
  if (a.z != b.z) return a.z > b.z ? a : b;
  return a.tie < b.tie ? a : b;
}

template <typename T, int NT>             // NT: threads of a CTA
struct Worker {
  static constexpr int NW = NT / 32;
  const SampleParams& p;
  SampleSmem& s;
  RowView<T> row;
  int nchunks, c_begin, c_end;             // chunks of the row, and those of this CTA
  int rank, C;
  double c;                                // log2(e) / tau
  double itau;                             // 1 / tau
  double span;                             // 1000 / c: logits further below a maximum weigh less than 2^-1000 of it
  int tab_hi, tab_lo;                      // 2^(lane/32)
  double M;                                // row maximum (known after pass A)
  Exp2 eM;                                 // weights relative to (nearly) M; corr makes them relative to M
  bool far;
  double corr;
  static constexpr int N = Row<T>::N, kGroup = 4;

  __device__ __forceinline__ int tid() const { return threadIdx.x; }
  __device__ __forceinline__ int lane() const { return threadIdx.x & 31; }
  __device__ __forceinline__ int warp() const { return threadIdx.x >> 5; }
  __device__ __forceinline__ SampleSmem* smem_of(int r) const {
    return C == 1 ? &s : cg::this_cluster().map_shared_rank(&s, r);
  }
  __device__ __forceinline__ void csync() const {
    if (C == 1) __syncthreads(); else cg::this_cluster().sync();
  }
  __device__ __forceinline__ double weight(float z) const { return exp(((double)z - M) * itau); }
  // smallest float whose weight relative to `ref` is worth counting (2^-1000 and more)
  __device__ __forceinline__ float low_of(double ref) const { return __double2float_ru(ref - span); }
  __device__ __forceinline__ void set_max(double m) {
    M = m;
    double R;
    eM.set(c, m, far, R);
    corr = far ? 1.0 : exp2(fma(-m, c, R));
  }

  // f(4 vectors, vector index of the first) over this lane's part of chunk ch, up to four vectors at a time; absent ones are -inf
  template <typename F> __device__ __forceinline__ void vectors(int ch, F f) const {
    const int s0 = ch * p.vecs * 32;
    // whole vectors throughout: no bounds to look at
    const bool inside = (int64_t)s0 * N >= row.head && (int64_t)(s0 + p.vecs * 32) * N - row.head <= row.V;
    const uint4 none = make_uint4(Row<T>::kFill, Row<T>::kFill, Row<T>::kFill, Row<T>::kFill);
    for (int i = 0; i < p.vecs; i += 4) {
      uint4 v[4];
      if (inside) {
        const uint4* src = reinterpret_cast<const uint4*>(row.row + ((int64_t)(s0 + i * 32 + lane()) * N - row.head));
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = i + k < p.vecs ? __ldg(src + k * 32) : none;
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = i + k < p.vecs ? row.load(s0 + (i + k) * 32 + lane()) : none;
      }
      f(v, s0 + i * 32 + lane(), min(4, p.vecs - i));
    }
  }
  // f(z, element index) over this lane's part of chunk ch
  template <typename F> __device__ __forceinline__ void each(int ch, F f) const {
    vectors(ch, [&](const uint4* v, int s0, int n) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (k >= n) break;
        float z[N];
        Row<T>::unpack(v[k], z);
        const int j0 = (s0 + k * 32) * N - row.head;
#pragma unroll
        for (int e = 0; e < N; ++e) f(z[e], j0 + e);
      }
    });
  }
  // sum of 2^(z c - R) over the elements of chunk ch.  Those below `low` count as `low`, less than 2^-800: where |max c| < 2^30 a float's
  // steps are less than 128 octaves.  Where that fails (far from zero, because `low` may round up to the maximum; where temperature is so
  // high that `low` would lie below all floats, because -inf must not count as one) EXACT leaves them out.
  template <bool EXACT> __device__ __forceinline__ double weigh_all(int ch, const Exp2& x, float low) const {
    double sum = 0.0;
    vectors(ch, [&](const uint4* v, int, int n) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (k >= n) break;
        float z[N];
        Row<T>::unpack(v[k], z);
#pragma unroll
        for (int e = 0; e < N; ++e) {
          double q, w;
          x.parts<EXACT>(fmaxf(z[e], low), tab_hi, tab_lo, q, w);
          if (!EXACT || z[e] >= low) sum = fma(q, w, sum);
        }
      }
    });
    return warp_sum(sum);
  }
  // sum over the elements that are worth counting and for which take(z, index) holds
  template <typename F> __device__ __forceinline__ double weigh(int ch, const Exp2& x, float low, F take) const {
    double sums[kGroup] = {};
    vectors(ch, [&](const uint4* v, int s0, int n) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (k >= n) break;
        float z[N], y[N];
        Row<T>::unpack(v[k], z);
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = fmaxf(z[e], low);
        const int j0 = (s0 + k * 32) * N - row.head;
#pragma unroll
        for (int e = 0; e < N; e += kGroup)
          x.template add_group<true, kGroup>(y + e, tab_hi, tab_lo, sums, [&](int i) { return take(z[e + i], j0 + e + i) && z[e + i] >= low; });
      }
    });
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kGroup; ++i) sum += sums[i];
    return warp_sum(sum);
  }
  // the same and the counts above three borders at once
  __device__ __forceinline__ void weigh3(int ch, float low, const float* border, double* sum, unsigned* n) const {
    double a[3] = {0, 0, 0};
    unsigned b[3] = {0, 0, 0};
    each(ch, [&](float z, int) {
      double q, w;
      eM.parts<true>(fmaxf(z, low), tab_hi, tab_lo, q, w);
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (z >= border[i]) { ++b[i]; if (z >= low) a[i] = fma(q, w, a[i]); }
    });
#pragma unroll
    for (int i = 0; i < 3; ++i) { sum[i] = warp_sum(a[i]); n[i] += __reduce_add_sync(0xffffffffu, b[i]); }
  }

  // ---- pass A ----
  __device__ void pass_a(bool want_sum, bool want_groups) const {
    SampleSmem* lead = smem_of(0);
    // Sums are of 2^(z c) as it stands where 2^(max z c) is well inside the range of doubles, so that maximum and sum come from one
    // look at the elements; what lies below 2^-900 then counts as 2^-900.  Otherwise (set apart after the maximum is known) the
    // chunk is summed relative to its maximum.
    Exp2 plain;
    bool far0;
    double zero;
    plain.set(c, 0.0, far0, zero);
    const float floor0 = __double2float_ru(-0.9 * span), safe = floor0 > -FLT_MAX ? (float)(0.8 * span) : -1.f;
    for (int ch = c_begin + warp(); ch < c_end; ch += NW) {
      float mx = -INFINITY;
      double sum = 0.0, ref = 0.0, sums[kGroup] = {};
      if (want_sum) {
        vectors(ch, [&](const uint4* v, int, int n) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (k >= n) break;
            mx = max_nan(mx, Row<T>::max_of(v[k]));
            float z[N];
            Row<T>::unpack(v[k], z);
#pragma unroll
            for (int e = 0; e < N; ++e) z[e] = fmaxf(z[e], floor0);
#pragma unroll
            for (int e = 0; e < N; e += kGroup) plain.add_group<false, kGroup>(z + e, tab_hi, tab_lo, sums, [](int) { return true; });
          }
        });
      } else {
        vectors(ch, [&](const uint4* v, int, int n) {
#pragma unroll
          for (int k = 0; k < 4; ++k) if (k < n) mx = max_nan(mx, Row<T>::max_of(v[k]));
        });
      }
      if (want_groups) lead->gmax[ch * 32 + lane()] = mx;
      const float cm = warp_max_nan(mx);
      if (want_sum) {
        if (fabsf(cm) < safe) {
#pragma unroll
          for (int i = 0; i < kGroup; ++i) sum += sums[i];
          sum = warp_sum(sum);
        } else if (cm > -INFINITY && cm < INFINITY) {
          Exp2 x;
          bool far_ch;
          x.set(c, (double)cm, far_ch, ref);
          const float low = low_of((double)cm);
          sum = far_ch || low == -FLT_MAX ? weigh_all<true>(ch, x, low) : weigh_all<false>(ch, x, low);
          if (far_ch) ref = NAN;
        } else {
          sum = 0.0;
        }
      }
      if (lane() == 0) { lead->cmax[ch] = cm; lead->csum[ch] = sum; lead->cref[ch] = ref; }
    }
  }

  // which step of 1/32 octave of weight below the maximum (a monotone function of z)
  __device__ __forceinline__ int bin_of(float z, float scale) const { return (int)fmaxf(0.f, fminf(((float)M - z) * scale, (float)(kSBins - 1))); }
  // smallest float (above -inf) that falls into a bin below b; +inf if there is none
  __device__ float border(int b) const {
    uint32_t lo = kKeyNegInf, hi = kKeyInf;              // bin_of(lo) >= b (or lo = -inf), bin_of(hi) < b (or hi = inf)
    while (hi - lo > 1) {
      const uint32_t mid = lo + (hi - lo) / 2;
      if (bin_of(of_key(mid), bin_scale()) < b) hi = mid; else lo = mid;
    }
    return of_key(hi);
  }
  __device__ __forceinline__ float bin_scale() const { return (float)(32.0 * c); }

  // ---- passes that the leader asks for ----
  __device__ void execute(const Cmd& k) const {
    SampleSmem* lead = smem_of(0);
    const float low = low_of(M);
    if (k.op == OP_PIVOTS || k.op == OP_SPLIT) {
      // masses and counts above three borders; OP_SPLIT: above one, chunk sums too, and a list of what reaches a second one
      double m[3] = {0, 0, 0};
      unsigned n[3] = {0, 0, 0};
      for (int ch = c_begin + warp(); ch < c_end; ch += NW) {
        if (k.op == OP_PIVOTS) {
          double one[3];
          weigh3(ch, low, k.v, one, n);
#pragma unroll
          for (int i = 0; i < 3; ++i) m[i] += one[i];
        } else {
          unsigned cnt = 0;
          auto above = [&](float z, int j) {
            const bool top = z >= k.v[0];
            if (z >= k.v[1] && !top) {
              const int at = atomicAdd(&lead->n_list, 1);
              if (at < kSList) lead->list[at] = ((unsigned long long)~key_of(z) << 32) | (uint32_t)j;
            }
            cnt += top;
            return top;
          };
          const double sum = corr * weigh(ch, eM, low, above);
          if (lane() == 0) lead->csum[ch] = sum;
          m[0] += sum;
          n[0] += __reduce_add_sync(0xffffffffu, cnt);
        }
      }
      // (every lane holds its warp's totals)
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (lane() == 0) { s.wmass[warp()][i] = k.op == OP_PIVOTS ? corr * m[i] : m[i]; s.wcnt[warp()][i] = n[i]; }
      __syncthreads();
      if (tid() < 3) {
        double a = 0.0;
        unsigned long long b = 0;
        for (int w = 0; w < NW; ++w) { a += s.wmass[w][tid()]; b += s.wcnt[w][tid()]; }
        lead->mass[rank][tid()] = a;
        lead->cnt[rank][tid()] = b;
      }
    } else if (k.op == OP_COMPACT) {
      for (int ch = c_begin + warp(); ch < c_end; ch += NW)
        each(ch, [&](float z, int j) {
          const uint32_t key = key_of(z);
          if (key >= k.lo && key < k.hi) {
            const int at = atomicAdd(&lead->n_list, 1);
            if (at < kSList) lead->list[at] = ((unsigned long long)~key << 32) | (uint32_t)j;
          }
        });
    } else if (k.op == OP_EQUAL) {
      for (int ch = c_begin + warp(); ch < c_end; ch += NW) {
        unsigned n = 0;
        each(ch, [&](float z, int) { n += (z == k.v[0]); });
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane() == 0) lead->csum[ch] = (double)n;
      }
    } else if (k.op == OP_CDF) {
      const Cut cut = {k.v[0], k.tie};
      auto take = [&](float z, int j) { return kept(cut, z, j); };
      for (int ch = c_begin + warp(); ch < c_end; ch += NW) {
        const double sum = corr * weigh(ch, eM, low, take);
        if (lane() == 0) lead->csum[ch] = sum;
      }
    } else if (k.op == OP_HIST) {
      for (int i = tid(); i < kSBins; i += NT) s.bins[i] = 0;
      __syncthreads();
      const float scale = bin_scale();
      for (int ch = c_begin + warp(); ch < c_end; ch += NW)
        each(ch, [&](float z, int j) {
          const int b = z > -INFINITY ? bin_of(z, scale) : kSBins - 1;
          if (b < kSBins - 1 && !(z > k.v[0] || (z == k.v[0] && j <= k.tie))) atomicAdd(&s.bins[b], 1u);       // (the last step takes all that is 64 octaves down and is not looked at)
        });
      __syncthreads();
    }
  }
  // Leader: hands a command to every CTA of the cluster and takes part; returns when all are done.
  __device__ void issue(const Cmd& k) const {
    __syncthreads();
    if (tid() < C) smem_of(tid())->cmd = k;
    csync();
    if (k.op == OP_DONE) return;
    execute(k);
    csync();
  }

  // ---- leader only, all threads ----
  // exclusive prefix sum over the threads; total in every thread
  __device__ double block_scan(double v, double& total) const {
    double inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const double x = __shfl_up_sync(0xffffffffu, inc, o); if (lane() >= o) inc += x; }
    __syncthreads();
    if (lane() == 31) s.red[warp()] = inc;
    __syncthreads();
    double before = 0.0, all = 0.0;
    for (int w = 0; w < NW; ++w) { if (w < warp()) before += s.red[w]; all += s.red[w]; }
    total = all;
    return before + (inc - v);
  }
  __device__ int block_min(int v) const {
    __syncthreads();
    if (tid() == 0) s.pick = INT_MAX;
    __syncthreads();
    v = __reduce_min_sync(0xffffffffu, v);
    if (lane() == 0) atomicMin(&s.pick, v);
    __syncthreads();
    return s.pick;
  }
  __device__ int block_count(int v) const {
    v = __reduce_add_sync(0xffffffffu, v);
    __syncthreads();                       // (the last call's sums have been read)
    if (lane() == 0) s.wsum[warp()] = v;
    __syncthreads();
    return __reduce_add_sync(0xffffffffu, lane() < NW ? s.wsum[lane()] : 0);
  }
  // ascending sort of list[0, n): logits descending, ids ascending
  __device__ void sort_list(int n) const {
    if (n <= NT) {                  // by rank: every entry counts those before it (all entries differ)
      const unsigned long long mine = tid() < n ? s.list[tid()] : 0;
      int r = 0;
      if (tid() < n) {
#pragma unroll 16
        for (int j = 0; j < n; ++j) r += s.list[j] < mine ? 1 : 0;
      }
      __syncthreads();
      if (tid() < n) s.list[r] = mine;
      __syncthreads();
      return;
    }
    int P = 32;
    while (P < n) P <<= 1;
    for (int i = n + tid(); i < P; i += NT) s.list[i] = ~0ull;
    __syncthreads();
    for (int k = 2; k <= P; k <<= 1)
      for (int j = k >> 1; j > 0; j >>= 1) {
        for (int t = tid(); t < P / 2; t += NT) {
          const int i = ((t & ~(j - 1)) << 1) | (t & (j - 1)), l = i | j;
          const unsigned long long a = s.list[i], b = s.list[l];
          if ((a > b) == ((i & k) == 0)) { s.list[i] = b; s.list[l] = a; }
        }
        __syncthreads();
      }
  }
  __device__ __forceinline__ float list_z(int i) const { return of_key(~(uint32_t)(s.list[i] >> 32)); }
  __device__ __forceinline__ int list_id(int i) const { return (int)(uint32_t)s.list[i]; }
  // pref[i] = sum of the first i + 1 weights of the list's first n entries
  __device__ double list_prefix(int n) const {
    const int per = (n + NT - 1) / NT, b = tid() * per, e = min(n, b + per);
    double v = 0.0;
    for (int i = b; i < e; ++i) { v += weight(list_z(i)); s.pref[i] = v; }
    double total;
    const double run = block_scan(v, total);
    for (int i = b; i < e; ++i) s.pref[i] += run;
    __syncthreads();
    return n > 0 ? s.pref[n - 1] : 0.0;
  }
  // the list's entries [0, n) in the order of their ids: lowest id whose running sum exceeds target
  __device__ int draw_from_list(int n, double u) const {
    const double target = u * s.pref[n - 1];
    int best = INT_MAX, last = -1;
    // (entries that weigh less than 2^-1000 come last in the list and are not drawn: rounding in pref may give them a step)
    const float low = low_of(M);
    int worth = 0;
    for (int i = tid(); i < n; i += NT) worth += list_z(i) >= low;
    n = block_count(worth);
    if (n <= NT / 2) {
      if (tid() < n) {
        const int me = list_id(tid());
        double run = 0.0;
        double before = 0.0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) { const double at = s.pref[j]; if (list_id(j) <= me) run += at - before; before = at; }
        if (run > target) best = me;
        last = me;
      }
    } else {
      __syncthreads();
      // turned round in place: ids in front, position in the list (for the weight) behind
      for (int i = tid(); i < n; i += NT) s.list[i] = ((unsigned long long)(uint32_t)list_id(i) << 32) | (uint32_t)i;
      __syncthreads();
      sort_list(n);
      const int per = (n + NT - 1) / NT, b = tid() * per, e = min(n, b + per);
      double v = 0.0;
      for (int i = b; i < e; ++i) { const int j = (int)(uint32_t)s.list[i]; v += s.pref[j] - (j ? s.pref[j - 1] : 0.0); }
      double total;
      double run = block_scan(v, total);
      for (int i = b; i < e; ++i) {
        const int j = (int)(uint32_t)s.list[i];
        run += s.pref[j] - (j ? s.pref[j - 1] : 0.0);
        last = (int)(s.list[i] >> 32);
        if (run > target) { best = last; break; }
      }
    }
    best = block_min(best);
    return best != INT_MAX ? best : -block_min(-last);         // rounding at the far end: the last one
  }
  // first chunk whose running sum of csum exceeds target, and the sum before it; the last non-empty one if there is none
  __device__ int find_chunk(double target, double& before) const {
    const double v = tid() < nchunks ? s.csum[tid()] : 0.0;
    double total;
    const double ex = block_scan(v, total);
    int ch = block_min((v > 0.0 && ex + v > target) ? tid() : INT_MAX);
    if (ch == INT_MAX) ch = -block_min(v > 0.0 ? -tid() : 0);
    if (tid() == ch) s.dval = ex;
    __syncthreads();
    before = s.dval;
    return ch;
  }
  // lowest element of chunk ch at which before + running sum of w(z, j) exceeds target; the last one with w > 0 otherwise.  A vector
  // per thread.  (w is evaluated by whole warps.)
  template <typename F> __device__ int find_in_chunk(int ch, double before, double target, F w) const {
    int best = INT_MAX, last = -1;
    double run = before;
    for (int v0 = 0; v0 < p.vecs * 32; v0 += NT) {
      const int sv = ch * p.vecs * 32 + v0 + tid();
      const uint4 none = make_uint4(Row<T>::kFill, Row<T>::kFill, Row<T>::kFill, Row<T>::kFill);
      const uint4 v = v0 + tid() < p.vecs * 32 ? row.load(sv) : none;
      float z[N];
      Row<T>::unpack(v, z);
      const int j0 = sv * N - row.head;
      double x[N], mine = 0.0, total;
#pragma unroll
      for (int e = 0; e < N; ++e) { x[e] = w(z[e], j0 + e); mine += x[e]; if (x[e] > 0.0) last = j0 + e; }
      double r = run + block_scan(mine, total);
#pragma unroll
      for (int e = 0; e < N; ++e) { r += x[e]; if (best == INT_MAX && x[e] > 0.0 && r > target) best = j0 + e; }
      run += total;
    }
    best = block_min(best);
    return best != INT_MAX ? best : -block_min(-last);
  }

  // find_cut's first try: the cut's neighbourhood from a histogram, then exactly.  False if it was missed.  On success csum + cfix are
  // the chunks' sums of the prefix.
  // known: the n_known largest are listed and weigh known_mass together; the estimate is about the others.
  __device__ bool guess(bool by_mass, unsigned long long count, double target, int n_known, double known_mass, Cut& cut, double& top_mass) const {
    Cmd k = {};
    k.op = OP_HIST;
    k.v[0] = n_known > 0 ? list_z(n_known - 1) : INFINITY;
    k.tie = n_known > 0 ? list_id(n_known - 1) : 0;
    issue(k);
    // each thread some adjacent bins: counts and estimated masses in order, then the bin in which the running sum gets there
    constexpr int kPer = kSBins / NT;
    double w[kPer], sum = 0.0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int b = tid() * kPer + i;
      unsigned c_ = 0;
      for (int r = 0; r < C; ++r) c_ += smem_of(r)->bins[b];
      w[i] = by_mass ? (double)c_ * exp2(-((double)b + 0.5) / 32.0) : (double)c_;
      sum += w[i];
    }
    double total;
    double run = (by_mass ? known_mass : (double)n_known) + block_scan(sum, total);
    const double goal = by_mass ? target : (double)count;
    int at = INT_MAX;
#pragma unroll
    for (int i = 0; i < kPer; ++i) { run += w[i]; if (at == INT_MAX && w[i] > 0.0 && run >= goal) at = tid() * kPer + i; }
    at = block_min(at);
    if (at == INT_MAX) { if (!by_mass) return false; at = kSBins - 2; }
    // one bin to either side (counts are exact and need none), as far as the list holds them
    const int side = by_mass ? 1 : 0;
    k.v[0] = border(max(0, at - side));
    k.v[1] = border(min(kSBins - 1, at + side + 1));
    __syncthreads();
    if (tid() == 0) s.n_list = 0;
    k.op = OP_SPLIT;
    issue(k);
    if (s.n_list > kSList || s.n_list == 0) return false;
    const int m = s.n_list;
    double above = 0.0;
    unsigned long long n_above = 0;
    for (int r = 0; r < C; ++r) { above += s.mass[r][0]; n_above += s.cnt[r][0]; }
    sort_list(m);
    list_prefix(m);
    int pos;
    if (by_mass) {
      if ((n_above > 0 && above >= target) || above + s.pref[m - 1] < target) return false;
      int b = INT_MAX;
      for (int i = tid(); i < m; i += NT) if (above + s.pref[i] >= target) { b = i; break; }
      pos = block_min(b);
    } else {
      if (n_above >= count || n_above + (unsigned long long)m < count) return false;
      pos = (int)(count - n_above) - 1;
    }
    cut.z = list_z(pos); cut.tie = list_id(pos);
    top_mass = above + s.pref[pos];
    // the listed part of the prefix joins its chunks (integers: no order to depend on; cut off at 2^-51, the whole list's error is below
    // 2e-12 of the largest weight, which the mass holds)
    if (tid() < nchunks) s.cfix[tid()] = 0;
    __syncthreads();
    for (int i = tid(); i <= pos; i += NT)
      atomicAdd(&s.cfix[(list_id(i) + row.head) / (N * 32 * p.vecs)], (unsigned long long)(weight(list_z(i)) * (double)kFixOne));
    __syncthreads();
    if (tid() < nchunks) s.csum[tid()] += (double)s.cfix[tid()] * (1.0 / (double)kFixOne);
    __syncthreads();
    return true;
  }

  // The cut after which the kept prefix (of all finite entries, in order) has `count` tokens (by_mass false), or is the
  // shortest one with mass >= target (by_mass true).  *top_mass: mass of that prefix.  False if the whole row is kept.
  // Overwrites list, pref and csum; *summed: csum holds the prefix's chunk sums.
  __device__ bool find_cut(bool by_mass, unsigned long long count, double target, double tau, int n_known, double known_mass, Cut& cut,
                           double& top_mass, bool* summed) const {
    *summed = false;
    if (guess(by_mass, count, target, n_known, known_mass, cut, top_mass)) { *summed = true; return true; }
    uint32_t lo = kKeyNegInf + 1, hi = kKeyInf;          // crit(key >= lo) holds, crit(key >= hi) does not
    unsigned long long n_hi = 0, n_lo = ~0ull;
    double m_hi = 0.0;
    for (int it = 0;; ++it) {
      uint32_t pv[3];
      const float vlo = of_key(lo), vhi = fminf(of_key(hi), (float)M);
      if (it == 0) {
        pv[0] = lo;
        pv[1] = key_of((float)(M - 9.0 * tau));
        pv[2] = key_of((float)(M - 4.0 * tau));
      } else {
        const double a = fmax((double)vlo, M - 40.0 * tau), b = (double)vhi;
        pv[0] = lo + (hi - lo) / 2;                      // halves the keys: ends the search whatever the values are
        pv[1] = key_of((float)(a + (b - a) / 3.0));
        pv[2] = key_of((float)(a + (b - a) * (2.0 / 3.0)));
      }
#pragma unroll
      for (int i = 0; i < 3; ++i) pv[i] = max(lo + (it ? 1u : 0u), min(hi - 1, pv[i]));
      if (pv[0] > pv[1]) { const uint32_t t = pv[0]; pv[0] = pv[1]; pv[1] = t; }
      if (pv[1] > pv[2]) { const uint32_t t = pv[1]; pv[1] = pv[2]; pv[2] = t; }
      if (pv[0] > pv[1]) { const uint32_t t = pv[0]; pv[0] = pv[1]; pv[1] = t; }
      Cmd k = {};
      k.op = OP_PIVOTS;
      for (int i = 0; i < 3; ++i) k.v[i] = of_key(pv[i]);
      issue(k);
      for (int i = 2; i >= 0; --i) {                     // from the highest pivot down
        double m = 0.0;
        unsigned long long n = 0;
        for (int r = 0; r < C; ++r) { m += s.mass[r][i]; n += s.cnt[r][i]; }
        const bool holds = by_mass ? n > 0 && m >= target : n >= count;      // (a target of 0, top_p = 0, asks for one token too)
        if (holds) { lo = pv[i]; n_lo = n; break; }
        hi = pv[i]; n_hi = n; m_hi = m;
        if (it == 0 && i == 0) { top_mass = m; return false; }
      }
      if (n_lo != ~0ull && (n_lo - n_hi <= (unsigned long long)kSList || hi - lo <= 1)) break;
    }
    const unsigned long long between = n_lo - n_hi;
    if (between <= (unsigned long long)kSList) {
      __syncthreads();
      if (tid() == 0) s.n_list = 0;
      Cmd k = {};
      k.op = OP_COMPACT; k.lo = lo; k.hi = hi;
      issue(k);
      const int n = s.n_list;
      sort_list(n);
      list_prefix(n);
      int at = n - 1;
      if (by_mass) {
        int b = INT_MAX;
        for (int i = tid(); i < n; i += NT) if (m_hi + s.pref[i] >= target) { b = i; break; }
        b = block_min(b);
        if (b != INT_MAX) at = b;
      } else {
        at = (int)(count - n_hi) - 1;
      }
      cut.z = list_z(at); cut.tie = list_id(at);
      top_mass = m_hi + s.pref[at];
      __syncthreads();
      return true;
    }
    // one value, more often than the list holds: the r-th of them in the order of the ids
    const float v = of_key(lo);
    const double w = weight(v);
    double r = by_mass ? ceil((target - m_hi) / w) : (double)(count - n_hi);
    r = fmin(fmax(r, 1.0), (double)between);
    Cmd k = {};
    k.op = OP_EQUAL; k.v[0] = v;
    issue(k);
    double before;
    const int ch = find_chunk(r - 0.5, before);
    cut.z = v;
    cut.tie = find_in_chunk(ch, before, r - 0.5, [&](float z, int) { return z == v ? 1.0 : 0.0; });
    top_mass = m_hi + r * w;
    return true;
  }

  // The list: every finite element whose key reaches a bound that at least kk of them reach (all finite ones if there are
  // fewer).  False: more than the list holds.
  __device__ bool make_list(int kk) const {
    uint32_t bound = kKeyNegInf + 1;
    const int G = nchunks * 32;
    if (kk * 10 <= nchunks * 9) {
      // The kk-th largest chunk maximum: kk chunks hold an element that reaches it, and with n chunks alike about
      // -n log(1 - kk / n) elements do.  Every chunk counts those before it; their numbers, in the place of the keys' last 8 bits
      // (which the bound then lacks), keep equal ones apart.
      static_assert(kSMaxChunks <= 256, "chunk numbers of 8 bits");
      __syncthreads();
      const uint32_t me = tid() < nchunks ? (key_of(s.cmax[tid()]) & ~255u) | (uint32_t)tid() : 0u;
      if (tid() < kSMaxChunks) s.bins[tid()] = me;
      __syncthreads();
      if (tid() < nchunks) {
        int r = 0;
#pragma unroll 8
        for (int i = 0; i < nchunks; i += 4) {
          const uint4 x = *reinterpret_cast<const uint4*>(s.bins + i);
          r += (int)(x.x > me) + (int)(x.y > me) + (int)(x.z > me) + (int)(x.w > me);
        }
        if (r == kk - 1) s.pick = (int)(me & ~255u);
      }
      __syncthreads();
      bound = max(bound, (uint32_t)s.pick);
    } else if (kk < G) {
      // A bound that at least kk group maxima reach and not many more, from an interval of values [lo, hi) that is cut in three at
      // a time (of keys now and then, which ends it whatever the values are).  The lowest chunk maximum is a lower end if there
      // are kk chunks; otherwise one is looked for in growing steps.
      constexpr int kPer = kSMaxChunks * 32 / NT;
      uint32_t g[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) { const int at = tid() + i * NT; g[i] = at < G ? key_of(s.gmax[at]) : 0u; }
      float low_max = INFINITY;
      for (int ch = lane(); ch < nchunks; ch += 32) low_max = fminf(low_max, s.cmax[ch]);
      low_max = -warp_max_nan(-low_max);
      uint32_t lo = bound, hi = key_of((float)M) + 1;
      bool open = kk > nchunks;                      // lo is not known to be one
      if (!open) lo = max(lo, key_of(low_max));
      float step = (float)M - low_max;
      for (int it = 0; it < 64 && hi - lo > 1; ++it) {
        const float vl = of_key(lo), vh = of_key(hi - 1);
        uint32_t a, b;                               // lo < a <= b < hi
        if (open && step > 0.f && step < 1e30f) {
          a = key_of(vh - 3.f * step); b = key_of(vh - step);
          step *= 4.f;
        } else if (!open && (it & 7) != 7) {
          a = key_of(vl + (vh - vl) * (1.f / 3.f)); b = key_of(vl + (vh - vl) * (2.f / 3.f));
        } else {
          a = lo + (hi - lo) / 3; b = lo + (hi - lo) / 3 * 2;
        }
        a = min(max(a, lo + 1), hi - 1);
        b = min(max(b, a), hi - 1);
        int n = 0;                                   // two counts, 16 bits each
#pragma unroll
        for (int i = 0; i < kPer; ++i) n += (g[i] >= a ? 1 : 0) + (g[i] >= b ? 65536 : 0);
        n = block_count(n);
        const int na = n & 0xffff, nb = (int)((unsigned)n >> 16);
        if (nb >= kk) lo = b; else { hi = b; if (na >= kk) lo = a; else hi = a; }
        const int got = nb >= kk ? nb : na;
        if (got >= kk) { open = false; if (got <= 2 * kk + 32) break; }
      }
      bound = lo;
    }
    __syncthreads();
    if (tid() == 0) s.n_list = 0;
    __syncthreads();
    // the groups that reach the bound (their numbers take the place of sorting space), then a thread per vector of each
    int* hits = reinterpret_cast<int*>(s.bins);
    if (tid() == 0) s.pick = 0;
    __syncthreads();
    const float reach = of_key(bound);
#pragma unroll 4
    for (int g = tid(); g < G; g += NT)
      if (s.gmax[g] >= reach) { const int at = atomicAdd(&s.pick, 1); if (at < kSBins) hits[at] = g; }
    __syncthreads();
    const int n_hits = s.pick;
    if (n_hits > kSBins) return false;
    for (int i = tid(); i < n_hits * p.vecs; i += NT) {
      const int g = hits[i / p.vecs], sv = ((g >> 5) * p.vecs + i % p.vecs) * 32 + (g & 31);
      const uint4 v = row.load(sv);
      float z[N];
      Row<T>::unpack(v, z);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const uint32_t key = key_of(z[e]);
        if (key >= bound) {
          const int at = atomicAdd(&s.n_list, 1);
          if (at < kSList) s.list[at] = ((unsigned long long)~key << 32) | (uint32_t)(sv * N - row.head + e);
        }
      }
    }
    __syncthreads();
    return s.n_list <= kSList;
  }
};

// 512 threads an SM (as one CTA where CTAs share rows, as two otherwise, so that one row's end overlaps another's pass) with 128
// registers each: the 64-bit chains need several elements in flight per thread more than they need warps.
template <typename T, int NT>
__global__ void __launch_bounds__(NT, 512 / NT) dppo_sample_kernel(SampleParams p, int C) {
  constexpr int NW = NT / 32;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  SampleSmem& s = *reinterpret_cast<SampleSmem*>(smem_raw);
  const int rank = (C == 1) ? 0 : (int)cluster_ctarank();
  const int64_t t = (int64_t)(blockIdx.x / (unsigned)C);
  const int tid = threadIdx.x;

  auto drop = [&](int bit) {
    if (rank == 0) {
      if (tid == 0) { p.ids[t] = 0; p.logp[t] = 0.f; if (bit) atomicOr(p.status, bit); }
      for (int i = tid; i < p.K; i += NT) { p.topk_ids[t * p.K + i] = 0; p.topk_p[t * p.K + i] = 0.f; }
    }
  };
  if (p.token_mask && p.token_mask[t] == 0) { drop(0); return; }          // the same decision in every CTA of the cluster
  double tau = p.temperature ? (double)p.temperature[t] : 1.0;
  int64_t k = p.top_k ? (int64_t)p.top_k[t] : 0;
  const double top_p = p.top_p ? (double)p.top_p[t] : 1.0, min_p = p.min_p ? (double)p.min_p[t] : 0.0, u = p.uniform[t];
  if (!(tau >= 0.0 && tau < INFINITY) || !(top_p >= 0.0) || !(min_p >= 0.0 && min_p <= 1.0) || !(u >= 0.0 && u < 1.0)) {
    drop(DPPO_STATUS_BAD_SAMPLING);
    return;
  }
  if (tau == 0.0) { tau = 1.0; k = 1; }
  const bool k_on = k > 0 && k < p.V, small_k = k_on && k <= kSMaxTop;
  const bool p_on = top_p < 1.0, m_on = min_p > 0.0;

  const T* base = reinterpret_cast<const T*>(p.logits) + t * p.ld;
  RowView<T> row;
  row.row = base;
  row.V = (int)p.V;
  row.head = (int)(((uintptr_t)base & 15) / sizeof(T));
  row.nvec = (int)(((int64_t)row.head + p.V + Row<T>::N - 1) / Row<T>::N);
  const int nchunks = (row.nvec + 32 * p.vecs - 1) / (32 * p.vecs), per = (nchunks + C - 1) / C;
  int kk = p.K;                                      // length of the list that is asked for
  if (small_k) kk = max(kk, (int)k);
  else if (p_on || m_on) kk = max(kk, min(kSProbe, max(1, nchunks * 3 / 4)));
  Worker<T, NT> w = {p, s, row, nchunks, min(nchunks, rank * per), min(nchunks, (rank + 1) * per), rank, C, kLog2eD / tau, 1.0 / tau, 1000.0 * tau / kLog2eD};

  const double mine = exp2((double)(tid & 31) / 32.0);
  w.tab_hi = __double2hiint(mine);
  w.tab_lo = __double2loint(mine);
  if (C > 1) w.csync();                              // every CTA of the cluster runs
  w.pass_a(!small_k, kk > 0);
  w.csync();

  // row maximum, known to the leader
  SampleSmem* lead = w.smem_of(0);
  float mx = -INFINITY;
  for (int ch = threadIdx.x & 31; ch < nchunks; ch += 32) mx = max_nan(mx, lead->cmax[ch]);
  mx = warp_max_nan(mx);
  if (!(mx > -INFINITY && mx < INFINITY)) {          // a NaN, an infinity, or nothing but -inf: every CTA sees the same
    drop(DPPO_STATUS_NONFINITE_ROW);
    w.csync();                                       // the leader's shared memory was read by all
    return;
  }
  w.set_max((double)mx);
  if (rank != 0) {                                   // passes that the leader asks for, until it is done
    for (;;) {
      w.csync();
      const Cmd cmd = s.cmd;
      if (cmd.op == OP_DONE) return;
      w.execute(cmd);
      w.csync();
    }
  }
  __syncthreads();

  double W = 0.0;                                    // mass of the kept tokens
  if (!small_k) {
    // chunk sums relative to the row maximum, and the whole mass
    double v = 0.0;
    if (tid < nchunks) {
      const double ref = s.cref[tid];                // (NaN: relative to the chunk's maximum)
      // (a chunk without an element worth counting has no mass, so that no chunk is chosen in which nothing can be drawn)
      if (s.cmax[tid] >= w.low_of(w.M)) v = s.csum[tid] * (ref == ref ? exp2(fma(-w.M, w.c, ref)) : exp(((double)s.cmax[tid] - w.M) * w.itau));
      s.csum[tid] = v;
    }
    w.block_scan(v, W);
    __syncthreads();
  }
  Cut cut = {-INFINITY, -1};
  bool cut_on = false, in_list = false;              // in_list: the kept tokens are the list's first n
  int n = 0, n_list = 0, n_rec = 0;
  if (kk > 0) {
    if (!w.make_list(kk)) {
      // ties or an order that puts thousands of the largest into few groups: the exact cut of the kk largest
      Cut kc = {-INFINITY, -1};
      double dummy;
      bool summed;
      w.find_cut(false, (unsigned long long)kk, 0.0, tau, 0, 0.0, kc, dummy, &summed);
      // the kk entries themselves
      __syncthreads();
      if (tid == 0) s.n_list = 0;
      Cmd cmd = {};
      cmd.op = OP_COMPACT; cmd.lo = key_of(kc.z) + 1; cmd.hi = kKeyInf;
      w.issue(cmd);
      // of the value at the cut the ones up to its tie, by a walk over the leader's view of the row
      for (int ch = tid >> 5; ch < nchunks; ch += NW)
        w.each(ch, [&](float z, int j) {
          if (z == kc.z && j <= kc.tie) {
            const int at = atomicAdd(&s.n_list, 1);
            if (at < kSList) s.list[at] = ((unsigned long long)~key_of(z) << 32) | (uint32_t)j;
          }
        });
      __syncthreads();
      if (!small_k) {                                // the search used csum: whole sums again
        Cmd all = {};
        all.op = OP_CDF; all.v[0] = -INFINITY; all.tie = -1;
        w.issue(all);
      }
    }
    n_list = s.n_list;
    w.sort_list(n_list);
    n_rec = min(n_list, p.K);
    for (int i = tid; i < n_rec; i += NT) { s.rec_z[i] = w.list_z(i); s.rec_id[i] = w.list_id(i); }
    if (small_k || p_on || m_on) {
      if (small_k) n_list = min(n_list, (int)k);
      const double total = w.list_prefix(n_list);
      if (small_k) W = total;
      n = n_list;
      in_list = small_k;
      // (top_p counts within the top_k: with a top_k beyond the list their mass has to be found first, below)
      if (!(k_on && !small_k && p_on)) {
        if (p_on) {
          const double target = top_p * W;
          int b = INT_MAX;
          for (int i = tid; i < n_list; i += NT) if (s.pref[i] >= target) { b = i; break; }
          b = w.block_min(b);
          if (b != INT_MAX) { n = min(n, b + 1); in_list = true; }
        }
        if (m_on) {
          int cnt = 0;
          for (int i = tid; i < n_list; i += NT) cnt += (w.weight(w.list_z(i)) >= min_p);
          cnt = w.block_count(cnt);
          if (cnt < n_list || small_k) { n = min(n, cnt); in_list = true; }
        }
        n = max(n, 1);
        if (in_list && k_on && !small_k) n = (int)min((int64_t)n, k);
      }
    }
  }
  int pick = 0;
  if (in_list) {
    W = s.pref[n - 1];
    cut.z = w.list_z(n - 1); cut.tie = w.list_id(n - 1);
    cut_on = true;
    __syncthreads();
    pick = w.draw_from_list(n, u);
  } else {
    bool summed = !(k_on || p_on || m_on);           // csum holds the sums of what is kept
    if (k_on) {                                      // top_k above kSMaxTop
      Cut kc;
      double mass;
      if (w.find_cut(false, (unsigned long long)k, 0.0, tau, 0, 0.0, kc, mass, &summed)) { cut = kc; cut_on = true; W = mass; }
    }
    if (p_on) {
      Cut pc;
      double mass;
      if (w.find_cut(true, 0, top_p * W, tau, k_on ? 0 : n_list, k_on || n_list == 0 ? 0.0 : s.pref[n_list - 1], pc, mass, &summed)) {
        if (cut_on) { const Cut both = tighter(cut, pc); summed = summed && both.z == pc.z && both.tie == pc.tie; cut = both; }
        else cut = pc;
        cut_on = true;
      }
    }
    if (m_on) {
      const Cut mc = {__double2float_ru(w.M + tau * log(min_p)), INT_MAX};
      const Cut both = cut_on ? tighter(cut, mc) : mc;
      summed = summed && cut_on && both.z == cut.z && both.tie == cut.tie;
      cut = both;
      cut_on = true;
    }
    if (!summed) {
      Cmd cmd = {};
      cmd.op = OP_CDF; cmd.v[0] = cut.z; cmd.tie = cut.tie;
      w.issue(cmd);
    }
    w.block_scan(tid < nchunks ? s.csum[tid] : 0.0, W);
    __syncthreads();
    const double target = u * W;
    double before;
    const int ch = w.find_chunk(target, before);
    const float low = w.low_of(w.M);
    pick = w.find_in_chunk(ch, before, target, [&](float z, int j) {
      double q, x;
      w.eM.template parts<true>(fmaxf(z, low), w.tab_hi, w.tab_lo, q, x);
      return (z >= low && (!cut_on || kept(cut, z, j))) ? w.corr * (q * x) : 0.0;
    });
  }
  if (tid == 0) {
    p.ids[t] = pick;
    p.logp[t] = (float)(((double)Row<T>::at(base, pick) - w.M) / tau - log(W));
  }
  // the record: the largest K in order, with what the draw gave them
  for (int i = tid; i < n_rec; i += NT) {
    p.topk_ids[t * p.K + i] = s.rec_id[i];
    p.topk_p[t * p.K + i] = (!cut_on || kept(cut, s.rec_z[i], s.rec_id[i])) ? (float)(w.weight(s.rec_z[i]) / W) : 0.f;
  }
  if (n_rec < p.K && tid < 32) {                     // fewer finite logits than K: -inf entries by their ids
    int at = n_rec;
    for (int64_t j0 = 0; j0 < p.V && at < p.K; j0 += 32) {
      const bool hit = j0 + tid < p.V && Row<T>::at(base, j0 + tid) == -INFINITY;
      const unsigned m = __ballot_sync(0xffffffffu, hit);
      const int me = at + __popc(m & ((1u << tid) - 1u));
      if (hit && me < p.K) { p.topk_ids[t * p.K + me] = (int)(j0 + tid); p.topk_p[t * p.K + me] = 0.f; }
      at += __popc(m);
    }
  }
  Cmd done = {};
  done.op = OP_DONE;
  w.issue(done);
}

template <typename T, int NT>
cudaError_t launch_sample(const SampleParams& p, int64_t T_rows, int C, cudaStream_t st) {
  auto kernel = dppo_sample_kernel<T, NT>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SampleSmem));
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(T_rows * C));
  cfg.blockDim = dim3(NT);
  cfg.dynamicSmemBytes = sizeof(SampleSmem);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)C; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = C > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, p, C);
}

}  // namespace
}  // namespace dppo

extern "C" int dppo_sample(const void* logits, int64_t T, int64_t V, int64_t logits_row_stride, int logits_dtype,
                           const double* uniform, const float* temperature, const int32_t* top_k, const float* top_p,
                           const float* min_p, const uint8_t* token_mask, int K,
                           int32_t* sampled_ids, float* mu_logp, int32_t* mu_topk_ids, float* mu_topk_p,
                           int32_t* status, void* cuda_stream) {
  using namespace dppo;
  if (T < 0 || V < 1 || V > ((int64_t)1 << 30) || K < 0 || (int64_t)K > V) return DPPO_ERR_SHAPE;
  if (logits_dtype != DPPO_F32 && logits_dtype != DPPO_BF16) return DPPO_ERR_DTYPE;
  if (K > DPPO_SAMPLE_MAX_TOPK) return DPPO_ERR_UNSUPPORTED;
  if (!status) return DPPO_ERR_NULL;
  if (T > 0 && (!logits || !uniform || !sampled_ids || !mu_logp)) return DPPO_ERR_NULL;
  if (T > 0 && K > 0 && (!mu_topk_ids || !mu_topk_p)) return DPPO_ERR_TOPK;
  if (logits_row_stride < V) return DPPO_ERR_STRIDE;
  const int es = logits_dtype == DPPO_BF16 ? 2 : 4;
  if (((uintptr_t)logits % es) || ((uintptr_t)uniform % 8)) return DPPO_ERR_ALIGN;
  const uintptr_t words = (uintptr_t)temperature | (uintptr_t)top_k | (uintptr_t)top_p | (uintptr_t)min_p | (uintptr_t)sampled_ids | (uintptr_t)mu_logp |
                          (uintptr_t)mu_topk_ids | (uintptr_t)mu_topk_p | (uintptr_t)status;
  if (words % 4) return DPPO_ERR_ALIGN;
  if (T == 0) return DPPO_OK;
  int dev = 0, sms = 148;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  const int64_t nvec = (V * es + 15) / 16 + 1;             // one more for a row that starts inside a vector
  // few rows: several SMs share a row, as long as there are SMs and vectors enough for all of their warps (bf16,
  // V = 151936, without cuts: one row 14 us on eight SMs, 33 us on one; 64 rows 25 us on two each, 33 us on one each)
  int C = 1;
  while (C < kSMaxCluster && T * C * 2 <= sms && nvec >= 64 * 2 * C * kSWarps) C *= 2;
  // vectors per lane and chunk: at most kSMaxChunks chunks; four where a CTA has the row to itself and chunks enough
  // (what a chunk costs besides its elements is spread over more of them: 256 fp32 rows of 50257 with top-p 88 us, 109 us with as
  // few as 256 chunks allow), no more than needed where the row is shared
  int vecs = (int)((nvec + 32 * kSMaxChunks - 1) / (32 * kSMaxChunks));
  if (C == 1 && vecs < 4 && nvec >= 32 * 4 * 4 * kSWarps) vecs = 4;
  SampleParams p = {logits, V, logits_row_stride, uniform, temperature, top_p, min_p, top_k, token_mask, K, vecs,
                    sampled_ids, mu_logp, mu_topk_ids, mu_topk_p, status};
  if (T > INT32_MAX / C) return DPPO_ERR_SHAPE;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  // a row to a CTA of 256 threads, two on an SM, once there are more rows than SMs (2048 rows of 151936: 451 us, in CTAs of 512 537 us;
  // 256 fp32 rows of 50257 with top-p: 88 and 129 us); 512 threads, on one SM or several, otherwise
  const bool many = T > sms;
  cudaError_t e;
  if (logits_dtype == DPPO_BF16) e = many ? launch_sample<__nv_bfloat16, 256>(p, T, C, st) : launch_sample<__nv_bfloat16, 512>(p, T, C, st);
  else e = many ? launch_sample<float, 256>(p, T, C, st) : launch_sample<float, 512>(p, T, C, st);
  return e == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
}
