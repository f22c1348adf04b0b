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
//   search    cuts that lie below the list (top-p over a broad row, top_k > 1024, ties by the thousand) are bracketed by passes
//             over the row (from L2), all CTAs of the cluster counting and summing above three pivots at a time, until what
//             lies between two pivots fits the list.
//   draw      inside the list, or, when the kept set is larger, in the one chunk that the running sum of the chunks' sums
//             points to.
#include <cooperative_groups.h>
#include <limits.h>

#include "dppo_common.cuh"
#include "dppo_pipe.cuh"

namespace dppo {
namespace {

namespace cg = cooperative_groups;

constexpr int kSThreads = 512, kSWarps = kSThreads / 32;
constexpr int kSMaxChunks = 320;       // chunks of a row; a longer row has longer chunks
constexpr int kSList = 4096;           // entries of the sorted list
constexpr int kSMaxTop = DPPO_SAMPLE_MAX_TOPK;      // largest list that is asked for
constexpr int kSProbe = 256;           // list length tried first for top-p / min-p alone
constexpr int kSMaxCluster = 8;
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

enum { OP_DONE = 0, OP_PIVOTS, OP_COMPACT, OP_EQUAL, OP_CDF };
struct Cmd {
  int op;
  uint32_t lo, hi;       // OP_COMPACT: keys [lo, hi)
  float v[3];            // OP_PIVOTS: ascending; OP_EQUAL, OP_CDF: v[0]
  int tie;               // OP_CDF
};

struct SampleSmem {
  double csum[kSMaxChunks];
  double tab[32];                         // 2^(i/32)
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
  float cmax[kSMaxChunks];
  float rec_z[kSMaxTop];
  int rec_id[kSMaxTop];
  int hist[256];
  Cmd cmd;
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

// 2^x for -1020 <= x <= 1000: x = n/32 + f, 2^x = 2^(n>>5) tab[n & 31] 2^f, |f| <= 1/64, with the Taylor polynomial of 2^f
// to the fourth power: the fifth term is below 1.3e-12.
__device__ __forceinline__ double exp2_tab(double d, double c, const double* tab) {       // 2^(d c)
  constexpr double kMagic = 6755399441055744.0 / 32.0;       // 1.5 2^52 / 32: adding it rounds to multiples of 1/32
  const double t = fma(d, c, kMagic);
  const double f = fma(d, c, -(t - kMagic));
  double p = fma(f, 9.6181291076284772e-3, 5.5504108664821580e-2);     // ln2^4 / 24, ln2^3 / 6
  p = fma(p, f, 2.4022650695910071e-1);                                // ln2^2 / 2
  p = fma(p, f, 6.9314718055994531e-1);
  p = fma(p, f, 1.0);
  const int n = __double2loint(t);
  const double s = tab[n & 31];
  return p * __hiloint2double(__double2hiint(s) + ((n >> 5) << 20), __double2loint(s));
}

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

template <typename T>
struct Worker {
  const SampleParams& p;
  SampleSmem& s;
  RowView<T> row;
  int nchunks, c_begin, c_end;             // chunks of the row, and those of this CTA
  int rank, C;
  double c;                                // log2(e) / tau
  double itau;                             // 1 / tau
  double M;                                // row maximum (known after pass A)
  static constexpr int N = Row<T>::N;

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
  __device__ __forceinline__ float low_of(double ref) const { return __double2float_ru(ref - 1000.0 / c); }

  // f(z, element index) over this thread's part of chunk ch
  template <typename F> __device__ __forceinline__ void each(int ch, F f) const {
    for (int i = 0; i < p.vecs; ++i) {
      const int sv = (ch * p.vecs + i) * 32 + lane();
      const uint4 v = row.load(sv);
      float z[N];
      Row<T>::unpack(v, z);
      const int j0 = sv * N - row.head;
#pragma unroll
      for (int e = 0; e < N; ++e) f(z[e], j0 + e);
    }
  }

  // ---- pass A ----
  __device__ void pass_a(bool want_sum, bool want_groups) const {
    SampleSmem* lead = smem_of(0);
    for (int ch = c_begin + warp(); ch < c_end; ch += kSWarps) {
      float mx = -INFINITY;
      for (int i = 0; i < p.vecs; i += 4) {
        uint4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) if (i + k < p.vecs) v[k] = row.load((ch * p.vecs + i + k) * 32 + lane());
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (i + k < p.vecs) {
            float z[N];
            Row<T>::unpack(v[k], z);
#pragma unroll
            for (int e = 0; e < N; ++e) mx = max_nan(mx, z[e]);
          }
      }
      if (want_groups) lead->gmax[ch * 32 + lane()] = mx;
      const float cm = warp_max_nan(mx);
      double sum = 0.0;
      if (want_sum && cm > -INFINITY && cm < INFINITY) {
        const float low = low_of((double)cm);
        each(ch, [&](float z, int) { const double w = exp2_tab((double)z - (double)cm, c, s.tab); if (z >= low) sum += w; });
        sum = warp_sum(sum);
      }
      if (lane() == 0) { lead->cmax[ch] = cm; lead->csum[ch] = sum; }
    }
  }

  // ---- passes that the leader asks for ----
  __device__ void execute(const Cmd& k) const {
    SampleSmem* lead = smem_of(0);
    if (k.op == OP_PIVOTS) {
      double m[3] = {0, 0, 0};
      unsigned n[3] = {0, 0, 0};
      const float low = low_of(M);
      for (int ch = c_begin + warp(); ch < c_end; ch += kSWarps)
        each(ch, [&](float z, int) {
          if (z >= k.v[0]) {
            const double w = z >= low ? exp2_tab((double)z - M, c, s.tab) : 0.0;
#pragma unroll
            for (int i = 0; i < 3; ++i) if (z >= k.v[i]) { m[i] += w; ++n[i]; }
          }
        });
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        const double mm = warp_sum(m[i]);
        const unsigned nn = __reduce_add_sync(0xffffffffu, n[i]);
        if (lane() == 0) { s.wmass[warp()][i] = mm; s.wcnt[warp()][i] = nn; }
      }
      __syncthreads();
      if (tid() < 3) {
        double a = 0.0;
        unsigned long long b = 0;
        for (int w = 0; w < kSWarps; ++w) { a += s.wmass[w][tid()]; b += s.wcnt[w][tid()]; }
        lead->mass[rank][tid()] = a;
        lead->cnt[rank][tid()] = b;
      }
    } else if (k.op == OP_COMPACT) {
      for (int ch = c_begin + warp(); ch < c_end; ch += kSWarps)
        each(ch, [&](float z, int j) {
          const uint32_t key = key_of(z);
          if (key >= k.lo && key < k.hi) {
            const int at = atomicAdd(&lead->n_list, 1);
            if (at < kSList) lead->list[at] = ((unsigned long long)~key << 32) | (uint32_t)j;
          }
        });
    } else if (k.op == OP_EQUAL) {
      for (int ch = c_begin + warp(); ch < c_end; ch += kSWarps) {
        unsigned n = 0;
        each(ch, [&](float z, int) { n += (z == k.v[0]); });
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane() == 0) lead->csum[ch] = (double)n;
      }
    } else if (k.op == OP_CDF) {
      const Cut cut = {k.v[0], k.tie};
      const float low = low_of(M);
      for (int ch = c_begin + warp(); ch < c_end; ch += kSWarps) {
        double sum = 0.0;
        each(ch, [&](float z, int j) { if (z >= low && kept(cut, z, j)) sum += exp2_tab((double)z - M, c, s.tab); });
        sum = warp_sum(sum);
        if (lane() == 0) lead->csum[ch] = sum;
      }
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
    for (int w = 0; w < kSWarps; ++w) { if (w < warp()) before += s.red[w]; all += s.red[w]; }
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
    __syncthreads();
    if (tid() == 0) s.pick = 0;
    __syncthreads();
    v = __reduce_add_sync(0xffffffffu, v);
    if (lane() == 0) atomicAdd(&s.pick, v);
    __syncthreads();
    return s.pick;
  }
  // ascending sort of list[0, n): logits descending, ids ascending
  __device__ void sort_list(int n) const {
    int P = 32;
    while (P < n) P <<= 1;
    for (int i = n + tid(); i < P; i += kSThreads) s.list[i] = ~0ull;
    __syncthreads();
    for (int k = 2; k <= P; k <<= 1)
      for (int j = k >> 1; j > 0; j >>= 1) {
        for (int t = tid(); t < P / 2; t += kSThreads) {
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
    const int per = (n + kSThreads - 1) / kSThreads, b = tid() * per, e = min(n, b + per);
    double v = 0.0;
    for (int i = b; i < e; ++i) v += weight(list_z(i));
    double total;
    double run = block_scan(v, total);
    for (int i = b; i < e; ++i) { run += weight(list_z(i)); s.pref[i] = run; }
    __syncthreads();
    return n > 0 ? s.pref[n - 1] : 0.0;
  }
  // the list's entries [0, n) in the order of their ids: lowest id whose running sum exceeds target
  __device__ int draw_from_list(int n, double u) const {
    const double target = u * s.pref[n - 1];
    int best = INT_MAX, last = -1;
    if (n <= kSThreads / 2) {
      if (tid() < n) {
        const int me = list_id(tid());
        double run = 0.0;
        for (int j = 0; j < n; ++j) if (list_id(j) <= me) run += s.pref[j] - (j ? s.pref[j - 1] : 0.0);
        if (run > target) best = me;
        last = me;
      }
    } else {
      __syncthreads();
      // turned round in place: ids in front, position in the list (for the weight) behind
      for (int i = tid(); i < n; i += kSThreads) s.list[i] = ((unsigned long long)(uint32_t)list_id(i) << 32) | (uint32_t)i;
      __syncthreads();
      sort_list(n);
      const int per = (n + kSThreads - 1) / kSThreads, b = tid() * per, e = min(n, b + per);
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
  // lowest element of chunk ch at which before + running sum of w(z, j) exceeds target; the last one with w > 0 otherwise
  template <typename F> __device__ int find_in_chunk(int ch, double before, double target, F w) const {
    __syncthreads();
    if (warp() == 0) {
      int best = INT_MAX, last = -1;
      double run = before;
      for (int i = 0; i < p.vecs && best == INT_MAX; ++i) {
        const int sv = (ch * p.vecs + i) * 32 + lane();
        const uint4 v = row.load(sv);
        float z[N];
        Row<T>::unpack(v, z);
        const int j0 = sv * N - row.head;
        double x[N], mine = 0.0;
#pragma unroll
        for (int e = 0; e < N; ++e) { x[e] = w(z[e], j0 + e); mine += x[e]; if (x[e] > 0.0) last = j0 + e; }
        double inc = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const double y = __shfl_up_sync(0xffffffffu, inc, o); if (lane() >= o) inc += y; }
        double r = run + (inc - mine);
        int b = INT_MAX;
#pragma unroll
        for (int e = 0; e < N; ++e) { r += x[e]; if (b == INT_MAX && x[e] > 0.0 && r > target) b = j0 + e; }
        best = __reduce_min_sync(0xffffffffu, b);
        run = run + __shfl_sync(0xffffffffu, inc, 31);
      }
      last = __reduce_max_sync(0xffffffffu, last);
      if (lane() == 0) s.pick = best != INT_MAX ? best : last;
    }
    __syncthreads();
    return s.pick;
  }

  // The cut after which the kept prefix (of all finite entries, in order) has `count` tokens (by_mass false), or is the
  // shortest one with mass >= target (by_mass true).  *top_mass: mass of that prefix.  False if the whole row is kept.
  // Overwrites list, pref and csum.
  __device__ bool find_cut(bool by_mass, unsigned long long count, double target, double tau, Cut& cut, double& top_mass) const {
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
        const bool holds = by_mass ? m >= target : n >= count;
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
        for (int i = tid(); i < n; i += kSThreads) if (m_hi + s.pref[i] >= target) { b = i; break; }
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
    if (kk < G) {
      // the two upper digits of the kk-th largest group maximum, by counting
      uint32_t prefix = 0;
      int want = kk;
      for (int d = 0; d < 2; ++d) {
        const int shift = 24 - 8 * d;
        for (int i = tid(); i < 256; i += kSThreads) s.hist[i] = 0;
        __syncthreads();
        for (int g = tid(); g < G; g += kSThreads) {
          const uint32_t k = key_of(s.gmax[g]);
          if (d == 0 || (k >> 24) == (prefix >> 24)) atomicAdd(&s.hist[(k >> shift) & 255], 1);
        }
        __syncthreads();
        if (warp() == 0) {                    // lane i: digits 255 - 8 i down to 248 - 8 i
          int n = 0;
          for (int q = 0; q < 8; ++q) n += s.hist[255 - 8 * lane() - q];
          int inc = n;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, inc, o); if (lane() >= o) inc += x; }
          int run = inc - n;
          if (run < want && inc >= want) {
            for (int q = 0; q < 8; ++q) {
              const int dg = 255 - 8 * lane() - q, h = s.hist[dg];
              if (run + h >= want) { s.pick = dg; s.n_list = run; break; }
              run += h;
            }
          }
        }
        __syncthreads();
        prefix |= (uint32_t)s.pick << shift;
        want -= s.n_list;
        __syncthreads();
      }
      bound = max(bound, prefix);
    }
    __syncthreads();
    if (tid() == 0) s.n_list = 0;
    __syncthreads();
    // a thread per vector of each group that reaches the bound
    for (int g0 = 0; g0 < G; g0 += kSThreads) {
      const int g = g0 + tid();
      const bool hit = g < G && key_of(s.gmax[g]) >= bound;
      if (hit) {
        const int ch = g >> 5, ln = g & 31;
        for (int i = 0; i < p.vecs; ++i) {
          const int sv = (ch * p.vecs + i) * 32 + ln;
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
      }
    }
    __syncthreads();
    return s.n_list <= kSList;
  }
};

template <typename T>
__global__ void __launch_bounds__(kSThreads, 2) dppo_sample_kernel(SampleParams p, int C) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  SampleSmem& s = *reinterpret_cast<SampleSmem*>(smem_raw);
  const int rank = (C == 1) ? 0 : (int)cluster_ctarank();
  const int64_t t = (int64_t)(blockIdx.x / (unsigned)C);
  const int tid = threadIdx.x;

  auto drop = [&](int bit) {
    if (rank == 0) {
      if (tid == 0) { p.ids[t] = 0; p.logp[t] = 0.f; if (bit) atomicOr(p.status, bit); }
      for (int i = tid; i < p.K; i += kSThreads) { p.topk_ids[t * p.K + i] = 0; p.topk_p[t * p.K + i] = 0.f; }
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
  int kk = p.K;
  if (small_k) kk = max(kk, (int)k);
  else if (p_on || m_on) kk = max(kk, kSProbe);

  const T* base = reinterpret_cast<const T*>(p.logits) + t * p.ld;
  RowView<T> row;
  row.row = base;
  row.V = (int)p.V;
  row.head = (int)(((uintptr_t)base & 15) / sizeof(T));
  row.nvec = (int)(((int64_t)row.head + p.V + Row<T>::N - 1) / Row<T>::N);
  const int nchunks = (row.nvec + 32 * p.vecs - 1) / (32 * p.vecs), per = (nchunks + C - 1) / C;
  Worker<T> w = {p, s, row, nchunks, min(nchunks, rank * per), min(nchunks, (rank + 1) * per), rank, C, kLog2eD / tau, 1.0 / tau, 0.0};

  if (tid < 32) s.tab[tid] = exp2((double)tid / 32.0);
  w.csync();                                         // tables ready; every CTA of the cluster runs
  w.pass_a(!small_k, kk > 0);
  w.csync();

  // row maximum, known to the leader
  SampleSmem* lead = w.smem_of(0);
  float mx = -INFINITY;
  for (int ch = threadIdx.x & 31; ch < nchunks; ch += 32) mx = max_nan(mx, lead->cmax[ch]);
  mx = warp_max_nan(mx);
  w.M = (double)mx;
  if (!(mx > -INFINITY && mx < INFINITY)) {          // a NaN, an infinity, or nothing but -inf: every CTA sees the same
    drop(DPPO_STATUS_NONFINITE_ROW);
    w.csync();                                       // the leader's shared memory was read by all
    return;
  }
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
      v = s.csum[tid] > 0.0 ? s.csum[tid] * exp(((double)s.cmax[tid] - w.M) * w.itau) : 0.0;
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
      w.find_cut(false, (unsigned long long)kk, 0.0, tau, kc, dummy);
      // the kk entries themselves
      __syncthreads();
      if (tid == 0) s.n_list = 0;
      Cmd cmd = {};
      cmd.op = OP_COMPACT; cmd.lo = key_of(kc.z) + 1; cmd.hi = kKeyInf;
      w.issue(cmd);
      // of the value at the cut the ones up to its tie, by a walk over the leader's view of the row
      for (int ch = tid >> 5; ch < nchunks; ch += kSWarps)
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
    for (int i = tid; i < n_rec; i += kSThreads) { s.rec_z[i] = w.list_z(i); s.rec_id[i] = w.list_id(i); }
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
          for (int i = tid; i < n_list; i += kSThreads) if (s.pref[i] >= target) { b = i; break; }
          b = w.block_min(b);
          if (b != INT_MAX) { n = min(n, b + 1); in_list = true; }
        }
        if (m_on) {
          int cnt = 0;
          for (int i = tid; i < n_list; i += kSThreads) cnt += (w.weight(w.list_z(i)) >= min_p);
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
    if (k_on) {                                      // top_k above kSMaxTop
      Cut kc;
      double mass;
      if (w.find_cut(false, (unsigned long long)k, 0.0, tau, kc, mass)) { cut = kc; cut_on = true; W = mass; }
    }
    if (p_on) {
      Cut pc;
      double mass;
      if (w.find_cut(true, 0, top_p * W, tau, pc, mass)) { cut = cut_on ? tighter(cut, pc) : pc; cut_on = true; }
    }
    if (m_on) {
      const Cut mc = {__double2float_ru(w.M + tau * log(min_p)), INT_MAX};
      cut = cut_on ? tighter(cut, mc) : mc;
      cut_on = true;
    }
    if (cut_on) {
      Cmd cmd = {};
      cmd.op = OP_CDF; cmd.v[0] = cut.z; cmd.tie = cut.tie;
      w.issue(cmd);
      w.block_scan(tid < nchunks ? s.csum[tid] : 0.0, W);
      __syncthreads();
    }
    const double target = u * W;
    double before;
    const int ch = w.find_chunk(target, before);
    const float low = w.low_of(w.M);
    pick = w.find_in_chunk(ch, before, target, [&](float z, int j) {
      return (z >= low && (!cut_on || kept(cut, z, j))) ? exp2_tab((double)z - w.M, w.c, s.tab) : 0.0;
    });
  }
  if (tid == 0) {
    p.ids[t] = pick;
    p.logp[t] = (float)(((double)Row<T>::at(base, pick) - w.M) / tau - log(W));
  }
  // the record: the largest K in order, with what the draw gave them
  for (int i = tid; i < n_rec; i += kSThreads) {
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

template <typename T>
cudaError_t launch_sample(const SampleParams& p, int64_t T_rows, int C, cudaStream_t st) {
  auto kernel = dppo_sample_kernel<T>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SampleSmem));
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(T_rows * C));
  cfg.blockDim = dim3(kSThreads);
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
  if (T < 0 || V < 1 || V > INT32_MAX || K < 0 || (int64_t)K > V) return DPPO_ERR_SHAPE;
  if (logits_dtype != DPPO_F32 && logits_dtype != DPPO_BF16) return DPPO_ERR_DTYPE;
  if (K > DPPO_SAMPLE_MAX_TOPK) return DPPO_ERR_UNSUPPORTED;
  if (!status) return DPPO_ERR_NULL;
  if (T > 0 && (!logits || !uniform || !sampled_ids || !mu_logp)) return DPPO_ERR_NULL;
  if (T > 0 && K > 0 && (!mu_topk_ids || !mu_topk_p)) return DPPO_ERR_TOPK;
  if (logits_row_stride < V) return DPPO_ERR_STRIDE;
  const int es = logits_dtype == DPPO_BF16 ? 2 : 4;
  if (((uintptr_t)logits % es) || ((uintptr_t)uniform % 8)) return DPPO_ERR_ALIGN;
  if (T == 0) return DPPO_OK;
  int dev = 0, sms = 148;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  const int64_t nvec = (V * es + 15) / 16 + 1;             // one more for a row that starts inside a vector
  SampleParams p = {logits, V, logits_row_stride, uniform, temperature, top_p, min_p, top_k, token_mask, K,
                    (int)((nvec + 32 * kSMaxChunks - 1) / (32 * kSMaxChunks)),
                    sampled_ids, mu_logp, mu_topk_ids, mu_topk_p, status};
  // few rows: several SMs share a row, as long as there are SMs and chunks enough for all of them
  int C = 1;
  const int64_t chunks = (nvec + 32 * (int64_t)p.vecs - 1) / (32 * (int64_t)p.vecs);
  while (C < kSMaxCluster && T * C * 2 <= sms && chunks >= 2 * C * kSWarps) C *= 2;
  if (T > INT32_MAX / C) return DPPO_ERR_SHAPE;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = logits_dtype == DPPO_BF16 ? launch_sample<__nv_bfloat16>(p, T, C, st) : launch_sample<float>(p, T, C, st);
  return e == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
}
