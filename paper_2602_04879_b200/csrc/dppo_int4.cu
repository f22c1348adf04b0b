// Weights in 4 bits with a scale per group of 32, 64 or 128 along a row: rounding to them, and their product with a few rows.
//
//   scale = amax / 7 rounded to bf16,   code = round(x / scale) + 8 in 1 .. 15, two codes to a byte, the even column in the low half
//   y[m, n] = sum_g scale[n, g] sum_{k in group g} x[m, k] (code[n, k] - 8)
//
// The codes are small whole numbers, so every product x (code - 8) is exact; a group's products are added up in fp32 and its scale is
// applied to that sum, so that no weight is rounded a second time.
#include <mutex>

#include "dppo_gemm.cuh"
#include "dppo_rowvec.cuh"

namespace dppo {
namespace {

// ---------------------------------------------------------------------------------------------------------- quantiser
struct QuantParams {
  const void* x;
  int64_t rows, cols, ldx;
  unsigned char* q;
  int64_t ldq;
  __nv_bfloat16* scale;
  int64_t lds;
  void* values;              // in the type of x, or null
  int64_t ldv;
  int32_t* status;
  int64_t slots;             // pieces of 8 columns of a row, a whole number of groups
  int x_whole, q_whole, v_whole;   // 16-byte loads, 4-byte stores, 16-byte stores of values allowed
};

constexpr int kQThreads = 256, kQItems = 4;

// amax / 7 rounded to bf16 once: the quotient is rounded towards zero with what was lost kept in the last bit
__device__ __forceinline__ float group_scale(float amax) {
  float t = __fdiv_rz(amax, 7.f);
  if (fmaf(t, 7.f, -amax) != 0.f) t = __uint_as_float(__float_as_uint(t) | 1u);
  return __bfloat162float(__float2bfloat16_rn(t));
}

// round(|x| / scale) to nearest, ties to even: the quotient's floor from an approximate reciprocal (it may be one off next to a whole
// number), and the sign of |x| - (floor + 1/2) scale, which one fma gives exactly
__device__ __forceinline__ int code_of(float x, float scale, float inv) {
  const float a = fabsf(x), f = fminf(floorf(a * inv), 7.f);
  const float d = fmaf(-(f + 0.5f), scale, a);
  const int k = (int)f;
  const int up = d > 0.f || (d == 0.f && (k & 1));
  const int c = min(k + up, 7);
  return x < 0.f ? -c : c;
}

template <typename InT, int G>
__global__ void __launch_bounds__(kQThreads) int4_quantize_kernel(QuantParams p) {
  constexpr int LANES = G / 8;
  const InT* X = reinterpret_cast<const InT*>(p.x);
  InT* Vv = reinterpret_cast<InT*>(p.values);
  const int64_t total = p.rows * p.slots;
  const int64_t first = (int64_t)blockIdx.x * (kQThreads * kQItems) + threadIdx.x;
  float v[kQItems][8];
  int64_t row[kQItems], col[kQItems];
#pragma unroll
  for (int k = 0; k < kQItems; ++k) {
    const int64_t i = first + k * kQThreads;
    row[k] = -1;
    col[k] = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[k][j] = 0.f;
    if (i < total) {
      row[k] = total <= 0xffffffffll ? (int64_t)((uint32_t)i / (uint32_t)p.slots) : i / p.slots;
      col[k] = (i - row[k] * p.slots) * 8;
      const InT* src = X + row[k] * p.ldx + col[k];
      if (p.x_whole && col[k] + 8 <= p.cols) {
        float2 z[4];
        if (sizeof(InT) == 2) {
          to_pairs<__nv_bfloat16>(ldg128_stream(src), z);
        } else {
          to_pairs<float>(ldg128_stream(src), z);
          to_pairs<float>(ldg128_stream(src + 4), z + 2);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) { v[k][2 * j] = z[j].x; v[k][2 * j + 1] = z[j].y; }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (col[k] + j < p.cols) v[k][j] = to_f32<InT>(src[j]);
      }
    }
  }
#pragma unroll
  for (int k = 0; k < kQItems; ++k) {
    float amax = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) amax = max_nan(amax, fabsf(v[k][j]));
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    if (row[k] < 0 || col[k] >= p.cols) continue;          // (a piece of the last group may lie behind the row)
    const bool bad = !(amax <= 3.4028234e38f);
    const float scale = bad ? NAN : group_scale(fmaxf(amax, 7.888609052210118e-31f)), inv = bad ? 0.f : __frcp_rn(scale);
    if ((threadIdx.x & (LANES - 1)) == 0) {
      p.scale[row[k] * p.lds + col[k] / G] = __float2bfloat16_rn(scale);
      if (bad) atomicOr(p.status, DPPO_STATUS_NONFINITE_ROW);
    }
    uint32_t w = 0;
    float val[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = bad ? 0 : code_of(v[k][j], scale, inv);
      w |= (uint32_t)(c + 8) << (4 * j);
      val[j] = (float)c * scale;
    }
    unsigned char* dst = p.q + row[k] * p.ldq + col[k] / 2;
    const int n = (int)min((int64_t)8, p.cols - col[k]);
    if (n < 8) w &= (1u << (4 * n)) - 1u;
    if (n == 8 && p.q_whole) {
      *reinterpret_cast<uint32_t*>(dst) = w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (2 * j < n) dst[j] = (unsigned char)(w >> (8 * j));
    }
    if (Vv) {
      InT* out = Vv + row[k] * p.ldv + col[k];
      if (n == 8 && p.v_whole) {
        Store<InT, 8>::run(out, 0u, val);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < n) out[j] = from_f32<InT>(val[j]);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------------------ product
struct MatvecParams {
  const __nv_bfloat16* x;
  int64_t ldx;
  const unsigned char* q;
  int64_t ldq;
  const __nv_bfloat16* scale;
  int64_t lds;
  int64_t M, N, K;
  int gshift;                // log2 of the group
  void* y;
  int64_t ldy;
  int y_bf16;
};

// ---- tensor cores ------------------------------------------------------------------------------------------------------
// D[n, m] = sum over a group of (code[n, k] - 8) x[m, k] for up to 128 rows n and NT rows m at a time: the weights are the operand with the many
// rows.  They come as they are stored by tensor copies (rows x 256 codes, 128-byte swizzle) into a ring; a thread per row turns
// 128 codes into bf16 pairs in registers and writes them to tensor memory, where tcgen05.mma takes its A operand from; x lies in
// shared memory for the whole launch.  The product of a group is read back, scaled by the row's scale (a thread's own) and added up in
// fp32 registers.  One persistent CTA per SM:
//   warp 0         tensor copies of the weights
//   warps 1, 2     allocate tensor memory (the first), issue the MMAs of every other chunk: a wait for a barrier costs 150 cycles even where nothing is to be
//                  waited for, and with one warp the tensor cores stood still for two of them a chunk (820 cycles instead of 380)
//   C x 4 warps    conversion, taking the chunks of 128 codes in turn
//   E x 4 warps    products: scale, add up, store; each warpgroup NT / E rows of x
// Where x does not fit, a pair of CTAs (a cluster) shares a tile, each half of K, and they exchange the sums of half of x's rows through
// distributed shared memory; where that is not enough either, x is loaded again for each part of K.
//
// A word of 8 codes c0 .. c7 gives the pairs (c0, c4), (c1, c5), (c2, c6), (c3, c7): a mask and an or put a code into the low mantissa bits of
// the bf16 number 128, and subtracting 136 leaves code - 8, exactly.  x is laid out in the order that this makes of k.
namespace mv {

constexpr int LANES = 128, CHUNK = 128;    // rows of a tile at most; codes that a thread converts at a time
constexpr int STAGE_BYTES = LANES * 128;   // two chunks
constexpr int XSPAN = 64;                  // k of a swizzled block of x

struct Params {
  const __nv_bfloat16* x;
  int64_t ldx;
  const __nv_bfloat16* scale;
  int64_t lds;
  int M, N, K;
  void* y;
  int64_t ldy;
  int y_bf16, x_vec;                       // x_vec: 16-byte loads of x allowed
  int rows, stages, seg, nseg, groups;     // rows of a tile; seg: codes of K that x lies in shared memory for (a multiple of 256), nseg of them to a CTA
  int pairs;                               // pairs of chunks of a CTA
  int32_t* status;
  unsigned long long wait_ns;
  int inject;
};

template <int NT, int G> struct Shape {
  static constexpr int E = NT == 64 ? 2 : 1, EN = NT / E;              // warpgroups for the products, rows of x of each
  static constexpr int A = CHUNK / 2, D = CHUNK / G * NT;              // columns of tensor memory of a chunk: operand, products
  static constexpr int BUFS = 512 / (A + D) >= 6 ? 6 : 512 / (A + D) / 2 * 2;     // chunks under way
  // Warpgroups that convert.  Barrier phases are known by their parity, so whoever waits for a buffer's last use has to know that the use before
  // that is over.  An issuing warp has made it itself, BUFS being even.  A converting warpgroup has seen the end of the MMAs of chunk
  // i - CONV - BUFS before its chunk i; CONV being even, that chunk and i - 2 BUFS are one issuing warp's, which takes them in order: CONV <= BUFS.
  static constexpr int CONV = NT == 64 || BUFS < 4 ? 2 : 4;
  static constexpr int THREADS = 96 + (CONV + E) * 128;
  static_assert(BUFS >= 2 && BUFS % 2 == 0 && CONV % 2 == 0 && CONV <= BUFS, "barrier phases");
};

__device__ __forceinline__ uint32_t elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p;
}
// A from tensor memory
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n"
               ::"r"(d), "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
      "%24,%25,%26,%27,%28,%29,%30,%31,%32};\n"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
        "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                 "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(taddr));
}
// the 8 codes of a word as four bf16 pairs (c0, c4), (c1, c5), (c2, c6), (c3, c7), less 8
__device__ __forceinline__ void convert(uint32_t w, uint32_t* r) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t v;
    asm("lop3.b32 %0, %1, 0x000f000f, 0x43004300, 0xea;" : "=r"(v) : "r"(w >> (4 * i)));
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r[i]) : "r"(v), "r"(0x43084308u));
  }
}

// x rows m0 .. m0 + NT - 1, codes k0 .. k0 + seg - 1 of K, into shared memory: blocks of 64 codes, NT rows of 128 bytes each, 128-byte
// swizzle, and within 8 codes the order that convert() makes of them.  Rows and codes that there are not are zero.
template <int NT, int T>
__device__ __forceinline__ void load_x(const Params& p, unsigned char* xs, int m0, int k0, int tid) {
  constexpr int AT_ONCE = 4;               // loads in flight
  const int octets = p.seg / 8, all = NT * octets;
  for (int i0 = tid; i0 < all; i0 += AT_ONCE * T) {
    uint4 v[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int i = i0 + u * T, m = i / octets, o = i - m * octets, k = k0 + 8 * o;
      v[u] = make_uint4(0u, 0u, 0u, 0u);
      if (i < all && m0 + m < p.M && k < p.K) {
        const __nv_bfloat16* src = p.x + (int64_t)(m0 + m) * p.ldx + k;
        if (p.x_vec && k + 8 <= p.K) {
          v[u] = *reinterpret_cast<const uint4*>(src);
        } else {
          uint32_t h[8] = {};
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (k + j < p.K) h[j] = __bfloat16_as_ushort(src[j]);
          v[u] = make_uint4(h[0] | (h[1] << 16), h[2] | (h[3] << 16), h[4] | (h[5] << 16), h[6] | (h[7] << 16));
        }
      }
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int i = i0 + u * T, m = i / octets, o = i - m * octets;
      if (i >= all) break;
      const int at = (o / 8) * (NT * 128) + m * 128 + ((16 * (o % 8)) ^ ((m & 7) << 4));
      // (0, 4), (1, 5), (2, 6), (3, 7)
      *reinterpret_cast<uint4*>(xs + at) = make_uint4(__byte_perm(v[u].x, v[u].z, 0x5410), __byte_perm(v[u].x, v[u].z, 0x7632), __byte_perm(v[u].y, v[u].w, 0x5410),
                                                      __byte_perm(v[u].y, v[u].w, 0x7632));
    }
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

struct Bars {
  unsigned long long full[12], empty[12];            // stages of weights
  unsigned long long a_full[6], done[6], d_free[6];  // chunk: operand written; MMAs done (operand free, products there); products read
  unsigned long long x_free, x_full;                 // x replaced
  unsigned long long sum_full, sum_free;             // pairs of CTAs: the other's sums are here; read by the other
  uint32_t tmem;
  int abort_flag;
};

template <int NT, int G, int CL>
__global__ void __launch_bounds__(Shape<NT, G>::THREADS, 1) matvec_int4_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ Params p) {
  using S = Shape<NT, G>;
  constexpr int NG = CHUNK / G, BUFS = S::BUFS, CONV = S::CONV, COLS = S::A + S::D, EN = S::EN, OWN = EN / CL;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* xs = smem + p.stages * STAGE_BYTES;
  float* sums = reinterpret_cast<float*>(xs + (size_t)p.seg * NT * 2);  // pairs: [E][OWN][LANES], from the other CTA
  Bars* bars = reinterpret_cast<Bars*>(sums + (CL > 1 ? NT / CL * LANES : 0));
  const uint32_t full0 = smem_u32(bars->full), empty0 = smem_u32(bars->empty), a0 = smem_u32(bars->a_full), done0 = smem_u32(bars->done), free0 = smem_u32(bars->d_free);
  const uint32_t x_free = smem_u32(&bars->x_free), x_full = smem_u32(&bars->x_full), sum_full = smem_u32(&bars->sum_full), sum_free = smem_u32(&bars->sum_free);
  const WaitCtl wc{&bars->abort_flag, p.wait_ns};
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = CL > 1 ? (int)cluster_ctarank() : 0;
  if (tid == 0) {
    for (int i = 0; i < 12; ++i) { mbar_init(full0 + 8 * i, 1); mbar_init(empty0 + 8 * i, 8); }
    for (int i = 0; i < 6; ++i) { mbar_init(a0 + 8 * i, 4); mbar_init(done0 + 8 * i, 1); mbar_init(free0 + 8 * i, 4 * S::E); }
    mbar_init(x_free, CONV * 4);
    mbar_init(x_full, CONV * 4);
    mbar_init(sum_full, 4 * S::E);
    mbar_init(sum_free, 4 * S::E);
    bars->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem)), "n"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = bars->tmem;
  if (CL > 1) cluster_sync_all();          // the other's barriers exist before anything is sent to them
  // A tile is `rows` rows of the weights times NT rows of x; the blocks of x are the slow index.  A CTA's chunks are counted in pairs (a stage).
  const int tiles_n = (p.N + p.rows - 1) / p.rows, tiles = tiles_n * ((p.M + NT - 1) / NT), seg_pairs = p.seg / 256;
  const int pair0 = rank * p.pairs, pairs = max(0, min(p.pairs, (p.K + 255) / 256 - pair0));      // this CTA's part of K
  const int first = blockIdx.x / CL, grid = gridDim.x / CL;

  if (warp == 0) {
    // ------------------------------------------------------------------ weights
    if (!(p.inject & DPPO_INJECT_NO_COPIES)) {
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int tile = first; tile < tiles && ok; tile += grid) {
        const int n0 = (tile % tiles_n) * p.rows;
        for (int c = 0; c < pairs; ++c) {
          if (!mbar_wait_warp(empty0 + 8 * s, ph ^ 1u, wc)) { ok = false; break; }
          if (lane == 0) {
            mbar_arrive_expect_tx(full0 + 8 * s, p.rows * 128);
            gemm::tma_load_2d(smem_u32(smem) + s * STAGE_BYTES, &map_q, (pair0 + c) * 128, n0, full0 + 8 * s);
          }
          if (++s == p.stages) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp < 3) {
    // ------------------------------------------------------------------ MMAs
    constexpr uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(NT >> 3) << 17) | ((uint32_t)(LANES >> 4) << 24);
    const uint64_t xdesc = gemm::make_desc_k_sw128(smem_u32(xs));
    int b = 0, odd = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (int tile = first; tile < tiles && ok; tile += grid) {
      int k = 0;                                           // within what shared memory holds of x
      for (int c = 0; c < 2 * pairs; ++c, k = k + CHUNK == p.seg ? 0 : k + CHUNK) {
        if (odd == warp - 1) {
          // (the operand first: once it is there, the buffer's products before are the last ones)
          ok = mbar_wait_warp(a0 + 8 * b, ph, wc) && mbar_wait_warp(free0 + 8 * b, ph ^ 1u, wc);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t ta = tmem + b * COLS, td = ta + S::A;
          if (elect_one()) {
#pragma unroll
            for (int i = 0; i < CHUNK / 16; ++i) {         // 16 codes an MMA
              const int at = (k + 16 * i) / XSPAN * (NT * 128) + (16 * i) % XSPAN * 2;
              mma_ts(td + (16 * i) / G * NT, ta + 8 * i, xdesc + (uint64_t)(at >> 4), idesc, (16 * i) % G != 0);
            }
            gemm::mma_commit(done0 + 8 * b);
          }
          __syncwarp();
        }
        odd ^= 1;
        if (++b == BUFS) { b = 0; ph ^= 1u; }
      }
    }
  } else if (warp < 3 + 4 * CONV) {
    // ------------------------------------------------------------------ conversion
    const int g = (warp - 3) >> 2, q = warp & 3, r = q * 32 + lane;     // (a warp's lanes of tensor memory are given by its number)
    const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16);
    const int mine = first < tiles ? (tiles - first + grid - 1) / grid : 0;      // tiles of this CTA
    const bool one = p.nseg == 1 && p.M <= NT;             // one part of x for everything
    const int parts = one ? (mine > 0 && pairs > 0 ? 1 : 0) : mine * p.nseg;
    int x_now = -1;                        // which part of x (block of rows, part of K) shared memory holds
    uint32_t n_x = 0;
    // this warpgroup's next chunk of all the CTA's: its number, its place in the ring (in chunks) and its buffer
    int i = g, at = g, b = g;
    uint32_t ph = 0, bph = 0;
    if (b >= BUFS) { b -= BUFS; bph ^= 1u; }
    bool ok = true;
    for (int part = 0; part < parts && ok; ++part) {
      int end = mine * 2 * pairs;
      if (!one || x_now < 0) {
        const int t = one ? 0 : part / p.nseg, seg = one ? 0 : part - t * p.nseg, start = t * 2 * pairs + seg * 2 * seg_pairs;
        if (!one) end = t * 2 * pairs + min(2 * pairs, (seg + 1) * 2 * seg_pairs);
        if (start >= end) continue;        // (a CTA's last part of K may be empty)
        const int block = (first + t * grid) / tiles_n, x_want = block * p.nseg + seg;
        if (x_now != x_want) {
          // once the MMAs with the part before are done: those of the chunk before this part's first, whoever converts it, are the last
          if (start > 0 && !mbar_wait_warp(done0 + 8 * ((start - 1) % BUFS), (uint32_t)((start - 1) / BUFS) & 1u, wc)) { ok = false; break; }
          __syncwarp();
          if (lane == 0) mbar_arrive(x_free);
          if (!mbar_wait_warp(x_free, n_x & 1u, wc)) { ok = false; break; }
          load_x<NT, CONV * 128>(p, xs, block * NT, (pair0 + seg * seg_pairs) * 256, tid - 96);
          __syncwarp();
          if (lane == 0) mbar_arrive(x_full);
          if (!mbar_wait_warp(x_full, n_x & 1u, wc)) { ok = false; break; }
          ++n_x;
          x_now = x_want;
        }
      }
      for (; i < end; i += CONV) {
        const int s = at >> 1;
        if (!mbar_wait_warp(full0 + 8 * s, ph, wc)) { ok = false; break; }
        const uint32_t src = smem_u32(smem) + s * STAGE_BYTES + r * 128;
        uint4 w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = lds128(src + ((((at & 1) * 4 + j) ^ (r & 7)) << 4));
        __syncwarp();
        if (lane == 0) mbar_arrive(empty0 + 8 * s);
        uint32_t v[32];
        auto half = [&](const uint4& x, const uint4& y) {
          convert(x.x, v); convert(x.y, v + 4); convert(x.z, v + 8); convert(x.w, v + 12);
          convert(y.x, v + 16); convert(y.y, v + 20); convert(y.z, v + 24); convert(y.w, v + 28);
        };
        half(w[0], w[1]);
        if (!mbar_wait_warp(done0 + 8 * b, bph ^ 1u, wc)) { ok = false; break; }       // the buffer's operand before has been used
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        tmem_st32(lane_base + b * COLS, v);
        half(w[2], w[3]);
        tmem_st32(lane_base + b * COLS + 32, v);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(a0 + 8 * b);
        at += CONV;
        if (at >= 2 * p.stages) { at -= 2 * p.stages; ph ^= 1u; }
        b += CONV;
        if (b >= BUFS) { b -= BUFS; bph ^= 1u; }
      }
    }
  } else {
    // ------------------------------------------------------------------ products
    const int e = (warp - 3 - 4 * CONV) >> 2, q = warp & 3, r = q * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16) + S::A + e * EN;
    int b = 0;
    uint32_t ph = 0, n_tile = 0;
    bool ok = true;
    int tn = first % tiles_n, block = first / tiles_n;     // of the tile under way
    const int ysize = p.y_bf16 ? 2 : 4;
    const int64_t ystep = p.ldy * ysize;
    auto y_at = [&](int n, int m) { return reinterpret_cast<char*>(p.y) + m * ystep + (int64_t)n * ysize; };
    auto put = [&](char* at, float v) {
      if (p.y_bf16) *reinterpret_cast<__nv_bfloat16*>(at) = __float2bfloat16_rn(v);
      else *reinterpret_cast<float*>(at) = v;
    };
    // The row's scales, fetched two pairs of chunks ahead (their latency is that of L2 or of memory), the next tile's first along with this
    // one's last.
    const int glim = min(max(p.groups - 2 * pair0 * NG, 0), 2 * pairs * NG);      // this CTA's groups
    auto scales_of = [&](int tile_n, bool there) {
      const int n = tile_n * p.rows + r;
      return there && r < p.rows && n < p.N ? reinterpret_cast<const unsigned short*>(p.scale) + (int64_t)n * p.lds + 2 * pair0 * NG : nullptr;
    };
    unsigned short sc[2][2 * NG];
    auto fetch = [&](const unsigned short* row, int c, unsigned short* to) {
#pragma unroll
      for (int h = 0; h < 2 * NG; ++h) {
        to[h] = 0;
        if (row && c * NG + h < glim) to[h] = __ldg(row + c * NG + h);
      }
    };
    const unsigned short* srow = scales_of(tn, first < tiles);
    fetch(srow, 0, sc[0]);
    fetch(srow, 2, sc[1]);
    // pairs of CTAs: this CTA's rows of x of the tile before wait for the other's sums
    float keep[CL > 1 ? OWN : 1];
    char* keep_at = nullptr;
    int keep_rows = -1;
    auto complete = [&]() {
      if (CL == 1 || keep_rows < 0) return true;
      if (!__all_sync(0xffffffffu, mbar_wait_cluster(sum_full, (n_tile - 1u) & 1u, wc))) return false;
      const float* theirs = sums + e * OWN * LANES + r;
      char* at = keep_at;
#pragma unroll
      for (int j = 0; j < (CL > 1 ? OWN : 0); ++j) {
        if (j >= keep_rows) break;
        const float o = theirs[j * LANES];
        if (keep_at) put(at, rank == 0 ? keep[j] + o : o + keep[j]);
        at += ystep;
      }
      __syncwarp();
      if (lane == 0) bar_arrive_cluster(map_to_cta(sum_free, (uint32_t)(rank ^ 1)));
      keep_rows = -1;
      return true;
    };
    for (int tile = first; tile < tiles && ok; tile += grid) {
      const int n = tn * p.rows + r, m0 = block * NT + e * EN;
      const bool live = srow != nullptr;
      tn += grid;
      while (tn >= tiles_n) { tn -= tiles_n; ++block; }
      const unsigned short* srow_next = scales_of(tn, tile + grid < tiles);
      float2 acc[EN / 2];
#pragma unroll
      for (int j = 0; j < EN / 2; ++j) acc[j] = make_float2(0.f, 0.f);
      for (int c0 = 0; c0 < 2 * pairs && ok; c0 += 4) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int c = c0 + 2 * u;
          if (c < 2 * pairs && ok) {                       // two chunks: buffers b and b + 1
            ok = mbar_wait_warp(done0 + 8 * b, ph, wc) && mbar_wait_warp(done0 + 8 * b + 8, ph, wc);
            if (ok) {
              asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
              for (int h = 0; h < NG; ++h) {
                const float s0 = __uint_as_float((uint32_t)sc[u][h] << 16), s1 = __uint_as_float((uint32_t)sc[u][NG + h] << 16);
#pragma unroll
                for (int j0 = 0; j0 < EN; j0 += 16) {
                  uint32_t v[32];
                  tmem_ld16(lane_base + b * COLS + h * NT + j0, v);
                  tmem_ld16(lane_base + (b + 1) * COLS + h * NT + j0, v + 16);
                  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                  for (int j = 0; j < 8; ++j) {
                    acc[j0 / 2 + j] = __ffma2_rn(make_float2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])), make_float2(s0, s0), acc[j0 / 2 + j]);
                    acc[j0 / 2 + j] = __ffma2_rn(make_float2(__uint_as_float(v[16 + 2 * j]), __uint_as_float(v[17 + 2 * j])), make_float2(s1, s1), acc[j0 / 2 + j]);
                  }
                }
              }
              asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
              __syncwarp();
              if (lane == 0) { mbar_arrive(free0 + 8 * b); mbar_arrive(free0 + 8 * b + 8); }
              if (c + 4 < 2 * pairs) fetch(srow, c + 4, sc[u]); else fetch(srow_next, 2 * u, sc[u]);
              b += 2;
              if (b == BUFS) { b = 0; ph ^= 1u; }
            }
          }
        }
        if (ok && c0 == 0) ok = complete();
      }
      if (!ok || !complete()) { ok = false; break; }
      if (CL == 1) {
        if (live) {
          char* at = y_at(n, m0);
          const int rows = p.M - m0;
#pragma unroll
          for (int j = 0; j < EN; ++j) {
            if (j >= rows) break;
            put(at, (j & 1) ? acc[j / 2].y : acc[j / 2].x);
            at += ystep;
          }
        }
      } else {
        // the other's rows of x go over there, once it has read what went before
        if (n_tile > 0 && !__all_sync(0xffffffffu, mbar_wait_cluster(sum_free, (n_tile - 1u) & 1u, wc))) { ok = false; break; }
        const uint32_t dst = map_to_cta(smem_u32(sums + e * OWN * LANES + r), (uint32_t)(rank ^ 1));
        const int rows = min(p.M - m0 - (rank ^ 1) * OWN, OWN);
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
          const float lo = (j & 1) ? acc[j / 2].y : acc[j / 2].x, hi = (j & 1) ? acc[(OWN + j) / 2].y : acc[(OWN + j) / 2].x;
          keep[CL > 1 ? j : 0] = rank == 0 ? lo : hi;
          if (j < rows) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(dst + (uint32_t)(j * LANES * 4)), "f"(rank == 0 ? hi : lo) : "memory");
        }
        __syncwarp();
        if (lane == 0) bar_arrive_cluster(map_to_cta(sum_full, (uint32_t)(rank ^ 1)));
        keep_rows = max(0, min(p.M - m0 - rank * OWN, OWN));
        keep_at = live ? y_at(n, m0 + rank * OWN) : nullptr;
      }
      srow = srow_next;
      ++n_tile;
    }
    if (ok) complete();
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (wc.aborted()) {                      // time for copies and tensor-core work still under way
    if (tid == 0) atomicOr(p.status, DPPO_STATUS_WAIT_LIMIT);
    drain_after_abort();
  }
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
  }
  if (CL > 1) cluster_sync_all();          // the other may still be sending to this CTA's shared memory
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn get_encode() {
  static EncodeFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &r) == cudaSuccess && r == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeFn>(ptr);
  });
  return fn;
}

template <int NT, int G, int CL>
cudaError_t launch_cl(Params p, const unsigned char* q, int64_t ldq, int sms, int smem_most, cudaStream_t st) {
  using S = Shape<NT, G>;
  constexpr int FIXED = (CL > 1 ? NT / CL * LANES * 4 : 0) + (int)sizeof(Bars) + 1024;
  const int room = smem_most - FIXED, total = (p.K + 255) / 256;
  p.pairs = (total + CL - 1) / CL;
  // x for all of this CTA's K where at least four stages are left besides it, else as much as leaves that many
  int most = (room - 4 * STAGE_BYTES) / (NT * 2) / 256;
  p.nseg = (p.pairs + most - 1) / most;
  p.seg = (p.pairs + p.nseg - 1) / p.nseg * 256;
  p.stages = (room - p.seg * NT * 2) / STAGE_BYTES;
  if (p.stages > 12) p.stages = 12;
  // rows of a tile: rounds of tiles over the CTAs that are as full as they can be
  const int64_t ctas = sms / CL, rounds = (p.N + ctas * LANES - 1) / (ctas * LANES);
  p.rows = (int)((p.N + ctas * rounds - 1) / (ctas * rounds));
  CUtensorMap map;
  const cuuint64_t dims[2] = {(cuuint64_t)((p.K + 1) / 2), (cuuint64_t)p.N}, strides[1] = {(cuuint64_t)ldq};
  const cuuint32_t box[2] = {128u, (cuuint32_t)p.rows}, ones[2] = {1u, 1u};
  EncodeFn enc = get_encode();
  if (!enc || enc(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<unsigned char*>(q), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  const int smem = p.stages * STAGE_BYTES + p.seg * NT * 2 + FIXED;
  const int64_t tiles = (int64_t)((p.N + p.rows - 1) / p.rows) * ((p.M + NT - 1) / NT);
  auto kernel = matvec_int4_kernel<NT, G, CL>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CL; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)((tiles < ctas ? tiles : ctas) * CL), 1, 1);
  cfg.blockDim = dim3(S::THREADS, 1, 1);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = CL > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, map, p);
}

template <int NT, int G>
cudaError_t launch(const Params& p, const unsigned char* q, int64_t ldq, int sms, int smem_most, cudaStream_t st) {
  // a pair of CTAs where one cannot hold x besides four stages of weights
  const int64_t x_bytes = (int64_t)((p.K + 255) / 256) * 256 * NT * 2;
  if (x_bytes + 4 * STAGE_BYTES + (int)sizeof(Bars) + 1024 > smem_most) return launch_cl<NT, G, 2>(p, q, ldq, sms, smem_most, st);
  return launch_cl<NT, G, 1>(p, q, ldq, sms, smem_most, st);
}

}  // namespace mv

// Any layout: a warp per row of the weights and up to 8 rows of x, lanes along K.
constexpr int kGThreads = 256, kGRows = 8;
__global__ void __launch_bounds__(kGThreads) matvec_int4_generic_kernel(MatvecParams p) {
  const int lane = threadIdx.x & 31;
  const int64_t blocks_m = (p.M + kGRows - 1) / kGRows;
  for (int64_t item = (int64_t)blockIdx.x * (kGThreads / 32) + (threadIdx.x >> 5); item < p.N * blocks_m; item += (int64_t)gridDim.x * (kGThreads / 32)) {
    const int64_t n = item / blocks_m, m0 = (item - n * blocks_m) * kGRows;
    float acc[kGRows] = {};
    for (int64_t k0 = 8 * lane; k0 < p.K; k0 += 256) {
      float w[8];
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        const unsigned b = k0 + j < p.K ? p.q[n * p.ldq + (k0 + j) / 2] : 0x88u;
        w[j] = (float)((int)(b & 15u) - 8);
        w[j + 1] = k0 + j + 1 < p.K ? (float)((int)(b >> 4) - 8) : 0.f;
      }
      const float s = __bfloat162float(p.scale[n * p.lds + (k0 >> p.gshift)]);
#pragma unroll
      for (int m = 0; m < kGRows; ++m) {
        if (m0 + m >= p.M) break;
        const __nv_bfloat16* x = p.x + (m0 + m) * p.ldx + k0;
        float part = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (k0 + j < p.K) part = fmaf(__bfloat162float(x[j]), w[j], part);
        acc[m] = fmaf(s, part, acc[m]);
      }
    }
#pragma unroll
    for (int m = 0; m < kGRows; ++m) {
      const float v = warp_sum_f32(acc[m]);
      if (lane == 0 && m0 + m < p.M) {
        if (p.y_bf16) reinterpret_cast<__nv_bfloat16*>(p.y)[(m0 + m) * p.ldy + n] = __float2bfloat16_rn(v);
        else reinterpret_cast<float*>(p.y)[(m0 + m) * p.ldy + n] = v;
      }
    }
  }
}

bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return na && nb && x < y + nb && y < x + na;
}

}  // namespace
}  // namespace dppo

extern "C" int dppo_int4_quantize(const void* x, int64_t rows, int64_t cols, int64_t x_row_stride, int x_dtype, int group,
                                  uint8_t* q, int64_t q_row_stride, void* scale, int64_t scale_row_stride,
                                  void* values, int64_t values_row_stride, int32_t* status, void* cuda_stream) {
  using namespace dppo;
  if (rows < 0 || cols < 0 || cols > ((int64_t)1 << 30) || rows > ((int64_t)1 << 38) || (cols > 0 && rows > ((int64_t)1 << 38) / cols)) return DPPO_ERR_SHAPE;
  if (x_dtype != DPPO_F32 && x_dtype != DPPO_BF16) return DPPO_ERR_DTYPE;
  if (group != 32 && group != 64 && group != 128) return DPPO_ERR_UNSUPPORTED;
  if (!status) return DPPO_ERR_NULL;
  if ((uintptr_t)status % 4) return DPPO_ERR_ALIGN;
  if (rows == 0 || cols == 0) return DPPO_OK;
  if (!x || !q || !scale) return DPPO_ERR_NULL;
  const int64_t groups = (cols + group - 1) / group;
  if (rows > 1 && (x_row_stride < cols || q_row_stride < (cols + 1) / 2 || scale_row_stride < groups || (values && values_row_stride < cols))) return DPPO_ERR_STRIDE;
  const size_t es = x_dtype == DPPO_BF16 ? 2 : 4;
  if ((uintptr_t)x % es || (uintptr_t)scale % 2 || (uintptr_t)values % es) return DPPO_ERR_ALIGN;
  const size_t nx = ((size_t)(rows - 1) * x_row_stride + cols) * es, nq = (size_t)(rows - 1) * q_row_stride + (cols + 1) / 2;
  const size_t ns = ((size_t)(rows - 1) * scale_row_stride + groups) * 2, nv = values ? ((size_t)(rows - 1) * values_row_stride + cols) * es : 0;
  if (overlaps(x, nx, q, nq) || overlaps(x, nx, scale, ns) || overlaps(q, nq, scale, ns) || overlaps(values, nv, q, nq) || overlaps(values, nv, scale, ns)) return DPPO_ERR_ALIAS;
  const bool in_place = values == x && (rows == 1 || values_row_stride == x_row_stride);
  if (!in_place && overlaps(values, nv, x, nx)) return DPPO_ERR_ALIAS;
  QuantParams p = {};
  p.x = x; p.rows = rows; p.cols = cols; p.ldx = x_row_stride; p.q = q; p.ldq = q_row_stride; p.scale = reinterpret_cast<__nv_bfloat16*>(scale);
  p.lds = scale_row_stride; p.values = values; p.ldv = values_row_stride; p.status = status;
  p.slots = groups * (group / 8);
  p.x_whole = (uintptr_t)x % 16 == 0 && (rows == 1 || (x_row_stride * es) % 16 == 0);
  p.q_whole = (uintptr_t)q % 4 == 0 && (rows == 1 || q_row_stride % 4 == 0);
  p.v_whole = values && (uintptr_t)values % 16 == 0 && (rows == 1 || (values_row_stride * es) % 16 == 0);
  const int64_t grid = (rows * p.slots + kQThreads * kQItems - 1) / (kQThreads * kQItems);
  if (grid > 0x7fffffffll) return DPPO_ERR_SHAPE;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const unsigned g = (unsigned)grid;
  if (x_dtype == DPPO_BF16) {
    if (group == 32) int4_quantize_kernel<__nv_bfloat16, 32><<<g, kQThreads, 0, st>>>(p);
    else if (group == 64) int4_quantize_kernel<__nv_bfloat16, 64><<<g, kQThreads, 0, st>>>(p);
    else int4_quantize_kernel<__nv_bfloat16, 128><<<g, kQThreads, 0, st>>>(p);
  } else {
    if (group == 32) int4_quantize_kernel<float, 32><<<g, kQThreads, 0, st>>>(p);
    else if (group == 64) int4_quantize_kernel<float, 64><<<g, kQThreads, 0, st>>>(p);
    else int4_quantize_kernel<float, 128><<<g, kQThreads, 0, st>>>(p);
  }
  return cudaGetLastError() == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
}

extern "C" int dppo_matvec_int4(const void* x, int64_t x_row_stride, const uint8_t* q, int64_t q_row_stride, const void* scale,
                                int64_t scale_row_stride, int group, int64_t M, int64_t N, int64_t K, void* y, int y_dtype,
                                int64_t y_row_stride, int32_t* status, const dppo_opts* opts, void* cuda_stream) {
  using namespace dppo;
  if (M < 0 || N < 0 || K < 0 || M > ((int64_t)1 << 30) || N > ((int64_t)1 << 30) || K > ((int64_t)1 << 30)) return DPPO_ERR_SHAPE;
  if (y_dtype != DPPO_F32 && y_dtype != DPPO_BF16) return DPPO_ERR_DTYPE;
  if (group != 32 && group != 64 && group != 128) return DPPO_ERR_UNSUPPORTED;
  if (opts && opts->wait_limit_us < 0) return DPPO_ERR_UNSUPPORTED;
  if (!status) return DPPO_ERR_NULL;
  if ((uintptr_t)status % 4) return DPPO_ERR_ALIGN;
  if (M == 0 || N == 0) return DPPO_OK;
  if (!y || (K > 0 && (!x || !q || !scale))) return DPPO_ERR_NULL;
  const int64_t groups = (K + group - 1) / group;
  if ((M > 1 && (x_row_stride < K || y_row_stride < N)) || (N > 1 && (q_row_stride < (K + 1) / 2 || scale_row_stride < groups))) return DPPO_ERR_STRIDE;
  const size_t ys = y_dtype == DPPO_BF16 ? 2 : 4;
  if ((uintptr_t)x % 2 || (uintptr_t)scale % 2 || (uintptr_t)y % ys) return DPPO_ERR_ALIGN;
  const size_t ny = ((size_t)(M - 1) * (M > 1 ? y_row_stride : 0) + N) * ys;
  if (K > 0 && (overlaps(y, ny, x, ((size_t)(M - 1) * (M > 1 ? x_row_stride : 0) + K) * 2) || overlaps(y, ny, q, (size_t)(N - 1) * (N > 1 ? q_row_stride : 0) + (K + 1) / 2) ||
                overlaps(y, ny, scale, ((size_t)(N - 1) * (N > 1 ? scale_row_stride : 0) + groups) * 2))) return DPPO_ERR_ALIAS;
  MatvecParams p = {};
  p.x = reinterpret_cast<const __nv_bfloat16*>(x); p.ldx = x_row_stride; p.q = q; p.ldq = q_row_stride;
  p.scale = reinterpret_cast<const __nv_bfloat16*>(scale); p.lds = scale_row_stride; p.M = M; p.N = N; p.K = K;
  p.gshift = group == 32 ? 5 : (group == 64 ? 6 : 7);
  p.y = y; p.ldy = y_row_stride; p.y_bf16 = y_dtype == DPPO_BF16;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  // bulk copies of the weights: rows on 16-byte boundaries
  const int64_t pitch = N > 1 ? q_row_stride : ((K + 1) / 2 + 15) / 16 * 16;
  if (K > 0 && (uintptr_t)q % 16 == 0 && pitch % 16 == 0 && N * ((M + 15) / 16) < ((int64_t)1 << 31)) {
    mv::Params m = {};
    m.x = p.x; m.ldx = p.ldx; m.scale = p.scale; m.lds = p.lds; m.M = (int)M; m.N = (int)N; m.K = (int)K; m.y = y; m.ldy = p.ldy; m.y_bf16 = p.y_bf16;
    m.x_vec = (uintptr_t)x % 16 == 0 && (M == 1 || x_row_stride % 8 == 0);
    m.groups = (int)groups;
    m.status = status; m.wait_ns = wait_limit_ns(opts ? opts->wait_limit_us : 0); m.inject = opts ? opts->test_inject : 0;
    int dev = 0, sms = 148, most = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    cudaDeviceGetAttribute(&most, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev);
    // rows of x that one pass over the weights serves (the products of 64 rows and groups of 32 would not fit tensor memory)
    cudaError_t e;
    if (M <= 16) {
      e = group == 128 ? mv::launch<16, 128>(m, q, pitch, sms, most, st) : group == 64 ? mv::launch<16, 64>(m, q, pitch, sms, most, st) : mv::launch<16, 32>(m, q, pitch, sms, most, st);
    } else if (M <= 32 || group == 32) {
      e = group == 128 ? mv::launch<32, 128>(m, q, pitch, sms, most, st) : group == 64 ? mv::launch<32, 64>(m, q, pitch, sms, most, st) : mv::launch<32, 32>(m, q, pitch, sms, most, st);
    } else {
      e = group == 128 ? mv::launch<64, 128>(m, q, pitch, sms, most, st) : mv::launch<64, 64>(m, q, pitch, sms, most, st);
    }
    return e == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
  }
  const int64_t warps = N * ((M + kGRows - 1) / kGRows), grid = (warps + kGThreads / 32 - 1) / (kGThreads / 32);
  matvec_int4_generic_kernel<<<(unsigned)(grid < (1 << 30) ? grid : (1 << 30)), kGThreads, 0, st>>>(p);
  return cudaGetLastError() == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
}
