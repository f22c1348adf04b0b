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
// D[n, m] = sum over a group of (code[n, k] - 8) x[m, k] for 128 rows n and NT rows m at a time: the weights are the operand with the many
// rows.  They come as they are stored by tensor copies (128 rows x 256 codes, 128-byte swizzle) into a ring; a thread per row turns its
// 128 codes into bf16 pairs in registers and writes them to tensor memory, where tcgen05.mma takes its A operand from; x lies in
// shared memory for the whole launch (or a segment of K at a time, where it does not fit).  The product of a group is read back, scaled
// by the row's scale (a thread's own) and added up in fp32 registers while the next codes are converted.
//   warp 0         tensor copies of the weights
//   warp 1         allocates tensor memory, issues the MMAs
//   WG x 4 warps   convert, scale and add up; warpgroup g takes the chunks g, g + WG, ... of 128 codes of a tile
// At a tile's end the warpgroups exchange their sums through shared memory; each finishes and stores a part of the rows of x.
//
// A word of 8 codes c0 .. c7 gives the pairs (c0, c4), (c1, c5), (c2, c6), (c3, c7): a mask and an or put a code into the low mantissa bits of
// the bf16 number 128, and subtracting 136 leaves code - 8, exactly.  x is laid out in the order that this makes of k.
namespace mv {

constexpr int ROWS = 128, CHUNK = 128;     // rows of a tile; codes that a thread converts at a time
constexpr int STAGE_BYTES = ROWS * 128;    // two chunks
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
  int stages, seg, nseg, groups;           // seg: codes of K that x lies in shared memory for (a multiple of 256), nseg of them
  int32_t* status;
  unsigned long long wait_ns;
  int inject;
};

template <int NT> struct Shape {
  static constexpr int WG = NT == 16 ? 4 : 2;              // what the registers hold: 32 for half of the converted codes, NT for the sums, 16 for a part of a product
  static constexpr int THREADS = 64 + WG * 128;
};
template <int NT, int G> struct Tmem {
  static constexpr int A = CHUNK / 2, D = CHUNK / G * NT;  // columns of a warpgroup's operand and products
  static constexpr int COLS = Shape<NT>::WG * (A + D) <= 256 ? 256 : 512;
  static_assert(Shape<NT>::WG * (A + D) <= 512, "tensor memory");
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
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
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
template <int NT>
__device__ __forceinline__ void load_x(const Params& p, unsigned char* xs, int m0, int k0, int tid, int threads) {
  const int octets = p.seg / 8;
  for (int i = tid; i < NT * octets; i += threads) {
    const int m = i / octets, o = i - m * octets, k = k0 + 8 * o;
    uint32_t h[8] = {};                                    // the eight entries
    if (m0 + m < p.M && k < p.K) {
      const __nv_bfloat16* src = p.x + (int64_t)(m0 + m) * p.ldx + k;
      if (p.x_vec && k + 8 <= p.K) {
        const uint4 v = *reinterpret_cast<const uint4*>(src);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = (w[j >> 1] >> (16 * (j & 1))) & 0xffffu;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (k + j < p.K) h[j] = __bfloat16_as_ushort(src[j]);
      }
    }
    const int at = (o / 8) * (NT * 128) + m * 128 + ((16 * (o % 8)) ^ ((m & 7) << 4));
    *reinterpret_cast<uint4*>(xs + at) = make_uint4(h[0] | (h[4] << 16), h[1] | (h[5] << 16), h[2] | (h[6] << 16), h[3] | (h[7] << 16));
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

template <int NT, int G>
__global__ void __launch_bounds__(Shape<NT>::THREADS, 1) matvec_int4_kernel(const __grid_constant__ CUtensorMap map_q, const Params p) {
  constexpr int WG = Shape<NT>::WG, NG = CHUNK / G, OWN = NT / WG;      // OWN: rows of x that a warpgroup finishes
  using TM = Tmem<NT, G>;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* xs = smem + p.stages * STAGE_BYTES;
  float* sums = reinterpret_cast<float*>(xs + (size_t)p.seg * NT * 2);  // [WG - 1][NT][ROWS]
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(sums + (WG - 1) * NT * ROWS);
  const uint32_t full0 = smem_u32(bars), empty0 = smem_u32(bars + 16), a0 = smem_u32(bars + 32), d0 = smem_u32(bars + 36);
  const uint32_t sum_full = smem_u32(bars + 40), sum_free = smem_u32(bars + 41), x_free = smem_u32(bars + 42), x_full = smem_u32(bars + 43);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 44);
  const WaitCtl wc{reinterpret_cast<volatile int*>(tmem_slot + 1), p.wait_ns};
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < p.stages; ++i) { mbar_init(full0 + 8 * i, 1); mbar_init(empty0 + 8 * i, 8); }
    for (int i = 0; i < WG; ++i) { mbar_init(a0 + 8 * i, 4); mbar_init(d0 + 8 * i, 1); }
    mbar_init(sum_full, WG * 4);
    mbar_init(sum_free, WG * 4);
    mbar_init(x_free, WG * 4);
    mbar_init(x_full, WG * 4);
    *wc.flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "n"(TM::COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (p.nseg == 1 && p.M <= NT) load_x<NT>(p, xs, 0, 0, tid, Shape<NT>::THREADS);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = *tmem_slot;
  // A tile is 128 rows of the weights times NT rows of x; the blocks of x are the slow index.  Its chunks are counted in pairs (a stage).
  const int tiles_n = (p.N + ROWS - 1) / ROWS, tiles = tiles_n * ((p.M + NT - 1) / NT), pairs = (p.K + 255) / 256, seg_pairs = p.seg / 256;

  if (warp == 0) {
    // ------------------------------------------------------------------ weights
    if (!(p.inject & DPPO_INJECT_NO_COPIES)) {
      int s = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
        const int n0 = (tile % tiles_n) * ROWS;
        for (int c = 0; c < pairs; ++c) {
          if (!mbar_wait_warp(empty0 + 8 * s, ph ^ 1u, wc)) { ok = false; break; }
          if (lane == 0) {
            mbar_arrive_expect_tx(full0 + 8 * s, STAGE_BYTES);
            gemm::tma_load_2d(smem_u32(smem) + s * STAGE_BYTES, &map_q, c * 128, n0, full0 + 8 * s);
          }
          if (++s == p.stages) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMAs
    constexpr uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(NT >> 3) << 17) | ((uint32_t)(ROWS >> 4) << 24);
    const uint64_t xdesc = gemm::make_desc_k_sw128(smem_u32(xs));
    uint32_t use = 0;                                      // chunks of each warpgroup so far (its phase)
    int g = 0;
    bool ok = true;
    for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
      for (int c = 0; c < 2 * pairs; ++c) {
        ok = mbar_wait_warp(a0 + 8 * g, use & 1u, wc);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const int k = (c % (2 * seg_pairs)) * CHUNK;       // within the segment
        const uint32_t ta = tmem + g * (TM::A + TM::D), td = ta + TM::A;
        if (elect_one()) {
#pragma unroll
          for (int i = 0; i < CHUNK / 16; ++i) {           // 16 codes an MMA
            const int at = (k + 16 * i) / XSPAN * (NT * 128) + (16 * i) % XSPAN * 2;
            mma_ts(td + (16 * i) / G * NT, ta + 8 * i, xdesc + (uint64_t)(at >> 4), idesc, (16 * i) % G != 0);
          }
          gemm::mma_commit(d0 + 8 * g);
        }
        __syncwarp();
        if (++g == WG) { g = 0; ++use; }
      }
    }
  } else {
    // ------------------------------------------------------------------ conversion and sums
    const int g = (warp - 2) >> 2, q = warp & 3, r = q * 32 + lane;     // warpgroup; a warp's lanes of tensor memory are given by its number
    const uint32_t ta = tmem + ((uint32_t)(q * 32) << 16) + g * (TM::A + TM::D), td = ta + TM::A;
    uint32_t n_d = 0, n_tile = 0, n_x = 0;                 // products awaited, tiles finished, segments of x loaded
    int s0 = 0;                                            // stage of the tile's first pair
    uint32_t ph0 = 0;
    int turn = 0;                                          // warpgroup of the tile's first chunk
    int x_now = p.nseg == 1 && p.M <= NT ? 0 : -1;         // which part of x (block of rows, segment) shared memory holds
    bool ok = true;
    for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
      const int n = (tile % tiles_n) * ROWS + r, m0 = (tile / tiles_n) * NT;
      const __nv_bfloat16* srow = p.scale + (int64_t)(n < p.N ? n : 0) * p.lds;
      float acc[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[j] = 0.f;
      float sc[NG] = {};                                   // scales of the product under way
      bool under_way = false;
      auto take_product = [&]() {
        if (!under_way) return true;
        if (!mbar_wait_warp(d0 + 8 * g, n_d & 1u, wc)) return false;
        ++n_d;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
        for (int h = 0; h < NG; ++h)
#pragma unroll
          for (int j0 = 0; j0 < NT; j0 += 16) {
            uint32_t v[16];
            tmem_ld16(td + h * NT + j0, v);
#pragma unroll
            for (int j = 0; j < 16; j += 2) {
              const float2 a = __ffma2_rn(make_float2(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), make_float2(sc[h], sc[h]), make_float2(acc[j0 + j], acc[j0 + j + 1]));
              acc[j0 + j] = a.x;
              acc[j0 + j + 1] = a.y;
            }
          }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        under_way = false;
        return true;
      };
      for (int seg = 0; seg < p.nseg && ok; ++seg) {
        const int x_want = (tile / tiles_n) * p.nseg + seg;
        if (x_now != x_want) {
          // once every warpgroup has seen its last product with the part before
          ok = take_product();
          if (!ok) break;
          __syncwarp();
          if (lane == 0) mbar_arrive(x_free);
          ok = mbar_wait_warp(x_free, n_x & 1u, wc);
          if (!ok) break;
          load_x<NT>(p, xs, m0, seg * p.seg, tid - 64, WG * 128);
          __syncwarp();
          if (lane == 0) mbar_arrive(x_full);
          ok = mbar_wait_warp(x_full, n_x & 1u, wc);
          if (!ok) break;
          ++n_x;
          x_now = x_want;
        }
        const int c_end = min(2 * pairs, 2 * seg_pairs * (seg + 1));
        for (int c = 2 * seg_pairs * seg + ((g - turn - 2 * seg_pairs * seg % WG + 2 * WG) % WG); c < c_end; c += WG) {
          const int pair = s0 + c / 2, s = pair % p.stages;
          const uint32_t ph = (ph0 + (uint32_t)(pair / p.stages)) & 1u;
          float nsc[NG];
#pragma unroll
          for (int h = 0; h < NG; ++h) {
            const int gi = c * NG + h;
            nsc[h] = (n < p.N && gi < p.groups) ? __bfloat162float(__ldg(srow + gi)) : 0.f;
          }
          ok = mbar_wait_warp(full0 + 8 * s, ph, wc);
          if (!ok) break;
          const uint32_t src = smem_u32(smem) + s * STAGE_BYTES + r * 128;
          uint4 w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = lds128(src + ((((c & 1) * 4 + i) ^ (r & 7)) << 4));
          __syncwarp();
          if (lane == 0) mbar_arrive(empty0 + 8 * s);
          uint32_t v[32];
          convert(w[0].x, v);
          convert(w[0].y, v + 4);
          convert(w[0].z, v + 8);
          convert(w[0].w, v + 12);
          convert(w[1].x, v + 16);
          convert(w[1].y, v + 20);
          convert(w[1].z, v + 24);
          convert(w[1].w, v + 28);
          ok = take_product();                             // of the chunk before: its operand may be overwritten now
          if (!ok) break;
          tmem_st32(ta, v);
          convert(w[2].x, v);
          convert(w[2].y, v + 4);
          convert(w[2].z, v + 8);
          convert(w[2].w, v + 12);
          convert(w[3].x, v + 16);
          convert(w[3].y, v + 20);
          convert(w[3].z, v + 24);
          convert(w[3].w, v + 28);
          tmem_st32(ta + 32, v);
          asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(a0 + 8 * g);
#pragma unroll
          for (int h = 0; h < NG; ++h) sc[h] = nsc[h];
          under_way = true;
        }
      }
      if (!ok || !take_product()) break;
      s0 += pairs;
      ph0 += (uint32_t)(s0 / p.stages);
      s0 %= p.stages;
      turn = (turn + 2 * pairs) % WG;
      // the warpgroups' sums: each leaves those of the others' rows of x, and finishes its own
      if (n_tile > 0 && !mbar_wait_warp(sum_free, (n_tile - 1u) & 1u, wc)) break;
      const int live = min(NT, p.M - m0);
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int owner = j / OWN;
        if (owner != g && j < live) sums[((g < owner ? g : g - 1) * NT + j) * ROWS + r] = acc[j];
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(sum_full);
      if (!mbar_wait_warp(sum_full, n_tile & 1u, wc)) break;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        if (j / OWN == g && j < live) {
          float v = 0.f;                                   // in the order of the warpgroups, whoever adds
#pragma unroll
          for (int o = 0; o < WG; ++o) v += o == j / OWN ? acc[j] : sums[((o < j / OWN ? o : o - 1) * NT + j) * ROWS + r];
          if (n < p.N) {
            if (p.y_bf16) reinterpret_cast<__nv_bfloat16*>(p.y)[(int64_t)(m0 + j) * p.ldy + n] = __float2bfloat16_rn(v);
            else reinterpret_cast<float*>(p.y)[(int64_t)(m0 + j) * p.ldy + n] = v;
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(sum_free);
      ++n_tile;
    }
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
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(TM::COLS) : "memory");
  }
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

template <int NT, int G>
cudaError_t launch(Params p, const unsigned char* q, int64_t ldq, int sms, int smem_most, cudaStream_t st) {
  CUtensorMap map;
  const cuuint64_t dims[2] = {(cuuint64_t)((p.K + 1) / 2), (cuuint64_t)p.N}, strides[1] = {(cuuint64_t)ldq};
  const cuuint32_t box[2] = {128u, (cuuint32_t)ROWS}, ones[2] = {1u, 1u};
  EncodeFn enc = get_encode();
  if (!enc || enc(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<unsigned char*>(q), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  constexpr int WG = Shape<NT>::WG, FIXED = (WG - 1) * NT * ROWS * 4 + 512 + 1024;
  // x for all of K where at least four stages are left besides it, else as much of K as leaves that many
  const int room = smem_most - FIXED, whole = (p.K + 255) / 256 * 256;
  p.seg = (room - 4 * STAGE_BYTES) / (NT * 2) / 256 * 256;
  if (p.seg > whole) p.seg = whole;
  p.nseg = (whole + p.seg - 1) / p.seg;
  p.stages = (room - p.seg * NT * 2) / STAGE_BYTES;
  if (p.stages > 12) p.stages = 12;
  const int smem = p.stages * STAGE_BYTES + p.seg * NT * 2 + FIXED;
  const int64_t tiles = (int64_t)((p.N + ROWS - 1) / ROWS) * ((p.M + NT - 1) / NT);
  auto kernel = matvec_int4_kernel<NT, G>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  kernel<<<(unsigned)(tiles < sms ? tiles : sms), Shape<NT>::THREADS, smem, st>>>(map, p);
  return cudaGetLastError();
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
