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
  int64_t slots;             // pairs of pieces of 8 columns of a row, a whole number of groups
  int step_rows, step_slots; // kQThreads pairs further on
  int x_whole, q_whole, v_whole;   // 16-byte loads, 4-byte stores, 16-byte stores of values allowed
};

constexpr int kQThreads = 256, kQItems = 2;

// amax / 7 rounded to bf16 once, ties to even: the bf16 number below an approximate quotient (it may be one off where the quotient is next to a bf16
// number, which the choice between it and the next one makes good), and the sign of amax - 7 (the middle above it), which one fma gives exactly
__device__ __forceinline__ float group_scale(float amax) {
  const uint32_t below = __float_as_uint(amax * 0.14285715f) & 0xffff0000u;
  const float d = fmaf(-7.f, __uint_as_float(below | 0x8000u), amax);
  return __uint_as_float(below + (d > 0.f || (d == 0.f && (below & 0x10000u)) ? 0x10000u : 0u));
}
__device__ __forceinline__ float about_one_over(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
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
// Eight numbers to a word of codes, and their values.  fp32: one by one.
__device__ __forceinline__ uint32_t codes_of(const float2* x, float scale, float inv, float2* val) {
  uint32_t w = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int c0 = code_of(x[j].x, scale, inv), c1 = code_of(x[j].y, scale, inv);
    w |= (uint32_t)(c0 + 8) << (8 * j) | (uint32_t)(c1 + 8) << (8 * j + 4);
    val[j] = make_float2((float)c0 * scale, (float)c1 * scale);
  }
  return w;
}
// bf16: x / scale is a quotient of two 8-bit mantissas, so it is the middle of two whole numbers or at least 2^-10 away from it (|2 x - (2 k + 1) scale| is
// a multiple of half of scale's last place at least).  So the product with the reciprocal, off by less than 2^-19, is first rounded to
// a multiple of 2^-11, which makes a middle exact, and then to a whole number, ties to even; both by adding 1.5 2^23 units.  The second sum's
// low bits are the code, and a word's codes are the sum of those bits, shifted, less what the rest of the bits come to.
__device__ __forceinline__ uint32_t codes_of_bf16(const float2* x, float scale, float inv, float2* val) {
  constexpr float FINE = 6144.f, WHOLE = 12582912.f + 8.f;
  constexpr uint32_t REST = 0x4B400000u + (0x4B400000u << 4) + (0x4B400000u << 8);
  const float2 s2 = make_float2(scale, scale), i2 = make_float2(inv, inv), f2 = make_float2(FINE, FINE), nf2 = make_float2(-FINE, -FINE);
  const float2 w2 = make_float2(WHOLE, WHOLE), nw2 = make_float2(-WHOLE, -WHOLE);
  uint32_t w = 0u - REST;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 b = __fadd2_rn(__fadd2_rn(__ffma2_rn(x[j], i2, f2), nf2), w2);
    val[j] = __fmul2_rn(__fadd2_rn(b, nw2), s2);
    w += (__float_as_uint(b.x) << (8 * j)) + (__float_as_uint(b.y) << (8 * j + 4));
  }
  return w;
}

// Bound by HBM: 151936 x 2048 bf16 in groups of 128 with the values, 1.41 GB, in 225 us, 97 % of the measured copy rate.  (With a piece to a thread, two
// divisions a piece for its place and two for its scale it was bound by the issue slots: 590 us with the fp32 way to the codes, 311 with the bf16 one.)
// A thread has pairs of pieces of 8 columns of a group, G / 2 columns apart, all of them loaded before the first is used; a group's G / 16 pairs lie in
// neighbouring lanes, whose loads are whole sectors.
template <typename InT, int G>
__global__ void __launch_bounds__(kQThreads) int4_quantize_kernel(QuantParams p) {
  constexpr bool BF16 = sizeof(InT) == 2;
  constexpr int LANES = G / 16, WORDS = BF16 ? 1 : 2;      // 16-byte words of a piece
  const InT* X = reinterpret_cast<const InT*>(p.x);
  InT* Vv = reinterpret_cast<InT*>(p.values);
  const uint32_t slots = (uint32_t)p.slots, cols = (uint32_t)p.cols;
  const int64_t first = (int64_t)blockIdx.x * (kQThreads * kQItems);
  int64_t row0 = first / slots;
  const uint32_t at0 = (uint32_t)(first - row0 * slots) + threadIdx.x, r0 = at0 / slots;
  row0 += r0;
  const uint32_t slot0 = at0 - r0 * slots;
  uint4 raw[kQItems][2][WORDS];
  {
    int64_t row = row0;
    uint32_t slot = slot0;
#pragma unroll
    for (int k = 0; k < kQItems; ++k) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t col = slot / LANES * G + slot % LANES * 8 + h * (G / 2);
#pragma unroll
        for (int u = 0; u < WORDS; ++u) raw[k][h][u] = make_uint4(0u, 0u, 0u, 0u);
        if (row < p.rows) {
          const InT* src = X + row * p.ldx + col;
          if (p.x_whole && col + 8 <= cols) {
#pragma unroll
            for (int u = 0; u < WORDS; ++u) raw[k][h][u] = ldg128_stream(src + u * 4);
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (col + j < cols) set_raw(raw[k][h][BF16 ? 0 : j / 4], BF16 ? j : j % 4, src[j]);
          }
        }
      }
      row += p.step_rows;
      slot += p.step_slots;
      if (slot >= slots) { slot -= slots; ++row; }
    }
  }
  int64_t row = row0;
  uint32_t slot = slot0;
#pragma unroll
  for (int k = 0; k < kQItems; ++k) {
    RawMax<InT> most;
    most.m = {};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int u = 0; u < WORDS; ++u) {
        constexpr uint32_t MAGNITUDE = BF16 ? 0x7fff7fffu : 0x7fffffffu;
        const uint4& v = raw[k][h][u];
        most.add(make_uint4(v.x & MAGNITUDE, v.y & MAGNITUDE, v.z & MAGNITUDE, v.w & MAGNITUDE));
      }
    float amax = most.value();
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    const uint32_t group = slot / LANES, col = group * G + slot % LANES * 8;
    if (row < p.rows) {
      const bool bad = !(amax <= 3.4028234e38f);
      const float scale = bad ? NAN : group_scale(fmaxf(amax, 7.888609052210118e-31f)), inv = about_one_over(scale);
      if (slot % LANES == 0) {
        p.scale[row * p.lds + group] = __float2bfloat16_rn(scale);
        if (bad) atomicOr(p.status, DPPO_STATUS_NONFINITE_ROW);
      }
      unsigned char* q = p.q + row * p.ldq + col / 2;
      InT* out = Vv + row * p.ldv + col;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int n = min(8, (int)cols - (int)(col + h * (G / 2)));
        if (n <= 0) break;                 // (a piece of the last group may lie behind the row)
        float2 x[4], val[4];
#pragma unroll
        for (int u = 0; u < WORDS; ++u) to_pairs<InT>(raw[k][h][u], x + 2 * u);
        uint32_t w = BF16 ? codes_of_bf16(x, scale, inv, val) : codes_of(x, scale, inv, val);
        if (bad) w = 0x88888888u;
        if (n < 8) w &= (1u << (4 * n)) - 1u;
        unsigned char* dst = q + h * (G / 4);
        if (n == 8 && p.q_whole) {
          *reinterpret_cast<uint32_t*>(dst) = w;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (2 * j < n) dst[j] = (unsigned char)(w >> (8 * j));
        }
        if (Vv) {
          InT* to = out + h * (G / 2);
          if (n == 8 && p.v_whole) {
            Store<InT, 8>::run(to, 0u, reinterpret_cast<const float*>(val));
          } else {
            const float* one = reinterpret_cast<const float*>(val);
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (j < n) to[j] = from_f32<InT>(one[j]);
          }
        }
      }
    }
    row += p.step_rows;
    slot += p.step_slots;
    if (slot >= slots) { slot -= slots; ++row; }
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
// D[n, m] = sum over a group of (code[n, k] - 8) x[m, k] for up to 128 rows n of the weights and a few rows m of x at a time: the weights are the
// operand with the many rows.  They come as they are stored by tensor copies (rows x 256 codes, 128-byte swizzle) into a ring; a thread per
// row turns a chunk of its codes into the tensor cores' type in registers and writes them to tensor memory, where tcgen05.mma takes its A
// operand from; x lies in shared memory for the whole launch.  The product of a group is read back, scaled by the row's scale (a thread's own)
// and added up in fp32 registers.  One persistent CTA per SM:
//   warp 0          tensor copies of the weights
//   warps 1 .. L    issue the MMAs (the first allocates tensor memory)
//   L x 4 warps     conversion
//   P x 4 warps     products: scale, add up, store
// Chunk i belongs to line i % L: a converting warpgroup, an issuing warp and B buffers in tensor memory, which each take their chunks in
// order.  (Barrier phases are known by their parity, which would not do for a line that could fall two uses of a buffer behind.  With one
// issuing warp the tensor cores stood still while it found its barriers ready, 150 cycles each.)
// Where x does not fit, a pair of CTAs (a cluster) shares a tile, each half of K, and they exchange the sums of half of x's rows through
// distributed shared memory; where that is not enough either, x is loaded again for each part of K.
//
// Two ways to the same sums:
//   bf16   A word of 8 codes c0 .. c7 gives the pairs (c0, c4), (c1, c5), (c2, c6), (c3, c7): a mask and an or put a code into the low mantissa bits of
//          the bf16 number 128, and subtracting 136 leaves code - 8, exactly.  11 instructions a word, chunks of 128 codes.
//   int8   (up to 4 rows of x) The codes stay whole numbers: two masks and a shift give a word's 8 bytes.  x is written as four signed 8-bit digits in
//          units of 2^-29 of the power of two at the largest entry of its group, a row of the operand each; the int32 products are exact, and
//          8 times the sum of the digits is taken off, exactly.  That holds entries down to 2^-22 of the largest with all of their 8 bits.  A group
//          with smaller ones, which may be all of its sum where the large one's weight is zero, is summed by the products' threads from x and
//          the codes as they stand, in fp32.  (Of groups of standard normal x one in 20000 to 80000.  151936 x 2048, one row: 31 us, with one
//          such group of the 16 49 us, with nothing else 191 us.)
//
// What bounds it, 151936 x 2048 in groups of 128 (166 MB; 25 us at the measured copy rate), calls back to back:
//   1 row     31 us.  A launch, x and the first weights take 5 us; then 4 warps convert, and 8 take the products of, 256 codes of 115 rows in some 650
//             cycles, where HBM delivers them in 640.
//   16 rows   55 us, 61 rows 81 us.  The issue slots (62 % busy with 61 rows, the rest latency from one warp to the next): a chunk of 128 codes costs
//             16 words x 11 instructions of conversion, and the products' warps some 100 each around their sums.  The tensor cores are not the
//             bound: an MMA takes 47 cycles with up to 96 columns, of bf16 (K = 16) as of int8 (K = 32): 374 cycles a chunk for bf16, 187 for int8, of
//             the 760 that it takes.
// Up to four rows, groups of 128: 31, 35, 41 us for 1, 2, 4 rows; groups of 32: 44 us for one row, 90 for four.
// Tried and left: the chunks' products in rotation over two or three parts for bf16 (32 rows 64 -> 72 us: more warps for the same issue slots), three or
// four lines for int8 (31 -> 33 us), int8 for 8 and 16 rows (see launch_rows), groups that digits do not hold within the loop over chunks.
//
// x is laid out in the order that the conversion makes of k.
namespace mv {

constexpr int LANES = 128;                 // rows of a tile at most
constexpr int STAGE_BYTES = LANES * 128;   // 256 codes of each row
constexpr int DIGITS = 4;

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
  int pairs;                               // blocks of 256 codes of a CTA
  int scales_together;                     // a chunk's scales lie on a boundary of their size
  const unsigned char* q;                  // the codes once more, for groups that are summed without the tensor cores
  int64_t ldq;
  int32_t* status;
  unsigned long long wait_ns;
  int inject;
};

// NT: columns of an MMA (bf16: rows of x; int8: DIGITS to a row of x)
template <int NT, int G, bool I8> struct Shape {
  static constexpr int XROWS = I8 ? NT / DIGITS : NT;                            // rows of x
  static constexpr int CHUNK = I8 ? 256 : 128, PER = 256 / CHUNK;      // codes that a thread converts at a time; chunks of a stage
  static constexpr int STEP = I8 ? 32 : 16;                            // codes of an MMA
  static constexpr int XBYTES = I8 ? NT : 2 * NT;                      // of shared memory for a code
  static constexpr int XSPAN = I8 ? 128 : 64;                          // codes of a swizzled block of x
  static constexpr int NG = CHUNK / G;
  // Warpgroups for the products: E share the rows of x.  int8: SPLIT parts, one for each line, whose sums meet at the tile's end (39 us for a row by one
  // part, 31 by two).  bf16: TURNS sets, which take tiles in rotation, so that one stores while the other adds up (61 rows: 110 us with one set, 81
  // with two); a single set for 17 to 32 rows, whose two warpgroups of 16 rows leave no registers for four (32 rows: 64 us, and 68 with two sets).
  static constexpr int E = I8 || NT == 16 ? 1 : 2, EN = XROWS / E, SPLIT = I8 ? 2 : 1, TURNS = I8 || NT == 32 ? 1 : 2;
  static constexpr int PRODUCTS = E * SPLIT * TURNS;                // in all; E of a chunk
  static constexpr int A = 64, D = NG * NT, COLS = A + D;              // columns of tensor memory of a chunk: operand, products
  // Lines and buffers: six buffers of tensor memory in three lines where they fit (16 rows 55 us; four lines of one buffer 66 us), else four.
  static constexpr int L = !I8 && NT == 16 ? (COLS * 6 <= 512 ? 3 : 4) : 2;
  static constexpr int B = COLS * 2 * L <= 512 ? 2 : 1;
  static constexpr int BUFS = L * B;
  static constexpr int THREADS = 32 + 32 * L + (L + PRODUCTS) * 128;
  static_assert(BUFS * COLS <= 512, "tensor memory");
};

__device__ __forceinline__ uint32_t elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p;
}
// Whether a phase is over, asked ahead of the wait for it, so that the answer comes while something else is done.
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool mbar_wait_warp(bool over, uint32_t bar, uint32_t parity, const WaitCtl& w) {
  return __all_sync(0xffffffffu, over) || dppo::mbar_wait_warp(bar, parity, w);
}
// A from tensor memory
template <bool I8> __device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  if (I8)
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::i8 [%0], [%1], %2, %3, p;\n}\n"
                 ::"r"(d), "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
  else
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
__device__ __forceinline__ void tmem_ld4(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];\n" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(taddr));
}
// What the loads before brought is there.  (It names their registers: the compiler sees no other reason to use, or to spill, them after it.)
template <int N> __device__ __forceinline__ void tmem_ld_wait(uint32_t* r) {
  static_assert(N % 4 == 0, "");
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; i += 4) asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]));
}
// the 8 codes of a word as four bf16 pairs (c0, c4), (c1, c5), (c2, c6), (c3, c7), less 8
__device__ __forceinline__ void convert_bf16(uint32_t w, uint32_t* r) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t v;
    asm("lop3.b32 %0, %1, 0x000f000f, 0x43004300, 0xea;" : "=r"(v) : "r"(w >> (4 * i)));
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r[i]) : "r"(v), "r"(0x43084308u));
  }
}
// the same as bytes (c0, c2, c4, c6), (c1, c3, c5, c7)
__device__ __forceinline__ void convert_i8(uint32_t w, uint32_t* r) {
  r[0] = w & 0x0f0f0f0fu;
  r[1] = (w >> 4) & 0x0f0f0f0fu;
}
// half of a chunk: 32 columns
template <bool I8> __device__ __forceinline__ void convert_half(const uint4* w, uint32_t* v) {
#pragma unroll
  for (int j = 0; j < (I8 ? 4 : 2); ++j) {
    if (I8) {
      convert_i8(w[j].x, v + 8 * j);
      convert_i8(w[j].y, v + 8 * j + 2);
      convert_i8(w[j].z, v + 8 * j + 4);
      convert_i8(w[j].w, v + 8 * j + 6);
    } else {
      convert_bf16(w[j].x, v + 16 * j);
      convert_bf16(w[j].y, v + 16 * j + 4);
      convert_bf16(w[j].z, v + 16 * j + 8);
      convert_bf16(w[j].w, v + 16 * j + 12);
    }
  }
}

// bf16: x rows m0 .. m0 + NT - 1, codes k0 .. k0 + seg - 1 of K, into shared memory: blocks of 64 codes, NT rows of 128 bytes each, 128-byte
// swizzle, and within 8 codes the order that the conversion makes of them.  Rows and codes that there are not are zero.
template <int NT, int WARPS>
__device__ __forceinline__ void load_x(const Params& p, unsigned char* xs, int m0, int k0, int warp, int lane) {
  constexpr int AT_ONCE = 8;               // loads in flight
  const int blocks = p.seg / 256, all = NT * blocks;       // a warp takes 256 codes of a row, 8 to a lane
  for (int i0 = warp; i0 < all; i0 += AT_ONCE * WARPS) {
    uint4 v[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int i = i0 + u * WARPS, m = i / blocks, k = k0 + (i - m * blocks) * 256 + 8 * lane;
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
      const int i = i0 + u * WARPS, m = i / blocks, o = (i - m * blocks) * 32 + lane;
      if (i >= all) break;
      const int at = (o / 8) * (NT * 128) + m * 128 + ((16 * (o % 8)) ^ ((m & 7) << 4));
      // (0, 4), (1, 5), (2, 6), (3, 7)
      *reinterpret_cast<uint4*>(xs + at) = make_uint4(__byte_perm(v[u].x, v[u].z, 0x5410), __byte_perm(v[u].x, v[u].z, 0x7632), __byte_perm(v[u].y, v[u].w, 0x5410),
                                                      __byte_perm(v[u].y, v[u].w, 0x7632));
    }
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// int8: the same for XROWS rows as digits (row 4 m + digit of the operand) in blocks of 128 codes, and for each group and row of x what
// the products need: -8 times the sum of the lower two digits (the second 256-fold) and of the upper two, and the group's unit.  A warp per row and
// group.  A group with an entry that is no whole number of units has zeros for digits and a negative unit, and is announced.  An entry that is no number,
// or infinite, makes the unit NaN.
template <int NT, int XROWS, int G, int WARPS>
__device__ __forceinline__ void load_x_digits(const Params& p, unsigned char* xs, int4* table, int* odd, int m0, int k0, int warp, int lane) {
  constexpr int AT_ONCE = 4;
  const int rows = min(XROWS, p.M - m0), all = p.seg / G * rows;           // (columns of rows that there are not are never read)
  for (int u0 = warp; u0 < all; u0 += AT_ONCE * WARPS) {
    float v[AT_ONCE][G / 32];
#pragma unroll
    for (int a = 0; a < AT_ONCE; ++a) {
      const int u = u0 + a * WARPS, gi = u / rows, m = u - gi * rows;
#pragma unroll
      for (int j = 0; j < G / 32; ++j) {
        const int k = k0 + gi * G + 32 * j + lane;
        v[a][j] = u < all && k < p.K ? __bfloat162float(p.x[(int64_t)(m0 + m) * p.ldx + k]) : 0.f;
      }
    }
#pragma unroll
    for (int a = 0; a < AT_ONCE; ++a) {
      const int u = u0 + a * WARPS, gi = u / rows, m = u - gi * rows, kg = gi * G;
      if (u >= all) break;
      float top = 0.f;
#pragma unroll
      for (int j = 0; j < G / 32; ++j) top = max_nan(top, fabsf(v[a][j]));
      top = warp_max_nan(top);
      const bool bad = !(top <= 3.4028234e38f);
      // unit 2^(e - 29) for a largest entry in [2^e, 2^(e + 1)), not below 2^-133, of which every bf16 number is a multiple; 1 / unit in two steps, as it
      // may be beyond fp32
      const int e = max((int)(__float_as_uint(top) >> 23) - 127, -104);
      const float up = __uint_as_float((uint32_t)(127 + 21 - e) << 23);
      bool whole = true;
#pragma unroll
      for (int j = 0; j < G / 32; ++j) {
        v[a][j] = v[a][j] * up * 256.f;
        whole = whole && rintf(v[a][j]) == v[a][j];
      }
      whole = __all_sync(0xffffffffu, whole);
      int sum[DIGITS] = {};
#pragma unroll
      for (int j = 0; j < G / 32; ++j) {
        int X = whole ? __float2int_rn(v[a][j]) : 0;
        const int k = kg + 32 * j + lane, byte = (k & 127 & ~7) + ((k & 1) * 4 + ((k & 7) >> 1));
#pragma unroll
        for (int d = 0; d < DIGITS; ++d) {
          const int digit = d == DIGITS - 1 ? X : ((X + 128) & 255) - 128, row = DIGITS * m + d;
          X = (X - digit) >> 8;
          sum[d] += digit;
          xs[k / 128 * (NT * 128) + row * 128 + (byte ^ ((row & 7) << 4))] = (unsigned char)digit;
        }
      }
#pragma unroll
      for (int d = 0; d < DIGITS; ++d) sum[d] = __reduce_add_sync(0xffffffffu, sum[d]);
      const uint32_t unit = e >= -97 ? (uint32_t)(127 + e - 29) << 23 : 1u << (e + 120);
      if (lane == 0) {
        table[gi * XROWS + m] = make_int4(-8 * (sum[0] + 256 * sum[1]), -8 * (sum[2] + 256 * sum[3]), (int)(bad ? 0x7fc00000u : (whole ? unit : unit | 0x80000000u)), 0);
        if (!whole && !bad) *odd = 1;
      }
    }
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// The sum of a group as it stands: n entries of x, their codes from q on, on a 16-byte boundary.
template <int G> __device__ __noinline__ float group_sum(const __nv_bfloat16* x, const unsigned char* q, int n) {
  float s = 0.f;
  if (n >= G) {
    uint4 w[G / 32];
#pragma unroll
    for (int j = 0; j < G / 32; ++j) w[j] = *reinterpret_cast<const uint4*>(q + 16 * j);
#pragma unroll
    for (int j = 0; j < G; ++j) s = fmaf(__bfloat162float(x[j]), (float)((int)(word_of(w[j / 32], j / 8 % 4) >> (4 * (j % 8)) & 15u) - 8), s);
  } else {
    for (int j = 0; j < n; ++j) s = fmaf(__bfloat162float(x[j]), (float)((int)(q[j / 2] >> (4 * (j % 2)) & 15u) - 8), s);
  }
  return s;
}

struct Bars {
  unsigned long long full[12], empty[12];  // stages of weights
  unsigned long long ready[6], done[6];    // chunk: operand written and the buffer's products before read; MMAs done (operand free, products there)
  unsigned long long x_free, x_full;       // x replaced
  unsigned long long turn[2];              // two sets: the other has read its tile's last products.  Two parts: the second's sums are there; read
  unsigned long long sum_full[2], sum_free[2];       // pairs of CTAs, by whose turn it is: the other's sums are here; read by the other
  uint32_t tmem;
  int abort_flag;
  int odd;                                 // int8: x has a group that digits do not hold
};

template <int NT, int G, int CL, bool I8>
__global__ void __launch_bounds__(Shape<NT, G, I8>::THREADS, 1) matvec_int4_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ Params p) {
  using S = Shape<NT, G, I8>;
  constexpr int NG = S::NG, L = S::L, B = S::B, BUFS = S::BUFS, COLS = S::COLS, EN = S::EN, OWN = EN / CL, PER = S::PER, XROWS = S::XROWS, TURNS = S::TURNS;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* xs = smem + p.stages * STAGE_BYTES;
  int4* table = reinterpret_cast<int4*>(xs + (size_t)p.seg * S::XBYTES);                       // int8: [groups of seg][XROWS]
  float* meet = reinterpret_cast<float*>(table + (I8 ? p.seg / G * XROWS : 0));              // int8: [XROWS][LANES], from the second part
  float* sums = meet + (I8 ? XROWS * LANES : 0);                                             // pairs of CTAs: [TURNS][E][OWN][LANES], from the other
  Bars* bars = reinterpret_cast<Bars*>(sums + (CL > 1 ? TURNS * S::E * OWN * LANES : 0));
  const uint32_t full0 = smem_u32(bars->full), empty0 = smem_u32(bars->empty), ready0 = smem_u32(bars->ready), done0 = smem_u32(bars->done);
  const uint32_t x_free = smem_u32(&bars->x_free), x_full = smem_u32(&bars->x_full);
  const WaitCtl wc{&bars->abort_flag, p.wait_ns};
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = CL > 1 ? (int)cluster_ctarank() : 0;
  if (tid == 0) {
    for (int i = 0; i < 12; ++i) { mbar_init(full0 + 8 * i, 1); mbar_init(empty0 + 8 * i, 4 * PER); }
    for (int i = 0; i < 6; ++i) { mbar_init(ready0 + 8 * i, 4 + 4 * S::E); mbar_init(done0 + 8 * i, 1); }
    mbar_init(x_free, L * 4);
    mbar_init(x_full, L * 4);
    for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&bars->turn[i]), 4 * S::E);
    for (int i = 0; i < TURNS; ++i) { mbar_init(smem_u32(&bars->sum_full[i]), 1); mbar_init(smem_u32(&bars->sum_free[i]), 4 * S::E); }
    bars->abort_flag = 0;
    bars->odd = 0;
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
  // A tile is `rows` rows of the weights times XROWS rows of x; the blocks of x are the slow index.
  const int tiles_n = (p.N + p.rows - 1) / p.rows, tiles = tiles_n * ((p.M + XROWS - 1) / XROWS);
  const int pair0 = rank * p.pairs, pairs = max(0, min(p.pairs, (p.K + 255) / 256 - pair0));      // this CTA's part of K
  const int first = blockIdx.x / CL, grid = gridDim.x / CL;
  const int mine = first < tiles ? (tiles - first + grid - 1) / grid : 0;                         // tiles of this CTA
  const int per_tile = PER * pairs, per_seg = PER * (p.seg / 256), chunks = mine * per_tile;

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
  } else if (warp <= L) {
    // ------------------------------------------------------------------ MMAs
    const int line = warp - 1;
    // D = fp32, A and B = bf16; or D = int32, A unsigned and B signed 8-bit; both K-major
    constexpr uint32_t idesc = (I8 ? (2u << 4) | (1u << 10) : (1u << 4) | (1u << 7) | (1u << 10)) | ((uint32_t)(NT >> 3) << 17) | ((uint32_t)(LANES >> 4) << 24);
    const uint64_t xdesc = gemm::make_desc_k_sw128(smem_u32(xs));
    int c = line, sub = 0;                 // place in the tile; buffer of the line
    uint32_t ph = 0;
    for (int i = line; i < chunks; i += L) {
      while (c >= per_tile) c -= per_tile;
      int in = c;                          // place in what shared memory holds of x
      while (in >= per_seg) in -= per_seg;
      const uint32_t b = (uint32_t)(line * B + sub), ta = tmem + b * COLS, td = ta + S::A;
      const uint64_t xd = xdesc + (uint64_t)((uint32_t)(in * (S::CHUNK * S::XBYTES)) >> 4);
      if (!mbar_wait_warp(ready0 + 8 * b, ph, wc)) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      if (elect_one()) {
#pragma unroll
        for (int j = 0; j < S::CHUNK / S::STEP; ++j) {     // 32 bytes of a row of x an MMA
          const int at = (S::STEP * j) / S::XSPAN * (NT * 128) + j * 32 % 128;
          mma_ts<I8>(td + (S::STEP * j) / G * NT, ta + 8 * j, xd + (uint64_t)(at >> 4), idesc, (S::STEP * j) % G != 0);
        }
        gemm::mma_commit(done0 + 8 * b);
      }
      __syncwarp();
      c += L;
      if (++sub == B) { sub = 0; ph ^= 1u; }
    }
  } else if (warp < 1 + L + 4 * L) {
    // ------------------------------------------------------------------ conversion
    const int line = (warp - 1 - L) >> 2, q = warp & 3, r = q * 32 + lane;      // (a warp's lanes of tensor memory are given by its number)
    const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16);
    const bool one = p.nseg == 1 && p.M <= XROWS;          // one part of x for everything
    const int parts = one ? (chunks > 0 ? 1 : 0) : mine * p.nseg;
    int x_now = -1;                        // which part of x (block of rows, part of K) shared memory holds
    uint32_t n_x = 0;
    int i = line, at = line, sub = 0;      // next chunk: its number, place in the ring (in chunks) and buffer of the line
    uint32_t ph = 0, bph = 0;
    bool ok = true;
    for (int part = 0; part < parts && ok; ++part) {
      int end = chunks;
      if (!one || x_now < 0) {
        const int t = one ? 0 : part / p.nseg, seg = one ? 0 : part - t * p.nseg, start = t * per_tile + seg * per_seg;
        if (!one) end = t * per_tile + min(per_tile, (seg + 1) * per_seg);
        if (start >= end) continue;        // (a CTA's last part of K may be empty)
        const int block = (first + t * grid) / tiles_n, x_want = block * p.nseg + seg;
        if (x_now != x_want) {
          // once the MMAs with the part before are done: this warpgroup's own last chunk, the others see to theirs
          const int last = i - L, lsub = sub ? sub - 1 : B - 1;
          if (last >= 0 && !mbar_wait_warp(done0 + 8 * (line * B + lsub), sub ? bph : bph ^ 1u, wc)) { ok = false; break; }
          __syncwarp();
          if (lane == 0) mbar_arrive(x_free);
          if (!mbar_wait_warp(x_free, n_x & 1u, wc)) { ok = false; break; }
          const int k0 = (pair0 + seg * (p.seg / 256)) * 256;
          if (I8) load_x_digits<NT, XROWS, G, L * 4>(p, xs, table, &bars->odd, block * XROWS, k0, warp - 1 - L, lane);
          else load_x<NT, L * 4>(p, xs, block * XROWS, k0, warp - 1 - L, lane);
          __syncwarp();
          if (lane == 0) mbar_arrive(x_full);
          if (!mbar_wait_warp(x_full, n_x & 1u, wc)) { ok = false; break; }
          ++n_x;
          x_now = x_want;
        }
      }
      bool over = false;
      for (; i < end; i += L) {
        const int s = at / PER, b = line * B + sub;
        if (!mbar_wait_warp(over, full0 + 8 * s, ph, wc)) { ok = false; break; }
        const uint32_t src = smem_u32(smem) + s * STAGE_BYTES + r * 128;
        constexpr int PIECES = S::CHUNK / 32;              // of 16 bytes
        uint4 w[PIECES];
#pragma unroll
        for (int j = 0; j < PIECES; ++j) w[j] = lds128(src + ((((at % PER) * PIECES + j) ^ (r & 7)) << 4));
        const bool used = mbar_test(done0 + 8 * b, bph ^ 1u);
        at += L;
        if (at >= PER * p.stages) { at -= PER * p.stages; ph ^= 1u; }
        over = mbar_test(full0 + 8 * (at / PER), ph);
        uint32_t v[32];
        convert_half<I8>(w, v);
        if (!mbar_wait_warp(used, done0 + 8 * b, bph ^ 1u, wc)) { ok = false; break; }       // the buffer's operand before has been used
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        tmem_st32(lane_base + b * COLS, v);
        convert_half<I8>(w + PIECES / 2, v);
        tmem_st32(lane_base + b * COLS + 32, v);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        // The stage is given back here, where its codes have been used: with the arrival right behind the loads, before the wait above, codes of
        // the stage's next content turned up among these.
        if (lane == 0) { mbar_arrive(ready0 + 8 * b); mbar_arrive(empty0 + 8 * s); }
        if (++sub == B) { sub = 0; bph ^= 1u; }
      }
    }
  } else {
    // ------------------------------------------------------------------ products
    constexpr int SPLIT = S::SPLIT;
    const int wg = (warp - 1 - L - 4 * L) >> 2, e = wg % S::E, turn = TURNS > 1 ? wg / S::E : 0, part = SPLIT > 1 ? wg : 0, q = warp & 3, r = q * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16) + S::A + (I8 ? 0 : e * EN);
    const uint32_t sum_full = smem_u32(&bars->sum_full[turn]), sum_free = smem_u32(&bars->sum_free[turn]);
    constexpr int PIECE = OWN % 4 == 0 ? 4 : 2;      // rows of x sent together
    float* inbox = sums + (turn * S::E + e) * OWN * LANES + r * PIECE;       // [OWN / PIECE][LANES][PIECE]
    if (turn == 0 && lane == 0)
      for (int i = part * B; i < (SPLIT > 1 ? (part + 1) * B : BUFS); ++i) mbar_arrive(ready0 + 8 * i);      // nothing to be read before a buffer's first use
    const int stride = TURNS * grid;       // between this set's tiles
    uint32_t n_tile = 0;
    bool ok = true;
    int tile = first + turn * grid, tn = tile % tiles_n, block = tile / tiles_n;
    const int ysize = p.y_bf16 ? 2 : 4;
    const int64_t ystep = p.ldy * ysize;
    auto y_at = [&](int n, int m) { return reinterpret_cast<char*>(p.y) + m * ystep + (int64_t)n * ysize; };
    auto put = [&](char* at, float v) {
      if (p.y_bf16) *reinterpret_cast<__nv_bfloat16*>(at) = __float2bfloat16_rn(v);
      else *reinterpret_cast<float*>(at) = v;
    };
    // The row's scales, fetched AHEAD chunks ahead (their latency is that of L2 or of memory), the next tile's first along with this one's last.
    constexpr int AHEAD = I8 ? 2 : 4;
    const int g0 = pair0 * (256 / G), glim = min(max(p.groups - g0, 0), per_tile * NG);           // this CTA's groups
    auto scales_of = [&](int tile_n, bool there) {
      const int n = tile_n * p.rows + r;
      return there && r < p.rows && n < p.N ? reinterpret_cast<const unsigned short*>(p.scale) + (int64_t)n * p.lds + g0 : nullptr;
    };
    // (a register each, and the loads by predicate: nothing here may wait for them)
    uint32_t sc[AHEAD][NG];
    // int8, four or eight groups to a chunk: all at once where they lie so (two to a register then; groups of 32, one row: 64 -> 56 us when x had three digits, 43 us now).
    constexpr bool MANY = I8 && NG >= 4;
    const bool together = MANY && p.scales_together;
    auto fetch = [&](const unsigned short* row, int c, uint32_t* to) {
      if constexpr (MANY) {
        if (together) {
          const unsigned short* src = row + c * NG;
          const int there = row ? min(max(glim - c * NG, 0), NG) : 0;
#pragma unroll
          for (int h = 0; h < NG; ++h) to[h] = 0u;
          if (there == NG) {
            if (NG == 8) asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(to[0]), "=r"(to[1 % NG]), "=r"(to[2 % NG]), "=r"(to[3 % NG]) : "l"(src));
            else asm volatile("ld.global.nc.v2.u32 {%0, %1}, [%2];" : "=r"(to[0]), "=r"(to[1 % NG]) : "l"(src));
          } else {
#pragma unroll
            for (int h = 0; h < NG; ++h)
              if (h < there) to[h / 2] |= (uint32_t)src[h] << (16 * (h & 1));
          }
          return;
        }
      }
#pragma unroll
      for (int h = 0; h < NG; ++h) {
        const int gi = c * NG + h;
        to[h] = 0u;
        asm volatile("{\n .reg .pred q;\n setp.ne.b32 q, %2, 0;\n @q ld.global.nc.u16 %0, [%1];\n}\n"
                     : "+r"(to[h]) : "l"(row + gi), "r"((int)(row && gi < glim)));
      }
    };
    auto scale_of = [&](const uint32_t* from, int h) {
      return __uint_as_float(together ? (h & 1 ? from[h / 2] & 0xffff0000u : from[h / 2] << 16) : from[h] << 16);
    };
    const unsigned short* srow = scales_of(tn, tile < tiles);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) fetch(srow, part + u * SPLIT, sc[u]);
    for (int k = turn; tile < tiles && ok; tile += stride, k += TURNS) {       // k: this CTA's tiles
      // the tile's first chunk: its line, and how often the line's buffers have been used
      const uint32_t i0 = (uint32_t)k * (uint32_t)per_tile;
      // (parts: the first of the tile's chunks that is of this line, and the same of the next tile)
      const int begin = SPLIT > 1 ? part ^ (int)(i0 & 1u) : 0, begin_next = SPLIT > 1 ? part ^ (int)((i0 + (uint32_t)per_tile) & 1u) : 0;
      int line = SPLIT > 1 ? part : (int)(i0 % L), sub = (int)((i0 + begin) / L % B);
      uint32_t ph = (i0 + begin) / (L * B) & 1u;
      const int n = tn * p.rows + r, m0 = block * XROWS + e * EN;
      const bool live = srow != nullptr;
      tn += stride;
      while (tn >= tiles_n) { tn -= tiles_n; ++block; }
      const unsigned short* srow_next = scales_of(tn, tile + stride < tiles);
      if (srow_next)                       // (a load that comes from memory would hold up the use of those before it)
        for (int i = 0; i < glim; i += 16) asm volatile("prefetch.global.L2 [%0];" ::"l"(srow_next + i));
      float2 acc[EN / 2];
#pragma unroll
      for (int j = 0; j < EN / 2; ++j) acc[j] = make_float2(0.f, 0.f);
      // Once the tile before has been read, by the other set: all uses of the buffers before this tile's are over then, as the parities want.
      if (TURNS > 1 && k > 0) ok = mbar_wait_warp(smem_u32(&bars->turn[turn]), (uint32_t)((k - 1) / 2) & 1u, wc);
      const int4* tab = table + begin * (NG * XROWS);        // int8: of the next chunk
      bool over = false;                   // whether the next chunk's products are there
      for (int c0 = begin; (c0 == begin || c0 < per_tile) && ok; c0 += AHEAD * SPLIT) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          const int c = c0 + u * SPLIT;
          if (c >= per_tile) {
            if (c0 == begin) fetch(srow_next, begin_next + u * SPLIT, sc[u]);
          } else if (ok) {
            const uint32_t b = (uint32_t)(line * B + sub), td = lane_base + b * COLS;
            ok = mbar_wait_warp(over, done0 + 8 * b, ph, wc);
            if (ok) {
              if (SPLIT > 1 || ++line == L) {
                if (SPLIT == 1) line = 0;
                if (++sub == B) { sub = 0; ph ^= 1u; }
              }
              // (64 rows: not worth the registers, 85 us against 90 for 61 x 151936 x 2048)
              over = NT < 64 && c + SPLIT < per_tile && mbar_test(done0 + 8 * (uint32_t)(line * B + sub), ph);
              asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
              if (I8) {
                float* a = reinterpret_cast<float*>(acc);
                auto add = [&](const uint32_t* v, int m, float s1, const int4& t) {
                  // the lower and the upper half of the sum: below 2^25 in magnitude; times a power of two, in fp32's range wherever the sum is: exact
                  const float low = (float)((int)v[0] + 256 * (int)v[1] + t.x), high = (float)((int)v[2] + 256 * (int)v[3] + t.y);
                  a[m] = fmaf(s1, fmaf(high, 65536.f, low) * fabsf(__int_as_float(t.z)), a[m]);
                };
                if (p.M == 1) {            // a single row: its digits only
                  uint32_t v[NG][4];
#pragma unroll
                  for (int h = 0; h < NG; ++h) tmem_ld4(td + h * NT, v[h]);
                  tmem_ld_wait<NG * 4>(v[0]);
#pragma unroll
                  for (int h = 0; h < NG; ++h) add(v[h], 0, scale_of(sc[u], h), tab[h * XROWS]);
                } else {
                  constexpr int AT = NG < 2 ? NG : 2;      // groups read together
#pragma unroll
                  for (int h1 = 0; h1 < NG; h1 += AT) {
                    uint32_t v[AT][16];
#pragma unroll
                    for (int h = 0; h < AT; ++h) tmem_ld16(td + (h1 + h) * NT, v[h]);
                    tmem_ld_wait<AT * 16>(v[0]);
#pragma unroll
                    for (int h = 0; h < AT; ++h)
#pragma unroll
                      for (int m = 0; m < XROWS; ++m) {
                        if (m0 + m >= p.M) break;
                        add(v[h] + 4 * m, m, scale_of(sc[u], h1 + h), tab[(h1 + h) * XROWS + m]);
                      }
                  }
                }
              } else {
#pragma unroll
                for (int h = 0; h < NG; ++h) {
                  const float s1 = scale_of(sc[u], h);
                  const float2 s2 = make_float2(s1, s1);
                  constexpr int AT = EN < 32 ? 16 : 32;    // columns read together
#pragma unroll
                  for (int j0 = 0; j0 < EN; j0 += AT) {
                    uint32_t v[AT];
                    tmem_ld16(td + h * NT + j0, v);
                    if (AT == 32) tmem_ld16(td + h * NT + j0 + 16, v + AT - 16);
                    tmem_ld_wait<AT>(v);
#pragma unroll
                    for (int j = 0; j < AT / 2; ++j) acc[j0 / 2 + j] = __ffma2_rn(make_float2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])), s2, acc[j0 / 2 + j]);
                  }
                }
              }
              asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
              __syncwarp();
              if (lane == 0) mbar_arrive(ready0 + 8 * b);
              if (c + AHEAD * SPLIT < per_tile) fetch(srow, c + AHEAD * SPLIT, sc[u]); else fetch(srow_next, begin_next + u * SPLIT, sc[u]);
              if (I8) tab += SPLIT * NG * XROWS;
            }
          }
        }
      }
      if (!ok) break;
      if (I8 && bars->odd) {               // the groups that digits do not hold (here, so that the loop above is rid of them: 4 rows 41 us, with them 45)
        float* a = reinterpret_cast<float*>(acc);
        for (int base = 0; base < per_tile * NG * XROWS; base += 32) {
          const int at = base + lane;
          const bool such = at < per_tile * NG * XROWS && at / (NG * XROWS) % SPLIT == begin && m0 + at % XROWS < p.M && table[at].z < 0;
          for (uint32_t left = __ballot_sync(0xffffffffu, such); left; left &= left - 1u) {
            const int i = base + __ffs((int)left) - 1, gi = i / XROWS, m = i % XROWS, k = pair0 * 256 + gi * G;
            if (!live) continue;
            const float sum = __bfloat162float(p.scale[(int64_t)n * p.lds + g0 + gi]) *
                              group_sum<G>(p.x + (int64_t)(m0 + m) * p.ldx + k, p.q + (int64_t)n * p.ldq + k / 2, p.K - k);
#pragma unroll
            for (int r = 0; r < XROWS; ++r) a[r] += r == m ? sum : 0.f;
          }
        }
      }
      if (TURNS > 1) {
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars->turn[turn ^ 1]));
      }
      if (SPLIT > 1) {
        // the parts' sums meet at the first
        float* a = reinterpret_cast<float*>(acc);
        const uint32_t here = smem_u32(&bars->turn[0]), read = smem_u32(&bars->turn[1]);
        if (part == 1) {
          if (n_tile > 0 && !mbar_wait_warp(read, (n_tile - 1u) & 1u, wc)) { ok = false; break; }
#pragma unroll
          for (int m = 0; m < XROWS; ++m)
            if (m0 + m < p.M) meet[m * LANES + r] = a[m];
          __syncwarp();
          if (lane == 0) mbar_arrive(here);
          srow = srow_next;
          ++n_tile;
          continue;
        }
        if (!mbar_wait_warp(here, n_tile & 1u, wc)) { ok = false; break; }
#pragma unroll
        for (int m = 0; m < XROWS; ++m)
          if (m0 + m < p.M) a[m] += meet[m * LANES + r];
        if ((!__any_sync(0xffffffffu, a[0] + a[1] + a[2] + a[3 % EN] == 1.f) || p.M > 0) && lane == 0) mbar_arrive(read);   // (once they have been read, see below)
      }
      const float* a = reinterpret_cast<const float*>(acc);
      float sum[OWN];
      int m_own = m0;
      if (CL == 1) {
#pragma unroll
        for (int j = 0; j < OWN; ++j) sum[j] = a[j];
      } else {
        // The other's rows of x go over there, once it has read what went before: asynchronous stores, which count on the barrier there themselves
        // (an arrival that releases ordinary ones takes some 3000 cycles, the stores to y before it among them).
        if (n_tile > 0 && !mbar_wait_warp(sum_free, (n_tile - 1u) & 1u, wc)) { ok = false; break; }
        const uint32_t dst = map_to_cta(smem_u32(inbox), (uint32_t)(rank ^ 1)), bar = map_to_cta(sum_full, (uint32_t)(rank ^ 1));
        if (e == 0 && q == 0 && lane == 0) mbar_arrive_expect_tx(sum_full, S::E * OWN * LANES * 4);
        float out[OWN];
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
          const float lo = a[j], hi = a[(OWN + j) % EN];
          sum[j] = rank == 0 ? lo : hi;
          out[j] = rank == 0 ? hi : lo;
        }
#pragma unroll
        for (int j = 0; j < OWN; j += PIECE) {
          if (PIECE == 4)
            asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
                         ::"r"(dst + (uint32_t)(j * LANES * 4)), "r"(__float_as_uint(out[j])), "r"(__float_as_uint(out[j + 1])), "r"(__float_as_uint(out[(j + 2) % OWN])),
                           "r"(__float_as_uint(out[(j + 3) % OWN])), "r"(bar) : "memory");
          else
            asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];"
                         ::"r"(dst + (uint32_t)(j * LANES * 4)), "r"(__float_as_uint(out[j])), "r"(__float_as_uint(out[j + 1])), "r"(bar) : "memory");
        }
        if (!mbar_wait_warp(sum_full, n_tile & 1u, wc)) { ok = false; break; }
#pragma unroll
        for (int j = 0; j < OWN; j += PIECE)
#pragma unroll
          for (int i = 0; i < PIECE; ++i) sum[j + i] += inbox[j * LANES + i];
        // Nothing but what was read is behind this arrival: a release would wait for the stores to y, a fence for loads under way.  The vote's answer does
        // not matter; it has the arrival wait for what was read, of which every vector is in it.
        float all = 0.f;
#pragma unroll
        for (int j = 0; j < OWN; ++j) all += sum[j];
        if ((!__any_sync(0xffffffffu, all == 1.f) || p.M > 0) && lane == 0)
          asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(map_to_cta(sum_free, (uint32_t)(rank ^ 1))) : "memory");
        m_own = m0 + rank * OWN;
      }
      if (live) {
        char* at = y_at(n, m_own);
        const int rows = p.M - m_own;
#pragma unroll
        for (int j = 0; j < OWN; ++j) {
          if (j >= rows) break;
          put(at, sum[j]);
          at += ystep;
        }
      }
      srow = srow_next;
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

template <int NT, int G, int CL, bool I8> struct Room {
  using S = Shape<NT, G, I8>;
  static constexpr int FIXED = (I8 ? S::XROWS * LANES * 4 : 0) + (CL > 1 ? S::TURNS * S::E * S::EN / CL * LANES * 4 : 0) + (int)sizeof(Bars) + 1024;
  static constexpr int X256 = 256 * S::XBYTES + (I8 ? 256 / G * S::XROWS * 16 : 0);        // shared memory for 256 codes of x
};
// blocks of 256 codes of x that fit besides four stages of weights
template <int NT, int G, int CL, bool I8> int x_blocks(int smem_most) {
  return (smem_most - Room<NT, G, CL, I8>::FIXED - 4 * STAGE_BYTES) / Room<NT, G, CL, I8>::X256;
}

template <int NT, int G, int CL, bool I8>
cudaError_t launch_cl(Params p, const unsigned char* q, int64_t ldq, int sms, int smem_most, cudaStream_t st) {
  using S = Shape<NT, G, I8>;
  constexpr int FIXED = Room<NT, G, CL, I8>::FIXED, X256 = Room<NT, G, CL, I8>::X256;
  const int room = smem_most - FIXED, total = (p.K + 255) / 256;
  p.pairs = (total + CL - 1) / CL;
  p.q = q; p.ldq = ldq;
  p.scales_together = (uintptr_t)p.scale % (2 * S::NG) == 0 && (p.N == 1 || p.lds % S::NG == 0);
  // x for all of this CTA's K where at least four stages are left besides it, else as much as leaves that many
  const int most = x_blocks<NT, G, CL, I8>(smem_most);
  p.nseg = (p.pairs + most - 1) / most;
  p.seg = (p.pairs + p.nseg - 1) / p.nseg * 256;
  p.stages = (room - p.seg / 256 * X256) / STAGE_BYTES;
  if (p.stages > 12) p.stages = 12;
  // A stage's contents are all of one line: a line that waits for one has then seen the one before, as the parity of its phases wants.
  while (p.stages * S::PER % S::L) --p.stages;
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
  const int smem = p.stages * STAGE_BYTES + p.seg / 256 * X256 + FIXED;
  const int64_t tiles = (int64_t)((p.N + p.rows - 1) / p.rows) * ((p.M + S::XROWS - 1) / S::XROWS);
  auto kernel = matvec_int4_kernel<NT, G, CL, I8>;
  // (the most there is, whatever this call takes: another thread may be between this and its launch)
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_most);
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

template <int NT, int G, bool I8>
cudaError_t launch(const Params& p, const unsigned char* q, int64_t ldq, int sms, int smem_most, cudaStream_t st) {
  // A pair of CTAs where one cannot hold x besides four stages of weights.  Where a pair cannot either, x comes in parts, and as bf16: the products
  // read what the digits came with from shared memory, after the MMAs.
  const int blocks = (p.K + 255) / 256;
  if (blocks <= x_blocks<NT, G, 1, I8>(smem_most)) return launch_cl<NT, G, 1, I8>(p, q, ldq, sms, smem_most, st);
  if constexpr (I8) {
    if ((blocks + 1) / 2 > x_blocks<NT, G, 2, true>(smem_most)) return launch<16, G, false>(p, q, ldq, sms, smem_most, st);
  }
  return launch_cl<NT, G, 2, I8>(p, q, ldq, sms, smem_most, st);
}

// Rows of x that one pass over the weights serves.  (Of 64 rows and groups of 32 the products would not fit tensor memory.)  Up to four rows as integers: a
// tile's int8 MMAs take half as long and its conversion a third of the instructions; above that the products take more than is saved (with
// three digits 8 rows 69 us against 54, 16 rows 135 against 55, at 151936 x 2048).
template <int G>
cudaError_t launch_rows(const Params& p, const unsigned char* q, int64_t ldq, int sms, int smem_most, cudaStream_t st) {
  if (p.M <= 4) return launch<16, G, true>(p, q, ldq, sms, smem_most, st);
  if (p.M <= 16) return launch<16, G, false>(p, q, ldq, sms, smem_most, st);
  if constexpr (G >= 64) if (p.M > 32) return launch<64, G, false>(p, q, ldq, sms, smem_most, st);
  return launch<32, G, false>(p, q, ldq, sms, smem_most, st);
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
  p.slots = groups * (group / 16);
  p.step_rows = (int)(kQThreads / p.slots);
  p.step_slots = (int)(kQThreads % p.slots);
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
  if (K > 0 && (uintptr_t)q % 16 == 0 && pitch % 16 == 0 && N * ((M + 3) / 4) * ((K + 127) / 128) < ((int64_t)1 << 31)) {
    mv::Params m = {};
    m.x = p.x; m.ldx = p.ldx; m.scale = p.scale; m.lds = p.lds; m.M = (int)M; m.N = (int)N; m.K = (int)K; m.y = y; m.ldy = p.ldy; m.y_bf16 = p.y_bf16;
    m.x_vec = (uintptr_t)x % 16 == 0 && (M == 1 || x_row_stride % 8 == 0);
    m.groups = (int)groups;
    m.status = status; m.wait_ns = wait_limit_ns(opts ? opts->wait_limit_us : 0); m.inject = opts ? opts->test_inject : 0;
    int dev = 0, sms = 148, most = 0;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    cudaDeviceGetAttribute(&most, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev);
    const cudaError_t e = group == 128 ? mv::launch_rows<128>(m, q, pitch, sms, most, st)
                                       : (group == 64 ? mv::launch_rows<64>(m, q, pitch, sms, most, st) : mv::launch_rows<32>(m, q, pitch, sms, most, st));
    return e == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
  }
  const int64_t warps = N * ((M + kGRows - 1) / kGRows), grid = (warps + kGThreads / 32 - 1) / (kGThreads / 32);
  matvec_int4_generic_kernel<<<(unsigned)(grid < (1 << 30) ? grid : (1 << 30)), kGThreads, 0, st>>>(p);
  return cudaGetLastError() == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
}
