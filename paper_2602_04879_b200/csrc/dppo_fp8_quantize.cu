// Rounding to 8-bit floating point (e4m3 or e5m2) with one fp32 scale for each 1 x 128 or 128 x 128 block, as stored and
// transposed, in one pass over the input.
//
//   scale = amax / B (B the largest finite value of the type),  q = x / scale rounded to nearest even.
//
// The quotient is formed as (7/8 x) / (amax 2^-n) with B = 7/8 2^n (448 = 7/8 2^9, 57344 = 7/8 2^16): one correctly rounded
// division, exact wherever x / scale lies half way between two 8-bit values (7/8 x is exact for bf16 inputs), so that ties go to
// even as the definition says.  Divided by amax / B rounded to fp32, such ties would go either way.  The division itself is
// one multiplication by the rounded reciprocal and Markstein's correction step (P. Markstein, IBM J. Res. Dev. 34, 1990),
// with the divisor scaled into [1, 2) first so that the remainder cannot underflow.
//
// Bounded by memory (2 or 4 bytes in, 1 byte out per orientation), and close behind it by instructions.  A CTA owns a tile of 128
// columns and 16 R rows; each thread holds an R x 8 block of it in registers, so the input is read once, whatever is written: row
// maxima come from the 16 threads of a row, column maxima (transposed form) from shared memory; one thread per row and one per column
// then works out the scale; products and corrections go in packed fp32 pairs.  The transposed bytes are turned round in shared
// memory, 8 x 8 bytes per thread, placed so that neither side collides on the banks.
//
// Measured on B200, bf16 in, both orientations out: [151936, 2048] in blocks of 128 x 128 230 us = 5.4 TB/s (83 % of a copy's rate),
// [2048, 151936] in blocks of 1 x 128 269 us = 4.6 TB/s (71 %; twice the scales to work out, and maxima across threads for the rows);
// [61, 2048] as stored 2.1 us, a launch.
#include <cuda_fp8.h>

#include "dppo_common.cuh"

namespace dppo {
namespace {

constexpr int kQThreads = 256;

struct QuantParams {
  const void* x;
  int64_t rows, cols, ldx;
  int block_rows, vec;             // vec: 16-byte loads allowed (aligned base and row stride)
  uint8_t* q;
  int64_t ldq;
  float* scale;
  int64_t s_row, s_k;
  uint8_t* qt;
  int64_t ldqt;
  float* scale_t;
  int64_t st_row, st_k;
  int32_t* status;
  int qvec, qtvec;                 // 8-byte stores allowed
  int64_t col_tiles;
};

// What turns an element of a block into its 8-bit value: num = x f, q = num / b; f = 7/8 2^(n - e), b = amax 2^-e in [1, 2), r = 1 / b
// (kept: f, -b, r and the scale).
// A block with an infinity or a NaN has f = NaN: all its values, and its scale, come out as NaN.
template <bool E5M2> __device__ __forceinline__ float4 block_scale(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) { const float nan = __int_as_float(0x7fffffff); return make_float4(nan, -1.f, 1.f, nan); }
  const float amax = fmaxf(__uint_as_float(amax_bits), 0x1p-100f);
  const int e = (int)(__float_as_uint(amax) >> 23) - 127;    // amax is a normal number
  const float b = __uint_as_float((__float_as_uint(amax) & 0x007fffffu) | 0x3f800000u);
  return make_float4(0.875f * __uint_as_float((uint32_t)((E5M2 ? 16 : 9) - e + 127) << 23), -b, __frcp_rn(b), __fdiv_rn(amax, E5M2 ? 57344.f : 448.f));
}
// two elements of blocks with the same scale, as two bytes
template <bool E5M2> __device__ __forceinline__ uint32_t round2(float x, float y, const float4& s) {
  const float2 num = __fmul2_rn(make_float2(x, y), make_float2(s.x, s.x)), r = make_float2(s.z, s.z);
  float2 q = __fmul2_rn(num, r);
  q = __ffma2_rn(__ffma2_rn(q, make_float2(s.y, s.y), num), r, q);
  return __nv_cvt_float2_to_fp8x2(q, __NV_SATFINITE, E5M2 ? __NV_E5M2 : __NV_E4M3);
}

// Eight consecutive elements of one row, as loaded; Max: their magnitudes' running maximum, NaNs and infinities above all else.
template <typename T> struct Oct;
template <> struct Oct<__nv_bfloat16> {
  uint4 v;
  __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = __ldg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void put(int i, __nv_bfloat16 x) {
    const uint32_t b = __bfloat16_as_ushort(x);
    (&v.x)[i >> 1] |= (i & 1) ? b << 16 : b;
  }
  __device__ __forceinline__ float at(int i) const {
    const uint32_t w = (&v.x)[i >> 1];
    return __uint_as_float((i & 1) ? (w & 0xffff0000u) : (w << 16));
  }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {         // of two pairs of magnitudes
    const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&m);
  }
  __device__ __forceinline__ uint32_t pair(int k) const { return (&v.x)[k] & 0x7fff7fffu; }
  __device__ __forceinline__ uint32_t row_max() const {      // as fp32 bits
    const uint32_t m = max2(max2(pair(0), pair(1)), max2(pair(2), pair(3)));
    return max(m << 16, m & 0xffff0000u);
  }
};
template <> struct Oct<float> {
  float4 a, b;
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load(const float* p) {
    a = __ldg(reinterpret_cast<const float4*>(p));
    b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ __forceinline__ void put(int i, float x) { if (i < 4) (&a.x)[i] = x; else (&b.x)[i - 4] = x; }
  __device__ __forceinline__ float at(int i) const { return i < 4 ? (&a.x)[i] : (&b.x)[i - 4]; }
  __device__ __forceinline__ uint32_t mag(int i) const { return __float_as_uint(at(i)) & 0x7fffffffu; }
  __device__ __forceinline__ uint32_t row_max() const {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, mag(j));
    return m;
  }
};
// maxima of eight columns over R rows, as fp32 bits
template <int R> __device__ __forceinline__ void col_max(const Oct<__nv_bfloat16>* v, uint32_t* m) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t x = v[0].pair(k);
#pragma unroll
    for (int i = 1; i < R; ++i) x = Oct<__nv_bfloat16>::max2(x, v[i].pair(k));
    m[2 * k] = x << 16;
    m[2 * k + 1] = x & 0xffff0000u;
  }
}
template <int R> __device__ __forceinline__ void col_max(const Oct<float>* v, uint32_t* m) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t x = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) x = max(x, v[i].mag(j));
    m[j] = x;
  }
}

// R rows per thread: 8 for whole 128 x 128 tiles, needed for 128 x 128 blocks and for the transposed form, and faster for rows that allow
// 16-byte loads once there are tiles for all SMs with more than half of their rows (1 x 128 blocks as stored, bf16: [2048, 151936] 158 us
// against 283 us, [4096, 2048] 6.9 against 9.3 us, [128, 151936] 13.7 against 19.7 us); 1 otherwise: up to eight times the CTAs, so that few
// rows still spread over the SMs, and rows on no 16-byte boundary are read by adjacent threads of many warps ([512, 2048] 4.8 against 5.7 us,
// [4, 151936] 3.3 against 11.7 us, [61, 151936] 10.8 against 17.4 us, [1024, 50257] 57 against 63 us, in fp32 63 against 72 us).
template <typename T, int R, bool E5M2>
__global__ void __launch_bounds__(kQThreads) dppo_quantize_kernel(QuantParams p) {
  static_assert(R == 8 || R == 1, "rows per thread");
  constexpr bool kTile = R == 8;
  __shared__ __align__(16) uint32_t colmax[kTile ? 8 : 1][kTile ? 128 : 4];
  __shared__ float4 row_s[16 * R], col_s[kTile ? 128 : 1];
  __shared__ uint32_t blockmax[8];
  __shared__ __align__(16) unsigned char tile[kTile ? 128 * 128 : 16];
  const int tid = threadIdx.x, cg = tid & 15, rg = tid >> 4, warp = tid >> 5;
  const int64_t rt = blockIdx.x / p.col_tiles, ct = blockIdx.x - rt * p.col_tiles;
  const int64_t r0 = rt * (16 * R) + rg * R, c0 = ct * 128 + cg * 8;      // this thread's block
  const T* x = reinterpret_cast<const T*>(p.x);
  Oct<T> v[R];
  const bool inner = p.vec && c0 + 8 <= p.cols && r0 + R <= p.rows;
  if (inner) {
    const T* src = x + r0 * p.ldx + c0;
#pragma unroll
    for (int i = 0; i < R; ++i) v[i].load(src + i * p.ldx);
  } else {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      v[i].zero();
      if (r0 + i < p.rows) {
#pragma unroll
        for (int j = 0; j < 8; ++j) if (c0 + j < p.cols) v[i].put(j, x[(r0 + i) * p.ldx + c0 + j]);
      }
    }
  }
  bool bad = false;
  const bool whole = kTile && p.block_rows == 128;           // one scale for the tile
  if (whole || p.q) {
    uint32_t m[R];
#pragma unroll
    for (int i = 0; i < R; ++i) m[i] = v[i].row_max();
    if (whole) {
#pragma unroll
      for (int i = 1; i < R; ++i) m[0] = max(m[0], m[i]);
      m[0] = __reduce_max_sync(0xffffffffu, m[0]);
      if ((tid & 31) == 0) blockmax[warp] = m[0];
    } else {
      // maxima over the 16 threads of a row, rows shared out on the way: with R = 8, thread cg ends up with row cg / 2
      int row = 0;
#pragma unroll
      for (int n = R / 2, o = 8; n > 0; n >>= 1, o >>= 1) {
        const bool up = cg & o;
#pragma unroll
        for (int i = 0; i < n; ++i) {
          const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? m[i] : m[i + n], o);
          m[i] = max(up ? m[i + n] : m[i], got);
        }
        row += up ? n : 0;
      }
#pragma unroll
      for (int o = R == 8 ? 1 : 8; o > 0; o >>= 1) m[0] = max(m[0], __shfl_xor_sync(0xffffffffu, m[0], o));
      const float4 s = block_scale<E5M2>(m[0]);
      bad |= s.w != s.w;
      if ((cg & (16 / R - 1)) == 0) {
        row_s[rg * R + row] = s;
        if (r0 + row < p.rows) p.scale[(r0 + row) * p.s_row + ct * p.s_k] = s.w;
      }
    }
  }
  if (kTile && p.qt && !whole) {
    uint32_t m[8];
    col_max<R>(v, m);
#pragma unroll
    for (int j = 0; j < 8; ++j) m[j] = max(m[j], __shfl_xor_sync(0xffffffffu, m[j], 16));
    if ((tid & 31) < 16) {
      uint4* dst = reinterpret_cast<uint4*>(&colmax[kTile ? warp : 0][kTile ? cg * 8 : 0]);
      dst[0] = make_uint4(m[0], m[1], m[2], m[3]);
      dst[kTile ? 1 : 0] = make_uint4(m[4], m[5], m[6], m[7]);
    }
  }
  __syncthreads();
  float4 bs = make_float4(0.f, -1.f, 1.f, 0.f);
  if (whole) {
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) m = max(m, blockmax[w]);
    bs = block_scale<E5M2>(m);
    bad |= bs.w != bs.w;
    if (tid == 0) {
      if (p.q) p.scale[rt * p.s_row + ct * p.s_k] = bs.w;
      if (p.qt) p.scale_t[ct * p.st_row + rt * p.st_k] = bs.w;
    }
  } else if (kTile && p.qt) {
    if (tid < 128) {                                         // a thread per column
      uint32_t m = 0;
#pragma unroll
      for (int w = 0; w < 8; ++w) m = max(m, colmax[kTile ? w : 0][kTile ? tid : 0]);
      const float4 s = block_scale<E5M2>(m);
      col_s[kTile ? (tid & ~7) | ((tid ^ (tid >> 3)) & 7) : 0] = s;       // (place: the readers take every eighth column at a time)
      bad |= s.w != s.w;
      if (ct * 128 + tid < p.cols) p.scale_t[(ct * 128 + tid) * p.st_row + rt * p.st_k] = s.w;
    }
    __syncthreads();
  }
  if (p.q) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float4 s = whole ? bs : row_s[rg * R + i];
      uint32_t o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = round2<E5M2>(v[i].at(2 * j), v[i].at(2 * j + 1), s);
      const uint2 b = make_uint2(o[0] | (o[1] << 16), o[2] | (o[3] << 16));
      if (r0 + i < p.rows) {
        uint8_t* dst = p.q + (r0 + i) * p.ldq + c0;
        if (p.qvec && c0 + 8 <= p.cols) {
          *reinterpret_cast<uint2*>(dst) = b;
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) if (c0 + j < p.cols) dst[j] = (uint8_t)((j < 4 ? b.x : b.y) >> (8 * (j & 3)));
        }
      }
    }
  }
  if (kTile && p.qt) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = cg * 8 + j;
      const float4 s = whole ? bs : col_s[kTile ? cg * 8 + ((j ^ cg) & 7) : 0];
      uint32_t o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = round2<E5M2>(v[kTile ? 2 * i : 0].at(j), v[kTile ? 2 * i + 1 : 0].at(j), s);
      *reinterpret_cast<uint2*>(tile + (kTile ? c * 128 + ((rg ^ (c >> 3)) * 8) : 0)) = make_uint2(o[0] | (o[1] << 16), o[2] | (o[3] << 16));
    }
    __syncthreads();
    const int64_t row0 = rt * 128 + cg * 8;                  // first of the eight input rows of this thread's piece
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = i * 16 + rg;
      const int64_t col = ct * 128 + c;
      if (col < p.cols) {
        const uint2 o = *reinterpret_cast<const uint2*>(tile + (kTile ? c * 128 + ((cg ^ (c >> 3)) * 8) : 0));
        uint8_t* dst = p.qt + col * p.ldqt + row0;
        if (p.qtvec && row0 + 8 <= p.rows) {
          *reinterpret_cast<uint2*>(dst) = o;
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) if (row0 + j < p.rows) dst[j] = (uint8_t)((j < 4 ? o.x : o.y) >> (8 * (j & 3)));
        }
      }
    }
  }
  if (bad) atomicOr(p.status, DPPO_STATUS_NONFINITE_ROW);
}

template <typename T, bool E5M2>
cudaError_t launch_quantize(QuantParams p, cudaStream_t st) {
  p.col_tiles = (p.cols + 127) / 128;
  int dev = 0, sms = 148;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  const int64_t grid = p.col_tiles * ((p.rows + 127) / 128);
  if (p.qt || p.block_rows == 128 || (p.vec && p.rows > 64 && grid >= 2 * sms)) {
    dppo_quantize_kernel<T, 8, E5M2><<<(unsigned)grid, kQThreads, 0, st>>>(p);
  } else {
    const int64_t grid = p.col_tiles * ((p.rows + 15) / 16);
    dppo_quantize_kernel<T, 1, E5M2><<<(unsigned)grid, kQThreads, 0, st>>>(p);
  }
  return cudaGetLastError();
}

}  // namespace
}  // namespace dppo

extern "C" int dppo_fp8_quantize(const void* x, int64_t rows, int64_t cols, int64_t x_row_stride, int x_dtype, int fp8_format,
                                 int block_rows, void* q, int64_t q_row_stride, float* q_scale, int64_t q_scale_row_stride,
                                 int64_t q_scale_k_stride, void* qt, int64_t qt_row_stride, float* qt_scale,
                                 int64_t qt_scale_row_stride, int64_t qt_scale_k_stride, int32_t* status, void* cuda_stream) {
  using namespace dppo;
  const int64_t big = (int64_t)1 << 38;                      // (the grid has to count in 31 bits too: below)
  if (rows < 0 || cols < 0 || (rows > 0 && cols > big / rows)) return DPPO_ERR_SHAPE;
  if (x_dtype != DPPO_F32 && x_dtype != DPPO_BF16) return DPPO_ERR_DTYPE;
  if (fp8_format != DPPO_E4M3 && fp8_format != DPPO_E5M2) return DPPO_ERR_DTYPE;
  if (block_rows != 1 && block_rows != 128) return DPPO_ERR_UNSUPPORTED;
  if (!status) return DPPO_ERR_NULL;
  if (rows == 0 || cols == 0) return DPPO_OK;
  if (!x || (!q && !qt) || (q && !q_scale) || (qt && !qt_scale)) return DPPO_ERR_NULL;
  if (x_row_stride < cols || (q && q_row_stride < cols) || (qt && qt_row_stride < rows)) return DPPO_ERR_STRIDE;
  // every scale has a place of its own: the two strides span [row blocks, column blocks] without overlap
  const int64_t kb = (cols + 127) / 128, rb = (rows + block_rows - 1) / block_rows;
  const int64_t kbt = (rows + 127) / 128, rbt = (cols + block_rows - 1) / block_rows;
  auto apart = [](int64_t s_row, int64_t s_k, int64_t nr, int64_t nk) {
    return s_row >= 1 && s_k >= 1 && (s_k >= s_row * nr || s_row >= s_k * nk || nr == 1 || nk == 1);
  };
  if (q && !apart(q_scale_row_stride, q_scale_k_stride, rb, kb)) return DPPO_ERR_STRIDE;
  if (qt && !apart(qt_scale_row_stride, qt_scale_k_stride, rbt, kbt)) return DPPO_ERR_STRIDE;
  const int es = x_dtype == DPPO_BF16 ? 2 : 4;
  if (((uintptr_t)x % es) || ((uintptr_t)q_scale % 4) || ((uintptr_t)qt_scale % 4) || ((uintptr_t)status % 4)) return DPPO_ERR_ALIGN;
  const int64_t tile_rows = qt || block_rows == 128 ? 128 : 16;
  if (kb * ((rows + tile_rows - 1) / tile_rows) > INT32_MAX) return DPPO_ERR_SHAPE;
  QuantParams p = {};
  p.x = x; p.rows = rows; p.cols = cols; p.ldx = x_row_stride; p.block_rows = block_rows;
  p.vec = ((uintptr_t)x % 16) == 0 && (x_row_stride * es) % 16 == 0;
  p.q = reinterpret_cast<uint8_t*>(q); p.ldq = q_row_stride; p.scale = q_scale; p.s_row = q_scale_row_stride; p.s_k = q_scale_k_stride;
  p.qt = reinterpret_cast<uint8_t*>(qt); p.ldqt = qt_row_stride; p.scale_t = qt_scale; p.st_row = qt_scale_row_stride; p.st_k = qt_scale_k_stride;
  p.status = status;
  p.qvec = ((uintptr_t)q % 8) == 0 && q_row_stride % 8 == 0;
  p.qtvec = ((uintptr_t)qt % 8) == 0 && qt_row_stride % 8 == 0;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaError_t e;
  if (fp8_format == DPPO_E5M2) e = x_dtype == DPPO_BF16 ? launch_quantize<__nv_bfloat16, true>(p, st) : launch_quantize<float, true>(p, st);
  else e = x_dtype == DPPO_BF16 ? launch_quantize<__nv_bfloat16, false>(p, st) : launch_quantize<float, false>(p, st);
  return e == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
}
