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
// Bounded by memory: 2 (or 4) bytes in, 1 byte out per orientation.  A CTA owns a tile of 128 columns and 16 R rows; each
// thread holds an R x 8 block of it in registers, so the input is read once, whatever is written: row scales come from a
// reduction over the 16 threads of a row, column scales (transposed form) from one over shared memory.  The transposed
// bytes are turned round in shared memory, 8 x 8 bytes per thread, placed so that neither side collides on the banks.
#include <cuda_fp8.h>

#include "dppo_common.cuh"

namespace dppo {
namespace {

constexpr int kQThreads = 256;

struct QuantParams {
  const void* x;
  int64_t rows, cols, ldx;
  int block_rows, e5m2, vec;       // vec: 16-byte loads allowed (aligned base and row stride)
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

// What turns an element of a block into its 8-bit value: num = x f, q = num / b.
struct BlockScale {
  float f, b, r;                   // f = 7/8 2^(n - e), b = amax 2^-e in [1, 2), r = 1 / b
  int bad;
};
__device__ __forceinline__ BlockScale block_scale(uint32_t amax_bits, int e5m2, float& scale) {
  BlockScale s;
  s.bad = amax_bits >= 0x7f800000u;                          // an infinity or a NaN in the block
  const float amax = fmaxf(__uint_as_float(s.bad ? 0x3f800000u : amax_bits), 0x1p-100f);
  scale = s.bad ? __int_as_float(0x7fffffff) : __fdiv_rn(amax, e5m2 ? 57344.f : 448.f);
  const int e = (int)(__float_as_uint(amax) >> 23) - 127;    // amax is a normal number
  s.b = __uint_as_float((__float_as_uint(amax) & 0x007fffffu) | 0x3f800000u);
  s.r = __frcp_rn(s.b);
  s.f = 0.875f * __uint_as_float((uint32_t)((e5m2 ? 16 : 9) - e + 127) << 23);
  return s;
}
__device__ __forceinline__ float quotient(float x, const BlockScale& s) {
  const float num = x * s.f, q = num * s.r;
  return fmaf(fmaf(-q, s.b, num), s.r, q);
}
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d, int e5m2) {
  const __nv_fp8_interpretation_t t = e5m2 ? __NV_E5M2 : __NV_E4M3;
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, t);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, t);
  return lo | (hi << 16);
}

// Eight consecutive elements of one row, as loaded.
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
};
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// R rows per thread: 8 for whole 128 x 128 tiles (needed for 128 x 128 blocks and for the transposed form), less otherwise.
template <typename T, int R>
__global__ void __launch_bounds__(kQThreads) dppo_quantize_kernel(QuantParams p) {
  __shared__ uint32_t colmax[R == 8 ? 8 : 1][128];
  __shared__ uint32_t blockmax[8];
  __shared__ __align__(16) unsigned char tile[R == 8 ? 128 * 128 : 16];
  const int tid = threadIdx.x, cg = tid & 15, rg = tid >> 4, warp = tid >> 5;
  const int64_t rt = blockIdx.x / p.col_tiles, ct = blockIdx.x - rt * p.col_tiles;
  const int64_t r0 = rt * (16 * R) + rg * R, c0 = ct * 128 + cg * 8;      // this thread's block
  const T* x = reinterpret_cast<const T*>(p.x);
  Oct<T> v[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    v[i].zero();
    const int64_t r = r0 + i;
    if (r < p.rows) {
      const T* src = x + r * p.ldx + c0;
      if (p.vec && c0 + 8 <= p.cols) {
        v[i].load(src);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) if (c0 + j < p.cols) v[i].put(j, src[j]);
      }
    }
  }
  uint32_t rowmax[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, abs_bits(v[i].at(j)));
    rowmax[i] = m;
  }
  int bad = 0;
  BlockScale bs = {};
  float block_value = 0.f;
  if (R == 8 && p.block_rows == 128) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) m = max(m, rowmax[i]);
    m = __reduce_max_sync(0xffffffffu, m);
    if ((tid & 31) == 0) blockmax[warp] = m;
    __syncthreads();
    m = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) m = max(m, blockmax[w]);
    bs = block_scale(m, p.e5m2, block_value);
    bad |= bs.bad;
    if (tid == 0) {
      if (p.q) p.scale[rt * p.s_row + ct * p.s_k] = block_value;
      if (p.qt) p.scale_t[ct * p.st_row + rt * p.st_k] = block_value;
    }
  }
  if (p.q) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      BlockScale s = bs;
      if (p.block_rows == 1) {
        uint32_t m = rowmax[i];
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        float sv;
        s = block_scale(m, p.e5m2, sv);
        bad |= s.bad;
        if (cg == 0 && r0 + i < p.rows) p.scale[(r0 + i) * p.s_row + ct * p.s_k] = sv;
      }
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = quotient(v[i].at(j), s);
      uint2 o = make_uint2(pack4(y[0], y[1], y[2], y[3], p.e5m2), pack4(y[4], y[5], y[6], y[7], p.e5m2));
      if (s.bad) o = make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);
      if (r0 + i < p.rows) {
        uint8_t* dst = p.q + (r0 + i) * p.ldq + c0;
        if (p.qvec && c0 + 8 <= p.cols) {
          *reinterpret_cast<uint2*>(dst) = o;
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) if (c0 + j < p.cols) dst[j] = (uint8_t)((j < 4 ? o.x : o.y) >> (8 * (j & 3)));
        }
      }
    }
  }
  if (R == 8 && p.qt) {
    BlockScale s = bs;
    if (p.block_rows == 1) {
      uint32_t cm[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < R; ++i) m = max(m, abs_bits(v[i].at(j)));
        cm[j] = max(m, __shfl_xor_sync(0xffffffffu, m, 16));
      }
      if ((tid & 31) < 16) {
#pragma unroll
        for (int j = 0; j < 8; ++j) colmax[R == 8 ? warp : 0][cg * 8 + j] = cm[j];
      }
      __syncthreads();
      // one thread per column: its scale, and what the column's threads need of it
      if (tid < 128) {
        uint32_t m = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) m = max(m, colmax[R == 8 ? w : 0][tid]);
        colmax[0][tid] = m;
      }
      __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = cg * 8 + j;
      if (p.block_rows == 1) {
        float sv;
        s = block_scale(colmax[0][c], p.e5m2, sv);
        bad |= s.bad;
        if (rg == 0 && c0 + j < p.cols) p.scale_t[(c0 + j) * p.st_row + rt * p.st_k] = sv;
      }
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = quotient(v[R == 8 ? i : 0].at(j), s);
      uint2 o = make_uint2(pack4(y[0], y[1], y[2], y[3], p.e5m2), pack4(y[4], y[5], y[6], y[7], p.e5m2));
      if (s.bad) o = make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);
      *reinterpret_cast<uint2*>(tile + c * 128 + ((rg ^ (c >> 3)) * 8)) = o;
    }
    __syncthreads();
    const int64_t row0 = rt * 128 + cg * 8;                  // first of the eight input rows of this thread's piece
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = i * 16 + rg;
      const int64_t col = ct * 128 + c;
      if (col < p.cols) {
        const uint2 o = *reinterpret_cast<const uint2*>(tile + c * 128 + ((cg ^ (c >> 3)) * 8));
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

template <typename T>
cudaError_t launch_quantize(QuantParams p, cudaStream_t st) {
  p.col_tiles = (p.cols + 127) / 128;
  if (p.qt || p.block_rows == 128) {
    const int64_t grid = p.col_tiles * ((p.rows + 127) / 128);
    if (grid > INT32_MAX) return cudaErrorInvalidValue;
    dppo_quantize_kernel<T, 8><<<(unsigned)grid, kQThreads, 0, st>>>(p);
  } else {
    const int64_t grid = p.col_tiles * ((p.rows + 15) / 16);
    if (grid > INT32_MAX) return cudaErrorInvalidValue;
    dppo_quantize_kernel<T, 1><<<(unsigned)grid, kQThreads, 0, st>>>(p);
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
  const int64_t big = (int64_t)1 << 38;                      // 128 x 128 tiles of it still count in 31 bits
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
  if (((uintptr_t)x % es) || ((uintptr_t)q_scale % 4) || ((uintptr_t)qt_scale % 4)) return DPPO_ERR_ALIGN;
  QuantParams p = {};
  p.x = x; p.rows = rows; p.cols = cols; p.ldx = x_row_stride; p.block_rows = block_rows; p.e5m2 = fp8_format == DPPO_E5M2;
  p.vec = ((uintptr_t)x % 16) == 0 && (x_row_stride * es) % 16 == 0;
  p.q = reinterpret_cast<uint8_t*>(q); p.ldq = q_row_stride; p.scale = q_scale; p.s_row = q_scale_row_stride; p.s_k = q_scale_k_stride;
  p.qt = reinterpret_cast<uint8_t*>(qt); p.ldqt = qt_row_stride; p.scale_t = qt_scale; p.st_row = qt_scale_row_stride; p.st_k = qt_scale_k_stride;
  p.status = status;
  p.qvec = ((uintptr_t)q % 8) == 0 && q_row_stride % 8 == 0;
  p.qtvec = ((uintptr_t)qt % 8) == 0 && qt_row_stride % 8 == 0;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  const cudaError_t e = x_dtype == DPPO_BF16 ? launch_quantize<__nv_bfloat16>(p, st) : launch_quantize<float>(p, st);
  return e == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
}
