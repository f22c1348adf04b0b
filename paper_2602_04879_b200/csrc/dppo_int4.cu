// Weights in 4 bits with a scale per group of 32, 64 or 128 along a row: rounding to them, and their product with a few rows.
//
//   scale = amax / 7 rounded to bf16,   code = round(x / scale) + 8 in 1 .. 15, two codes to a byte, the even column in the low half
//   y[m, n] = sum_g scale[n, g] sum_{k in group g} x[m, k] (code[n, k] - 8)
//
// The codes are small whole numbers, so every product x (code - 8) is exact; a group's products are added up in fp32 and its scale is
// applied to that sum, so that no weight is rounded a second time.
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
  const int64_t warps = N * ((M + kGRows - 1) / kGRows), grid = (warps + kGThreads / 32 - 1) / (kGThreads / 32);
  matvec_int4_generic_kernel<<<(unsigned)(grid < (1 << 30) ? grid : (1 << 30)), kGThreads, 0, st>>>(p);
  return cudaGetLastError() == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
}
