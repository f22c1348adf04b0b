// A row of logits as 16-byte vectors, whatever element it starts at, for the kernels that read it with plain loads.
//
// A row's image starts at the 16-byte boundary at or below its first element, `head` elements early; vector v is elements
// [v N - head, v N - head + N) of the row.  Vectors inside the row are one 16-byte load; the one or two at its ends are put together from
// single elements, so that nothing outside the row is read or written.  The other tensors of a call are cut along the same vectors: where
// their rows do not lie on the same phase they are read and written element by element.
#pragma once

#include "dppo_common.cuh"
#include "dppo_pipe.cuh"
#include "dppo_rowtools.cuh"

namespace dppo {

// Logits at or below this (the lowest bf16 number; the lowest fp32 number too) count as probability zero, as -inf does.  Entries are clamped
// to it, so that differences of logits stay finite: where the weight is zero, 0 * (a difference) must be 0.
constexpr float kLowest = -3.3895313892515355e38f;

// Raw bits of -inf in both halves (bf16) or in the word (fp32): the filling of a vector outside its row.
template <typename T> struct RawOf;
template <> struct RawOf<__nv_bfloat16> { static constexpr uint32_t kNegInf = 0xFF80FF80u; };
template <> struct RawOf<float> { static constexpr uint32_t kNegInf = 0xFF800000u; };

__device__ __forceinline__ uint4 ldg128_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// a raw vector with its entries clamped to kLowest from below (NaN stays NaN)
template <typename T> __device__ __forceinline__ uint4 clamp_raw(const uint4& v);
template <> __device__ __forceinline__ uint4 clamp_raw<__nv_bfloat16>(const uint4& v) {
  constexpr uint32_t low = 0xFF7FFF7Fu;
  return make_uint4(max_nan_bf16x2(v.x, low), max_nan_bf16x2(v.y, low), max_nan_bf16x2(v.z, low), max_nan_bf16x2(v.w, low));
}
template <> __device__ __forceinline__ uint4 clamp_raw<float>(const uint4& v) {
  return make_uint4(__float_as_uint(max_nan(__uint_as_float(v.x), kLowest)), __float_as_uint(max_nan(__uint_as_float(v.y), kLowest)),
                    __float_as_uint(max_nan(__uint_as_float(v.z), kLowest)), __float_as_uint(max_nan(__uint_as_float(v.w), kLowest)));
}
// running maximum of raw entries, kept raw (two bf16 lanes, or one fp32), and its value
template <typename T> struct RawMax;
template <> struct RawMax<__nv_bfloat16> {
  uint32_t m = 0xFF7FFF7Fu;
  __device__ __forceinline__ void add(const uint4& v) { m = max_nan_bf16x2(max_nan_bf16x2(m, v.x), max_nan_bf16x2(max_nan_bf16x2(v.y, v.z), v.w)); }
  __device__ __forceinline__ float value() const { return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u)); }
};
template <> struct RawMax<float> {
  float m = kLowest;
  __device__ __forceinline__ void add(const uint4& v) {
    m = max_nan(max_nan(m, __uint_as_float(v.x)), max_nan(max_nan(__uint_as_float(v.y), __uint_as_float(v.z)), __uint_as_float(v.w)));
  }
  __device__ __forceinline__ float value() const { return m; }
};
// a raw vector as pairs of floats
template <typename T> __device__ __forceinline__ void to_pairs(const uint4& v, float2* z);
template <> __device__ __forceinline__ void to_pairs<__nv_bfloat16>(const uint4& v, float2* z) {
  z[0] = make_float2(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u));
  z[1] = make_float2(__uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
  z[2] = make_float2(__uint_as_float(v.z << 16), __uint_as_float(v.z & 0xffff0000u));
  z[3] = make_float2(__uint_as_float(v.w << 16), __uint_as_float(v.w & 0xffff0000u));
}
template <> __device__ __forceinline__ void to_pairs<float>(const uint4& v, float2* z) {
  z[0] = make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
  z[1] = make_float2(__uint_as_float(v.z), __uint_as_float(v.w));
}
// the entries of a raw vector less m, as pairs of floats (bf16: one instruction an entry, which widens it as well)
template <typename T> __device__ __forceinline__ void less_pairs(const uint4& v, float m, float2* d);
__device__ __forceinline__ float2 less_bf16x2(uint32_t w, float nm) {
  float2 d;
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n add.f32.bf16 %0, l, %3;\n add.f32.bf16 %1, h, %3;\n}\n" : "=f"(d.x), "=f"(d.y) : "r"(w), "f"(nm));
  return d;
}
template <> __device__ __forceinline__ void less_pairs<__nv_bfloat16>(const uint4& v, float m, float2* d) {
  d[0] = less_bf16x2(v.x, -m);
  d[1] = less_bf16x2(v.y, -m);
  d[2] = less_bf16x2(v.z, -m);
  d[3] = less_bf16x2(v.w, -m);
}
template <> __device__ __forceinline__ void less_pairs<float>(const uint4& v, float m, float2* d) {
  const float2 nm = make_float2(-m, -m);
  d[0] = __fadd2_rn(make_float2(__uint_as_float(v.x), __uint_as_float(v.y)), nm);
  d[1] = __fadd2_rn(make_float2(__uint_as_float(v.z), __uint_as_float(v.w)), nm);
}
// exp(d) for |d| < kNearZero, to 2^-41: for what a log-sum-exp loses when it is rounded to fp32, which is that little unless it is above 2^17
constexpr double kNearZero = 0.0078125;
__device__ __forceinline__ double exp_series(double d) { return 1.0 + d * (1.0 + d * (1.0 / 2 + d * (1.0 / 6 + d * (1.0 / 24)))); }
__device__ __forceinline__ float warp_max_nan(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float warp_sum_f32(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ uint32_t cluster_nctarank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
// the two halves of cluster_sync_all
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }

__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i == 0 ? v.x : (i == 1 ? v.y : (i == 2 ? v.z : v.w)); }
__device__ __forceinline__ void set_word(uint4& v, int i, uint32_t w) {
  if (i == 0) v.x = w; else if (i == 1) v.y = w; else if (i == 2) v.z = w; else v.w = w;
}
// element i of a raw vector
__device__ __forceinline__ void set_raw(uint4& v, int i, __nv_bfloat16 x) {
  const uint32_t b = (uint32_t)__bfloat16_as_ushort(x), w = word_of(v, i >> 1);
  set_word(v, i >> 1, (i & 1) ? ((w & 0xffffu) | (b << 16)) : ((w & 0xffff0000u) | b));
}
__device__ __forceinline__ void set_raw(uint4& v, int i, float x) { set_word(v, i, __float_as_uint(x)); }

template <typename T>
__device__ __forceinline__ uint32_t head_of(const T* row) { return (uint32_t)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(T)); }

// A row of V elements T cut into vectors of N elements, the first of which starts `head` elements in front of the row.  Vectors lo .. hi - 1
// lie inside the row and are aligned in this tensor: 16-byte accesses; the others of the nvec go element by element.
template <typename T, int N>
struct RowRef {
  T* row;
  int V, head, nvec, lo, hi;
  __device__ __forceinline__ RowRef(T* r, uint32_t h, int64_t v) : row(r), V((int)v), head((int)h) {
    nvec = (head + V + N - 1) / N;
    const bool whole = ((reinterpret_cast<uintptr_t>(r) - (uintptr_t)h * sizeof(T)) & 15u) == 0;
    lo = whole ? (head ? 1 : 0) : 0;
    hi = whole ? (head + V) / N : 0;
  }
  __device__ __forceinline__ bool inside(int v) const { return v >= lo && v < hi; }
  __device__ __forceinline__ T* at(int v) const { return row + ((int64_t)v * N - head); }
};

// raw = 16 bytes at p where `yes`, unchanged otherwise: loads of several vectors stay in flight together
__device__ __forceinline__ void ldg128_if(uint4& raw, const void* p, bool yes) {
  asm volatile("{\n .reg .pred q;\n setp.ne.b32 q, %5, 0;\n @q ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];\n}\n"
               : "+r"(raw.x), "+r"(raw.y), "+r"(raw.z), "+r"(raw.w) : "l"(p), "r"((int)yes));
}

// Vectors v0, v0 + step, ... (NV of them) in front of `end`; entries outside the row, and vectors from `end` on, read as -inf.
template <int NV, typename T, int N>
__device__ __forceinline__ void load_vecs(uint4* raw, const RowRef<const T, N>& r, int v0, int step, int end) {
  constexpr uint32_t inf = RawOf<T>::kNegInf;
  bool edge = false;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int v = v0 + k * step;
    raw[k] = make_uint4(inf, inf, inf, inf);
    ldg128_if(raw[k], r.at(v), r.inside(v) && v < end);
    edge |= v < end && !r.inside(v);
  }
  if (edge) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = v0 + k * step;
      if (v < end && !r.inside(v)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int j = v * N - r.head + i;
          if (j >= 0 && j < r.V) set_raw(raw[k], i, r.row[j]);
        }
      }
    }
  }
}

template <typename OutT, int N>
__device__ __forceinline__ void store_vec(const RowRef<OutT, N>& r, int v, const float* x) {
  if (r.inside(v)) { Store<OutT, N>::run(r.at(v), 0u, x); return; }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int j = v * N - r.head + i;
    if (j >= 0 && j < r.V) r.row[j] = from_f32<OutT>(x[i]);
  }
}

// this CTA's share (part of parts) of a row of zeros
template <typename OutT, int N>
__device__ __forceinline__ void zero_row(const RowRef<OutT, N>& r, int part, int parts, int threads) {
  const float zero[N] = {};
  for (int v = part * threads + (int)threadIdx.x; v < r.nvec; v += parts * threads) store_vec<OutT, N>(r, v, zero);
}

}  // namespace dppo
