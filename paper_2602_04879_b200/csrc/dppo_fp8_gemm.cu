// C[M, N] = A[M, K] . B[N, K]^T for 8-bit floating-point operands with an fp32 scale per block of 128 along K.
//
//   C[m, n] = sum_kb sa[m, kb] sb[n, kb] P_kb[m, n],   P_kb[m, n] = sum_{k in block kb} A[m, k] B[n, k]
//
// The tensor cores form P_kb alone (tcgen05.mma kind::f8f6f4, fp32 accumulators in tensor memory, one K block of 128 = four
// instructions); no accumulator carries more than one block, because the scales differ from block to block.  Eight
// promotion warps read each P_kb back (tcgen05.ld), scale it and add it to fp32 sums in their registers, while the tensor cores
// work on the next block in the other half of tensor memory.
//
// One persistent CTA per SM, tiles of 128 x 256:
//   warp 0       TMA producer: 128 x 128-byte boxes of A and 256 x 128-byte boxes of B, 128-byte swizzle, 4 stages
//   warp 1       allocates tensor memory (512 columns: two P_kb buffers) and issues the MMAs
//   warps 2, 3   copy the tile's scales of each K block into a ring of their own (cp.async)
//   warps 4-11   promotion: a warp owns 32 rows (its quarter of the tensor-memory lanes) and 128 of the 256 columns, 128 fp32
//                sums per thread (setmaxnreg moves registers from warps 0-3 to them)
// Every wait is bounded (dppo_pipe.cuh).
#include <mutex>

#include "dppo_common.cuh"
#include "dppo_gemm.cuh"

namespace dppo {
namespace {

namespace f8 {

constexpr int BM = 128, BN = 256, BK = 128;
constexpr int STAGES = 4, SRING = 8;
constexpr int A_BYTES = BM * BK, B_BYTES = BN * BK, STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int SCALE_FLOATS = BM + BN;
constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + SRING * SCALE_FLOATS * 4 + 512 + 1024;
constexpr int THREADS = 384, PROMO_WARPS = 8;
// 384 threads x 168 registers at launch = 64512 = 128 x 72 + 256 x 216
constexpr int REGS_LOW = 72, REGS_HIGH = 216;
static_assert(128 * REGS_LOW + 256 * REGS_HIGH <= THREADS * 168, "register split");

struct Params {
  int M, N, K;
  int a_shift, b_shift;              // log2 of the rows that share a scale (0 or 7)
  const float* sa;
  int64_t sa_row, sa_k;
  const float* sb;
  int64_t sb_row, sb_k;
  void* C;
  int64_t ldc;
  int c_bf16, c_vec;                 // c_vec: 16-byte stores allowed
  uint32_t idesc;
  int32_t* status;
  unsigned long long wait_ns;
  int inject;
};

__device__ __forceinline__ void mma_f8(uint32_t tmem_c, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n"
      ::"r"(tmem_c), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// 4-byte asynchronous copy; zero when not `valid`
__device__ __forceinline__ void cp_async4(uint32_t dst, const float* src, bool valid) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(valid ? 4 : 0) : "memory");
}
// this thread's arrival on the barrier once its copies so far have landed
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

template <bool B_ROW_SCALES>       // B_ROW_SCALES: b_block_rows = 1
__global__ void __launch_bounds__(THREADS, 1) gemm_tn_fp8_kernel(const __grid_constant__ CUtensorMap map_a,
                                                                 const __grid_constant__ CUtensorMap map_b, Params p) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* sring = reinterpret_cast<float*>(smem + STAGES * STAGE_BYTES);
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(sring + SRING * SCALE_FLOATS);
  const uint32_t full0 = smem_u32(bars), empty0 = smem_u32(bars + STAGES);
  const uint32_t tfull0 = smem_u32(bars + 2 * STAGES), tempty0 = smem_u32(bars + 2 * STAGES + 2);
  const uint32_t sfull0 = smem_u32(bars + 2 * STAGES + 4), sempty0 = smem_u32(bars + 2 * STAGES + 4 + SRING);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 4 + 2 * SRING);
  const WaitCtl wc{reinterpret_cast<volatile int*>(tmem_slot + 1), p.wait_ns};
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(full0 + 8 * i, 1); mbar_init(empty0 + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(tfull0 + 8 * i, 1); mbar_init(tempty0 + 8 * i, PROMO_WARPS); }
    for (int i = 0; i < SRING; ++i) { mbar_init(sfull0 + 8 * i, 64); mbar_init(sempty0 + 8 * i, PROMO_WARPS); }
    *wc.flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(2 * BN) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_base = *tmem_slot;

  const int tiles_m = (p.M + BM - 1) / BM, tiles_n = (p.N + BN - 1) / BN;
  const int64_t ntiles = (int64_t)tiles_m * tiles_n;
  const int kblocks = (p.K + BK - 1) / BK;
  const uint32_t smem_base = smem_u32(smem);

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_LOW));
    if (warp == 0) {
      if (lane == 0 && !(p.inject & DPPO_INJECT_NO_COPIES)) {
        int s = 0;
        uint32_t ph = 0;
        bool ok = true;
        for (int64_t tile = blockIdx.x; tile < ntiles && ok; tile += gridDim.x) {
          const int m0 = (int)(tile % tiles_m) * BM, n0 = (int)(tile / tiles_m) * BN;
          for (int kb = 0; kb < kblocks; ++kb) {
            if (!mbar_wait(empty0 + 8 * s, ph ^ 1u, wc)) { ok = false; break; }
            const uint32_t a_dst = smem_base + s * STAGE_BYTES;
            mbar_arrive_expect_tx(full0 + 8 * s, STAGE_BYTES);
            gemm::tma_load_2d(a_dst, &map_a, kb * BK, m0, full0 + 8 * s);
            gemm::tma_load_2d(a_dst + A_BYTES, &map_b, kb * BK, n0, full0 + 8 * s);
            if (++s == STAGES) { s = 0; ph ^= 1u; }
          }
        }
      }
    } else if (warp == 1) {
      if (lane == 0) {
        int s = 0;
        uint32_t ph = 0, it = 0;
        bool ok = true;
        for (int64_t tile = blockIdx.x; tile < ntiles && ok; tile += gridDim.x) {
          for (int kb = 0; kb < kblocks; ++kb, ++it) {
            const uint32_t b = it & 1u, use = it >> 1;
            if (!mbar_wait(tempty0 + 8 * b, (use & 1u) ^ 1u, wc) || !mbar_wait(full0 + 8 * s, ph, wc)) { ok = false; break; }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint64_t adesc = gemm::make_desc_k_sw128(smem_base + s * STAGE_BYTES);
            const uint64_t bdesc = gemm::make_desc_k_sw128(smem_base + s * STAGE_BYTES + A_BYTES);
#pragma unroll
            for (int k = 0; k < BK / 32; ++k)        // 32 elements = 32 bytes along K inside the swizzle atom
              mma_f8(tmem_base + b * BN, adesc + (uint64_t)(k * 2), bdesc + (uint64_t)(k * 2), p.idesc, k != 0);
            gemm::mma_commit(empty0 + 8 * s);
            gemm::mma_commit(tfull0 + 8 * b);
            if (++s == STAGES) { s = 0; ph ^= 1u; }
          }
        }
      }
    } else {
      const int i = tid - 64;                        // 0..63
      int sl = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int64_t tile = blockIdx.x; tile < ntiles && ok; tile += gridDim.x) {
        const int m0 = (int)(tile % tiles_m) * BM, n0 = (int)(tile / tiles_m) * BN;
        for (int kb = 0; kb < kblocks; ++kb) {
          if (!mbar_wait_warp(sempty0 + 8 * sl, ph ^ 1u, wc)) { ok = false; break; }
          const uint32_t dst = smem_u32(sring + sl * SCALE_FLOATS);
          const float* sa = p.sa + kb * p.sa_k;
          const float* sb = p.sb + kb * p.sb_k;
#pragma unroll
          for (int j = i; j < BM; j += 64) {
            const bool in = m0 + j < p.M;
            cp_async4(dst + 4u * j, in ? sa + (int64_t)((m0 + j) >> p.a_shift) * p.sa_row : p.sa, in);
          }
          if (B_ROW_SCALES) {
#pragma unroll
            for (int j = i; j < BN; j += 64) {
              const bool in = n0 + j < p.N;
              cp_async4(dst + 4u * (BM + j), in ? sb + (int64_t)(n0 + j) * p.sb_row : p.sb, in);
            }
          } else if (i < 2) {
            const int n = n0 + i * 128;
            const bool in = n < p.N;
            cp_async4(dst + 4u * (BM + i), in ? sb + (int64_t)(n >> 7) * p.sb_row : p.sb, in);
          }
          cp_async_arrive(sfull0 + 8 * sl);
          if (++sl == SRING) { sl = 0; ph ^= 1u; }
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_HIGH));
    const int q = warp & 3, half = (warp - 4) >> 2;
    uint32_t it = 0, sph = 0;
    int sl = 0;
    bool ok = true;
    for (int64_t tile = blockIdx.x; tile < ntiles && ok; tile += gridDim.x) {
      const int m0 = (int)(tile % tiles_m) * BM, n0 = (int)(tile / tiles_m) * BN + half * 128;
      float acc[128];
#pragma unroll
      for (int j = 0; j < 128; ++j) acc[j] = 0.f;
      for (int kb = 0; kb < kblocks; ++kb, ++it) {
        const uint32_t b = it & 1u, use = it >> 1;
        if (!mbar_wait_warp(sfull0 + 8 * sl, sph, wc)) { ok = false; break; }
        const float* sc = sring + sl * SCALE_FLOATS;
        const float sa = sc[q * 32 + lane];
        const float s = B_ROW_SCALES ? sa : sa * sc[BM + half];
        if (!mbar_wait_warp(tfull0 + 8 * b, use & 1u, wc)) { ok = false; break; }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + b * BN + half * 128;
#pragma unroll
        for (int c = 0; c < 128; c += 32) {
          uint32_t r[32];
          gemm::tmem_ld32(taddr + c, r);
#pragma unroll
          for (int j = 0; j < 32; j += 4) {
            float4 f = make_float4(__uint_as_float(r[j]), __uint_as_float(r[j + 1]), __uint_as_float(r[j + 2]), __uint_as_float(r[j + 3]));
            if (B_ROW_SCALES) {
              const float4 w = *reinterpret_cast<const float4*>(sc + BM + half * 128 + c + j);
              f.x *= w.x; f.y *= w.y; f.z *= w.z; f.w *= w.w;
            }
            acc[c + j] = fmaf(f.x, s, acc[c + j]);
            acc[c + j + 1] = fmaf(f.y, s, acc[c + j + 1]);
            acc[c + j + 2] = fmaf(f.z, s, acc[c + j + 2]);
            acc[c + j + 3] = fmaf(f.w, s, acc[c + j + 3]);
          }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) { mbar_arrive(tempty0 + 8 * b); mbar_arrive(sempty0 + 8 * sl); }
        if (++sl == SRING) { sl = 0; sph ^= 1u; }
      }
      if (!ok) break;
      const int row = m0 + q * 32 + lane;
      if (row < p.M) {
        if (p.c_bf16) {
          __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.C) + (int64_t)row * p.ldc + n0;
#pragma unroll
          for (int j = 0; j < 128; j += 8) {
            if (p.c_vec && n0 + j + 8 <= p.N) {
              uint32_t o[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(acc[j + 2 * e], acc[j + 2 * e + 1]);
                o[e] = *reinterpret_cast<const uint32_t*>(&h);
              }
              *reinterpret_cast<uint4*>(dst + j) = make_uint4(o[0], o[1], o[2], o[3]);
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) if (n0 + j + e < p.N) dst[j + e] = __float2bfloat16_rn(acc[j + e]);
            }
          }
        } else {
          float* dst = reinterpret_cast<float*>(p.C) + (int64_t)row * p.ldc + n0;
#pragma unroll
          for (int j = 0; j < 128; j += 4) {
            if (p.c_vec && n0 + j + 4 <= p.N) {
              *reinterpret_cast<float4*>(dst + j) = make_float4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) if (n0 + j + e < p.N) dst[j + e] = acc[j + e];
            }
          }
        }
      }
    }
  }

  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (wc.aborted()) {
    if (tid == 0 && p.status) atomicOr(p.status, DPPO_STATUS_WAIT_LIMIT);
    drain_after_abort();
  }
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(2 * BN) : "memory");
  }
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn get_encode() {
  static EncodeFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeFn>(ptr);
  });
  return fn;
}
// bytes [rows, cols], boxes of 128 bytes x box_rows rows, 128-byte swizzle; out of range reads as 0
bool make_map(CUtensorMap* map, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  EncodeFn enc = get_encode();
  if (!enc) return false;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld};
  cuuint32_t box[2] = {128u, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1u, 1u};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t launch(const Params& p, const CUtensorMap& ma, const CUtensorMap& mb, cudaStream_t st) {
  int dev = 0, sms = 0;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  const int64_t ntiles = (int64_t)((p.M + BM - 1) / BM) * ((p.N + BN - 1) / BN);
  const unsigned grid = (unsigned)(ntiles < sms ? ntiles : sms);
  auto kernel = p.b_shift ? gemm_tn_fp8_kernel<false> : gemm_tn_fp8_kernel<true>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES);
  if (e != cudaSuccess) return e;
  kernel<<<grid, THREADS, SMEM_BYTES, st>>>(ma, mb, p);
  return cudaGetLastError();
}

}  // namespace f8
}  // namespace
}  // namespace dppo

extern "C" int dppo_gemm_tn_fp8(const void* A, int64_t lda, int a_format, int a_block_rows, const float* a_scale,
                                int64_t a_scale_row_stride, int64_t a_scale_k_stride,
                                const void* B, int64_t ldb, int b_format, int b_block_rows, const float* b_scale,
                                int64_t b_scale_row_stride, int64_t b_scale_k_stride,
                                int M, int N, int K, void* C, int c_dtype, int64_t ldc,
                                int32_t* status, const dppo_opts* opts, void* cuda_stream) {
  using namespace dppo;
  if (M < 0 || N < 0 || K < 0) return DPPO_ERR_SHAPE;
  if (a_format != DPPO_E4M3 && a_format != DPPO_E5M2) return DPPO_ERR_DTYPE;
  if (b_format != DPPO_E4M3 && b_format != DPPO_E5M2) return DPPO_ERR_DTYPE;
  if (c_dtype != DPPO_F32 && c_dtype != DPPO_BF16) return DPPO_ERR_DTYPE;
  if ((a_block_rows != 1 && a_block_rows != 128) || (b_block_rows != 1 && b_block_rows != 128)) return DPPO_ERR_UNSUPPORTED;
  dppo_opts o = {};
  if (opts) o = *opts;
  if (o.wait_limit_us < 0) return DPPO_ERR_UNSUPPORTED;
  if (M == 0 || N == 0) return DPPO_OK;
  if (!C || (K > 0 && (!A || !B || !a_scale || !b_scale))) return DPPO_ERR_NULL;
  if (ldc < N || (K > 0 && (lda < K || ldb < K))) return DPPO_ERR_STRIDE;
  if (K > 0 && (a_scale_row_stride < 0 || a_scale_k_stride < 0 || b_scale_row_stride < 0 || b_scale_k_stride < 0)) return DPPO_ERR_STRIDE;
  const int es = c_dtype == DPPO_BF16 ? 2 : 4;
  if ((uintptr_t)C % es) return DPPO_ERR_ALIGN;
  if (K > 0 && (((uintptr_t)A % 16) || ((uintptr_t)B % 16) || (lda % 16) || (ldb % 16) || ((uintptr_t)a_scale % 4) || ((uintptr_t)b_scale % 4)))
    return DPPO_ERR_ALIGN;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (K == 0)                                            // an empty sum
    return cudaMemset2DAsync(C, (size_t)ldc * es, 0, (size_t)N * es, (size_t)M, st) == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
  f8::Params p = {};
  p.M = M; p.N = N; p.K = K;
  p.a_shift = a_block_rows == 128 ? 7 : 0; p.b_shift = b_block_rows == 128 ? 7 : 0;
  p.sa = a_scale; p.sa_row = a_scale_row_stride; p.sa_k = a_scale_k_stride;
  p.sb = b_scale; p.sb_row = b_scale_row_stride; p.sb_k = b_scale_k_stride;
  p.C = C; p.ldc = ldc; p.c_bf16 = c_dtype == DPPO_BF16;
  p.c_vec = ((uintptr_t)C % 16) == 0 && (ldc * es) % 16 == 0;
  // D = f32 (bit 4), formats of A (bits 7-9) and B (bits 10-12), both K-major, N / 8 (bit 17), M / 16 (bit 24)
  p.idesc = (1u << 4) | ((uint32_t)a_format << 7) | ((uint32_t)b_format << 10) | ((uint32_t)(f8::BN >> 3) << 17) | ((uint32_t)(f8::BM >> 4) << 24);
  p.status = status; p.wait_ns = wait_limit_ns(o.wait_limit_us); p.inject = o.test_inject;
  CUtensorMap ma, mb;
  if (!f8::make_map(&ma, A, M, K, lda, f8::BM) || !f8::make_map(&mb, B, N, K, ldb, f8::BN)) return DPPO_ERR_CUDA;
  return f8::launch(p, ma, mb, st) == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
}
