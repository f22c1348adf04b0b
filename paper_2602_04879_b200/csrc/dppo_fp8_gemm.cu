// C[M, N] = A[M, K] . B[N, K]^T for 8-bit floating-point operands with an fp32 scale per block of 128 along K.
//
//   C[m, n] = sum_kb sa[m, kb] sb[n, kb] P_kb[m, n],   P_kb[m, n] = sum_{k in block kb} A[m, k] B[n, k]
//
// The tensor cores form P_kb alone (tcgen05.mma kind::f8f6f4, fp32 accumulators in tensor memory, one K block of 128 = four
// instructions); no accumulator carries more than one block, because the scales differ from block to block.  Eight
// promotion warps read each P_kb back (tcgen05.ld), scale it and add it to fp32 sums in their registers, while the tensor cores
// work on the next block in the other half of tensor memory.
//
// Persistent CTAs, one per SM:
//   warp 0       TMA producer: boxes of 128 bytes along K, 128-byte swizzle, 4 stages; with each stage the scales of the tile's rows
//                (and of its columns, if each has its own) for that K block, into a ring of 8
//   warp 1       allocates tensor memory (two P_kb buffers) and issues the MMAs
//   warps 2, 3   stand between the mbarriers and the promotion warps: warp 3 waits for a finished P_kb and lets them go, warp 2 hears
//                that they have read it and frees the buffer.  Promotion warps see only named barriers, which cost them a few
//                cycles where polling, and arriving on, an mbarrier cost a few hundred
//   warps 4-11   promotion: a warp owns 32 rows (its quarter of the tensor-memory lanes) and half of the tile's columns, its
//                fp32 sums in registers (setmaxnreg moves registers from warps 0-3 to these); finished tiles leave through shared
//                memory and bulk tensor stores
// CG = 2: pairs of CTAs (a cluster of two SMs, tcgen05 cta_group::2) on tiles of 256 x 192, each CTA staging its 128 rows of A
// and half of the tile's rows of B and promoting its own 128 x 192 sums (96 per thread: a promotion warp then has registers for
// all of its columns of a P_kb at once, reads them in one go and frees the buffer before it adds them up).  CG = 1: single CTAs on tiles of 128 x 128.
// Every wait is bounded.
//
// What bounds it is the hand-over of the P_kb buffers (MMA done -> sums read -> buffer free), two of which are in flight: scales have no
// barrier of their own (the MMA waited for them along with the operands), and the arrival that frees a buffer is relaxed.
#include <mutex>

#include "dppo_common.cuh"
#include "dppo_gemm.cuh"

namespace dppo {
namespace {

namespace f8 {

constexpr int BM = 128, BK = 128;
constexpr int THREADS = 384, PROMO_WARPS = 8;
constexpr int SRING = 8;
// 384 threads x 168 registers at launch = 64512 = 128 x 72 + 256 x 216
constexpr int REGS_LOW = 72, REGS_HIGH = 216;
static_assert(128 * REGS_LOW + 32 * PROMO_WARPS * REGS_HIGH <= THREADS * 168, "register split");

template <int CG> struct Cfg {
  static constexpr int TILE_M = BM * CG, BN = 256;
  static constexpr int B_ROWS = BN / CG;                    // rows of B that one CTA stages
  static constexpr int COLS = 128;                          // columns of a promotion warp
  static constexpr int A_BYTES = BM * BK, B_BYTES = B_ROWS * BK, STAGE_BYTES = A_BYTES + B_BYTES;
  static constexpr int STAGES = CG == 2 ? 5 : 3;
  static constexpr int OUT_BYTES = PROMO_WARPS * 4096;      // 32 rows x 32 columns per promotion warp (two such blocks for bf16)
  static constexpr int SCALES = BM + BN;
  static constexpr int TMEM_BUF = 256, TMEM_COLS = 2 * TMEM_BUF;      // columns between / of the two buffers (a power of two)
  static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + OUT_BYTES + SRING * SCALES * 4 + 512 + 1024;
};

struct Params {
  int M, N, K;
  int a_shift;                       // log2 of the rows of A that share a scale (0 or 7)
  const float* sa;
  int64_t sa_row, sa_k;
  const float* sb;
  int64_t sb_row, sb_k;
  int kblocks;
  int a_tma, b_tma;                  // the scales of the rows of A / B come with the operands (map_sa / map_sb)
  void* C;
  int64_t ldc;
  int c_bf16, c_vec, tma_store;      // c_vec: 16-byte stores allowed; tma_store: map_c describes C
  uint32_t formats;                  // bits of the instruction descriptor
  int32_t* status;
  unsigned long long wait_ns;
  int inject;
};

template <int CG>
__device__ __forceinline__ void mma_f8(uint32_t tmem_c, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  if (CG == 2)
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n"
        ::"r"(tmem_c), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
  else
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n"
        ::"r"(tmem_c), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
template <int CG> __device__ __forceinline__ void commit(uint32_t bar) {
  if (CG == 2) gemm::mma_commit_pair(bar); else gemm::mma_commit(bar);
}
// N columns of this warp's lanes, all on their way before the first is waited for
template <int N> __device__ __forceinline__ void read_columns(uint32_t taddr, uint32_t* r);
template <> __device__ __forceinline__ void read_columns<64>(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%64];\n"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%65];\n"
      "tcgen05.wait::ld.sync.aligned;\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31]), "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]), "=r"(r[40]),
        "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]), "=r"(r[48]), "=r"(r[49]), "=r"(r[50]),
        "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]), "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]),
        "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
      : "r"(taddr + 0), "r"(taddr + 32)
      : "memory");
}
__device__ __forceinline__ uint32_t elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p;
}
// named barriers: promotion warps and one helper warp; one of each kind per P_kb buffer
constexpr int BAR_THREADS = PROMO_WARPS * 32 + 32;
__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("barrier.cta.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void full_sync(uint32_t b) {
  if (b) asm volatile("barrier.cta.sync 4, %0;" ::"n"(BAR_THREADS) : "memory"); else asm volatile("barrier.cta.sync 3, %0;" ::"n"(BAR_THREADS) : "memory");
}
__device__ __forceinline__ void full_arrive(uint32_t b) {
  if (b) asm volatile("barrier.cta.arrive 4, %0;" ::"n"(BAR_THREADS) : "memory"); else asm volatile("barrier.cta.arrive 3, %0;" ::"n"(BAR_THREADS) : "memory");
}
__device__ __forceinline__ void empty_sync(uint32_t b) {
  if (b) asm volatile("barrier.cta.sync 6, %0;" ::"n"(BAR_THREADS) : "memory"); else asm volatile("barrier.cta.sync 5, %0;" ::"n"(BAR_THREADS) : "memory");
}
__device__ __forceinline__ void empty_arrive(uint32_t b) {
  if (b) asm volatile("barrier.cta.arrive 6, %0;" ::"n"(BAR_THREADS) : "memory"); else asm volatile("barrier.cta.arrive 5, %0;" ::"n"(BAR_THREADS) : "memory");
}
// Arrivals that order none of this thread's memory accesses: what they hand over is a tensor-memory buffer that has been read
// (tcgen05.fence orders that), not shared memory.  A release would wait for the thread's loads of the coming scales, and at cluster
// scope for much more: the tensor cores waited 1000 and 2000 cycles a block for it.
__device__ __forceinline__ void arrive_relaxed(uint32_t bar) {
  asm volatile("mbarrier.arrive.relaxed.cta.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void arrive_relaxed_cluster(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void st128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint32_t bf16x2(float2 v) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// acc[0, 16) += s * r (* the column's scale): 32 columns of one row, packed fp32 pairs
template <bool B_ROW_SCALES>
__device__ __forceinline__ void promote32(float2* acc, const uint32_t* r, float s, const float* sb) {
  const float2 s2 = make_float2(s, s);
#pragma unroll
  for (int j = 0; j < 32; j += 4) {
    float2 u = make_float2(__uint_as_float(r[j]), __uint_as_float(r[j + 1])), v = make_float2(__uint_as_float(r[j + 2]), __uint_as_float(r[j + 3]));
    if (B_ROW_SCALES) {
      const float4 w = *reinterpret_cast<const float4*>(sb + j);
      u = __fmul2_rn(u, make_float2(w.x, w.y));
      v = __fmul2_rn(v, make_float2(w.z, w.w));
    }
    acc[j / 2] = __ffma2_rn(u, s2, acc[j / 2]);
    acc[j / 2 + 1] = __ffma2_rn(v, s2, acc[j / 2 + 1]);
  }
}

template <int CG, bool B_ROW_SCALES>       // B_ROW_SCALES: b_block_rows = 1
__global__ void __launch_bounds__(THREADS, 1) gemm_tn_fp8_kernel(const __grid_constant__ CUtensorMap map_a,
                                                                 const __grid_constant__ CUtensorMap map_b,
                                                                 const __grid_constant__ CUtensorMap map_c,
                                                                 const __grid_constant__ CUtensorMap map_sa,
                                                                 const __grid_constant__ CUtensorMap map_sb, Params p) {
  using C = Cfg<CG>;
  constexpr int STAGES = C::STAGES, STAGE_BYTES = C::STAGE_BYTES, BN = C::BN, COLS = C::COLS;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* out_stage = smem + STAGES * STAGE_BYTES;
  float* sring = reinterpret_cast<float*>(out_stage + C::OUT_BYTES);
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(sring + SRING * C::SCALES);
  const uint32_t full0 = smem_u32(bars), done0 = smem_u32(bars + STAGES);
  const uint32_t tempty0 = smem_u32(bars + 2 * STAGES);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 2);
  const WaitCtl wc{reinterpret_cast<volatile int*>(tmem_slot + 1), p.wait_ns};
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = (CG == 2) ? cluster_ctarank() : 0u;       // 0: leader of the pair
  const int group = (int)blockIdx.x / CG, ngroups = (int)gridDim.x / CG;

  if (tid == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(full0 + 8 * i, 1); mbar_init(done0 + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) mbar_init(tempty0 + 8 * i, CG);
    *wc.flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    if (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(C::TMEM_COLS) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(C::TMEM_COLS) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG == 2) cluster_sync_all();      // the peer's barriers exist before anything is sent to them
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_base = *tmem_slot;

  const int tiles_m = (p.M + C::TILE_M - 1) / C::TILE_M, tiles_n = (p.N + BN - 1) / BN;
  const int64_t ntiles = (int64_t)tiles_m * tiles_n;
  const int kblocks = p.kblocks;
  const uint32_t smem_base = smem_u32(smem);

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_LOW));
    if (warp == 0) {
      // ---------------------------------------------------------------- TMA producer (of this CTA's operand slices)
      if (lane == 0 && !(p.inject & DPPO_INJECT_NO_COPIES)) {
        constexpr uint32_t kSlot = C::SCALES * 4;
        const uint32_t bytes = STAGE_BYTES + (p.a_tma ? BM * 4 : 0) + (B_ROW_SCALES && p.b_tma ? BN * 4 : 0), ring = smem_u32(sring);
        int s = 0;
        uint32_t ph = 0, it = 0;
        bool ok = true;
        for (int64_t tile = group; tile < ntiles && ok; tile += ngroups) {
          const int m0 = (int)(tile % tiles_m) * C::TILE_M + (int)rank * BM, n0 = (int)(tile / tiles_m) * BN;
          for (int kb = 0; kb < kblocks; ++kb, ++it) {
            if (!mbar_wait(done0 + 8 * s, ph ^ 1u, wc)) { ok = false; break; }
            const uint32_t a_dst = smem_base + s * STAGE_BYTES, b_dst = a_dst + C::A_BYTES;
            // The slot's last scales were those of 8 K blocks ago.  A stage is free once the MMAs of 4 blocks ago are done, and
            // those began after every promotion warp had read the block 2 before them: nobody reads the slot any more.
            const uint32_t sc_dst = ring + (it % SRING) * kSlot;
            if (CG == 2) {       // both CTAs' bytes are counted on the leader's barrier
              const uint32_t bar = map_to_cta(full0 + 8 * s, 0);
              if (rank == 0) mbar_arrive_expect_tx(full0 + 8 * s, 2 * bytes);
              gemm::tma_load_2d_pair(a_dst, &map_a, kb * BK, m0, bar);
              gemm::tma_load_2d_pair(b_dst, &map_b, kb * BK, n0 + (int)rank * C::B_ROWS, bar);
              if (p.a_tma) gemm::tma_load_2d_pair(sc_dst, &map_sa, m0, kb, bar);
              if (B_ROW_SCALES && p.b_tma) gemm::tma_load_2d_pair(sc_dst + BM * 4, &map_sb, n0, kb, bar);
            } else {
              mbar_arrive_expect_tx(full0 + 8 * s, bytes);
              gemm::tma_load_2d(a_dst, &map_a, kb * BK, m0, full0 + 8 * s);
              gemm::tma_load_2d(b_dst, &map_b, kb * BK, n0, full0 + 8 * s);
              if (p.a_tma) gemm::tma_load_2d(sc_dst, &map_sa, m0, kb, full0 + 8 * s);
              if (B_ROW_SCALES && p.b_tma) gemm::tma_load_2d(sc_dst + BM * 4, &map_sb, n0, kb, full0 + 8 * s);
            }
            if (++s == STAGES) { s = 0; ph ^= 1u; }
          }
        }
      }
    } else if (warp == 1) {
      // ---------------------------------------------------------------- MMA issuer (in a pair: the leader's only)
      // (the whole warp runs the loop, so that descriptors and addresses are warp-uniform values for the compiler, and one elected
      // lane issues: with a single lane in the loop each MMA took three times as long to issue)
      if (rank == 0) {
        const uint32_t idesc = p.formats | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(C::TILE_M >> 4) << 24);
        const uint64_t adesc0 = gemm::make_desc_k_sw128(smem_base), bdesc0 = gemm::make_desc_k_sw128(smem_base + C::A_BYTES);
        int s = 0;
        uint32_t ph = 0, it = 0;
        bool ok = true;
        for (int64_t tile = group; tile < ntiles && ok; tile += ngroups) {
          for (int kb = 0; kb < kblocks; ++kb, ++it) {
            const uint32_t b = it & 1u, use = it >> 1;
            ok = mbar_wait(tempty0 + 8 * b, (use & 1u) ^ 1u, wc) && mbar_wait(full0 + 8 * s, ph, wc);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint64_t adesc = adesc0 + (uint64_t)(s * (STAGE_BYTES >> 4)), bdesc = bdesc0 + (uint64_t)(s * (STAGE_BYTES >> 4));
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < BK / 32; ++k)      // 32 elements = 32 bytes along K inside the swizzle atom
                mma_f8<CG>(tmem_base + b * C::TMEM_BUF, adesc + (uint64_t)(k * 2), bdesc + (uint64_t)(k * 2), idesc, k != 0);
              commit<CG>(done0 + 8 * s);             // the stage may be filled again, and P_kb is complete
            }
            __syncwarp();
            if (++s == STAGES) { s = 0; ph ^= 1u; }
          }
        }
      }
    } else {
      // ---------------------------------------------------------------- helpers.  They serve every K block even after a wait ran
      // out (mbar_wait then returns at once), so that no one is left at a named barrier.
      const uint32_t tempty = CG == 2 ? map_to_cta(tempty0, 0) : tempty0;
      int s = 0;
      uint32_t it = 0, ph = 0;
      for (int64_t tile = group; tile < ntiles; tile += ngroups) {
        for (int kb = 0; kb < kblocks; ++kb, ++it) {
          const uint32_t b = it & 1u;
          if (warp == 3) {
            if (!wc.aborted()) mbar_wait(done0 + 8 * s, ph, wc);
            __syncwarp();
            if (++s == STAGES) { s = 0; ph ^= 1u; }
            full_arrive(b);
          } else {
            empty_sync(b);
            if (lane == 0) { if (CG == 2) arrive_relaxed_cluster(tempty + 8 * b); else arrive_relaxed(tempty + 8 * b); }
          }
        }
      }
    }
  } else {
    // ------------------------------------------------------------------ promotion
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_HIGH));
    const int q = warp & 3, part = (warp - 4) >> 2;
    const uint32_t wbuf = smem_u32(out_stage) + (uint32_t)(warp - 4) * 4096u;
    const bool a_direct = !p.a_shift && !p.a_tma, b_direct = B_ROW_SCALES && !p.b_tma;
    uint32_t it = 0, out_it = 0;
    for (int64_t tile = group; tile < ntiles; tile += ngroups) {
      const int m0 = (int)(tile % tiles_m) * C::TILE_M + (int)rank * BM + q * 32, n0 = (int)(tile / tiles_m) * BN + part * COLS;
      const bool live = m0 < p.M && n0 < p.N;        // this warp's part of the tile meets C (what it adds up otherwise is not stored)
      float2 acc[COLS / 2];
#pragma unroll
      for (int j = 0; j < COLS / 2; ++j) acc[j] = make_float2(0.f, 0.f);
      // scales that all rows (columns) of this warp share: lane i keeps the one of K block kb0 + i
      for (int kb0 = 0; kb0 < kblocks; kb0 += 32) {
        float shared_s = 1.f;
        if (live && kb0 + lane < kblocks) {
          if (p.a_shift) shared_s = p.sa[(int64_t)(m0 >> 7) * p.sa_row + (kb0 + lane) * p.sa_k];
          if (!B_ROW_SCALES) shared_s *= p.sb[(int64_t)(n0 >> 7) * p.sb_row + (kb0 + lane) * p.sb_k];
        }
        const int kn = min(32, kblocks - kb0);
        float s = __shfl_sync(0xffffffffu, shared_s, 0);
#pragma unroll 1
        for (int i = 0; i < kn; ++i, ++it) {
          const uint32_t b = it & 1u;
          float* sc = sring + (it % SRING) * C::SCALES;
          float* sbv = sc + BM + part * COLS;
          full_sync(b);
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const float sa = p.a_tma ? sc[q * 32 + lane] : 1.f;
          const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + b * C::TMEM_BUF + part * COLS;
          uint32_t r[64];
          read_columns<64>(taddr, r);
          s *= sa;
          if (a_direct && m0 + lane < p.M) s *= p.sa[(int64_t)(m0 + lane) * p.sa_row + (kb0 + i) * p.sa_k];
          if (b_direct) {                            // column scales of a layout that no tensor map describes: one by one, a part each
            for (int j = q * 32 + lane; j < COLS; j += 128) sbv[j] = n0 + j < p.N ? p.sb[(int64_t)(n0 + j) * p.sb_row + (kb0 + i) * p.sb_k] : 0.f;
            bar_sync(7 + part, 128);
          }
          promote32<B_ROW_SCALES>(acc, r, s, sbv);
          promote32<B_ROW_SCALES>(acc + 16, r + 32, s, sbv + 32);
          read_columns<64>(taddr + 64, r);
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          empty_arrive(b);                           // buffer read
          const float s_next = __shfl_sync(0xffffffffu, shared_s, (i + 1) & 31);
          promote32<B_ROW_SCALES>(acc + 32, r, s, sbv + 64);
          promote32<B_ROW_SCALES>(acc + 48, r + 32, s, sbv + 96);
          s = s_next;
          if (b_direct) bar_sync(7 + part, 128);     // before the slot's scales are written again
        }
      }
      if (!live) continue;
      const int row = m0 + lane;
      if (p.tma_store) {
        // 32 rows x 32 columns at a time through the warp's block(s), 16-byte pieces placed by the 128-byte (fp32) or
        // 64-byte (bf16) swizzle
#pragma unroll
        for (int c = 0; c < COLS / 32; ++c) {
          if (n0 + c * 32 >= p.N) break;
          const uint32_t buf = wbuf + (p.c_bf16 ? (out_it & 1u) * 2048u : 0u);
          const float2* v = acc + c * 16;
          if (lane == 0) { if (p.c_bf16) gemm::bulk_wait_read<1>(); else gemm::bulk_wait_read<0>(); }
          __syncwarp();
          if (p.c_bf16) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              st128(buf + (uint32_t)lane * 64u + (uint32_t)((j ^ ((lane >> 1) & 3)) * 16), bf16x2(v[4 * j]), bf16x2(v[4 * j + 1]), bf16x2(v[4 * j + 2]), bf16x2(v[4 * j + 3]));
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
              st128(buf + (uint32_t)lane * 128u + (uint32_t)((j ^ (lane & 7)) * 16), __float_as_uint(v[2 * j].x), __float_as_uint(v[2 * j].y),
                    __float_as_uint(v[2 * j + 1].x), __float_as_uint(v[2 * j + 1].y));
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) { gemm::tma_store_2d(&map_c, buf, n0 + c * 32, m0); gemm::bulk_commit(); }
          ++out_it;
        }
      } else if (row < p.M) {
        if (p.c_bf16) {
          __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.C) + (int64_t)row * p.ldc + n0;
#pragma unroll
          for (int j = 0; j < COLS; j += 2) {
            if (n0 + j < p.N) dst[j] = __float2bfloat16_rn(acc[j / 2].x);
            if (n0 + j + 1 < p.N) dst[j + 1] = __float2bfloat16_rn(acc[j / 2].y);
          }
        } else {
          float* dst = reinterpret_cast<float*>(p.C) + (int64_t)row * p.ldc + n0;
#pragma unroll
          for (int j = 0; j < COLS; j += 2) {
            if (n0 + j < p.N) dst[j] = acc[j / 2].x;
            if (n0 + j + 1 < p.N) dst[j + 1] = acc[j / 2].y;
          }
        }
      }
    }
    if (lane == 0 && out_it > 0) gemm::bulk_wait_all<0>();
  }

  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  // after a wait ran out: time for loads and tensor-core work still under way
  if (wc.aborted()) {
    if (tid == 0 && p.status) atomicOr(p.status, DPPO_STATUS_WAIT_LIMIT);
    drain_after_abort();
  }
  if (CG == 2) cluster_sync_all();      // a pair leaves together
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::TMEM_COLS) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::TMEM_COLS) : "memory");
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
// Row-major matrix [rows, cols], boxes of box_cols x box_rows (64 or 128 bytes wide, swizzled alike); out of range reads as 0
bool make_map(CUtensorMap* map, CUtensorMapDataType type, int es, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_cols, int box_rows) {
  EncodeFn enc = get_encode();
  if (!enc) return false;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld * es};
  cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1u, 1u};
  return enc(map, type, 2, const_cast<void*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, box_cols * es == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Scales [rows, kblocks] with adjacent rows, boxes of `box` rows of one K block; false if the layout does not allow a map
bool make_scale_map(CUtensorMap* map, const float* base, int64_t rows, int64_t row_stride, int64_t kblocks, int64_t k_stride, int box) {
  EncodeFn enc = get_encode();
  if (!enc || row_stride != 1 || k_stride % 4 != 0 || k_stride < rows || ((uintptr_t)base % 16) != 0) return false;
  cuuint64_t dims[2] = {(cuuint64_t)rows, (cuuint64_t)kblocks};
  cuuint64_t strides[1] = {(cuuint64_t)k_stride * 4};
  cuuint32_t boxes[2] = {(cuuint32_t)box, 1u};
  cuuint32_t estr[2] = {1u, 1u};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, const_cast<float*>(base), dims, strides, boxes, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int CG, bool B_ROW_SCALES>
cudaError_t launch(Params p, const void* A, int64_t lda, const void* B, int64_t ldb, int sms, cudaStream_t st) {
  using C = Cfg<CG>;
  CUtensorMap ma, mb, mc, msa, msb;
  if (!make_map(&ma, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, A, p.M, p.K, lda, 128, BM)) return cudaErrorInvalidValue;
  if (!make_map(&mb, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, B, p.N, p.K, ldb, 128, C::B_ROWS)) return cudaErrorInvalidValue;
  mc = msa = msb = ma;
  p.a_tma = !p.a_shift && make_scale_map(&msa, p.sa, p.M, p.sa_row, p.kblocks, p.sa_k, BM);
  p.b_tma = B_ROW_SCALES && make_scale_map(&msb, p.sb, p.N, p.sb_row, p.kblocks, p.sb_k, C::BN);
  p.tma_store = p.c_vec && make_map(&mc, p.c_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, p.c_bf16 ? 2 : 4, p.C, p.M, p.N,
                                    p.ldc, 32, 32);
  auto kernel = gemm_tn_fp8_kernel<CG, B_ROW_SCALES>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM_BYTES);
  if (e != cudaSuccess) return e;
  const int64_t ntiles = (int64_t)((p.M + C::TILE_M - 1) / C::TILE_M) * ((p.N + C::BN - 1) / C::BN);
  const int slots = sms / CG;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((ntiles < slots ? ntiles : slots) * CG));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = C::SMEM_BYTES;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CG; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = (CG > 1) ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, ma, mb, mc, msa, msb, p);
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
  if (o.gemm_cta_group < 0 || o.gemm_cta_group > 2 || o.wait_limit_us < 0) return DPPO_ERR_UNSUPPORTED;
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
  p.a_shift = a_block_rows == 128 ? 7 : 0;
  p.sa = a_scale; p.sa_row = a_scale_row_stride; p.sa_k = a_scale_k_stride;
  p.sb = b_scale; p.sb_row = b_scale_row_stride; p.sb_k = b_scale_k_stride;
  p.kblocks = (K + f8::BK - 1) / f8::BK;
  p.C = C; p.ldc = ldc; p.c_bf16 = c_dtype == DPPO_BF16;
  p.c_vec = ((uintptr_t)C % 16) == 0 && (ldc * es) % 16 == 0;
  // instruction descriptor: D = f32 (bit 4), formats of A (bits 7-9) and B (bits 10-12), both K-major
  p.formats = (1u << 4) | ((uint32_t)a_format << 7) | ((uint32_t)b_format << 10);
  p.status = status; p.wait_ns = wait_limit_ns(o.wait_limit_us); p.inject = o.test_inject;
  int dev = 0, sms = 0;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  const int64_t pair_tiles = (int64_t)((M + 255) / 256) * ((N + 255) / 256);
  const bool pairs = o.gemm_cta_group == 2 || (o.gemm_cta_group == 0 && M > 128 && pair_tiles >= sms / 4);
  cudaError_t e;
  if (pairs) e = b_block_rows == 1 ? f8::launch<2, true>(p, A, lda, B, ldb, sms, st) : f8::launch<2, false>(p, A, lda, B, ldb, sms, st);
  else e = b_block_rows == 1 ? f8::launch<1, true>(p, A, lda, B, ldb, sms, st) : f8::launch<1, false>(p, A, lda, B, ldb, sms, st);
  return e == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
}
