// C[M, N] = A[M, K] . B[N, K]^T for 8-bit floating-point operands with an fp32 scale per block of 128 along K.
//
//   C[m, n] = sum_kb sa[m, kb] sb[n, kb] P_kb[m, n],   P_kb[m, n] = sum_{k in block kb} A[m, k] B[n, k]
//
// The tensor cores form P_kb alone (tcgen05.mma kind::f8f6f4, fp32 accumulators in tensor memory, one K block of 128 = four
// instructions); no accumulator carries more than one block, because the scales differ from block to block.  Eight
// promotion warps read each P_kb back (tcgen05.ld), scale it and add it to fp32 sums in their registers, while the tensor cores
// work on the next block in the other half of tensor memory.
//
// Persistent CTAs, one per SM, tiles of 128 x w (w = 256 or 128, chosen per call):
//   warp 0       producer: TMA boxes of 128 bytes along K, 128-byte swizzle, 3 stages; with each stage the scales of the tile's rows and
//                columns for that K block by 4-byte asynchronous copies (any strides) into a ring of 8
//   warp 1       allocates tensor memory (two P_kb buffers) and issues the MMAs
//   warps 2, 3   stand between the mbarriers and the promotion warps: warp 3 waits for a finished P_kb and lets them go, warp 2 hears
//                that they have read it and frees the buffer.  Promotion warps see only named barriers, which cost them a few
//                cycles where polling, and arriving on, an mbarrier cost a few hundred
//   warps 4-11   promotion: a warp owns 32 rows (its quarter of the tensor-memory lanes) and 128 of the columns, its fp32 sums in
//                registers (setmaxnreg moves registers from warps 0-3 to these); finished tiles leave through shared memory and
//                bulk tensor stores
// With few tiles and a long K a cluster of S CTAs shares a tile: each sums an S-th part of the K blocks, leaves its sums in its shared
// memory, and all add up a part of the rows each, CTA after CTA (a fixed order), through distributed shared memory.
// Every wait on an mbarrier is bounded (dppo_pipe.cuh).  The named barriers come to an end because warps 2 and 3 serve every block of
// every tile whatever happened before (the rule stands at their loop), the cluster barriers because then every warp's loop ends.
//
// What bounds the K loop is the hand-over of the P_kb buffers (MMA done -> sums read -> buffer free), two of which are in flight, and the
// fp32 additions themselves (256 of the 512 cycles that the MMAs of a block take at their nominal rate).  Scales have no barrier of
// their own: the MMA waits for them along with the operands.  Outside the K loop: the promotion warps store a finished tile themselves,
// and the tensor cores stop once both buffers are full (per busy SM, tiles of 16 K blocks run at 14.2 TFLOP/s, of 1187 at 16.1); tiles
// run with M fastest, so that an A beyond L2 is read again for each column of tiles (151936 x 2048 x 2048: 2.58 GB read where A and
// B are 315 MB); a last round of few tiles leaves SMs idle (2048 x 2048: 128 tiles on 148 SMs).
//
// Measured on B200 (the same call over and over; e4m3, scales 1 x 128 for A and 128 x 128 for B unless said): 4096 x 151936 x 2048 to bf16
// 1.21 ms = 2.11 PFLOP/s (a bf16 GEMM peaks at 1.67 here; on a GPU warm from other work, inputs changed from call to call, 1.39 ms =
// 1.84 PFLOP/s); 151936 x 2048 x 2048 with scales 1 x 128 on both sides 1.02-1.04 ms = 1.23-1.25 PFLOP/s; 61 x 151936 x 2048 65 us =
// 5.0 TB/s, 77 % of a copy's rate; 64 x 2048 x 151936 87 us, 500 us without the split along K; to a C that no tensor map describes,
// 1796 x 50257 x 1024 to fp32 233 us, 132 us with N = 50256.  Single-SM tiles were as fast as pairs of SMs (the hand-over sets the pace, not
// the operands), and simpler to feed scales to.
#include <cooperative_groups.h>
#include <mutex>

#include "dppo_common.cuh"
#include "dppo_gemm.cuh"

namespace dppo {
namespace {

namespace f8 {

constexpr int BM = 128, BN = 256, BK = 128;                // BN: the widest tile
constexpr int COLS = 128;                                  // columns of a promotion warp
constexpr int THREADS = 384, PROMO_WARPS = 8;
constexpr int STAGES = 3, SRING = 8, SCALES = BM + BN;
constexpr int A_BYTES = BM * BK, STAGE_BYTES = (BM + BN) * BK;
constexpr int OUT_BYTES = PROMO_WARPS * 8192;              // two blocks of 32 rows x 128 bytes per promotion warp
constexpr int PART_PITCH = BN + 4;                         // floats; a CTA's sums of a shared tile, in the stages' memory
constexpr int MAX_SPLIT = 8;
constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + OUT_BYTES + SRING * SCALES * 4 + 512 + 1024;
static_assert(BM * PART_PITCH * 4 <= STAGES * STAGE_BYTES, "partial tile");
// 384 threads x 168 registers at launch = 64512 = 128 x 72 + 256 x 216
constexpr int REGS_LOW = 72, REGS_HIGH = 216;
static_assert(128 * REGS_LOW + 32 * PROMO_WARPS * REGS_HIGH <= THREADS * 168, "register split");

struct Params {
  int M, N, bn, split;               // bn: columns of a tile; split: CTAs that share a tile
  int a_shift;                       // log2 of the rows of A that share a scale (0 or 7; B: the template argument)
  const float* sa;
  int64_t sa_row, sa_k;
  const float* sb;
  int64_t sb_row, sb_k;
  int kblocks;
  void* C;
  int64_t ldc;
  int c_bf16, c_vec;                 // c_vec: 16-byte stores allowed
  int n_tma;                         // columns of C that map_c describes: whole 16-byte pieces of a row (0: no map)
  uint32_t formats;                  // bits of the instruction descriptor
  int32_t* status;
  unsigned long long wait_ns;
  int inject;
};

__device__ __forceinline__ void mma_f8(uint32_t tmem_c, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n"
      ::"r"(tmem_c), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// 64 columns of this warp's 32 lanes: r[j] is column j of the thread's row
__device__ __forceinline__ void read_rows(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
      "%24,%25,%26,%27,%28,%29,%30,%31,%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,"
      "%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%64];\n"
      "tcgen05.wait::ld.sync.aligned;\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]),
        "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
        "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
        "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]),
        "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
      : "r"(taddr)
      : "memory");
}
// 64 columns of 16 lanes in the layout of a matrix-instruction accumulator: r[4 g], r[4 g + 1] are columns 8 g + 2 (lane % 4), + 1 of row
// lane / 4, r[4 g + 2], r[4 g + 3] those of row lane / 4 + 8
__device__ __forceinline__ void read_fragment(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
      "%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
      "tcgen05.wait::ld.sync.aligned;\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
// 4-byte asynchronous copy of base[at]; zero when not `valid`
__device__ __forceinline__ void cp_async4(uint32_t dst, const float* base, int64_t at, bool valid) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(valid ? base + at : base), "r"(valid ? 4 : 0) : "memory");
}
// this thread's arrival on the barrier once its copies so far have landed
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(p));
  return p;
}
// named barriers: promotion warps and one helper warp; one of each kind per P_kb buffer
constexpr int BAR_THREADS = PROMO_WARPS * 32 + 32;
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
__device__ __forceinline__ void st128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void st64(uint32_t addr, float2 v) {
  asm volatile("st.shared.v2.f32 [%0], {%1,%2};" ::"r"(addr), "f"(v.x), "f"(v.y) : "memory");
}
__device__ __forceinline__ void st32(uint32_t addr, uint32_t v) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ uint32_t bf16x2(float2 v) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// acc += s * r: 64 columns of one row, packed fp32 pairs
__device__ __forceinline__ void promote_rows(float2* acc, const uint32_t* r, float s) {
  const float2 s2 = make_float2(s, s);
#pragma unroll
  for (int j = 0; j < 32; ++j) acc[j] = __ffma2_rn(make_float2(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1])), s2, acc[j]);
}
// Reads a fragment of 16 rows x 64 columns (LAST: of buffer b); acc += s0, s1 (the two rows) * sb (the columns') * fragment.  The thread
// needs only every fourth pair of the column scales: read by one row per thread, each warp would fetch all 128 of them for every
// block, and the shared memory's 128 bytes a cycle would be what bounds the kernel.
// (The products of the scales are formed before the fragment is waited for.)
template <bool LAST> __device__ __forceinline__ void read_and_promote(uint32_t taddr, float2* acc, float s0, float s1, const float* sb, uint32_t b) {
  float2 w0[8], w1[8];
#pragma unroll
  for (int g = 0; g < 8; ++g) {
    const float2 w = *reinterpret_cast<const float2*>(sb + 8 * g);
    w0[g] = __fmul2_rn(w, make_float2(s0, s0));
    w1[g] = __fmul2_rn(w, make_float2(s1, s1));
  }
  uint32_t r[32];
  read_fragment(taddr, r);
  if (LAST) {                              // buffer b read
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    empty_arrive(b);
  }
#pragma unroll
  for (int g = 0; g < 8; ++g) {
    acc[2 * g] = __ffma2_rn(make_float2(__uint_as_float(r[4 * g]), __uint_as_float(r[4 * g + 1])), w0[g], acc[2 * g]);
    acc[2 * g + 1] = __ffma2_rn(make_float2(__uint_as_float(r[4 * g + 2]), __uint_as_float(r[4 * g + 3])), w1[g], acc[2 * g + 1]);
  }
}

// element (r, in) of a warp's two staged blocks (32 rows x 128 bytes each, 128-byte swizzle) to C[at]
__device__ __forceinline__ void store_staged(const Params& p, const unsigned char* blocks, int r, int in, int64_t at) {
  const int ncol = p.c_bf16 ? 64 : 32, byte = (in % ncol) * (p.c_bf16 ? 2 : 4);
  const unsigned char* src = blocks + (in / ncol) * 4096 + r * 128 + ((((byte >> 4) ^ (r & 7)) << 4) | (byte & 15));
  if (p.c_bf16) reinterpret_cast<unsigned short*>(p.C)[at] = *reinterpret_cast<const unsigned short*>(src);
  else reinterpret_cast<float*>(p.C)[at] = *reinterpret_cast<const float*>(src);
}

template <bool B_ROW_SCALES>       // b_block_rows = 1
__global__ void __launch_bounds__(THREADS, 1) gemm_tn_fp8_kernel(const __grid_constant__ CUtensorMap map_a,
                                                                 const __grid_constant__ CUtensorMap map_b,
                                                                 const __grid_constant__ CUtensorMap map_c, Params p) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* out_stage = smem + STAGES * STAGE_BYTES;
  float* sring = reinterpret_cast<float*>(out_stage + OUT_BYTES);
  unsigned long long* bars = reinterpret_cast<unsigned long long*>(sring + SRING * SCALES);
  const uint32_t full0 = smem_u32(bars), done0 = smem_u32(bars + STAGES), tempty0 = smem_u32(bars + 2 * STAGES);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 2);
  const WaitCtl wc{reinterpret_cast<volatile int*>(tmem_slot + 1), p.wait_ns};
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = p.split > 1 ? (int)cluster_ctarank() : 0;
  const int group = (int)blockIdx.x / p.split, ngroups = (int)gridDim.x / p.split;

  if (tid == 0) {
    for (int i = 0; i < STAGES; ++i) { mbar_init(full0 + 8 * i, 1 + 32); mbar_init(done0 + 8 * i, 2); }
    for (int i = 0; i < 2; ++i) mbar_init(tempty0 + 8 * i, 1);
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

  const int bn = p.bn, tiles_m = (p.M + BM - 1) / BM, tiles_n = (p.N + bn - 1) / bn;
  const int ntiles = tiles_m * tiles_n;
  const int per = (p.kblocks + p.split - 1) / p.split, kb_first = min(p.kblocks, rank * per);
  const int kblocks = min(p.kblocks, kb_first + per) - kb_first;      // this CTA's K blocks of each tile
  const uint32_t smem_base = smem_u32(smem);

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_LOW));
    if (warp == 0) {
      // ---------------------------------------------------------------- producer
      if (!(p.inject & DPPO_INJECT_NO_COPIES)) {
        const uint32_t bytes = A_BYTES + bn * BK, ring = smem_u32(sring);
        int s = 0;
        uint32_t ph = 0, it = 0;
        bool ok = true;
        for (int tile = group; tile < ntiles && ok; tile += ngroups) {
          const int m0 = (tile % tiles_m) * BM, n0 = (tile / tiles_m) * bn;
          const float* sa = p.sa + (int64_t)(m0 >> p.a_shift) * p.sa_row + kb_first * p.sa_k;
          const float* sb = p.sb + (int64_t)(B_ROW_SCALES ? n0 : n0 >> 7) * p.sb_row + kb_first * p.sb_k;
          for (int kb = kb_first; kb < kb_first + kblocks; ++kb, ++it) {
            if (!mbar_wait_warp(done0 + 8 * s, ph ^ 1u, wc)) { ok = false; break; }
            const uint32_t a_dst = smem_base + s * STAGE_BYTES, bar = full0 + 8 * s;
            if (lane == 0) {
              mbar_arrive_expect_tx(bar, bytes);
              gemm::tma_load_2d(a_dst, &map_a, kb * BK, m0, bar);
              gemm::tma_load_2d(a_dst + A_BYTES, &map_b, kb * BK, n0, bar);
            }
            // Scales are plain shared-memory data, which a commit does not order.  They reach the promotion warps through the issuer:
            // its wait for `full` sees them landed, its own arrival on `done` passes that on, warp 3 and a named barrier hand it over.  And
            // back: the slot's last scales were those of 8 K blocks ago; a stage is free once the issuer has arrived for the block 3
            // before, after its wait for the buffer that every promotion warp had left with the block 5 before.  Nobody reads the slot.
            const uint32_t sc = ring + (it % SRING) * (SCALES * 4);
            if (!p.a_shift) {
#pragma unroll
              for (int j = 0; j < BM; j += 32) cp_async4(sc + 4 * (j + lane), sa, (int64_t)(j + lane) * p.sa_row, m0 + j + lane < p.M);
            } else if (lane == 0) {
              cp_async4(sc, sa, 0, true);
            }
            if (B_ROW_SCALES) {
#pragma unroll
              for (int j = 0; j < BN; j += 32) cp_async4(sc + 4 * (BM + j + lane), sb, (int64_t)(j + lane) * p.sb_row, n0 + j + lane < p.N);
            } else if (lane < 2) {
              cp_async4(sc + 4 * (BM + lane), sb, lane * p.sb_row, n0 + lane * 128 < p.N);
            }
            cp_async_arrive(bar);
            sa += p.sa_k;
            sb += p.sb_k;
            if (++s == STAGES) { s = 0; ph ^= 1u; }
          }
        }
      }
    } else if (warp == 1) {
      // ---------------------------------------------------------------- MMA issuer
      // (the whole warp runs the loop, so that descriptors and addresses are warp-uniform values for the compiler, and one elected
      // lane issues: with a single lane in the loop each MMA took three times as long to issue)
      const uint32_t idesc = p.formats | ((uint32_t)(bn >> 3) << 17) | ((uint32_t)(BM >> 4) << 24);
      const uint64_t adesc0 = gemm::make_desc_k_sw128(smem_base), bdesc0 = gemm::make_desc_k_sw128(smem_base + A_BYTES);
      int s = 0;
      uint32_t ph = 0, it = 0;
      bool ok = true;
      for (int tile = group; tile < ntiles && ok; tile += ngroups) {
        for (int kb = 0; kb < kblocks; ++kb, ++it) {
          const uint32_t b = it & 1u, use = it >> 1;
          ok = mbar_wait(tempty0 + 8 * b, (use & 1u) ^ 1u, wc) && mbar_wait(full0 + 8 * s, ph, wc);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint64_t adesc = adesc0 + (uint64_t)(s * (STAGE_BYTES >> 4)), bdesc = bdesc0 + (uint64_t)(s * (STAGE_BYTES >> 4));
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < BK / 32; ++k)        // 32 elements = 32 bytes along K inside the swizzle atom
              mma_f8(tmem_base + b * BN, adesc + (uint64_t)(k * 2), bdesc + (uint64_t)(k * 2), idesc, k != 0);
            gemm::mma_commit(done0 + 8 * s);         // the stage may be filled again, and P_kb is complete
            mbar_arrive(done0 + 8 * s);              // (the commit speaks for the tensor cores, this for the scales: see the producer)
          }
          __syncwarp();
          if (++s == STAGES) { s = 0; ph ^= 1u; }
        }
      }
    } else {
      // ---------------------------------------------------------------- helpers.  They serve every K block even after a wait ran out
      // (then without waiting for the tensor cores), so that no one is left at a named barrier.  Warp 3 may not arrive for a
      // block before the buffer's previous block has been read, or its arrival would count for that one.  A finished block
      // implies that; after an abort it waits for the buffer itself, which the promotion warps and warp 2 free without fail:
      // they only ever wait for warp 3.
      int s = 0;
      uint32_t it = 0, ph = 0;
      for (int tile = group; tile < ntiles; tile += ngroups) {
        for (int kb = 0; kb < kblocks; ++kb, ++it) {
          const uint32_t b = it & 1u;
          if (warp == 3) {
            if (wc.aborted() || !mbar_wait(done0 + 8 * s, ph, wc)) {
#pragma unroll 1
              for (int i = 0; i < (1 << 24) && !mbar_try_wait(tempty0 + 8 * b, ((it >> 1) & 1u) ^ 1u); ++i) {}
            }
            __syncwarp();
            if (++s == STAGES) { s = 0; ph ^= 1u; }
            full_arrive(b);
          } else {
            empty_sync(b);
            if (lane == 0) mbar_arrive(tempty0 + 8 * b);
          }
        }
      }
    }
  } else {
    // ------------------------------------------------------------------ promotion
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_HIGH));
    const int q = warp & 3, part = (warp - 4) >> 2;
    const uint32_t wbuf = smem_u32(out_stage) + (uint32_t)(warp - 4) * 8192u;
    uint32_t it = 0;
    for (int tile = group; tile < ntiles; tile += ngroups) {
      const int m0 = (tile % tiles_m) * BM + q * 32, n0 = (tile / tiles_m) * bn + part * COLS;
      const int n_end = min(p.N, n0 - part * COLS + bn);             // the tile's columns end here
      const bool live = m0 < p.M && n0 < n_end;      // this warp's part of the tile meets C (what it adds up otherwise is not stored)
      float2 acc[COLS / 2];
#pragma unroll
      for (int j = 0; j < COLS / 2; ++j) acc[j] = make_float2(0.f, 0.f);
#pragma unroll 1
      for (int kb = 0; kb < kblocks; ++kb, ++it) {
        const uint32_t b = it & 1u, taddr = tmem_base + ((uint32_t)(q * 32) << 16) + b * BN + part * COLS;
        const float* sc = sring + (it % SRING) * SCALES;
        full_sync(b);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (B_ROW_SCALES) {
          const float* sv = sc + BM + part * COLS + 2 * (lane & 3);
          const float* sr = sc + (p.a_shift ? 0 : q * 32 + (lane >> 2));
          const int r8 = p.a_shift ? 0 : 8;
          const float s0 = sr[0], s1 = sr[r8];
          read_and_promote<false>(taddr, acc, s0, s1, sv, b);
          read_and_promote<false>(taddr + 64, acc + 16, s0, s1, sv + 64, b);
          const float s2 = sr[2 * r8], s3 = sr[3 * r8];
          read_and_promote<false>(taddr + (16u << 16), acc + 32, s2, s3, sv, b);
          read_and_promote<true>(taddr + 64 + (16u << 16), acc + 48, s2, s3, sv + 64, b);
        } else {
          const float sa = sc[p.a_shift ? 0 : q * 32 + lane], sb = sc[BM + part];
          uint32_t r[64];
          read_rows(taddr, r);
          const float x = sa * sb;
          promote_rows(acc, r, x);
          read_rows(taddr + 64, r);
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          empty_arrive(b);                           // buffer read
          promote_rows(acc + 32, r, x);
        }
      }
      // pair j of the thread's sums: which row of the warp's 32 and which column of its 128 (a pair is two adjacent columns)
      auto pair_row = [&](int j) { return B_ROW_SCALES ? (j >> 5) * 16 + (j & 1) * 8 + (lane >> 2) : lane; };
      auto pair_col = [&](int j) { return B_ROW_SCALES ? ((j & 31) >> 1) * 8 + 2 * (lane & 3) : 2 * j; };
      if (p.split > 1) {
        // the tile's only owner of these K blocks: its sums go where the operands were (all of them have been used)
        float* part_sums = reinterpret_cast<float*>(smem) + (q * 32) * PART_PITCH + part * COLS;
#pragma unroll
        for (int j = 0; j < COLS / 2; ++j) *reinterpret_cast<float2*>(part_sums + pair_row(j) * PART_PITCH + pair_col(j)) = acc[j];
      } else if (live) {
        // Blocks of 32 rows x 128 bytes (32 fp32 or 64 bf16 columns), 16-byte pieces placed by the 128-byte swizzle, two of them in
        // the warp's 8 KB at a time: one wait for the stores before, one proxy fence.  (Rows of 64 bytes took the copy engine,
        // which the operand loads need too, twice as long.)
        const int ncol = p.c_bf16 ? 64 : 32;
#pragma unroll
        for (int g = 0; g < 2; ++g) {                // bf16: all four quarters of the columns at once; fp32: two and two
          if (g == 1 && p.c_bf16) break;
          if (p.n_tma && lane == 0) gemm::bulk_wait_read<0>();
          __syncwarp();
          if (p.c_bf16) {
#pragma unroll
            for (int j = 0; j < COLS / 2; j += B_ROW_SCALES ? 1 : 4) {
              const int row = pair_row(j), col = pair_col(j), unit = (col & 63) >> 3;
              const uint32_t at = wbuf + (uint32_t)((col >> 6) * 4096 + row * 128 + ((unit ^ (row & 7)) << 4));
              if (B_ROW_SCALES) st32(at + (col & 7) * 2, bf16x2(acc[j]));
              else st128(at, bf16x2(acc[j]), bf16x2(acc[j + 1]), bf16x2(acc[j + 2]), bf16x2(acc[j + 3]));
            }
          } else {
#pragma unroll
            for (int j = 0; j < COLS / 2; j += B_ROW_SCALES ? 1 : 2) {
              // (columns 64 g to 64 g + 63)
              if ((B_ROW_SCALES ? (j & 31) >> 4 : j >> 5) != g) continue;
              const int row = pair_row(j), col = pair_col(j), unit = (col & 31) >> 2;
              const uint32_t at = wbuf + (uint32_t)(((col >> 5) & 1) * 4096 + row * 128 + ((unit ^ (row & 7)) << 4));
              if (B_ROW_SCALES) st64(at + (col & 3) * 4, acc[j]);
              else st128(at, __float_as_uint(acc[j].x), __float_as_uint(acc[j].y), __float_as_uint(acc[j + 1].x), __float_as_uint(acc[j + 1].y));
            }
          }
          if (p.n_tma) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
              for (int c = 0; c < 2; ++c) {
                const int col = n0 + (2 * g + c) * ncol;
                if (col < n_end && col < p.n_tma) gemm::tma_store_2d(&map_c, wbuf + c * 4096u, col, m0);
              }
              gemm::bulk_commit();
            }
            // The copies write whole 16-byte pieces, beyond the map's last column too: where C's rows end inside a piece the map ends
            // before it, and a lane per row stores what is left (1796 x 50257 x 1024 to fp32 with rows of 50260: 155 us, 233 us by
            // the stores below).
            const int first = max(p.n_tma, n0 + 2 * g * ncol), last = min(n_end, n0 + 2 * (g + 1) * ncol);
            if (first < last && m0 + lane < p.M) {
              const unsigned char* blocks = out_stage + (warp - 4) * 8192;
              for (int col = first; col < last; ++col) store_staged(p, blocks, lane, col - n0 - 2 * g * ncol, (int64_t)(m0 + lane) * p.ldc + col);
            }
          } else {
            // a C that no tensor map describes (its rows do not start on 16-byte boundaries): the blocks' rows by plain stores of
            // adjacent elements
            __syncwarp();
            const unsigned char* blocks = out_stage + (warp - 4) * 8192;
            const int rows = min(32, p.M - m0);
            for (int r = 0; r < rows; ++r) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                if (i >= 2 && !p.c_bf16) break;
                const int in = i * 32 + lane, col = n0 + 2 * g * ncol + in;      // bf16: 128 columns, fp32: 64
                if (col >= n_end) continue;
                store_staged(p, blocks, r, in, (int64_t)(m0 + r) * p.ldc + col);
              }
            }
          }
        }
      }
    }
    if (lane == 0) gemm::bulk_wait_all<0>();         // the stores still read this CTA's memory
  }

  __syncwarp();
  if (p.split > 1) {
    // each CTA of the cluster adds up a part of the tile's rows
    cooperative_groups::cluster_group cl = cooperative_groups::this_cluster();
    cl.sync();
    const int m0 = (group % tiles_m) * BM, n0 = (group / tiles_m) * bn, n_end = min(p.N, n0 + bn);
    const int r_first = BM * rank / p.split, rows = BM * (rank + 1) / p.split - r_first;
    for (int i = tid; i < rows * (BN / 4); i += THREADS) {
      const int r = r_first + i / (BN / 4), c = (i % (BN / 4)) * 4, row = m0 + r, col = n0 + c;
      if (row >= p.M || col >= n_end) continue;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int o = 0; o < p.split; ++o) {
        const float4 w = *reinterpret_cast<const float4*>(cl.map_shared_rank(reinterpret_cast<float*>(smem), o) + r * PART_PITCH + c);
        v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
      }
      const float e[4] = {v.x, v.y, v.z, v.w};
      const int64_t at = (int64_t)row * p.ldc + col;
      if (p.c_bf16) {
        __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.C) + at;
        if (p.c_vec && col + 4 <= n_end) *reinterpret_cast<uint2*>(dst) = make_uint2(bf16x2(make_float2(v.x, v.y)), bf16x2(make_float2(v.z, v.w)));
        else for (int k = 0; k < 4; ++k) if (col + k < n_end) dst[k] = __float2bfloat16_rn(e[k]);
      } else {
        float* dst = reinterpret_cast<float*>(p.C) + at;
        if (p.c_vec && col + 4 <= n_end) *reinterpret_cast<float4*>(dst) = v;
        else for (int k = 0; k < 4; ++k) if (col + k < n_end) dst[k] = e[k];
      }
    }
    cl.sync();                          // nobody leaves while its sums are read
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  // after a wait ran out: time for loads and tensor-core work still under way
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
// Row-major matrix [rows, cols], boxes of 128 bytes (the swizzle span) x box_rows; out of range reads as 0.  (Stores clip columns at
// whole 16-byte pieces only: see n_tma.)
bool make_map(CUtensorMap* map, CUtensorMapDataType type, int es, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  EncodeFn enc = get_encode();
  if (!enc) return false;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld * es};
  cuuint32_t box[2] = {128u / es, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1u, 1u};
  return enc(map, type, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool B_ROW_SCALES>
cudaError_t launch(Params p, const void* A, int64_t lda, const void* B, int64_t ldb, int K, int sms, cudaStream_t st) {
  // Tile width (whole blocks of 128 columns) and split: the time of a K block of a tile hardly depends on the width (the hand-over's
  // latency), so a block is counted as 256 + width, a shared tile's exchange as two blocks (four in clusters of 3, 5, 6 or 7, which
  // take a microsecond or two longer: 30 x 1215 x 2500 12.4 us in sevens, 10.4 in eights), and the cheapest choice is taken.
  // Measured: 600 x 2048 x 151936 210 us in threes, 292 in pairs; 64 x 2048 x 151936 87 us in eights, 500 alone; 512 x 2048 x 8192 19
  // and 35 us; 4096 x 151936 x 2048 1.17 ms in tiles of 256, 1.79 ms in tiles of 128; where few tiles leave SMs idle the narrow
  // ones win by a tenth.
  const int64_t tm = (p.M + BM - 1) / BM;
  int64_t best = INT64_MAX;
  for (int w = BN; w >= 128; w -= 128) {
    const int64_t tiles = tm * ((p.N + w - 1) / w);
    if (tiles > INT32_MAX / 2) return cudaErrorInvalidValue;
    for (int S = 1; S <= MAX_SPLIT; ++S) {
      // (a cluster lies in one GPC, whose SMs are not a multiple of every size: of 148 SMs 112 can be counted on for clusters of 5 to
      // 8, nine in ten for 3, whose tiles would otherwise take a second round)
      const int64_t room = S > 4 ? sms * 3 / 4 : S == 3 ? sms * 9 / 10 : sms;
      if (S > 1 && (tiles * S > room || p.kblocks < 2 * S)) continue;
      const int64_t cost = ((tiles * S + sms - 1) / sms) * ((p.kblocks + S - 1) / S + (S == 1 ? 0 : (S & (S - 1)) ? 4 : 2)) * (256 + w);
      if (cost < best) { best = cost; p.bn = w; p.split = S; }
    }
  }
  CUtensorMap ma, mb, mc;
  if (!make_map(&ma, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, A, p.M, K, lda, BM)) return cudaErrorInvalidValue;
  if (!make_map(&mb, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, B, p.N, K, ldb, p.bn)) return cudaErrorInvalidValue;
  mc = ma;
  p.n_tma = p.c_vec ? p.N & ~(p.c_bf16 ? 7 : 3) : 0;
  if (p.n_tma && !make_map(&mc, p.c_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, p.c_bf16 ? 2 : 4, p.C, p.M, p.n_tma,
                           p.ldc, 32))
    p.n_tma = 0;
  auto kernel = gemm_tn_fp8_kernel<B_ROW_SCALES>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES);
  if (e != cudaSuccess) return e;
  const int64_t ctas = tm * ((p.N + p.bn - 1) / p.bn) * p.split;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(ctas < sms ? ctas : sms));           // a shared tile never has to wait for another: ctas <= sms then
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = SMEM_BYTES;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)p.split; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.split > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, ma, mb, mc, p);
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
  const int most = 1 << 30;                              // tile bounds are counted in int
  if (M < 0 || N < 0 || K < 0 || M > most || N > most || K > most) return DPPO_ERR_SHAPE;
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
  if ((uintptr_t)C % es || (uintptr_t)status % 4) return DPPO_ERR_ALIGN;
  if (K > 0 && (((uintptr_t)A % 16) || ((uintptr_t)B % 16) || (lda % 16) || (ldb % 16) || ((uintptr_t)a_scale % 4) || ((uintptr_t)b_scale % 4)))
    return DPPO_ERR_ALIGN;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(cuda_stream);
  if (K == 0)                                            // an empty sum
    return cudaMemset2DAsync(C, (size_t)ldc * es, 0, (size_t)N * es, (size_t)M, st) == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
  f8::Params p = {};
  p.M = M; p.N = N;
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
  const cudaError_t e = b_block_rows == 1 ? f8::launch<true>(p, A, lda, B, ldb, K, sms, st) : f8::launch<false>(p, A, lda, B, ldb, K, sms, st);
  return e == cudaSuccess ? DPPO_OK : DPPO_ERR_CUDA;
}
