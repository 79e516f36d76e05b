// The persistent tcgen05 pipeline of the linear-layer operators: D = A . B^T on tiles of 128*CG x BN, an epilogue of the
// operator's own on the accumulator while the next tile's products run.
//
// Same machine as the bf16 GEMM (TMA producer warp, MMA issuer warp, epilogue warps, two accumulator buffers in
// TMEM, mbarriers only, every wait bounded), cut down to what these operators need: a fixed stride through the slots
// of a tile order, optionally repeated for `splits` slices of the k axis, and an `Epi` type that is handed the accumulator.
// Eight epilogue warps, two on each quarter of the TMEM lanes: a warp moves its 32 rows x half of the columns to registers, hands
// the buffer back at once and only then computes (with four warps that worked on the buffer piece by piece the
// epilogue of the cross entropy took 11.5 thousand cycles a tile and bounded every D up to 1024).
// Operands are 8-bit integers (kind::i8, exact 32-bit integer sums) or 16-bit floats (kind::f16, fp32 sums); 16-bit operands may
// be stored with k or with their other axis contiguous.
//
// One stage holds 128 bytes of k per row (one swizzle row): 128 int8 or 64 16-bit elements.  CTA pairs (CG = 2) compute
// 256 rows per tile; each CTA supplies half of the B columns.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdio.h>

#include "internal.h"
#include "ptx.cuh"

namespace sp {

constexpr uint32_t kProdSmemLimit = 232448;  // 227 KiB opt-in maximum per CTA
constexpr uint32_t kProdBarrierBytes = 1024;

// status word: (role << 8) | which wait
enum : int { kProdProducer = 0x11, kProdMma = 0x12, kProdEpilogue = 0x13 };

enum : int { kElemI8 = 0, kElem16 = 1 };

template <int CG, int BN, int ELEM, uint32_t EPI_BYTES>
struct ProdCfg {
  static constexpr int kBK = ELEM == kElemI8 ? 128 : 64;        // elements of k per stage
  static constexpr int kBCols = BN / CG;                        // columns of B one CTA supplies
  static constexpr uint32_t kABytes = 128 * 128;
  static constexpr uint32_t kBBytes = kBCols * 128;
  static constexpr uint32_t kStageBytes = kABytes + kBBytes;
  static constexpr int kFit = (kProdSmemLimit - kProdBarrierBytes - 1024 - EPI_BYTES) / kStageBytes;
  static constexpr int kStages = kFit > 8 ? 8 : kFit;
  static constexpr uint32_t kSmemBytes = kStages * kStageBytes + EPI_BYTES + kProdBarrierBytes + 1024;  // + alignment slack
  static constexpr int kTmemCols = 2 * BN;                      // two accumulator buffers (a power of two)
  // Warps: producer, MMA issuer, two that idle, eight of the epilogue.  The register file is re-divided between groups of four
  // warps: 128 threads x 72 + 256 x 216 = 64512, what 384 threads x 168 were launched with.
  static constexpr int kEpiWarps = 8, kEpi0 = 4;
  static constexpr int kThreads = 32 * (kEpi0 + kEpiWarps);
  static constexpr int kRegsIssue = 72, kRegsEpilogue = 216;
};

struct ProdArgs {
  const int32_t* perm;   // tile table (orders that are not arithmetic), else nullptr
  const int32_t* live;   // Epi::kLive: on the device, rows of A that are there (an order in bands of tile rows, one slice)
  int32_t* status;
  int M, N;              // rows of A, rows of B
  int bn;                // columns of a tile: BN, or less where that fills the last wave better (a multiple of 32; B k-major)
  int kblocks;           // stages that cover k
  int splits;            // slices of k: slice z takes stages z, z + splits, z + 2 splits, ...: units that run together read k in step
  int kb_sum;            // stages whose products one accumulator takes before the epilogue adds it to its own sum (Epi::kSums; else a slice)
  int turn;              // 1: units start their walk along k at different places (one tile row: all read the same few lines of A, and
                         //    in step they would queue for them in one L2 slice: one token's scores, 131072 x 4096, 219 us in step, 191 so)
  // A product that reads nothing of the kernel before it may run beside it: it goes straight to work (everything before that kernel is
  // complete, see pdl_begin) and waits before it ends instead, so that whatever follows it follows both.
  int overlap;
  int units;             // CTAs or CTA pairs launched
  uint32_t idesc;        // instruction descriptor
  Sched sched;
};

// Shared-memory operand descriptor: start address, leading / stride byte offsets in 16-byte units, version 1, 128-byte swizzle.
__device__ __forceinline__ uint64_t prod_desc(uint32_t lbo_bytes, uint32_t sbo_bytes) {
  return ((uint64_t)((lbo_bytes >> 4) & 0x3FFFu) << 16) | ((uint64_t)((sbo_bytes >> 4) & 0x3FFFu) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint64_t prod_desc_at(uint64_t base, uint32_t addr) { return base + (uint64_t)((addr & 0x3FFFFu) >> 4); }

// Instruction descriptors.  kind::i8: D s32, A and B signed 8-bit.  kind::f16: D fp32, A and B both fp16 or both bf16,
// each k-major or (bit 15 / 16) contiguous along its other axis.
inline uint32_t idesc_i8(int m, int n) {
  return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
inline uint32_t idesc_16(int m, int n, bool bf16, bool a_mn, bool b_mn) {
  const uint32_t t = bf16 ? 1u : 0u;
  return (1u << 4) | (t << 7) | (t << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(m >> 4) << 24);
}

template <int CG, int ELEM>
__device__ __forceinline__ void prod_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (ELEM == kElem16) {
    umma_bf16<CG>(d, a, b, idesc, accumulate);   // kind::f16: fp16 or bf16 by the instruction descriptor
  } else if constexpr (CG == 1) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
  } else {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
  }
}

__device__ __forceinline__ void pdl_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Waits for the kernel before this one, and only then lets the one behind it start.  So whatever starts early, a product with `overlap` or an sp_gemm with
// SP_FLAG_OVERLAP, runs beside one kernel only, the one before it: everything before that is complete.
__device__ __forceinline__ void pdl_begin() {
  pdl_wait();
  pdl_launch_dependents();
}

__device__ __forceinline__ uint32_t pack_16(float lo, float hi, bool bf16) {
  if (bf16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// What an epilogue is given with the values of its part of a tile's accumulator (one row per lane).
struct EpiTile {
  int row0, col0;    // row of lane 0, first column of the part
  int part;          // number of the part among all columns: 2 x tile column + half
  int z;             // slice of k
};

// Staging of one epilogue warp: 32 rows x 128 bytes on their way to a bulk store.
struct EpiStage {
  uint32_t slice;
  int lane;
  __device__ __forceinline__ uint32_t free() const {   // whole warp: the last store has read the slice
    if (lane == 0) bulk_wait_read_0();
    __syncwarp();
    return slice;
  }
};

// 128 bytes of this lane's row into a slice, 128-byte swizzle (16-byte unit j of row r at j ^ (r % 8)): conflict-free,
// and what a bulk tensor store with that swizzle reads back.
__device__ __forceinline__ void stage_row(uint32_t slice, int lane, const uint32_t (&v)[32]) {
  const uint32_t row = slice + (uint32_t)lane * 128u, sw = (uint32_t)lane & 7u;
#pragma unroll
  for (uint32_t j = 0; j < 8; ++j) st_shared_16(row + ((j ^ sw) << 4), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
}

__device__ __forceinline__ uint32_t ld_shared_32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}

// A staged slice to a matrix whose rows a bulk store cannot take (row pitch or address not a multiple of 16 bytes, but whole elements).
// The slices of a part come from left to right.  Each row is cut where its own addresses are multiples of 16: a window takes its first
// bytes from the slice before (its last 16 bytes are carried over) and the rest from this one, so that all but a part's two edges is
// written 16 bytes at a time, four rows per instruction.  (One element per lane, a row per instruction: 2001 x 4999 fp32 results of a
// 2048-long product 50 us, this way 28.6; rows of 5000, by bulk stores, 23.5.)  `len`: bytes of this slice inside the matrix.
template <int ELT>
__device__ __forceinline__ void store_slice_plain(uint32_t carry, uint32_t slice, int lane, char* out, int64_t ld_bytes, int row0, int col, int M, int len,
                                                  bool first, bool last) {
  __syncwarp();
  auto scalar = [&](int row, int w) {      // a window that is not whole: element by element
    char* a = out + (int64_t)(row0 + row) * ld_bytes + (int64_t)col * ELT;
    const int p = 16 * w - (int)((uintptr_t)a & 15u), lo = first && p < 0 ? 0 : p, hi = min(p + 16, len);
#pragma unroll 1
    for (int q = lo; q < hi; q += ELT) {
      const uint32_t b = (uint32_t)q & 127u, addr = q < 0 ? carry + (uint32_t)row * 16u + (b & 12u)
                                                          : slice + (uint32_t)row * 128u + ((((b >> 4) ^ ((uint32_t)row & 7u)) << 4) | (b & 12u));
      const uint32_t v = ld_shared_32(addr);
      if constexpr (ELT == 4) *reinterpret_cast<uint32_t*>(a + q) = v;
      else *reinterpret_cast<uint16_t*>(a + q) = (uint16_t)(b & 2u ? v >> 16 : v);
    }
  };
  // Lane 8 i + w has window w of rows i, i + 4, ...: bytes 16 w - m on, m the row's address modulo 16, are the tail of unit w - 1 and the head of
  // unit w, put together by a shift of m bytes.  Two warps run per scheduler here, so the count of instructions is what costs.
  const int w = lane & 7, i0 = lane >> 3;
  char* a = out + (int64_t)(row0 + i0) * ld_bytes + (int64_t)col * ELT;
  const uint32_t ua = (uint32_t)i0 * 128u + (((uint32_t)w ^ (uint32_t)i0) << 4), ub = (uint32_t)i0 * 128u + (((uint32_t)(w - 1) ^ (uint32_t)i0) << 4);
  // straight-line code: the eight rounds' reads are in flight together
#pragma unroll
  for (int r = 0; r < 32; r += 4, a += 4 * ld_bytes) {
    const uint32_t m = (uint32_t)(uintptr_t)a & 15u;
    const int p = 16 * w - (int)m;
    uint32_t x[4], y[4], t[5], o[5];
    const uint32_t flip = r & 4 ? 64u : 0u;      // bit 2 of the row turns the unit by 4
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(w ? slice + (uint32_t)r * 128u + (ub ^ flip) : carry + (uint32_t)(r + i0) * 16u));
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(y[0]), "=r"(y[1]), "=r"(y[2]), "=r"(y[3]) : "r"(slice + (uint32_t)r * 128u + (ua ^ flip)));
    const bool m8 = m & 8u, m4 = m & 4u;      // x, y shifted by two words, by one word, by half a word
    t[0] = m8 ? x[1] : x[3]; t[1] = m8 ? x[2] : y[0]; t[2] = m8 ? x[3] : y[1]; t[3] = m8 ? y[0] : y[2]; t[4] = m8 ? y[1] : y[3];
    o[0] = m4 ? (m8 ? x[0] : x[2]) : t[0];
#pragma unroll
    for (int i = 1; i < 5; ++i) o[i] = m4 ? t[i - 1] : t[i];
    if constexpr (ELT == 2) {
      const uint32_t sel = m & 2u ? 0x5432u : 0x7654u;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = __byte_perm(o[i], o[i + 1], sel);
#pragma unroll
      for (int i = 4; i > 0; --i) o[i] = o[i - 1];
    }
    if (row0 + r + i0 < M && p + 16 <= len && !(first && p < 0)) *reinterpret_cast<uint4*>(a + p) = make_uint4(o[1], o[2], o[3], o[4]);
  }
  if ((first || last) && row0 + lane < M) {      // a row's two edges in this tile
    const int m = (int)((uintptr_t)(out + (int64_t)(row0 + lane) * ld_bytes + (int64_t)col * ELT) & 15u), end = (len + m) >> 4;
    if (first && m) scalar(lane, 0);
    if (last && ((len + m) & 15) && !(first && m && end == 0)) scalar(lane, end);
  }
  __syncwarp();
  if (!last) {      // unit 7 of each row goes on to the next slice
    uint32_t x[4];
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                 : "r"(slice + (uint32_t)lane * 128u + ((7u ^ ((uint32_t)lane & 7u)) << 4)));
    st_shared_16(carry + (uint32_t)lane * 16u, x[0], x[1], x[2], x[3]);
    __syncwarp();
  }
}

template <int CG, int BN, int ELEM, bool A_MN, bool B_MN, class Epi>
__global__ void __launch_bounds__(384, 1)
product_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmC,
               const ProdArgs args, const typename Epi::Args eargs) {
  using C = ProdCfg<CG, BN, ELEM, Epi::kBytes>;
  constexpr int S = C::kStages;
  static_assert(ELEM == kElem16 || (!A_MN && !B_MN), "8-bit operands are k-major");

  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t epi_base = smem_base + S * C::kStageBytes;      // 1024-byte aligned
  const uint32_t bar_base = epi_base + Epi::kBytes;
  const uint32_t bar_full = bar_base, bar_empty = bar_base + 8 * S, bar_tfull = bar_base + 16 * S, bar_tempty = bar_tfull + 16;
  const uint32_t tmem_slot = bar_tempty + 16;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 1 ? 0u : cluster_ctarank();
  const int unit = blockIdx.x / CG;
  const int T = args.sched.T, Tn = args.sched.Tn;

  if (threadIdx.x == 32) { prefetch_tensormap(&tmA); prefetch_tensormap(&tmB); }
  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(bar_tfull + 8 * i, 1); mbar_init(bar_tempty + 8 * i, C::kEpiWarps * CG); }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    tmem_alloc<CG>(tmem_slot, C::kTmemCols);
    tmem_relinquish<CG>();
  }
  tcgen05_fence_before();
  unit_sync<CG>();
  tcgen05_fence_after();
  const uint32_t tmem_base = ld_shared_32(tmem_slot);
  if (!args.overlap) pdl_begin();   // set-up may overlap the kernel before this one; global memory is touched only from here on

  auto tile_at = [&](int s, int& tm, int& tn, int& z) {
    z = s / T;
    const int o = s - z * T;
    const int t = args.sched.use_table ? __ldg(args.perm + o) : slot_to_tile(args.sched, o);
    tm = t / Tn; tn = t - tm * Tn;
  };
  // Rows that are known on the device only: tiles beyond them are passed over, and bands beyond them, whose slots are the last, not walked at all.
  int live = 0, total = T * args.splits;
  if constexpr (Epi::kLive) {
    live = *args.live;
    const int64_t band = 128 * CG * args.sched.group;
    total = (int)min((int64_t)T, (live + band - 1) / band * args.sched.group * Tn);
  }
  auto passed_over = [&](int tm) { return Epi::kLive && tm * 128 * CG >= live; };
  auto stages_of = [&](int z) { return (args.kblocks - z + args.splits - 1) / args.splits; };

  if (warp < C::kEpi0) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRegsIssue));
  if (warp == 0) {
    // ---------------------------------------------------------------- TMA producer
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int s = unit; s < total && ok; s += args.units) {
      int tm, tn, z;
      tile_at(s, tm, tn, z);
      if (passed_over(tm)) continue;
      const int n = stages_of(z);
      const int row0 = tm * 128 * CG + (int)rank * 128, col0 = tn * args.bn + (int)rank * (args.bn / CG);
      int at = args.turn ? (unit * 5) % n : 0;      // the stage to load, of this slice's
      for (int kb = 0; kb < n; ++kb) {
        ok = mbar_wait(bar_empty + 8 * stage, phase ^ 1u, args.status, (kProdProducer << 8) | 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const uint32_t full_local = bar_full + 8 * stage;
        const uint32_t full_leader = CG == 1 ? full_local : mapa(full_local, 0);
        const uint32_t sa = smem_base + stage * C::kStageBytes, sb = sa + C::kABytes;
        const int k = (z + at * args.splits) * C::kBK;
        if (++at == n) at = 0;
        if (elect_one()) {
          if (rank == 0) mbar_arrive_expect_tx(full_local, CG * C::kABytes + (uint32_t)args.bn * 128u);
          if constexpr (A_MN) {
#pragma unroll
            for (int j = 0; j < 2; ++j) tma_load_2d<CG>(sa + j * 8192, &tmA, row0 + j * 64, k, full_leader);   // boxes of 64 k x 64 rows
          } else {
            tma_load_2d<CG>(sa, &tmA, k, row0, full_leader);
          }
          if constexpr (B_MN) {
#pragma unroll
            for (int j = 0; j < C::kBCols / 64; ++j) tma_load_2d<CG>(sb + j * 8192, &tmB, col0 + j * 64, k, full_leader);
          } else {
            tma_load_2d<CG>(sb, &tmB, k, col0, full_leader);
          }
        }
        __syncwarp();
        if (++stage == S) { stage = 0; phase ^= 1u; }
      }
    }
    // every stage handed out must have been released before this CTA may exit: no commit arrival (or, after a failure,
    // no copy) is still in flight towards its shared memory
    for (int i = 0; i < S && ok; ++i) {
      ok = mbar_wait(bar_empty + 8 * stage, phase ^ 1u, args.status, (kProdProducer << 8) | 2);
      ok = __all_sync(0xffffffffu, ok);
      if (++stage == S) { stage = 0; phase ^= 1u; }
    }
    if (!ok) {
      const unsigned long long t0 = globaltimer();
      while (globaltimer() - t0 < 1000000ull) __nanosleep(1000);   // let copies in flight land
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer (leader CTA only)
    if (rank == 0) {
      // k-major: rows of 128 bytes, groups of 8 rows 1024 bytes apart, k advances 32 bytes inside the swizzle row.
      // Other axis contiguous: a box is 64 k-rows of 128 bytes; groups of 8 k-rows 1024 bytes apart (stride offset), the
      // next 64 rows of the operand in the next box, 8192 bytes on (leading offset); 16 k are 2048 bytes.
      const uint64_t da0 = A_MN ? prod_desc(8192, 1024) : prod_desc(16, 1024);
      const uint64_t db0 = B_MN ? prod_desc(8192, 1024) : prod_desc(16, 1024);
      constexpr uint32_t ka = A_MN ? 2048 : 32, kb_ = B_MN ? 2048 : 32;
      int stage = 0;
      uint32_t phase = 0;
      int it = 0;
      bool ok = true;
      for (int s = unit; s < total && ok; s += args.units) {
        int tm, tn, z;
        tile_at(s, tm, tn, z);
        if (passed_over(tm)) continue;
        const int n = stages_of(z);
        for (int ks = 0; ks < n && ok; ks += args.kb_sum, ++it) {
          const int ke = min(n, ks + args.kb_sum), buf = it & 1;
          ok = mbar_wait(bar_tempty + 8 * buf, ((uint32_t)(it >> 1) & 1u) ^ 1u, args.status, (kProdMma << 8) | 1);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tcgen05_fence_after();
          const uint32_t d = tmem_base + (uint32_t)(buf * BN);
          for (int kb = ks; kb < ke; ++kb) {
            ok = mbar_wait(bar_full + 8 * stage, phase, args.status, (kProdMma << 8) | 2);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tcgen05_fence_after();
            if (elect_one()) {
              const uint32_t sa = smem_base + stage * C::kStageBytes, sb = sa + C::kABytes;
#pragma unroll
              for (int k = 0; k < 4; ++k)
                prod_mma<CG, ELEM>(d, prod_desc_at(da0, sa + k * ka), prod_desc_at(db0, sb + k * kb_), args.idesc, (uint32_t)(kb > ks || k != 0));
              umma_commit<CG>(bar_empty + 8 * stage);
              if (kb == ke - 1) umma_commit<CG>(bar_tfull + 8 * buf);
            }
            __syncwarp();
            if (++stage == S) { stage = 0; phase ^= 1u; }
          }
        }
      }
    }
    __syncwarp();
  }
  } else {
    // ---------------------------------------------------------------- epilogue
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kRegsEpilogue));
    constexpr int kCols = BN / 2;   // columns of one warp
    const int quarter = warp & 3, half = (warp - C::kEpi0) >> 2;   // TMEM lanes [32 * quarter, 32 * quarter + 32)
    const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * kCols);
    Epi epi(eargs, &tmC, epi_base, warp - C::kEpi0, lane);
    int it = 0;
    bool ok = true;
    for (int s = unit; s < total && ok; s += args.units) {
      EpiTile e;
      int tm, tn;
      tile_at(s, tm, tn, e.z);
      if (passed_over(tm)) continue;
      const int n = stages_of(e.z);
      e.row0 = tm * 128 * CG + (int)rank * 128 + quarter * 32;
      e.col0 = tn * args.bn + half * kCols;
      e.part = 2 * tn + half;
      const int edge = min(args.N, (tn + 1) * args.bn);   // what the accumulator holds beyond the tile's own columns is not used
      epi.before(e, args.M, edge);
      uint32_t v[kCols];
      const auto full = [&]() {      // the next accumulator is complete
        ok = mbar_wait(bar_tfull + 8 * (it & 1), (uint32_t)(it >> 1) & 1u, args.status, (kProdEpilogue << 8) | 1);
        ok = __all_sync(0xffffffffu, ok);
        tcgen05_fence_after();
      };
      const auto hand_back = [&]() {
        tcgen05_fence_before();
        __syncwarp();
        // Relaxed: the values are in registers, nothing was written that the issuer reads.  With release the arrival would wait for the
        // stores of the tile before to reach memory.
        if (lane == 0) {
          if constexpr (CG == 1) mbar_arrive_relaxed(bar_tempty + 8 * (it & 1));
          else mbar_arrive_relaxed_cluster(mapa(bar_tempty + 8 * (it & 1), 0));
        }
        ++it;
      };
      full();
      if (!ok) break;
#pragma unroll
      for (int q = 0; q < kCols / 32; ++q) tmem_ld_32x32b_x32(taddr + (uint32_t)((it & 1) * BN + q * 32), *reinterpret_cast<uint32_t(*)[32]>(v + q * 32));
      tmem_ld_wait();
      hand_back();
      if constexpr (Epi::kSums) {
        for (int ks = args.kb_sum; ks < n; ks += args.kb_sum) {
          full();
          if (!ok) break;
#pragma unroll
          for (int q = 0; q < kCols / 16; ++q) {      // 16 columns at a time: v and 32 more do not fit the registers
            uint32_t w[16];
            tmem_ld_32x32b_x16(taddr + (uint32_t)((it & 1) * BN + q * 16), w);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) v[q * 16 + j] = __float_as_uint(__uint_as_float(v[q * 16 + j]) + __uint_as_float(w[j]));
          }
          hand_back();
        }
      }
      if (!ok) break;
      epi.template finish<kCols>(v, e, args.M, edge);
    }
    if (lane == 0) bulk_wait_all();   // every store of this warp has reached global memory
    __syncwarp();
  }

  tcgen05_fence_before();
  unit_sync<CG>();
  if (warp == 1) tmem_dealloc<CG>(tmem_base, C::kTmemCols);
  if (args.overlap && threadIdx.x == 0) pdl_begin();
}

// Columns of a tile of 128 * CG rows for M x N results: the width, from 256 down in steps of `step`, with the least waves x (width + 48) (the
// tensor cores' time goes with the width, the operands' way through L2 with 256 + width), while 256 would make up to three waves.  8-bit
// 1000 x 3000 x 4000: 13.4 us at 192 columns, 16.2 at 256; 2001 x 4999 x 2048: 25.8 and 28.6.  Beyond three waves the power limit decides, not
// the last wave (4096^3: 54.7 and 52.6), and with one tile row the reading of B does (16 tokens x 65536 x 4096: 101 and 97).
inline int tile_width(int64_t M, int64_t N, int cg, int step) {
  const int64_t units = 148 / cg, rows = (M + 128 * cg - 1) / (128 * cg);
  int best = 256;
  int64_t least = 0;
  if (rows == 1 || rows * ((N + 255) / 256) > 3 * units) return best;
  for (int w = 256; w >= 160; w -= step) {
    const int64_t cost = (rows * ((N + w - 1) / w) + units - 1) / units * (w + 48);
    if (least == 0 || cost < least) { least = cost; best = w; }
  }
  return best;
}

// Launch with programmatic stream serialisation: the next kernel's set-up overlaps this one's tail.
template <class... KArgs, class... Args>
inline int launch_pdl(const char* what, void (*kern)(KArgs...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  if (log_enabled()) fprintf(stderr, "[swizzleperf] %s: grid=%u threads=%d cluster=%d smem=%zu\n", what, grid.x, threads, cluster, smem);
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...);
  if (e != cudaSuccess) { set_error("launching %s failed: %s", what, cudaGetErrorString(e)); return SP_ERR_CUDA; }
  return SP_OK;
}

// Fills args.idesc, args.units and launches one product.  The caller has set M, N, bn, kblocks, splits (at most kblocks), sched, perm, status.
template <int CG, int BN, int ELEM, bool A_MN, bool B_MN, class Epi>
int launch_product(const char* what, const CUtensorMap& tmA, const CUtensorMap& tmB, const CUtensorMap& tmC, ProdArgs args, bool bf16,
                   const typename Epi::Args& eargs, cudaStream_t stream) {
  using C = ProdCfg<CG, BN, ELEM, Epi::kBytes>;
  auto kern = product_kernel<CG, BN, ELEM, A_MN, B_MN, Epi>;
  static uint64_t configured = 0;   // per instantiation, one bit per device
  if (first_use_on_this_device(configured)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kSmemBytes);
    if (e != cudaSuccess) { configured = 0; set_error("cudaFuncSetAttribute(smem=%u) failed: %s", C::kSmemBytes, cudaGetErrorString(e)); return SP_ERR_CUDA; }
  }
  const int64_t work = (int64_t)args.sched.T * args.splits;
  if (work > 0x3fffffff) { set_error("%s: too many tiles", what); return SP_ERR_UNSUPPORTED; }
  args.units = gemm_units(128 * CG, BN, work);   // one CTA per SM, or as many CTA pairs as fit: same as sp_gemm's tiles of this shape
  if (args.units <= 0) { set_error("could not size the grid"); return SP_ERR_CUDA; }
  if (!Epi::kSums) args.kb_sum = args.kblocks;
  args.idesc = ELEM == kElemI8 ? idesc_i8(128 * CG, args.bn) : idesc_16(128 * CG, args.bn, bf16, A_MN, B_MN);
  return launch_pdl(what, kern, dim3((unsigned)(args.units * CG)), C::kThreads, C::kSmemBytes, CG, stream, tmA, tmB, tmC, args, eargs);
}

}  // namespace sp
