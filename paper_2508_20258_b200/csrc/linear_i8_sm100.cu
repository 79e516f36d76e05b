// The linear layer in 8-bit integers: rows quantised with one scale each, the product of two 8-bit matrices in exact
// 32-bit integer sums on the tensor cores, scaled per row (token) and per column (output channel) on the way out.
#include <new>
#include <mutex>
#include <vector>

#include "product.cuh"

namespace sp {

// ------------------------------------------------------------------ quantiser
// scale = max|x| / 127 (rounded once to fp32), q = the integer nearest to x / scale, halves to even.
//
// A quotient taken in fp32 can land on the wrong side of a half.  So the cheap product with 1 / scale decides only where
// it is clear (its error is below 2^-16 for |q| <= 127); within 2^-12 of a half the remainder x - q * scale decides.  That
// remainder is exact in fp32: near a half, x and q * scale are multiples of ulp(scale) / 2 and differ by about scale / 2.
//
// Bound: one read of x, one write of q; each thread keeps its vectors of the row in registers between the two passes.
constexpr int kQuantThreads = 256;
constexpr int kQuantVecs = 4;        // vectors of 8 elements a thread holds

template <class T> __device__ __forceinline__ float quant_to_float(T v);
template <> __device__ __forceinline__ float quant_to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float quant_to_float(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float quant_to_float(float v) { return v; }

// Elements [c, c + 8) of a row; columns at or beyond `cols` read as zero.  `vec`: rows start on 16-byte boundaries.
template <class T>
__device__ __forceinline__ void quant_load(const T* row, int64_t c, int64_t cols, bool vec, float (&v)[8]) {
  if (vec && c + 8 <= cols) {
    constexpr int kWords = (int)sizeof(T) * 8 / 16;
    __align__(16) T e[8];
#pragma unroll
    for (int i = 0; i < kWords; ++i) reinterpret_cast<uint4*>(e)[i] = __ldg(reinterpret_cast<const uint4*>(row + c) + i);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = quant_to_float(e[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? quant_to_float(row[c + i]) : 0.f;
  }
}

__device__ __forceinline__ int quant_one(float x, float s, float inv, bool divide) {
  const float y = divide ? __fdiv_rn(x, s) : x * inv;
  float q = rintf(y);
  const float f = fabsf(y - q);
  if (f > 0.5f - 0x1p-12f) {
    const float r = fmaf(-q, s, x), two = 2.f * fabsf(r);
    if (two > s || (two == s && (((int)q) & 1))) q += r > 0.f ? 1.f : -1.f;
  }
  return (int)fminf(fmaxf(q, -127.f), 127.f);
}

// TPR threads share a row (32: eight rows per block; 256: one).
template <class T, int TPR>
__global__ void __launch_bounds__(kQuantThreads) quantize_kernel(const T* x, int rows, int64_t cols, int64_t kp, int8_t* q, float* scale) {
  pdl_wait();
  // Only now may the next kernel start: one that reads nothing of this kernel before its own wait then finds everything
  // before this kernel complete (the few-token product fetches weights that early).
  pdl_launch_dependents();
  constexpr int kRows = kQuantThreads / TPR;
  const int t = threadIdx.x % TPR;
  const int row = blockIdx.x * kRows + threadIdx.x / TPR;
  const bool live = row < rows;
  const T* xr = x + (int64_t)(live ? row : 0) * cols;
  const bool vec = (((uintptr_t)x | (uintptr_t)(cols * (int64_t)sizeof(T))) & 15u) == 0;
  const int64_t nvec = kp / 8;
  float v[kQuantVecs][8];
  uint32_t top = 0;      // |x| as bits: orders like the values, infinities and NaN above all
#pragma unroll
  for (int i = 0; i < kQuantVecs; ++i) {
    const int64_t j = t + (int64_t)i * TPR;
    if (j < nvec) {
      quant_load(xr, j * 8, cols, vec, v[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[i][e]) & 0x7fffffffu);
    }
  }
  for (int64_t j = t + (int64_t)kQuantVecs * TPR; j < nvec; j += TPR) {   // long rows: read again below
    float w[8];
    quant_load(xr, j * 8, cols, vec, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(w[e]) & 0x7fffffffu);
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if constexpr (TPR > 32) {
    __shared__ uint32_t part[kQuantThreads / 32];
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kQuantThreads / 32; ++i) top = max(top, part[i]);
  }
  if (!live) return;
  const bool bad = top >= 0x7f800000u;
  const float s = bad ? __uint_as_float(0x7fffffffu) : __fdiv_rn(__uint_as_float(top), 127.f);
  if (t == 0) scale[row] = s;
  const bool zero = bad || s == 0.f;
  const bool divide = !(s > 0x1p-100f && s < 0x1p100f);   // 1 / scale must be a normal number
  const float inv = divide ? 0.f : 1.f / s;
  int8_t* qr = q + (int64_t)row * kp;
  auto store = [&](int64_t j, const float (&w)[8]) {
    uint32_t lo = 0, hi = 0;
    if (!zero) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        lo |= (uint32_t)(quant_one(w[e], s, inv, divide) & 0xff) << (8 * e);
        hi |= (uint32_t)(quant_one(w[e + 4], s, inv, divide) & 0xff) << (8 * e);
      }
    }
    *reinterpret_cast<uint2*>(qr + j * 8) = make_uint2(lo, hi);
  };
#pragma unroll
  for (int i = 0; i < kQuantVecs; ++i) {
    const int64_t j = t + (int64_t)i * TPR;
    if (j < nvec) store(j, v[i]);
  }
  for (int64_t j = t + (int64_t)kQuantVecs * TPR; j < nvec; j += TPR) {
    float w[8];
    quant_load(xr, j * 8, cols, vec, w);
    store(j, w);
  }
}

// ------------------------------------------------------------------ epilogue of the tiled product
// c = (float(acc) * a_scale[row]) * b_scale[col]: the integer rounds once to fp32, then one rounding per factor (the two
// scales are not multiplied first: their product can leave fp32's range where the result does not).
template <bool OUT_F32>
struct EpiI8 {
  static constexpr uint32_t kBytes = 4 * 2 * 4096 + 4 * 256;   // staging, then 64 column scales per warp
  struct Args {
    const float* a_scale;
    const float* b_scale;
    char* C;
    int64_t ld_bytes;
    int bf16;     // 16-bit output: bf16, else fp16
    int plain;    // rows of C that a bulk store cannot take
  };
  const Args& a;
  const CUtensorMap* map;
  EpiStage stage;
  uint32_t scales;
  int lane;
  float rs;
  float bs[8];
  __device__ EpiI8(const Args& args, const CUtensorMap* m, uint32_t base, int w, int l)
      : a(args), map(m), stage{base + (uint32_t)w * 8192u, 0}, scales(base + 32768u + (uint32_t)w * 256u), lane(l) {}
  __device__ __forceinline__ void before(const EpiTile& e, int M, int N) {
    rs = e.row0 + lane < M ? __ldg(a.a_scale + e.row0 + lane) : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int c = e.col0 + i * 32 + lane;
      bs[i] = c < N ? __ldg(a.b_scale + c) : 0.f;   // beyond the tile's own columns: loaded, never used
    }
  }
  template <int BN>
  __device__ __forceinline__ void tile(const EpiTile& e, int M, int N) {
    constexpr int kCols = OUT_F32 ? 32 : 64;
#pragma unroll
    for (int q = 0; q < BN / kCols; ++q) {
      uint32_t v[32], w[32];
      tmem_ld_32x32b_x32(e.taddr + (uint32_t)(q * kCols), v);
      if constexpr (!OUT_F32) tmem_ld_32x32b_x32(e.taddr + (uint32_t)(q * kCols + 32), w);
      const float b0 = bs[OUT_F32 ? q : 2 * q], b1 = OUT_F32 ? 0.f : bs[2 * q + (OUT_F32 ? 0 : 1)];
      asm volatile("st.shared.f32 [%0], %1;" ::"r"(scales + lane * 4), "f"(b0) : "memory");
      if constexpr (!OUT_F32) asm volatile("st.shared.f32 [%0], %1;" ::"r"(scales + 128 + lane * 4), "f"(b1) : "memory");
      __syncwarp();
      tmem_ld_wait();
      auto scaled = [&](uint32_t (&r)[32], uint32_t at) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float4 f;
          asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w) : "r"(at + j * 16) : "memory");
          r[4 * j] = __float_as_uint((float)(int)r[4 * j] * rs * f.x);
          r[4 * j + 1] = __float_as_uint((float)(int)r[4 * j + 1] * rs * f.y);
          r[4 * j + 2] = __float_as_uint((float)(int)r[4 * j + 2] * rs * f.z);
          r[4 * j + 3] = __float_as_uint((float)(int)r[4 * j + 3] * rs * f.w);
        }
      };
      scaled(v, scales);
      if constexpr (!OUT_F32) {
        scaled(w, scales + 128);
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = pack_16(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]), a.bf16);
#pragma unroll
        for (int j = 0; j < 16; ++j) v[16 + j] = pack_16(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]), a.bf16);
      }
      const uint32_t slice = stage.next(lane);
      stage_row(slice, lane, v);
      const int col = e.col0 + q * kCols;
      const bool inside = e.row0 < M && col < N;
      if (a.plain) {
        if (inside) store_slice_plain<OUT_F32 ? 4 : 2>(slice, lane, a.C, a.ld_bytes, e.row0, col, M, N);
        else __syncwarp();
      } else {
        fence_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (inside) tma_store_2d(map, slice, col, e.row0);
          bulk_commit();   // also when nothing was stored: keeps the group count in step
        }
      }
    }
  }
};

// ------------------------------------------------------------------ few tokens
// At most NT rows of A: the call is bound by reading the weights once, so the weights take the 128-row side of the MMA and the
// tokens its N side, and the k axis of each 128-row block is split over the S CTAs of a cluster to occupy every SM.  The
// partial sums are integers: they meet through distributed shared memory, in any order with one result.
template <int NT>
struct FewCfg {
  static constexpr uint32_t kWBytes = 128 * 128, kQBytes = NT * 128, kStageBytes = kWBytes + kQBytes;
  static constexpr int kFit = (114688 - 1024 - 512) / kStageBytes;    // two CTAs per SM
  static constexpr int kStages = kFit > 6 ? 6 : kFit;
  static constexpr uint32_t kSmemBytes = kStages * kStageBytes + 512 + 1024;
  static constexpr int kTmemCols = NT < 32 ? 32 : NT;
  static_assert(kStages * kStageBytes >= NT * 128 * 4, "the partial sums reuse the stages");
};

struct FewArgs {
  const float* a_scale;
  const float* b_scale;
  char* C;
  int32_t* status;
  int M, N;
  int kblocks, kb_split;
  int out;          // SP_BF16, SP_FP32, SP_FP16
  int early;        // 1: the kernel before this one writes no weights, and everything before that one is complete
  uint32_t idesc;
};

__device__ __forceinline__ void few_store(const FewArgs& a, int tok, int n, int acc) {
  const float y = (float)acc * __ldg(a.a_scale + tok) * __ldg(a.b_scale + n);
  const int64_t at = (int64_t)tok * a.N + n;
  if (a.out == SP_FP32) reinterpret_cast<float*>(a.C)[at] = y;
  else if (a.out == SP_BF16) reinterpret_cast<__nv_bfloat16*>(a.C)[at] = __float2bfloat16_rn(y);
  else reinterpret_cast<__half*>(a.C)[at] = __float2half_rn(y);
}

template <int NT>
__global__ void __launch_bounds__(192, 2)
few_tokens_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmQ, const FewArgs args) {
  using C = FewCfg<NT>;
  constexpr int S = C::kStages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t bar_full = smem_base + S * C::kStageBytes, bar_empty = bar_full + 8 * S, bar_done = bar_empty + 8 * S;
  const uint32_t tmem_slot = bar_done + 8;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank(), nranks = cluster_nctarank();
  const int n0 = (int)(blockIdx.x / nranks) * 128;
  const int k0 = (int)rank * args.kb_split, k1 = min(args.kblocks, k0 + args.kb_split);

  pdl_launch_dependents();
  if (threadIdx.x == 32) { prefetch_tensormap(&tmW); prefetch_tensormap(&tmQ); }
  if (threadIdx.x == 0) {
    for (int i = 0; i < S; ++i) { mbar_init(bar_full + 8 * i, 1); mbar_init(bar_empty + 8 * i, 1); }
    mbar_init(bar_done, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    tmem_alloc<1>(tmem_slot, C::kTmemCols);
    tmem_relinquish<1>();
  }
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  const uint32_t tmem = ld_shared_32(tmem_slot);

  if (warp == 0) {
    bool ok = true;
    auto stage_addr = [&](int i) { return smem_base + (uint32_t)(i % S) * C::kStageBytes; };
    const int ahead = min(S, k1 - k0);
    if (!args.early) pdl_wait();
    if (elect_one()) {
      for (int i = 0; i < ahead; ++i) {
        mbar_arrive_expect_tx(bar_full + 8 * i, C::kStageBytes);
        tma_load_2d<1>(stage_addr(i), &tmW, (k0 + i) * 128, n0, bar_full + 8 * i);
      }
    }
    __syncwarp();
    if (args.early) pdl_wait();
    if (elect_one()) {
      for (int i = 0; i < ahead; ++i) tma_load_2d<1>(stage_addr(i) + C::kWBytes, &tmQ, (k0 + i) * 128, 0, bar_full + 8 * i);
    }
    __syncwarp();
    for (int i = S; i < k1 - k0; ++i) {
      const int st = i % S;
      ok = mbar_wait(bar_empty + 8 * st, (uint32_t)(i / S - 1) & 1u, args.status, (kProdProducer << 8) | 3);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      if (elect_one()) {
        mbar_arrive_expect_tx(bar_full + 8 * st, C::kStageBytes);
        tma_load_2d<1>(stage_addr(i), &tmW, (k0 + i) * 128, n0, bar_full + 8 * st);
        tma_load_2d<1>(stage_addr(i) + C::kWBytes, &tmQ, (k0 + i) * 128, 0, bar_full + 8 * st);
      }
      __syncwarp();
    }
    // every stage in use must have been released: no commit arrival is in flight towards this CTA when it exits
    for (int i = max(0, k1 - k0 - S); i < k1 - k0 && ok; ++i) {
      ok = mbar_wait(bar_empty + 8 * (i % S), (uint32_t)(i / S) & 1u, args.status, (kProdProducer << 8) | 4);
      ok = __all_sync(0xffffffffu, ok);
    }
    if (!ok) {
      const unsigned long long t0 = globaltimer();
      while (globaltimer() - t0 < 1000000ull) __nanosleep(1000);   // let copies in flight land
    }
    __syncwarp();
  } else if (warp == 1) {
    pdl_wait();
    bool ok = true;
    for (int i = 0; i < k1 - k0; ++i) {
      const int st = i % S;
      ok = mbar_wait(bar_full + 8 * st, (uint32_t)(i / S) & 1u, args.status, (kProdMma << 8) | 3);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tcgen05_fence_after();
      if (elect_one()) {
        const uint64_t d0 = prod_desc(16, 1024);
        const uint32_t sw = smem_base + (uint32_t)st * C::kStageBytes, sq = sw + C::kWBytes;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          prod_mma<1, kElemI8>(tmem, prod_desc_at(d0, sw + k * 32), prod_desc_at(d0, sq + k * 32), args.idesc, (uint32_t)(i > 0 || k != 0));
        umma_commit<1>(bar_empty + 8 * st);
        if (i == k1 - k0 - 1) umma_commit<1>(bar_done);
      }
      __syncwarp();
    }
  } else {
    pdl_wait();
    const int quarter = warp & 3, row = quarter * 32 + lane, n = n0 + row;
    bool ok = mbar_wait(bar_done, 0, args.status, (kProdEpilogue << 8) | 3);
    ok = __all_sync(0xffffffffu, ok);
    tcgen05_fence_after();
    if (ok) {
#pragma unroll
      for (int q = 0; q < (NT + 31) / 32; ++q) {
        uint32_t v[32];
        tmem_ld_32x32b_x32(tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(q * 32), v);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < (NT < 32 ? NT : 32); ++j) {
          const int tok = q * 32 + j;
          if (tok >= args.M) break;
          if (nranks == 1) {
            if (n < args.N) few_store(args, tok, n, (int)v[j]);
          } else {
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(smem_base + (uint32_t)(tok * 128 + row) * 4u), "r"(v[j]) : "memory");
          }
        }
      }
    }
  }
  tcgen05_fence_before();
  if (nranks > 1) {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (warp >= 2) {
      const int row = (int)threadIdx.x - 64, n = n0 + row;
      for (int tok = (int)rank; tok < args.M; tok += (int)nranks) {
        int acc = 0;
        for (uint32_t r = 0; r < nranks; ++r) {
          int p;
          asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(p) : "r"(mapa(smem_base + (uint32_t)(tok * 128 + row) * 4u, r)) : "memory");
          acc += p;
        }
        if (n < args.N) few_store(args, tok, n, acc);
      }
    }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");   // nobody leaves while a peer may read its partial sums
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  } else {
    __syncthreads();
  }
  if (warp == 1) {
    tcgen05_fence_after();
    tmem_dealloc<1>(tmem, C::kTmemCols);
  }
}

// ------------------------------------------------------------------ host side
static std::mutex g_i8_mu;   // per-kernel set-up below is done under it

static size_t elt_bytes(int dtype) { return dtype == SP_FP32 ? 4 : 2; }

template <class T>
static int launch_quantize(const void* x, int64_t M, int64_t K, int8_t* q, float* scale, cudaStream_t stream) {
  const int64_t kp = (K + 15) / 16 * 16;
  // a warp per row while the row fits its registers (8 rows per block), else a block per row
  if (kp <= 32 * kQuantVecs * 8)
    return launch_pdl("quantize", quantize_kernel<T, 32>, dim3((unsigned)((M + 7) / 8)), kQuantThreads, 0, 1, stream, (const T*)x, (int)M, K, kp, q, scale);
  return launch_pdl("quantize", quantize_kernel<T, kQuantThreads>, dim3((unsigned)M), kQuantThreads, 0, 1, stream, (const T*)x, (int)M, K, kp, q, scale);
}

static int check_quantize(const void* x, int32_t dtype, int64_t M, int64_t K, const void* q, const void* scale) {
  if (!x || !q || !scale) { set_error("x, q and scale must not be NULL"); return SP_ERR_INVALID_ARG; }
  if (M <= 0 || K <= 0) { set_error("M and K must be positive"); return SP_ERR_INVALID_ARG; }
  if (M >= (1ll << 31) - 256 || K >= (1ll << 31) - 256) { set_error("dimension too large"); return SP_ERR_UNSUPPORTED; }
  if (dtype != SP_BF16 && dtype != SP_FP32 && dtype != SP_FP16) { set_error("x must be bf16, fp32 or fp16"); return SP_ERR_INVALID_ARG; }
  if (((uintptr_t)q & 15u) || ((uintptr_t)scale & 3u) || ((uintptr_t)x & (elt_bytes(dtype) - 1))) {
    set_error("q must be 16-byte aligned, scale and x aligned to their elements");
    return SP_ERR_ALIGNMENT;
  }
  return SP_OK;
}

static int quantize(const void* x, int32_t dtype, int64_t M, int64_t K, int8_t* q, float* scale, cudaStream_t stream) {
  if (dtype == SP_BF16) return launch_quantize<__nv_bfloat16>(x, M, K, q, scale, stream);
  if (dtype == SP_FP16) return launch_quantize<__half>(x, M, K, q, scale, stream);
  return launch_quantize<float>(x, M, K, q, scale, stream);
}

struct I8Call {
  const void *A, *B;
  const float *a_scale, *b_scale;
  void* C;
  int64_t M, N, K;
  int out;
  int few;              // few-token form (library's choice of tile and order, M <= kFewTokens)
  int tile_m, tile_n;
  Sched sched;
  std::vector<int32_t> host_perm;
};

constexpr int64_t kFewTokens = 128;

// Checks everything the host can check; chooses tile and order where they are left to the library.
static int check_i8(const void* A, const void* a_scale, const void* B, const void* b_scale, const void* C, int64_t M, int64_t N, int64_t K,
                    int scheme, const sp_params* params, I8Call* call) {
  if (!A || !a_scale || !B || !b_scale || !C) { set_error("A, B, C and the scales must not be NULL"); return SP_ERR_INVALID_ARG; }
  if (M <= 0 || N <= 0 || K <= 0) { set_error("M, N, K must be positive"); return SP_ERR_INVALID_ARG; }
  if (M >= (1ll << 31) - 512 || N >= (1ll << 31) - 512) { set_error("dimension too large"); return SP_ERR_UNSUPPORTED; }
  if (K > SP_I8_MAX_K) { set_error("K must be at most %d: a longer sum can leave 32 bits", SP_I8_MAX_K); return SP_ERR_UNSUPPORTED; }
  if (params && params->struct_size != sizeof(sp_params)) {
    set_error("sp_params.struct_size is %u, expected %zu", params->struct_size, sizeof(sp_params));
    return SP_ERR_INVALID_ARG;
  }
  const int out = params ? params->out_dtype : SP_BF16;
  if (out != SP_BF16 && out != SP_FP32 && out != SP_FP16) { set_error("bad out_dtype"); return SP_ERR_INVALID_ARG; }
  if (params && params->b_layout != 1) { set_error("8-bit products take B as N x K (b_layout = 1)"); return SP_ERR_UNSUPPORTED; }
  if (params && (params->flags & ~SP_FLAG_SERPENTINE)) { set_error("of the flags only SP_FLAG_SERPENTINE applies to 8-bit products"); return SP_ERR_INVALID_ARG; }
  if ((K % 16) != 0) { set_error("K must be a multiple of 16 (16-byte row pitch; pad with zeros)"); return SP_ERR_ALIGNMENT; }
  if ((((uintptr_t)A | (uintptr_t)B) & 15u) || (((uintptr_t)a_scale | (uintptr_t)b_scale) & 3u) || ((uintptr_t)C & (elt_bytes(out) - 1))) {
    set_error("A and B must be 16-byte aligned, C and the scales aligned to their elements");
    return SP_ERR_ALIGNMENT;
  }
  int tile_m = params ? params->tile_m : 0, tile_n = params ? params->tile_n : 0;
  const bool pick = tile_m == 0 && tile_n == 0;
  if (!pick && !((tile_m == 256 && tile_n == 256) || (tile_m == 128 && (tile_n == 256 || tile_n == 128)))) {
    set_error("unsupported tile %dx%d (supported: 128x128, 128x256, 256x256)", tile_m, tile_n);
    return SP_ERR_UNSUPPORTED;
  }
  call->A = A; call->B = B; call->a_scale = (const float*)a_scale; call->b_scale = (const float*)b_scale; call->C = const_cast<void*>(C);
  call->M = M; call->N = N; call->K = K; call->out = out;
  call->few = scheme == SP_ORDER_AUTO && pick && M <= kFewTokens;
  if (call->few) return SP_OK;
  if (pick) {
    // the tile with the least waves x area / (CTAs per tile x relative rate of its shape); rates measured at 4096^3 and 8192^3
    static const struct { int tm, tn; double eff; } kTiles[] = {{256, 256, 1.00}, {128, 256, 0.92}, {128, 128, 0.70}};
    double best = 0;
    for (const auto& t : kTiles) {
      const int64_t T = ((M + t.tm - 1) / t.tm) * ((N + t.tn - 1) / t.tn);
      const int cg = t.tm / 128, units = 148 / cg;
      const double cost = (double)((T + units - 1) / units) * t.tm * t.tn / (cg * t.eff);
      if (tile_m == 0 || cost < best) { tile_m = t.tm; tile_n = t.tn; best = cost; }
    }
  }
  sp_params own = {};
  own.struct_size = sizeof own;
  if (scheme == SP_ORDER_AUTO) {
    // bands of eight tile rows, walked serpentine-wise, once the operands no longer fit in L2 together
    scheme = (M + N) * K > (64ll << 20) ? SP_GROUP_M : SP_ROW_MAJOR;
    own.group = 8;
    own.flags = SP_FLAG_SERPENTINE;
    params = &own;
  }
  call->tile_m = tile_m; call->tile_n = tile_n;
  int rc = resolve_sched(M, N, tile_m, tile_n, scheme, params, &call->sched);
  if (rc != SP_OK) return rc;
  if (scheme == kCustom || !already_validated(call->sched)) {
    rc = build_perm_host(call->sched, params ? params->custom_perm : nullptr, call->host_perm);
    if (rc != SP_OK) return rc;
    if (scheme != kCustom) remember_validated(call->sched);
  }
  return SP_OK;
}

template <int NT>
static int launch_few(const I8Call& c, const CUtensorMap& tmW, FewArgs args, cudaStream_t stream) {
  using C = FewCfg<NT>;
  CUtensorMap tmQ;
  int rc = make_map_any(&tmQ, c.A, 1, c.M, c.K, c.K, NT, 128);
  if (rc != SP_OK) return rc;
  auto kern = few_tokens_kernel<NT>;
  static uint64_t configured = 0;
  if (first_use_on_this_device(configured)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kSmemBytes);
    if (e != cudaSuccess) { configured = 0; set_error("cudaFuncSetAttribute(smem=%u) failed: %s", C::kSmemBytes, cudaGetErrorString(e)); return SP_ERR_CUDA; }
  }
  const int64_t blocks = (c.N + 127) / 128;
  // as many slices of k as two CTAs per SM allow, each with at least two stages of work
  int split = 1;
  while (split < 8 && blocks * split * 2 <= 2 * 148 && args.kblocks >= split * 2 * 2) split *= 2;
  args.kb_split = (args.kblocks + split - 1) / split;
  while (split > 1 && (split - 1) * args.kb_split >= args.kblocks) { split /= 2; args.kb_split = (args.kblocks + split - 1) / split; }   // every slice has work
  args.idesc = idesc_i8(128, NT);
  return launch_pdl("few-token product", kern, dim3((unsigned)(blocks * split)), 192, C::kSmemBytes, split, stream, tmW, tmQ, args);
}

template <bool OUT_F32>
static int launch_tiles(const I8Call& c, const ProdArgs& pa, const typename EpiI8<OUT_F32>::Args& ea, const CUtensorMap& tmA, const CUtensorMap& tmB,
                        const CUtensorMap& tmC, cudaStream_t stream) {
  if (c.tile_m == 256) return launch_product<2, 256, kElemI8, false, false, EpiI8<OUT_F32>>("8-bit product", tmA, tmB, tmC, pa, false, ea, stream);
  if (c.tile_n == 256) return launch_product<1, 256, kElemI8, false, false, EpiI8<OUT_F32>>("8-bit product", tmA, tmB, tmC, pa, false, ea, stream);
  return launch_product<1, 128, kElemI8, false, false, EpiI8<OUT_F32>>("8-bit product", tmA, tmB, tmC, pa, false, ea, stream);
}

static int run_i8(const I8Call& c, bool early, cudaStream_t stream) {
  LibraryState st;
  int rc = library_state(c.few ? nullptr : &c.sched, c.host_perm, stream, &st);
  if (rc != SP_OK) return rc;
  CUtensorMap tmA, tmB, tmC;
  if (c.few) {
    rc = make_map_any(&tmB, c.B, 1, c.N, c.K, c.K, 128, 128);
    if (rc != SP_OK) return rc;
    FewArgs a = {};
    a.a_scale = c.a_scale; a.b_scale = c.b_scale; a.C = (char*)c.C; a.status = st.status;
    a.M = (int)c.M; a.N = (int)c.N; a.kblocks = (int)((c.K + 127) / 128); a.out = c.out; a.early = early ? 1 : 0;
    if (c.M <= 16) return launch_few<16>(c, tmB, a, stream);
    if (c.M <= 32) return launch_few<32>(c, tmB, a, stream);
    if (c.M <= 64) return launch_few<64>(c, tmB, a, stream);
    return launch_few<128>(c, tmB, a, stream);
  }
  ProdArgs pa = {};
  pa.perm = st.perm; pa.status = st.status; pa.M = (int)c.M; pa.N = (int)c.N;
  pa.kblocks = (int)((c.K + 127) / 128); pa.splits = 1; pa.kb_split = pa.kblocks;
  pa.sched = c.sched;
  const int cg = c.tile_m / 128;
  rc = make_map_any(&tmA, c.A, 1, c.M, c.K, c.K, 128, 128);
  if (rc == SP_OK) rc = make_map_any(&tmB, c.B, 1, c.N, c.K, c.K, c.tile_n / cg, 128);
  if (rc != SP_OK) return rc;
  const int elt = (int)elt_bytes(c.out);
  const int64_t ld = c.N * elt;
  const bool plain = ((uintptr_t)c.C & 15u) || (ld & 15);
  if (plain) tmC = tmB;    // not used
  else rc = make_map_any(&tmC, c.C, elt, c.M, c.N, c.N, 32, 128 / elt);
  if (rc != SP_OK) return rc;
  if (c.out == SP_FP32) {
    EpiI8<true>::Args ea = {c.a_scale, c.b_scale, (char*)c.C, ld, 0, plain};
    return launch_tiles<true>(c, pa, ea, tmA, tmB, tmC, stream);
  }
  EpiI8<false>::Args ea = {c.a_scale, c.b_scale, (char*)c.C, ld, c.out == SP_BF16, plain};
  return launch_tiles<false>(c, pa, ea, tmA, tmB, tmC, stream);
}

}  // namespace sp

using namespace sp;

extern "C" {

int sp_quantize_i8(const void* x, int32_t x_dtype, int64_t M, int64_t K, int8_t* q, float* scale, void* stream) {
  int rc = check_quantize(x, x_dtype, M, K, q, scale);
  if (rc != SP_OK) return rc;
  int dev = 0;
  rc = current_device(&dev);
  if (rc != SP_OK) return rc;
  return quantize(x, x_dtype, M, K, q, scale, (cudaStream_t)stream);
}

int sp_gemm_i8(const int8_t* A, const float* a_scale, const int8_t* B, const float* b_scale, void* C, int64_t M, int64_t N, int64_t K,
               int scheme, const sp_params* params, void* stream) try {
  I8Call call;
  int rc = check_i8(A, a_scale, B, b_scale, C, M, N, K, scheme, params, &call);
  if (rc != SP_OK) return rc;
  int dev = 0;
  rc = current_device(&dev);
  if (rc != SP_OK) return rc;
  std::lock_guard<std::mutex> lock(g_i8_mu);
  return run_i8(call, false, (cudaStream_t)stream);
} catch (const std::exception& e) {
  set_error("sp_gemm_i8: %s", e.what());
  return SP_ERR_CUDA;
}

int sp_linear_i8(const void* x, int32_t x_dtype, int8_t* q, float* q_scale, const int8_t* W, const float* w_scale, void* y, int64_t M, int64_t N,
                 int64_t K, int scheme, const sp_params* params, void* stream) try {
  int rc = check_quantize(x, x_dtype, M, K, q, q_scale);
  if (rc != SP_OK) return rc;
  I8Call call;
  rc = check_i8(q, q_scale, W, w_scale, y, M, N, (K + 15) / 16 * 16, scheme, params, &call);
  if (rc != SP_OK) return rc;
  int dev = 0;
  rc = current_device(&dev);
  if (rc != SP_OK) return rc;
  std::lock_guard<std::mutex> lock(g_i8_mu);
  rc = quantize(x, x_dtype, M, K, q, q_scale, (cudaStream_t)stream);
  if (rc != SP_OK) return rc;
  return run_i8(call, true, (cudaStream_t)stream);
} catch (const std::exception& e) {
  set_error("sp_linear_i8: %s", e.what());
  return SP_ERR_CUDA;
}

}  // extern "C"
