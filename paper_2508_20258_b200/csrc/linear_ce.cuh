// What the losses of a vocabulary product share: row statistics and their joining, the plan of pieces and workspace, the scores' product under an epilogue of the
// loss's own, and the gradients' products behind it.  (linear_ce_sm100.cu has the parts that are not templates.)
#pragma once
#include <math_constants.h>

#include <mutex>

#include "product.cuh"

namespace sp {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kCeTile = 256;     // vocabulary columns of one tile, at most
constexpr int kCePart = 128;     // and of one epilogue warp, at most
constexpr int kMaxSplits = 64;   // slices of the vocabulary in the product for dh
constexpr int kCeSum = 8;      // stages of 64 products per accumulator

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ void row_values(uint32_t u, int bf16, float& lo, float& hi) {
  if (bf16) {
    lo = __uint_as_float(u << 16); hi = __uint_as_float(u & 0xffff0000u);
  } else {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u));
    lo = f.x; hi = f.y;
  }
}

__device__ __forceinline__ void join_pair(float2& a, float2 p) {
  const float m = fmaxf(a.x, p.x), ref = m == -CUDART_INF_F ? 0.f : m;      // nothing finite yet: every term is exp2(-inf) = 0
  a = make_float2(m, a.y * ex2(a.x - ref) + p.y * ex2(p.x - ref));
}

// Mean or sum of the per-token losses in a fixed order, in fp64.  One block.  kept(t): the token counts.
template <class Kept>
__device__ __forceinline__ void reduce_losses(const float* each, int T, bool mean, float* loss, const Kept& kept) {
  __shared__ double part_s[32];
  __shared__ int part_n[32];
  double s = 0;
  int n = 0;
  for (int64_t t = threadIdx.x; t < T; t += blockDim.x) {
    s += each[t];
    n += kept(t);
  }
  for (int o = 16; o; o >>= 1) {
    s += __shfl_xor_sync(0xffffffffu, s, o);
    n += __shfl_xor_sync(0xffffffffu, n, o);
  }
  if ((threadIdx.x & 31) == 0) { part_s[threadIdx.x >> 5] = s; part_n[threadIdx.x >> 5] = n; }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < (int)blockDim.x / 32; ++i) { s += part_s[i]; n += part_n[i]; }
    loss[0] = (float)(mean ? s / n : s);     // no token left by the mask: 0 / 0
  }
}

// Pairs of 2^shift rows to one each.  blockDim >> shift threads share a row's pairs, whose reads do not wait
// for one another.  (Eight threads per row, joining pair after pair, took 6 us for one token's 296 pairs: a chain of trips to L2.)  `part`: 1024 pairs in shared memory.
__device__ __forceinline__ void join_rows(const float2* stats, int T, int tiles, int64_t first, int shift, float2* part) {
  const int rows = 1 << shift, groups = (int)blockDim.x >> shift;
  const int r = threadIdx.x & (rows - 1), g = threadIdx.x >> shift, lane = threadIdx.x & 31;
  float2 pair = make_float2(-CUDART_INF_F, 0.f);
  if (first + r < T) {
    const float2* at = stats + first + r;
    for (int i = g; i < tiles; i += 8 * groups) {
      float2 p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = i + j * groups < tiles ? __ldg(at + (int64_t)(i + j * groups) * T) : make_float2(-CUDART_INF_F, 0.f);
      float m = pair.x;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = fmaxf(m, p[j].x);
      const float ref = m == -CUDART_INF_F ? 0.f : m;
      float s = pair.y * ex2(pair.x - ref);
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fmaf(p[j].y, ex2(p[j].x - ref), s);
      pair = make_float2(m, s);
    }
  }
  part[threadIdx.x] = pair;
  __syncthreads();
  if (groups > 8) {      // a warp per row first
    for (int row = threadIdx.x >> 5; row < rows; row += blockDim.x >> 5) {
      pair = make_float2(-CUDART_INF_F, 0.f);
      for (int i = lane; i < groups; i += 32) join_pair(pair, part[i * rows + row]);
#pragma unroll
      for (int o = 16; o; o >>= 1) join_pair(pair, make_float2(__shfl_xor_sync(0xffffffffu, pair.x, o), __shfl_xor_sync(0xffffffffu, pair.y, o)));
      if (lane == 0) part[row] = pair;      // slot `row` is group 0's of this row: read above by this warp only
    }
    __syncthreads();
  }
}
// Row r's pair then.
__device__ __forceinline__ float2 joined_row(const float2* part, int r, int shift) {
  const int groups = (int)blockDim.x >> shift;
  float2 pair = part[r];
  for (int i = 1; i < groups && groups <= 8; ++i) join_pair(pair, part[(i << shift) + r]);
  return pair;
}

struct CePrep {
  const int64_t* target;      // cross entropy: the tokens' words, `ignore` for those that do not count
  const float* lse;           // else nullptr; distillation: +infinity for those that do not count
  const float* grad;     // per token (none) or one number; nullptr: 1
  float* coef;           // per token
  float* factor;         // one number
  const uint4* h;        // rows of `vecs` vectors of 8 elements ...
  uint4* rows;           // ... copied to rows of `ld` vectors
  int64_t T;
  int vecs, ld;
  int V;
  int64_t ignore;
  int reduction, fp16;
  float times;           // of `factor`
  int masked;            // 1: rows of ignored tokens become zeros
  int twice;             // 1: all rows once more behind the first T
  unsigned long long* rest;   // per token: set to 0 ...
  int32_t* count;             // ... and this one number too

  __device__ __forceinline__ bool kept(int64_t t) const { return lse != nullptr ? __ldg(lse + t) != CUDART_INF_F : __ldg(target + t) != ignore; }
};

// One staged slice of 64 16-bit columns to a matrix.
__device__ __forceinline__ void store_part(const EpiStage& stage, const CUtensorMap* map, int lane, const uint32_t (&p)[32], bool inside, int col, int row) {
  const uint32_t slice = stage.free();
  stage_row(slice, lane, p);
  fence_async_smem();
  __syncwarp();
  if (lane == 0 && inside) {
    tma_store_2d(map, slice, col, row);
    bulk_commit();
  }
}

// ------------------------------------------------------------------ host side
extern std::mutex g_ce_mu;   // per-kernel set-up is done under it

inline int64_t up256(int64_t b) { return (b + 255) & ~255ll; }
inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Everything that follows from the sizes alone.
struct CePlan {
  int64_t T, V, D;
  bool row;                   // forward: the form for one token
  int64_t tiles;              // pairs per token that the forward product leaves: two per vocabulary tile, or one per block
  int64_t piece, ld_g;        // gradient: vocabulary rows of a piece, row pitch of g
  int pieces;
  int slices;                 // of the vocabulary in the product for dh
  int halves;                 // 2: the second half of the T rows of h and g repeats the first, g as the rounding errors of the first half's: both add up to one row of dh
  bool copy;                  // forward: the tokens' rows are copied to cache lines of their own
  int64_t ld_h;               // row pitch of such copies
  int64_t off_picked, off_each, off_rows, forward_bytes;
  int64_t off_factor, off_rest, off_list, off_grad_rows, off_g, off_acc, off_sure, grad_bytes;
  bool summed() const { return pieces > 1 || slices > 1 || halves > 1; }      // dh passes through fp32 sums
};

// Rows of a token tile: a CTA pair's 256, or one CTA's 128 where no more tokens are there.  (Also for token counts that fill their last tile
// badly the smaller one does not pay: it moves half as much again through L2 per product.  777 x 20011 x 1032: forward 54 us on
// 4 x 256 rows, 58 on 7 x 128; dh 51 and 55.)
inline int ce_rows(int64_t T) { return T <= 128 ? 128 : 256; }

CePlan ce_plan(int64_t T, int64_t V, int64_t D, int halves = 1);
bool ce_sizes(int64_t T, int64_t V, int64_t D);      // whether the calls take them
int ce_sched(int64_t M, int64_t N, int tile_m, int tile_n, Sched* out, bool rows = false);
ProdArgs ce_args(const Sched& sched, int32_t* status, int64_t M, int64_t N, int64_t K, int slices);
CePrep ce_rows_args(const CePlan& p, const void* h, void* rows, const int64_t* target, int64_t ignore, bool masked);
unsigned ce_copy_blocks(const CePlan& p);
int launch_ce_rows(const CePlan& p, const CePrep& a, cudaStream_t stream);
int launch_ce_prep(const CePlan& p, const CePrep& a, cudaStream_t stream);
int ce_products(const CePlan& p, const void* Wp, char* ws, void* dh, void* dW, int64_t v0, int64_t cols, bool bf16, int32_t* status, cudaStream_t stream);
int ce_finish(const CePlan& p, char* ws, void* dh, bool bf16, cudaStream_t stream);

// h . W_piece^T with an epilogue of scores.
template <class Epi>
int ce_scores(const char* what, const CePlan& p, const void* h, int64_t ld_h, const void* W, int64_t cols, int32_t* status, bool bf16, const CUtensorMap* tmC,
                     const typename Epi::Args& ea, cudaStream_t stream, const int32_t* live = nullptr, int overlap = 0) {
  CUtensorMap tmA, tmB;
  Sched sched;
  const int rows = ce_rows(p.T), width = tile_width(p.T, cols, rows / 128, tmC ? 64 : 32);      // g is stored 64 columns at a time
  int rc = ce_sched(p.T, cols, rows, width, &sched);
  if (rc == SP_OK) rc = make_map_any(&tmA, h, 2, p.T, p.D, ld_h, 128, 64);
  if (rc == SP_OK) rc = make_map_any(&tmB, W, 2, cols, p.D, p.D, width / (rows / 128), 64);
  if (rc != SP_OK) return rc;
  ProdArgs a = ce_args(sched, status, p.T, cols, p.D, 1);
  a.turn = sched.Tm == 1;
  a.live = live;
  a.overlap = overlap;
  a.bn = width;
  if (rows == 256) return launch_product<2, 256, kElem16, false, false, Epi>(what, tmA, tmB, tmC ? *tmC : tmA, a, bf16, ea, stream);
  return launch_product<1, 256, kElem16, false, false, Epi>(what, tmA, tmB, tmC ? *tmC : tmA, a, bf16, ea, stream);
}

// Both gradients, the vocabulary piece by piece: scores(v0, columns, W's rows, map of g) leaves g of a piece.
template <class Scores>
int ce_gradients(const CePlan& p, const void* W, char* ws, void* dh, void* dW, bool bf16, int32_t* status, cudaStream_t stream, const Scores& scores) {
  for (int64_t v0 = 0; v0 < p.V; v0 += p.piece) {
    const int64_t cols = p.V - v0 < p.piece ? p.V - v0 : p.piece;
    const char* Wp = (const char*)W + v0 * p.D * 2;
    CUtensorMap tmG;
    int rc = make_map_any(&tmG, ws + p.off_g, 2, p.T, cols, p.ld_g, 32, 64);
    if (rc == SP_OK) rc = scores(v0, cols, Wp, tmG);
    if (rc == SP_OK) rc = ce_products(p, Wp, ws, dh, dW, v0, cols, bf16, status, stream);
    if (rc != SP_OK) return rc;
  }
  return dh ? ce_finish(p, ws, dh, bf16, stream) : SP_OK;
}

}  // namespace sp
