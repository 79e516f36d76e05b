// Softmax cross entropy of a vocabulary product without keeping the scores, and its gradients.
//
//   z = h . W^T  (T x V),   lse_t = log sum_v exp z_tv,   loss_t = lse_t - z_t,target(t)
//   g_tv = c_t (exp(z_tv - lse_t) - [v = target(t)]),     dh = g . W,   dW = g^T . h
//
// Forward: the product runs tile by tile on the tensor cores; the epilogue reduces 128 columns of a row to a
// (maximum, sum of exponentials) pair, the row's target left out, so T x V scores become about T x V / 128 pairs, which a second kernel joins.
// Gradient: the vocabulary is walked in pieces.  A piece's scores are made again, turned into g in the epilogue and written as 16 bits;
// two more products read them: dh += g . W_piece (k = the vocabulary) and dW_piece = g^T . h (k = the tokens).  Where a token is nearly
// certain of its word, its own entry is made from the others' (see kRestStep).
#include <new>
#include <vector>

#include "linear_ce.cuh"

namespace sp {

__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];"
               ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(src) : "memory");
}
__device__ __forceinline__ void tma_add_3d(const CUtensorMap* map, uint32_t src, int x, int y, int z) {
  asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2, %3}], [%4];"
               ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(src) : "memory");
}

// ------------------------------------------------------------------ forward: statistics of a tile's rows
// Per row and 128 columns the maximum m (in powers of two: m = max z * log2 e, rounded once) and s = sum 2^(z log2 e - m).  Any m serves
// as long as the joined result uses the same one, so its rounding costs nothing.  The row's target is left out of both: its score
// goes to `picked`, and the join adds its term, so that a loss of 1e-6 is a sum of the others' terms and not a difference of 32-bit numbers.
//
// The tensor cores cut what they add off behind the accumulator's last bit, 16 products at a time, always towards zero: over D = 4096 lse
// came out 1.8e-6 too small, over 8192 4e-6.  So an accumulator takes 512 products only and the epilogue adds such sums, rounded to
// nearest: 2e-7, in the same time (256 products: 1e-7, and 11 % more time at D = 1024).
// What bounds it: 128 x 256 exponentials per CTA and tile at 16 a clock, 2048 cycles beside 512 for every 64 of D.
struct EpiStats {
  static constexpr uint32_t kBytes = 0;
  static constexpr bool kSums = true;
  static constexpr bool kLive = false;
  struct Args {
    float2* stats;            // [part of the columns][row]
    float* picked;            // score of the row's target
    const int64_t* target;
  };
  const Args& a;
  int lane;
  int rel;                    // the row's target, as a column of this part; -1: not here
  __device__ EpiStats(const Args& args, const CUtensorMap*, uint32_t, int, int l) : a(args), lane(l) {}
  __device__ __forceinline__ void before(const EpiTile& e, int M, int N) {
    const int row = e.row0 + lane;
    const int64_t t = row < M ? __ldg(a.target + row) : -1;
    rel = t >= e.col0 && t < N && t < (int64_t)e.col0 + kCePart ? (int)(t - e.col0) : -1;      // N: the tile's edge
  }
  template <int COLS>
  __device__ __forceinline__ void finish(uint32_t (&v)[COLS], const EpiTile& e, int M, int N) {
    static_assert(COLS == kCePart, "");
    if (e.col0 + COLS > N) {     // columns beyond the tile or the vocabulary
#pragma unroll
      for (int j = 0; j < COLS; ++j)
        if (e.col0 + j >= N) v[j] = 0xff800000u;
    }
    float hit = 0.f;
    if (__any_sync(0xffffffffu, rel >= 0)) {
#pragma unroll
      for (int j = 0; j < COLS; ++j)
        if (rel == j) { hit = __uint_as_float(v[j]); v[j] = 0xff800000u; }
    }
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = __uint_as_float(v[i]);
#pragma unroll
    for (int j = 8; j < COLS; j += 16) {
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = j + 8 + i < COLS ? fmaxf(fmaxf(t[i], __uint_as_float(v[j + i])), __uint_as_float(v[j + 8 + i])) : fmaxf(t[i], __uint_as_float(v[j + i]));
    }
    const float m = fmaxf(fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])), fmaxf(fmaxf(t[4], t[5]), fmaxf(t[6], t[7]))) * kLog2e;
    const float ref = m == -CUDART_INF_F ? 0.f : m;    // nothing finite here: every term is exp2(-inf) = 0
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = 0.f;
#pragma unroll
    for (int j = 0; j < COLS; j += 8)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] += ex2(fmaf(__uint_as_float(v[j + i]), kLog2e, -ref));
    const int row = e.row0 + lane;
    if (row < M) {
      a.stats[(int64_t)e.part * M + row] = make_float2(m, ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7])));
      if (rel >= 0) a.picked[row] = hit;
    }
  }
};

// ------------------------------------------------------------------ forward: one token
// The call is one read of W, so what counts is that every SM reads the same share of it, whatever V is, from the first cycle to the
// last: in the tiled form 256 words per CTA leave 20 of 148 SMs without work at 32768 words.  Here a warp takes two rows of W,
// asks for 4 KiB of each at once, straight to registers, multiplies in fp32 and keeps the running (maximum, sum) of its
// rows' scores; a block leaves one pair.  Measured at 32768 x 4096: 52 us, tiled 66.  For one token only: every further one
// costs the fp32 units as much again (two tokens 60 us, tiled 55).
constexpr int kRowThreads = 256, kRowUnroll = 8;
constexpr int64_t kRowMaxD = 16384;       // the token as fp32 in 64 KiB of shared memory

struct RowArgs {
  const uint16_t* W;
  const uint16_t* h;
  const int64_t* target;
  float2* stats;        // [block]
  float* picked;
  int V, D;
  int bf16;
};

__global__ void __launch_bounds__(kRowThreads, 2) row_stats_kernel(const RowArgs a) {
  extern __shared__ __align__(16) float row_token[];      // D
  __shared__ float2 part[kRowThreads / 32];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, warp = blockIdx.x * (kRowThreads / 32) + wid;
  const int step = gridDim.x * (kRowThreads / 32) * 2;
  pdl_begin();
  int4 w[2][kRowUnroll];
  auto fetch = [&](int64_t n, int k) {      // elements [k, k + 2048) of rows n and n + 1
#pragma unroll
    for (int u = 0; u < kRowUnroll; ++u)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int c = k + u * 256 + lane * 8;
        w[r][u] = n + r < a.V && c < a.D ? __ldcs(reinterpret_cast<const int4*>(a.W + (n + r) * a.D + c)) : make_int4(0, 0, 0, 0);
      }
  };
  fetch(warp * 2, 0);
  for (int i = threadIdx.x; i < a.D / 2; i += kRowThreads) {
    float lo, hi;
    row_values(__ldg(reinterpret_cast<const uint32_t*>(a.h) + i), a.bf16, lo, hi);
    reinterpret_cast<float2*>(row_token)[i] = make_float2(lo, hi);
  }
  const int64_t want = __ldg(a.target);
  __syncthreads();
  float2 pair = make_float2(-CUDART_INF_F, 0.f);
  for (int64_t n = (int64_t)warp * 2; n < a.V; n += step) {
    float acc[2] = {};
    for (int k = 0; k < a.D; k += kRowUnroll * 256) {
#pragma unroll
      for (int u = 0; u < kRowUnroll; ++u) {
        const int c = k + u * 256 + lane * 8;
        if (c < a.D) {
          const float4 p = *reinterpret_cast<const float4*>(row_token + c), q = *reinterpret_cast<const float4*>(row_token + c + 4);
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float lo, hi;
            row_values((uint32_t)w[r][u].x, a.bf16, lo, hi); acc[r] = fmaf(lo, p.x, acc[r]); acc[r] = fmaf(hi, p.y, acc[r]);
            row_values((uint32_t)w[r][u].y, a.bf16, lo, hi); acc[r] = fmaf(lo, p.z, acc[r]); acc[r] = fmaf(hi, p.w, acc[r]);
            row_values((uint32_t)w[r][u].z, a.bf16, lo, hi); acc[r] = fmaf(lo, q.x, acc[r]); acc[r] = fmaf(hi, q.y, acc[r]);
            row_values((uint32_t)w[r][u].w, a.bf16, lo, hi); acc[r] = fmaf(lo, q.z, acc[r]); acc[r] = fmaf(hi, q.w, acc[r]);
          }
        }
      }
      if (k + kRowUnroll * 256 < a.D) fetch(n, k + kRowUnroll * 256);
      else if (n + step < a.V) fetch(n + step, 0);
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
#pragma unroll
      for (int o = 16; o; o >>= 1) acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], o);
      if (want == n + r) {      // the target's term is the join's
        if (lane == 0 && n + r < a.V) *a.picked = acc[r];
      } else if (n + r < a.V) {
        const float m = fmaxf(pair.x, acc[r] * kLog2e), ref = m == -CUDART_INF_F ? 0.f : m;
        pair = make_float2(m, fmaf(pair.y, ex2(pair.x - ref), ex2(fmaf(acc[r], kLog2e, -ref))));
      }
    }
  }
  if (lane == 0) part[wid] = pair;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kRowThreads / 32; ++i) join_pair(pair, part[i]);
    a.stats[blockIdx.x] = pair;
  }
}

struct CeJoin {
  const float2* stats;  // without the target
  const float* picked;  // the target's score
  const int64_t* target;
  float* lse;
  float* each;        // loss per token
  float* loss;        // the reduced loss (mean, sum), else nullptr
  int T, V, tiles;
  int64_t ignore;
  int mean;
};

// 2^shift rows per block.
__global__ void __launch_bounds__(1024) ce_join_kernel(const CeJoin a, int shift) {
  pdl_begin();
  __shared__ float2 part[1024];
  const int rows = 1 << shift, r = threadIdx.x & (rows - 1);
  for (int64_t first = (int64_t)blockIdx.x << shift; first < a.T; first += (int64_t)gridDim.x << shift) {
    const bool ends = (int)threadIdx.x < rows && first + r < a.T;      // this thread finishes a row
    const int64_t y = ends ? __ldg(a.target + first + r) : -1;
    const bool hit = ends && y >= 0 && y < a.V;
    const float picked = hit ? a.picked[first + r] : -CUDART_INF_F;      // no word of the vocabulary: no term of its own
    join_rows(a.stats, a.T, a.tiles, first, shift, part);
    if (ends) {
      const float2 pair = joined_row(part, r, shift);
      // With `own` the target's exponent against the larger maximum, its product not rounded, and `rest` the sum of the others: lse = ref + log2(rest +
      // 2^own), and the loss is log(1 + rest / 2^own), whose digits do not depend on the size of the scores.  (lse - picked, in scores of 30:
      // losses below 1e-5 were noise of +-4e-6.)
      const float top = fmaxf(pair.x, picked * kLog2e), ref = top == -CUDART_INF_F ? 0.f : top;
      const float own = fmaf(picked, kLog2e, -ref), mine = ex2(own), rest = pair.y * ex2(pair.x - ref);
      const float bits = log2f(rest + mine);
      a.lse[first + r] = (ref + bits) * kLn2;
      a.each[first + r] = y == a.ignore ? 0.f : !hit ? CUDART_NAN_F : rest < mine ? log1pf(rest / mine) : (bits - own) * kLn2;
    }
    __syncthreads();      // before the next rows' pairs
  }
  if (a.loss != nullptr && gridDim.x == 1) {
    __syncthreads();
    reduce_losses(a.each, a.T, a.mean, a.loss, [&](int64_t t) { return a.target[t] != a.ignore; });
  }
}

__global__ void __launch_bounds__(1024) ce_reduce_kernel(const CeJoin a) {
  pdl_begin();
  reduce_losses(a.each, a.T, a.mean, a.loss, [&](int64_t t) { return a.target[t] != a.ignore; });
}

// ------------------------------------------------------------------ gradient
// The tokens' rows once more, each on a cache line of its own (a row of a tile's 128 bytes then takes one line of L2, not two: 1001 x 50001 x
// 1032 forward 123 us without, 116 with) and, for the gradient, zeros where a token does not count: dW adds 0 x h for those, and what an
// ignored row holds need not be finite.
__device__ __forceinline__ void ce_copy_rows(const CePrep& a, int block, int blocks) {
  const int64_t n = a.T * a.vecs;
  for (int64_t i = (int64_t)block * blockDim.x + threadIdx.x; i < n; i += (int64_t)blocks * blockDim.x) {
    const int64_t t = i / a.vecs;
    const uint4 v = __ldg(a.h + i);
    const uint4 w = a.masked && !a.kept(t) ? make_uint4(0u, 0u, 0u, 0u) : v;
    a.rows[t * a.ld + (i - t * a.vecs)] = w;
    if (a.twice) a.rows[(t + a.T) * a.ld + (i - t * a.vecs)] = w;
  }
}

__global__ void __launch_bounds__(1024) ce_rows_kernel(const CePrep a) {
  pdl_begin();
  ce_copy_rows(a, blockIdx.x, gridDim.x);
}

// What the loss's gradient puts on each token, c_t = factor * coef_t: g is made with coef_t and rounded to 16 bits, the two products
// multiply by `factor` in fp32.
//   One number for all tokens (mean, sum): it all goes to `factor`, so that its own rounding does not repeat in every token's
//   largest entry, p - 1 ~ -1, which 16 bits hold well.
//   A weight per token (none): coef_t.
// fp16 reaches down to 2^-24 only, and p ranges down to 1 / V and below: there coef is scaled by a power of two that brings
// its largest value to [2^14, 2^15] (|g| <= coef stays below 65504), and `factor` by the inverse.  Block 0; the others copy rows.
__global__ void __launch_bounds__(1024) ce_prep_kernel(const CePrep a) {
  pdl_begin();
  if (blockIdx.x > 0) {
    ce_copy_rows(a, blockIdx.x - 1, gridDim.x - 1);
    return;
  }
  __shared__ int part_n[32];
  __shared__ float part_m[32];
  int n = 0;
  float top = 0.f;
  for (int64_t t = threadIdx.x; t < a.T; t += 1024) {
    const bool kept = a.kept(t);
    n += kept;
    if (kept && a.reduction == SP_REDUCE_NONE && a.grad) top = fmaxf(top, fabsf(a.grad[t]));
  }
  for (int o = 16; o; o >>= 1) {
    n += __shfl_xor_sync(0xffffffffu, n, o);
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  }
  if ((threadIdx.x & 31) == 0) { part_n[threadIdx.x >> 5] = n; part_m[threadIdx.x >> 5] = top; }
  __syncthreads();
  n = 0; top = 0.f;
  for (int i = 0; i < 32; ++i) { n += part_n[i]; top = fmaxf(top, part_m[i]); }
  const bool each = a.reduction == SP_REDUCE_NONE && a.grad;
  float factor = 1.f;
  if (!each) {
    factor = a.grad ? a.grad[0] : 1.f;
    if (a.reduction == SP_REDUCE_MEAN) factor = n > 0 ? factor / (float)n : 0.f;
    top = 1.f;
  }
  // not finite (an overflowed loss scale): onto the tokens that count, so that it does not meet the zeros of the ignored ones
  const float wild = fabsf(factor) < CUDART_INF_F ? 1.f : factor;
  if (wild != 1.f) factor = 1.f;
  int up = 0;
  if (a.fp16 && top > 0.f && top < CUDART_INF_F) {
    int e;
    frexpf(top, &e);                     // top in [2^(e-1), 2^e)
    up = max(-100, min(100, each ? 15 - e : 15));
  }
  const float scale = exp2f((float)up);
  for (int64_t t = threadIdx.x; t < a.T; t += 1024) {
    float c = 0.f;
    if (a.kept(t)) c = a.lse == nullptr && (a.target[t] < 0 || a.target[t] >= a.V) ? CUDART_NAN_F : (each ? a.grad[t] : wild) * scale;
    a.coef[t] = c;
    a.rest[t] = 0;
  }
  if (threadIdx.x == 0) { *a.factor = factor * a.times * exp2f((float)-up); *a.count = 0; }
}

// The entry of a token's own word, p - 1, is the one that cancels: lse is a 32-bit number of the size of the scores, so p is off by |lse| 2^-23 or so,
// and of a token that is sure of its word (1 - p = 1e-5, scores of 30) nothing would be left.  But 1 - p is also the sum of the
// others' p, each good to a few 2^-23 of itself.  So that sum is what such tokens get.
//
// It is added up by all tiles of a row in any order, in whole steps of 2^-62: 62 bits and two to spare, the same result whatever the order.
constexpr float kRestStep = 0x1p-62f;
constexpr unsigned long long kRestNone = ~0ull;

// Scores of a part's columns to p, in place, and the sum of them.  The row's own word (`rel`, -1: not here) and what lies beyond the vocabulary or the
// tile count nothing and become 0; `hit`: the own word's score.  (Taken out before the exponentials, so that these and the additions run together.)
template <int COLS>
__device__ __forceinline__ float ce_probabilities(uint32_t (&v)[COLS], float lse2, int rel, int cols, float& hit) {
  hit = 0.f;
  if (__any_sync(0xffffffffu, rel >= 0)) {
#pragma unroll
    for (int j = 0; j < COLS; ++j)
      if (rel == j) { hit = __uint_as_float(v[j]); v[j] = 0xff800000u; }
  }
  if (cols < COLS) {
#pragma unroll
    for (int j = 0; j < COLS; ++j)
      if (j >= cols) v[j] = 0xff800000u;
  }
  const uint64_t scale = pair_of(kLog2e, kLog2e), off = pair_of(-lse2, -lse2);
  uint64_t s[4] = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < COLS; j += 8)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = j + 2 * i;
      float lo, hi;
      halves_of(fma_pair(pair_of(__uint_as_float(v[k]), __uint_as_float(v[k + 1])), scale, off), lo, hi);
      lo = ex2(lo); hi = ex2(hi);
      s[i] = add_pair(s[i], pair_of(lo, hi));
      v[k] = __float_as_uint(lo); v[k + 1] = __float_as_uint(hi);
    }
  float lo, hi;
  halves_of(add_pair(add_pair(s[0], s[1]), add_pair(s[2], s[3])), lo, hi);
  return lo + hi;
}

// While the vocabulary is one piece, the gradient's own tiles add the sums up and this kernel puts them into g, before anything reads g.  (Tokens whose
// p is at most 1/2 keep p - 1, which does not cancel there.)  Sums and launch cost 2 us in a short step (1 x 2000 x 512 from
// a graph: 26.7 to 28.6), 3 % at 777 x 20011 x 1032.
struct CeOwn {
  const int64_t* target;
  const float* lse;
  const float* coef;
  const unsigned long long* rest;
  uint16_t* g;
  int64_t ld;
  int T, V, bf16;
};

__global__ void __launch_bounds__(256) ce_own_kernel(const CeOwn a) {
  pdl_begin();
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= a.T) return;
  const int64_t y = __ldg(a.target + t);
  const float c = __ldg(a.coef + t), rest = __ull2float_rn(a.rest[t]) * kRestStep;
  const bool finite = fabsf(__ldg(a.lse + t)) < CUDART_INF_F && fabsf(c) < CUDART_INF_F;      // else the row is NaN as it stands
  if (finite && c != 0.f && y >= 0 && y < a.V && rest < 0.5f) a.g[t * a.ld + y] = (uint16_t)pack_16(-rest * c, 0.f, a.bf16);
}

// With the vocabulary in pieces the sum has to be there before the first piece is used.  So the tokens that are sure of their word (and only
// they) are put together in rows of their own, and one more product over the whole vocabulary makes their sums.  A warp per token:
// its own score, and with it 1 - p, well enough to tell.  Tokens with 1 - p of 1/16 + |lse| 2^-9 and more keep p - 1: it is off by
// |lse| 2^-23 / (1 - p) < 2^-13 relative there, less than 16 bits keep.
// The price is a fourth product for the share of tokens that are sure.  Gradient of 8192 x 131072 x 4096: 20.5 ms where none is, 22.7 where 30 % are, 27.5
// where all are.
struct CeSure {
  const int64_t* target;
  const float* lse;
  const float* coef;
  unsigned long long* rest;    // kRestNone for the tokens that are not sure
  const uint4* rows;           // the tokens, and the same pitch for
  uint4* sure;                 // those that are sure
  int32_t* list;               // whose these are
  int32_t* count;
  const uint4* W;
  int vecs, ld;
  int T, V, bf16;
};

__global__ void __launch_bounds__(256) ce_sure_kernel(const CeSure a) {
  pdl_begin();
  const int lane = threadIdx.x & 31;
  for (int64_t t = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); t < a.T; t += (int64_t)gridDim.x * 8) {
    const int64_t y = __ldg(a.target + t);
    const float lse = __ldg(a.lse + t), c = a.coef[t];
    bool sure = fabsf(lse) < CUDART_INF_F && fabsf(c) < CUDART_INF_F && c != 0.f && y >= 0 && y < a.V;
    const uint4* row = a.rows + t * a.ld;
    if (sure) {
      float z = 0.f;
      for (int i = lane; i < a.vecs; i += 32) {
        const uint4 p = row[i], q = __ldg(a.W + y * a.vecs + i);
        const uint32_t u[4] = {p.x, p.y, p.z, p.w}, w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float ul, uh, wl, wh;
          row_values(u[k], a.bf16, ul, uh);
          row_values(w[k], a.bf16, wl, wh);
          z = fmaf(ul, wl, z);
          z = fmaf(uh, wh, z);
        }
      }
      for (int o = 16; o; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
      sure = -expm1f(z - lse) < fminf(0.5f, 0.0625f + fabsf(lse) * 0x1p-9f);
    }
    if (!sure) {
      if (lane == 0) a.rest[t] = kRestNone;
      continue;
    }
    int at = 0;
    if (lane == 0) {
      at = atomicAdd(a.count, 1);      // any order: a token's sum does not depend on its place
      a.list[at] = (int)t;
    }
    at = __shfl_sync(0xffffffffu, at, 0);
    for (int i = lane; i < a.vecs; i += 32) a.sure[(int64_t)at * a.ld + i] = row[i];
  }
}

// The sums of the tokens that are sure.
struct EpiRest {
  static constexpr uint32_t kBytes = 0;
  static constexpr bool kSums = true;
  static constexpr bool kLive = true;
  struct Args {
    const float* lse;
    const int64_t* target;
    const int32_t* list;
    const int32_t* count;
    unsigned long long* rest;
  };
  const Args& a;
  int lane, token, rel;
  float lse2;
  __device__ EpiRest(const Args& args, const CUtensorMap*, uint32_t, int, int l) : a(args), lane(l) {}
  __device__ __forceinline__ void before(const EpiTile& e, int, int) {
    token = e.row0 + lane < *a.count ? a.list[e.row0 + lane] : -1;
    lse2 = token >= 0 ? __ldg(a.lse + token) * kLog2e : 0.f;
    const int64_t t = token >= 0 ? __ldg(a.target + token) - e.col0 : -1;
    rel = t >= 0 && t < kCePart ? (int)t : -1;
  }
  template <int COLS>
  __device__ __forceinline__ void finish(uint32_t (&v)[COLS], const EpiTile& e, int, int N) {
    float hit;
    const float s = ce_probabilities<COLS>(v, lse2, rel, N - e.col0, hit);
    if (token >= 0) atomicAdd(a.rest + token, __float2ull_rn(s / kRestStep));
  }
};

// g of a tile, to 16 bits: its rounding (at most half a step, 2^-8 of bf16 or 2^-11 of fp16 relative) is independent from entry to entry and
// enters sums over the vocabulary or the tokens, so it moves a gradient by less than the gradient's own rounding to the same type.
struct EpiG {
  static constexpr uint32_t kBytes = 8 * 4096;
  static constexpr bool kSums = true;       // the scores as the forward product made them: a sum that is cut off all along D is too small, and with it every p
  static constexpr bool kLive = false;
  struct Args {
    const float* lse;
    const float* coef;
    const int64_t* target;
    int64_t v0;              // first column of the piece
    unsigned long long* rest;
    int given;               // 1: sums of the others' p are in `rest` (or kRestNone), 0: they are added up there
    int bf16;
  };
  const Args& a;
  const CUtensorMap* map;
  EpiStage stage;
  int lane, rel;
  float lse2, c, minus;      // minus: 1 - p of the own word, where it is given
  __device__ EpiG(const Args& args, const CUtensorMap* m, uint32_t base, int w, int l) : a(args), map(m), stage{base + (uint32_t)w * 4096u, l}, lane(l) {}
  __device__ __forceinline__ void before(const EpiTile& e, int M, int) {
    const int row = e.row0 + lane;
    const bool in = row < M;
    c = in ? __ldg(a.coef + row) : 0.f;
    lse2 = in ? __ldg(a.lse + row) * kLog2e : 0.f;
    const int64_t t = in ? __ldg(a.target + row) - a.v0 - e.col0 : -1;
    rel = t >= 0 && t < kCePart ? (int)t : -1;
    minus = -1.f;
    if (a.given && rel >= 0) {
      const unsigned long long r = a.rest[row];
      if (r != kRestNone) minus = __ull2float_rn(r) * kRestStep;
    }
  }
  template <int COLS>
  __device__ __forceinline__ void finish(uint32_t (&v)[COLS], const EpiTile& e, int M, int N) {
    float hit;
    const float s = ce_probabilities<COLS>(v, lse2, rel, N - e.col0, hit);
    if (!a.given && e.row0 + lane < M && c != 0.f) atomicAdd(a.rest + e.row0 + lane, __float2ull_rn(s / kRestStep));
    const float own = minus >= 0.f ? -minus : ex2(fmaf(hit, kLog2e, -lse2)) - 1.f;
#pragma unroll
    for (int q = 0; q < COLS / 64; ++q) {
      uint32_t p[32];
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        p[j] = pack_16(__uint_as_float(v[q * 64 + 2 * j]) * c, __uint_as_float(v[q * 64 + 2 * j + 1]) * c, a.bf16);
        if (c == 0.f) p[j] = 0;     // a token that does not count: exactly nothing, whatever its scores are
      }
      const uint32_t slice = stage.free();
      stage_row(slice, lane, p);
      const uint32_t at = (uint32_t)(rel - q * 64);
      if (at < 64u && c != 0.f)      // the own word's entry, over the zero
        asm volatile("st.shared.b16 [%0], %1;" ::"r"(slice + (uint32_t)lane * 128u + (((at >> 3) ^ ((uint32_t)lane & 7u)) << 4) + (at & 7u) * 2u),
                     "h"((uint16_t)pack_16(own * c, 0.f, a.bf16)) : "memory");
      fence_async_smem();
      __syncwarp();
      const int col = e.col0 + q * 64;
      if (lane == 0 && e.row0 < M && col < N) {
        tma_store_2d(map, slice, col, e.row0);
        bulk_commit();
      }
    }
  }
};

// Both gradients are sums of 512 products added to each other in fp32, as the scores are: over 65536 tokens one accumulator came out 4e-4 too
// small, nearly half a step of fp16.
//
// fp32 sums of a slice of the vocabulary: stored by the first piece, added to by the later ones (each element once per piece,
// in stream order: the same bits every time).
struct EpiSum {
  static constexpr uint32_t kBytes = 8 * 4096;
  static constexpr bool kSums = true;
  static constexpr bool kLive = false;
  struct Args { int add; };
  const Args& a;
  const CUtensorMap* map;
  EpiStage stage;
  int lane;
  __device__ EpiSum(const Args& args, const CUtensorMap* m, uint32_t base, int w, int l) : a(args), map(m), stage{base + (uint32_t)w * 4096u, l}, lane(l) {}
  __device__ __forceinline__ void before(const EpiTile&, int, int) {}
  template <int COLS>
  __device__ __forceinline__ void finish(uint32_t (&v)[COLS], const EpiTile& e, int M, int N) {
#pragma unroll
    for (int q = 0; q < COLS / 32; ++q) {
      const uint32_t slice = stage.free();
      stage_row(slice, lane, *reinterpret_cast<uint32_t(*)[32]>(v + q * 32));
      fence_async_smem();
      __syncwarp();
      const int col = e.col0 + q * 32;
      if (lane == 0 && e.row0 < M && col < N) {
        if (a.add) tma_add_3d(map, slice, col, e.row0, e.z);
        else tma_store_3d(map, slice, col, e.row0, e.z);
        bulk_commit();
      }
    }
  }
};

// A finished gradient, to its 16-bit type.  Rows of dh of tokens that do not count are zero also where W is not finite (0 x infinity).
// TOKENS: rows are tokens (dh); else words (dW, whose writing bounds it for few tokens: 16 x 65536 x 4096 takes 484 us a step with the test of a row, 399
// without).
template <bool TOKENS>
struct EpiOut16 {
  static constexpr uint32_t kBytes = 8 * 4096;
  static constexpr bool kSums = true;
  static constexpr bool kLive = false;
  struct Args {
    const float* factor;
    const float* coef;       // of the tokens
    int bf16;
  };
  const Args& a;
  const CUtensorMap* map;
  EpiStage stage;
  int lane;
  float factor;
  bool none;
  __device__ EpiOut16(const Args& args, const CUtensorMap* m, uint32_t base, int w, int l)
      : a(args), map(m), stage{base + (uint32_t)w * 4096u, l}, lane(l), factor(__ldg(args.factor)) {}
  __device__ __forceinline__ void before(const EpiTile& e, int M, int) {
    if constexpr (TOKENS) none = e.row0 + lane < M && __ldg(a.coef + e.row0 + lane) == 0.f;
  }
  template <int COLS>
  __device__ __forceinline__ void finish(uint32_t (&v)[COLS], const EpiTile& e, int M, int N) {
#pragma unroll
    for (int q = 0; q < COLS / 64; ++q) {
      uint32_t p[32];
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        p[j] = pack_16(__uint_as_float(v[q * 64 + 2 * j]) * factor, __uint_as_float(v[q * 64 + 2 * j + 1]) * factor, a.bf16);
        if (TOKENS && none) p[j] = 0;
      }
      store_part(stage, map, lane, p, e.row0 < M && e.col0 + q * 64 < N, e.col0 + q * 64, e.row0);
    }
  }
};

// dh from the fp32 sums of its slices, added in slice order.  Four elements per thread (D is a multiple of 8); zeros as above.
__global__ void __launch_bounds__(256) ce_finish_kernel(const float4* acc, int64_t n4, int d4, int slices, const float* factor, const float* coef, int bf16, uint2* out) {
  pdl_begin();
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n4) return;
  float4 s = __ldcs(acc + i);
  for (int z = 1; z < slices; ++z) {
    const float4 p = __ldcs(acc + (int64_t)z * n4 + i);
    s.x += p.x; s.y += p.y; s.z += p.z; s.w += p.w;
  }
  const float f = __ldg(factor);
  out[i] = __ldg(coef + i / d4) == 0.f ? make_uint2(0u, 0u) : make_uint2(pack_16(s.x * f, s.y * f, bf16), pack_16(s.z * f, s.w * f, bf16));
}

// ------------------------------------------------------------------ host side
std::mutex g_ce_mu;

CePlan ce_plan(int64_t T, int64_t V, int64_t D, int halves) {
  CePlan p = {};
  T *= halves;
  p.T = T; p.V = V; p.D = D; p.halves = halves;
  p.row = T == 1 && D <= kRowMaxD;
  p.tiles = 2 * div_up(V, tile_width(T, V, ce_rows(T) / 128, 32));
  if (p.row) p.tiles = div_up(V, 2 * kRowThreads / 32) < 2 * 148 ? div_up(V, 2 * kRowThreads / 32) : 2 * 148;   // blocks: two per SM
  p.off_picked = up256(p.tiles * T * 8);
  p.off_each = p.off_picked + up256(T * 4);
  p.ld_h = (D + 63) / 64 * 64;
  // a launch of its own pays from about 50 us of products on
  p.copy = D % 64 != 0 && T > 128 && (double)T * (double)V * (double)D > 2.5e10;
  p.off_rows = p.off_each + up256(T * 4);
  p.forward_bytes = p.off_rows + (p.copy ? up256(T * p.ld_h * 2) : 0);
  // g of one piece takes 256 MiB, 27 waves of tiles on the whole device, or 2 KiB for each token (four tiles in width) where that is more; and the padding of
  // its rows
  constexpr int64_t kEntries = 128ll << 20;
  p.piece = V;
  if (T * V > kEntries) {
    p.piece = kEntries / T / kCeTile * kCeTile;
    if (p.piece < 4 * kCeTile) p.piece = 4 * kCeTile;
    if (p.piece > V) p.piece = V;
  }
  p.pieces = (int)div_up(V, p.piece);
  p.ld_g = (p.piece + 63) / 64 * 64;      // rows of g start on cache lines
  // Few tiles of dh and a long k axis: the vocabulary is cut into slices of at least four stages until every SM has one.
  const int64_t out_tiles = div_up(T, ce_rows(T)) * div_up(D, 256), units = ce_rows(T) == 256 ? 74 : 148, kb = div_up(p.piece, 64);
  int64_t s = out_tiles < units ? units / out_tiles : 1;
  if (s > kb / 4) s = kb / 4;
  if (s > kMaxSplits) s = kMaxSplits;
  if (s < 1) s = 1;
  p.slices = (int)s;
  p.off_factor = up256(T * 4);
  p.off_rest = p.off_factor + 256;
  p.off_list = p.off_rest + up256(T * 8);
  p.off_grad_rows = p.off_list + (p.pieces > 1 ? up256(T * 4) : 0);
  p.off_g = p.off_grad_rows + up256(T * p.ld_h * 2);
  p.off_acc = p.off_g + up256(T * p.ld_g * 2);
  p.grad_bytes = p.off_acc + (p.summed() ? up256(p.slices * T * D * 4) : 0);
  // With pieces, rows of the tokens that are sure lie where g or the sums of dh come later: a row of g has at least 1024 entries of 2 bytes, one of dh's sums D of 4.
  p.off_sure = p.ld_h <= p.ld_g ? p.off_g : p.off_acc;
  return p;
}

// Sizes that every grid of tiles of the two calls can hold (kMaxTiles of at least 128 x 160), and below 2^31 each: asked before anything is launched.
bool ce_sizes(int64_t T, int64_t V, int64_t D) {
  if (T <= 0 || V <= 0 || D <= 0 || T >= (1ll << 31) - 512 || V >= (1ll << 31) - 512 || D >= (1ll << 31) - 512) return false;
  const int64_t rows = div_up(T, ce_rows(T)), width = tile_width(T, V, ce_rows(T) / 128, 32);
  return rows * div_up(V, width) <= kMaxTiles && rows * div_up(D, 256) <= kMaxTiles && div_up(V, 256) * div_up(D, 256) <= kMaxTiles;
}

static int check_ce(const void* h, const void* W, const void* target, const void* lse, int64_t T, int64_t V, int64_t D, int32_t dtype, int32_t reduction,
                    const void* workspace) {
  if (!h || !W || !target || !lse || !workspace) { set_error("h, W, target, lse and workspace must not be NULL"); return SP_ERR_INVALID_ARG; }
  if (T <= 0 || V <= 0 || D <= 0) { set_error("T, V, D must be positive"); return SP_ERR_INVALID_ARG; }
  if (!ce_sizes(T, V, D)) { set_error("sizes too large"); return SP_ERR_UNSUPPORTED; }
  if (dtype != SP_BF16 && dtype != SP_FP16) { set_error("h and W must both be bf16 or both fp16"); return SP_ERR_UNSUPPORTED; }
  if (reduction != SP_REDUCE_NONE && reduction != SP_REDUCE_MEAN && reduction != SP_REDUCE_SUM) { set_error("unknown reduction %d", reduction); return SP_ERR_INVALID_ARG; }
  if ((D % 8) != 0) { set_error("D must be a multiple of 8 (16-byte row pitch)"); return SP_ERR_ALIGNMENT; }
  if ((((uintptr_t)h | (uintptr_t)W | (uintptr_t)workspace) & 15u) || ((uintptr_t)target & 7u) || ((uintptr_t)lse & 3u)) {
    set_error("h, W and workspace must be 16-byte aligned, target and lse aligned to their elements");
    return SP_ERR_ALIGNMENT;
  }
  return SP_OK;
}

// The tile grid of one product in bands of eight tile rows, walked serpentine-wise: a wave of tiles is then about as
// tall as it is wide, so it needs few operand panels, and a band starts on the panels the last one used last.  `rows`: row-major, for an
// output whose writing is what bounds the product: a wave then writes whole rows (dW of 16 tokens, 65536 x 4096: 106 us, in bands 114).
int ce_sched(int64_t M, int64_t N, int tile_m, int tile_n, Sched* out, bool rows) {
  if (rows) return resolve_sched(M, N, tile_m, tile_n, SP_ROW_MAJOR, nullptr, out);
  sp_params p = {};
  p.struct_size = sizeof p;
  p.group = 8;
  p.flags = SP_FLAG_SERPENTINE;
  return resolve_sched(M, N, tile_m, tile_n, SP_GROUP_M, &p, out);
}

ProdArgs ce_args(const Sched& sched, int32_t* status, int64_t M, int64_t N, int64_t K, int slices) {
  ProdArgs a = {};
  a.status = status;
  a.M = (int)M; a.N = (int)N; a.bn = 256;
  a.kblocks = (int)div_up(K, 64);
  a.splits = a.kblocks < slices ? a.kblocks : slices;
  a.kb_sum = kCeSum;
  a.sched = sched;
  return a;
}

CePrep ce_rows_args(const CePlan& p, const void* h, void* rows, const int64_t* target, int64_t ignore, bool masked) {
  CePrep a = {};
  a.target = target; a.h = (const uint4*)h; a.rows = (uint4*)rows; a.T = p.T / p.halves; a.twice = p.halves > 1; a.vecs = (int)(p.D / 8); a.ld = (int)(p.ld_h / 8);
  a.ignore = ignore; a.masked = masked; a.times = 1.f;
  return a;
}

unsigned ce_copy_blocks(const CePlan& p) {      // four vectors per thread, at most two blocks per SM
  const int64_t b = div_up(p.T * (p.D / 8), 4096);
  return (unsigned)(b < 296 ? b : 296);
}

// The two products of a piece of the vocabulary, [v0, v0 + cols): dh (its first piece if v0 = 0) and dW's rows.
int ce_products(const CePlan& p, const void* Wp, char* ws, void* dh, void* dW, int64_t v0, int64_t cols, bool bf16, int32_t* status, cudaStream_t stream) {
  const int64_t T = p.T, D = p.D;
  const float *coef = (const float*)ws, *factor = (const float*)(ws + p.off_factor);
  char *g = ws + p.off_g, *rows = ws + p.off_grad_rows, *acc = ws + p.off_acc;
  const bool summed = p.summed();
  CUtensorMap tmA, tmB, tmC;
  int rc = SP_OK;
  if (dh) {
    Sched sched;
    rc = ce_sched(T, D, ce_rows(T), 256, &sched);
    if (rc == SP_OK) rc = make_map_any(&tmA, g, 2, T, cols, p.ld_g, 128, 64);
    if (rc == SP_OK) rc = make_map_any(&tmB, Wp, 2, cols, D, D, 64, 64);
    if (rc != SP_OK) return rc;
    ProdArgs a = ce_args(sched, status, T, D, cols, p.slices);
    if (summed) {
      rc = make_map_3d_f32(&tmC, acc, p.slices, T, D, 32, 32);
      if (rc != SP_OK) return rc;
      const EpiSum::Args es = {v0 > 0};
      rc = ce_rows(T) == 256 ? launch_product<2, 256, kElem16, false, true, EpiSum>("gradient of h", tmA, tmB, tmC, a, bf16, es, stream)
                           : launch_product<1, 256, kElem16, false, true, EpiSum>("gradient of h", tmA, tmB, tmC, a, bf16, es, stream);
    } else {
      rc = make_map_any(&tmC, dh, 2, T, D, D, 32, 64);
      if (rc != SP_OK) return rc;
      const EpiOut16<true>::Args eo = {factor, coef, bf16};
      rc = ce_rows(T) == 256 ? launch_product<2, 256, kElem16, false, true, EpiOut16<true>>("gradient of h", tmA, tmB, tmC, a, bf16, eo, stream)
                           : launch_product<1, 256, kElem16, false, true, EpiOut16<true>>("gradient of h", tmA, tmB, tmC, a, bf16, eo, stream);
    }
    if (rc != SP_OK) return rc;
  }
  if (dW) {
    Sched sched;
    rc = ce_sched(cols, D, 256, 256, &sched, T * D <= (8ll << 20));
    if (rc == SP_OK) rc = make_map_any(&tmA, g, 2, T, cols, p.ld_g, 64, 64);
    if (rc == SP_OK) rc = make_map_any(&tmB, rows, 2, T, D, p.ld_h, 64, 64);
    if (rc == SP_OK) rc = make_map_any(&tmC, (char*)dW + v0 * D * 2, 2, cols, D, D, 32, 64);
    if (rc != SP_OK) return rc;
    ProdArgs a = ce_args(sched, status, cols, D, T, 1);
    a.overlap = dh != nullptr;      // it reads g and h only: its CTAs take the SMs that dh leaves free
    const EpiOut16<false>::Args eo = {factor, nullptr, bf16};
    rc = launch_product<2, 256, kElem16, true, true, EpiOut16<false>>("gradient of W", tmA, tmB, tmC, a, bf16, eo, stream);
    if (rc != SP_OK) return rc;
  }
  return rc;
}

// dh from its sums, where it has passed through them.
int ce_finish(const CePlan& p, char* ws, void* dh, bool bf16, cudaStream_t stream) {
  if (!p.summed()) return SP_OK;
  const int64_t n4 = p.T / p.halves * p.D / 4;
  return launch_pdl("sum of the slices", ce_finish_kernel, dim3((unsigned)div_up(n4, 256)), 256, 0, 1, stream, (const float4*)(ws + p.off_acc), n4, (int)(p.D / 4), p.slices * p.halves,
                    (const float*)(ws + p.off_factor), (const float*)ws, (int)bf16, (uint2*)dh);
}

int launch_ce_rows(const CePlan& p, const CePrep& a, cudaStream_t stream) {
  return launch_pdl("copy of the tokens", ce_rows_kernel, dim3(ce_copy_blocks(p)), 1024, 0, 1, stream, a);
}

int launch_ce_prep(const CePlan& p, const CePrep& a, cudaStream_t stream) {
  return launch_pdl("coefficients and rows of the tokens", ce_prep_kernel, dim3(1 + ce_copy_blocks(p)), 1024, 0, 1, stream, a);
}

static int launch_row(const RowArgs& a, int blocks, cudaStream_t stream) {
  static uint64_t configured = 0;
  if (first_use_on_this_device(configured)) {
    const cudaError_t e = cudaFuncSetAttribute(row_stats_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kRowMaxD * 4));
    if (e != cudaSuccess) { configured = 0; set_error("cudaFuncSetAttribute failed: %s", cudaGetErrorString(e)); return SP_ERR_CUDA; }
  }
  return launch_pdl("row products", row_stats_kernel, dim3((unsigned)blocks), kRowThreads, (size_t)a.D * 4, 1, stream, a);
}

}  // namespace sp

using namespace sp;

using Bytes = unsigned __int128;

extern "C" {

int64_t sp_linear_ce_workspace(int64_t T, int64_t V, int64_t D, int32_t grad) {
  if (!ce_sizes(T, V, D)) return -1;
  const CePlan p = ce_plan(T, V, D);
  return grad ? p.grad_bytes : p.forward_bytes;
}

int sp_linear_ce(const void* h, const void* W, const int64_t* target, float* lse, float* loss, int64_t T, int64_t V, int64_t D, int32_t dtype,
                 int64_t ignore_index, int32_t reduction, void* workspace, int64_t workspace_bytes, void* stream) try {
  int rc = check_ce(h, W, target, lse, T, V, D, dtype, reduction, workspace);
  if (rc != SP_OK) return rc;
  if (!loss) { set_error("loss must not be NULL"); return SP_ERR_INVALID_ARG; }
  if ((uintptr_t)loss & 3u) { set_error("loss must be aligned to its elements"); return SP_ERR_ALIGNMENT; }
  const CePlan p = ce_plan(T, V, D);
  if (workspace_bytes < p.forward_bytes) { set_error("workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)p.forward_bytes); return SP_ERR_INVALID_ARG; }
  const Span spans[] = {{"lse", lse, (Bytes)T * 4}, {"loss", loss, reduction == SP_REDUCE_NONE ? (Bytes)T * 4 : 4}, {"workspace", workspace, (Bytes)p.forward_bytes},
                        {"h", h, (Bytes)T * (Bytes)D * 2}, {"W", W, (Bytes)V * (Bytes)D * 2}, {"target", target, (Bytes)T * 8}};
  rc = refuse_overlaps(spans, 3, 6);
  if (rc != SP_OK) return rc;
  int dev = 0;
  rc = current_device(&dev);
  if (rc != SP_OK) return rc;
  std::lock_guard<std::mutex> lock(g_ce_mu);
  LibraryState st;
  rc = library_state(nullptr, {}, (cudaStream_t)stream, &st);
  if (rc != SP_OK) return rc;
  char* ws = (char*)workspace;
  const EpiStats::Args ea = {(float2*)ws, (float*)(ws + p.off_picked), target};
  if (p.row) {
    const RowArgs ra = {(const uint16_t*)W, (const uint16_t*)h, target, ea.stats, ea.picked, (int)V, (int)D, dtype == SP_BF16};
    rc = launch_row(ra, (int)p.tiles, (cudaStream_t)stream);
  } else {
    if (p.copy) {
      CePrep prep = ce_rows_args(p, h, ws + p.off_rows, target, ignore_index, false);
      rc = launch_ce_rows(p, prep, (cudaStream_t)stream);
      if (rc != SP_OK) return rc;
    }
    rc = ce_scores<EpiStats>("vocabulary product", p, p.copy ? ws + p.off_rows : h, p.copy ? p.ld_h : D, W, V, st.status, dtype == SP_BF16, nullptr, ea, (cudaStream_t)stream);
  }
  if (rc != SP_OK) return rc;
  CeJoin j = {};
  j.stats = ea.stats; j.picked = ea.picked; j.target = target; j.lse = lse;
  j.each = reduction == SP_REDUCE_NONE ? loss : (float*)(ws + p.off_each);
  j.loss = reduction == SP_REDUCE_NONE ? nullptr : loss;
  j.T = (int)T; j.V = (int)V; j.tiles = (int)p.tiles; j.ignore = ignore_index; j.mean = reduction == SP_REDUCE_MEAN;
  // 256 threads while a row's pairs are one batch of reads, else 1024
  // One block does up to 64 tokens of few pairs, and the sum of their losses with them: a launch less.
  const int shift = T <= 4 ? 2 : 5, threads = p.tiles <= 8 * (256 >> shift) ? 256 : 1024;
  const unsigned blocks = j.loss && T <= 64 && p.tiles <= 256 ? 1u : (unsigned)div_up(T, 1 << shift);
  rc = launch_pdl("join of the row statistics", ce_join_kernel, dim3(blocks), threads, 0, 1, (cudaStream_t)stream, j, shift);
  if (rc == SP_OK && j.loss && blocks > 1) rc = launch_pdl("sum of the losses", ce_reduce_kernel, dim3(1), 1024, 0, 1, (cudaStream_t)stream, j);
  return rc;
} catch (const std::exception& e) {
  set_error("sp_linear_ce: %s", e.what());
  return SP_ERR_CUDA;
}

int sp_linear_ce_grad(const void* h, const void* W, const int64_t* target, const float* lse, const float* grad_loss, void* dh, void* dW, int64_t T,
                      int64_t V, int64_t D, int32_t dtype, int64_t ignore_index, int32_t reduction, void* workspace, int64_t workspace_bytes,
                      void* stream_) try {
  int rc = check_ce(h, W, target, lse, T, V, D, dtype, reduction, workspace);
  if (rc != SP_OK) return rc;
  if (!dh && !dW) { set_error("dh and dW must not both be NULL"); return SP_ERR_INVALID_ARG; }
  if ((((uintptr_t)dh | (uintptr_t)dW) & 15u) || ((uintptr_t)grad_loss & 3u)) { set_error("dh and dW must be 16-byte aligned, grad_loss aligned to its elements"); return SP_ERR_ALIGNMENT; }
  const CePlan p = ce_plan(T, V, D);
  if (workspace_bytes < p.grad_bytes) { set_error("workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)p.grad_bytes); return SP_ERR_INVALID_ARG; }
  const Span spans[] = {{"dh", dh, (Bytes)T * (Bytes)D * 2}, {"dW", dW, (Bytes)V * (Bytes)D * 2}, {"workspace", workspace, (Bytes)p.grad_bytes},
                        {"h", h, (Bytes)T * (Bytes)D * 2}, {"W", W, (Bytes)V * (Bytes)D * 2}, {"target", target, (Bytes)T * 8}, {"lse", lse, (Bytes)T * 4},
                        {"grad_loss", grad_loss, reduction == SP_REDUCE_NONE ? (Bytes)T * 4 : 4}};
  rc = refuse_overlaps(spans, 3, 8);
  if (rc != SP_OK) return rc;
  int dev = 0;
  rc = current_device(&dev);
  if (rc != SP_OK) return rc;
  cudaStream_t stream = (cudaStream_t)stream_;
  std::lock_guard<std::mutex> lock(g_ce_mu);
  LibraryState st;
  rc = library_state(nullptr, {}, stream, &st);
  if (rc != SP_OK) return rc;
  const bool bf16 = dtype == SP_BF16;
  char* ws = (char*)workspace;
  float *coef = (float*)ws, *factor = (float*)(ws + p.off_factor);
  char* g = ws + p.off_g;
  char* rows = ws + p.off_grad_rows;
  auto* rest = (unsigned long long*)(ws + p.off_rest);
  int32_t *count = (int32_t*)(ws + p.off_factor + 4), *list = (int32_t*)(ws + p.off_list);
  CePrep prep = ce_rows_args(p, h, rows, target, ignore_index, true);
  prep.rest = rest; prep.count = count;
  prep.grad = grad_loss; prep.coef = coef; prep.factor = factor; prep.V = (int)V; prep.reduction = reduction; prep.fp16 = !bf16;
  rc = launch_ce_prep(p, prep, stream);
  if (rc != SP_OK) return rc;
  if (p.pieces > 1) {
    uint4* sure = (uint4*)(ws + p.off_sure);
    const CeSure cs = {target, lse, coef, rest, (const uint4*)rows, sure, list, count, (const uint4*)W, (int)(D / 8), (int)(p.ld_h / 8), (int)T, (int)V, bf16};
    const int64_t blocks = div_up(T, 8);
    rc = launch_pdl("tokens that are sure", ce_sure_kernel, dim3((unsigned)(blocks < 8 * 148 ? blocks : 8 * 148)), 256, 0, 1, stream, cs);
    if (rc != SP_OK) return rc;
    const EpiRest::Args er = {lse, target, list, count, rest};
    rc = ce_scores<EpiRest>("sums of the others", p, sure, p.ld_h, W, V, st.status, bf16, nullptr, er, stream, count);
    if (rc != SP_OK) return rc;
  }
  const auto scores = [&](int64_t v0, int64_t cols, const void* Wp, const CUtensorMap& tmG) {
    const EpiG::Args ea = {lse, coef, target, v0, rest, p.pieces > 1, bf16};
    int rc = ce_scores<EpiG>("gradient of the scores", p, rows, p.ld_h, Wp, cols, st.status, bf16, &tmG, ea, stream);
    if (rc == SP_OK && p.pieces == 1) {
      const CeOwn co = {target, lse, coef, rest, (uint16_t*)g, p.ld_g, (int)T, (int)V, bf16};
      rc = launch_pdl("own words", ce_own_kernel, dim3((unsigned)div_up(T, 256)), 256, 0, 1, stream, co);
    }
    return rc;
  };
  rc = ce_gradients(p, W, ws, dh, dW, bf16, st.status, stream, scores);
  return rc;
} catch (const std::exception& e) {
  set_error("sp_linear_ce_grad: %s", e.what());
  return SP_ERR_CUDA;
}

}  // extern "C"
