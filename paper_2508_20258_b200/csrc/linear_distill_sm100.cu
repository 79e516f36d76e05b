// Distillation from a teacher's top logits under a vocabulary product, without keeping the scores, and its gradients.
//
//   z = h . W^T / tau,   lse_t = log sum_v exp z_tv,   p = exp(z - lse),   q: softmax of a token's K logits / tau, 0 for all other words
//   loss_t = tau^2 sum_v q_v (log q_v - log p_v),   g_tv = c_t tau (p_tv - q_tv),   dh = g . W,   dW = g^T . h
//
// Beside the products, which are those of the cross entropy, K words per token have to be met.  Forward: a first kernel sorts each token's words; the product's epilogue
// finds those of its 128 columns by an index of the sorted list, hands their scores on and leaves them out of its (maximum, sum) pair; the join makes
// lse, the loss and p - q of the token's words.  Gradient: the tiles write c p in 16 bits, and a kernel puts c (p - q) over it where the teacher has words: T x K
// scattered entries, a fraction of a percent of g.
//
// The loss is tau^2 (sum of the other words' p + sum over the teacher's words of q d - q + p), d = log q - log p, whose terms are not negative; p - q of a word with p above 1/2 is the
// sum of all other q less the sum of all other p, and its d (with q above 1/2 too) made from those: a student that is sure and right keeps its digits.  For words below 1/2, p - q and d are
// differences of fp32 numbers, good to the scores' error and a few 2^-23 of p, q and their logarithms.
#include <new>

#include "linear_ce.cuh"

namespace sp {

constexpr int kMaxTop = 1024;
constexpr int kNoWord = 0x7fffffff;

// ------------------------------------------------------------------ the teacher's words in order
struct TeacherArgs {
  const int64_t* index;      // [T][K]
  const void* logit;
  int logit_dtype;
  float scale;               // log2 e / tau
  int32_t* word;             // [T][K] ascending, then kNoWord
  int32_t* slot;             // where it stood
  float* q;                  // of the first of equal words their sum (of the others nothing is read)
  float* lq;                 // log2 of it
  uint16_t* start;           // [T][parts + 1]: how many words come before a part of the columns
  int32_t* state;            // [T]: kIgnored, ...
  int64_t T;
  int V, K, size;            // size: K, at least 32, up to a power of two
  int parts, bn;             // of the scores' tiles
};
enum : int { kIgnored = 0, kKept = 1, kInvalid = 2 };      // no word, or none with a logit above minus infinity; a word outside the vocabulary

// Sorts 32 KEYS keys, the c-th of a lane being element 32 c + lane, in registers (4096 tokens of 64 words by way of shared memory 15.6 us, so 10.4).
template <int KEYS>
__device__ __forceinline__ void sort_keys(uint64_t (&key)[KEYS], int lane) {
#pragma unroll
  for (int k = 2; k <= 32 * KEYS; k *= 2)
#pragma unroll
    for (int o = k / 2; o; o /= 2) {
      if (o >= 32) {
#pragma unroll
        for (int c = 0; c < KEYS; ++c)
          if ((c & (o / 32)) == 0) {
            uint64_t &u = key[c], &w = key[c | (o / 32)];
            if ((u > w) == ((c * 32 & k) == 0)) {
              const uint64_t t = u;
              u = w; w = t;
            }
          }
      } else {
#pragma unroll
        for (int c = 0; c < KEYS; ++c) {
          const uint64_t w = __shfl_xor_sync(0xffffffffu, key[c], o);
          const bool low = ((c * 32 + lane) & k) == 0 == ((lane & o) == 0);      // this one keeps the smaller
          if ((w < key[c]) == low) key[c] = w;
        }
      }
    }
}

// GROUP threads per token, 32 KEYS keys: a warp, sorting in registers, or (KEYS 0: `size` of them) the block, in shared memory.
template <int GROUP, int KEYS>
__global__ void __launch_bounds__(256) teacher_kernel(const TeacherArgs a) {
  extern __shared__ uint64_t teacher_keys[];
  __shared__ float part[8];
  const int group = threadIdx.x / GROUP, i0 = threadIdx.x % GROUP, lane = threadIdx.x & 31;
  uint64_t* key = teacher_keys + group * a.size;                                               // word, and where it stood
  float* value = reinterpret_cast<float*>(teacher_keys + 256 / GROUP * a.size) + group * a.size;      // logits as they stood
  const auto sync = [] {
    if constexpr (GROUP == 32) __syncwarp();
    else __syncthreads();
  };
  const auto over_group = [&](float v, bool max) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const float w = __shfl_xor_sync(0xffffffffu, v, o);
      v = max ? fmaxf(v, w) : v + w;
    }
    if constexpr (GROUP > 32) {
      __syncthreads();
      if (lane == 0) part[threadIdx.x >> 5] = v;
      __syncthreads();
      v = part[0];
      for (int i = 1; i < GROUP / 32; ++i) v = max ? fmaxf(v, part[i]) : v + part[i];
    }
    return v;
  };
  pdl_begin();
  for (int64_t t = (int64_t)blockIdx.x * (256 / GROUP) + group; t < a.T; t += (int64_t)gridDim.x * (256 / GROUP)) {
    const auto logit = [&](int j) {
      const int64_t at = t * a.K + j;
      if (a.logit_dtype == SP_FP32) return __ldg((const float*)a.logit + at);
      float lo, hi;
      row_values(__ldg((const uint16_t*)a.logit + at), a.logit_dtype == SP_BF16, lo, hi);
      return lo;
    };
    float state = kIgnored, top = -CUDART_INF_F;
    uint64_t mine[KEYS ? KEYS : 1];
#pragma unroll
    for (int j = i0, c = 0; KEYS ? c < KEYS : j < a.size; j += GROUP, ++c) {
      int word = kNoWord;
      if (j < a.K) {
        const int64_t v = __ldg(a.index + t * a.K + j);
        const float l = logit(j);
        value[j] = l;
        if (v >= a.V) state = kInvalid;
        else if (v >= 0) {
          word = (int)v;
          top = fmaxf(top, l);
          if (l != -CUDART_INF_F) state = fmaxf(state, kKept);
        }
      }
      const uint64_t k = (uint64_t)word << 32 | (uint32_t)j;
      if constexpr (KEYS > 0) mine[c] = k;
      else key[j] = k;
    }
    state = over_group(state, true);
    top = over_group(top, true);
    if constexpr (KEYS > 0) {
      sort_keys<KEYS>(mine, lane);
#pragma unroll
      for (int c = 0; c < KEYS; ++c) key[c * 32 + lane] = mine[c];
      sync();
    } else {
      sync();
      for (int k = 2; k <= a.size; k *= 2)      // bitonic, as in registers
        for (int o = k / 2; o; o /= 2) {
          for (int i = i0; i < a.size / 2; i += GROUP) {
            const int x = (i & ~(o - 1)) * 2 + (i & (o - 1)), y = x + o;
            const uint64_t u = key[x], w = key[y];
            if ((u > w) == ((x & k) == 0)) { key[x] = w; key[y] = u; }
          }
          sync();
        }
    }
    float sum = 0.f;
    const auto term = [&](int i) { return ex2((value[(uint32_t)key[i]] - top) * a.scale); };      // a NaN, an infinity: all NaN
    for (int i = i0; i < a.K; i += GROUP)
      if ((int)(key[i] >> 32) != kNoWord) sum += term(i);
    sum = over_group(sum, false);
    const float log_sum = log2f(sum);
    for (int i = i0; i < a.K; i += GROUP) {
      const int word = (int)(key[i] >> 32), j = (int)(uint32_t)key[i];
      float q = 0.f, lq = -CUDART_INF_F;
      if (word != kNoWord && (i == 0 || (int)(key[i - 1] >> 32) != word)) {
        q = term(i);
        lq = fmaf(value[j] - top, a.scale, -log_sum);
        int n = i + 1;
        for (; n < a.K && (int)(key[n] >> 32) == word; ++n) q += term(n);
        if (n > i + 1) lq = log2f(q) - log_sum;
        q /= sum;
      }
      a.word[t * a.K + i] = word; a.slot[t * a.K + i] = j; a.q[t * a.K + i] = q; a.lq[t * a.K + i] = lq;
    }
    // Words before each part's first column: the i-th word makes that i from the part behind the word's before on, up to its own.  Before the first and behind the last all
    // threads write; `used` words are in a part.
    const auto part_of = [&](uint32_t word) { return (int)(word / a.bn * 2 + (word % a.bn >= (uint32_t)kCePart)); };
    uint16_t* start = a.start + t * (a.parts + 1);
    int used = 0;
    for (int i = i0; i < a.K; i += GROUP) {
      const uint32_t word = (uint32_t)(key[i] >> 32);
      if (word == kNoWord) break;
      used = i + 1;
      if (i > 0)
        for (int p = part_of((uint32_t)(key[i - 1] >> 32)) + 1, end = part_of(word); p <= end; ++p) start[p] = (uint16_t)i;
    }
    used = (int)over_group((float)used, true);
    const int first = used ? part_of((uint32_t)(key[0] >> 32)) : a.parts, last = used ? part_of((uint32_t)(key[used - 1] >> 32)) : a.parts;
    for (int p = i0; p <= first; p += GROUP) start[p] = 0;
    for (int p = last + 1 + i0; p <= a.parts; p += GROUP) start[p] = (uint16_t)used;
    if (i0 == 0) a.state[t] = (int)state;
    sync();
  }
}

// ------------------------------------------------------------------ forward: statistics of a tile's rows
// As the cross entropy's: per row and part the maximum (in powers of two) and the sum, all of the teacher's words left out and their scores handed on.  A warp looks at 32
// columns at a time as long as one of its rows has a word there: 64 words per token cost 4096 x 32768 x 2048 3 % (327 to 339 us).
struct EpiDistill {
  static constexpr uint32_t kBytes = 0;
  static constexpr bool kSums = true;
  static constexpr bool kLive = false;
  struct Args {
    float2* stats;            // [part of the columns][row]
    float* picked;            // [row][K]: scores of the words in their order
    const int32_t* word;
    const uint16_t* start;
    float scale;              // log2 e / tau
    int K, parts;
  };
  const Args& a;
  int lane;
  int at, end, next;          // of the row's words: the next one in this part, the part's end; its column in the part
  __device__ EpiDistill(const Args& args, const CUtensorMap*, uint32_t, int, int l) : a(args), lane(l) {}
  __device__ __forceinline__ void before(const EpiTile& e, int M, int) {
    const int64_t row = e.row0 + lane;
    at = end = 0;
    next = kNoWord;
    if (row < M) {
      const uint16_t* s = a.start + row * (a.parts + 1) + e.part;
      at = s[0]; end = s[1];      // written while this kernel was running: not by way of the read-only cache
      if (at < end) next = a.word[row * a.K + at] - e.col0;
    }
  }
  template <int COLS>
  __device__ __forceinline__ void finish(uint32_t (&v)[COLS], const EpiTile& e, int M, int N) {
    static_assert(COLS == kCePart, "");
    const int64_t row = e.row0 + lane;
    if (e.col0 + COLS > N) {     // columns beyond the tile or the vocabulary
#pragma unroll
      for (int j = 0; j < COLS; ++j)
        if (e.col0 + j >= N) v[j] = 0xff800000u;
    }
#pragma unroll
    for (int q = 0; q < COLS; q += 32)
      while (__any_sync(0xffffffffu, next < q + 32)) {
        const bool mine = next < q + 32;
        const int rel = mine ? next : -1;
        if (mine) {      // on its way while the columns are looked at
          next = at + 1 < end ? a.word[row * a.K + at + 1] - e.col0 : kNoWord;
        }
        float hit = -CUDART_INF_F;      // the second of two equal words finds its column empty
#pragma unroll
        for (int j = q; j < q + 32; ++j)
          if (rel == j) { hit = __uint_as_float(v[j]); v[j] = 0xff800000u; }
        if (mine) { a.picked[row * a.K + at] = hit; ++at; }
      }
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = __uint_as_float(v[i]);
#pragma unroll
    for (int j = 8; j < COLS; j += 16) {
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = j + 8 + i < COLS ? fmaxf(fmaxf(t[i], __uint_as_float(v[j + i])), __uint_as_float(v[j + 8 + i])) : fmaxf(t[i], __uint_as_float(v[j + i]));
    }
    const float m = fmaxf(fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])), fmaxf(fmaxf(t[4], t[5]), fmaxf(t[6], t[7]))) * a.scale;
    const float ref = m == -CUDART_INF_F ? 0.f : m;    // nothing finite here: every term is exp2(-inf) = 0
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = 0.f;
#pragma unroll
    for (int j = 0; j < COLS; j += 8)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] += ex2(fmaf(__uint_as_float(v[j + i]), a.scale, -ref));
    if (row < M) a.stats[(int64_t)e.part * M + row] = make_float2(m, ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7])));
  }
};

// ------------------------------------------------------------------ forward: join
struct DistillJoin {
  const float2* stats;
  const float* picked;
  const int32_t* word;
  const int32_t* slot;
  const float* q;
  const float* lq;
  const int32_t* state;
  float* lse;
  float* diff;        // [T][K], in the caller's order
  float* each;        // loss per token
  float* loss;        // the reduced loss (mean, sum), else nullptr
  const uint4* h;     // rows of `vecs` vectors of 8 elements
  const uint4* W;
  int vecs, bf16;
  int T, K, tiles;
  float scale, tau;
  int mean;
};

// q (log(q / p) - 1 + p / q): the part of the divergence that one word adds.  For d = log(q / p) near 0 by its series d^2 / 2 - d^3 / 6 + ..., whose terms up to d^10 leave
// 2^-24 of it at d = 1/2.
__device__ __forceinline__ float divergence(float q, float p, float d) {
  if (q == 0.f) return p;
  if (fabsf(d) < 0.5f) {
    float s = 1.f / 3628800.f;
    s = fmaf(s, -d, 1.f / 362880.f);
    s = fmaf(s, -d, 1.f / 40320.f);
    s = fmaf(s, -d, 1.f / 5040.f);
    s = fmaf(s, -d, 1.f / 720.f);
    s = fmaf(s, -d, 1.f / 120.f);
    s = fmaf(s, -d, 1.f / 24.f);
    s = fmaf(s, -d, 1.f / 6.f);
    s = fmaf(s, -d, 0.5f);
    return q * d * d * s;
  }
  return fmaf(q, d, p - q);
}

// 2^shift rows per block: their pairs are joined as the cross entropy's, a warp takes a row's words.  Up to 32 WORDS of them per row are in registers, asked for before
// the pairs are joined; more are read where they are needed (WORDS 0).
template <int WORDS>
__global__ void __launch_bounds__(1024) distill_join_kernel(const DistillJoin a, int shift) {
  pdl_begin();
  __shared__ float2 part[1024];
  __shared__ float2 joined[32];
  const int rows = 1 << shift, r = threadIdx.x & (rows - 1), lane = threadIdx.x & 31;
  const auto total_of = [](float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  };
  // A word's score once more, by a warp.  The tensor cores cut sums off towards zero, of products that are all positive, as where a state lies along its word's row of W, a little each time,
  // and more where products are long: of tokens that have settled on a word the score of fp16 was 2.7e-6 of itself too small (512 to 4096 products), so 1e-8 on average and 4e-8 in the root of the
  // mean square, and p - q of a batch with them off by 2 to 4e-6 (24 x 32768 x 1024), so 1e-7.  It takes the reading of a row of h and one of W, 1 to 2 us.  (bf16, whose products have 16 bits for 22:
  // scores 4.7e-7 too small, p - q off by 0.3 to 1.7e-6, left so.)
  const auto score_of = [&](int64_t t, int word) {
    const uint4 *u = a.h + t * a.vecs, *w = a.W + (int64_t)word * a.vecs;
    float z = 0.f;
#pragma unroll 4
    for (int i = lane; i < a.vecs; i += 32) {
      const uint4 p = __ldg(u + i), q = __ldg(w + i);
      const uint32_t pu[4] = {p.x, p.y, p.z, p.w}, qu[4] = {q.x, q.y, q.z, q.w};
      float s[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float ul, uh, wl, wh;
        row_values(pu[k], a.bf16, ul, uh);
        row_values(qu[k], a.bf16, wl, wh);
        s[k] = fmaf(uh, wh, ul * wl);
      }
      z += (s[0] + s[1]) + (s[2] + s[3]);
    }
    return total_of(z);
  };
  struct Word {
    int word, slot;
    bool first;      // of equals
    float z, q, lq;
  };
  for (int64_t first = (int64_t)blockIdx.x << shift; first < a.T; first += (int64_t)gridDim.x << shift) {
    Word held[WORDS ? WORDS : 1];
    const auto word_at = [&](int64_t base, int i) {
      Word w = {kNoWord, 0, false, 0.f, 0.f, 0.f};
      if (i < a.K) {
        w.word = a.word[base + i];
        w.slot = a.slot[base + i];
        w.first = w.word != kNoWord && (i == 0 || a.word[base + i - 1] != w.word);
        w.z = a.picked[base + i];
        w.q = a.q[base + i];
        w.lq = a.lq[base + i];
      }
      return w;
    };
    const auto hold = [&](int w) {
#pragma unroll
      for (int c = 0; c < WORDS; ++c) held[c] = word_at((first + w) * a.K, c * 32 + lane);
    };
    const int w0 = threadIdx.x >> 5;
    if (w0 < rows && first + w0 < a.T) hold(w0);
    join_rows(a.stats, a.T, a.tiles, first, shift, part);
    if ((int)threadIdx.x < rows) joined[r] = joined_row(part, r, shift);
    __syncthreads();
    for (int w = w0; w < rows && first + w < a.T; w += blockDim.x >> 5) {
      if (w != w0) hold(w);
      const int64_t t = first + w, base = t * a.K;
      const auto each_word = [&](const auto& f) {
        if constexpr (WORDS > 0) {
#pragma unroll
          for (int c = 0; c < WORDS; ++c)
            if (c * 32 + lane < a.K) f(c * 32 + lane, held[c]);
        } else {
          for (int i = lane; i < a.K; i += 32) f(i, word_at(base, i));
        }
      };
      const float2 pair = joined[w];
      const int state = a.state[t];
      // The largest score, and which of the teacher's words has it (the first of them).  A NaN counts as the largest: the order is total, and all lanes settle on the same word whatever the scores
      // are.
      const auto order = [](float z) { return z == z ? z : CUDART_INF_F; };
      float own_top = -CUDART_INF_F;
      int own_at = 0, own_word = kNoWord;
      each_word([&](int i, const Word& x) {
        if (x.first && (order(x.z) > order(own_top) || i == 0)) { own_top = x.z; own_at = i; own_word = x.word; }
      });
#pragma unroll
      for (int o = 16; o; o >>= 1) {
        const float z = __shfl_xor_sync(0xffffffffu, own_top, o);
        const int at = __shfl_xor_sync(0xffffffffu, own_at, o), word = __shfl_xor_sync(0xffffffffu, own_word, o);
        if (word != kNoWord && (own_word == kNoWord || order(z) > order(own_top) || (order(z) == order(own_top) && at < own_at))) { own_top = z; own_at = at; own_word = word; }
      }
      const bool kept = state == kKept;
      if (kept && !a.bf16) {      // p is at most this, without the teacher's other words; of p below 1/64 the error does not count
        const float top = fmaxf(pair.x, own_top * a.scale), own = ex2(fmaf(own_top, a.scale, -top));
        if (__any_sync(0xffffffffu, own > (own + pair.y * ex2(pair.x - top)) * 0x1p-6f)) own_top = score_of(t, own_word);      // all lanes or none: it sums over the warp
      }
      const float top = fmaxf(pair.x, own_top * a.scale), ref = top == -CUDART_INF_F ? 0.f : top;
      const float others = pair.y * ex2(pair.x - ref);      // the words that are not the teacher's
      const auto exponent = [&](int i, const Word& x) { return fmaf(i == own_at ? own_top : x.z, a.scale, -ref); };
      float mine = 0.f, q_rest = 0.f, largest = 0.f;         // all of the teacher's but the largest, and that one
      each_word([&](int i, const Word& x) {
        if (!x.first) return;
        const float e = ex2(exponent(i, x));
        if (i == own_at) largest = e;
        else { mine += e; q_rest += x.q; }
      });
      mine = total_of(mine);
      q_rest = total_of(q_rest);
      largest = total_of(largest);
      const float rest = others + mine, total = rest + largest;
      const float bits = log2f(total);
      float sum = 0.f;
      each_word([&](int i, const Word& x) {
        float diff = state == kInvalid ? CUDART_NAN_F : 0.f;
        if (kept && x.word != kNoWord) {
          if (!x.first) return;      // the first of its equals writes
          const float e = exponent(i, x), p = ex2(e) / total;
          const bool most = i == own_at && p > 0.5f;      // of it 1 - p is better known than p, and 1 - q than q
          sum += divergence(x.q, p, most && x.q > 0.5f ? log1pf(-q_rest) + log1pf(rest / largest) : (x.lq - (e - bits)) * kLn2);
          diff = most ? q_rest - rest / total : p - x.q;
          for (int n = i + 1; n < a.K && a.word[base + n] == x.word; ++n) a.diff[base + a.slot[base + n]] = diff;
        }
        a.diff[base + x.slot] = diff;
      });
      sum = total_of(sum);
      if (lane == 0) {
        a.lse[t] = state == kIgnored ? CUDART_INF_F : state == kInvalid ? CUDART_NAN_F : (ref + bits) * kLn2;
        a.each[t] = state == kIgnored ? 0.f : state == kInvalid ? CUDART_NAN_F : a.tau * a.tau * (others / total + sum);
      }
    }
    __syncthreads();      // before the next rows' pairs
  }
  if (a.loss != nullptr && gridDim.x == 1) {
    __syncthreads();
    reduce_losses(a.each, a.T, a.mean, a.loss, [&](int64_t t) { return a.state[t] != kIgnored; });
  }
}

__global__ void __launch_bounds__(1024) distill_reduce_kernel(const DistillJoin a) {
  pdl_begin();
  reduce_losses(a.each, a.T, a.mean, a.loss, [&](int64_t t) { return a.state[t] != kIgnored; });
}

// ------------------------------------------------------------------ gradient
// c p of a tile, to 16 bits: its rounding (at most half a step, 2^-8 of bf16 or 2^-11 of fp16 relative) is independent from entry to entry and moves a gradient about as much as the
// gradient's own rounding to the same type does.  With few tokens, though, a word's row of dW is one or two entries' product and may have all of it.  So up to kSplitTokens
// tokens have two rows of g, the second one for what the first one's rounding has left: the products, bound by W, take 2 to 7 % longer (16 x 65536 x 4096 290 to 296 us, 64 x
// 32768 x 512 51 to 66), and the errors of dh and dW go from 1.4 to 1.0 times those of their own rounding.  (Up to 128 tokens, in a tile of 256 rows: 568 to 693 us at 65 x
// 131072 x 4096.)
constexpr int kSplitTokens = 64;      // two rows of each fill a tile of 128
struct EpiProb {
  static constexpr uint32_t kBytes = 8 * 4096;
  static constexpr bool kSums = true;       // the scores as the forward product made them
  static constexpr bool kLive = false;
  struct Args {
    const float* lse;
    const float* coef;
    float scale;
    int T, bf16;             // rows of T and beyond: the rounding errors of those before
  };
  const Args& a;
  const CUtensorMap* map;
  EpiStage stage;
  int lane;
  bool errors;
  float lse2, c;
  __device__ EpiProb(const Args& args, const CUtensorMap* m, uint32_t base, int w, int l) : a(args), map(m), stage{base + (uint32_t)w * 4096u, l}, lane(l) {}
  __device__ __forceinline__ void before(const EpiTile& e, int M, int) {
    const int row = e.row0 + lane;
    const bool in = row < M;
    errors = row >= a.T;
    const int token = errors ? row - a.T : row;
    c = in ? __ldg(a.coef + token) : 0.f;
    lse2 = in ? __ldg(a.lse + token) * kLog2e : 0.f;
  }
  template <int COLS>
  __device__ __forceinline__ void finish(uint32_t (&v)[COLS], const EpiTile& e, int M, int N) {
    const uint64_t scale = pair_of(a.scale, a.scale), off = pair_of(-lse2, -lse2);
#pragma unroll
    for (int q = 0; q < COLS / 64; ++q) {
      uint32_t p[32];
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        float lo, hi;
        halves_of(fma_pair(pair_of(__uint_as_float(v[q * 64 + 2 * j]), __uint_as_float(v[q * 64 + 2 * j + 1])), scale, off), lo, hi);
        lo = ex2(lo) * c;
        hi = ex2(hi) * c;
        p[j] = pack_16(lo, hi, a.bf16);
        if (errors) {
          float near_lo, near_hi;
          row_values(p[j], a.bf16, near_lo, near_hi);
          p[j] = pack_16(lo - near_lo, hi - near_hi, a.bf16);
        }
        if (c == 0.f) p[j] = 0;     // a token that does not count: exactly nothing, whatever its scores are
      }
      store_part(stage, map, lane, p, e.row0 < M && e.col0 + q * 64 < N, e.col0 + q * 64, e.row0);
    }
  }
};

// c (p - q) over c p where the teacher has words, of the piece [v0, v0 + cols).  Equal words of a token write the same value.
struct PlaceArgs {
  const int64_t* index;
  const float* diff;
  const float* coef;
  uint16_t* g;
  int64_t n, ld;        // T x K
  int64_t v0, cols;
  int64_t errors;       // entries of g from a token's row to the one for its rounding errors, or 0
  int K, bf16;
};

__global__ void __launch_bounds__(256) distill_place_kernel(const PlaceArgs a) {
  pdl_begin();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.n; i += (int64_t)gridDim.x * 256) {
    const int64_t word = __ldg(a.index + i);
    if (word < a.v0 || word >= a.v0 + a.cols) continue;
    const int64_t t = i / a.K, v = word - a.v0;
    const float c = __ldg(a.coef + t), d = __ldg(a.diff + i);
    if (c == 0.f) continue;
    const uint32_t near = pack_16(d * c, 0.f, a.bf16);
    a.g[t * a.ld + v] = (uint16_t)near;
    if (a.errors) {
      float lo, hi;
      row_values(near, a.bf16, lo, hi);
      a.g[a.errors + t * a.ld + v] = (uint16_t)pack_16(d * c - lo, 0.f, a.bf16);
    }
  }
}

// ------------------------------------------------------------------ host side
struct DistillPlan {
  CePlan ce;
  int64_t K;
  int width, parts;           // of the forward product's tiles
  int64_t off_picked, off_each, off_rows, off_word, off_slot, off_q, off_lq, off_start, off_state, forward_bytes;
};

static DistillPlan distill_plan(int64_t T, int64_t V, int64_t D, int64_t K) {
  DistillPlan p = {};
  p.ce = ce_plan(T, V, D);
  p.K = K;
  p.width = tile_width(T, V, ce_rows(T) / 128, 32);
  p.parts = (int)(2 * div_up(V, p.width));
  p.off_picked = up256((int64_t)p.parts * T * 8);
  p.off_each = p.off_picked + up256(T * K * 4);
  p.off_word = p.off_each + up256(T * 4);
  p.off_slot = p.off_word + up256(T * K * 4);
  p.off_q = p.off_slot + up256(T * K * 4);
  p.off_lq = p.off_q + up256(T * K * 4);
  p.off_start = p.off_lq + up256(T * K * 4);
  p.off_state = p.off_start + up256(T * (p.parts + 1) * 2);
  p.off_rows = p.off_state + up256(T * 4);
  p.forward_bytes = p.off_rows + (p.ce.copy ? up256(T * p.ce.ld_h * 2) : 0);
  return p;
}

static CePlan distill_grad_plan(int64_t T, int64_t V, int64_t D) { return ce_plan(T, V, D, T <= kSplitTokens ? 2 : 1); }

static bool distill_sizes(int64_t T, int64_t V, int64_t D, int64_t K) { return K > 0 && K <= kMaxTop && ce_sizes(T, V, D); }

static int check_distill(const void* h, const void* W, const void* index, const void* lse, const void* diff, int64_t T, int64_t V, int64_t D, int64_t K, int32_t dtype,
                         float temperature, int32_t reduction, const void* workspace) {
  if (!h || !W || !index || !lse || !diff || !workspace) { set_error("h, W, top_index, lse, diff and workspace must not be NULL"); return SP_ERR_INVALID_ARG; }
  if (T <= 0 || V <= 0 || D <= 0 || K <= 0) { set_error("T, V, D, K must be positive"); return SP_ERR_INVALID_ARG; }
  if (!distill_sizes(T, V, D, K)) { set_error("sizes too large (K up to %d)", kMaxTop); return SP_ERR_UNSUPPORTED; }
  if (dtype != SP_BF16 && dtype != SP_FP16) { set_error("h and W must both be bf16 or both fp16"); return SP_ERR_UNSUPPORTED; }
  if (!(temperature >= SP_DISTILL_MIN_TEMPERATURE && temperature <= SP_DISTILL_MAX_TEMPERATURE)) { set_error("temperature out of range"); return SP_ERR_INVALID_ARG; }
  if (reduction != SP_REDUCE_NONE && reduction != SP_REDUCE_MEAN && reduction != SP_REDUCE_SUM) { set_error("unknown reduction %d", reduction); return SP_ERR_INVALID_ARG; }
  if ((D % 8) != 0) { set_error("D must be a multiple of 8 (16-byte row pitch)"); return SP_ERR_ALIGNMENT; }
  if ((((uintptr_t)h | (uintptr_t)W | (uintptr_t)workspace) & 15u) || ((uintptr_t)index & 7u) || (((uintptr_t)lse | (uintptr_t)diff) & 3u)) {
    set_error("h, W and workspace must be 16-byte aligned, top_index, lse and diff aligned to their elements");
    return SP_ERR_ALIGNMENT;
  }
  return SP_OK;
}

static int launch_teacher(TeacherArgs& a, cudaStream_t stream) {
  a.size = 32;
  while (a.size < a.K) a.size *= 2;
  const int per_block = a.size <= 256 ? 8 : 1;      // tokens
  const int64_t blocks = div_up(a.T, per_block);
  const unsigned grid = (unsigned)(blocks < 148 * 8 ? blocks : 148 * 8);
  const size_t smem = (size_t)per_block * a.size * 12;
  void (*kern)(TeacherArgs) = teacher_kernel<256, 0>;
  if (a.size == 32) kern = teacher_kernel<32, 1>;
  else if (a.size == 64) kern = teacher_kernel<32, 2>;
  else if (a.size == 128) kern = teacher_kernel<32, 4>;
  else if (a.size == 256) kern = teacher_kernel<32, 8>;
  return launch_pdl("teacher's words", kern, dim3(grid), 256, smem, 1, stream, a);
}

}  // namespace sp

using namespace sp;

using Bytes = unsigned __int128;

extern "C" {

int64_t sp_linear_distill_workspace(int64_t T, int64_t V, int64_t D, int64_t K, int32_t grad) {
  if (!distill_sizes(T, V, D, K)) return -1;
  return grad ? distill_grad_plan(T, V, D).grad_bytes : distill_plan(T, V, D, K).forward_bytes;
}

int sp_linear_distill(const void* h, const void* W, const int64_t* top_index, const void* top_logit, int32_t top_dtype, float* lse, float* diff, float* loss, int64_t T,
                      int64_t V, int64_t D, int64_t K, int32_t dtype, float temperature, int32_t reduction, void* workspace, int64_t workspace_bytes, void* stream_) try {
  int rc = check_distill(h, W, top_index, lse, diff, T, V, D, K, dtype, temperature, reduction, workspace);
  if (rc != SP_OK) return rc;
  if (!loss || !top_logit) { set_error("loss and top_logit must not be NULL"); return SP_ERR_INVALID_ARG; }
  if (top_dtype != SP_BF16 && top_dtype != SP_FP32 && top_dtype != SP_FP16) { set_error("unknown type of top_logit %d", top_dtype); return SP_ERR_UNSUPPORTED; }
  const int logit_bytes = top_dtype == SP_FP32 ? 4 : 2;
  if (((uintptr_t)loss & 3u) || ((uintptr_t)top_logit & (uintptr_t)(logit_bytes - 1))) { set_error("loss and top_logit must be aligned to their elements"); return SP_ERR_ALIGNMENT; }
  const DistillPlan p = distill_plan(T, V, D, K);
  if (workspace_bytes < p.forward_bytes) { set_error("workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)p.forward_bytes); return SP_ERR_INVALID_ARG; }
  const Span spans[] = {{"lse", lse, (Bytes)T * 4}, {"diff", diff, (Bytes)T * K * 4}, {"loss", loss, reduction == SP_REDUCE_NONE ? (Bytes)T * 4 : 4},
                        {"workspace", workspace, (Bytes)p.forward_bytes}, {"h", h, (Bytes)T * D * 2}, {"W", W, (Bytes)V * D * 2}, {"top_index", top_index, (Bytes)T * K * 8},
                        {"top_logit", top_logit, (Bytes)T * K * logit_bytes}};
  rc = refuse_overlaps(spans, 4, 8);
  if (rc != SP_OK) return rc;
  int dev = 0;
  rc = current_device(&dev);
  if (rc != SP_OK) return rc;
  cudaStream_t stream = (cudaStream_t)stream_;
  std::lock_guard<std::mutex> lock(g_ce_mu);
  LibraryState st;
  rc = library_state(nullptr, {}, stream, &st);
  if (rc != SP_OK) return rc;
  char* ws = (char*)workspace;
  const float scale = kLog2e / temperature;
  TeacherArgs ta = {top_index, top_logit, top_dtype, scale, (int32_t*)(ws + p.off_word), (int32_t*)(ws + p.off_slot), (float*)(ws + p.off_q), (float*)(ws + p.off_lq),
                    (uint16_t*)(ws + p.off_start), (int32_t*)(ws + p.off_state), T, (int)V, (int)K, 0, p.parts, p.width};
  if (p.ce.copy) {
    CePrep prep = ce_rows_args(p.ce, h, ws + p.off_rows, nullptr, 0, false);
    rc = launch_ce_rows(p.ce, prep, stream);
    if (rc != SP_OK) return rc;
  }
  rc = launch_teacher(ta, stream);
  if (rc != SP_OK) return rc;
  const EpiDistill::Args ea = {(float2*)ws, (float*)(ws + p.off_picked), ta.word, ta.start, scale, (int)K, p.parts};
  rc = ce_scores<EpiDistill>("vocabulary product", p.ce, p.ce.copy ? ws + p.off_rows : h, p.ce.copy ? p.ce.ld_h : D, W, V, st.status, dtype == SP_BF16, nullptr, ea, stream,
                             nullptr, 2);
  if (rc != SP_OK) return rc;
  DistillJoin j = {};
  j.stats = ea.stats; j.picked = ea.picked; j.word = ta.word; j.slot = ta.slot; j.q = ta.q; j.lq = ta.lq; j.state = ta.state; j.lse = lse; j.diff = diff;
  j.each = reduction == SP_REDUCE_NONE ? loss : (float*)(ws + p.off_each);
  j.loss = reduction == SP_REDUCE_NONE ? nullptr : loss;
  j.h = (const uint4*)h; j.W = (const uint4*)W; j.vecs = (int)(D / 8); j.bf16 = dtype == SP_BF16;
  j.T = (int)T; j.K = (int)K; j.tiles = p.parts; j.scale = scale; j.tau = temperature; j.mean = reduction == SP_REDUCE_MEAN;
  // A warp per token: eight to a block, or all in one block, with the sum of their losses, while 32 warps suffice.  (32 to a block of 8 warps, as the cross entropy has them: 110 x 1216 x 688, 75
  // words, 27 us in this kernel alone, so 10.)
  const bool one = j.loss && T <= 32;
  const int shift = one ? 5 : 3, threads = 32 << shift;
  const unsigned blocks = (unsigned)div_up(T, 1 << shift);
  rc = launch_pdl("join of the row statistics", K <= 32 ? distill_join_kernel<1> : K <= 128 ? distill_join_kernel<4> : distill_join_kernel<0>, dim3(blocks), threads, 0, 1, stream, j, shift);
  if (rc == SP_OK && j.loss && blocks > 1) rc = launch_pdl("sum of the losses", distill_reduce_kernel, dim3(1), 1024, 0, 1, stream, j);
  return rc;
} catch (const std::exception& e) {
  set_error("sp_linear_distill: %s", e.what());
  return SP_ERR_CUDA;
}

int sp_linear_distill_grad(const void* h, const void* W, const int64_t* top_index, const float* lse, const float* diff, const float* grad_loss, void* dh, void* dW, int64_t T,
                           int64_t V, int64_t D, int64_t K, int32_t dtype, float temperature, int32_t reduction, void* workspace, int64_t workspace_bytes, void* stream_) try {
  int rc = check_distill(h, W, top_index, lse, diff, T, V, D, K, dtype, temperature, reduction, workspace);
  if (rc != SP_OK) return rc;
  if (!dh && !dW) { set_error("dh and dW must not both be NULL"); return SP_ERR_INVALID_ARG; }
  if ((((uintptr_t)dh | (uintptr_t)dW) & 15u) || ((uintptr_t)grad_loss & 3u)) { set_error("dh and dW must be 16-byte aligned, grad_loss aligned to its elements"); return SP_ERR_ALIGNMENT; }
  const CePlan p = distill_grad_plan(T, V, D);
  if (workspace_bytes < p.grad_bytes) { set_error("workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)p.grad_bytes); return SP_ERR_INVALID_ARG; }
  const Span spans[] = {{"dh", dh, (Bytes)T * D * 2}, {"dW", dW, (Bytes)V * D * 2}, {"workspace", workspace, (Bytes)p.grad_bytes}, {"h", h, (Bytes)T * D * 2},
                        {"W", W, (Bytes)V * D * 2}, {"top_index", top_index, (Bytes)T * K * 8}, {"lse", lse, (Bytes)T * 4}, {"diff", diff, (Bytes)T * K * 4},
                        {"grad_loss", grad_loss, reduction == SP_REDUCE_NONE ? (Bytes)T * 4 : 4}};
  rc = refuse_overlaps(spans, 3, 9);
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
  float* coef = (float*)ws;
  char *g = ws + p.off_g, *rows = ws + p.off_grad_rows;
  CePrep prep = ce_rows_args(p, h, rows, nullptr, 0, true);
  prep.lse = lse; prep.times = temperature;
  prep.rest = (unsigned long long*)(ws + p.off_rest); prep.count = (int32_t*)(ws + p.off_factor + 4);
  prep.grad = grad_loss; prep.coef = coef; prep.factor = (float*)(ws + p.off_factor); prep.V = (int)V; prep.reduction = reduction; prep.fp16 = !bf16;
  rc = launch_ce_prep(p, prep, stream);
  if (rc != SP_OK) return rc;
  const int64_t n = T * K, blocks = div_up(n, 256);
  const auto scores = [&](int64_t v0, int64_t cols, const void* Wp, const CUtensorMap& tmG) {
    const EpiProb::Args ea = {lse, coef, kLog2e / temperature, (int)T, bf16};
    int rc = ce_scores<EpiProb>("gradient of the scores", p, rows, p.ld_h, Wp, cols, st.status, bf16, &tmG, ea, stream);
    if (rc != SP_OK) return rc;
    const PlaceArgs pa = {top_index, diff, coef, (uint16_t*)g, n, p.ld_g, v0, cols, p.halves > 1 ? T * p.ld_g : 0, (int)K, bf16};
    return launch_pdl("teacher's words", distill_place_kernel, dim3((unsigned)(blocks < 148 * 16 ? blocks : 148 * 16)), 256, 0, 1, stream, pa);
  };
  return ce_gradients(p, W, ws, dh, dW, bf16, st.status, stream, scores);
} catch (const std::exception& e) {
  set_error("sp_linear_distill_grad: %s", e.what());
  return SP_ERR_CUDA;
}

}  // extern "C"
