// Layer norm of the rows of a matrix, and its gradients.
//
//   y = (x - mean) rstd gamma + beta,   mean = sum x / N,   rstd = 1 / sqrt(sum (x - mean)^2 / N + eps)
//   xh = (x - mean) rstd,   u = dy gamma,   dx = rstd (u - sum u / N - xh sum (u xh) / N),   dgamma = sum over rows of dy xh,   dbeta = of dy
//
// Both are bound by HBM: x is read and y written, or x and dy read and dx written, each once.  A row is held in registers from its one read to its
// one write, 32 or (backward, beside the columns' sums) 16 elements per thread, by 1 to 16 warps, beyond a block's width by the CTAs of a cluster, which exchange
// their sums through distributed shared memory.  Each group of warps walks its own rows with the next ones on their way through shared memory.
// The issue slots are what comes next (23 bytes a clock and SM leave 8 instructions for an element of 16 bits, read and written), so all arithmetic is on
// pairs.  Sums are 32-bit and taken in a fixed order: the same bits every time.
#include <float.h>

#include <mutex>

#include "product.cuh"

namespace sp {

constexpr int kLnThreads = 512;                   // of a block: 16 warps in groups
constexpr int kLnMaxCluster = 8;               // portable
constexpr int kLnSums = 2;                        // of a group of warps at once, at most
constexpr int64_t kLnMaxN = 32768;
constexpr int kLnSms = 148;
constexpr int kLnRing = 192 << 10;                // bytes of rows on their way, at most

// How a row lies in the lanes of its group.
enum : int {
  kLnWhole,     // 16-byte units, the rows being whole units at 16-byte addresses
  kLnEdges,     // 16-byte units of memory, the first and the last of a row shared with its neighbours; a group's rows all begin at the same place in their unit
  kLnSingle     // single elements: x, dy and the result do not begin at the same place
};

struct LnArgs {
  const char* x;
  const char* dy;
  const void* gamma;
  const void* beta;
  char* out;                // y, or dx (nullptr: not wanted)
  float* mean;
  float* rstd;
  float* part;              // backward: sums of a CTA cluster's rows, [cluster][dgamma, dbeta][pitch]; nullptr: not wanted, or one cluster has them all
  void* dgamma;             // one cluster: where they go (nullptr: not wanted)
  void* dbeta;
  int64_t M;
  int N;
  int slice;                // columns of one CTA, a multiple of 16
  int clusters;             // launched
  int pitch;
  int w_dtype;
  float eps;
  uint32_t slot;            // bytes of one row's slice in shared memory, for one matrix
};

__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src, int bytes) {      // what lies beyond `bytes` becomes zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ld_shared_16(uint32_t addr, uint32_t (&v)[4]) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr) : "memory");
}

// Element types: 16 bytes to pairs of floats and back; one element.
template <bool BF16>
struct Ln16 {
  static constexpr int kBytes = 2;
  static __device__ __forceinline__ float one(uint32_t bits) {
    float lo, hi;
    halves(bits, lo, hi);
    return lo;
  }
  static __device__ __forceinline__ void halves(uint32_t v, float& lo, float& hi) {
    if constexpr (BF16) {
      lo = __uint_as_float(v << 16); hi = __uint_as_float(v & 0xffff0000u);
    } else {
      const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&v));
      lo = p.x; hi = p.y;
    }
  }
  static __device__ __forceinline__ uint32_t twice_from_shared(uint32_t at) {
    uint16_t b;
    asm volatile("ld.shared.b16 %0, [%1];" : "=h"(b) : "r"(at) : "memory");
    return b * 0x10001u;
  }
  static __device__ __forceinline__ float first(uint32_t v) { return one(v); }
  static __device__ __forceinline__ float from_shared(uint32_t at) { return one(twice_from_shared(at)); }
  static __device__ __forceinline__ void unpack(const uint32_t (&v)[4], uint64_t* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float lo, hi;
      halves(v[i], lo, hi);
      f[i] = pair_of(lo, hi);
    }
  }
  static __device__ __forceinline__ void pack(const uint64_t* f, uint32_t (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float lo, hi;
      halves_of(f[i], lo, hi);
      v[i] = pack_16(lo, hi, BF16);
    }
  }
  static __device__ __forceinline__ void copy_from_shared(char* to, uint32_t at) { *reinterpret_cast<uint16_t*>(to) = (uint16_t)twice_from_shared(at); }
  static __device__ __forceinline__ void store_one(char* at, float f) { *reinterpret_cast<uint16_t*>(at) = (uint16_t)pack_16(f, 0.f, BF16); }
};
struct Ln32 {
  static constexpr int kBytes = 4;
  static __device__ __forceinline__ uint32_t twice_from_shared(uint32_t at) { return ld_shared_32(at); }
  static __device__ __forceinline__ float first(uint32_t v) { return __uint_as_float(v); }
  static __device__ __forceinline__ float from_shared(uint32_t at) { return __uint_as_float(ld_shared_32(at)); }
  static __device__ __forceinline__ void unpack(const uint32_t (&v)[4], uint64_t* f) {
#pragma unroll
    for (int i = 0; i < 2; ++i) f[i] = pair_of(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
  }
  static __device__ __forceinline__ void pack(const uint64_t* f, uint32_t (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float lo, hi;
      halves_of(f[i], lo, hi);
      v[2 * i] = __float_as_uint(lo); v[2 * i + 1] = __float_as_uint(hi);
    }
  }
  static __device__ __forceinline__ void copy_from_shared(char* to, uint32_t at) { *reinterpret_cast<uint32_t*>(to) = ld_shared_32(at); }
  static __device__ __forceinline__ void store_one(char* at, float f) { *reinterpret_cast<float*>(at) = f; }
};

// A group of W warps and its part of a row, PER elements per thread as PER / 2 pairs.
//   Units: a lane's u-th is unit (u W + warp) 32 + lane.  With edges the slice begins `lead` elements inside its first unit; what the first and the last
//   unit hold beside it counts as zeros and is not written.
//   Single elements: a lane's i-th is column (i W + warp) 32 + lane.
template <class E, int W, int PER, int MODE>
struct LnGroup {
  static constexpr int kGroups = kLnThreads / 32 / W, kGroupThreads = 32 * W, kPairs = PER / 2;
  static constexpr bool kUnits = MODE != kLnSingle;
  static constexpr int kElems = kUnits ? 16 / E::kBytes : 1;           // next to each other
  static constexpr int kChunks = PER / kElems;                         // such stretches
  static constexpr int kStep = kUnits ? 1 : 2;                         // chunks that are done together, kWide pairs
  static constexpr int kWide = kStep * kElems / 2;
  int lane, wg, group, tid;
  int rank, ranks;             // of the CTA in its cluster
  int cols, lead;              // of the slice
  // Rows with edges: which of the warp's units the slice has in part only (bit i: among the i-th ones); shared memory of the warp: what of its first and last such unit is
  // the slice's (all bits of an element set), and the two on their way out; the element of them that this lane writes, its place in the slice's row or -1.
  uint32_t edges, rim;
  int rim_at;
  uint32_t red, far;           // shared memory: sums of warps, sums of CTAs (two of each, used in turn)
  uint32_t parity;

  __device__ __forceinline__ LnGroup(const LnArgs& a, uint32_t red_) : lead(0), edges(0), rim_at(-1), red(red_), parity(0) {
    const int warp = threadIdx.x >> 5;
    lane = threadIdx.x & 31;
    wg = warp % W; group = warp / W; tid = threadIdx.x % kGroupThreads;
    ranks = W == 16 ? (int)cluster_nctarank() : 1;
    rank = W == 16 ? (int)cluster_ctarank() : 0;
    cols = max(0, min(a.slice, a.N - rank * a.slice));
    far = red + 2 * 16 * 4 * kLnSums;
    rim = far + 2 * kLnMaxCluster * 4 * kLnSums + warp * 64;
    if (W == 16 && ranks > 1) unit_sync<2>();      // every CTA of the cluster is there before one writes to its shared memory
  }
  // `m`: address modulo 16 of the group's rows
  __device__ __forceinline__ void begin_at(int m) {
    if constexpr (MODE == kLnEdges) {
      lead = m / E::kBytes;
#pragma unroll
      for (int i = 0; i < kChunks; ++i)
        if (__any_sync(0xffffffffu, has(i) && !full(i))) edges |= 1u << i;
      const int last = (lead + cols - 1) / kElems, e = lane & 7;      // lanes 0 to 7: the elements of unit 0, 8 to 15: of the last one
      const int unit = lane < 8 ? 0 : last, c = unit * kElems - lead + e;
      const bool mine = wg == unit / 32 % W && (lane < 8 || last > 0) && c >= 0 && c < cols;
      if (lane < 16 && e < kElems) {
        if constexpr (E::kBytes == 2) asm volatile("st.shared.b16 [%0], %1;" ::"r"(rim + lane * 2), "h"((uint16_t)(mine ? 0xffff : 0)) : "memory");
        else asm volatile("st.shared.b32 [%0], %1;" ::"r"(rim + (lane < 8 ? 0 : 16) + e * 4), "r"(mine ? 0xffffffffu : 0u) : "memory");
        if (mine && (unit * kElems - lead < 0 || unit * kElems - lead + kElems > cols)) rim_at = c * E::kBytes;      // in a unit that is not whole
      }
      __syncwarp();
    }
  }
  // A branch that is taken by few warps and, for the compiler, not to be made part of the straight line.
  __device__ __forceinline__ bool edge(int i) const {
    if constexpr (MODE != kLnEdges) return false;
    if ((edges >> i & 1u) == 0) return false;
    __syncwarp();
    return true;
  }
  __device__ __forceinline__ int chunk(int i) const { return (i * W + wg) * 32 + lane; }
  __device__ __forceinline__ int column(int i) const { return MODE == kLnEdges ? chunk(i) * kElems - lead : chunk(i) * kElems; }
  __device__ __forceinline__ bool any(int i) const { return (i * W + wg) * 32 * kElems < cols + (MODE == kLnEdges ? lead : 0); }      // of the warp's i-th chunks
  __device__ __forceinline__ bool has(int i) const { return column(i) < cols; }
  __device__ __forceinline__ bool full(int i) const { return MODE != kLnEdges || (column(i) >= 0 && column(i) + kElems <= cols); }
  __device__ __forceinline__ void sync() const {
    if constexpr (W == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(kGroupThreads) : "memory");
  }

  // A row's slice on its way to shared memory, as whole 16-byte units of global memory.  [lo, hi): the matrix, outside of which nothing is read.
  __device__ __forceinline__ void fetch(uint32_t dst, const char* row, const char* lo, const char* hi) const {
    if constexpr (MODE == kLnWhole) {      // the units a lane will read itself
#pragma unroll
      for (int u = 0; u < kChunks; ++u)
        if (has(u)) cp_async_16(dst + chunk(u) * 16, row + chunk(u) * 16, 16);
    } else if (MODE == kLnEdges && row - lead * E::kBytes >= lo && row + cols * E::kBytes + 15 <= hi) {
      row -= lead * E::kBytes;
#pragma unroll
      for (int u = 0; u < kChunks; ++u)
        if (has(u)) cp_async_16(dst + chunk(u) * 16, row + chunk(u) * 16, 16);
    } else {
      const int m = (int)((uintptr_t)row & 15u), n = (m + cols * E::kBytes + 15) >> 4;
      const auto unit = [&](int j) {
        const char* p = row - m + 16 * j;
        if (p >= lo) cp_async_16(dst + 16 * j, p, (int)min((int64_t)16, (int64_t)(hi - p)));
        else      // the matrix starts inside this unit
          for (int b = 0; b < 16; b += E::kBytes)
            if (p + b >= lo && p + b < hi) {
              if constexpr (E::kBytes == 4) asm volatile("st.shared.b32 [%0], %1;" ::"r"(dst + 16 * j + b), "r"(*reinterpret_cast<const uint32_t*>(p + b)) : "memory");
              else asm volatile("st.shared.b16 [%0], %1;" ::"r"(dst + 16 * j + b), "h"(*reinterpret_cast<const uint16_t*>(p + b)) : "memory");
            }
      };
      if constexpr (kUnits) {
        for (int u = 0; u < kChunks; ++u)
          if (chunk(u) < n) unit(chunk(u));
      } else {
        for (int j = tid; j < n; j += kGroupThreads) unit(j);
      }
    }
  }
  // A lane's pairs of chunk i from shared memory, `m`: the row's address modulo 16.  Columns outside the slice become zeros.
  __device__ __forceinline__ void take(uint32_t src, int i, int m, uint64_t* f) const {
    int none;
    float filler;
    take<false>(src, i, m, f, none, filler);
  }
  // FILL: what an edge holds beside the slice becomes the slice's own first element there, `extra` times `filler`, which the sums are relieved of again.  (It
  // is an element of the row, at most sqrt(N) deviations from the mean, so at most 15 rows' worth of squares are added and taken away.)
  template <bool FILL>
  __device__ __forceinline__ void take(uint32_t src, int i, int m, uint64_t* f, int& extra, float& filler) const {
    if constexpr (kUnits) {
      uint32_t v[4] = {0u, 0u, 0u, 0u};
      if (has(i)) ld_shared_16(src + 16 * chunk(i), v);
      if (edge(i) && has(i) && !full(i)) {
        const bool begin = chunk(i) == 0;
        uint32_t k[4], fill = 0;
        ld_shared_16(rim + (begin ? 0 : 16), k);
        if constexpr (FILL) {
          fill = E::twice_from_shared(src + 16 * chunk(i) + (begin ? lead * E::kBytes : 0));
          filler = E::first(fill);
          extra = kElems - min(kElems, cols - column(i)) + max(0, -column(i));
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) v[w] = (v[w] & k[w]) | (fill & ~k[w]);
      }
      E::unpack(v, f);
    } else {
      const uint32_t at = src + m + column(i) * E::kBytes;
      f[0] = pair_of(has(i) ? E::from_shared(at) : 0.f, has(i + 1) ? E::from_shared(at + 32 * W * E::kBytes) : 0.f);
    }
  }
  // f - v in the columns that the lane holds, else 0 as before
  __device__ __forceinline__ void subtract(int i, float v, uint64_t* f) const {
    if constexpr (kUnits) {
      const float m = has(i) ? -v : 0.f;
#pragma unroll
      for (int k = 0; k < kWide; ++k) f[k] = add_pair(f[k], pair_of(m, m));
    } else {
      f[0] = add_pair(f[0], pair_of(has(i) ? -v : 0.f, has(i + 1) ? -v : 0.f));
    }
  }
  __device__ __forceinline__ void put(char* row, int i, const uint64_t* f) const {
    if constexpr (kUnits) {
      char* at = row + column(i) * E::kBytes;
      uint32_t v[4];
      E::pack(f, v);
      if (has(i) && full(i)) *reinterpret_cast<uint4*>(at) = make_uint4(v[0], v[1], v[2], v[3]);
      if (edge(i) && has(i) && !full(i)) st_shared_16(rim + (chunk(i) == 0 ? 32 : 48), v[0], v[1], v[2], v[3]);
    } else {
      float lo, hi;
      halves_of(f[0], lo, hi);
      char* at = row + column(i) * E::kBytes;
      if (has(i)) E::store_one(at, lo);
      if (has(i + 1)) E::store_one(at + 32 * W * E::kBytes, hi);
    }
  }
  // After the row's put: what the edges have of it, an element per lane.
  __device__ __forceinline__ void put_rim(char* row) const {
    if constexpr (MODE == kLnEdges) {
      if (edges == 0) return;
      __syncwarp();
      if (rim_at >= 0) E::copy_from_shared(row + rim_at, rim + 32 + (lane < 8 ? 0 : 16) + (lane & 7) * E::kBytes);
      __syncwarp();
    }
  }
  // gamma or beta of this lane's columns.  All of a kind of loads are in flight together, 16 bytes each where they can be: a block starts with them.
  __device__ __forceinline__ void weights(const void* w, int dtype, int col0, float none, uint64_t* f) const {
    if (w == nullptr) {
#pragma unroll
      for (int k = 0; k < kPairs; ++k) f[k] = pair_of(none, none);
    } else if (dtype == SP_FP32) {
      const float* p = (const float*)w + col0;
      if (MODE == kLnWhole && ((uintptr_t)w & 15u) == 0) {
#pragma unroll
        for (int i = 0; i < kChunks; ++i)
#pragma unroll
          for (int q = 0; q < kElems / 4; ++q) {
            const float4 v = has(i) ? __ldg(reinterpret_cast<const float4*>(p + column(i)) + q) : make_float4(none, none, none, none);
            f[i * kElems / 2 + 2 * q] = pair_of(v.x, v.y);
            f[i * kElems / 2 + 2 * q + 1] = pair_of(v.z, v.w);
          }
      } else {
        one_by_one(f, none, [&](int c) { return __ldg(p + c); });
      }
    } else {      // the rows' type
      if constexpr (E::kBytes == 2) {
        const uint16_t* p = (const uint16_t*)w + col0;
        if (MODE == kLnWhole && ((uintptr_t)w & 15u) == 0) {
#pragma unroll
          for (int i = 0; i < kChunks; ++i) {
            const uint4 q = has(i) ? __ldg(reinterpret_cast<const uint4*>(p + column(i))) : make_uint4(0u, 0u, 0u, 0u);
            const uint32_t v[4] = {q.x, q.y, q.z, q.w};
            if constexpr (kUnits) E::unpack(v, f + i * kElems / 2);
          }
        } else {
          one_by_one(f, none, [&](int c) { return E::one(__ldg(p + c)); });
        }
      }
    }
  }
  template <class Load>
  __device__ __forceinline__ void one_by_one(uint64_t* f, float none, const Load& load) const {
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
      float v[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int e = 2 * k + h, c = column(e / kElems) + e % kElems;
        v[h] = c >= 0 && c < cols ? load(c) : none;
      }
      f[k] = pair_of(v[0], v[1]);
    }
  }

  // n sums over the row (n: a power of two): lanes, warps, CTAs, in this order.  Of several sums every step of the lanes' leaves half to each half of the lanes.
  template <int n>
  __device__ __forceinline__ void sum(float* s) {
    int o = 16;
#pragma unroll
    for (int left = n / 2; left; left /= 2, o /= 2) {
      const bool upper = lane & o;
#pragma unroll
      for (int j = 0; j < left; ++j) {
        const float give = upper ? s[j] : s[j + left], keep = upper ? s[j + left] : s[j];
        s[j] = keep + __shfl_xor_sync(0xffffffffu, give, o);
      }
    }
#pragma unroll
    for (; o; o /= 2) s[0] += __shfl_xor_sync(0xffffffffu, s[0], o);
    constexpr int kLanes = 32 / n;      // lanes [j kLanes, (j + 1) kLanes) have sum j
    if constexpr (W == 1) {
      const float all = s[0];
#pragma unroll
      for (int j = 0; j < n; ++j) s[j] = n == 1 ? all : __shfl_sync(0xffffffffu, all, j * kLanes);
    } else {
      const uint32_t at = red + (parity * 16 + group * W) * (4 * kLnSums);      // [sum][warp]
      if (lane % kLanes == 0) asm volatile("st.shared.f32 [%0], %1;" ::"r"(at + (lane / kLanes * W + wg) * 4), "f"(s[0]) : "memory");
      sync();
      if constexpr (W == 16) {      // a lane per warp and sum: an instruction each for what one thread would do 16 times (2048 x 16384 fp32 58.9 to 53 us; of 8 warps the shuffles take longer)
        float v = __uint_as_float(ld_shared_32(at + lane % (n * W) * 4));
#pragma unroll
        for (int o = W / 2; o; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
#pragma unroll
        for (int j = 0; j < n; ++j) s[j] = n == 1 ? v : __shfl_sync(0xffffffffu, v, j * W);
      } else if constexpr (W >= 4) {
#pragma unroll
        for (int j = 0; j < n; ++j) {
          s[j] = 0.f;
#pragma unroll
          for (int i = 0; i < W / 4; ++i) {
            uint32_t v[4];
            ld_shared_16(at + j * W * 4 + i * 16, v);
            s[j] += (__uint_as_float(v[0]) + __uint_as_float(v[1])) + (__uint_as_float(v[2]) + __uint_as_float(v[3]));
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < n; ++j) {
          float p, q;
          asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(p), "=f"(q) : "r"(at + j * 8) : "memory");
          s[j] = p + q;
        }
      }
      if constexpr (W == 16)
        if (ranks > 1) {
          const uint32_t here = far + parity * kLnMaxCluster * 4 * kLnSums;      // [CTA][sum]
          if (tid < ranks) {
#pragma unroll
            for (int j = 0; j < n; ++j) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(mapa(here + (rank * kLnSums + j) * 4, tid)), "f"(s[j]) : "memory");
          }
          unit_sync<2>();      // all threads of the cluster
#pragma unroll
          for (int j = 0; j < n; ++j) s[j] = 0.f;
          for (int i = 0; i < ranks; ++i)
#pragma unroll
            for (int j = 0; j < n; ++j) s[j] += __uint_as_float(ld_shared_32(here + (i * kLnSums + j) * 4));
        }
      parity ^= 1u;
    }
  }
};

// Bytes of shared memory beside the rows: sums of warps and of CTAs, two of each, and the warps' rims.
constexpr uint32_t kLnRedBytes = 2 * (16 + kLnMaxCluster) * 4 * kLnSums + 16 * 64;

// Batches of `rows` rows' slices on their way.
template <class E, int PER, int ROWS>
constexpr int kLnDepth = kLnRing / (kLnThreads * PER * E::kBytes * ROWS) < 4 ? kLnRing / (kLnThreads * PER * E::kBytes * ROWS) : 4;

// 1 / sqrt(v): the hardware's, which is good to two steps, and one step of Newton's method.
__device__ __forceinline__ float ln_rsqrt(float v) {
  const float r = rsqrtf(v), s = r * fmaf(-0.5f * v * r, r, 1.5f);
  return s == s ? s : r;      // 0 and infinity
}

__device__ __forceinline__ float halves_sum(uint64_t s) {
  float lo, hi;
  halves_of(s, lo, hi);
  return lo + hi;
}

template <class E, int W, int PER, int MODE>
__global__ void __launch_bounds__(kLnThreads, 1) layernorm_kernel(const LnArgs a) {
  extern __shared__ __align__(16) uint8_t ln_smem[];
  using G = LnGroup<E, W, PER, MODE>;
  constexpr int D = kLnDepth<E, PER, 1>, P = G::kWide;
  const uint32_t base = smem_u32(ln_smem);
  G g(a, base);
  const uint32_t ring = base + kLnRedBytes + g.group * D * a.slot;
  const uint32_t total = a.clusters * G::kGroups, last = (uint32_t)a.M - 1;      // unsigned: beyond the last row they may pass 2^31
  const int64_t pitch = (int64_t)a.N * E::kBytes, hop = (int64_t)total * pitch, all = a.M * pitch;
  uint32_t row = blockIdx.x / g.ranks * G::kGroups + g.group;
  int64_t here = (int64_t)row * pitch + (int64_t)g.rank * a.slice * E::kBytes, next = here;
  g.begin_at((int)((uintptr_t)(a.x + here) & 15u));
  pdl_begin();
  const auto fetch = [&](uint32_t at, uint32_t r) {
    if (r <= last) g.fetch(at, a.x + next, a.x, a.x + all);
    next += hop;
    cp_async_commit();
  };
  uint32_t ahead = row;
#pragma unroll
  for (int i = 0; i < D; ++i, ahead += total) fetch(ring + i * a.slot, ahead);
  uint64_t gamma[G::kPairs], beta[G::kPairs];
  g.weights(a.gamma, a.w_dtype, g.rank * a.slice, 1.f, gamma);
  g.weights(a.beta, a.w_dtype, g.rank * a.slice, 0.f, beta);
  const float inv = 1.f / (float)a.N;
  uint32_t at = ring;
  for (; row <= last; row += total, here += hop) {
    cp_async_wait<D - 1>();
    if constexpr (MODE == kLnSingle) g.sync();      // the others' copies
    uint64_t x[G::kPairs], s2[2] = {0, 0}, v2[2] = {0, 0};
    float filler[2] = {0.f, 0.f};
    int extra[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < G::kChunks; i += G::kStep)
      if (g.any(i)) {
        uint64_t* f = x + i * G::kElems / 2;
        g.template take<true>(at, i, (int)((uintptr_t)(a.x + here) & 15u), f, extra[i > 0], filler[i > 0]);      // at most two units of a lane are edges
#pragma unroll
        for (int k = 0; k < P; ++k) s2[k & 1] = add_pair(s2[k & 1], f[k]);
      }
    float s = halves_sum(add_pair(s2[0], s2[1]));
    if constexpr (MODE == kLnEdges) s -= extra[0] * filler[0] + extra[1] * filler[1];
    g.template sum<1>(&s);
    fetch(at, ahead);
    ahead += total;
    at = at + a.slot == ring + D * a.slot ? ring : at + a.slot;
    // The differences' own sum corrects what the rounded mean leaves: of rows whose mean is a thousand deviations, too, variance and y keep their digits.
    const float about = s * inv;
    s2[0] = s2[1] = 0;
#pragma unroll
    for (int i = 0; i < G::kChunks; i += G::kStep)
      if (g.any(i)) {
        uint64_t* f = x + i * G::kElems / 2;
        g.subtract(i, about, f);
#pragma unroll
        for (int k = 0; k < P; ++k) {
          s2[k & 1] = add_pair(s2[k & 1], f[k]);
          v2[k & 1] = fma_pair(f[k], f[k], v2[k & 1]);
        }
      }
    float sv[2] = {halves_sum(add_pair(s2[0], s2[1])), halves_sum(add_pair(v2[0], v2[1]))};
    if constexpr (MODE == kLnEdges)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const float e = filler[q] - about;
        sv[0] -= extra[q] * e;
        sv[1] -= extra[q] * e * e;
      }
    g.template sum<2>(sv);
    const float off = sv[0] * inv, var = fmaf(-off, off, sv[1] * inv), rstd = ln_rsqrt((var < 0.f ? 0.f : var) + a.eps);
    if (g.tid == 0 && g.rank == 0) {
      if (a.mean != nullptr) a.mean[row] = about + off;
      if (a.rstd != nullptr) a.rstd[row] = rstd;
    }
    const uint64_t scale = pair_of(rstd, rstd), minus = pair_of(-off, -off);
#pragma unroll
    for (int i = 0; i < G::kChunks; i += G::kStep)
      if (g.any(i)) {
        const int o = i * G::kElems / 2;
#pragma unroll
        for (int k = o; k < o + P; ++k) x[k] = fma_pair(mul_pair(add_pair(x[k], minus), scale), gamma[k], beta[k]);
        g.put(a.out + here, i, x + o);
      }
    g.put_rim(a.out + here);
  }
}

__device__ __forceinline__ void store_weight(void* out, int dtype, int col, float s) {
  if (out == nullptr) return;
  if (dtype == SP_FP32) ((float*)out)[col] = s;
  else ((uint16_t*)out)[col] = (uint16_t)pack_16(s, 0.f, dtype == SP_BF16);
}

// (A row finished beside the sums of the next, between the same two barriers, its x and dy read twice from shared memory: 16384 x 4096 86 us, so 75. Instructions bound it.)
template <class E, int W, int PER, int MODE>
__global__ void __launch_bounds__(kLnThreads, 1) layernorm_grad_kernel(const LnArgs a) {
  extern __shared__ __align__(16) uint8_t ln_smem[];
  using G = LnGroup<E, W, PER, MODE>;
  constexpr int D = kLnDepth<E, PER, 2>, P = G::kWide;
  const uint32_t base = smem_u32(ln_smem);
  G g(a, base);
  const uint32_t ring = base + kLnRedBytes + g.group * D * 2 * a.slot, batch = 2 * a.slot;
  const uint32_t total = a.clusters * G::kGroups, last = (uint32_t)a.M - 1;
  const int col0 = g.rank * a.slice;
  const int64_t pitch = (int64_t)a.N * E::kBytes, hop = (int64_t)total * pitch, all = a.M * pitch;
  uint32_t row = blockIdx.x / g.ranks * G::kGroups + g.group;
  int64_t here = (int64_t)row * pitch + (int64_t)col0 * E::kBytes, next = here;
  g.begin_at((int)((uintptr_t)(a.x + here) & 15u));
  pdl_begin();
  const auto fetch = [&](uint32_t at, uint32_t r) {
    if (r <= last) {
      g.fetch(at, a.x + next, a.x, a.x + all);
      g.fetch(at + a.slot, a.dy + next, a.dy, a.dy + all);
    }
    next += hop;
    cp_async_commit();
  };
  uint32_t ahead = row;
#pragma unroll
  for (int i = 0; i < D; ++i, ahead += total) fetch(ring + i * batch, ahead);
  uint64_t gamma[G::kPairs], dg[G::kPairs], db[G::kPairs];
  g.weights(a.gamma, a.w_dtype, col0, 1.f, gamma);
#pragma unroll
  for (int k = 0; k < G::kPairs; ++k) dg[k] = db[k] = 0;
  const float inv = 1.f / (float)a.N;
  float mean = 0.f, rstd = 0.f;
  if (row <= last) { mean = __ldg(a.mean + row); rstd = __ldg(a.rstd + row); }
  uint32_t at = ring;
  for (; row <= last; row += total, here += hop) {
    float next_mean = 0.f, next_rstd = 0.f;
    if (row + total <= last) { next_mean = __ldg(a.mean + row + total); next_rstd = __ldg(a.rstd + row + total); }
    cp_async_wait<D - 1>();
    if constexpr (MODE == kLnSingle) g.sync();
    uint64_t x[G::kPairs], y[G::kPairs], s2[2] = {0, 0}, t2[2] = {0, 0};      // xh and u
    const uint64_t minus = pair_of(-mean, -mean), scale = pair_of(rstd, rstd);
#pragma unroll
    for (int i = 0; i < G::kChunks; i += G::kStep)
      if (g.any(i)) {
        const int o = i * G::kElems / 2;
        g.take(at, i, (int)((uintptr_t)(a.x + here) & 15u), x + o);
        g.take(at + a.slot, i, (int)((uintptr_t)(a.dy + here) & 15u), y + o);      // 0 outside the slice, and with it all that x adds there
#pragma unroll
        for (int k = o; k < o + P; ++k) {
          x[k] = mul_pair(add_pair(x[k], minus), scale);
          dg[k] = fma_pair(y[k], x[k], dg[k]);
          db[k] = add_pair(db[k], y[k]);
          y[k] = mul_pair(y[k], gamma[k]);
          s2[k & 1] = add_pair(s2[k & 1], y[k]);
          t2[k & 1] = fma_pair(y[k], x[k], t2[k & 1]);
        }
      }
    float st[2] = {halves_sum(add_pair(s2[0], s2[1])), halves_sum(add_pair(t2[0], t2[1]))};
    g.template sum<2>(st);
    fetch(at, ahead);
    ahead += total;
    at = at + batch == ring + D * batch ? ring : at + batch;
    if (a.out != nullptr) {
      const uint64_t c1 = pair_of(-st[0] * inv, -st[0] * inv), c2 = pair_of(-st[1] * inv, -st[1] * inv);
#pragma unroll
      for (int i = 0; i < G::kChunks; i += G::kStep)
        if (g.any(i)) {
          uint64_t* f = x + i * G::kElems / 2;
#pragma unroll
          for (int k = 0; k < P; ++k) f[k] = mul_pair(scale, fma_pair(c2, f[k], add_pair(y[i * G::kElems / 2 + k], c1)));
          g.put(a.out + here, i, f);
        }
      g.put_rim(a.out + here);
    }
    mean = next_mean; rstd = next_rstd;
  }
  if (a.part == nullptr && a.dgamma == nullptr && a.dbeta == nullptr) return;
  // the groups' sums to one, in their order
  float* all_groups = reinterpret_cast<float*>(ln_smem + kLnRedBytes);
  cp_async_wait<0>();
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const auto out = [&](int c, float s) {
      if (a.part != nullptr) a.part[((int64_t)(blockIdx.x / g.ranks) * 2 + w) * a.pitch + col0 + c] = s;
      else store_weight(w == 0 ? a.dgamma : a.dbeta, a.w_dtype, col0 + c, s);
    };
    if constexpr (G::kGroups > 1) __syncthreads();
#pragma unroll
    for (int k = 0; k < G::kPairs; ++k) {
      float v[2];
      halves_of(w == 0 ? dg[k] : db[k], v[0], v[1]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int e = 2 * k + h, c = g.column(e / G::kElems) + e % G::kElems;
        if (c >= 0 && c < g.cols) {
          if constexpr (G::kGroups > 1) all_groups[g.group * a.pitch + c] = v[h];
          else out(c, v[h]);
        }
      }
    }
    if constexpr (G::kGroups > 1) {
      __syncthreads();
      for (int c = threadIdx.x; c < a.N; c += kLnThreads) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < G::kGroups; ++i) s += all_groups[i * a.pitch + c];
        out(c, s);
      }
    }
  }
}

// dgamma (blockIdx.y 0) and dbeta (1) from the clusters' sums, in a fixed order: 16 rows of 32 columns side by side.
__global__ void __launch_bounds__(512) layernorm_weights_kernel(const float* part, int rows, int pitch, int N, int dtype, void* dgamma, void* dbeta) {
  pdl_begin();
  __shared__ float sums[16][32];
  void* out = blockIdx.y == 0 ? dgamma : dbeta;
  if (out == nullptr) return;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (col < N) {
    const float* p = part + (int64_t)blockIdx.y * pitch + col;
#pragma unroll 8
    for (int i = w; i < rows; i += 16) s += __ldcg(p + (int64_t)i * 2 * pitch);
  }
  sums[w][lane] = s;
  __syncthreads();
  if (w != 0 || col >= N) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) s += sums[i][lane];
  store_weight(out, dtype, col, s);
}

// ------------------------------------------------------------------ host side
static std::mutex g_ln_mu;   // per-kernel set-up is done under it

static int ln_bytes(int32_t dtype) { return dtype == SP_FP32 ? 4 : 2; }

// What follows from the sizes and from how rows lie in the lanes.
struct LnPlan {
  int mode, per;            // elements per thread
  int ranks, slice;         // CTAs that share a row, columns of one
  int warps, clusters;      // of a group; launched
  int pitch;
};

static LnPlan ln_plan(int64_t M, int64_t N, int elt, bool grad, int mode) {
  LnPlan p = {};
  p.mode = mode;
  const int edge = mode == kLnEdges ? 16 / elt : 0;      // of elements before the slice, at most one unit less
  // Forward 32 elements per thread: per row half the warps, with what a warp costs beside its elements (8192 x 4096 bf16: 25.9 us, with 16: 31.9).  Rows with edges, whose bookkeeping wants
  // registers, 16 where these are well filled: 5001 x 2035 fp16 16.4 us, with 32: 20.3; 16384 x 1031, half filled, 41.4 and 33.7.
  const auto width = [&](int per) {
    for (p.ranks = 1;; p.ranks *= 2) {
      p.slice = (int)(((N + p.ranks - 1) / p.ranks + 15) / 16 * 16);
      if ((N < p.slice ? N : p.slice) + edge <= kLnThreads * per) break;
    }
    p.per = per;
    const int w = (int)(N < p.slice ? N : p.slice) + edge;
    for (p.warps = 1; p.warps * 32 * per < w; p.warps *= 2) {}
    return 4 * w > 3 * p.warps * 32 * per;      // more than three quarters used
  };
  if (grad) width(16);
  else if (mode != kLnEdges || !width(16) || p.ranks > 1) width(32);
  if (mode == kLnSingle || p.ranks > 1) p.warps = 16;
  const int groups = kLnThreads / 32 / p.warps;
  // One block per SM; backward, whose blocks each leave a row of sums, at least two rows for every group, and one block for up to four.
  const int64_t most = kLnSms / p.ranks, rows = grad ? (M <= 4 * groups ? 4 : 2) : 1, want = (M + groups * rows - 1) / (groups * rows);
  p.clusters = (int)(want < most ? want : most);
  if (mode == kLnEdges && (int64_t)p.clusters * groups < M) {      // a group's rows are a multiple of 16 bytes apart
    int apart = 1;
    while (((int64_t)apart * groups * N * elt) % 16) apart *= 2;
    p.clusters = p.clusters < apart ? apart : p.clusters / apart * apart;
  }
  p.pitch = (int)((N + 15) / 16 * 16);
  return p;
}

template <class E, int W, int PER, int MODE>
static int ln_launch(bool grad, const LnArgs& a, const LnPlan& p, cudaStream_t stream) {
  const int slots = grad ? 2 * kLnDepth<E, PER, 2> : kLnDepth<E, PER, 1>;
  const uint32_t smem = kLnRedBytes + (uint32_t)(kLnThreads / 32 / W * slots) * a.slot;
  void (*kern)(LnArgs) = layernorm_kernel<E, W, PER, MODE>;
  if constexpr (PER == 16)
    if (grad) kern = layernorm_grad_kernel<E, W, PER, MODE>;
  static uint64_t configured[2] = {0, 0};
  if (first_use_on_this_device(configured[grad])) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kProdSmemLimit);
    if (e != cudaSuccess) { configured[grad] = 0; set_error("cudaFuncSetAttribute failed: %s", cudaGetErrorString(e)); return SP_ERR_CUDA; }
  }
  return launch_pdl(grad ? "layer norm gradient" : "layer norm", kern, dim3((unsigned)(p.clusters * p.ranks)), kLnThreads, smem, p.ranks, stream, a);
}

template <class E, int PER, int MODE>
static int ln_warps(bool grad, const LnArgs& a, const LnPlan& p, cudaStream_t stream) {
  if constexpr (MODE != kLnSingle) {
    switch (p.warps) {
      case 1: return ln_launch<E, 1, PER, MODE>(grad, a, p, stream);
      case 2: return ln_launch<E, 2, PER, MODE>(grad, a, p, stream);
      case 4: return ln_launch<E, 4, PER, MODE>(grad, a, p, stream);
      case 8: return ln_launch<E, 8, PER, MODE>(grad, a, p, stream);
    }
  }
  return ln_launch<E, 16, PER, MODE>(grad, a, p, stream);
}

template <class E>
static int ln_run(bool grad, const LnArgs& a, const LnPlan& p, cudaStream_t stream) {
  switch (p.mode) {
    case kLnWhole: return p.per == 16 ? ln_warps<E, 16, kLnWhole>(grad, a, p, stream) : ln_warps<E, 32, kLnWhole>(grad, a, p, stream);
    case kLnEdges: return p.per == 16 ? ln_warps<E, 16, kLnEdges>(grad, a, p, stream) : ln_warps<E, 32, kLnEdges>(grad, a, p, stream);
    default: return p.per == 16 ? ln_warps<E, 16, kLnSingle>(grad, a, p, stream) : ln_warps<E, 32, kLnSingle>(grad, a, p, stream);
  }
}

// How the rows lie.
static int ln_mode(const LnArgs& a, int elt) {
  const uintptr_t x = (uintptr_t)a.x, dy = a.dy ? (uintptr_t)a.dy : x, out = a.out ? (uintptr_t)a.out : x;
  if (((x ^ dy) | (x ^ out)) & 15u) return kLnSingle;
  return (x & 15u) == 0 && (int64_t)a.N * elt % 16 == 0 ? kLnWhole : kLnEdges;
}

static int ln_any(bool grad, LnArgs& a, int32_t dtype, cudaStream_t stream, const LnPlan& p) {
  a.slice = p.slice; a.clusters = p.clusters; a.pitch = p.pitch;
  a.slot = (uint32_t)p.slice * ln_bytes(dtype) + 16;
  std::lock_guard<std::mutex> lock(g_ln_mu);
  if (dtype == SP_BF16) return ln_run<Ln16<true>>(grad, a, p, stream);
  if (dtype == SP_FP16) return ln_run<Ln16<false>>(grad, a, p, stream);
  return ln_run<Ln32>(grad, a, p, stream);
}

static int check_ln(int64_t M, int64_t N, int32_t dtype, int32_t w_dtype) {
  if (M <= 0 || N <= 0) { set_error("M, N must be positive"); return SP_ERR_INVALID_ARG; }
  if (M >= (1ll << 31) || N > kLnMaxN) { set_error("M below 2^31 and N up to %lld", (long long)kLnMaxN); return SP_ERR_UNSUPPORTED; }
  if (dtype != SP_BF16 && dtype != SP_FP32 && dtype != SP_FP16) { set_error("unknown element type %d", dtype); return SP_ERR_UNSUPPORTED; }
  if (w_dtype != dtype && w_dtype != SP_FP32) { set_error("gamma and beta must have the rows' type or be fp32"); return SP_ERR_UNSUPPORTED; }
  return SP_OK;
}

}  // namespace sp

using namespace sp;

using Bytes = unsigned __int128;

extern "C" {

int sp_layernorm(const void* x, const void* gamma, const void* beta, void* y, float* mean, float* rstd, int64_t M, int64_t N, int32_t dtype,
                 int32_t w_dtype, float eps, void* stream) {
  if (!x || !y) { set_error("x and y must not be NULL"); return SP_ERR_INVALID_ARG; }
  int rc = check_ln(M, N, dtype, w_dtype);
  if (rc != SP_OK) return rc;
  if (!(eps >= 0.f) || eps > FLT_MAX) { set_error("eps must be finite and not negative"); return SP_ERR_INVALID_ARG; }
  const uintptr_t e = ln_bytes(dtype), ew = ln_bytes(w_dtype);
  if ((((uintptr_t)x | (uintptr_t)y) & (e - 1)) || (((uintptr_t)gamma | (uintptr_t)beta) & (ew - 1)) || (((uintptr_t)mean | (uintptr_t)rstd) & 3u)) {
    set_error("pointers must be aligned to their elements");
    return SP_ERR_ALIGNMENT;
  }
  const Span spans[] = {{"y", y, (Bytes)M * N * e}, {"mean", mean, (Bytes)M * 4}, {"rstd", rstd, (Bytes)M * 4},
                        {"x", x, (Bytes)M * N * e}, {"gamma", gamma, (Bytes)N * ew}, {"beta", beta, (Bytes)N * ew}};
  rc = refuse_overlaps(spans, 3, 6);
  if (rc != SP_OK) return rc;
  int dev = 0;
  rc = current_device(&dev);
  if (rc != SP_OK) return rc;
  LnArgs a = {};
  a.x = (const char*)x; a.gamma = gamma; a.beta = beta; a.out = (char*)y; a.mean = mean; a.rstd = rstd;
  a.M = M; a.N = (int)N; a.w_dtype = w_dtype; a.eps = eps;
  return ln_any(false, a, dtype, (cudaStream_t)stream, ln_plan(M, N, ln_bytes(dtype), false, ln_mode(a, ln_bytes(dtype))));
}

int64_t sp_layernorm_workspace(int64_t M, int64_t N) {
  if (M <= 0 || N <= 0 || M >= (1ll << 31) || N > kLnMaxN) return -1;
  int64_t most = 0;      // whatever the type and the addresses are
  for (int mode : {kLnWhole, kLnEdges, kLnSingle})
    for (int elt : {2, 4}) {
      const LnPlan p = ln_plan(M, N, elt, true, mode);
      if ((int64_t)p.clusters * 2 * p.pitch * 4 > most) most = (int64_t)p.clusters * 2 * p.pitch * 4;
    }
  return most;
}

int sp_layernorm_grad(const void* dy, const void* x, const void* gamma, const float* mean, const float* rstd, void* dx, void* dgamma, void* dbeta,
                      int64_t M, int64_t N, int32_t dtype, int32_t w_dtype, void* workspace, int64_t workspace_bytes, void* stream) {
  if (!dy || !x || !mean || !rstd) { set_error("dy, x, mean and rstd must not be NULL"); return SP_ERR_INVALID_ARG; }
  if (!dx && !dgamma && !dbeta) { set_error("dx, dgamma and dbeta must not all be NULL"); return SP_ERR_INVALID_ARG; }
  int rc = check_ln(M, N, dtype, w_dtype);
  if (rc != SP_OK) return rc;
  const bool weights = dgamma || dbeta;
  const int64_t need = weights ? sp_layernorm_workspace(M, N) : 0;
  if (weights && (!workspace || workspace_bytes < need)) {
    set_error("workspace of %lld bytes, %lld needed for dgamma and dbeta", workspace ? (long long)workspace_bytes : 0ll, (long long)need);
    return SP_ERR_INVALID_ARG;
  }
  const uintptr_t e = ln_bytes(dtype), ew = ln_bytes(w_dtype);
  if ((((uintptr_t)x | (uintptr_t)dy | (uintptr_t)dx) & (e - 1)) || (((uintptr_t)gamma | (uintptr_t)dgamma | (uintptr_t)dbeta) & (ew - 1)) ||
      (((uintptr_t)mean | (uintptr_t)rstd) & 3u) || (weights && ((uintptr_t)workspace & 15u))) {
    set_error("pointers must be aligned to their elements, workspace to 16 bytes");
    return SP_ERR_ALIGNMENT;
  }
  const Span spans[] = {{"dx", dx, (Bytes)M * N * e}, {"dgamma", dgamma, (Bytes)N * ew}, {"dbeta", dbeta, (Bytes)N * ew},
                        {"workspace", weights ? workspace : nullptr, (Bytes)need}, {"dy", dy, (Bytes)M * N * e}, {"x", x, (Bytes)M * N * e},
                        {"gamma", gamma, (Bytes)N * ew}, {"mean", mean, (Bytes)M * 4}, {"rstd", rstd, (Bytes)M * 4}};
  rc = refuse_overlaps(spans, 4, 9);
  if (rc != SP_OK) return rc;
  int dev = 0;
  rc = current_device(&dev);
  if (rc != SP_OK) return rc;
  LnArgs a = {};
  a.x = (const char*)x; a.dy = (const char*)dy; a.gamma = gamma; a.out = (char*)dx; a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  a.M = M; a.N = (int)N; a.w_dtype = w_dtype;
  const LnPlan p = ln_plan(M, N, ln_bytes(dtype), true, ln_mode(a, ln_bytes(dtype)));
  if (p.clusters > 1) a.part = weights ? (float*)workspace : nullptr;
  else { a.dgamma = dgamma; a.dbeta = dbeta; }
  rc = ln_any(true, a, dtype, (cudaStream_t)stream, p);
  if (rc == SP_OK && a.part)
    rc = launch_pdl("layer norm gradient of the weights", layernorm_weights_kernel, dim3((unsigned)((N + 31) / 32), 2), 512, 0, 1, (cudaStream_t)stream,
                    (const float*)a.part, p.clusters, p.pitch, (int)N, w_dtype, dgamma, dbeta);
  return rc;
}

}  // extern "C"
