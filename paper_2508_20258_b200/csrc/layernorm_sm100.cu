// Layer norm of the rows of a matrix, and its gradients.
//
//   y = (x - mean) rstd gamma + beta,   mean = sum x / N,   rstd = 1 / sqrt(sum (x - mean)^2 / N + eps)
//   xh = (x - mean) rstd,   u = dy gamma,   dx = rstd (u - sum u / N - xh sum (u xh) / N),   dgamma = sum over rows of dy xh,   dbeta = of dy
//
// Both are bound by HBM: x is read and y written, or x and dy read and dx written, each once (16384 x 4096 bf16: 45 us, 5.9 TB/s, and 70 us, 5.8 TB/s; a copy of as many bytes 43 and 64).
// A row is held in registers from its one read to its one write, up to 32 or (backward, beside the columns' sums) 16 or 24 elements per thread, by 1 to 16 warps, beyond a
// block's width by the CTAs of a cluster, which exchange their sums through distributed shared memory (backward such rows stay in shared memory, and sums cross beside another row's work).  Each group of warps walks its own rows with the next ones on their
// way through shared memory.
// What comes next are issue slots and the chain of a row, read, sums, barriers, write, with 16 warps on an SM to hide it (half of the slots are used): so all arithmetic is on pairs, kernels have no
// branch among a thread's elements, and rows wider than 4096 (backward) or 8192, whose one group per SM has nothing beside it, are slower: 4096 x 8192 27.7 and 44.5 us, 2048 x 16384 fp32
// 53 and 87 (copies 22.6 and 33, 43 and 64).
// Sums are 32-bit and taken in a fixed order: the same bits every time.
#include <float.h>

#include <mutex>

#include "product.cuh"

namespace sp {

constexpr int kLnThreads = 512;                   // of a block: 16 warps in groups
constexpr int kLnMaxCluster = 4;
constexpr int kLnSums = 2;                        // of a group of warps at once, at most
constexpr int64_t kLnMaxN = 32768;
constexpr int kLnSms = 148;
// Clusters of four that find room at once, as the occupancy calculator has it for the devices seen (which SMs share a GPC decides): with 37 a second wave (1000 x 32768 fp32 164 us, with 33: 101).
// A constant, not asked of each device: it decides in which order dgamma and dbeta are added up.  Where fewer find room, that second wave is what it costs.
constexpr int kLnFours = 33;
constexpr uint32_t kLnSumBytes = 2 * (16 + kLnMaxCluster) * 4 * kLnSums;      // of shared memory: sums of warps and of CTAs, two of each
constexpr int kLnRing = 192 << 10;                // bytes of rows on their way, at most

// How a row lies in the lanes of its group.
enum : int {
  kLnWhole,     // 16-byte units, the rows being whole units at 16-byte addresses
  kLnEdges,     // whole 16-byte units of memory, and the few elements before the first and behind the last; a group's rows all begin at the same place in a unit
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
// Asked for here, not where it is used: the compiler would move an ordinary read there.
__device__ __forceinline__ float ask_for(const float* at) {
  float v;
  asm volatile("ld.global.nc.f32 %0, [%1];" : "=f"(v) : "l"(at));
  return v;
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ld_shared_16(uint32_t addr, uint32_t (&v)[4]) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr) : "memory");
}

// The same where reads may be moved beside each other and beside arithmetic: of a row that has arrived, at an address that came through `arrived`.
__device__ __forceinline__ void ld_row_16(uint32_t addr, uint32_t (&v)[4]) {
  asm("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr));
}
__device__ __forceinline__ uint32_t arrived(uint32_t at) {
  asm volatile("" : "+r"(at)::"memory");
  return at;
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
  static __device__ __forceinline__ float from_shared(uint32_t at) {
    uint16_t b;
    asm volatile("ld.shared.b16 %0, [%1];" : "=h"(b) : "r"(at) : "memory");
    return one(b);
  }
  static __device__ __forceinline__ float load(const char* at) {
    uint16_t b;
    asm volatile("ld.global.nc.b16 %0, [%1];" : "=h"(b) : "l"(at));
    return one(b);
  }
  static __device__ __forceinline__ void store(char* at, float f) { *reinterpret_cast<uint16_t*>(at) = (uint16_t)pack_16(f, 0.f, BF16); }
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
};
struct Ln32 {
  static constexpr int kBytes = 4;
  static __device__ __forceinline__ float from_shared(uint32_t at) { return __uint_as_float(ld_shared_32(at)); }
  static __device__ __forceinline__ float load(const char* at) { return ask_for(reinterpret_cast<const float*>(at)); }
  static __device__ __forceinline__ void store(char* at, float f) { *reinterpret_cast<float*>(at) = f; }
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
};

// A group of W warps and its part of a row, PER elements per thread as PER / 2 pairs.
//   Units: a lane's u-th is unit (u W + warp) 32 + lane.  With edges, `head` elements come before the first unit and at most as many behind the last: lanes 0 to 7 and 8 to 15
//   of the first warp have one each, beside their units.
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
  int cols;                    // of the slice
  int head, chunks;            // elements before the first unit; units (or single elements)
  int edge;                    // column of the lane's edge element, -1: none
  uint32_t red, far;           // shared memory: sums of warps, sums of CTAs (two of each, used in turn)
  uint32_t scratch;            // with edges: a warp's chunk of weights for each warp
  uint32_t parity;

  __device__ __forceinline__ LnGroup(const LnArgs& a, uint32_t red_) : head(0), edge(-1), red(red_), parity(0) {
    const int warp = threadIdx.x >> 5;
    lane = threadIdx.x & 31;
    wg = warp % W; group = warp / W; tid = threadIdx.x % kGroupThreads;
    ranks = W == 16 ? (int)cluster_nctarank() : 1;
    rank = W == 16 ? (int)cluster_ctarank() : 0;
    cols = max(0, min(a.slice, a.N - rank * a.slice));
    chunks = cols / kElems;
    far = red + 2 * 16 * 4 * kLnSums;
    scratch = red + kLnSumBytes;
    if (W == 16 && ranks > 1) unit_sync<2>();      // every CTA of the cluster is there before one writes to its shared memory
  }
  // `m`: address modulo 16 of the group's rows
  __device__ __forceinline__ void begin_at(int m) {
    if constexpr (MODE == kLnEdges) {
      head = min(((16 - m) & 15) / E::kBytes, cols);
      chunks = (cols - head) / kElems;
      const int e = lane < 8 ? lane : head + chunks * kElems + lane - 8;
      if (wg == 0 && lane < 16 && e < (lane < 8 ? head : cols)) edge = e;
    }
  }
  __device__ __forceinline__ int chunk(int i) const { return (i * W + wg) * 32 + lane; }
  __device__ __forceinline__ int column(int i) const { return head + chunk(i) * kElems; }
  // PER is the least number of elements, in steps of 8, that holds the row: only the last 8 may be missing, and no warp passes any over.  (Groups of 16 warps ask, as the CTAs of a cluster have
  // unequal slices.)
  static constexpr int kSure = kUnits && W < 16 ? (PER - 8) / kElems : 0;
  __device__ __forceinline__ bool any(int i) const { return kUnits || (i * W + wg) * 32 < chunks; }
  __device__ __forceinline__ bool has(int i) const { return i < kSure || chunk(i) < chunks; }
  __device__ __forceinline__ bool edges() const { return MODE == kLnEdges && wg == 0; }        // the warp that has them
  __device__ __forceinline__ float edge_of(const char* row) const { return edge >= 0 ? E::load(row + edge * E::kBytes) : 0.f; }
  __device__ __forceinline__ void sync() const {
    if constexpr (W == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(kGroupThreads) : "memory");
  }

  // A row's slice on its way to shared memory: the units that a lane will read itself, or all whole 16-byte units of global memory that hold it.  [lo, hi): the matrix, outside of
  // which nothing is read.
  __device__ __forceinline__ void fetch(uint32_t dst, const char* row, const char* lo, const char* hi) const {
    if constexpr (kUnits) {
      row += head * E::kBytes;
#pragma unroll
      for (int u = 0; u < kChunks; ++u)
        if (has(u)) cp_async_16(dst + chunk(u) * 16, row + chunk(u) * 16, 16);
    } else {
      const int m = (int)((uintptr_t)row & 15u), n = (m + cols * E::kBytes + 15) >> 4;
      for (int j = tid; j < n; j += kGroupThreads) {
        const char* p = row - m + 16 * j;
        if (p >= lo) cp_async_16(dst + 16 * j, p, (int)min((int64_t)16, (int64_t)(hi - p)));
        else      // the matrix starts inside this unit
          for (int b = 0; b < 16; b += E::kBytes)
            if (p + b >= lo && p + b < hi) {
              if constexpr (E::kBytes == 4) asm volatile("st.shared.b32 [%0], %1;" ::"r"(dst + 16 * j + b), "r"(*reinterpret_cast<const uint32_t*>(p + b)) : "memory");
              else asm volatile("st.shared.b16 [%0], %1;" ::"r"(dst + 16 * j + b), "h"(*reinterpret_cast<const uint16_t*>(p + b)) : "memory");
            }
      }
    }
  }
  // A lane's pairs of chunk i from shared memory, `m`: the row's address modulo 16.  Zeros where it has none.
  __device__ __forceinline__ void take(uint32_t src, int i, int m, uint64_t* f) const {
    if constexpr (kUnits) {
      uint32_t v[4] = {0u, 0u, 0u, 0u};
      if (has(i)) ld_row_16(src + 16 * chunk(i), v);
      E::unpack(v, f);
    } else {
      const uint32_t at = src + m + column(i) * E::kBytes;
      f[0] = pair_of(has(i) ? E::from_shared(at) : 0.f, has(i + 1) ? E::from_shared(at + 32 * W * E::kBytes) : 0.f);
    }
  }
  // f - v where the lane has something, else 0 as before
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
    char* at = row + column(i) * E::kBytes;
    if constexpr (kUnits) {
      uint32_t v[4];
      E::pack(f, v);
      if (has(i)) *reinterpret_cast<uint4*>(at) = make_uint4(v[0], v[1], v[2], v[3]);
    } else {
      float lo, hi;
      halves_of(f[0], lo, hi);
      if (has(i)) E::store(at, lo);
      if (has(i + 1)) E::store(at + 32 * W * E::kBytes, hi);
    }
  }
  // gamma or beta in one column of the slice
  __device__ __forceinline__ float weight(const void* w, int dtype, int col0, int c, float none) const {
    if (w == nullptr || c < 0) return none;
    if (dtype == SP_FP32) return __ldg((const float*)w + col0 + c);
    return E::load((const char*)w + (int64_t)(col0 + c) * E::kBytes);
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
        one_by_one<kSpread>(f, none, [&](int c) { return __ldg(p + c); });
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
          one_by_one<false>(f, none, [&](int c) { return E::one(__ldg(p + c)); });
        }
      }
    }
  }
  // SPREAD: the lanes' loads next to each other, and through shared memory to those that want them.  32-bit weights of 16-bit rows lie 32 bytes apart from lane to lane otherwise (5001 x
  // 2035 19.8 us, so 17.9; 16-bit ones 16 bytes, where it costs 1.7 us more than it saves).
  static constexpr bool kSpread = MODE == kLnEdges && E::kBytes == 2;
  template <bool SPREAD, class Load>
  __device__ __forceinline__ void one_by_one(uint64_t* f, float none, const Load& load) const {
    if constexpr (SPREAD) {
      float v[PER];
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const int c = ((e / kElems * W + wg) * 32) * kElems + e % kElems * 32 + lane;
        v[e] = c < chunks * kElems ? load(head + c) : none;
      }
      const uint32_t mine = scratch + (threadIdx.x >> 5) * 32 * kElems * 4;
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
#pragma unroll
        for (int k = 0; k < kElems; ++k) asm volatile("st.shared.f32 [%0], %1;" ::"r"(mine + (k * 32 + lane) * 4), "f"(v[i * kElems + k]) : "memory");
        __syncwarp();
#pragma unroll
        for (int k = 0; k < kElems; k += 4) {
          uint32_t q[4];
          ld_shared_16(mine + (lane * kElems + k) * 4, q);
          f[(i * kElems + k) / 2] = pair_of(__uint_as_float(q[0]), __uint_as_float(q[1]));
          f[(i * kElems + k) / 2 + 1] = pair_of(__uint_as_float(q[2]), __uint_as_float(q[3]));
        }
        __syncwarp();
      }
    } else {
#pragma unroll
      for (int k = 0; k < kPairs; ++k) {
        float v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int e = 2 * k + h;
          v[h] = has(e / kElems) ? load(column(e / kElems) + e % kElems) : none;
        }
        f[k] = pair_of(v[0], v[1]);
      }
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
        if (ranks > 1) {      // (Every warp's sums straight to all CTAs behind one barrier: gradient of 2048 x 16384 fp32 97.8 us, so 91.9.  Groups of 8 warps in twice the CTAs, whose sums complete on
                              // barriers of their own by st.async, so that a CTA's two groups need not wait for each other: 137.)
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

// Bytes of shared memory before the rows.
template <class E, int MODE>
constexpr uint32_t kLnBefore = kLnSumBytes + (MODE == kLnEdges && E::kBytes == 2 ? kLnThreads * 8 * 4 : 0);

// Backward with 24 elements per thread, gamma waits in shared memory, where the rows' ring leaves room for it (16 bits): 4096 x 12288 78 us, in registers, which it overfills, 96.  Every
// thread keeps its own, 16 bytes of each side by side.
template <class E, int PER>
constexpr bool kLnFarGamma = PER == 24 && E::kBytes == 2;

// Batches of `rows` rows' slices on their way.
template <class E, int PER, int ROWS>
constexpr int kLnDepth = kLnRing / (kLnThreads * PER * E::kBytes * ROWS) < 3 ? kLnRing / (kLnThreads * PER * E::kBytes * ROWS) : 3;

// Of the kernel that finishes a row beside the sums of the next: sums of all warps of a cluster, [turn][CTA][sum][warp].
constexpr uint32_t kLnTurnSums = kLnMaxCluster * 2 * 16 * 4;

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
  const uint32_t ring = base + kLnBefore<E, MODE> + g.group * D * a.slot;
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
  const float edge_gamma = g.weight(a.gamma, a.w_dtype, g.rank * a.slice, g.edge, 1.f), edge_beta = g.weight(a.beta, a.w_dtype, g.rank * a.slice, g.edge, 0.f);
  float edge = row <= last ? g.edge_of(a.x + here) : 0.f;      // of the row to come
  const float inv = 1.f / (float)a.N;
  uint32_t at = ring;
  for (; row <= last; row += total, here += hop) {
    cp_async_wait<D - 1>();
    if constexpr (MODE == kLnSingle) g.sync();      // the others' copies
    const uint32_t here_at = arrived(at);
    uint64_t x[G::kPairs], s2[2] = {0, 0}, v2[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < G::kChunks; i += G::kStep)
      if (g.any(i)) {
        uint64_t* f = x + i * G::kElems / 2;
        g.take(here_at, i, (int)((uintptr_t)(a.x + here) & 15u), f);
#pragma unroll
        for (int k = 0; k < P; ++k) s2[k & 1] = add_pair(s2[k & 1], f[k]);
      }
    float s = halves_sum(add_pair(s2[0], s2[1]));
    const float xe = edge;
    if (g.edges()) {
      s += xe;
      if (row + total <= last) edge = g.edge_of(a.x + here + hop);
    }
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
    const float de = g.edge >= 0 ? xe - about : 0.f;
    if (g.edges()) {
      sv[0] += de;
      sv[1] = fmaf(de, de, sv[1]);
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
    if (g.edges() && g.edge >= 0) E::store(a.out + here + g.edge * E::kBytes, fmaf((de - off) * rstd, edge_gamma, edge_beta));
  }
}

__device__ __forceinline__ void store_weight(void* out, int dtype, int col, float s) {
  if (out == nullptr) return;
  if (dtype == SP_FP32) ((float*)out)[col] = s;
  else ((uint16_t*)out)[col] = (uint16_t)pack_16(s, 0.f, dtype == SP_BF16);
}

// The block's sums of columns, to its row of the workspace or to dgamma and dbeta.
template <class E, int MODE, class G>
__device__ __forceinline__ void ln_column_sums(const G& g, const LnArgs& a, const uint64_t* dg, const uint64_t* db, float edge_dg, float edge_db, float* all_groups) {
  constexpr int P = G::kWide;
  if (a.part == nullptr && a.dgamma == nullptr && a.dbeta == nullptr) return;
  // The groups' sums to one, in their order, by way of shared memory: written to global memory as the lanes hold them, 32 bytes apart, they took 4 us longer.
  cp_async_wait<0>();
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    __syncthreads();      // all rows, and the sums before these, have been read
    float* mine = all_groups + g.group * a.slice;
#pragma unroll
    for (int i = 0; i < G::kChunks; i += G::kStep)
      if (g.any(i)) {
        const uint64_t* f = (w == 0 ? dg : db) + i * G::kElems / 2;
        if constexpr (MODE == kLnWhole) {
          if (g.has(i)) {
#pragma unroll
            for (int k = 0; k < P; k += 2) {
              float4 v;
              halves_of(f[k], v.x, v.y);
              halves_of(f[k + 1], v.z, v.w);
              *reinterpret_cast<float4*>(mine + g.column(i) + 2 * k) = v;
            }
          }
        } else {
#pragma unroll
          for (int k = 0; k < P; ++k) {
            float v[2];
            halves_of(f[k], v[0], v[1]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int e = 2 * k + h;
              if (g.has(i + e / G::kElems)) mine[g.column(i + e / G::kElems) + e % G::kElems] = v[h];
            }
          }
        }
      }
    if (g.edge >= 0) mine[g.edge] = w == 0 ? edge_dg : edge_db;
    __syncthreads();
    for (int c = threadIdx.x; c < g.cols; c += kLnThreads) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < G::kGroups; ++i) s += all_groups[i * a.slice + c];
      if (a.part != nullptr) a.part[((int64_t)(blockIdx.x / g.ranks) * 2 + w) * a.pitch + g.rank * a.slice + c] = s;
      else store_weight(w == 0 ? a.dgamma : a.dbeta, a.w_dtype, g.rank * a.slice + c, s);
    }
  }
}

template <class E, int W, int PER, int MODE>
__global__ void __launch_bounds__(kLnThreads, 1) layernorm_grad_kernel(const LnArgs a) {
  extern __shared__ __align__(16) uint8_t ln_smem[];
  using G = LnGroup<E, W, PER, MODE>;
  constexpr int D = kLnDepth<E, PER, 2>, P = G::kWide;
  const uint32_t base = smem_u32(ln_smem);
  G g(a, base);
  constexpr bool kFar = kLnFarGamma<E, PER>;
  const uint32_t gammas = base + kLnBefore<E, MODE> + threadIdx.x * 16;
  const uint32_t ring = base + kLnBefore<E, MODE> + (kFar ? kLnThreads * PER * 4 : 0) + g.group * D * 2 * a.slot, batch = 2 * a.slot;
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
  if constexpr (kFar) {
#pragma unroll
    for (int k = 0; k < G::kPairs; k += 2) asm volatile("st.shared.v2.b64 [%0], {%1, %2};" :: "r"(gammas + k * 8 * kLnThreads), "l"(gamma[k]), "l"(gamma[k + 1]) : "memory");
  }
#pragma unroll
  for (int k = 0; k < G::kPairs; ++k) dg[k] = db[k] = 0;
  const float inv = 1.f / (float)a.N;
  const float edge_gamma = g.weight(a.gamma, a.w_dtype, col0, g.edge, 1.f);
  float edge_x = 0.f, edge_dy = 0.f, edge_dg = 0.f, edge_db = 0.f;      // of the row to come; sums
  float mean = 0.f, rstd = 0.f;
  if (row <= last) {
    edge_x = g.edge_of(a.x + here);
    edge_dy = g.edge_of(a.dy + here);
  }
  if (row <= last) { mean = __ldg(a.mean + row); rstd = __ldg(a.rstd + row); }
  uint32_t at = ring;
  for (; row <= last; row += total, here += hop) {
    float next_mean = 0.f, next_rstd = 0.f;
    if (row + total <= last) { next_mean = ask_for(a.mean + row + total); next_rstd = ask_for(a.rstd + row + total); }
    cp_async_wait<D - 1>();
    if constexpr (MODE == kLnSingle) g.sync();
    const uint32_t here_at = arrived(at);
    uint64_t x[G::kPairs], y[G::kPairs], s2[2] = {0, 0}, t2[2] = {0, 0};      // xh and u
    const uint64_t minus = pair_of(-mean, -mean), scale = pair_of(rstd, rstd);
#pragma unroll
    for (int i = 0; i < G::kChunks; i += G::kStep)
      if (g.any(i)) {
        const int o = i * G::kElems / 2;
        g.take(here_at, i, (int)((uintptr_t)(a.x + here) & 15u), x + o);
        if constexpr (kFar) {
#pragma unroll
          for (int k = o; k < o + P; k += 2) asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(gamma[k]), "=l"(gamma[k + 1]) : "r"(gammas + k * 8 * kLnThreads) : "memory");
        }
        g.take(here_at + a.slot, i, (int)((uintptr_t)(a.dy + here) & 15u), y + o);      // 0 outside the slice, and with it all that x adds there
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
    float xe = 0.f, ue = 0.f;
    if (g.edges()) {
      if (g.edge >= 0) {
        xe = (edge_x - mean) * rstd;
        edge_dg = fmaf(edge_dy, xe, edge_dg);
        edge_db += edge_dy;
        ue = edge_dy * edge_gamma;
        st[0] += ue;
        st[1] = fmaf(ue, xe, st[1]);
      }
      if (row + total <= last) {
        edge_x = g.edge_of(a.x + here + hop);
        edge_dy = g.edge_of(a.dy + here + hop);
      }
    }
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
      if (g.edges() && g.edge >= 0) E::store(a.out + here + g.edge * E::kBytes, rstd * fmaf(-st[1] * inv, xe, ue - st[0] * inv));
    }
    mean = next_mean; rstd = next_rstd;
  }
  ln_column_sums<E, MODE>(g, a, dg, db, edge_dg, edge_db, reinterpret_cast<float*>(ln_smem + kLnBefore<E, MODE>));
}

// The same by groups of 16 warps that finish a row beside the sums of the next, which cross the cluster (or the block) meanwhile: for rows that clusters share, whose barrier had nothing beside it,
// and those that only fit one CTA this way, since x and dy are read from shared memory twice and the registers hold gamma and the columns' sums alone (gradients of 2048 x 16384 fp32 92 to 87 us,
// 3000 x 16384 bf16 in one CTA instead of two 89 to 80, 1000 x 24576 fp32 96 to 84).  Narrower rows lose more by the second reading and conversion (4096 x 5120 36 to 45 us, 4096 x 12288 78 to 82,
// 16384 x 4096 75 to 86).
template <class E, int PER, int MODE>
__global__ void __launch_bounds__(kLnThreads, 1) layernorm_grad_ahead_kernel(const LnArgs a) {
  extern __shared__ __align__(16) uint8_t ln_smem[];
  using G = LnGroup<E, 16, PER, MODE>;
  constexpr int D = kLnDepth<E, PER, 2>, P = G::kWide;
  static_assert(D == 3, "a row to finish, one to sum, one on its way");
  const uint32_t base = smem_u32(ln_smem);
  G g(a, base);
  const uint32_t sums = base + kLnBefore<E, MODE>;
  const uint32_t ring = sums + 2 * kLnTurnSums, batch = 2 * a.slot;
  const uint32_t total = a.clusters, last = (uint32_t)a.M - 1;
  const int col0 = g.rank * a.slice;
  const int64_t pitch = (int64_t)a.N * E::kBytes, hop = (int64_t)total * pitch, all = a.M * pitch;
  uint32_t row = blockIdx.x / g.ranks;
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
  const float edge_gamma = g.weight(a.gamma, a.w_dtype, col0, g.edge, 1.f);
  float edge_x = 0.f, edge_dy = 0.f, edge_dg = 0.f, edge_db = 0.f;      // of the row to come; sums
  float mean = 0.f, rstd = 0.f, mean_before = 0.f, rstd_before = 0.f, xe_before = 0.f, ue_before = 0.f;
  if (row <= last) {
    edge_x = g.edge_of(a.x + here);
    edge_dy = g.edge_of(a.dy + here);
    mean = __ldg(a.mean + row); rstd = __ldg(a.rstd + row);
  }
  uint32_t at = ring, at_before = ring, turn = 0;
  for (bool first = true;; first = false) {
    const bool more = row <= last;
    float next_mean = 0.f, next_rstd = 0.f, st[2], xe = 0.f, ue = 0.f;
    if (more) {
      if (row + total <= last) { next_mean = ask_for(a.mean + row + total); next_rstd = ask_for(a.rstd + row + total); }
      cp_async_wait<D - 2>();
      const uint32_t here_at = arrived(at);
      uint64_t s2[2] = {0, 0}, t2[2] = {0, 0};
      const uint64_t minus = pair_of(-mean, -mean), scale = pair_of(rstd, rstd);
#pragma unroll
      for (int i = 0; i < G::kChunks; ++i) {
        const int o = i * G::kElems / 2;
        uint64_t x[P], y[P];
        g.take(here_at, i, 0, x);
        g.take(here_at + a.slot, i, 0, y);
#pragma unroll
        for (int k = 0; k < P; ++k) {
          x[k] = mul_pair(add_pair(x[k], minus), scale);
          dg[o + k] = fma_pair(y[k], x[k], dg[o + k]);
          db[o + k] = add_pair(db[o + k], y[k]);
          y[k] = mul_pair(y[k], gamma[o + k]);
          s2[k & 1] = add_pair(s2[k & 1], y[k]);
          t2[k & 1] = fma_pair(y[k], x[k], t2[k & 1]);
        }
      }
      st[0] = halves_sum(add_pair(s2[0], s2[1]));
      st[1] = halves_sum(add_pair(t2[0], t2[1]));
      if (g.edges()) {
        if (g.edge >= 0) {
          xe = (edge_x - mean) * rstd;
          edge_dg = fmaf(edge_dy, xe, edge_dg);
          edge_db += edge_dy;
          ue = edge_dy * edge_gamma;
          st[0] += ue;
          st[1] = fmaf(ue, xe, st[1]);
        }
        if (row + total <= last) {
          edge_x = g.edge_of(a.x + here + hop);
          edge_dy = g.edge_of(a.dy + here + hop);
        }
      }
      // lanes 0-15 keep the first sum, 16-31 the second
      const bool upper = g.lane & 16;
      float v = (upper ? st[1] : st[0]) + __shfl_xor_sync(0xffffffffu, upper ? st[0] : st[1], 16);
#pragma unroll
      for (int o = 8; o; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
      st[0] = v;
    }
    float c1 = 0.f, c2 = 0.f;
    if (!first) {      // all CTAs' sums of the row before; they have read those of the row before that, whose place is free
      asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
      const uint32_t from = sums + ((turn & 1u) ^ 1u) * (kLnTurnSums) + g.lane * 4;
      float v = 0.f;
      for (int i = 0; i < g.ranks; ++i) v += __uint_as_float(ld_shared_32(from + i * 128));
#pragma unroll
      for (int o = 8; o; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
      c1 = -__shfl_sync(0xffffffffu, v, 0) * inv;
      c2 = -__shfl_sync(0xffffffffu, v, 16) * inv;
    }
    if (more) {
      if ((g.lane & 15) < g.ranks)
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(mapa(sums + (turn & 1u) * (kLnTurnSums) + g.rank * 128 + (g.lane >> 4) * 64 + g.wg * 4, g.lane & 15)), "f"(st[0]) : "memory");
      asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
      ++turn;
    }
    if (!first) {
      if (a.out != nullptr) {
        const uint32_t here_at = arrived(at_before);
        char* out = a.out + here - hop;
        const uint64_t minus = pair_of(-mean_before, -mean_before), scale = pair_of(rstd_before, rstd_before), p1 = pair_of(c1, c1), p2 = pair_of(c2, c2);
#pragma unroll
        for (int i = 0; i < G::kChunks; ++i) {
          const int o = i * G::kElems / 2;
          uint64_t x[P], y[P];
          g.take(here_at, i, 0, x);
          g.take(here_at + a.slot, i, 0, y);
#pragma unroll
          for (int k = 0; k < P; ++k) {
            x[k] = mul_pair(add_pair(x[k], minus), scale);
            x[k] = mul_pair(scale, fma_pair(p2, x[k], fma_pair(y[k], gamma[o + k], p1)));
          }
          g.put(out, i, x);
        }
        if (g.edges() && g.edge >= 0) E::store(out + g.edge * E::kBytes, rstd_before * fmaf(c2, xe_before, ue_before + c1));
      }
      fetch(at_before, ahead);
      ahead += total;
    }
    if (!more) break;
    mean_before = mean; rstd_before = rstd; xe_before = xe; ue_before = ue; at_before = at;
    mean = next_mean; rstd = next_rstd;
    at = at + batch == ring + D * batch ? ring : at + batch;
    row += total; here += hop;
  }
  cp_async_wait<0>();
  ln_column_sums<E, MODE>(g, a, dg, db, edge_dg, edge_db, reinterpret_cast<float*>(ln_smem + kLnBefore<E, MODE> + 2 * kLnTurnSums));
}
// dgamma (blockIdx.y 0) and dbeta (1) from the clusters' sums, in a fixed order: 32 rows of 32 columns side by side, up to five of them for a thread, asked for at once.
__global__ void __launch_bounds__(1024) layernorm_weights_kernel(const float* part, int rows, int pitch, int N, int dtype, void* dgamma, void* dbeta) {
  pdl_begin();
  __shared__ float sums[32][33];
  void* out = blockIdx.y == 0 ? dgamma : dbeta;
  if (out == nullptr) return;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  float v[5];
#pragma unroll
  for (int i = 0; i < 5; ++i) v[i] = col < N && w + 32 * i < rows ? __ldcg(part + ((int64_t)(w + 32 * i) * 2 + blockIdx.y) * pitch + col) : 0.f;
  sums[w][lane] = ((v[0] + v[1]) + (v[2] + v[3])) + v[4];
  __syncthreads();
  float s = sums[lane][w];      // a warp per column
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0 && blockIdx.x * 32 + w < N) store_weight(out, dtype, blockIdx.x * 32 + w, s);
}
static_assert(kLnSms <= 5 * 32, "rows of sums that the kernel above adds");

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
  // Forward up to 32 elements per thread: per row half the warps, with what a warp costs beside its elements, that up to 16 take (8192 x 4096 bf16: 25.9 us, with 16: 31.9).  Backward up to
  // 16, beside the columns' sums: 24 in half the warps are slower (16 bits: 8192 x 3000 42 us, with 16: 35; fp32, where some of it leaves the registers: 4096 x 5120 70, with 16: 49).  But in 16
  // bits 16 warps of 24, and of 32 with the rows in shared memory alone, save a cluster CTAs (4096 x 12288 in one CTA 78 us, in two 105).
  const int most_per = grad ? 16 : 32, widest = grad && elt == 2 && mode != kLnSingle ? 32 : most_per;
  for (p.ranks = 1;; p.ranks *= 2) {
    p.slice = (int)(((N + p.ranks - 1) / p.ranks + 15) / 16 * 16);
    if ((N < p.slice ? N : p.slice) <= kLnThreads * widest) break;
  }
  // With edges only whole units count: 1031 elements of 16 bits have at most 128.
  const int cols = (int)(N < p.slice ? N : p.slice), width = mode == kLnEdges ? cols / (16 / elt) * (16 / elt) : cols;
  for (p.warps = 1; p.warps < 16 && p.warps * 32 * most_per < width; p.warps *= 2) {}
  if (mode == kLnSingle || p.ranks > 1) p.warps = 16;
  for (p.per = 8; p.per < widest && (p.warps * 32 * p.per < width || mode == kLnSingle); p.per += 8) {}
  const int groups = kLnThreads / 32 / p.warps;
  // One block per SM; backward, whose blocks each leave a row of sums, at least two rows for every group, and one block for up to four.
  const int64_t most = p.ranks < 4 ? kLnSms / p.ranks : kLnFours, rows = grad ? (M <= 4 * groups ? 4 : 2) : 1, want = (M + groups * rows - 1) / (groups * rows);
  p.clusters = (int)(want < most ? want : most);
  if (mode == kLnEdges && (int64_t)p.clusters * groups < M) {      // a group's rows are a multiple of 16 bytes apart
    int apart = 1;
    while (((int64_t)apart * groups * N * elt) % 16) apart *= 2;
    p.clusters = p.clusters < apart ? apart : p.clusters / apart * apart;
  }
  p.pitch = (int)((N + 15) / 16 * 16);
  return p;
}

template <bool GRAD, class E, int W, int PER, int MODE, bool AHEAD = false>
static int ln_launch(const LnArgs& a, const LnPlan& p, cudaStream_t stream) {
  const int slots = GRAD ? 2 * kLnDepth<E, PER, 2> : kLnDepth<E, PER, 1>;
  const uint32_t smem = kLnBefore<E, MODE> + (uint32_t)(kLnThreads / 32 / W * slots) * a.slot + (AHEAD ? 2 * kLnTurnSums : GRAD && kLnFarGamma<E, PER> ? kLnThreads * PER * 4 : 0);
  void (*kern)(LnArgs);
  if constexpr (AHEAD) kern = layernorm_grad_ahead_kernel<E, PER, MODE>;
  else if constexpr (GRAD) kern = layernorm_grad_kernel<E, W, PER, MODE>;
  else kern = layernorm_kernel<E, W, PER, MODE>;
  static uint64_t configured = 0;
  if (first_use_on_this_device(configured)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kProdSmemLimit);
    if (e != cudaSuccess) { configured = 0; set_error("cudaFuncSetAttribute failed: %s", cudaGetErrorString(e)); return SP_ERR_CUDA; }
  }
  return launch_pdl(GRAD ? "layer norm gradient" : "layer norm", kern, dim3((unsigned)(p.clusters * p.ranks)), kLnThreads, smem, p.ranks, stream, a);
}

// More than one warp is taken where half as many would not do, clusters where one CTA would not: each thread then has more than half of the most (backward, 16 warps of
// 16 bits have up to 32).
template <bool GRAD, class E, int W, int MODE>
static int ln_width(const LnArgs& a, const LnPlan& p, cudaStream_t stream) {
  if constexpr (W == 1) {
    if (p.per == 8) return ln_launch<GRAD, E, W, 8, MODE>(a, p, stream);
    if (!GRAD && p.per == 16) return ln_launch<false, E, W, 16, MODE>(a, p, stream);
  }
  if constexpr (GRAD && W == 16 && E::kBytes == 2) {
    if (p.per == 24 && p.ranks == 1) return ln_launch<true, E, W, 24, MODE>(a, p, stream);
    if (p.per == 24) return ln_launch<true, E, W, 24, MODE, true>(a, p, stream);
    if (p.per == 32) return ln_launch<true, E, W, 32, MODE, true>(a, p, stream);
  }
  if constexpr (GRAD && W == 16 && E::kBytes == 4) {
    if (p.ranks > 1) return ln_launch<true, E, W, 16, MODE, true>(a, p, stream);
  }
  if constexpr (GRAD) return ln_launch<true, E, W, 16, MODE>(a, p, stream);
  else if (p.per == 24) return ln_launch<false, E, W, 24, MODE>(a, p, stream);
  else return ln_launch<false, E, W, 32, MODE>(a, p, stream);
}

template <bool GRAD, class E, int MODE>
static int ln_warps(const LnArgs& a, const LnPlan& p, cudaStream_t stream) {
  switch (p.warps) {
    case 1: return ln_width<GRAD, E, 1, MODE>(a, p, stream);
    case 2: return ln_width<GRAD, E, 2, MODE>(a, p, stream);
    case 4: return ln_width<GRAD, E, 4, MODE>(a, p, stream);
    case 8: return ln_width<GRAD, E, 8, MODE>(a, p, stream);
    default: return ln_width<GRAD, E, 16, MODE>(a, p, stream);
  }
}

template <bool GRAD, class E>
static int ln_run(const LnArgs& a, const LnPlan& p, cudaStream_t stream) {
  switch (p.mode) {
    case kLnWhole: return ln_warps<GRAD, E, kLnWhole>(a, p, stream);
    case kLnEdges: return ln_warps<GRAD, E, kLnEdges>(a, p, stream);
    default: return ln_launch<GRAD, E, 16, GRAD ? 16 : 32, kLnSingle>(a, p, stream);
  }
}

// How the rows lie.
static int ln_mode(const LnArgs& a, int elt) {
  const uintptr_t x = (uintptr_t)a.x, dy = a.dy ? (uintptr_t)a.dy : x, out = a.out ? (uintptr_t)a.out : x;
  if (((x ^ dy) | (x ^ out)) & 15u) return kLnSingle;
  return (x & 15u) == 0 && (int64_t)a.N * elt % 16 == 0 ? kLnWhole : kLnEdges;
}

template <bool GRAD>
static int ln_any(LnArgs& a, int32_t dtype, cudaStream_t stream, const LnPlan& p) {
  a.slice = p.slice; a.clusters = p.clusters; a.pitch = p.pitch;
  a.slot = (uint32_t)p.slice * ln_bytes(dtype) + 16;
  std::lock_guard<std::mutex> lock(g_ln_mu);
  if (dtype == SP_BF16) return ln_run<GRAD, Ln16<true>>(a, p, stream);
  if (dtype == SP_FP16) return ln_run<GRAD, Ln16<false>>(a, p, stream);
  return ln_run<GRAD, Ln32>(a, p, stream);
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
  return ln_any<false>(a, dtype, (cudaStream_t)stream, ln_plan(M, N, ln_bytes(dtype), false, ln_mode(a, ln_bytes(dtype))));
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
  rc = ln_any<true>(a, dtype, (cudaStream_t)stream, p);
  if (rc == SP_OK && a.part)
    rc = launch_pdl("layer norm gradient of the weights", layernorm_weights_kernel, dim3((unsigned)((N + 31) / 32), 2), 1024, 0, 1, (cudaStream_t)stream,
                    (const float*)a.part, p.clusters, p.pitch, (int)N, w_dtype, dgamma, dbeta);
  return rc;
}

}  // extern "C"
