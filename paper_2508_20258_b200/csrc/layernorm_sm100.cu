// Layer norm of the rows of a matrix, and its gradients.
//
//   y = (x - mean) rstd gamma + beta,   mean = sum x / N,   rstd = 1 / sqrt(sum (x - mean)^2 / N + eps)
//   xh = (x - mean) rstd,   u = dy gamma,   dx = rstd (u - sum u / N - xh sum (u xh) / N),   dgamma = sum over rows of dy xh,   dbeta = of dy
//
// Both are bound by HBM: x is read and y written, or x and dy read and dx written, each once.  A row is held in registers from its one read to its
// one write, 16 elements per thread, by 1, 2, 4 or 8 warps, beyond 4096 elements by the CTAs of a cluster, which exchange their sums through
// distributed shared memory.  Each group of warps walks its own rows with the next four on their way through shared memory.
// Sums are 32-bit and taken in a fixed order: the same bits every time.
#include <float.h>

#include <mutex>

#include "product.cuh"

namespace sp {

constexpr int kLnThreads = 256, kLnPer = 16;      // threads of a block, elements per thread
constexpr int kLnDepth = 4;                       // rows on their way per group of warps
constexpr int kLnSlice = kLnThreads * kLnPer;     // columns of a CTA, at most
constexpr int kLnMaxCluster = 8;
constexpr int64_t kLnMaxN = (int64_t)kLnSlice * kLnMaxCluster;
constexpr int kLnSms = 148;

struct LnArgs {
  const char* x;
  const char* dy;
  const void* gamma;
  const void* beta;
  char* out;                // y, or dx (nullptr: not wanted)
  float* mean;
  float* rstd;
  float* part;              // backward: sums of a CTA cluster's rows, [cluster][dgamma, dbeta][pitch]; nullptr: not wanted
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

// Element types: 16 bytes to floats and back.
struct LnBf16 {
  static constexpr int kBytes = 2;
  static __device__ __forceinline__ void unpack(const uint32_t (&v)[4], float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(v[i] << 16); f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u); }
  }
  static __device__ __forceinline__ void pack(const float* f, uint32_t (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack_16(f[2 * i], f[2 * i + 1], true);
  }
};
struct LnFp16 {
  static constexpr int kBytes = 2;
  static __device__ __forceinline__ void unpack(const uint32_t (&v)[4], float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&v[i]));
      f[2 * i] = p.x; f[2 * i + 1] = p.y;
    }
  }
  static __device__ __forceinline__ void pack(const float* f, uint32_t (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack_16(f[2 * i], f[2 * i + 1], false);
  }
};
struct LnFp32 {
  static constexpr int kBytes = 4;
  static __device__ __forceinline__ void unpack(const uint32_t (&v)[4], float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
  }
  static __device__ __forceinline__ void pack(const float* f, uint32_t (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(f[i]);
  }
};

// Bytes s .. s + 15 of a and b one behind the other; s from 0 to 15, a multiple of the element size.
template <int ELT>
__device__ __forceinline__ void shift_16(const uint32_t (&a)[4], const uint32_t (&b)[4], int s, uint32_t (&o)[4]) {
  const uint32_t v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  uint32_t t[6], q[5];
#pragma unroll
  for (int i = 0; i < 6; ++i) t[i] = s & 8 ? v[i + 2] : v[i];
#pragma unroll
  for (int i = 0; i < 5; ++i) q[i] = s & 4 ? t[i + 1] : t[i];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = ELT == 2 && (s & 2) ? __funnelshift_r(q[i], q[i + 1], 16) : q[i];
}

// Element i of 16 bytes to global memory.
template <int ELT>
__device__ __forceinline__ void store_element(char* at, const uint32_t (&v)[4], int i) {
  if constexpr (ELT == 4) *reinterpret_cast<uint32_t*>(at) = v[i];
  else *reinterpret_cast<uint16_t*>(at) = (uint16_t)(i & 1 ? v[i >> 1] >> 16 : v[i >> 1]);
}

__device__ __forceinline__ float ln_weight(const void* w, int dtype, int col) {
  if (dtype == SP_FP32) return __ldg((const float*)w + col);
  const uint16_t b = __ldg((const uint16_t*)w + col);
  if (dtype == SP_BF16) return __uint_as_float((uint32_t)b << 16);
  __half_raw r;
  r.x = b;
  return __half2float(__half(r));
}

// A group of W warps and its part of a row: 16-byte units of the slice, unit (wg U + u) 32 + lane the u-th of a lane, so that a warp's units are one stretch.
template <class E, int W, bool ALIGNED>
struct LnGroup {
  static constexpr int kGroups = kLnThreads / 32 / W, kGroupThreads = 32 * W;
  static constexpr int kElems = 16 / E::kBytes, kUnits = kLnPer / kElems;
  int lane, wg, group, tid;
  int rank, ranks;             // of the CTA in its cluster
  int cols;                    // of the slice
  uint32_t red, far;           // shared memory: sums of warps, sums of CTAs (two of each, used in turn)
  uint32_t parity;

  __device__ __forceinline__ LnGroup(const LnArgs& a, uint32_t red_) : red(red_), parity(0) {
    const int warp = threadIdx.x >> 5;
    lane = threadIdx.x & 31;
    wg = warp % W; group = warp / W; tid = threadIdx.x % kGroupThreads;
    ranks = W == 8 ? (int)cluster_nctarank() : 1;
    rank = W == 8 ? (int)cluster_ctarank() : 0;
    cols = max(0, min(a.slice, a.N - rank * a.slice));
    far = red + 2 * 8 * 8;
    if (W == 8 && ranks > 1) unit_sync<2>();      // every CTA of the cluster is there before one writes to its shared memory
  }
  __device__ __forceinline__ int unit(int u) const { return (wg * kUnits + u) * 32 + lane; }
  __device__ __forceinline__ void sync() const {
    if constexpr (W == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(kGroupThreads) : "memory");
  }

  // A row's slice on its way to shared memory, as whole 16-byte units of global memory.  [lo, hi): the matrix, outside of which nothing is read.
  __device__ __forceinline__ void fetch(uint32_t dst, const char* row, const char* lo, const char* hi) const {
    const int bytes = cols * E::kBytes;
    if constexpr (ALIGNED) {      // the units a lane will read itself
#pragma unroll
      for (int u = 0; u < kUnits; ++u)
        if (unit(u) * 16 < bytes) cp_async_16(dst + unit(u) * 16, row + unit(u) * 16, 16);
    } else {
      const int m = (int)((uintptr_t)row & 15u), n = (m + bytes + 15) >> 4;
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
  // Unit k of the slice from shared memory, `m`: its row's address modulo 16.  Columns beyond the slice become zeros.
  __device__ __forceinline__ void take(uint32_t src, int k, int m, float* f) const {
    uint32_t v[4] = {0u, 0u, 0u, 0u};
    const int left = cols - k * kElems;
    if (left > 0) {
      ld_shared_16(src + 16 * k, v);
      if constexpr (!ALIGNED) {
        if (m) {
          uint32_t w[4], o[4];
          ld_shared_16(src + 16 * k + 16, w);
          shift_16<E::kBytes>(v, w, m, o);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = o[i];
        }
      }
    }
    E::unpack(v, f);
    if constexpr (!ALIGNED)
      if (left < kElems) {
#pragma unroll
        for (int i = 0; i < kElems; ++i)
          if (i >= left) f[i] = 0.f;
      }
  }
  // A lane's units to the row's slice.  Unaligned rows: a lane writes the 16-byte unit of global memory in which its own begins, the first part of it
  // from the lane before; element by element where a stretch of the warp or the slice begins or ends.
  __device__ __forceinline__ void put(char* row, const float* f) const {
    const int bytes = cols * E::kBytes;
    if constexpr (ALIGNED) {
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        uint32_t v[4];
        E::pack(f + u * kElems, v);
        if (unit(u) * 16 < bytes) *reinterpret_cast<uint4*>(row + unit(u) * 16) = make_uint4(v[0], v[1], v[2], v[3]);
      }
    } else {
      const int m = (int)((uintptr_t)row & 15u);
      if (wg * kUnits * 512 >= bytes + 16) return;      // a warp with no part of the row
      uint32_t before[4] = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        uint32_t v[4], p[4], o[4];
        E::pack(f + u * kElems, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t r = __shfl_sync(0xffffffffu, v[i], (lane + 31) & 31);
          p[i] = lane == 0 ? before[i] : r;
          before[i] = r;
          o[i] = v[i];
        }
        if (m) shift_16<E::kBytes>(p, v, 16 - m, o);
        const int at = unit(u) * 16 - m;                                             // of the row: where this unit of global memory begins
        const int first = u == 0 && lane == 0 ? at + m : at, end = min(at + 16, bytes);
        if (first == at && end == at + 16) *reinterpret_cast<uint4*>(row + at) = make_uint4(o[0], o[1], o[2], o[3]);
        else if (first < end) {
#pragma unroll
          for (int i = 0; i < kElems; ++i)
            if (at + i * E::kBytes >= first && at + i * E::kBytes < end) store_element<E::kBytes>(row + at + i * E::kBytes, o, i);
        }
        if (u == kUnits - 1 && lane == 31 && m) {      // the end of the warp's stretch
#pragma unroll
          for (int i = 0; i < kElems; ++i)
            if (i * E::kBytes >= 16 - m && at + m + i * E::kBytes < bytes) store_element<E::kBytes>(row + at + m + i * E::kBytes, v, i);
        }
      }
    }
  }
  // Sums of a and b over the row: lanes, warps, CTAs, in this order.
  __device__ __forceinline__ void sum(float& a, float& b) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      a += __shfl_xor_sync(0xffffffffu, a, o);
      b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    if constexpr (W > 1) {
      const uint32_t at = red + (parity * 8 + group * W) * 8;
      if (lane == 0) asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(at + wg * 8), "f"(a), "f"(b) : "memory");
      sync();
      a = b = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        float p, q;
        asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(p), "=f"(q) : "r"(at + i * 8) : "memory");
        a += p; b += q;
      }
    }
    if constexpr (W == 8)
      if (ranks > 1) {
        const uint32_t at = far + parity * kLnMaxCluster * 8;
        if (tid < ranks) asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(mapa(at + rank * 8, tid)), "f"(a), "f"(b) : "memory");
        unit_sync<2>();      // all threads of the cluster
        a = b = 0.f;
        for (int i = 0; i < ranks; ++i) {
          float p, q;
          asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(p), "=f"(q) : "r"(at + i * 8) : "memory");
          a += p; b += q;
        }
      }
    parity ^= 1u;
  }
};

// Bytes of shared memory beside the rows: sums of warps and of CTAs, two of each.
constexpr uint32_t kLnRedBytes = 2 * 8 * 8 + 2 * kLnMaxCluster * 8;

// 1 / sqrt(v): the hardware's, which is good to two steps, and one step of Newton's method.
__device__ __forceinline__ float ln_rsqrt(float v) {
  const float r = rsqrtf(v), s = r * fmaf(-0.5f * v * r, r, 1.5f);
  return s == s ? s : r;      // 0 and infinity
}

template <class E, int W, bool ALIGNED>
__global__ void __launch_bounds__(kLnThreads, 3) layernorm_kernel(const LnArgs a) {
  extern __shared__ __align__(16) uint8_t ln_smem[];
  using G = LnGroup<E, W, ALIGNED>;
  constexpr int U = G::kUnits, K = G::kElems;
  const uint32_t base = smem_u32(ln_smem);
  G g(a, base);
  const uint32_t ring = base + kLnRedBytes + g.group * kLnDepth * a.slot;
  const int64_t first = (int64_t)(blockIdx.x / g.ranks) * G::kGroups + g.group, step = (int64_t)a.clusters * G::kGroups;
  const int col0 = g.rank * a.slice;
  const int64_t pitch = (int64_t)a.N * E::kBytes, from = (int64_t)col0 * E::kBytes;
  const char* end = a.x + a.M * pitch;
  pdl_begin();
#pragma unroll
  for (int i = 0; i < kLnDepth; ++i) {
    if (first + i * step < a.M) g.fetch(ring + i * a.slot, a.x + (first + i * step) * pitch + from, a.x, end);
    cp_async_commit();
  }
  float gamma[kLnPer], beta[kLnPer];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < K; ++i) {
      const int c = g.unit(u) * K + i;
      gamma[u * K + i] = a.gamma != nullptr && c < g.cols ? ln_weight(a.gamma, a.w_dtype, col0 + c) : 1.f;
      beta[u * K + i] = a.beta != nullptr && c < g.cols ? ln_weight(a.beta, a.w_dtype, col0 + c) : 0.f;
    }
  const float inv = 1.f / (float)a.N;
  int slot = 0;
  for (int64_t row = first; row < a.M; row += step) {
    cp_async_wait<kLnDepth - 1>();
    if constexpr (!ALIGNED) g.sync();      // the others' copies
    const char* src = a.x + row * pitch + from;
    float x[kLnPer];
#pragma unroll
    for (int u = 0; u < U; ++u) g.take(ring + slot * a.slot, g.unit(u), (int)((uintptr_t)src & 15u), x + u * K);
    float s = 0.f, t = 0.f;
#pragma unroll
    for (int i = 0; i < kLnPer; i += 2) { s += x[i]; t += x[i + 1]; }
    s += t; t = 0.f;
    if constexpr (W == 1 && !ALIGNED) __syncwarp();      // all have read the slot
    g.sum(s, t);
    if (row + kLnDepth * step < a.M) g.fetch(ring + slot * a.slot, src + kLnDepth * step * pitch, a.x, end);
    cp_async_commit();
    slot = slot + 1 == kLnDepth ? 0 : slot + 1;
    // The differences' own sum corrects what the rounded mean leaves: of rows whose mean is a thousand deviations, too, variance and y keep their digits.
    const float about = s * inv;
    float d = 0.f, v = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < K; ++i) {
        float& e = x[u * K + i];
        e = g.unit(u) * K + (ALIGNED ? 0 : i) < g.cols ? e - about : 0.f;
        d += e;
        v = fmaf(e, e, v);
      }
    g.sum(d, v);
    const float off = d * inv, var = fmaf(-off, off, v * inv), rstd = ln_rsqrt((var < 0.f ? 0.f : var) + a.eps);
    if (g.tid == 0 && g.rank == 0) {
      if (a.mean != nullptr) a.mean[row] = about + off;
      if (a.rstd != nullptr) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < kLnPer; ++i) x[i] = fmaf((x[i] - off) * rstd, gamma[i], beta[i]);
    g.put(a.out + row * pitch + from, x);
  }
}

template <class E, int W, bool ALIGNED>
__global__ void __launch_bounds__(kLnThreads, 2) layernorm_grad_kernel(const LnArgs a) {
  extern __shared__ __align__(16) uint8_t ln_smem[];
  using G = LnGroup<E, W, ALIGNED>;
  constexpr int U = G::kUnits, K = G::kElems;
  const uint32_t base = smem_u32(ln_smem);
  G g(a, base);
  const uint32_t ring = base + kLnRedBytes + g.group * kLnDepth * 2 * a.slot;
  const int64_t first = (int64_t)(blockIdx.x / g.ranks) * G::kGroups + g.group, step = (int64_t)a.clusters * G::kGroups;
  const int col0 = g.rank * a.slice;
  const int64_t pitch = (int64_t)a.N * E::kBytes, from = (int64_t)col0 * E::kBytes, all = a.M * pitch;
  pdl_begin();
  const auto fetch = [&](int slot, int64_t row) {
    const uint32_t at = ring + slot * 2 * a.slot;
    g.fetch(at, a.x + row * pitch + from, a.x, a.x + all);
    g.fetch(at + a.slot, a.dy + row * pitch + from, a.dy, a.dy + all);
  };
#pragma unroll
  for (int i = 0; i < kLnDepth; ++i) {
    if (first + i * step < a.M) fetch(i, first + i * step);
    cp_async_commit();
  }
  float gamma[kLnPer], dg[kLnPer], db[kLnPer];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < K; ++i) {
      const int c = g.unit(u) * K + i;
      gamma[u * K + i] = a.gamma != nullptr && c < g.cols ? ln_weight(a.gamma, a.w_dtype, col0 + c) : 1.f;
      dg[u * K + i] = db[u * K + i] = 0.f;
    }
  const float inv = 1.f / (float)a.N;
  float mean = 0.f, rstd = 0.f;
  if (first < a.M) { mean = __ldg(a.mean + first); rstd = __ldg(a.rstd + first); }
  int slot = 0;
  for (int64_t row = first; row < a.M; row += step) {
    float next_mean = 0.f, next_rstd = 0.f;
    if (row + step < a.M) { next_mean = __ldg(a.mean + row + step); next_rstd = __ldg(a.rstd + row + step); }
    cp_async_wait<kLnDepth - 1>();
    if constexpr (!ALIGNED) g.sync();
    const char *src = a.x + row * pitch + from, *src_dy = a.dy + row * pitch + from;
    const uint32_t at = ring + slot * 2 * a.slot;
    float x[kLnPer], y[kLnPer];      // xh and u
    float s = 0.f, t = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      g.take(at, g.unit(u), (int)((uintptr_t)src & 15u), x + u * K);
      g.take(at + a.slot, g.unit(u), (int)((uintptr_t)src_dy & 15u), y + u * K);
#pragma unroll
      for (int i = u * K; i < u * K + K; ++i) {
        x[i] = (x[i] - mean) * rstd;
        dg[i] = fmaf(y[i], x[i], dg[i]);
        db[i] += y[i];
        y[i] *= gamma[i];
        s += y[i];
        t = fmaf(y[i], x[i], t);
      }
    }
    if constexpr (W == 1 && !ALIGNED) __syncwarp();      // all have read the slot
    if (a.out != nullptr || W > 1) g.sum(s, t);
    if (row + kLnDepth * step < a.M) fetch(slot, row + kLnDepth * step);
    cp_async_commit();
    slot = slot + 1 == kLnDepth ? 0 : slot + 1;
    if (a.out != nullptr) {
      s *= inv; t *= inv;
#pragma unroll
      for (int i = 0; i < kLnPer; ++i) x[i] = rstd * fmaf(-t, x[i], y[i] - s);
      g.put(a.out + row * pitch + from, x);
    }
    mean = next_mean; rstd = next_rstd;
  }
  if (a.part == nullptr) return;
  // the groups' sums to one, in their order
  float* part = a.part + (int64_t)(blockIdx.x / g.ranks) * 2 * a.pitch + col0;
  cp_async_wait<0>();
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    float* v = w == 0 ? dg : db;
    if constexpr (G::kGroups > 1) {
      float* all_groups = reinterpret_cast<float*>(ln_smem + kLnRedBytes);
      const int width = (a.N + 15) & ~15;
      __syncthreads();
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < K; ++i)
          if (g.unit(u) * K + i < width) all_groups[g.group * width + g.unit(u) * K + i] = v[u * K + i];
      __syncthreads();
      for (int c = threadIdx.x; c < a.N; c += kLnThreads) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < G::kGroups; ++i) s += all_groups[i * width + c];
        part[w * a.pitch + c] = s;
      }
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < K; i += 4)
          if (g.unit(u) * K + i < g.cols) *reinterpret_cast<float4*>(part + w * a.pitch + g.unit(u) * K + i) = make_float4(v[u * K + i], v[u * K + i + 1], v[u * K + i + 2], v[u * K + i + 3]);
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
  if (dtype == SP_FP32) ((float*)out)[col] = s;
  else ((uint16_t*)out)[col] = (uint16_t)pack_16(s, 0.f, dtype == SP_BF16);
}

// ------------------------------------------------------------------ host side
static std::mutex g_ln_mu;   // per-kernel set-up is done under it

static int ln_bytes(int32_t dtype) { return dtype == SP_FP32 ? 4 : 2; }

// What follows from the sizes: how many CTAs share a row, how many warps a group has, how many clusters run.
struct LnPlan {
  int ranks, warps, slice, clusters, pitch;
};

static LnPlan ln_plan(int64_t M, int64_t N, bool grad) {
  LnPlan p = {};
  p.ranks = 1;
  while ((int64_t)p.ranks * kLnSlice < N) p.ranks *= 2;
  p.slice = (int)(((N + p.ranks - 1) / p.ranks + 15) / 16 * 16);
  p.warps = 1;
  while (p.warps * 32 * kLnPer < p.slice) p.warps *= 2;
  const int groups = kLnThreads / 32 / p.warps;
  // Two (backward) or three blocks per SM; and backward, whose blocks each leave a row of sums, at least four rows for every group.
  const int64_t most = (grad ? 2 : 3) * kLnSms / p.ranks, per = grad ? 4 : 1, want = (M + groups * per - 1) / (groups * per);
  p.clusters = (int)(want < most ? want : most);
  p.pitch = (int)((N + 15) / 16 * 16);
  return p;
}

template <class E, int W, bool ALIGNED>
static int ln_launch(bool grad, const LnArgs& a, const LnPlan& p, cudaStream_t stream) {
  const uint32_t smem = kLnRedBytes + (uint32_t)(kLnThreads / 32 / W) * kLnDepth * (grad ? 2 : 1) * a.slot;
  auto kern = grad ? layernorm_grad_kernel<E, W, ALIGNED> : layernorm_kernel<E, W, ALIGNED>;
  static uint64_t configured[2] = {0, 0};
  if (first_use_on_this_device(configured[grad])) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kProdSmemLimit);
    if (e != cudaSuccess) { configured[grad] = 0; set_error("cudaFuncSetAttribute failed: %s", cudaGetErrorString(e)); return SP_ERR_CUDA; }
  }
  return launch_pdl(grad ? "layer norm gradient" : "layer norm", kern, dim3((unsigned)(p.clusters * p.ranks)), kLnThreads, smem, p.ranks, stream, a);
}

template <class E>
static int ln_run(bool grad, const LnArgs& a, const LnPlan& p, bool aligned, cudaStream_t stream) {
  switch (p.warps) {
    case 1: return aligned ? ln_launch<E, 1, true>(grad, a, p, stream) : ln_launch<E, 1, false>(grad, a, p, stream);
    case 2: return aligned ? ln_launch<E, 2, true>(grad, a, p, stream) : ln_launch<E, 2, false>(grad, a, p, stream);
    case 4: return aligned ? ln_launch<E, 4, true>(grad, a, p, stream) : ln_launch<E, 4, false>(grad, a, p, stream);
    default: return aligned ? ln_launch<E, 8, true>(grad, a, p, stream) : ln_launch<E, 8, false>(grad, a, p, stream);
  }
}

static int ln_any(bool grad, LnArgs& a, int32_t dtype, cudaStream_t stream, LnPlan* plan) {
  const LnPlan p = ln_plan(a.M, a.N, grad);
  a.slice = p.slice; a.clusters = p.clusters; a.pitch = p.pitch;
  a.slot = (uint32_t)p.slice * ln_bytes(dtype) + 16;
  // rows of whole 16-byte units at 16-byte addresses
  const bool aligned = ((int64_t)a.N * ln_bytes(dtype)) % 16 == 0 && (((uintptr_t)a.x | (uintptr_t)a.dy | (uintptr_t)a.out) & 15u) == 0;
  *plan = p;
  std::lock_guard<std::mutex> lock(g_ln_mu);
  if (dtype == SP_BF16) return ln_run<LnBf16>(grad, a, p, aligned, stream);
  if (dtype == SP_FP16) return ln_run<LnFp16>(grad, a, p, aligned, stream);
  return ln_run<LnFp32>(grad, a, p, aligned, stream);
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
  LnPlan p;
  return ln_any(false, a, dtype, (cudaStream_t)stream, &p);
}

int64_t sp_layernorm_workspace(int64_t M, int64_t N) {
  if (M <= 0 || N <= 0 || M >= (1ll << 31) || N > kLnMaxN) return -1;
  const LnPlan p = ln_plan(M, N, true);
  return (int64_t)p.clusters * 2 * p.pitch * 4;
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
  a.part = weights ? (float*)workspace : nullptr;
  a.M = M; a.N = (int)N; a.w_dtype = w_dtype;
  LnPlan p;
  rc = ln_any(true, a, dtype, (cudaStream_t)stream, &p);
  if (rc == SP_OK && weights)
    rc = launch_pdl("layer norm gradient of the weights", layernorm_weights_kernel, dim3((unsigned)((N + 31) / 32), 2), 512, 0, 1, (cudaStream_t)stream,
                    (const float*)a.part, p.clusters, p.pitch, (int)N, w_dtype, dgamma, dbeta);
  return rc;
}

}  // extern "C"
