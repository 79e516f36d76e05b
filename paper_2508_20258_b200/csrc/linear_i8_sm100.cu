// The linear layer in 8-bit integers: rows quantised with one scale each, the product of two 8-bit matrices in exact
// 32-bit integer sums on the tensor cores, scaled per row (token) and per column (output channel) on the way out.
#include <new>
#include <mutex>
#include <type_traits>
#include <vector>

#include "product.cuh"

namespace sp {

// ------------------------------------------------------------------ quantiser
// scale = max|x| / 127 (rounded once to fp32), q = the integer nearest to x / scale, halves to even.
//
// A quotient taken in fp32 can land on the wrong side of a half.  So the product with 1 / scale decides only where it is clear; next to a
// half the remainder x - q * scale decides, which is exact in fp32 there: x and q * scale are multiples of ulp(scale) / 2
// and differ by about scale / 2.
//
// Bound: one read of x, one write of q; each thread keeps its vectors of the row in registers, as they were read, between the two
// passes.  What it has to be careful with is instructions: 67 million elements at 18 each take longer than their bytes.
constexpr int kQuantThreads = 256;
constexpr int kQuantVecs = 4;        // vectors of 8 elements a thread holds

// Eight elements of a row as they lie in memory, their largest |x| as bits, and their values.
template <class T>
struct Vec8 {
  uint4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {      // 16-byte aligned
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
  }
  // 16-bit elements at any address, from the two 16-byte units that hold them (the caller has checked that both lie in the matrix): two reads
  // and a shift of (address modulo 16) bytes instead of eight reads.
  __device__ __forceinline__ void load_shifted(const T* p) {
    static_assert(sizeof(T) == 2, "");
    const uint4* at = reinterpret_cast<const uint4*>((uintptr_t)p & ~(uintptr_t)15);
    const uint4 a = __ldg(at), b = __ldg(at + 1);
    const uint32_t m = (uint32_t)(uintptr_t)p & 15u;
    const bool m8 = m & 8u, m4 = m & 4u;
    const uint32_t t[6] = {m8 ? a.z : a.x, m8 ? a.w : a.y, m8 ? b.x : a.z, m8 ? b.y : a.w, m8 ? b.z : b.x, m8 ? b.w : b.y};
    uint32_t o[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) o[i] = m4 ? t[i + 1] : t[i];
    const uint32_t sel = m & 2u ? 0x5432u : 0x3210u;
    w[0] = make_uint4(__byte_perm(o[0], o[1], sel), __byte_perm(o[1], o[2], sel), __byte_perm(o[2], o[3], sel), __byte_perm(o[3], o[4], sel));
  }
  __device__ __forceinline__ void load_some(const T* p, int n) {      // any address; elements from n on are zero
    uint32_t* u = reinterpret_cast<uint32_t*>(w);
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = i < n ? __ldg(reinterpret_cast<const uint32_t*>(p) + i) : 0u;
    } else {
      const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) u[i] = (2 * i < n ? (uint32_t)__ldg(h + 2 * i) : 0u) | (2 * i + 1 < n ? (uint32_t)__ldg(h + 2 * i + 1) << 16 : 0u);
    }
  }
  // Bits of |x| order like the values, infinities and NaN above all; 16-bit elements are compared in pairs.
  __device__ __forceinline__ uint32_t larger(uint32_t top) const {
    const uint32_t* u = reinterpret_cast<const uint32_t*>(w);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) * 2; i += 2) {
      if constexpr (sizeof(T) == 4) top = __vimax3_u32(top, u[i] & 0x7fffffffu, u[i + 1] & 0x7fffffffu);
      else top = __vimax3_u16x2(top, u[i] & 0x7fff7fffu, u[i + 1] & 0x7fff7fffu);
    }
    return top;
  }
  __device__ __forceinline__ void values(float (&v)[8]) const { values_as<T>(v); }
  template <class U>
  __device__ __forceinline__ void values_as(float (&v)[8]) const {
    const uint32_t* u = reinterpret_cast<const uint32_t*>(w);
    if constexpr (sizeof(U) == 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(u[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (std::is_same<U, __half>::value) {
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(u + i));
          v[2 * i] = f.x; v[2 * i + 1] = f.y;
        } else {
          v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
      }
    }
  }
};

// The row's largest |x| as a float from the bits above.
template <class T>
__device__ __forceinline__ float quant_top(uint32_t bits) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(bits);
  const uint32_t b = max(bits & 0xffffu, bits >> 16);
  if constexpr (std::is_same<T, __half>::value) return __half2float(__ushort_as_half((unsigned short)b));
  return __uint_as_float(b << 16);
}

struct QuantScale {
  float s, inv;
  bool zero;      // all q are zero: a row of zeros, or one that is not finite
  __device__ __forceinline__ QuantScale(float scale, float inverse) : s(scale), inv(inverse), zero(inverse < 0.f) {}   // made before; inverse -1: zero
  __device__ __forceinline__ explicit QuantScale(float top) {
    const bool bad = !(top <= 3.402823466e38f);
    s = bad ? __uint_as_float(0x7fffffffu) : __fdiv_rn(top, 127.f);
    zero = bad || s == 0.f;
    inv = s > 0x1p-100f && s < 0x1p100f ? 1.f / s : 0.f;    // 0: 1 / s may not be a normal number
  }
};

// Eight elements to 8 bits.  z = x / s + 384.5 lies in [257, 512), where fp32 has 15 bits behind the point: bits 15 to 22 of z are
// floor(x / s + 1/2) + 128, and z is off by less than its last bit, so that floor is right unless all 15 bits are zero.  Those
// elements (exact halves among them, which coarse types meet often: 0.7 % of bf16 normal numbers) are decided by the
// remainder.  No conversion instruction, of which an SM does few per clock.
__device__ __forceinline__ uint2 quant_pack(const float (&v)[8], const QuantScale& k) {
  uint32_t z[8], low = 0xffffffffu;
#pragma unroll
  for (int e = 0; e < 8; ++e) z[e] = __float_as_uint(fmaf(v[e], k.inv, 384.5f)) << 1;      // integer in byte 2, fraction in the low half
#pragma unroll
  for (int e = 0; e < 8; e += 4) low = __vimin3_u16x2(low, __byte_perm(z[e], z[e + 1], 0x5410), __byte_perm(z[e + 2], z[e + 3], 0x5410));
  if ((low & 0xffffu) == 0 || (low >> 16) == 0) {
    const float h = 0.5f * k.s;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // x / s is within 2^-15 of n - 1/2: n, or n - 1 where the remainder says so, or on a tie where n is odd
      const float n = __uint_as_float((z[e] >> 1) & 0xffff8000u | 0x43800000u) - 384.f;
      const float r = fmaf(-n, k.s, v[e]);
      if ((z[e] & 0xffffu) == 0 && (r < -h || (r == -h && (z[e] & 0x10000u)))) z[e] -= 0x10000u;
    }
  }
  return make_uint2(__byte_perm(__byte_perm(z[0], z[1], 0x0062), __byte_perm(z[2], z[3], 0x0062), 0x5410) ^ 0x80808080u,
                    __byte_perm(__byte_perm(z[4], z[5], 0x0062), __byte_perm(z[6], z[7], 0x0062), 0x5410) ^ 0x80808080u);
}

// One element of a row whose scale has no normal inverse.
static __device__ __noinline__ int8_t quant_by_remainder(float x, float s) {
  float n = fminf(fmaxf(rintf(__fdiv_rn(x, s)), -127.f), 127.f);
  const float r = fmaf(-n, s, x), two = 2.f * fabsf(r);
  if (two > s || (two == s && ((int)n & 1))) n += r > 0.f ? 1.f : -1.f;
  return (int8_t)(int)fminf(fmaxf(n, -127.f), 127.f);
}

// Elements [c, c + 8) of such a row.
template <class T>
__device__ __forceinline__ void quant_extreme(const T* row, int64_t c, int64_t cols, float s, int8_t* q) {
#pragma unroll 1
  for (int e = 0; e < 8; ++e, ++c) q[c] = c < cols ? quant_by_remainder((float)row[c], s) : (int8_t)0;
}

// TPR threads share a row: as few as hold it in registers (8192 x 4096 bf16: 128 threads 22.5 us, 256 27.6).
template <class T, int TPR>
__global__ void __launch_bounds__(kQuantThreads, sizeof(T) == 2 ? 5 : 4) quantize_kernel(const T* x, int rows, int64_t cols, int64_t kp, int8_t* q, float* scale) {
  pdl_begin();      // the few-token products fetch weights while this kernel runs: everything before it is complete
  constexpr int kRows = kQuantThreads / TPR;
  const int t = threadIdx.x % TPR;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
  const bool live = row < rows;
  const T* xr = x + (live ? row : 0) * cols;
  const int nvec = live ? (int)(kp / 8) : 0;
  const int nfull = (((uintptr_t)x | (uintptr_t)(cols * (int64_t)sizeof(T))) & 15u) == 0 ? (int)(cols / 8) : 0;   // vectors read whole
  const uintptr_t end = (uintptr_t)(x + rows * cols);
  auto load = [&](int j, Vec8<T>& w) {
    const T* p = xr + (int64_t)j * 8;
    if (j < nfull) {
      w.load(p);
      return;
    }
    if constexpr (sizeof(T) == 2) {
      const uintptr_t unit = (uintptr_t)p & ~(uintptr_t)15;
      if ((int64_t)j * 8 + 8 <= cols && unit >= (uintptr_t)x && unit + 32 <= end) {
        w.load_shifted(p);
        return;
      }
    }
    w.load_some(p, (int)min((int64_t)8, max((int64_t)0, cols - (int64_t)j * 8)));
  };
  Vec8<T> v[kQuantVecs];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kQuantVecs; ++i)
    if (t + i * TPR < nvec) load(t + i * TPR, v[i]);
#pragma unroll
  for (int i = 0; i < kQuantVecs; ++i)
    if (t + i * TPR < nvec) top = v[i].larger(top);
  for (int j = t + kQuantVecs * TPR; j < nvec; j += TPR) {   // long rows: read again below
    Vec8<T> w;
    load(j, w);
    top = w.larger(top);
  }
  uint32_t big = __reduce_max_sync(0xffffffffu, __float_as_uint(quant_top<T>(top)));
  if constexpr (TPR > 32) {
    __shared__ uint32_t part[kQuantThreads / 32];
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = big;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TPR / 32; ++i) big = max(big, part[threadIdx.x / TPR * (TPR / 32) + i]);
  }
  if (!live) return;
  const QuantScale k(__uint_as_float(big));
  if (t == 0) scale[row] = k.s;
  int8_t* qr = q + row * kp;
  if (k.zero) {
    for (int j = t; j < nvec; j += TPR) *reinterpret_cast<uint2*>(qr + (int64_t)j * 8) = make_uint2(0u, 0u);
    return;
  }
  if (k.inv == 0.f) {
    for (int j = t; j < nvec; j += TPR) quant_extreme(xr, (int64_t)j * 8, cols, k.s, qr);
    return;
  }
  auto store = [&](int j, const Vec8<T>& w) {
    float f[8];
    w.values(f);
    *reinterpret_cast<uint2*>(qr + (int64_t)j * 8) = quant_pack(f, k);
  };
#pragma unroll
  for (int i = 0; i < kQuantVecs; ++i)
    if (t + i * TPR < nvec) store(t + i * TPR, v[i]);
  for (int j = t + kQuantVecs * TPR; j < nvec; j += TPR) {
    Vec8<T> w;
    load(j, w);
    store(j, w);
  }
}

// ------------------------------------------------------------------ epilogue of the tiled product
// PLAIN: rows of C that a bulk store cannot take.
// c = (float(acc) * a_scale[row]) * b_scale[col]: the integer rounds once to fp32, then one rounding per factor (the two
// scales are not multiplied first: their product can leave fp32's range where the result does not).
template <bool OUT_F32, bool PLAIN>
struct EpiI8 {
  static constexpr uint32_t kBytes = 8 * 4096 + (PLAIN ? 8 * 512 : 0);   // staging, then what rows without bulk stores carry from slice to slice
  static constexpr bool kSums = false;
  static constexpr bool kLive = false;
  struct Args {
    const float* a_scale;
    const float* b_scale;
    char* C;
    int64_t ld_bytes;
    int bf16;     // 16-bit output: bf16, else fp16
  };
  const Args& a;
  const CUtensorMap* map;
  EpiStage stage;
  uint32_t carry;
  int lane;
  float rs;
  float bs[4];      // column scales: column 32 i + lane
  __device__ EpiI8(const Args& args, const CUtensorMap* m, uint32_t base, int w, int l)
      : a(args), map(m), stage{base + (uint32_t)w * 4096u, l}, carry(base + 32768u + (uint32_t)w * 512u), lane(l) {}
  __device__ __forceinline__ void before(const EpiTile& e, int M, int N) {
    rs = e.row0 + lane < M ? __ldg(a.a_scale + e.row0 + lane) : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) bs[i] = e.col0 + 32 * i + lane < N ? __ldg(a.b_scale + e.col0 + 32 * i + lane) : 0.f;
  }
  template <int COLS>
  __device__ __forceinline__ void finish(uint32_t (&v)[COLS], const EpiTile& e, int M, int N) {
    // the column scales pass through the (free) slice: every lane needs all of them
    const uint32_t slice = stage.free();
#pragma unroll
    for (int i = 0; i < COLS / 32; ++i) asm volatile("st.shared.f32 [%0], %1;" ::"r"(slice + i * 128 + lane * 4), "f"(bs[i]) : "memory");
    __syncwarp();
#pragma unroll
    for (int j = 0; j < COLS / 4; ++j) {
      float4 f;
      asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w) : "r"(slice + j * 16));
      v[4 * j] = __float_as_uint((float)(int)v[4 * j] * rs * f.x);
      v[4 * j + 1] = __float_as_uint((float)(int)v[4 * j + 1] * rs * f.y);
      v[4 * j + 2] = __float_as_uint((float)(int)v[4 * j + 2] * rs * f.z);
      v[4 * j + 3] = __float_as_uint((float)(int)v[4 * j + 3] * rs * f.w);
    }
    __syncwarp();
    constexpr int kCols = OUT_F32 ? 32 : 64;
#pragma unroll
    for (int q = 0; q < COLS / kCols; ++q) {
      uint32_t p[32];
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        if constexpr (OUT_F32) p[j] = v[q * 32 + j];
        else p[j] = pack_16(__uint_as_float(v[q * 64 + 2 * j]), __uint_as_float(v[q * 64 + 2 * j + 1]), a.bf16);
      }
      if (q) stage.free();
      stage_row(slice, lane, p);
      const int col = e.col0 + q * kCols;
      const bool inside = e.row0 < M && col < N;
      if constexpr (PLAIN) {
        constexpr int kElt = OUT_F32 ? 4 : 2;
        if (inside) store_slice_plain<kElt>(carry, slice, lane, a.C, a.ld_bytes, e.row0, col, M, min(128, (N - col) * kElt), q == 0,
                                            q == COLS / kCols - 1 || col + kCols >= N);
      } else {
        fence_async_smem();
        __syncwarp();
        if (lane == 0 && inside) {
          tma_store_2d(map, slice, col, e.row0);
          bulk_commit();
        }
      }
    }
  }
};

// One result, rounded to the output's type.
__device__ __forceinline__ void store_y(char* C, int out, int64_t at, float y) {
  if (out == SP_FP32) reinterpret_cast<float*>(C)[at] = y;
  else if (out == SP_BF16) reinterpret_cast<__nv_bfloat16*>(C)[at] = __float2bfloat16_rn(y);
  else reinterpret_cast<__half*>(C)[at] = __float2half_rn(y);
}

// ------------------------------------------------------------------ a handful of tokens
// One or two tokens, or up to four under a small matrix: what counts is the time from launch to the first weight and from the last
// weight to the result.  So no tensor memory, barriers or clusters: a warp takes two weight rows, asks for 4 KiB of each at
// once (16 bytes per lane and load, straight to registers), multiplies them with the tokens in shared memory four bytes at a
// time, and sums over the warp.  Two blocks per SM walk the rows with a fixed stride.  Where the tokens are short and 16-bit,
// each block quantises them itself while its first weights are on their way: a launch less.
// Measured (us; weights from HBM; the few-token form below in brackets): 1 x 1024 x 1024 2.6 (4.1), 1 x 4096 x 4096 4.6 (6.8), 4 x 4096 x 4096
// 5.7 (6.8), 1 x 8192 x 8192 13.7 (14.7), 4 x 16384 x 8192 27.4 (25.2), 8 x 8192 x 8192 21.5 (15.0): every token costs the
// integer units as much again.
constexpr int kDotThreads = 256, kDotUnroll = 8, kDotTokens = 4;
constexpr int64_t kDotAlways = 2;           // tokens up to which this form is taken whatever the matrix ...
constexpr int64_t kDotWeights = 1 << 25;    // ... and bytes of weights up to which it is for kDotTokens
constexpr int64_t kDotBytes = 65536;        // tokens x K that a block holds
constexpr int64_t kDotQuantize = 4096;      // tokens x K up to which a block quantises for itself
constexpr int kDotVecs = (int)(kDotQuantize / 8 / kDotThreads);

struct DotArgs {
  const int8_t* W;
  const float* w_scale;
  const int8_t* q;        // tokens, already 8 bits ...
  const float* q_scale;
  const uint16_t* x;      // ... or not (QUANT): quantised here, into q_out and scale_out as well
  int x_bf16;             // bf16, else fp16
  int64_t cols;           // of x
  int8_t* q_out;
  float* scale_out;
  char* C;
  int M, N, K;
  int out;
  int early;              // as FewArgs
};

// The tokens to 8 bits, by the whole block.  Their vectors were asked for before the first weights: behind those they would arrive last.
__device__ __forceinline__ void dot_fetch_tokens(const DotArgs& a, Vec8<uint16_t> (&v)[kDotVecs]) {
  const int nvec = a.K / 8, total = a.M * nvec;
  const bool aligned = (((uintptr_t)a.x | (uintptr_t)(a.cols * 2)) & 15u) == 0;
#pragma unroll
  for (int i = 0; i < kDotVecs; ++i) {
    const int at = (int)threadIdx.x + i * kDotThreads;
    if (at < total) {
      const int m = at / nvec, j = at - m * nvec;
      const uint16_t* p = a.x + (int64_t)m * a.cols + (int64_t)j * 8;
      const int n = (int)min((int64_t)8, max((int64_t)0, a.cols - (int64_t)j * 8));
      if (n == 8 && aligned) v[i].load(p);
      else v[i].load_some(p, n);
    }
  }
}

__device__ __forceinline__ float dot_top(uint32_t bits, int bf16) { return bf16 ? quant_top<__nv_bfloat16>(bits) : quant_top<__half>(bits); }

__device__ __forceinline__ void dot_quantize(const DotArgs& a, const Vec8<uint16_t> (&v)[kDotVecs], int8_t* tokens, float* scales, float* inverses, uint32_t* tops) {
  const int nvec = a.K / 8, total = a.M * nvec, lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < kDotVecs; ++i) {
    const int first = (int)threadIdx.x - lane + i * kDotThreads;      // of this warp
    if (first < total) {
      const int at = first + lane, m = at / nvec;
      const uint32_t top = at < total ? __float_as_uint(dot_top(v[i].larger(0u), a.x_bf16)) : 0u;
      if (first / nvec == (first + 31) / nvec) {       // the warp is inside one row
        const uint32_t all = __reduce_max_sync(0xffffffffu, top);
        if (lane == 0) atomicMax(tops + m, all);
      } else if (at < total) {
        atomicMax(tops + m, top);
      }
    }
  }
  __syncthreads();
  if (threadIdx.x < (unsigned)a.M) {
    const QuantScale k(__uint_as_float(tops[threadIdx.x]));
    scales[threadIdx.x] = k.s;
    inverses[threadIdx.x] = k.zero ? -1.f : k.inv;
    if (blockIdx.x == 0) a.scale_out[threadIdx.x] = k.s;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kDotVecs; ++i) {
    const int at = (int)threadIdx.x + i * kDotThreads;
    if (at < total) {
      const int m = at / nvec, j = at - m * nvec;
      const QuantScale k(scales[m], inverses[m]);
      uint2 b = make_uint2(0u, 0u);
      if (!k.zero) {
        float f[8];
        if (a.x_bf16) v[i].template values_as<__nv_bfloat16>(f);
        else v[i].template values_as<__half>(f);
        if (k.inv != 0.f) {
          b = quant_pack(f, k);
        } else {
          uint64_t bytes = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) bytes |= (uint64_t)(uint8_t)quant_by_remainder(f[e], k.s) << (8 * e);
          b = make_uint2((uint32_t)bytes, (uint32_t)(bytes >> 32));
        }
      }
      *reinterpret_cast<uint2*>(tokens + (int64_t)m * a.K + (int64_t)j * 8) = b;
      if (blockIdx.x == 0) *reinterpret_cast<uint2*>(a.q_out + (int64_t)m * a.K + (int64_t)j * 8) = b;
    }
  }
}

// QUANT: the tokens are quantised here (its registers would cost the other form half a microsecond).
template <int MT, bool QUANT>
__global__ void __launch_bounds__(kDotThreads, 2) dot_tokens_kernel(const DotArgs a) {
  extern __shared__ __align__(16) int8_t dot_tokens[];     // MT rows of K bytes; rows beyond M are read and not used
  __shared__ float scales[kDotTokens], inverses[kDotTokens];
  __shared__ uint32_t tops[kDotTokens];
  const int lane = threadIdx.x & 31, warp = blockIdx.x * (kDotThreads / 32) + (threadIdx.x >> 5);
  const int step = gridDim.x * (kDotThreads / 32) * 2;
  int4 w[2][kDotUnroll];
  auto fetch = [&](int64_t n, int k) {     // bytes [k, k + 4096) of rows n and n + 1
#pragma unroll
    for (int u = 0; u < kDotUnroll; ++u)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int c = k + u * 512 + lane * 16;
        w[r][u] = n + r < a.N && c < a.K ? __ldcs(reinterpret_cast<const int4*>(a.W + (n + r) * a.K + c)) : make_int4(0, 0, 0, 0);
      }
  };
  Vec8<uint16_t> own[QUANT ? kDotVecs : 1];
  if (!a.early) pdl_begin();
  if constexpr (QUANT) dot_fetch_tokens(a, own);
  fetch(warp * 2, 0);
  if (a.early) pdl_begin();
  if constexpr (QUANT) {
    if (threadIdx.x < kDotTokens) tops[threadIdx.x] = 0;
    __syncthreads();
    dot_quantize(a, own, dot_tokens, scales, inverses, tops);
  } else {
    for (int i = threadIdx.x; i < a.M * (a.K / 16); i += kDotThreads)
      reinterpret_cast<int4*>(dot_tokens)[i] = __ldg(reinterpret_cast<const int4*>(a.q) + i);
    if (threadIdx.x < a.M) scales[threadIdx.x] = __ldg(a.q_scale + threadIdx.x);
  }
  __syncthreads();
  for (int64_t n = (int64_t)warp * 2; n < a.N; n += step) {
    int acc[2][MT] = {};
    for (int k = 0; k < a.K; k += kDotUnroll * 512) {
#pragma unroll
      for (int u = 0; u < kDotUnroll; ++u) {
        const int c = k + u * 512 + lane * 16;
        if (c < a.K) {
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const int4 x = *reinterpret_cast<const int4*>(dot_tokens + m * a.K + c);
#pragma unroll
            for (int r = 0; r < 2; ++r)
              acc[r][m] = __dp4a(w[r][u].x, x.x, __dp4a(w[r][u].y, x.y, __dp4a(w[r][u].z, x.z, __dp4a(w[r][u].w, x.w, acc[r][m]))));
          }
        }
      }
      if (k + kDotUnroll * 512 < a.K) fetch(n, k + kDotUnroll * 512);
      else if (n + step < a.N) fetch(n + step, 0);
    }
    int mine = 0;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int sum = __reduce_add_sync(0xffffffffu, acc[r][m]);
        if (lane == 2 * m + r) mine = sum;
      }
    const int m = lane >> 1;
    const int64_t col = n + (lane & 1);
    if (m < a.M && col < a.N) store_y(a.C, a.out, (int64_t)m * a.N + col, (float)mine * scales[m] * __ldg(a.w_scale + col));
  }
}

// ------------------------------------------------------------------ few tokens
// At most NT rows of A: the call is bound by reading the weights once, so the weights take the 128-row side of the MMA and the
// tokens its N side, and the k axis of each 128-row block is split over the S CTAs of a cluster to occupy every SM.  The
// partial sums are integers: they meet through distributed shared memory, in any order with one result.
// Measured (us; as tiles in brackets): 16 x 4096 x 4096 6.6 (12.3), 24 x 16384 x 8192 26.0 (28.6), 64 x 1024 x 1024 5.1 (6.1), 128 x 4096 x 4096 10.9
// (12.9), 256 x 4096 x 11008 20.0 (28.9); on the other side of the rule 128 x 1024 x 1024 6.7 (6.1), 128 x 11008 x 4096 17.7 (14.4).
template <int NT>
struct FewCfg {
  static constexpr uint32_t kWBytes = 128 * 128, kQBytes = NT * 128, kStageBytes = kWBytes + kQBytes;
  static constexpr int kPerSm = NT > 128 ? 1 : 2;                     // CTAs per SM
  static constexpr int kFit = (229376 / kPerSm - 1024 - 512) / kStageBytes;
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


template <int NT>
__global__ void __launch_bounds__(192, FewCfg<NT>::kPerSm)
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
    // Blocks start their walk along k at different places: they all read the same few lines of the tokens, and in step would queue for
    // them in one L2 slice.
    const int n_k = k1 - k0, turn = (int)(blockIdx.x / nranks) * 5 % n_k;
    auto k_at = [&](int i) { return (k0 + (i + turn < n_k ? i + turn : i + turn - n_k)) * 128; };
    const int ahead = min(S, k1 - k0);
    if (!args.early) pdl_begin();
    if (elect_one()) {
      for (int i = 0; i < ahead; ++i) {
        mbar_arrive_expect_tx(bar_full + 8 * i, C::kStageBytes);
        tma_load_2d<1>(stage_addr(i), &tmW, k_at(i), n0, bar_full + 8 * i);
      }
    }
    __syncwarp();
    if (args.early) pdl_begin();
    if (elect_one()) {
      for (int i = 0; i < ahead; ++i) tma_load_2d<1>(stage_addr(i) + C::kWBytes, &tmQ, k_at(i), 0, bar_full + 8 * i);
    }
    __syncwarp();
    for (int i = S; i < k1 - k0; ++i) {
      const int st = i % S;
      ok = mbar_wait(bar_empty + 8 * st, (uint32_t)(i / S - 1) & 1u, args.status, (kProdProducer << 8) | 3);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      if (elect_one()) {
        mbar_arrive_expect_tx(bar_full + 8 * st, C::kStageBytes);
        tma_load_2d<1>(stage_addr(i), &tmW, k_at(i), n0, bar_full + 8 * st);
        tma_load_2d<1>(stage_addr(i) + C::kWBytes, &tmQ, k_at(i), 0, bar_full + 8 * st);
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
    pdl_begin();
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
    pdl_begin();
    const int quarter = warp & 3;
    bool ok = mbar_wait(bar_done, 0, args.status, (kProdEpilogue << 8) | 3);
    ok = __all_sync(0xffffffffu, ok);
    tcgen05_fence_after();
    if (ok) {
      // [token][row of W] in shared memory, over the stages; a short loop: code that runs once costs its own loading (unrolled over the tokens:
      // 125 cycles per token, 128 x 4096 x 4096 17.4 us)
#pragma unroll 1
      for (int q = 0; q < (args.M + 31) / 32; ++q) {
        uint32_t v[32];
        tmem_ld_32x32b_x32(tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(q * 32), v);
        tmem_ld_wait();
        const uint32_t at = smem_base + (uint32_t)(q * 32 * 128 + quarter * 32 + lane) * 4u;
#pragma unroll
        for (int j = 0; j < (NT < 32 ? NT : 32); ++j) asm volatile("st.shared.b32 [%0], %1;" ::"r"(at + j * 512u), "r"(v[j]) : "memory");
      }
    }
  }
  tcgen05_fence_before();
  __syncwarp();
  if (nranks > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  } else {
    __syncthreads();
  }
  if (warp >= 2) {
    // Each CTA of the cluster finishes every S-th token: a warp per token, four rows per lane, the reads of all partial sums in flight
    // together (one element at a time, trip after trip between SMs, 24 tokens x 16384 x 8192 took 36 us).
    const int row = lane * 4, n = n0 + row;
    float bs[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) bs[i] = n + i < args.N ? __ldg(args.b_scale + n + i) : 0.f;
    const bool whole = n + 3 < args.N && (args.N & 3) == 0 && ((uintptr_t)args.C & 15u) == 0;
#pragma unroll 2
    for (int tok = (int)rank + (warp - 2) * (int)nranks; tok < args.M; tok += 4 * (int)nranks) {
      const float as = __ldg(args.a_scale + tok);
      int p[8][4];
#pragma unroll
      for (uint32_t r = 0; r < 8; ++r) {
        p[r][0] = p[r][1] = p[r][2] = p[r][3] = 0;
        if (r < nranks)
          asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(p[r][0]), "=r"(p[r][1]), "=r"(p[r][2]), "=r"(p[r][3])
                       : "r"(mapa(smem_base, r) + (uint32_t)(tok * 128 + row) * 4u));
      }
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        int acc = 0;
#pragma unroll
        for (int r = 0; r < 8; ++r) acc += p[r][i];
        y[i] = (float)acc * as * bs[i];
      }
      const int64_t at = (int64_t)tok * args.N + n;
      if (whole) {
        if (args.out == SP_FP32) *reinterpret_cast<float4*>(args.C + at * 4) = make_float4(y[0], y[1], y[2], y[3]);
        else *reinterpret_cast<uint2*>(args.C + at * 2) = make_uint2(pack_16(y[0], y[1], args.out == SP_BF16), pack_16(y[2], y[3], args.out == SP_BF16));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (n + i < args.N) store_y(args.C, args.out, at + i, y[i]);
      }
    }
  }
  __syncwarp();
  if (nranks > 1) {      // nobody leaves while a peer may read its partial sums
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
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
  const auto run = [&](auto tpr) {
    constexpr int kTpr = decltype(tpr)::value;
    return launch_pdl("quantize", quantize_kernel<T, kTpr>, dim3((unsigned)((M + kQuantThreads / kTpr - 1) / (kQuantThreads / kTpr))), kQuantThreads, 0, 1,
                      stream, (const T*)x, (int)M, K, kp, q, scale);
  };
  const int64_t held = (kp + 8 * kQuantVecs - 1) / (8 * kQuantVecs);      // threads that hold a row
  if (held <= 32) return run(std::integral_constant<int, 32>());
  if (held <= 64) return run(std::integral_constant<int, 64>());
  if (held <= 128) return run(std::integral_constant<int, 128>());
  return run(std::integral_constant<int, kQuantThreads>());
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
  bool plain;           // rows of C that a bulk store cannot take
  Sched sched;
  std::vector<int32_t> host_perm;
};

// The few-token form: always up to 64 tokens; up to 256 where 128 x 128 tiles would occupy less than half of the SMs and k is long enough to split.
constexpr int64_t kFewAlways = 64, kFewTokens = 256;

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
  if (!pick && !((tile_m == 256 && tile_n == 256) || (tile_m == 128 && tile_n == 128))) {
    set_error("unsupported tile %dx%d (supported: 128x128, 256x256)", tile_m, tile_n);
    return SP_ERR_UNSUPPORTED;
  }
  if (pick && scheme == kCustom) { set_error("SP_CUSTOM needs tile_m and tile_n: its table is that grid's"); return SP_ERR_INVALID_ARG; }
  call->A = A; call->B = B; call->a_scale = (const float*)a_scale; call->b_scale = (const float*)b_scale; call->C = const_cast<void*>(C);
  call->M = M; call->N = N; call->K = K; call->out = out;
  call->few = scheme == SP_ORDER_AUTO && pick && (M <= kFewAlways || (M <= kFewTokens && K >= 2048 && (M + 127) / 128 * ((N + 127) / 128) <= 64));
  if (call->few) return SP_OK;
  const int64_t ld = N * (int64_t)elt_bytes(out);
  call->plain = ((uintptr_t)C & 15u) || (ld & 15);
  if (pick) {
    // 256 rows by the width that fills the waves best (bulk stores of 16-bit results come in 64 columns), or 128 x 128 where that is less: a tile of
    // 128 x 128 runs at 0.70 of the rate of 256 x 256 (4096^3 and 8192^3)
    tile_m = 256;
    tile_n = tile_width(M, N, 2, out == SP_FP32 || call->plain ? 32 : 64);
    const auto waves = [&](int tm, int tn, int units) { return (double)((((M + tm - 1) / tm) * ((N + tn - 1) / tn) + units - 1) / units); };
    if (waves(128, 128, 148) * 128 * 128 * (304.0 / 256) / 0.70 < waves(256, tile_n, 74) * 128 * (tile_n + 48)) tile_m = tile_n = 128;
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

template <int MT, bool QUANT>
static int launch_dot(const DotArgs& a, cudaStream_t stream) {
  auto kern = dot_tokens_kernel<MT, QUANT>;
  static uint64_t configured = 0;
  if (first_use_on_this_device(configured)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kDotBytes);
    if (e != cudaSuccess) { configured = 0; set_error("cudaFuncSetAttribute failed: %s", cudaGetErrorString(e)); return SP_ERR_CUDA; }
  }
  const int64_t blocks = (a.N + 15) / 16;
  return launch_pdl("dot products", kern, dim3((unsigned)(blocks < 2 * 148 ? blocks : 2 * 148)), kDotThreads, (size_t)MT * a.K, 1, stream, a);
}

// The tokens come quantised (x == nullptr) or are quantised by every block.
static int run_dot(const I8Call& c, const void* x, int x_dtype, int64_t cols, bool early, cudaStream_t stream) {   // x: bf16 or fp16
  DotArgs a = {};
  a.W = (const int8_t*)c.B; a.w_scale = c.b_scale; a.q = (const int8_t*)c.A; a.q_scale = c.a_scale;
  a.x = (const uint16_t*)x; a.x_bf16 = x_dtype == SP_BF16; a.cols = cols; a.q_out = (int8_t*)const_cast<void*>(c.A); a.scale_out = const_cast<float*>(c.a_scale);
  a.C = (char*)c.C; a.M = (int)c.M; a.N = (int)c.N; a.K = (int)c.K; a.out = c.out; a.early = early ? 1 : 0;
  if (c.M <= 1) return x ? launch_dot<1, true>(a, stream) : launch_dot<1, false>(a, stream);
  if (c.M <= 2) return x ? launch_dot<2, true>(a, stream) : launch_dot<2, false>(a, stream);
  return x ? launch_dot<4, true>(a, stream) : launch_dot<4, false>(a, stream);
}

static bool takes_dot(const I8Call& c) {
  const int64_t mt = c.M <= 2 ? c.M : 4;      // rows of shared memory
  return c.few && (c.M <= kDotAlways || (c.M <= kDotTokens && c.N * c.K <= kDotWeights)) && mt * c.K <= kDotBytes;
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
  // as many slices of k as the CTAs that run at once allow, each with at least two stages of work
  int split = 1;
  while (split < 8 && blocks * split * 2 <= C::kPerSm * 148 && args.kblocks >= split * 2 * 2) split *= 2;
  args.kb_split = (args.kblocks + split - 1) / split;
  while (split > 1 && (split - 1) * args.kb_split >= args.kblocks) { split /= 2; args.kb_split = (args.kblocks + split - 1) / split; }   // every slice has work
  args.idesc = idesc_i8(128, NT);
  return launch_pdl("few-token product", kern, dim3((unsigned)(blocks * split)), 192, C::kSmemBytes, split, stream, tmW, tmQ, args);
}

template <bool OUT_F32, bool PLAIN>
static int launch_tiles(const I8Call& c, const ProdArgs& pa, const CUtensorMap& tmA, const CUtensorMap& tmB, const CUtensorMap& tmC, cudaStream_t stream) {
  using Epi = EpiI8<OUT_F32, PLAIN>;
  const typename Epi::Args ea = {c.a_scale, c.b_scale, (char*)c.C, c.N * (OUT_F32 ? 4 : 2), c.out == SP_BF16};
  if (c.tile_m == 256) return launch_product<2, 256, kElemI8, false, false, Epi>("8-bit product", tmA, tmB, tmC, pa, false, ea, stream);
  return launch_product<1, 128, kElemI8, false, false, Epi>("8-bit product", tmA, tmB, tmC, pa, false, ea, stream);
}

static int run_i8(const I8Call& c, bool early, cudaStream_t stream) {
  if (takes_dot(c)) return run_dot(c, nullptr, 0, 0, early, stream);
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
    if (c.M <= 128) return launch_few<128>(c, tmB, a, stream);
    return launch_few<256>(c, tmB, a, stream);
  }
  ProdArgs pa = {};
  pa.perm = st.perm; pa.status = st.status; pa.M = (int)c.M; pa.N = (int)c.N; pa.bn = c.tile_n;
  pa.kblocks = (int)((c.K + 127) / 128); pa.splits = 1;
  pa.sched = c.sched;
  const int cg = c.tile_m / 128;
  rc = make_map_any(&tmA, c.A, 1, c.M, c.K, c.K, 128, 128);
  if (rc == SP_OK) rc = make_map_any(&tmB, c.B, 1, c.N, c.K, c.K, c.tile_n / cg, 128);
  if (rc != SP_OK) return rc;
  const int elt = (int)elt_bytes(c.out);
  if (c.plain) tmC = tmB;    // not used
  else rc = make_map_any(&tmC, c.C, elt, c.M, c.N, c.N, 32, 128 / elt);
  if (rc != SP_OK) return rc;
  if (c.out == SP_FP32) return c.plain ? launch_tiles<true, true>(c, pa, tmA, tmB, tmC, stream) : launch_tiles<true, false>(c, pa, tmA, tmB, tmC, stream);
  return c.plain ? launch_tiles<false, true>(c, pa, tmA, tmB, tmC, stream) : launch_tiles<false, false>(c, pa, tmA, tmB, tmC, stream);
}

}  // namespace sp

using namespace sp;

using Bytes = unsigned __int128;

extern "C" {

int sp_quantize_i8(const void* x, int32_t x_dtype, int64_t M, int64_t K, int8_t* q, float* scale, void* stream) {
  int rc = check_quantize(x, x_dtype, M, K, q, scale);
  if (rc != SP_OK) return rc;
  const Span spans[] = {{"q", q, (Bytes)M * (Bytes)((K + 15) / 16 * 16)}, {"scale", scale, (Bytes)M * 4}, {"x", x, (Bytes)M * (Bytes)K * elt_bytes(x_dtype)}};
  rc = refuse_overlaps(spans, 2, 3);
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
  const Span spans[] = {{"C", C, (Bytes)M * (Bytes)N * elt_bytes(call.out)}, {"A", A, (Bytes)M * (Bytes)K}, {"a_scale", a_scale, (Bytes)M * 4},
                        {"B", B, (Bytes)N * (Bytes)K}, {"b_scale", b_scale, (Bytes)N * 4}};
  rc = refuse_overlaps(spans, 1, 5);
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
  const int64_t kp = (K + 15) / 16 * 16;
  rc = check_i8(q, q_scale, W, w_scale, y, M, N, kp, scheme, params, &call);
  if (rc != SP_OK) return rc;
  const Span spans[] = {{"y", y, (Bytes)M * (Bytes)N * elt_bytes(call.out)}, {"q", q, (Bytes)M * (Bytes)kp}, {"q_scale", q_scale, (Bytes)M * 4},
                        {"x", x, (Bytes)M * (Bytes)K * elt_bytes(x_dtype)}, {"W", W, (Bytes)N * (Bytes)kp}, {"w_scale", w_scale, (Bytes)N * 4}};
  rc = refuse_overlaps(spans, 3, 6);
  if (rc != SP_OK) return rc;
  int dev = 0;
  rc = current_device(&dev);
  if (rc != SP_OK) return rc;
  std::lock_guard<std::mutex> lock(g_i8_mu);
  if (takes_dot(call) && M * call.K <= kDotQuantize && x_dtype != SP_FP32) return run_dot(call, x, x_dtype, K, false, (cudaStream_t)stream);
  rc = quantize(x, x_dtype, M, K, q, q_scale, (cudaStream_t)stream);
  if (rc != SP_OK) return rc;
  return run_i8(call, true, (cudaStream_t)stream);
} catch (const std::exception& e) {
  set_error("sp_linear_i8: %s", e.what());
  return SP_ERR_CUDA;
}

}  // extern "C"
