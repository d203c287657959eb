// Device code shared by the FP8 kernels: a lane's piece of a row, its largest magnitude, its cast and where scales lie.
#pragma once

#include <cuda_fp8.h>

#include <atomic>

#include "btx_fp8.cuh"
#include "btx_route_dev.cuh"

namespace btx {
namespace fp8 {
namespace {

constexpr unsigned kAll = 0xffffffffu;

// Two fp32 numbers in a pair of registers, and the instructions that work on both.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b) {
  f32x2 d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ void unpack2(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// N elements of a lane as they were loaded, two of bf16 or one of fp32 per word.
template <typename T, int N> struct Piece {
  static constexpr int WORDS = N * (int)sizeof(T) / 4;
  uint32_t w[WORDS];

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = 0;
  }
  // the first n (any number) of N elements; vec: p is on a 16-byte boundary
  __device__ __forceinline__ void load(const T* p, int n, bool vec) {
    if (vec && n >= N) {
#pragma unroll
      for (int i = 0; i < WORDS; i += 4) {
        const uint4 q = __ldcs(reinterpret_cast<const uint4*>(p) + i / 4);
        w[i] = q.x; w[i + 1] = q.y; w[i + 2] = q.z; w[i + 3] = q.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        if (sizeof(T) == 4) {
          w[i] = i < n ? __float_as_uint(to_f32(p[i])) : 0u;
        } else {
          const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
          w[i] = (2 * i < n ? (uint32_t)h[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)h[2 * i + 1] << 16 : 0u);
        }
      }
    }
  }
  __device__ __forceinline__ void store(T* p, int n, bool vec) const {
    if (vec && n >= N) {
#pragma unroll
      for (int i = 0; i < WORDS; i += 4) __stcs(reinterpret_cast<uint4*>(p) + i / 4, make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]));
    } else {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        if (sizeof(T) == 4) {
          if (i < n) reinterpret_cast<uint32_t*>(p)[i] = w[i];
        } else {
          uint16_t* h = reinterpret_cast<uint16_t*>(p);
          if (2 * i < n) h[2 * i] = (uint16_t)w[i];
          if (2 * i + 1 < n) h[2 * i + 1] = (uint16_t)(w[i] >> 16);
        }
      }
    }
  }
  __device__ __forceinline__ void values(float (&v)[N]) const {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      if (sizeof(T) == 4) {
        v[i] = __uint_as_float(w[i]);
      } else {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ void set(const float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      if (sizeof(T) == 4) {
        w[i] = __float_as_uint(v[i]);
      } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
  }
  __device__ __forceinline__ void pairs(f32x2 (&v)[N / 2]) const {
    float f[N];
    values(f);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) v[i] = pack2(f[2 * i], f[2 * i + 1]);
  }
  __device__ __forceinline__ void set(const f32x2 (&v)[N / 2]) {
    float f[N];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) unpack2(v[i], f[2 * i], f[2 * i + 1]);
    set(f);
  }
  // largest magnitude as the bits of a float (NaN and infinities compare above every number)
  __device__ __forceinline__ uint32_t amax() const {
    uint32_t m = 0;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) m = max(m, w[i] & 0x7fffffffu);
      return m;
    } else {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
      return max(m & 0xffff0000u, m << 16);
    }
  }
};

__device__ __forceinline__ float max_abs(float a, float b) {       // NaN if either is
  float d;
  asm("{\n\t.reg .f32 x, y;\n\tabs.f32 x, %1;\n\tabs.f32 y, %2;\n\tmax.NaN.f32 %0, x, y;\n\t}" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
template <int N> __device__ __forceinline__ uint32_t amax_of(const float (&v)[N]) {
  float m[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) m[i] = max_abs(v[2 * i], v[2 * i + 1]);
#pragma unroll
  for (int k = N / 4; k > 0; k /= 2)
#pragma unroll
    for (int i = 0; i < k; ++i) m[i] = max_abs(m[i], m[i + k]);
  return __float_as_uint(m[0]) & 0x7fffffffu;
}
// the largest over groups of LANES neighbouring lanes
template <int LANES> __device__ __forceinline__ uint32_t lanes_max(uint32_t m) {
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) m = max(m, __shfl_xor_sync(kAll, m, o));
  return m;
}

__device__ __forceinline__ uint32_t codes2(float a, float b) { return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3); }
// N codes of a lane's elements, whose block's scale byte is `byte` (255: a block that is not a number has codes 0)
template <int N> __device__ __forceinline__ void cast_codes(const float (&v)[N], uint32_t byte, uint32_t inv_bits, uint32_t (&q)[N / 4]) {
  const f32x2 inv = pack2(__uint_as_float(inv_bits), __uint_as_float(inv_bits));
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    float a, b, c, d;
    unpack2(mul2(pack2(v[4 * i], v[4 * i + 1]), inv), a, b);
    unpack2(mul2(pack2(v[4 * i + 2], v[4 * i + 3]), inv), c, d);
    q[i] = byte == 255u ? 0u : codes2(a, b) | codes2(c, d) << 16;
  }
}
__device__ __forceinline__ float scale_value(uint32_t byte) {
  return __uint_as_float(byte == 255u ? 0x7fffffffu : (byte == 0u ? 0x00400000u : byte << 23));
}

// byte of the scale of row `row` (of a matrix whose first row tile is tile0), elements `block` * 128 ..
__device__ __forceinline__ size_t scale_offset(size_t tile0, int row, int kt, int block) {
  return ((tile0 + row / kTileRows) * (size_t)kt + block / 4) * kTileBytes + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}

// once per device and kernel: the attribute outlives the call
inline bool allow_smem(const void* kernel, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0ull;
  if (bit != 0 && (done.load(std::memory_order_relaxed) & bit)) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  done.fetch_or(bit, std::memory_order_relaxed);
  return true;
}

}  // namespace
}  // namespace fp8
}  // namespace btx
