// Root-mean-square norm of the rows in front of a feed-forward sublayer, with the residual's addition and an FP8 output, and
// its backward pass.  Both are bound by memory: a row stays on the chip between the sum over it and its outputs.
//
//   forward   h = round(x + residual), s = 1 / sqrt(sum h^2 / d + eps), y = h s w; y is rounded to the output's type, and cast to
//             FP8 from its fp32 value
//   backward  g = dy w, m = sum(g h s) / d: dx = dh + s (g - h s m), dw = sum over rows of dy h s.  s is formed again
//             from h in the pass that reads h anyway.  A block keeps its share of dw in registers over all of its rows; a
//             second kernel adds the blocks' shares in order, so the result repeats
//
// A row is shared by blockDim.x threads, V vectors of 16 bytes each; a block works on blockDim.y rows at a time.  Blocks are
// resident and walk over the rows.  Every thread fetches its own vectors of the next rows into its own places in shared memory
// (cp.async), so what is in flight does not depend on registers and nobody waits for another thread's copy.
//
// Measured on one B200 (16384 x 4096, replayed; the floor is the bytes at the 6561 GB/s of a copy; a replay finds part of its data in
// the L2).  Forward, bf16: with residual, h and y 83 us (81.8), and codes too 94-95 (92), y alone 47 (40.9); fp32 with codes 176 (174).
// Backward with dh, bf16: 82.5 us (81.8), 3 of these for the second kernel, 93 from a cold L2; fp32 158.  Issue slots are taken to
// 52-56 %.  One row of 4096: 2.3 us, a launch.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "btx_fp8_dev.cuh"

namespace btx {
namespace fp8 {
namespace {

constexpr int kSmem = 220 * 1024;          // shared memory of a multiprocessor that the rings of its blocks share

// Sums over the threads of a row, in every one of them; `slot` alternates between calls.  Rows of a block wait for themselves
// only (a named barrier each).
template <int N> __device__ __forceinline__ void row_sum(float (&a)[N], float (*part)[32][N], int slot) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a[i] += __shfl_xor_sync(kAll, a[i], o);
  const int warps = blockDim.x >> 5;
  if (warps == 1) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, first = threadIdx.y * warps;
  if (lane == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) part[slot][first + warp][i] = a[i];
  asm volatile("bar.sync %0, %1;" ::"r"(1 + threadIdx.y), "r"(blockDim.x) : "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) {
    a[i] = lane < warps ? part[slot][first + lane][i] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a[i] += __shfl_xor_sync(kAll, a[i], o);
  }
}

// whether `yes` is true for any thread of a row
__device__ __forceinline__ bool row_any(bool yes) {
  if (blockDim.x == 32) return __any_sync(kAll, yes);
  int any = yes;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %0, 0;\n\tbarrier.cta.red.or.pred q, %1, %2, p;\n\tselp.s32 %0, 1, 0, q;\n\t}"
               : "+r"(any) : "r"(1 + threadIdx.y), "r"(blockDim.x) : "memory");
  return any;
}

// 1 / sqrt(m) of the fp32 m = sum / d + eps, and a step of Newton's method on it (with the product m s in two words), which leaves
// about half an ulp of its two roundings: a row's elements share this error, and those near the middle between two FP8 values show it.
__device__ __forceinline__ float inv_rms(float sum, int d, float eps) {
  const float m = sum / (float)d + eps, s = 1.0f / sqrtf(m);
  if (!(m > 0.f && m < INFINITY)) return s;
  const float t = m * s, low = fmaf(m, s, -t);
  return fmaf(0.5f * s, fmaf(-t, s, 1.0f) - low * s, s);
}

// A thread's columns and its places in shared memory: STAGES rows of each of ARRAYS tensors, V vectors a row.  VEC: every
// vector of every tensor is whole and on a 16-byte boundary.
//
// Otherwise rows go by words of 4 bytes.  A row of bf16 that starts in the middle of a word is kept and written as the words that
// hold it: word k of a vector has elements 2k - 1 and 2k, element 7 is in the next lane's word 0, which the warp's last lane
// fetches for itself.  Words that reach over an end of the row are put together from single elements.  Words of fp32 (TURNED) are
// fetched and written 32 neighbours at a time and change hands in shared memory (16384 x 4097, gradients: 246 us, 279 without; bf16, where
// half words change hands too, does not gain).  Latency of the longer way of a row bounds these (32-39 % of the issue slots, 28 % of
// the shared memory's): 16384 x 4098 bf16 with residual, h and y 203 us, 4099 231, where 4096 takes 83 (single elements took 403;
// aligned 16-byte pieces and shifts were slower, as the pieces at a row's ends then have to be waited for).
template <typename T, int V, int ARRAYS, int STAGES, bool VEC> struct Rows {
  static constexpr int VN = 16 / (int)sizeof(T);
  static constexpr bool HALVES = !VEC && sizeof(T) == 2, TURNED = !VEC && sizeof(T) == 4;
  int d, c0, dc;                           // elements of a row, first column, columns from one vector to the next
  uint32_t base, step;                     // first place, bytes from one place to the next
  uint32_t turned;                         // words: the warp's vectors on their way out
  uint32_t more;                           // HALVES: the last lane's places of single words
  uint32_t odd;                            // HALVES: bit stage * ARRAYS + array: that row starts in the middle of a word
  const T* from[ARRAYS];                   // first column of the next row to fetch
  long long ahead[ARRAYS];                 // elements to the row after it

  __device__ __forceinline__ void init(uint8_t* smem, int d_) {
    d = d_; c0 = threadIdx.x * VN; dc = blockDim.x * VN;
    const int threads = blockDim.x * blockDim.y, me = threadIdx.y * blockDim.x + threadIdx.x;
    step = threads * 16;
    const uint32_t first = (uint32_t)__cvta_generic_to_shared(smem);
    base = first + me * 16;
    turned = first + STAGES * ARRAYS * V * step + (me >> 5) * 512;
    more = first + (STAGES * ARRAYS * V + 1) * step + (me >> 5) * (STAGES * ARRAYS * V * 4);
    odd = 0;
    // places behind the last column are never written again
    for (int k = 0; k < STAGES * ARRAYS * V; ++k)
      asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(base + k * step), "r"(0) : "memory");
  }
  __device__ __forceinline__ void source(int array, const void* p, long long stride, long long row, long long rows_ahead) {
    from[array] = (const T*)p + row * stride + c0;
    ahead[array] = rows_ahead * stride;
  }
  __device__ __forceinline__ int col(int i) const { return c0 + i * dc; }
  __device__ __forceinline__ uint32_t place(int stage, int array, int i) const { return base + ((stage * ARRAYS + array) * V + i) * step; }
  // word with elements e and e + 1 of the row, of which the vector at `at` begins with element c
  __device__ __forceinline__ void fetch_word(uint32_t to, const T* at, int c, int e) const {
    if (e >= 0 && e + 1 < d) {
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(at + (e - c)) : "memory");
    } else {
      const uint16_t* h = reinterpret_cast<const uint16_t*>(at) + (e - c);
      const uint32_t w = (e >= 0 && e < d ? (uint32_t)h[0] : 0u) | (e + 1 < d ? (uint32_t)h[1] << 16 : 0u);
      asm volatile("st.shared.u32 [%0], %1;" ::"r"(to), "r"(w) : "memory");
    }
  }
  // the next row, if there is one, into a stage
  __device__ __forceinline__ void fetch(int stage, bool in) {
    if (TURNED) __syncwarp();              // all lanes have read what was here
#pragma unroll
    for (int a = 0; a < ARRAYS; ++a) {
      if (in) {
        int off = 0;
        if constexpr (HALVES) {
          const uint32_t bit = 1u << (stage * ARRAYS + a);
          off = (int)((uintptr_t)from[a] >> 1 & 1);
          odd = off ? odd | bit : odd & ~bit;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const uint32_t to = place(stage, a, i);
          const T* at = from[a] + i * dc;
          if constexpr (VEC) {
            if (col(i) < d) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(at) : "memory");
          } else if constexpr (HALVES) {
            if (col(i) <= d) {               // (the vector behind the last one may hold its last element)
#pragma unroll
              for (int k = 0; k < 4; ++k) fetch_word(to + 4 * k, at, col(i), col(i) + 2 * k - off);
            }
            if (off && (threadIdx.x & 31) == 31) fetch_word(more + ((stage * ARRAYS + a) * V + i) * 4, at, col(i), col(i) + 7);
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (col(i) + word(k) < d)
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to + 4 * word(k)), "l"(at + word(k)) : "memory");
          }
        }
      }
      from[a] += ahead[a];
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  // word `k`, `lane` of the warp's 32 vectors, counted from the lane's own
  __device__ __forceinline__ static int word(int k) { return k * 32 - 3 * (int)(threadIdx.x & 31); }
  // the row of the oldest fetch has landed
  __device__ __forceinline__ void wait() const {
    asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
    if (TURNED) __syncwarp();
  }
  __device__ __forceinline__ void read(int stage, int array, int i, f32x2 (&v)[VN / 2]) const {
    Piece<T, VN> q;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.w[0]), "=r"(q.w[1]), "=r"(q.w[2]), "=r"(q.w[3])
                 : "r"(place(stage, array, i)) : "memory");
    if constexpr (HALVES) {
      if (odd >> (stage * ARRAYS + array) & 1) {         // (the same for the whole warp)
        uint32_t next = __shfl_down_sync(kAll, q.w[0], 1);
        if ((threadIdx.x & 31) == 31)
          asm volatile("ld.shared.u32 %0, [%1];" : "=r"(next) : "r"(more + ((stage * ARRAYS + array) * V + i) * 4) : "memory");
#pragma unroll
        for (int k = 0; k < 4; ++k) q.w[k] = __funnelshift_r(q.w[k], k < 3 ? q.w[k + 1 < 4 ? k + 1 : 3] : next, 16);
      }
    }
    q.pairs(v);
  }
  // (called by whole warps)
  __device__ __forceinline__ void write(T* row, int i, const Piece<T, VN>& q) const {
    T* at = row + i * dc;
    if constexpr (VEC) {
      if (col(i) < d) q.store(at, VN, true);
    } else if constexpr (HALVES) {
      const int lane = threadIdx.x & 31, off = (int)((uintptr_t)at >> 1 & 1), n = d - col(i);
      uint16_t* h = reinterpret_cast<uint16_t*>(at);
      uint32_t w[4];
      const uint32_t before = __shfl_up_sync(kAll, q.w[3], 1);
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = off ? __funnelshift_r(k > 0 ? q.w[k > 0 ? k - 1 : 0] : before, q.w[k], 16) : q.w[k];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int e = 2 * k - off;           // (element -1: the lane's before, which leaves it to this one)
        if (e + 1 < n && (e >= 0 || lane > 0)) {
          *reinterpret_cast<uint32_t*>(h + e) = w[k];
        } else {
          if (e < n && (e >= 0 || lane > 0)) h[e] = (uint16_t)w[k];
          if (e + 1 < n) h[e + 1] = (uint16_t)(w[k] >> 16);
        }
      }
      if (off && lane == 31 && 7 < n) h[7] = (uint16_t)(q.w[3] >> 16);
    } else {
      const int lane = threadIdx.x & 31, n = d - col(i);
      __syncwarp();                        // (the vector before has been read)
      asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(turned + lane * 16), "r"(q.w[0]), "r"(q.w[1]), "r"(q.w[2]), "r"(q.w[3]) : "memory");
      __syncwarp();
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t w;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(turned + (k * 32 + lane) * 4) : "memory");
        if (word(k) < n) reinterpret_cast<uint32_t*>(at)[word(k)] = w;
      }
    }
  }
  // this thread's weights, ones where there are none
  __device__ __forceinline__ void weights(const void* w, f32x2 (&v)[V][VN / 2]) const {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      Piece<T, VN> q;
      q.load((const T*)w + col(i), w == nullptr ? 0 : d - col(i), VEC);
      q.pairs(v[i]);
      if (w == nullptr)
#pragma unroll
        for (int j = 0; j < VN / 2; ++j) v[i][j] = pack2(1.f, 1.f);
    }
  }
};

// Threads of a multiprocessor that the registers are meant for.  What is in flight should be about 64 KB: with a residual (two
// loads a vector) or in the backward pass 512 threads have that, with one tensor to read it takes 1024
// (16384 x 4096 without a residual: bf16 47 us, with 512 threads 53; fp32 83 and 107).
constexpr int resident_threads(int v, int threads, int arrays) { return threads == 1024 || (arrays == 1 && v == 2) ? 1024 : 512; }

template <typename T, int V, int THREADS, bool RESIDUAL, bool VEC>
__global__ void __launch_bounds__(THREADS, resident_threads(V, THREADS, RESIDUAL ? 2 : 1) / THREADS)
norm_kernel(const __grid_constant__ NormParams p) {
  constexpr int VN = 16 / (int)sizeof(T), STAGES = THREADS == 1024 ? 1 : 2;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float part[2][32][1];
  const int pitch = (int)row_pitch(p.d), kt = (int)scale_tiles_k(p.d);
  const int step = gridDim.x * blockDim.y;
  long long t = (long long)blockIdx.x * blockDim.y + threadIdx.y;
  Rows<T, V, RESIDUAL ? 2 : 1, STAGES, VEC> rows;
  rows.init(smem, p.d);
  rows.source(0, p.x, p.x_stride, t, step);
  if (RESIDUAL) rows.source(RESIDUAL ? 1 : 0, p.residual, p.residual_stride, t, step);
  allow_dependents();
  grid_dependency_wait();
  if (STAGES > 1) rows.fetch(0, t < p.T);
  f32x2 w[V][VN / 2];
  rows.weights(p.w, w);
  T *h = (T*)p.h + t * p.h_stride + rows.c0, *y = (T*)p.y + t * p.y_stride + rows.c0;
  uint8_t* codes = p.codes + t * pitch + rows.c0;
  int slot = 0;
  for (long long b = (long long)blockIdx.x * blockDim.y; b < p.T; b += step, t += step) {      // (the same for all rows of the block)
    const bool in = t < p.T;
    const int stage = STAGES > 1 ? slot : 0;
    rows.fetch(STAGES > 1 ? slot ^ 1 : 0, t + (STAGES > 1 ? step : 0) < p.T);
    rows.wait();
    f32x2 v[V][VN / 2], sums = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      rows.read(stage, 0, i, v[i]);
      Piece<T, VN> q;
      if (RESIDUAL) {
        f32x2 r[VN / 2];
        rows.read(stage, RESIDUAL ? 1 : 0, i, r);
#pragma unroll
        for (int j = 0; j < VN / 2; ++j) v[i][j] = add2(v[i][j], r[j]);
        q.set(v[i]);
        q.pairs(v[i]);
      } else {
        q.set(v[i]);
      }
      if (p.h != nullptr && in) rows.write(h, i, q);
#pragma unroll
      for (int j = 0; j < VN / 2; ++j) sums = fma2(v[i][j], v[i][j], sums);
    }
    float sum[1], other;
    unpack2(sums, sum[0], other);
    sum[0] += other;
    row_sum(sum, part, slot);
    const float s = inv_rms(sum[0], p.d, p.eps);
    // s in two factors, a power of two and a number from 1 to 2 (all of an s that is infinite or not a number in the first).  bf16:
    // h 2^k is exact (in [2^-141, sqrt(d)]; smaller ones lose bits), and so is its product with w unless it leaves fp32, which y
    // then does too: one rounding, whatever the sizes of h and w.
    const uint32_t bits = __float_as_uint(s);
    const float power = sizeof(T) == 4 || (bits & 0x7f800000u) == 0x7f800000u ? s : __uint_as_float(bits & 0x7f800000u);
    const float rest = __uint_as_float((bits & 0x007fffffu) | 0x3f800000u);
    const f32x2 first = pack2(power, power), second = pack2(rest, rest);
    uint8_t* scales = p.scales + scale_offset(0, (int)t, kt, 0);
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
      for (int j = 0; j < VN / 2; ++j) {
        v[i][j] = mul2(mul2(v[i][j], first), w[i][j]);
        if (sizeof(T) == 2) v[i][j] = mul2(v[i][j], second);
      }
      if (p.y != nullptr && in) {
        Piece<T, VN> q;
        q.set(v[i]);
        rows.write(y, i, q);
      }
      if (p.codes != nullptr) {
        constexpr int LANES = kBlock / VN;
        const int c = rows.col(i);
        float f[VN];
#pragma unroll
        for (int j = 0; j < VN / 2; ++j) unpack2(v[i][j], f[2 * j], f[2 * j + 1]);
        if (c + VN > p.d) {                  // behind the last element (0 times an infinite s otherwise)
#pragma unroll
          for (int j = 0; j < VN; ++j)
            if (c + j >= p.d) f[j] = 0.f;
        }
        uint32_t inv, q[VN / 4];
        const uint32_t byte = scale_byte(lanes_max<LANES>(amax_of(f)), inv);
        cast_codes(f, byte, inv, q);
        if (in && c < pitch) {
          if constexpr (VN == 8) *reinterpret_cast<uint2*>(codes + i * rows.dc) = make_uint2(q[0], q[1]);
          else *reinterpret_cast<uint32_t*>(codes + i * rows.dc) = q[0];
          if ((threadIdx.x & (LANES - 1)) == 0 && c < p.d) scales[c / (4 * kBlock) * kTileBytes + c / kBlock % 4] = (uint8_t)byte;
        }
      }
    }
    h += step * p.h_stride;
    y += step * p.y_stride;
    codes += (long long)step * pitch;
    slot ^= 1;
  }
}

// sum h^2 and, with u = dy w, sum u h; then dw += dy (h s) and dx = dh + s (u - m (h s)), m = s sum(u h) / d.  h s is of size 1, so
// that s^2, which may leave fp32 where dx does not, is not formed.
template <typename T, int V, int THREADS, bool ADD, bool VEC>
__global__ void __launch_bounds__(THREADS, resident_threads(V, THREADS, 3) / THREADS)
norm_grad_kernel(const __grid_constant__ NormGradParams p) {
  constexpr int VN = 16 / (int)sizeof(T), STAGES = THREADS == 1024 ? 1 : 2;
  // h and dy stay in registers for dx where these hold them, else they are read again: bf16 rows of three and four vectors a thread
  // (2048 x 16384 80-84 us spilling, 50 so; 16384 x 4096 with two 83, 84 so).
  constexpr bool KEEP = sizeof(T) == 4 || V == 2;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float part[2][32][2], part_again[1][32][1];       // (between two uses of the second lies a barrier of the first's)
  const int step = gridDim.x * blockDim.y;
  long long t = (long long)blockIdx.x * blockDim.y + threadIdx.y;
  Rows<T, V, ADD ? 3 : 2, STAGES, VEC> rows;
  rows.init(smem, p.d);
  rows.source(0, p.h, p.h_stride, t, step);
  rows.source(1, p.dy, p.dy_stride, t, step);
  if (ADD) rows.source(ADD ? 2 : 0, p.dh, p.dh_stride, t, step);
  allow_dependents();
  grid_dependency_wait();
  if (blockIdx.x == 0)
    for (int i = threadIdx.y * blockDim.x + threadIdx.x; i < kStatusWords; i += blockDim.x * blockDim.y) p.status[i] = 0;
  if (STAGES > 1) rows.fetch(0, t < p.T);
  f32x2 w[V][VN / 2], dw[V][VN / 2];
  rows.weights(p.w, w);
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int j = 0; j < VN / 2; ++j) dw[i][j] = 0;
  T* dx = (T*)p.dx + t * p.dx_stride + rows.c0;
  int slot = 0;
  for (long long b = (long long)blockIdx.x * blockDim.y; b < p.T; b += step, t += step) {
    const int stage = STAGES > 1 ? slot : 0;
    rows.fetch(STAGES > 1 ? slot ^ 1 : 0, t + (STAGES > 1 ? step : 0) < p.T);
    rows.wait();
    f32x2 h[KEEP ? V : 1][VN / 2], dy[KEEP ? V : 1][VN / 2], sums[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int k = KEEP ? i : 0;
      rows.read(stage, 0, i, h[k]);
      rows.read(stage, 1, i, dy[k]);
#pragma unroll
      for (int j = 0; j < VN / 2; ++j) {
        sums[0] = fma2(h[k][j], h[k][j], sums[0]);
        sums[1] = fma2(mul2(dy[k][j], w[i][j]), h[k][j], sums[1]);
      }
    }
    float sum[2], other;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      unpack2(sums[i], sum[i], other);
      sum[i] += other;
    }
    row_sum(sum, part, slot);
    const float s = inv_rms(sum[0], p.d, p.eps);
    const f32x2 s2 = pack2(s, s);
    float m = sum[1] / (float)p.d * s;
    // Products u h may leave fp32 where dx does not: their sum is infinite, not a number, or below 2^-60, of which 2^15 products
    // below the normal numbers are no part.  Then with h s, unless all dy are 0, as in padded rows.
    if (!(fabsf(sum[1]) >= 0x1p-60f && fabsf(sum[1]) < INFINITY)) {
      f32x2 any = 0;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int k = KEEP ? i : 0;
        if (!KEEP) rows.read(stage, 1, i, dy[k]);
#pragma unroll
        for (int j = 0; j < VN / 2; ++j) any |= dy[k][j];
      }
      m = 0.f;
      if (row_any((any & 0x7fffffff7fffffffull) != 0)) {
        f32x2 units = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          f32x2 hi[VN / 2], di[VN / 2];
          if (!KEEP) {
            rows.read(stage, 0, i, hi);
            rows.read(stage, 1, i, di);
          }
#pragma unroll
          for (int j = 0; j < VN / 2; ++j) {
            if (KEEP) {                      // (copies that nothing of the way of other rows is computed from)
              asm volatile("mov.b64 %0, %1;" : "=l"(hi[j]) : "l"(h[KEEP ? i : 0][j]));
              asm volatile("mov.b64 %0, %1;" : "=l"(di[j]) : "l"(dy[KEEP ? i : 0][j]));
            }
            units = fma2(mul2(di[j], w[i][j]), mul2(hi[j], s2), units);
          }
        }
        float again[1];
        unpack2(units, again[0], other);
        again[0] += other;
        row_sum(again, part_again, 0);
        m = again[0] / (float)p.d;
      }
    }
    const f32x2 m2 = pack2(-m, -m);
    if (t < p.T) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int k = KEEP ? i : 0;
        f32x2 g[VN / 2];
        if (!KEEP) {
          rows.read(stage, 0, i, h[k]);
          rows.read(stage, 1, i, dy[k]);
        }
        if (ADD) {
          rows.read(stage, ADD ? 2 : 0, i, g);
        } else {
#pragma unroll
          for (int j = 0; j < VN / 2; ++j) g[j] = 0;
        }
#pragma unroll
        for (int j = 0; j < VN / 2; ++j) {
          const f32x2 unit = mul2(h[k][j], s2);
          dw[i][j] = fma2(dy[k][j], unit, dw[i][j]);
          g[j] = fma2(fma2(unit, m2, mul2(dy[k][j], w[i][j])), s2, g[j]);
        }
        Piece<T, VN> q;
        q.set(g);
        rows.write(dx, i, q);
      }
    }
    dx += step * p.dx_stride;
    slot ^= 1;
  }
  if (p.dw == nullptr) return;
  if (blockDim.y > 1) {                      // the rows of the block, in order (its ring has room for a place per value)
    f32x2* sh = reinterpret_cast<f32x2*>(smem);
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < VN / 2; ++j) sh[((threadIdx.y * V + i) * (VN / 2) + j) * blockDim.x + threadIdx.x] = dw[i][j];
    __syncthreads();
    if (threadIdx.y > 0) return;
    for (int r = 1; r < (int)blockDim.y; ++r)
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < VN / 2; ++j) dw[i][j] = add2(dw[i][j], sh[((r * V + i) * (VN / 2) + j) * blockDim.x + threadIdx.x]);
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = rows.col(i);
    Piece<float, VN> out;
    out.set(dw[i]);
    out.store(p.part + (size_t)blockIdx.x * p.d + c, p.d - c, p.d % 4 == 0);
  }
}

// dw[c] (+)= the sum of column c over `parts` rows: 32 columns a block, its 32 warps take every 32nd row, eight of them at once
constexpr int kSumWarps = 32, kSumAhead = 8;
__global__ void __launch_bounds__(32 * kSumWarps)
norm_sum_kernel(const float* part, int parts, int d, int accumulate, float* dw) {
  __shared__ float share[kSumWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  allow_dependents();
  grid_dependency_wait();
  float a = 0.f;
  if (c < d)
    for (int i0 = warp; i0 < parts; i0 += kSumWarps * kSumAhead) {
      float v[kSumAhead];
#pragma unroll
      for (int u = 0; u < kSumAhead; ++u) {
        const int i = i0 + u * kSumWarps;
        v[u] = i < parts ? __ldcs(part + (size_t)i * d + c) : 0.f;
      }
#pragma unroll
      for (int u = 0; u < kSumAhead; ++u) a += v[u];
    }
  share[warp][lane] = a;
  __syncthreads();
  if (warp == 0 && c < d) {
    a = accumulate ? dw[c] : 0.f;
#pragma unroll
    for (int i = 0; i < kSumWarps; ++i) a += share[i][lane];
    dw[c] = a;
  }
}

// Vectors of 16 bytes a thread, threads of a row, rows of a block; blocks that a multiprocessor holds, bytes of their ring.
// More than 512 threads (which leaves 64 registers for each and one stage) only for rows of more than 32 KB; the backward pass, with
// 32 floats of dw and of w in bf16, spills there: 2048 x 32768 159 us, with a floor of 82.
struct Shape { int v, threads, rows, blocks, smem; };
Shape shape_of(int T, int vecs, int esize, int arrays) {
  Shape s;
  // as many rows as make 512 threads (few blocks leave few shares of dw to add up)
  auto with = [&](int v) {
    s.v = v;
    s.threads = (vecs + 32 * v - 1) / (32 * v) * 32;
    s.rows = s.threads < 512 ? 512 / s.threads : 1;
    return s.threads <= 512 || v == 4 ? s.rows * vecs : 0;
  };
  // The fewest vectors a thread with which 700 are at work, or the most there can be: 16384 x 5120 bf16 (640 of them) with codes 120 us
  // with two rows of 224 threads, 142 with one of 320, gradients 101 and 124; 16384 x 4099 with codes 266
  // and 413.  (By the row's length alone, so that its sums do not depend on the rows around it.)
  const int most = std::max(with(2), std::max(with(3), with(4)));
  for (int v = 2; with(v) < (most < 700 ? most : 700); ++v) {}
  // as long as every multiprocessor has some
  const int fill = T / sm_count();
  if (s.rows > fill) s.rows = fill > 0 ? fill : 1;
  const int block = s.threads * s.rows, bound = s.threads <= 512 ? 512 : 1024;
  s.blocks = resident_threads(s.v, bound, arrays) / block;
  s.smem = (bound == 1024 ? 1 : 2) * s.v * arrays * (block * 16 + block / 32 * 4);       // places, and words of last lanes
  const int shares = s.rows > 1 ? block * s.v * (16 / esize) * 4 : 0;
  if (s.smem < shares) s.smem = shares;
  return s;
}
template <bool X> using Bool = std::integral_constant<bool, X>;
template <int X> using Int = std::integral_constant<int, X>;
template <typename F> cudaError_t by_shape(const Shape& s, bool more, bool vec, F&& f) {
  auto with = [&](auto v, auto threads) {
    if (more) return vec ? f(v, threads, Bool<true>(), Bool<true>()) : f(v, threads, Bool<true>(), Bool<false>());
    return vec ? f(v, threads, Bool<false>(), Bool<true>()) : f(v, threads, Bool<false>(), Bool<false>());
  };
  if (s.v == 2) return with(Int<2>(), Int<512>());
  if (s.v == 3) return with(Int<3>(), Int<512>());
  return s.threads <= 512 ? with(Int<4>(), Int<512>()) : with(Int<4>(), Int<1024>());
}
int vectors(long long d, int esize) { return (int)((d * esize + 15) / 16); }

// (a tensor that is not there does no harm)
bool rows16(const void* p, long long stride, int esize) { return p == nullptr || (((uintptr_t)p & 15) == 0 && stride * esize % 16 == 0); }

template <typename T> cudaError_t norm(const NormParams& p, cudaStream_t st) {
  const int e = sizeof(T);
  const Shape s = shape_of(p.T, vectors(row_pitch(p.d), e), e, p.residual != nullptr ? 2 : 1);
  const bool vec = p.d * e % 16 == 0 && rows16(p.x, p.x_stride, e) && rows16(p.residual, p.residual_stride, e) && rows16(p.w, 0, e) &&
                   rows16(p.h, p.h_stride, e) && rows16(p.y, p.y_stride, e);
  const long long want = (p.T + s.rows - 1ll) / s.rows, most = (long long)s.blocks * sm_count();
  const dim3 grid((unsigned)(want < most ? want : most)), block(s.threads, s.rows);
  const int smem = s.smem + (vec ? 0 : s.threads * s.rows * 16);
  return by_shape(s, p.residual != nullptr, vec, [&](auto v, auto threads, auto residual, auto whole) {
    static std::atomic<uint64_t> done{0};
    auto kernel = norm_kernel<T, decltype(v)::value, decltype(threads)::value, decltype(residual)::value, decltype(whole)::value>;
    if (!allow_smem((const void*)kernel, kSmem, done)) return cudaErrorInvalidValue;
    return launch_after_predecessor(kernel, grid, block, smem, st, true, p);
  });
}

int grad_parts(int T, const Shape& s) {
  const long long want = (T + s.rows - 1ll) / s.rows, most = (long long)s.blocks * sm_count();
  return (int)(want < most ? (want > 0 ? want : 1) : most);
}

template <typename T> cudaError_t norm_grad(const NormGradParams& p, cudaStream_t st) {
  const int e = sizeof(T);
  const Shape s = shape_of(p.T, vectors(p.d, e), e, 3);
  const bool vec = p.d * e % 16 == 0 && rows16(p.h, p.h_stride, e) && rows16(p.w, 0, e) && rows16(p.dy, p.dy_stride, e) &&
                   rows16(p.dh, p.dh_stride, e) && rows16(p.dx, p.dx_stride, e);
  const int parts = grad_parts(p.T, s);
  const dim3 grid((unsigned)parts), block(s.threads, s.rows);
  const int smem = s.smem + (vec ? 0 : s.threads * s.rows * 16);
  const cudaError_t r = by_shape(s, p.dh != nullptr, vec, [&](auto v, auto threads, auto add, auto whole) {
    static std::atomic<uint64_t> done{0};
    auto kernel = norm_grad_kernel<T, decltype(v)::value, decltype(threads)::value, decltype(add)::value, decltype(whole)::value>;
    if (!allow_smem((const void*)kernel, kSmem, done)) return cudaErrorInvalidValue;
    return launch_after_predecessor(kernel, grid, block, smem, st, true, p);
  });
  if (r != cudaSuccess || p.dw == nullptr) return r;
  return launch_after_predecessor(norm_sum_kernel, dim3((p.d + 31) / 32), dim3(32 * kSumWarps), 0, st, true, (const float*)p.part, parts,
                                  p.d, p.accumulate, p.dw);
}

}  // namespace

// Blocks of the backward pass, each with a share of dw: as many as are resident at once.
int norm_grad_parts(int T, int d, int dtype) {
  const int e = dtype == BTX_BF16 ? 2 : 4;
  return grad_parts(T, shape_of(T, vectors(d, e), e, 3));
}

cudaError_t launch_norm(const NormParams& p, int dtype, cudaStream_t st) {
  return dtype == BTX_BF16 ? norm<__nv_bfloat16>(p, st) : norm<float>(p, st);
}
cudaError_t launch_norm_grad(const NormGradParams& p, int dtype, cudaStream_t st) {
  return dtype == BTX_BF16 ? norm_grad<__nv_bfloat16>(p, st) : norm_grad<float>(p, st);
}

}  // namespace fp8
}  // namespace btx
