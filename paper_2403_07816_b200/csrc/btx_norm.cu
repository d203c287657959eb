// Root-mean-square norm of the rows in front of a feed-forward sublayer, with the residual's addition and an FP8 output, and
// its backward pass.  Both are bound by memory: a row stays in registers between the sum over it and its outputs.
//
//   forward   h = round(x + residual), s = 1 / sqrt(sum h^2 / d + eps), y = h s w; y is rounded to the output's type, and cast to
//             FP8 from its fp32 value
//   backward  g = dy w, m = s sum(g h) / d: dx = dh + s (g - h s m), dw = sum over rows of dy h s.  s is formed again
//             from h in the pass that reads h anyway.  A block keeps its share of dw in registers over all of its rows; a
//             second kernel adds the blocks' shares in order, so the result repeats
//
// A row is shared by the threads of a block (threadIdx.y: another row), V vectors of 16 bytes for each of them.
#include <type_traits>

#include "btx_fp8_dev.cuh"

namespace btx {
namespace fp8 {
namespace {


// Sums over the threads of a row, in every one of them; `slot` alternates between calls.
template <int N> __device__ __forceinline__ void row_sum(float (&a)[N], float (*part)[32][N], int slot) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a[i] += __shfl_xor_sync(kAll, a[i], o);
  const int warps = blockDim.x >> 5;
  if (warps == 1) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) part[slot][warp][i] = a[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    a[i] = lane < warps ? part[slot][lane][i] : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a[i] += __shfl_xor_sync(kAll, a[i], o);
  }
}

__device__ __forceinline__ float inv_rms(float sum, int d, float eps) { return 1.0f / sqrtf(sum / (float)d + eps); }

// vec: bit 0 x, 1 residual, 2 w, 3 h, 4 y
template <typename T, int V, int THREADS>
__global__ void __launch_bounds__(THREADS)
norm_kernel(const NormParams p, int vec) {
  constexpr int VN = 16 / (int)sizeof(T);
  __shared__ float part[2][32][1];
  const int kt = (int)scale_tiles_k(p.d), pitch = (int)row_pitch(p.d);
  allow_dependents();
  grid_dependency_wait();
  const int rows = blockDim.y;
  int slot = 0;
  for (long long t0 = (long long)blockIdx.x * rows; t0 < p.T; t0 += (long long)gridDim.x * rows, slot ^= 1) {
    const bool in = t0 + threadIdx.y < p.T;
    const int t = (int)(in ? t0 + threadIdx.y : 0);
    Piece<T, VN> x[V], r[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * VN, n = in ? p.d - c : 0;
      x[i].load((const T*)p.x + t * p.x_stride + c, n, vec & 1);
      if (p.residual != nullptr) r[i].load((const T*)p.residual + t * p.residual_stride + c, n, vec & 2);
    }
    float sum[1] = {0.f};
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * VN, n = in ? p.d - c : 0;
      float v[VN];
      x[i].values(v);
      if (p.residual != nullptr) {
        float a[VN];
        r[i].values(a);
#pragma unroll
        for (int j = 0; j < VN; ++j) v[j] += a[j];
        x[i].set(v);
        x[i].values(v);
      }
      if (p.h != nullptr) x[i].store((T*)p.h + t * p.h_stride + c, n, vec & 8);
#pragma unroll
      for (int j = 0; j < VN; ++j) sum[0] = fmaf(v[j], v[j], sum[0]);
    }
    row_sum(sum, part, slot);
    const float s = inv_rms(sum[0], p.d, p.eps);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * VN, n = in ? p.d - c : 0;
      float v[VN];
      x[i].values(v);
      Piece<T, VN> out;
      if (p.w != nullptr) {
        float w[VN];
        const T* from = (const T*)p.w + c;
        if ((vec & 4) && n >= VN) {
          const uint4 q = *reinterpret_cast<const uint4*>(from);
          out.w[0] = q.x; out.w[1] = q.y; out.w[2] = q.z; out.w[3] = q.w;
        } else {
          out.load(from, n, false);
        }
        out.values(w);
#pragma unroll
        for (int j = 0; j < VN; ++j) v[j] = v[j] * s * w[j];
      } else {
#pragma unroll
        for (int j = 0; j < VN; ++j) v[j] *= s;
      }
      if (p.y != nullptr) {
        out.set(v);
        out.store((T*)p.y + t * p.y_stride + c, n, vec & 16);
      }
      if (p.codes != nullptr) {
        constexpr int LANES = kBlock / VN;
#pragma unroll
        for (int j = 0; j < VN; ++j)
          if (j >= n) v[j] = 0.f;            // behind the last element (0 times an infinite s otherwise)
        uint32_t inv, q[VN / 4];
        const uint32_t byte = scale_byte(lanes_max<LANES>(amax_of(v)), inv);
        cast_codes(v, byte, inv, q);
        if (in && c < pitch) {
          uint8_t* to = p.codes + (size_t)t * pitch + c;
          if constexpr (VN == 8) *reinterpret_cast<uint2*>(to) = make_uint2(q[0], q[1]);
          else *reinterpret_cast<uint32_t*>(to) = q[0];
        }
        if (n > 0 && (threadIdx.x & (LANES - 1)) == 0) p.scales[scale_offset(0, t, kt, c / kBlock)] = (uint8_t)byte;
      }
    }
  }
}

// vec: bit 0 h, 1 w, 2 dy, 3 dh, 4 dx, 5 the shares of dw
template <typename T, int V, int THREADS>
__global__ void __launch_bounds__(THREADS)
norm_grad_kernel(const NormGradParams p, int vec) {
  constexpr int VN = 16 / (int)sizeof(T);
  __shared__ float part[2][32][2];
  allow_dependents();
  grid_dependency_wait();
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < kStatusWords; i += blockDim.x) p.status[i] = 0;
  float dw[V][VN];
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int j = 0; j < VN; ++j) dw[i][j] = 0.f;
  int slot = 0;
  for (int t = blockIdx.x; t < p.T; t += gridDim.x, slot ^= 1) {
    Piece<T, VN> h[V], dy[V], dh[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * VN, n = p.d - c;
      h[i].load((const T*)p.h + t * p.h_stride + c, n, vec & 1);
      dy[i].load((const T*)p.dy + t * p.dy_stride + c, n, vec & 4);
      if (p.dh != nullptr) dh[i].load((const T*)p.dh + t * p.dh_stride + c, n, vec & 8);
    }
    float sum[2] = {0.f, 0.f};
    auto weights = [&](int i, float (&w)[VN]) {
      const int c = (i * blockDim.x + threadIdx.x) * VN, n = p.d - c;
      Piece<T, VN> q;
      if ((vec & 2) && n >= VN) {
        const uint4 u = *reinterpret_cast<const uint4*>((const T*)p.w + c);
        q.w[0] = u.x; q.w[1] = u.y; q.w[2] = u.z; q.w[3] = u.w;
      } else {
        q.load((const T*)p.w + c, n, false);
      }
      q.values(w);
    };
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float a[VN], g[VN];
      h[i].values(a);
      dy[i].values(g);
      if (p.w != nullptr) {
        float w[VN];
        weights(i, w);
#pragma unroll
        for (int j = 0; j < VN; ++j) g[j] *= w[j];
      }
#pragma unroll
      for (int j = 0; j < VN; ++j) {
        sum[0] = fmaf(a[j], a[j], sum[0]);
        sum[1] = fmaf(g[j], a[j], sum[1]);
      }
    }
    row_sum(sum, part, slot);
    const float s = inv_rms(sum[0], p.d, p.eps), m = sum[1] / (float)p.d * s;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * VN, n = p.d - c;
      float a[VN], g[VN];
      h[i].values(a);
      dy[i].values(g);
#pragma unroll
      for (int j = 0; j < VN; ++j) {
        a[j] *= s;
        if (j < n) dw[i][j] = fmaf(g[j], a[j], dw[i][j]);
      }
      if (p.w != nullptr) {
        float w[VN];
        weights(i, w);
#pragma unroll
        for (int j = 0; j < VN; ++j) g[j] *= w[j];
      }
#pragma unroll
      for (int j = 0; j < VN; ++j) g[j] = s * (g[j] - a[j] * m);
      if (p.dh != nullptr) {
        float r[VN];
        dh[i].values(r);
#pragma unroll
        for (int j = 0; j < VN; ++j) g[j] += r[j];
      }
      Piece<T, VN> out;
      out.set(g);
      out.store((T*)p.dx + t * p.dx_stride + c, n, vec & 16);
    }
  }
  if (p.dw != nullptr)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (i * blockDim.x + threadIdx.x) * VN;
      float* to = p.part + (size_t)blockIdx.x * p.d + c;
      if ((vec & 32) && c + VN <= p.d) {
#pragma unroll
        for (int j = 0; j < VN; j += 4) *reinterpret_cast<float4*>(to + j) = make_float4(dw[i][j], dw[i][j + 1], dw[i][j + 2], dw[i][j + 3]);
      } else {
#pragma unroll
        for (int j = 0; j < VN; ++j)
          if (c + j < p.d) to[j] = dw[i][j];
      }
    }
}

// dw[c] (+)= the sum of column c over `parts` rows: 32 columns a block, its 16 warps take every sixteenth row
constexpr int kSumWarps = 16;
__global__ void __launch_bounds__(32 * kSumWarps)
norm_sum_kernel(const float* part, int parts, int d, int accumulate, float* dw) {
  __shared__ float share[kSumWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  allow_dependents();
  grid_dependency_wait();
  float a = 0.f;
  if (c < d)
    for (int i = warp; i < parts; i += kSumWarps) a += __ldcs(part + (size_t)i * d + c);
  share[warp][lane] = a;
  __syncthreads();
  if (warp == 0 && c < d) {
    a = accumulate ? dw[c] : 0.f;
#pragma unroll
    for (int i = 0; i < kSumWarps; ++i) a += share[i][lane];
    dw[c] = a;
  }
}

// Vectors of 16 bytes a thread and threads of a row: few vectors, so that many rows are in flight; more than 512 threads
// (which leaves 64 registers for each) only for rows of more than 32 KB.
struct Shape { int v, threads; };
Shape shape_of(int vecs) {
  for (int v = 1; v < 4; v *= 2)
    if (vecs <= v * (v == 1 ? 64 : 512)) return {v, (vecs + 32 * v - 1) / (32 * v) * 32};
  return {4, (vecs + 127) / 128 * 32};
}
template <typename F> cudaError_t by_shape(const Shape& s, F&& f) {
  using std::integral_constant;
  if (s.v == 1) return f(integral_constant<int, 1>(), integral_constant<int, 256>());
  if (s.v == 2) return f(integral_constant<int, 2>(), integral_constant<int, 512>());
  if (s.threads <= 512) return f(integral_constant<int, 4>(), integral_constant<int, 512>());
  return f(integral_constant<int, 4>(), integral_constant<int, 1024>());
}

template <typename T> int vectors(long long d) { return (int)((d + 16 / (int)sizeof(T) - 1) / (16 / (int)sizeof(T))); }

bool rows16(const void* p, long long stride, int esize) { return ((uintptr_t)p & 15) == 0 && stride * esize % 16 == 0; }

template <typename T> cudaError_t norm(const NormParams& p, cudaStream_t st) {
  const Shape s = shape_of(vectors<T>(p.codes != nullptr ? row_pitch(p.d) : p.d));
  const int rows = s.threads == 32 ? 8 : 1;
  const int e = sizeof(T);
  const int vec = rows16(p.x, p.x_stride, e) | rows16(p.residual, p.residual_stride, e) << 1 | rows16(p.w, 0, e) << 2 |
                  rows16(p.h, p.h_stride, e) << 3 | rows16(p.y, p.y_stride, e) << 4;
  const long long want = (p.T + rows - 1ll) / rows, most = 64ll * sm_count();
  const dim3 grid((unsigned)(want < most ? want : most)), block(s.threads, rows);
  return by_shape(s, [&](auto v, auto threads) {
    return launch_after_predecessor(norm_kernel<T, decltype(v)::value, decltype(threads)::value>, grid, block, 0, st, true, p, vec);
  });
}

template <typename T> cudaError_t norm_grad(const NormGradParams& p, cudaStream_t st) {
  const Shape s = shape_of(vectors<T>(p.d));
  const int e = sizeof(T);
  const int vec = rows16(p.h, p.h_stride, e) | rows16(p.w, 0, e) << 1 | rows16(p.dy, p.dy_stride, e) << 2 |
                  rows16(p.dh, p.dh_stride, e) << 3 | rows16(p.dx, p.dx_stride, e) << 4 | (p.d % 4 == 0) << 5;
  const int parts = norm_grad_parts(p.T, p.d, sizeof(T) == 2 ? BTX_BF16 : BTX_F32);
  const dim3 grid((unsigned)parts), block(s.threads);
  const cudaError_t r = by_shape(s, [&](auto v, auto threads) {
    return launch_after_predecessor(norm_grad_kernel<T, decltype(v)::value, decltype(threads)::value>, grid, block, 0, st, true, p, vec);
  });
  if (r != cudaSuccess || p.dw == nullptr) return r;
  return launch_after_predecessor(norm_sum_kernel, dim3((p.d + 31) / 32), dim3(32 * kSumWarps), 0, st, true, (const float*)p.part, parts,
                                  p.d, p.accumulate, p.dw);
}

}  // namespace

// Blocks of the backward pass, each with a share of dw: about 1024 threads for every multiprocessor.
int norm_grad_parts(int T, int d, int dtype) {
  const Shape s = shape_of(dtype == BTX_BF16 ? vectors<__nv_bfloat16>(d) : vectors<float>(d));
  const long long most = (1024 / s.threads) * (long long)sm_count();
  return (int)(T < most ? (T > 0 ? T : 1) : most);
}

cudaError_t launch_norm(const NormParams& p, int dtype, cudaStream_t st) {
  return dtype == BTX_BF16 ? norm<__nv_bfloat16>(p, st) : norm<float>(p, st);
}
cudaError_t launch_norm_grad(const NormGradParams& p, int dtype, cudaStream_t st) {
  return dtype == BTX_BF16 ? norm_grad<__nv_bfloat16>(p, st) : norm_grad<float>(p, st);
}

}  // namespace fp8
}  // namespace btx
