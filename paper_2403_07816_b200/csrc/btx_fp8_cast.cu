// FP8 casts: one power-of-two scale for 128 elements of a row, or for a block of 128 x 128.
//
//   quantize_rows   a scale per row and 128 elements, as the rows stand: sixteen lanes share a block, eight elements each, the
//                   maximum takes four shuffles
//   quantize_tiles  square blocks and transposed outputs: a block of threads holds a 128 x 128 tile in registers (8 rows of 8
//                   elements a thread), which gives the largest of its rows, of its columns or of all; x is read once
//                   for both outputs.  Transposed codes turn through shared memory, 8 bytes (of 8 rows) at a time
//   dequantize      the mapping of quantize_rows backwards
//   dispatch_rows   quantize_rows of the expert layer's tokens, or a copy of their FP8 form, to the k rows of every token
#include "btx_fp8_dev.cuh"
#include "btx_fp8_gemm.cuh"

namespace btx {
namespace fp8 {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;                 // 256-element chunks a warp has in flight

template <typename T, typename I>
__global__ void __launch_bounds__(kThreads)
quantize_rows_kernel(const CastParams p, int vec, I items, int groups) {
  const int lane = threadIdx.x & 31;
  const int kt = (int)scale_tiles_k(p.K), pitch = (int)row_pitch(p.K);
  const size_t tiles = (size_t)row_tiles(p.out_rows);
  allow_dependents();
  grid_dependency_wait();
  for (I w = ((I)blockIdx.x * kThreads + threadIdx.x) >> 5; w < items; w += (I)gridDim.x * (kThreads / 32)) {
    const I r = w / (I)groups;
    const int g = (int)(w - r * (I)groups);
    const int b = (int)(r / (I)p.rows), row = (int)(r - (I)b * (I)p.rows);
    const T* src = (const T*)p.src + b * p.batch_stride + row * p.row_stride;
    const int out_row = p.first + row * p.step;
    const int c0 = g * kUnroll * 256 + lane * 8;
    Piece<T, 8> x[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) x[u].load(src + c0 + u * 256, p.K - (c0 + u * 256), vec != 0);
    uint8_t* codes = p.codes + ((size_t)b * p.out_rows + out_row) * pitch + c0;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int c = c0 + u * 256;
      uint32_t inv, q[2];
      const uint32_t byte = scale_byte(lanes_max<16>(x[u].amax()), inv);
      float v[8];
      x[u].values(v);
      cast_codes(v, byte, inv, q);
      if (c < pitch) *reinterpret_cast<uint2*>(codes + u * 256) = make_uint2(q[0], q[1]);
      if ((lane & 15) == 0 && c < p.K) p.scales[scale_offset(b * tiles, out_row, kt, c / kBlock)] = (uint8_t)byte;
    }
  }
}

// A thread's eight rows are neighbours: rows rg * 8 .. of its eight columns cg * 8 ..
template <typename T>
__global__ void __launch_bounds__(kThreads)
quantize_tiles_kernel(const CastParams p, int vec, long long items, int col_tiles) {
  __shared__ __align__(16) uint8_t turned[128 * 128];
  __shared__ uint32_t part[8][128];        // largest of every column over a warp's 16 rows (square: [warp][0], of all)
  __shared__ uint32_t inv_of[128];
  __shared__ uint8_t byte_of[128];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cg = tid & 15, rg = tid >> 4;
  const int kt = (int)scale_tiles_k(p.K), pitch = (int)row_pitch(p.K);
  const int kt_t = (int)scale_tiles_k(p.rows), pitch_t = (int)row_pitch(p.rows);
  const size_t tiles = (size_t)row_tiles(p.out_rows), tiles_t = (size_t)row_tiles(p.K);
  const long long per = (long long)col_tiles * row_tiles(p.rows);
  allow_dependents();
  grid_dependency_wait();
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int b = (int)(it / per);
    const int rt = (int)((it - b * per) / col_tiles), ct = (int)(it - b * per - (long long)rt * col_tiles);
    const int r0 = rt * 128 + rg * 8, c0 = ct * 128 + cg * 8;
    const T* src = (const T*)p.src + b * p.batch_stride + r0 * p.row_stride + c0;
    Piece<T, 8> x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (r0 + i < p.rows) x[i].load(src + i * p.row_stride, p.K - c0, vec != 0);
      else x[i].zero();
    }
    uint32_t byte = 0, inv = 0;              // square: of the tile
    if (p.square) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, x[i].amax());
      m = __reduce_max_sync(kAll, m);
      if (lane == 0) part[warp][0] = m;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, part[i][0]);
      byte = scale_byte(m, inv);
    }
    if (p.codes != nullptr) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t bi = byte, vi = inv, q[2];
        if (!p.square) bi = scale_byte(lanes_max<16>(x[i].amax()), vi);
        float v[8];
        x[i].values(v);
        cast_codes(v, bi, vi, q);
        if (r0 + i < p.rows) {
          const int row = p.first + (r0 + i) * p.step;
          if (c0 < pitch) *reinterpret_cast<uint2*>(p.codes + ((size_t)b * p.out_rows + row) * pitch + c0) = make_uint2(q[0], q[1]);
          if (cg == 0) p.scales[scale_offset(b * tiles, row, kt, ct)] = (uint8_t)bi;
        }
      }
    }
    if (p.codes_t != nullptr) {
      float v[8][8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i].values(v[i]);
      if (!p.square) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          uint32_t m = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i][j]) & 0x7fffffffu);
          m = max(m, __shfl_xor_sync(kAll, m, 16));
          if (lane < 16) part[warp][cg * 8 + j] = m;
        }
        __syncthreads();
        if (tid < 128) {
          uint32_t m = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) m = max(m, part[i][tid]);
          uint32_t iv;
          byte_of[tid] = (uint8_t)scale_byte(m, iv);
          inv_of[tid] = iv;
        }
        __syncthreads();
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int col = cg * 8 + j;
        const uint32_t bj = p.square ? byte : byte_of[col], vj = p.square ? inv : inv_of[col];
        float t[8];
        uint32_t q[2];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = v[i][j];
        cast_codes(t, bj, vj, q);
        // 8-byte slot rg of the column, moved about so that sixteen lanes meet sixteen different pairs of banks
        *reinterpret_cast<uint2*>(turned + col * 128 + ((rg ^ cg) * 8)) = make_uint2(q[0], q[1]);
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int col = i * 32 + (tid >> 3), k = tid & 7, s = col >> 3;   // slots 2k and 2k + 1 of the column
        uint4 q = *reinterpret_cast<const uint4*>(turned + col * 128 + ((k ^ (s >> 1)) * 16));
        if (s & 1) q = make_uint4(q.z, q.w, q.x, q.y);
        const int row = ct * 128 + col;
        if (row < p.K && rt * 128 + k * 16 < pitch_t)
          *reinterpret_cast<uint4*>(p.codes_t + ((size_t)b * p.K + row) * pitch_t + rt * 128 + k * 16) = q;
      }
      if (tid < 128 && ct * 128 + tid < p.K)
        p.scales_t[scale_offset(b * tiles_t, ct * 128 + tid, kt_t, rt)] = (uint8_t)(p.square ? byte : byte_of[tid]);
    }
    __syncthreads();                         // the next tile's maxima and codes go to the same places
  }
}

template <typename T, typename I>
__global__ void __launch_bounds__(kThreads)
dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int rows, int K, I items, int groups, int vec,
                  T* __restrict__ dst) {
  const int lane = threadIdx.x & 31;
  const int kt = (int)scale_tiles_k(K), pitch = (int)row_pitch(K);
  const size_t tiles = (size_t)row_tiles(rows);
  allow_dependents();
  grid_dependency_wait();
  for (I w = ((I)blockIdx.x * kThreads + threadIdx.x) >> 5; w < items; w += (I)gridDim.x * (kThreads / 32)) {
    const I r = w / (I)groups;
    const int g = (int)(w - r * (I)groups);
    const size_t b = (size_t)(r / (I)rows);
    const int row = (int)(r - (I)b * (I)rows);
    uint2 q[kUnroll];
    uint32_t byte[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int c = (g * kUnroll + u) * 256 + lane * 8;
      q[u] = make_uint2(0, 0); byte[u] = 0;
      if (c < K) {
        q[u] = __ldcs(reinterpret_cast<const uint2*>(codes + (size_t)r * pitch + c));
        byte[u] = scales[scale_offset(b * tiles, row, kt, c / kBlock)];
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int c = (g * kUnroll + u) * 256 + lane * 8;
      if (c >= K) break;
      const float s = scale_value(byte[u]);
      float v[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t word = i < 2 ? q[u].x : q[u].y;
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(word >> (16 * (i & 1))), __NV_E4M3);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
        v[2 * i] = f.x * s;                  // exact: four significant bits times a power of two
        v[2 * i + 1] = f.y * s;
      }
      Piece<T, 8> out;
      out.set(v);
      out.store(dst + (size_t)r * K + c, K - c, vec != 0);
    }
  }
}

// T: type of x, or uint8_t where x is FP8 already (its scales in tiles of their own).  d is a multiple of 16.
template <typename T, typename I>
__global__ void __launch_bounds__(kThreads)
dispatch_rows_kernel(const mx4::Dispatch q, const T* __restrict__ x, const uint8_t* __restrict__ x_scales, uint8_t* __restrict__ codes,
                     uint8_t* __restrict__ scales, I items, int groups) {
  const int lane = threadIdx.x & 31;
  const int kt = (int)scale_tiles_k(q.d);
  allow_dependents();
  grid_dependency_wait();
  for (I w = ((I)blockIdx.x * kThreads + threadIdx.x) >> 5; w < items; w += (I)gridDim.x * (kThreads / 32)) {
    const size_t t = (size_t)(w / (I)groups);
    const int g = (int)(w - (I)t * (I)groups);
    const int c0 = g * kUnroll * 256 + lane * 8;
    const T* from = x + t * q.d + c0;
    uint2 code[kUnroll];
    uint32_t byte[kUnroll];
    if constexpr (sizeof(T) == 1) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        code[u] = make_uint2(0, 0); byte[u] = 0;
        if (c0 + u * 256 < q.d) {
          code[u] = __ldcs(reinterpret_cast<const uint2*>(from + u * 256));
          byte[u] = x_scales[scale_offset(0, (int)t, kt, (c0 + u * 256) / kBlock)];
        }
      }
    } else {
      Piece<T, 8> v[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) v[u].load(from + u * 256, q.d - (c0 + u * 256), true);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        uint32_t inv, out[2];
        float f[8];
        byte[u] = scale_byte(lanes_max<16>(v[u].amax()), inv);
        v[u].values(f);
        cast_codes(f, byte[u], inv, out);
        code[u] = make_uint2(out[0], out[1]);
      }
    }
    for (int j = 0; j < q.k; ++j) {
      const int row = q.flat2row[t * q.k + j];
      if (row < 0) continue;
      uint8_t* to = codes + (size_t)row * q.d + c0;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int c = c0 + u * 256;
        if (c < q.d) {
          *reinterpret_cast<uint2*>(to + u * 256) = code[u];
          if ((lane & 15) == 0) scales[scale_offset(0, row, kt, c / kBlock)] = (uint8_t)byte[u];
        }
      }
    }
  }
}

int cast_blocks(long long items) {
  const long long want = (items + kThreads / 32 - 1) / (kThreads / 32), most = 32ll * sm_count();
  return (int)(want < most ? want : most);
}
int cast_groups(int K) { return (int)((row_pitch(K) + 256 * kUnroll - 1) / (256 * kUnroll)); }

template <typename F> cudaError_t by_index(long long items, F&& f) {
  // numbers reach items plus one round of the grid
  return items < (1ll << 31) ? f((uint32_t)items) : f((uint64_t)items);
}

template <typename T> cudaError_t quantize(const CastParams& p, cudaStream_t st) {
  const int vec = ((uintptr_t)p.src & 15) == 0 && p.row_stride * sizeof(T) % 16 == 0 && p.batch_stride * sizeof(T) % 16 == 0;
  if (p.square || p.codes_t != nullptr) {
    const int col_tiles = (int)((p.K + 127ll) / 128);
    const long long items = (long long)p.batch * row_tiles(p.rows) * col_tiles, most = 8ll * sm_count();
    return launch_after_predecessor(quantize_tiles_kernel<T>, dim3((unsigned)(items < most ? items : most)), dim3(kThreads), 0, st, true,
                                    p, vec, items, col_tiles);
  }
  const int groups = cast_groups(p.K);
  const long long items = (long long)p.batch * p.rows * groups;
  return by_index(items, [&](auto n) {
    return launch_after_predecessor(quantize_rows_kernel<T, decltype(n)>, dim3(cast_blocks(items)), dim3(kThreads), 0, st, true, p, vec,
                                    n, groups);
  });
}

template <typename T>
cudaError_t dequantize(const uint8_t* codes, const uint8_t* scales, int batch, int rows, int K, T* dst, cudaStream_t st) {
  const int groups = cast_groups(K);
  const long long items = (long long)batch * rows * groups;
  const int vec = K * sizeof(T) % 16 == 0;
  return by_index(items, [&](auto n) {
    return launch_after_predecessor(dequantize_kernel<T, decltype(n)>, dim3(cast_blocks(items)), dim3(kThreads), 0, st, true, codes,
                                    scales, rows, K, n, groups, vec, dst);
  });
}

template <typename T>
cudaError_t dispatch_rows(const mx4::Dispatch& q, const T* x, const uint8_t* x_scales, uint8_t* codes, uint8_t* scales, cudaStream_t st) {
  const int groups = cast_groups(q.d);
  const long long items = (long long)q.T * groups;
  return by_index(items, [&](auto n) {
    return launch_after_predecessor(dispatch_rows_kernel<T, decltype(n)>, dim3(cast_blocks(items)), dim3(kThreads), 0, st, true, q, x,
                                    x_scales, codes, scales, n, groups);
  });
}

}  // namespace

cudaError_t launch_dispatch_rows(const mx4::Dispatch& q, int dtype, const void* x, const uint8_t* x_scales, uint8_t* codes,
                                 uint8_t* scales, cudaStream_t st) {
  if (x_scales != nullptr) return dispatch_rows(q, (const uint8_t*)x, x_scales, codes, scales, st);
  return dtype == BTX_BF16 ? dispatch_rows(q, (const __nv_bfloat16*)x, x_scales, codes, scales, st)
                           : dispatch_rows(q, (const float*)x, x_scales, codes, scales, st);
}

cudaError_t launch_quantize(const CastParams& p, int dtype, cudaStream_t st) {
  return dtype == BTX_BF16 ? quantize<__nv_bfloat16>(p, st) : quantize<float>(p, st);
}

cudaError_t launch_dequantize(const uint8_t* codes, const uint8_t* scales, int batch, int rows, int K, int dtype, void* dst,
                              cudaStream_t st) {
  return dtype == BTX_BF16 ? dequantize(codes, scales, batch, rows, K, (__nv_bfloat16*)dst, st)
                           : dequantize(codes, scales, batch, rows, K, (float*)dst, st);
}

}  // namespace fp8
}  // namespace btx
