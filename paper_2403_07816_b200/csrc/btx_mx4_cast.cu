// MXFP4 casts and the row dispatch of the expert layer on MXFP4 weights: the memory-bound steps around the products.
//
//   quantize     per 32 elements: scale 2^(floor(log2 max|x|) - 2), elements to the nearest e2m1 value (ties to the
//                even code, at most 6).  Four lanes share a block, eight elements each: a warp reads 256 consecutive
//                elements with 16-byte loads, the maximum takes two shuffles, a lane stores four bytes of codes and
//                every fourth the scale byte.  2 + 17/32 bytes per bf16 element, 6.0 TB/s for large matrices, 0.93 of the
//                measured copy rate, at 88 % of the issue slots.
//   dequantize   the same mapping backwards
//   dispatch     stable counting sort of the assignments by expert, padded to 128-row tiles
//   quantize_rows  quantize of x with every row written to the k rows of its token: x is read once
#include "btx_mx4_dev.cuh"

namespace btx {
namespace mx4 {
namespace {

constexpr int kCastThreads = 256;
constexpr int kSortThreads = 512;
constexpr int kSortOne = 2048;             // assignments that one block dispatches on its own

// A warp takes kCastUnroll chunks of 256 elements of one row at a time.  I: the type that numbers them; the two divisions
// in 64 bits cost as many instructions as the cast of the chunks.
template <typename T, typename I>
__global__ void __launch_bounds__(kCastThreads)
quantize_kernel(const CastParams p, int vec, I items, int groups) {
  const int lane = threadIdx.x & 31;
  const int kt = (int)scale_tiles_k(p.K);
  allow_dependents();
  grid_dependency_wait();
  const size_t tiles = ((size_t)p.out_rows + kTileRows - 1) / kTileRows;
  for (I w = ((I)blockIdx.x * kCastThreads + threadIdx.x) >> 5; w < items; w += (I)gridDim.x * (kCastThreads / 32)) {
    const I r = w / (I)groups;
    const int g = (int)(w - r * (I)groups);
    const int b = (int)(r / (I)p.rows), row = (int)(r - (I)b * (I)p.rows);
    const T* src = (const T*)p.src + b * p.batch_stride + row * p.row_stride;
    const int out_row = p.first + row * p.step;
    const int c0 = g * kCastUnroll * 256 + lane * 8;
    Eight<T> x[kCastUnroll];
#pragma unroll
    for (int u = 0; u < kCastUnroll; ++u) {
      if (c0 + u * 256 < p.K) x[u].load(src + c0 + u * 256, vec != 0);
      else x[u].zero();
    }
    uint8_t* codes = p.codes + ((size_t)b * p.out_rows + out_row) * (p.K / 2) + c0 / 2;
    uint8_t* scales = p.scales + scale_offset(b * tiles, out_row, kt, c0 / 128) + (c0 / kBlock & 3);
#pragma unroll
    for (int u = 0; u < kCastUnroll; ++u) {
      uint32_t byte;
      const uint32_t q = cast8(x[u], byte);
      if (c0 + u * 256 < p.K) *reinterpret_cast<uint32_t*>(codes + u * 128) = q;
      if ((lane & 3) == 0 && c0 + u * 256 < kt * 128) scales[u * 2 * kTileBytes] = (uint8_t)byte;
    }
  }
}

template <typename T> __device__ __forceinline__ void store8(T* p, const float (&v)[8]);
template <> __device__ __forceinline__ void store8<float>(float* p, const float (&v)[8]) {
  __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
  __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
}
template <> __device__ __forceinline__ void store8<__nv_bfloat16>(__nv_bfloat16* p, const float (&v)[8]) {
  __nv_bfloat162 h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
  __stcs(reinterpret_cast<uint4*>(p), *reinterpret_cast<uint4*>(h));
}

template <typename T, typename I>
__global__ void __launch_bounds__(kCastThreads)
dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int rows, int K, I items, int groups,
                  T* __restrict__ dst) {
  const int lane = threadIdx.x & 31;
  const int kt = (int)scale_tiles_k(K);
  allow_dependents();
  grid_dependency_wait();
  const size_t tiles = ((size_t)rows + kTileRows - 1) / kTileRows;
  for (I w = ((I)blockIdx.x * kCastThreads + threadIdx.x) >> 5; w < items; w += (I)gridDim.x * (kCastThreads / 32)) {
    const I r = w / (I)groups;
    const int g = (int)(w - r * (I)groups);
    const size_t b = (size_t)(r / (I)rows);
    const int row = (int)(r - (I)b * (I)rows);
    uint32_t q[kCastUnroll], byte[kCastUnroll];
#pragma unroll
    for (int u = 0; u < kCastUnroll; ++u) {
      const int c = (g * kCastUnroll + u) * 256 + lane * 8;
      q[u] = 0; byte[u] = 0;
      if (c < K) {
        q[u] = *reinterpret_cast<const uint32_t*>(codes + (size_t)r * (K / 2) + c / 2);
        byte[u] = scales[scale_offset(b * tiles, row, kt, c / 128) + (c / kBlock & 3)];
      }
    }
#pragma unroll
    for (int u = 0; u < kCastUnroll; ++u) {
      const int c = (g * kCastUnroll + u) * 256 + lane * 8;
      if (c >= K) break;
      const float s = byte[u] == 255u ? __uint_as_float(0x7fffffffu)
                                      : __uint_as_float(byte[u] == 0u ? 0x00400000u : byte[u] << 23);
      float v[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)(q[u] >> (8 * i)), __NV_E2M1);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
        v[2 * i] = f.x * s;                 // exact: at most two significant bits times a power of two
        v[2 * i + 1] = f.y * s;
      }
      store8<T>(dst + (size_t)r * K + c, v);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Dispatch
// ---------------------------------------------------------------------------------------------
// Offsets of the experts' padded segments from their counts in shared memory (one block): pad[e], and the list of
// the expert of every tile.
__device__ __forceinline__ void place_experts(int E, int pad_tiles, const int* cnt, int* pad, int* __restrict__ scan,
                                              int32_t* __restrict__ tile_expert, int32_t* __restrict__ tile_rows,
                                              int32_t* __restrict__ n_tiles, int32_t* __restrict__ pad_offsets) {
  const int tid = threadIdx.x;               // kSortThreads >= kMaxExperts4: a thread per expert
  const int lane = tid & 31, warp = tid >> 5;
  const int unit = pad_tiles * kTileRows;
  const int tiles = tid < E ? (cnt[tid] + unit - 1) / unit * pad_tiles : 0;
  int incl = tiles;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(kAll, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) scan[warp] = incl;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < warp; ++w) before += scan[w];
  const int first = before + incl - tiles;
  if (tid < E) {
    pad[tid] = first * kTileRows;
    if (pad_offsets != nullptr) pad_offsets[tid] = first * kTileRows;
    for (int j = 0; j < tiles; ++j) {
      tile_expert[first + j] = tid;
      tile_rows[first + j] = max(0, min(kTileRows, cnt[tid] - j * kTileRows));
    }
  }
  if (tid == E - 1) {
    n_tiles[0] = first + tiles;
    if (pad_offsets != nullptr) pad_offsets[E] = (first + tiles) * kTileRows;
  }
  __syncthreads();
}

// Stable ranks of one block's assignments inside their experts, in rounds of kSortThreads; running[e] is the rank
// the next one gets.  Bucket E takes assignments without an expert.
__device__ __forceinline__ void scatter_rounds(int begin, int end, int E, const int32_t* __restrict__ topk_idx,
                                               int* running, int (*wcnt)[kMaxExperts4 + 1], const int* pad,
                                               int32_t* __restrict__ flat2row, int32_t* __restrict__ rowmap) {
  constexpr int NW = kSortThreads / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int r0 = begin; r0 < end; r0 += kSortThreads) {
    for (int j = threadIdx.x; j <= E; j += kSortThreads)
#pragma unroll
      for (int w = 0; w < NW; ++w) wcnt[w][j] = 0;
    __syncthreads();
    const int i = r0 + threadIdx.x;
    int e = E;
    if (i < end) {
      e = topk_idx[i];
      if ((unsigned)e >= (unsigned)E) e = E;
    }
    const unsigned same = __match_any_sync(kAll, e);
    const int rank = __popc(same & ((1u << lane) - 1u));
    if (rank == 0) wcnt[warp][e] = __popc(same);
    __syncthreads();
    if (i < end) {
      int row = -1;
      if (e < E) {
        int before = 0;
        for (int w = 0; w < warp; ++w) before += wcnt[w][e];
        row = pad[e] + running[e] + before + rank;
        rowmap[row] = i;
      }
      flat2row[i] = row;
    }
    __syncthreads();
    for (int q = threadIdx.x; q < E; q += kSortThreads) {
      int s = 0;
      for (int w = 0; w < NW; ++w) s += wcnt[w][q];
      running[q] += s;
    }
    __syncthreads();
  }
}

// padding rows of all experts: a warp per expert
__device__ __forceinline__ void clear_padding(int E, int pad_tiles, const int* cnt, const int* pad, int32_t* __restrict__ rowmap) {
  const int unit = pad_tiles * kTileRows;
  for (int e = threadIdx.x >> 5; e < E; e += blockDim.x >> 5)
    for (int r = cnt[e] + (threadIdx.x & 31); r < (cnt[e] + unit - 1) / unit * unit; r += 32) rowmap[pad[e] + r] = -1;
}

struct SortShared {
  int wcnt[kSortThreads / 32][kMaxExperts4 + 1];
  int cnt[kMaxExperts4 + 1], running[kMaxExperts4 + 1], pad[kMaxExperts4 + 1], scan[kSortThreads / 32];
};

// The whole dispatch of a batch of at most kSortOne assignments in one block.
__global__ void __launch_bounds__(kSortThreads)
dispatch_one_kernel(const Dispatch q) {
  __shared__ SortShared s;
  allow_dependents();
  grid_dependency_wait();
  if (threadIdx.x < kStatusWords) q.status[threadIdx.x] = 0;
  for (int i = threadIdx.x; i <= kMaxExperts4; i += kSortThreads) { s.cnt[i] = 0; s.running[i] = 0; }
  __syncthreads();
  for (int i = threadIdx.x; i < q.R; i += kSortThreads) {
    const int e = q.topk_idx[i];
    if ((unsigned)e < (unsigned)q.E) atomicAdd(&s.cnt[e], 1);
  }
  __syncthreads();
  place_experts(q.E, q.pad_tiles, s.cnt, s.pad, s.scan, q.tile_expert, q.tile_rows, q.n_tiles, nullptr);
  clear_padding(q.E, q.pad_tiles, s.cnt, s.pad, q.rowmap);
  scatter_rounds(0, q.R, q.E, q.topk_idx, s.running, s.wcnt, s.pad, q.flat2row, q.rowmap);
}

__global__ void __launch_bounds__(kSortThreads)
dispatch_count_kernel(const Dispatch q) {
  __shared__ int hist[kMaxExperts4];
  allow_dependents();
  grid_dependency_wait();
  if (blockIdx.x == 0 && threadIdx.x < kStatusWords) q.status[threadIdx.x] = 0;
  for (int i = threadIdx.x; i < q.E; i += kSortThreads) hist[i] = 0;
  __syncthreads();
  const int begin = blockIdx.x * q.chunk, end = min(q.R, begin + q.chunk);
  for (int i = begin + threadIdx.x; i < end; i += kSortThreads) {
    const int e = q.topk_idx[i];
    if ((unsigned)e < (unsigned)q.E) atomicAdd(&hist[e], 1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < q.E; i += kSortThreads) q.block_counts[(size_t)blockIdx.x * q.E + i] = hist[i];
}

// counts per block -> the rank each block starts at, in place; segments and tiles of the experts
__global__ void __launch_bounds__(kSortThreads)
dispatch_scan_kernel(const Dispatch q) {
  __shared__ int cnt[kMaxExperts4 + 1], pad[kMaxExperts4 + 1], scan[kSortThreads / 32];
  allow_dependents();
  grid_dependency_wait();
  const int e = threadIdx.x;
  if (e < q.E) {
    int run = 0;
    for (int b0 = 0; b0 < q.blocks; b0 += 8) {
      int v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = b0 + i < q.blocks ? q.block_counts[(size_t)(b0 + i) * q.E + e] : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (b0 + i < q.blocks) q.block_counts[(size_t)(b0 + i) * q.E + e] = run;
        run += v[i];
      }
    }
    cnt[e] = run;
  }
  __syncthreads();
  place_experts(q.E, q.pad_tiles, cnt, pad, scan, q.tile_expert, q.tile_rows, q.n_tiles, q.pad_offsets);
  clear_padding(q.E, q.pad_tiles, cnt, pad, q.rowmap);
}

__global__ void __launch_bounds__(kSortThreads)
dispatch_scatter_kernel(const Dispatch q) {
  __shared__ SortShared s;
  allow_dependents();
  grid_dependency_wait();
  for (int i = threadIdx.x; i < q.E; i += kSortThreads) {
    s.running[i] = q.block_counts[(size_t)blockIdx.x * q.E + i];
    s.pad[i] = q.pad_offsets[i];
  }
  __syncthreads();
  const int begin = blockIdx.x * q.chunk;
  scatter_rounds(begin, min(q.R, begin + q.chunk), q.E, q.topk_idx, s.running, s.wcnt, s.pad, q.flat2row, q.rowmap);
}

template <typename T, typename I>
__global__ void __launch_bounds__(kCastThreads)
quantize_rows_kernel(const Dispatch q, const T* __restrict__ x, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                     I items, int groups) {
  const int lane = threadIdx.x & 31;
  allow_dependents();
  grid_dependency_wait();
  for (I w = ((I)blockIdx.x * kCastThreads + threadIdx.x) >> 5; w < items; w += (I)gridDim.x * (kCastThreads / 32)) {
    const size_t t = (size_t)(w / (I)groups);
    const int g = (int)(w - (I)t * (I)groups);
    cast_token_rows<T>(x + t * q.d, q.d, g, lane, q.k, q.flat2row + t * q.k, codes, scales);
  }
}

// A thread owns 16 bytes of y; slots are added in order, in fp32, and rounded once.
template <typename T>
__global__ void __launch_bounds__(256)
combine_rows_kernel(int Tn, int d, int k, const float* __restrict__ rows, const int32_t* __restrict__ flat2row,
                    T* __restrict__ y) {
  constexpr int VN = Vec<T>::N;
  const int vecs = d / VN;
  allow_dependents();
  grid_dependency_wait();
  for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < (size_t)Tn * vecs; i += (size_t)gridDim.x * blockDim.x) {
    const size_t t = i / vecs;
    const int c = (int)(i - t * vecs) * VN;
    float acc[VN];
#pragma unroll
    for (int j = 0; j < VN; ++j) acc[j] = 0.f;
    for (int s = 0; s < k; ++s) {
      if (flat2row[t * k + s] < 0) continue;               // its row was never written
      const float* r = rows + (t * k + s) * d + c;
#pragma unroll
      for (int j = 0; j < VN; j += 4) {
        const float4 q = __ldcs(reinterpret_cast<const float4*>(r + j));
        acc[j] += q.x; acc[j + 1] += q.y; acc[j + 2] += q.z; acc[j + 3] += q.w;
      }
    }
    __align__(16) T out[VN];
#pragma unroll
    for (int j = 0; j < VN; ++j) out[j] = from_f32<T>(acc[j]);
    *reinterpret_cast<uint4*>(y + t * d + c) = *reinterpret_cast<const uint4*>(out);
  }
}

// More blocks than fit at once: with 32 for every multiprocessor the cast of four 11008 x 4096 matrices (bf16) takes 76 us
// and the way back 74, with 8 86 and 86 (all blocks walk through memory in step), with 64 78 and 76.
int cast_blocks(long long items) {
  const long long want = (items + kCastThreads / 32 - 1) / (kCastThreads / 32), most = 32ll * sm_count();
  return (int)(want < most ? want : most);
}
int cast_groups(int K) { return (K + 256 * kCastUnroll - 1) / (256 * kCastUnroll); }

}  // namespace

template <typename F> static cudaError_t by_index(long long items, F&& f) {
  // numbers reach items plus one round of the grid
  return items < (1ll << 31) ? f((uint32_t)items) : f((uint64_t)items);
}

cudaError_t launch_quantize(const CastParams& p, int dtype, cudaStream_t st) {
  const int groups = cast_groups(p.K);
  const long long items = (long long)p.batch * p.rows * groups;
  const int esize = dtype == BTX_BF16 ? 2 : 4;
  const int vec = ((uintptr_t)p.src & 15) == 0 && p.row_stride * esize % 16 == 0 && p.batch_stride * esize % 16 == 0;
  return by_index(items, [&](auto n) {
    using I = decltype(n);
    if (dtype == BTX_BF16)
      return launch_after_predecessor(quantize_kernel<__nv_bfloat16, I>, dim3(cast_blocks(items)), dim3(kCastThreads), 0, st, true, p,
                                      vec, n, groups);
    return launch_after_predecessor(quantize_kernel<float, I>, dim3(cast_blocks(items)), dim3(kCastThreads), 0, st, true, p, vec, n,
                                    groups);
  });
}

cudaError_t launch_dequantize(const uint8_t* codes, const uint8_t* scales, int batch, int rows, int K, int dtype, void* dst,
                              cudaStream_t st) {
  const int groups = cast_groups(K);
  const long long items = (long long)batch * rows * groups;
  return by_index(items, [&](auto n) {
    using I = decltype(n);
    if (dtype == BTX_BF16)
      return launch_after_predecessor(dequantize_kernel<__nv_bfloat16, I>, dim3(cast_blocks(items)), dim3(kCastThreads), 0, st, true,
                                      codes, scales, rows, K, n, groups, (__nv_bfloat16*)dst);
    return launch_after_predecessor(dequantize_kernel<float, I>, dim3(cast_blocks(items)), dim3(kCastThreads), 0, st, true, codes,
                                    scales, rows, K, n, groups, (float*)dst);
  });
}

// Assignments per block: whole rounds of the block's threads, few enough rounds that at most 592 blocks share a batch (the
// scan walks over the blocks).
int dispatch_chunk(long long R) {
  if (R <= kSortOne) return kSortOne;
  const long long rounds = (R + kSortThreads * 592ll - 1) / (kSortThreads * 592ll);
  return (int)(rounds * kSortThreads);
}

cudaError_t launch_dispatch(const Dispatch& q, cudaStream_t st) {
  if (q.blocks <= 1) {
    return launch_after_predecessor(dispatch_one_kernel, dim3(1), dim3(kSortThreads), 0, st, true, q);
  }
  cudaError_t e = launch_after_predecessor(dispatch_count_kernel, dim3(q.blocks), dim3(kSortThreads), 0, st, true, q);
  if (e != cudaSuccess) return e;
  if ((e = launch_after_predecessor(dispatch_scan_kernel, dim3(1), dim3(kSortThreads), 0, st, true, q)) != cudaSuccess) return e;
  return launch_after_predecessor(dispatch_scatter_kernel, dim3(q.blocks), dim3(kSortThreads), 0, st, true, q);
}

cudaError_t launch_quantize_rows(const Dispatch& q, int dtype, const void* x, uint8_t* codes, uint8_t* scales, cudaStream_t st) {
  const int groups = cast_groups(q.d);
  const long long items = (long long)q.T * groups;
  return by_index(items, [&](auto n) {
    using I = decltype(n);
    if (dtype == BTX_BF16)
      return launch_after_predecessor(quantize_rows_kernel<__nv_bfloat16, I>, dim3(cast_blocks(items)), dim3(kCastThreads), 0, st,
                                      true, q, (const __nv_bfloat16*)x, codes, scales, n, groups);
    return launch_after_predecessor(quantize_rows_kernel<float, I>, dim3(cast_blocks(items)), dim3(kCastThreads), 0, st, true, q,
                                    (const float*)x, codes, scales, n, groups);
  });
}

cudaError_t launch_combine_rows(const Dispatch& q, int dtype, const float* rows, void* y, cudaStream_t st) {
  const size_t n = (size_t)q.T * (q.d / (dtype == BTX_BF16 ? 8 : 4));
  const size_t want = (n + 255) / 256, most = (size_t)sm_count() * 32;
  const dim3 grid((unsigned)(want < most ? want : most));
  if (dtype == BTX_BF16)
    return launch_after_predecessor(combine_rows_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, true, q.T, q.d, q.k, rows,
                                    (const int32_t*)q.flat2row, (__nv_bfloat16*)y);
  return launch_after_predecessor(combine_rows_kernel<float>, grid, dim3(256), 0, st, true, q.T, q.d, q.k, rows,
                                  (const int32_t*)q.flat2row, (float*)y);
}

}  // namespace mx4
}  // namespace btx
