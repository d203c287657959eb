// FP8 casts: one power-of-two scale for 128 elements of a row, or for a block of 128 x 128.
//
//   quantize_rows   a scale per row and 128 elements, as the rows stand: a warp takes 256 elements at a time
//   quantize_tiles  square blocks and transposed outputs: a block of threads works on 128 x 128 tiles, eight neighbouring rows of
//                   16 bytes a thread, which gives the largest of its rows, of its columns or of all; x is read once for
//                   both outputs.  The next tile is on its way meanwhile (cp.async into the thread's own places in shared
//                   memory).  Transposed codes turn through shared memory, 8 bytes (of 8 rows) at a time
//   dequantize      the mapping of quantize_rows backwards
//   dispatch_rows   quantize_rows of the expert layer's tokens, or a copy of their FP8 form, to the k rows of every token
//
// VEC: rows start on 16-byte boundaries and hold whole vectors; otherwise they are read element by element, by the same lanes.
//
// All are bound by memory and by the instructions of the casts.  Measured on one B200 (replayed; the floor is the bytes at the
// 6561 GB/s of a copy): 16384 x 4096 bf16 as rows 29.7 us (30.7), as rows and transposed 54.4 (40.9), back to bf16 31.6 (30.7);
// 2 x 11008 x 4096 fp32 in square blocks, both ways, 101 (82.5), back 42.3 (41.3).  quantize_tiles is at 69 % of the issue slots.
// Rows off 16-byte boundaries: rows 60, both ways 110, back 64.
#include <atomic>

#include "btx_fp8_dev.cuh"
#include "btx_fp8_gemm.cuh"

namespace btx {
namespace fp8 {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;                 // 256-element chunks a warp has in flight

// A warp takes kUnroll chunks of 256 elements of one row at a time, eight neighbours a lane: sixteen lanes share a block.
template <typename T, bool VEC, typename I>
__global__ void __launch_bounds__(kThreads)
quantize_rows_kernel(const __grid_constant__ CastParams p, I items, int groups) {
  const int lane = threadIdx.x & 31;
  const int kt = (int)scale_tiles_k(p.K), pitch = (int)row_pitch(p.K);
  const size_t tiles = (size_t)row_tiles(p.out_rows);
  allow_dependents();
  grid_dependency_wait();
  for (I w = ((I)blockIdx.x * kThreads + threadIdx.x) >> 5; w < items; w += (I)gridDim.x * (kThreads / 32)) {
    const I r = w / (I)groups;
    const int g = (int)(w - r * (I)groups);
    const int b = (int)(r / (I)p.rows), row = (int)(r - (I)b * (I)p.rows);
    const int out_row = p.first + row * p.step;
    const int c0 = g * kUnroll * 256 + lane * 8, left = p.K - c0;
    const T* src = (const T*)p.src + b * p.batch_stride + row * p.row_stride + c0;
    uint8_t* codes = p.codes + ((size_t)b * p.out_rows + out_row) * pitch + c0;
    uint8_t* scales = p.scales + scale_offset(b * tiles, out_row, kt, g * kUnroll * 2);    // (two scale tiles, eight blocks)
    Piece<T, 8> x[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (u * 256 < left) x[u].load(src + u * 256, VEC ? 8 : left - u * 256, VEC);
      else x[u].zero();
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      uint32_t inv, q[2];
      const uint32_t byte = scale_byte(lanes_max<16>(x[u].amax()), inv);
      float v[8];
      x[u].values(v);
      cast_codes(v, byte, inv, q);
      if (u * 256 < left + pitch - p.K) *reinterpret_cast<uint2*>(codes + u * 256) = make_uint2(q[0], q[1]);
      if ((lane & 15) == 0 && u * 256 < left) scales[(u >> 1) * kTileBytes + (u & 1) * 2 + (lane >> 4)] = (uint8_t)byte;
    }
  }
}

// Threads of a tile: 16 groups of eight rows, 16 bytes of a row each.
template <typename T> struct Tile {
  static constexpr int VN = 16 / (int)sizeof(T), LANES = 128 / VN, THREADS = 16 * LANES;
  static constexpr int ROWS_BYTES = THREADS * 8 * 16, SMEM = ROWS_BYTES + 128 * 128;
  static constexpr int BLOCKS = sizeof(T) == 2 ? 3 : 2;       // resident on a multiprocessor
};
// magnitudes of the elements of a word, and the larger ones of two words (as integers: NaN and infinities are above all numbers)
template <typename T> __device__ __forceinline__ uint32_t word_abs(uint32_t w) { return w & (sizeof(T) == 2 ? 0x7fff7fffu : 0x7fffffffu); }
template <typename T> __device__ __forceinline__ uint32_t word_max(uint32_t a, uint32_t b) { return sizeof(T) == 2 ? __vmaxu2(a, b) : max(a, b); }

// Largest magnitudes of eight rows over the LANES lanes that share them, from m[i], the lane's words of row i.  Lanes hand each
// other half of what is left to reduce, so a lane ends up with one row (bf16: two in a word); their scale bytes go to row_byte.
template <typename T> __device__ __forceinline__ void rows_scales(const uint32_t (&m)[8], int cg, uint8_t* row_byte) {
  if constexpr (sizeof(T) == 2) {
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __vmaxu2(__byte_perm(m[2 * i], m[2 * i + 1], 0x5410), __byte_perm(m[2 * i], m[2 * i + 1], 0x7632));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t got = __shfl_xor_sync(kAll, cg & 8 ? r[i] : r[i + 2], 8);
      r[i] = __vmaxu2(cg & 8 ? r[i + 2] : r[i], got);
    }
    const uint32_t got = __shfl_xor_sync(kAll, cg & 4 ? r[0] : r[1], 4);
    uint32_t a = __vmaxu2(cg & 4 ? r[1] : r[0], got);
    a = __vmaxu2(a, __shfl_xor_sync(kAll, a, 2));
    a = __vmaxu2(a, __shfl_xor_sync(kAll, a, 1));
    uint32_t inv;
    const uint32_t lo = scale_byte(a << 16, inv), hi = scale_byte(a & 0xffff0000u, inv);
    if ((cg & 3) == 0) *reinterpret_cast<uint16_t*>(row_byte + (cg >> 2) * 2) = (uint16_t)(lo | hi << 8);
  } else {
    uint32_t r[4], t[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = max(cg & 16 ? m[i + 4] : m[i], __shfl_xor_sync(kAll, cg & 16 ? m[i] : m[i + 4], 16));
#pragma unroll
    for (int i = 0; i < 2; ++i) t[i] = max(cg & 8 ? r[i + 2] : r[i], __shfl_xor_sync(kAll, cg & 8 ? r[i] : r[i + 2], 8));
    uint32_t a = max(cg & 4 ? t[1] : t[0], __shfl_xor_sync(kAll, cg & 4 ? t[0] : t[1], 4)), inv;
    a = max(a, __shfl_xor_sync(kAll, a, 2));
    a = max(a, __shfl_xor_sync(kAll, a, 1));
    if ((cg & 3) == 0) row_byte[cg >> 2] = (uint8_t)scale_byte(a, inv);
  }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(Tile<T>::THREADS, Tile<T>::BLOCKS)
quantize_tiles_kernel(const __grid_constant__ CastParams p, long long items, int col_tiles, int words) {
  using G = Tile<T>;
  constexpr int VN = G::VN, LANES = G::LANES, WARPS = G::THREADS / 32, PER = VN / 4;      // PER: elements of a word
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ uint32_t part[WARPS][128 / PER];       // largest of every column over a warp's rows
  __shared__ uint32_t whole[2][WARPS];     // of a square block, for tiles in turn
  __shared__ uint32_t inv_of[128];
  __shared__ uint8_t byte_of[128];
  __shared__ __align__(8) uint8_t row_byte[128];
  uint8_t* turned = smem + G::ROWS_BYTES;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cg = tid % LANES, rg = tid / LANES;
  const int kt = (int)scale_tiles_k(p.K), pitch = (int)row_pitch(p.K);
  const int kt_t = (int)scale_tiles_k(p.rows), pitch_t = (int)row_pitch(p.rows);
  const size_t tiles = (size_t)row_tiles(p.out_rows), tiles_t = (size_t)row_tiles(p.K);
  const long long per = (long long)col_tiles * row_tiles(p.rows);
  const uint32_t places = (uint32_t)__cvta_generic_to_shared(smem) + tid * 16;
  auto place = [&](int i) { return places + i * G::THREADS * 16; };
  allow_dependents();
  grid_dependency_wait();

  auto locate = [&](long long it, int& b, int& rt, int& ct) {
    b = (int)(it / per);
    rt = (int)((it - b * per) / col_tiles);
    ct = (int)(it - b * per - (long long)rt * col_tiles);
  };
  auto fetch = [&](long long it) {
    if (it < items) {
      int b, rt, ct;
      locate(it, b, rt, ct);
      const int r0 = rt * 128 + rg * 8, left = max(0, p.K - ct * 128 - cg * VN);       // elements of a row from here on
      const T* src = (const T*)p.src + b * p.batch_stride + r0 * p.row_stride + ct * 128 + cg * VN;
      if (VEC || words) {                    // copies of 16 or 4 bytes; nothing is read where the size is 0
        const int bytes = min(16, left * (int)sizeof(T));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int n = r0 + i < p.rows ? bytes : 0;
          const uint8_t* from = n > 0 ? reinterpret_cast<const uint8_t*>(src + i * p.row_stride) : reinterpret_cast<const uint8_t*>(p.src);
          if (VEC) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(place(i)), "l"(from), "r"(n) : "memory");
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(place(i) + 4 * k), "l"(4 * k < n ? from + 4 * k : from), "r"(4 * k < n ? 4 : 0) : "memory");
          }
        }
      } else {
        Piece<T, VN> q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i].load(src + i * p.row_stride, r0 + i < p.rows ? left : 0, false);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(place(i)), "r"(q[i].w[0]), "r"(q[i].w[1]), "r"(q[i].w[2]),
                       "r"(q[i].w[3]) : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  fetch(blockIdx.x);
  int turn = 0;
  for (long long it = blockIdx.x; it < items; it += gridDim.x, turn ^= 1) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    int b, rt, ct;
    locate(it, b, rt, ct);
    const int r0 = rt * 128 + rg * 8, c0 = ct * 128;
    Piece<T, VN> x[8];
    uint32_t most[4], row_most[8];           // words of magnitudes: largest of the thread's columns, of its rows
#pragma unroll
    for (int i = 0; i < 8; ++i)
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x[i].w[0]), "=r"(x[i].w[1]), "=r"(x[i].w[2]), "=r"(x[i].w[3]) : "r"(place(i)) : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t a[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        a[k] = word_abs<T>(x[i].w[k]);
        most[k] = i == 0 ? a[k] : word_max<T>(most[k], a[k]);
      }
      row_most[i] = word_max<T>(word_max<T>(a[0], a[1]), word_max<T>(a[2], a[3]));
    }
    fetch(it + gridDim.x);                   // the places are free: this tile is in registers
    uint32_t byte = 0, inv = 0;              // square: of the tile
    if (p.square) {
      uint32_t m = word_max<T>(word_max<T>(most[0], most[1]), word_max<T>(most[2], most[3]));
      m = __reduce_max_sync(kAll, PER == 2 ? max(m & 0xffff0000u, m << 16) : m);
      if (lane == 0) whole[turn][warp] = m;
      __syncthreads();
      byte = scale_byte(__reduce_max_sync(kAll, whole[turn][lane % WARPS]), inv);
    } else if (p.codes_t != nullptr) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (LANES == 16) most[k] = word_max<T>(most[k], __shfl_xor_sync(kAll, most[k], 16));
        if (lane < LANES) part[warp][cg * 4 + k] = most[k];
      }
    }
    if (p.codes != nullptr) {
      uint8_t* to = p.codes + ((size_t)b * p.out_rows + p.first + (size_t)r0 * p.step) * pitch + c0 + cg * VN;
      const size_t next = (size_t)p.step * pitch;
      const int n = c0 + cg * VN < pitch ? p.rows - r0 : 0;                              // rows to write
      uint2 bytes = make_uint2(0, 0);
      if (!p.square) {
        rows_scales<T>(row_most, cg, row_byte + rg * 8);
        __syncwarp();
        bytes = *reinterpret_cast<const uint2*>(row_byte + rg * 8);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t bi = byte, vi = inv, q[VN / 4];
        if (!p.square) {
          bi = (i < 4 ? bytes.x : bytes.y) >> (8 * (i & 3)) & 255u;
          vi = (254u - bi) << 23;            // (of no use where the byte is 255)
        }
        float v[VN];
        x[i].values(v);
        cast_codes(v, bi, vi, q);
        if (i < n) {
          if constexpr (VN == 8) *reinterpret_cast<uint2*>(to + i * next) = make_uint2(q[0], q[1]);
          else *reinterpret_cast<uint32_t*>(to + i * next) = q[0];
        }
      }
    }
    if (!p.square) {
      __syncthreads();
      if (p.codes_t != nullptr && tid < 128 / PER) {
        uint32_t m = part[0][tid];
#pragma unroll
        for (int i = 1; i < WARPS; ++i) m = word_max<T>(m, part[i][tid]);
#pragma unroll
        for (int k = 0; k < PER; ++k)
          byte_of[tid * PER + k] = (uint8_t)scale_byte(PER == 1 ? m : k == 0 ? m << 16 : m & 0xffff0000u, inv_of[tid * PER + k]);
      }
    }
    if (p.codes != nullptr && tid < 128 && rt * 128 + tid < p.rows)
      p.scales[scale_offset(b * tiles, p.first + (rt * 128 + tid) * p.step, kt, ct)] = p.square ? (uint8_t)byte : row_byte[tid];
    if (p.codes_t == nullptr) continue;
    if (!p.square) __syncthreads();
    uint32_t q[VN][2];                       // eight rows of every column
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      float v[4][VN];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[g * 4 + i].values(v[i]);
#pragma unroll
      for (int j = 0; j < VN; ++j) {
        const uint32_t bj = p.square ? byte : byte_of[cg * VN + j], vj = p.square ? inv : inv_of[cg * VN + j];
        const float t[4] = {v[0][j], v[1][j], v[2][j], v[3][j]};
        uint32_t word[1];
        cast_codes(t, bj, vj, word);
        q[j][g] = word[0];
      }
    }
    // 8-byte slot rg of a column, moved about so that sixteen lanes meet sixteen different pairs of banks
#pragma unroll
    for (int j = 0; j < VN; ++j) *reinterpret_cast<uint2*>(turned + (cg * VN + j) * 128 + ((rg ^ (cg & 15)) * 8)) = make_uint2(q[j][0], q[j][1]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 1024 / G::THREADS; ++i) {
      const int c = (i * G::THREADS + tid) >> 3, k = tid & 7, s = c / VN & 15;   // slots 2k and 2k + 1 of the column
      uint4 w = *reinterpret_cast<const uint4*>(turned + c * 128 + ((k ^ (s >> 1)) * 16));
      if (s & 1) w = make_uint4(w.z, w.w, w.x, w.y);
      if (c0 + c < p.K && rt * 128 + k * 16 < pitch_t)
        *reinterpret_cast<uint4*>(p.codes_t + ((size_t)b * p.K + c0 + c) * pitch_t + rt * 128 + k * 16) = w;
    }
    if (tid < 128 && c0 + tid < p.K) p.scales_t[scale_offset(b * tiles_t, c0 + tid, kt_t, rt)] = (uint8_t)(p.square ? byte : byte_of[tid]);
    if (p.square) __syncthreads();           // (otherwise the next tile's maxima come between)
  }
}

template <typename T, bool VEC, typename I>
__global__ void __launch_bounds__(kThreads)
dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int rows, int K, I items, int groups,
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
    const int row = (int)(r - (I)b * (I)rows), at = g * kUnroll * 256;
    const uint8_t* from = codes + (size_t)r * pitch + at;
    const uint8_t* sc = scales + scale_offset(b * tiles, row, kt, at / kBlock);
    T* to = dst + (size_t)r * K + at;
    auto value2 = [](uint32_t two) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
      return __half22float2(*reinterpret_cast<const __half2*>(&h));
    };
    if constexpr (VEC) {
      const int c0 = lane * 8, left = K - at - c0;
      uint2 q[kUnroll];
      uint32_t byte[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        q[u] = make_uint2(0, 0); byte[u] = 0;
        if (u * 256 < left) {
          q[u] = __ldcs(reinterpret_cast<const uint2*>(from + c0 + u * 256));
          byte[u] = sc[(u >> 1) * kTileBytes + (u & 1) * 2 + (lane >> 4)];
        }
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (u * 256 >= left) break;
        const float s = scale_value(byte[u]);
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 f = value2((i < 2 ? q[u].x : q[u].y) >> (16 * (i & 1)));
          v[2 * i] = f.x * s;                // exact: four significant bits times a power of two
          v[2 * i + 1] = f.y * s;
        }
        Piece<T, 8> out;
        out.set(v);
        out.store(to + c0 + u * 256, 8, true);
      }
    } else if constexpr (sizeof(T) == 2) {
      // Two neighbours a lane, in a word of dst.  In a row that starts in the middle of a word they are the second of the lane's
      // two codes and the first of the next lane's; the row's first element is by itself.
      constexpr int PAIRS = kUnroll * 4, BLOCKS = kUnroll * 2;
      const int off = (int)((uintptr_t)to >> 1 & 1), left = K - at;
      uint32_t q[PAIRS + 1];
      float scale[BLOCKS + 1];
#pragma unroll
      for (int j = 0; j < PAIRS; ++j) {
        const int c = j * 64 + lane * 2;
        q[j] = c < left ? (uint32_t)__ldcs(reinterpret_cast<const uint16_t*>(from + c)) : 0u;
      }
      q[PAIRS] = PAIRS * 64 < left ? from[PAIRS * 64] : 0u;
#pragma unroll
      for (int k = 0; k <= BLOCKS; ++k) scale[k] = k * kBlock < left ? scale_value(sc[(k >> 2) * kTileBytes + (k & 3)]) : 0.f;
      if (off && g == 0 && lane == 0) to[0] = __float2bfloat16_rn(value2(q[0]).x * scale[0]);
#pragma unroll
      for (int j = 0; j < PAIRS; ++j) {
        const int c = j * 64 + lane * 2 + off;
        uint32_t two = q[j];
        float s = scale[j / 2];
        if (off) {
          uint32_t next = __shfl_down_sync(kAll, q[j], 1);
          const uint32_t first = __shfl_sync(kAll, q[j + 1], 0);
          if (lane == 31) {
            next = first;
            if (j & 1) s = scale[j / 2 + 1];
          }
          two = two >> 8 | next << 8;
        }
        const float2 f = value2(two & 0xffffu);
        const __nv_bfloat162 h = __floats2bfloat162_rn(f.x * scale[j / 2], f.y * s);
        if (c + 1 < left) *reinterpret_cast<__nv_bfloat162*>(to + c) = h;
        else if (c < left) to[c] = __low2bfloat16(h);
      }
    } else {
      uint32_t q[kUnroll][8];
      uint32_t byte[kUnroll][2];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
#pragma unroll
        for (int j = 0; j < 8; ++j) q[u][j] = at + u * 256 + j * 32 + lane < K ? __ldcs(from + u * 256 + j * 32 + lane) : 0u;
#pragma unroll
        for (int h = 0; h < 2; ++h) byte[u][h] = at + u * 256 + h * 128 < K ? sc[(u >> 1) * kTileBytes + (u & 1) * 2 + h] : 0u;
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const float2 f = value2(q[u][j] | q[u][j + 1] << 8);
          const float s = scale_value(byte[u][j / 4]);
          const int c = u * 256 + j * 32 + lane;
          if (at + c < K) to[c] = from_f32<T>(f.x * s);
          if (at + c + 32 < K) to[c + 32] = from_f32<T>(f.y * s);
        }
    }
  }
}

// T: type of x, or uint8_t where x is FP8 already (its scales in tiles of their own).  d is a multiple of 16.
template <typename T, typename I>
__global__ void __launch_bounds__(kThreads)
dispatch_rows_kernel(const mx4::Dispatch q, const T* __restrict__ x, const uint8_t* __restrict__ x_scales, uint8_t* __restrict__ codes,
                     uint8_t* __restrict__ scales, I items, int groups) {
  const int lane = threadIdx.x & 31;
  const int kt = (int)scale_tiles_k(q.d), pitch = (int)row_pitch(q.d);
  grid_dependency_wait();
  allow_dependents();                        // in this order: the products start after the dispatch, see fp8_gemm_kernel
  for (I w = ((I)blockIdx.x * kThreads + threadIdx.x) >> 5; w < items; w += (I)gridDim.x * (kThreads / 32)) {
    const size_t t = (size_t)(w / (I)groups);
    const int g = (int)(w - (I)t * (I)groups);
    const int c0 = g * kUnroll * 256 + lane * 8;
    const T* from = x + t * (sizeof(T) == 1 ? pitch : q.d) + c0;
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
      uint8_t* to = codes + (size_t)row * pitch + c0;
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

template <typename T, bool VEC> cudaError_t quantize(const CastParams& p, int words, cudaStream_t st) {
  if (p.square || p.codes_t != nullptr) {
    static std::atomic<uint64_t> done{0};
    const int col_tiles = (int)((p.K + 127ll) / 128);
    const long long items = (long long)p.batch * row_tiles(p.rows) * col_tiles, most = Tile<T>::BLOCKS * (long long)sm_count();
    if (!allow_smem((const void*)quantize_tiles_kernel<T, VEC>, Tile<T>::SMEM, done)) return cudaErrorInvalidValue;
    return launch_after_predecessor(quantize_tiles_kernel<T, VEC>, dim3((unsigned)(items < most ? items : most)), dim3(Tile<T>::THREADS),
                                    Tile<T>::SMEM, st, true, p, items, col_tiles, words);
  }
  const int groups = cast_groups(p.K);
  const long long items = (long long)p.batch * p.rows * groups;
  return by_index(items, [&](auto n) {
    return launch_after_predecessor(quantize_rows_kernel<T, VEC, decltype(n)>, dim3(cast_blocks(items)), dim3(kThreads), 0, st, true, p, n,
                                    groups);
  });
}
template <typename T> cudaError_t quantize(const CastParams& p, cudaStream_t st) {
  const size_t e = sizeof(T);
  const bool vec = ((uintptr_t)p.src & 15) == 0 && p.K * e % 16 == 0 && p.K % 8 == 0 && p.row_stride * e % 16 == 0 && p.batch_stride * e % 16 == 0;
  const int words = ((uintptr_t)p.src & 3) == 0 && p.K * e % 4 == 0 && p.row_stride * e % 4 == 0 && p.batch_stride * e % 4 == 0;
  return vec ? quantize<T, true>(p, words, st) : quantize<T, false>(p, words, st);
}

template <typename T>
cudaError_t dequantize(const uint8_t* codes, const uint8_t* scales, int batch, int rows, int K, T* dst, cudaStream_t st) {
  const int groups = cast_groups(K);
  const long long items = (long long)batch * rows * groups;
  return by_index(items, [&](auto n) {
    const dim3 grid(cast_blocks(items)), block(kThreads);
    if (K % 8 == 0)
      return launch_after_predecessor(dequantize_kernel<T, true, decltype(n)>, grid, block, 0, st, true, codes, scales, rows, K, n, groups, dst);
    return launch_after_predecessor(dequantize_kernel<T, false, decltype(n)>, grid, block, 0, st, true, codes, scales, rows, K, n, groups, dst);
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
