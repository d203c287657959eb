// Device code shared by the MXFP4 kernels (btx_mx4_cast.cu, btx_mx4_gemm.cu, btx_mx4_layer.cu): the cast of eight
// elements of a block by a lane, the PTX of the one-CTA tensor-core forms, and what becomes of an accumulator.
#pragma once

#include <cuda_fp4.h>

#include <atomic>

#include "btx_mx4.cuh"
#include "btx_route_dev.cuh"
#include "btx_tc_ptx.cuh"

namespace btx {
namespace mx4 {
namespace {

using namespace tcx;
using routedev::Vec;

constexpr unsigned kAll = 0xffffffffu;

// ---------------------------------------------------------------------------------------------
// Cast
// ---------------------------------------------------------------------------------------------
constexpr int kCastUnroll = 4;             // 256-element chunks a warp has in flight

// Eight elements of a lane as they were loaded: their largest magnitude as the bits of a float (NaN and infinities
// compare above every number), and their values.
template <typename T> struct Eight;
template <> struct Eight<float> {
  uint4 a, b;
  __device__ __forceinline__ void zero() { a = b = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void load(const float* p, bool vec) {
    if (vec) {
      a = __ldcs(reinterpret_cast<const uint4*>(p));
      b = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
    } else {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(p);
      a = make_uint4(w[0], w[1], w[2], w[3]);
      b = make_uint4(w[4], w[5], w[6], w[7]);
    }
  }
  __device__ __forceinline__ uint32_t block_max() const {
    constexpr uint32_t M = 0x7fffffffu;
    uint32_t m = max(max(max(a.x & M, a.y & M), max(a.z & M, a.w & M)), max(max(b.x & M, b.y & M), max(b.z & M, b.w & M)));
    m = max(m, __shfl_xor_sync(kAll, m, 1));
    return max(m, __shfl_xor_sync(kAll, m, 2));
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
    v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y); v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
  }
};
template <> struct Eight<__nv_bfloat16> {
  uint4 a;
  __device__ __forceinline__ void zero() { a = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void load(const __nv_bfloat16* p, bool vec) {
    if (vec) {
      a = __ldcs(reinterpret_cast<const uint4*>(p));
    } else {
      const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
      a = make_uint4(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16, h[4] | (uint32_t)h[5] << 16, h[6] | (uint32_t)h[7] << 16);
    }
  }
  // two 16-bit maxima per instruction: half the comparisons of the widened values
  __device__ __forceinline__ uint32_t block_max() const {
    constexpr uint32_t M = 0x7fff7fffu;
    uint32_t m = __vimax3_u16x2(a.x & M, a.y & M, a.z & M);
    m = __vimax3_u16x2(m, a.w & M, __shfl_xor_sync(kAll, __vimax3_u16x2(m, a.w & M, 0u), 1));
    m = __vimax3_u16x2(m, __shfl_xor_sync(kAll, m, 2), 0u);
    return max(m & 0xffff0000u, m << 16);
  }
  __device__ __forceinline__ void values(float (&v)[8]) const { Vec<__nv_bfloat16>::unpack(a, v); }
};

// Four bytes of codes of eight elements times `inv`.
__device__ __forceinline__ uint32_t pack_e2m1(const float (&v)[8], float inv) {
  uint32_t q;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
      "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
      : "=r"(q)
      : "f"(v[0] * inv), "f"(v[1] * inv), "f"(v[2] * inv), "f"(v[3] * inv), "f"(v[4] * inv), "f"(v[5] * inv), "f"(v[6] * inv),
        "f"(v[7] * inv));
  return q;
}

// Eight elements of a block shared by four neighbouring lanes: four bytes of codes and the block's scale byte.
template <typename T> __device__ __forceinline__ uint32_t cast8(const Eight<T>& x, uint32_t& byte) {
  float inv, v[8];
  byte = scale_byte(x.block_max(), inv);
  x.values(v);
  const uint32_t q = pack_e2m1(v, inv);
  return byte == 255u ? 0u : q;
}
__device__ __forceinline__ size_t scale_offset(size_t tile_row0, int row, int kt, int chunk) {
  return ((tile_row0 + row / kTileRows) * (size_t)kt + chunk) * kTileBytes + (row & 31) * 16 + ((row >> 5) & 3) * 4;
}

// kCastUnroll chunks of 256 elements of a token, cast once and written to the rows of its slots.
template <typename T>
__device__ __forceinline__ void cast_token_rows(const T* __restrict__ x, int d, int g, int lane, int k, const int* rows,
                                                uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  const int kt = (int)scale_tiles_k(d);
  const int c0 = g * kCastUnroll * 256 + lane * 8;
  Eight<T> v[kCastUnroll];
#pragma unroll
  for (int u = 0; u < kCastUnroll; ++u) {
    if (c0 + u * 256 < d) v[u].load(x + c0 + u * 256, true);
    else v[u].zero();
  }
  uint32_t code[kCastUnroll], byte[kCastUnroll];
#pragma unroll
  for (int u = 0; u < kCastUnroll; ++u) code[u] = cast8(v[u], byte[u]);
  for (int j = 0; j < k; ++j) {
    const int row = rows[j];
    if (row < 0) continue;
    uint8_t* to = codes + (size_t)row * (d / 2) + c0 / 2;
    uint8_t* sc = scales + scale_offset(0, row, kt, c0 / 128) + (c0 / kBlock & 3);
#pragma unroll
    for (int u = 0; u < kCastUnroll; ++u) {
      if (c0 + u * 256 < d) *reinterpret_cast<uint32_t*>(to + u * 128) = code[u];
      if ((lane & 3) == 0 && c0 + u * 256 < kt * 128) sc[u * 2 * kTileBytes] = (uint8_t)byte[u];
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Products
// ---------------------------------------------------------------------------------------------
constexpr int SK = 256;                                  // contraction elements per stage (128 bytes of codes)
constexpr int BM = kTileRows;
constexpr int BN = 128;
constexpr int EPI_WARPS = 8;
constexpr int A_BYTES = BM * SK / 2, B_BYTES = BN * SK / 2;
constexpr int SF_BYTES = 2 * kTileBytes;                 // scales of a stage, of A or of B
constexpr int MAX_STAGES = 10, SF_COLS = 16;             // tensor-memory columns of a stage's scales
static_assert(2 * BN + MAX_STAGES * SF_COLS <= 512, "accumulators and scales fit in tensor memory");
constexpr int GROUP_N = 8;                               // column tiles per raster group

enum Mode { STORE = 0, GATE_UP = 1, DOWN = 2 };

// bytes of a ring stage whose A part has `rows` rows, and how many fit
inline __host__ __device__ int stage_bytes(int rows) { return rows * (SK / 2) + 2 * SF_BYTES + B_BYTES; }
inline __host__ __device__ int stage_count(int rows, int ring_bytes) {
  const int n = ring_bytes / stage_bytes(rows);
  return n < MAX_STAGES ? n : MAX_STAGES;
}

struct Params {
  int M, N, K;                      // STORE: rows and columns of y; grouped: N = B rows per expert
  int m_tiles, n_tiles, batch;
  int grouped;
  int tile_step;                    // 128-row tiles per row tile of this launch (1, or 2 for CTA pairs)
  const int32_t* n_row_tiles;       // grouped: row tiles in use (device)
  const int32_t* tile_expert;
  const int32_t* tile_rows;         // grouped: rows of a tile that hold an assignment
  const int32_t* rowmap;
  int a_rows, a_box;                // rows of A per stage, rows per TMA operation
  int split;                        // CTAs that share a tile's contraction
  const uint8_t* a_scales;
  const uint8_t* b_scales;
  long long a_scale_batch, b_scale_batch;   // bytes from one matrix to the next
  int kt;                           // scale tiles along K
  int a_row_tiles, b_row_tiles;     // scale row tiles of one matrix
  const float* gates;
  void* y;
  uint8_t* act_codes;
  uint8_t* act_scales;
  int out_bf16;
  int wide;                         // output rows start on 32-byte boundaries
  int32_t* status;
};

// ---- PTX of the one-CTA forms ----
__device__ __forceinline__ void load_3d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
}
__device__ __forceinline__ void load_bulk(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                         uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accum) : "memory");
}
// This lane's 16 bytes of two 512-byte scale tiles to eight tensor-memory columns of the warp's 32-lane quarter.  Word
// c of a lane's 16 bytes belongs to row c * 32 + lane of a tile: it goes to column c, the same in all four quarters.
__device__ __forceinline__ void store_scales(uint32_t taddr, const uint4& lo, const uint4& hi) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(lo.x), "r"(lo.y), "r"(lo.z), "r"(lo.w), "r"(hi.x), "r"(hi.y), "r"(hi.z), "r"(hi.w) : "memory");
}
__device__ __forceinline__ void arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// A bounded wait of a whole warp: it gives up for all lanes or for none.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* status) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, status));
}

__device__ __forceinline__ uint4 ld_shared_v4(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared::cta.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

struct Item { int mt, nt, b, e; };

// Tile number -> (row tile, column tile): groups of GROUP_N column tiles, rows advance slowest inside a group.
__device__ __forceinline__ void raster(int m_tiles, int n_tiles, int t, int& mt, int& nt) {
  const int full = n_tiles / GROUP_N, in_full = full * m_tiles * GROUP_N;
  int g, width, rem;
  if (t < in_full) { g = t / (m_tiles * GROUP_N); rem = t - g * m_tiles * GROUP_N; width = GROUP_N; }
  else { g = full; rem = t - in_full; width = n_tiles - full * GROUP_N; }
  mt = rem / width;
  nt = g * GROUP_N + rem - mt * width;
}
__device__ __forceinline__ Item get_item(const Params& p, int m_tiles, int t) {
  Item it;
  const int per = m_tiles * p.n_tiles;
  it.b = t / per;
  raster(m_tiles, p.n_tiles, t - it.b * per, it.mt, it.nt);
  it.e = p.grouped ? p.tile_expert[it.mt * p.tile_step] : it.b;
  return it;
}

// 64 accumulator columns of one row per thread, by a whole warp
__device__ __forceinline__ void load_chunk(uint32_t taddr, float (&v)[64]) {
  uint32_t r[64];
  __syncwarp();                                           // the tensor-memory load needs the whole warp
#pragma unroll
  for (int h = 0; h < 2; ++h)
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[32 * h + 0]), "=r"(r[32 * h + 1]), "=r"(r[32 * h + 2]), "=r"(r[32 * h + 3]), "=r"(r[32 * h + 4]),
          "=r"(r[32 * h + 5]), "=r"(r[32 * h + 6]), "=r"(r[32 * h + 7]), "=r"(r[32 * h + 8]), "=r"(r[32 * h + 9]),
          "=r"(r[32 * h + 10]), "=r"(r[32 * h + 11]), "=r"(r[32 * h + 12]), "=r"(r[32 * h + 13]), "=r"(r[32 * h + 14]),
          "=r"(r[32 * h + 15]), "=r"(r[32 * h + 16]), "=r"(r[32 * h + 17]), "=r"(r[32 * h + 18]), "=r"(r[32 * h + 19]),
          "=r"(r[32 * h + 20]), "=r"(r[32 * h + 21]), "=r"(r[32 * h + 22]), "=r"(r[32 * h + 23]), "=r"(r[32 * h + 24]),
          "=r"(r[32 * h + 25]), "=r"(r[32 * h + 26]), "=r"(r[32 * h + 27]), "=r"(r[32 * h + 28]), "=r"(r[32 * h + 29]),
          "=r"(r[32 * h + 30]), "=r"(r[32 * h + 31])
        : "r"(taddr + 32 * h));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 64; ++i) v[i] = __uint_as_float(r[i]);
}

// What becomes of them (columns n0 .. n0 + 63 of the product).  m: the row of A; flat: its row of y (STORE) or its
// assignment, -1 for a row that nobody asked for.
template <int MODE>
__device__ __forceinline__ void finish_chunk(const Params& p, const Item& it, float (&v)[64], int n0, int m, int flat,
                                             size_t y_offset = 0) {
  if (flat < 0 || n0 >= (MODE == GATE_UP ? (p.N + 255) / 256 * 256 : p.N)) return;
  const bool wide = p.wide != 0;
  if constexpr (MODE == GATE_UP) {
    const int F = p.N / 2;
    const int f0 = n0 / 2;                                // 32 hidden units: one block
    float a[32];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      a[i] = fast_swiglu(v[2 * i], v[2 * i + 1]);
      amax = max(amax, __float_as_uint(a[i]) & 0x7fffffffu);
    }
    float inv;
    uint32_t byte = scale_byte(amax, inv);
    uint32_t w[4] = {0, 0, 0, 0};
    if (byte != 255u) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        w[i / 4] |= (uint32_t)__nv_cvt_float2_to_fp4x2(make_float2(a[2 * i] * inv, a[2 * i + 1] * inv), __NV_E2M1,
                                                       cudaRoundNearest) << (8 * (i & 3));
    }
    // past the last unit there is no block, but the other half of an MMA's 64 elements wants a finite scale
    if (f0 >= F) byte = 0;
    const int blk = f0 / kBlock, akt = (int)scale_tiles_k(F);
    if (blk < 4 * akt)
      p.act_scales[((size_t)(m / kTileRows) * akt + blk / 4) * kTileBytes + (m & 31) * 16 + (m >> 5 & 3) * 4 + (blk & 3)] = (uint8_t)byte;
    if (f0 < F) *reinterpret_cast<uint4*>(p.act_codes + (size_t)m * (F / 2) + f0 / 2) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
    const size_t o = (MODE == STORE ? ((size_t)it.b * p.M + flat) * p.N : (size_t)flat * p.N) + n0 + y_offset;
    if (MODE == DOWN) {
      const float g = p.gates[flat];
#pragma unroll
      for (int i = 0; i < 64; ++i) v[i] *= g;
    }
    if (MODE == STORE && p.out_bf16) {
      __nv_bfloat16* y = (__nv_bfloat16*)p.y + o;
      if (wide && n0 + 64 <= p.N) {
#pragma unroll
        for (int i = 0; i < 64; i += 16) st32(y + i, pack8(v + i), pack8(v + i + 8), true);
      } else {
#pragma unroll
        for (int i = 0; i < 64; ++i)
          if (n0 + i < p.N) y[i] = __float2bfloat16_rn(v[i]);
      }
    } else {
      float* y = (float*)p.y + o;
      if (wide && n0 + 64 <= p.N) {
#pragma unroll
        for (int i = 0; i < 64; i += 8) st32(y + i, f4(v + i), f4(v + i + 4), true);
      } else {
#pragma unroll
        for (int i = 0; i < 64; ++i)
          if (n0 + i < p.N) y[i] = v[i];
      }
    }
  }
}

// STORE where rows of y do not start on 32-byte boundaries: a thread's 64 values of a row would go out one by one, 32
// rows per instruction (894 instead of 150 us for M = 8192, N = 11007, K = 4096, bf16).  The warp turns them through
// shared memory, 16 words at a time, and writes two rows of 16 neighbouring words per instruction (171 us; bf16
// rows of even length go out as pairs, 156 us for N = 11004).
constexpr int TURN_PITCH = 17, TURN_BYTES = 32 * TURN_PITCH * 4;       // of a warp
template <typename W, int PER, typename Value>
__device__ __forceinline__ void turn_words(W* y, int N, int rows, int cols, int lane, uint32_t* st, Value value) {
  // W: a word of PER columns; y: first row and column of the chunk; value(i): this thread's word i
  const int sub = lane >> 4, c = lane & 15;
  const long long step = 2ll * N / PER;
#pragma unroll
  for (int g = 0; g < 4 / PER; ++g) {
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 16; ++j) st[lane * TURN_PITCH + j] = value(g * 16 + j);
    __syncwarp();
    const bool in = (g * 16 + c) * PER < cols;
    W* to = y + (long long)sub * N / PER + g * 16 + c;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t w = st[(2 * i + sub) * TURN_PITCH + c];
      if (in && 2 * i + sub < rows) {
        if (sizeof(W) == 2) *reinterpret_cast<uint16_t*>(to) = (uint16_t)w;
        else *reinterpret_cast<uint32_t*>(to) = w;
      }
      to += step;
    }
  }
}
__device__ __forceinline__ void store_turned(const Params& p, const Item& it, const float (&v)[64], int n0, int m0, int lane, uint32_t* st) {
  const size_t o = ((size_t)it.b * p.M + m0) * p.N + n0;
  const int rows = p.M - m0, cols = p.N - n0;
  if (!p.out_bf16) {
    turn_words<uint32_t, 1>((uint32_t*)p.y + o, p.N, rows, cols, lane, st, [&](int i) { return __float_as_uint(v[i]); });
  } else if ((p.N & 1) == 0 && ((uintptr_t)p.y & 3) == 0) {
    turn_words<uint32_t, 2>((uint32_t*)((__nv_bfloat16*)p.y + o), p.N, rows, cols, lane, st, [&](int i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      return *reinterpret_cast<const uint32_t*>(&h);
    });
  } else {
    turn_words<uint16_t, 1>((uint16_t*)p.y + o, p.N, rows, cols, lane, st, [&](int i) {
      return (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(v[i]));
    });
  }
}

// codes [batch][rows][K/2] as bytes, box of 128 bytes x box_rows
inline bool make_codes_map(CUtensorMap* m, const void* base, long long K, long long rows, long long batch, uint32_t box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)K / 2, (cuuint64_t)rows, (cuuint64_t)batch};
  cuuint64_t strides[2] = {(cuuint64_t)K / 2, (cuuint64_t)(K / 2 * rows)};
  cuuint32_t box[3] = {SK / 2, box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
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
}  // namespace mx4
}  // namespace btx
