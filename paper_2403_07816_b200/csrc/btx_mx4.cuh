// Shared declarations of the MXFP4 path: the format, the launchers of its kernels and the plan of the expert layer
// on MXFP4 weights (btx_mx4_cast.cu, btx_mx4_gemm.cu, btx_mx4_api.cu).
//
// Format (include/btx.h): e2m1 codes, two per byte along K, rows of K/2 bytes; one scale byte (2^(b-127)) per 32
// elements, stored in tiles of 128 rows x 4 blocks = 512 bytes, [row tile][K/128][512], byte (r % 32) * 16 +
// (r / 32 % 4) * 4 + j for block 4c + j of row r: lane r % 32 of a warp takes 16 neighbouring bytes, whose four words are
// the four columns of tensor memory that the MMAs read (tcgen05.st), so no kernel rearranges scales.
#pragma once

#include "btx_common.cuh"

namespace btx {
namespace mx4 {

constexpr int kBlock = 32;                 // elements per scale
constexpr int kTileRows = 128;             // rows of a scale tile, of an MMA and of an expert's row padding
constexpr int kTileBytes = 512;
constexpr int kMaxExperts4 = 512;

inline __host__ __device__ long long scale_tiles_k(long long K) { return (K + 127) / 128; }

// A cast of [batch, rows, K] with any row and batch stride into codes and scales of [batch, out_rows, K]: source row
// r becomes row first + r * step.
struct CastParams {
  const void* src;
  long long row_stride, batch_stride;      // elements
  int batch, rows, K, out_rows, first, step;
  uint8_t* codes;
  uint8_t* scales;
};
cudaError_t launch_quantize(const CastParams& p, int dtype, cudaStream_t st);
cudaError_t launch_dequantize(const uint8_t* codes, const uint8_t* scales, int batch, int rows, int K, int dtype, void* dst,
                              cudaStream_t st);

// Row dispatch of the expert layer: rows of an expert are consecutive, in the order of t*k+slot, and padded to whole
// tiles of 128 rows or pairs of them.
struct Dispatch {
  int T, k, R, E, d;                       // R = T*k
  int pad_tiles;                           // an expert's rows are padded to this many row tiles (2: products by CTA pairs)
  int m_tiles_max;                         // upper bound of the padded row tiles
  const int32_t* topk_idx;                 // an index outside 0..E-1: no expert
  int32_t* flat2row;                       // [R] padded row of an assignment, -1 without an expert
  int32_t* rowmap;                         // [m_tiles_max * 128] assignment of a padded row, -1 for padding
  int32_t* tile_expert;                    // [m_tiles_max]
  int32_t* tile_rows;                      // [m_tiles_max] rows of a tile with an assignment
  int32_t* n_tiles;                        // [1] padded row tiles in use
  int32_t* block_counts;                   // [blocks * E] (batches of more than one block)
  int32_t* pad_offsets;                    // [E + 1] first padded row of every expert
  int chunk, blocks;                       // assignments per block of the dispatch kernels, blocks
  int32_t* status;                         // cleared by the first kernel
};
int dispatch_chunk(long long R);
cudaError_t launch_dispatch(const Dispatch& q, cudaStream_t st);
// x [T, d] cast to MXFP4 and written to the k padded rows of every token
cudaError_t launch_quantize_rows(const Dispatch& q, int dtype, const void* x, uint8_t* codes, uint8_t* scales, cudaStream_t st);
// y[t] = sum over slots with an expert of rows[t*k+slot]
cudaError_t launch_combine_rows(const Dispatch& q, int dtype, const float* rows, void* y, cudaStream_t st);

// Products.  A: codes [batch, M, K] (grouped: the padded rows), B: codes [batch or experts, N, K].
struct GemmArgs {
  const uint8_t *a_codes, *a_scales, *b_codes, *b_scales;
  int batch, M, N, K;                      // grouped: batch = 1, M = padded rows (upper bound), N rows per expert
  int experts;                             // B matrices
  int32_t* status;
};
// Whether the expert layer's products run on CTA pairs (256-row tiles): enough rows per expert to fill them.
bool pairs_fit(long long rows, long long experts, long long d, long long F);
btx_status launch_matmul(const GemmArgs& g, int dtype, void* y, cudaStream_t st);
// W1/W3 product (rows interleaved) with silu(h1) * h3 cast to MXFP4
btx_status launch_gate_up(const GemmArgs& g, const Dispatch& q, uint8_t* act_codes, uint8_t* act_scales, cudaStream_t st);
// W2 product, gate-scaled fp32 rows at [t*k+slot]
btx_status launch_down(const GemmArgs& g, const Dispatch& q, const float* gates, float* rows, cudaStream_t st);

// The whole layer of a small batch as one cooperative kernel; BTX_ERR_UNSUPPORTED, nothing launched, where not every
// block can be resident.  `rows` holds layer_rows_floats floats.
bool layer_fits(const Dispatch& q);
size_t layer_rows_floats(const Dispatch& q);
btx_status launch_layer(const GemmArgs& up, const GemmArgs& down, const Dispatch& q, int dtype, const void* x, const float* gates,
                        float* rows, uint8_t* act_codes, uint8_t* act_scales, void* y, cudaStream_t st);

// 32 values of a lane group are cast with one scale: the byte is floor(log2 max) - 2 (bias 127, not below 0), 255
// when the block holds an infinity or NaN; `inv` is the exact reciprocal of the scale.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits, float& inv) {
  if (amax_bits >= 0x7f800000u) { inv = 0.f; return 255u; }
  const int e = (int)(amax_bits >> 23) - 2;
  const uint32_t b = e > 0 ? (uint32_t)e : 0u;
  inv = __uint_as_float((254u - b) << 23);
  return b;
}

}  // namespace mx4
}  // namespace btx
