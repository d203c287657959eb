// Shared declarations of the FP8 path: the format, the launchers of its kernels and of the norm in front of it
// (btx_fp8_cast.cu, btx_norm.cu; called by btx_fp8_api.cu).
//
// Format (include/btx.h): e4m3 codes, a byte each, rows of `pitch` bytes (K rounded up to 32, zeros behind K); one scale
// byte (2^(b-127)) per row and 128 elements, in tiles of 128 rows x 4 blocks = 512 bytes, [row tile][ceil(K/512)][512], byte
// (r % 32) * 16 + (r / 32 % 4) * 4 + j for block 4c + j of row r.  These are the tiles of the MXFP4 path with wider
// blocks: a word of tensor memory holds the scales of four neighbouring blocks of a row, and an MMA names the byte it takes.
#pragma once

#include "btx_common.cuh"

namespace btx {
namespace fp8 {

constexpr int kBlock = 128;                // elements per scale, and rows of a square block
constexpr int kTileRows = 128;             // rows of a scale tile
constexpr int kTileBytes = 512;
constexpr int kTileK = 512;                // elements of a row whose scales lie in one tile

// Whole sectors of 32 bytes: a box of 128 bytes of a row at any multiple of 16 touches five of them (8192 x 4096 x 4080: 116 us with
// rows of 4080 bytes, 102 with rows of 4096; rows of 4064 and 4032 bytes are no slower than those).
inline __host__ __device__ long long row_pitch(long long K) { return (K + 31) / 32 * 32; }
inline __host__ __device__ long long scale_tiles_k(long long K) { return (K + kTileK - 1) / kTileK; }
inline __host__ __device__ long long row_tiles(long long rows) { return (rows + kTileRows - 1) / kTileRows; }

// A cast of [batch, rows, K] with any row and batch stride: as it stands into codes and scales of [batch, out_rows, K], source
// row r to row first + r * step (codes == nullptr: not wanted), and transposed into [batch, K, rows] (codes_t == nullptr:
// not wanted).
struct CastParams {
  const void* src;
  long long row_stride, batch_stride;      // elements
  int batch, rows, K, out_rows, first, step;
  int square;                              // one scale per 128 x 128 block instead of one per row
  uint8_t *codes, *scales, *codes_t, *scales_t;
};
cudaError_t launch_quantize(const CastParams& p, int dtype, cudaStream_t st);
cudaError_t launch_dequantize(const uint8_t* codes, const uint8_t* scales, int batch, int rows, int K, int dtype, void* dst,
                              cudaStream_t st);

struct NormParams {
  int T, d;
  float eps;
  const void *x, *residual, *w;            // residual, w: may be null
  void *h, *y;                             // may be null
  long long x_stride, residual_stride, h_stride, y_stride;
  uint8_t *codes, *scales;                 // may be null
};
cudaError_t launch_norm(const NormParams& p, int dtype, cudaStream_t st);

struct NormGradParams {
  int T, d;
  float eps;
  const void *h, *w, *dy, *dh;             // w, dh: may be null
  void* dx;
  float* dw;                               // may be null
  long long h_stride, dy_stride, dh_stride, dx_stride;
  int accumulate;
  float* part;                             // [norm_grad_parts][d]
  int32_t* status;
};
int norm_grad_parts(int T, int d, int dtype);
cudaError_t launch_norm_grad(const NormGradParams& p, int dtype, cudaStream_t st);

// Scale byte of a block from the bits of its largest magnitude: the smallest 2^e, not below 2^-127, with
// max / 2^e <= 448 = 1.75 * 2^8, so e is the exponent less 8, or less 7 where the significand is above 1.75; 255 when the
// block holds an infinity or NaN.  `inv` is the exact reciprocal of the scale.
__host__ __device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits, uint32_t& inv_bits) {
  if (amax_bits >= 0x7f800000u) { inv_bits = 0; return 255u; }
  const int e = (int)((amax_bits + 0x1fffffu) >> 23) - 8;
  const uint32_t b = e > 0 ? (uint32_t)e : 0u;
  inv_bits = (254u - b) << 23;
  return b;
}

}  // namespace fp8
}  // namespace btx
