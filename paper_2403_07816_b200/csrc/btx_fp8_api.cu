// C ABI of the FP8 path and of the norm in front of it: argument checks and launches.
#include <cmath>

#include "btx_fp8.cuh"

namespace btx {
namespace fp8 {
namespace {

constexpr int kMaxSide = 1 << 30;                    // rows and columns, and the ends of the tiles past the last one, fit 32 bits
constexpr long long kMaxCodes = 1ll << 40;           // bytes of a matrix of codes: a tensor map's stride is below this
constexpr int kMaxNorm = 1 << 16;                    // bytes of a row that a block keeps in registers

btx_status check_shape(int batch, int rows, int K) {
  if (batch < 0 || rows < 0 || K < 1) return BTX_ERR_INVALID_ARG;
  if (rows > kMaxSide || K > kMaxSide) return BTX_ERR_UNSUPPORTED;
  const long long codes = rows * row_pitch(K), scales = row_tiles(rows) * scale_tiles_k(K) * kTileBytes;
  if (codes >= kMaxCodes || (batch > 0 && (codes > scales ? codes : scales) > (1ll << 62) / batch)) return BTX_ERR_UNSUPPORTED;
  return BTX_OK;
}

bool bad_dtype(int dtype) { return dtype != BTX_F32 && dtype != BTX_BF16; }
bool off_element(const void* p, int dtype) { return ((uintptr_t)p & (dtype == BTX_BF16 ? 1 : 3)) != 0; }

btx_status check_norm(const btx_norm_desc* d) {
  if (!d || d->T < 0 || d->d_model < 1 || bad_dtype(d->dtype)) return BTX_ERR_INVALID_ARG;
  if (!(d->eps >= 0.f) || std::isinf(d->eps)) return BTX_ERR_INVALID_ARG;
  if (d->d_model > kMaxNorm / (d->dtype == BTX_BF16 ? 2 : 4) || d->T > kMaxSide) return BTX_ERR_UNSUPPORTED;
  return BTX_OK;
}
// rows of d elements, `stride` apart, that do not overlap
bool bad_rows(const void* p, int64_t stride, const btx_norm_desc* d) {
  return off_element(p, d->dtype) || (d->T > 1 && stride < d->d_model) || stride < 0 || stride > (1ll << 40);
}

}  // namespace
}  // namespace fp8
}  // namespace btx

using namespace btx;
using namespace btx::fp8;

extern "C" btx_status btx_fp8_sizes(int32_t batch, int32_t rows, int32_t K, size_t* code_bytes, size_t* scale_bytes) {
  btx_status s = check_shape(batch, rows, K);
  if (s != BTX_OK) return s;
  if (code_bytes) *code_bytes = (size_t)batch * rows * row_pitch(K);
  if (scale_bytes) *scale_bytes = (size_t)batch * row_tiles(rows) * scale_tiles_k(K) * kTileBytes;
  return BTX_OK;
}

extern "C" btx_status btx_fp8_quantize(int32_t dtype, const void* src, int64_t row_stride, int64_t batch_stride, int32_t batch,
                                       int32_t rows, int32_t K, int32_t block_rows, int32_t out_rows, int32_t row_first,
                                       int32_t row_step, void* codes, void* scales, void* codes_t, void* scales_t, void* stream) {
  btx_status s = check_shape(batch, rows, K);
  if (s != BTX_OK) return s;
  if (bad_dtype(dtype) || (block_rows != 1 && block_rows != kBlock)) return BTX_ERR_INVALID_ARG;
  if (!codes != !scales || !codes_t != !scales_t) return BTX_ERR_INVALID_ARG;
  if (codes) {
    if (row_first < 0 || row_step < 1 || out_rows < 0) return BTX_ERR_INVALID_ARG;
    if ((s = check_shape(batch, out_rows, K)) != BTX_OK) return s;
    if (rows > 0 && (long long)row_first + (long long)(rows - 1) * row_step >= out_rows) return BTX_ERR_INVALID_ARG;
  }
  if (codes_t && rows > 0 && (s = check_shape(batch, K, rows)) != BTX_OK) return s;
  if (batch == 0 || rows == 0) return BTX_OK;
  if (!src || (!codes && !codes_t)) return BTX_ERR_INVALID_ARG;
  if (row_stride < 0 || batch_stride < 0) return BTX_ERR_INVALID_ARG;
  if (off_element(src, dtype) || misaligned(codes) || misaligned(scales) || misaligned(codes_t) || misaligned(scales_t))
    return BTX_ERR_INVALID_ARG;
  if ((s = check_device()) != BTX_OK) return s;
  CastParams p = {};
  p.src = src; p.row_stride = row_stride; p.batch_stride = batch_stride; p.batch = batch; p.rows = rows; p.K = K;
  p.out_rows = out_rows; p.first = row_first; p.step = row_step; p.square = block_rows == kBlock;
  p.codes = (uint8_t*)codes; p.scales = (uint8_t*)scales; p.codes_t = (uint8_t*)codes_t; p.scales_t = (uint8_t*)scales_t;
  return launch_quantize(p, dtype, (cudaStream_t)stream) == cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
}

extern "C" btx_status btx_fp8_dequantize(int32_t dtype, const void* codes, const void* scales, int32_t batch, int32_t rows,
                                         int32_t K, void* dst, void* stream) {
  btx_status s = check_shape(batch, rows, K);
  if (s != BTX_OK) return s;
  if (bad_dtype(dtype)) return BTX_ERR_INVALID_ARG;
  if (batch == 0 || rows == 0) return BTX_OK;
  if (!codes || !scales || !dst || misaligned(codes) || misaligned(scales) || misaligned(dst)) return BTX_ERR_INVALID_ARG;
  if ((s = check_device()) != BTX_OK) return s;
  return launch_dequantize((const uint8_t*)codes, (const uint8_t*)scales, batch, rows, K, dtype, dst, (cudaStream_t)stream) ==
                 cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
}

extern "C" btx_status btx_rms_norm(const btx_norm_desc* desc, const void* x, int64_t x_stride, const void* residual,
                                   int64_t residual_stride, const void* weight, void* h, int64_t h_stride, void* y,
                                   int64_t y_stride, void* codes, void* scales, void* stream) {
  btx_status s = check_norm(desc);
  if (s != BTX_OK) return s;
  if (!codes != !scales) return BTX_ERR_INVALID_ARG;
  if (desc->T == 0) return BTX_OK;
  if (!x || (!h && !y && !codes)) return BTX_ERR_INVALID_ARG;
  if (bad_rows(x, x_stride, desc) || (residual && bad_rows(residual, residual_stride, desc)) || (h && bad_rows(h, h_stride, desc)) ||
      (y && bad_rows(y, y_stride, desc)) || off_element(weight, desc->dtype) || misaligned(codes) || misaligned(scales))
    return BTX_ERR_INVALID_ARG;
  if ((s = check_device()) != BTX_OK) return s;
  NormParams p = {};
  p.T = desc->T; p.d = desc->d_model; p.eps = desc->eps; p.x = x; p.residual = residual; p.w = weight; p.h = h; p.y = y;
  p.x_stride = x_stride; p.residual_stride = residual_stride; p.h_stride = h_stride; p.y_stride = y_stride;
  p.codes = (uint8_t*)codes; p.scales = (uint8_t*)scales;
  return launch_norm(p, desc->dtype, (cudaStream_t)stream) == cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
}

extern "C" btx_status btx_rms_norm_backward_workspace_size(const btx_norm_desc* desc, size_t* workspace_bytes) {
  btx_status s = check_norm(desc);
  if (s != BTX_OK) return s;
  if (!workspace_bytes) return BTX_ERR_INVALID_ARG;
  *workspace_bytes = kStatusWords * 4 + (size_t)norm_grad_parts(desc->T, desc->d_model, desc->dtype) * desc->d_model * 4;
  return BTX_OK;
}

extern "C" btx_status btx_rms_norm_backward(const btx_norm_desc* desc, const void* h, int64_t h_stride, const void* weight,
                                            const void* dy, int64_t dy_stride, const void* dh, int64_t dh_stride, void* dx,
                                            int64_t dx_stride, float* dweight, int32_t accumulate, void* workspace,
                                            size_t workspace_bytes, void* stream) {
  size_t need = 0;
  btx_status s = btx_rms_norm_backward_workspace_size(desc, &need);
  if (s != BTX_OK) return s;
  if (!workspace || misaligned(workspace)) return BTX_ERR_INVALID_ARG;
  if (desc->T > 0) {
    if (!h || !dy || !dx) return BTX_ERR_INVALID_ARG;
    if (bad_rows(h, h_stride, desc) || bad_rows(dy, dy_stride, desc) || (dh && bad_rows(dh, dh_stride, desc)) ||
        bad_rows(dx, dx_stride, desc))
      return BTX_ERR_INVALID_ARG;
  }
  if (off_element(weight, desc->dtype) || ((uintptr_t)dweight & 3)) return BTX_ERR_INVALID_ARG;
  if (workspace_bytes < need) return BTX_ERR_WORKSPACE;
  if (desc->T == 0 && (!dweight || accumulate)) return BTX_OK;
  if ((s = check_device()) != BTX_OK) return s;
  NormGradParams p = {};
  p.T = desc->T; p.d = desc->d_model; p.eps = desc->eps; p.h = h; p.w = weight; p.dy = dy; p.dh = dh; p.dx = dx; p.dw = dweight;
  p.h_stride = h_stride; p.dy_stride = dy_stride; p.dh_stride = dh_stride; p.dx_stride = dx_stride;
  p.accumulate = accumulate != 0; p.status = (int32_t*)workspace; p.part = (float*)((char*)workspace + kStatusWords * 4);
  return launch_norm_grad(p, desc->dtype, (cudaStream_t)stream) == cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
}
