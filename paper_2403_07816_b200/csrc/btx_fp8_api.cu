// C ABI of the FP8 path and of the norm in front of it: argument checks and launches.
#include <cmath>

#include "btx_fp8_gemm.cuh"

namespace btx {
namespace fp8 {
namespace {

constexpr int kMaxSide = 1 << 30;                    // rows and columns, and the ends of the tiles past the last one, fit 32 bits
constexpr long long kMaxCodes = 1ll << 40;           // bytes of a matrix of codes: a tensor map's stride is below this
constexpr long long kMaxItems = 1ll << 30;           // output tiles of a product are numbered in 32 bits
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

btx_status check_matmul(int dtype, int batch, int M, int N, int K) {
  if (bad_dtype(dtype) || batch < 0 || M < 0 || N < 1) return BTX_ERR_INVALID_ARG;
  btx_status s = check_shape(batch, M, K);
  if (s != BTX_OK) return s;
  if ((s = check_shape(batch, N, K)) != BTX_OK) return s;
  if (row_tiles(M) * row_tiles(N) > kMaxItems || row_tiles(M) * row_tiles(N) * batch > kMaxItems) return BTX_ERR_UNSUPPORTED;
  return BTX_OK;
}

struct MoePlan {
  mx4::Dispatch q;
  size_t w_status, w_flat2row, w_rowmap, w_tile_expert, w_tile_rows, w_n_tiles, w_block_counts, w_pad_offsets, w_xs, w_xs_scales, w_act,
      w_act_scales, w_rows, bytes;
};

btx_status make_moe_plan(const btx_fp8_moe_desc* d, MoePlan* pl) {
  if (!d || !pl) return BTX_ERR_INVALID_ARG;
  if (d->T < 0 || d->d_model < 1 || d->d_ff < 1 || d->E < 1 || d->k < 1 || d->k > d->E || bad_dtype(d->dtype)) return BTX_ERR_INVALID_ARG;
  if (d->E > mx4::kMaxExperts4 || d->d_model % 16 || d->d_ff % 16 || d->d_model > kMaxSide || d->d_ff > kMaxSide / 2)
    return BTX_ERR_UNSUPPORTED;
  const long long R = (long long)d->T * d->k;
  if (R > (1ll << 28)) return BTX_ERR_UNSUPPORTED;
  const long long used = R < d->E ? R : d->E;        // experts that can hold a row
  const int pad_tiles = pairs_fit(R, used, d->d_model, d->d_ff) ? 2 : 1;
  const long long unit = pad_tiles * kTileRows;
  const long long tiles = (R + used * (unit - 1)) / unit * pad_tiles;
  const long long d_pitch = row_pitch(d->d_model), f_pitch = row_pitch(d->d_ff);
  const long long wide = d_pitch > f_pitch ? d_pitch : f_pitch;             // codes of the rows, of W1 and W3, of W2
  if (tiles * kTileRows * wide >= kMaxCodes || 2 * (long long)d->d_ff * d_pitch >= kMaxCodes || d->d_model * f_pitch >= kMaxCodes) return BTX_ERR_UNSUPPORTED;
  const long long widest = d->d_model > 2 * (long long)d->d_ff ? d->d_model : 2 * (long long)d->d_ff;
  if (tiles * (row_tiles(widest) + 1) > kMaxItems) return BTX_ERR_UNSUPPORTED;
  *pl = MoePlan();
  mx4::Dispatch& q = pl->q;
  q.T = d->T; q.k = d->k; q.R = (int)R; q.E = d->E; q.d = d->d_model;
  q.pad_tiles = pad_tiles;
  q.m_tiles_max = (int)tiles;
  q.chunk = mx4::dispatch_chunk(R);
  q.blocks = (int)((R + q.chunk - 1) / q.chunk);
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o = (o + bytes + 255) / 256 * 256; return at; };
  const size_t rp = (size_t)tiles * kTileRows;
  pl->w_status = take(kStatusWords * 4);
  pl->w_flat2row = take((size_t)R * 4);
  pl->w_rowmap = take(rp * 4);
  pl->w_tile_expert = take((size_t)tiles * 4);
  pl->w_tile_rows = take((size_t)tiles * 4);
  pl->w_n_tiles = take(4);
  pl->w_block_counts = take((size_t)q.blocks * d->E * 4);
  pl->w_pad_offsets = take((size_t)(d->E + 1) * 4);
  pl->w_xs = take(rp * d_pitch);
  pl->w_xs_scales = take((size_t)tiles * scale_tiles_k(d->d_model) * kTileBytes);
  pl->w_act = take(rp * f_pitch);
  pl->w_act_scales = take((size_t)tiles * scale_tiles_k(d->d_ff) * kTileBytes);
  pl->w_rows = take((size_t)R * d->d_model * 4);
  pl->bytes = o;
  return BTX_OK;
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

extern "C" btx_status btx_fp8_matmul_workspace_size(int32_t dtype, int32_t batch, int32_t M, int32_t N, int32_t K,
                                                    size_t* workspace_bytes) {
  btx_status s = check_matmul(dtype, batch, M, N, K);
  if (s != BTX_OK) return s;
  if (!workspace_bytes) return BTX_ERR_INVALID_ARG;
  *workspace_bytes = kStatusWords * 4;
  return BTX_OK;
}

extern "C" btx_status btx_fp8_matmul(int32_t dtype, int32_t batch, int32_t M, int32_t N, int32_t K, const void* a_codes,
                                     const void* a_scales, const void* b_codes, const void* b_scales, void* y,
                                     int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  btx_status s = btx_fp8_matmul_workspace_size(dtype, batch, M, N, K, &need);
  if (s != BTX_OK) return s;
  if (accumulate && dtype != BTX_F32) return BTX_ERR_UNSUPPORTED;
  if (batch == 0 || M == 0) return BTX_OK;
  if (!a_codes || !a_scales || !b_codes || !b_scales || !y || !workspace) return BTX_ERR_INVALID_ARG;
  if (misaligned(a_codes) || misaligned(a_scales) || misaligned(b_codes) || misaligned(b_scales) || misaligned(y) ||
      misaligned(workspace))
    return BTX_ERR_INVALID_ARG;
  if (workspace_bytes < need) return BTX_ERR_WORKSPACE;
  if ((s = check_device()) != BTX_OK) return s;
  GemmArgs g = {};
  g.a_codes = (const uint8_t*)a_codes; g.a_scales = (const uint8_t*)a_scales;
  g.b_codes = (const uint8_t*)b_codes; g.b_scales = (const uint8_t*)b_scales;
  g.batch = batch; g.experts = batch; g.M = M; g.N = N; g.K = K; g.status = (int32_t*)workspace;
  return fp8::launch_matmul(g, dtype, y, accumulate != 0, (cudaStream_t)stream);
}

extern "C" btx_status btx_fp8_moe_workspace_size(const btx_fp8_moe_desc* desc, size_t* workspace_bytes) {
  MoePlan pl;
  btx_status s = make_moe_plan(desc, &pl);
  if (s != BTX_OK) return s;
  if (!workspace_bytes) return BTX_ERR_INVALID_ARG;
  *workspace_bytes = pl.bytes;
  return BTX_OK;
}

extern "C" btx_status btx_fp8_moe_forward(const btx_fp8_moe_desc* desc, const void* x, const void* x_scales,
                                          const int32_t* topk_idx, const float* gates, const void* w13_codes,
                                          const void* w13_scales, const void* w2_codes, const void* w2_scales, void* y,
                                          void* workspace, size_t workspace_bytes, void* stream) {
  MoePlan pl;
  btx_status s = make_moe_plan(desc, &pl);
  if (s != BTX_OK) return s;
  if (desc->T == 0) return BTX_OK;
  if (!x || !topk_idx || !gates || !w13_codes || !w13_scales || !w2_codes || !w2_scales || !y || !workspace)
    return BTX_ERR_INVALID_ARG;
  if (misaligned(x) || misaligned(x_scales) || misaligned(w13_codes) || misaligned(w13_scales) || misaligned(w2_codes) ||
      misaligned(w2_scales) || misaligned(y) || misaligned(workspace) || (((uintptr_t)topk_idx | (uintptr_t)gates) & 3))
    return BTX_ERR_INVALID_ARG;
  if (workspace_bytes < pl.bytes) return BTX_ERR_WORKSPACE;
  if ((s = check_device()) != BTX_OK) return s;
  cudaStream_t st = (cudaStream_t)stream;
  char* ws = (char*)workspace;
  mx4::Dispatch q = pl.q;
  q.topk_idx = topk_idx;
  q.status = (int32_t*)(ws + pl.w_status);
  q.flat2row = (int32_t*)(ws + pl.w_flat2row); q.rowmap = (int32_t*)(ws + pl.w_rowmap);
  q.tile_expert = (int32_t*)(ws + pl.w_tile_expert); q.tile_rows = (int32_t*)(ws + pl.w_tile_rows); q.n_tiles = (int32_t*)(ws + pl.w_n_tiles);
  q.block_counts = (int32_t*)(ws + pl.w_block_counts); q.pad_offsets = (int32_t*)(ws + pl.w_pad_offsets);
  uint8_t *xs = (uint8_t*)ws + pl.w_xs, *xs_scales = (uint8_t*)ws + pl.w_xs_scales;
  uint8_t *act = (uint8_t*)ws + pl.w_act, *act_scales = (uint8_t*)ws + pl.w_act_scales;
  float* rows = (float*)(ws + pl.w_rows);
  GemmArgs up = {}, down = {};
  up.batch = 1; up.M = q.m_tiles_max * kTileRows; up.experts = desc->E; up.status = q.status;
  up.a_codes = xs; up.a_scales = xs_scales; up.b_codes = (const uint8_t*)w13_codes; up.b_scales = (const uint8_t*)w13_scales;
  up.N = 2 * desc->d_ff; up.K = desc->d_model;
  down = up;
  down.a_codes = act; down.a_scales = act_scales; down.b_codes = (const uint8_t*)w2_codes; down.b_scales = (const uint8_t*)w2_scales;
  down.N = desc->d_model; down.K = desc->d_ff;
  // every kernel is a programmatic dependent of the one before it
  if (mx4::launch_dispatch(q, st) != cudaSuccess) return BTX_ERR_CUDA;
  if (launch_dispatch_rows(q, desc->dtype, x, (const uint8_t*)x_scales, xs, xs_scales, st) != cudaSuccess) return BTX_ERR_CUDA;
  if ((s = fp8::launch_gate_up(up, q, act, act_scales, st)) != BTX_OK) return s;
  if ((s = fp8::launch_down(down, q, gates, rows, st)) != BTX_OK) return s;
  return mx4::launch_combine_rows(q, desc->dtype, rows, y, st) == cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
}
