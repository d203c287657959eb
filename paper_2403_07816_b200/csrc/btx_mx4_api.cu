// C ABI of the MXFP4 path: argument checks, the buffer plan and the launch sequence of the expert layer.
#include "btx_mx4.cuh"

namespace btx {
namespace mx4 {
namespace {

constexpr long long kMaxItems = 1ll << 30;           // output tiles of a product are numbered in 32 bits
constexpr int kMaxSide = 1 << 30;                    // so are rows and columns, and the ends of the tiles past the last one
constexpr long long kMaxCodes = 1ll << 40;           // bytes of a matrix of codes: a tensor map's stride is below this

thread_local bool g_separate = false;                // btx_selftest_separate_launches

size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

long long row_tiles(long long rows) { return (rows + kTileRows - 1) / kTileRows; }

btx_status check_shape(int batch, int rows, int K) {
  if (batch < 0 || rows < 0 || K < 1) return BTX_ERR_INVALID_ARG;
  if (K % kBlock != 0 || rows > kMaxSide || K > kMaxSide) return BTX_ERR_UNSUPPORTED;
  const long long codes = rows * (long long)(K / 2), scales = row_tiles(rows) * scale_tiles_k(K) * kTileBytes;
  if (codes >= kMaxCodes || (batch > 0 && (codes > scales ? codes : scales) > (1ll << 62) / batch)) return BTX_ERR_UNSUPPORTED;
  return BTX_OK;
}

struct MoePlan {
  Dispatch q;
  size_t w_status, w_flat2row, w_rowmap, w_tile_expert, w_tile_rows, w_n_tiles, w_block_counts, w_pad_offsets, w_xs, w_xs_scales, w_act,
      w_act_scales, w_rows, bytes;
};

btx_status make_moe_plan(const btx_mx4_moe_desc* d, MoePlan* pl) {
  if (!d || !pl) return BTX_ERR_INVALID_ARG;
  if (d->T < 0 || d->d_model < 1 || d->d_ff < 1 || d->E < 1 || d->k < 1 || d->k > d->E) return BTX_ERR_INVALID_ARG;
  if (d->dtype != BTX_F32 && d->dtype != BTX_BF16) return BTX_ERR_INVALID_ARG;
  if (d->E > kMaxExperts4 || d->d_model % kBlock || d->d_ff % kBlock || d->d_model > kMaxSide || d->d_ff > kMaxSide / 2)
    return BTX_ERR_UNSUPPORTED;
  const long long R = (long long)d->T * d->k;
  if (R > (1ll << 28)) return BTX_ERR_UNSUPPORTED;
  const long long used = R < d->E ? R : d->E;        // experts that can hold a row
  const int pad_tiles = pairs_fit(R, used, d->d_model, d->d_ff) ? 2 : 1;
  const long long unit = pad_tiles * kTileRows;
  const long long tiles = (R + used * (unit - 1)) / unit * pad_tiles;
  const long long wide = d->d_model > d->d_ff ? d->d_model : d->d_ff;       // codes of the rows, of W1 and W3, of W2
  if (tiles * kTileRows * (wide / 2) >= kMaxCodes || (long long)d->d_ff * d->d_model >= kMaxCodes) return BTX_ERR_UNSUPPORTED;
  const long long widest = d->d_model > 2 * (long long)d->d_ff ? d->d_model : 2 * (long long)d->d_ff;
  if (tiles * row_tiles(widest) > kMaxItems) return BTX_ERR_UNSUPPORTED;
  *pl = MoePlan();
  Dispatch& q = pl->q;
  q.T = d->T; q.k = d->k; q.R = (int)R; q.E = d->E; q.d = d->d_model;
  q.pad_tiles = pad_tiles;
  q.m_tiles_max = (int)tiles;
  q.chunk = dispatch_chunk(R);
  q.blocks = (int)((R + q.chunk - 1) / q.chunk);
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o = align_up(o + bytes, 256); return at; };
  const size_t rp = (size_t)tiles * kTileRows;
  pl->w_status = take(kStatusWords * 4);
  pl->w_flat2row = take((size_t)R * 4);
  pl->w_rowmap = take(rp * 4);
  pl->w_tile_expert = take((size_t)tiles * 4);
  pl->w_tile_rows = take((size_t)tiles * 4);
  pl->w_n_tiles = take(4);
  pl->w_block_counts = take((size_t)q.blocks * d->E * 4);
  pl->w_pad_offsets = take((size_t)(d->E + 1) * 4);
  pl->w_xs = take(rp * (d->d_model / 2));
  pl->w_xs_scales = take((size_t)tiles * scale_tiles_k(d->d_model) * kTileBytes);
  pl->w_act = take(rp * (d->d_ff / 2));
  pl->w_act_scales = take((size_t)tiles * scale_tiles_k(d->d_ff) * kTileBytes);
  pl->w_rows = take((layer_fits(q) ? layer_rows_floats(q) : (size_t)R * d->d_model) * 4);
  pl->bytes = o;
  return BTX_OK;
}

btx_status check_matmul(int dtype, int batch, int M, int N, int K) {
  if (dtype != BTX_F32 && dtype != BTX_BF16) return BTX_ERR_INVALID_ARG;
  if (batch < 0 || M < 0 || N < 1) return BTX_ERR_INVALID_ARG;
  btx_status s = check_shape(batch, M, K);
  if (s != BTX_OK) return s;
  if ((s = check_shape(batch, N, K)) != BTX_OK) return s;
  if (row_tiles(M) * row_tiles(N) > kMaxItems || row_tiles(M) * row_tiles(N) * batch > kMaxItems) return BTX_ERR_UNSUPPORTED;
  return BTX_OK;
}

}  // namespace
}  // namespace mx4
}  // namespace btx

using namespace btx;
using namespace btx::mx4;

extern "C" btx_status btx_mx4_sizes(int32_t batch, int32_t rows, int32_t K, size_t* code_bytes, size_t* scale_bytes) {
  btx_status s = check_shape(batch, rows, K);
  if (s != BTX_OK) return s;
  if (code_bytes) *code_bytes = (size_t)batch * rows * (K / 2);
  if (scale_bytes) *scale_bytes = (size_t)batch * row_tiles(rows) * scale_tiles_k(K) * kTileBytes;
  return BTX_OK;
}

extern "C" btx_status btx_mx4_quantize(int32_t dtype, const void* src, int64_t row_stride, int64_t batch_stride, int32_t batch,
                                       int32_t rows, int32_t K, int32_t out_rows, int32_t row_first, int32_t row_step,
                                       void* codes, void* scales, void* stream) {
  btx_status s = check_shape(batch, rows, K);
  if (s != BTX_OK) return s;
  if (dtype != BTX_F32 && dtype != BTX_BF16) return BTX_ERR_INVALID_ARG;
  if (row_first < 0 || row_step < 1 || out_rows < 0) return BTX_ERR_INVALID_ARG;
  if ((s = check_shape(batch, out_rows, K)) != BTX_OK) return s;
  if (rows > 0 && (long long)row_first + (long long)(rows - 1) * row_step >= out_rows) return BTX_ERR_INVALID_ARG;
  if (batch == 0 || rows == 0) return BTX_OK;
  if (!src || !codes || !scales) return BTX_ERR_INVALID_ARG;
  if (row_stride < 0 || batch_stride < 0) return BTX_ERR_INVALID_ARG;
  if (((uintptr_t)src & (dtype == BTX_BF16 ? 1 : 3)) || misaligned(codes) || misaligned(scales)) return BTX_ERR_INVALID_ARG;
  if ((s = check_device()) != BTX_OK) return s;
  CastParams p = {};
  p.src = src; p.row_stride = row_stride; p.batch_stride = batch_stride; p.batch = batch; p.rows = rows; p.K = K;
  p.out_rows = out_rows; p.first = row_first; p.step = row_step; p.codes = (uint8_t*)codes; p.scales = (uint8_t*)scales;
  return launch_quantize(p, dtype, (cudaStream_t)stream) == cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
}

extern "C" btx_status btx_mx4_dequantize(int32_t dtype, const void* codes, const void* scales, int32_t batch, int32_t rows,
                                         int32_t K, void* dst, void* stream) {
  btx_status s = check_shape(batch, rows, K);
  if (s != BTX_OK) return s;
  if (dtype != BTX_F32 && dtype != BTX_BF16) return BTX_ERR_INVALID_ARG;
  if (batch == 0 || rows == 0) return BTX_OK;
  if (!codes || !scales || !dst || misaligned(codes) || misaligned(scales) || misaligned(dst)) return BTX_ERR_INVALID_ARG;
  if ((s = check_device()) != BTX_OK) return s;
  return launch_dequantize((const uint8_t*)codes, (const uint8_t*)scales, batch, rows, K, dtype, dst, (cudaStream_t)stream) ==
                 cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
}

extern "C" btx_status btx_mx4_matmul_workspace_size(int32_t dtype, int32_t batch, int32_t M, int32_t N, int32_t K,
                                                    size_t* workspace_bytes) {
  btx_status s = check_matmul(dtype, batch, M, N, K);
  if (s != BTX_OK) return s;
  if (!workspace_bytes) return BTX_ERR_INVALID_ARG;
  *workspace_bytes = kStatusWords * 4;
  return BTX_OK;
}

extern "C" btx_status btx_mx4_matmul(int32_t dtype, int32_t batch, int32_t M, int32_t N, int32_t K, const void* a_codes,
                                     const void* a_scales, const void* b_codes, const void* b_scales, void* y,
                                     void* workspace, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  btx_status s = btx_mx4_matmul_workspace_size(dtype, batch, M, N, K, &need);
  if (s != BTX_OK) return s;
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
  return launch_matmul(g, dtype, y, (cudaStream_t)stream);
}

extern "C" btx_status btx_mx4_moe_workspace_size(const btx_mx4_moe_desc* desc, size_t* workspace_bytes) {
  MoePlan pl;
  btx_status s = make_moe_plan(desc, &pl);
  if (s != BTX_OK) return s;
  if (!workspace_bytes) return BTX_ERR_INVALID_ARG;
  *workspace_bytes = pl.bytes;
  return BTX_OK;
}

extern "C" btx_status btx_mx4_moe_forward(const btx_mx4_moe_desc* desc, const void* x, const int32_t* topk_idx,
                                          const float* gates, const void* w13_codes, const void* w13_scales,
                                          const void* w2_codes, const void* w2_scales, void* y, void* workspace,
                                          size_t workspace_bytes, void* stream) {
  MoePlan pl;
  btx_status s = make_moe_plan(desc, &pl);
  if (s != BTX_OK) return s;
  if (desc->T == 0) return BTX_OK;
  if (!x || !topk_idx || !gates || !w13_codes || !w13_scales || !w2_codes || !w2_scales || !y || !workspace)
    return BTX_ERR_INVALID_ARG;
  if (misaligned(x) || misaligned(w13_codes) || misaligned(w13_scales) || misaligned(w2_codes) || misaligned(w2_scales) ||
      misaligned(y) || misaligned(workspace) || (((uintptr_t)topk_idx | (uintptr_t)gates) & 3))
    return BTX_ERR_INVALID_ARG;
  if (workspace_bytes < pl.bytes) return BTX_ERR_WORKSPACE;
  if ((s = check_device()) != BTX_OK) return s;
  cudaStream_t st = (cudaStream_t)stream;
  char* ws = (char*)workspace;
  Dispatch q = pl.q;
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
  if (layer_fits(q) && !g_separate) {
    s = launch_layer(up, down, q, desc->dtype, x, gates, rows, act, act_scales, y, st);
    if (s != BTX_ERR_UNSUPPORTED) return s;  // else not every block can be resident: the launches below do the same work
  }
  // every kernel is a programmatic dependent of the one before it
  if (launch_dispatch(q, st) != cudaSuccess) return BTX_ERR_CUDA;
  if (launch_quantize_rows(q, desc->dtype, x, xs, xs_scales, st) != cudaSuccess) return BTX_ERR_CUDA;
  if ((s = launch_gate_up(up, q, act, act_scales, st)) != BTX_OK) return s;
  if ((s = launch_down(down, q, gates, rows, st)) != BTX_OK) return s;
  return launch_combine_rows(q, desc->dtype, rows, y, st) == cudaSuccess ? BTX_OK : BTX_ERR_CUDA;
}

extern "C" btx_status btx_selftest_separate_launches(int32_t on) {
  g_separate = on != 0;
  return BTX_OK;
}
