// Launchers of the FP8 products (btx_fp8_gemm.cu) and of the expert layer's dispatch (btx_fp8_cast.cu).
#pragma once

#include "btx_fp8.cuh"
#include "btx_mx4.cuh"

namespace btx {
namespace fp8 {

// A: codes [batch, M, K] (grouped: the padded rows), B: codes [batch or experts, N, K].  Sizes as in mx4::GemmArgs.
using GemmArgs = mx4::GemmArgs;
// x [T, d], in dtype or (x_scales != nullptr) as FP8 codes, to the padded rows of every token's experts
cudaError_t launch_dispatch_rows(const mx4::Dispatch& q, int dtype, const void* x, const uint8_t* x_scales, uint8_t* codes,
                                 uint8_t* scales, cudaStream_t st);
bool pairs_fit(long long rows, long long experts, long long d, long long F);
// accumulate: fp32 y is added to
btx_status launch_matmul(const GemmArgs& g, int dtype, void* y, int accumulate, cudaStream_t st);
// W1/W3 product (rows interleaved) with silu(h1) * h3 cast to FP8
btx_status launch_gate_up(const GemmArgs& g, const mx4::Dispatch& q, uint8_t* act_codes, uint8_t* act_scales, cudaStream_t st);
// W2 product, gate-scaled fp32 rows at [t*k+slot]
btx_status launch_down(const GemmArgs& g, const mx4::Dispatch& q, const float* gates, float* rows, cudaStream_t st);

}  // namespace fp8
}  // namespace btx
