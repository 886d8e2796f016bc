// Launchers of the operators in 8 bits (kernels_fp8.hip, kernels_fp8_matmul.hip); all asynchronous on `stream`.
#pragma once

#include "internal.h"

namespace demon {

// rows in e4m3 with the scales [blocks of 128 channels][row] of their blocks
struct RowsFp8 { int rows, channels; uint8_t* q; long long q_stride; float* scale; long long scale_stride; };
// y = x, or (gated) silu(x[0 .. channels)) * x[channels .. 2 channels)
hipError_t launch_quantize_fp8(const RowsFp8& a, const void* x, long long x_stride, bool gated, bool bf16, hipStream_t stream);
// h = x (+ residual), written to `sum` if given; y = h / sqrt(mean(h^2) + eps) * weight
struct NormFp8 { const void* x; long long x_stride; const void* residual; long long residual_stride; const float* weight; float eps;
                 void* sum; long long sum_stride; };
constexpr int kNormFp8Channels = 32768;      // a row is held in the registers of at most 1024 threads
constexpr int kFp8Rows = (1 << 22) - 1;      // of rows that are written in 8 bits: a launch has at most 2^32 - 1 threads
hipError_t launch_rms_norm_fp8(const RowsFp8& a, const NormFp8& n, bool bf16, hipStream_t stream);
// weights [n][k] in e4m3 with the scales [blocks of 128 rows][blocks of 128 columns]
hipError_t launch_quantize_weights_fp8(const void* w, long long w_stride, int n, int k, bool bf16, uint8_t* q, long long q_stride, float* scale,
                                       hipStream_t stream);
// out = a w^T by the blocks' scales (+ bias), fp32 or bf16; n_frames > 0: out is [rows / n_frames][n][n_frames].  fp32_sums: bf16 outputs' too.
// hipErrorNotSupported: more outputs than a launch has threads for (nothing was launched)
struct MatmulFp8 { const uint8_t* a; long long a_stride; const float* a_scale; long long a_scale_stride; const uint8_t* w; long long w_stride;
                   const float* w_scale; const float* bias; void* out; long long out_stride; int rows, n, k, n_frames; };
hipError_t launch_matmul_fp8(const MatmulFp8& a, bool bf16, bool fp32_sums, hipStream_t stream);

}  // namespace demon
