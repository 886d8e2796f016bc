// C entry points of the operands in 8 bits and of their product: argument checks, then one launch each.
#include "fp8.h"

using namespace demon;

namespace {

demon_status launched(hipError_t e, const char* what)
{
    return e == hipSuccess ? DEMON_OK : fail(DEMON_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

int blocks_of(int n) { return n / 128 + (n % 128 != 0); }

// the 8-bit rows and their scales that an operator writes
demon_status check_rows(int rows, int channels, demon_dtype dtype, const void* q, long long q_stride, const float* scale, long long scale_stride)
{
    if (!q || !scale) return fail(DEMON_ERR_INVALID_ARG, "NULL argument");
    if (rows < 1 || channels < 1) return fail(DEMON_ERR_INVALID_ARG, "rows and channels must be >= 1");
    if (dtype != DEMON_F32 && dtype != DEMON_BF16) return fail(DEMON_ERR_INVALID_ARG, "unknown dtype");
    if (q_stride < channels) return fail(DEMON_ERR_INVALID_ARG, "8-bit rows overlap");
    if (scale_stride < rows) return fail(DEMON_ERR_INVALID_ARG, "scales of blocks overlap");
    if (rows > kFp8Rows) return fail(DEMON_ERR_UNSUPPORTED, "more than %d rows", kFp8Rows);
    return DEMON_OK;
}

demon_status matmul(const MatmulFp8& a, demon_dtype out_dtype, bool fp32_sums, void* stream)
{
    clear_error();
    if (!a.a || !a.a_scale || !a.w || !a.w_scale || !a.out) return fail(DEMON_ERR_INVALID_ARG, "NULL argument");
    if (a.rows < 1 || a.n < 1 || a.k < 1) return fail(DEMON_ERR_INVALID_ARG, "rows, n and k must be >= 1");
    if (out_dtype != DEMON_F32 && out_dtype != DEMON_BF16) return fail(DEMON_ERR_INVALID_ARG, "unknown dtype");
    if (a.a_stride < 0 || a.w_stride < 0) return fail(DEMON_ERR_INVALID_ARG, "negative row stride");
    if (a.a_scale_stride < a.rows) return fail(DEMON_ERR_INVALID_ARG, "scales of blocks overlap");
    if (a.n_frames < 0 || (a.n_frames > 0 && a.rows % a.n_frames != 0)) return fail(DEMON_ERR_INVALID_ARG, "rows must be a multiple of n_frames");
    if (a.n_frames == 0 && a.out_stride < a.n) return fail(DEMON_ERR_INVALID_ARG, "output rows overlap");
    if (a.rows > (1 << 24) || a.n > (1 << 24) || a.k > (1 << 24)) return fail(DEMON_ERR_UNSUPPORTED, "more than 16777216 rows, columns or values of K");
    const hipError_t e = launch_matmul_fp8(a, out_dtype == DEMON_BF16, fp32_sums, (hipStream_t)stream);
    if (e == hipErrorNotSupported) return fail(DEMON_ERR_UNSUPPORTED, "more outputs than a launch has threads for");
    return launched(e, "matrix product");
}

}  // namespace

extern "C" {

demon_status demon_vae_quantize_fp8(const void* d_x, long long x_stride, int rows, int channels, int gated, demon_dtype dtype,
                                    void* d_q, long long q_stride, float* d_scale, long long scale_stride, void* stream)
{
    clear_error();
    if (!d_x) return fail(DEMON_ERR_INVALID_ARG, "NULL argument");
    if (const demon_status rc = check_rows(rows, channels, dtype, d_q, q_stride, d_scale, scale_stride); rc != DEMON_OK) return rc;
    if (x_stride < 0) return fail(DEMON_ERR_INVALID_ARG, "negative row stride");
    if (channels > (1 << 24)) return fail(DEMON_ERR_UNSUPPORTED, "more than 16777216 channels");
    const RowsFp8 a = {rows, channels, (uint8_t*)d_q, q_stride, d_scale, scale_stride};
    return launched(launch_quantize_fp8(a, d_x, x_stride, gated != 0, dtype == DEMON_BF16, (hipStream_t)stream), "quantize");
}

demon_status demon_vae_rms_norm_fp8(const void* d_x, long long x_stride, const void* d_residual, long long residual_stride, const float* d_weight,
                                    int rows, int channels, float eps, demon_dtype dtype, void* d_sum, long long sum_stride,
                                    void* d_q, long long q_stride, float* d_scale, long long scale_stride, void* stream)
{
    clear_error();
    if (!d_x || !d_weight) return fail(DEMON_ERR_INVALID_ARG, "NULL argument");
    if (const demon_status rc = check_rows(rows, channels, dtype, d_q, q_stride, d_scale, scale_stride); rc != DEMON_OK) return rc;
    if (!(eps >= 0.f) || eps > 3.0e38f) return fail(DEMON_ERR_INVALID_ARG, "eps must be >= 0 and finite");
    if (x_stride < 0 || (d_residual && residual_stride < 0)) return fail(DEMON_ERR_INVALID_ARG, "negative row stride");
    if (d_sum && sum_stride < channels) return fail(DEMON_ERR_INVALID_ARG, "rows of the sum overlap");
    if (d_sum && ((d_sum == d_x && sum_stride != x_stride) || (d_sum == d_residual && sum_stride != residual_stride)))
        return fail(DEMON_ERR_INVALID_ARG, "a sum in place must have the input's row stride");
    if (channels > kNormFp8Channels) return fail(DEMON_ERR_UNSUPPORTED, "more than %d channels", kNormFp8Channels);
    const RowsFp8 a = {rows, channels, (uint8_t*)d_q, q_stride, d_scale, scale_stride};
    const NormFp8 n = {d_x, x_stride, d_residual, residual_stride, d_weight, eps, d_sum, sum_stride};
    return launched(launch_rms_norm_fp8(a, n, dtype == DEMON_BF16, (hipStream_t)stream), "rms norm");
}

demon_status demon_vae_quantize_weights_fp8(const void* d_w, long long w_stride, int n, int k, demon_dtype dtype,
                                            void* d_q, long long q_stride, float* d_scale, void* stream)
{
    clear_error();
    if (!d_w || !d_q || !d_scale) return fail(DEMON_ERR_INVALID_ARG, "NULL argument");
    if (n < 1 || k < 1) return fail(DEMON_ERR_INVALID_ARG, "n and k must be >= 1");
    if (dtype != DEMON_F32 && dtype != DEMON_BF16) return fail(DEMON_ERR_INVALID_ARG, "unknown dtype");
    if (w_stride < 0) return fail(DEMON_ERR_INVALID_ARG, "negative row stride");
    if (q_stride < k) return fail(DEMON_ERR_INVALID_ARG, "8-bit rows overlap");
    if (n > (1 << 24) || k > (1 << 24) || (long long)blocks_of(n) * blocks_of(k) >= (1 << 24)) return fail(DEMON_ERR_UNSUPPORTED, "matrix too large");
    return launched(launch_quantize_weights_fp8(d_w, w_stride, n, k, dtype == DEMON_BF16, (uint8_t*)d_q, q_stride, d_scale, (hipStream_t)stream),
                    "quantize weights");
}

demon_status demon_vae_matmul_fp8(const void* d_a, long long a_stride, const float* d_a_scale, long long a_scale_stride,
                                  const void* d_w, long long w_stride, const float* d_w_scale, const float* d_bias, int rows, int n, int k,
                                  int n_frames, demon_dtype out_dtype, void* d_out, long long out_stride, void* stream)
{
    const MatmulFp8 a = {(const uint8_t*)d_a, a_stride, d_a_scale, a_scale_stride, (const uint8_t*)d_w, w_stride, d_w_scale, d_bias,
                         d_out, out_stride, rows, n, k, n_frames};
    return matmul(a, out_dtype, false, stream);
}

demon_status demon_vae_matmul_fp8_fp32_sums(const void* d_a, long long a_stride, const float* d_a_scale, long long a_scale_stride,
                                            const void* d_w, long long w_stride, const float* d_w_scale, const float* d_bias, int rows, int n, int k,
                                            int n_frames, demon_dtype out_dtype, void* d_out, long long out_stride, void* stream)
{
    const MatmulFp8 a = {(const uint8_t*)d_a, a_stride, d_a_scale, a_scale_stride, (const uint8_t*)d_w, w_stride, d_w_scale, d_bias,
                         d_out, out_stride, rows, n, k, n_frames};
    return matmul(a, out_dtype, true, stream);
}

}  // extern "C"
