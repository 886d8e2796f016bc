// Matrix product of rows and weights in 8 bits (e4m3), with a scale for each block of 128 along K:
//
//   out[m][n] = bias[n] + sum over blocks b of  a_scale[b][m] w_scale[n / 128][b]  sum over k in b of a[m][k] w[n][k]
//
// A product of two e4m3 values is exact in fp32.  The inner sum of 256 outputs starts from zero in the MFMA, and its result is added to the fp32
// accumulators with the block's two scales, one multiply-add an output.  There are two ways to it:
//   output bf16: one 16 x 16 x 128 MFMA on the 8-bit operands.  The matrix unit aligns the products of 8-bit operands to the largest of those it adds
//     at once and keeps about 13 bits below it (every shape of that MFMA does: 1.3e-5 of the result for normal values in the 2-norm, at most
//     2^-11.7 of the block's largest product in any output), a hundredth of the output's rounding of 2^-8;
//   output fp32: the operands widened to halves, which hold every e4m3 value, and four 16 x 16 x 32 MFMAs of halves, which add in fp32 (7e-8).  The
//     matrix unit does half as many of these a second.
// The weights are the rows of the MFMA's result (operand A) and the rows of `a` its columns (operand B): a lane then holds results of
// one row of `a`, and the product of the scales is one value a lane and tile.
//
// Operand layout: lane l of either operand holds row l % 16 of its tile and, of a block of 128 values of K, the pieces of 16 bytes
// l / 16 and l / 16 + 4.  Which values of K a lane holds is free as long as A and B agree, since the MFMA sums over all of them; with these
// pieces one load of a wave reads 64 bytes that follow each other of each of 16 rows.
#include "device_common.h"

namespace demon {

namespace {

constexpr int kBlock = 128;
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef u32x4 loose16 __attribute__((aligned(1)));

struct Frag { u32x4 lo, hi; };

// Operands of the MFMAs of a block, as the output's type has them multiplied.
template <typename O> struct Operand;
template <> struct Operand<uint16_t> {
    i32x8 v;
    __device__ __forceinline__ void set(const Frag& f)
    {
        v = i32x8{(int)f.lo[0], (int)f.lo[1], (int)f.lo[2], (int)f.lo[3], (int)f.hi[0], (int)f.hi[1], (int)f.hi[2], (int)f.hi[3]};
    }
};
template <> struct Operand<float> {
    f16x8 v[4];
    __device__ __forceinline__ void set(const Frag& f)
    {
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                const int bits = (int)(s < 2 ? f.lo[2 * s + d] : f.hi[2 * s + d - 4]);
                const f16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(bits, 1.f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(bits, 1.f, true);
                v[s][4 * d] = lo[0]; v[s][4 * d + 1] = lo[1]; v[s][4 * d + 2] = hi[0]; v[s][4 * d + 3] = hi[1];
            }
    }
};

__device__ __forceinline__ f32x4 block_product(const Operand<uint16_t>& a, const Operand<uint16_t>& b)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
}
__device__ __forceinline__ f32x4 block_product(const Operand<float>& a, const Operand<float>& b)
{
    f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < 4; ++s) p = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.v[s], b.v[s], p, 0, 0, 0);
    return p;
}

// A piece of 16 values at p, of which the first `left` belong to the row; zeros for the others, which are not read.
__device__ __forceinline__ u32x4 load_piece(const uint8_t* p, int left)
{
    u32x4 v = {};
    if (left >= 16) v = *reinterpret_cast<const loose16*>(p);
    else {
#pragma unroll
        for (int e = 0; e < 15; ++e)
            if (e < left) v[e / 4] |= (uint32_t)p[e] << (8 * (e % 4));
    }
    return v;
}

__device__ __forceinline__ void store_out(uint16_t* p, float v) { *p = f32_to_bf16_bits(v); }
__device__ __forceinline__ void store_out(float* p, float v) { *p = v; }

// Where out[m][n] is: rows of n values, or the latent [clip][n][frame] of rows m = clip * n_frames + frame.
template <typename O> __device__ __forceinline__ O* out_at(const MatmulFp8& a, long long m, long long n)
{
    O* out = (O*)a.out;
    if (a.n_frames == 0) return out + m * a.out_stride + n;
    const long long clip = m / a.n_frames, frame = m - clip * a.n_frames;
    return out + (clip * a.n + n) * a.n_frames + frame;
}

}  // namespace

// ---------------------------------------------------------------------------------- operands straight from memory
// A workgroup of W waves takes 16 FN weight rows by 16 FM rows; each wave sums every W-th block of K, from operands that it loads into
// registers itself, and the waves' sums are added in their order through LDS.  Reads any alignment and any K.
template <typename O, int FN, int FM, int W>
__global__ __launch_bounds__(64 * W) void matmul_direct_kernel(MatmulFp8 a)
{
    __shared__ f32x4 part[W][FN * FM][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, piece = lane >> 4;
    const int tiles_n = (a.n + 16 * FN - 1) / (16 * FN);
    const int n0 = (int)(blockIdx.x % tiles_n) * 16 * FN, m0 = (int)(blockIdx.x / tiles_n) * 16 * FM;
    const int blocks = (a.k + kBlock - 1) / kBlock;
    const uint8_t *pw[FN], *pa[FM];
    const float* ps[FM];
#pragma unroll
    for (int i = 0; i < FN; ++i) pw[i] = a.w + (long long)min(n0 + 16 * i + col, a.n - 1) * a.w_stride + piece * 16;   // rows behind the last:
#pragma unroll
    for (int j = 0; j < FM; ++j) {                                                                                     // the last again, not stored
        const int m = min(m0 + 16 * j + col, a.rows - 1);
        pa[j] = a.a + (long long)m * a.a_stride + piece * 16;
        ps[j] = a.a_scale + m;
    }
    const float* pws = a.w_scale + (long long)(n0 / kBlock) * blocks;
    f32x4 acc[FN][FM] = {};
    for (int b = wave; b < blocks; b += W) {
        const long long at = (long long)b * kBlock;
        const int left = (int)min((long long)a.k - at, (long long)kBlock) - piece * 16;
        Operand<O> fw[FN], fa[FM];
#pragma unroll
        for (int i = 0; i < FN; ++i) fw[i].set({load_piece(pw[i] + at, left), load_piece(pw[i] + at + 64, left - 64)});
#pragma unroll
        for (int j = 0; j < FM; ++j) fa[j].set({load_piece(pa[j] + at, left), load_piece(pa[j] + at + 64, left - 64)});
        const float sw = pws[b];
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            const float s = sw * ps[j][b * a.a_scale_stride];
#pragma unroll
            for (int i = 0; i < FN; ++i) {
                const f32x4 p = block_product(fw[i], fa[j]);
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][j][r] = fmaf(s, p[r], acc[i][j][r]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) part[wave][i * FM + j][lane] = acc[i][j];
    __syncthreads();
    for (int t = wave; t < FN * FM; t += W) {
        f32x4 v = part[0][t][lane];
#pragma unroll
        for (int w = 1; w < W; ++w) v += part[w][t][lane];
        const int m = m0 + 16 * (t % FM) + col;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int n = n0 + 16 * (t / FM) + 4 * piece + r;
            if (m < a.rows && n < a.n) store_out(out_at<O>(a, m, n), v[r] + (a.bias ? a.bias[n] : 0.f));
        }
    }
}

template <typename O> static hipError_t launch_direct(const MatmulFp8& a, hipStream_t stream)
{
    constexpr int FN = 2, FM = 2, W = 4;
    const long long tiles = (long long)((a.n + 16 * FN - 1) / (16 * FN)) * ((a.rows + 16 * FM - 1) / (16 * FM));
    if (tiles > 0x7fffffffll) return hipErrorInvalidValue;
    hipLaunchKernelGGL((matmul_direct_kernel<O, FN, FM, W>), dim3((unsigned)tiles), dim3(64 * W), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_matmul_fp8(const MatmulFp8& a, bool bf16, hipStream_t stream)
{
    return bf16 ? launch_direct<uint16_t>(a, stream) : launch_direct<float>(a, stream);
}

}  // namespace demon
