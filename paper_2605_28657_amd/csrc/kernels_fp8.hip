// Rows and weights in 8 bits: the operands of the 8-bit matrix product (kernels_fp8_matmul.hip), in e4m3 (sign, 4 bits of exponent, 3 of
// mantissa; largest value 448, no infinity) with one fp32 scale for each block of 128 channels of a row, or for each 128 x 128 block of a
// weight matrix.
//
//   scale = max(max |y|, 2^-100) / 448,   q = e4m3(y * (1 / scale)), round to nearest even
//
// so that the block's largest value becomes 448 and its other ones are off by at most 2^-4 of themselves (2^-10 scale where e4m3 is
// subnormal).  The smallest scale keeps 1 / scale finite: a block of zeros has the scale 2^-100 / 448 and zeros.  The maximum is taken on the
// bit patterns of |y| as integers, which order like the values with the NaNs above infinity: a block with a NaN has a NaN as its
// scale and is NaN throughout, one with an infinity has an infinite scale, NaN where the infinities were and zeros elsewhere.  All
// arithmetic is fp32.
//
// A thread holds 8 channels that follow each other (16 bytes of bf16, 32 of fp32), so that a block is 16 lanes, the row of the wave's
// cross-lane moves: its maximum needs no LDS.  Loads and stores of whole chunks take any alignment that the type has (the hardware's 16-byte
// loads do); the chunk that the row ends in is read and written by elements.
#include <type_traits>

#include "device_common.h"
#include "fp8.h"

namespace demon {

namespace {

constexpr int kBlock = 128;
constexpr float kLargest = 448.f;
constexpr uint32_t kFloorBits = (127 - 100) << 23;          // 2^-100

// Rows of more than this are read past the caches: what comes last would push out what came first before anything finds it there, and their lines would
// take the place of the results (gate of 12000 x 5632 rows, 270 MB: 63.4 -> 55.3 us, norm of 12000 x 2048 with a residual, 98 MB: 35.2 -> 31.2; rows of
// 12000 x 2048, 49 MB, which the 256 MB of the last cache may well hold from whoever wrote them, 12.7 -> 14.2).
constexpr long long kStreamBytes = 64ll << 20;

template <typename T> struct Chunk;                          // 8 channels as they lie in memory
template <> struct Chunk<uint16_t> {
    typedef u32x4 loose __attribute__((aligned(2)));
    u32x4 v = {};
    template <bool STREAM = false> __device__ void load(const uint16_t* p)
    {
        const loose* q = reinterpret_cast<const loose*>(p);
        v = STREAM ? (u32x4)__builtin_nontemporal_load(q) : (u32x4)*q;
    }
    __device__ float get(int e) const { return __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16); }
    __device__ void set(int e, uint16_t x) { v[e / 2] = e & 1 ? (v[e / 2] & 0xffffu) | (uint32_t)x << 16 : (v[e / 2] & 0xffff0000u) | x; }
};
template <> struct Chunk<float> {
    typedef u32x4 loose __attribute__((aligned(4)));
    u32x4 v[2] = {};
    template <bool STREAM = false> __device__ void load(const float* p)
    {
        const loose *q = reinterpret_cast<const loose*>(p), *r = reinterpret_cast<const loose*>(p + 4);
        v[0] = STREAM ? (u32x4)__builtin_nontemporal_load(q) : (u32x4)*q;
        v[1] = STREAM ? (u32x4)__builtin_nontemporal_load(r) : (u32x4)*r;
    }
    __device__ float get(int e) const { return __uint_as_float(v[e / 4][e % 4]); }
    __device__ void set(int e, float x) { v[e / 4][e % 4] = __float_as_uint(x); }
};

// Elements 0 .. n - 1 (0 < n < 8) of a chunk, zeros behind them, which no maximum or sum of squares sees.  The elements of one end are requested together, the last one for those that
// are not there: behind a branch of its own each would wait for the one before (weights of 517 x 1111 in bf16: 8.6 us, so 6.2; norm of 75 x 5631 6.2 -> 5.2).  Several ends of a
// thread (rows of the weights, chunks and operands of the norm) are still waited for one after another.
template <typename T> __device__ __forceinline__ void load_tail(Chunk<T>& c, const T* p, int n)
{
    T v[7];
#pragma unroll
    for (int e = 0; e < 7; ++e) v[e] = p[e < n ? e : n - 1];
#pragma unroll
    for (int e = 0; e < 7; ++e) c.set(e, e < n ? v[e] : (T)0);
}

__device__ __forceinline__ void store8(uint16_t* p, const float (&y)[8])
{
    typedef u32x4 loose __attribute__((aligned(2)));
    const u32x4 v = {pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])};
    *reinterpret_cast<loose*>(p) = v;
}
__device__ __forceinline__ void store8(float* p, const float (&y)[8])
{
    typedef f32x4 loose __attribute__((aligned(4)));
    const f32x4 lo = {y[0], y[1], y[2], y[3]}, hi = {y[4], y[5], y[6], y[7]};
    *reinterpret_cast<loose*>(p) = lo;
    *reinterpret_cast<loose*>(p + 4) = hi;
}
__device__ __forceinline__ void store1(uint16_t* p, float y) { *p = f32_to_bf16_bits(y); }
__device__ __forceinline__ void store1(float* p, float y) { *p = y; }

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Largest of the 16 lanes of a block, in all of them: rotations of the row by 8, 4, 2 and 1.
template <int N> __device__ __forceinline__ uint32_t rotated(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + N, 0xf, 0xf, false); }
__device__ __forceinline__ uint32_t max16(uint32_t v)
{
    v = umax(v, rotated<8>(v));
    v = umax(v, rotated<4>(v));
    v = umax(v, rotated<2>(v));
    return umax(v, rotated<1>(v));
}

__device__ __forceinline__ uint32_t magnitude(const float (&y)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = umax(m, __float_as_uint(y[e]) & 0x7fffffffu);
    return m;
}

// One multiplication by the rounded 1 / 448: off by less than 2 steps of 2^-24 from the quotient, which costs ten instructions.
__device__ __forceinline__ float scale_of(uint32_t largest) { return __uint_as_float(umax(largest, kFloorBits)) * (1.f / kLargest); }

// 1 / scale within a step: the hardware's reciprocal, which is off by up to two, and one Newton step.  0 for an infinite scale.
__device__ __forceinline__ float inverse(float scale)
{
    const float r = __builtin_amdgcn_rcpf(scale);
    return r == 0.f ? 0.f : fmaf(fmaf(-scale, r, 1.f), r, r);
}

// g / (1 + exp(-g)), the exponential and the reciprocal as the hardware has them: off by a few steps of 2^-24 (and of the exponent's rounding, 2^-24 |g| log2 e),
// the value's 8 bits keep 2^-4
__device__ __forceinline__ float silu(float g) { return g * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * -1.44269504f)); }

// Writes the first n (at most 8) values of a chunk.
__device__ __forceinline__ void store_q(uint8_t* p, const float (&y)[8], float inv, int n)
{
    typedef u32x2 loose __attribute__((aligned(1)));
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] * inv, y[1] * inv, lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2] * inv, y[3] * inv, lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4] * inv, y[5] * inv, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6] * inv, y[7] * inv, hi, true);
    if (n >= 8) {
        const u32x2 v = {(uint32_t)lo, (uint32_t)hi};
        *reinterpret_cast<loose*>(p) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) p[e] = (uint8_t)((e < 4 ? lo : hi) >> (8 * (e % 4)));
    }
}

}  // namespace

// ---------------------------------------------------------------------------------- rows, with or without a gate
// y = x, or y = g / (1 + exp(-g)) * u of rows [g | u].  Blocks have nothing to do with each other: a workgroup's 16 groups of lanes take
// 2^log2_rows rows by 16 / 2^log2_rows blocks, U times, all requested before the first is used; as few rows as their blocks fill it, since long runs of a row
// count for more than scales of rows side by side (gate of 12000 x 5632 rows: 16 rows 70.5 us, 4 69.7, 1 63.4: 5360 GB/s, a copy of its size 5390).
template <typename T, bool GATED, bool STREAM, int U>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ x, long long x_stride, int rows, int channels, uint8_t* __restrict__ q,
                                                            long long q_stride, float* __restrict__ scale, long long scale_stride, int log2_rows)
{
    const int group = threadIdx.x >> 4, lane = threadIdx.x & 15;
    const long long row = ((long long)blockIdx.x << log2_rows) + (group & ((1 << log2_rows) - 1));
    if (row >= rows) return;
    const int step = 16 >> log2_rows, first = blockIdx.y * step * U + (group >> log2_rows);
    const T* p = x + row * x_stride;
    Chunk<T> a[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long long c = (long long)(first + u * step) * kBlock + lane * 8;
        if (c + 8 <= channels) {
            a[u].template load<STREAM>(p + c);
            if (GATED) b[u].template load<STREAM>(p + channels + c);
        } else if (c < channels) {
            load_tail(a[u], p + c, (int)(channels - c));
            if (GATED) load_tail(b[u], p + channels + c, (int)(channels - c));
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long long block = first + u * step, c = block * kBlock + lane * 8;
        if (block * kBlock >= channels) return;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            y[e] = a[u].get(e);
            if (GATED) y[e] = silu(y[e]) * b[u].get(e);
        }
        const float s = scale_of(max16(magnitude(y)));
        if (lane == 0) scale[block * scale_stride + row] = s;
        store_q(q + row * q_stride + c, y, inverse(s), (int)(channels - c));
    }
}

hipError_t launch_quantize_fp8(const RowsFp8& a, const void* x, long long x_stride, bool gated, bool bf16, hipStream_t stream)
{
    constexpr int U = 4;
    const int blocks = (a.channels + kBlock - 1) / kBlock;
    int log2_rows = 0;
    while (log2_rows < 4 && (16 >> (log2_rows + 1)) * U >= blocks && (1 << log2_rows) < a.rows) ++log2_rows;
    const int span = (16 >> log2_rows) * U;
    const dim3 grid((unsigned)((a.rows + (1ll << log2_rows) - 1) >> log2_rows), (unsigned)((blocks + span - 1) / span));
    const bool stream_in = (long long)a.rows * a.channels * (gated ? 2 : 1) * (bf16 ? 2 : 4) > kStreamBytes;
    auto go = [&](auto kernel, auto* p) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, p, x_stride, a.rows, a.channels, a.q, a.q_stride, a.scale, a.scale_stride, log2_rows);
    };
    auto by_size = [&](auto* p) {
        typedef std::remove_const_t<std::remove_pointer_t<decltype(p)>> T;
        if (gated) stream_in ? go(quantize_rows_kernel<T, true, true, U>, p) : go(quantize_rows_kernel<T, true, false, U>, p);
        else stream_in ? go(quantize_rows_kernel<T, false, true, U>, p) : go(quantize_rows_kernel<T, false, false, U>, p);
    };
    bf16 ? by_size((const uint16_t*)x) : by_size((const float*)x);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------------- root-mean-square norm
// h = x + residual;  y = h / sqrt(mean(h^2) + eps) * weight, in 8 bits.  A row belongs to N threads that hold it in registers (V chunks
// each) from its one read to its one write; h is summed, squared and normed as it is before it is rounded for `sum`.  A thread writes
// of `sum` what it has read of x and residual, so that `sum` may be either of them.  12000 x 2048 bf16 rows with a residual, 173 MB: 31.2 us, 5550 GB/s with two
// waves a row, 32.2 with one, 32.8 with four.
template <typename T, int N, int V, bool STREAM>
__global__ __launch_bounds__(N < 256 ? 256 : N) void rms_norm_kernel(const T* x, long long x_stride, const T* residual, long long residual_stride,
                                                                     const float* __restrict__ weight, int rows, int channels, float eps,
                                                                     T* sum, long long sum_stride, uint8_t* __restrict__ q, long long q_stride,
                                                                     float* __restrict__ scale, long long scale_stride)
{
    constexpr int R = N < 256 ? 256 / N : 1;
    const int t = threadIdx.x % N;
    const long long mine = (long long)blockIdx.x * R + threadIdx.x / N, row = mine < rows ? mine : rows - 1;
    const bool here = mine < rows;                          // behind the last row the last again, not written
    const T* px = x + row * x_stride;
    const T* pr = residual + row * residual_stride;
    Chunk<T> a[V], b[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = (v * N + t) * 8;
        if (c + 8 <= channels) {
            a[v].template load<STREAM>(px + c);
            if (residual) b[v].template load<STREAM>(pr + c);
        } else if (c < channels) {
            load_tail(a[v], px + c, channels - c);
            if (residual) load_tail(b[v], pr + c, channels - c);
        }
    }
    float h[V][8], squares = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = (v * N + t) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            h[v][e] = a[v].get(e);
            if (residual) h[v][e] += b[v].get(e);
            squares = fmaf(h[v][e], h[v][e], squares);
        }
        if (sum && here && c < channels) {
            T* ps = sum + row * sum_stride + c;
            if (c + 8 <= channels) store8(ps, h[v]);
            else {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (e < channels - c) store1(ps + e, h[v][e]);
            }
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) squares += __shfl_xor(squares, o, 64);
    if constexpr (N > 64) {
        __shared__ float part[R][N / 64];
        if ((t & 63) == 0) part[threadIdx.x / N][t >> 6] = squares;
        __syncthreads();
        squares = 0.f;
#pragma unroll
        for (int w = 0; w < N / 64; ++w) squares += part[threadIdx.x / N][w];
    }
    if (!here) return;
    const float inv = rsqrtf(squares / (float)channels + eps);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int c = (v * N + t) * 8;
        if (c - (t & 15) * 8 >= channels) break;            // the 16 lanes of a block leave together
        Chunk<float> w;
        if (c + 8 <= channels) w.load(weight + c);
        else if (c < channels) load_tail(w, weight + c, channels - c);
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = h[v][e] * inv * w.get(e);
        // behind the last channel h and w are zeros, and 0 * inv is NaN where inv is not finite: such values are not the row's
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = c + e < channels ? y[e] : 0.f;
        const float s = scale_of(max16(magnitude(y)));
        if ((t & 15) == 0) scale[(long long)(c / kBlock) * scale_stride + row] = s;
        store_q(q + row * q_stride + c, y, inverse(s), channels - c);
    }
}

hipError_t launch_rms_norm_fp8(const RowsFp8& a, const NormFp8& n, bool bf16, hipStream_t stream)
{
    const bool stream_in = (long long)a.rows * a.channels * (n.residual ? 2 : 1) * (bf16 ? 2 : 4) > kStreamBytes;
    auto go = [&](auto type, auto threads, auto chunks) {
        typedef decltype(type) T;
        constexpr int N = threads(), V = chunks(), R = N < 256 ? 256 / N : 1;
        hipLaunchKernelGGL((stream_in ? rms_norm_kernel<T, N, V, true> : rms_norm_kernel<T, N, V, false>), dim3((unsigned)((a.rows - 1) / R + 1)), dim3(N < 256 ? 256 : N), 0, stream,
                           (const T*)n.x, n.x_stride, (const T*)n.residual, n.residual_stride, n.weight, a.rows, a.channels, n.eps,
                           (T*)n.sum, n.sum_stride, a.q, a.q_stride, a.scale, a.scale_stride);
    };
    auto by_channels = [&](auto type) {
        using std::integral_constant;
        const int c = a.channels;
        if (c <= 512) go(type, integral_constant<int, 64>(), integral_constant<int, 1>());
        else if (c <= 1024) go(type, integral_constant<int, 64>(), integral_constant<int, 2>());
        else if (c <= 2048) go(type, integral_constant<int, 128>(), integral_constant<int, 2>());
        else if (c <= 4096) go(type, integral_constant<int, 256>(), integral_constant<int, 2>());
        else if (c <= 8192) go(type, integral_constant<int, 256>(), integral_constant<int, 4>());
        else if (c <= 16384) go(type, integral_constant<int, 1024>(), integral_constant<int, 2>());
        else go(type, integral_constant<int, 1024>(), integral_constant<int, 4>());
    };
    if (a.channels > kNormFp8Channels) return hipErrorInvalidValue;
    bf16 ? by_channels(uint16_t()) : by_channels(float());
    return hipGetLastError();
}

// ---------------------------------------------------------------------------------- weights
// A workgroup takes a 128 x 128 block: a row of it in 16 lanes, 8 rows a thread, held in registers between the maximum and the write.  Bound by the bytes
// (11264 x 2048 in bf16, 69 MB, 11.8 us: 5900 GB/s).
template <typename T>
__global__ __launch_bounds__(256) void quantize_weights_kernel(const T* __restrict__ w, long long w_stride, int n, int k, uint8_t* __restrict__ q,
                                                               long long q_stride, float* __restrict__ scale)
{
    __shared__ uint32_t part[4];
    const int t = threadIdx.x, blocks = (k + kBlock - 1) / kBlock, bn = blockIdx.x / blocks, bk = blockIdx.x % blocks;
    const int c = bk * kBlock + (t & 15) * 8, row0 = bn * kBlock + (t >> 4);
    Chunk<T> a[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = row0 + 16 * i;
        const T* p = w + row * w_stride + c;
        if (row < n) {
            if (c + 8 <= k) a[i].load(p);
            else if (c < k) load_tail(a[i], p, k - c);
        }
    }
    float y[8][8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[i][e] = a[i].get(e);
        m = umax(m, magnitude(y[i]));
    }
    m = max16(m);
    m = umax(m, (uint32_t)__shfl_xor((int)m, 16, 64));
    m = umax(m, (uint32_t)__shfl_xor((int)m, 32, 64));
    if ((t & 63) == 0) part[t >> 6] = m;
    __syncthreads();
    const float s = scale_of(umax(umax(part[0], part[1]), umax(part[2], part[3])));
    if (t == 0) scale[blockIdx.x] = s;
    if (c >= k) return;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (const int row = row0 + 16 * i; row < n) store_q(q + row * q_stride + c, y[i], inverse(s), k - c);
}

hipError_t launch_quantize_weights_fp8(const void* w, long long w_stride, int n, int k, bool bf16, uint8_t* q, long long q_stride, float* scale,
                                       hipStream_t stream)
{
    const long long blocks = (long long)((n + kBlock - 1) / kBlock) * ((k + kBlock - 1) / kBlock);
    if (bf16) hipLaunchKernelGGL(quantize_weights_kernel<uint16_t>, dim3((unsigned)blocks), dim3(256), 0, stream, (const uint16_t*)w, w_stride, n, k, q, q_stride, scale);
    else hipLaunchKernelGGL(quantize_weights_kernel<float>, dim3((unsigned)blocks), dim3(256), 0, stream, (const float*)w, w_stride, n, k, q, q_stride, scale);
    return hipGetLastError();
}

}  // namespace demon
