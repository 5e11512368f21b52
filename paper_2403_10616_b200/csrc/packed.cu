// Packed matrices: conversion from and to dense ones, the layer norm and the GELU that write their
// result and their input as packed checkpoints, and the GELU's gradient from such a checkpoint (see
// include/dipaco.h for the format).
//
//   gelu(a) = a s, s = 1 / (1 + exp(-2u)), u = sqrt(2/pi) (a + 0.044715 a^3)   (the tanh form: 2s = 1 + tanh u)
//   gelu'(a) = s + a s (1 - s) 2 u',  u' = sqrt(2/pi) (1 + 3 * 0.044715 a^2)
//
// One block of threads per block of 128 x 128 values: the values are read once and stay in registers
// while the block's largest magnitude is found.
#include "inner_common.cuh"

#include <cmath>

using namespace dipaco;

namespace {

constexpr int THREADS = 512;
constexpr int VALUES = PACK_BLOCK * PACK_BLOCK / THREADS;  // of one thread

// Where a thread's values lie: U consecutive columns in every STEP-th row of the block.
template <typename T> struct Layout {
    static constexpr int U = 16 / (int)sizeof(T);
    static constexpr int PER_ROW = PACK_BLOCK / U;
    static constexpr int STEP = THREADS / PER_ROW;
    static constexpr int UNITS = VALUES / U;
};

struct Extent {
    int rows, cols, block_cols;
};

// U values of a row from column c, those from `cols` on as zero.  Rows may start at any element.
template <typename T>
__device__ __forceinline__ void load_unit(const T *row, int c, int cols, bool aligned, float *f)
{
    constexpr int U = Layout<T>::U;
    const int n = min(cols - c, U);
    if (aligned) {
        Unit<T>::widen(__ldcs(reinterpret_cast<const uint4 *>(row + c)), f);
    } else {
        // the aligned 16-byte units that hold the values, the second only where it holds one
        const uintptr_t at = reinterpret_cast<uintptr_t>(row + c);
        const unsigned s = (unsigned)(at & 15u);
        const uint4 *unit = reinterpret_cast<const uint4 *>(at - s);
        const uint4 lo = unit[0];
        uint4 hi = make_uint4(0u, 0u, 0u, 0u);
        if (s + n * sizeof(T) > 16u) hi = unit[1];
        Unit<T>::widen(cut16(lo, hi, s), f);
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
        if (i >= n) f[i] = 0.0f;
}

template <int U> __device__ __forceinline__ void store_codes(uint8_t *p, int n, const float *f, float reciprocal)
{
    unsigned w[U / 4];
#pragma unroll
    for (int i = 0; i < U / 4; ++i) w[i] = encode4(f + 4 * i, reciprocal);
    if (n >= U) {
        if constexpr (U == 8)
            *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
        else
            *reinterpret_cast<unsigned *>(p) = w[0];
    } else {
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (i < n) p[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
    }
}

// The largest of the block's values, on every thread.
__device__ __forceinline__ unsigned block_max(unsigned m, unsigned *shared)
{
    m = __reduce_max_sync(0xffffffffu, m);
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = m;
    __syncthreads();
    return __reduce_max_sync(0xffffffffu, threadIdx.x % 32 < THREADS / 32 ? shared[threadIdx.x % 32] : 0u);
}

template <int N> __device__ __forceinline__ unsigned largest(const float *v)
{
    unsigned m = 0u;
#pragma unroll
    for (int i = 0; i < N; ++i) m = max(m, finite_magnitude(v[i]));
    return m;
}

struct PackedOut {
    uint8_t *codes, *scales;
    long long stride;
};

// Writes the thread's values v, whose block has the largest magnitude m.
template <typename T>
__device__ __forceinline__ void write_block(const PackedOut &out, const Extent &x, int row0, int col, int rows_from,
                                            const float *v, unsigned m)
{
    constexpr int U = Layout<T>::U;
    const unsigned byte = scale_byte(m);
    const float reciprocal = scale_reciprocal(byte);
    if (threadIdx.x == 0) out.scales[blockIdx.x] = (uint8_t)byte;
#pragma unroll
    for (int j = 0; j < Layout<T>::UNITS; ++j) {
        const long long r = (long long)row0 + rows_from + j * Layout<T>::STEP;
        if (r < x.rows && col < x.cols)
            store_codes<U>(out.codes + r * out.stride + col, x.cols - col, v + j * U, reciprocal);
    }
}

// exp(-2u); 2u log2(e) = a (c1 + c3 a^2)
__device__ __forceinline__ float gelu_decay(float a)
{
    constexpr float c1 = 2.0f * 0.7978845608028654f * 1.4426950408889634f;
    constexpr float c3 = c1 * 0.044715f;
    return exp2f(-a * fmaf(c3, a * a, c1));
}

enum : int { OP_PACK, OP_NORM, OP_GELU, OP_GELU_BACK };

struct BlockArgs {
    const void *x;  // dense input (the gradient for OP_GELU_BACK)
    long long x_stride;
    bool aligned;
    Extent extent;
    PackedOut first;   // the packed result
    PackedOut second;  // the packed input (OP_NORM, OP_GELU); codes NULL: not wanted
    // OP_GELU_BACK: the packed input of the GELU
    const uint8_t *codes, *scales;
    long long codes_stride;
    // OP_NORM
    const float *mean, *rstd;
    const void *gamma, *beta;
    bool params_bf16, gamma_aligned, beta_aligned;
};

template <typename T, int OP>
__global__ void __launch_bounds__(THREADS) block_kernel(BlockArgs a)
{
    using L = Layout<T>;
    constexpr int U = L::U;
    __shared__ unsigned shared[2][THREADS / 32];
    const int row0 = (int)(blockIdx.x / a.extent.block_cols) * PACK_BLOCK;
    const int col = (int)(blockIdx.x % a.extent.block_cols) * PACK_BLOCK + (int)(threadIdx.x % L::PER_ROW) * U;
    const int rows_from = threadIdx.x / L::PER_ROW;

    float x[VALUES], y[OP == OP_PACK ? 1 : VALUES];
#pragma unroll
    for (int j = 0; j < L::UNITS; ++j) {
        const long long r = (long long)row0 + rows_from + j * L::STEP;
        if (r < a.extent.rows && col < a.extent.cols) {
            load_unit<T>(static_cast<const T *>(a.x) + r * a.x_stride, col, a.extent.cols, a.aligned, x + j * U);
        } else {
#pragma unroll
            for (int i = 0; i < U; ++i) x[j * U + i] = 0.0f;
        }
    }
    if constexpr (OP == OP_NORM) {
        float gamma[U], beta[U];
#pragma unroll
        for (int i = 0; i < U; ++i) { gamma[i] = 1.0f; beta[i] = 0.0f; }
        if (a.gamma) load_params<U>(a.gamma, a.params_bf16, a.gamma_aligned, col, a.extent.cols, gamma);
        if (a.beta) load_params<U>(a.beta, a.params_bf16, a.beta_aligned, col, a.extent.cols, beta);
#pragma unroll
        for (int j = 0; j < L::UNITS; ++j) {
            const long long r = (long long)row0 + rows_from + j * L::STEP;
            const bool in = r < a.extent.rows;
            const float mean = in ? a.mean[r] : 0.0f, rstd = in ? a.rstd[r] : 0.0f;
#pragma unroll
            for (int i = 0; i < U; ++i)
                y[j * U + i] = in && col + i < a.extent.cols
                                   ? (x[j * U + i] - mean) * rstd * gamma[i] + beta[i]
                                   : 0.0f;
        }
    } else if constexpr (OP == OP_GELU) {
#pragma unroll
        for (int e = 0; e < VALUES; ++e) y[e] = x[e] * __fdividef(1.0f, 1.0f + gelu_decay(x[e]));
    } else if constexpr (OP == OP_GELU_BACK) {
        constexpr float k = 2.0f * 0.7978845608028654f;
#pragma unroll
        for (int j = 0; j < L::UNITS; ++j) {
            const long long r = (long long)row0 + rows_from + j * L::STEP;
            const float scale = scale_value(a.scales[blockIdx.x]);
            const bool in = r < a.extent.rows && col < a.extent.cols;
            const uint8_t *q = a.codes + r * a.codes_stride + col;
#pragma unroll
            for (int i = 0; i < U; i += 4) {
                float v[4];
                // rows of codes are padded to 16 bytes: four of them can be read wherever one can
                decode4(in && col + i < a.extent.cols ? *reinterpret_cast<const unsigned *>(q + i) : 0u, scale, v);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const int e = j * U + i + t;
                    // s (1 - s) = d s^2 with d = exp(-2u): no cancellation where s is near 1
                    const float decay = gelu_decay(v[t]), d = decay > 3e38f ? 3e38f : decay;
                    const float s = __fdividef(1.0f, 1.0f + d), w = d * s * s;
                    // w is zero before its factors overflow (a code times its scale may itself exceed
                    // the largest fp32 value)
                    const float bend = w == 0.0f ? 0.0f : v[t] * w * fmaf(3.0f * 0.044715f * k, v[t] * v[t], k);
                    const float slope = s + bend;
                    y[e] = col + i + t < a.extent.cols ? x[e] * slope : 0.0f;
                }
            }
        }
    }

    if constexpr (OP == OP_PACK) {
        write_block<T>(a.first, a.extent, row0, col, rows_from, x, block_max(largest<VALUES>(x), shared[0]));
    } else {
        const unsigned m = block_max(largest<VALUES>(y), shared[0]);
        write_block<T>(a.first, a.extent, row0, col, rows_from, y, m);
        if (OP != OP_GELU_BACK && a.second.codes)
            write_block<T>(a.second, a.extent, row0, col, rows_from, x, block_max(largest<VALUES>(x), shared[1]));
    }
}

// Four codes per thread.
template <typename T>
__global__ void __launch_bounds__(256) unpack_kernel(const uint8_t *codes, long long codes_stride,
                                                     const uint8_t *scales, T *y, long long y_stride, int rows,
                                                     int cols, bool aligned)
{
    const long long per_row = (cols + 3) / 4, scale_cols = (cols + PACK_BLOCK - 1) / PACK_BLOCK;
    const long long step = (long long)gridDim.x * blockDim.x;
    for (long long u = (long long)blockIdx.x * blockDim.x + threadIdx.x; u < per_row * rows; u += step) {
        const long long r = u / per_row;
        const int c = (int)(u - r * per_row) * 4;
        float f[4];
        decode4(*reinterpret_cast<const unsigned *>(codes + r * codes_stride + c),
                scale_value(scales[r / PACK_BLOCK * scale_cols + c / PACK_BLOCK]), f);
        T *p = y + r * y_stride + c;
        if (aligned && c + 4 <= cols) {
            if constexpr (sizeof(T) == 4)
                *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
            else
                *reinterpret_cast<uint2 *>(p) = make_uint2(Unit<T>::pack(f[0], f[1]), Unit<T>::pack(f[2], f[3]));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + i < cols) p[i] = narrow1<T>(f[i]);
        }
    }
}

PackedOut packed_out(const dipaco_packed *p)
{
    if (!p) return {nullptr, nullptr, 0};
    return {static_cast<uint8_t *>(p->codes), static_cast<uint8_t *>(p->scales), p->stride};
}

template <int OP>
int launch_blocks(BlockArgs a, int dtype, int64_t rows, int64_t cols, cudaStream_t stream)
{
    const int64_t block_cols = ceil_div(cols, PACK_BLOCK), blocks = ceil_div(rows, PACK_BLOCK) * block_cols;
    if (blocks > INT32_MAX) return DIPACO_ELIMIT;
    a.extent = {(int)rows, (int)cols, (int)block_cols};
    a.aligned = rows_aligned16(a.x, a.x_stride, rows, dense_size(dtype));
    if (dtype == DIPACO_BF16)
        block_kernel<__nv_bfloat16, OP><<<(unsigned)blocks, THREADS, 0, stream>>>(a);
    else
        block_kernel<float, OP><<<(unsigned)blocks, THREADS, 0, stream>>>(a);
    return launch_status();
}

int check_dense(const void *x, int64_t stride, int64_t rows, int64_t cols, int dtype, int device)
{
    if (!is_dense_dtype(dtype) || device < 0) return DIPACO_EINVAL;
    if (const int rc = check_extents(rows, cols)) return rc;
    return dense_ok(x, stride, rows, cols, dtype) ? DIPACO_OK : DIPACO_EINVAL;
}

} // namespace

extern "C" {

int dipaco_pack(const void *x, int64_t x_stride, int32_t dtype, const dipaco_packed *out, int32_t device,
                void *cuda_stream)
{
    if (!out) return DIPACO_EINVAL;
    const int64_t rows = out->rows, cols = out->cols;
    if (const int rc = check_dense(x, x_stride, rows, cols, dtype, device)) return rc;
    if (!packed_ok(out, rows, cols)) return DIPACO_EINVAL;
    if (rows == 0 || cols == 0) return DIPACO_OK;
    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    BlockArgs a = {};
    a.x = x;
    a.x_stride = x_stride;
    a.first = packed_out(out);
    return launch_blocks<OP_PACK>(a, dtype, rows, cols, static_cast<cudaStream_t>(cuda_stream));
}

int dipaco_unpack(const dipaco_packed *x, void *y, int64_t y_stride, int32_t dtype, int32_t device,
                  void *cuda_stream)
{
    if (!x) return DIPACO_EINVAL;
    const int64_t rows = x->rows, cols = x->cols;
    if (const int rc = check_dense(y, y_stride, rows, cols, dtype, device)) return rc;
    if (!packed_ok(x, rows, cols)) return DIPACO_EINVAL;
    if (rows == 0 || cols == 0) return DIPACO_OK;
    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(ceil_div(cols, 4) * rows, 256), 148 * 32);
    const bool aligned = rows_aligned16(y, y_stride, rows, dense_size(dtype));
    const uint8_t *codes = static_cast<const uint8_t *>(x->codes), *scales = static_cast<const uint8_t *>(x->scales);
    if (dtype == DIPACO_BF16)
        unpack_kernel<__nv_bfloat16><<<grid, 256, 0, stream>>>(codes, x->stride, scales,
                                                               static_cast<__nv_bfloat16 *>(y), y_stride,
                                                               (int)rows, (int)cols, aligned);
    else
        unpack_kernel<float><<<grid, 256, 0, stream>>>(codes, x->stride, scales, static_cast<float *>(y), y_stride,
                                                       (int)rows, (int)cols, aligned);
    return launch_status();
}

int dipaco_layer_norm_pack(const void *x, int64_t x_stride, const void *gamma, const void *beta,
                           const dipaco_packed *y, const dipaco_packed *x_packed, float *mean, float *rstd,
                           float eps, int32_t dtype, int32_t param_dtype, int32_t device, void *cuda_stream)
{
    if (!y) return DIPACO_EINVAL;
    const int64_t rows = y->rows, cols = y->cols;
    if (const int rc = check_dense(x, x_stride, rows, cols, dtype, device)) return rc;
    if (!is_dense_dtype(param_dtype) || !(eps >= 0.0f) || !std::isfinite(eps)) return DIPACO_EINVAL;
    if (!packed_ok(y, rows, cols) || (x_packed && !packed_ok(x_packed, rows, cols))) return DIPACO_EINVAL;
    const int psize = dense_size(param_dtype);
    if (!vector_ok(gamma, psize) || !vector_ok(beta, psize) || !vector_ok(mean, 4) || !vector_ok(rstd, 4))
        return DIPACO_EINVAL;
    if (rows == 0 || cols == 0) return DIPACO_OK;
    if (!mean || !rstd) return DIPACO_EINVAL;
    if (const int rc = dipaco_layer_norm(x, x_stride, nullptr, nullptr, nullptr, 0, mean, rstd, rows, cols, eps,
                                         dtype, param_dtype, device, cuda_stream))
        return rc;
    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    BlockArgs a = {};
    a.x = x;
    a.x_stride = x_stride;
    a.first = packed_out(y);
    a.second = packed_out(x_packed);
    a.mean = mean;
    a.rstd = rstd;
    a.gamma = gamma;
    a.beta = beta;
    a.params_bf16 = param_dtype == DIPACO_BF16;
    a.gamma_aligned = (uintptr_t)gamma % 16 == 0;
    a.beta_aligned = (uintptr_t)beta % 16 == 0;
    return launch_blocks<OP_NORM>(a, dtype, rows, cols, static_cast<cudaStream_t>(cuda_stream));
}

int dipaco_gelu_pack(const void *x, int64_t x_stride, int32_t dtype, const dipaco_packed *y,
                     const dipaco_packed *x_packed, int32_t device, void *cuda_stream)
{
    if (!y) return DIPACO_EINVAL;
    const int64_t rows = y->rows, cols = y->cols;
    if (const int rc = check_dense(x, x_stride, rows, cols, dtype, device)) return rc;
    if (!packed_ok(y, rows, cols) || (x_packed && !packed_ok(x_packed, rows, cols))) return DIPACO_EINVAL;
    if (rows == 0 || cols == 0) return DIPACO_OK;
    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    BlockArgs a = {};
    a.x = x;
    a.x_stride = x_stride;
    a.first = packed_out(y);
    a.second = packed_out(x_packed);
    return launch_blocks<OP_GELU>(a, dtype, rows, cols, static_cast<cudaStream_t>(cuda_stream));
}

int dipaco_gelu_pack_backward(const void *dy, int64_t dy_stride, int32_t dtype, const dipaco_packed *x_packed,
                              const dipaco_packed *dx, int32_t device, void *cuda_stream)
{
    if (!dx || !x_packed) return DIPACO_EINVAL;
    const int64_t rows = dx->rows, cols = dx->cols;
    if (const int rc = check_dense(dy, dy_stride, rows, cols, dtype, device)) return rc;
    if (!packed_ok(dx, rows, cols) || !packed_ok(x_packed, rows, cols)) return DIPACO_EINVAL;
    if (rows == 0 || cols == 0) return DIPACO_OK;
    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    BlockArgs a = {};
    a.x = dy;
    a.x_stride = dy_stride;
    a.first = packed_out(dx);
    a.codes = static_cast<const uint8_t *>(x_packed->codes);
    a.scales = static_cast<const uint8_t *>(x_packed->scales);
    a.codes_stride = x_packed->stride;
    return launch_blocks<OP_GELU_BACK>(a, dtype, rows, cols, static_cast<cudaStream_t>(cuda_stream));
}

} // extern "C"
