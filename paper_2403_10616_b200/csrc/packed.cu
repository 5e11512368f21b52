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

// The unit of 16 bytes that starts at p, of which the first n values belong to the matrix.  Rows may
// start at any element: the values are cut out of the aligned units that hold them, the second of which
// is read only where it holds one.
template <typename T> __device__ __forceinline__ uint4 load_unit(const T *p, int n, bool aligned)
{
    if (aligned) return *reinterpret_cast<const uint4 *>(p);
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    const unsigned s = (unsigned)(at & 15u);
    const uint4 *unit = reinterpret_cast<const uint4 *>(at - s);
    const uint4 lo = unit[0];
    uint4 hi = make_uint4(0u, 0u, 0u, 0u);
    if (s + n * sizeof(T) > 16u) hi = unit[1];
    return cut16(lo, hi, s);
}

// The first n values of a unit, the others zero.
template <typename T> __device__ __forceinline__ uint4 keep_first(uint4 v, int n)
{
    float f[Layout<T>::U];
    Unit<T>::widen(v, f);
#pragma unroll
    for (int i = 0; i < Layout<T>::U; ++i)
        if (i >= n) f[i] = 0.0f;
    return Unit<T>::narrow(f);  // exact
}

// The largest of the block's values, on every thread.
__device__ __forceinline__ unsigned block_max(unsigned m, unsigned *shared)
{
    m = __reduce_max_sync(0xffffffffu, m);
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = m;
    __syncthreads();
    return __reduce_max_sync(0xffffffffu, threadIdx.x % 32 < THREADS / 32 ? shared[threadIdx.x % 32] : 0u);
}

struct PackedOut {
    uint8_t *codes, *scales;
    long long stride;
};

// The thread's values of one matrix: as they were loaded, or computed in fp32.
template <typename T> struct LoadedValues {
    const uint4 *raw;
    __device__ __forceinline__ void unit(int j, float *f) const { Unit<T>::widen(raw[j], f); }
    // Bits of the largest magnitude; at least those of infinity if there is an infinity or NaN.
    __device__ __forceinline__ unsigned largest() const
    {
        unsigned m = 0u;
#pragma unroll
        for (int j = 0; j < Layout<T>::UNITS; ++j) {
            const unsigned w[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 2)
                    m = __vmaxu2(m, w[i] & 0x7fff7fffu);
                else
                    m = max(m, w[i] & 0x7fffffffu);
            }
        }
        return sizeof(T) == 2 ? max(m << 16, m & 0xffff0000u) : m;
    }
};
template <typename T> struct ComputedValues {
    const float *v;
    __device__ __forceinline__ void unit(int j, float *f) const
    {
#pragma unroll
        for (int i = 0; i < Layout<T>::U; ++i) f[i] = v[j * Layout<T>::U + i];
    }
    __device__ __forceinline__ unsigned largest() const  // of the values that are not NaN
    {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < VALUES; ++i) m = fmaxf(m, fabsf(v[i]));
        return __float_as_uint(m);
    }
};

template <int U, bool SPECIAL> __device__ __forceinline__ void store_codes(uint8_t *p, int n, const float *f, float reciprocal)
{
    unsigned w[U / 4];
#pragma unroll
    for (int i = 0; i < U / 4; ++i) w[i] = SPECIAL ? encode4(f + 4 * i, reciprocal) : encode4_finite(f + 4 * i, reciprocal);
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

// Writes the block's codes and scale.  Infinities and NaN are rare: where the largest magnitude is not
// finite, the block looks for the largest finite one and encodes with care for infinities.
template <typename T, typename Values>
__device__ __forceinline__ void write_block(const PackedOut &out, const Extent &x, int row0, int col, const Values &v,
                                            unsigned *shared)
{
    using L = Layout<T>;
    unsigned m = block_max(v.largest(), shared);
    const bool special = m >= 0x7f800000u;
    if (special) {
        m = 0u;
#pragma unroll
        for (int j = 0; j < L::UNITS; ++j) {
            float f[L::U];
            v.unit(j, f);
#pragma unroll
            for (int i = 0; i < L::U; ++i) m = max(m, finite_magnitude(f[i]));
        }
        m = block_max(m, shared + THREADS / 32);
    }
    const unsigned byte = scale_byte(m);
    const float reciprocal = scale_reciprocal(byte);
    if (threadIdx.x == 0) out.scales[blockIdx.x] = (uint8_t)byte;
    if (col >= x.cols) return;
    uint8_t *p = out.codes + (long long)row0 * out.stride + col;
#pragma unroll
    for (int j = 0; j < L::UNITS; ++j) {
        if (row0 + j * L::STEP < x.rows) {
            float f[L::U];
            v.unit(j, f);
            if (special)
                store_codes<L::U, true>(p, x.cols - col, f, reciprocal);
            else
                store_codes<L::U, false>(p, x.cols - col, f, reciprocal);
        }
        p += L::STEP * out.stride;
    }
}

// exp(-2u); 2u log2(e) = a (c1 + c3 a^2).  The approximations are good to two units in the last place.
__device__ __forceinline__ float gelu_decay(float a)
{
    constexpr float c1 = 2.0f * 0.7978845608028654f * 1.4426950408889634f;
    constexpr float c3 = c1 * 0.044715f;
    float d;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(-a * fmaf(c3, a * a, c1)));
    return d;
}
__device__ __forceinline__ float reciprocal_of(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
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
__global__ void __launch_bounds__(THREADS, 2) block_kernel(const __grid_constant__ BlockArgs a)
{
    using L = Layout<T>;
    constexpr int U = L::U;
    __shared__ unsigned shared[2][2 * THREADS / 32];
    const int rows = a.extent.rows, cols = a.extent.cols;
    const int row0 = (int)(blockIdx.x / a.extent.block_cols) * PACK_BLOCK + (int)threadIdx.x / L::PER_ROW;
    const int col = (int)(blockIdx.x % a.extent.block_cols) * PACK_BLOCK + (int)(threadIdx.x % L::PER_ROW) * U;
    const bool edge = (int)(blockIdx.x % a.extent.block_cols + 1) * PACK_BLOCK > cols ||
                      (int)(blockIdx.x / a.extent.block_cols + 1) * PACK_BLOCK > rows;  // the same for the whole block

    uint4 raw[L::UNITS];
    const T *x = static_cast<const T *>(a.x) + (long long)row0 * a.x_stride + col;
#pragma unroll
    for (int j = 0; j < L::UNITS; ++j) {
        if (!edge) {
            raw[j] = load_unit<T>(x, U, a.aligned);
        } else if (row0 + j * L::STEP < rows && col < cols) {
            raw[j] = keep_first<T>(load_unit<T>(x, cols - col, a.aligned), cols - col);
        } else {
            raw[j] = make_uint4(0u, 0u, 0u, 0u);
        }
        x += L::STEP * a.x_stride;
    }
    const LoadedValues<T> loaded = {raw};
    if constexpr (OP == OP_PACK) {
        write_block<T>(a.first, a.extent, row0, col, loaded, shared[0]);
        return;
    }

    float y[VALUES];
    if constexpr (OP == OP_NORM) {
        float gamma[U], beta[U];
#pragma unroll
        for (int i = 0; i < U; ++i) { gamma[i] = 1.0f; beta[i] = 0.0f; }
        if (a.gamma) load_params<U>(a.gamma, a.params_bf16, a.gamma_aligned, col, cols, gamma);
        if (a.beta) load_params<U>(a.beta, a.params_bf16, a.beta_aligned, col, cols, beta);
#pragma unroll
        for (int j = 0; j < L::UNITS; ++j) {
            const int r = row0 + j * L::STEP;
            const float mean = r < rows ? a.mean[r] : 0.0f, rstd = r < rows ? a.rstd[r] : 0.0f;
            float *f = y + j * U;
            loaded.unit(j, f);
#pragma unroll
            for (int i = 0; i < U; ++i) f[i] = fmaf((f[i] - mean) * rstd, gamma[i], beta[i]);
            if (edge) {
#pragma unroll
                for (int i = 0; i < U; ++i)
                    if (r >= rows || col + i >= cols) f[i] = 0.0f;
            }
        }
    } else if constexpr (OP == OP_GELU) {
#pragma unroll
        for (int j = 0; j < L::UNITS; ++j) {
            float *f = y + j * U;
            loaded.unit(j, f);
#pragma unroll
            for (int i = 0; i < U; ++i) f[i] *= reciprocal_of(1.0f + gelu_decay(f[i]));
        }
    } else {
        constexpr float k = 2.0f * 0.7978845608028654f;
        const float scale = scale_value(a.scales[blockIdx.x]);
        const uint8_t *q = a.codes + (long long)row0 * a.codes_stride + col;
#pragma unroll
        for (int j = 0; j < L::UNITS; ++j) {
            float *f = y + j * U;
            loaded.unit(j, f);
            const bool in = !edge || (row0 + j * L::STEP < rows && col < cols);
#pragma unroll
            for (int i = 0; i < U; i += 4) {
                float v[4];
                // rows of codes are padded to 16 bytes: four of them can be read wherever one can
                decode4(in && (!edge || col + i < cols) ? *reinterpret_cast<const unsigned *>(q + i) : 0u, scale, v);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    // s (1 - s) = d s^2 with d = exp(-2u): no cancellation where s is near 1
                    const float decay = gelu_decay(v[t]), d = decay > 3e38f ? 3e38f : decay;
                    const float s = reciprocal_of(1.0f + d), w = d * s * s;
                    // w is zero before its factors overflow (a code times its scale may itself exceed
                    // the largest fp32 value)
                    const float bend = w == 0.0f ? 0.0f : v[t] * w * fmaf(3.0f * 0.044715f * k, v[t] * v[t], k);
                    f[i + t] *= s + bend;
                }
            }
            if (edge) {
#pragma unroll
                for (int i = 0; i < U; ++i)
                    if (col + i >= cols) f[i] = 0.0f;
            }
            q += L::STEP * a.codes_stride;
        }
    }
    const ComputedValues<T> computed = {y};
    write_block<T>(a.first, a.extent, row0, col, computed, shared[0]);
    if (OP != OP_GELU_BACK && a.second.codes) write_block<T>(a.second, a.extent, row0, col, loaded, shared[1]);
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
