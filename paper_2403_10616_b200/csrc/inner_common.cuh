// Shared by the operators of the inner phase (layer_norm.cu, packed.cu, packed_matmul.cu): argument
// checks, loads at any element alignment, and the 8-bit block format.
//
// Packed matrix: e4m3 codes, one e8m0 scale 2^e per block of 128 x 128 values, e the least exponent
// with max|x| <= 448 * 2^e over the block's finite values (448: the largest e4m3 value).
#pragma once

#include "../../include/dipaco.h"

#include <cuda.h>
#include <cuda_fp8.h>

#include "kernels.cuh"

namespace dipaco {

constexpr int PACK_BLOCK = 128;
constexpr int64_t MAX_EXTENT = (int64_t)INT32_MAX - 65536;  // rows or columns: steps beyond the last fit an int

// ------------------------------------------------------------------------------------------ host

struct DeviceScope {
    int prev = -1;
    bool ok = true;
    explicit DeviceScope(int dev)
    {
        if (cudaGetDevice(&prev) != cudaSuccess) { cudaGetLastError(); ok = false; prev = -1; return; }
        if (prev == dev) { prev = -1; return; }
        if (cudaSetDevice(dev) != cudaSuccess) { cudaGetLastError(); ok = false; }
    }
    ~DeviceScope()
    {
        if (prev >= 0) cudaSetDevice(prev);
    }
};

inline bool is_dense_dtype(int dtype) { return dtype == DIPACO_F32 || dtype == DIPACO_BF16; }
inline int dense_size(int dtype) { return dtype == DIPACO_BF16 ? 2 : 4; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline int check_extents(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0) return DIPACO_EINVAL;
    return rows > MAX_EXTENT || cols > MAX_EXTENT ? DIPACO_ELIMIT : DIPACO_OK;
}

// A dense matrix argument: elements at their own alignment, rows that do not overlap.
inline bool dense_ok(const void *p, int64_t stride, int64_t rows, int64_t cols, int dtype)
{
    if (rows == 0 || cols == 0) return true;
    return p && (uintptr_t)p % dense_size(dtype) == 0 && (stride >= cols || rows == 1) && stride >= 0;
}

// A vector argument (gamma, mean, ...); NULL where the entry point allows it is checked there.
inline bool vector_ok(const void *p, int size) { return (uintptr_t)p % size == 0; }

// A packed matrix argument of the given extents.
inline bool packed_ok(const dipaco_packed *p, int64_t rows, int64_t cols)
{
    if (!p || p->rows != rows || p->cols != cols) return false;
    if (rows == 0 || cols == 0) return true;
    return p->codes && p->scales && (uintptr_t)p->codes % 16 == 0 && p->stride >= cols && p->stride % 16 == 0;
}

inline bool rows_aligned16(const void *p, int64_t stride, int64_t rows, int size)
{
    return (uintptr_t)p % 16 == 0 && (rows == 1 || stride * size % 16 == 0);
}

inline int launch_status()
{
    const cudaError_t err = cudaGetLastError();
    return err == cudaSuccess ? DIPACO_OK : err == cudaErrorMemoryAllocation ? DIPACO_ENOMEM : DIPACO_ECUDA;
}

// Tensor maps are encoded by the driver, whose entry point is looked up once.
using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                 const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiled encode_tiled()
{
    static const EncodeTiled fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

// A word that kernels set when a bounded wait runs out: reads and clears it.  False: a CUDA call failed.
template <typename Symbol> bool take_error_word(const Symbol &symbol, bool &expired)
{
    int word = 0;
    if (cudaMemcpyFromSymbol(&word, symbol, sizeof(int)) != cudaSuccess) return false;
    if (word == 0) return true;
    expired = true;
    word = 0;
    return cudaMemcpyToSymbol(symbol, &word, sizeof(int)) == cudaSuccess;
}
bool take_packing_error(bool &expired);  // of packed.cu
bool take_norm_error(bool &expired);     // of layer_norm.cu
bool take_linear_error(bool &expired);   // of packed_linear.cu
bool take_residual_norm_error(bool &expired);  // of residual_norm.cu

// The norm of rows whose statistics are known, and unless x_packed is NULL the rows themselves, packed (of packed.cu):
// checked arguments, the device current, values to work on.
int pack_normalised(const void *x, int64_t x_stride, int dtype, const float *mean, const float *rstd, const void *gamma,
                    const void *beta, int param_dtype, const dipaco_packed *y, const dipaco_packed *x_packed,
                    cudaStream_t stream);

// The activation of dense fp32 rows, and unless x_packed is NULL the rows themselves, packed (of packed.cu): as above.
int pack_activated(const float *x, int64_t x_stride, int activation, const dipaco_packed *y, const dipaco_packed *x_packed,
                   cudaStream_t stream);

// Launches of a warp whose wait runs out (dipaco_selftest_inner_wait_expiry).
int expire_packing_wait(unsigned long long limit_ns, cudaStream_t stream);
int expire_norm_wait(unsigned long long limit_ns, cudaStream_t stream);
int expire_linear_wait(unsigned long long limit_ns, cudaStream_t stream);
int expire_residual_norm_wait(unsigned long long limit_ns, cudaStream_t stream);

// ------------------------------------------------------------------------------------------ device

// True on one thread of the warp.  Asynchronous copies and products are issued under it: the compiler
// then keeps their operands in uniform registers, which it does not under a test of the lane.
__device__ __forceinline__ bool elect_one()
{
    unsigned ok;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok));
    return ok != 0;
}

// Two fp32 values in one register pair: additions and products take one issue slot for both.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pair_of(float lo, float hi)
{
    f32x2 p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(lo), "f"(hi));
    return p;
}
__device__ __forceinline__ f32x2 pair_of(float both) { return pair_of(both, both); }
__device__ __forceinline__ float2 values_of(f32x2 p)
{
    float2 v;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(p));
    return v;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float sum_of(f32x2 p)
{
    const float2 v = values_of(p);
    return v.x + v.y;
}
// 16 bytes to pairs, and pairs to 16 bytes (rounded).
template <typename T> __device__ __forceinline__ void widen_pairs(const uint4 &v, f32x2 *p)
{
    float f[Unit<T>::UE];
    Unit<T>::widen(v, f);
#pragma unroll
    for (int i = 0; i < Unit<T>::UE / 2; ++i) p[i] = pair_of(f[2 * i], f[2 * i + 1]);
}
template <typename T> __device__ __forceinline__ uint4 narrow_pairs(const f32x2 *p)
{
    float f[Unit<T>::UE];
#pragma unroll
    for (int i = 0; i < Unit<T>::UE / 2; ++i) {
        const float2 v = values_of(p[i]);
        f[2 * i] = v.x;
        f[2 * i + 1] = v.y;
    }
    return Unit<T>::narrow(f);
}

// The first n of a unit's values, the others zero.
template <int U> __device__ __forceinline__ void keep_inside(f32x2 *p, int n)
{
#pragma unroll
    for (int i = 0; i < U / 2; ++i) {
        const float2 v = values_of(p[i]);
        p[i] = pair_of(2 * i < n ? v.x : 0.0f, 2 * i + 1 < n ? v.y : 0.0f);
    }
}

// The value of an e8m0 byte: 2^(b-127), which bf16 holds; 255 is NaN.
__device__ __forceinline__ float scale_value(unsigned b)
{
    unsigned r;
    asm("cvt.rn.bf16x2.ue8m0x2 %0, %1;" : "=r"(r) : "h"((unsigned short)b));
    return __uint_as_float(r << 16);
}

// Magnitude bits that take part in a block's maximum: those of infinities and NaN do not.
__device__ __forceinline__ unsigned finite_magnitude(float x)
{
    const unsigned m = __float_as_uint(x) & 0x7fffffffu;
    return m < 0x7f800000u ? m : 0u;
}

// The e8m0 byte for a block whose largest finite magnitude has the bits m.  448 = 1.75 * 2^8, so the
// exponent is that of m less 8, one more where m's significand is over 1.75.  The byte is at least 1
// (2^-126), which keeps both the scale and its reciprocal normal; a block of zeros gets 127 (1.0).
__device__ __forceinline__ unsigned scale_byte(unsigned m)
{
    if (m == 0u) return 127u;
    const int e = (int)(m >> 23) - 8 + ((m & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (unsigned)max(e, 1);
}
__device__ __forceinline__ float scale_reciprocal(unsigned byte) { return __uint_as_float((254u - byte) << 23); }

// Two codes (x in the low byte).  y + 0*y turns an infinity into NaN and leaves every other value as
// it is: the conversion would saturate an infinity to 448.
__device__ __forceinline__ unsigned encode2(float x, float y, float reciprocal)
{
    x *= reciprocal;
    y *= reciprocal;
    const float2 v = make_float2(__fmaf_rn(x, 0.0f, x), __fmaf_rn(y, 0.0f, y));
    return __nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ unsigned encode4(const float *f, float reciprocal)
{
    return encode2(f[0], f[1], reciprocal) | (encode2(f[2], f[3], reciprocal) << 16);
}
// The same where no value is infinite.
__device__ __forceinline__ unsigned encode4_finite(const f32x2 *p, f32x2 reciprocal)
{
    const unsigned lo = __nv_cvt_float2_to_fp8x2(values_of(mul2(p[0], reciprocal)), __NV_SATFINITE, __NV_E4M3);
    const unsigned hi = __nv_cvt_float2_to_fp8x2(values_of(mul2(p[1], reciprocal)), __NV_SATFINITE, __NV_E4M3);
    return __byte_perm(lo, hi, 0x5410);
}
__device__ __forceinline__ float2 decode2(unsigned codes)
{
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)codes, __NV_E4M3);
    return __half22float2(__half2(h));
}
__device__ __forceinline__ f32x2 decode_pair(unsigned codes)
{
    const float2 v = decode2(codes & 0xffffu);
    return pair_of(v.x, v.y);
}
__device__ __forceinline__ void decode4(unsigned codes, float scale, float *f)
{
    const float2 a = decode2(codes & 0xffffu), b = decode2(codes >> 16);
    f[0] = a.x * scale; f[1] = a.y * scale; f[2] = b.x * scale; f[3] = b.y * scale;
}

template <typename T> __device__ __forceinline__ float widen1(T v);
template <> __device__ __forceinline__ float widen1<float>(float v) { return v; }
template <> __device__ __forceinline__ float widen1<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T narrow1(float v);
template <> __device__ __forceinline__ float narrow1<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 narrow1<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ float load_param(const void *p, bool bf16, int64_t i)
{
    return bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]) : static_cast<const float *>(p)[i];
}

// U consecutive parameters from column c (U a multiple of 4), those from `cols` on as zero.
template <int U>
__device__ __forceinline__ void load_params(const void *p, bool bf16, bool aligned, int c, int cols, float *f)
{
    if (aligned && c + U <= cols) {
        if (bf16) {
            const uint2 *q = reinterpret_cast<const uint2 *>(static_cast<const __nv_bfloat16 *>(p) + c);
#pragma unroll
            for (int i = 0; i < U / 4; ++i) {
                const uint2 v = __ldg(q + i);
                f[4 * i] = __uint_as_float(v.x << 16);
                f[4 * i + 1] = __uint_as_float(v.x & 0xffff0000u);
                f[4 * i + 2] = __uint_as_float(v.y << 16);
                f[4 * i + 3] = __uint_as_float(v.y & 0xffff0000u);
            }
        } else {
            const float4 *q = reinterpret_cast<const float4 *>(static_cast<const float *>(p) + c);
#pragma unroll
            for (int i = 0; i < U / 4; ++i) {
                const float4 v = __ldg(q + i);
                f[4 * i] = v.x; f[4 * i + 1] = v.y; f[4 * i + 2] = v.z; f[4 * i + 3] = v.w;
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < U; ++i) f[i] = c + i < cols ? load_param(p, bf16, c + i) : 0.0f;
}

template <int U>
__device__ __forceinline__ void param_pairs(const void *p, bool bf16, bool aligned, int c, int cols, f32x2 *pairs)
{
    float f[U];
    load_params<U>(p, bf16, aligned, c, cols, f);
#pragma unroll
    for (int i = 0; i < U / 2; ++i) pairs[i] = pair_of(f[2 * i], f[2 * i + 1]);
}

} // namespace dipaco
