// Layer norm of the rows of a matrix, forward and backward (see include/dipaco.h).
//
//   mean = sum x / C, var = sum (x - mean)^2 / C, rstd = (var + eps)^-1/2, y = (x - mean) rstd gamma + beta
//   g = dy gamma, h = (x - mean) rstd, dx = rstd (g - mean(g) - h mean(g h)), dgamma = sum dy h, dbeta = sum dy
//
// All sums are fp32.  The variance is summed from the centred values of the row, which is held in
// registers, so it does not cancel for rows whose mean is large beside their spread.
#include "inner_common.cuh"

#include <cmath>

using namespace dipaco;

namespace {

// ------------------------------------------------------------------------------------------ sums over a row

// Sum over the TPR threads of a row.  Rows of up to 32 threads lie inside a warp; of wider ones every
// thread of the block takes part, and `shared` (one slot per warp) is used once.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *shared)
{
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (TPR > 32) {
        constexpr int WARPS = TPR / 32;
        const int warp = threadIdx.x >> 5;
        if ((threadIdx.x & 31) == 0) shared[warp] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) v += shared[warp / WARPS * WARPS + w];
    }
    return v;
}

// ------------------------------------------------------------------------------------------ forward

struct NormArgs {
    const void *x;
    void *y;  // NULL: statistics only
    const void *gamma, *beta;
    float *mean, *rstd;
    long long x_stride, y_stride;
    int rows, cols;
    float eps;
    bool params_bf16, gamma_aligned, beta_aligned;
};

// One row per TPR threads, the row in registers: NU units of 16 bytes per thread (VEC: rows on 16-byte
// boundaries), or as many single values.  Bound by memory: about nine instructions per value, and enough
// rows in flight with a warp per row up to 2048 values in bf16 (1024 in fp32); wider rows take a block.
template <typename T, bool VEC, int TPR, int NU>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) norm_rows_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int U = VEC ? 16 / (int)sizeof(T) : 1;
    constexpr int E = NU * 16 / (int)sizeof(T);
    constexpr int UNITS = E / U;
    __shared__ float shared[2][32];
    const int lane = threadIdx.x % TPR;
    const int row = blockIdx.x * (blockDim.x / TPR) + threadIdx.x / TPR;
    const bool live = row < a.rows;
    const int cols = live ? a.cols : 0;
    const T *x = static_cast<const T *>(a.x) + (live ? row : 0) * a.x_stride;

    float v[E];
    float sum = 0.0f;
    if constexpr (VEC) {
        uint4 raw[UNITS];
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            const int c = (j * TPR + lane) * U;
            raw[j] = c < cols ? *reinterpret_cast<const uint4 *>(x + c) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            const int c = (j * TPR + lane) * U;
            Unit<T>::widen(raw[j], v + j * U);
            if (c < cols && c + U > cols) {
#pragma unroll
                for (int i = 0; i < U; ++i)
                    if (c + i >= cols) v[j * U + i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < U; ++i) sum += v[j * U + i];
        }
    } else {
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            const int c = j * TPR + lane;
            v[j] = c < cols ? widen1<T>(x[c]) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < UNITS; ++j) sum += v[j];
    }
    const float mean = row_sum<TPR>(sum, shared[0]) / (float)a.cols;
    sum = 0.0f;
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        const int c = (j * TPR + lane) * U;
        if (c < cols) {
#pragma unroll
            for (int i = 0; i < U; ++i) v[j * U + i] -= mean;
            if (VEC && c + U > cols) {
#pragma unroll
                for (int i = 0; i < U; ++i)
                    if (c + i >= cols) v[j * U + i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < U; ++i) sum = fmaf(v[j * U + i], v[j * U + i], sum);
        }
    }
    const float rstd = 1.0f / sqrtf(row_sum<TPR>(sum, shared[1]) / (float)a.cols + a.eps);
    if (!live) return;
    if (lane == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    if (!a.y) return;
    T *y = static_cast<T *>(a.y) + row * a.y_stride;
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        const int c = (j * TPR + lane) * U;
        if (c >= cols) continue;
        float *r = v + j * U;
#pragma unroll
        for (int i = 0; i < U; ++i) r[i] *= rstd;
        if constexpr (VEC) {
            float p[U];
            if (a.gamma) {
                load_params<U>(a.gamma, a.params_bf16, a.gamma_aligned, c, cols, p);
#pragma unroll
                for (int i = 0; i < U; ++i) r[i] *= p[i];
            }
            if (a.beta) {
                load_params<U>(a.beta, a.params_bf16, a.beta_aligned, c, cols, p);
#pragma unroll
                for (int i = 0; i < U; ++i) r[i] += p[i];
            }
            if (c + U <= cols) {
                *reinterpret_cast<uint4 *>(y + c) = Unit<T>::narrow(r);
            } else {
#pragma unroll
                for (int i = 0; i < U; ++i)
                    if (c + i < cols) y[c + i] = narrow1<T>(r[i]);
            }
        } else {
            if (a.gamma) r[0] *= load_param(a.gamma, a.params_bf16, c);
            if (a.beta) r[0] += load_param(a.beta, a.params_bf16, c);
            y[c] = narrow1<T>(r[0]);
        }
    }
}

// Rows that do not fit a block's registers: one block per row, which reads the row three times.
template <typename T>
__global__ void __launch_bounds__(1024) norm_long_rows_kernel(NormArgs a)
{
    __shared__ float shared[2][32];
    const T *x = static_cast<const T *>(a.x) + (long long)blockIdx.x * a.x_stride;
    float sum = 0.0f;
    for (long long c = threadIdx.x; c < a.cols; c += 1024) sum += widen1<T>(x[c]);
    const float mean = row_sum<1024>(sum, shared[0]) / (float)a.cols;
    sum = 0.0f;
    for (long long c = threadIdx.x; c < a.cols; c += 1024) {
        const float d = widen1<T>(x[c]) - mean;
        sum = fmaf(d, d, sum);
    }
    const float rstd = 1.0f / sqrtf(row_sum<1024>(sum, shared[1]) / (float)a.cols + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[blockIdx.x] = mean;
        if (a.rstd) a.rstd[blockIdx.x] = rstd;
    }
    if (!a.y) return;
    T *y = static_cast<T *>(a.y) + (long long)blockIdx.x * a.y_stride;
    for (long long c = threadIdx.x; c < a.cols; c += 1024) {
        float r = (widen1<T>(x[c]) - mean) * rstd;
        if (a.gamma) r *= load_param(a.gamma, a.params_bf16, c);
        if (a.beta) r += load_param(a.beta, a.params_bf16, c);
        y[c] = narrow1<T>(r);
    }
}

template <typename T, bool VEC>
void launch_norm(const NormArgs &a, cudaStream_t stream)
{
    const int64_t units = ceil_div(a.cols, 16 / (int)sizeof(T));
#define NORM_CASE(TPR, NU)                                                                                         \
    if (units <= TPR * NU) {                                                                                       \
        constexpr int threads = TPR < 128 ? 128 : TPR;                                                             \
        norm_rows_kernel<T, VEC, TPR, NU><<<(unsigned)ceil_div(a.rows, threads / TPR), threads, 0, stream>>>(a);   \
        return;                                                                                                    \
    }
    NORM_CASE(8, 1)
    NORM_CASE(16, 1)
    NORM_CASE(32, 1)
    NORM_CASE(32, 2)
    NORM_CASE(32, 4)
    NORM_CASE(32, 8)
    NORM_CASE(128, 4)
    NORM_CASE(128, 8)
    NORM_CASE(256, 8)
    NORM_CASE(512, 8)
#undef NORM_CASE
    norm_long_rows_kernel<T><<<(unsigned)a.rows, 1024, 0, stream>>>(a);
}

// ------------------------------------------------------------------------------------------ backward

struct NormBackArgs {
    const void *dy;
    const void *x;  // dense, or the codes of a packed matrix
    const uint8_t *scales;
    const float *mean, *rstd;
    const void *gamma;
    void *dx;                // may be NULL
    float *dgamma, *dbeta;   // rows of `part_stride` values, one per block; may be NULL
    long long dy_stride, x_stride, dx_stride, part_stride;
    int rows, cols, scale_cols;
    bool params_bf16, gamma_aligned;
};

// What a thread loads of a row, before conversion.
template <typename T, bool PACKED, bool VEC> struct BackRow {
    static constexpr int U = 16 / (int)sizeof(T);
    static constexpr int E = 2 * U;
    uint4 dy4[VEC ? 2 : 1], x4[VEC && !PACKED ? 2 : 1];
    unsigned codes[VEC && PACKED ? 2 * U / 4 : 1];
    float dy1[VEC ? 1 : E], x1[VEC ? 1 : E];
    float scale[PACKED && VEC ? 2 : 1];
    float mean, rstd;

    __device__ __forceinline__ void load(const NormBackArgs &a, long long row, int lane, int threads)
    {
        mean = a.mean[row];
        rstd = a.rstd[row];
        const T *dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
        const uint8_t *scales = PACKED ? a.scales + row / PACK_BLOCK * a.scale_cols : nullptr;
        constexpr int STEPS = VEC ? 2 : E, W = VEC ? U : 1;
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
            const int c = (j * threads + lane) * W;
            if (c >= a.cols) continue;
            if constexpr (VEC)
                dy4[j] = *reinterpret_cast<const uint4 *>(dy + c);
            else
                dy1[j] = widen1<T>(dy[c]);
            if constexpr (PACKED) {
                const uint8_t *q = static_cast<const uint8_t *>(a.x) + row * a.x_stride + c;
                const float s = scale_value(scales[c / PACK_BLOCK]);
                if constexpr (VEC) scale[j] = s;
                if constexpr (!VEC) {
                    x1[j] = decode2(*q).x * s;
                } else if constexpr (U == 8) {
                    const uint2 w = *reinterpret_cast<const uint2 *>(q);
                    codes[2 * j] = w.x;
                    codes[2 * j + 1] = w.y;
                } else {
                    codes[j] = *reinterpret_cast<const unsigned *>(q);
                }
            } else {
                const T *q = static_cast<const T *>(a.x) + row * a.x_stride + c;
                if constexpr (VEC)
                    x4[j] = *reinterpret_cast<const uint4 *>(q);
                else
                    x1[j] = widen1<T>(*q);
            }
        }
    }
    // dy and h of step j.
    __device__ __forceinline__ void convert(int j, float *dy, float *hat) const
    {
        if constexpr (VEC) {
            Unit<T>::widen(dy4[j], dy);
            if constexpr (PACKED) {
#pragma unroll
                for (int i = 0; i < U; i += 4) {
                    const float2 p = decode2(codes[(j * U + i) / 4] & 0xffffu), q = decode2(codes[(j * U + i) / 4] >> 16);
                    hat[i] = fmaf(p.x, scale[j], -mean); hat[i + 1] = fmaf(p.y, scale[j], -mean);
                    hat[i + 2] = fmaf(q.x, scale[j], -mean); hat[i + 3] = fmaf(q.y, scale[j], -mean);
                }
            } else {
                Unit<T>::widen(x4[j], hat);
#pragma unroll
                for (int i = 0; i < U; ++i) hat[i] -= mean;
            }
#pragma unroll
            for (int i = 0; i < U; ++i) hat[i] *= rstd;
        } else {
            dy[0] = dy1[j];
            hat[0] = (x1[j] - mean) * rstd;
        }
    }
};

// TPR threads per row, each with the same two units of 16 bytes of every row that its block passes over:
// the sums of dgamma and dbeta stay in registers and leave the block once.  The next row is loaded while
// this one is reduced.
template <typename T, bool PACKED, bool VEC, int TPR>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR, TPR < 512 ? 2 : 1) norm_back_kernel(const __grid_constant__ NormBackArgs a)
{
    using Row = BackRow<T, PACKED, VEC>;
    constexpr int E = Row::E;
    constexpr int U = VEC ? Row::U : 1;
    constexpr int UNITS = E / U;
    constexpr int THREADS = TPR < 256 ? 256 : TPR;
    constexpr int GROUPS = THREADS / TPR;
    constexpr int WARPS = TPR / 32;
    __shared__ float2 shared[2][THREADS / 32];
    __shared__ float columns[GROUPS > 1 ? 2 * TPR * E : 1];
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const float inv_cols = 1.0f / (float)a.cols;

    float gamma[E], sum_g[E], sum_b[E];
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        const int c = (j * TPR + lane) * U;
#pragma unroll
        for (int i = 0; i < U; ++i) sum_g[j * U + i] = sum_b[j * U + i] = 0.0f;
        if constexpr (VEC) {
            if (a.gamma) {
                load_params<U>(a.gamma, a.params_bf16, a.gamma_aligned, c, a.cols, gamma + j * U);
            } else {
#pragma unroll
                for (int i = 0; i < U; ++i) gamma[j * U + i] = 1.0f;
            }
        } else {
            gamma[j] = !a.gamma ? 1.0f : c < a.cols ? load_param(a.gamma, a.params_bf16, c) : 0.0f;
        }
    }

    const long long step = (long long)gridDim.x * GROUPS;
    long long row = (long long)blockIdx.x * GROUPS + group;
    Row now, ahead;
    if (VEC && row < a.rows) now.load(a, row, lane, TPR);
    int parity = 0;
    for (; row - group < a.rows; row += step) {
        const bool live = row < a.rows;
        if constexpr (VEC) {
            if (row + step < a.rows) ahead.load(a, row + step, lane, TPR);
        } else {
            if (live) now.load(a, row, lane, TPR);
        }
        float hat[E], g[E];
        float2 both = make_float2(0.0f, 0.0f);  // sums of g and of g h
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            const int c = (j * TPR + lane) * U;
            if (c < a.cols && live) {
                now.convert(j, g + j * U, hat + j * U);
                if (VEC && c + U > a.cols) {
#pragma unroll
                    for (int i = 0; i < U; ++i)
                        if (c + i >= a.cols) g[j * U + i] = hat[j * U + i] = 0.0f;
                }
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const int e = j * U + i;
                    sum_g[e] = fmaf(g[e], hat[e], sum_g[e]);
                    sum_b[e] += g[e];
                    g[e] *= gamma[e];
                    both.x += g[e];
                    both.y = fmaf(g[e], hat[e], both.y);
                }
            }
        }
#pragma unroll
        for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1) {
            both.x += __shfl_xor_sync(0xffffffffu, both.x, o);
            both.y += __shfl_xor_sync(0xffffffffu, both.y, o);
        }
        if constexpr (TPR > 32) {
            // two sets of slots in turn: a slot is written again only after the barrier of the next row,
            // which every thread of the row's group reaches after it has read this row's
            const int warp = threadIdx.x >> 5;
            if ((threadIdx.x & 31) == 0) shared[parity][warp] = both;
            if constexpr (GROUPS == 1)
                __syncthreads();
            else
                asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(TPR) : "memory");
            both = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float2 s = shared[parity][group * WARPS + w];
                both.x += s.x;
                both.y += s.y;
            }
            parity ^= 1;
        }
        if (live && a.dx) {
            const float g1 = both.x * inv_cols, g2 = both.y * inv_cols, rstd = now.rstd;
#pragma unroll
            for (int j = 0; j < UNITS; ++j) {
                const int c = (j * TPR + lane) * U;
                if (c >= a.cols) continue;
                T *d = static_cast<T *>(a.dx) + row * a.dx_stride + c;
                float r[U];
#pragma unroll
                for (int i = 0; i < U; ++i) r[i] = fmaf(-hat[j * U + i], g2, g[j * U + i] - g1) * rstd;
                if constexpr (VEC) {
                    if (c + U <= a.cols) {
                        *reinterpret_cast<uint4 *>(d) = Unit<T>::narrow(r);
                    } else {
#pragma unroll
                        for (int i = 0; i < U; ++i)
                            if (c + i < a.cols) d[i] = narrow1<T>(r[i]);
                    }
                } else {
                    *d = narrow1<T>(r[0]);
                }
            }
        }
        if constexpr (VEC) now = ahead;
    }

    if (!a.dgamma && !a.dbeta) return;
    if constexpr (GROUPS > 1) {  // the block's groups in ascending order
        for (int g = 0; g < GROUPS; ++g) {
            __syncthreads();
            if (group == g) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int at = (e / U * TPR + lane) * U + e % U;
                    columns[at] = (g ? columns[at] : 0.0f) + sum_g[e];
                    columns[TPR * E + at] = (g ? columns[TPR * E + at] : 0.0f) + sum_b[e];
                }
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < a.cols; c += THREADS) {
            if (a.dgamma) a.dgamma[blockIdx.x * a.part_stride + c] = columns[c];
            if (a.dbeta) a.dbeta[blockIdx.x * a.part_stride + c] = columns[TPR * E + c];
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int c = (e / U * TPR + lane) * U + e % U;
            if (c < a.cols) {
                if (a.dgamma) a.dgamma[blockIdx.x * a.part_stride + c] = sum_g[e];
                if (a.dbeta) a.dbeta[blockIdx.x * a.part_stride + c] = sum_b[e];
            }
        }
    }
}

// Rows that do not fit a block's registers: dx by one block per row, which reads the row twice, and
// dgamma, dbeta by blocks of 256 columns over a share of the rows.
template <typename T, bool PACKED>
__device__ __forceinline__ float back_value(const NormBackArgs &a, long long row, long long c)
{
    if constexpr (PACKED)
        return decode2(static_cast<const uint8_t *>(a.x)[row * a.x_stride + c]).x *
               scale_value(a.scales[row / PACK_BLOCK * a.scale_cols + c / PACK_BLOCK]);
    else
        return widen1<T>(static_cast<const T *>(a.x)[row * a.x_stride + c]);
}

template <typename T, bool PACKED>
__global__ void __launch_bounds__(1024) norm_back_long_rows_kernel(NormBackArgs a)
{
    __shared__ float shared[2][32];
    const long long row = blockIdx.x;
    const T *dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float g1 = 0.0f, g2 = 0.0f;
    for (long long c = threadIdx.x; c < a.cols; c += 1024) {
        const float g = widen1<T>(dy[c]) * (a.gamma ? load_param(a.gamma, a.params_bf16, c) : 1.0f);
        g1 += g;
        g2 = fmaf(g, (back_value<T, PACKED>(a, row, c) - mean) * rstd, g2);
    }
    g1 = row_sum<1024>(g1, shared[0]) / (float)a.cols;
    g2 = row_sum<1024>(g2, shared[1]) / (float)a.cols;
    T *dx = static_cast<T *>(a.dx) + row * a.dx_stride;
    for (long long c = threadIdx.x; c < a.cols; c += 1024) {
        const float g = widen1<T>(dy[c]) * (a.gamma ? load_param(a.gamma, a.params_bf16, c) : 1.0f);
        dx[c] = narrow1<T>((g - g1 - (back_value<T, PACKED>(a, row, c) - mean) * rstd * g2) * rstd);
    }
}

template <typename T, bool PACKED>
__global__ void __launch_bounds__(256) norm_back_long_columns_kernel(NormBackArgs a)
{
    const long long c = (long long)blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols) return;
    float sum_g = 0.0f, sum_b = 0.0f;
    for (long long row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float dy = widen1<T>(static_cast<const T *>(a.dy)[row * a.dy_stride + c]);
        sum_g = fmaf(dy, (back_value<T, PACKED>(a, row, c) - a.mean[row]) * a.rstd[row], sum_g);
        sum_b += dy;
    }
    if (a.dgamma) a.dgamma[blockIdx.y * a.part_stride + c] = sum_g;
    if (a.dbeta) a.dbeta[blockIdx.y * a.part_stride + c] = sum_b;
}

// The blocks' sums, in the order of the blocks within each of 32 strands and then of the strands.
__global__ void __launch_bounds__(1024) norm_back_join_kernel(const float *parts_g, const float *parts_b, int parts,
                                                              long long part_stride, int cols, float *dgamma,
                                                              float *dbeta)
{
    __shared__ float shared[32][33];
    const float *parts_of = blockIdx.y ? parts_b : parts_g;
    float *out = blockIdx.y ? dbeta : dgamma;
    if (!out) return;
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + tx;
    float sum = 0.0f;
    if (c < cols)
#pragma unroll 10
        for (int p = ty; p < parts; p += 32) sum += parts_of[p * part_stride + c];
    shared[ty][tx] = sum;
    __syncthreads();
    sum = shared[tx][ty];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const long long at = (long long)blockIdx.x * 32 + ty;
    if (tx == 0 && at < cols) out[at] = sum;
}

constexpr int BACK_BLOCKS = 296;       // two blocks of the row kernel on each of 148 SMs
constexpr int BACK_LONG_SHARES = 32;

// The widest row that a block holds, and the threads for a row: two units of 16 bytes each.
int64_t back_widest(int dtype) { return dtype == DIPACO_BF16 ? 16384 : 8192; }
int back_threads_per_row(int64_t cols, int dtype)
{
    int tpr = 8;
    while (tpr * (32 / dense_size(dtype)) < cols) tpr *= 2;
    return tpr;
}

// Blocks that write their own sums of dgamma and dbeta.
int64_t back_parts(int64_t rows, int64_t cols, int dtype)
{
    if (cols > back_widest(dtype)) return std::min<int64_t>(BACK_LONG_SHARES, ceil_div(rows, 64));
    const int tpr = back_threads_per_row(cols, dtype);
    return std::min<int64_t>(BACK_BLOCKS, ceil_div(rows, tpr < 256 ? 256 / tpr : 1));
}

template <typename T, bool PACKED, bool VEC>
void launch_back(const NormBackArgs &a, int blocks, cudaStream_t stream)
{
    const int tpr = back_threads_per_row(a.cols, sizeof(T) == 2 ? DIPACO_BF16 : DIPACO_F32);
#define BACK_CASE(TPR)                                                                              \
    case TPR:                                                                                       \
        norm_back_kernel<T, PACKED, VEC, TPR><<<blocks, TPR < 256 ? 256 : TPR, 0, stream>>>(a);     \
        return;
    switch (tpr) {
        BACK_CASE(8)
        BACK_CASE(16)
        BACK_CASE(32)
        BACK_CASE(64)
        BACK_CASE(128)
        BACK_CASE(256)
        BACK_CASE(512)
        BACK_CASE(1024)
    }
#undef BACK_CASE
}

template <typename T, bool PACKED>
void launch_back_any(const NormBackArgs &a, int blocks, bool vec, cudaStream_t stream)
{
    if (a.cols > back_widest(sizeof(T) == 2 ? DIPACO_BF16 : DIPACO_F32)) {
        if (a.dx) norm_back_long_rows_kernel<T, PACKED><<<a.rows, 1024, 0, stream>>>(a);
        if (a.dgamma || a.dbeta)
            norm_back_long_columns_kernel<T, PACKED>
                <<<dim3((unsigned)ceil_div(a.cols, 256), blocks), 256, 0, stream>>>(a);
    } else if (vec) {
        launch_back<T, PACKED, true>(a, blocks, stream);
    } else {
        launch_back<T, PACKED, false>(a, blocks, stream);
    }
}

} // namespace

extern "C" {

int dipaco_layer_norm(const void *x, int64_t x_stride, const void *gamma, const void *beta, void *y,
                      int64_t y_stride, float *mean, float *rstd, int64_t rows, int64_t cols, float eps,
                      int32_t dtype, int32_t param_dtype, int32_t device, void *cuda_stream)
{
    if (!is_dense_dtype(dtype) || !is_dense_dtype(param_dtype) || device < 0) return DIPACO_EINVAL;
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return DIPACO_EINVAL;
    if (const int rc = check_extents(rows, cols)) return rc;
    if (!dense_ok(x, x_stride, rows, cols, dtype)) return DIPACO_EINVAL;
    if (y ? !dense_ok(y, y_stride, rows, cols, dtype) : !mean && !rstd && rows > 0 && cols > 0) return DIPACO_EINVAL;
    const int psize = dense_size(param_dtype);
    if (!vector_ok(gamma, psize) || !vector_ok(beta, psize) || !vector_ok(mean, 4) || !vector_ok(rstd, 4))
        return DIPACO_EINVAL;
    if (rows == 0 || cols == 0) return DIPACO_OK;

    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    NormArgs a = {x, y, gamma, beta, mean, rstd, x_stride, y_stride, (int)rows, (int)cols, eps,
                  param_dtype == DIPACO_BF16, (uintptr_t)gamma % 16 == 0, (uintptr_t)beta % 16 == 0};
    const int size = dense_size(dtype);
    const bool vec = rows_aligned16(x, x_stride, rows, size) && (!y || rows_aligned16(y, y_stride, rows, size));
    if (dtype == DIPACO_BF16)
        vec ? launch_norm<__nv_bfloat16, true>(a, stream) : launch_norm<__nv_bfloat16, false>(a, stream);
    else
        vec ? launch_norm<float, true>(a, stream) : launch_norm<float, false>(a, stream);
    return launch_status();
}

int dipaco_layer_norm_workspace(int64_t rows, int64_t cols, int64_t *bytes)
{
    if (!bytes) return DIPACO_EINVAL;
    if (const int rc = check_extents(rows, cols)) return rc;
    int64_t parts = 0;  // the most of either dtype
    if (rows > 0 && cols > 0) parts = std::max(back_parts(rows, cols, DIPACO_F32), back_parts(rows, cols, DIPACO_BF16));
    *bytes = parts > 1 ? parts * 2 * cols * (int64_t)sizeof(float) : 0;
    return DIPACO_OK;
}

int dipaco_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride,
                               const dipaco_packed *x_packed, const float *mean, const float *rstd,
                               const void *gamma, void *dx, int64_t dx_stride, float *dgamma, float *dbeta,
                               int64_t rows, int64_t cols, int32_t dtype, int32_t param_dtype, void *workspace,
                               int64_t workspace_bytes, int32_t device, void *cuda_stream)
{
    if (!is_dense_dtype(dtype) || !is_dense_dtype(param_dtype) || device < 0) return DIPACO_EINVAL;
    if (const int rc = check_extents(rows, cols)) return rc;
    if (!dx && !dgamma && !dbeta) return DIPACO_EINVAL;
    if (cols == 0) return DIPACO_OK;
    if (!vector_ok(dgamma, 4) || !vector_ok(dbeta, 4) || !vector_ok(gamma, dense_size(param_dtype)))
        return DIPACO_EINVAL;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (rows > 0) {
        if ((x != nullptr) == (x_packed != nullptr)) return DIPACO_EINVAL;
        if (!dense_ok(dy, dy_stride, rows, cols, dtype)) return DIPACO_EINVAL;
        if (x ? !dense_ok(x, x_stride, rows, cols, dtype) : !packed_ok(x_packed, rows, cols)) return DIPACO_EINVAL;
        if (dx && !dense_ok(dx, dx_stride, rows, cols, dtype)) return DIPACO_EINVAL;
        if (!mean || !rstd || !vector_ok(mean, 4) || !vector_ok(rstd, 4)) return DIPACO_EINVAL;
        int64_t need = 0;
        dipaco_layer_norm_workspace(rows, cols, &need);
        if ((dgamma || dbeta) && need > 0 &&
            (!workspace || (uintptr_t)workspace % 16 != 0 || workspace_bytes < need))
            return DIPACO_EINVAL;
    }
    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    if (rows == 0) {  // sums over no rows
        if (dgamma && cudaMemsetAsync(dgamma, 0, cols * sizeof(float), stream) != cudaSuccess) return launch_status();
        if (dbeta && cudaMemsetAsync(dbeta, 0, cols * sizeof(float), stream) != cudaSuccess) return launch_status();
        return DIPACO_OK;
    }
    const int parts = (int)back_parts(rows, cols, dtype);
    NormBackArgs a = {};
    a.dy = dy;
    a.x = x_packed ? x_packed->codes : x;
    a.scales = x_packed ? static_cast<const uint8_t *>(x_packed->scales) : nullptr;
    a.mean = mean;
    a.rstd = rstd;
    a.gamma = gamma;
    a.dx = dx;
    a.dy_stride = dy_stride;
    a.x_stride = x_packed ? x_packed->stride : x_stride;
    a.dx_stride = dx_stride;
    a.rows = (int)rows;
    a.cols = (int)cols;
    a.scale_cols = (int)ceil_div(cols, PACK_BLOCK);
    a.params_bf16 = param_dtype == DIPACO_BF16;
    a.gamma_aligned = (uintptr_t)gamma % 16 == 0;
    if (parts > 1) {
        float *w = static_cast<float *>(workspace);
        a.dgamma = dgamma ? w : nullptr;
        a.dbeta = dbeta ? w + cols : nullptr;
        a.part_stride = 2 * cols;
    } else {
        a.dgamma = dgamma;
        a.dbeta = dbeta;
    }
    const int size = dense_size(dtype);
    const bool vec = rows_aligned16(dy, dy_stride, rows, size) && (!x || rows_aligned16(x, x_stride, rows, size)) &&
                     (!dx || rows_aligned16(dx, dx_stride, rows, size));
    if (dtype == DIPACO_BF16)
        x ? launch_back_any<__nv_bfloat16, false>(a, parts, vec, stream)
          : launch_back_any<__nv_bfloat16, true>(a, parts, vec, stream);
    else
        x ? launch_back_any<float, false>(a, parts, vec, stream) : launch_back_any<float, true>(a, parts, vec, stream);
    if (parts > 1 && (dgamma || dbeta))
        norm_back_join_kernel<<<dim3((unsigned)ceil_div(cols, 32), 2), 1024, 0, stream>>>(
            a.dgamma, a.dbeta, parts, a.part_stride, (int)cols, dgamma, dbeta);
    return launch_status();
}

} // extern "C"
