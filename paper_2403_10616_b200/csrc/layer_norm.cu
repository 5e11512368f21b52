// Layer norm of the rows of a matrix, forward and backward (see include/dipaco.h).
//
//   mean = sum x / C, var = sum (x - mean)^2 / C, rstd = (var + eps)^-1/2, y = (x - mean) rstd gamma + beta
//   g = dy gamma, h = (x - mean) rstd, dx = rstd (g - mean(g) - h mean(g h)), dgamma = sum dy h, dbeta = sum dy
//
// All sums are fp32.  The variance is summed from the centred values of the row, which is held in
// registers, so it does not cancel for rows whose mean is large beside their spread.  The mean of fp32
// values is corrected by the mean of x - mean: its own roundings, up to some units in the last place, can
// be more than the spread (a row of 1000.1 had results up to 0.15 instead of 0 at eps = 1e-5).
#include "inner_common.cuh"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

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

// Two sums at once.
template <int TPR> __device__ __forceinline__ float2 row_sums(float a, float b, float2 *shared)
{
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    if constexpr (TPR > 32) {
        constexpr int WARPS = TPR / 32;
        const int warp = threadIdx.x >> 5;
        if ((threadIdx.x & 31) == 0) shared[warp] = make_float2(a, b);
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float2 v = shared[warp / WARPS * WARPS + w];
            a += v.x;
            b += v.y;
        }
    }
    return make_float2(a, b);
}

// ------------------------------------------------------------------------------------------ forward

struct NormArgs {
    const void *x;
    void *y;  // NULL: statistics only
    const void *gamma, *beta;
    float *mean, *rstd;
    long long x_stride, y_stride;
    int rows, cols;
    float eps, inv_cols;
    bool params_bf16;
};

// (square / cols + eps)^-1/2.  Its error is that of every value of the row, so it is kept to the last rounding:
// the product with 1 / cols is corrected by its remainder, and one Newton step takes the approximation's
// residual with what the product v r rounds off (rms error 2.8e-8 instead of 5.3e-8 without either).
__device__ __forceinline__ float inverse_root(float square, float cols, float inv_cols, float eps)
{
    float v = __fmul_rn(square, inv_cols);
    if (v < 1e30f) v = fmaf(fmaf(-v, cols, square), inv_cols, v);
    v = __fadd_rn(v, eps);  // not contracted: the same value wherever this is compiled
    const float r = rsqrtf(v), t = __fmul_rn(v, r), rest = fmaf(v, r, -t);
    const float better = fmaf(0.5f * r, fmaf(-rest, r, fmaf(-t, r, 1.0f)), r);
    return v > 1e-30f && v < 1e30f ? better : 1.0f / sqrtf(v);  // where the step's products stay normal
}

// Corrects a mean and the sum of squares around it by `rest`, the sum of the values less that mean, and returns
// what the values less that mean still have to lose.  Where sums leave the range of fp32 nothing is corrected.
__device__ __forceinline__ float correct_mean(float &mean, float &square, float rest, float cols)
{
    const float shift = rest / cols;
    if (!(fabsf(shift) < 1e30f)) return 0.0f;
    mean += shift;
    const float less = fmaf(-shift, rest, square);
    if (less < square) square = fmaxf(less, 0.0f);
    return shift;
}

template <typename T> __device__ __forceinline__ void store_first(T *p, const uint4 &v, int n)
{
#pragma unroll
    for (int i = 0; i < 16 / (int)sizeof(T); ++i)
        if (i < n) store_element(p + i, v, i);
}

constexpr int NORM_WIDEST = 16384;  // values of a row with gamma and beta in shared memory

// How rows are read: by single values, by units of 16 bytes, or by units of which a row's last is partly outside.
enum : int { ROWS_SINGLE, ROWS_UNITS, ROWS_RAGGED };

// One row at a time per TPR threads, in registers: NU units of 16 bytes per thread, of which the last PART
// may lie outside the row, or as many single values.  Bound by memory, if little else is done: the next row
// is on its way while this one is summed, sums run in four chains, and gamma and beta wait in shared memory
// in fp32 (with both read and widened for every row: 16384x2048 43 us).  A warp per row up to 2048 values
// in bf16 (1024 in fp32) keeps sums inside warps; two or four warps per row took 35 and 37 us there.
// STATS (nothing written but mean and rstd) sums in fp32 pairs and takes fewer registers, for more warps: the
// first launch of the packed norm, 32768x896, 15 -> 13 us; with y to write pairs were slower.
// Measured: 16384x2048 in bf16 with statistics 32 us, 4.2 TB/s; what is left is the warps' waiting for
// their own chains of sums and exchanges (they issue in a third of the cycles), not instructions.
// The blocks on an SM are those of widths to 2048 with y written; from 7161 bf16 values on gamma and beta leave room in
// shared memory for fewer than the grid assumes, and its last blocks run in a second wave (8192x7000 86 us).
// Rows off 16 bytes are read by single values and spill registers: 16384x2048 in bf16 98 us.  fp32: 16384x2048
// 51 us, 32768x896 46 us (with the mean corrected; 45 without).
constexpr int norm_blocks(int tpr, int nu, bool stats) { return tpr > 128 ? 1 : nu > 4 ? 4 : stats ? 8 : 6; }  // on an SM

template <typename T, int MODE, int TPR, int NU, int PART, bool STATS>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR, norm_blocks(TPR, NU, STATS))
    norm_rows_kernel(const __grid_constant__ NormArgs a)
{
    constexpr bool VEC = MODE != ROWS_SINGLE;
    constexpr int U = VEC ? 16 / (int)sizeof(T) : 1;
    constexpr int E = NU * 16 / (int)sizeof(T);
    constexpr int UNITS = E / U, SURE = VEC ? NU - PART : 0;  // units that are inside for certain
    constexpr int THREADS = TPR < 128 ? 128 : TPR, GROUPS = THREADS / TPR;
    using Raw = typename std::conditional<VEC, uint4, T>::type;
    extern __shared__ __align__(16) float params[];  // gamma, beta, each padded to whole units
    // bf16: the sums of equal values, or of others of one size, are exact up to 2^16 of them
    constexpr bool CORRECT = std::is_same<T, float>::value;
    __shared__ float shared[2][TPR > 32 ? TPR / 32 : 1];  // the first sum of a row, of two rows in turn
    __shared__ float2 shared2[2][TPR > 32 ? TPR / 32 : 1];  // the sums around its mean
    const int lane = threadIdx.x % TPR;
    const int step = (int)gridDim.x * GROUPS;
    int row = (int)blockIdx.x * GROUPS + (int)threadIdx.x / TPR;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride + lane * U;
    T *y = static_cast<T *>(a.y) + row * a.y_stride + lane * U;
    const int cols = a.cols - lane * U;  // a unit j of this thread is inside while j * TPR * U < cols
    const int padded = (a.cols + 7) & ~7;

    Raw raw[UNITS];
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        if constexpr (VEC) raw[j] = make_uint4(0u, 0u, 0u, 0u);
        if (row < a.rows && (j < SURE || j * TPR * U < cols)) raw[j] = *reinterpret_cast<const Raw *>(x + j * TPR * U);
    }
    if constexpr (!STATS) {
        for (int c = threadIdx.x; c < padded; c += THREADS) {
            const bool in = c < a.cols;
            params[c] = !in ? 0.0f : a.gamma ? load_param(a.gamma, a.params_bf16, c) : 1.0f;
            params[padded + c] = in && a.beta ? load_param(a.beta, a.params_bf16, c) : 0.0f;
        }
        __syncthreads();
    }
    int turn = 0;
    // rows beyond the last keep the warp together: what they compute is not written
    for (int first = (int)blockIdx.x * GROUPS; first < a.rows; first += step, row += step) {
        // statistics alone: the same sums in fp32 pairs
        f32x2 pairs[STATS && VEC ? E / 2 : 1], sum2[2] = {0ull, 0ull};
        float v[STATS && VEC ? 1 : E], sums[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            if constexpr (STATS && VEC) {
                f32x2 *p = pairs + j * U / 2;
                widen_pairs<T>(raw[j], p);
                if (MODE == ROWS_RAGGED && j >= SURE) keep_inside<U>(p, cols - j * TPR * U);
#pragma unroll
                for (int i = 0; i < U / 2; ++i) sum2[i & 1] = add2(sum2[i & 1], p[i]);
            } else {
                if constexpr (VEC)
                    Unit<T>::widen(raw[j], v + j * U);
                else
                    v[j] = j * TPR < cols ? widen1<T>(raw[j]) : 0.0f;
                if constexpr (MODE == ROWS_RAGGED) {
                    if (j >= SURE) {
#pragma unroll
                        for (int i = 1; i < U; ++i)
                            if (j * TPR * U + i >= cols) v[j * U + i] = 0.0f;
                    }
                }
#pragma unroll
                for (int i = 0; i < U; ++i) sums[(j * U + i) & 3] += v[j * U + i];
            }
        }
        x += step * a.x_stride;
        if (row + step < a.rows) {
#pragma unroll
            for (int j = 0; j < UNITS; ++j)
                if (j < SURE || j * TPR * U < cols) raw[j] = *reinterpret_cast<const Raw *>(x + j * TPR * U);
        }
        // divided, not multiplied: the mean of equal values is that value where their sum is exact
        const auto sum = [&] { return STATS && VEC ? sum_of(sum2[0]) + sum_of(sum2[1]) : (sums[0] + sums[1]) + (sums[2] + sums[3]); };
        float mean = row_sum<TPR>(sum(), shared[turn]) / (float)a.cols;
        f32x2 rest2 = 0ull;
        float rest = 0.0f;
        sum2[0] = sum2[1] = 0ull;
        sums[0] = sums[1] = sums[2] = sums[3] = 0.0f;
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            if constexpr (STATS && VEC) {
                f32x2 *p = pairs + j * U / 2;
#pragma unroll
                for (int i = 0; i < U / 2; ++i) p[i] = add2(p[i], pair_of(-mean));
                if (j >= SURE) keep_inside<U>(p, cols - j * TPR * U);
#pragma unroll
                for (int i = 0; i < U / 2; ++i) {
                    sum2[i & 1] = fma2(p[i], p[i], sum2[i & 1]);
                    if constexpr (CORRECT) rest2 = add2(rest2, p[i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < U; ++i) v[j * U + i] -= mean;
                if (j >= SURE) {  // what lies outside does not count
#pragma unroll
                    for (int i = 0; i < U; ++i)
                        if (j * TPR * U + (MODE == ROWS_RAGGED ? i : 0) >= cols) v[j * U + i] = 0.0f;
                }
#pragma unroll
                for (int i = 0; i < U; ++i) sums[(j * U + i) & 3] = fmaf(v[j * U + i], v[j * U + i], sums[(j * U + i) & 3]);
                if constexpr (CORRECT) {
#pragma unroll
                    for (int i = 0; i < U; ++i) rest += v[j * U + i];
                }
            }
        }
        float square, shift = 0.0f;
        if constexpr (CORRECT) {
            const float2 both = row_sums<TPR>(sum(), STATS && VEC ? sum_of(rest2) : rest, shared2[turn]);
            square = both.x;
            shift = correct_mean(mean, square, both.y, (float)a.cols);
        } else {
            square = row_sum<TPR>(sum(), &shared2[turn][0].x);
        }
        const float rstd = inverse_root(square, (float)a.cols, a.inv_cols, a.eps);
        const float loss = shift == 0.0f ? 0.0f : -shift * rstd;  // of (x - mean) rstd
        turn ^= 1;
        if (row < a.rows) {
            if (lane == 0) {
                if (a.mean) a.mean[row] = mean;
                if (a.rstd) a.rstd[row] = rstd;
            }
            if constexpr (!STATS) {
                const float *gamma = params + lane * U, *beta = gamma + padded;
                const auto hat = [&](float d) { return CORRECT ? fmaf(d, rstd, loss) : d * rstd; };
#pragma unroll
                for (int j = 0; j < UNITS; ++j) {
                    if (j >= SURE && j * TPR * U >= cols) continue;
                    float *r = v + j * U;
                    if constexpr (VEC) {
#pragma unroll
                        for (int i = 0; i < U; i += 4) {
                            const float4 g = *reinterpret_cast<const float4 *>(gamma + j * TPR * U + i);
                            const float4 b = *reinterpret_cast<const float4 *>(beta + j * TPR * U + i);
                            r[i] = fmaf(hat(r[i]), g.x, b.x);
                            r[i + 1] = fmaf(hat(r[i + 1]), g.y, b.y);
                            r[i + 2] = fmaf(hat(r[i + 2]), g.z, b.z);
                            r[i + 3] = fmaf(hat(r[i + 3]), g.w, b.w);
                        }
                        const uint4 out = Unit<T>::narrow(r);
                        if (MODE != ROWS_RAGGED || j < SURE || j * TPR * U + U <= cols)
                            *reinterpret_cast<uint4 *>(y + j * TPR * U) = out;
                        else
                            store_first(y + j * TPR * U, out, cols - j * TPR * U);
                    } else {
                        y[j * TPR] = narrow1<T>(fmaf(hat(r[0]), gamma[j * TPR], beta[j * TPR]));
                    }
                }
            }
        }
        y += step * a.y_stride;
    }
}

// Rows that do not fit a block's registers: one block per row, which reads the row three times.
template <typename T>
__global__ void __launch_bounds__(1024) norm_long_rows_kernel(NormArgs a)
{
    __shared__ float shared[32];
    __shared__ float2 shared2[32];
    const T *x = static_cast<const T *>(a.x) + (long long)blockIdx.x * a.x_stride;
    float sum = 0.0f, rest = 0.0f;
    for (long long c = threadIdx.x; c < a.cols; c += 1024) sum += widen1<T>(x[c]);
    const float first = row_sum<1024>(sum, shared) / (float)a.cols;
    sum = 0.0f;
    for (long long c = threadIdx.x; c < a.cols; c += 1024) {
        const float d = widen1<T>(x[c]) - first;
        sum = fmaf(d, d, sum);
        rest += d;
    }
    const float2 both = row_sums<1024>(sum, rest, shared2);
    float mean = first, square = both.x;
    const float shift = correct_mean(mean, square, both.y, (float)a.cols);
    const float rstd = inverse_root(square, (float)a.cols, a.inv_cols, a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[blockIdx.x] = mean;
        if (a.rstd) a.rstd[blockIdx.x] = rstd;
    }
    if (!a.y) return;
    T *y = static_cast<T *>(a.y) + (long long)blockIdx.x * a.y_stride;
    for (long long c = threadIdx.x; c < a.cols; c += 1024) {
        float r = (widen1<T>(x[c]) - first - shift) * rstd;
        if (a.gamma) r *= load_param(a.gamma, a.params_bf16, c);
        if (a.beta) r += load_param(a.beta, a.params_bf16, c);
        y[c] = narrow1<T>(r);
    }
}

template <typename T, int MODE, int TPR, int NU, int PART, bool STATS>
int launch_norm_kernel(const NormArgs &a, cudaStream_t stream)
{
    constexpr int threads = TPR < 128 ? 128 : TPR;
    const auto kernel = norm_rows_kernel<T, MODE, TPR, NU, PART, STATS>;
    const int64_t full = 148 * norm_blocks(TPR, NU, STATS);
    const unsigned grid = (unsigned)std::min<int64_t>(full, ceil_div(a.rows, threads / TPR));
    const int smem = STATS ? 0 : 2 * (int)ceil_div(a.cols, 8) * 8 * (int)sizeof(float);
    // always the largest there can be: threads that launch different sizes share the attribute
    if (smem > 48 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 2 * NORM_WIDEST * (int)sizeof(float)) != cudaSuccess)
        return launch_status();
    kernel<<<grid, threads, smem, stream>>>(a);
    return launch_status();
}

template <typename T, int MODE, int TPR, int NU, int PART> int launch_norm_shape(const NormArgs &a, cudaStream_t stream)
{
    return a.y ? launch_norm_kernel<T, MODE, TPR, NU, PART, false>(a, stream)
               : launch_norm_kernel<T, MODE, TPR, NU, PART, true>(a, stream);
}

// Up to 2048 values in bf16 the units are dealt out so that only a thread's last can lie outside.
template <typename T, int MODE> int launch_norm(const NormArgs &a, cudaStream_t stream)
{
    const int64_t units = ceil_div(a.cols, 16 / (int)sizeof(T));
    if (units <= 8) return launch_norm_shape<T, MODE, 8, 1, 1>(a, stream);
    if (units <= 16) return launch_norm_shape<T, MODE, 16, 1, 1>(a, stream);
    switch (ceil_div(units, 32)) {
    case 1: return launch_norm_shape<T, MODE, 32, 1, 1>(a, stream);
    case 2: return launch_norm_shape<T, MODE, 32, 2, 1>(a, stream);
    case 3: return launch_norm_shape<T, MODE, 32, 3, 1>(a, stream);
    case 4: return launch_norm_shape<T, MODE, 32, 4, 1>(a, stream);
    case 5: return launch_norm_shape<T, MODE, 32, 5, 1>(a, stream);
    case 6: return launch_norm_shape<T, MODE, 32, 6, 1>(a, stream);
    case 7: return launch_norm_shape<T, MODE, 32, 7, 1>(a, stream);
    case 8: return launch_norm_shape<T, MODE, 32, 8, 1>(a, stream);
    }
    if (units <= 128 * 4) return launch_norm_shape<T, MODE, 128, 4, 2>(a, stream);
    if (units <= 128 * 8) return launch_norm_shape<T, MODE, 128, 8, 4>(a, stream);
    if (units <= 256 * 8) return launch_norm_shape<T, MODE, 256, 8, 4>(a, stream);
    if constexpr (sizeof(T) == 4)  // in bf16 256 threads hold the widest row
        if (a.cols <= NORM_WIDEST) return launch_norm_shape<T, MODE, 512, 8, 4>(a, stream);
    norm_long_rows_kernel<T><<<(unsigned)a.rows, 1024, 0, stream>>>(a);
    return launch_status();
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

// Bytes of the 16-byte units that hold n bytes at p.
__device__ __forceinline__ int around(const uint8_t *p, int n) { return ((int)((uintptr_t)p & 15) + n + 15) & ~15; }

// The first n of 16 bytes to shared memory, the others zero.
__device__ __forceinline__ void copy_filled(void *to, const void *from, int n)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ptx::smem_addr(to)), "l"(from), "r"(n) : "memory");
}

static __device__ int g_norm_error;  // set by a bounded wait that ran out
constexpr int BACK_MAX_STAGES = 4;

// How the threads of a block share rows: TPR threads for a row, each with 32 bytes of it (two
// units of 16, or single values), ROWS rows at a time.  SYNC threads go together; the block's others go their own way.
template <typename T, bool PACKED, bool VEC, int TPR> struct BackShape {
    static constexpr int U = VEC ? 16 / (int)sizeof(T) : 1;
    static constexpr int E = 32 / (int)sizeof(T);
    static constexpr int UNITS = E / U;
    static constexpr int ROWS = TPR <= 256 ? 2 : 1;
    static constexpr int THREADS = TPR < 512 ? 512 : TPR;
    static constexpr int GROUPS = THREADS / TPR;
    static constexpr int SYNC = TPR < 32 ? 32 : TPR;  // threads that take rows together: whole warps
    static constexpr int SYNCS = THREADS / SYNC;
    static constexpr int TAKEN = SYNC / TPR * ROWS;   // rows at a time
    using Raw = typename std::conditional<VEC, uint4, T>::type;
    using X = typename std::conditional<PACKED, uint8_t, T>::type;
    using RawX = typename std::conditional<!PACKED, Raw, typename std::conditional<!VEC, uint8_t,
                 typename std::conditional<U == 8, uint2, unsigned>::type>::type>::type;

    // x - mean of a unit, or of two single values.
    static __device__ __forceinline__ void centred(const RawX *x, float scale, float scale1, float mean, f32x2 *h)
    {
        const f32x2 minus = pair_of(-mean);
        if constexpr (PACKED && VEC) {  // a code times its scale is exact
            unsigned w[U / 4];
            memcpy(w, x, sizeof(w));
#pragma unroll
            for (int i = 0; i < U / 2; ++i) h[i] = fma2(decode_pair(w[i / 2] >> (16 * (i & 1))), pair_of(scale), minus);
        } else if constexpr (PACKED) {
            h[0] = fma2(pair_of(decode2(x[0]).x, decode2(x[1]).x), pair_of(scale, scale1), minus);
        } else if constexpr (VEC) {
            widen_pairs<T>(*x, h);
#pragma unroll
            for (int i = 0; i < U / 2; ++i) h[i] = add2(h[i], minus);
        } else {
            h[0] = add2(pair_of(widen1<T>(x[0]), widen1<T>(x[1])), minus);
        }
    }
};

// Sums over the warp of four values at once: afterwards lane l has the sum of value l / 8.  Each step
// halves what a lane carries, which takes 6 exchanges instead of 20.
__device__ __forceinline__ float warp_sum4(const float *v)
{
    const int lane = threadIdx.x & 31;
    const bool high = lane & 16, upper = lane & 8;
    const float a = (high ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, high ? v[0] : v[2], 16);
    const float b = (high ? v[3] : v[1]) + __shfl_xor_sync(0xffffffffu, high ? v[1] : v[3], 16);
    float s = (upper ? b : a) + __shfl_xor_sync(0xffffffffu, upper ? a : b, 8);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}

// The sums of dgamma and dbeta stay in registers, as each thread has the same columns of every row that its
// block passes over, and leave the block once.  Two rows are taken at a time, which halves the work of
// their reductions.  Rows are brought to shared memory by bulk copies, a few steps ahead: a thread has no
// registers to spare for them (4999x2047 in fp32 from registers: 50 us).  On 16-byte boundaries (VEC) a last,
// partial unit of a row is copied by itself and filled up with zeros, which take no part in any sum; rows
// elsewhere are copied with the 16-byte units around them and read value by value.  fp32 arithmetic goes in
// pairs (f32x2): without, 32768x2048 from 8 bits takes 97 us.  Bound by instructions, about 24 for a value:
// 32768x2048 86 us from 8 bits (3.9 TB/s) and 78 us from bf16 (5.1 TB/s), 4999x2047 in fp32 31 us (rows of
// stride 2049, inputs in L2: 39 us from memory).
template <typename T, bool PACKED, bool VEC, int TPR>
__global__ void __launch_bounds__(TPR < 512 ? 512 : TPR, 1)
    norm_back_kernel(const __grid_constant__ NormBackArgs a, int stages, int dy_bytes, int x_bytes)
{
    using S = BackShape<T, PACKED, VEC, TPR>;
    constexpr int E = S::E, U = S::U, UNITS = S::UNITS, ROWS = S::ROWS, THREADS = S::THREADS, GROUPS = S::GROUPS;
    constexpr int WARPS = TPR / 32;
    constexpr int PAIRS = VEC ? U / 2 : 1, SINGLE = VEC ? 1 : 2;  // of a unit; single values that make a pair
    extern __shared__ uint8_t raw_ring[];
    __shared__ uint64_t bars[S::SYNCS][BACK_MAX_STAGES];
    __shared__ float4 shared[2][THREADS / 32];
    __shared__ float columns[GROUPS > 1 ? 2 * TPR * E : 1];
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const int sync = threadIdx.x / S::SYNC, in_sync = threadIdx.x % S::SYNC;
    uint64_t *full = bars[sync];
    const int column = lane * U, cols = a.cols - column;
    const float inv_cols = 1.0f / (float)a.cols;
    const int row_bytes = dy_bytes + x_bytes, stage_bytes = S::TAKEN * row_bytes;
    uint8_t *ring = raw_ring + ((128u - (ptx::smem_addr(raw_ring) & 127u)) & 127u) + sync * stages * stage_bytes;
    constexpr bool X_UNITS = VEC || PACKED;  // rows of x on 16-byte boundaries
    const int dy_row_bytes = a.cols * (int)sizeof(T), x_row_bytes = a.cols * (int)sizeof(typename S::X);
    const int dy_tail = VEC ? dy_row_bytes & 15 : 0, x_tail = VEC ? x_row_bytes & 15 : 0;

    const int step = (int)gridDim.x * S::SYNCS * S::TAKEN, begin = ((int)blockIdx.x * S::SYNCS + sync) * S::TAKEN;
    // one thread: the rows from `first` on into a stage
    const auto request = [&](int first, int stage) {
        const int rows = min(S::TAKEN, a.rows - first);
        uint8_t *to = ring + stage * stage_bytes;
        const uint8_t *dy = reinterpret_cast<const uint8_t *>(static_cast<const T *>(a.dy) + first * a.dy_stride);
        const uint8_t *x = reinterpret_cast<const uint8_t *>(static_cast<const typename S::X *>(a.x) + first * a.x_stride);
        const long long dy_step = a.dy_stride * (long long)sizeof(T), x_step = a.x_stride * (long long)sizeof(typename S::X);
        if constexpr (VEC) {
            const int dy_whole = dy_row_bytes & ~15, x_whole = x_row_bytes & ~15;
            ptx::mbar_arrive_expect_tx(&full[stage], rows * (dy_whole + x_whole));
            for (int r = 0; r < rows; ++r, to += row_bytes, dy += dy_step, x += x_step) {
                if (dy_whole) ptx::bulk_load(to, dy, dy_whole, &full[stage]);
                if (x_whole) ptx::bulk_load(to + dy_bytes, x, x_whole, &full[stage]);
                if (dy_tail) copy_filled(to + dy_whole, dy + dy_whole, dy_tail);
                if (x_tail) copy_filled(to + dy_bytes + x_whole, x + x_whole, x_tail);
            }
            if (dy_tail || x_tail)  // arrives when this thread's own copies have landed
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(ptx::smem_addr(&full[stage])) : "memory");
        } else {
            int bytes = 0;
            for (int r = 0; r < rows; ++r)
                bytes += around(dy + r * dy_step, dy_row_bytes) + around(x + r * x_step, x_row_bytes);
            ptx::mbar_arrive_expect_tx(&full[stage], bytes);
            for (int r = 0; r < rows; ++r, to += row_bytes, dy += dy_step, x += x_step) {
                ptx::bulk_load(to, dy - ((uintptr_t)dy & 15), around(dy, dy_row_bytes), &full[stage]);
                ptx::bulk_load(to + dy_bytes, x - ((uintptr_t)x & 15), around(x, x_row_bytes), &full[stage]);
            }
        }
    };
    if (in_sync == 0) {
        for (int s = 0; s < stages; ++s) ptx::mbar_init(&full[s], dy_tail || x_tail ? 2 : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (in_sync == 0)
        for (int s = 0; s < stages; ++s)
            if (begin + s * (long long)step < a.rows) request(begin + s * step, s);

    f32x2 gamma[E / 2], sum_g[E / 2], sum_b[E / 2];
#pragma unroll
    for (int e = 0; e < E / 2; ++e) {
        sum_g[e] = sum_b[e] = 0ull;
        gamma[e] = pair_of(1.0f);
    }
    if (a.gamma) {
#pragma unroll
        for (int j = 0; j < UNITS; j += SINGLE) {
            const int c = column + j * TPR * U;
            if constexpr (VEC) {
                if (c < a.cols) param_pairs<U>(a.gamma, a.params_bf16, a.gamma_aligned, c, a.cols, gamma + j * PAIRS);
            } else {
                gamma[j / 2] = pair_of(c < a.cols ? load_param(a.gamma, a.params_bf16, c) : 0.0f,
                                       c + TPR < a.cols ? load_param(a.gamma, a.params_bf16, c + TPR) : 0.0f);
            }
        }
    }

    int row = begin + in_sync / TPR * ROWS;
    // of the next rows; two rows that are taken together lie in one row of scales
    float mean_ahead[ROWS], rstd_ahead[ROWS];
    uint8_t scale_ahead[PACKED ? UNITS : 1];
    const auto look_ahead = [&](int row) {
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            if (row + k < a.rows) {
                mean_ahead[k] = a.mean[row + k];
                rstd_ahead[k] = a.rstd[row + k];
            }
        }
        if (PACKED && row < a.rows) {
            const uint8_t *scales = a.scales + (long long)(row / PACK_BLOCK) * a.scale_cols + column / PACK_BLOCK;
#pragma unroll
            for (int j = 0; j < UNITS; ++j)
                if (j * TPR * U < cols)
                    scale_ahead[PACKED ? j : 0] = TPR * U % PACK_BLOCK == 0 ? scales[j * (TPR * U / PACK_BLOCK)]
                                                                          : scales[(column + j * TPR * U) / PACK_BLOCK - column / PACK_BLOCK];
        }
    };
    look_ahead(row);
    T *dx = static_cast<T *>(a.dx) + row * a.dx_stride + column;
    // where a row starts inside its first unit
    unsigned dy_at = (unsigned)(uintptr_t)(static_cast<const T *>(a.dy) + row * a.dy_stride);
    unsigned x_at = (unsigned)(uintptr_t)(static_cast<const typename S::X *>(a.x) + row * a.x_stride);
    const unsigned dy_step = (unsigned)(a.dy_stride * (long long)sizeof(T)), x_step = (unsigned)(a.x_stride * (long long)sizeof(typename S::X));
    int parity = 0, stage = 0;
    unsigned phase = 0;
    for (int first = begin; first < a.rows; first += step, row += step) {
        if (!__all_sync(0xffffffffu, bounded_wait(&full[stage], phase, &g_norm_error, 1))) {
            for (int i = 0; i < 2000; ++i) __nanosleep(1000);  // copies in flight land before the block ends
            // other warps may have seen the rows arrive: the barriers that they come to are met
            if constexpr (TPR > 32 && GROUPS > 1)
                for (; first < a.rows; first += step) asm volatile("bar.sync %0, %1;" ::"r"(1 + sync), "n"(S::SYNC) : "memory");
            return;
        }
        const uint8_t *mine = ring + stage * stage_bytes + in_sync / TPR * ROWS * row_bytes;
        // the pairs of dy of unit j, or of single values j and j + 1, of row k
        const auto dy_pairs = [&](int k, int j, f32x2 *p) {
            if constexpr (VEC) {
                widen_pairs<T>(reinterpret_cast<const uint4 *>(mine + k * row_bytes)[lane + j * TPR], p);
            } else {
                const T *r = reinterpret_cast<const T *>(mine + k * row_bytes + (dy_at + k * dy_step & 15u)) + column + j * TPR;
                const bool both = (j + 1) * TPR < cols;
                p[0] = pair_of(widen1<T>(r[0]), both ? widen1<T>(r[TPR]) : 0.0f);
            }
        };
        f32x2 hat[ROWS][E / 2];
        f32x2 sum2[4] = {0ull, 0ull, 0ull, 0ull};  // of g and g h, of either row
        float rstd[ROWS];
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            rstd[k] = rstd_ahead[k];
            if (row + k < a.rows) {
#pragma unroll
                for (int j = 0; j < UNITS; j += SINGLE) {
                    const int c = j * TPR * U;
                    if (c < cols) {
                        f32x2 dy[PAIRS], *h = hat[k] + j * PAIRS / SINGLE;
                        dy_pairs(k, j, dy);
                        const uint8_t *at = mine + k * row_bytes + dy_bytes;
                        if constexpr (VEC) {
                            const typename S::RawX x = reinterpret_cast<const typename S::RawX *>(at)[lane + j * TPR];
                            S::centred(&x, PACKED ? scale_value(scale_ahead[PACKED ? j : 0]) : 0.0f, 0.0f, mean_ahead[k], h);
                        } else {
                            const typename S::RawX *r =
                                reinterpret_cast<const typename S::RawX *>(at + (X_UNITS ? 0u : x_at + k * x_step & 15u)) + column + c;
                            const bool both = c + TPR < cols;  // the second value is inside too
                            const typename S::RawX x[2] = {r[0], r[both ? TPR : 0]};
                            S::centred(x, PACKED ? scale_value(scale_ahead[PACKED ? j : 0]) : 0.0f,
                                       PACKED ? scale_value(scale_ahead[PACKED ? (both ? j + 1 : j) : 0]) : 0.0f, mean_ahead[k], h);
                        }
#pragma unroll
                        for (int i = 0; i < PAIRS; ++i) {
                            const int e = j * PAIRS / SINGLE + i;
                            h[i] = mul2(h[i], pair_of(rstd[k]));
                            const f32x2 p = mul2(dy[i], h[i]);
                            sum_g[e] = add2(sum_g[e], p);
                            sum_b[e] = add2(sum_b[e], dy[i]);
                            sum2[2 * k] = fma2(dy[i], gamma[e], sum2[2 * k]);
                            sum2[2 * k + 1] = fma2(p, gamma[e], sum2[2 * k + 1]);
                        }
                    }
                }
            }
        }
        float sums[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[i] = sum_of(sum2[i]);
        look_ahead(row + step);
        if constexpr (TPR < 32) {
#pragma unroll
            for (int i = 0; i < 2 * ROWS; ++i)
#pragma unroll
                for (int o = TPR / 2; o > 0; o >>= 1) sums[i] += __shfl_xor_sync(0xffffffffu, sums[i], o);
        } else {
            const float s = warp_sum4(sums);
            if constexpr (TPR == 32) {
#pragma unroll
                for (int i = 0; i < 2 * ROWS; ++i) sums[i] = __shfl_sync(0xffffffffu, s, 8 * i);
            } else {
                const int warp = threadIdx.x >> 5;
                if ((threadIdx.x & 7) == 0) reinterpret_cast<float *>(&shared[parity][warp])[(threadIdx.x & 31) >> 3] = s;
            }
        }
        // Behind this barrier every thread is done with the rows before these: their stage is free, and so
        // are the slots of `shared` that the next rows use.
        if constexpr (TPR <= 32)
            __syncwarp();
        else if constexpr (GROUPS == 1)
            __syncthreads();
        else
            asm volatile("bar.sync %0, %1;" ::"r"(1 + sync), "n"(S::SYNC) : "memory");
        if constexpr (TPR > 32) {
            sums[0] = sums[1] = sums[2] = sums[3] = 0.0f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float4 q = shared[parity][group * WARPS + w];
                sums[0] += q.x; sums[1] += q.y; sums[2] += q.z; sums[3] += q.w;
            }
            parity ^= 1;
        }
        const long long next = first + (stages - 1) * (long long)step;
        if (in_sync == 0 && first != begin && next < a.rows) request((int)next, stage == 0 ? stages - 1 : stage - 1);
        if (a.dx) {
#pragma unroll
            for (int k = 0; k < ROWS; ++k) {
                if (row + k >= a.rows) continue;
                const f32x2 g1 = pair_of(-sums[2 * k] * inv_cols), g2 = pair_of(-sums[2 * k + 1] * inv_cols);
                T *out = dx + k * a.dx_stride;
#pragma unroll
                for (int j = 0; j < UNITS; j += SINGLE) {
                    const int c = j * TPR * U;
                    if (c >= cols) continue;
                    f32x2 r[PAIRS];
                    dy_pairs(k, j, r);
#pragma unroll
                    for (int i = 0; i < PAIRS; ++i) {
                        const int e = j * PAIRS / SINGLE + i;
                        r[i] = mul2(fma2(hat[k][e], g2, fma2(r[i], gamma[e], g1)), pair_of(rstd[k]));
                    }
                    if constexpr (VEC) {
                        const uint4 unit = narrow_pairs<T>(r);
                        if (c + U <= cols)
                            *reinterpret_cast<uint4 *>(out + c) = unit;
                        else
                            store_first(out + c, unit, cols - c);
                    } else {
                        const float2 v = values_of(r[0]);
                        out[c] = narrow1<T>(v.x);
                        if (c + TPR < cols) out[c + TPR] = narrow1<T>(v.y);
                    }
                }
            }
        }
        dx += step * a.dx_stride;
        dy_at += step * dy_step;
        x_at += step * x_step;
        if (++stage == stages) { stage = 0; phase ^= 1; }
    }

    if (!a.dgamma && !a.dbeta) return;
    // the column of value e of this thread
    const auto column_of = [&](int e) { return VEC ? (e / U * TPR + lane) * U + e % U : e * TPR + lane; };
    if constexpr (GROUPS > 1) {  // the block's groups in ascending order
        for (int g = 0; g < GROUPS; ++g) {
            __syncthreads();
            if (group == g) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int at = column_of(e);
                    const float2 vg = values_of(sum_g[e / 2]), vb = values_of(sum_b[e / 2]);
                    columns[at] = (g ? columns[at] : 0.0f) + (e & 1 ? vg.y : vg.x);
                    columns[TPR * E + at] = (g ? columns[TPR * E + at] : 0.0f) + (e & 1 ? vb.y : vb.x);
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
            const int c = column_of(e);
            const float2 vg = values_of(sum_g[e / 2]), vb = values_of(sum_b[e / 2]);
            if (c < a.cols) {
                if (a.dgamma) a.dgamma[blockIdx.x * a.part_stride + c] = e & 1 ? vg.y : vg.x;
                if (a.dbeta) a.dbeta[blockIdx.x * a.part_stride + c] = e & 1 ? vb.y : vb.x;
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

// The blocks' sums, in the order of the blocks within each of 32 strands and then of the strands.  A second
// launch instead of atomics: the order never changes.  At most 148 rows of sums, about 3 us.
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

constexpr int BACK_LONG_SHARES = 32;
constexpr int BACK_RING = 192 * 1024;  // bytes of shared memory for rows on their way

// The widest row that a block holds, and the threads for a row: 32 bytes each.
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
    const int tpr = back_threads_per_row(cols, dtype), rows_at_once = tpr <= 256 ? 2 : 1;
    return std::min<int64_t>(148, ceil_div(rows, std::max(tpr, 512) / tpr * rows_at_once));
}

template <typename T, bool PACKED, bool VEC, int TPR>
int launch_back_shape(const NormBackArgs &a, int blocks, cudaStream_t stream)
{
    using S = BackShape<T, PACKED, VEC, TPR>;
    // of a row in shared memory; rows that start inside a unit can take one more
    const int dy_bytes = (int)ceil_div(a.cols * (int)sizeof(T), 16) * 16 + (VEC ? 0 : 16);
    const int x_bytes = (int)ceil_div(a.cols * (int)sizeof(typename S::X), 16) * 16 + (VEC || PACKED ? 0 : 16);
    const int stage = S::SYNCS * S::TAKEN * (dy_bytes + x_bytes);
    // a stage takes 64 KB and some for rows off 16-byte boundaries at most
    const int stages = std::max(2, std::min(BACK_MAX_STAGES, BACK_RING / stage)), smem = stages * stage + 128;
    // always the largest there can be: threads that launch different sizes share the attribute
    if (cudaFuncSetAttribute(norm_back_kernel<T, PACKED, VEC, TPR>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             BACK_RING + 128) != cudaSuccess)
        return launch_status();
    norm_back_kernel<T, PACKED, VEC, TPR><<<blocks, S::THREADS, smem, stream>>>(a, stages, dy_bytes, x_bytes);
    return launch_status();
}

template <typename T, bool PACKED, bool VEC>
int launch_back(const NormBackArgs &a, int blocks, cudaStream_t stream)
{
    switch (back_threads_per_row(a.cols, sizeof(T) == 2 ? DIPACO_BF16 : DIPACO_F32)) {
    case 8: return launch_back_shape<T, PACKED, VEC, 8>(a, blocks, stream);
    case 16: return launch_back_shape<T, PACKED, VEC, 16>(a, blocks, stream);
    case 32: return launch_back_shape<T, PACKED, VEC, 32>(a, blocks, stream);
    case 64: return launch_back_shape<T, PACKED, VEC, 64>(a, blocks, stream);
    case 128: return launch_back_shape<T, PACKED, VEC, 128>(a, blocks, stream);
    case 256: return launch_back_shape<T, PACKED, VEC, 256>(a, blocks, stream);
    case 512: return launch_back_shape<T, PACKED, VEC, 512>(a, blocks, stream);
    default: return launch_back_shape<T, PACKED, VEC, 1024>(a, blocks, stream);
    }
}

template <typename T, bool PACKED>
int launch_back_any(const NormBackArgs &a, int blocks, bool vec, cudaStream_t stream)
{
    if (a.cols > back_widest(sizeof(T) == 2 ? DIPACO_BF16 : DIPACO_F32)) {
        if (a.dx) norm_back_long_rows_kernel<T, PACKED><<<a.rows, 1024, 0, stream>>>(a);
        if (a.dgamma || a.dbeta)
            norm_back_long_columns_kernel<T, PACKED>
                <<<dim3((unsigned)ceil_div(a.cols, 256), blocks), 256, 0, stream>>>(a);
        return launch_status();
    }
    return vec ? launch_back<T, PACKED, true>(a, blocks, stream) : launch_back<T, PACKED, false>(a, blocks, stream);
}

// A warp waits, for a limited time, on a barrier that nothing completes: no copy is in flight.
__global__ void __launch_bounds__(32) wait_expiry_kernel(unsigned long long limit_ns)
{
    __shared__ uint64_t bar;
    if (threadIdx.x == 0) {
        ptx::mbar_init(&bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    __all_sync(0xffffffffu, bounded_wait(&bar, 0, &g_norm_error, 9, limit_ns));
}

} // namespace

bool dipaco::take_norm_error(bool &expired) { return take_error_word(g_norm_error, expired); }

int dipaco::expire_norm_wait(unsigned long long limit_ns, cudaStream_t stream)
{
    wait_expiry_kernel<<<1, 32, 0, stream>>>(limit_ns);
    return launch_status();
}

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
    if (rows == 0 || (cols == 0 && !mean && !rstd)) return DIPACO_OK;

    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (cols == 0) {  // statistics of nothing: bytes of ones are a NaN
        if (mean && cudaMemsetAsync(mean, 0xff, rows * sizeof(float), stream) != cudaSuccess) return launch_status();
        if (rstd && cudaMemsetAsync(rstd, 0xff, rows * sizeof(float), stream) != cudaSuccess) return launch_status();
        return DIPACO_OK;
    }
    NormArgs a = {x, y, gamma, beta, mean, rstd, x_stride, y_stride, (int)rows, (int)cols, eps, 1.0f / (float)cols,
                  param_dtype == DIPACO_BF16};
    const int size = dense_size(dtype);
    const bool vec = rows_aligned16(x, x_stride, rows, size) && (!y || rows_aligned16(y, y_stride, rows, size));
    const int mode = !vec ? ROWS_SINGLE : cols * size % 16 ? ROWS_RAGGED : ROWS_UNITS;
    if (dtype == DIPACO_BF16)
        return mode == ROWS_SINGLE  ? launch_norm<__nv_bfloat16, ROWS_SINGLE>(a, stream)
               : mode == ROWS_UNITS ? launch_norm<__nv_bfloat16, ROWS_UNITS>(a, stream)
                                    : launch_norm<__nv_bfloat16, ROWS_RAGGED>(a, stream);
    return mode == ROWS_SINGLE  ? launch_norm<float, ROWS_SINGLE>(a, stream)
           : mode == ROWS_UNITS ? launch_norm<float, ROWS_UNITS>(a, stream)
                                : launch_norm<float, ROWS_RAGGED>(a, stream);
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
    const int size = dense_size(dtype);
    const bool vec = rows_aligned16(dy, dy_stride, rows, size) && (!x || rows_aligned16(x, x_stride, rows, size)) &&
                     (!dx || rows_aligned16(dx, dx_stride, rows, size));
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
    if (const int rc = dtype == DIPACO_BF16 ? (x ? launch_back_any<__nv_bfloat16, false>(a, parts, vec, stream)
                                                 : launch_back_any<__nv_bfloat16, true>(a, parts, vec, stream))
                                            : (x ? launch_back_any<float, false>(a, parts, vec, stream)
                                                 : launch_back_any<float, true>(a, parts, vec, stream)))
        return rc;
    if (parts > 1 && (dgamma || dbeta))
        norm_back_join_kernel<<<dim3((unsigned)ceil_div(cols, 32), 2), 1024, 0, stream>>>(
            a.dgamma, a.dbeta, parts, a.part_stride, (int)cols, dgamma, dbeta);
    return launch_status();
}

} // extern "C"
