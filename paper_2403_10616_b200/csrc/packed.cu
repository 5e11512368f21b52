// Packed matrices: conversion from and to dense ones, the layer norm and the GELU that write their
// result and their input as packed checkpoints, and the GELU's gradient from such a checkpoint (see
// include/dipaco.h for the format).
//
//   gelu(a) = a s, s = 1 / (1 + exp(-2u)), u = sqrt(2/pi) (a + 0.044715 a^3)   (the tanh form: 2s = 1 + tanh u)
//   gelu'(a) = s + a s (1 - s) 2 u',  u' = sqrt(2/pi) (1 + 3 * 0.044715 a^2)
//
// One block of threads per block of 128 x 128 values, which is read once: the largest magnitude has to be
// known before the first code is.
//
//   stream_kernel  bf16 rows on 16-byte boundaries: persistent, the copy engine brings the next blocks to
//                  shared memory while one is worked on
//   block_kernel   fp32, and rows at any alignment: the values are loaded to registers
//
// Measured on 32768x3584 in bf16: pack 59 us (6.0 TB/s: bound by memory), GELU with both results 102 to 104 us
// and its gradient 102 to 106 us (4.5 TB/s).  Powers and reciprocals, two for a value, would take 52 us of those two,
// instructions 60 and memory 72: the three overlap in part.  The norm's two launches on 32768x896 take
// 41 us, 13 of them for the statistics; its second reads x from L2.  From fp32 (block_kernel) the GELU and its
// gradient take 182 and 214 us, and the norm of 32768x896 takes 85 us with its statistics: they spill registers.
#include "activations.cuh"
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

// Magnitudes of pairs of bf16 values: the larger of each half (NaN only where both are), and the larger half
// as the bits of an fp32 value.
__device__ __forceinline__ unsigned larger_bf16x2(unsigned magnitudes, unsigned w)
{
    asm("max.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(magnitudes) : "r"(w));  // the sign is not used
    return magnitudes;
}
__device__ __forceinline__ unsigned wider_bf16x2(unsigned magnitudes)
{
    magnitudes &= 0x7fff7fffu;
    return max(magnitudes << 16, magnitudes & 0xffff0000u);
}

__device__ __forceinline__ float larger(float magnitude, f32x2 p)  // NaN does not count
{
    const float2 v = values_of(p);
    asm("max.abs.f32 %0, %0, %1, %2;" : "+f"(magnitude) : "f"(v.x), "f"(v.y));
    return magnitude;
}

// The thread's values of one matrix: as they were loaded, or computed in fp32.
template <typename T> struct LoadedValues {
    const uint4 *raw;
    __device__ __forceinline__ void unit(int j, f32x2 *p) const { widen_pairs<T>(raw[j], p); }
    __device__ __forceinline__ void unit_at(int j, f32x2 *p) const  // j not known when compiling
    {
        uint4 r = raw[0];
#pragma unroll
        for (int k = 1; k < Layout<T>::UNITS; ++k)
            if (j == k) r = raw[k];
        widen_pairs<T>(r, p);
    }
    // Bits of the largest magnitude; at least those of infinity if there is an infinity.
    __device__ __forceinline__ unsigned largest() const
    {
        unsigned m = 0u;
#pragma unroll
        for (int j = 0; j < Layout<T>::UNITS; ++j) {
            const unsigned w[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 2)
                    m = larger_bf16x2(m, w[i]);
                else
                    m = max(m, w[i] & 0x7fffffffu);
            }
        }
        return sizeof(T) == 2 ? wider_bf16x2(m) : m;
    }
};
template <typename T> struct ComputedValues {
    const f32x2 *v;
    __device__ __forceinline__ void unit(int j, f32x2 *p) const
    {
#pragma unroll
        for (int i = 0; i < Layout<T>::U / 2; ++i) p[i] = v[j * Layout<T>::U / 2 + i];
    }
    __device__ __forceinline__ void unit_at(int j, f32x2 *p) const
    {
        unit(0, p);
#pragma unroll
        for (int k = 1; k < Layout<T>::UNITS; ++k)
            if (j == k) unit(k, p);
    }
    __device__ __forceinline__ unsigned largest() const  // of the values that are not NaN
    {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < VALUES / 2; ++i) m = larger(m, v[i]);
        return __float_as_uint(m);
    }
};

template <int U, bool SPECIAL>
__device__ __forceinline__ void store_codes(uint8_t *p, int n, const f32x2 *v, float reciprocal)
{
    unsigned w[U / 4];
#pragma unroll
    for (int i = 0; i < U / 4; ++i) {
        if constexpr (SPECIAL) {
            const float2 a = values_of(v[2 * i]), b = values_of(v[2 * i + 1]);
            const float f[4] = {a.x, a.y, b.x, b.y};
            w[i] = encode4(f, reciprocal);
        } else {
            w[i] = encode4_finite(v + 2 * i, pair_of(reciprocal));
        }
    }
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

// Writes the codes and the scale of block `index`, given the bits m of its largest magnitude.  Infinities
// are rare: where m is not finite, the block looks for its largest finite magnitude and encodes with care.
template <typename T, typename Values>
__device__ __forceinline__ void write_codes(const PackedOut &out, const Extent &x, long long index, int row0, int col,
                                            bool edge, const Values &v, unsigned m, unsigned *shared)
{
    using L = Layout<T>;
    const bool special = m >= 0x7f800000u;
    if (special) {
        m = 0u;
#pragma unroll
        for (int j = 0; j < L::UNITS; ++j) {
            f32x2 f[L::U / 2];
            v.unit(j, f);
#pragma unroll
            for (int i = 0; i < L::U / 2; ++i)
                m = max(m, max(finite_magnitude(values_of(f[i]).x), finite_magnitude(values_of(f[i]).y)));
        }
        m = block_max(m, shared);
    }
    const unsigned byte = scale_byte(m);
    const float reciprocal = scale_reciprocal(byte);
    if (threadIdx.x == 0) out.scales[index] = (uint8_t)byte;
    uint8_t *p = out.codes + row0 * out.stride + col;
    const long long step = L::STEP * out.stride;
    if (!edge && !special) {
#pragma unroll
        for (int j = 0; j < L::UNITS; ++j) {
            f32x2 f[L::U / 2];
            v.unit(j, f);
            store_codes<L::U, false>(p, L::U, f, reciprocal);
            p += step;
        }
        return;
    }
    if (col >= x.cols) return;
#pragma unroll 1
    for (int j = 0; j < L::UNITS; ++j) {
        if (row0 + j * L::STEP < x.rows) {
            f32x2 f[L::U / 2];
            v.unit_at(j, f);
            store_codes<L::U, true>(p, x.cols - col, f, reciprocal);
        }
        p += step;
    }
}

enum : int { OP_PACK, OP_NORM, OP_GELU, OP_GELU_BACK, OP_ACTIVATE };  // OP_ACTIVATE: of block_kernel

struct BlockArgs {
    const void *x;  // dense input (the gradient for OP_GELU_BACK)
    long long x_stride;
    bool aligned;
    Extent extent;
    PackedOut first;   // the packed result
    PackedOut second;  // the packed input (OP_NORM, OP_GELU, OP_ACTIVATE); codes NULL: not wanted
    int activation;    // OP_ACTIVATE
    // OP_GELU_BACK: the packed input of the GELU
    const uint8_t *codes, *scales;
    long long codes_stride;
    // OP_NORM
    const float *mean, *rstd;
    const void *gamma, *beta;
    bool params_bf16, gamma_aligned, beta_aligned;
};

// gamma and beta of U columns.
template <int U> __device__ __forceinline__ void norm_params(const BlockArgs &a, int col, f32x2 *gamma, f32x2 *beta)
{
#pragma unroll
    for (int i = 0; i < U / 2; ++i) { gamma[i] = pair_of(1.0f); beta[i] = 0ull; }
    if (a.gamma) param_pairs<U>(a.gamma, a.params_bf16, a.gamma_aligned, col, a.extent.cols, gamma);
    if (a.beta) param_pairs<U>(a.beta, a.params_bf16, a.beta_aligned, col, a.extent.cols, beta);
}
template <int U>
__device__ __forceinline__ void normalise(f32x2 *f, float mean, float rstd, const f32x2 *gamma, const f32x2 *beta)
{
#pragma unroll
    for (int i = 0; i < U / 2; ++i) f[i] = fma2(mul2(add2(f[i], pair_of(-mean)), pair_of(rstd)), gamma[i], beta[i]);
}

template <typename T, int OP>
__global__ void __launch_bounds__(THREADS, 2) block_kernel(const __grid_constant__ BlockArgs a)
{
    using L = Layout<T>;
    constexpr int U = L::U;
    __shared__ unsigned shared[4][THREADS / 32];
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
        write_codes<T>(a.first, a.extent, blockIdx.x, row0, col, edge, loaded, block_max(loaded.largest(), shared[0]), shared[1]);
        return;
    }

    f32x2 y[VALUES / 2];
    if constexpr (OP == OP_NORM) {
        f32x2 gamma[U / 2], beta[U / 2];
        norm_params<U>(a, col, gamma, beta);
#pragma unroll
        for (int j = 0; j < L::UNITS; ++j) {
            const int r = row0 + j * L::STEP;
            const float mean = r < rows ? a.mean[r] : 0.0f, rstd = r < rows ? a.rstd[r] : 0.0f;
            f32x2 *f = y + j * U / 2;
            loaded.unit(j, f);
            normalise<U>(f, mean, rstd, gamma, beta);
            if (edge) keep_inside<U>(f, r < rows ? cols - col : 0);
        }
    } else if constexpr (OP == OP_GELU) {
#pragma unroll
        for (int j = 0; j < L::UNITS; ++j) {
            f32x2 *f = y + j * U / 2;
            loaded.unit(j, f);
#pragma unroll
            for (int i = 0; i < U / 2; ++i) f[i] = gelu(f[i]);
        }
    } else if constexpr (OP == OP_ACTIVATE) {
#pragma unroll
        for (int j = 0; j < L::UNITS; ++j) {
            f32x2 *f = y + j * U / 2;
            loaded.unit(j, f);
#pragma unroll
            for (int i = 0; i < U / 2; ++i)
                f[i] = a.activation == DIPACO_ACTIVATION_SILU ? activate<DIPACO_ACTIVATION_SILU>(f[i])
                                                              : activate<DIPACO_ACTIVATION_RELU>(f[i]);
        }
    } else {
        const f32x2 scale = pair_of(scale_value(a.scales[blockIdx.x]));
        const uint8_t *q = a.codes + (long long)row0 * a.codes_stride + col;
#pragma unroll
        for (int j = 0; j < L::UNITS; ++j) {
            f32x2 *f = y + j * U / 2;
            loaded.unit(j, f);
            const bool in = !edge || (row0 + j * L::STEP < rows && col < cols);
#pragma unroll
            for (int i = 0; i < U; i += 4) {
                // rows of codes are padded to 16 bytes: four of them can be read wherever one can
                const unsigned w = in && (!edge || col + i < cols) ? *reinterpret_cast<const unsigned *>(q + i) : 0u;
                f[i / 2] = mul2(f[i / 2], gelu_slope(mul2(decode_pair(w), scale)));
                f[i / 2 + 1] = mul2(f[i / 2 + 1], gelu_slope(mul2(decode_pair(w >> 16), scale)));
            }
            if (edge) keep_inside<U>(f, cols - col);
            q += L::STEP * a.codes_stride;
        }
    }
    const ComputedValues<T> computed = {y};
    write_codes<T>(a.first, a.extent, blockIdx.x, row0, col, edge, computed, block_max(computed.largest(), shared[0]), shared[1]);
    if (OP != OP_GELU_BACK && a.second.codes)
        write_codes<T>(a.second, a.extent, blockIdx.x, row0, col, edge, loaded, block_max(loaded.largest(), shared[2]), shared[3]);
}

// ------------------------------------------------------------------------------------------ streamed blocks

static __device__ int g_packing_error;  // set by a bounded wait that ran out

constexpr int DENSE_BYTES = PACK_BLOCK * PACK_BLOCK * 2;  // of a block in bf16
constexpr int CODE_BYTES = PACK_BLOCK * PACK_BLOCK;

// Buffers for blocks on their way.  A buffer is free once every thread is past the barrier of the block in
// it (OP_GELU_BACK, which has read it then) or of the next block (the others read it again to pack it).
template <int OP> struct Stream {
    static constexpr int BUFFERS = OP == OP_GELU_BACK ? 2 : 3;
    static constexpr int BYTES = DENSE_BYTES + (OP == OP_GELU_BACK ? CODE_BYTES : 0);
    static constexpr int SMEM = BUFFERS * BYTES + 128;
};

// A thread's values in shared memory: as LoadedValues.
struct SharedValues {
    const uint4 *unit0;
    __device__ __forceinline__ uint4 at(int j) const { return unit0[j * THREADS]; }
    __device__ __forceinline__ void unit(int j, f32x2 *p) const { widen_pairs<__nv_bfloat16>(at(j), p); }
    __device__ __forceinline__ void unit_at(int j, f32x2 *p) const { unit(j, p); }
};

__device__ __forceinline__ void load_box(void *to, const CUtensorMap *map, int x, int y, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
            ptx::smem_addr(to)),
        "l"(map), "r"(x), "r"(y), "r"(ptx::smem_addr(bar))
        : "memory");
}

template <int OP>
__global__ void __launch_bounds__(THREADS, 2)
    stream_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap codes_map,
                  const __grid_constant__ BlockArgs a, int blocks)
{
    using T = __nv_bfloat16;
    using L = Layout<T>;
    using S = Stream<OP>;
    constexpr int U = L::U;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t full[S::BUFFERS];
    __shared__ unsigned maxima[2][2][THREADS / 32], special[2][THREADS / 32];
    uint8_t *buffers = raw + ((128u - (ptx::smem_addr(raw) & 127u)) & 127u);
    const int rows = a.extent.rows, cols = a.extent.cols;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;

    if (threadIdx.x == 0) {
        for (int b = 0; b < S::BUFFERS; ++b) ptx::mbar_init(&full[b], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    const auto request = [&](int index, int buffer) {  // one thread
        ptx::mbar_arrive_expect_tx(&full[buffer], S::BYTES);
        const int x = index % a.extent.block_cols * PACK_BLOCK, y = index / a.extent.block_cols * PACK_BLOCK;
        load_box(buffers + buffer * S::BYTES, &x_map, x, y, &full[buffer]);
        if (OP == OP_GELU_BACK) load_box(buffers + buffer * S::BYTES + DENSE_BYTES, &codes_map, x, y, &full[buffer]);
    };
    if (threadIdx.x == 0)
        for (int b = 0; b < S::BUFFERS; ++b)
            if (blockIdx.x + (long long)b * gridDim.x < blocks) request(blockIdx.x + b * gridDim.x, b);

    f32x2 gamma[U / 2], beta[U / 2];  // of the columns from `held` on
    int held = -1;
    int buffer = 0, previous = S::BUFFERS - 1;
    unsigned phase = 0, turn = 0;
    // the block's place among the blocks, moved on without a division
    const int rows_on = gridDim.x / a.extent.block_cols * PACK_BLOCK, cols_on = gridDim.x % a.extent.block_cols * PACK_BLOCK;
    const int all_cols = a.extent.block_cols * PACK_BLOCK;
    int first_row = blockIdx.x / a.extent.block_cols * PACK_BLOCK, col0 = blockIdx.x % a.extent.block_cols * PACK_BLOCK;
    for (int index = blockIdx.x; index < blocks; index += gridDim.x) {
        const int row0 = first_row + (int)threadIdx.x / L::PER_ROW;
        const int col = col0 + (int)(threadIdx.x % L::PER_ROW) * U;
        float mean[L::UNITS], rstd[L::UNITS];
        if constexpr (OP == OP_NORM) {
            if (col0 != held) norm_params<U>(a, col, gamma, beta);
            held = col0;
#pragma unroll
            for (int j = 0; j < L::UNITS; ++j) {
                const int r = min(row0 + j * L::STEP, rows - 1);
                mean[j] = a.mean[r];
                rstd[j] = a.rstd[r];
            }
        }
        const f32x2 scale = pair_of(OP == OP_GELU_BACK ? scale_value(a.scales[index]) : 0.0f);
        const bool edge = col0 + PACK_BLOCK > cols || first_row + PACK_BLOCK > rows;
        const SharedValues x = {reinterpret_cast<const uint4 *>(buffers + buffer * S::BYTES) + threadIdx.x};
        if (!__all_sync(0xffffffffu, bounded_wait(&full[buffer], phase, &g_packing_error, 1))) {  // whole warps leave
            for (int i = 0; i < 2000; ++i) __nanosleep(1000);  // copies in flight land before the block ends
            return;
        }

        f32x2 y[OP == OP_PACK ? 1 : VALUES / 2];
        unsigned mx = 0u;
        float my = 0.0f;
#pragma unroll
        for (int j = 0; j < L::UNITS; ++j) {
            const uint4 unit = x.at(j);  // zero outside the matrix
            if constexpr (OP != OP_GELU_BACK) {
                mx = larger_bf16x2(mx, unit.x);
                mx = larger_bf16x2(mx, unit.y);
                mx = larger_bf16x2(mx, unit.z);
                mx = larger_bf16x2(mx, unit.w);
            }
            if constexpr (OP != OP_PACK) {
                f32x2 *f = y + j * U / 2;
                widen_pairs<T>(unit, f);
                if constexpr (OP == OP_NORM) {
                    normalise<U>(f, mean[j], rstd[j], gamma, beta);
                } else if constexpr (OP == OP_GELU) {
#pragma unroll
                    for (int i = 0; i < U / 2; ++i) f[i] = gelu(f[i]);
                } else {
                    const uint2 c = reinterpret_cast<const uint2 *>(buffers + buffer * S::BYTES + DENSE_BYTES)[threadIdx.x + j * THREADS];
#pragma unroll
                    for (int i = 0; i < U / 2; ++i)
                        f[i] = mul2(f[i], gelu_slope(mul2(decode_pair((i < 2 ? c.x : c.y) >> (16 * (i & 1))), scale)));
                }
#pragma unroll
                for (int i = 0; i < U / 2; ++i) my = larger(my, f[i]);
            }
        }
        if (OP == OP_NORM && edge) {  // what lies outside is not zero here: it is made so, and the maximum taken again
            my = 0.0f;
#pragma unroll
            for (int j = 0; j < (OP == OP_NORM ? L::UNITS : 0); ++j) {
                f32x2 *f = y + j * U / 2;
                keep_inside<U>(f, row0 + j * L::STEP < rows ? cols - col : 0);
#pragma unroll
                for (int i = 0; i < U / 2; ++i) my = larger(my, f[i]);
            }
        }
        const unsigned wx = __reduce_max_sync(0xffffffffu, wider_bf16x2(mx));
        const unsigned wy = __reduce_max_sync(0xffffffffu, __float_as_uint(my));
        if (lane == 0) {
            maxima[turn][0][warp] = wx;
            maxima[turn][1][warp] = wy;
        }
        __syncthreads();
        const int freed = OP == OP_GELU_BACK ? buffer : previous;
        const long long next = index + (long long)gridDim.x * (OP == OP_GELU_BACK ? S::BUFFERS : S::BUFFERS - 1);
        if (threadIdx.x == 0 && next < blocks && (OP == OP_GELU_BACK || index != (int)blockIdx.x)) request((int)next, freed);
        if constexpr (OP != OP_PACK) {
            const ComputedValues<T> computed = {y};
            const unsigned m = __reduce_max_sync(0xffffffffu, maxima[turn][1][lane % (THREADS / 32)]);
            write_codes<T>(a.first, a.extent, index, row0, col, edge, computed, m, special[0]);
        }
        if (OP == OP_PACK || (OP != OP_GELU_BACK && a.second.codes)) {
            const unsigned m = __reduce_max_sync(0xffffffffu, maxima[turn][0][lane % (THREADS / 32)]);
            write_codes<T>(OP == OP_PACK ? a.first : a.second, a.extent, index, row0, col, edge, x, m, special[1]);
        }
        previous = buffer;
        if (++buffer == S::BUFFERS) { buffer = 0; phase ^= 1; }
        turn ^= 1;
        first_row += rows_on;
        col0 += cols_on;
        if (col0 >= all_cols) { col0 -= all_cols; first_row += PACK_BLOCK; }
    }
}

// Four codes per thread.  32768x3584 to bf16 107 us, to fp32 125 us (3.3 and 4.7 TB/s): bound by instructions (22 for a
// value, 71 % of the issue slots, a division of 64-bit numbers among them), with DRAM at 34 % for bf16.
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

bool box_map(CUtensorMap *map, const void *data, int64_t rows, int64_t cols, int64_t row_bytes, bool codes)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)row_bytes};
    const cuuint32_t box[2] = {PACK_BLOCK, PACK_BLOCK}, steps[2] = {1, 1};
    return encode(map, codes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2,
                  const_cast<void *>(data), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int OP> int launch_stream(const BlockArgs &a, int blocks, cudaStream_t stream)
{
    const int64_t rows = a.extent.rows, cols = a.extent.cols;
    CUtensorMap x_map, codes_map = {};
    // the stride of a single row is never used, but has to be a possible one
    const int64_t x_bytes = rows == 1 ? ceil_div(cols, 8) * 16 : a.x_stride * 2;
    if (!box_map(&x_map, a.x, rows, cols, x_bytes, false)) return DIPACO_ECUDA;
    if (OP == OP_GELU_BACK && !box_map(&codes_map, a.codes, rows, cols, a.codes_stride, true)) return DIPACO_ECUDA;
    if (cudaFuncSetAttribute(stream_kernel<OP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Stream<OP>::SMEM) != cudaSuccess)
        return launch_status();
    int grid = 296;  // two on each SM
    // with few blocks in a row of them, a block of threads keeps to one column of blocks, and to its parameters
    if (OP == OP_NORM && a.extent.block_cols <= 16) grid = grid / a.extent.block_cols * a.extent.block_cols;
    stream_kernel<OP><<<std::min(blocks, grid), THREADS, Stream<OP>::SMEM, stream>>>(x_map, codes_map, a, blocks);
    return launch_status();
}

template <int OP>
int launch_blocks(BlockArgs a, int dtype, int64_t rows, int64_t cols, cudaStream_t stream)
{
    const int64_t block_cols = ceil_div(cols, PACK_BLOCK), blocks = ceil_div(rows, PACK_BLOCK) * block_cols;
    if (blocks > INT32_MAX - 4096) return DIPACO_ELIMIT;
    a.extent = {(int)rows, (int)cols, (int)block_cols};
    a.aligned = rows_aligned16(a.x, a.x_stride, rows, dense_size(dtype));
    if (dtype == DIPACO_BF16 && a.aligned) return launch_stream<OP>(a, (int)blocks, stream);
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

// A warp waits, for a limited time, on a barrier that nothing completes: no copy is in flight.
__global__ void __launch_bounds__(32) wait_expiry_kernel(unsigned long long limit_ns)
{
    __shared__ uint64_t bar;
    if (threadIdx.x == 0) {
        ptx::mbar_init(&bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    __all_sync(0xffffffffu, bounded_wait(&bar, 0, &g_packing_error, 9, limit_ns));
}

} // namespace

bool dipaco::take_packing_error(bool &expired) { return take_error_word(g_packing_error, expired); }

int dipaco::expire_packing_wait(unsigned long long limit_ns, cudaStream_t stream)
{
    wait_expiry_kernel<<<1, 32, 0, stream>>>(limit_ns);
    return launch_status();
}

int dipaco::pack_normalised(const void *x, int64_t x_stride, int dtype, const float *mean, const float *rstd,
                            const void *gamma, const void *beta, int param_dtype, const dipaco_packed *y,
                            const dipaco_packed *x_packed, cudaStream_t stream)
{
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
    return launch_blocks<OP_NORM>(a, dtype, y->rows, y->cols, stream);
}

int dipaco::pack_activated(const float *x, int64_t x_stride, int activation, const dipaco_packed *y,
                           const dipaco_packed *x_packed, cudaStream_t stream)
{
    BlockArgs a = {};
    a.x = x;
    a.x_stride = x_stride;
    a.first = packed_out(y);
    a.second = packed_out(x_packed);
    a.activation = activation;
    if (activation == DIPACO_ACTIVATION_GELU) return launch_blocks<OP_GELU>(a, DIPACO_F32, y->rows, y->cols, stream);
    if (activation == DIPACO_ACTIVATION_NONE) {
        if (x_packed) {
            BlockArgs b = a;
            b.first = a.second;
            if (const int rc = launch_blocks<OP_PACK>(b, DIPACO_F32, y->rows, y->cols, stream)) return rc;
        }
        return launch_blocks<OP_PACK>(a, DIPACO_F32, y->rows, y->cols, stream);
    }
    const int64_t block_cols = ceil_div(y->cols, PACK_BLOCK), blocks = ceil_div(y->rows, PACK_BLOCK) * block_cols;
    if (blocks > INT32_MAX - 4096) return DIPACO_ELIMIT;
    a.extent = {(int)y->rows, (int)y->cols, (int)block_cols};
    a.aligned = rows_aligned16(x, x_stride, y->rows, 4);
    block_kernel<float, OP_ACTIVATE><<<(unsigned)blocks, THREADS, 0, stream>>>(a);
    return launch_status();
}

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
    if (rows == 0) return DIPACO_OK;
    if (!mean || !rstd) return DIPACO_EINVAL;
    if (const int rc = dipaco_layer_norm(x, x_stride, nullptr, nullptr, nullptr, 0, mean, rstd, rows, cols, eps,
                                         dtype, param_dtype, device, cuda_stream))
        return rc;
    if (cols == 0) return DIPACO_OK;
    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    return pack_normalised(x, x_stride, dtype, mean, rstd, gamma, beta, param_dtype, y, x_packed,
                           static_cast<cudaStream_t>(cuda_stream));
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
