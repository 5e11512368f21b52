// The norms after and before a block, with its gate and its scaled residual (see include/dipaco.h):
//
//   p = LN(f) post_gamma + post_beta,  z = s x + g p (rounded to x's type),  n = LN(z) gamma + beta
//
// and the gradients.  With h_z = (z - mean_z) rstd_z, u = dn gamma, and the same for f:
//
//   d = dz + rstd_z (u - mean(u) - h_z mean(u h_z))      the whole gradient of z
//   dx = s d,  q = d g post_gamma,  df = rstd_f (q - mean(q) - h_f mean(q h_f))
//   dg = d (h_f post_gamma + post_beta), summed where g is broadcast
//   dgamma = sum dn h_z,  dbeta = sum dn,  dpost_gamma = sum d g h_f,  dpost_beta = sum d g   (over rows)
//
//   group_rows_kernel a group of warps per row, which stays in their registers: up to 8192 columns
//   rows_kernel       a block per row, which is read again for every sum: any width
//   group_back_kernel every gradient in one pass, a row in the registers of a group: up to 4096 columns
//   back_rows_kernel  as rows_kernel for dx, df and the two means that d needs; back_columns_kernel the sums over rows
#include "inner_common.cuh"

#include <algorithm>
#include <cmath>

using namespace dipaco;

namespace {

// A [rows, cols] matrix that is read: dense, or packed.
struct Source {
    const void *dense;
    const uint8_t *codes, *scales;
    long long stride;
    int scale_cols;
};

struct NormArgs {
    int rows, cols;
    const void *post_gamma, *post_beta, *gamma, *beta;
    bool params_bf16;
    const void *gate;
    long long gate_stride;
    int gate_kind;
    bool gate_bf16;
    float scale, eps;
    bool post_norm, norm;
    // forward
    Source x, f, z;  // z: of the backward pass
    void *z_out, *n;
    long long z_stride, n_stride;
    float *stats;  // [4][rows]
    // backward
    Source dn, dz;
    const float *saved;  // [4][rows]
    void *dx, *df, *dgate;
    long long dx_stride, df_stride, dgate_stride;
    float *row_means;  // [2][rows]: mean(u), mean(u h_z)
    float *partial;    // [parts][4][cols]: sums over rows of dn h_z, dn, w h_f, w
    int parts;
};

template <typename T> __device__ __forceinline__ float load_value(const Source &s, long long row, int col)
{
    if (s.dense) return widen1<T>(static_cast<const T *>(s.dense)[row * s.stride + col]);
    const __half_raw h = __nv_cvt_fp8_to_halfraw(s.codes[row * s.stride + col], __NV_E4M3);
    return __half2float(__half(h)) * scale_value(s.scales[row / PACK_BLOCK * s.scale_cols + col / PACK_BLOCK]);
}

__device__ __forceinline__ float param_or(const void *p, bool bf16, int c, float otherwise)
{
    return p ? load_param(p, bf16, c) : otherwise;
}

template <typename T> __device__ __forceinline__ float gate_at(const NormArgs &a, long long row, int col)
{
    switch (a.gate_kind) {
    case DIPACO_GATE_COLS: return load_param(a.gate, a.gate_bf16, col);
    case DIPACO_GATE_ROWS: return load_param(a.gate, a.gate_bf16, row);
    case DIPACO_GATE_FULL: return widen1<T>(static_cast<const T *>(a.gate)[row * a.gate_stride + col]);
    default: return 1.0f;
    }
}

constexpr int ROW_THREADS = 256;

// Sums of two values over the block, on every thread, in a fixed order.
__device__ __forceinline__ float2 block_sums(float a, float b, float2 *shared)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = make_float2(a, b);
    __syncthreads();
    float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int w = 0; w < ROW_THREADS / 32; ++w) {
        sum.x += shared[w].x;
        sum.y += shared[w].y;
    }
    return sum;
}

// Mean and 1 / sqrt(var + eps) of the row value(c).  The mean is corrected by the mean of what is left after
// it: the roundings of a sum can be more than the spread of a row whose values are nearly equal.
template <typename Value>
__device__ __forceinline__ float2 row_statistics(int cols, float eps, float2 *shared, Value value)
{
    float sum = 0.0f;
    for (int c = threadIdx.x; c < cols; c += ROW_THREADS) sum += value(c);
    const float mean = block_sums(sum, 0.0f, shared).x / (float)cols;
    float left = 0.0f, squares = 0.0f;
    for (int c = threadIdx.x; c < cols; c += ROW_THREADS) {
        const float d = value(c) - mean;
        left += d;
        squares = fmaf(d, d, squares);
    }
    const float2 s = block_sums(left, squares, shared);
    const float off = s.x / (float)cols;
    return make_float2(mean + off, 1.0f / sqrtf(fmaxf(s.y / (float)cols - off * off, 0.0f) + eps));
}

template <typename T> __global__ void __launch_bounds__(ROW_THREADS) rows_kernel(const __grid_constant__ NormArgs a)
{
    __shared__ float2 shared[ROW_THREADS / 32];
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        float2 of_f = make_float2(0.0f, 1.0f), of_z = make_float2(0.0f, 1.0f);
        if (a.post_norm)
            of_f = row_statistics(a.cols, a.eps, shared, [&](int c) { return load_value<T>(a.f, row, c); });
        T *z = static_cast<T *>(a.z_out) + row * a.z_stride;
        for (int c = threadIdx.x; c < a.cols; c += ROW_THREADS) {
            float p = load_value<T>(a.f, row, c);
            if (a.post_norm)
                p = fmaf((p - of_f.x) * of_f.y, param_or(a.post_gamma, a.params_bf16, c, 1.0f),
                         param_or(a.post_beta, a.params_bf16, c, 0.0f));
            z[c] = narrow1<T>(fmaf(gate_at<T>(a, row, c), p, a.scale * load_value<T>(a.x, row, c)));
        }
        if (a.norm) {  // a thread reads what it wrote itself
            of_z = row_statistics(a.cols, a.eps, shared, [&](int c) { return widen1<T>(z[c]); });
            if (a.n) {
                T *n = static_cast<T *>(a.n) + row * a.n_stride;
                for (int c = threadIdx.x; c < a.cols; c += ROW_THREADS)
                    n[c] = narrow1<T>(fmaf((widen1<T>(z[c]) - of_z.x) * of_z.y, param_or(a.gamma, a.params_bf16, c, 1.0f),
                                           param_or(a.beta, a.params_bf16, c, 0.0f)));
            }
        }
        if (threadIdx.x == 0) {
            a.stats[row] = of_f.x;
            a.stats[a.rows + row] = of_f.y;
            a.stats[2ll * a.rows + row] = of_z.x;
            a.stats[3ll * a.rows + row] = of_z.y;
        }
    }
}

// ------------------------------------------------------------------------------------------ rows in registers

// A group of `warps` warps has a row, eight values for each thread: consecutive ones where rows are on 16-byte
// boundaries (VEC), else every (32 * warps)-th, so that a warp's accesses stay whole.  What does not change from row
// to row, the columns' parameters, stays in registers too (HOLD), and the next row is loaded while one is worked on.

constexpr int PER_THREAD = 8;

struct Group {
    int warps, index, warp, lane, thread;  // thread: of the group
    int other;                             // the warp whose values this lane joins
    float count;                           // how many values that warp has; 0: none to join
    float of_first, of_warp, of_row;       // 1 / number of values of the warp's first lane, of the warp, of the row
    float2 *slots;                         // [2][warps][rows], shared
    int parity = 0;

    // A barrier of this group's own.
    __device__ __forceinline__ void sync() const
    {
        asm volatile("bar.sync %0, %1;" ::"r"(index + 1), "r"(warps * 32) : "memory");
    }
};

template <bool VEC> __device__ __forceinline__ int column(const Group &g, int j)
{
    return VEC ? g.thread * PER_THREAD + j : j * g.warps * 32 + g.thread;
}
// Which of the thread's values belong to the row.
template <bool VEC> __device__ __forceinline__ unsigned valid_values(const Group &g, int cols)
{
    unsigned valid = 0u;
#pragma unroll
    for (int j = 0; j < PER_THREAD; ++j)
        if (column<VEC>(g, j) < cols) valid |= 1u << j;
    return valid;
}
constexpr unsigned ALL_VALID = (1u << PER_THREAD) - 1u;
// Makes the others zero.
__device__ __forceinline__ void keep_valid(unsigned valid, f32x2 *v)
{
    if (valid == ALL_VALID) return;
#pragma unroll
    for (int i = 0; i < PER_THREAD / 2; ++i) {
        const float2 w = values_of(v[i]);
        v[i] = pair_of(valid >> (2 * i) & 1u ? w.x : 0.0f, valid >> (2 * i + 1) & 1u ? w.y : 0.0f);
    }
}

// A thread's values of a row as they are in memory.
template <typename T> struct RowRaw {
    unsigned w[PER_THREAD * sizeof(T) / 4];
};
template <typename T, bool VEC>
__device__ __forceinline__ void load_row(const T *row, const Group &g, unsigned valid, RowRaw<T> &raw)
{
    constexpr int UE = Unit<T>::UE;
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < PER_THREAD / UE; ++i) {
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (valid >> (i * UE) & 1u) v = __ldcs(reinterpret_cast<const uint4 *>(row + g.thread * PER_THREAD) + i);
            raw.w[4 * i] = v.x; raw.w[4 * i + 1] = v.y; raw.w[4 * i + 2] = v.z; raw.w[4 * i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < PER_THREAD; ++j) {
            unsigned v = 0u;
            if (valid >> j & 1u) {
                if constexpr (sizeof(T) == 2)
                    v = __ldcs(reinterpret_cast<const unsigned short *>(row) + column<false>(g, j));
                else
                    v = __ldcs(reinterpret_cast<const unsigned *>(row) + column<false>(g, j));
            }
            if (sizeof(T) == 4)
                raw.w[j] = v;
            else if (j & 1)
                raw.w[j / 2] |= v << 16;
            else
                raw.w[j / 2] = v;
        }
    }
}
// Values that do not belong to the row are zero.
template <typename T> __device__ __forceinline__ void widen_row(const RowRaw<T> &raw, unsigned valid, f32x2 *v)
{
    constexpr int UE = Unit<T>::UE;
#pragma unroll
    for (int i = 0; i < PER_THREAD / UE; ++i)
        widen_pairs<T>(make_uint4(raw.w[4 * i], raw.w[4 * i + 1], raw.w[4 * i + 2], raw.w[4 * i + 3]), v + i * UE / 2);
    keep_valid(valid, v);
}
template <typename T> __device__ __forceinline__ void narrow_row(const f32x2 *v, RowRaw<T> &raw)
{
    constexpr int UE = Unit<T>::UE;
#pragma unroll
    for (int i = 0; i < PER_THREAD / UE; ++i) {
        const uint4 u = narrow_pairs<T>(v + i * UE / 2);
        raw.w[4 * i] = u.x; raw.w[4 * i + 1] = u.y; raw.w[4 * i + 2] = u.z; raw.w[4 * i + 3] = u.w;
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store_row(T *row, const Group &g, unsigned valid, const RowRaw<T> &raw)
{
    constexpr int UE = Unit<T>::UE;
    if constexpr (VEC) {
        if (valid == ALL_VALID) {
#pragma unroll
            for (int i = 0; i < PER_THREAD / UE; ++i)
                reinterpret_cast<uint4 *>(row + g.thread * PER_THREAD)[i] =
                    make_uint4(raw.w[4 * i], raw.w[4 * i + 1], raw.w[4 * i + 2], raw.w[4 * i + 3]);
            return;
        }
    }
#pragma unroll
    for (int j = 0; j < PER_THREAD; ++j)
        if (valid >> j & 1u) {
            if constexpr (sizeof(T) == 2)
                reinterpret_cast<unsigned short *>(row)[column<VEC>(g, j)] = (unsigned short)(raw.w[j / 2] >> 16 * (j & 1));
            else
                reinterpret_cast<unsigned *>(row)[column<VEC>(g, j)] = raw.w[j];
        }
}
// Parameters of the thread's columns.
template <bool VEC>
__device__ __forceinline__ void load_columns(const void *p, bool bf16, const Group &g, int cols, float otherwise, f32x2 *v)
{
    if (!p) {
#pragma unroll
        for (int i = 0; i < PER_THREAD / 2; ++i) v[i] = pair_of(otherwise);
    } else if (VEC) {
        param_pairs<PER_THREAD>(p, bf16, reinterpret_cast<uintptr_t>(p) % 16 == 0, g.thread * PER_THREAD, cols, v);
    } else {
#pragma unroll
        for (int i = 0; i < PER_THREAD / 2; ++i) {
            const int c0 = column<VEC>(g, 2 * i), c1 = column<VEC>(g, 2 * i + 1);
            v[i] = pair_of(c0 < cols ? load_param(p, bf16, c0) : 0.0f, c1 < cols ? load_param(p, bf16, c1) : 0.0f);
        }
    }
}

__device__ __forceinline__ float sum_pairs(const f32x2 *v)
{
    return sum_of(add2(add2(v[0], v[1]), add2(v[2], v[3])));
}

// Sums of pairs of values over the group, R at a time, on every thread: over warps in shared memory, in two sets that
// take turns, so that a set is written again only after everyone has read it.  Up to eight warps are joined in three
// steps by every eight lanes, more in five.
template <int R> __device__ __forceinline__ void join_warps(const Group &g, float2 *sums)
{
    for (int o = g.warps <= 8 ? 4 : 16; o > 0; o >>= 1)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            sums[r].x += __shfl_xor_sync(0xffffffffu, sums[r].x, o);
            sums[r].y += __shfl_xor_sync(0xffffffffu, sums[r].y, o);
        }
}
template <int R> __device__ __forceinline__ void warp_sums(float2 *sums)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            sums[r].x += __shfl_xor_sync(0xffffffffu, sums[r].x, o);
            sums[r].y += __shfl_xor_sync(0xffffffffu, sums[r].y, o);
        }
}
// Hands the warps' values round: [warp][row].
template <int R> __device__ __forceinline__ const float2 *exchange(Group &g, const float2 *own)
{
    float2 *slots = g.slots + g.parity * g.warps * R;
    if (g.lane == 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) slots[g.warp * R + r] = own[r];
    }
    g.sync();
    g.parity ^= 1;
    return slots;
}

// Mean and 1 / sqrt(var + eps) of the group's R rows.  Differences are taken from the mean of the warp's first lane's
// values: it is exact where all values are equal, and no farther from the warp's mean than the spread of its 256
// values times sqrt(32), so that the squares lose five bits at most.  The warps are joined about the first one's mean.
template <int R, bool VEC>
__device__ __forceinline__ void group_statistics(Group &g, const f32x2 (*v)[PER_THREAD / 2], unsigned valid, float eps, float2 *found)
{
    float2 sums[R];
    float centre[R];
#pragma unroll
    for (int r = 0; r < R; ++r) centre[r] = __shfl_sync(0xffffffffu, sum_pairs(v[r]) * g.of_first, 0);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        f32x2 d[PER_THREAD / 2], squares = 0ull;
#pragma unroll
        for (int i = 0; i < PER_THREAD / 2; ++i) d[i] = add2(v[r][i], pair_of(-centre[r]));
        keep_valid(valid, d);
#pragma unroll
        for (int i = 0; i < PER_THREAD / 2; ++i) squares = fma2(d[i], d[i], squares);
        sums[r] = make_float2(sum_pairs(d), sum_of(squares));
    }
    warp_sums<R>(sums);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float off = sums[r].x * g.of_warp;
        sums[r] = make_float2(centre[r] + off, fmaxf(fmaf(-off, sums[r].x, sums[r].y), 0.0f));
    }
    if (g.warps > 1) {
        const float2 *slots = exchange<R>(g, sums);
        float first[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            first[r] = slots[r].x;
            const float2 of = slots[g.other * R + r];
            const float apart = of.x - first[r];
            sums[r] = g.count > 0.0f ? make_float2(g.count * apart, fmaf(g.count * apart, apart, of.y)) : make_float2(0.0f, 0.0f);
        }
        join_warps<R>(g, sums);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float off = sums[r].x * g.of_row;
            sums[r] = make_float2(first[r] + off, fmaxf(fmaf(-off, sums[r].x, sums[r].y), 0.0f));
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) found[r] = make_float2(sums[r].x, rsqrtf(fmaf(sums[r].y, g.of_row, eps)));
}

// How many values a warp of the group has, and its first lane.
template <bool VEC> __device__ __forceinline__ int values_of_warp(int warps, int warp, int cols)
{
    if (VEC) return min(max(cols - warp * 32 * PER_THREAD, 0), 32 * PER_THREAD);
    int n = 0;
#pragma unroll
    for (int j = 0; j < PER_THREAD; ++j) n += min(max(cols - (j * warps + warp) * 32, 0), 32);
    return n;
}
template <bool VEC> __device__ __forceinline__ int values_of_first_lane(int warps, int warp, int cols)
{
    if (VEC) return min(max(cols - warp * 32 * PER_THREAD, 0), PER_THREAD);
    int n = 0;
#pragma unroll
    for (int j = 0; j < PER_THREAD; ++j) n += (j * warps + warp) * 32 < cols;
    return n;
}

// A group of the block, with `slots` of 2 * rows float2 for each of the block's warps.
template <bool VEC> __device__ __forceinline__ Group make_group(int warps, int cols, float2 *slots, int rows)
{
    Group g;
    g.warps = warps;
    g.lane = threadIdx.x & 31;
    g.index = (int)(threadIdx.x >> 5) / warps;
    g.warp = (int)(threadIdx.x >> 5) - g.index * warps;
    g.thread = g.warp * 32 + g.lane;
    g.slots = slots + 2 * g.index * warps * rows;
    const int joined = warps <= 8 ? g.lane & 7 : g.lane;
    g.other = min(joined, warps - 1);
    g.count = joined < warps ? (float)values_of_warp<VEC>(warps, joined, cols) : 0.0f;
    g.of_first = 1.0f / (float)values_of_first_lane<VEC>(warps, g.warp, cols);
    g.of_warp = 1.0f / (float)values_of_warp<VEC>(warps, g.warp, cols);
    g.of_row = 1.0f / (float)cols;
    return g;
}

// GATE: what a thread needs for it.
enum : int { GATE_IN_COLUMNS, GATE_OF_ROW, GATE_OF_VALUES };

constexpr int MAX_GROUP_COLS = 32 * 32 * PER_THREAD;

// HOLD: blocks of up to 16 warps; R rows at a time.
template <typename T, bool VEC, int GATE, bool HOLD, int R>
__global__ void __launch_bounds__(HOLD ? 512 : 1024, 1)
    group_rows_kernel(const __grid_constant__ NormArgs a, int warps)
{
    __shared__ float2 slots[2 * 32 * R];
    Group g = make_group<VEC>(warps, a.cols, slots, R);
    const int groups = (int)(blockDim.x >> 5) / warps;
    const unsigned valid = valid_values<VEC>(g, a.cols);
    // p = h factor + shift, a gate of columns in both
    f32x2 factor[PER_THREAD / 2], shift[PER_THREAD / 2], gamma[PER_THREAD / 2], beta[PER_THREAD / 2];
    const auto load_block_columns = [&] {
        load_columns<VEC>(a.post_gamma, a.params_bf16, g, a.cols, 1.0f, factor);
        load_columns<VEC>(a.post_beta, a.params_bf16, g, a.cols, 0.0f, shift);
        if (GATE == GATE_IN_COLUMNS && a.gate_kind == DIPACO_GATE_COLS) {
            f32x2 gate[PER_THREAD / 2];
            load_columns<VEC>(a.gate, a.gate_bf16, g, a.cols, 1.0f, gate);
#pragma unroll
            for (int i = 0; i < PER_THREAD / 2; ++i) {
                factor[i] = mul2(factor[i], gate[i]);
                shift[i] = mul2(shift[i], gate[i]);
            }
        }
    };
    const auto load_next_columns = [&] {
        load_columns<VEC>(a.gamma, a.params_bf16, g, a.cols, 1.0f, gamma);
        load_columns<VEC>(a.beta, a.params_bf16, g, a.cols, 0.0f, beta);
    };
    const long long between = (long long)gridDim.x * groups, step = between * R;  // the R rows are `between` apart
    long long row = (long long)blockIdx.x * groups + g.index;
    RowRaw<T> next_x[R], next_f[R];
    const auto load_next = [&](long long first) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const long long at = min(first + r * between, (long long)a.rows - 1);  // the last row again where there is none
            load_row<T, VEC>(static_cast<const T *>(a.f.dense) + at * a.f.stride, g, valid, next_f[r]);
            load_row<T, VEC>(static_cast<const T *>(a.x.dense) + at * a.x.stride, g, valid, next_x[r]);
        }
    };
    if (row < a.rows) load_next(row);
    if (HOLD) {
        load_block_columns();
        if (a.n) load_next_columns();
    }
    for (; row < a.rows; row += step) {
        f32x2 v[R][PER_THREAD / 2];
        RowRaw<T> x[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            widen_row<T>(next_f[r], valid, v[r]);
            x[r] = next_x[r];
        }
        if (row + step < a.rows) load_next(row + step);
        float2 of_f[R], of_z[R];
#pragma unroll
        for (int r = 0; r < R; ++r) of_f[r] = of_z[r] = make_float2(0.0f, 1.0f);
        if (a.post_norm) group_statistics<R, VEC>(g, v, valid, a.eps, of_f);
        if (!HOLD) load_block_columns();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const long long at = row + r * between;
            if (R > 1 && at >= a.rows) break;
            f32x2 gate[PER_THREAD / 2], stream[PER_THREAD / 2];
            if (GATE == GATE_OF_ROW) {
                const float of_row = load_param(a.gate, a.gate_bf16, at);
#pragma unroll
                for (int i = 0; i < PER_THREAD / 2; ++i) gate[i] = pair_of(of_row);
            } else if (GATE == GATE_OF_VALUES) {
                RowRaw<T> raw;
                load_row<T, VEC>(static_cast<const T *>(a.gate) + at * a.gate_stride, g, valid, raw);
                widen_row<T>(raw, valid, gate);
            }
            widen_row<T>(x[r], valid, stream);
#pragma unroll
            for (int i = 0; i < PER_THREAD / 2; ++i) {
                const f32x2 scaled = mul2(stream[i], pair_of(a.scale));
                const f32x2 p = fma2(mul2(add2(v[r][i], pair_of(-of_f[r].x)), pair_of(of_f[r].y)), factor[i], shift[i]);
                v[r][i] = GATE == GATE_IN_COLUMNS ? add2(p, scaled) : fma2(gate[i], p, scaled);
            }
            RowRaw<T> raw;
            narrow_row<T>(v[r], raw);
            store_row<T, VEC>(static_cast<T *>(a.z_out) + at * a.z_stride, g, valid, raw);
            widen_row<T>(raw, valid, v[r]);
        }
        if (a.norm) {
            group_statistics<R, VEC>(g, v, valid, a.eps, of_z);
            if (a.n) {
                if (!HOLD) load_next_columns();
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const long long at = row + r * between;
                    if (R > 1 && at >= a.rows) break;
#pragma unroll
                    for (int i = 0; i < PER_THREAD / 2; ++i)
                        v[r][i] = fma2(mul2(add2(v[r][i], pair_of(-of_z[r].x)), pair_of(of_z[r].y)), gamma[i], beta[i]);
                    RowRaw<T> raw;
                    narrow_row<T>(v[r], raw);
                    store_row<T, VEC>(static_cast<T *>(a.n) + at * a.n_stride, g, valid, raw);
                }
            }
        }
        if (g.thread < R) {
            const long long at = row + g.thread * between;
            const float2 f = R > 1 && g.thread ? of_f[R - 1] : of_f[0], z = R > 1 && g.thread ? of_z[R - 1] : of_z[0];
            if (at < a.rows) {
                a.stats[at] = f.x;
                a.stats[a.rows + at] = f.y;
                a.stats[2ll * a.rows + at] = z.x;
                a.stats[3ll * a.rows + at] = z.y;
            }
        }
    }
}

// ------------------------------------------------------------------------------------------ gradients

// What a row's statistics and the means of its gradient say about its values.
struct RowOf {
    float mean_f, rstd_f, mean_z, rstd_z, mean_u, mean_uh;
};
struct ValueOf {
    float dn, h_z, d, h_f;
};
template <typename T>
__device__ __forceinline__ ValueOf value_of(const NormArgs &a, const RowOf &r, long long row, int c)
{
    ValueOf v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (a.dz.dense) v.d = load_value<T>(a.dz, row, c);
    if (a.norm) {
        v.dn = load_value<T>(a.dn, row, c);
        v.h_z = (load_value<T>(a.z, row, c) - r.mean_z) * r.rstd_z;
        const float u = v.dn * param_or(a.gamma, a.params_bf16, c, 1.0f);
        v.d += r.rstd_z * (u - r.mean_u - v.h_z * r.mean_uh);
    }
    v.h_f = (load_value<T>(a.f, row, c) - r.mean_f) * r.rstd_f;
    return v;
}
__device__ __forceinline__ RowOf row_of(const NormArgs &a, long long row)
{
    RowOf r = {0.0f, 1.0f, 0.0f, 1.0f, 0.0f, 0.0f};
    if (a.post_norm) {
        r.mean_f = a.saved[row];
        r.rstd_f = a.saved[a.rows + row];
    }
    if (a.norm) {
        r.mean_z = a.saved[2ll * a.rows + row];
        r.rstd_z = a.saved[3ll * a.rows + row];
    }
    return r;
}

template <typename T> __global__ void __launch_bounds__(ROW_THREADS) back_rows_kernel(const __grid_constant__ NormArgs a)
{
    __shared__ float2 shared[ROW_THREADS / 32];
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        RowOf r = row_of(a, row);
        if (a.norm) {
            float s1 = 0.0f, s2 = 0.0f;
            for (int c = threadIdx.x; c < a.cols; c += ROW_THREADS) {
                const float u = load_value<T>(a.dn, row, c) * param_or(a.gamma, a.params_bf16, c, 1.0f);
                s1 += u;
                s2 = fmaf(u, (load_value<T>(a.z, row, c) - r.mean_z) * r.rstd_z, s2);
            }
            const float2 s = block_sums(s1, s2, shared);
            r.mean_u = s.x / (float)a.cols;
            r.mean_uh = s.y / (float)a.cols;
            if (threadIdx.x == 0) {
                a.row_means[row] = r.mean_u;
                a.row_means[a.rows + row] = r.mean_uh;
            }
        }
        float s3 = 0.0f, s4 = 0.0f, s5 = 0.0f;
        for (int c = threadIdx.x; c < a.cols; c += ROW_THREADS) {
            const ValueOf v = value_of<T>(a, r, row, c);
            const float post = param_or(a.post_gamma, a.params_bf16, c, 1.0f);
            const float p = a.post_norm ? fmaf(v.h_f, post, param_or(a.post_beta, a.params_bf16, c, 0.0f)) : v.h_f;
            const float q = v.d * gate_at<T>(a, row, c) * post;
            s3 += q;
            s4 = fmaf(q, v.h_f, s4);
            s5 = fmaf(v.d, p, s5);
            if (a.dx) static_cast<T *>(a.dx)[row * a.dx_stride + c] = narrow1<T>(a.scale * v.d);
            if (a.gate_kind == DIPACO_GATE_FULL && a.dgate)
                static_cast<T *>(a.dgate)[row * a.dgate_stride + c] = narrow1<T>(v.d * p);
        }
        float2 s = make_float2(0.0f, 0.0f);
        if (a.post_norm) {
            s = block_sums(s3, s4, shared);
            s.x /= (float)a.cols;
            s.y /= (float)a.cols;
        }
        if (a.gate_kind == DIPACO_GATE_ROWS && a.dgate) {
            s5 = block_sums(s5, 0.0f, shared).x;
            if (threadIdx.x == 0) static_cast<float *>(a.dgate)[row] = s5;
        }
        if (a.df)
            for (int c = threadIdx.x; c < a.cols; c += ROW_THREADS) {
                const ValueOf v = value_of<T>(a, r, row, c);
                float q = v.d * gate_at<T>(a, row, c);
                if (a.post_norm)
                    q = r.rstd_f * (q * param_or(a.post_gamma, a.params_bf16, c, 1.0f) - s.x - v.h_f * s.y);
                static_cast<T *>(a.df)[row * a.df_stride + c] = narrow1<T>(q);
            }
    }
}

// A row of f or z: as load_row, or eight codes.
template <typename T, bool VEC>
__device__ __forceinline__ void load_source(const Source &s, long long row, const Group &g, unsigned valid, RowRaw<T> &raw)
{
    if (s.dense) {
        load_row<T, VEC>(static_cast<const T *>(s.dense) + row * s.stride, g, valid, raw);
        return;
    }
    const uint8_t *codes = s.codes + row * s.stride;
    raw.w[0] = raw.w[1] = 0u;
    if constexpr (VEC) {
        if (valid) {  // rows of codes are padded to 16 bytes
            const uint2 v = __ldcs(reinterpret_cast<const uint2 *>(codes) + g.thread);
            raw.w[0] = v.x;
            raw.w[1] = v.y;
        }
    } else {
#pragma unroll
        for (int j = 0; j < PER_THREAD; ++j)
            if (valid >> j & 1u) raw.w[j / 4] |= (unsigned)__ldcs(codes + column<false>(g, j)) << 8 * (j % 4);
    }
}
// Their values (zero outside the row).
template <typename T, bool VEC>
__device__ __forceinline__ void widen_source(const Source &s, long long row, const Group &g, unsigned valid, const RowRaw<T> &raw, f32x2 *v)
{
    if (s.dense) {
        widen_row<T>(raw, valid, v);
        return;
    }
    const uint8_t *scales = s.scales + row / PACK_BLOCK * s.scale_cols;
    const f32x2 one = VEC && valid ? pair_of(scale_value(scales[g.thread * PER_THREAD / PACK_BLOCK])) : 0ull;
#pragma unroll
    for (int i = 0; i < PER_THREAD / 2; ++i) {
        f32x2 scale = one;
        if (!VEC)
            scale = pair_of(valid >> (2 * i) & 1u ? scale_value(scales[column<VEC>(g, 2 * i) / PACK_BLOCK]) : 0.0f,
                            valid >> (2 * i + 1) & 1u ? scale_value(scales[column<VEC>(g, 2 * i + 1) / PACK_BLOCK]) : 0.0f);
        v[i] = mul2(decode_pair(raw.w[i / 2] >> 16 * (i & 1)), scale);
    }
    keep_valid(valid, v);
}

// Sums of pairs over the group, on every thread.
template <int R> __device__ __forceinline__ void group_sums(Group &g, float2 *sums)
{
    warp_sums<R>(sums);
    if (g.warps == 1) return;
    const float2 *slots = exchange<R>(g, sums);
#pragma unroll
    for (int r = 0; r < R; ++r) sums[r] = g.count > 0.0f ? slots[g.other * R + r] : make_float2(0.0f, 0.0f);
    join_warps<R>(g, sums);
}

constexpr int MAX_BACK_COLS = 16 * 32 * PER_THREAD;

// A persistent block of groups, each with a row at a time; a thread keeps the sums over its rows of its columns.  The
// next row's values are loaded where this row's have been used for the last time.
template <typename T, bool VEC, int GATE>
__global__ void __launch_bounds__(512, 1) group_back_kernel(const __grid_constant__ NormArgs a, int warps)
{
    constexpr int P = PER_THREAD / 2;
    __shared__ float2 slots[2 * 16 * 2];
    __shared__ float joined[MAX_BACK_COLS];
    Group g = make_group<VEC>(warps, a.cols, slots, 2);
    const int groups = (int)(blockDim.x >> 5) / warps;
    const unsigned valid = valid_values<VEC>(g, a.cols);
    const long long step = (long long)gridDim.x * groups;
    long long row = (long long)blockIdx.x * groups + g.index;
    RowRaw<T> dn = {}, dz = {}, z = {}, f = {};
    const auto load_z = [&](long long at) {
        if (a.norm) {
            load_row<T, VEC>(static_cast<const T *>(a.dn.dense) + at * a.dn.stride, g, valid, dn);
            load_source<T, VEC>(a.z, at, g, valid, z);
        }
        if (a.dz.dense) load_row<T, VEC>(static_cast<const T *>(a.dz.dense) + at * a.dz.stride, g, valid, dz);
    };
    if (row < a.rows) {
        load_z(row);
        load_source<T, VEC>(a.f, row, g, valid, f);
    }
    f32x2 gamma[P], factor[P], shift[P];  // factor: post_gamma, times a gate of columns
    load_columns<VEC>(a.gamma, a.params_bf16, g, a.cols, 1.0f, gamma);
    load_columns<VEC>(a.post_gamma, a.params_bf16, g, a.cols, 1.0f, factor);
    if (GATE == GATE_IN_COLUMNS) {
        if (a.gate_kind == DIPACO_GATE_COLS) {
            f32x2 gate[P];
            load_columns<VEC>(a.gate, a.gate_bf16, g, a.cols, 1.0f, gate);
#pragma unroll
            for (int i = 0; i < P; ++i) factor[i] = mul2(factor[i], gate[i]);
        }
    } else {
        load_columns<VEC>(a.post_beta, a.params_bf16, g, a.cols, 0.0f, shift);
    }
    f32x2 sums[4][P];
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < P; ++i) sums[q][i] = 0ull;

    for (; row < a.rows; row += step) {
        const bool more = row + step < a.rows;
        f32x2 d[P], h[P];
        widen_row<T>(dz, valid, d);
        if (a.norm) {
            const float mean = a.saved[2ll * a.rows + row], rstd = a.saved[3ll * a.rows + row];
            f32x2 u[P];
            widen_row<T>(dn, valid, u);
            widen_source<T, VEC>(a.z, row, g, valid, z, h);
            f32x2 all[2] = {0ull, 0ull};
#pragma unroll
            for (int i = 0; i < P; ++i) {
                h[i] = mul2(add2(h[i], pair_of(-mean)), pair_of(rstd));
                sums[0][i] = fma2(u[i], h[i], sums[0][i]);
                sums[1][i] = add2(sums[1][i], u[i]);
                u[i] = mul2(u[i], gamma[i]);
                all[0] = add2(all[0], u[i]);
                all[1] = fma2(u[i], h[i], all[1]);
            }
            float2 of[1] = {make_float2(sum_of(all[0]), sum_of(all[1]))};
            group_sums<1>(g, of);
            const f32x2 mean_u = pair_of(-of[0].x * g.of_row), mean_uh = pair_of(-of[0].y * g.of_row);
#pragma unroll
            for (int i = 0; i < P; ++i) d[i] = fma2(fma2(h[i], mean_uh, add2(u[i], mean_u)), pair_of(rstd), d[i]);
            keep_valid(valid, d);
        }
        if (more) load_z(row + step);
        f32x2 out[P];
        RowRaw<T> raw;
        if (a.dx) {
#pragma unroll
            for (int i = 0; i < P; ++i) out[i] = mul2(d[i], pair_of(a.scale));
            narrow_row<T>(out, raw);
            store_row<T, VEC>(static_cast<T *>(a.dx) + row * a.dx_stride, g, valid, raw);
        }
        const float mean = a.post_norm ? a.saved[row] : 0.0f, rstd = a.post_norm ? a.saved[a.rows + row] : 1.0f;
        widen_source<T, VEC>(a.f, row, g, valid, f, h);
#pragma unroll
        for (int i = 0; i < P; ++i) h[i] = mul2(add2(h[i], pair_of(-mean)), pair_of(rstd));
        if (more) load_source<T, VEC>(a.f, row + step, g, valid, f);
        f32x2 of_gate = 0ull;
        if (GATE != GATE_IN_COLUMNS) {
            f32x2 gate[P];
            if (GATE == GATE_OF_ROW) {
                const float of_row = load_param(a.gate, a.gate_bf16, row);
#pragma unroll
                for (int i = 0; i < P; ++i) gate[i] = pair_of(of_row);
            } else {
                load_row<T, VEC>(static_cast<const T *>(a.gate) + row * a.gate_stride, g, valid, raw);
                widen_row<T>(raw, valid, gate);
            }
#pragma unroll
            for (int i = 0; i < P; ++i) {
                out[i] = mul2(d[i], fma2(h[i], factor[i], shift[i]));
                if (GATE == GATE_OF_ROW) of_gate = add2(of_gate, out[i]);
                d[i] = mul2(d[i], gate[i]);
            }
            if (GATE == GATE_OF_VALUES && a.dgate) {
                narrow_row<T>(out, raw);
                store_row<T, VEC>(static_cast<T *>(a.dgate) + row * a.dgate_stride, g, valid, raw);
            }
        }
        f32x2 all[2] = {0ull, 0ull};
#pragma unroll
        for (int i = 0; i < P; ++i) {
            sums[2][i] = fma2(d[i], h[i], sums[2][i]);
            sums[3][i] = add2(sums[3][i], d[i]);
            d[i] = mul2(d[i], factor[i]);
            all[0] = add2(all[0], d[i]);
            all[1] = fma2(d[i], h[i], all[1]);
        }
        float2 of[2] = {make_float2(sum_of(all[0]), sum_of(all[1])), make_float2(sum_of(of_gate), 0.0f)};
        if (GATE == GATE_OF_ROW) {
            group_sums<2>(g, of);
            if (g.thread == 0 && a.dgate) static_cast<float *>(a.dgate)[row] = of[1].x;
        } else if (a.post_norm) {
            group_sums<1>(g, of);
        }
        if (a.df) {
            if (a.post_norm) {
                const f32x2 mean_q = pair_of(-of[0].x * g.of_row), mean_qh = pair_of(-of[0].y * g.of_row);
#pragma unroll
                for (int i = 0; i < P; ++i) d[i] = mul2(fma2(h[i], mean_qh, add2(d[i], mean_q)), pair_of(rstd));
            }
            narrow_row<T>(d, raw);
            store_row<T, VEC>(static_cast<T *>(a.df) + row * a.df_stride, g, valid, raw);
        }
    }
    // the groups' sums, one group after another
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        for (int turn = 0; turn < groups; ++turn) {
            if (g.index == turn) {
#pragma unroll
                for (int j = 0; j < PER_THREAD; ++j) {
                    const float2 w = values_of(sums[q][j / 2]);
                    const float own = j & 1 ? w.y : w.x;
                    if (valid >> j & 1u) {
                        float &at = joined[column<VEC>(g, j)];
                        at = turn ? at + own : own;
                    }
                }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x) a.partial[((long long)blockIdx.x * 4 + q) * a.cols + c] = joined[c];
        __syncthreads();
    }
}

// A gate that is one for all rows leaves the sums over rows of d h_f and d for join_kernel, any other goes into them.
__device__ __forceinline__ bool gate_at_the_end(const NormArgs &a)
{
    return a.gate_kind == DIPACO_GATE_NONE || a.gate_kind == DIPACO_GATE_COLS;
}

constexpr int COLUMN_THREADS = 128;
constexpr int MAX_PARTS = 64;

template <typename T>
__global__ void __launch_bounds__(COLUMN_THREADS) back_columns_kernel(const __grid_constant__ NormArgs a)
{
    const int c = blockIdx.x * COLUMN_THREADS + threadIdx.x;
    if (c >= a.cols) return;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const long long first = (long long)a.rows * blockIdx.y / gridDim.y, last = (long long)a.rows * (blockIdx.y + 1) / gridDim.y;
    for (long long row = first; row < last; ++row) {
        RowOf r = row_of(a, row);
        if (a.norm) {
            r.mean_u = a.row_means[row];
            r.mean_uh = a.row_means[a.rows + row];
        }
        const ValueOf v = value_of<T>(a, r, row, c);
        const float w = gate_at_the_end(a) ? v.d : v.d * gate_at<T>(a, row, c);
        s[0] = fmaf(v.dn, v.h_z, s[0]);
        s[1] += v.dn;
        s[2] = fmaf(w, v.h_f, s[2]);
        s[3] += w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) a.partial[((long long)blockIdx.y * 4 + i) * a.cols + c] = s[i];
}

struct JoinArgs {
    const float *partial;
    int parts, cols;
    const void *gate, *post_gamma, *post_beta;
    bool gate_bf16, params_bf16, post_norm, gate_cols;
    float *dgate, *dgamma, *dbeta, *dpost_gamma, *dpost_beta;
};

constexpr int JOIN_SLICES = 8;

// The parts' sums in order, 32 columns of a block in JOIN_SLICES slices of parts, and the gradients they make.
__global__ void __launch_bounds__(32 * JOIN_SLICES) join_kernel(const __grid_constant__ JoinArgs a)
{
    __shared__ float shared[4][JOIN_SLICES][32];
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (c < a.cols) {
#pragma unroll 4
        for (int p = slice; p < a.parts; p += JOIN_SLICES)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] += a.partial[((long long)p * 4 + i) * a.cols + c];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) shared[i][slice][lane] = s[i];
    __syncthreads();
    if (slice != 0 || c >= a.cols) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < JOIN_SLICES; ++w) s[i] += shared[i][w][lane];
    }
    if (a.dgamma) a.dgamma[c] = s[0];
    if (a.dbeta) a.dbeta[c] = s[1];
    const float gate = a.gate_cols ? load_param(a.gate, a.gate_bf16, c) : 1.0f;
    if (a.dpost_gamma) a.dpost_gamma[c] = gate * s[2];
    if (a.dpost_beta) a.dpost_beta[c] = gate * s[3];
    if (a.dgate)
        a.dgate[c] = a.post_norm ? fmaf(param_or(a.post_gamma, a.params_bf16, c, 1.0f), s[2],
                                        param_or(a.post_beta, a.params_bf16, c, 0.0f) * s[3])
                                 : s[2];
}

// Rows without values: statistics are those of nothing.
__global__ void empty_rows_kernel(float *stats, int rows, bool post_norm, bool norm)
{
    const float nan = __int_as_float(0x7fffffff);
    for (long long r = blockIdx.x * 256ll + threadIdx.x; r < rows; r += gridDim.x * 256ll) {
        stats[r] = post_norm ? nan : 0.0f;
        stats[rows + r] = post_norm ? nan : 1.0f;
        stats[2ll * rows + r] = norm ? nan : 0.0f;
        stats[3ll * rows + r] = norm ? nan : 1.0f;
    }
}

// ------------------------------------------------------------------------------------------ host

Source dense_source(const void *p, int64_t stride) { return {p, nullptr, nullptr, stride, 0}; }
Source source(const void *p, int64_t stride, const dipaco_packed *packed)
{
    if (!packed) return dense_source(p, stride);
    return {nullptr, static_cast<const uint8_t *>(packed->codes), static_cast<const uint8_t *>(packed->scales),
            packed->stride, (int)ceil_div(packed->cols, PACK_BLOCK)};
}

int check_args(const dipaco_residual_norm_args *a, int32_t device)
{
    if (!a || device < 0 || !is_dense_dtype(a->dtype) || !is_dense_dtype(a->param_dtype) || !is_dense_dtype(a->gate_dtype))
        return DIPACO_EINVAL;
    if (const int rc = check_extents(a->rows, a->cols)) return rc;
    if (!(a->eps >= 0.0f) || !std::isfinite(a->eps) || !std::isfinite(a->residual_scale)) return DIPACO_EINVAL;
    if (a->gate_kind < DIPACO_GATE_NONE || a->gate_kind > DIPACO_GATE_FULL) return DIPACO_EINVAL;
    const int psize = dense_size(a->param_dtype);
    for (const void *p : {a->post_gamma, a->post_beta, a->gamma, a->beta})
        if (!vector_ok(p, psize)) return DIPACO_EINVAL;
    if (!a->post_norm && (a->post_gamma || a->post_beta)) return DIPACO_EINVAL;
    if (!a->norm && (a->gamma || a->beta)) return DIPACO_EINVAL;
    if (a->rows == 0 || a->cols == 0 || a->gate_kind == DIPACO_GATE_NONE) return DIPACO_OK;
    if (!a->gate || !vector_ok(a->gate, dense_size(a->gate_dtype))) return DIPACO_EINVAL;
    if (a->gate_kind == DIPACO_GATE_FULL &&
        (a->gate_dtype != a->dtype || !dense_ok(a->gate, a->gate_stride, a->rows, a->cols, a->dtype)))
        return DIPACO_EINVAL;
    return DIPACO_OK;
}

NormArgs norm_args(const dipaco_residual_norm_args *a)
{
    NormArgs n = {};
    n.rows = (int)a->rows;
    n.cols = (int)a->cols;
    n.post_gamma = a->post_gamma;
    n.post_beta = a->post_beta;
    n.gamma = a->gamma;
    n.beta = a->beta;
    n.params_bf16 = a->param_dtype == DIPACO_BF16;
    n.gate = a->gate;
    n.gate_stride = a->gate_stride;
    n.gate_kind = a->gate_kind;
    n.gate_bf16 = a->gate_dtype == DIPACO_BF16;
    n.scale = a->residual_scale;
    n.eps = a->eps;
    n.post_norm = a->post_norm != 0;
    n.norm = a->norm != 0;
    return n;
}

template <typename T, bool VEC, int GATE> int launch_groups(const NormArgs &a, cudaStream_t stream)
{
    const int warps = (int)ceil_div(a.cols, 32 * PER_THREAD);
    const int groups = (warps <= 16 ? 16 : 32) / warps;
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(a.rows, groups), 148), threads = groups * warps * 32;
    if (warps > 16)
        group_rows_kernel<T, VEC, GATE, false, 1><<<grid, threads, 0, stream>>>(a, warps);
    else if (a.rows <= (int64_t)grid * groups)
        group_rows_kernel<T, VEC, GATE, true, 1><<<grid, threads, 0, stream>>>(a, warps);
    else
        group_rows_kernel<T, VEC, GATE, true, 2><<<grid, threads, 0, stream>>>(a, warps);
    return launch_status();
}

template <typename T> int launch_rows(const NormArgs &a, cudaStream_t stream)
{
    if (a.cols > MAX_GROUP_COLS) {
        rows_kernel<T><<<(unsigned)std::min<int64_t>(a.rows, 148 * 8), ROW_THREADS, 0, stream>>>(a);
        return launch_status();
    }
    const auto aligned = [&](const void *p, long long stride) { return !p || rows_aligned16(p, stride, a.rows, sizeof(T)); };
    const bool vec = aligned(a.x.dense, a.x.stride) && aligned(a.f.dense, a.f.stride) && aligned(a.z_out, a.z_stride) &&
                     aligned(a.n, a.n_stride) && (a.gate_kind != DIPACO_GATE_FULL || aligned(a.gate, a.gate_stride));
    switch (a.gate_kind) {
    case DIPACO_GATE_ROWS:
        return vec ? launch_groups<T, true, GATE_OF_ROW>(a, stream) : launch_groups<T, false, GATE_OF_ROW>(a, stream);
    case DIPACO_GATE_FULL:
        return vec ? launch_groups<T, true, GATE_OF_VALUES>(a, stream) : launch_groups<T, false, GATE_OF_VALUES>(a, stream);
    default:
        return vec ? launch_groups<T, true, GATE_IN_COLUMNS>(a, stream) : launch_groups<T, false, GATE_IN_COLUMNS>(a, stream);
    }
}

struct BackPlan {
    int groups;  // of a block of group_back_kernel; 0: the kernels for any width
    int parts;
    int64_t partial_bytes, bytes;
};
BackPlan plan_back(int64_t rows, int64_t cols)
{
    BackPlan p;
    if (cols <= MAX_BACK_COLS) {
        const int64_t warps = std::max<int64_t>(1, ceil_div(cols, 32 * PER_THREAD));
        p.groups = (int)(16 / warps);
        p.parts = (int)std::max<int64_t>(1, std::min<int64_t>(148, ceil_div(rows, p.groups)));
        p.partial_bytes = p.bytes = (int64_t)p.parts * 4 * cols * 4;
        return p;
    }
    const int64_t columns = ceil_div(cols, COLUMN_THREADS);
    p.groups = 0;
    p.parts = (int)std::max<int64_t>(1, std::min<int64_t>({MAX_PARTS, ceil_div(rows, 16), ceil_div(148 * 8, columns)}));
    p.partial_bytes = (int64_t)p.parts * 4 * cols * 4;
    p.bytes = ceil_div(p.partial_bytes, 16) * 16 + rows * 8;
    return p;
}

template <typename T, bool VEC> int launch_back_groups(const NormArgs &a, const BackPlan &plan, cudaStream_t stream)
{
    const int warps = (int)ceil_div(a.cols, 32 * PER_THREAD), threads = plan.groups * warps * 32;
    if (a.gate_kind == DIPACO_GATE_ROWS)
        group_back_kernel<T, VEC, GATE_OF_ROW><<<plan.parts, threads, 0, stream>>>(a, warps);
    else if (a.gate_kind == DIPACO_GATE_FULL)
        group_back_kernel<T, VEC, GATE_OF_VALUES><<<plan.parts, threads, 0, stream>>>(a, warps);
    else
        group_back_kernel<T, VEC, GATE_IN_COLUMNS><<<plan.parts, threads, 0, stream>>>(a, warps);
    return launch_status();
}

template <typename T> int launch_back(const NormArgs &a, const BackPlan &plan, cudaStream_t stream)
{
    if (plan.groups == 0) {
        back_rows_kernel<T><<<(unsigned)std::min<int64_t>(a.rows, 148 * 8), ROW_THREADS, 0, stream>>>(a);
        if (const int rc = launch_status()) return rc;
        const dim3 columns((unsigned)ceil_div(a.cols, COLUMN_THREADS), (unsigned)plan.parts);
        back_columns_kernel<T><<<columns, COLUMN_THREADS, 0, stream>>>(a);
        return launch_status();
    }
    const auto aligned = [&](const void *p, long long stride) { return !p || rows_aligned16(p, stride, a.rows, sizeof(T)); };
    const bool vec = aligned(a.dn.dense, a.dn.stride) && aligned(a.dz.dense, a.dz.stride) && aligned(a.f.dense, a.f.stride) &&
                     aligned(a.z.dense, a.z.stride) && aligned(a.dx, a.dx_stride) && aligned(a.df, a.df_stride) &&
                     (a.gate_kind != DIPACO_GATE_FULL || (aligned(a.gate, a.gate_stride) && aligned(a.dgate, a.dgate_stride)));
    return vec ? launch_back_groups<T, true>(a, plan, stream) : launch_back_groups<T, false>(a, plan, stream);
}

} // namespace

extern "C" {

int dipaco_residual_norm(const dipaco_residual_norm_args *args, const void *x, int64_t x_stride, const void *f,
                         int64_t f_stride, void *z, int64_t z_stride, void *n, int64_t n_stride,
                         const dipaco_packed *n_packed, const dipaco_packed *z_packed, float *stats, int32_t device,
                         void *cuda_stream)
{
    if (const int rc = check_args(args, device)) return rc;
    const int64_t rows = args->rows, cols = args->cols;
    if (!dense_ok(x, x_stride, rows, cols, args->dtype) || !dense_ok(f, f_stride, rows, cols, args->dtype) ||
        !dense_ok(z, z_stride, rows, cols, args->dtype))
        return DIPACO_EINVAL;
    if ((n || n_packed) && !args->norm) return DIPACO_EINVAL;
    if ((n && n_packed) || (z_packed && !n_packed)) return DIPACO_EINVAL;
    if (n && !dense_ok(n, n_stride, rows, cols, args->dtype)) return DIPACO_EINVAL;
    if ((n_packed && !packed_ok(n_packed, rows, cols)) || (z_packed && !packed_ok(z_packed, rows, cols))) return DIPACO_EINVAL;
    if (!vector_ok(stats, 4)) return DIPACO_EINVAL;
    if (rows == 0) return DIPACO_OK;
    if (!stats) return DIPACO_EINVAL;

    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    NormArgs a = norm_args(args);
    if (cols == 0) {
        empty_rows_kernel<<<(unsigned)std::min<int64_t>(ceil_div(rows, 256), 148), 256, 0, stream>>>(stats, a.rows, a.post_norm, a.norm);
        return launch_status();
    }
    a.x = dense_source(x, x_stride);
    a.f = dense_source(f, f_stride);
    a.z_out = z;
    a.z_stride = z_stride;
    a.n = n;
    a.n_stride = n_stride;
    a.stats = stats;
    if (const int rc = args->dtype == DIPACO_BF16 ? launch_rows<__nv_bfloat16>(a, stream) : launch_rows<float>(a, stream)) return rc;
    if (!n_packed) return DIPACO_OK;
    return pack_normalised(z, z_stride, args->dtype, stats + 2 * rows, stats + 3 * rows, args->gamma, args->beta,
                           args->param_dtype, n_packed, z_packed, stream);
}

int dipaco_residual_norm_workspace(int64_t rows, int64_t cols, int64_t *bytes)
{
    if (!bytes) return DIPACO_EINVAL;
    if (const int rc = check_extents(rows, cols)) return rc;
    *bytes = rows == 0 || cols == 0 ? 0 : plan_back(rows, cols).bytes;
    return DIPACO_OK;
}

int dipaco_residual_norm_backward(const dipaco_residual_norm_args *args, const void *dn, int64_t dn_stride, const void *dz,
                                  int64_t dz_stride, const void *f, int64_t f_stride, const dipaco_packed *f_packed,
                                  const void *z, int64_t z_stride, const dipaco_packed *z_packed, const float *stats,
                                  void *dx, int64_t dx_stride, void *df, int64_t df_stride, void *dgate,
                                  int64_t dgate_stride, float *dgamma, float *dbeta, float *dpost_gamma,
                                  float *dpost_beta, void *workspace, int64_t workspace_bytes, int32_t device,
                                  void *cuda_stream)
{
    if (const int rc = check_args(args, device)) return rc;
    const int64_t rows = args->rows, cols = args->cols;
    const int dtype = args->dtype;
    const bool values = rows > 0 && cols > 0;
    if (args->norm) {
        if (!dense_ok(dn, dn_stride, rows, cols, dtype)) return DIPACO_EINVAL;
        if (values && !z == !z_packed) return DIPACO_EINVAL;
        if (z_packed ? !packed_ok(z_packed, rows, cols) : !dense_ok(z, z_stride, rows, cols, dtype)) return DIPACO_EINVAL;
    } else if (dn || dgamma || dbeta) {
        return DIPACO_EINVAL;
    }
    if (dz && !dense_ok(dz, dz_stride, rows, cols, dtype)) return DIPACO_EINVAL;
    if (values && !f == !f_packed) return DIPACO_EINVAL;
    if (f_packed ? !packed_ok(f_packed, rows, cols) : !dense_ok(f, f_stride, rows, cols, dtype)) return DIPACO_EINVAL;
    if (!args->post_norm && (dpost_gamma || dpost_beta)) return DIPACO_EINVAL;
    if (dgate && args->gate_kind == DIPACO_GATE_NONE) return DIPACO_EINVAL;
    if ((dx && !dense_ok(dx, dx_stride, rows, cols, dtype)) || (df && !dense_ok(df, df_stride, rows, cols, dtype))) return DIPACO_EINVAL;
    if (dgate && args->gate_kind == DIPACO_GATE_FULL && !dense_ok(dgate, dgate_stride, rows, cols, dtype)) return DIPACO_EINVAL;
    if (args->gate_kind != DIPACO_GATE_FULL && !vector_ok(dgate, 4)) return DIPACO_EINVAL;
    for (const void *p : {(const void *)stats, (const void *)dgamma, (const void *)dbeta, (const void *)dpost_gamma, (const void *)dpost_beta})
        if (!vector_ok(p, 4)) return DIPACO_EINVAL;
    if (values && !stats) return DIPACO_EINVAL;
    const BackPlan plan = plan_back(rows, cols);
    if (values && (!workspace || (uintptr_t)workspace % 16 != 0 || workspace_bytes < plan.bytes)) return DIPACO_EINVAL;
    if (!values && rows == 0 && cols == 0) return DIPACO_OK;

    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    float *const dgate_cols = args->gate_kind == DIPACO_GATE_COLS ? static_cast<float *>(dgate) : nullptr;
    if (!values) {  // sums over nothing
        for (float *p : {dgate_cols, dgamma, dbeta, dpost_gamma, dpost_beta})
            if (p && cols > 0 && cudaMemsetAsync(p, 0, cols * sizeof(float), stream) != cudaSuccess) return launch_status();
        if (args->gate_kind == DIPACO_GATE_ROWS && dgate && rows > 0 &&
            cudaMemsetAsync(dgate, 0, rows * sizeof(float), stream) != cudaSuccess)
            return launch_status();
        return DIPACO_OK;
    }
    NormArgs a = norm_args(args);
    a.dn = dense_source(dn, dn_stride);
    a.dz = dense_source(dz, dz_stride);
    a.f = source(f, f_stride, f_packed);
    a.z = source(z, z_stride, z_packed);
    a.saved = stats;
    a.dx = dx;
    a.dx_stride = dx_stride;
    a.df = df;
    a.df_stride = df_stride;
    a.dgate = args->gate_kind == DIPACO_GATE_COLS ? nullptr : dgate;
    a.dgate_stride = dgate_stride;
    a.partial = static_cast<float *>(workspace);
    a.row_means = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + ceil_div(plan.partial_bytes, 16) * 16);
    a.parts = plan.parts;
    if (const int rc = dtype == DIPACO_BF16 ? launch_back<__nv_bfloat16>(a, plan, stream) : launch_back<float>(a, plan, stream)) return rc;
    if (!dgate_cols && !dgamma && !dbeta && !dpost_gamma && !dpost_beta) return DIPACO_OK;
    JoinArgs j = {};
    j.partial = a.partial;
    j.parts = plan.parts;
    j.cols = a.cols;
    j.gate = args->gate;
    j.gate_cols = args->gate_kind == DIPACO_GATE_COLS;
    j.gate_bf16 = a.gate_bf16;
    j.post_gamma = args->post_gamma;
    j.post_beta = args->post_beta;
    j.params_bf16 = a.params_bf16;
    j.post_norm = a.post_norm;
    j.dgate = dgate_cols;
    j.dgamma = dgamma;
    j.dbeta = dbeta;
    j.dpost_gamma = dpost_gamma;
    j.dpost_beta = dpost_beta;
    join_kernel<<<(unsigned)ceil_div(cols, 32), 32 * JOIN_SLICES, 0, stream>>>(j);
    return launch_status();
}

} // extern "C"
