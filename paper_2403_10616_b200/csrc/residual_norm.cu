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
//   group_back_kernel every gradient in one pass, a row in the registers of a group: up to 8192 columns
//   back_rows_kernel  as rows_kernel for dx, df and the two means that d needs; back_columns_kernel the sums over rows
//
// Measured: 16384x2048 in bf16 54 us (5.0 TB/s) and its gradient 97 (4.1 TB/s), 32768x896 49 and 98, with n and z
// packed 64 (the packing kernel reads z from L2) and from such checkpoints 108, 4999x2047 in fp32 45 and 66, 4096x8192 in
// bf16 77 and 171 (gates of columns); a single row of 896 4.5 and 10.
// Two reads and two writes would take 41 us of the first, four and two 61 of its gradient.  The forward kernel is bound by
// chains (each row's two sums, one after the other, in 16 warps; issue slots 54 % used), the gradient too: its sums over
// rows take half of the registers, which leaves 12 warps (issue slots 46 %).
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

// A group of warps has a row, 8 U values for each thread, which stay in registers from the first sum to the last
// result.  VEC (rows on 16-byte boundaries, of whole units of eight): a thread's units are `threads` units apart; else a
// thread has every `threads`-th value, so that a warp's accesses stay whole.  Parameters wait in shared memory.

struct Group {
    int warps, index, warp, lane;
    int thread, threads;              // of the group
    int other;                        // the warp whose values this lane joins
    float count;                      // how many values that warp has; 0: none to join
    float of_first, of_warp, of_row;  // 1 / number of values of the warp's first lane, of the warp, of the row
    float2 *slots;                    // [2][warps][rows], shared
    int parity = 0;

    // A barrier of this group's own.
    __device__ __forceinline__ void sync() const
    {
        asm volatile("bar.sync %0, %1;" ::"r"(index + 1), "r"(threads) : "memory");
    }
};

// Value j of a thread of the group, and whether it belongs to the row.
template <bool VEC> __device__ __forceinline__ int column(int threads, int thread, int j)
{
    return VEC ? ((j >> 3) * threads + thread) * 8 + (j & 7) : j * threads + thread;
}
template <bool VEC, int U> __device__ __forceinline__ unsigned valid_values(int threads, int thread, int cols)
{
    unsigned valid = 0u;
#pragma unroll
    for (int j = 0; j < 8 * U; ++j)
        if (column<VEC>(threads, thread, j) < cols) valid |= 1u << j;
    return valid;
}

template <bool VEC, int U>
__device__ __forceinline__ Group make_group(int warps, int cols, float2 *slots, int rows)
{
    Group g;
    g.warps = warps;
    g.threads = warps * 32;
    g.lane = threadIdx.x & 31;
    g.index = (int)(threadIdx.x >> 5) / warps;
    g.warp = (int)(threadIdx.x >> 5) - g.index * warps;
    g.thread = g.warp * 32 + g.lane;
    g.slots = slots + 2 * g.index * warps * rows;
    const auto values_of_warp = [&](int warp) {  // its 32 threads' runs of units, or of values
        int n = 0;
#pragma unroll
        for (int u = 0; u < (VEC ? U : 8 * U); ++u) {
            constexpr int run = VEC ? 8 : 1;
            n += min(max(cols - (u * g.threads + warp * 32) * run, 0), 32 * run);
        }
        return n;
    };
    const int joined = warps <= 8 ? g.lane & 7 : g.lane;
    g.other = min(joined, warps - 1);
    g.count = joined < warps ? (float)values_of_warp(joined) : 0.0f;
    g.of_first = 1.0f / (float)__popc(valid_values<VEC, U>(g.threads, g.warp * 32, cols));
    g.of_warp = 1.0f / (float)values_of_warp(g.warp);
    g.of_row = 1.0f / (float)cols;
    return g;
}

// A thread's values of a row as they are in memory.
template <typename T, int U> struct RowRaw {
    unsigned w[8 * U * sizeof(T) / 4];
};
template <typename T, bool VEC, int U>
__device__ __forceinline__ void load_row(const void *row, const Group &g, unsigned valid, RowRaw<T, U> &raw)
{
    constexpr int UE = Unit<T>::UE;
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < 8 * U / UE; ++i) {
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (valid >> (i * UE) & 1u) v = __ldcs(static_cast<const uint4 *>(row) + column<true>(g.threads, g.thread, i * UE) / UE);
            raw.w[4 * i] = v.x; raw.w[4 * i + 1] = v.y; raw.w[4 * i + 2] = v.z; raw.w[4 * i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8 * U; ++j) {
            unsigned v = 0u;
            if (valid >> j & 1u) {
                if constexpr (sizeof(T) == 2)
                    v = __ldcs(static_cast<const unsigned short *>(row) + column<false>(g.threads, g.thread, j));
                else
                    v = __ldcs(static_cast<const unsigned *>(row) + column<false>(g.threads, g.thread, j));
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
// A row of a gate of values that the next pass loads, into L2.  Without and with it, us:
//   forward    bf16 gains (16384x2048 76 and 70, 32768x896 66 and 60, 2048x8191 107 and 95), fp32 loses (8192x2048 65.5 and
//              66.5, 4999x2047 57 and 60, 3001x5555 115 and 123)
//   gradient   up to 6144 columns bf16 gains (133 and 121, 128 and 118, 4000x6144 116 and 104), and fp32 value by value in
//              most (82 and 78, 175 and 158; 20000x333 67.6 and 69); whole units of fp32 lose (107.5 and 114.5), and more
//              columns in either type (4096x8192 bf16 236 and 256, 2048x8191 fp32 226 and 250)
template <typename T, bool VEC, int U>
__device__ __forceinline__ void prefetch_row(const void *row, const Group &g, unsigned valid)
{
    constexpr int EACH = VEC ? Unit<T>::UE : 1;  // values of a load
    if (g.lane % (128 / EACH / (int)sizeof(T)) != 0) return;  // a lane for each 128 bytes
#pragma unroll
    for (int j = 0; j < 8 * U; j += EACH)
        if (valid >> j & 1u)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const T *>(row) + column<VEC>(g.threads, g.thread, j)));
}
template <typename T, int U> __device__ __forceinline__ void widen_row(const RowRaw<T, U> &raw, f32x2 *v)
{
    constexpr int UE = Unit<T>::UE;
#pragma unroll
    for (int i = 0; i < 8 * U / UE; ++i)
        widen_pairs<T>(make_uint4(raw.w[4 * i], raw.w[4 * i + 1], raw.w[4 * i + 2], raw.w[4 * i + 3]), v + i * UE / 2);
}
template <typename T, int U> __device__ __forceinline__ void narrow_row(const f32x2 *v, RowRaw<T, U> &raw)
{
    constexpr int UE = Unit<T>::UE;
#pragma unroll
    for (int i = 0; i < 8 * U / UE; ++i) {
        const uint4 u = narrow_pairs<T>(v + i * UE / 2);
        raw.w[4 * i] = u.x; raw.w[4 * i + 1] = u.y; raw.w[4 * i + 2] = u.z; raw.w[4 * i + 3] = u.w;
    }
}
template <typename T, bool VEC, int U>
__device__ __forceinline__ void store_row(void *row, const Group &g, unsigned valid, const RowRaw<T, U> &raw)
{
    constexpr int UE = Unit<T>::UE;
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < 8 * U / UE; ++i)
            if (valid >> (i * UE) & 1u)
                static_cast<uint4 *>(row)[column<true>(g.threads, g.thread, i * UE) / UE] =
                    make_uint4(raw.w[4 * i], raw.w[4 * i + 1], raw.w[4 * i + 2], raw.w[4 * i + 3]);
    } else {
#pragma unroll
        for (int j = 0; j < 8 * U; ++j)
            if (valid >> j & 1u) {
                if constexpr (sizeof(T) == 2)
                    static_cast<unsigned short *>(row)[column<false>(g.threads, g.thread, j)] = (unsigned short)(raw.w[j / 2] >> 16 * (j & 1));
                else
                    static_cast<unsigned *>(row)[column<false>(g.threads, g.thread, j)] = raw.w[j];
            }
    }
}

// A vector of parameters in shared memory, as the threads read it: in VEC form the first and the last four of every
// unit apart, so that a warp's loads do not conflict.
template <bool VEC> __device__ __forceinline__ int param_place(int col, int cols)
{
    return VEC ? ((col >> 2 & 1) * (cols >> 3) + (col >> 3)) * 4 + (col & 3) : col;
}
// Which of the row's units are the thread's (VEC); any that is there, where there is none.
template <int U> struct Places {
    int thread, threads, last;
    __device__ Places(const Group &g, int cols) : thread(g.thread), threads(g.threads), last(max((cols >> 3) - 1, 0)) {}
    __device__ __forceinline__ int unit(int u) const { return min(u * threads + thread, last); }
};
// Parameters to shared memory, in the gradient some times the gate of columns.  The loads of four columns are all under
// way before the first is used: one after another they were half of a call of few rows (40x6316 in fp32 19.7 us, now 10.2).
struct HeldParam {
    const void *p;
    bool bf16;
    float otherwise;
    const void *gate;  // of columns, or NULL
};
template <bool VEC, int N>
__device__ __forceinline__ void hold_params(const NormArgs &a, const HeldParam *params, float *held)
{
    const auto bits_at = [](const void *p, bool bf16, int c) -> unsigned {
        if (!p) return 0u;
        return bf16 ? __ldg(static_cast<const unsigned short *>(p) + c) : __ldg(static_cast<const unsigned *>(p) + c);
    };
    const auto value_of_bits = [](unsigned bits, bool bf16) { return __uint_as_float(bf16 ? bits << 16 : bits); };
    for (int first = threadIdx.x; first < a.cols; first += 4 * blockDim.x) {
        unsigned bits[4][N], gate_bits[4][N];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = min(first + i * (int)blockDim.x, a.cols - 1);
#pragma unroll
            for (int q = 0; q < N; ++q) {
                bits[i][q] = bits_at(params[q].p, params[q].bf16, c);
                gate_bits[i][q] = bits_at(params[q].gate, a.gate_bf16, c);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = first + i * (int)blockDim.x;
            if (c >= a.cols) break;
#pragma unroll
            for (int q = 0; q < N; ++q) {
                float v = params[q].p ? value_of_bits(bits[i][q], params[q].bf16) : params[q].otherwise;
                if (params[q].gate) v *= value_of_bits(gate_bits[i][q], a.gate_bf16);
                held[q * a.cols + param_place<VEC>(c, a.cols)] = v;
            }
        }
    }
}
template <bool VEC, int U>
__device__ __forceinline__ void held_columns(const float *held, const Group &g, const Places<U> &places, int cols, int unit, f32x2 *v)
{
    if constexpr (VEC) {
        const int at = places.unit(unit);
        const float4 *p = reinterpret_cast<const float4 *>(held);
        const float4 lo = p[at], hi = p[(cols >> 3) + at];
        v[0] = pair_of(lo.x, lo.y); v[1] = pair_of(lo.z, lo.w);
        v[2] = pair_of(hi.x, hi.y); v[3] = pair_of(hi.z, hi.w);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = pair_of(held[min(column<false>(g.threads, g.thread, 8 * unit + 2 * i), cols - 1)],
                           held[min(column<false>(g.threads, g.thread, 8 * unit + 2 * i + 1), cols - 1)]);
    }
}

// What a unit adds to a sum: nothing from values that are not the row's.
template <bool VEC> __device__ __forceinline__ void keep_valid(unsigned valid, int unit, f32x2 *v)  // before the sum
{
    if constexpr (!VEC) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 w = values_of(v[i]);
            v[i] = pair_of(valid >> (8 * unit + 2 * i) & 1u ? w.x : 0.0f, valid >> (8 * unit + 2 * i + 1) & 1u ? w.y : 0.0f);
        }
    }
}
template <bool VEC> __device__ __forceinline__ f32x2 if_valid(unsigned valid, int unit, f32x2 sum)  // after it
{
    return !VEC || (valid >> (8 * unit) & 1u) ? sum : 0ull;
}
__device__ __forceinline__ f32x2 sum4(const f32x2 *v) { return add2(add2(v[0], v[1]), add2(v[2], v[3])); }

// Sums of R pairs of values over the warp.
template <int R, int FROM = 16> __device__ __forceinline__ void warp_sums(float2 *sums)
{
#pragma unroll
    for (int o = FROM; o > 0; o >>= 1)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            sums[r].x += __shfl_xor_sync(0xffffffffu, sums[r].x, o);
            sums[r].y += __shfl_xor_sync(0xffffffffu, sums[r].y, o);
        }
}
// The same of what lanes have of the warps: of up to eight by every eight lanes.
template <int R> __device__ __forceinline__ void join_warps(const Group &g, float2 *sums)
{
    if (g.warps <= 8)
        warp_sums<R, 4>(sums);
    else
        warp_sums<R>(sums);
}
// Hands the warps' values round, [warp][R], in two sets that take turns: a set is written again only after everyone
// has read it.
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

// Mean and 1 / sqrt(var + eps) of the group's row.  Differences are taken from the mean of the warp's first lane's
// values: it is exact where all values are equal, and no farther from the warp's mean than the spread of the warp's
// values times sqrt(32), so that the squares lose five bits at most.  The warps are joined about the first one's mean.
// In units that are not the row's there may be anything (VEC; zeros otherwise): they are left out of every sum.
template <bool VEC, int U>
__device__ __forceinline__ float2 group_statistics(Group &g, const f32x2 *v, unsigned valid, float eps)
{
    f32x2 first = sum4(v);  // the first lane's first unit is the row's
#pragma unroll
    for (int u = 1; u < U; ++u) first = add2(first, if_valid<VEC>(valid, u, sum4(v + 4 * u)));
    const float centre = __shfl_sync(0xffffffffu, sum_of(first) * g.of_first, 0);
    f32x2 all = 0ull, squares = 0ull;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        f32x2 d[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = add2(v[4 * u + i], pair_of(-centre));
        keep_valid<VEC>(valid, u, d);
        f32x2 s = mul2(d[0], d[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) s = fma2(d[i], d[i], s);
        all = add2(all, if_valid<VEC>(valid, u, sum4(d)));
        squares = add2(squares, if_valid<VEC>(valid, u, s));
    }
    float2 sums = make_float2(sum_of(all), sum_of(squares));
    warp_sums<1>(&sums);
    float off = sums.x * g.of_warp;
    sums = make_float2(centre + off, fmaxf(fmaf(-off, sums.x, sums.y), 0.0f));
    if (g.warps > 1) {
        const float2 *slots = exchange<1>(g, &sums);
        const float about = slots[0].x;
        const float2 of = slots[g.other];
        const float apart = of.x - about;
        sums = g.count > 0.0f ? make_float2(g.count * apart, fmaf(g.count * apart, apart, of.y)) : make_float2(0.0f, 0.0f);
        join_warps<1>(g, &sums);
        off = sums.x * g.of_row;
        sums = make_float2(about + off, fmaxf(fmaf(-off, sums.x, sums.y), 0.0f));
    }
    return make_float2(sums.x, rsqrtf(fmaf(sums.y, g.of_row, eps)));
}

// GATE: what a thread needs for it.
enum : int { GATE_IN_COLUMNS, GATE_OF_ROW, GATE_OF_VALUES };

constexpr int MAX_GROUP_COLS = 8192;  // 160 KB of parameters in shared memory

// Vectors that the threads of group_rows_kernel read from there.  A gate of columns is one of its own: multiplied into
// the others it would turn gate (h post_gamma + 0) into NaN where it is infinite, and overflow where gate p does not.
template <int GATE> constexpr int HELD_VECTORS = GATE == GATE_IN_COLUMNS ? 5 : 4;

template <typename T, bool VEC, int GATE, int U>
__global__ void __launch_bounds__(512, 1) group_rows_kernel(const __grid_constant__ NormArgs a, int warps)
{
    constexpr int P = 4 * U;
    extern __shared__ __align__(16) float held[];  // [HELD_VECTORS][cols]: p = h factor + shift; gamma, beta; gate
    __shared__ float2 slots[2 * 16];
    Group g = make_group<VEC, U>(warps, a.cols, slots, 1);
    const int groups = (int)(blockDim.x >> 5) / warps;
    const unsigned valid = valid_values<VEC, U>(g.threads, g.thread, a.cols);
    const Places<U> places(g, a.cols);
    const int row_step = gridDim.x * groups;
    int row = blockIdx.x * groups + g.index;
    const T *f_row = static_cast<const T *>(a.f.dense) + row * a.f.stride, *x_row = static_cast<const T *>(a.x.dense) + row * a.x.stride;
    const long long f_step = row_step * a.f.stride, x_step = row_step * a.x.stride;
    RowRaw<T, U> next_x, next_f;
    if (row < a.rows) {
        load_row<T, VEC, U>(f_row, g, valid, next_f);
        load_row<T, VEC, U>(x_row, g, valid, next_x);
    }
    const bool bf16 = a.params_bf16;
    const HeldParam params[5] = {{a.post_gamma, bf16, 1.0f, nullptr}, {a.post_beta, bf16, 0.0f, nullptr},
                                 {a.gamma, bf16, 1.0f, nullptr}, {a.beta, bf16, 0.0f, nullptr},
                                 {a.gate_kind == DIPACO_GATE_COLS ? a.gate : nullptr, a.gate_bf16, 1.0f, nullptr}};
    hold_params<VEC, HELD_VECTORS<GATE>>(a, params, held);
    __syncthreads();
    for (; row < a.rows; row += row_step) {
        f32x2 v[P];
        widen_row<T, U>(next_f, v);
        const RowRaw<T, U> x = next_x;
        if (row < a.rows - row_step) {
            f_row += f_step;
            x_row += x_step;
            load_row<T, VEC, U>(f_row, g, valid, next_f);
            load_row<T, VEC, U>(x_row, g, valid, next_x);
            if (GATE == GATE_OF_VALUES && sizeof(T) == 2) prefetch_row<T, VEC, U>(static_cast<const T *>(a.gate) + (row + row_step) * a.gate_stride, g, valid);
        }
        float2 of_f = make_float2(0.0f, 1.0f), of_z = make_float2(0.0f, 1.0f);
        if (a.post_norm) of_f = group_statistics<VEC, U>(g, v, valid, a.eps);
        RowRaw<T, U> raw;
        if (GATE == GATE_OF_VALUES) load_row<T, VEC, U>(static_cast<const T *>(a.gate) + row * a.gate_stride, g, valid, raw);
        const f32x2 of_row = pair_of(GATE == GATE_OF_ROW ? load_param(a.gate, a.gate_bf16, row) : 0.0f);
        f32x2 stream[P], gate[P];
        widen_row<T, U>(x, stream);
        if (GATE == GATE_OF_VALUES) widen_row<T, U>(raw, gate);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            f32x2 factor[4], shift[4], by[4];
            held_columns<VEC, U>(held, g, places, a.cols, u, factor);
            held_columns<VEC, U>(held + a.cols, g, places, a.cols, u, shift);
            if (GATE == GATE_IN_COLUMNS) held_columns<VEC, U>(held + 4 * a.cols, g, places, a.cols, u, by);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = 4 * u + i;
                const f32x2 p = fma2(mul2(add2(v[k], pair_of(-of_f.x)), pair_of(of_f.y)), factor[i], shift[i]);
                v[k] = fma2(GATE == GATE_IN_COLUMNS ? by[i] : GATE == GATE_OF_ROW ? of_row : gate[k], p,
                            mul2(stream[k], pair_of(a.scale)));
            }
            keep_valid<VEC>(valid, u, v + 4 * u);
        }
        narrow_row<T, U>(v, raw);
        store_row<T, VEC, U>(static_cast<T *>(a.z_out) + row * a.z_stride, g, valid, raw);
        if (a.norm) {
            widen_row<T, U>(raw, v);
            of_z = group_statistics<VEC, U>(g, v, valid, a.eps);
            if (a.n) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    f32x2 gamma[4], beta[4];
                    held_columns<VEC, U>(held + 2 * a.cols, g, places, a.cols, u, gamma);
                    held_columns<VEC, U>(held + 3 * a.cols, g, places, a.cols, u, beta);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        v[4 * u + i] = fma2(mul2(add2(v[4 * u + i], pair_of(-of_z.x)), pair_of(of_z.y)), gamma[i], beta[i]);
                }
                narrow_row<T, U>(v, raw);
                store_row<T, VEC, U>(static_cast<T *>(a.n) + row * a.n_stride, g, valid, raw);
            }
        }
        if (g.thread == 0) {
            a.stats[row] = of_f.x;
            a.stats[a.rows + row] = of_f.y;
            a.stats[2ll * a.rows + row] = of_z.x;
            a.stats[3ll * a.rows + row] = of_z.y;
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

static __device__ int g_residual_norm_error;  // set by a bounded wait that ran out

// Rows on their way to shared memory: bulk copies of the 16-byte units that hold a row, a stage of the ring for a row of
// dn, z, dz and f.
struct Feed {
    const uint8_t *first;  // row 0
    long long step;        // bytes from row to row
    int bytes;             // of a row; 0: not there

    __device__ __forceinline__ const uint8_t *row(long long at) const { return first + at * step; }
    // How far into its first unit a row begins.
    __device__ __forceinline__ int ahead(long long at) const { return (int)(reinterpret_cast<uintptr_t>(row(at)) & 15u); }
    __device__ __forceinline__ unsigned copied(long long at) const { return (unsigned)(ahead(at) + bytes + 15) & ~15u; }
};
template <typename T> __device__ __forceinline__ Feed make_feed(const Source &s, int cols)
{
    if (s.codes) return {s.codes, s.stride, cols};
    return {static_cast<const uint8_t *>(s.dense), s.stride * (long long)sizeof(T), s.dense ? cols * (int)sizeof(T) : 0};
}

// A row's values in shared memory; where there are none, any of the row.
template <typename T, bool VEC, int U>
__device__ __forceinline__ void read_row(const uint8_t *at, const Group &g, const Places<U> &places, int cols, f32x2 *v)
{
    constexpr int UE = Unit<T>::UE;
    if constexpr (VEC) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint4 *p = reinterpret_cast<const uint4 *>(at) + places.unit(u) * (8 / UE);
#pragma unroll
            for (int i = 0; i < 8 / UE; ++i) widen_pairs<T>(p[i], v + 4 * u + i * UE / 2);
        }
    } else {
        const T *p = reinterpret_cast<const T *>(at);
#pragma unroll
        for (int i = 0; i < 4 * U; ++i)
            v[i] = pair_of(widen1<T>(p[min(column<false>(g.threads, g.thread, 2 * i), cols - 1)]),
                           widen1<T>(p[min(column<false>(g.threads, g.thread, 2 * i + 1), cols - 1)]));
    }
}
template <typename T, bool VEC, int U>
__device__ __forceinline__ void read_source(const Source &s, int row, const uint8_t *at, const Group &g, const Places<U> &places, int cols, f32x2 *v)
{
    if (s.dense) {
        read_row<T, VEC, U>(at, g, places, cols, v);
        return;
    }
    const uint8_t *scales = s.scales + (long long)(row / PACK_BLOCK) * s.scale_cols;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if constexpr (VEC) {
            const int unit = places.unit(u);
            const uint2 w = reinterpret_cast<const uint2 *>(at)[unit];
            const f32x2 scale = pair_of(scale_value(scales[unit * 8 / PACK_BLOCK]));
            v[4 * u] = mul2(decode_pair(w.x), scale);
            v[4 * u + 1] = mul2(decode_pair(w.x >> 16), scale);
            v[4 * u + 2] = mul2(decode_pair(w.y), scale);
            v[4 * u + 3] = mul2(decode_pair(w.y >> 16), scale);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c0 = min(column<false>(g.threads, g.thread, 8 * u + 2 * i), cols - 1);
                const int c1 = min(column<false>(g.threads, g.thread, 8 * u + 2 * i + 1), cols - 1);
                v[4 * u + i] = mul2(decode_pair(at[c0] | (unsigned)at[c1] << 8),
                                    pair_of(scale_value(scales[c0 / PACK_BLOCK]), scale_value(scales[c1 / PACK_BLOCK])));
            }
        }
    }
}
// Zeros where there are no values.
template <bool VEC, int U> __device__ __forceinline__ void keep_valid_row(unsigned valid, f32x2 *v)
{
    if (valid == (1u << (8 * U)) - 1u) return;
#pragma unroll
    for (int i = 0; i < 4 * U; ++i) {
        const float2 w = values_of(v[i]);
        v[i] = pair_of(valid >> (2 * i) & 1u ? w.x : 0.0f, valid >> (2 * i + 1) & 1u ? w.y : 0.0f);
    }
}

// Sums of R pairs over the group, on every thread.
template <int R> __device__ __forceinline__ void group_sums(Group &g, float2 *sums)
{
    warp_sums<R>(sums);
    if (g.warps == 1) return;
    const float2 *slots = exchange<R>(g, sums);
#pragma unroll
    for (int r = 0; r < R; ++r) sums[r] = g.count > 0.0f ? slots[g.other * R + r] : make_float2(0.0f, 0.0f);
    join_warps<R>(g, sums);
}

constexpr int MAX_BACK_COLS = 8192;
constexpr int MAX_STAGES = 4;
constexpr int BACK_SMEM = 226 * 1024;

// A persistent block of groups, each with a row at a time; a thread keeps the sums over its rows of its columns.  A
// ring of `stages` rows on their way for each group.
template <typename T, bool VEC, int GATE, int U, int THREADS>
__global__ void __launch_bounds__(THREADS, 1) group_back_kernel(const __grid_constant__ NormArgs a, int warps, int stages, int buffer)
{
    constexpr int P = 4 * U;
    extern __shared__ __align__(16) float held[];  // [3][cols]: gamma; post_gamma, times a gate of columns; post_beta
    __shared__ float2 slots[2 * 16 * 2];
    __shared__ uint64_t full[16 * MAX_STAGES];
    Group g = make_group<VEC, U>(warps, a.cols, slots, 2);
    const int groups = (int)(blockDim.x >> 5) / warps;
    const unsigned valid = valid_values<VEC, U>(g.threads, g.thread, a.cols);
    const Places<U> places(g, a.cols);
    const int row_step = gridDim.x * groups;
    int row = blockIdx.x * groups + g.index;
    uint8_t *ring = reinterpret_cast<uint8_t *>(held) + (a.cols * 12 + 15) / 16 * 16 + g.index * stages * 4 * buffer;
    uint64_t *arrived = full + g.index * stages;
    const Feed dn = make_feed<T>(a.dn, a.cols), z = make_feed<T>(a.z, a.cols), dz = make_feed<T>(a.dz, a.cols), f = make_feed<T>(a.f, a.cols);
    const auto request = [&](int at, int stage) {  // one thread
        uint8_t *to = ring + stage * 4 * buffer;
        unsigned bytes = f.copied(at);
        if (a.norm) bytes += dn.copied(at) + z.copied(at);
        if (dz.bytes) bytes += dz.copied(at);
        ptx::mbar_arrive_expect_tx(&arrived[stage], bytes);
        if (a.norm) {
            ptx::bulk_load(to, dn.row(at) - dn.ahead(at), dn.copied(at), &arrived[stage]);
            ptx::bulk_load(to + buffer, z.row(at) - z.ahead(at), z.copied(at), &arrived[stage]);
        }
        if (dz.bytes) ptx::bulk_load(to + 2 * buffer, dz.row(at) - dz.ahead(at), dz.copied(at), &arrived[stage]);
        ptx::bulk_load(to + 3 * buffer, f.row(at) - f.ahead(at), f.copied(at), &arrived[stage]);
    };
    if (g.thread == 0) {
        for (int s = 0; s < stages; ++s) ptx::mbar_init(&arrived[s], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int s = 0; s < stages && row + (long long)s * row_step < a.rows; ++s) request(row + s * row_step, s);
    }
    const bool bf16 = a.params_bf16;
    const HeldParam params[3] = {{a.gamma, bf16, 1.0f, nullptr},
                                 {a.post_gamma, bf16, 1.0f, a.gate_kind == DIPACO_GATE_COLS ? a.gate : nullptr},
                                 {a.post_beta, bf16, 0.0f, nullptr}};
    hold_params<VEC, 3>(a, params, held);
    __syncthreads();
    f32x2 sums[4][P];
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < P; ++i) sums[q][i] = 0ull;

    int stage = 0;
    unsigned phase = 0;
    bool ok = true;  // a wait that runs out leaves the results undefined, but every barrier is met
    for (; row < a.rows; row += row_step) {
        const uint8_t *from = ring + stage * 4 * buffer;
        float mean_f = 0.0f, rstd_f = 1.0f, mean_z = 0.0f, rstd_z = 1.0f;
        if (a.post_norm) {
            mean_f = a.saved[row];
            rstd_f = a.saved[a.rows + row];
        }
        if (a.norm) {
            mean_z = a.saved[2ll * a.rows + row];
            rstd_z = a.saved[3ll * a.rows + row];
        }
        const float of_row = GATE == GATE_OF_ROW ? load_param(a.gate, a.gate_bf16, row) : 1.0f;
        constexpr bool wide = U == 2 && THREADS == 512;  // over 6144 columns
        if (GATE == GATE_OF_VALUES && !wide && (sizeof(T) == 2 || !VEC) && row < a.rows - row_step)
            prefetch_row<T, VEC, U>(static_cast<const T *>(a.gate) + (row + row_step) * a.gate_stride, g, valid);
        if (ok) ok = __all_sync(0xffffffffu, bounded_wait(&arrived[stage], phase, &g_residual_norm_error, 1));  // one answer for a warp
        f32x2 d[P], h[P];
        if (dz.bytes) {
            read_row<T, VEC, U>(from + 2 * buffer + (VEC ? 0 : dz.ahead(row)), g, places, a.cols, d);
        } else {
#pragma unroll
            for (int k = 0; k < P; ++k) d[k] = 0ull;
        }
        if (a.norm) {
            f32x2 y[P], all[2] = {0ull, 0ull};
            read_row<T, VEC, U>(from + (VEC ? 0 : dn.ahead(row)), g, places, a.cols, y);
            read_source<T, VEC, U>(a.z, row, from + buffer + (VEC ? 0 : z.ahead(row)), g, places, a.cols, h);
            keep_valid_row<VEC, U>(valid, y);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                f32x2 gamma[4];
                held_columns<VEC, U>(held, g, places, a.cols, u, gamma);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int k = 4 * u + i;
                    h[k] = mul2(add2(h[k], pair_of(-mean_z)), pair_of(rstd_z));
                    sums[0][k] = fma2(y[k], h[k], sums[0][k]);
                    sums[1][k] = add2(sums[1][k], y[k]);
                    y[k] = mul2(y[k], gamma[i]);
                    all[0] = add2(all[0], y[k]);
                    all[1] = fma2(y[k], h[k], all[1]);
                }
            }
            float2 of = make_float2(sum_of(all[0]), sum_of(all[1]));
            group_sums<1>(g, &of);
            const f32x2 mean_u = pair_of(-of.x * g.of_row), mean_uh = pair_of(-of.y * g.of_row);
#pragma unroll
            for (int k = 0; k < P; ++k) d[k] = fma2(fma2(h[k], mean_uh, add2(y[k], mean_u)), pair_of(rstd_z), d[k]);
        }
        keep_valid_row<VEC, U>(valid, d);
        RowRaw<T, U> raw;
        if (a.dx) {
            f32x2 out[P];
#pragma unroll
            for (int k = 0; k < P; ++k) out[k] = mul2(d[k], pair_of(a.scale));
            narrow_row<T, U>(out, raw);
            store_row<T, VEC, U>(static_cast<T *>(a.dx) + row * a.dx_stride, g, valid, raw);
        }
        read_source<T, VEC, U>(a.f, row, from + 3 * buffer + (VEC ? 0 : f.ahead(row)), g, places, a.cols, h);
        // d is zero outside the row, but its product with an infinite f is not (through the norm all of that row is NaN)
        if (GATE == GATE_OF_ROW && !a.post_norm) keep_valid_row<VEC, U>(valid, h);
        f32x2 gate[P], of_gate = 0ull, all[2] = {0ull, 0ull};
        if (GATE == GATE_OF_VALUES) {
            load_row<T, VEC, U>(static_cast<const T *>(a.gate) + row * a.gate_stride, g, valid, raw);
            widen_row<T, U>(raw, gate);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            f32x2 factor[4], shift[4];
            held_columns<VEC, U>(held + a.cols, g, places, a.cols, u, factor);
            if (GATE != GATE_IN_COLUMNS) held_columns<VEC, U>(held + 2 * a.cols, g, places, a.cols, u, shift);
#pragma unroll
            for (int i = 0; i < 4; ++i) {  // d is zero outside the row
                const int k = 4 * u + i;
                h[k] = mul2(add2(h[k], pair_of(-mean_f)), pair_of(rstd_f));
                if (GATE != GATE_IN_COLUMNS) {
                    const f32x2 dp = mul2(d[k], fma2(h[k], factor[i], shift[i]));
                    d[k] = mul2(d[k], GATE == GATE_OF_ROW ? pair_of(of_row) : gate[k]);
                    if (GATE == GATE_OF_ROW)
                        of_gate = add2(of_gate, dp);
                    else
                        gate[k] = dp;
                }
                sums[2][k] = fma2(d[k], h[k], sums[2][k]);
                sums[3][k] = add2(sums[3][k], d[k]);
                d[k] = mul2(d[k], factor[i]);
                all[0] = add2(all[0], d[k]);
                all[1] = fma2(d[k], h[k], all[1]);
            }
        }
        if (GATE == GATE_OF_VALUES && a.dgate) {
            narrow_row<T, U>(gate, raw);
            store_row<T, VEC, U>(static_cast<T *>(a.dgate) + row * a.dgate_stride, g, valid, raw);
        }
        float2 of[2] = {make_float2(sum_of(all[0]), sum_of(all[1])), make_float2(sum_of(of_gate), 0.0f)};
        if (GATE == GATE_OF_ROW) {
            group_sums<2>(g, of);
            if (g.thread == 0 && a.dgate) static_cast<float *>(a.dgate)[row] = of[1].x;
        } else if (a.post_norm) {
            group_sums<1>(g, of);
        } else if (g.warps > 1) {
            g.sync();
        }
        // every warp of the group is past its reads of this stage
        __syncwarp();
        if (g.warp == 0 && ok && row + (long long)stages * row_step < a.rows) {
            if (elect_one()) request(row + stages * row_step, stage);
            __syncwarp();
        }
        if (++stage == stages) { stage = 0; phase ^= 1u; }
        if (a.df) {
            if (a.post_norm) {
                const f32x2 mean_q = pair_of(-of[0].x * g.of_row), mean_qh = pair_of(-of[0].y * g.of_row);
#pragma unroll
                for (int k = 0; k < P; ++k) d[k] = mul2(fma2(h[k], mean_qh, add2(d[k], mean_q)), pair_of(rstd_f));
            }
            narrow_row<T, U>(d, raw);
            store_row<T, VEC, U>(static_cast<T *>(a.df) + row * a.df_stride, g, valid, raw);
        }
    }
    if (!ok)  // a wait ran out: let the copies in flight land before the block ends
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    // the groups' sums, [group][4][cols] in the place of the rows, which everyone has read, then added in their order
    __syncthreads();
    float *const own = held + g.index * 4 * a.cols;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if constexpr (VEC) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (valid >> (8 * u) & 1u) {
                    float4 *const to = reinterpret_cast<float4 *>(own + q * a.cols) + 2 * places.unit(u);
                    const f32x2 *const w = &sums[q][4 * u];
                    const float2 w0 = values_of(w[0]), w1 = values_of(w[1]), w2 = values_of(w[2]), w3 = values_of(w[3]);
                    to[0] = make_float4(w0.x, w0.y, w1.x, w1.y);
                    to[1] = make_float4(w2.x, w2.y, w3.x, w3.y);
                }
        } else {
#pragma unroll
            for (int j = 0; j < 8 * U; ++j) {
                const float2 w = values_of(sums[q][j / 2]);
                if (valid >> j & 1u) own[q * a.cols + column<false>(g.threads, g.thread, j)] = j & 1 ? w.y : w.x;
            }
        }
    }
    __syncthreads();
    const int with_rows = min(groups, a.rows - (int)blockIdx.x * groups);
    float *const part = a.partial + blockIdx.x * 4ll * a.cols;
    if constexpr (VEC) {
        for (int c = threadIdx.x; c < a.cols; c += blockDim.x) {
            const float4 *at = reinterpret_cast<const float4 *>(held) + c;
            float4 sum = *at;
            for (int i = 1; i < with_rows; ++i) {
                at += a.cols;
                const float4 w = *at;
                sum = make_float4(sum.x + w.x, sum.y + w.y, sum.z + w.z, sum.w + w.w);
            }
            reinterpret_cast<float4 *>(part)[c] = sum;
        }
    } else {
        for (int c = threadIdx.x; c < 4 * a.cols; c += blockDim.x) {
            float sum = held[c];
            for (int i = 1; i < with_rows; ++i) sum += held[i * 4 * a.cols + c];
            part[c] = sum;
        }
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

constexpr int JOIN_SLICES = 32;

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

template <typename T, bool VEC, int GATE, int U> int launch_groups(const NormArgs &a, cudaStream_t stream)
{
    const auto kernel = group_rows_kernel<T, VEC, GATE, U>;
    const int warps = (int)ceil_div(a.cols, 256 * U), groups = 16 / warps;
    constexpr int held = HELD_VECTORS<GATE> * (int)sizeof(float);  // bytes of a column
    if (a.cols * held > 48 * 1024 &&
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_GROUP_COLS * held) != cudaSuccess)
        return launch_status();
    kernel<<<(unsigned)std::min<int64_t>(ceil_div(a.rows, groups), 148), groups * warps * 32, a.cols * held, stream>>>(a, warps);
    return launch_status();
}
template <typename T, bool VEC, int GATE> int launch_groups(const NormArgs &a, cudaStream_t stream)
{
    if (a.cols <= 256) return launch_groups<T, VEC, GATE, 1>(a, stream);
    if constexpr (sizeof(T) == 2 && VEC) {  // value by value four units spill registers (5662x3345 121 us)
        if (a.cols > 512) return launch_groups<T, VEC, GATE, 4>(a, stream);
    }
    return launch_groups<T, VEC, GATE, 2>(a, stream);
}

template <typename T> int launch_rows(const NormArgs &a, cudaStream_t stream)
{
    if (a.cols > MAX_GROUP_COLS) {
        rows_kernel<T><<<(unsigned)std::min<int64_t>(a.rows, 148 * 8), ROW_THREADS, 0, stream>>>(a);
        return launch_status();
    }
    const auto aligned = [&](const void *p, long long stride) { return !p || rows_aligned16(p, stride, a.rows, sizeof(T)); };
    const bool vec = a.cols % 8 == 0 && aligned(a.x.dense, a.x.stride) && aligned(a.f.dense, a.f.stride) && aligned(a.z_out, a.z_stride) &&
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
    bool grouped;  // group_back_kernel; else the kernels for any width
    int parts;
    int64_t partial_bytes, bytes;
};
BackPlan plan_back(int64_t rows, int64_t cols)
{
    BackPlan p;
    if (cols <= MAX_BACK_COLS) {  // as many groups as any type's, so that the workspace does not depend on it
        p.grouped = true;
        p.parts = (int)std::max<int64_t>(1, std::min<int64_t>(148, rows));
        p.partial_bytes = p.bytes = (int64_t)p.parts * 4 * cols * 4;
        return p;
    }
    const int64_t columns = ceil_div(cols, COLUMN_THREADS);
    p.grouped = false;
    p.parts = (int)std::max<int64_t>(1, std::min<int64_t>({MAX_PARTS, ceil_div(rows, 16), ceil_div(148 * 8, columns)}));
    p.partial_bytes = (int64_t)p.parts * 4 * cols * 4;
    p.bytes = ceil_div(p.partial_bytes, 16) * 16 + rows * 8;
    return p;
}

template <typename T, bool VEC, int GATE, int U, int THREADS> int launch_back_groups(NormArgs &a, cudaStream_t stream)
{
    const auto kernel = group_back_kernel<T, VEC, GATE, U, THREADS>;
    const int warps = (int)ceil_div(a.cols, 256 * U), groups = THREADS / 32 / warps;
    a.parts = (int)std::min<int64_t>(ceil_div(a.rows, groups), a.parts);
    // a row of any kind and alignment, and how many fit beside the parameters
    const int buffer = (a.cols * (int)sizeof(T) + 30) / 16 * 16, parameters = (a.cols * 12 + 15) / 16 * 16;
    const int stages = std::min(MAX_STAGES, (BACK_SMEM - parameters) / (groups * 4 * buffer));
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, BACK_SMEM) != cudaSuccess) return launch_status();
    const int smem = std::max(parameters + groups * stages * 4 * buffer, groups * 16 * a.cols);  // rows, and at the end sums
    kernel<<<a.parts, groups * warps * 32, smem, stream>>>(a, warps, stages, buffer);
    return launch_status();
}
// One unit for a thread leaves registers for 16 warps, two for 12, which have less to do for each value: they are faster
// (16384x2048 in bf16 101 us against 128, 8192x4096 128 against 134, 8192x2048 in fp32 87 against 95) but for a single
// unit, which 4096x64 takes 19.5 against 21.5, and where values come one by one (16384x2048 at odd addresses 234 against
// 146).  More than 4096 columns need two units all the same, and more than 6144 16 warps of them, whose registers do not
// hold everything (3500x5120 in fp32 159 against 103, 3001x5555 218 against 161).
template <typename T, bool VEC, int GATE> int launch_back_groups(NormArgs &a, cudaStream_t stream)
{
    if (a.cols > 6144) return launch_back_groups<T, VEC, GATE, 2, 512>(a, stream);
    if (a.cols > (VEC ? 256 : 4096)) return launch_back_groups<T, VEC, GATE, 2, 384>(a, stream);
    return launch_back_groups<T, VEC, GATE, 1, 512>(a, stream);
}
template <typename T, bool VEC> int launch_back_groups(NormArgs &a, cudaStream_t stream)
{
    if (a.gate_kind == DIPACO_GATE_ROWS) return launch_back_groups<T, VEC, GATE_OF_ROW>(a, stream);
    if (a.gate_kind == DIPACO_GATE_FULL) return launch_back_groups<T, VEC, GATE_OF_VALUES>(a, stream);
    return launch_back_groups<T, VEC, GATE_IN_COLUMNS>(a, stream);
}

// a.parts: how many parts there may be, and then are.
template <typename T> int launch_back(NormArgs &a, const BackPlan &plan, cudaStream_t stream)
{
    if (!plan.grouped) {
        back_rows_kernel<T><<<(unsigned)std::min<int64_t>(a.rows, 148 * 8), ROW_THREADS, 0, stream>>>(a);
        if (const int rc = launch_status()) return rc;
        const dim3 columns((unsigned)ceil_div(a.cols, COLUMN_THREADS), (unsigned)plan.parts);
        back_columns_kernel<T><<<columns, COLUMN_THREADS, 0, stream>>>(a);
        return launch_status();
    }
    const auto aligned = [&](const void *p, long long stride) { return !p || rows_aligned16(p, stride, a.rows, sizeof(T)); };
    const bool vec = a.cols % 8 == 0 && aligned(a.dn.dense, a.dn.stride) && aligned(a.dz.dense, a.dz.stride) && aligned(a.f.dense, a.f.stride) &&
                     aligned(a.z.dense, a.z.stride) && aligned(a.dx, a.dx_stride) && aligned(a.df, a.df_stride) &&
                     (a.gate_kind != DIPACO_GATE_FULL || (aligned(a.gate, a.gate_stride) && aligned(a.dgate, a.dgate_stride)));
    return vec ? launch_back_groups<T, true>(a, stream) : launch_back_groups<T, false>(a, stream);
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
    __all_sync(0xffffffffu, bounded_wait(&bar, 0, &g_residual_norm_error, 9, limit_ns));
}

} // namespace

bool dipaco::take_residual_norm_error(bool &expired) { return take_error_word(g_residual_norm_error, expired); }

int dipaco::expire_residual_norm_wait(unsigned long long limit_ns, cudaStream_t stream)
{
    wait_expiry_kernel<<<1, 32, 0, stream>>>(limit_ns);
    return launch_status();
}

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
    j.parts = a.parts;
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
