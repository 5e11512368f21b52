// Linear layers on packed matrices (see include/dipaco.h): the products of product_pairs.cuh with what surrounds them
// in a block done in their epilogue, on the sums as they leave tensor memory.
//
//   dense  y = act(x w^T + bias) + residual
//   pack   a = x w^T + bias and act(a), both packed.  A tile's 256 rows and 128 or 256 columns are whole blocks of
//          128 x 128, so that a block's largest magnitude is known on one SM: the sums are read from tensor memory
//          twice, once for it and once to encode.  Of act(a) it is the activation of the largest a where that is
//          large enough (grows_from); else every value is activated once more for it.
//   back   da = (dy w) act'(a) packed, and its sums over rows.  The products with the slope go back to tensor memory
//          until the block's largest is known.
//
// Few tokens through a weight: their sums go to fp32 and are packed by a second launch.
#include "activations.cuh"
#include "product_pairs.cuh"

#include <algorithm>

namespace dipaco {
namespace {

// ------------------------------------------------------------------------------------------ dense

// act(v + bias) + residual.
struct Linear {
    static constexpr bool NOTHING = false;
    const void *bias, *residual;
    long long residual_row;
    int activation;
    bool bias_bf16, bias_aligned, residual_bf16, residual_aligned;

    __device__ __forceinline__ f32x2 act(f32x2 v) const
    {
        switch (activation) {
        case DIPACO_ACTIVATION_RELU: return activate<DIPACO_ACTIVATION_RELU>(v);
        case DIPACO_ACTIVATION_SILU: return activate<DIPACO_ACTIVATION_SILU>(v);
        case DIPACO_ACTIVATION_GELU: return activate<DIPACO_ACTIVATION_GELU>(v);
        default: return v;
        }
    }
    __device__ __forceinline__ float value(float v, long long row, int col) const
    {
        if (bias) v += load_param(bias, bias_bf16, col);
        v = values_of(act(pair_of(v))).x;
        if (residual) v += load_param(residual, residual_bf16, row * residual_row + col);
        return v;
    }
    // 32 columns of a row
    __device__ __forceinline__ void columns(float *v, long long row, int col, int m, int n) const
    {
        f32x2 p[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = pair_of(v[2 * i], v[2 * i + 1]);
        if (bias) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x2 b[4];
                param_pairs<8>(bias, bias_bf16, bias_aligned, col + 8 * i, n, b);
#pragma unroll
                for (int j = 0; j < 4; ++j) p[4 * i + j] = add2(p[4 * i + j], b[j]);
            }
        }
        switch (activation) {
        case DIPACO_ACTIVATION_RELU: each<DIPACO_ACTIVATION_RELU>(p); break;
        case DIPACO_ACTIVATION_SILU: each<DIPACO_ACTIVATION_SILU>(p); break;
        case DIPACO_ACTIVATION_GELU: each<DIPACO_ACTIVATION_GELU>(p); break;
        }
        if (residual && row < m) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f32x2 r[4];
                const long long at = row * residual_row + col + 8 * i;
                const void *from = residual_bf16 ? static_cast<const void *>(static_cast<const __nv_bfloat16 *>(residual) + at)
                                                 : static_cast<const void *>(static_cast<const float *>(residual) + at);
                param_pairs<8>(from, residual_bf16, residual_aligned, 0, n - (col + 8 * i), r);
#pragma unroll
                for (int j = 0; j < 4; ++j) p[4 * i + j] = add2(p[4 * i + j], r[j]);
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float2 w = values_of(p[i]);
            v[2 * i] = w.x;
            v[2 * i + 1] = w.y;
        }
    }
    template <int ACTIVATION> static __device__ __forceinline__ void each(f32x2 *p)
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = activate<ACTIVATION>(p[i]);
    }
};

// Nothing is contracted: every sum is zero.
template <typename T> __global__ void __launch_bounds__(256) empty_sums_kernel(T *y, long long y_row, long long m, int n, Linear finish)
{
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < m * n; i += gridDim.x * 256ll) {
        const long long row = i / n;
        const int col = (int)(i - row * n);
        y[row * y_row + col] = narrow1<T>(finish.value(0.0f, row, col));
    }
}

// ------------------------------------------------------------------------------------------ packed results

struct PackedCodes {
    uint8_t *codes, *scales;
    long long stride;
    bool wide;  // rows on 32-byte boundaries
};

struct PackArgs : ProductArgs {
    PackedCodes first, second;  // act(a) and a; or da.  codes NULL: not wanted
    const void *bias;
    bool bias_bf16;
    // back
    const uint8_t *a_codes, *of_a_scales;
    long long a_stride;
    float *row_sums;  // [blocks of 128 rows][n]
};

// What the epilogue warps share.  The barrier's phases are the exchanges of maxima; a warp is at most one exchange
// ahead of another, so that two sets of maxima do.
struct PackShared {
    uint64_t exchanged;
    unsigned maxima[2][2][2][PAIR_EPILOGUE_WARPS];  // [exchange][block][of act(a), of a]
};

// 32 codes of a row, of which the first `left` are the matrix's.
__device__ __forceinline__ void store_codes(const PackedCodes &out, long long row, int col, int left, const unsigned *w)
{
    uint8_t *p = out.codes + row * out.stride + col;
    if (left >= 32 && out.wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                     "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
        return;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (left >= 16 * h + 16) {
            *reinterpret_cast<uint4 *>(p + 16 * h) = make_uint4(w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (16 * h + i < left) p[16 * h + i] = (uint8_t)(w[4 * h + i / 4] >> 8 * (i % 4));
        }
    }
}

// The codes of 32 values: CAREFUL where there may be infinities.
template <bool CAREFUL> __device__ __forceinline__ void encode32(const f32x2 *v, float reciprocal, unsigned *w)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (CAREFUL) {
            const float2 a = values_of(v[2 * i]), b = values_of(v[2 * i + 1]);
            const float f[4] = {a.x, a.y, b.x, b.y};
            w[i] = encode4(f, reciprocal);
        } else {
            w[i] = encode4_finite(v + 2 * i, pair_of(reciprocal));
        }
    }
}

__device__ __forceinline__ float larger3(float most, f32x2 p)  // NaN does not count
{
    const float2 v = values_of(p);
    asm("max.f32 %0, %0, %1, %2;" : "+f"(most) : "f"(v.x), "f"(v.y));
    return most;
}
__device__ __forceinline__ float larger_magnitude(float most, f32x2 p)
{
    const float2 v = values_of(p);
    asm("max.abs.f32 %0, %0, %1, %2;" : "+f"(most) : "f"(v.x), "f"(v.y));
    return most;
}
__device__ __forceinline__ unsigned finite_magnitudes(unsigned most, f32x2 p)
{
    const float2 v = values_of(p);
    return max(most, max(finite_magnitude(v.x), finite_magnitude(v.y)));
}

// An epilogue warp's part of the exchanges.
struct Exchange {
    PackShared &shared;
    int warp, lane;
    unsigned count = 0;

    // This warp's largest values of block `block` (bits; the lanes' largest is taken).
    __device__ __forceinline__ void put(int block, unsigned first, unsigned second)
    {
        first = __reduce_max_sync(0xffffffffu, first);
        second = __reduce_max_sync(0xffffffffu, second);
        if (lane == 0) {
            shared.maxima[count & 1][block][0][warp] = first;
            shared.maxima[count & 1][block][1][warp] = second;
        }
    }
    // All warps' largest, once every warp has put its own; false if the wait ran out.
    __device__ __forceinline__ bool meet(int blocks, unsigned (*most)[2])
    {
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&shared.exchanged);
        if (!warp_wait(&shared.exchanged, count & 1, 11)) return false;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int q = 0; q < 2; ++q)
                most[b][q] = b < blocks ? __reduce_max_sync(0xffffffffu, shared.maxima[count & 1][b][q][lane & 7]) : 0u;
        ++count;
        return true;
    }
};

// A warp's way through a tile: its quarter of the rows, every other group of 32 columns, from the columns that the
// sets of sums share.
struct TileWalk {
    int own, blocks;  // groups of this warp, blocks of 128 columns
    int odd;
    bool down;
    __device__ __forceinline__ int group(int t) const { return 2 * (down ? own - 1 - t : t) + odd; }
};

template <int ACTIVATION>
__device__ __forceinline__ void pack_epilogue(const PackArgs &p, const PairBlock &b, PackShared &shared,
                                              float (*bias)[PAIR_MAX_N / 64][32])
{
    constexpr bool GROWS = ACTIVATION == DIPACO_ACTIVATION_GELU || ACTIVATION == DIPACO_ACTIVATION_SILU;
    const int lane = b.lane, quarter = b.warp & 3;
    const uint32_t read_bars[2] = {cluster_addr(ptx::smem_addr(&b.sums_read[0]), 0),
                                   cluster_addr(ptx::smem_addr(&b.sums_read[1]), 0)};
    const int scale_cols = (p.n + 127) / 128;
    const bool keep = p.second.codes != nullptr;
    TileWalk walk = {p.tile_n / 64, p.tile_n / 128, b.warp >> 2, false};
    Exchange exchange = {shared, b.warp, lane};
    PairWalk items(p, b.pair);
    PairItem item;
    for (int sets = 0; items.take(p, b.pair, item); ++sets) {
        const int n0 = item.tile_n * p.tile_n, row0 = item.tile_m * PAIR_ROWS + (int)b.rank * 128;
        const int row = row0 + quarter * 32 + lane;
        float (*columns_bias)[32] = bias[b.warp];
        __syncwarp();
#pragma unroll
        for (int t = 0; t < PAIR_MAX_N / 64; ++t) {
            const int col = n0 + (2 * t + walk.odd) * 32 + lane;
            columns_bias[t][lane] = t < walk.own && p.bias && col < p.n ? load_param(p.bias, p.bias_bf16, col) : 0.0f;
        }
        __syncwarp();
        if (!warp_wait(&b.sums_full[sets & 1], (sets >> 1) & 1, 4)) return;
        fence_after_sync();
        const uint32_t from = b.tmem + ((uint32_t)(quarter * 32) << 16) + ((sets & 1) ? b.second_set : 0);
        walk.down = !(sets & 1);
        const uint32_t read_bar = read_bars[sets & 1];
        // a of a group
        const auto with_bias = [&](int group, const uint32_t *r, f32x2 *a) {
            const float4 *add = reinterpret_cast<const float4 *>(columns_bias[group >> 1]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float4 w = add[i];
                a[2 * i] = add2(pair_of(__uint_as_float(r[4 * i]), __uint_as_float(r[4 * i + 1])), pair_of(w.x, w.y));
                a[2 * i + 1] = add2(pair_of(__uint_as_float(r[4 * i + 2]), __uint_as_float(r[4 * i + 3])), pair_of(w.z, w.w));
            }
        };
        uint32_t held[32];  // the group whose columns the next tile's products overwrite
        f32x2 a[16];
        unsigned most[2][2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (half >= walk.blocks) break;
            float top = 0.0f, magnitude = 0.0f;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int group = walk.group(2 * half + i);
                uint32_t other[32];
                uint32_t *r = half + i == 0 ? held : other;
                tmem_load32(from + group * 32, r);
                tmem_wait(r);
                if (half + i == 0 && !b.apart) {
                    fence_before_sync();
                    if (lane == 0) arrive_remote(read_bar);
                    __syncwarp();
                }
                with_bias(group, r, a);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    if (ACTIVATION != DIPACO_ACTIVATION_NONE) top = larger3(top, a[j]);
                    magnitude = larger_magnitude(magnitude, a[j]);
                }
            }
            if (row >= p.m) top = magnitude = 0.0f;  // the bias is not the matrix's there
            exchange.put(walk.down ? walk.blocks - 1 - half : half, __float_as_uint(top), __float_as_uint(magnitude));
        }
        if (!exchange.meet(walk.blocks, most)) return;
        bool careful = false;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (k >= walk.blocks || n0 + k * 128 >= p.n || row0 >= p.m) continue;
            careful |= most[k][1] >= 0x7f800000u;
            if (GROWS) careful |= most[k][0] < __float_as_uint(grows_from<ACTIVATION>());
            if (ACTIVATION == DIPACO_ACTIVATION_NONE)
                most[k][0] = most[k][1];
            else
                most[k][0] = __float_as_uint(values_of(activate<ACTIVATION>(pair_of(__uint_as_float(most[k][0])))).x);
        }
        if (careful) {  // the same for all epilogue warps of the block
#pragma unroll 1
            for (int half = 0; half < walk.blocks; ++half) {
                unsigned of_y = 0u, of_a = 0u;
#pragma unroll 1
                for (int i = 0; i < 2; ++i) {
                    const int group = walk.group(2 * half + i);
                    if (half + i == 0) {
                        with_bias(group, held, a);
                    } else {
                        uint32_t r[32];
                        tmem_load32(from + group * 32, r);
                        tmem_wait(r);
                        with_bias(group, r, a);
                    }
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        of_y = finite_magnitudes(of_y, activate<ACTIVATION>(a[j]));
                        of_a = finite_magnitudes(of_a, a[j]);
                    }
                }
                if (row >= p.m) of_y = of_a = 0u;
                exchange.put(walk.down ? walk.blocks - 1 - half : half, of_y, of_a);
            }
            if (!exchange.meet(walk.blocks, most)) return;
        }
        unsigned bytes[2][2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            bytes[k][0] = scale_byte(most[k][0]);
            bytes[k][1] = scale_byte(most[k][1]);
        }
        if (b.warp == 0 && lane < walk.blocks && n0 + lane * 128 < p.n && row0 < p.m) {
            const long long at = (long long)(row0 / 128) * scale_cols + n0 / 128 + lane;
            p.first.scales[at] = (uint8_t)(lane ? bytes[1][0] : bytes[0][0]);
            if (keep) p.second.scales[at] = (uint8_t)(lane ? bytes[1][1] : bytes[0][1]);
        }
        const auto store = [&](int group) {
            const int left = p.n - (n0 + group * 32);
            const bool inside = row < p.m && left > 0;
            const float by_y = scale_reciprocal(group >> 2 ? bytes[1][0] : bytes[0][0]);
            unsigned w[8];
            if (keep) {
                const float by_a = scale_reciprocal(group >> 2 ? bytes[1][1] : bytes[0][1]);
                if (careful)
                    encode32<true>(a, by_a, w);
                else
                    encode32<false>(a, by_a, w);
                if (inside) store_codes(p.second, row, n0 + group * 32, left, w);
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) a[j] = activate<ACTIVATION>(a[j]);
            if (careful)
                encode32<true>(a, by_y, w);
            else
                encode32<false>(a, by_y, w);
            if (inside) store_codes(p.first, row, n0 + group * 32, left, w);
        };
        with_bias(walk.group(0), held, a);
        store(walk.group(0));
#pragma unroll 1
        for (int t = 1; t < walk.own; ++t) {
            uint32_t r[32];
            tmem_load32(from + walk.group(t) * 32, r);
            tmem_wait(r);
            if (b.apart && t + 1 == walk.own) {
                fence_before_sync();
                if (lane == 0) arrive_remote(read_bar);
                __syncwarp();
            }
            with_bias(walk.group(t), r, a);
            store(walk.group(t));
        }
    }
}

// Sums over the warp's 32 rows of 32 columns, a column for a lane: at each step a lane hands on the half of its
// values that the lane across keeps.
__device__ __forceinline__ float column_sums(float *v, int lane)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const bool upper = lane & o;
#pragma unroll
        for (int i = 0; i < o; ++i) {
            const float give = upper ? v[i] : v[i + o];
            v[i] = (upper ? v[i + o] : v[i]) + __shfl_xor_sync(0xffffffffu, give, o);
        }
    }
    return v[0];
}

__device__ __forceinline__ void tmem_store32(uint32_t address, const f32x2 *v)
{
    uint32_t r[32];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float2 w = values_of(v[i]);
        r[2 * i] = __float_as_uint(w.x);
        r[2 * i + 1] = __float_as_uint(w.y);
    }
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(address), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
        "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

template <int ACTIVATION>
__device__ __forceinline__ void back_epilogue(const PackArgs &p, const PairBlock &b, PackShared &shared,
                                              float (*sums)[PAIR_MAX_N / 32][4][32])
{
    const int lane = b.lane, quarter = b.warp & 3;
    const uint32_t read_bars[2] = {cluster_addr(ptx::smem_addr(&b.sums_read[0]), 0),
                                   cluster_addr(ptx::smem_addr(&b.sums_read[1]), 0)};
    const int scale_cols = (p.n + 127) / 128;
    TileWalk walk = {p.tile_n / 64, p.tile_n / 128, b.warp >> 2, false};
    Exchange exchange = {shared, b.warp, lane};
    PairWalk items(p, b.pair);
    PairItem item;
    for (int sets = 0; items.take(p, b.pair, item); ++sets) {
        const int n0 = item.tile_n * p.tile_n, row0 = item.tile_m * PAIR_ROWS + (int)b.rank * 128;
        const int row = row0 + quarter * 32 + lane;
        walk.down = !(sets & 1);
        // codes of a, two units of 16 for a group (rows of codes are padded to whole units), and their scales
        const auto load_codes = [&](int group, uint4 *codes) {
            if constexpr (ACTIVATION == DIPACO_ACTIVATION_NONE) return;
            const uint8_t *at = p.a_codes + row * p.a_stride + n0 + group * 32;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                codes[h] = row < p.m && n0 + group * 32 + 16 * h < p.n ? __ldcs(reinterpret_cast<const uint4 *>(at + 16 * h))
                                                                       : make_uint4(0u, 0u, 0u, 0u);
        };
        uint4 codes[2] = {};
        load_codes(walk.group(0), codes);
        float scales[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int block = n0 / 128 + k;
            scales[k] = ACTIVATION != DIPACO_ACTIVATION_NONE && k < walk.blocks && block < scale_cols && row0 < p.m
                            ? scale_value(p.of_a_scales[(long long)(row0 / 128) * scale_cols + block])
                            : 0.0f;
        }
        if (!warp_wait(&b.sums_full[sets & 1], (sets >> 1) & 1, 4)) return;
        fence_after_sync();
        const uint32_t from = b.tmem + ((uint32_t)(quarter * 32) << 16) + ((sets & 1) ? b.second_set : 0);
        const uint32_t read_bar = read_bars[sets & 1];
        f32x2 held[16];
        unsigned most[2][2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (half >= walk.blocks) break;
            float magnitude = 0.0f;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int t = 2 * half + i, group = walk.group(t);
                uint32_t r[32];
                tmem_load32(from + group * 32, r);
                tmem_wait(r);
                if (t == 0 && !b.apart) {
                    fence_before_sync();
                    if (lane == 0) arrive_remote(read_bar);
                    __syncwarp();
                }
                const unsigned words[8] = {codes[0].x, codes[0].y, codes[0].z, codes[0].w,
                                           codes[1].x, codes[1].y, codes[1].z, codes[1].w};
                if (t + 1 < walk.own) load_codes(walk.group(t + 1), codes);
                const f32x2 scale = pair_of(group >> 2 ? scales[1] : scales[0]);
                f32x2 other[16];
                f32x2 *v = t == 0 ? held : other;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    v[j] = pair_of(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
                    if constexpr (ACTIVATION != DIPACO_ACTIVATION_NONE)
                        v[j] = mul2(v[j], slope<ACTIVATION>(mul2(decode_pair(words[j / 2] >> 16 * (j & 1)), scale)));
                    if (row >= p.m) v[j] = 0ull;
                    magnitude = larger_magnitude(magnitude, v[j]);
                }
                if (t > 0) tmem_store32(from + group * 32, v);
                if (p.row_sums) {
                    float f[32];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float2 w = values_of(v[j]);
                        f[2 * j] = w.x;
                        f[2 * j + 1] = w.y;
                    }
                    sums[sets & 1][group][quarter][lane] = column_sums(f, lane);
                }
            }
            exchange.put(walk.down ? walk.blocks - 1 - half : half, __float_as_uint(magnitude), 0u);
        }
        tmem_stored();
        if (!exchange.meet(walk.blocks, most)) return;
        if (p.row_sums && b.warp < p.tile_n / 32 && row0 < p.m && n0 + b.warp * 32 + lane < p.n) {
            const float(*s)[32] = sums[sets & 1][b.warp];
            p.row_sums[(long long)(row0 / 128) * p.n + n0 + b.warp * 32 + lane] = (s[0][lane] + s[1][lane]) + (s[2][lane] + s[3][lane]);
        }
        const bool careful = most[0][0] >= 0x7f800000u || most[1][0] >= 0x7f800000u;
        if (careful) {  // the same for all epilogue warps of the block
#pragma unroll 1
            for (int half = 0; half < walk.blocks; ++half) {
                unsigned finite = 0u;
#pragma unroll 1
                for (int i = 0; i < 2; ++i) {
                    const int group = walk.group(2 * half + i);
                    if (half + i == 0) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) finite = finite_magnitudes(finite, held[j]);
                    } else {
                        uint32_t r[32];
                        tmem_load32(from + group * 32, r);
                        tmem_wait(r);
#pragma unroll
                        for (int j = 0; j < 32; ++j) finite = max(finite, finite_magnitude(__uint_as_float(r[j])));
                    }
                }
                exchange.put(walk.down ? walk.blocks - 1 - half : half, finite, 0u);
            }
            if (!exchange.meet(walk.blocks, most)) return;
        }
        const unsigned bytes[2] = {scale_byte(most[0][0]), scale_byte(most[1][0])};
        if (b.warp == 0 && lane < walk.blocks && n0 + lane * 128 < p.n && row0 < p.m)
            p.first.scales[(long long)(row0 / 128) * scale_cols + n0 / 128 + lane] = (uint8_t)(lane ? bytes[1] : bytes[0]);
        const auto store = [&](int group, const f32x2 *v) {
            const int left = p.n - (n0 + group * 32);
            const float by = scale_reciprocal(group >> 2 ? bytes[1] : bytes[0]);
            unsigned w[8];
            if (careful)
                encode32<true>(v, by, w);
            else
                encode32<false>(v, by, w);
            if (row < p.m && left > 0) store_codes(p.first, row, n0 + group * 32, left, w);
        };
        store(walk.group(0), held);
#pragma unroll 1
        for (int t = 1; t < walk.own; ++t) {
            uint32_t r[32];
            tmem_load32(from + walk.group(t) * 32, r);
            tmem_wait(r);
            if (b.apart && t + 1 == walk.own) {
                fence_before_sync();
                if (lane == 0) arrive_remote(read_bar);
                __syncwarp();
            }
            f32x2 v[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = pair_of(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
            store(walk.group(t), v);
        }
    }
}

template <int ACTIVATION, bool BACK>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(PAIR_THREADS, 1)
    packed_pair_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
                       const __grid_constant__ PackArgs p)
{
    __shared__ PackShared shared;
    // biases of the warps' columns; or sums over rows of the tile's columns, for two tiles
    __shared__ __align__(16) float columns[BACK ? 2 * PAIR_MAX_N * 4 : PAIR_EPILOGUE_WARPS * PAIR_MAX_N / 2];
    if (threadIdx.x == 64) ptx::mbar_init(&shared.exchanged, PAIR_EPILOGUE_WARPS);  // seen after run_pair's first barrier
    run_pair<false>(a_map, b_map, p, [&](const PairBlock &b) {
        if constexpr (BACK)
            back_epilogue<ACTIVATION>(p, b, shared, reinterpret_cast<float(*)[PAIR_MAX_N / 32][4][32]>(columns));
        else
            pack_epilogue<ACTIVATION>(p, b, shared, reinterpret_cast<float(*)[PAIR_MAX_N / 64][32]>(columns));
    });
}

constexpr int SLICES = 8;

// The sums over all rows from those over blocks of 128, in a fixed order.
__global__ void __launch_bounds__(32 * SLICES) row_sums_kernel(const float *partial, int parts, int n, float *out)
{
    __shared__ float shared[SLICES][32];
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (col < n) {
#pragma unroll 8
        for (int i = slice; i < parts; i += SLICES) s += partial[(long long)i * n + col];
    }
    shared[slice][lane] = s;
    __syncthreads();
    if (slice != 0 || col >= n) return;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < SLICES; ++i) s += shared[i][lane];
    out[col] = s;
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
    warp_wait(&bar, 0, 9, limit_ns);
}

// ------------------------------------------------------------------------------------------ host

PackedCodes packed_codes(const dipaco_packed *p)
{
    if (!p) return {};
    return {static_cast<uint8_t *>(p->codes), static_cast<uint8_t *>(p->scales), p->stride,
            (uintptr_t)p->codes % 32 == 0 && (p->stride % 32 == 0 || p->rows == 1)};
}

// Tiles of whole blocks: 256 columns, or 128 where that takes less time by the estimate of plan_pairs.
void plan_blocks(PackArgs &p)
{
    double best = 0.0;
    for (const int tile_n : {256, 128}) {
        const int64_t tiles = ceil_div(p.m, PAIR_ROWS) * ceil_div(p.n, tile_n);
        const double time = (double)ceil_div(tiles, PAIRS) * (p.steps * std::max(2.0 * tile_n, 64.0 * 4 + tile_n) + 12.0 * tile_n);
        if (best != 0.0 && time >= best) continue;
        best = time;
        p.tile_n = tile_n;
        p.tiles_m = (int)ceil_div(p.m, PAIR_ROWS);
        p.tiles_n = (int)ceil_div(p.n, tile_n);
        p.pairs = (int)std::min<int64_t>(PAIRS, tiles);
        p.whole_tiles = (int)tiles;
    }
    p.chunk = CHUNK_BF16;
}

template <bool BACK> int launch_packed(const CUtensorMap &a_map, const CUtensorMap &b_map, const PackArgs &p, int activation, cudaStream_t stream)
{
    const auto kernel = activation == DIPACO_ACTIVATION_RELU   ? packed_pair_kernel<DIPACO_ACTIVATION_RELU, BACK>
                        : activation == DIPACO_ACTIVATION_SILU ? packed_pair_kernel<DIPACO_ACTIVATION_SILU, BACK>
                        : activation == DIPACO_ACTIVATION_GELU ? packed_pair_kernel<DIPACO_ACTIVATION_GELU, BACK>
                                                               : packed_pair_kernel<DIPACO_ACTIVATION_NONE, BACK>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PAIR_SMEM) != cudaSuccess) return launch_status();
    kernel<<<2 * p.pairs, PAIR_THREADS, PAIR_SMEM, stream>>>(a_map, b_map, p);
    return launch_status();
}

bool is_activation(int activation) { return activation >= DIPACO_ACTIVATION_NONE && activation <= DIPACO_ACTIVATION_GELU; }

// A product whose sums are taken in one go.
int check_contraction(int64_t m, int64_t n, int64_t k)
{
    if (k < 0) return DIPACO_EINVAL;
    if (const int rc = check_extents(m, n)) return rc;
    return k > (int64_t)CHUNK_BF16 * STEP || ceil_div(m, PAIR_ROWS) * ceil_div(n, 128) > INT32_MAX ? DIPACO_ELIMIT : DIPACO_OK;
}

// Few tokens, and sums over nothing, are packed from fp32.
bool by_way_of_fp32(int64_t m, int64_t n, int64_t k) { return k == 0 || (m <= n && are_few(m, n, k, false, true)); }

bool workspace_ok(const void *workspace, int64_t bytes, int64_t need)
{
    return need == 0 || (workspace && (uintptr_t)workspace % 16 == 0 && bytes >= need);
}

} // namespace
} // namespace dipaco

using namespace dipaco;

bool dipaco::take_linear_error(bool &expired) { return take_error_word(g_product_error, expired); }

int dipaco::expire_linear_wait(unsigned long long limit_ns, cudaStream_t stream)
{
    wait_expiry_kernel<<<1, 32, 0, stream>>>(limit_ns);
    return launch_status();
}

extern "C" {

int dipaco_packed_linear(const dipaco_packed *x, const dipaco_packed *w, const void *bias, int32_t bias_dtype,
                         int32_t activation, const void *residual, int64_t residual_stride, void *y, int64_t y_stride,
                         int32_t dtype, void *workspace, int64_t workspace_bytes, int32_t device, void *cuda_stream)
{
    if (!x || !w || !is_dense_dtype(dtype) || !is_dense_dtype(bias_dtype) || !is_activation(activation) || device < 0 || x->cols != w->cols)
        return DIPACO_EINVAL;
    const int64_t m = x->rows, n = w->rows, k = x->cols;
    int64_t need = 0;
    if (const int rc = dipaco_packed_matmul_workspace(m, n, k, &need)) return rc;
    if (!packed_ok(x, m, k) || !packed_ok(w, n, k) || !dense_ok(y, y_stride, m, n, dtype)) return DIPACO_EINVAL;
    if (!vector_ok(bias, dense_size(bias_dtype)) || (residual && !dense_ok(residual, residual_stride, m, n, dtype))) return DIPACO_EINVAL;
    const bool few = are_few(m, n, k, false, true);
    if (!few && !workspace_ok(workspace, workspace_bytes, need)) return DIPACO_EINVAL;
    if (m == 0 || n == 0) return DIPACO_OK;

    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const Linear finish = {bias, residual, residual_stride, activation, bias_dtype == DIPACO_BF16, (uintptr_t)bias % 16 == 0,
                           dtype == DIPACO_BF16, rows_aligned16(residual, residual_stride, m, dense_size(dtype))};
    if (k == 0) {
        const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(m, 256) * n, 148 * 8);
        if (dtype == DIPACO_BF16)
            empty_sums_kernel<<<grid, 256, 0, stream>>>(static_cast<__nv_bfloat16 *>(y), y_stride, m, (int)n, finish);
        else
            empty_sums_kernel<<<grid, 256, 0, stream>>>(static_cast<float *>(y), y_stride, m, (int)n, finish);
        return launch_status();
    }
    if (few) return launch_few(x, w, y, y_stride, dtype, false, finish, stream);
    return launch_product(x, w, false, true, y, y_stride, dtype, false, finish, workspace, stream);
}

int dipaco_packed_linear_pack_workspace(int64_t m, int64_t n, int64_t k, int64_t *bytes)
{
    if (!bytes) return DIPACO_EINVAL;
    if (const int rc = check_contraction(m, n, k)) return rc;
    *bytes = by_way_of_fp32(m, n, k) ? m * ceil_div(n, 4) * 16 : 0;
    return DIPACO_OK;
}

int dipaco_packed_linear_pack(const dipaco_packed *x, const dipaco_packed *w, const void *bias, int32_t bias_dtype,
                              int32_t activation, const dipaco_packed *y, const dipaco_packed *a, void *workspace,
                              int64_t workspace_bytes, int32_t device, void *cuda_stream)
{
    if (!x || !w || !y || !is_dense_dtype(bias_dtype) || !is_activation(activation) || device < 0 || x->cols != w->cols) return DIPACO_EINVAL;
    const int64_t m = x->rows, n = w->rows, k = x->cols;
    int64_t need = 0;
    if (const int rc = dipaco_packed_linear_pack_workspace(m, n, k, &need)) return rc;
    if (!packed_ok(x, m, k) || !packed_ok(w, n, k) || !packed_ok(y, m, n) || (a && !packed_ok(a, m, n))) return DIPACO_EINVAL;
    if (!vector_ok(bias, dense_size(bias_dtype)) || !workspace_ok(workspace, workspace_bytes, need)) return DIPACO_EINVAL;
    if (m == 0 || n == 0) return DIPACO_OK;

    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (need > 0) {
        const Linear finish = {bias, nullptr, 0, DIPACO_ACTIVATION_NONE, bias_dtype == DIPACO_BF16, (uintptr_t)bias % 16 == 0, false, false};
        float *sums = static_cast<float *>(workspace);
        const int64_t stride = ceil_div(n, 4) * 4;
        if (k == 0) {
            empty_sums_kernel<<<(unsigned)std::min<int64_t>(ceil_div(m, 256) * n, 148 * 8), 256, 0, stream>>>(sums, stride, m, (int)n, finish);
            if (const int rc = launch_status()) return rc;
        } else if (const int rc = launch_few(x, w, sums, stride, DIPACO_F32, false, finish, stream)) {
            return rc;
        }
        return pack_activated(sums, stride, activation, y, a, stream);
    }
    PackArgs p = {};
    set_operands(p, x, w, false, true);
    plan_blocks(p);
    p.first = packed_codes(y);
    p.second = packed_codes(a);
    p.bias = bias;
    p.bias_bf16 = bias_dtype == DIPACO_BF16;
    CUtensorMap a_map, b_map;
    if (!operand_map(&a_map, x, 128) || !operand_map(&b_map, w, p.tile_n / 2)) return DIPACO_ECUDA;
    return launch_packed<false>(a_map, b_map, p, activation, stream);
}

int dipaco_packed_linear_pack_backward_workspace(int64_t m, int64_t n, int64_t k, int64_t *bytes)
{
    if (!bytes) return DIPACO_EINVAL;
    if (const int rc = check_contraction(m, n, k)) return rc;
    *bytes = ceil_div(ceil_div(m, PACK_BLOCK) * n, 4) * 16;
    return DIPACO_OK;
}

int dipaco_packed_linear_pack_backward(const dipaco_packed *dy, const dipaco_packed *w, const dipaco_packed *a, int32_t activation,
                                       const dipaco_packed *da, float *dbias, void *workspace, int64_t workspace_bytes,
                                       int32_t device, void *cuda_stream)
{
    if (!dy || !w || !da || !is_activation(activation) || device < 0 || dy->cols != w->rows) return DIPACO_EINVAL;
    const int64_t m = dy->rows, n = w->cols, k = dy->cols;
    int64_t need = 0;
    if (const int rc = dipaco_packed_linear_pack_backward_workspace(m, n, k, &need)) return rc;
    if (!packed_ok(dy, m, k) || !packed_ok(w, k, n) || !packed_ok(da, m, n)) return DIPACO_EINVAL;
    const bool slopes = activation != DIPACO_ACTIVATION_NONE;
    if (slopes && !packed_ok(a, m, n)) return DIPACO_EINVAL;
    if (!vector_ok(dbias, 4) || (dbias && !workspace_ok(workspace, workspace_bytes, need))) return DIPACO_EINVAL;
    if (n == 0) return DIPACO_OK;

    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (m == 0 || k == 0) {  // sums over nothing
        if (dbias && cudaMemsetAsync(dbias, 0, n * sizeof(float), stream) != cudaSuccess) return launch_status();
        if (m == 0) return DIPACO_OK;
        const int64_t scales = ceil_div(m, PACK_BLOCK) * ceil_div(n, PACK_BLOCK);
        if (cudaMemset2DAsync(da->codes, m == 1 ? n : da->stride, 0, n, m, stream) != cudaSuccess ||
            cudaMemsetAsync(da->scales, 127, scales, stream) != cudaSuccess)
            return launch_status();
        return DIPACO_OK;
    }
    PackArgs p = {};
    set_operands(p, dy, w, false, false);
    plan_blocks(p);
    p.first = packed_codes(da);
    p.a_codes = slopes ? static_cast<const uint8_t *>(a->codes) : nullptr;
    p.of_a_scales = slopes ? static_cast<const uint8_t *>(a->scales) : nullptr;
    p.a_stride = slopes ? a->stride : 0;
    p.row_sums = dbias ? static_cast<float *>(workspace) : nullptr;
    CUtensorMap a_map, b_map;
    if (!operand_map(&a_map, dy, 128) || !operand_map(&b_map, w, 128)) return DIPACO_ECUDA;
    if (const int rc = launch_packed<true>(a_map, b_map, p, activation, stream)) return rc;
    if (dbias)
        row_sums_kernel<<<(unsigned)ceil_div(n, 32), 32 * SLICES, 0, stream>>>(p.row_sums, (int)ceil_div(m, PACK_BLOCK), p.n, dbias);
    return launch_status();
}

} // extern "C"
