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
// Few tokens through a weight, packed: few_pack_kernel, in one launch.
//
// Measured (one B200, short runs; the bare product of the same operands to bf16 takes 100 us for the first two and 176 for
// the third): 32768x3584x896 packed with GELU and checkpoint 174 us, 164 without the checkpoint, 117 without either;
// with an argument over 7.2 in every block 191, where every block has a NaN or no argument of 0.3 291;
// the gradient of the same extents through the GELU 195, 174 without the sums over rows, 115 without the slopes;
// 16384x2048x8192 with bias and residual 188; one token through 3584x896, packed, 5.8 on the device.  Results in fp32
// over more than 2048 values spill the running totals: 4096x1024x4096 43 us, 51 with a residual, where bf16 takes 27 and 29.
// What bounds the packed forms is the epilogue: 11,300 clocks for a tile whose products take 3,600, of which activations
// are 3,150 (two powers and one reciprocal for two values at 8 clocks each, all their unit gives).  Its warps wait for
// their own chains: with 12 or 16 of them registers spill, and with twice the instructions in a loop they no longer stay
// in the instruction caches (the dense epilogue with its groups unrolled: 210 us instead of 135).
#include "activations.cuh"
#include "product_pairs.cuh"

#include <algorithm>
#include <type_traits>

namespace dipaco {
namespace {

// ------------------------------------------------------------------------------------------ dense

// act(v + bias) + residual.
struct Linear {
    static constexpr bool NOTHING = false;
    const void *bias, *residual;
    long long residual_row;
    int activation;
    bool bias_bf16, residual_bf16, residual_aligned;

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
    // of 32 columns
    __device__ __forceinline__ void act32(f32x2 *v) const
    {
        switch (activation) {
        case DIPACO_ACTIVATION_RELU: each<DIPACO_ACTIVATION_RELU>(v); break;
        case DIPACO_ACTIVATION_SILU: each<DIPACO_ACTIVATION_SILU>(v); break;
        case DIPACO_ACTIVATION_GELU: each<DIPACO_ACTIVATION_GELU>(v); break;
        }
    }
    template <int ACTIVATION> static __device__ __forceinline__ void each(f32x2 *p)
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = activate<ACTIVATION>(p[i]);
    }
};

// With 168 registers a thread.  12 and 16 warps spill: 32768x3584x896 packed 181 and 328 us instead of 174.
constexpr int EPILOGUE_WARPS = 8;
constexpr int SUBS = EPILOGUE_WARPS / 4;                  // warps that share a quarter of the rows
constexpr int GROUPS = (PAIR_MAX_N / 32 + SUBS - 1) / SUBS;  // of 32 columns, of one warp, at most
constexpr int BUFFERS = 3;                                // of a warp, for results on their way out
static_assert(EPILOGUE_WARPS * BUFFERS <= PAIR_EPILOGUE_WARPS * PAIR_STAGING, "staging");

// A warp's way through a tile: its quarter of the rows, every SUBS-th group of 32 columns, first those columns that the
// sets of sums share.
struct TileWalk {
    int sub, own;  // the first group, how many
    bool down;
    __device__ __forceinline__ int slot(int t) const { return down ? own - 1 - t : t; }  // which of its groups is t-th
    __device__ __forceinline__ int column(int slot) const { return (SUBS * slot + sub) * 32; }
    __device__ __forceinline__ int group(int t) const { return SUBS * slot(t) + sub; }
    __device__ __forceinline__ int block(int t) const { return group(t) >> 2; }  // of 128 columns
    __device__ __forceinline__ bool ends_block(int t) const { return t + 1 == own || block(t + 1) != block(t); }
};
__device__ __forceinline__ TileWalk make_walk(int warp, int tile_n)
{
    const int sub = warp >> 2;
    return {sub, (tile_n / 32 - sub + SUBS - 1) / SUBS, false};
}

// Parameters of the warp's columns from n0 on, for all lanes to read: the next tile's are on their way while one is
// worked on.
__device__ __forceinline__ void load_next_columns(const void *p, bool bf16, const TileWalk &walk, int n0, int n, int lane, float *next)
{
#pragma unroll
    for (int s = 0; s < GROUPS; ++s) {
        const int col = n0 + walk.column(s) + lane;
        next[s] = s < walk.own && p && col < n ? load_param(p, bf16, col) : 0.0f;
    }
}
__device__ __forceinline__ void put_next_columns(const float *next, int lane, float (*to)[32])
{
    __syncwarp();
#pragma unroll
    for (int s = 0; s < GROUPS; ++s) to[s][lane] = next[s];
    __syncwarp();
}
__device__ __forceinline__ void add_columns(const float *columns, const uint32_t *r, f32x2 *v)
{
    const float4 *add = reinterpret_cast<const float4 *>(columns);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float4 w = add[i];
        v[2 * i] = add2(pair_of(__uint_as_float(r[4 * i]), __uint_as_float(r[4 * i + 1])), pair_of(w.x, w.y));
        v[2 * i + 1] = add2(pair_of(__uint_as_float(r[4 * i + 2]), __uint_as_float(r[4 * i + 3])), pair_of(w.z, w.w));
    }
}

// The residual of 32 rows and 64 bytes of columns, as a warp loads it whole: lane l has unit l % 4 of rows l / 4 + 8 i.
__device__ __forceinline__ void load_residual(const DenseArgs<Linear> &p, int row0, int col, int lane, uint4 *units)
{
    const int size = p.c_bf16 ? 2 : 4, at = col + (lane & 3) * (16 / size);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = row0 + (lane >> 2) + 8 * i;
        units[i] = make_uint4(0u, 0u, 0u, 0u);
        if (row < p.m && at < p.n)
            units[i] = __ldcs(reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(p.finish.residual) +
                                                              (row * p.finish.residual_row + at) * size));
    }
}

// 32 columns of the warp's rows to C, by the copy engine (TMA) or at any alignment.  units: the residual of the first 64
// bytes, where it is read that way.
template <bool TMA>
__device__ __forceinline__ void finish_linear(const DenseArgs<Linear> &p, const CUtensorMap &c_map, const PairItem &item,
                                              int row0, int quarter, unsigned rank, int lane, int group, const uint32_t *sums,
                                              const float *bias, uint4 *units, bool by_units, uint8_t *buffers, int &buffer)
{
    if (item.slot >= 0) {
        float *out = p.partial + partial_offset(p, item.slot, rank) + (long long)group * 32 * 128 + quarter * 32 + lane;
#pragma unroll
        for (int i = 0; i < 32; ++i) out[i * 128] = __uint_as_float(sums[i]);
        return;
    }
    const int col0 = item.tile_n * p.tile_n + group * 32;
    f32x2 v[16];
    add_columns(bias, sums, v);
    uint4 second[4];  // the residual of the other 64 bytes, in fp32
    if (by_units && !p.c_bf16) load_residual(p, row0, col0 + 16, lane, second);
    p.finish.act32(v);
    if constexpr (TMA) {
        if (p.finish.residual && !by_units && row0 + lane < p.m) {  // a residual at another alignment
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const long long at = (row0 + lane) * p.finish.residual_row + col0 + 2 * i;
                v[i] = add2(v[i], pair_of(col0 + 2 * i < p.n ? load_param(p.finish.residual, p.finish.residual_bf16, at) : 0.0f,
                                          col0 + 2 * i + 1 < p.n ? load_param(p.finish.residual, p.finish.residual_bf16, at + 1) : 0.0f));
            }
        }
        // rows of 64 bytes in the copy engine's swizzle of that width
        const int parts = p.c_bf16 ? 1 : 2, size = p.c_bf16 ? 2 : 4;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            if (part >= parts) break;
            const int col = col0 + part * 16;
            asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(BUFFERS - 1) : "memory");  // the buffer's last
            __syncwarp();
            uint8_t *staging = buffers + buffer * PAIR_STAGING_BYTES;
            if (++buffer == BUFFERS) buffer = 0;
            const auto place = [&](int row, int unit) {
                return reinterpret_cast<uint4 *>(staging + row * 64 + ((unit ^ ((row >> 1) & 3)) * 16));
            };
            if (by_units) {
#pragma unroll
                for (int i = 0; i < 4; ++i) *place((lane >> 2) + 8 * i, lane & 3) = part ? second[i] : units[i];
                __syncwarp();
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint4 *at = place(lane, i);
                if (p.c_bf16) {
                    f32x2 r[4];
                    if (by_units) {
                        widen_pairs<__nv_bfloat16>(*at, r);
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[4 * i + j] = add2(v[4 * i + j], r[j]);
                    }
                    *at = narrow_pairs<__nv_bfloat16>(v + 4 * i);
                } else {
                    f32x2 *w = v + 8 * part + 2 * i, r[2];
                    if (by_units) {
                        widen_pairs<float>(*at, r);
                        w[0] = add2(w[0], r[0]);
                        w[1] = add2(w[1], r[1]);
                    }
                    *at = narrow_pairs<float>(w);
                }
            }
            ptx::fence_proxy_async();
            __syncwarp();
            // rows outside C and columns from whole_n on are not written
            if (elect_one()) {
                if (row0 < p.m && col < p.whole_n) tma_store_2d(&c_map, ptx::smem_addr(staging), col, row0);
                ptx::bulk_commit();
            }
            __syncwarp();
            const int ahead = (p.whole_n - col) * size;
            if (p.whole_n < p.n && ahead >= 0 && ahead < 64 && row0 + lane < p.m)  // the unit that C's rows end in
                store_head(static_cast<uint8_t *>(p.c) + ((row0 + lane) * p.c_row + p.whole_n) * size, *place(lane, ahead >> 4),
                           (p.n - p.whole_n) * size);
        }
        return;
    }
    // any alignment: rows through shared memory, a lane per column
    float *at = reinterpret_cast<float *>(buffers);
    for (int part = 0; part < 2; ++part) {  // 16 rows at a time
        __syncwarp();
        if (lane >> 4 == part) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float2 w = values_of(v[i]);
                at[(lane & 15) * 32 + ((2 * i + lane) & 31)] = w.x;
                at[(lane & 15) * 32 + ((2 * i + 1 + lane) & 31)] = w.y;
            }
        }
        __syncwarp();
        const int first = row0 + part * 16, rows = min(16, p.m - first);
        if (col0 + lane >= p.n) continue;
        const auto sum = [&](int r) { return at[r * 32 + ((lane + part * 16 + r) & 31)]; };
        if (!p.finish.residual) {
            for (int r = 0; r < rows; ++r) store_c(p, first + r, col0 + lane, sum(r));
            continue;
        }
#pragma unroll 1
        for (int r0 = 0; r0 < rows; r0 += 8) {
            float add[8];
#pragma unroll
            for (int r = 0; r < 8; ++r)
                add[r] = load_param(p.finish.residual, p.finish.residual_bf16, (long long)min(first + r0 + r, p.m - 1) * p.finish.residual_row + col0 + lane);
#pragma unroll
            for (int r = 0; r < 8; ++r)
                if (r0 + r < rows) store_c(p, first + r0 + r, col0 + lane, sum(r0 + r) + add[r]);
        }
    }
}

template <bool CHUNKED, bool TMA>
__device__ __forceinline__ void linear_epilogue(const DenseArgs<Linear> &p, const CUtensorMap &c_map, const PairBlock &b,
                                                float (*columns)[GROUPS][32])
{
    const int lane = b.lane, quarter = b.warp & 3;
    float (*bias)[32] = columns[b.warp];
    uint8_t *staging = b.aligned + PAIR_STAGING_AT + b.warp * BUFFERS * PAIR_STAGING_BYTES;
    int buffer = 0;
    const uint32_t read_bars[2] = {cluster_addr(ptx::smem_addr(&b.sums_read[0]), 0),
                                   cluster_addr(ptx::smem_addr(&b.sums_read[1]), 0)};
    const bool by_units = TMA && p.finish.residual && p.finish.residual_aligned;
    TileWalk walk = make_walk(b.warp, p.tile_n);
    PairWalk items(p, b.pair);
    PairItem item, ahead;
    bool more = items.take(p, b.pair, ahead);
    float next[GROUPS];
    if (more) load_next_columns(p.finish.bias, p.finish.bias_bf16, walk, ahead.tile_n * p.tile_n, p.n, lane, next);
    int sets = 0;
    uint4 units[4], units_ahead[4] = {};  // of this group and of the next one
    const auto load_first = [&](bool down) {  // of the next tile
        const int slot = down ? walk.own - 1 : 0;
        load_residual(p, ahead.tile_m * PAIR_ROWS + (int)b.rank * 128 + quarter * 32, ahead.tile_n * p.tile_n + walk.column(slot), lane, units_ahead);
    };
    if (by_units && more && ahead.slot < 0) load_first(!CHUNKED);
    while (more) {
        item = ahead;
        const int n0 = item.tile_n * p.tile_n, row0 = item.tile_m * PAIR_ROWS + (int)b.rank * 128 + quarter * 32;
        put_next_columns(next, lane, bias);
        more = items.take(p, b.pair, ahead);
        if (more) load_next_columns(p.finish.bias, p.finish.bias_bf16, walk, ahead.tile_n * p.tile_n, p.n, lane, next);
        const int chunks = CHUNKED ? (item.last - item.first + p.chunk - 1) / p.chunk : 1;
        const bool units_of = by_units && item.slot < 0;
        float total[CHUNKED ? GROUPS : 1][32];
        if constexpr (CHUNKED) {
#pragma unroll
            for (int s = 0; s < GROUPS; ++s)
#pragma unroll
                for (int i = 0; i < 32; ++i) total[s][i] = 0.0f;
        }
        for (int chunk = 0; chunk < chunks; ++chunk, ++sets) {
            walk.down = !(sets & 1);
            if (!warp_wait(&b.sums_full[sets & 1], (sets >> 1) & 1, 4)) {
                ptx::bulk_wait_all();  // results on their way are read from this block's shared memory
                return;
            }
            fence_after_sync();
            const uint32_t from = b.tmem + ((uint32_t)(quarter * 32) << 16) + ((sets & 1) ? b.second_set : 0);
            const auto read_over = [&] {
                fence_before_sync();
                if (lane == 0) arrive_remote(read_bars[sets & 1]);
                __syncwarp();
            };
            uint32_t r[32];
            if constexpr (CHUNKED) {
#pragma unroll
                for (int s = 0; s < GROUPS; ++s) {  // in any order: a chunk's products take longer than this
                    if (s >= walk.own) break;
                    tmem_load32(from + walk.column(s), r);
                    tmem_wait(r);
#pragma unroll
                    for (int i = 0; i < 32; ++i) total[s][i] += __uint_as_float(r[i]);
                }
                read_over();
            } else {
#pragma unroll 1
                for (int t = 0; t < walk.own; ++t) {
                    tmem_load32(from + walk.column(walk.slot(t)), r);
                    tmem_wait(r);
                    if (t == (b.apart ? walk.own - 1 : 0)) read_over();
#pragma unroll
                    for (int i = 0; i < 4; ++i) units[i] = units_ahead[i];
                    if (units_of && t + 1 < walk.own)
                        load_residual(p, row0, n0 + walk.column(walk.slot(t + 1)), lane, units_ahead);
                    else if (by_units && t + 1 == walk.own && more && ahead.slot < 0)
                        load_first(!walk.down);
                    finish_linear<TMA>(p, c_map, item, row0, quarter, b.rank, lane, walk.group(t), r, bias[walk.slot(t)], units, units_of, staging, buffer);
                }
            }
        }
        if constexpr (CHUNKED) {
#pragma unroll 1
            for (int s = 0; s < walk.own; ++s) {  // on total[0]
                const int group = SUBS * s + walk.sub;
#pragma unroll
                for (int i = 0; i < 4; ++i) units[i] = units_ahead[i];
                if (units_of && s + 1 < walk.own)
                    load_residual(p, row0, n0 + walk.column(s + 1), lane, units_ahead);
                else if (by_units && s + 1 == walk.own && more && ahead.slot < 0)
                    load_first(false);
                finish_linear<TMA>(p, c_map, item, row0, quarter, b.rank, lane, group, reinterpret_cast<const uint32_t *>(total[0]), bias[s], units,
                              units_of, staging, buffer);
#pragma unroll
                for (int j = 0; j + 1 < GROUPS; ++j)
#pragma unroll
                    for (int i = 0; i < 32; ++i) total[j][i] = total[j + 1][i];
            }
        }
    }
    ptx::bulk_wait_all();
}

template <bool CHUNKED, bool TMA>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(pair_threads(EPILOGUE_WARPS), 1)
    linear_pair_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
                       const __grid_constant__ CUtensorMap c_map, const __grid_constant__ DenseArgs<Linear> p)
{
    __shared__ __align__(16) float columns[EPILOGUE_WARPS][GROUPS][32];
    run_pair<CHUNKED, EPILOGUE_WARPS>(a_map, b_map, p, [&](const PairBlock &b) { linear_epilogue<CHUNKED, TMA>(p, c_map, b, columns); });
}

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
    unsigned maxima[2][2][2][EPILOGUE_WARPS];  // [exchange][block][of act(a), of a]
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
__device__ __forceinline__ float larger_magnitude(float most, f32x2 p)  // NaN stays
{
    const float2 v = values_of(p);
    asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(most) : "f"(v.x), "f"(v.y));
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
    __device__ __forceinline__ void arrive()
    {
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&shared.exchanged);
    }
    // All warps' largest, once every warp has put its own and arrived; false if the wait ran out.
    __device__ __forceinline__ bool take(int blocks, unsigned (*most)[2])
    {
        if (!warp_wait(&shared.exchanged, count & 1, 11)) return false;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int q = 0; q < 2; ++q)
                most[b][q] = b < blocks ? __reduce_max_sync(0xffffffffu, shared.maxima[count & 1][b][q][min(lane, EPILOGUE_WARPS - 1)]) : 0u;
        ++count;
        return true;
    }
    __device__ __forceinline__ bool meet(int blocks, unsigned (*most)[2])
    {
        arrive();
        return take(blocks, most);
    }
};

template <int ACTIVATION>
__device__ __forceinline__ void pack_epilogue(const PackArgs &p, const PairBlock &b, PackShared &shared, float (*columns)[GROUPS][32])
{
    constexpr bool GROWS = ACTIVATION == DIPACO_ACTIVATION_GELU || ACTIVATION == DIPACO_ACTIVATION_SILU;
    const int lane = b.lane, quarter = b.warp & 3;
    float (*bias)[32] = columns[b.warp];
    const uint32_t read_bars[2] = {cluster_addr(ptx::smem_addr(&b.sums_read[0]), 0),
                                   cluster_addr(ptx::smem_addr(&b.sums_read[1]), 0)};
    const int scale_cols = (p.n + 127) / 128, blocks = p.tile_n / 128;
    const bool keep = p.second.codes != nullptr;
    TileWalk walk = make_walk(b.warp, p.tile_n);
    Exchange exchange = {shared, b.warp, lane};
    float next[GROUPS];
    int tile_m, tile_n, sets = 0;
    PairWalk::place(p, b.pair, tile_m, tile_n);
    load_next_columns(p.bias, p.bias_bf16, walk, tile_n * p.tile_n, p.n, lane, next);
    for (int tile = b.pair; tile < p.whole_tiles; tile += p.pairs, ++sets) {  // as PairWalk takes them
        const int n0 = tile_n * p.tile_n, row0 = tile_m * PAIR_ROWS + (int)b.rank * 128;
        const int row = row0 + quarter * 32 + lane;
        put_next_columns(next, lane, bias);
        if (!warp_wait(&b.sums_full[sets & 1], (sets >> 1) & 1, 4)) return;
        fence_after_sync();
        const uint32_t from = b.tmem + ((uint32_t)(quarter * 32) << 16) + ((sets & 1) ? b.second_set : 0);
        walk.down = !(sets & 1);
        uint32_t held[32], r[32];  // held: the first group, whose columns the next tile's products overwrite
        f32x2 a[16];
        tmem_load32(from + walk.column(walk.slot(0)), held);
        tmem_wait(held);
        if (!b.apart) {
            fence_before_sync();
            if (lane == 0) arrive_remote(read_bars[sets & 1]);
            __syncwarp();
        }
        unsigned most[2][2];
        add_columns(bias[walk.slot(0)], held, a);
        float top = 0.0f, magnitude = 0.0f;
#pragma unroll 1
        for (int t = 0; t < walk.own; ++t) {
            if (t + 1 < walk.own) tmem_load32(from + walk.column(walk.slot(t + 1)), r);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                if (ACTIVATION != DIPACO_ACTIVATION_NONE) top = larger3(top, a[j]);
                magnitude = larger_magnitude(magnitude, a[j]);
            }
            if (walk.ends_block(t)) {
                if (row >= p.m) top = magnitude = 0.0f;  // the bias is not the matrix's there
                exchange.put(walk.block(t), __float_as_uint(top), __float_as_uint(magnitude));
                top = magnitude = 0.0f;
            }
            if (t + 1 < walk.own) {
                tmem_wait(r);
                add_columns(bias[walk.slot(t + 1)], r, a);
            }
        }
        exchange.arrive();
        // the next tile's place and biases while the others arrive
        if (tile + p.pairs < p.whole_tiles) {
            PairWalk::place(p, tile + p.pairs, tile_m, tile_n);
            load_next_columns(p.bias, p.bias_bf16, walk, tile_n * p.tile_n, p.n, lane, next);
        }
        if (!exchange.take(blocks, most)) return;
        bool careful = false, in_pairs = true;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (k >= blocks || n0 + k * 128 >= p.n || row0 >= p.m) continue;
            careful |= most[k][1] >= 0x7f800000u;
            if (GROWS) careful |= most[k][0] < __float_as_uint(grows_from<ACTIVATION>());
            in_pairs &= most[k][1] <= __float_as_uint(pairs_up_to<ACTIVATION>());
            if (ACTIVATION == DIPACO_ACTIVATION_NONE)
                most[k][0] = most[k][1];
            else
                most[k][0] = __float_as_uint(values_of(activate<ACTIVATION>(pair_of(__uint_as_float(most[k][0])))).x);
        }
        if (careful) {  // the same for all epilogue warps of the block
            unsigned of_y = 0u, of_a = 0u;
#pragma unroll 1
            for (int t = 0; t < walk.own; ++t) {
                if (t == 0) {
                    add_columns(bias[walk.slot(0)], held, a);
                } else {
                    tmem_load32(from + walk.column(walk.slot(t)), r);
                    tmem_wait(r);
                    add_columns(bias[walk.slot(t)], r, a);
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    of_y = finite_magnitudes(of_y, activate<ACTIVATION>(a[j]));
                    of_a = finite_magnitudes(of_a, a[j]);
                }
                if (walk.ends_block(t)) {
                    if (row >= p.m) of_y = of_a = 0u;
                    exchange.put(walk.block(t), of_y, of_a);
                    of_y = of_a = 0u;
                }
            }
            if (!exchange.meet(blocks, most)) return;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            most[k][0] = scale_byte(most[k][0]);
            most[k][1] = scale_byte(most[k][1]);
        }
        if (b.warp == 0 && lane < blocks && n0 + lane * 128 < p.n && row0 < p.m) {
            const long long at = (long long)(row0 / 128) * scale_cols + n0 / 128 + lane;
            p.first.scales[at] = (uint8_t)(lane ? most[1][0] : most[0][0]);
            if (keep) p.second.scales[at] = (uint8_t)(lane ? most[1][1] : most[0][1]);
        }
        // One loop for the ordinary blocks and another for the rare ones: code that is jumped over costs instruction cache.
        const auto encode_tile = [&](auto rare) {
            constexpr bool RARE = decltype(rare)::value;
            add_columns(bias[walk.slot(0)], held, a);
#pragma unroll 1
            for (int t = 0; t < walk.own; ++t) {
                const int slot = walk.slot(t), col = n0 + walk.column(slot), left = p.n - col;
                const bool inside = row < p.m && left > 0, second = walk.block(t);
                if (t + 1 < walk.own) tmem_load32(from + walk.column(walk.slot(t + 1)), r);
                unsigned w[8];
                if (keep) {
                    encode32<RARE>(a, scale_reciprocal(second ? most[1][1] : most[0][1]), w);
                    if (inside) store_codes(p.second, row, col, left, w);
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) a[j] = RARE ? activate<ACTIVATION>(a[j]) : activate_in_pairs<ACTIVATION>(a[j]);
                encode32<RARE>(a, scale_reciprocal(second ? most[1][0] : most[0][0]), w);
                if (inside) store_codes(p.first, row, col, left, w);
                if (t + 1 < walk.own) {
                    tmem_wait(r);
                    if (b.apart && t + 2 == walk.own) {  // a warp has two groups or four
                        fence_before_sync();
                        if (lane == 0) arrive_remote(read_bars[sets & 1]);
                        __syncwarp();
                    }
                    add_columns(bias[walk.slot(t + 1)], r, a);
                }
            }
        };
        if (careful || !in_pairs)
            encode_tile(std::true_type());
        else
            encode_tile(std::false_type());
    }
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

// 16 of the warp's rows of 32 columns of tensor memory: lane l has columns 8 i + 2 (l % 4) + {0, 1} of two of them, of the
// four lanes that share l % 4 in every other register pair.
__device__ __forceinline__ void tmem_load_across(uint32_t address, uint32_t *r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(address));
}

// Sums over the warp's 32 rows of 32 columns that are in tensor memory, a column for a lane.  Read across, a lane has
// eight columns' values of four rows, so that three exchanges are left; with a row for a lane it would take five.
__device__ __forceinline__ float column_sums(uint32_t address, int lane)
{
    uint32_t r[32];
    tmem_load_across(address, r);
    tmem_load_across(address + (16u << 16), r + 16);
    tmem_wait(r);
    float s[8];  // columns 8 (i / 2) + 2 (lane % 4) + i % 2
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int at = i / 2 * 4 + i % 2;
        s[i] = (__uint_as_float(r[at]) + __uint_as_float(r[at + 2])) + (__uint_as_float(r[at + 16]) + __uint_as_float(r[at + 18]));
    }
    // a lane hands on the half of its columns that the lane across keeps
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) {
        const bool upper = lane & (4 * o);
#pragma unroll
        for (int i = 0; i < o; ++i) {
            const float give = upper ? s[i] : s[i + o];
            s[i] = (upper ? s[i + o] : s[i]) + __shfl_xor_sync(0xffffffffu, give, 4 * o);
        }
    }
    return s[0];
}
// Which column that is.
__device__ __forceinline__ int column_of_sum(int lane) { return (lane >> 3) * 8 + 2 * (lane & 3) + (lane >> 2 & 1); }

// What the epilogue warps of the gradient share, where the others have their results' buffers.
struct BackShared {
    float sums[2][PAIR_MAX_N / 32][4][32];  // over 32 rows, for two tiles
    // The slopes at all values that a code stands for in the tile's blocks of a, for two tiles: a block has one scale, so
    // that a value's slope is looked up in place of two powers and reciprocals and 13 products for every pair.
    float slopes[2][2][256];
};
static_assert(sizeof(BackShared) <= PAIR_EPILOGUE_WARPS * PAIR_STAGING * PAIR_STAGING_BYTES, "in the place of the buffers");

// Steps whose sums are taken in one go.  dbias is a result in fp32, whose sums would otherwise lose 1.3e-4 of themselves
// over 65536 values of one sign (1.2e-6 in parts; over 8192 in one go 8e-6).  Parts cost the wide tiles: 16384x2048x8192
// takes 197 us in one go and 289 in parts of 2048.  da goes with dbias and does not depend on whether that is wanted.
constexpr int BACK_STEPS = 64;

// The sums of a tile that are taken out of the products' sets a chunk at a time: added up in columns of tensor memory that
// the sets leave free, each by the warp that reads it.  Counts the sets; false if a wait ran out.
__device__ __forceinline__ bool add_chunks(const PackArgs &p, const PairBlock &b, const TileWalk &walk, const uint32_t *read_bars,
                                           uint32_t totals, int &sets)
{
    const uint32_t rows = (uint32_t)(b.warp & 3) * 32 << 16;
    for (int first = 0; first < p.steps; first += p.chunk, ++sets) {
        if (!warp_wait(&b.sums_full[sets & 1], (sets >> 1) & 1, 4)) return false;
        fence_after_sync();
        const uint32_t from = b.tmem + rows + ((sets & 1) ? b.second_set : 0);
#pragma unroll 1
        for (int s = 0; s < walk.own; ++s) {
            uint32_t r[32], before[32];
            f32x2 v[16];
            tmem_load32(from + walk.column(s), r);
            tmem_wait(r);
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = pair_of(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
            if (first > 0) {
                tmem_load32(totals + walk.column(s), before);
                tmem_wait(before);
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    v[j] = add2(pair_of(__uint_as_float(before[2 * j]), __uint_as_float(before[2 * j + 1])), v[j]);
            }
            tmem_store32(totals + walk.column(s), v);
        }
        tmem_stored();
        fence_before_sync();
        if (b.lane == 0) arrive_remote(read_bars[sets & 1]);
        __syncwarp();
    }
    return true;
}

template <int ACTIVATION, bool CHUNKED>
__device__ __forceinline__ void back_epilogue(const PackArgs &p, const PairBlock &b, PackShared &shared)
{
    BackShared &of_tiles = *reinterpret_cast<BackShared *>(b.aligned + PAIR_STAGING_AT);
    const int lane = b.lane, quarter = b.warp & 3;
    const uint32_t read_bars[2] = {cluster_addr(ptx::smem_addr(&b.sums_read[0]), 0),
                                   cluster_addr(ptx::smem_addr(&b.sums_read[1]), 0)};
    const int scale_cols = (p.n + 127) / 128, blocks = p.tile_n / 128;
    TileWalk walk = make_walk(b.warp, p.tile_n);
    Exchange exchange = {shared, b.warp, lane};
    constexpr bool SLOPES = ACTIVATION != DIPACO_ACTIVATION_NONE;
    // a group's codes of a, two units of 16 (rows of codes are padded to whole units)
    const auto load_codes = [&](int row, int col, uint4 *codes) {
        codes[0] = codes[1] = make_uint4(0u, 0u, 0u, 0u);
        if (!SLOPES || row >= p.m) return;
        const uint4 *at = reinterpret_cast<const uint4 *>(p.a_codes + row * p.a_stride + col);
        if (col < p.n) codes[0] = __ldcs(at);
        if (col + 16 < p.n) codes[1] = __ldcs(at + 1);
    };
    // the scales of a tile's blocks of a, and the slopes of this thread's code in them
    const auto load_scales = [&](int tile_m, int tile_n, float *scales) {
        const int row = tile_m * PAIR_ROWS + (int)b.rank * 128;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int block = tile_n * p.tile_n / 128 + k;
            scales[k] = SLOPES && k < blocks && row < p.m && block < scale_cols ? scale_value(p.of_a_scales[(long long)(row / 128) * scale_cols + block]) : 0.0f;
        }
    };
    const auto put_slopes = [&](int set, const float *scales) {
        static_assert(EPILOGUE_WARPS * 32 == 256, "a code for a thread");
        const int code = b.warp * 32 + lane;
        const float v = decode2((unsigned)code).x;
        const float2 s = values_of(slope<ACTIVATION>(mul2(pair_of(v), pair_of(scales[0], scales[1]))));
        of_tiles.slopes[set][0][code] = s.x;
        of_tiles.slopes[set][1][code] = s.y;
    };
    int tile_m, tile_n, turn = 0, sets = 0;  // tiles, and sets of sums, so far
    PairWalk::place(p, b.pair, tile_m, tile_n);
    uint4 codes[2];
    float scales[2];
    unsigned most[2][2];
    walk.down = true;
    load_codes(tile_m * PAIR_ROWS + (int)b.rank * 128 + quarter * 32 + lane, tile_n * p.tile_n + walk.column(walk.slot(0)), codes);
    load_scales(tile_m, tile_n, scales);
    if (SLOPES) put_slopes(0, scales);
    if (!exchange.meet(0, most)) return;
    for (int tile = b.pair; tile < p.whole_tiles; tile += p.pairs, ++turn) {  // as PairWalk takes them
        const int n0 = tile_n * p.tile_n, row0 = tile_m * PAIR_ROWS + (int)b.rank * 128;
        const int row = row0 + quarter * 32 + lane;
        uint32_t from = b.tmem + ((uint32_t)(quarter * 32) << 16);
        const int set = turn & 1;  // of sums, unless they are chunks'
        if constexpr (CHUNKED) {
            from += p.tile_n;
            if (!add_chunks(p, b, walk, read_bars, from, sets)) return;
        } else {
            if (!warp_wait(&b.sums_full[set], (turn >> 1) & 1, 4)) return;
            fence_after_sync();
            from += set ? b.second_set : 0;
        }
        walk.down = !(turn & 1);
        const bool more = tile + p.pairs < p.whole_tiles;
        if (more) {
            PairWalk::place(p, tile + p.pairs, tile_m, tile_n);
            load_scales(tile_m, tile_n, scales);
        }
        f32x2 held[16], v[16];  // held: the first group's results, as the next tile's products overwrite its columns
        float magnitude = 0.0f;
        uint32_t r[32];
        tmem_load32(from + walk.column(walk.slot(0)), r);
#pragma unroll 1
        for (int t = 0; t < walk.own; ++t) {
            const int slot = walk.slot(t);
            const unsigned words[8] = {codes[0].x, codes[0].y, codes[0].z, codes[0].w, codes[1].x, codes[1].y, codes[1].z, codes[1].w};
            if (t + 1 < walk.own) {
                load_codes(row, n0 + walk.column(walk.slot(t + 1)), codes);
            } else if (more) {  // the next tile's first
                TileWalk then = walk;
                then.down = !walk.down;
                load_codes(tile_m * PAIR_ROWS + (int)b.rank * 128 + quarter * 32 + lane, tile_n * p.tile_n + then.column(then.slot(0)), codes);
            }
            tmem_wait(r);
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = pair_of(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
            if (t + 1 < walk.own) tmem_load32(from + walk.column(walk.slot(t + 1)), r);
            if constexpr (SLOPES) {
                const float *slopes = of_tiles.slopes[turn & 1][walk.block(t)];
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const unsigned w = words[j / 2] >> 16 * (j & 1);
                    v[j] = mul2(v[j], pair_of(slopes[w & 255u], slopes[w >> 8 & 255u]));
                }
            }
            if (row >= p.m) {  // zero times a NaN of the weights
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = 0ull;
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) magnitude = larger_magnitude(magnitude, v[j]);
            if (t > 0 || p.row_sums) tmem_store32(from + walk.column(slot), v);
            if (p.row_sums) {
                tmem_stored();
                of_tiles.sums[turn & 1][walk.group(t)][quarter][column_of_sum(lane)] = column_sums(from + walk.column(slot), lane);
            }
            if (t == 0) {
                if (!CHUNKED && !b.apart) {
                    fence_before_sync();
                    if (lane == 0) arrive_remote(read_bars[set]);
                    __syncwarp();
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) held[j] = v[j];
            }
            if (walk.ends_block(t)) {
                exchange.put(walk.block(t), __float_as_uint(magnitude), 0u);
                magnitude = 0.0f;
            }
        }
        tmem_stored();
        if (SLOPES && more) put_slopes(~turn & 1, scales);
        if (!exchange.meet(blocks, most)) return;
        if (p.row_sums && b.warp < p.tile_n / 32 && row0 < p.m && n0 + b.warp * 32 + lane < p.n) {
            const float(*s)[32] = of_tiles.sums[turn & 1][b.warp];
            p.row_sums[(long long)(row0 / 128) * p.n + n0 + b.warp * 32 + lane] = (s[0][lane] + s[1][lane]) + (s[2][lane] + s[3][lane]);
        }
        // the results of the t-th group
        const auto results = [&](int t) {
            if (t == 0) {
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = held[j];
            } else {
                tmem_load32(from + walk.column(walk.slot(t)), r);
                tmem_wait(r);
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = pair_of(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
            }
        };
        const bool careful = most[0][0] >= 0x7f800000u || most[1][0] >= 0x7f800000u;
        if (careful) {  // the same for all epilogue warps of the block
            unsigned finite = 0u;
#pragma unroll 1
            for (int t = 0; t < walk.own; ++t) {
                results(t);
#pragma unroll
                for (int j = 0; j < 16; ++j) finite = finite_magnitudes(finite, v[j]);
                if (walk.ends_block(t)) {
                    exchange.put(walk.block(t), finite, 0u);
                    finite = 0u;
                }
            }
            if (!exchange.meet(blocks, most)) return;
        }
        const unsigned bytes[2] = {scale_byte(most[0][0]), scale_byte(most[1][0])};
        if (b.warp == 0 && lane < blocks && n0 + lane * 128 < p.n && row0 < p.m)
            p.first.scales[(long long)(row0 / 128) * scale_cols + n0 / 128 + lane] = (uint8_t)(lane ? bytes[1] : bytes[0]);
        const auto encode_tile = [&](auto rare) {
#pragma unroll 1
            for (int t = 0; t < walk.own; ++t) {
                const int slot = walk.slot(t), col = n0 + walk.column(slot), left = p.n - col;
                results(t);
                if (!CHUNKED && b.apart && t + 1 == walk.own) {
                    fence_before_sync();
                    if (lane == 0) arrive_remote(read_bars[set]);
                    __syncwarp();
                }
                if (left <= 0) continue;
                unsigned w[8];
                encode32<decltype(rare)::value>(v, scale_reciprocal(walk.block(t) ? bytes[1] : bytes[0]), w);
                if (row < p.m) store_codes(p.first, row, col, left, w);
            }
        };
        if (careful)
            encode_tile(std::true_type());
        else
            encode_tile(std::false_type());
    }
}

template <int ACTIVATION, bool BACK, bool CHUNKED>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(pair_threads(EPILOGUE_WARPS), 1)
    packed_pair_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
                       const __grid_constant__ PackArgs p)
{
    __shared__ PackShared shared;
    __shared__ __align__(16) float columns[EPILOGUE_WARPS][GROUPS][32];  // biases of the warps' columns
    if (threadIdx.x == 64) ptx::mbar_init(&shared.exchanged, EPILOGUE_WARPS);  // seen after run_pair's first barrier
    run_pair<CHUNKED, EPILOGUE_WARPS>(a_map, b_map, p, [&](const PairBlock &b) {
        if constexpr (BACK)
            back_epilogue<ACTIVATION, CHUNKED>(p, b, shared);
        else
            pack_epilogue<ACTIVATION>(p, b, shared, columns);
    });
}

// Few tokens through a weight, packed: a cluster of eight blocks has a block of 128 columns, whose largest values its
// blocks read from one another's shared memory.
constexpr int FEW_CLUSTER = 8;
static_assert(FEW_CLUSTER * FEW_THREADS / 32 * FEW_OUTPUTS == PACK_BLOCK && FEW_OUTPUTS == 2, "a block of columns");

struct FewPackArgs : FewArgs {
    Linear finish;  // bias and activation
    PackedCodes first, second;
};

template <int M>
__global__ void __cluster_dims__(FEW_CLUSTER, 1, 1) __launch_bounds__(FEW_THREADS) few_pack_kernel(const __grid_constant__ FewPackArgs p)
{
    extern __shared__ __align__(16) __half tokens[];
    __shared__ unsigned of_warps[2][FEW_THREADS / 32], of_block[2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint8_t *token_scales = reinterpret_cast<uint8_t *>(tokens + M * p.steps * STEP);
    const int col = (int)(blockIdx.x * (FEW_THREADS / 32) + warp) * FEW_OUTPUTS;  // and the next
    few_tokens<M>(p, tokens, token_scales);
    __syncthreads();
    float a[FEW_OUTPUTS][M] = {}, y[FEW_OUTPUTS][M];
    if (col < p.outputs) few_sums<M>(p, tokens, token_scales, col, lane, a);
    unsigned most[2] = {0u, 0u};
#pragma unroll
    for (int r = 0; r < FEW_OUTPUTS; ++r) {
        const float bias = p.finish.bias && col + r < p.outputs ? load_param(p.finish.bias, p.finish.bias_bf16, col + r) : 0.0f;
#pragma unroll
        for (int t = 0; t < M; ++t) {
            a[r][t] += bias;
            y[r][t] = values_of(p.finish.act(pair_of(a[r][t]))).x;
            if (col + r < p.outputs) {
                most[0] = max(most[0], finite_magnitude(y[r][t]));
                most[1] = max(most[1], finite_magnitude(a[r][t]));
            }
        }
    }
    if (lane == 0) {
        of_warps[0][warp] = most[0];
        of_warps[1][warp] = most[1];
    }
    __syncthreads();
    if (threadIdx.x < 2) {
        unsigned m = 0u;
        for (int w = 0; w < FEW_THREADS / 32; ++w) m = max(m, of_warps[threadIdx.x][w]);
        of_block[threadIdx.x] = m;
    }
    cluster_sync();
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        unsigned m = 0u;
        if (lane < FEW_CLUSTER)
            asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(m) : "r"(cluster_addr(ptx::smem_addr(&of_block[q]), lane)) : "memory");
        most[q] = scale_byte(__reduce_max_sync(0xffffffffu, m));
    }
    // no block ends while its values may still be read
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    const int block = (int)blockIdx.x / FEW_CLUSTER;
    if (threadIdx.x == 0 && blockIdx.x % FEW_CLUSTER == 0) {
        p.first.scales[block] = (uint8_t)most[0];
        if (p.second.codes) p.second.scales[block] = (uint8_t)most[1];
    }
    const auto store = [&](const PackedCodes &out, unsigned scale, const float (*v)[M]) {
#pragma unroll
        for (int t = 0; t < M; ++t) {
            const unsigned codes = encode2(v[0][t], v[1][t], scale_reciprocal(scale));
            uint8_t *at = out.codes + t * out.stride + col;
            if (lane != t || col >= p.outputs) continue;
            if (col + 1 < p.outputs)
                *reinterpret_cast<unsigned short *>(at) = (unsigned short)codes;
            else
                *at = (uint8_t)codes;
        }
    };
    store(p.first, most[0], y);
    if (p.second.codes) store(p.second, most[1], a);
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
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

// Tiles of whole blocks: 256 columns, or 128 where that takes less time by the estimate of plan_pairs (and some clocks
// for a column's epilogue that the next products wait for).  Sums taken in chunks are added up in the columns of tensor
// memory that tiles of 128 leave free.
void plan_blocks(PackArgs &p, bool chunked)
{
    double best = 0.0;
    for (const int tile_n : {256, 128}) {
        if (chunked && tile_n > 128) continue;
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
    p.chunk = chunked ? CHUNK_F32 : CHUNK_BF16;
}

template <bool BACK, bool CHUNKED>
int launch_packed(const CUtensorMap &a_map, const CUtensorMap &b_map, const PackArgs &p, int activation, cudaStream_t stream)
{
    const auto kernel = activation == DIPACO_ACTIVATION_RELU   ? packed_pair_kernel<DIPACO_ACTIVATION_RELU, BACK, CHUNKED>
                        : activation == DIPACO_ACTIVATION_SILU ? packed_pair_kernel<DIPACO_ACTIVATION_SILU, BACK, CHUNKED>
                        : activation == DIPACO_ACTIVATION_GELU ? packed_pair_kernel<DIPACO_ACTIVATION_GELU, BACK, CHUNKED>
                                                               : packed_pair_kernel<DIPACO_ACTIVATION_NONE, BACK, CHUNKED>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PAIR_SMEM) != cudaSuccess) return launch_status();
    kernel<<<2 * p.pairs, pair_threads(EPILOGUE_WARPS), PAIR_SMEM, stream>>>(a_map, b_map, p);
    return launch_status();
}

bool is_activation(int activation) { return activation >= DIPACO_ACTIVATION_NONE && activation <= DIPACO_ACTIVATION_GELU; }

// A product whose sums are taken in one go.
int check_contraction(int64_t m, int64_t n, int64_t k)
{
    if (k < 0) return DIPACO_EINVAL;
    if (const int rc = check_extents(m, n)) return rc;
    // tiles and the step to a pair's next one fit an int
    return k > (int64_t)CHUNK_BF16 * STEP || ceil_div(m, PAIR_ROWS) * ceil_div(n, 128) > INT32_MAX - 65536 ? DIPACO_ELIMIT : DIPACO_OK;
}

int launch_few_pack(const FewPackArgs &p, int tokens, cudaStream_t stream)
{
    const auto kernel = tokens == 1 ? few_pack_kernel<1> : tokens == 2 ? few_pack_kernel<2> : tokens == 3 ? few_pack_kernel<3> : few_pack_kernel<4>;
    const int smem = few_smem(p, tokens);
    // always the largest there can be, as in launch_few
    if (smem > 48 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, FEW_SMEM) != cudaSuccess)
        return launch_status();
    kernel<<<(unsigned)ceil_div(p.outputs, PACK_BLOCK) * FEW_CLUSTER, FEW_THREADS, smem, stream>>>(p);
    return launch_status();
}

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
    const Linear finish = {bias, residual, residual_stride, activation, bias_dtype == DIPACO_BF16,
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
    const DenseKernels<Linear> kernels = {{linear_pair_kernel<false, false>, linear_pair_kernel<false, true>},
                                          {linear_pair_kernel<true, false>, linear_pair_kernel<true, true>},
                                          pair_threads(EPILOGUE_WARPS),
                                          true};
    return launch_product(x, w, false, true, y, y_stride, dtype, false, finish, kernels, workspace, stream);
}

int dipaco_packed_linear_pack_workspace(int64_t m, int64_t n, int64_t k, int64_t *bytes)
{
    if (!bytes) return DIPACO_EINVAL;
    if (const int rc = check_contraction(m, n, k)) return rc;
    *bytes = k == 0 ? m * ceil_div(n, 4) * 16 : 0;  // sums over nothing are packed from fp32
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
    const Linear finish = {bias, nullptr, 0, activation, bias_dtype == DIPACO_BF16, false, false};
    if (k == 0) {
        Linear sums_finish = finish;
        sums_finish.activation = DIPACO_ACTIVATION_NONE;
        float *sums = static_cast<float *>(workspace);
        const int64_t stride = ceil_div(n, 4) * 4;
        empty_sums_kernel<<<(unsigned)std::min<int64_t>(ceil_div(m, 256) * n, 148 * 8), 256, 0, stream>>>(sums, stride, m, (int)n, sums_finish);
        if (const int rc = launch_status()) return rc;
        return pack_activated(sums, stride, activation, y, a, stream);
    }
    if (m <= n && are_few(m, n, k, false, true)) {
        FewPackArgs p = {few_args(x, w), finish, packed_codes(y), packed_codes(a)};
        return launch_few_pack(p, (int)m, stream);
    }
    PackArgs p = {};
    set_operands(p, x, w, false, true);
    plan_blocks(p, false);
    p.first = packed_codes(y);
    p.second = packed_codes(a);
    p.bias = bias;
    p.bias_bf16 = bias_dtype == DIPACO_BF16;
    CUtensorMap a_map, b_map;
    if (!operand_map(&a_map, x, 128) || !operand_map(&b_map, w, p.tile_n / 2)) return DIPACO_ECUDA;
    return launch_packed<false, false>(a_map, b_map, p, activation, stream);
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
    const bool chunked = p.steps > BACK_STEPS;
    plan_blocks(p, chunked);
    p.first = packed_codes(da);
    p.a_codes = slopes ? static_cast<const uint8_t *>(a->codes) : nullptr;
    p.of_a_scales = slopes ? static_cast<const uint8_t *>(a->scales) : nullptr;
    p.a_stride = slopes ? a->stride : 0;
    p.row_sums = dbias ? static_cast<float *>(workspace) : nullptr;
    CUtensorMap a_map, b_map;
    if (!operand_map(&a_map, dy, 128) || !operand_map(&b_map, w, 128)) return DIPACO_ECUDA;
    if (const int rc = chunked ? launch_packed<true, true>(a_map, b_map, p, activation, stream)
                               : launch_packed<true, false>(a_map, b_map, p, activation, stream))
        return rc;
    if (dbias)
        row_sums_kernel<<<(unsigned)ceil_div(n, 32), 32 * SLICES, 0, stream>>>(p.row_sums, (int)ceil_div(m, PACK_BLOCK), p.n, dbias);
    return launch_status();
}

} // extern "C"
