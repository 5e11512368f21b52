// Products of packed matrices on pairs of SMs (see packed_matmul.cu, which states what they measured): the kernels,
// and what their epilogues have in common with those that do more than store (packed_linear.cu).
#pragma once

#include "inner_common.cuh"

#include <algorithm>
#include <cmath>

namespace dipaco {
namespace {

static __device__ int g_product_error;  // set by a bounded wait that ran out

// ------------------------------------------------------------------------------------------ PTX

// An address of this block's shared memory as seen from, or for, block `rank` of the cluster.
__device__ __forceinline__ uint32_t cluster_addr(uint32_t address, unsigned rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(address), "r"(rank));
    return r;
}
__device__ __forceinline__ unsigned cluster_rank()
{
    unsigned r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Orders what this thread wrote to shared memory before what the waiting block does.
__device__ __forceinline__ void arrive_cluster(uint32_t cluster_bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// Where only reads of tensor memory have to be over (fence_before_sync orders those).
__device__ __forceinline__ void arrive_remote(uint32_t cluster_bar)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ bool try_wait_cluster(uint64_t *bar, unsigned parity)
{
    unsigned ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(ptx::smem_addr(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}
// Whether the phase is over, without waiting: the same answer on the whole warp.
__device__ __forceinline__ bool test_arrived(uint64_t *bar, unsigned parity)
{
    unsigned ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(ptx::smem_addr(bar)), "r"(parity)
        : "memory");
    return __all_sync(0xffffffffu, ok);
}
// Bounded wait of a whole warp, which agrees on how it ended: what follows takes all its lanes.  CLUSTER:
// ordered after what the other block of the pair did before it arrived.
template <bool CLUSTER = false>
__device__ __forceinline__ bool warp_wait(uint64_t *bar, unsigned parity, int code, unsigned long long limit_ns = BULK_WAIT_LIMIT_NS)
{
    const auto arrived = [&] {
        const bool ok = CLUSTER ? try_wait_cluster(bar, parity) : ptx::mbar_try_wait(bar, parity);
        return __all_sync(0xffffffffu, ok) != 0;
    };
    if (arrived()) return true;
    const unsigned long long t0 = ptx::global_timer_ns();
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 256; ++i)
            if (arrived()) return true;
        if (__any_sync(0xffffffffu, ptx::global_timer_ns() - t0 > limit_ns)) {
            atomicCAS(&g_product_error, 0, code);
            return false;
        }
    }
}
// Of a pair's block; the barrier may be the other block's.
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], "
        "[%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, uint32_t src, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x),
                 "r"(y), "r"(src)
                 : "memory");
}
__device__ __forceinline__ void tmem_alloc(uint32_t *result, int columns)
{
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(ptx::smem_addr(result)),
                 "r"(columns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t address, int columns)
{
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(address), "r"(columns));
}
// 32 lanes x 16 bytes of shared memory to four columns of each 32-lane quarter of tensor memory, in both blocks
__device__ __forceinline__ void tmem_copy_scales(uint32_t address, uint64_t desc)
{
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(address), "l"(desc) : "memory");
}
__device__ __forceinline__ void mma_block_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t scale_a,
                                                 uint32_t scale_b, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(scale_a), "r"(scale_b), "r"((unsigned)add)
        : "memory");
}
// Arrives on the barrier of both blocks of the pair once the products issued so far are done.
__device__ __forceinline__ void mma_commit(uint64_t *bar)
{
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
            ptx::smem_addr(bar)),
        "h"((unsigned short)3)
        : "memory");
}
__device__ __forceinline__ void fence_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

__device__ __forceinline__ void tmem_load32(uint32_t address, uint32_t *r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(address));
}
// Waits for the loads so far; names the registers, which hold nothing before.
__device__ __forceinline__ void tmem_wait(uint32_t *r)
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                   "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]),
                   "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]),
                   "+r"(r[30]), "+r"(r[31])::"memory");
}

// ------------------------------------------------------------------------------------------ descriptors

// Shared-memory operand in the 128-byte swizzle: rows of 128 bytes, eight to a swizzle atom.  Contracted
// along the row (K-major) or across rows (MN-major); atoms follow one another either way.
__device__ __forceinline__ uint64_t operand_desc(uint32_t address)
{
    return (uint64_t)((address & 0x3ffffu) >> 4) | (uint64_t)(16384u >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 |
           1ull << 46 | 2ull << 61;
}
// Scale words: no swizzle, eight rows of 16 bytes to a 128-byte group.
__device__ __forceinline__ uint64_t scales_desc(uint32_t address)
{
    return (uint64_t)((address & 0x3ffffu) >> 4) | (uint64_t)(128u >> 4) << 16 | (uint64_t)(128u >> 4) << 32 | 1ull << 46;
}

// ------------------------------------------------------------------------------------------ common

constexpr int STEP = 128;                 // contracted values per step: one block
constexpr int CONTRACTED_PER_MMA = 32;
constexpr int SCALE_BYTES = 512;          // of shared memory for four columns: 32 lanes x 16 bytes
// A scale word holds the bytes of QUAD steps, and the instruction descriptor says which byte counts: the
// words are copied to tensor memory once for four steps.  Copies take the tensor cores' time: one for
// each step cost 20 % (8192^3: 555 us, 445 without any copy).
constexpr int QUAD = 4;
// The tensor cores truncate when they add 32 products to an fp32 sum: each of them to a quarter of the sum's last place
// (2^-25 of it) and the new sum to its own (2^-23).  Products that are alike lose 2^-24 of the sum so far, 2.4e-5 over
// 65501 of them; small ones beside a large one are lost whole, 3.7e-5 of a sum of 2048 built for it, and 2^-14 + 2^-17
// at most.  Sums that are returned in fp32 are therefore taken out of tensor memory every 16 steps, 2048 values, and added
// up in registers: under 2^-18 where products are alike, under 1e-6 where signs mix.  A result in bf16 has 2^-9 of
// rounding of its own: its sums are taken out every 512 steps, 65536 values, 2^-13 where products are alike.  (In one
// sum 2^21 positive products were off by a unit everywhere, 0.8 %.  Every 16 steps cost a product in bf16 up to 8 %:
// 8192x2048x131072 1570 -> 1700 us.)
constexpr int CHUNK_F32 = 16, CHUNK_BF16 = 512;  // powers of two

struct ProductArgs {
    const uint8_t *a_scales, *b_scales;
    int a_scale_cols, b_scale_cols;
    int transpose_a, transpose_b;  // A is stored [K, M]; B is stored [N, K]
    int m, n, steps;
    void *c;
    long long c_row;  // stride of C in elements
    int c_bf16, accumulate;
    // pair_kernel
    int chunk;  // steps after which a sum is taken out of tensor memory
    int tile_n, tiles_m, tiles_n;
    int pairs;
    int whole_tiles;  // tiles that one pair computes from end to end
    int head, helpers;  // of the others a pair does the first `head` steps, and `helpers` pairs share the rest
    int store_by_tma;
    int whole_n;  // columns in whole units of 16 bytes: the copy engine's
    float *partial;
};

// What becomes of a finished sum before it is rounded and stored: nothing.
struct AsItIs {
    static constexpr bool NOTHING = true;
};
template <class F> struct DenseArgs : ProductArgs {
    F finish;
};

// Bits: A and B e4m3 (0), A and B major-ness, N/8, e8m0 scales, M/16; scale_byte_desc adds the scale words'
// byte for B and A.
__device__ __forceinline__ uint32_t instruction_desc(const ProductArgs &p, int m, int n)
{
    return (uint32_t)(p.transpose_a ? 1 : 0) << 15 | (uint32_t)(p.transpose_b ? 0 : 1) << 16 | (uint32_t)(n >> 3) << 17 |
           1u << 23 | (uint32_t)(m >> 4) << 24;
}

__device__ __forceinline__ uint32_t scale_byte_desc(int byte) { return (uint32_t)byte << 4 | (uint32_t)byte << 29; }
__device__ __forceinline__ uint32_t byte_at(uint32_t word, int shift) { return word >> shift & 255u; }

__device__ __forceinline__ void store_c(const ProductArgs &p, long long row, long long col, float v)
{
    const long long at = row * p.c_row + col;
    if (p.c_bf16) {
        __nv_bfloat16 *c = static_cast<__nv_bfloat16 *>(p.c) + at;
        if (p.accumulate) v += __bfloat162float(*c);
        *c = __float2bfloat16_rn(v);
    } else {
        float *c = static_cast<float *>(p.c) + at;
        if (p.accumulate) v += *c;
        *c = v;
    }
}

// ------------------------------------------------------------------------------------------ pairs of SMs

// Each block of the pair holds 128 rows of A and half the tile's columns of B per stage.  Tensor memory:
// two sets of sums, and scales of five quads of steps at the end.  With 256 columns the sets overlap: the
// first set's last columns are the second's first.  They are read out first, and the products of the
// next tile start as soon as that is done; with fewer columns the sets are apart and the next tile's
// products only wait for the tile before the last to be read out.
constexpr int PAIR_STAGES = 5;
constexpr int PAIR_OPERAND_BYTES = 128 * STEP;
constexpr int PAIR_STAGE_BYTES = 2 * PAIR_OPERAND_BYTES;
constexpr int PAIR_WORDS_BYTES = 3 * SCALE_BYTES;  // scale words of a quad: of A, and of B twice four columns
// Scale words are written for eight steps at a time: a signal between the blocks for each step held the
// tensor cores up (16384x2048x8192: 427 us against 285).
constexpr int PAIR_WORDS_STEPS = 8;
constexpr int PAIR_WORDS_SET = PAIR_WORDS_STEPS / QUAD * PAIR_WORDS_BYTES;
constexpr int PAIR_EPILOGUE_WARPS = 8;
constexpr int PAIR_STAGING = 3;           // buffers of an epilogue warp
constexpr int PAIR_STAGING_BYTES = 2048;  // of one: 32 rows of 64 bytes
// shared memory: operands and staging on 1024-byte boundaries (the swizzle goes by address), then scale words
constexpr int PAIR_STAGING_AT = PAIR_STAGES * PAIR_STAGE_BYTES;
constexpr int PAIR_WORDS_AT = PAIR_STAGING_AT + PAIR_EPILOGUE_WARPS * PAIR_STAGING * PAIR_STAGING_BYTES;
constexpr int PAIR_SMEM = PAIR_WORDS_AT + 2 * PAIR_WORDS_SET + 1024;
constexpr int pair_threads(int epilogue_warps) { return (epilogue_warps + 3) * 32; }  // + loads, products, scale words
// Scale columns are written again five quads later, when the last step of the quad that had them is done:
// the step that begins the new quad has been loaded where the step PAIR_STAGES before it was, which is
// thus done, and only quads of single steps (short contractions) are closer together than that.
constexpr int PAIR_SCALE_COLUMNS = 12;
constexpr int PAIR_SCALE_SLOTS = 5;
constexpr int PAIR_SCALES_AT = 512 - PAIR_SCALE_SLOTS * PAIR_SCALE_COLUMNS;
// With 256 columns the sets of sums share 60, the first two groups of 32 that are read out.
static_assert(PAIR_WORDS_STEPS == 2 * QUAD && CHUNK_F32 % QUAD == 0 && CHUNK_BF16 % QUAD == 0 && PAIR_SCALE_SLOTS <= PAIR_STAGES && 2 * 256 - PAIR_SCALES_AT <= 64 && 2 * 224 <= PAIR_SCALES_AT, "quads and tensor memory");
constexpr int PAIR_MAX_N = 256;
constexpr int PAIR_ROWS = 256;
constexpr int RASTER = 8;  // row tiles that share column tiles while those are in L2

// A piece of work: steps [first, last) of a tile.
struct PairItem {
    int tile_m, tile_n, first, last;
    int slot;  // where a partial sum goes; -1: the tile is finished here
};

// The pieces of one pair.  Whole tiles come first, one for each pair and round.  The tiles of a last,
// unfilled round have a pair each for their first `head` steps, and the other pairs share the steps that
// are left evenly: all pairs are done at about the same time, and most of them are at the same place of
// the contraction at the same time, so that they share what they load in L2.
struct PairWalk {
    int tile;
    long long next, end;  // a helper's share of the last steps, counted through the tiles
    bool first_share = true;

    __device__ PairWalk(const ProductArgs &p, int pair) : tile(pair)
    {
        next = end = 0;
        if (p.helpers > 0 && pair >= p.pairs - p.helpers) share(p, pair - (p.pairs - p.helpers), next, end);
    }
    // Of helper h: units [begin, end) of the (steps - head) of every dealt tile.
    static __device__ void share(const ProductArgs &p, int h, long long &begin, long long &end)
    {
        const long long units = (long long)(p.tiles_m * p.tiles_n - p.whole_tiles) * (p.steps - p.head);
        begin = units * h / p.helpers;
        end = units * (h + 1) / p.helpers;
    }
    __device__ bool take(const ProductArgs &p, int pair, PairItem &item)
    {
        const int tiles = p.tiles_m * p.tiles_n;
        int index;
        if (tile < tiles) {
            index = tile;
            tile += p.pairs;
            item.first = 0;
            item.last = index < p.whole_tiles ? p.steps : p.head;
            item.slot = index < p.whole_tiles ? -1 : index - p.whole_tiles;
        } else {
            if (next >= end) return false;
            const int tail = p.steps - p.head, dealt = (int)(next / tail);
            index = p.whole_tiles + dealt;
            item.first = p.head + (int)(next % tail);
            item.last = (int)min((long long)p.steps, item.first + (end - next));
            item.slot = helper_slot(p, pair - (p.pairs - p.helpers), !first_share, item.first == p.head && item.last == p.steps, dealt);
            next += item.last - item.first;
            first_share = false;
        }
        place(p, index, item.tile_m, item.tile_n);
        return true;
    }
    // Partial sums: of the heads, of tails done by one helper, and two per helper for what it shares with others.
    static __device__ int helper_slot(const ProductArgs &p, int h, bool later, bool whole_tail, int dealt)
    {
        const int tiles = p.tiles_m * p.tiles_n - p.whole_tiles;
        return whole_tail ? tiles + dealt : 2 * tiles + 2 * h + (later ? 1 : 0);
    }
    static __host__ __device__ void place(const ProductArgs &p, int index, int &tile_m, int &tile_n)
    {
        const int group = index / (RASTER * p.tiles_n), rest = index % (RASTER * p.tiles_n);
        const int rows = p.tiles_m - group * RASTER < RASTER ? p.tiles_m - group * RASTER : RASTER;
        tile_m = group * RASTER + rest % rows;
        tile_n = rest / rows;
    }
};

// Partial sums: [slot][block of the pair][column][128 rows].
__device__ __forceinline__ long long partial_offset(const ProductArgs &p, int slot, unsigned rank)
{
    return ((long long)slot * 2 + rank) * p.tile_n * 128;
}

// The first bytes of a unit, an even number of them.
__device__ __forceinline__ void store_head(uint8_t *to, uint4 unit, int bytes)
{
    if (bytes & 8) {
        *reinterpret_cast<uint2 *>(to) = make_uint2(unit.x, unit.y);
        unit = make_uint4(unit.z, unit.w, 0u, 0u);
        to += 8;
    }
    if (bytes & 4) {
        *reinterpret_cast<unsigned *>(to) = unit.x;
        unit.x = unit.y;
        to += 4;
    }
    if (bytes & 2) *reinterpret_cast<unsigned short *>(to) = (unsigned short)unit.x;
}

// Where an epilogue warp puts 32 columns of its 32 rows.
template <class F>
__device__ __forceinline__ void finish_columns(const DenseArgs<F> &p, const CUtensorMap &c_map, const PairItem &item,
                                               unsigned rank, int quarter, int lane, int c0, const uint32_t *words,
                                               uint8_t *staging, int &buffer)
{
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(words[i]);
    if (item.slot >= 0) {
        float *out = p.partial + partial_offset(p, item.slot, rank) + (long long)c0 * 128 + quarter * 32 + lane;
#pragma unroll
        for (int i = 0; i < 32; ++i) out[i * 128] = v[i];
        return;
    }
    const int row0 = item.tile_m * PAIR_ROWS + (int)rank * 128 + quarter * 32;
    const int col0 = item.tile_n * p.tile_n + c0;
    if (p.store_by_tma) {
        // rows of 64 bytes in the copy engine's swizzle of that width: no bank conflicts
        const int parts = p.c_bf16 ? 1 : 2;
        for (int part = 0; part < parts; ++part) {
            asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PAIR_STAGING - 1) : "memory");  // the buffer's last
            __syncwarp();
            uint8_t *at = staging + buffer * PAIR_STAGING_BYTES;
            if (++buffer == PAIR_STAGING) buffer = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint4 unit;
                if (p.c_bf16)
                    unit = Unit<__nv_bfloat16>::narrow(v + 8 * i);
                else if (part == 0)
                    unit = Unit<float>::narrow(v + 4 * i);
                else
                    unit = Unit<float>::narrow(v + 16 + 4 * i);
                *reinterpret_cast<uint4 *>(at + lane * 64 + ((i ^ ((lane >> 1) & 3)) * 16)) = unit;
            }
            ptx::fence_proxy_async();
            __syncwarp();
            // rows outside C and columns from whole_n on are not written
            const int col = col0 + part * 16;
            if (elect_one()) {
                if (row0 < p.m && col < p.whole_n) tma_store_2d(&c_map, ptx::smem_addr(at), col, row0);
                ptx::bulk_commit();
            }
            __syncwarp();
        }
        if (p.whole_n < p.n) {
            // the unit that C's rows end in: the copy engine would write it whole, with zeros behind them
            const int size = p.c_bf16 ? 2 : 4, ahead = (p.whole_n - col0) * size;
            if (ahead >= 0 && ahead < 64 * parts && row0 + lane < p.m) {
                int of = buffer - parts + (ahead >> 6);
                if (of < 0) of += PAIR_STAGING;
                const uint8_t *at = staging + of * PAIR_STAGING_BYTES + lane * 64 + ((ahead & 48) ^ ((lane >> 1) & 3) * 16);
                store_head(static_cast<uint8_t *>(p.c) + ((row0 + lane) * p.c_row + p.whole_n) * size,
                           *reinterpret_cast<const uint4 *>(at), (p.n - p.whole_n) * size);
            }
        }
        return;
    }
    // any alignment, and sums with what is there: rows through shared memory, a lane per column
    float *at = reinterpret_cast<float *>(staging);
    for (int part = 0; part < 2; ++part) {  // 16 rows at a time
        __syncwarp();
        if (lane >> 4 == part) {
#pragma unroll
            for (int i = 0; i < 32; ++i) at[(lane & 15) * 32 + ((i + lane) & 31)] = v[i];
        }
        __syncwarp();
        const int rows = min(16, p.m - row0 - part * 16);
        if (col0 + lane < p.n)
            for (int r = 0; r < rows; ++r)
                store_c(p, row0 + part * 16 + r, col0 + lane, at[r * 32 + ((lane + part * 16 + r) & 31)]);
    }
}

// What an epilogue warp finds: the sums of the pair's next piece of work are in tensor memory, in turn in the first
// and the second set, once sums_full of the set is; and it has read them (or what the sets share of them) when it
// arrives on the first block's sums_read.
struct PairBlock {
    uint8_t *aligned;  // shared memory
    uint64_t *sums_full, *sums_read;
    uint32_t tmem;
    int second_set;
    bool apart;
    unsigned rank;
    int pair, warp, lane;
};

// A block of a pair: loads, scale words and products each by a warp, and epilogue(PairBlock) by the first
// EPILOGUE_WARPS.
template <bool CHUNKED, int EPILOGUE_WARPS, class Epilogue>
__device__ __forceinline__ void run_pair(const CUtensorMap &a_map, const CUtensorMap &b_map, const ProductArgs &p,
                                         const Epilogue &epilogue)
{
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t full[PAIR_STAGES], empty[PAIR_STAGES], sums_full[2], sums_read[2], words_full[2], words_empty[2],
        ended;
    __shared__ uint32_t tmem_base;
    const uint32_t base = (ptx::smem_addr(raw) + 1023u) & ~1023u;
    uint8_t *aligned = raw + (base - ptx::smem_addr(raw));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const unsigned rank = cluster_rank();
    const int pair = blockIdx.x >> 1;

    if (warp == 0) tmem_alloc(&tmem_base, 512);
    if (threadIdx.x == 32) {
        for (int s = 0; s < PAIR_STAGES; ++s) {
            ptx::mbar_init(&full[s], 1);
            ptx::mbar_init(&empty[s], 1);
        }
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(&sums_full[s], 1);
            ptx::mbar_init(&sums_read[s], 2 * EPILOGUE_WARPS);
            ptx::mbar_init(&words_full[s], 2);  // of either block
            ptx::mbar_init(&words_empty[s], 1);
        }
        ptx::mbar_init(&ended, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    fence_before_sync();
    cluster_sync();
    fence_after_sync();
    const uint32_t tmem = tmem_base;
    const int second_set = PAIR_SCALES_AT - p.tile_n;  // column of the second set of sums
    const bool apart = second_set >= p.tile_n;
    const int half_n = p.tile_n / 2;

    if (warp == EPILOGUE_WARPS) {
        // ---- loads: this block's halves of A and B
        const unsigned b_bytes = p.transpose_b ? half_n * STEP : PAIR_OPERAND_BYTES;
        PairWalk walk(p, pair);
        PairItem item;
        int stage = 0;
        unsigned phase = 0;
        bool ok = true;
        while (ok && walk.take(p, pair, item)) {
            const int m0 = item.tile_m * PAIR_ROWS + (int)rank * 128, nb = item.tile_n * p.tile_n + (int)rank * half_n;
            for (int i = item.first; i < item.last; ++i) {
                ok = warp_wait(&empty[stage], phase ^ 1, 1);
                if (!ok) break;
                if (elect_one()) {
                    const uint32_t to = base + stage * PAIR_STAGE_BYTES;
                    const uint32_t bar = cluster_addr(ptx::smem_addr(&full[stage]), 0);
                    if (rank == 0) ptx::mbar_arrive_expect_tx(&full[stage], 2 * (PAIR_OPERAND_BYTES + b_bytes));
                    if (p.transpose_a)
                        tma_load_2d(to, &a_map, m0, i * STEP, bar);
                    else
                        tma_load_2d(to, &a_map, i * STEP, m0, bar);
                    if (p.transpose_b)
                        tma_load_2d(to + PAIR_OPERAND_BYTES, &b_map, i * STEP, nb, bar);
                    else
                        tma_load_2d(to + PAIR_OPERAND_BYTES, &b_map, nb, i * STEP, bar);
                }
                __syncwarp();
                if (++stage == PAIR_STAGES) { stage = 0; phase ^= 1; }
            }
        }
        // the barriers of the last stages are arrived on from the first block: both stay until then
        for (int s = 0; ok && s < PAIR_STAGES; ++s) {
            ok = warp_wait(&empty[stage], phase ^ 1, 2);
            if (++stage == PAIR_STAGES) { stage = 0; phase ^= 1; }
        }
        if (!ok)  // a wait ran out: let the copies in flight land before the block ends
            for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    } else if (warp == EPILOGUE_WARPS + 2) {
        // ---- scale words of this block's tensor memory
        const int a_blocks = (p.m + 127) / 128, b_blocks = (p.n + 127) / 128;
        PairWalk walk(p, pair);
        PairItem item;
        int set = 0;
        unsigned phase = 0;
        bool ok = true;
        while (ok && walk.take(p, pair, item)) {
            const int block_a = item.tile_m * 2 + (int)rank;
            const int n0 = item.tile_n * p.tile_n, block_b = n0 >> 7;
            unsigned held = 0;  // scale bytes of 32 steps, one step per lane: of A's block and of up to three of B
            for (int i0 = item.first; i0 < item.last; i0 += PAIR_WORDS_STEPS) {
                const int at = (i0 - item.first) & 31;
                if (at == 0 && i0 + lane < item.last) {
                    const long long kb = i0 + lane;
                    held = 127u;
                    if (block_a < a_blocks)
                        held = p.a_scales[p.transpose_a ? kb * p.a_scale_cols + block_a
                                                        : (long long)block_a * p.a_scale_cols + kb];
#pragma unroll
                    for (int b = 0; b < 3; ++b) {
                        unsigned byte = 127u;
                        if (block_b + b < b_blocks)
                            byte = p.b_scales[p.transpose_b ? (long long)(block_b + b) * p.b_scale_cols + kb
                                                            : kb * p.b_scale_cols + block_b + b];
                        held |= byte << (8 * b + 8);
                    }
                }
                ok = warp_wait(&words_empty[set], phase ^ 1, 7);
                if (!ok) break;
                uint4 *words = reinterpret_cast<uint4 *>(aligned + PAIR_WORDS_AT + set * PAIR_WORDS_SET) + lane;
                for (int i = 0; i < PAIR_WORDS_STEPS && i0 + i < item.last; i += QUAD) {
                    // the quad's bytes of A's block and of the three of B (after the last step: not used)
                    unsigned wa = 0u, w0 = 0u, w1 = 0u, w2 = 0u;
#pragma unroll
                    for (int j = 0; j < QUAD; ++j) {
                        const unsigned bytes = __shfl_sync(0xffffffffu, held, at + i + j);
                        wa |= byte_at(bytes, 0) << 8 * j;
                        w0 |= byte_at(bytes, 8) << 8 * j;
                        w1 |= byte_at(bytes, 16) << 8 * j;
                        w2 |= byte_at(bytes, 24) << 8 * j;
                    }
                    unsigned wb[8];  // of the eight groups of 32 columns
#pragma unroll
                    for (int g = 0; g < 8; ++g) {
                        const int b = ((n0 + 32 * g) >> 7) - block_b;
                        wb[g] = b == 0 ? w0 : b == 1 ? w1 : w2;
                    }
                    words[0] = make_uint4(wa, wa, wa, wa);
                    words[32] = make_uint4(wb[0], wb[1], wb[2], wb[3]);
                    words[64] = make_uint4(wb[4], wb[5], wb[6], wb[7]);
                    words += PAIR_WORDS_BYTES / 16;
                }
                ptx::fence_proxy_async();
                __syncwarp();
                if (elect_one()) arrive_cluster(cluster_addr(ptx::smem_addr(&words_full[set]), 0));
                __syncwarp();
                if (++set == 2) { set = 0; phase ^= 1; }
            }
        }
        for (int s = 0; ok && s < 2; ++s) {  // as for the stages
            ok = warp_wait(&words_empty[set], phase ^ 1, 8);
            if (++set == 2) { set = 0; phase ^= 1; }
        }
    } else if (warp == EPILOGUE_WARPS + 1) {
        // ---- products: one thread of the first block issues them for both.  This warp's own instructions
        // bound the kernel if there are many: what can be is done once for a quad, and whether the next
        // step has been loaded is asked for while this one is issued.
        if (rank == 0) {
            const uint32_t idesc = instruction_desc(p, PAIR_ROWS, p.tile_n);
            // 32 contracted values further on: 32 bytes along a row, or 32 rows of 128 bytes
            const uint32_t step_a = (p.transpose_a ? CONTRACTED_PER_MMA * 128 : CONTRACTED_PER_MMA) >> 4;
            const uint32_t step_b = (p.transpose_b ? CONTRACTED_PER_MMA : CONTRACTED_PER_MMA * 128) >> 4;
            const uint64_t desc_a = operand_desc(base), desc_b = operand_desc(base + PAIR_OPERAND_BYTES);
            const bool wide = p.tile_n > 128;
            PairWalk walk(p, pair);
            PairItem item;
            int stage = 0, sets = 0;  // sets of sums begun
            int words_set = 0, slot = 0;
            int issued = 0;  // steps
            int ends[PAIR_SCALE_SLOTS] = {};  // where the last quads ended, the latest first
            unsigned phase = 0, words_phase = 0;
            bool ok = true, loaded = false;  // loaded: the next step is known to be
            while (ok && walk.take(p, pair, item)) {
                for (int at = 0; at < item.last - item.first; at += QUAD) {
                    const int left = item.last - item.first - at;
                    const bool words_begin = at % PAIR_WORDS_STEPS == 0;
                    const bool words_end = left <= QUAD || at % PAIR_WORDS_STEPS == PAIR_WORDS_STEPS - QUAD;
                    const bool set_begin = CHUNKED ? (at & (p.chunk - 1)) == 0 : at == 0;
                    const bool set_end = left <= QUAD || (CHUNKED && (at & (p.chunk - 1)) == p.chunk - QUAD);
                    if (words_begin) ok = warp_wait<true>(&words_full[words_set], words_phase, 9);
                    if (set_begin) {
                        // the set before this one (its shared columns), or the one before that, has been read
                        const int before = sets - (apart ? 2 : 1);
                        if (ok && before >= 0) ok = warp_wait(&sums_read[before & 1], (before >> 1) & 1, 5);
                    }
                    const int last = ends[PAIR_SCALE_SLOTS - 1] - 1;
                    if (ok && last >= 0 && last > issued - PAIR_STAGES)
                        ok = warp_wait(&empty[last % PAIR_STAGES], last / PAIR_STAGES & 1, 6);
                    if (!ok) break;
                    const uint32_t sums = tmem + ((sets & 1) ? second_set : 0);
                    const uint32_t scale_a = tmem + PAIR_SCALES_AT + slot * PAIR_SCALE_COLUMNS, scale_b = scale_a + 4;
#pragma unroll
                    for (int i = 0; i < QUAD; ++i) {
                        if (i >= left) break;
                        if (!loaded) ok = warp_wait(&full[stage], phase, 3);
                        if (!ok) break;
                        const int ahead = stage + 1 == PAIR_STAGES ? 0 : stage + 1;
                        loaded = test_arrived(&full[ahead], ahead ? phase : phase ^ 1);
                        fence_after_sync();
                        if (elect_one()) {
                            if (i == 0) {
                                const uint32_t words = base + PAIR_WORDS_AT + words_set * PAIR_WORDS_SET +
                                                       (words_begin ? 0 : PAIR_WORDS_BYTES);
                                tmem_copy_scales(scale_a, scales_desc(words));
                                tmem_copy_scales(scale_b, scales_desc(words + SCALE_BYTES));
                                if (wide) tmem_copy_scales(scale_b + 4, scales_desc(words + 2 * SCALE_BYTES));
                            }
                            const uint64_t da = desc_a + (uint32_t)(stage * (PAIR_STAGE_BYTES >> 4));
                            const uint64_t db = desc_b + (uint32_t)(stage * (PAIR_STAGE_BYTES >> 4));
#pragma unroll
                            for (int j = 0; j < STEP / CONTRACTED_PER_MMA; ++j)
                                mma_block_scaled(sums, da + j * step_a, db + j * step_b, idesc | scale_byte_desc(i), scale_a,
                                                 scale_b, i + j > 0 || !set_begin);
                            mma_commit(&empty[stage]);
                            if (i + 1 == QUAD || i + 1 == left) {
                                if (words_end) mma_commit(&words_empty[words_set]);
                                if (set_end) mma_commit(&sums_full[sets & 1]);
                            }
                        }
                        __syncwarp();
                        stage = ahead;
                        if (ahead == 0) phase ^= 1;
                    }
                    if (!ok) break;
                    issued += min(left, QUAD);
                    if (set_end) ++sets;
                    if (words_end && ++words_set == 2) { words_set = 0; words_phase ^= 1; }
                    if (++slot == PAIR_SCALE_SLOTS) slot = 0;
#pragma unroll
                    for (int q = PAIR_SCALE_SLOTS - 1; q > 0; --q) ends[q] = ends[q - 1];
                    ends[0] = issued;
                }
            }
            if (!ok) {  // products in flight end before the tensor memory is freed
                if (elect_one()) mma_commit(&ended);
                warp_wait(&ended, 0, 10);
            }
        }
    } else {
        epilogue(PairBlock{aligned, sums_full, sums_read, tmem, second_set, apart, rank, pair, warp, lane});
    }
    __syncwarp();
    fence_before_sync();
    cluster_sync();
    fence_after_sync();
    if (warp == 0) tmem_free(tmem, 512);
}

// Results to a dense matrix: a warp reads its quarter of the rows and every other group of 32 columns.
template <bool CHUNKED, class F>
__device__ __forceinline__ void dense_epilogue(const DenseArgs<F> &p, const CUtensorMap &c_map, const PairBlock &b)
{
    const int lane = b.lane, quarter = b.warp & 3, odd = b.warp >> 2;
    const uint32_t tmem = b.tmem;
    const int second_set = b.second_set;
    const bool apart = b.apart;
    uint8_t *staging = b.aligned + PAIR_STAGING_AT + b.warp * PAIR_STAGING * PAIR_STAGING_BYTES;
    const uint32_t read_bars[2] = {cluster_addr(ptx::smem_addr(&b.sums_read[0]), 0),
                                   cluster_addr(ptx::smem_addr(&b.sums_read[1]), 0)};
    const int groups = p.tile_n / 32;
    PairWalk walk(p, b.pair);
    PairItem item;
    int sets = 0, buffer = 0;
    bool ok = true;
    float total[CHUNKED ? 128 : 1];
    while (ok && walk.take(p, b.pair, item)) {
        const int parts = CHUNKED ? (item.last - item.first + p.chunk - 1) / p.chunk : 1;
        if constexpr (CHUNKED) {
#pragma unroll
            for (int i = 0; i < 128; ++i) total[i] = 0.0f;
        }
        for (int part = 0; part < parts; ++part, ++sets) {
            ok = warp_wait(&b.sums_full[sets & 1], (sets >> 1) & 1, 4);
            if (!ok) break;
            fence_after_sync();
            const uint32_t from = tmem + ((uint32_t)(quarter * 32) << 16) + ((sets & 1) ? second_set : 0);
            const bool down = !(sets & 1);  // the columns shared with the other set come first
            const uint32_t read_bar = down ? read_bars[0] : read_bars[1];
            if constexpr (CHUNKED) {
#pragma unroll
                for (int t = 0; t < PAIR_MAX_N / 64; ++t) {
                    // the total's registers need fixed indexes: both orders are written out
#pragma unroll
                    for (int order = 0; order < 2; ++order) {
                        const int u = order ? PAIR_MAX_N / 64 - 1 - t : t, g = 2 * u + odd;
                        if (down == (order == 1) && g < groups) {
                            uint32_t r[32];
                            tmem_load32(from + g * 32, r);
                            tmem_wait(r);
#pragma unroll
                            for (int i = 0; i < 32; ++i) total[u * 32 + i] += __uint_as_float(r[i]);
                        }
                    }
                    if (!apart && t == 0) {
                        fence_before_sync();
                        if (lane == 0) arrive_remote(read_bar);
                        __syncwarp();
                    }
                }
            } else {
                // the next group is on its way while one is rounded and stored
                const int own = (groups - odd + 1) / 2;  // of this warp: odd, odd + 2, ...
                const auto group = [&](int t) { return 2 * (down ? own - 1 - t : t) + odd; };
                uint32_t r[2][32];
                tmem_load32(from + group(0) * 32, r[0]);
#pragma unroll
                for (int t = 0; t < PAIR_MAX_N / 64; ++t) {
                    if (t >= own) break;
                    tmem_wait(r[t & 1]);
                    if (!apart && t == 0) {
                        fence_before_sync();
                        if (lane == 0) arrive_remote(read_bar);
                        __syncwarp();
                    }
                    if (t + 1 < own) tmem_load32(from + group(t + 1) * 32, r[~t & 1]);
                    finish_columns(p, c_map, item, b.rank, quarter, lane, group(t) * 32, r[t & 1], staging, buffer);
                }
            }
            if (apart) {
                fence_before_sync();
                if (lane == 0) arrive_remote(read_bar);
                __syncwarp();
            }
        }
        if constexpr (CHUNKED) {
            if (ok) {
#pragma unroll
                for (int u = 0; u < PAIR_MAX_N / 64; ++u)
                    if (2 * u + odd < groups)
                        finish_columns(p, c_map, item, b.rank, quarter, lane, (2 * u + odd) * 32,
                                       reinterpret_cast<const uint32_t *>(total + u * 32),
                                       staging, buffer);
            }
        }
    }
    ptx::bulk_wait_all();
}

template <bool CHUNKED, class F>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(pair_threads(PAIR_EPILOGUE_WARPS), 1)
    pair_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
                const __grid_constant__ CUtensorMap c_map, const __grid_constant__ DenseArgs<F> p)
{
    run_pair<CHUNKED, PAIR_EPILOGUE_WARPS>(a_map, b_map, p, [&](const PairBlock &b) { dense_epilogue<CHUNKED>(p, c_map, b); });
}

// Tiles whose steps were dealt out: their partial sums in the order of the steps.  A block joins 32
// columns of one block's 128 rows.
template <class F> __global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ DenseArgs<F> p)
{
    __shared__ float shared[128][33];
    const int groups = p.tile_n / 32;
    const int group = blockIdx.x % groups;
    const unsigned rank = blockIdx.x / groups % 2;
    const int tile = blockIdx.x / (2 * groups);  // among those dealt out
    const int row = threadIdx.x & 127, side = threadIdx.x >> 7;
    const long long at = (long long)(group * 32 + side * 16) * 128 + row;
    float v[16];
    const float *in = p.partial + partial_offset(p, tile, rank) + at;
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = in[i * 128];
    const int tail = p.steps - p.head;
    const long long from = (long long)tile * tail, to = from + tail;
    const long long units = (long long)(p.tiles_m * p.tiles_n - p.whole_tiles) * tail;
    int h = (int)(from * p.helpers / units);  // the helper that has unit `from`, or the one before it
    for (; h < p.helpers; ++h) {
        long long begin, end;
        PairWalk::share(p, h, begin, end);
        if (begin >= to) break;
        if (end <= from || begin == end) continue;
        const int slot = PairWalk::helper_slot(p, h, begin / tail != tile, begin <= from && end >= to, tile);
        in = p.partial + partial_offset(p, slot, rank) + at;
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] += in[i * 128];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) shared[row][side * 16 + i] = v[i];
    __syncthreads();
    int tile_m, tile_n;
    PairWalk::place(p, p.whole_tiles + tile, tile_m, tile_n);
    const long long row0 = (long long)tile_m * PAIR_ROWS + rank * 128;
    const long long col = (long long)tile_n * p.tile_n + group * 32 + (threadIdx.x & 31);
    if (col < p.n)
        for (int r = threadIdx.x >> 5; r < 128 && row0 + r < p.m; r += 8) {
            float v = shared[r][threadIdx.x & 31];
            if constexpr (!F::NOTHING) v = p.finish.value(v, row0 + r, (int)col);
            store_c(p, row0 + r, col, v);
        }
}

// ------------------------------------------------------------------------------------------ a few rows

// Up to four rows of A (tokens) against the rows of B^T (a weight's outputs), both contracted along their
// rows: bound by reading the weight once.  The tokens wait in shared memory in f16, which holds every code;
// a warp takes two outputs, 16 codes per lane and step, all within one block, and multiplies in fp32.  The
// tensor cores' path takes 9.3 us for one token through 3584x896, this one 3.6 us; through 8192x8192 it takes
// 20 us (3.3 TB/s: bound by the conversions and additions, about four instructions for a weight).
constexpr int FEW_MAX = 4;
constexpr int FEW_THREADS = 256;
constexpr int FEW_OUTPUTS = 2;  // of a warp
constexpr int FEW_SMEM = 96 * 1024;

struct FewArgs {
    const uint8_t *tokens, *token_scales, *weight, *weight_scales;
    long long token_stride, weight_stride;
    int outputs, k, steps;
    void *c;
    long long c_token, c_output;  // strides of C
    int c_bf16, accumulate, tokens_first;  // tokens_first: they are C's rows
};
template <class F> struct FinishedFew : FewArgs {
    F finish;
};

template <class F> __device__ __forceinline__ void store_few(const FinishedFew<F> &p, int token, int output, float v)
{
    if constexpr (!F::NOTHING) v = p.finish.value(v, p.tokens_first ? token : output, p.tokens_first ? output : token);
    const long long at = token * p.c_token + output * p.c_output;
    if (p.c_bf16) {
        __nv_bfloat16 *c = static_cast<__nv_bfloat16 *>(p.c) + at;
        *c = __float2bfloat16_rn(p.accumulate ? v + __bfloat162float(*c) : v);
    } else {
        float *c = static_cast<float *>(p.c) + at;
        *c = p.accumulate ? v + *c : v;
    }
}

// v times the product of two scales, whose exponents are added first: two halves of the sum are always
// exponents of fp32, where the scales' product itself might not be.
__device__ __forceinline__ float scaled(float v, unsigned a, unsigned b)
{
    if (a == 255u || b == 255u) return __uint_as_float(0x7fc00000u);
    const int e = (int)(a + b) - 254, half = e >> 1;
    return v * __uint_as_float((unsigned)(half + 127) << 23) * __uint_as_float((unsigned)(e - half + 127) << 23);
}

// The products of 16 codes of each output and each token, added to the sums.
template <int M>
__device__ __forceinline__ void few_products(const uint4 *codes, const unsigned *scale, unsigned token_scale,
                                             const __half *tokens, int padded, int k, float (*sums)[M])
{
                float part[FEW_OUTPUTS][M] = {};
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    float w[FEW_OUTPUTS][8];
#pragma unroll
                    for (int r = 0; r < FEW_OUTPUTS; ++r) {
                        decode4(q ? codes[r].z : codes[r].x, 1.0f, w[r]);
                        decode4(q ? codes[r].w : codes[r].y, 1.0f, w[r] + 4);
                    }
#pragma unroll
                    for (int t = 0; t < M; ++t) {
                        const uint4 raw = *reinterpret_cast<const uint4 *>(tokens + t * padded + q * (padded / 2) + k / 2);
                        const unsigned words[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&words[i]));
#pragma unroll
                            for (int r = 0; r < FEW_OUTPUTS; ++r) {
                                part[r][t] = fmaf(w[r][2 * i], v.x, part[r][t]);
                                part[r][t] = fmaf(w[r][2 * i + 1], v.y, part[r][t]);
                            }
                        }
                    }
                }
#pragma unroll
                for (int r = 0; r < FEW_OUTPUTS; ++r)
#pragma unroll
                    for (int t = 0; t < M; ++t) sums[r][t] += scaled(part[r][t], scale[r], token_scale);
}

// The tokens in shared memory, [M][2][padded / 16][8]: the halves of every 16 codes apart, so that a warp's loads do not
// conflict; and their scale bytes.
template <int M> __device__ __forceinline__ void few_tokens(const FewArgs &p, __half *tokens, uint8_t *token_scales)
{
    const int padded = p.steps * STEP;
    for (int i = threadIdx.x; i < M * padded / 4; i += FEW_THREADS) {
        const int t = i * 4 / padded, k = i * 4 % padded;
        unsigned w = 0u;
        if (k < p.k) {
            w = *reinterpret_cast<const unsigned *>(p.tokens + t * p.token_stride + k);
            if (k + 4 > p.k) w &= 0xffffffffu >> 8 * (k + 4 - p.k);
        }
        const __half2_raw lo = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w & 0xffffu), __NV_E4M3);
        const __half2_raw hi = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> 16), __NV_E4M3);
        *reinterpret_cast<uint2 *>(tokens + t * padded + (k >> 3 & 1) * (padded / 2) + (k >> 4) * 8 + (k & 7)) =
            make_uint2(lo.x | (unsigned)lo.y << 16, hi.x | (unsigned)hi.y << 16);
    }
    for (int i = threadIdx.x; i < p.steps; i += FEW_THREADS) token_scales[i] = p.token_scales[i];  // one block of rows
}

// The products of outputs first, first + 1, ... with every token, on all lanes of the warp.
template <int M>
__device__ __forceinline__ void few_sums(const FewArgs &p, const __half *tokens, const uint8_t *token_scales, int first, int lane,
                                         float (*sums)[M])
{
    const int padded = p.steps * STEP;
    const uint8_t *rows[FEW_OUTPUTS], *scales[FEW_OUTPUTS];
#pragma unroll
    for (int r = 0; r < FEW_OUTPUTS; ++r) {
        const int row = min(first + r, p.outputs - 1);
        rows[r] = p.weight + row * p.weight_stride;
        scales[r] = p.weight_scales + (long long)(row / PACK_BLOCK) * p.steps;
    }
    const int whole = p.k / 512 * 512;
#pragma unroll(M == 1 ? 4 : 2)
    for (int k = lane * 16; k < whole; k += 512) {
        uint4 codes[FEW_OUTPUTS];
        unsigned scale[FEW_OUTPUTS];
#pragma unroll
        for (int r = 0; r < FEW_OUTPUTS; ++r) {
            codes[r] = __ldcs(reinterpret_cast<const uint4 *>(rows[r] + k));
            scale[r] = scales[r][k / STEP];
        }
        few_products<M>(codes, scale, token_scales[k / STEP], tokens, padded, k, sums);
    }
    if (const int k = whole + lane * 16; k < p.k) {
        uint4 codes[FEW_OUTPUTS];
        unsigned scale[FEW_OUTPUTS];
#pragma unroll
        for (int r = 0; r < FEW_OUTPUTS; ++r) {
            codes[r] = __ldcs(reinterpret_cast<const uint4 *>(rows[r] + k));
            scale[r] = scales[r][k / STEP];
        }
        if (k + 16 > p.k) {  // rows of codes are padded to 16 bytes with anything
            const int n = p.k - k;
#pragma unroll
            for (int r = 0; r < FEW_OUTPUTS; ++r) {
                codes[r].x &= n >= 4 ? ~0u : (1u << 8 * n) - 1u;
                codes[r].y &= n >= 8 ? ~0u : n > 4 ? (1u << 8 * (n - 4)) - 1u : 0u;
                codes[r].z &= n >= 12 ? ~0u : n > 8 ? (1u << 8 * (n - 8)) - 1u : 0u;
                codes[r].w &= n > 12 ? (1u << 8 * (n - 12)) - 1u : 0u;
            }
        }
        few_products<M>(codes, scale, token_scales[k / STEP], tokens, padded, k, sums);
    }
#pragma unroll
    for (int r = 0; r < FEW_OUTPUTS; ++r)
#pragma unroll
        for (int t = 0; t < M; ++t)
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sums[r][t] += __shfl_xor_sync(0xffffffffu, sums[r][t], o);
}

template <int M, class F> __global__ void __launch_bounds__(FEW_THREADS) few_kernel(const __grid_constant__ FinishedFew<F> p)
{
    extern __shared__ __align__(16) __half tokens[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint8_t *token_scales = reinterpret_cast<uint8_t *>(tokens + M * p.steps * STEP);
    few_tokens<M>(p, tokens, token_scales);
    __syncthreads();

    const int step = gridDim.x * (FEW_THREADS / 32) * FEW_OUTPUTS;
    for (int first = (blockIdx.x * (FEW_THREADS / 32) + warp) * FEW_OUTPUTS; first < p.outputs; first += step) {
        float sums[FEW_OUTPUTS][M] = {};
        few_sums<M>(p, tokens, token_scales, first, lane, sums);
#pragma unroll
        for (int r = 0; r < FEW_OUTPUTS; ++r)
#pragma unroll
            for (int t = 0; t < M; ++t)
                if (lane == 0 && first + r < p.outputs) store_few(p, t, first + r, sums[r][t]);
    }
}

// ------------------------------------------------------------------------------------------ host

// Boxes of `rows` x 128 codes in the 128-byte swizzle; codes outside the matrix read as zero.
inline bool operand_map(CUtensorMap *map, const dipaco_packed *x, int rows)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)x->cols, (cuuint64_t)x->rows};
    const cuuint64_t strides[1] = {(cuuint64_t)x->stride};
    const cuuint32_t box[2] = {128, (cuuint32_t)rows}, steps[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, x->codes, dims, strides, box, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Boxes of 32 rows of 64 bytes of results, in the swizzle of that width.  n is a multiple of 16 bytes.
inline bool result_map(CUtensorMap *map, void *c, int64_t m, int64_t n, int64_t stride, int dtype)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const bool bf16 = dtype == DIPACO_BF16;
    const cuuint64_t dims[2] = {(cuuint64_t)n, (cuuint64_t)m};
    const cuuint64_t strides[1] = {(cuuint64_t)(stride * dense_size(dtype))};
    const cuuint32_t box[2] = {bf16 ? 32u : 16u, 32}, steps[2] = {1, 1};
    return encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, c, dims, strides,
                  box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
                  CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int PAIRS = 74;  // pairs of the 148 SMs

// How a product is cut up: the columns of a tile, from 64 to 256, and whether the last round's steps are dealt
// out, by an estimate in clocks of one SM.  Fewer columns than 256 pay where they divide the result better
// (224 for multiples of 896) or keep the sets of sums apart.
struct PairPlan {
    int tile_n = 256, tiles_m = 0, tiles_n = 0, pairs = 0, whole_tiles = 0, head = 0, helpers = 0;
    int64_t workspace = 0;
};

inline PairPlan plan_pairs(int64_t m, int64_t n, int64_t steps)
{
    PairPlan best;
    double best_time = 0.0;
    for (int tile_n = 256; tile_n >= 64; tile_n -= 32) {
        PairPlan plan;
        plan.tile_n = tile_n;
        plan.tiles_m = (int)ceil_div(m, PAIR_ROWS);
        plan.tiles_n = (int)ceil_div(n, tile_n);
        const int64_t tiles = (int64_t)plan.tiles_m * plan.tiles_n;
        plan.pairs = (int)std::min<int64_t>(PAIRS, tiles);
        plan.whole_tiles = (int)tiles;
        // a step is bound by the products (2 clocks per column) or by its operands' way from L2
        const double step = std::max(2.0 * tile_n, 64.0 * 4 + tile_n * 1.0);
        const double gap = tile_n > PAIR_SCALES_AT / 2 ? 500.0 : 0.0;  // sets of sums that overlap
        double time = (double)ceil_div(tiles, PAIRS) * (steps * step + gap);
        // a last, unfilled round with its steps dealt out to all pairs, and a second launch that joins sums
        const int64_t dealt = tiles % PAIRS, helpers = PAIRS - dealt, head = ceil_div(dealt * steps, PAIRS);
        if (dealt > 0 && head < steps) {
            const double join = 8000.0 + 3.0 * dealt * tile_n * 256 * 4 / 4000.0;
            const double shared = (double)(tiles / PAIRS) * (steps * step + gap) + head * step + 2 * gap + join;
            if (shared < time) {
                time = shared;
                plan.pairs = PAIRS;
                plan.whole_tiles = (int)(tiles - dealt);
                plan.head = (int)head;
                plan.helpers = (int)helpers;
                plan.workspace = (2 * dealt + 2 * helpers) * PAIR_ROWS * tile_n * (int64_t)sizeof(float);
            }
        }
        if (best_time == 0.0 || time < best_time) {
            best_time = time;
            best = plan;
        }
    }
    return best;
}

// Tokens of few_kernel: the shorter side, where both operands are contracted along their rows.
inline bool are_few(int64_t m, int64_t n, int64_t k, bool transpose_a, bool transpose_b)
{
    // more than two tokens only through smaller weights: four through 3584x896 take 5.5 us here and 8.7 us on
    // the tensor cores, four through 8192x8192 41 us and 29 us
    const int64_t few = std::min(m, n);
    return (few <= 2 || (few <= FEW_MAX && std::max(m, n) * k <= (int64_t)1 << 24)) && !transpose_a && transpose_b && few * ceil_div(k, STEP) * STEP * 2 + ceil_div(k, STEP) <= FEW_SMEM;
}

// Arguments for few tokens; the rest is for those who store.
inline FewArgs few_args(const dipaco_packed *tokens, const dipaco_packed *weight)
{
    FewArgs p = {};
    p.tokens = static_cast<const uint8_t *>(tokens->codes);
    p.token_scales = static_cast<const uint8_t *>(tokens->scales);
    p.weight = static_cast<const uint8_t *>(weight->codes);
    p.weight_scales = static_cast<const uint8_t *>(weight->scales);
    p.token_stride = tokens->stride;
    p.weight_stride = weight->stride;
    p.outputs = (int)weight->rows;
    p.k = (int)weight->cols;
    p.steps = (int)ceil_div(weight->cols, STEP);
    return p;
}
inline int few_smem(const FewArgs &p, int64_t tokens) { return (int)tokens * p.steps * STEP * 2 + p.steps; }

template <class F>
int launch_few(const dipaco_packed *a, const dipaco_packed *b, void *c, int64_t c_stride, int dtype, bool accumulate,
               const F &finish, cudaStream_t stream)
{
    const bool tokens_first = a->rows <= b->rows;
    const dipaco_packed *tokens = tokens_first ? a : b, *weight = tokens_first ? b : a;
    FinishedFew<F> p = {few_args(tokens, weight), finish};
    p.c = c;
    p.c_token = tokens_first ? c_stride : 1;
    p.c_output = tokens_first ? 1 : c_stride;
    p.c_bf16 = dtype == DIPACO_BF16;
    p.accumulate = accumulate;
    p.tokens_first = tokens_first;
    const int m = (int)tokens->rows;
    const int smem = few_smem(p, m);
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(p.outputs, FEW_THREADS / 32 * FEW_OUTPUTS), 148 * 2);
    const auto kernel = m == 1 ? few_kernel<1, F> : m == 2 ? few_kernel<2, F> : m == 3 ? few_kernel<3, F> : few_kernel<4, F>;
    // always the largest there can be: threads that launch different sizes share the attribute
    if (smem > 48 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, FEW_SMEM) != cudaSuccess)
        return launch_status();
    kernel<<<grid, FEW_THREADS, smem, stream>>>(p);
    return launch_status();
}

// The kernels of a product that stores to a dense matrix, whose sums are taken in one go or in chunks.
template <class F> struct DenseKernels {
    using Kernel = void (*)(CUtensorMap, CUtensorMap, CUtensorMap, DenseArgs<F>);
    Kernel whole[2], chunked[2];  // [1]: where the copy engine stores the results
    int threads;
    bool whole_f32;  // results in fp32 take the first too where there is one chunk
};

inline void set_operands(ProductArgs &p, const dipaco_packed *a, const dipaco_packed *b, bool transpose_a, bool transpose_b)
{
    p.a_scales = static_cast<const uint8_t *>(a->scales);
    p.b_scales = static_cast<const uint8_t *>(b->scales);
    p.a_scale_cols = (int)ceil_div(a->cols, PACK_BLOCK);
    p.b_scale_cols = (int)ceil_div(b->cols, PACK_BLOCK);
    p.transpose_a = transpose_a;
    p.transpose_b = transpose_b;
    p.m = (int)(transpose_a ? a->cols : a->rows);
    p.n = (int)(transpose_b ? b->rows : b->cols);
    p.steps = (int)ceil_div(transpose_a ? a->rows : a->cols, STEP);
}

// The product of checked operands with something to contract, finished and stored to C.
template <class F>
int launch_product(const dipaco_packed *a, const dipaco_packed *b, bool transpose_a, bool transpose_b, void *c,
                   int64_t c_stride, int dtype, bool accumulate, const F &finish, const DenseKernels<F> &kernels,
                   void *workspace, cudaStream_t stream)
{
    DenseArgs<F> p = {};
    set_operands(p, a, b, transpose_a, transpose_b);
    p.finish = finish;
    const int64_t m = p.m, n = p.n;
    p.c = c;
    p.c_row = c_stride;
    p.c_bf16 = dtype == DIPACO_BF16;
    p.accumulate = accumulate;

    if (ceil_div(m, PAIR_ROWS) * ceil_div(n, 64) > INT32_MAX) return DIPACO_ELIMIT;
    const PairPlan plan = plan_pairs(m, n, p.steps);
    p.tile_n = plan.tile_n;
    p.tiles_m = plan.tiles_m;
    p.tiles_n = plan.tiles_n;
    p.pairs = plan.pairs;
    p.whole_tiles = plan.whole_tiles;
    p.head = plan.head;
    p.helpers = plan.helpers;
    p.partial = static_cast<float *>(workspace);
    CUtensorMap a_map, b_map, c_map = {};
    if (!operand_map(&a_map, a, 128) || !operand_map(&b_map, b, transpose_b ? plan.tile_n / 2 : 128)) return DIPACO_ECUDA;
    p.whole_n = (int)(n / (16 / dense_size(dtype)) * (16 / dense_size(dtype)));
    p.store_by_tma = !accumulate && p.whole_n > 0 && rows_aligned16(c, c_stride, m, dense_size(dtype));
    if (p.store_by_tma && !result_map(&c_map, c, m, p.whole_n, m == 1 ? ceil_div(n, 8) * 8 : c_stride, dtype)) return DIPACO_ECUDA;
    p.chunk = p.c_bf16 ? CHUNK_BF16 : CHUNK_F32;
    const bool chunked = (!p.c_bf16 && !kernels.whole_f32) || p.steps > p.chunk;
    const auto kernel = (chunked ? kernels.chunked : kernels.whole)[p.store_by_tma != 0];
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PAIR_SMEM) != cudaSuccess) return launch_status();
    kernel<<<2 * plan.pairs, kernels.threads, PAIR_SMEM, stream>>>(a_map, b_map, c_map, p);
    if (const int rc = launch_status()) return rc;
    const int64_t dealt = (int64_t)plan.tiles_m * plan.tiles_n - plan.whole_tiles;
    if (dealt > 0)
        join_kernel<F><<<(unsigned)(dealt * 2 * (plan.tile_n / 32)), 256, 0, stream>>>(p);
    return launch_status();
}

} // namespace
} // namespace dipaco
