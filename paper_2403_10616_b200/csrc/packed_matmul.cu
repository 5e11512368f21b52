// Product of two packed matrices (see include/dipaco.h): C = op(A) op(B), codes e4m3, one scale per
// block of 128 x 128, fp32 sums.
//
// The contraction is walked in steps of 128, one block of A against one of B, on the tensor cores'
// block-scaled 8-bit form (tcgen05.mma kind::mxf8f6f4).  That form takes one scale per row and 32
// contracted values; here all of them are equal over a block, so the scale operands in tensor memory
// are constant words and a block may be contracted along either side: the operand's major-ness in the
// instruction descriptor is all that differs between the forward product and the two gradients.
#include "inner_common.cuh"

#include <cuda.h>

#include <cmath>

using namespace dipaco;

namespace {

static __device__ int g_product_error;  // set by a bounded wait that ran out

// ------------------------------------------------------------------------------------------ PTX

__device__ __forceinline__ bool elect_one()
{
    unsigned ok;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok));
    return ok != 0;
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint64_t *bar)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
            dst),
        "l"(map), "r"(x), "r"(y), "r"(ptx::smem_addr(bar))
        : "memory");
}
__device__ __forceinline__ void tmem_alloc(uint32_t *result, int columns)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(ptx::smem_addr(result)),
                 "r"(columns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t address, int columns)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(address), "r"(columns));
}
// 32 lanes x 16 bytes of shared memory to four columns of each 32-lane quarter of tensor memory
__device__ __forceinline__ void tmem_copy_scales(uint32_t address, uint64_t desc)
{
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(address), "l"(desc) : "memory");
}
__device__ __forceinline__ void mma_block_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t scale_a,
                                                 uint32_t scale_b, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(scale_a), "r"(scale_b), "r"((unsigned)add)
        : "memory");
}
__device__ __forceinline__ void mma_commit(uint64_t *bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
                     ptx::smem_addr(bar))
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
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
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

// ------------------------------------------------------------------------------------------ kernel

constexpr int TILE = 128;                     // of C and of the contraction: one block
constexpr int TILE_BYTES = TILE * TILE;       // of codes
constexpr int SCALE_BYTES = 512;              // 32 lanes x 16 bytes
constexpr int STAGES = 3;                     // two resident blocks per SM
constexpr int STAGE_BYTES = 2 * TILE_BYTES + 2 * SCALE_BYTES;
constexpr int PRODUCT_SMEM = STAGES * STAGE_BYTES + 1024;
constexpr int PRODUCT_THREADS = 192;          // four epilogue warps, load warp, issuing warp
constexpr int TMEM_COLUMNS = 256;             // 128 of sums, 8 of scales per stage
constexpr int CONTRACTED_PER_MMA = 32;
// The tensor cores truncate when they add to an fp32 sum, which drifts by about 1.2e-8 of the sum for
// every 32 contracted values (measured: 2.4e-5 over 65501).  Sums are therefore taken out of tensor
// memory every CHUNK steps, 2048 values, and added up in registers.
constexpr int CHUNK = 16;

struct ProductArgs {
    const uint8_t *a_scales, *b_scales;
    int a_scale_cols, b_scale_cols;
    int transpose_a, transpose_b;  // A is stored [K, M]; B is stored [N, K]
    int m, n, k;
    void *c;
    long long c_stride;
    int c_bf16, accumulate;
};

__global__ void __launch_bounds__(PRODUCT_THREADS)
    product_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map, ProductArgs p)
{
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t full[STAGES], empty[STAGES], done, drained;
    __shared__ uint32_t tmem_base;
    const uint32_t base = (ptx::smem_addr(raw) + 1023u) & ~1023u;
    uint8_t *aligned = raw + (base - ptx::smem_addr(raw));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tiles_n = (p.n + TILE - 1) / TILE;
    const int tile_m = blockIdx.x / tiles_n, tile_n = blockIdx.x % tiles_n;
    const int steps = (p.k + TILE - 1) / TILE;

    if (warp == 5) tmem_alloc(&tmem_base, TMEM_COLUMNS);
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            ptx::mbar_init(&full[s], 1);
            ptx::mbar_init(&empty[s], 1);
        }
        ptx::mbar_init(&done, 1);
        ptx::mbar_init(&drained, 128);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t sums = tmem_base, scale_columns = tmem_base + TILE;

    if (warp == 4) {
        int issued = 0;
        bool ok = true;
        unsigned held_a = 0, held_b = 0;  // scale bytes of 32 steps, one per lane
        for (int i = 0; i < steps; ++i) {
            if (i % 32 == 0 && i + lane < steps) {
                const int kb = i + lane;
                held_a = p.a_scales[p.transpose_a ? (long long)kb * p.a_scale_cols + tile_m
                                                  : (long long)tile_m * p.a_scale_cols + kb];
                held_b = p.b_scales[p.transpose_b ? (long long)tile_n * p.b_scale_cols + kb
                                                  : (long long)kb * p.b_scale_cols + tile_n];
            }
            const int s = i % STAGES;
            ok = bounded_wait(&empty[s], ((i / STAGES) & 1) ^ 1, &g_product_error, 1);
            if (!ok) break;
            const unsigned wa = __shfl_sync(0xffffffffu, held_a, i % 32) * 0x01010101u;
            const unsigned wb = __shfl_sync(0xffffffffu, held_b, i % 32) * 0x01010101u;
            uint8_t *stage = aligned + s * STAGE_BYTES;
            uint4 *words = reinterpret_cast<uint4 *>(stage + 2 * TILE_BYTES);
            words[lane] = make_uint4(wa, wa, wa, wa);
            words[32 + lane] = make_uint4(wb, wb, wb, wb);
            ptx::fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                ptx::mbar_arrive_expect_tx(&full[s], 2 * TILE_BYTES);
                const uint32_t at = base + s * STAGE_BYTES;
                if (p.transpose_a)
                    tma_load_2d(at, &a_map, tile_m * TILE, i * TILE, &full[s]);
                else
                    tma_load_2d(at, &a_map, i * TILE, tile_m * TILE, &full[s]);
                if (p.transpose_b)
                    tma_load_2d(at + TILE_BYTES, &b_map, i * TILE, tile_n * TILE, &full[s]);
                else
                    tma_load_2d(at + TILE_BYTES, &b_map, tile_n * TILE, i * TILE, &full[s]);
            }
            ++issued;
        }
        if (!ok)  // copies in flight end before the block does
            for (int i = max(0, issued - STAGES); i < issued; ++i)
                bounded_wait(&full[i % STAGES], (i / STAGES) & 1, &g_product_error, 2);
    } else if (warp == 5) {
        // bits: A and B e4m3 (0), A and B major-ness, N/8, e8m0 scales, M/16
        const uint32_t idesc = (uint32_t)(p.transpose_a ? 1 : 0) << 15 | (uint32_t)(p.transpose_b ? 0 : 1) << 16 |
                               (TILE >> 3) << 17 | 1u << 23 | (TILE >> 4) << 24;
        // 32 contracted values further on: 32 bytes along a row, or 32 rows of 128 bytes
        const uint32_t step_a = (p.transpose_a ? CONTRACTED_PER_MMA * 128 : CONTRACTED_PER_MMA) >> 4;
        const uint32_t step_b = (p.transpose_b ? CONTRACTED_PER_MMA : CONTRACTED_PER_MMA * 128) >> 4;
        bool ok = true;
        for (int i = 0; i < steps; ++i) {
            const int s = i % STAGES;
            ok = bounded_wait(&full[s], (i / STAGES) & 1, &g_product_error, 3);
            if (!ok) break;
            if (i > 0 && i % CHUNK == 0) {
                ok = bounded_wait(&drained, (i / CHUNK - 1) & 1, &g_product_error, 5);
                if (!ok) break;
            }
            fence_after_sync();
            if (elect_one()) {
                const uint32_t at = base + s * STAGE_BYTES;
                const uint32_t scale_a = scale_columns + s * 8, scale_b = scale_a + 4;
                tmem_copy_scales(scale_a, scales_desc(at + 2 * TILE_BYTES));
                tmem_copy_scales(scale_b, scales_desc(at + 2 * TILE_BYTES + SCALE_BYTES));
                const uint64_t da = operand_desc(at), db = operand_desc(at + TILE_BYTES);
#pragma unroll
                for (int j = 0; j < TILE / CONTRACTED_PER_MMA; ++j)
                    mma_block_scaled(sums, da + j * step_a, db + j * step_b, idesc, scale_a, scale_b, i % CHUNK + j > 0);
                mma_commit(&empty[s]);
                if (i + 1 == steps || i % CHUNK == CHUNK - 1) mma_commit(&done);
            }
            __syncwarp();
        }
    } else {
        float sum[TILE];
#pragma unroll
        for (int i = 0; i < TILE; ++i) sum[i] = 0.0f;
        bool ok = true;
        for (int chunk = 0; chunk * CHUNK < steps; ++chunk) {
            ok = bounded_wait(&done, chunk & 1, &g_product_error, 4);
            if (!ok) break;
            fence_after_sync();
#pragma unroll
            for (int c0 = 0; c0 < TILE; c0 += 32) {
                uint32_t r[32];
                tmem_load32(sums + ((uint32_t)(warp * 32) << 16) + c0, r);
#pragma unroll
                for (int i = 0; i < 32; ++i) sum[c0 + i] += __uint_as_float(r[i]);
            }
            fence_before_sync();
            ptx::mbar_arrive(&drained);
        }
        const long long row = (long long)tile_m * TILE + warp * 32 + lane;
        if (ok && row < p.m) {
#pragma unroll
            for (int i = 0; i < TILE; ++i) {
                const int col = tile_n * TILE + i;
                if (col < p.n) {
                    float v = sum[i];
                    if (p.c_bf16) {
                        __nv_bfloat16 *c = static_cast<__nv_bfloat16 *>(p.c) + row * p.c_stride + col;
                        if (p.accumulate) v += __bfloat162float(*c);
                        *c = __float2bfloat16_rn(v);
                    } else {
                        float *c = static_cast<float *>(p.c) + row * p.c_stride + col;
                        if (p.accumulate) v += *c;
                        *c = v;
                    }
                }
            }
        }
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    if (warp == 5) tmem_free(tmem_base, TMEM_COLUMNS);
}

// ------------------------------------------------------------------------------------------ host

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                 const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
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

// Boxes of 128 x 128 codes in the 128-byte swizzle; codes outside the matrix read as zero.
bool operand_map(CUtensorMap *map, const dipaco_packed *x)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)x->cols, (cuuint64_t)x->rows};
    const cuuint64_t strides[1] = {(cuuint64_t)x->stride};
    const cuuint32_t box[2] = {TILE, TILE}, steps[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, x->codes, dims, strides, box, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

} // namespace

extern "C" {

int dipaco_packed_matmul_workspace(int64_t m, int64_t n, int64_t k, int64_t *bytes)
{
    if (!bytes || k < 0) return DIPACO_EINVAL;
    if (const int rc = check_extents(m, n)) return rc;
    if (k > MAX_EXTENT) return DIPACO_ELIMIT;
    *bytes = 0;
    return DIPACO_OK;
}

int dipaco_packed_matmul(const dipaco_packed *a, const dipaco_packed *b, int32_t transpose_a, int32_t transpose_b,
                         void *c, int64_t c_stride, int32_t dtype, int32_t accumulate, void *workspace,
                         int64_t workspace_bytes, int32_t device, void *cuda_stream)
{
    if (!a || !b || !is_dense_dtype(dtype) || device < 0) return DIPACO_EINVAL;
    const int64_t m = transpose_a ? a->cols : a->rows, k = transpose_a ? a->rows : a->cols;
    const int64_t n = transpose_b ? b->rows : b->cols;
    if ((transpose_b ? b->cols : b->rows) != k) return DIPACO_EINVAL;
    int64_t need = 0;
    if (const int rc = dipaco_packed_matmul_workspace(m, n, k, &need)) return rc;
    if (!packed_ok(a, a->rows, a->cols) || !packed_ok(b, b->rows, b->cols)) return DIPACO_EINVAL;
    if (!dense_ok(c, c_stride, m, n, dtype)) return DIPACO_EINVAL;
    if (need > 0 && (!workspace || (uintptr_t)workspace % 16 != 0 || workspace_bytes < need)) return DIPACO_EINVAL;
    if (m == 0 || n == 0 || (k == 0 && accumulate)) return DIPACO_OK;

    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (k == 0) {  // a sum over nothing
        const size_t size = dense_size(dtype);
        const size_t pitch = m == 1 ? n * size : c_stride * size;
        return cudaMemset2DAsync(c, pitch, 0, n * size, m, stream) == cudaSuccess ? DIPACO_OK : launch_status();
    }
    const int64_t tiles = ceil_div(m, TILE) * ceil_div(n, TILE);
    if (tiles > INT32_MAX) return DIPACO_ELIMIT;
    CUtensorMap a_map, b_map;
    if (!operand_map(&a_map, a) || !operand_map(&b_map, b)) return DIPACO_ECUDA;
    ProductArgs p = {static_cast<const uint8_t *>(a->scales), static_cast<const uint8_t *>(b->scales),
                     (int)ceil_div(a->cols, PACK_BLOCK), (int)ceil_div(b->cols, PACK_BLOCK),
                     transpose_a != 0, transpose_b != 0, (int)m, (int)n, (int)k, c, c_stride,
                     dtype == DIPACO_BF16, accumulate != 0};
    if (cudaFuncSetAttribute(product_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PRODUCT_SMEM) != cudaSuccess)
        return launch_status();
    product_kernel<<<(unsigned)tiles, PRODUCT_THREADS, PRODUCT_SMEM, stream>>>(a_map, b_map, p);
    return launch_status();
}

int dipaco_packed_matmul_status(int32_t device, void *cuda_stream)
{
    if (device < 0) return DIPACO_EINVAL;
    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    if (cudaStreamSynchronize(static_cast<cudaStream_t>(cuda_stream)) != cudaSuccess) return DIPACO_ECUDA;
    int word = 0;
    if (cudaMemcpyFromSymbol(&word, g_product_error, sizeof(int)) != cudaSuccess) return launch_status();
    if (word == 0) return DIPACO_OK;
    word = 0;
    cudaMemcpyToSymbol(g_product_error, &word, sizeof(int));
    return DIPACO_ETIMEOUT;
}

} // extern "C"
