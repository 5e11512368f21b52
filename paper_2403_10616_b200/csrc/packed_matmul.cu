// Product of two packed matrices (see include/dipaco.h): C = op(A) op(B), codes e4m3, one scale per
// block of 128 x 128, fp32 sums.
//
// The contraction is walked in steps of 128, one block of A against one of B, on the tensor cores'
// block-scaled 8-bit form (tcgen05.mma kind::mxf8f6f4).  That form takes one scale per row and 32
// contracted values; here all of them are equal over a block, so the scale operands in tensor memory
// are constant words and a block may be contracted along either side: the operand's major-ness in the
// instruction descriptor is all that differs between the forward product and the two gradients.
//
//   pair_kernel    persistent; two SMs share a tile of 256 rows and up to 256 columns (cta_group::2):
//                  each loads half of A and half of B and keeps half of the sums
//   few_kernel     a few tokens through a weight: every weight is read once and multiplied in registers
//
// Measured: 8192^3 380 us in short runs (2.9 PFLOP/s) and 455 us under the 1000 W cap, 16384x2048x8192 176
// and 227 us, 32768x3584x896 100 and 124 us, the weight's gradient 3584x896 over 65501 198 and 244 us, 12 of them
// to join partial sums.  In long runs power sets the clock (1.3 to 1.45 GHz).  The tensor cores are busy for 86 %
// of the second's cycles, 52 % of the third's (seven steps to a tile, whose operands come from L2: 1.28 GB in 108 us,
// and 235 MB of results) and 65 % of the last's.  Adding to C takes longer, a dependent read of C for every row of a
// group of 32 columns: 32768x3584x896 in bf16 1.33 ms instead of 0.10, 16384x2048x8192 0.49.
#include "product_pairs.cuh"

#include <exception>
#include <map>
#include <mutex>
#include <utility>

namespace dipaco {
namespace {

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


} // namespace
} // namespace dipaco

using namespace dipaco;

extern "C" {

int dipaco_packed_matmul_workspace(int64_t m, int64_t n, int64_t k, int64_t *bytes)
{
    if (!bytes || k < 0) return DIPACO_EINVAL;
    if (const int rc = check_extents(m, n)) return rc;
    if (k > MAX_EXTENT) return DIPACO_ELIMIT;
    *bytes = m == 0 || n == 0 || k == 0 ? 0 : plan_pairs(m, n, ceil_div(k, STEP)).workspace;
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
    const bool few = are_few(m, n, k, transpose_a, transpose_b);
    if (!few && need > 0 && (!workspace || (uintptr_t)workspace % 16 != 0 || workspace_bytes < need)) return DIPACO_EINVAL;
    if (m == 0 || n == 0 || (k == 0 && accumulate)) return DIPACO_OK;

    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (k == 0) {  // a sum over nothing
        const size_t size = dense_size(dtype);
        const size_t pitch = m == 1 ? n * size : c_stride * size;
        return cudaMemset2DAsync(c, pitch, 0, n * size, m, stream) == cudaSuccess ? DIPACO_OK : launch_status();
    }
    if (few) return launch_few(a, b, c, c_stride, dtype, accumulate != 0, AsItIs{}, stream);
    const DenseKernels<AsItIs> kernels = {{pair_kernel<false, AsItIs>, pair_kernel<false, AsItIs>},
                                          {pair_kernel<true, AsItIs>, pair_kernel<true, AsItIs>},
                                          pair_threads(PAIR_EPILOGUE_WARPS),
                                          false};
    return launch_product(a, b, transpose_a != 0, transpose_b != 0, c, c_stride, dtype, accumulate != 0, AsItIs{}, kernels,
                          workspace, stream);
}

int dipaco_selftest_inner_wait_expiry(int32_t operators, int64_t limit_ns, int32_t device, void *cuda_stream)
{
    if (operators < 0 || operators > 2 || limit_ns < 1 || limit_ns > 1000000000ll || device < 0) return DIPACO_EINVAL;
    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (operators == 0) {
        if (const int rc = expire_norm_wait(limit_ns, stream)) return rc;
        return expire_residual_norm_wait(limit_ns, stream);
    }
    if (operators == 1) return expire_packing_wait(limit_ns, stream);
    wait_expiry_kernel<<<1, 32, 0, stream>>>(limit_ns);
    if (const int rc = launch_status()) return rc;
    return expire_linear_wait(limit_ns, stream);
}

int dipaco_inner_status(int32_t device, void *cuda_stream)
{
    if (device < 0) return DIPACO_EINVAL;
    DeviceScope scope(device);
    if (!scope.ok) return DIPACO_ECUDA;
    if (cudaStreamSynchronize(static_cast<cudaStream_t>(cuda_stream)) != cudaSuccess) return DIPACO_ECUDA;
    try {
        // A word is cleared by whoever reads it first, so that the news is kept here for the streams that ask later.
        static std::mutex mutex;
        static std::map<int32_t, uint64_t> &happened = *new std::map<int32_t, uint64_t>;  // time-outs on a device
        static std::map<std::pair<int32_t, void *>, uint64_t> &told = *new std::map<std::pair<int32_t, void *>, uint64_t>;
        const std::lock_guard<std::mutex> lock(mutex);
        uint64_t &count = happened[device], &known = told[{device, cuda_stream}];
        bool expired = false;
        const bool read = take_error_word(g_product_error, expired) && take_packing_error(expired) && take_norm_error(expired) &&
                          take_linear_error(expired) && take_residual_norm_error(expired);
        if (expired) ++count;
        if (!read) return launch_status();
        if (known == count) return DIPACO_OK;
        known = count;
        return DIPACO_ETIMEOUT;
    } catch (const std::exception &) {  // no memory for the books: nothing has been read
        return DIPACO_ENOMEM;
    }
}

} // extern "C"
