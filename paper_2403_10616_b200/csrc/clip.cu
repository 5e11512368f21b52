// The norm of many gradients together, and the gradients times min(1, most / norm) (see include/dipaco.h).
//
// The gradients are cut into chunks, each of one tensor, which blocks take in turn: sums_kernel leaves one sum of
// squares for each block, scale_kernel joins them in every block and goes through the chunks again, the last
// first, as those are the ones still in L2.  Few values take one launch of a cluster of blocks instead, whose sums
// meet in distributed shared memory (cluster_kernel).  Tensors are listed in the kernels' arguments, so that a call
// copies nothing and can be captured; longer lists take several launches.  Where neither a limit nor the norm is asked
// for, scale_kernel alone makes the copies.
//
// Bound by memory: gradients are read once for the norm and once more to be scaled.  144M in fp32, gathered: 286 us, 1.08
// of what those bytes take at a copy's rate (the floor without the second reading is 176); 526,080 in two launches 6.7.
#include "inner_common.cuh"

#include <algorithm>
#include <cfloat>
#include <exception>
#include <vector>

using namespace dipaco;

namespace {

constexpr int CHUNK = 8192, WARP_CHUNK = 2048;  // values, of a block and of a warp
constexpr int THREADS = 256;
constexpr int CLUSTER = 8, CLUSTER_THREADS = 512, CLUSTER_WARPS = CLUSTER * CLUSTER_THREADS / 32;
// One launch instead of two and a workspace, which saves the host 5.5 us of a call, while eight SMs take no longer than all
// of them.  In a replayed graph, mean of 1, 6 and 60 tensors in fp32 and 6 in bf16: 4.8 us for 1000 values (two launches
// 4.7), 6.5 for 64,000 (6.1), 6.6 for 96,000 (6.7), 7.4 for 128,000 (6.2), 9.2 for 256,000 (6.6), 13.8 for 526,080 (6.5).
// A warp has a chunk to itself: tensors are small, and a block to each chunk took 14 us for 64 of 1000 values, which take
// 6.6 now.
constexpr int CLUSTER_VALUES = 100000;
constexpr int FEW_TENSORS = 64, MANY_TENSORS = 640;  // 2 and 20 KB of arguments
constexpr int MAX_BLOCKS = 148 * 8;
constexpr int MAX_JOINED = 4096;  // sums that every block of scale_kernel joins by itself

struct Piece {
    const void *in;
    void *out;
    long long numel;
    unsigned first_chunk;
    unsigned char in_bf16, out_bf16;
};
template <int CAPACITY> struct Pieces {
    int count;
    unsigned chunks;
    Piece piece[CAPACITY];
};

// Chunk `chunk` is values [begin, end) of its piece, which is returned.
template <int SIZE = CHUNK, int CAPACITY>
__device__ __forceinline__ const Piece &find_chunk(const Pieces<CAPACITY> &t, unsigned chunk, long long &begin, long long &end)
{
    int low = 0, high = t.count - 1;  // the last piece whose first chunk is not after this one (it has a chunk)
    while (low < high) {
        const int mid = (low + high + 1) >> 1;
        if (t.piece[mid].first_chunk <= chunk)
            low = mid;
        else
            high = mid - 1;
    }
    const Piece &p = t.piece[low];
    begin = (long long)(chunk - p.first_chunk) * SIZE;
    end = min(p.numel, begin + SIZE);
    return p;
}

// The units of 16 bytes that hold values [begin, end) of a tensor: rows of them may begin and end inside one.
template <typename T> struct Units {
    static constexpr int UE = Unit<T>::UE;
    const uint4 *first;
    int lead, values, count;  // values of the first unit that come before, values, units
    __device__ Units(const void *p, long long begin, long long end)
    {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p) + begin * sizeof(T);
        first = reinterpret_cast<const uint4 *>(at & ~(uintptr_t)15);
        lead = (int)(at & 15) / (int)sizeof(T);
        values = (int)(end - begin);
        count = (lead + values + UE - 1) / UE;
    }
    __device__ __forceinline__ bool whole(int u) const { return u * UE >= lead && (u + 1) * UE <= lead + values; }
    __device__ __forceinline__ bool holds(int u, int i) const { return u * UE + i >= lead && u * UE + i < lead + values; }
};

template <typename T> __device__ __forceinline__ uint4 load_masked(const Units<T> &units, int u)
{
    uint4 v = __ldg(units.first + u);
    if (!units.whole(u)) {
        float f[Unit<T>::UE];
        Unit<T>::widen(v, f);
#pragma unroll
        for (int i = 0; i < Unit<T>::UE; ++i)
            if (!units.holds(u, i)) f[i] = 0.0f;
        v = Unit<T>::narrow(f);  // exact
    }
    return v;
}

template <typename T> __device__ __forceinline__ void add_squares(const uint4 &v, f32x2 *sum, unsigned &bits)
{
    bits |= v.x | v.y | v.z | v.w;
    f32x2 w[Unit<T>::UE / 2];
    widen_pairs<T>(v, w);
#pragma unroll
    for (int i = 0; i < Unit<T>::UE / 2; ++i) sum[i & 1] = fma2(w[i], w[i], sum[i & 1]);
}

// The sum of squares of thread me's values of a chunk, one of N.  Squares are added in fp32, at most 80 of them in four
// chains, and where that overflows or loses small values, once more in fp64.
template <typename T, int N, int SIZE> __device__ __forceinline__ double chunk_squares(const void *p, long long begin, long long end, int me)
{
    constexpr int UE = Unit<T>::UE, EACH = SIZE / UE / N;  // units of a thread
    const Units<T> units(p, begin, end);
    f32x2 sum[2] = {0ull, 0ull};
    unsigned bits = 0u;
    if (units.lead == 0 && units.values == SIZE) {  // all loads at once
        uint4 v[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) v[i] = __ldg(units.first + me + i * N);
#pragma unroll
        for (int i = 0; i < EACH; ++i) add_squares<T>(v[i], sum, bits);
    } else {
#pragma unroll 4
        for (int u = me; u < units.count; u += N) add_squares<T>(load_masked(units, u), sum, bits);
    }
    const float s = sum_of(add2(sum[0], sum[1]));
    const bool nothing = (bits & (sizeof(T) == 2 ? 0x7fff7fffu : 0x7fffffffu)) == 0u;
    if ((s >= 1e-28f && s <= 1e38f) || nothing) return s;
    double exact = 0.0;
    for (int u = me; u < units.count; u += N) {
        float f[UE];
        Unit<T>::widen(load_masked(units, u), f);
#pragma unroll
        for (int i = 0; i < UE; ++i) exact = fma((double)f[i], (double)f[i], exact);
    }
    return exact;
}
template <int N, int SIZE> __device__ __forceinline__ double piece_squares(const Piece &p, long long begin, long long end, int me)
{
    return p.in_bf16 ? chunk_squares<__nv_bfloat16, N, SIZE>(p.in, begin, end, me) : chunk_squares<float, N, SIZE>(p.in, begin, end, me);
}

// The sum over the block, on every thread.
template <int N = THREADS> __device__ __forceinline__ double block_sum(double v, double *shared)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < N / 32; ++w) v += shared[w];
    return v;
}

template <int CAPACITY>
__global__ void __launch_bounds__(THREADS) sums_kernel(const __grid_constant__ Pieces<CAPACITY> t, double *sums)
{
    __shared__ double shared[THREADS / 32];
    double sum = 0.0;
    for (unsigned c = blockIdx.x; c < t.chunks; c += gridDim.x) {
        long long begin, end;
        const Piece &p = find_chunk(t, c, begin, end);
        sum += piece_squares<THREADS, CHUNK>(p, begin, end, threadIdx.x);
    }
    sum = block_sum(sum, shared);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

__device__ __forceinline__ double joined(const double *sums, int count, double *shared)
{
    double sum = 0.0;
    for (int i = threadIdx.x; i < count; i += THREADS) sum += sums[i];
    return block_sum(sum, shared);
}

// Many sums to one, in their place.
__global__ void __launch_bounds__(THREADS) fold_kernel(double *sums, int count)
{
    __shared__ double shared[THREADS / 32];
    const double sum = joined(sums, count, shared);  // all have been read after its barrier
    if (threadIdx.x == 0) sums[0] = sum;
}

__global__ void __launch_bounds__(THREADS) norm_kernel(const double *sums, int count, float *norm)
{
    __shared__ double shared[THREADS / 32];
    const double sum = joined(sums, count, shared);
    if (threadIdx.x == 0) *norm = (float)sqrt(sum);
}

// A unit of values times `by`, to q.
template <typename T, typename O> __device__ __forceinline__ void store_scaled(const uint4 &v, float by, O *q)
{
    constexpr int UE = Unit<T>::UE, OE = Unit<O>::UE;
    float f[UE];
    Unit<T>::widen(v, f);
#pragma unroll
    for (int i = 0; i < UE; ++i) f[i] *= by;
    if constexpr (UE < OE) {  // four values to 8 bytes
        __stcs(reinterpret_cast<uint2 *>(q), make_uint2(Unit<O>::pack(f[0], f[1]), Unit<O>::pack(f[2], f[3])));
    } else {
#pragma unroll
        for (int i = 0; i < UE / OE; ++i) __stcs(reinterpret_cast<uint4 *>(q) + i, Unit<O>::narrow(f + i * OE));
    }
}

template <typename T, typename O, int N, int SIZE>
__device__ __forceinline__ void scale_chunk(const Piece &p, long long begin, long long end, float by, int me)
{
    constexpr int UE = Unit<T>::UE, EACH = SIZE / UE / N;
    constexpr int AT_ONCE = N == 32 ? 16 : 8;  // loads that wait for no store: the few warps of a cluster need more
    const T *const in = static_cast<const T *>(p.in) + begin;
    O *const out = static_cast<O *>(p.out) + begin;
    const Units<T> units(in, 0, end - begin);
    O *const to = out - units.lead;  // where the first unit's first value would go
    int head = 0, tail = 0;          // values before the whole units; the first one after them
    if (reinterpret_cast<uintptr_t>(to) % (UE * sizeof(O) < 16 ? UE * sizeof(O) : 16) == 0) {
        if (units.lead == 0 && units.values == SIZE) {
            uint4 v[EACH];
#pragma unroll
            for (int i = 0; i < EACH; ++i) v[i] = __ldcs(units.first + me + i * N);
#pragma unroll
            for (int i = 0; i < EACH; ++i) store_scaled<T, O>(v[i], by, to + (me + i * N) * UE);
            return;
        }
        const int whole = units.lead ? 1 : 0, last = (units.lead + units.values) / UE;
        head = min(units.values, whole * UE - units.lead);
        tail = max(head, last * UE - units.lead);
        int u = whole + me;
#pragma unroll 1
        for (; u + (AT_ONCE / 4 - 1) * N < last; u += AT_ONCE / 4 * N) {
            uint4 v[AT_ONCE / 4];
#pragma unroll
            for (int k = 0; k < AT_ONCE / 4; ++k) v[k] = __ldcs(units.first + u + k * N);
#pragma unroll
            for (int k = 0; k < AT_ONCE / 4; ++k) store_scaled<T, O>(v[k], by, to + (u + k * N) * UE);
        }
#pragma unroll 1
        for (; u < last; u += N) store_scaled<T, O>(__ldcs(units.first + u), by, to + u * UE);
        if (me < head) out[me] = narrow1<O>(widen1<T>(in[me]) * by);
    }
    // the rest, or all where results lie at another place within 16 bytes than the values: value by value
    int i = tail + me;
#pragma unroll 1
    for (; i + (AT_ONCE - 1) * N < units.values; i += AT_ONCE * N) {
        T v[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) v[k] = in[i + k * N];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) out[i + k * N] = narrow1<O>(widen1<T>(v[k]) * by);
    }
#pragma unroll 1
    for (; i < units.values; i += N) out[i] = narrow1<O>(widen1<T>(in[i]) * by);
}
// The same with a factor that fp32 holds to fewer bits than its own (gradients near the largest value): in fp64.
template <typename T, typename O, int N>
__device__ __noinline__ void scale_exactly(const Piece &p, long long begin, long long end, double by, int me)
{
    for (long long i = begin + me; i < end; i += N)
        static_cast<O *>(p.out)[i] = narrow1<O>((float)((double)widen1<T>(static_cast<const T *>(p.in)[i]) * by));
}
template <int N, int SIZE> __device__ __forceinline__ void scale_piece(const Piece &p, long long begin, long long end, double factor, int me)
{
    const float by = (float)factor;
    if (p.in == p.out && by == 1.0f) return;
    if (factor > 0.0 && factor < FLT_MIN) {
        if (p.in_bf16) {
            if (p.out_bf16)
                scale_exactly<__nv_bfloat16, __nv_bfloat16, N>(p, begin, end, factor, me);
            else
                scale_exactly<__nv_bfloat16, float, N>(p, begin, end, factor, me);
        } else {
            if (p.out_bf16)
                scale_exactly<float, __nv_bfloat16, N>(p, begin, end, factor, me);
            else
                scale_exactly<float, float, N>(p, begin, end, factor, me);
        }
        return;
    }
    if (p.in_bf16) {
        if (p.out_bf16)
            scale_chunk<__nv_bfloat16, __nv_bfloat16, N, SIZE>(p, begin, end, by, me);
        else
            scale_chunk<__nv_bfloat16, float, N, SIZE>(p, begin, end, by, me);
    } else {
        if (p.out_bf16)
            scale_chunk<float, __nv_bfloat16, N, SIZE>(p, begin, end, by, me);
        else
            scale_chunk<float, float, N, SIZE>(p, begin, end, by, me);
    }
}
__device__ __forceinline__ double factor(double norm, double most)
{
    return norm <= most || most == INFINITY ? 1.0 : most / norm;  // with a limit a NaN makes all results NaN
}

template <int CAPACITY>
__global__ void __launch_bounds__(THREADS)
    scale_kernel(const __grid_constant__ Pieces<CAPACITY> t, const double *sums, int count, double most, float *norm)
{
    __shared__ double shared[THREADS / 32];
    const double of_all = sqrt(joined(sums, count, shared));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)of_all;
    const double by = factor(of_all, most);
    for (unsigned i = blockIdx.x; i < t.chunks; i += gridDim.x) {
        long long begin, end;
        const Piece &p = find_chunk(t, t.chunks - 1 - i, begin, end);
        scale_piece<THREADS, CHUNK>(p, begin, end, by, threadIdx.x);
    }
}

// Everything at once, on one cluster: its blocks' sums are read from one another's shared memory.
__global__ void __cluster_dims__(CLUSTER, 1, 1) __launch_bounds__(CLUSTER_THREADS, 1)
    cluster_kernel(const __grid_constant__ Pieces<FEW_TENSORS> t, bool scale, double most, float *norm)
{
    __shared__ double shared[CLUSTER_THREADS / 32], of_block;
    const unsigned warp = threadIdx.x / 32 * CLUSTER + blockIdx.x;  // of the cluster
    const int lane = threadIdx.x & 31;
    double sum = 0.0;
    for (unsigned c = warp; c < t.chunks; c += CLUSTER_WARPS) {
        long long begin, end;
        const Piece &p = find_chunk<WARP_CHUNK>(t, c, begin, end);
        sum += piece_squares<32, WARP_CHUNK>(p, begin, end, lane);
    }
    sum = block_sum<CLUSTER_THREADS>(sum, shared);
    if (threadIdx.x == 0) of_block = sum;
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    sum = 0.0;
#pragma unroll
    for (int r = 0; r < CLUSTER; ++r) {
        uint32_t at;
        double v;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(ptx::smem_addr(&of_block)), "r"(r));
        asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(at) : "memory");
        sum += v;
    }
    // no block ends while its sum may still be read
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    const double of_all = sqrt(sum);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)of_all;
    if (scale) {
        const double by = factor(of_all, most);
        for (unsigned c = warp; c < t.chunks; c += CLUSTER_WARPS) {
            long long begin, end;
            const Piece &p = find_chunk<WARP_CHUNK>(t, c, begin, end);
            scale_piece<32, WARP_CHUNK>(p, begin, end, by, lane);
        }
    }
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ------------------------------------------------------------------------------------------ host

// What a call launches: tensors without values are left out.
struct Launches {
    std::vector<int> tensors;  // with values, in order
    int per_launch = 0, launches = 0;
    bool one_cluster = false;
    int64_t sums = 0;  // of the workspace
};

int64_t chunks_of(int64_t numel, int size = CHUNK) { return ceil_div(numel, size); }

int plan(const int64_t *numel, int32_t count, Launches &plan)
{
    if (count < 0 || (count > 0 && !numel)) return DIPACO_EINVAL;
    int64_t chunks = 0, values = 0;
    for (int i = 0; i < count; ++i) {
        if (numel[i] < 0) return DIPACO_EINVAL;
        if (numel[i] == 0) continue;
        if (numel[i] > ((int64_t)1 << 44)) return DIPACO_ELIMIT;
        plan.tensors.push_back(i);
        chunks += chunks_of(numel[i]);
        values += numel[i];
        if (chunks > INT32_MAX) return DIPACO_ELIMIT;
    }
    const int tensors = (int)plan.tensors.size();
    plan.per_launch = tensors <= FEW_TENSORS ? FEW_TENSORS : MANY_TENSORS;
    plan.launches = (int)ceil_div(tensors, plan.per_launch);
    plan.one_cluster = tensors <= FEW_TENSORS && values <= CLUSTER_VALUES;
    plan.sums = plan.one_cluster ? 0 : (int64_t)plan.launches * MAX_BLOCKS;
    return DIPACO_OK;
}

// Whether results overlap one another or values other than the ones they come from.
bool results_overlap(const Launches &plan, const void *const *grads, void *const *out, const int64_t *numel,
                     const int32_t *dtypes, const int32_t *out_dtypes)
{
    struct Range {
        uintptr_t begin, end;
        int tensor;
        bool result;
    };
    std::vector<Range> ranges;
    ranges.reserve(2 * plan.tensors.size());
    for (const int i : plan.tensors) {
        const uintptr_t in = (uintptr_t)grads[i], to = (uintptr_t)out[i];
        if (in != to || dtypes[i] != out_dtypes[i]) ranges.push_back({in, in + numel[i] * dense_size(dtypes[i]), i, false});
        ranges.push_back({to, to + numel[i] * dense_size(out_dtypes[i]), i, true});
    }
    std::sort(ranges.begin(), ranges.end(), [](const Range &a, const Range &b) { return a.begin < b.begin; });
    uintptr_t read = 0, written = 0;  // up to where ranges so far go
    for (const Range &r : ranges) {
        if (r.begin < written || (r.result && r.begin < read)) return true;
        uintptr_t &end = r.result ? written : read;
        end = std::max(end, r.end);
    }
    return false;
}

// Neither a limit nor the norm is asked for: results are copies, and no square is added.
bool are_copies(void *const *out, double most, const float *norm) { return out && most == INFINITY && !norm; }

template <int CAPACITY>
int launch(const Launches &plan, const void *const *grads, void *const *out, const int64_t *numel,
           const int32_t *dtypes, const int32_t *out_dtypes, double most, float *norm, double *sums, cudaStream_t stream)
{
    Pieces<CAPACITY> t;
    const bool copies = are_copies(out, most, norm), one_cluster = plan.one_cluster && !copies;
    const auto fill = [&](int launch) {
        const int first = launch * CAPACITY, last = std::min(first + CAPACITY, (int)plan.tensors.size());
        t.count = last - first;
        t.chunks = 0;
        for (int k = first; k < last; ++k) {
            const int i = plan.tensors[k];
            t.piece[k - first] = {grads[i], out ? out[i] : nullptr, numel[i], t.chunks, dtypes[i] == DIPACO_BF16,
                                  (unsigned char)(out && out_dtypes[i] == DIPACO_BF16)};
            t.chunks += (unsigned)chunks_of(numel[i], one_cluster ? WARP_CHUNK : CHUNK);
        }
    };
    if constexpr (CAPACITY == FEW_TENSORS) {
        if (one_cluster) {
            fill(0);
            cluster_kernel<<<CLUSTER, CLUSTER_THREADS, 0, stream>>>(t, out != nullptr, most, norm);
            return launch_status();
        }
    }
    int count = 0;
    for (int l = 0; l < (copies ? 0 : plan.launches); ++l) {
        fill(l);
        const int blocks = (int)std::min<int64_t>(t.chunks, MAX_BLOCKS);
        sums_kernel<CAPACITY><<<blocks, THREADS, 0, stream>>>(t, sums + count);
        count += blocks;
    }
    if (count > MAX_JOINED) {
        fold_kernel<<<1, THREADS, 0, stream>>>(sums, count);
        count = 1;
    }
    if (!out) {
        if (norm) norm_kernel<<<1, THREADS, 0, stream>>>(sums, count, norm);
        return launch_status();
    }
    for (int l = plan.launches - 1; l >= 0; --l) {
        if (plan.launches > 1 || copies) fill(l);
        const int blocks = (int)std::min<int64_t>(t.chunks, MAX_BLOCKS);
        scale_kernel<CAPACITY><<<blocks, THREADS, 0, stream>>>(t, sums, count, most, l == 0 ? norm : nullptr);
    }
    return launch_status();
}

} // namespace

extern "C" {

int dipaco_clip_gradients_workspace(const int64_t *numel, int32_t count, int64_t *bytes)
{
    if (!bytes) return DIPACO_EINVAL;
    try {
        Launches p;
        if (const int rc = plan(numel, count, p)) return rc;
        *bytes = p.sums * (int64_t)sizeof(double);
        return DIPACO_OK;
    } catch (const std::exception &) {
        return DIPACO_ENOMEM;
    }
}

int dipaco_clip_gradients(const void *const *grads, void *const *out, const int64_t *numel, const int32_t *dtypes,
                          const int32_t *out_dtypes, int32_t count, double max_norm, float *norm, void *workspace,
                          int64_t workspace_bytes, int32_t device, void *cuda_stream)
{
    if (device < 0 || (out && !(max_norm >= 0.0)) || !vector_ok(norm, 4)) return DIPACO_EINVAL;
    if (count > 0 && (!grads || !dtypes || (out && !out_dtypes))) return DIPACO_EINVAL;
    try {
        Launches p;
        if (const int rc = plan(numel, count, p)) return rc;
        for (const int i : p.tensors) {
            if (!is_dense_dtype(dtypes[i]) || !grads[i] || !vector_ok(grads[i], dense_size(dtypes[i]))) return DIPACO_EINVAL;
            if (out && (!is_dense_dtype(out_dtypes[i]) || !out[i] || !vector_ok(out[i], dense_size(out_dtypes[i])))) return DIPACO_EINVAL;
        }
        if (out && results_overlap(p, grads, out, numel, dtypes, out_dtypes)) return DIPACO_EINVAL;
        if (p.sums > 0 && !are_copies(out, max_norm, norm) &&
            (!workspace || (uintptr_t)workspace % 16 != 0 || workspace_bytes < p.sums * (int64_t)sizeof(double)))
            return DIPACO_EINVAL;
        DeviceScope scope(device);
        if (!scope.ok) return DIPACO_ECUDA;
        const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
        if (p.tensors.empty())
            return !norm || cudaMemsetAsync(norm, 0, sizeof(float), stream) == cudaSuccess ? DIPACO_OK : launch_status();
        double *sums = static_cast<double *>(workspace);
        return p.per_launch == FEW_TENSORS
                   ? launch<FEW_TENSORS>(p, grads, out, numel, dtypes, out_dtypes, max_norm, norm, sums, stream)
                   : launch<MANY_TENSORS>(p, grads, out, numel, dtypes, out_dtypes, max_norm, norm, sums, stream);
    } catch (const std::exception &) {  // no memory for the list
        return DIPACO_ENOMEM;
    }
}

} // extern "C"
