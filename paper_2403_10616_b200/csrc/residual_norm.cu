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
//   rows_kernel       a block per row, which is read once for every sum: any width
//   back_rows_kernel  the same for dx, df and the two means that d needs; back_columns_kernel the sums over rows
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

struct BackPlan {
    int parts;
    int64_t partial_bytes, bytes;
};
BackPlan plan_back(int64_t rows, int64_t cols)
{
    const int64_t columns = std::max<int64_t>(1, ceil_div(cols, COLUMN_THREADS));
    BackPlan p;
    p.parts = (int)std::max<int64_t>(1, std::min<int64_t>({MAX_PARTS, ceil_div(rows, 16), ceil_div(148 * 8, columns)}));
    p.partial_bytes = (int64_t)p.parts * 4 * cols * 4;
    p.bytes = ceil_div(p.partial_bytes, 16) * 16 + rows * 8;
    return p;
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
    const unsigned grid = (unsigned)std::min<int64_t>(rows, 148 * 8);
    if (args->dtype == DIPACO_BF16)
        rows_kernel<__nv_bfloat16><<<grid, ROW_THREADS, 0, stream>>>(a);
    else
        rows_kernel<float><<<grid, ROW_THREADS, 0, stream>>>(a);
    if (const int rc = launch_status()) return rc;
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
    const unsigned grid = (unsigned)std::min<int64_t>(rows, 148 * 8);
    const dim3 columns((unsigned)ceil_div(cols, COLUMN_THREADS), (unsigned)plan.parts);
    if (dtype == DIPACO_BF16) {
        back_rows_kernel<__nv_bfloat16><<<grid, ROW_THREADS, 0, stream>>>(a);
        back_columns_kernel<__nv_bfloat16><<<columns, COLUMN_THREADS, 0, stream>>>(a);
    } else {
        back_rows_kernel<float><<<grid, ROW_THREADS, 0, stream>>>(a);
        back_columns_kernel<float><<<columns, COLUMN_THREADS, 0, stream>>>(a);
    }
    if (const int rc = launch_status()) return rc;
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
