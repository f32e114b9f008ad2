// Softmax cross-entropy of the labelled vertices, with the gradient of the class scores in the same pass.
//
// For a row x of C scores with label t:   m = max_j x_j,  s = sum_j exp(x_j - m),  loss = log s + m - x_t,
//     dx_j = w (exp(x_j - m) / s - [j = t]),   w = scale, or scale / number of labelled rows.
// A row without a label is not read; its gradient is 0.  Every row is read once and stays in registers, 16 bytes a lane: LANES lanes
// of a wavefront (or a whole workgroup) have a row.  Rows wider than that are read twice.
//
// Three launches: the labelled rows of every piece of the label array are counted, the rows are done with the sum of these
// counts, and the workgroups' sums of row losses are added in their order; results do not depend on timing.
#include "common.h"
#include "rows.h"

namespace {

constexpr int kThreads = 256;
constexpr int kCountBlocks = 256;   // partial counts
constexpr int kLossBlocks = 4096;   // partial losses at most

struct Labels {
    const void *p;
    int is_64;
    int64_t C;
    // the label of a row, -1 where it has none
    __device__ __forceinline__ int64_t at(int64_t r) const {
        const int64_t t = is_64 ? static_cast<const int64_t *>(p)[r] : int64_t(static_cast<const int32_t *>(p)[r]);
        return t >= 0 && t < C ? t : -1;
    }
};

template <int THREADS, typename V, typename F> __device__ __forceinline__ V group_reduce(V v, V *red, F f) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = f(v, __shfl_xor(v, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < THREADS / 64; ++i) v = f(v, red[i]);
    return v;
}

__global__ void __launch_bounds__(kThreads) count_labels_kernel(const Labels labels, int64_t N, int32_t *__restrict__ counts) {
    __shared__ int red[kThreads / 64];
    const int64_t each = (N + gridDim.x - 1) / gridDim.x, r0 = each * blockIdx.x, r1 = r0 + each < N ? r0 + each : N;
    int n = 0;
    for (int64_t r = r0 + threadIdx.x; r < r1; r += kThreads) n += labels.at(r) >= 0;
    n = group_reduce<kThreads>(n, red, [](int a, int b) { return a + b; });
    if (threadIdx.x == 0) counts[blockIdx.x] = n;
}

// scale, or scale / number of labelled rows; the same in every thread of a workgroup
__device__ __forceinline__ float row_weight(const int32_t *counts, float scale) {
    if (!counts) return scale;
    __shared__ int red[kThreads / 64];
    static_assert(kCountBlocks == kThreads, "one count a thread");
    const int n = group_reduce<kThreads>(counts[threadIdx.x], red, [](int a, int b) { return a + b; });
    return scale / float(n > 1 ? n : 1);
}

// max that keeps NaN
__device__ __forceinline__ float max_nan(float a, float b) { return a != a ? a : b != b ? b : a > b ? a : b; }

// Rows in registers: LANES lanes with NV vectors of VEC elements each.  The last vector of a row ends with the row; elements that
// it shares with the one before (or, of a lane without a vector, all) are left out of the sums.
template <typename T, int VEC, int LANES, int NV>
__global__ void __launch_bounds__(kThreads) xent_kernel(const T *__restrict__ X, int64_t ldx, const Labels labels, T *__restrict__ dX, int64_t ldg,
                                                        float *__restrict__ loss_rows, const int32_t *__restrict__ counts, float scale,
                                                        float *__restrict__ loss_part, int64_t N, int C) {
    __shared__ float red[kThreads / 64];
    const float w = row_weight(counts, scale);
    constexpr int ROWS = kThreads / LANES;
    const int lane = int(threadIdx.x) % LANES, team = int(threadIdx.x) / LANES;
    int col[NV], skip[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int c = (lane + k * LANES) * VEC;
        col[k] = c < C - VEC ? c : C - VEC;
        skip[k] = c < C ? c - col[k] : VEC;
    }
    float sum = 0.0f;
    for (int64_t r = int64_t(blockIdx.x) * ROWS + team; r < N; r += int64_t(gridDim.x) * ROWS) {
        const int64_t t = labels.at(r);
        float v[NV][VEC];
        float loss = 0.0f;
        if (t >= 0) {
            float m = -__builtin_inff();
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if (skip[k] < VEC) gnn_load_row<T, VEC>(X + r * ldx + col[k], v[k]);
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (j >= skip[k]) m = max_nan(m, v[k][j]);
            }
            auto larger = [](float a, float b) { return max_nan(a, b); };
            auto add = [](float a, float b) { return a + b; };
            if constexpr (LANES <= 64) {
#pragma unroll
                for (int d = LANES / 2; d > 0; d >>= 1) m = larger(m, __shfl_xor(m, d));
            } else m = group_reduce<kThreads>(m, red, larger);
            float s = 0.0f, xt = 0.0f;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    if (j < skip[k]) continue;
                    if (col[k] + j == t) xt = v[k][j];
                    v[k][j] = __expf(v[k][j] - m);
                    s += v[k][j];
                }
            if constexpr (LANES <= 64) {
#pragma unroll
                for (int d = LANES / 2; d > 0; d >>= 1) { s = add(s, __shfl_xor(s, d)); xt = add(xt, __shfl_xor(xt, d)); }
            } else { s = group_reduce<kThreads>(s, red, add); xt = group_reduce<kThreads>(xt, red, add); }
            loss = logf(s) + (m - xt);
            const float inv = w / s;
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[k][j] = v[k][j] * inv - (col[k] + j == t ? w : 0.0f);
        } else {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[k][j] = 0.0f;
        }
        if (dX) {
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if (skip[k] == 0) gnn_store_row<T, VEC>(dX + r * ldg + col[k], v[k]);
                else
#pragma unroll
                    for (int j = 0; j < VEC; ++j)
                        if (j >= skip[k]) gnn_rows<T>::set(dX + r * ldg + col[k] + j, v[k][j]);
            }
        }
        if (lane == 0) {
            if (loss_rows) loss_rows[r] = loss;
            sum += loss;
        }
    }
    sum = group_reduce<kThreads>(sum, red, [](float a, float b) { return a + b; });
    if (threadIdx.x == 0) loss_part[blockIdx.x] = sum * w;
}

// Rows beyond the registers: a workgroup reads its row twice, first for the running maximum and the sum of the exponentials.
template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads) xent_wide_kernel(const T *__restrict__ X, int64_t ldx, const Labels labels, T *__restrict__ dX, int64_t ldg,
                                                             float *__restrict__ loss_rows, const int32_t *__restrict__ counts, float scale,
                                                             float *__restrict__ loss_part, int64_t N, int64_t C) {
    __shared__ float red[kThreads / 64];
    const float w = row_weight(counts, scale);
    const int64_t whole = C / VEC * VEC;
    float sum = 0.0f;
    for (int64_t r = blockIdx.x; r < N; r += gridDim.x) {
        const int64_t t = labels.at(r);
        const T *x = X + r * ldx;
        T *g = dX ? dX + r * ldg : nullptr;
        float loss = 0.0f, top = 0.0f, inv = 0.0f;
        if (t >= 0) {
            float m = -__builtin_inff(), s = 0.0f;
            auto take = [&](float v) {
                const float up = max_nan(m, v);
                if (up != m) {  // also NaN
                    s = m == -__builtin_inff() ? 0.0f : s * __expf(m - up);
                    m = up;
                }
                if (m != -__builtin_inff()) s += __expf(v - m);
            };
            for (int64_t c = int64_t(threadIdx.x) * VEC; c < whole; c += int64_t(kThreads) * VEC) {
                float v[VEC];
                gnn_load_row<T, VEC>(x + c, v);
#pragma unroll
                for (int j = 0; j < VEC; ++j) take(v[j]);
            }
            if (whole + threadIdx.x < C) take(gnn_rows<T>::get(x + whole + threadIdx.x));
            top = group_reduce<kThreads>(m, red, [](float a, float b) { return max_nan(a, b); });
            s = group_reduce<kThreads>(m == -__builtin_inff() ? 0.0f : s * __expf(m - top), red, [](float a, float b) { return a + b; });
            loss = logf(s) + (top - gnn_rows<T>::get(x + t));
            inv = w / s;
        }
        if (g) {
            for (int64_t c = int64_t(threadIdx.x) * VEC; c < whole; c += int64_t(kThreads) * VEC) {
                float v[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[j] = 0.0f;
                if (t >= 0) {
                    gnn_load_row<T, VEC>(x + c, v);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) v[j] = __expf(v[j] - top) * inv - (c + j == t ? w : 0.0f);
                }
                gnn_store_row<T, VEC>(g + c, v);
            }
            if (whole + threadIdx.x < C) {
                const int64_t c = whole + threadIdx.x;
                gnn_rows<T>::set(g + c, t >= 0 ? __expf(gnn_rows<T>::get(x + c) - top) * inv - (c == t ? w : 0.0f) : 0.0f);
            }
        }
        if (threadIdx.x == 0) {
            if (loss_rows) loss_rows[r] = loss;
            sum += loss;
        }
    }
    if (threadIdx.x == 0) loss_part[blockIdx.x] = sum * w;
}

__global__ void __launch_bounds__(kThreads) add_losses_kernel(const float *__restrict__ part, int n, float *__restrict__ loss) {
    __shared__ double red[kThreads / 64];
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += kThreads) s += part[i];
    s = group_reduce<kThreads>(s, red, [](double a, double b) { return a + b; });
    if (threadIdx.x == 0) *loss = float(s);
}

struct Call {
    Labels labels;
    float *loss_rows, *loss, *part;
    int32_t *counts;
    float scale;
    int64_t N, C, ldx, ldg;
    hipStream_t stream;
};

int blocks_of(int64_t N, int rows) {
    const int64_t b = (N + rows - 1) / rows;
    return int(b < kLossBlocks ? b : kLossBlocks);
}

template <typename T, int VEC, int LANES, int NV> int launch(const T *X, T *dX, const Call &c) {
    const int blocks = blocks_of(c.N, kThreads / LANES);
    xent_kernel<T, VEC, LANES, NV><<<blocks, kThreads, 0, c.stream>>>(X, c.ldx, c.labels, dX, c.ldg, c.loss_rows, c.counts, c.scale, c.part, c.N, int(c.C));
    return blocks;
}

template <typename T> int xent(const T *X, T *dX, const Call &c) {
    constexpr int V = gnn_rows<T>::VEC;
    if (c.counts) count_labels_kernel<<<kCountBlocks, kThreads, 0, c.stream>>>(c.labels, c.N, c.counts);
    int blocks;
    if (c.C < V) blocks = launch<T, 1, 8, 1>(X, dX, c);
    else if (c.C <= 4 * V) blocks = launch<T, V, 4, 1>(X, dX, c);
    else if (c.C <= 8 * V) blocks = launch<T, V, 8, 1>(X, dX, c);
    else if (c.C <= 16 * V) blocks = launch<T, V, 16, 1>(X, dX, c);
    else if (c.C <= 32 * V) blocks = launch<T, V, 32, 1>(X, dX, c);
    else if (c.C <= 64 * V) blocks = launch<T, V, 64, 1>(X, dX, c);
    else if (c.C <= 128 * V) blocks = launch<T, V, 64, 2>(X, dX, c);
    else if (c.C <= 256 * V) blocks = launch<T, V, 256, 1>(X, dX, c);
    else if (c.C <= 512 * V) blocks = launch<T, V, 256, 2>(X, dX, c);
    else if (c.C <= 1024 * V) blocks = launch<T, V, 256, 4>(X, dX, c);
    else {
        blocks = blocks_of(c.N, 1);
        xent_wide_kernel<T, V><<<blocks, kThreads, 0, c.stream>>>(X, c.ldx, c.labels, dX, c.ldg, c.loss_rows, c.counts, c.scale, c.part, c.N, c.C);
    }
    add_losses_kernel<<<1, kThreads, 0, c.stream>>>(c.part, blocks, c.loss);
    GNN_HIP_TRY(hipGetLastError());
    return GNN_OK;
}

__global__ void zero_loss_kernel(float *loss) { *loss = 0.0f; }

}  // namespace

extern "C" GNN_API int64_t gnn_softmax_xent_workspace_bytes(int64_t N, int64_t C) {
    if (N <= 0 || C <= 0) return 0;
    return kCountBlocks * 4 + kLossBlocks * 4;
}

extern "C" GNN_API int gnn_softmax_xent(const void *X, const void *labels, float *loss, void *dX, float *loss_rows, int64_t N, int64_t C,
                                        const gnn_loss_opts *opts) {
    if (!opts) return GNN_ERR_INVALID_ARG;
    gnn_loss_opts o = *opts;
    if (o.dtype != GNN_F32 && o.dtype != GNN_BF16) return GNN_ERR_INVALID_ARG;
    if (o.reduction != GNN_LOSS_SUM && o.reduction != GNN_LOSS_MEAN) return GNN_ERR_INVALID_ARG;
    if (N < 0 || C < 0 || N > INT32_MAX || C > INT32_MAX || !loss) return GNN_ERR_INVALID_ARG;
    if (o.ldx == 0) o.ldx = C;
    if (o.ldg == 0) o.ldg = C;
    if (o.ldx < C || o.ldg < C) return GNN_ERR_INVALID_ARG;
    hipStream_t stream = static_cast<hipStream_t>(o.stream);
    (void)hipGetLastError();
    if (N == 0 || C == 0) {
        zero_loss_kernel<<<1, 1, 0, stream>>>(loss);
        GNN_HIP_TRY(hipGetLastError());
        return GNN_OK;
    }
    if (!X || !labels || X == dX) return GNN_ERR_INVALID_ARG;
    if (!o.workspace || o.workspace_bytes < gnn_softmax_xent_workspace_bytes(N, C) || reinterpret_cast<uintptr_t>(o.workspace) % 16)
        return GNN_ERR_INVALID_ARG;
    Call c{};
    c.labels = Labels{labels, o.labels_is_64, C};
    c.counts = o.reduction == GNN_LOSS_MEAN ? static_cast<int32_t *>(o.workspace) : nullptr;
    c.part = reinterpret_cast<float *>(static_cast<char *>(o.workspace) + kCountBlocks * 4);
    c.loss = loss;
    c.loss_rows = loss_rows;
    c.scale = o.scale;
    c.N = N;
    c.C = C;
    c.ldx = o.ldx;
    c.ldg = o.ldg;
    c.stream = stream;
    if (o.dtype == GNN_F32) return xent(static_cast<const float *>(X), static_cast<float *>(dX), c);
    return xent(static_cast<const gnn_bf16 *>(X), static_cast<gnn_bf16 *>(dX), c);
}
