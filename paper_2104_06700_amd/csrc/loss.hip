// Softmax cross-entropy of the labelled vertices, with the gradient of the class scores in the same pass.
//
// For a row x of C scores with label t:   m = max_j x_j,  s = sum_j exp(x_j - m),  loss = log s + m - x_t,
//     dx_j = w (exp(x_j - m) / s - [j = t]),   w = scale, or scale / number of labelled rows.
// exp and log are one instruction and a product in 32 bits each; an exponential of d is off by about (1 + |d|) 2^-22, less than a gradient in bf16 keeps.
// A row without a label is not read; its gradient is 0.  Every row is read once and stays in registers, 16 bytes a lane: LANES lanes
// of a wavefront (or a whole workgroup) have a row, and a workgroup ends with its rows.  Rows wider than that are read twice.
//
// Three launches: the labelled rows of every piece of the label array are counted, the rows are done with the sum of these
// counts, and the workgroups' sums of row losses are added in their order; results do not depend on timing.  Of few rows every workgroup
// counts by itself, which is one launch less.
//
// Bound by the memory in wide rows (24,490 x 8,195 bf16, all labelled, 176 us = 4.6 TB/s, a workgroup's row waits twice for all its wavefronts), by
// instructions in narrow ones (2.4 M x 47 fp32, 8 % labelled, 98 us = 5.2 TB/s).
#include "common.h"
#include "rows.h"

namespace {

constexpr int kThreads = 256;
constexpr int kCountBlocks = 256;       // partial counts
// Rows up to which every workgroup counts all labels; Wide: where a row is a workgroup, so that the labels are read once a row (us, counted there and by a
// launch of its own: 4,096 rows of 16, 47, 200, 500 fp32 7.9 10.4, 8.9 10.4, 9.9 10.5, 9.5 10.4; 5,000 8.7 9.5, 9.9 9.6, 11.2 10.3, 11.1 10.2; 16,384 14.9
// 10.3 to 37.6 18.0.  Rows of 1,100: 1,300 9.2 11.2, 2,048 11.9 11.9, 2,900 15.4 12.8, 4,096 21.6 14.8, 16,384 151 33).
constexpr int64_t kCountHere = 4096, kCountHereWide = 2048;
constexpr int kLossBlocks = 65536;      // partial losses at most
constexpr int64_t kMostStride = 1 << 22;  // 128 rows of it are offsets of 32 bits

struct Labels {
    const void *p;
    int is_64;
    unsigned classes;
    // the label of a row, -1 where it has none
    __device__ __forceinline__ int at(int64_t r) const {
        if (is_64) {
            const int64_t t = static_cast<const int64_t *>(p)[r];
            return uint64_t(t) < classes ? int(t) : -1;
        }
        const int t = static_cast<const int32_t *>(p)[r];
        return unsigned(t) < classes ? t : -1;
    }
    // of row first + r, with a 32-bit offset
    template <typename I> __device__ __forceinline__ int at(int64_t first, I r) const {
        if (is_64) return at(first + int64_t(r));
        const int t = (static_cast<const int32_t *>(p) + first)[r];
        return unsigned(t) < classes ? t : -1;
    }
};

// f over LANES neighbouring lanes, in all of them
template <int LANES, typename F> __device__ __forceinline__ float lanes_reduce(float v, F f) {
    if constexpr (LANES >= 2) v = f(v, gnn_from_lane<0xB1>(v));    // the other of a pair
    if constexpr (LANES >= 4) v = f(v, gnn_from_lane<0x4E>(v));    // the other pair of four
    if constexpr (LANES >= 8) v = f(v, gnn_from_lane<0x141>(v));   // mirrored in eight: the other four
    if constexpr (LANES >= 16) v = f(v, gnn_from_lane<0x140>(v));  // mirrored in sixteen: the other eight
    if constexpr (LANES >= 32) v = f(v, __shfl_xor(v, 16));
    if constexpr (LANES >= 64) v = f(v, __shfl_xor(v, 32));
    return v;
}
// f over a workgroup, in all of its threads; red: a value for every wavefront
template <int THREADS, typename F> __device__ __forceinline__ float group_reduce(float v, float *red, F f) {
    v = lanes_reduce<64>(v, f);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < THREADS / 64; ++i) v = f(v, red[i]);
    return v;
}
struct Add { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };
struct Max { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };  // (a NaN is met by the sum)

__device__ __forceinline__ int wave_add(int n) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) n += __shfl_xor(n, d);
    return __builtin_amdgcn_readfirstlane(n);
}

// labelled rows among r0 + threadIdx.x, every THREADS-th of them up to r1; eight loads in flight
template <int THREADS> __device__ __forceinline__ int count_rows(const Labels &labels, int64_t r0, int64_t r1) {
    constexpr int U = 8;
    int n = 0;
    for (int64_t r = r0 + threadIdx.x; r < r1; r += THREADS * U) {
        int t[U];
#pragma unroll
        for (int u = 0; u < U; ++u) t[u] = r + u * THREADS < r1 ? labels.at(r + u * THREADS) : -1;
#pragma unroll
        for (int u = 0; u < U; ++u) n += t[u] >= 0;
    }
    return n;
}
template <int THREADS> __device__ __forceinline__ int group_count(int n, int *red) {
    n = wave_add(n);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = n;
    __syncthreads();
    n = red[0];
#pragma unroll
    for (int i = 1; i < THREADS / 64; ++i) n += red[i];
    return n;
}

__global__ void __launch_bounds__(1024) count_labels_kernel(const Labels labels, int64_t N, int32_t *__restrict__ counts) {
    __shared__ int red[1024 / 64];
    const int64_t each = (N + gridDim.x - 1) / gridDim.x, r0 = each * blockIdx.x, r1 = r0 + each < N ? r0 + each : N;
    const int n = group_count<1024>(count_rows<1024>(labels, r0, r1), red);
    if (threadIdx.x == 0) counts[blockIdx.x] = n;
}

enum Weight { kSum, kMeanCounted, kMeanHere };
// scale, or scale / number of labelled rows; the same in every thread of a workgroup.  Every wavefront adds up the counts: no barrier.
template <int WEIGHT, int THREADS> __device__ __forceinline__ float row_weight(const Labels &labels, int64_t N, const int32_t *counts, float scale, int *red) {
    if constexpr (WEIGHT == kSum) return scale;
    int n = 0;
    if constexpr (WEIGHT == kMeanCounted) {
        static_assert(kCountBlocks == 4 * 64, "four counts a lane");
        const int4 c = reinterpret_cast<const int4 *>(counts)[threadIdx.x & 63];
        n = wave_add((c.x + c.y) + (c.z + c.w));
    } else n = group_count<THREADS>(count_rows<THREADS>(labels, 0, N), red);
    return scale / float(n > 1 ? n : 1);
}

// Rows in registers: LANES lanes with NV vectors of VEC elements each.  The last vector of a row ends with the row; elements that
// it shares with the one before are left out of the sum and written twice, alike.  PASSES rows a team, all fetched first.
// Addresses are 32-bit offsets from the workgroup's first row (wide strides go the other way): 64-bit products for every row are
// a good part of a row's vector instructions (2.4 M rows of 47 scores, 8 % labelled: 107 -> 98 us).  Listing the labelled rows first and sharing them
// among the teams saves instructions where labels are few and no time: 98 us, and a row per workgroup pays for its barriers (177 -> 194).
template <typename T, int VEC, int LANES, int NV, int PASSES, int WEIGHT>
__global__ void __launch_bounds__(kThreads) xent_kernel(const T *__restrict__ X, int64_t ldx, const Labels labels, T *__restrict__ dX, int64_t ldg,
                                                        float *__restrict__ loss_rows, const int32_t *__restrict__ counts, float scale,
                                                        float *__restrict__ loss_part, int64_t N, int C) {
    __shared__ float red[kThreads / 64];
    __shared__ int red_n[kThreads / 64];
    constexpr int ROWS = kThreads / LANES;
    const int lane = int(threadIdx.x) % LANES, team = LANES == kThreads ? 0 : int(threadIdx.x) / LANES;
    const unsigned sx = unsigned(ldx), sg = unsigned(ldg);
    const int vecs = (C + VEC - 1) / VEC;
    unsigned col[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) col[k] = unsigned((lane + k * LANES) * VEC < C - VEC ? (lane + k * LANES) * VEC : C - VEC);
    float sum = 0.0f, w = 0.0f;
    bool weighed = false;
    for (int64_t b0 = int64_t(blockIdx.x) * (ROWS * PASSES); b0 < N; b0 += int64_t(gridDim.x) * (ROWS * PASSES)) {
        const int left = N - b0 < ROWS * PASSES ? int(N - b0) : ROWS * PASSES;
        const T *const x0 = X + b0 * ldx;
        T *const g0 = dX ? dX + b0 * ldg : nullptr;
        int t[PASSES];
        float xt[PASSES];
        gnn_strip<T, VEC, false> strip[PASSES][NV];
#pragma unroll
        for (int q = 0; q < PASSES; ++q) t[q] = team + q * ROWS < left ? labels.at(b0, unsigned(team + q * ROWS)) : -1;
#pragma unroll
        for (int q = 0; q < PASSES; ++q)
            if (t[q] >= 0) {
                const unsigned row = unsigned(team + q * ROWS) * sx;
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    if (lane + k * LANES < vecs) strip[q][k].load(x0 + (row + col[k]));
                xt[q] = gnn_rows<T>::get(x0 + (row + unsigned(t[q])));
            }
        if (!weighed) {  // while the rows are under way
            w = row_weight<WEIGHT, kThreads>(labels, N, counts, scale, red_n);
            weighed = true;
        }
#pragma unroll
        for (int q = 0; q < PASSES; ++q) {
            const int r = team + q * ROWS;
            if (r >= left) break;
            float v[NV][VEC];
            float loss = 0.0f;
            if (t[q] >= 0) {
                float m = -__builtin_inff();
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    if (lane + k * LANES < vecs) {
                        strip[q][k].get(v[k]);
#pragma unroll
                        for (int j = 0; j < VEC; ++j) m = fmaxf(m, v[k][j]);
                    }
                if constexpr (LANES <= 64) m = lanes_reduce<LANES>(m, Max());
                else m = group_reduce<kThreads>(m, red, Max());
                float s = 0.0f;
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    if (lane + k * LANES < vecs) {
                        if constexpr (VEC == 8 && NV > 1) {
                            strip[q][k].forget();
                            strip[q][k].get(v[k]);
                        }
                        float part = 0.0f;
#pragma unroll
                        for (int j = 0; j < VEC; ++j) {
                            v[k][j] = __expf(v[k][j] - m);
                            part += v[k][j];
                        }
                        const int over = (lane + k * LANES) * VEC - (C - VEC);  // > 0: so many elements are the vector's before, too
                        if (over > 0) {
                            part = 0.0f;
#pragma unroll
                            for (int j = 0; j < VEC; ++j) part += j >= over ? v[k][j] : 0.0f;
                        }
                        s += part;
                    }
                if constexpr (LANES <= 64) s = lanes_reduce<LANES>(s, Add());
                else s = group_reduce<kThreads>(s, red, Add());
                loss = __logf(s) + (m - xt[q]);
                const float inv = w / s;
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    const unsigned at = unsigned(t[q]) - col[k];
#pragma unroll
                    for (int j = 0; j < VEC; ++j) v[k][j] *= inv;
                    if (at < unsigned(VEC)) {  // one vector of the row, or two that share the element
#pragma unroll
                        for (int j = 0; j < VEC; ++j) v[k][j] -= j == int(at) ? w : 0.0f;
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) v[k][j] = 0.0f;
            }
            if (g0) {
                const unsigned row = unsigned(r) * sg;
#pragma unroll
                for (int k = 0; k < NV; ++k)
                    if (lane + k * LANES < vecs) gnn_store_row<T, VEC, true>(g0 + (row + col[k]), v[k]);
            }
            if (loss_rows && lane == 0) loss_rows[b0 + r] = loss;
            sum += loss;
        }
    }
    sum = group_reduce<kThreads>(lane == 0 ? sum : 0.0f, red, Add());
    if (threadIdx.x == 0) loss_part[blockIdx.x] = sum * w;
}

// Rows beyond the registers: a workgroup reads its row twice, first for the running maximum and the sum of the exponentials.
template <typename T, int VEC, int WEIGHT>
__global__ void __launch_bounds__(kThreads) xent_wide_kernel(const T *__restrict__ X, int64_t ldx, const Labels labels, T *__restrict__ dX, int64_t ldg,
                                                             float *__restrict__ loss_rows, const int32_t *__restrict__ counts, float scale,
                                                             float *__restrict__ loss_part, int64_t N, int64_t C) {
    __shared__ float red[kThreads / 64];
    __shared__ int red_n[kThreads / 64];
    const float w = row_weight<WEIGHT, kThreads>(labels, N, counts, scale, red_n);
    const int64_t whole = C / VEC * VEC;
    float sum = 0.0f;
    for (int64_t r = blockIdx.x; r < N; r += gridDim.x) {
        const int t = labels.at(r);
        const T *x = X + r * ldx;
        T *g = dX ? dX + r * ldg : nullptr;
        float loss = 0.0f, top = 0.0f, inv = 0.0f;
        if (t >= 0) {
            float m = -__builtin_inff(), s = 0.0f;
            // the maximum of so many, then their exponentials; before the first finite score there is nothing to scale
            auto take = [&](const float *v, int n) {
                float up = m;
                for (int j = 0; j < n; ++j) up = fmaxf(up, v[j]);
                if (up == -__builtin_inff()) {
                    for (int j = 0; j < n; ++j) s += v[j] != v[j] ? v[j] : 0.0f;
                    return;
                }
                s *= m == up ? 1.0f : __expf(m - up);
                m = up;
                for (int j = 0; j < n; ++j) s += __expf(v[j] - m);
            };
            for (int64_t c = int64_t(threadIdx.x) * VEC; c < whole; c += int64_t(kThreads) * VEC) {
                float v[VEC];
                gnn_load_row<T, VEC>(x + c, v);
                take(v, VEC);
            }
            if (whole + threadIdx.x < C) {
                const float v = gnn_rows<T>::get(x + whole + threadIdx.x);
                take(&v, 1);
            }
            top = group_reduce<kThreads>(m, red, Max());
            s = group_reduce<kThreads>(m == -__builtin_inff() ? s : s * __expf(m - top), red, Add());
            loss = __logf(s) + (top - gnn_rows<T>::get(x + t));
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
                gnn_store_row<T, VEC, true>(g + c, v);
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

// All loads of the up to kLossBlocks values are in flight together.
template <int THREADS, int U> __global__ void __launch_bounds__(THREADS) add_losses_kernel(const float *__restrict__ part, int n, float *__restrict__ loss) {
    __shared__ double red[THREADS / 64];
    static_assert(THREADS * U * 4 <= kLossBlocks, "one round");
    float4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = (u * THREADS + int(threadIdx.x)) * 4;
        if (i + 3 < n) v[u] = *reinterpret_cast<const float4 *>(part + i);
        else v[u] = make_float4(i < n ? part[i] : 0.0f, i + 1 < n ? part[i + 1] : 0.0f, i + 2 < n ? part[i + 2] : 0.0f, 0.0f);
    }
    double s = 0.0;
#pragma unroll
    for (int u = 0; u < U; ++u) s += (double(v[u].x) + double(v[u].y)) + (double(v[u].z) + double(v[u].w));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < THREADS / 64; ++i) s += red[i];
        *loss = float(s);
    }
}

struct Call {
    Labels labels;
    float *loss_rows, *loss, *part;
    int32_t *counts;
    bool mean;
    float scale;
    int64_t N, C, ldx, ldg;
    hipStream_t stream;
};

int blocks_of(int64_t N, int rows) {
    const int64_t b = (N + rows - 1) / rows;
    return int(b < kLossBlocks ? b : kLossBlocks);
}

template <typename T, int VEC, int LANES, int NV, int PASSES, int WEIGHT> int launch(const T *X, T *dX, const Call &c) {
    const int blocks = blocks_of(c.N, kThreads / LANES * PASSES);
    xent_kernel<T, VEC, LANES, NV, PASSES, WEIGHT><<<blocks, kThreads, 0, c.stream>>>(X, c.ldx, c.labels, dX, c.ldg, c.loss_rows, c.counts, c.scale, c.part, c.N,
                                                                                  int(c.C));
    return blocks;
}

// a workgroup has one row at a time
template <typename T> bool wide(const Call &c) { return c.C > 128 * gnn_rows<T>::VEC || c.ldx >= kMostStride || c.ldg >= kMostStride; }

template <typename T, int WEIGHT> int rows(const T *X, T *dX, const Call &c) {
    constexpr int V = gnn_rows<T>::VEC;
    if (c.ldx < kMostStride && c.ldg < kMostStride) {
        if (c.C < V) return launch<T, 1, 8, 1, 4, WEIGHT>(X, dX, c);
        if (c.C <= 4 * V) return launch<T, V, 4, 1, 2, WEIGHT>(X, dX, c);
        if (c.C <= 8 * V) return launch<T, V, 8, 1, 4, WEIGHT>(X, dX, c);
        if (c.C <= 16 * V) return launch<T, V, 16, 1, 4, WEIGHT>(X, dX, c);
        if (c.C <= 32 * V) return launch<T, V, 32, 1, 4, WEIGHT>(X, dX, c);
        if (c.C <= 64 * V) return launch<T, V, 64, 1, 4, WEIGHT>(X, dX, c);
        if (c.C <= 128 * V) return launch<T, V, 64, 2, 2, WEIGHT>(X, dX, c);
        if (c.C <= 512 * V) return launch<T, V, 256, 2, 1, WEIGHT>(X, dX, c);
        if (c.C <= 1024 * V) return launch<T, V, 256, 4, 1, WEIGHT>(X, dX, c);
        if (c.C <= 1536 * V) return launch<T, V, 256, 6, 1, WEIGHT>(X, dX, c);
        if (c.C <= 2048 * V) return launch<T, V, 256, 8, 1, WEIGHT>(X, dX, c);
    }
    const int blocks = blocks_of(c.N, 1);
    xent_wide_kernel<T, V, WEIGHT><<<blocks, kThreads, 0, c.stream>>>(X, c.ldx, c.labels, dX, c.ldg, c.loss_rows, c.counts, c.scale, c.part, c.N, c.C);
    return blocks;
}

template <typename T> int xent(const T *X, T *dX, const Call &c) {
    int blocks;
    if (!c.mean) blocks = rows<T, kSum>(X, dX, c);
    else if (c.N <= (wide<T>(c) ? kCountHereWide : kCountHere)) blocks = rows<T, kMeanHere>(X, dX, c);
    else {
        count_labels_kernel<<<kCountBlocks, 1024, 0, c.stream>>>(c.labels, c.N, c.counts);
        blocks = rows<T, kMeanCounted>(X, dX, c);
    }
    if (blocks <= 1024) add_losses_kernel<256, 1><<<1, 256, 0, c.stream>>>(c.part, blocks, c.loss);
    else if (blocks <= 16384) add_losses_kernel<1024, 4><<<1, 1024, 0, c.stream>>>(c.part, blocks, c.loss);
    else add_losses_kernel<1024, 16><<<1, 1024, 0, c.stream>>>(c.part, blocks, c.loss);
    GNN_HIP_TRY(hipGetLastError());
    return GNN_OK;
}

__global__ void zero_loss_kernel(float *loss) { *loss = 0.0f; }

}  // namespace

extern "C" GNN_API int64_t gnn_softmax_xent_workspace_bytes(int64_t N, int64_t C) {
    if (N <= 0 || C <= 0) return 0;
    return kCountBlocks * 4 + (N < kLossBlocks ? N : kLossBlocks) * 4;
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
    c.labels = Labels{labels, o.labels_is_64, unsigned(C)};
    c.mean = o.reduction == GNN_LOSS_MEAN;
    c.counts = static_cast<int32_t *>(o.workspace);
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
