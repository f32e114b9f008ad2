// Group norm with an activation over vertex features, channels last, and its gradients.
//
// A sample is a run of rows (a graph of a batch; the whole graph; one vertex), a group K = C / G neighbouring channels.  With
// n = rows of the sample * K, per sample and group
//     mean = sum x / n,  var = sum (x - mean)^2 / n,  rstd = 1 / sqrt(var + eps),
//     xh = (x - mean) rstd,  z = xh gamma[c] + beta[c],  y = act(z);
// backward, with dz = dY act'(z):
//     dbeta[c] = sum dz,  dgamma[c] = sum dz xh  (over all rows),
//     s1 = sum dz gamma / n,  s2 = sum dz gamma xh / n  (over the sample and group),  dX = rstd (dz gamma - s1 - xh s2).
//
// Rows are cut into tiles of equal size whatever the samples' sizes are, one workgroup each.  A tile adds up each sample's part of
// it per column; the partial sums of tile t and sample b lie in slot t + b (from one pair to the next at least one of the two
// grows, so no two share a slot).  A second kernel merges the slots of every sample, in their order: results do not depend on
// timing.  A third reads the rows again and writes the result.
#include "common.h"
#include "rows.h"

namespace {

constexpr int kThreads = 256;
constexpr int64_t kMaxTiles = 2048;  // as many workgroups as are resident at once

// Rows of every sample: from `ptr` (ragged), or `rows` of them each.  What ptr holds is kept inside the matrix.
struct Samples {
    const void *ptr;
    int is_64;
    int64_t rows, count, N;
    __device__ __forceinline__ int64_t begin(int64_t b) const {
        if (!ptr) return b * rows;
        const int64_t v = is_64 ? static_cast<const int64_t *>(ptr)[b] : int64_t(static_cast<const int32_t *>(ptr)[b]);
        return v < 0 ? 0 : v > N ? N : v;
    }
    // the first sample that ends behind `row`
    __device__ __forceinline__ int64_t of(int64_t row) const {
        if (!ptr) return row / rows;
        int64_t lo = 0, hi = count;
        while (lo < hi) {
            const int64_t mid = (lo + hi) >> 1;
            if (begin(mid + 1) > row) hi = mid;
            else lo = mid + 1;
        }
        return lo;
    }
};

template <int ACT> __device__ __forceinline__ float activate(float z) {
    if constexpr (ACT == GNN_ACT_RELU) return z > 0.0f ? z : z == z ? 0.0f : z;  // NaN stays
    else if constexpr (ACT == GNN_ACT_SILU) return z / (1.0f + __expf(-z));
    else return z;
}
// the activation's derivative
template <int ACT> __device__ __forceinline__ float slope(float z) {
    if constexpr (ACT == GNN_ACT_RELU) return z > 0.0f ? 1.0f : z == z ? 0.0f : z;
    else if constexpr (ACT == GNN_ACT_SILU) {
        const float s = 1.0f / (1.0f + __expf(-z));
        return s * (1.0f + z * (1.0f - s));
    } else return 1.0f;
}

struct Shape {
    Samples samples;
    int64_t N, tile_rows;
    int C, group_width, G;
    int cols;       // vectors of columns of a workgroup; threads: cols x row_lanes
    int row_lanes;
};

// What a thread of a tile works on: VEC neighbouring columns from `col`, every row_lanes-th row.  The last vector of a row starts
// where it ends with the row: columns that it shares with the one before are computed twice, to the same bits.
template <int VEC> struct Place {
    int lane, row_lane, col;
    bool active;
    __device__ __forceinline__ explicit Place(const Shape &s) {
        lane = int(threadIdx.x) % s.cols;
        row_lane = int(threadIdx.x) / s.cols;
        const int vec = int(blockIdx.y) * s.cols + lane;
        active = row_lane < s.row_lanes && vec * VEC < s.C;
        col = vec * VEC < s.C - VEC ? vec * VEC : s.C - VEC;
    }
};

// Runs f(sample, first row, row behind the last) for the parts of the samples in this workgroup's tile.  The same for all threads.
template <typename F> __device__ __forceinline__ void for_parts(const Shape &s, F f) {
    const int64_t r0 = int64_t(blockIdx.x) * s.tile_rows;
    const int64_t r1 = r0 + s.tile_rows < s.N ? r0 + s.tile_rows : s.N;
    int64_t row = r0;
    for (int64_t b = s.samples.of(r0); b < s.samples.count && row < r1; ++b) {
        const int64_t end = s.samples.begin(b + 1);
        const int64_t stop = end < r1 ? end : r1;
        if (stop <= row) continue;
        f(b, row, stop);
        row = stop;
    }
}

// Per part and column: the mean and the sum of squared distances from it.  Sums are taken of the distances from the thread's first
// row, which is of the values' own size, so that a mean far from zero costs no bits.
template <typename T, int VEC>
__global__ void __launch_bounds__(kThreads) norm_part_kernel(const T *__restrict__ X, int64_t ldx, const Shape s, float2 *__restrict__ part) {
    __shared__ float red_mean[kThreads * VEC], red_m2[kThreads * VEC];
    const Place<VEC> at(s);
    for_parts(s, [&](int64_t b, int64_t row, int64_t stop) {
        float mean[VEC], m2[VEC];
        const int64_t first = row + at.row_lane;
        if (at.active && first < stop) {
            float pivot[VEC], s1[VEC], s2[VEC];
            gnn_load_row<T, VEC>(X + first * ldx + at.col, pivot);
#pragma unroll
            for (int j = 0; j < VEC; ++j) s1[j] = s2[j] = 0.0f;
            int n = 1;
            for (int64_t r = first + s.row_lanes; r < stop; r += s.row_lanes, ++n) {
                float x[VEC];
                gnn_load_row<T, VEC>(X + r * ldx + at.col, x);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float d = x[j] - pivot[j];
                    s1[j] += d;
                    s2[j] += d * d;
                }
            }
            const float inv = 1.0f / float(n);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                mean[j] = pivot[j] + s1[j] * inv;
                m2[j] = s2[j] - s1[j] * s1[j] * inv;
                m2[j] = m2[j] < 0.0f ? 0.0f : m2[j];
            }
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            red_mean[threadIdx.x * VEC + j] = mean[j];
            red_m2[threadIdx.x * VEC + j] = m2[j];
        }
        __syncthreads();
        if (at.active && at.row_lane == 0) {
            const int64_t rows = stop - row;
            const int lanes = rows < s.row_lanes ? int(rows) : s.row_lanes;
            const int64_t full = rows / s.row_lanes, rest = rows % s.row_lanes;
            float2 out[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                float sum = 0.0f;
                const float base = red_mean[at.lane * VEC + j];
                for (int l = 0; l < lanes; ++l) sum += float(full + (l < rest)) * (red_mean[(l * s.cols + at.lane) * VEC + j] - base);
                const float m = base + sum / float(rows);
                float q = 0.0f;
                for (int l = 0; l < lanes; ++l) {
                    const int i = (l * s.cols + at.lane) * VEC + j;
                    const float d = red_mean[i] - m;
                    q += red_m2[i] + float(full + (l < rest)) * d * d;
                }
                out[j] = make_float2(m, q);
            }
            float2 *o = part + (int64_t(blockIdx.x) + b) * s.C + at.col;
#pragma unroll
            for (int j = 0; j < VEC; ++j) o[j] = out[j];
        }
        __syncthreads();
    });
}

template <int THREADS> __device__ __forceinline__ double team_sum(double v, double *red) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    if constexpr (THREADS > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0;
        for (int i = 0; i < THREADS / 64; ++i) v += red[i];
    }
    return v;
}

// Mean and reciprocal deviation of a sample and group from its parts: THREADS threads for a pair.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) norm_stats_kernel(const float2 *__restrict__ part, const Shape s, float eps, float *__restrict__ mean,
                                                             float *__restrict__ rstd) {
    __shared__ double red[THREADS / 64];
    const int64_t pairs = s.samples.count * s.G;
    for (int64_t p = blockIdx.x; p < pairs; p += gridDim.x) {
        const int64_t b = p / s.G;
        const int g = int(p % s.G);
        const int64_t lo = s.samples.begin(b), hi = s.samples.begin(b + 1);
        double m = 0.0, q = 0.0;
        const double n = double(hi > lo ? hi - lo : 0) * s.group_width;
        if (hi > lo) {
            const int64_t t0 = lo / s.tile_rows, t1 = (hi - 1) / s.tile_rows;
            const int64_t items = (t1 - t0 + 1) * s.group_width;
            for (int64_t i = threadIdx.x; i < items; i += THREADS) {
                const int64_t t = t0 + i / s.group_width;
                const int64_t r0 = t * s.tile_rows > lo ? t * s.tile_rows : lo;
                const int64_t r1 = (t + 1) * s.tile_rows < hi ? (t + 1) * s.tile_rows : hi;
                m += double(r1 - r0) * part[(t + b) * s.C + g * s.group_width + i % s.group_width].x;
            }
            m = team_sum<THREADS>(m, red) / n;
            for (int64_t i = threadIdx.x; i < items; i += THREADS) {
                const int64_t t = t0 + i / s.group_width;
                const int64_t r0 = t * s.tile_rows > lo ? t * s.tile_rows : lo;
                const int64_t r1 = (t + 1) * s.tile_rows < hi ? (t + 1) * s.tile_rows : hi;
                const float2 v = part[(t + b) * s.C + g * s.group_width + i % s.group_width];
                const double d = v.x - m;
                q += double(v.y) + double(r1 - r0) * d * d;
            }
            q = team_sum<THREADS>(q, red) / n;
        }
        if (threadIdx.x == 0) {
            mean[p] = float(m);
            rstd[p] = float(1.0 / sqrt(q + double(eps)));
        }
    }
}

// gamma and beta of a thread's columns, and their groups
template <int VEC> struct Affine {
    float gamma[VEC], beta[VEC];
    int group[VEC];
    __device__ __forceinline__ Affine(const Shape &s, int col, const float *g, const float *b) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            gamma[j] = g ? g[col + j] : 1.0f;
            beta[j] = b ? b[col + j] : 0.0f;
            group[j] = (col + j) / s.group_width;
        }
    }
};

template <typename T, int VEC, int ACT>
__global__ void __launch_bounds__(kThreads) norm_apply_kernel(const T *__restrict__ X, int64_t ldx, const Shape s, const float *__restrict__ gamma,
                                                              const float *__restrict__ beta, const float *__restrict__ mean,
                                                              const float *__restrict__ rstd, T *__restrict__ Y, int64_t ldy) {
    const Place<VEC> at(s);
    if (!at.active) return;
    const Affine<VEC> aff(s, at.col, gamma, beta);
    for_parts(s, [&](int64_t b, int64_t row, int64_t stop) {
        float m[VEC], a[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            m[j] = mean[b * s.G + aff.group[j]];
            a[j] = rstd[b * s.G + aff.group[j]] * aff.gamma[j];
        }
        for (int64_t r = row + at.row_lane; r < stop; r += s.row_lanes) {
            float x[VEC];
            gnn_load_row<T, VEC>(X + r * ldx + at.col, x);
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[j] = activate<ACT>((x[j] - m[j]) * a[j] + aff.beta[j]);
            gnn_store_row<T, VEC>(Y + r * ldy + at.col, x);
        }
    });
}

// Per part and column: sum dz and sum dz xh; per tile and column their sums over its parts (total; NULL where there is one sample).
template <typename T, int VEC, int ACT>
__global__ void __launch_bounds__(kThreads) norm_bwd_part_kernel(const T *__restrict__ X, int64_t ldx, const T *__restrict__ dY, int64_t ldy, const Shape s,
                                                                 const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                 const float *__restrict__ mean, const float *__restrict__ rstd,
                                                                 float2 *__restrict__ part, float2 *__restrict__ total) {
    __shared__ float red_1[kThreads * VEC], red_x[kThreads * VEC];
    const Place<VEC> at(s);
    const Affine<VEC> aff(s, at.col, gamma, beta);
    float t1[VEC], tx[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) t1[j] = tx[j] = 0.0f;
    for_parts(s, [&](int64_t b, int64_t row, int64_t stop) {
        float a1[VEC], ax[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) a1[j] = ax[j] = 0.0f;
        if (at.active) {
            float m[VEC], r[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                m[j] = mean[b * s.G + aff.group[j]];
                r[j] = rstd[b * s.G + aff.group[j]];
            }
            for (int64_t i = row + at.row_lane; i < stop; i += s.row_lanes) {
                float x[VEC], d[VEC];
                gnn_load_row<T, VEC>(X + i * ldx + at.col, x);
                gnn_load_row<T, VEC>(dY + i * ldy + at.col, d);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float xh = (x[j] - m[j]) * r[j];
                    const float dz = d[j] * slope<ACT>(xh * aff.gamma[j] + aff.beta[j]);
                    a1[j] += dz;
                    ax[j] += dz * xh;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            red_1[threadIdx.x * VEC + j] = a1[j];
            red_x[threadIdx.x * VEC + j] = ax[j];
        }
        __syncthreads();
        if (at.active && at.row_lane == 0) {
            float2 *o = part + (int64_t(blockIdx.x) + b) * s.C + at.col;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                float u1 = 0.0f, ux = 0.0f;
                for (int l = 0; l < s.row_lanes; ++l) {
                    u1 += red_1[(l * s.cols + at.lane) * VEC + j];
                    ux += red_x[(l * s.cols + at.lane) * VEC + j];
                }
                o[j] = make_float2(u1, ux);
                t1[j] += u1;
                tx[j] += ux;
            }
        }
        __syncthreads();
    });
    if (total && at.active && at.row_lane == 0) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) total[int64_t(blockIdx.x) * s.C + at.col + j] = make_float2(t1[j], tx[j]);
    }
}

// s1 and s2 of a sample and group from its parts.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) norm_bwd_stats_kernel(const float2 *__restrict__ part, const Shape s, const float *__restrict__ gamma,
                                                                 float2 *__restrict__ sums) {
    __shared__ double red[THREADS / 64];
    const int64_t pairs = s.samples.count * s.G;
    for (int64_t p = blockIdx.x; p < pairs; p += gridDim.x) {
        const int64_t b = p / s.G;
        const int g = int(p % s.G);
        const int64_t lo = s.samples.begin(b), hi = s.samples.begin(b + 1);
        if (hi <= lo) continue;
        const int64_t t0 = lo / s.tile_rows, t1 = (hi - 1) / s.tile_rows;
        const int64_t items = (t1 - t0 + 1) * s.group_width;
        double u1 = 0.0, ux = 0.0;
        for (int64_t i = threadIdx.x; i < items; i += THREADS) {
            const int c = g * s.group_width + int(i % s.group_width);
            const float2 v = part[(t0 + i / s.group_width + b) * s.C + c];
            const double w = gamma ? gamma[c] : 1.0f;
            u1 += w * v.x;
            ux += w * v.y;
        }
        u1 = team_sum<THREADS>(u1, red);
        ux = team_sum<THREADS>(ux, red);
        const double n = double(hi - lo) * s.group_width;
        if (threadIdx.x == 0) sums[p] = make_float2(float(u1 / n), float(ux / n));
    }
}

// dbeta and dgamma: the sums of all tiles' totals, 16 columns and 16 row lanes a workgroup.
__global__ void __launch_bounds__(256) norm_bwd_columns_kernel(const float2 *__restrict__ total, int64_t tiles, int C, float *__restrict__ dgamma,
                                                               float *__restrict__ dbeta) {
    __shared__ double red_1[256], red_x[256];
    const int c = int(blockIdx.x) * 16 + int(threadIdx.x & 15);
    double u1 = 0.0, ux = 0.0;
    if (c < C)
        for (int64_t t = threadIdx.x >> 4; t < tiles; t += 16) {
            const float2 v = total[t * C + c];
            u1 += v.x;
            ux += v.y;
        }
    red_1[threadIdx.x] = u1;
    red_x[threadIdx.x] = ux;
    __syncthreads();
    if (threadIdx.x < 16 && c < C) {
        for (int l = 1; l < 16; ++l) {
            u1 += red_1[l * 16 + threadIdx.x];
            ux += red_x[l * 16 + threadIdx.x];
        }
        if (dbeta) dbeta[c] = float(u1);
        if (dgamma) dgamma[c] = float(ux);
    }
}

template <typename T, int VEC, int ACT>
__global__ void __launch_bounds__(kThreads) norm_bwd_apply_kernel(const T *__restrict__ X, int64_t ldx, const T *__restrict__ dY, int64_t ldy, const Shape s,
                                                                  const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                  const float *__restrict__ mean, const float *__restrict__ rstd,
                                                                  const float2 *__restrict__ sums, T *__restrict__ dX, int64_t lddx) {
    const Place<VEC> at(s);
    if (!at.active) return;
    const Affine<VEC> aff(s, at.col, gamma, beta);
    for_parts(s, [&](int64_t b, int64_t row, int64_t stop) {
        float m[VEC], r[VEC];
        float2 u[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            m[j] = mean[b * s.G + aff.group[j]];
            r[j] = rstd[b * s.G + aff.group[j]];
            u[j] = sums[b * s.G + aff.group[j]];
        }
        for (int64_t i = row + at.row_lane; i < stop; i += s.row_lanes) {
            float x[VEC], d[VEC];
            gnn_load_row<T, VEC>(X + i * ldx + at.col, x);
            gnn_load_row<T, VEC>(dY + i * ldy + at.col, d);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float xh = (x[j] - m[j]) * r[j];
                const float dz = d[j] * slope<ACT>(xh * aff.gamma[j] + aff.beta[j]);
                x[j] = r[j] * (dz * aff.gamma[j] - u[j].x - xh * u[j].y);
            }
            gnn_store_row<T, VEC>(dX + i * lddx + at.col, x);
        }
    });
}

// ---------------------------------------------------------------- host

int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// A tile has at least about 4096 values, and there are at most kMaxTiles of them.
int64_t tile_rows_of(int64_t N, int64_t C) {
    const int64_t least = C < 1024 ? 4096 / C : 4;
    const int64_t even = (N + kMaxTiles - 1) / kMaxTiles;
    return even > least ? even : least;
}

struct Layout {
    int64_t tile_rows, tiles, part_off, total_off, sums_off, bytes;
};

Layout layout_of(int64_t N, int64_t C, int64_t G, int64_t B, bool backward) {
    Layout L{};
    L.tile_rows = tile_rows_of(N, C);
    L.tiles = (N + L.tile_rows - 1) / L.tile_rows;
    int64_t off = round_up((L.tiles + B) * C * int64_t(sizeof(float2)), 256);
    if (backward) {
        L.total_off = off;
        if (B > 1) off += round_up(L.tiles * C * int64_t(sizeof(float2)), 256);
        L.sums_off = off;
        off += round_up(B * G * int64_t(sizeof(float2)), 256);
    }
    L.bytes = off;
    return L;
}

int check_norm(int64_t N, int64_t C, int64_t G, int64_t B, const void *sample_ptr, const gnn_norm_opts *opts, gnn_norm_opts &o) {
    if (!opts) return GNN_ERR_INVALID_ARG;
    o = *opts;
    if (o.dtype != GNN_F32 && o.dtype != GNN_BF16) return GNN_ERR_INVALID_ARG;
    if (o.act < GNN_ACT_NONE || o.act > GNN_ACT_SILU) return GNN_ERR_INVALID_ARG;
    if (N < 0 || C < 0 || B < 0 || G <= 0 || N > INT64_MAX / 2 || C > (1 << 24) || B > INT32_MAX || N > INT32_MAX) return GNN_ERR_INVALID_ARG;
    if (C % G) return GNN_ERR_INVALID_ARG;
    if (!(o.eps >= 0.0f)) return GNN_ERR_INVALID_ARG;
    if (N > 0 && (B == 0 || (!sample_ptr && N % B))) return GNN_ERR_INVALID_ARG;
    if (o.ldx == 0) o.ldx = C;
    if (o.ldy == 0) o.ldy = C;
    if (o.lddx == 0) o.lddx = C;
    if (o.ldx < C || o.ldy < C || o.lddx < C || o.max_sample_rows < 0) return GNN_ERR_INVALID_ARG;
    return GNN_OK;
}

Shape shape_of(int64_t N, int64_t C, int64_t G, int64_t B, const void *sample_ptr, const gnn_norm_opts &o, const Layout &L, int vec, dim3 *grid) {
    Shape s{};
    s.samples.ptr = sample_ptr;
    s.samples.is_64 = o.ptr_is_64;
    s.samples.count = B;
    s.samples.rows = sample_ptr ? 0 : N / B;
    s.samples.N = N;
    s.N = N;
    s.C = int(C);
    s.G = int(G);
    s.group_width = int(C / G);
    s.tile_rows = L.tile_rows;
    const int64_t vecs = (C + vec - 1) / vec, chunks = (vecs + kThreads - 1) / kThreads;
    s.cols = int((vecs + chunks - 1) / chunks);
    s.row_lanes = kThreads / s.cols;
    *grid = dim3(unsigned(L.tiles), unsigned(chunks));
    return s;
}

template <typename T, int VEC>
int norm_fwd(const T *X, const float *gamma, const float *beta, T *Y, float *mean, float *rstd, Shape s, dim3 grid, const gnn_norm_opts &o, const Layout &L) {
    hipStream_t stream = static_cast<hipStream_t>(o.stream);
    float2 *part = static_cast<float2 *>(o.workspace);
    norm_part_kernel<T, VEC><<<grid, kThreads, 0, stream>>>(X, o.ldx, s, part);
    const int64_t pairs = s.samples.count * s.G;
    if (pairs < 4096) norm_stats_kernel<256><<<unsigned(pairs), 256, 0, stream>>>(part, s, o.eps, mean, rstd);
    else norm_stats_kernel<64><<<unsigned(pairs < 65536 ? pairs : 65536), 64, 0, stream>>>(part, s, o.eps, mean, rstd);
    if (o.act == GNN_ACT_RELU) norm_apply_kernel<T, VEC, GNN_ACT_RELU><<<grid, kThreads, 0, stream>>>(X, o.ldx, s, gamma, beta, mean, rstd, Y, o.ldy);
    else if (o.act == GNN_ACT_SILU) norm_apply_kernel<T, VEC, GNN_ACT_SILU><<<grid, kThreads, 0, stream>>>(X, o.ldx, s, gamma, beta, mean, rstd, Y, o.ldy);
    else norm_apply_kernel<T, VEC, GNN_ACT_NONE><<<grid, kThreads, 0, stream>>>(X, o.ldx, s, gamma, beta, mean, rstd, Y, o.ldy);
    GNN_HIP_TRY(hipGetLastError());
    return GNN_OK;
}

template <typename T, int VEC, int ACT>
int norm_bwd(const T *X, const float *gamma, const float *beta, const float *mean, const float *rstd, const T *dY, T *dX, float *dgamma, float *dbeta,
             Shape s, dim3 grid, const gnn_norm_opts &o, const Layout &L) {
    hipStream_t stream = static_cast<hipStream_t>(o.stream);
    char *ws = static_cast<char *>(o.workspace);
    float2 *part = reinterpret_cast<float2 *>(ws), *sums = reinterpret_cast<float2 *>(ws + L.sums_off);
    float2 *total = s.samples.count > 1 ? reinterpret_cast<float2 *>(ws + L.total_off) : nullptr;
    norm_bwd_part_kernel<T, VEC, ACT><<<grid, kThreads, 0, stream>>>(X, o.ldx, dY, o.ldy, s, gamma, beta, mean, rstd, part, total);
    if (dgamma || dbeta)
        norm_bwd_columns_kernel<<<unsigned((s.C + 15) / 16), 256, 0, stream>>>(total ? total : part, L.tiles, s.C, dgamma, dbeta);
    if (dX) {
        const int64_t pairs = s.samples.count * s.G;
        if (pairs < 4096) norm_bwd_stats_kernel<256><<<unsigned(pairs), 256, 0, stream>>>(part, s, gamma, sums);
        else norm_bwd_stats_kernel<64><<<unsigned(pairs < 65536 ? pairs : 65536), 64, 0, stream>>>(part, s, gamma, sums);
        norm_bwd_apply_kernel<T, VEC, ACT><<<grid, kThreads, 0, stream>>>(X, o.ldx, dY, o.ldy, s, gamma, beta, mean, rstd, sums, dX, o.lddx);
    }
    GNN_HIP_TRY(hipGetLastError());
    return GNN_OK;
}

template <typename T, int VEC, typename... A> int norm_bwd_act(const gnn_norm_opts &o, A... a) {
    if (o.act == GNN_ACT_RELU) return norm_bwd<T, VEC, GNN_ACT_RELU>(a...);
    if (o.act == GNN_ACT_SILU) return norm_bwd<T, VEC, GNN_ACT_SILU>(a...);
    return norm_bwd<T, VEC, GNN_ACT_NONE>(a...);
}

__global__ void __launch_bounds__(256) norm_zero_kernel(float *__restrict__ a, float *__restrict__ b, int64_t n) {
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) {
        if (a) a[i] = 0.0f;
        if (b) b[i] = 0.0f;
    }
}

}  // namespace

extern "C" GNN_API int64_t gnn_group_norm_workspace_bytes(int64_t N, int64_t C, int64_t G, int64_t B, int backward) {
    if (N <= 0 || C <= 0 || G <= 0 || B <= 0) return 0;
    return layout_of(N, C, G, B, backward != 0).bytes;
}

extern "C" GNN_API int gnn_group_norm_fwd(const void *X, const float *gamma, const float *beta, const void *sample_ptr, void *Y, float *mean, float *rstd,
                                          int64_t N, int64_t C, int64_t G, int64_t B, const gnn_norm_opts *opts) {
    gnn_norm_opts o;
    const int rc = check_norm(N, C, G, B, sample_ptr, opts, o);
    if (rc != GNN_OK) return rc;
    if (N == 0 || C == 0) return GNN_OK;
    if (!X || !Y || !mean || !rstd || X == Y) return GNN_ERR_INVALID_ARG;
    const Layout L = layout_of(N, C, G, B, false);
    if (!o.workspace || o.workspace_bytes < L.bytes || reinterpret_cast<uintptr_t>(o.workspace) % 16) return GNN_ERR_INVALID_ARG;
    (void)hipGetLastError();
    dim3 grid;
    if (o.dtype == GNN_F32) {
        const float *x = static_cast<const float *>(X);
        float *y = static_cast<float *>(Y);
        if (C >= 4) { const Shape s = shape_of(N, C, G, B, sample_ptr, o, L, 4, &grid); return norm_fwd<float, 4>(x, gamma, beta, y, mean, rstd, s, grid, o, L); }
        const Shape s = shape_of(N, C, G, B, sample_ptr, o, L, 1, &grid);
        return norm_fwd<float, 1>(x, gamma, beta, y, mean, rstd, s, grid, o, L);
    }
    const gnn_bf16 *x = static_cast<const gnn_bf16 *>(X);
    gnn_bf16 *y = static_cast<gnn_bf16 *>(Y);
    if (C >= 8) { const Shape s = shape_of(N, C, G, B, sample_ptr, o, L, 8, &grid); return norm_fwd<gnn_bf16, 8>(x, gamma, beta, y, mean, rstd, s, grid, o, L); }
    const Shape s = shape_of(N, C, G, B, sample_ptr, o, L, 1, &grid);
    return norm_fwd<gnn_bf16, 1>(x, gamma, beta, y, mean, rstd, s, grid, o, L);
}

extern "C" GNN_API int gnn_group_norm_bwd(const void *X, const float *gamma, const float *beta, const float *mean, const float *rstd, const void *dY,
                                          const void *sample_ptr, void *dX, float *dgamma, float *dbeta, int64_t N, int64_t C, int64_t G, int64_t B,
                                          const gnn_norm_opts *opts) {
    gnn_norm_opts o;
    const int rc = check_norm(N, C, G, B, sample_ptr, opts, o);
    if (rc != GNN_OK) return rc;
    if (C == 0 || (!dX && !dgamma && !dbeta)) return GNN_OK;
    hipStream_t stream = static_cast<hipStream_t>(o.stream);
    (void)hipGetLastError();
    if (N == 0) {
        if (dgamma || dbeta) norm_zero_kernel<<<64, 256, 0, stream>>>(dgamma, dbeta, C);
        GNN_HIP_TRY(hipGetLastError());
        return GNN_OK;
    }
    if (!X || !dY || !mean || !rstd || dX == X || dX == dY) return GNN_ERR_INVALID_ARG;
    const Layout L = layout_of(N, C, G, B, true);
    if (!o.workspace || o.workspace_bytes < L.bytes || reinterpret_cast<uintptr_t>(o.workspace) % 16) return GNN_ERR_INVALID_ARG;
    dim3 grid;
    if (o.dtype == GNN_F32) {
        const float *x = static_cast<const float *>(X), *dy = static_cast<const float *>(dY);
        float *dx = static_cast<float *>(dX);
        if (C >= 4) {
            const Shape s = shape_of(N, C, G, B, sample_ptr, o, L, 4, &grid);
            return norm_bwd_act<float, 4>(o, x, gamma, beta, mean, rstd, dy, dx, dgamma, dbeta, s, grid, o, L);
        }
        const Shape s = shape_of(N, C, G, B, sample_ptr, o, L, 1, &grid);
        return norm_bwd_act<float, 1>(o, x, gamma, beta, mean, rstd, dy, dx, dgamma, dbeta, s, grid, o, L);
    }
    const gnn_bf16 *x = static_cast<const gnn_bf16 *>(X), *dy = static_cast<const gnn_bf16 *>(dY);
    gnn_bf16 *dx = static_cast<gnn_bf16 *>(dX);
    if (C >= 8) {
        const Shape s = shape_of(N, C, G, B, sample_ptr, o, L, 8, &grid);
        return norm_bwd_act<gnn_bf16, 8>(o, x, gamma, beta, mean, rstd, dy, dx, dgamma, dbeta, s, grid, o, L);
    }
    const Shape s = shape_of(N, C, G, B, sample_ptr, o, L, 1, &grid);
    return norm_bwd_act<gnn_bf16, 1>(o, x, gamma, beta, mean, rstd, dy, dx, dgamma, dbeta, s, grid, o, L);
}
