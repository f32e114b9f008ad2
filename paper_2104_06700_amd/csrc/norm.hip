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
// Sums of up to a few tens of values are formed in fp32, what they come to is joined in 64 bits or in a second level of fp32.  Neither statistic is a difference of
// large numbers: variances are sums of squared distances from the mean or from a value close to it, and a mean keeps what fp32 rounds off it until the
// result is formed.  The backward pass is given the rounded one.
//
// Three ways.  Rows that are samples of their own stay in the registers of a few lanes (row_kernel, row_bwd_kernel; 2.4 M x 256 fp32 in one group 851 us =
// 5.9 TB/s, gradients 1457 = 5.2).  Samples that fit a workgroup, or nearly, are read once and done in one launch (small_kernel, small_bwd_kernel; 2,449
// graphs of 25 vertices x 100 fp32 forward 21 us, gradients 31, bound by the chain load, sum, barrier, store of each).  All others: the
// rows are cut into tiles of equal size whatever the samples' sizes are, one workgroup each, which adds up each sample's part of
// it per column.  A sample inside a tile is finished there; of one that crosses tiles, each leaves its partial sums in a slot of its own, and a second
// kernel merges them in their order: results do not depend on timing.  A third reads the rows again and writes the result.  Both readers are bound by the
// memory: 2.4 M x 256 fp32 in 32 groups forward 385 us (6.5 TB/s) and 777 (6.5), gradients 743 (6.8) and 1190 (6.3), merging 12 to 14.
#include "common.h"
#include "rows.h"

namespace {

// Tiles of at least kTileValues values, at most kTiles of them with kThreads threads each; matrices of kLarge values and more in kLargeTiles with
// kLargeThreads.  Few tiles are few partial sums to merge (103 K x 141 bf16 in 3 groups, backward, 512 tiles 43 us, 1024 49, 2048 of half the threads
// 47); beside much data that does not count (2.4 M x 256 fp32 forward, 512 tiles 1154 us, 2048 of half the threads 1171; 3.5 M x 128 bf16 backward 748, 738).
constexpr int kThreads = 512, kLargeThreads = 256;
constexpr int64_t kTiles = 512, kLargeTiles = 2048, kLarge = int64_t(1) << 28, kTileValues = 16384;
constexpr int64_t kSmallParts = 4096;   // at most so many workgroups of samples that fit one leave column sums
constexpr int64_t kRowParts = 2048;     // and of workgroups that have samples of one row
constexpr int64_t kJoined = 4096;       // partial sums that the writing kernel joins by itself
constexpr int64_t kSlice = 1024;        // columns of many samples that a workgroup of tiles has at once

// A dimension of a grid has less than 2^32 threads.  Kernels with a thread for every piece of the rows spread their workgroups over x and z.
__device__ __forceinline__ int64_t workgroup() { return int64_t(blockIdx.z) * gridDim.x + blockIdx.x; }
constexpr int64_t most_workgroups(int64_t threads) { return ((int64_t(1) << 32) - 1) / threads; }
dim3 spread(int64_t workgroups, unsigned y, unsigned threads) {  // threads: of a workgroup in x
    const int64_t most = most_workgroups(threads), z = (workgroups + most - 1) / most;
    return dim3(unsigned((workgroups + z - 1) / z), y, unsigned(z));
}

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
        if (!ptr) return count == 1 ? 0 : int64_t(uint32_t(row) / uint32_t(rows));
        int64_t lo = 0, hi = count;
        while (lo < hi) {
            const int64_t mid = (lo + hi) >> 1;
            if (begin(mid + 1) > row) hi = mid;
            else lo = mid + 1;
        }
        return lo;
    }
};

constexpr float kLog2e = 1.44269504088896340736f;
// 1 / (1 + exp(-z)): exp2 of a product, sum, reciprocal
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * z)); }
template <int ACT> __device__ __forceinline__ float activate(float z) {
    if constexpr (ACT == GNN_ACT_RELU) return z > 0.0f ? z : z == z ? 0.0f : z;  // NaN stays
    else if constexpr (ACT == GNN_ACT_SILU) return z * sigmoid(z);
    else return z;
}
// the activation's derivative
template <int ACT> __device__ __forceinline__ float slope(float z) {
    if constexpr (ACT == GNN_ACT_RELU) return z > 0.0f ? 1.0f : z == z ? 0.0f : z;
    else if constexpr (ACT == GNN_ACT_SILU) {
        const float s = sigmoid(z);
        return s + s * (z - z * s);
    } else return 1.0f;
}

// rstd (dz gamma - s1 - xh s2).  The product is rounded by itself, as in the sum that s1 is: where a group has one value it is s1, and the
// gradient exactly 0.
__device__ __forceinline__ float gradient(float dz, float gamma, float xh, float r, float2 s) {
#pragma clang fp contract(off)
    const float t = dz * gamma;
    const float u = t - s.x;
    return r * __builtin_fmaf(-xh, s.y, u);
}

// a b, rounded: not part of a fused operation that takes distances from the product as it was before
__device__ __forceinline__ float product(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}
// sum / n with inv = 1 / n: what the product with inv is off by is taken back, so that the mean of equal values is that value
__device__ __forceinline__ float quotient(float sum, float n, float inv) {
    const float q = sum * inv;
    return __builtin_fmaf(__builtin_fmaf(-q, n, sum), inv, q);
}

struct Shape {
    Samples samples;
    int64_t N, tile_rows;
    int C, group_width, G;
    int cols;       // vectors of columns of a workgroup; threads: cols x row_lanes
    int row_lanes;
    int join;       // row lanes that are left after the first joining of their moments: a power of two of groups of a thread for each column
    int32_t *sample_of;  // [N] ragged samples: the sample of every row, for the kernels that write results
    bool many;      // samples: those inside a tile are finished there
    // Columns are worked on in slices of at most `slice`: of neighbouring vectors where there is one sample, else of whole groups, or a group in `pieces`
    // that one workgroup has after the other.
    int slice, pieces;
    double2 *open;  // [samples][G] what the pieces before have come to
};

// The slot of a sample's part in tile t.  Of many: at most one comes into a tile from the one before (2 t), one goes out of it (2 t + 1).
__device__ __forceinline__ int64_t slot_of(const Shape &s, int64_t t, int64_t begin) {
    return !s.many ? t : begin > t * s.tile_rows ? 2 * t + 1 : 2 * t;
}

// What a tile kernel knows when it is compiled: there is one sample; there are many; many, and groups in pieces
enum Tiles { kOneSample, kManySamples, kPieces };

// Columns c0 .. c1 - 1, in runs of `run` that belong to a group each.
template <Tiles HOW> struct Slice {
    int c0, c1, run, groups, group;  // group: the first
    bool first, last;                // piece of it
    __device__ __forceinline__ Slice(const Shape &s, int p) {
        const int y = int(blockIdx.y);
        if (HOW != kPieces) {
            c0 = y * s.slice;
            c1 = c0 + s.slice < s.C ? c0 + s.slice : s.C;
            run = s.group_width;
            group = c0 / s.group_width;
        } else {
            const int end = (y + 1) * s.group_width;
            c0 = y * s.group_width + p * s.slice;
            c1 = c0 + s.slice < end ? c0 + s.slice : end;
            run = c1 - c0;
            group = y;
        }
        groups = (c1 - c0) / run;
        first = HOW != kPieces || p == 0;
        last = HOW != kPieces || p == s.pieces - 1;
    }
};

// What a thread of a tile works on: VEC neighbouring columns from `col`, every row_lanes-th row.  The last vector of a row starts
// where it ends with the slice: columns that it shares with the one before (in a narrow last slice, with the slice before) are computed twice, to the same bits.
template <int VEC> struct Place {
    int lane, row_lane, col;
    bool active;
    template <Tiles HOW> __device__ __forceinline__ Place(const Shape &s, const Slice<HOW> &slice) {
        lane = int(threadIdx.x) % s.cols;
        row_lane = int(threadIdx.x) / s.cols;
        const int c = slice.c0 + lane * VEC;
        active = row_lane < s.row_lanes && c < slice.c1;
        col = c < slice.c1 - VEC ? c : slice.c1 - VEC;
    }
};

// Runs f(sample, first row, row behind the last) for the parts of the samples in this workgroup's tile; ONE: there is one sample.  The same for all
// threads.  map: the rows' samples are written down.
template <bool ONE, typename F> __device__ __forceinline__ void for_parts(const Shape &s, bool map, F f) {
    const int64_t r0 = int64_t(blockIdx.x) * s.tile_rows;
    const int64_t r1 = r0 + s.tile_rows < s.N ? r0 + s.tile_rows : s.N;
    if constexpr (ONE) return f(int64_t(0), r0, r1);
    int64_t row = r0;
    for (int64_t b = s.samples.of(r0); b < s.samples.count && row < r1; ++b) {
        const int64_t end = s.samples.begin(b + 1);
        const int64_t stop = end < r1 ? end : r1;
        if (stop <= row) continue;
        if (map)
            for (int64_t r = row + threadIdx.x; r < stop; r += blockDim.x) s.sample_of[r] = int32_t(b);
        f(b, row, stop);
        row = stop;
    }
}

// sums over the row lanes of a tile: red [row_lanes][cols * VEC]; the sum of lane 0's columns is left in lane 0's places
template <int VEC> __device__ __forceinline__ void add_row_lanes(float *a, float *b, const Shape &s, const Place<VEC> &at, int lanes) {
    const int width = s.cols * VEC;
    while (lanes > 1) {
        const int half = (lanes + 1) >> 1;
        __syncthreads();
        if (at.row_lane + half < lanes) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int i = at.row_lane * width + at.lane * VEC + j;
                a[i] += a[i + half * width];
                b[i] += b[i + half * width];
            }
        }
        lanes = half;
    }
    __syncthreads();
}

// Sums of `groups` runs of n values each, sixteen to one at a time, between two areas of LDS; returns where they are.  All threads of the
// workgroup call it together, `threads` of them with their number i (others with i >= threads).
__device__ __forceinline__ void add_to(float &a, float b) { a += b; }
__device__ __forceinline__ void add_to(float2 &a, float2 b) { a.x += b.x; a.y += b.y; }
__device__ __forceinline__ void add_to(double2 &a, double2 b) { a.x += b.x; a.y += b.y; }
template <typename V> __device__ __forceinline__ const V *group_sums(V *from, V *to, int groups, int n, int i, int threads) {
    while (n > 1) {
        const int out = (n + 15) >> 4;
        __syncthreads();
        if (i < threads)
            for (int k = i; k < groups * out; k += threads) {
                const int g = out == 1 ? k : int(unsigned(k) / unsigned(out)), o = k - g * out;
                V t = from[g * n + o];
                for (int e = o + out; e < n; e += out) add_to(t, from[g * n + e]);
                to[k] = t;
            }
        n = out;
        V *const swap = from;
        from = to;
        to = swap;
    }
    __syncthreads();
    return from;
}

// What a tile has in LDS, in floats: `each` for every column of a thread.  Their place is taken by what finishes samples, the columns' contributions (V) by
// group and the room to add these up, once the threads' values have been added up.
// slice: columns to finish (0: none), in groups of K or one piece of a group
template <typename V> __host__ __device__ constexpr int64_t tile_values(int64_t threads, int64_t vec, int64_t each, int64_t slice, int64_t K) {
    const int64_t run = K < slice ? K : slice, sixteenth = run > 1 ? slice / run * ((run + 15) / 16) : 0;
    const int64_t own = each * threads * vec, sums = int64_t(sizeof(V) / 4) * (slice + sixteenth);
    return (own > sums ? own : sums) + 3 & ~int64_t(3);
}

// A mean in fp32 and what it loses there.  The results are formed from both: of values whose mean is 10,000 times their deviation a half unit of
// the mean's last place is 5e-4 of the deviation.
__device__ __forceinline__ float2 two_floats(double mean) { return make_float2(float(mean), float(mean - double(float(mean)))); }

// The moments (mean, sum of squared distances from it) of a tile's row lanes, each of `each` rows and one more in the first `rest` lanes, are joined in
// LDS: mean and m2 [row_lanes][cols * VEC], the result in row lane 0's places.  A thread has a column and every `join`-th row lane, eight or
// more of them, and so on to the last sixteen at most: narrow rows have more threads a column.  About the mean of a join's first lane,
// sum n d^2 - (sum n d)^2 / n takes off at most as many times what it leaves as there are lanes in it.
__device__ __forceinline__ void join_row_lanes(double *mean, float *m2, const Shape &s, int width, int each, int rest) {
    const int group = int(threadIdx.x) / width, first = int(threadIdx.x) - group * width;
    int have = s.row_lanes;  // so many moments of each column, of the lanes l, l + have, ..
    for (int groups = s.join; have > 1; groups = groups > 16 ? groups >> 3 : 1) {
        const auto rows = [&](int l) {
            return have == s.row_lanes ? each + (l < rest) : each * ((s.row_lanes - l + have - 1) / have) + (rest > l ? (rest - l + have - 1) / have : 0);
        };
        __syncthreads();
        if (group < groups)
            for (int c = first; c < width; c += int(blockDim.x)) {
                const int at = group * width + c;
                const double center = mean[at];
                float n = float(rows(group)), a = 0.0f, q = m2[at];
                for (int l = group + groups; l < have; l += groups) {
                    const float k = float(rows(l)), d = float(mean[l * width + c] - center);
                    n += k;
                    a += k * d;
                    q += m2[l * width + c] + k * d * d;
                }
                if (n > 0.0f) {
                    const float off = a * __builtin_amdgcn_rcpf(n), rest_of = q - a * off;
                    mean[at] = center + double(off);
                    m2[at] = rest_of < 0.0f ? 0.0f : rest_of;
                }
            }
        have = groups;
    }
    __syncthreads();
}

// Per part and column: the mean and the sum of squared distances from it.  A thread takes its rows in runs of up to 32 and sums up their distances from
// a value that no single row can move far: the mean of the rows before, for the first run that of its first four.  Each run's moments are then
// joined to those of the rows before (d = difference of the means: m2 = m2 + m2' + d^2 n n' / (n + n'), all terms positive), so that
// the difference s2 - s1^2 / n takes off at most what the run is worth, whatever row comes first: with all distances taken from a part's first row instead a zero
// row in front of 16,384 of mean 100 and deviation 1 costs rstd 4e-4.
template <typename T, int VEC, bool NT, int THREADS, Tiles HOW>
__global__ void __launch_bounds__(THREADS) norm_part_kernel(const T *__restrict__ X, int64_t ldx, const Shape s, double2 *__restrict__ part, float eps,
                                                             float *__restrict__ mean_out, float *__restrict__ rstd_out, float2 *__restrict__ exact) {
    constexpr bool ONE = HOW == kOneSample;
    extern __shared__ double tile_lds[];
    double *const red_1 = tile_lds;
    float *const red_2 = reinterpret_cast<float *>(tile_lds + blockDim.x * VEC);
    double2 *const sums = reinterpret_cast<double2 *>(tile_lds);
    double *const means = tile_lds + tile_values<double2>(blockDim.x, VEC, 3, ONE ? 0 : s.slice, s.group_width) / 2;
    if (!ONE && s.samples.ptr && blockIdx.y == 0)  // samples without rows are in no tile
        for (int64_t b = int64_t(blockIdx.x) * blockDim.x + threadIdx.x; b < s.samples.count; b += int64_t(gridDim.x) * blockDim.x)
            if (s.samples.begin(b + 1) <= s.samples.begin(b))
                for (int g = 0; g < s.G; ++g) {
                    mean_out[b * s.G + g] = 0.0f;
                    rstd_out[b * s.G + g] = 1.0f / sqrtf(eps);
                }  // (no row asks for their place in `exact`)
    for (int piece = 0; piece < (HOW == kPieces ? s.pieces : 1); ++piece) {
        const Slice<HOW> slice(s, piece);
        const Place<VEC> at(s, slice);
        for_parts<ONE>(s, s.sample_of && blockIdx.y == 0 && piece == 0, [&](int64_t b, int64_t row, int64_t stop) {
            constexpr int U = 4, RUN = 32;
            const int rows = int(stop - row), each = int(unsigned(rows) / unsigned(s.row_lanes)), rest = rows - each * s.row_lanes;
            float base[VEC], off[VEC], m2[VEC];  // the mean is base + off
#pragma unroll
            for (int j = 0; j < VEC; ++j) base[j] = off[j] = m2[j] = 0.0f;
            if (at.active) {
                const T *x = X + (row + at.row_lane) * ldx + at.col;
                const int64_t step = s.row_lanes * ldx;
                int left = each + (at.row_lane < rest);  // rows of this thread
                float before = 0.0f;
                if (left > 0) {
                    float v[U][VEC];
#pragma unroll
                    for (int u = 0; u < U; ++u) gnn_load_row<T, VEC>(x + (u < left ? u : 0) * step, v[u]);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) base[j] = v[0][j] + 0.25f * ((v[1][j] - v[0][j]) + (v[2][j] - v[0][j]) + (v[3][j] - v[0][j]));
                }
                while (left > 0) {
                    const int run = left < RUN ? left : RUN;
                    float t1[VEC], t2[VEC];
#pragma unroll
                    for (int j = 0; j < VEC; ++j) t1[j] = t2[j] = 0.0f;
                    for (int k = 0; k < run; k += U, x += U * step) {
                        gnn_strip<T, VEC, NT> strip[U];
#pragma unroll
                        for (int u = 0; u < U; ++u) strip[u].load(x + (k + u < run ? u : 0) * step);
                        float v[U][VEC];
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            strip[u].get(v[u]);
                            if (u > 0)
#pragma unroll
                                for (int j = 0; j < VEC; ++j) v[u][j] = k + u < run ? v[u][j] : base[j];
                        }
#pragma unroll
                        for (int j = 0; j < VEC; ++j) {
#pragma unroll
                            for (int u = 0; u < U; ++u) v[u][j] -= base[j];
                            t1[j] += (v[0][j] + v[1][j]) + (v[2][j] + v[3][j]);
                            t2[j] += (v[0][j] * v[0][j] + v[1][j] * v[1][j]) + (v[2][j] * v[2][j] + v[3][j] * v[3][j]);
                        }
                    }
                    const float n = float(run), inv = __builtin_amdgcn_rcpf(n), share = n * __builtin_amdgcn_rcpf(before + n), weight = share * before;
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float o = t1[j] * inv, q = t2[j] - t1[j] * o;
                        const float d = o - off[j];
                        off[j] += d * share;
                        m2[j] += (q < 0.0f ? 0.0f : q) + d * d * weight;
                        const float next = base[j] + off[j];  // the next run's distances are from here
                        off[j] -= next - base[j];
                        base[j] = next;
                    }
                    before += n;
                    left -= run;
                }
            }
            if (at.active)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    red_1[threadIdx.x * VEC + j] = double(base[j]) + double(off[j]);
                    red_2[threadIdx.x * VEC + j] = m2[j];
                }
            join_row_lanes(red_1, red_2, s, s.cols * VEC, each, rest);
            const int64_t begin = ONE ? 0 : s.samples.begin(b);
            const bool whole = !ONE && begin == row && s.samples.begin(b + 1) == stop;  // the same for all threads
            const bool mine = at.active && at.row_lane == 0;
            double2 v[VEC];
            if (mine)
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[j] = make_double2(red_1[at.lane * VEC + j], red_2[at.lane * VEC + j]);
            if (!whole) {
                if (mine) {
                    double2 *o = part + slot_of(s, blockIdx.x, begin) * s.C + at.col;
#pragma unroll
                    for (int j = 0; j < VEC; ++j) o[j] = v[j];
                }
            } else {
                const double inv = 1.0 / (double(rows) * slice.run);
                const int width = slice.c1 - slice.c0, k0 = at.col - slice.c0;  // (k0 < 0: columns of the slice before)
                if (mine)
#pragma unroll
                    for (int j = 0; j < VEC; ++j)
                        if (k0 + j >= 0) means[k0 + j] = v[j].x;
                __syncthreads();
                if (mine) {
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const int k = k0 + j;
                        if (k < 0) continue;
                        const double d = v[j].x - means[k - k % slice.run];
                        sums[k] = make_double2(double(rows) * d, v[j].y + double(rows) * d * d);
                    }
                }
                const double2 *all = group_sums(sums, sums + width, slice.groups, slice.run, int(threadIdx.x), int(blockDim.x));
                for (int g = int(threadIdx.x); g < slice.groups; g += int(blockDim.x)) {
                    const double off = all[g].x * inv;
                    double var = all[g].y * inv - off * off, mid = means[g * slice.run] + off;
                    if constexpr (HOW == kPieces) {  // one group: this thread's in every piece
                        double2 so_far = make_double2(mid, var * slice.run);
                        if (!slice.first) {  // the mean, and the sum over columns of squared distances from it
                            const double2 before = s.open[b * s.G + slice.group];
                            const double n = slice.run, m = slice.c0 - int(blockIdx.y) * s.group_width, d = mid - before.x;
                            so_far = make_double2(before.x + d * (n / (m + n)), before.y + so_far.y + d * d * (m * n / (m + n)));
                        }
                        if (!slice.last) {
                            s.open[b * s.G + slice.group] = so_far;
                            continue;
                        }
                        mid = so_far.x;
                        var = so_far.y / s.group_width;
                    }
                    const int64_t p = b * s.G + slice.group + g;
                    mean_out[p] = float(mid);
                    exact[p] = two_floats(mid);
                    rstd_out[p] = 1.0f / sqrtf(float(var < 0.0 ? 0.0 : var) + eps);
                }
            }
            __syncthreads();
        });
    }
}

template <int THREADS> __device__ __forceinline__ double2 team_sum(double2 v, double2 *red) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        v.x += __shfl_xor(v.x, d);
        v.y += __shfl_xor(v.y, d);
    }
    if constexpr (THREADS > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int i = 1; i < THREADS / 64; ++i) {
            v.x += red[i].x;
            v.y += red[i].y;
        }
    }
    return v;
}

// A sample's tiles, and THREADS threads on them: `wide` neighbouring columns of a group side by side, every `deep`-th tile.
template <int THREADS> struct Merge {
    int64_t lo, hi, t0, t1;
    int wide, deep, k, d;
    bool done;  // by the tile that the sample is in
    __device__ __forceinline__ Merge(const Shape &s, int64_t b) {
        lo = s.samples.begin(b);
        hi = s.samples.begin(b + 1);
        t0 = lo / s.tile_rows;
        t1 = hi > lo ? (hi - 1) / s.tile_rows : t0 - 1;
        done = s.many && t1 <= t0;
        wide = s.group_width < THREADS ? s.group_width : THREADS;
        deep = THREADS / wide;
        k = int(threadIdx.x) % wide;
        d = int(threadIdx.x) / wide;
    }
    // f(rows of the sample in tile t, partial sums of column c there), four loads in flight
    template <typename V, typename F> __device__ __forceinline__ void tiles(const Shape &s, const V *part, int c, F f) const {
        constexpr int U = 4;
        if (d >= deep) return;
        for (int64_t t = t0 + d; t <= t1; t += U * deep) {
            V v[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (t + u * deep <= t1) v[u] = part[slot_of(s, t + u * deep, lo) * s.C + c];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t w = t + u * deep;
                if (w > t1) continue;
                const int64_t r0 = w * s.tile_rows > lo ? w * s.tile_rows : lo, r1 = (w + 1) * s.tile_rows < hi ? (w + 1) * s.tile_rows : hi;
                f(double(r1 - r0), v[u]);
            }
        }
    }
};

// Sample and group of pair p: by sample, or, where there are fewer tiles than samples, the sample that goes out of tile p / G; -1: none does.
__device__ __forceinline__ int64_t sample_of_pair(const Shape &s, int64_t p, int64_t tiles, int *group) {
    const int64_t i = p / s.G;
    *group = int(p - i * s.G);
    if (s.samples.count <= tiles) return i;
    const int64_t end = (i + 1) * s.tile_rows;
    if (end >= s.N) return -1;
    const int64_t b = s.samples.of(end - 1);
    return b < s.samples.count && s.samples.begin(b) >= i * s.tile_rows && s.samples.begin(b + 1) > end ? b : -1;
}

// Mean and reciprocal deviation of a sample and group from its parts: THREADS threads for a pair.  One sample: also for every column the mean o, and w and b of
// the result act((x - o) w + b).
template <int THREADS>
__global__ void __launch_bounds__(THREADS) norm_stats_kernel(const double2 *__restrict__ part, const Shape s, float eps, float *__restrict__ mean,
                                                             float *__restrict__ rstd, float2 *__restrict__ exact, const float *__restrict__ gamma,
                                                             const float *__restrict__ beta, float *__restrict__ table) {
    __shared__ double2 red[THREADS / 64];
    const int64_t tiles = (s.N + s.tile_rows - 1) / s.tile_rows;
    const int64_t pairs = (s.samples.count > tiles ? tiles : s.samples.count) * s.G;
    for (int64_t i = blockIdx.x; i < pairs; i += gridDim.x) {
        int group;
        const int64_t b = sample_of_pair(s, i, tiles, &group);
        if (b < 0) continue;
        const int c0 = group * s.group_width;
        const int64_t p = b * s.G + group;
        const Merge<THREADS> m(s, b);
        if (m.done) continue;
        double mid = 0.0, var = 0.0;
        if (m.hi > m.lo) {
            const double pivot = part[slot_of(s, m.t0, m.lo) * s.C + c0].x;
            double2 u = {0.0, 0.0};
            for (int k = m.k; k < s.group_width; k += m.wide)
                m.tiles(s, part, c0 + k, [&](double rows, double2 v) {
                    const double d = v.x - pivot;
                    u.x += rows * d;
                    u.y += v.y + rows * d * d;
                });
            u = team_sum<THREADS>(u, red);
            const double n = double(m.hi - m.lo) * s.group_width, off = u.x / n;
            mid = pivot + off;
            var = u.y / n - off * off;
            var = var < 0.0 ? 0.0 : var;  // (NaN stays)
        }
        const float r = float(1.0 / sqrt(var + double(eps)));
        if (threadIdx.x == 0) {
            mean[p] = float(mid);
            rstd[p] = r;
            exact[p] = two_floats(mid);
        }
        if (table)
            for (int k = int(threadIdx.x); k < s.group_width; k += THREADS) {
                const float w = gamma ? r * gamma[c0 + k] : r;
                table[c0 + k] = float(mid);
                table[s.C + c0 + k] = w;
                table[2 * int64_t(s.C) + c0 + k] = (beta ? beta[c0 + k] : 0.0f) - two_floats(mid).y * w;
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
            gamma[j] = 1.0f;
            beta[j] = 0.0f;
        }
        if (g) columns(g + col, gamma);
        if (b) columns(b + col, beta);
        const int first = col / s.group_width;
        int g0 = first, left = (first + 1) * s.group_width - col;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            if (left == 0) { ++g0; left = s.group_width; }
            group[j] = g0;
            --left;
        }
    }
    static __device__ __forceinline__ void columns(const float *p, float (&out)[VEC]) {
        if constexpr (VEC == 1) out[0] = *p;
        else
#pragma unroll
            for (int j = 0; j < VEC; j += 4) {
                const gnn_f32x4 v = *reinterpret_cast<const gnn_f32x4 *>(p + j);
                out[j] = v.x; out[j + 1] = v.y; out[j + 2] = v.z; out[j + 3] = v.w;
            }
    }
    template <typename V> __device__ __forceinline__ void gather(const Shape &s, const V *stat, int64_t b, V (&out)[VEC]) const {
        const V *p = stat + b * s.G;
        if (group[0] == group[VEC - 1]) {  // one load where a vector has one group
            const V v = p[group[0]];
#pragma unroll
            for (int j = 0; j < VEC; ++j) out[j] = v;
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j) out[j] = p[group[j]];
        }
    }
};

// The kernels that write results: a workgroup of cols x row_lanes threads has rows_of() * row_lanes neighbouring rows and ends with them, a thread
// rows_of() vectors of one column.  Small workgroups that end are faster here than ones that stay and walk: the writes
// and reads of all of them move through the matrix as one front (2.5 GB copied by one-vector threads 6.5 TB/s, four vectors 6.1, resident
// workgroups 5.0; norm of 2.4 M x 256 fp32 in workgroups of 128 threads with 1, 2, 4, 8 rows each 1301, 1170, 1225, 1242 us, of 256 threads with 2 1200).
constexpr int kBlockMost = 128;
template <int VEC> __device__ __forceinline__ int column_of_block(const Shape &s) {
    const int vec = int(blockIdx.y) * s.cols + int(threadIdx.x);
    return vec * VEC >= s.C ? -1 : vec * VEC < s.C - VEC ? vec * VEC : s.C - VEC;
}
// One sample of few tiles: the writing kernel joins their partial sums (V) by itself, every workgroup for all columns, which costs less than a
// launch.  f(partial, rows, column) -> what a column's tiles add up; g(group, sum over its columns) -> what the group keeps, in as many bytes.
// The threads are (vector of columns, row lane) of all columns.  Returns the groups' results in LDS.
template <int VEC, typename R, typename V, typename F, typename G>
__device__ __forceinline__ const R *join_tiles(const Shape &s, const V *part, int64_t tiles, int col, F f, G g) {
    static_assert(sizeof(R) == sizeof(V), "the results take the sums' places");
    extern __shared__ double2 join_lds[];
    V *const sums = reinterpret_cast<V *>(join_lds), *const next = sums + s.row_lanes * s.C;
    V u[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) u[j] = V{0, 0};
    constexpr int U = 64 / (VEC * int(sizeof(V) / 4)) < 4 ? 64 / (VEC * int(sizeof(V) / 4)) : 4;  // in at most 64 registers
    for (int64_t t = threadIdx.y; t < tiles; t += U * s.row_lanes) {
        V v[U][VEC];
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (t + k * s.row_lanes < tiles)
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[k][j] = part[(t + k * s.row_lanes) * s.C + col + j];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t w = t + k * s.row_lanes;
            if (w >= tiles) break;
            const float rows = float(w + 1 < tiles ? s.tile_rows : s.N - w * s.tile_rows);
#pragma unroll
            for (int j = 0; j < VEC; ++j) add_to(u[j], f(v[k][j], rows, col + j));
        }
    }
    const int i = int(threadIdx.y) * s.cols + int(threadIdx.x), threads = s.cols * s.row_lanes;
    int run = s.row_lanes * s.group_width;
    if (s.group_width % VEC == 0) {  // [group][row lane][vector of it]
        const int each = s.group_width / VEC, vec = col / VEC, group = int(unsigned(vec) / unsigned(each));
#pragma unroll
        for (int j = 1; j < VEC; ++j) add_to(u[0], u[j]);
        sums[(group * s.row_lanes + threadIdx.y) * each + vec - group * each] = u[0];
        run = s.row_lanes * each;
    } else {  // [group][row lane][column of it]; columns that two vectors share are written twice, alike
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const int group = int(unsigned(col + j) / unsigned(s.group_width));
            sums[(group * s.row_lanes + threadIdx.y) * s.group_width + col + j - group * s.group_width] = u[j];
        }
    }
    const V *all = group_sums(sums, next, s.G, run, i, threads);
    R *const out = reinterpret_cast<R *>(all == sums ? next : sums);
    __syncthreads();
    for (int k = i; k < s.G; k += threads) out[k] = g(k, all[k]);
    __syncthreads();
    return out;
}
__device__ __forceinline__ int64_t sample_of_row(const Shape &s, int64_t r) {
    if (!s.sample_of) return s.samples.of(r);
    const uint32_t b = uint32_t(s.sample_of[r]), last = uint32_t(s.samples.count - 1);
    return b < last ? b : last;  // a row that ptr leaves to no sample was given none
}

enum Stats { kMany, kOne, kJoin };  // statistics of many samples, of one (a table of columns), of one that has to be joined from tiles first

// rows of a thread: with two the parameters of the gradient of a bf16 vector, six for each of eight columns, are more than its data (3.5 M x 128, two
// 786 us, four 736, eight 735; its forward pass 445, 445, 448)
template <typename T> __host__ __device__ constexpr int rows_of(bool backward) { return sizeof(T) == 4 || !backward ? 2 : 4; }

template <typename T, int VEC, int ACT, bool NT, Stats STATS>
__global__ void __launch_bounds__(512) norm_apply_kernel(const T *__restrict__ X, int64_t ldx, const Shape s, const float *__restrict__ gamma,
                                                         const float *__restrict__ beta, float *__restrict__ mean, float *__restrict__ rstd,
                                                         const float2 *__restrict__ exact, T *__restrict__ Y, int64_t ldy, const double2 *__restrict__ part, float eps, const float *__restrict__ table) {
    constexpr int kRows = rows_of<T>(false);
    const int col = column_of_block<VEC>(s);
    const int64_t r0 = workgroup() * (kRows * s.row_lanes) + threadIdx.y;
    if (STATS != kJoin && (col < 0 || r0 >= s.N)) return;
    gnn_strip<T, VEC, NT> strip[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u)
        if (r0 + u * s.row_lanes < s.N) strip[u].load(X + (r0 + u * s.row_lanes) * ldx + col);
    const Affine<VEC> aff(s, col, STATS == kOne ? nullptr : gamma, STATS == kOne ? nullptr : beta);
    // z = (x - o) w + (beta - l w): the mean is o + l.  A value that is the mean gives beta where rstd is finite.
    float w[VEC], o[VEC], l[VEC], bt[VEC];
    auto fold = [&]() {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            w[j] *= aff.gamma[j];
            bt[j] = aff.beta[j] - l[j] * w[j];
        }
    };
    if constexpr (STATS == kOne) {
        if (s.group_width % VEC == 0) aff.gather(s, mean, 0, o);  // a vector has one group
        else Affine<VEC>::columns(table + col, o);
        Affine<VEC>::columns(table + s.C + col, w);
        Affine<VEC>::columns(table + 2 * int64_t(s.C) + col, bt);
    } else if constexpr (STATS == kJoin) {
        // distances from the first tile's mean of the group's first column
        const double inv = 1.0 / (double(s.N) * s.group_width);
        const float4 *stat = join_tiles<VEC, float4>(s, part, (s.N + s.tile_rows - 1) / s.tile_rows, col,
            [&](double2 v, float rows, int c) {
                const double d = v.x - part[c - c % s.group_width].x;
                return make_double2(double(rows) * d, v.y + double(rows) * d * d);
            },
            [&](int g, double2 u) {
                const double off = u.x * inv, var = u.y * inv - off * off, mid = part[g * s.group_width].x + off;
                const float2 m = two_floats(mid);
                const float4 r = make_float4(m.x, 1.0f / sqrtf(float(var < 0.0 ? 0.0 : var) + eps), m.y, 0.0f);
                if (workgroup() == 0) {
                    mean[g] = r.x;
                    rstd[g] = r.y;
                }
                return r;
            });
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            o[j] = stat[aff.group[j]].x;
            w[j] = stat[aff.group[j]].y;
            l[j] = stat[aff.group[j]].z;
        }
        fold();
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const int64_t r = r0 + u * s.row_lanes;
        if (r >= s.N) break;
        if constexpr (STATS == kMany) {
            const int64_t b = sample_of_row(s, r);
            float2 m[VEC];
            aff.gather(s, exact, b, m);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                o[j] = m[j].x;
                l[j] = m[j].y;
            }
            aff.gather(s, rstd, b, w);
            fold();
        }
        float x[VEC];
        strip[u].get(x);
#pragma unroll
        for (int j = 0; j < VEC; ++j) x[j] = activate<ACT>((x[j] - o[j]) * w[j] + bt[j]);
        gnn_store_row<T, VEC, NT>(Y + r * ldy + col, x);
    }
}

// Per part and column: sum dz and sum dz xh; per tile and column their sums over its parts (total; NULL where there is one sample).  These are added up in 64
// bits in LDS: a tile of samples of one row has as many parts as rows, and 8,192 equal terms one after the other in fp32 are off by 3e-5.
// (Four wavefronts a SIMD at most: the seven that have room in bf16 read slower, 1.1 M x 351 785 -> 808 us.)
template <typename T, int VEC, int ACT, bool NT, int THREADS, Tiles HOW>
__global__ void __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(1, 4))) norm_bwd_part_kernel(const T *__restrict__ X, int64_t ldx, const T *__restrict__ dY, int64_t ldy, const Shape s,
                                                                 const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                 const float *__restrict__ mean, const float *__restrict__ rstd,
                                                                 float2 *__restrict__ part, float2 *__restrict__ total, float2 *__restrict__ sums_out) {
    constexpr bool ONE = HOW == kOneSample;
    extern __shared__ double tile_lds[];
    float *const red_1 = reinterpret_cast<float *>(tile_lds), *const red_x = red_1 + blockDim.x * VEC;
    float2 *const sums = reinterpret_cast<float2 *>(tile_lds);
    double2 *const totals = reinterpret_cast<double2 *>(tile_lds + tile_values<float2>(blockDim.x, VEC, 2, ONE ? 0 : s.slice, s.group_width) / 2);
    for (int piece = 0; piece < (HOW == kPieces ? s.pieces : 1); ++piece) {
        const Slice<HOW> slice(s, piece);
        const Place<VEC> at(s, slice);
        const Affine<VEC> aff(s, at.col, gamma, beta);
        if (!ONE && at.row_lane == 0)
#pragma unroll
            for (int j = 0; j < VEC; ++j) totals[at.lane * VEC + j] = make_double2(0.0, 0.0);
        for_parts<ONE>(s, s.sample_of && blockIdx.y == 0 && piece == 0, [&](int64_t b, int64_t row, int64_t stop) {
            constexpr int U = 4;
            float a1[VEC], ax[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) a1[j] = ax[j] = 0.0f;
            if (at.active) {
                float o[VEC], rs[VEC];
                aff.gather(s, mean, b, o);
                aff.gather(s, rstd, b, rs);
                int64_t r = row + at.row_lane;
                while (r < stop) {
                    float c1[VEC], cx[VEC];
#pragma unroll
                    for (int j = 0; j < VEC; ++j) c1[j] = cx[j] = 0.0f;
                    for (int k = 0; k < 32 / U && r < stop; ++k, r += U * s.row_lanes) {
                        gnn_strip<T, VEC, NT> sx[U], sd[U];
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            const int64_t i = r + u * s.row_lanes;
                            if (i < stop) {
                                sx[u].load(X + i * ldx + at.col);
                                sd[u].load(dY + i * ldy + at.col);
                            }
                        }
#pragma unroll
                        for (int u = 0; u < U; ++u) {
                            if (r + u * s.row_lanes >= stop) break;
                            float x[VEC], d[VEC];
                            sx[u].get(x);
                            sd[u].get(d);
#pragma unroll
                            for (int j = 0; j < VEC; ++j) {
                                const float xh = (x[j] - o[j]) * rs[j];
                                const float dz = d[j] * slope<ACT>(xh * aff.gamma[j] + aff.beta[j]);
                                c1[j] += dz;
                                cx[j] += dz * xh;
                            }
                        }
                    }
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        a1[j] += c1[j];
                        ax[j] += cx[j];
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                red_1[threadIdx.x * VEC + j] = a1[j];
                red_x[threadIdx.x * VEC + j] = ax[j];
            }
            add_row_lanes<VEC>(red_1, red_x, s, at, s.row_lanes);
            const int64_t begin = ONE ? 0 : s.samples.begin(b);
            const bool whole = !ONE && begin == row && s.samples.begin(b + 1) == stop;  // the same for all threads
            const bool mine = at.active && at.row_lane == 0;
            float u1[VEC], ux[VEC];
            if (mine) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    u1[j] = red_1[at.lane * VEC + j];
                    ux[j] = red_x[at.lane * VEC + j];
                    if constexpr (!ONE) add_to(totals[at.lane * VEC + j], make_double2(u1[j], ux[j]));
                }
                if (!whole) {
                    float2 *o = part + slot_of(s, blockIdx.x, begin) * s.C + at.col;
#pragma unroll
                    for (int j = 0; j < VEC; ++j) o[j] = make_float2(u1[j], ux[j]);
                }
            }
            if (whole && sums_out) {
                __syncthreads();
                const int k0 = at.col - slice.c0;
                if (mine)
#pragma unroll
                    for (int j = 0; j < VEC; ++j)
                        if (k0 + j >= 0) sums[k0 + j] = make_float2(u1[j] * aff.gamma[j], ux[j] * aff.gamma[j]);
                const float2 *all = group_sums(sums, sums + (slice.c1 - slice.c0), slice.groups, slice.run, int(threadIdx.x), int(blockDim.x));
                const float n = float(stop - row) * float(s.group_width);
                for (int g = int(threadIdx.x); g < slice.groups; g += int(blockDim.x)) {
                    float2 sum = all[g];
                    if constexpr (HOW == kPieces) {  // one group: this thread's in every piece
                        double2 so_far = make_double2(sum.x, sum.y);
                        if (!slice.first) add_to(so_far, s.open[b * s.G + slice.group]);
                        if (!slice.last) {
                            s.open[b * s.G + slice.group] = so_far;
                            continue;
                        }
                        sum = make_float2(float(so_far.x), float(so_far.y));
                    }
                    sums_out[b * s.G + slice.group + g] = make_float2(sum.x / n, sum.y / n);
                }
            }
            __syncthreads();
        });
        if (!ONE && total && at.active && at.row_lane == 0) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const double2 t = totals[at.lane * VEC + j];
                total[int64_t(blockIdx.x) * s.C + at.col + j] = make_float2(float(t.x), float(t.y));
            }
        }
    }
}

// sums over the `deep` rows of THREADS / wide threads each, left in the first row; wide * deep <= THREADS
template <int THREADS> __device__ __forceinline__ double2 add_deep(double2 v, double2 *red, int wide, int deep) {
    __syncthreads();
    red[threadIdx.x] = v;
    const int d = int(threadIdx.x) / wide;
    while (deep > 1) {
        const int half = (deep + 1) >> 1;
        __syncthreads();
        if (d + half < deep) {
            red[threadIdx.x].x += red[threadIdx.x + half * wide].x;
            red[threadIdx.x].y += red[threadIdx.x + half * wide].y;
        }
        deep = half;
    }
    __syncthreads();
    return red[threadIdx.x];
}

// s1 and s2 of a sample and group from its parts.  With one sample its columns' sums are dbeta and dgamma too.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) norm_bwd_stats_kernel(const float2 *__restrict__ part, const Shape s, const float *__restrict__ gamma,
                                                                 float2 *__restrict__ sums, float *__restrict__ dgamma, float *__restrict__ dbeta,
                                                                 const float *__restrict__ mean, const float *__restrict__ rstd, float *__restrict__ table) {
    __shared__ double2 red[THREADS];
    const int64_t tiles = (s.N + s.tile_rows - 1) / s.tile_rows;
    const int64_t pairs = (s.samples.count > tiles ? tiles : s.samples.count) * s.G;
    for (int64_t i = blockIdx.x; i < pairs; i += gridDim.x) {
        int group;
        const int64_t b = sample_of_pair(s, i, tiles, &group);
        if (b < 0) continue;
        const int c0 = group * s.group_width;
        const int64_t p = b * s.G + group;
        const Merge<THREADS> m(s, b);
        if (m.done) continue;
        if (m.hi <= m.lo) continue;
        double2 all = {0.0, 0.0};
        for (int k0 = 0; k0 < s.group_width; k0 += m.wide) {
            const int c = c0 + k0 + m.k;
            const bool there = k0 + m.k < s.group_width;
            double2 u = {0.0, 0.0};
            if (there) m.tiles(s, part, c, [&](double, float2 v) { u.x += v.x; u.y += v.y; });
            if (dgamma || dbeta) {
                u = add_deep<THREADS>(u, red, m.wide, m.deep);
                if (there && m.d == 0) {
                    if (dbeta) dbeta[c] = float(u.x);
                    if (dgamma) dgamma[c] = float(u.y);
                } else u = {0.0, 0.0};
            }
            const double w = there ? gamma ? gamma[c] : 1.0f : 0.0;
            if (there) { all.x += w * u.x; all.y += w * u.y; }
        }
        all = team_sum<THREADS>(all, red);
        const double n = double(m.hi - m.lo) * s.group_width;
        if (threadIdx.x == 0 && sums) sums[p] = make_float2(float(all.x / n), float(all.y / n));
        if (table) {
            const float v[4] = {mean[p], rstd[p], float(all.x / n), float(all.y / n)};
            for (int k = int(threadIdx.x); k < s.group_width; k += THREADS)
#pragma unroll
                for (int i = 0; i < 4; ++i) table[int64_t(i) * s.C + c0 + k] = v[i];
        }
        __syncthreads();
    }
}

// dbeta and dgamma: the sums of n rows of partial sums, 16 columns and 64 row lanes a workgroup.
__global__ void __launch_bounds__(1024) norm_bwd_columns_kernel(const float2 *__restrict__ total, int64_t n, int C, float *__restrict__ dgamma,
                                                                float *__restrict__ dbeta) {
    __shared__ double2 red[16][16];
    constexpr int U = 16;
    const int c = int(blockIdx.x) * 16 + int(threadIdx.x & 15);
    double2 u = {0.0, 0.0};
    if (c < C)
        for (int64_t t = threadIdx.x >> 4; t < n; t += 64 * U) {
            float2 v[U];
#pragma unroll
            for (int k = 0; k < U; ++k) v[k] = t + 64 * k < n ? total[(t + 64 * k) * C + c] : make_float2(0.0f, 0.0f);
#pragma unroll
            for (int k = 0; k < U; ++k) { u.x += v[k].x; u.y += v[k].y; }
        }
    // the four row lanes of a wavefront, then the sixteen wavefronts
#pragma unroll
    for (int d = 16; d <= 32; d <<= 1) {
        u.x += __shfl_xor(u.x, d);
        u.y += __shfl_xor(u.y, d);
    }
    if ((threadIdx.x & 63) < 16) red[threadIdx.x >> 6][threadIdx.x & 15] = u;
    __syncthreads();
    if (threadIdx.x < 16 && c < C) {
        for (int w = 1; w < 16; ++w) {
            u.x += red[w][threadIdx.x].x;
            u.y += red[w][threadIdx.x].y;
        }
        if (dbeta) dbeta[c] = float(u.x);
        if (dgamma) dgamma[c] = float(u.y);
    }
}

template <typename T, int VEC, int ACT, bool NT, Stats STATS>
__global__ void __launch_bounds__(512) norm_bwd_apply_kernel(const T *__restrict__ X, int64_t ldx, const T *__restrict__ dY, int64_t ldy, const Shape s,
                                                             const float *__restrict__ gamma, const float *__restrict__ beta,
                                                             const float *__restrict__ mean, const float *__restrict__ rstd,
                                                             const float2 *__restrict__ sums, T *__restrict__ dX, int64_t lddx, const float2 *__restrict__ part, const float *__restrict__ table) {
    constexpr int kRows = rows_of<T>(true);
    const int col = column_of_block<VEC>(s);
    const int64_t r0 = workgroup() * (kRows * s.row_lanes) + threadIdx.y;
    if (STATS != kJoin && (col < 0 || r0 >= s.N)) return;
    gnn_strip<T, VEC, NT> sx[kRows], sd[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u)
        if (r0 + u * s.row_lanes < s.N) {
            sx[u].load(X + (r0 + u * s.row_lanes) * ldx + col);
            sd[u].load(dY + (r0 + u * s.row_lanes) * ldy + col);
        }
    const Affine<VEC> aff(s, col, gamma, beta);
    float r[VEC], o[VEC];  // xh = (x - o) r
    auto fold = [&](int64_t b) {
        aff.gather(s, mean, b, o);
        aff.gather(s, rstd, b, r);
    };
    float2 w[VEC];
    if constexpr (STATS == kOne) {
        if (s.group_width % VEC == 0) {
            aff.gather(s, sums, 0, w);
            fold(0);
        } else {
            Affine<VEC>::columns(table + col, o);
            Affine<VEC>::columns(table + s.C + col, r);
            float a[VEC], b[VEC];
            Affine<VEC>::columns(table + 2 * int64_t(s.C) + col, a);
            Affine<VEC>::columns(table + 3 * int64_t(s.C) + col, b);
#pragma unroll
            for (int j = 0; j < VEC; ++j) w[j] = make_float2(a[j], b[j]);
        }
    } else if constexpr (STATS == kJoin) {
        const float n = float(s.N) * float(s.group_width);
        const float2 *stat = join_tiles<VEC, float2>(s, part, (s.N + s.tile_rows - 1) / s.tile_rows, col,
            [&](float2 v, float, int c) {
                const float k = gamma ? gamma[c] : 1.0f;
                return make_float2(v.x * k, v.y * k);
            },
            [&](int, float2 u) { return make_float2(u.x / n, u.y / n); });
#pragma unroll
        for (int j = 0; j < VEC; ++j) w[j] = stat[aff.group[j]];
        fold(0);
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const int64_t i = r0 + u * s.row_lanes;
        if (i >= s.N) break;
        if constexpr (STATS == kMany) {
            const int64_t b = sample_of_row(s, i);
            aff.gather(s, sums, b, w);
            fold(b);
        }
        float x[VEC], d[VEC];
        sx[u].get(x);
        sd[u].get(d);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float xh = (x[j] - o[j]) * r[j];
            const float dz = d[j] * slope<ACT>(xh * aff.gamma[j] + aff.beta[j]);
            x[j] = gradient(dz, aff.gamma[j], xh, r[j], w[j]);
        }
        gnn_store_row<T, VEC, NT>(dX + i * lddx + col, x);
    }
}

// ---------------------------------------------------------------- samples that fit a workgroup

// Vectors of a thread: 16 values, in backward of each of the two matrices
template <typename T> __host__ __device__ constexpr int held() { return 16 / gnn_rows<T>::VEC; }

// A team of threads has a sample's rows of `groups` neighbouring groups in registers: cols x lanes threads, thread (lane, row
// lane) the vector `lane` of every lanes-th row.  The last vector ends with the columns: those that it shares with the one before it are computed by
// both to the same bits (a short last vector in its place was a third slower: 2,449 graphs of 25 vertices x 100 bf16, backward, 90 us and 69).  Fewer columns than a
// vector has are one short vector.
struct Small {
    Samples samples;
    int C, G, K;
    int groups;        // of a team (blockIdx.y: which); the last one may have fewer
    int cols, lanes, team, teams;
    int len;           // partial sums of a group: lanes x K, or x K / VEC where vectors lie inside groups
    int team_sums;     // pairs of a team in LDS
};

// How vectors lie: inside groups; across groups; across groups, and there is a slice of fewer columns than a vector has
enum Vectors { kInside, kAcross, kShort };

// WHOLE: a thread with columns has a whole vector.  Without the partial loads and stores the forward kernel takes a fifth fewer registers (612 graphs of
// 100 vertices x 128 fp32 in 16 groups 23 -> 17 us); the backward kernel is faster so across groups (2,449 graphs of 25 x 100 bf16 49 -> 44), slower
// inside (x 64 fp32 27 -> 30).
template <int VEC, Vectors HOW, bool WHOLE> struct Team {
    static constexpr bool INSIDE = HOW == kInside, kWhole = WHOLE;
    int team, i, lane, row_lane, col, have, c0, groups;
    bool active;
    float2 *room;  // of the team's sums, a value or a pair each
    int g0, k0;  // group of the first column, and its place there
    __device__ __forceinline__ Team(const Small &s, float2 *lds) {
        team = int(threadIdx.x / unsigned(s.team));
        i = int(threadIdx.x) - team * s.team;
        row_lane = int(unsigned(i) / unsigned(s.cols));
        lane = i - row_lane * s.cols;
        c0 = int(blockIdx.y) * s.groups * s.K;
        const int left = (s.C - c0) / s.K;
        groups = left < s.groups ? left : s.groups;
        const int columns = groups * s.K;
        col = lane * VEC < columns - VEC || columns < VEC ? lane * VEC : columns - VEC;
        have = lane * VEC >= columns ? 0 : columns < VEC ? columns : VEC;
        active = team < s.teams && row_lane < s.lanes && have > 0;
        room = lds + (team < s.teams ? team : 0) * s.team_sums;
        g0 = int(unsigned(col) / unsigned(s.K));
        k0 = col - g0 * s.K;
    }
    // f(j, group of column j, place of its sum)
    template <typename F> __device__ __forceinline__ void columns(const Small &s, F f) const {
        int g = g0, k = k0, at = g0 * s.len + row_lane * s.K + k0;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            if (kWhole || j < have) f(j, g, at);
            if constexpr (!INSIDE) {
                ++at;
                if (++k == s.K) {
                    k = 0;
                    ++g;
                    at += s.len - s.K;
                }
            }
        }
    }
    // the sums of every group over the team's threads' v; the places that are returned hold them until the next call.  Sixteen to one at a
    // time; all threads of the workgroup call it together.
    // (v: of every column, or one of all columns of a vector that lies inside a group)
    template <typename V, int S> __device__ __forceinline__ const V *reduce(const Small &s, const V (&v)[S]) const {
        static_assert(S == VEC || (INSIDE && S == 1), "columns");
        V *const sums = reinterpret_cast<V *>(room);
        __syncthreads();
        if (active) {
            if constexpr (INSIDE) {
                V t = v[0];
#pragma unroll
                for (int j = 1; j < S; ++j) add_to(t, v[j]);
                sums[g0 * s.len + row_lane * (s.K / VEC) + k0 / VEC] = t;
            } else {
                columns(s, [&](int j, int, int at) { sums[at] = v[j]; });
            }
        }
        return group_sums(sums, sums + s.groups * s.len, groups, s.len, team < s.teams ? i : s.team, s.team);
    }
};

// A thread's vectors of a sample: `mine` of them, `step` elements apart from `p` on.  The first held() are in registers; a sample of more
// rows than the caller said is fetched again by every pass.
template <typename T, typename P> struct Held {
    static constexpr int VEC = gnn_rows<T>::VEC;
    typename gnn_rows<T>::raw v[held<T>()];
    __device__ __forceinline__ static typename gnn_rows<T>::raw one(const P &t, const T *p) {
        if (P::kWhole || t.have == VEC) return gnn_rows<T>::fetch(p);
        float f[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) f[j] = j < t.have ? gnn_rows<T>::get(p + j) : 0.0f;
        return gnn_rows<T>::pack(f);
    }
    __device__ __forceinline__ void fetch(const P &t, const T *p, int64_t step, int mine) {
#pragma unroll
        for (int k = 0; k < held<T>(); ++k)
            if (k < mine) v[k] = one(t, p + k * step);
    }
    // the vector of row k, from the registers where k is a constant
    __device__ __forceinline__ void get(int k, float (&f)[VEC]) const {
        typename gnn_rows<T>::raw t = v[k];
        if constexpr (VEC == 8) asm volatile("" : "+v"(t));  // unpacked again by every pass: kept unpacked it takes twice the registers
        gnn_rows<T>::unpack(t, f);
    }
    __device__ __forceinline__ static void get_far(const P &t, const T *p, int64_t step, int k, float (&f)[VEC]) { gnn_rows<T>::unpack(one(t, p + k * step), f); }
};
template <typename T, typename P> __device__ __forceinline__ void put_row(const P &t, T *q, const float (&f)[gnn_rows<T>::VEC]) {
    constexpr int VEC = gnn_rows<T>::VEC;
    if (P::kWhole || t.have == VEC) gnn_store_row<T, VEC>(q, f);
    else
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (j < t.have) gnn_rows<T>::set(q + j, f[j]);
}
// the sample of a team: its first row, rows, and how many of them a thread has
struct Span {
    int64_t lo;
    int rows, mine;
    bool there;
    template <typename P> __device__ __forceinline__ Span(const Small &s, const P &t, int64_t b) {
        there = t.team < s.teams && b < s.samples.count;
        lo = there ? s.samples.begin(b) : 0;
        const int64_t hi = there ? s.samples.begin(b + 1) : 0;
        rows = hi > lo ? int(hi - lo) : 0;
        mine = t.active && rows > t.row_lane ? (rows - t.row_lane + s.lanes - 1) / s.lanes : 0;
    }
};

// Forward.  Mean first, then the distances from it and their squares, both from the registers; the distances' mean takes off the rounding of the first (as in
// row_kernel).
template <typename T, int ACT, Vectors HOW>
__global__ void __launch_bounds__(1024) small_kernel(const T *X, int64_t ldx, const Small s, const float *__restrict__ gamma,
                                                     const float *__restrict__ beta, float eps, float *__restrict__ mean, float *__restrict__ rstd,
                                                     T *Y, int64_t ldy) {
    extern __shared__ float2 small_lds2[];
    constexpr int VEC = gnn_rows<T>::VEC;
    typedef Team<VEC, HOW, HOW != kShort> P;
    const P t(s, small_lds2);
    // gamma and beta wait in LDS: in registers they are what a third workgroup of 512 threads a CU has no room for
    float2 *const affine = small_lds2 + s.teams * s.team_sums;
    for (int c = int(threadIdx.x); c < t.groups * s.K; c += int(blockDim.x))
        affine[c] = make_float2(gamma ? gamma[t.c0 + c] : 1.0f, beta ? beta[t.c0 + c] : 0.0f);  // read behind the sums' barriers
    const int64_t xstep = s.lanes * ldx, ystep = s.lanes * ldy;
    for (int64_t b0 = int64_t(blockIdx.x) * s.teams; b0 < s.samples.count; b0 += int64_t(gridDim.x) * s.teams) {
        const int64_t b = b0 + t.team;
        const Span n(s, t, b);
        const T *x = X + (n.lo + t.row_lane) * ldx + t.c0 + t.col;
        Held<T, P> h;
        h.fetch(t, x, xstep, n.mine);
        const float count = float(n.rows > 0 ? n.rows : 1) * float(s.K), inv = 1.0f / count;
        // sums over the thread's rows; beyond the registers by thirty-two at a time, so that long sums do not lose bits
        // (by column, or of a vector's columns where it has one group)
        constexpr bool INSIDE = P::INSIDE;
        constexpr int S = INSIDE ? 1 : VEC;
        auto add_row = [&](auto (&to)[S], const float (&f)[VEC], auto term) {
            auto v = term(f[0], 0);
            if constexpr (INSIDE) {
                decltype(v) w[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) w[j] = term(f[j], j);
#pragma unroll
                for (int d = VEC / 2; d > 0; d /= 2)
#pragma unroll
                    for (int j = 0; j < d; ++j) add_to(w[j], w[j + d]);
                add_to(to[0], w[0]);
            } else {
                add_to(to[0], v);
#pragma unroll
                for (int j = 1; j < VEC; ++j) add_to(to[j], term(f[j], j));
            }
        };
        auto sum_rows = [&](auto (&a)[S], auto term) {
            typedef decltype(term(0.0f, 0)) V;
#pragma unroll
            for (int j = 0; j < S; ++j) a[j] = V{};
#pragma unroll
            for (int k = 0; k < held<T>(); ++k)
                if (k < n.mine) {
                    float f[VEC];
                    h.get(k, f);
                    add_row(a, f, term);
                }
#pragma clang loop unroll(disable)
            for (int k0 = held<T>(); k0 < n.mine; k0 += 32) {
                V part[S];
#pragma unroll
                for (int j = 0; j < S; ++j) part[j] = V{};
#pragma clang loop unroll(disable)
                for (int k = k0; k < k0 + 32 && k < n.mine; ++k) {
                    float f[VEC];
                    h.get_far(t, x, xstep, k, f);
                    add_row(part, f, term);
                }
#pragma unroll
                for (int j = 0; j < S; ++j) add_to(a[j], part[j]);
            }
        };
        float m[VEC];
        const float *sum;
        {
            float a[S];
            sum_rows(a, [](float f, int) { return f; });
            sum = t.reduce(s, a);
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) m[j] = 0.0f;
        t.columns(s, [&](int j, int g, int) { m[j] = product(sum[g], inv); });
        float *const first = reinterpret_cast<float *>(t.room + s.team_sums - ((s.groups + 1) >> 1));  // by group: kept for the same threads
        if (t.team < s.teams)
            for (int g = t.i; g < t.groups; g += s.team) first[g] = product(sum[g], inv);
        float2 b2[S];
        sum_rows(b2, [&](float f, int j) {
            const float d = f - m[j];
            return make_float2(d, d * d);
        });
        float2 *const both = const_cast<float2 *>(t.reduce(s, b2));
        // a group's thread turns its sums into the rest of the mean and the reciprocal deviation: every column's thread by itself is more registers
        // than bf16 has
        for (int g = t.i; g < t.groups && t.team < s.teams; g += s.team) {
            const float rest = quotient(both[g].x, count, inv), var = both[g].y * inv - rest * rest;
            const float r = 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps);
            both[g] = make_float2(rest, r);
            if (n.there) {
                const int64_t p = b * s.G + int(blockIdx.y) * s.groups + g;
                mean[p] = first[g] + rest;
                rstd[p] = r;
            }
        }
        __syncthreads();
        float a[VEC], e[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) a[j] = e[j] = 0.0f;
        t.columns(s, [&](int j, int g, int) {
            e[j] = both[g].x;
            a[j] = both[g].y;
        });
        float bt[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float2 p = j < t.have ? affine[t.col + j] : make_float2(0.0f, 0.0f);
            a[j] *= p.x;
            bt[j] = p.y;
        }
        T *y = Y + (n.lo + t.row_lane) * ldy + t.c0 + t.col;
        auto write = [&](int k, float (&f)[VEC]) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) f[j] = activate<ACT>(((f[j] - m[j]) - e[j]) * a[j] + bt[j]);
            put_row<T>(t, y + k * ystep, f);
        };
#pragma unroll
        for (int k = 0; k < held<T>(); ++k)
            if (k < n.mine) {
                float f[VEC];
                h.get(k, f);
                write(k, f);
            }
#pragma clang loop unroll(disable)
        for (int k = held<T>(); k < n.mine; ++k) {
            float f[VEC];
            h.get_far(t, x, xstep, k, f);
            write(k, f);
        }
    }
}

// Backward.  A workgroup adds up its samples' column sums for dbeta and dgamma and leaves them in its row of `part`.  In fp32 the registers
// of X and dY take xh and dz, so that the activation's derivative is formed once; bf16 pairs are unpacked twice.
template <typename T, int ACT, Vectors HOW>
__global__ void __launch_bounds__(512) small_bwd_kernel(const T *X, int64_t ldx, const T *dY, int64_t ldy, const Small s,
                                                        const float *__restrict__ gamma, const float *__restrict__ beta, const float *__restrict__ mean,
                                                        const float *__restrict__ rstd, T *dX, int64_t lddx, float2 *__restrict__ part) {
    extern __shared__ float2 small_lds2[];
    constexpr int VEC = gnn_rows<T>::VEC;
    constexpr bool KEEP = VEC == 4;
    typedef Team<VEC, HOW, HOW == kAcross> P;
    const P t(s, small_lds2);
    float gm[VEC], bt[VEC];
    double2 total[VEC];  // over all samples of a team: thousands, where they are small
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        const int c = t.c0 + t.col + j;
        gm[j] = gamma && j < t.have ? gamma[c] : 1.0f;
        bt[j] = beta && j < t.have ? beta[c] : 0.0f;
        total[j] = make_double2(0.0, 0.0);
    }
    const int64_t xstep = s.lanes * ldx, ystep = s.lanes * ldy, ostep = s.lanes * lddx;
    for (int64_t b0 = int64_t(blockIdx.x) * s.teams; b0 < s.samples.count; b0 += int64_t(gridDim.x) * s.teams) {
        const int64_t b = b0 + t.team;
        const Span n(s, t, b);
        const T *xp = X + (n.lo + t.row_lane) * ldx + t.c0 + t.col, *dp = dY + (n.lo + t.row_lane) * ldy + t.c0 + t.col;
        Held<T, P> x, d;
        x.fetch(t, xp, xstep, n.mine);
        d.fetch(t, dp, ystep, n.mine);
        float m[VEC], r[VEC];
        float2 a[VEC];
        const int64_t first = b * s.G + int64_t(blockIdx.y) * s.groups;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            m[j] = r[j] = 0.0f;
            a[j] = make_float2(0.0f, 0.0f);
        }
        if (n.mine)
            t.columns(s, [&](int j, int g, int) {
                m[j] = mean[first + g];
                r[j] = rstd[first + g];
            });
        // x, dY -> xh, dz
        auto turn = [&](float (&f)[VEC], float (&g)[VEC]) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                f[j] = (f[j] - m[j]) * r[j];
                g[j] *= slope<ACT>(f[j] * gm[j] + bt[j]);
            }
        };
        auto add = [&](float2 (&to)[VEC], const float (&f)[VEC], const float (&g)[VEC]) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                to[j].x += g[j];
                to[j].y += g[j] * f[j];
            }
        };
#pragma unroll
        for (int k = 0; k < held<T>(); ++k)
            if (k < n.mine) {
                float f[VEC], g[VEC];
                x.get(k, f);
                d.get(k, g);
                turn(f, g);
                add(a, f, g);
                if constexpr (KEEP) {
                    x.v[k] = gnn_rows<T>::pack(f);
                    d.v[k] = gnn_rows<T>::pack(g);
                }
            }
#pragma clang loop unroll(disable)
        for (int k0 = held<T>(); k0 < n.mine; k0 += 32) {
            float2 some[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) some[j] = make_float2(0.0f, 0.0f);
#pragma clang loop unroll(disable)
            for (int k = k0; k < k0 + 32 && k < n.mine; ++k) {
                float f[VEC], g[VEC];
                x.get_far(t, xp, xstep, k, f);
                d.get_far(t, dp, ystep, k, g);
                turn(f, g);
                add(some, f, g);
            }
#pragma unroll
            for (int j = 0; j < VEC; ++j) { a[j].x += some[j].x; a[j].y += some[j].y; }
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            add_to(total[j], make_double2(a[j].x, a[j].y));
            a[j].x *= gm[j];
            a[j].y *= gm[j];
        }
        if (!dX) continue;  // the same for the whole launch
        const float2 *sum = t.reduce(s, a);
        const float inv = 1.0f / (float(n.rows > 0 ? n.rows : 1) * float(s.K));
        t.columns(s, [&](int j, int g, int) { a[j] = make_float2(sum[g].x * inv, sum[g].y * inv); });
        T *o = dX + (n.lo + t.row_lane) * lddx + t.c0 + t.col;
        auto write = [&](int k, float (&f)[VEC], const float (&g)[VEC]) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) f[j] = gradient(g[j], gm[j], f[j], r[j], a[j]);
            put_row<T>(t, o + k * ostep, f);
        };
#pragma unroll
        for (int k = 0; k < held<T>(); ++k)
            if (k < n.mine) {
                float f[VEC], g[VEC];
                x.get(k, f);
                d.get(k, g);
                if constexpr (!KEEP) turn(f, g);
                write(k, f, g);
            }
#pragma clang loop unroll(disable)
        for (int k = held<T>(); k < n.mine; ++k) {
            float f[VEC], g[VEC];
            x.get_far(t, xp, xstep, k, f);
            d.get_far(t, dp, ystep, k, g);
            turn(f, g);
            write(k, f, g);
        }
    }
    if (!part) return;  // the same for the whole launch
    // the column sums of all teams and row lanes: units of cols * VEC places
    const int width = s.cols * VEC;
    int units = s.teams * s.lanes;
    const int unit = t.team * s.lanes + t.row_lane;
    const bool in = t.team < s.teams && t.row_lane < s.lanes;
    __syncthreads();
    if (in)
#pragma unroll
        for (int j = 0; j < VEC; ++j) small_lds2[unit * width + t.lane * VEC + j] = make_float2(float(total[j].x), float(total[j].y));
    while (units > 1) {
        const int half = (units + 1) >> 1;
        __syncthreads();
        if (in && unit + half < units)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                float2 &w = small_lds2[unit * width + t.lane * VEC + j];
                const float2 u = small_lds2[(unit + half) * width + t.lane * VEC + j];
                w.x += u.x;
                w.y += u.y;
            }
        units = half;
    }
    if (in && unit == 0)
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (j < t.have) part[int64_t(blockIdx.x) * s.C + t.c0 + t.col + j] = small_lds2[t.lane * VEC + j];
}

// ---------------------------------------------------------------- samples of one row

// Per vertex: `lanes` lanes of a wavefront, a power of two, have a row in registers, vector i of a lane in columns (i lanes + lane) VEC.  A
// group is `width` neighbouring lanes, or the row; sums go by lane permutations, without LDS and without waiting for other wavefronts.
struct PerRow {
    int64_t N;
    int C, G, K;
    int lanes, shift, width;  // lanes = 1 << shift
};
constexpr int kRowThreads = 256;

// sums of M values over `width` neighbouring lanes, in all of them; all lanes of the wavefront are here
template <int M> __device__ __forceinline__ void add_lanes(float (&v)[M], int width) {
    const auto step = [&](auto other) {
        float o[M];
#pragma unroll
        for (int i = 0; i < M; ++i) o[i] = other(v[i]);
#pragma unroll
        for (int i = 0; i < M; ++i) v[i] += o[i];
    };
    if (width >= 2) step([](float f) { return gnn_from_lane<0xB1>(f); });    // the other of a pair
    if (width >= 4) step([](float f) { return gnn_from_lane<0x4E>(f); });    // the other pair of four
    if (width >= 8) step([](float f) { return gnn_from_lane<0x141>(f); });   // mirrored in eight: the other four
    if (width >= 16) step([](float f) { return gnn_from_lane<0x140>(f); });  // mirrored in sixteen: the other eight
    if (width >= 32) step([](float f) { return __shfl_xor(f, 16); });
    if (width >= 64) step([](float f) { return __shfl_xor(f, 32); });
}

// The last vector of a row ends with it; its first `skip` columns are the vector's before it, computed by both to the same bits and counted there.
template <int VEC, int NV> struct RowPlace {
    int lane, unit, units;
    int col[NV], skip[NV];
    bool active[NV];
    __device__ __forceinline__ explicit RowPlace(const PerRow &s) {
        lane = int(threadIdx.x) & (s.lanes - 1);
        unit = int(threadIdx.x) >> s.shift;
        units = kRowThreads >> s.shift;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * s.lanes + lane) * VEC;
            active[i] = c < s.C;
            col[i] = c < s.C - VEC ? c : s.C - VEC;
            skip[i] = active[i] ? c - col[i] : VEC;
        }
    }
    // a[i]: of vector i; sums of the groups they belong to.  Of two quantities at once: the second's steps wait with the first's
    template <int M> __device__ __forceinline__ void groups(const PerRow &s, float (&a)[M]) const {
        static_assert(M % NV == 0, "a value for every vector");
        if (s.G == 1) {
            float t[M / NV];
#pragma unroll
            for (int k = 0; k < M / NV; ++k) {
                t[k] = a[k * NV];
#pragma unroll
                for (int i = 1; i < NV; ++i) t[k] += a[k * NV + i];
            }
            add_lanes(t, s.width);
#pragma unroll
            for (int i = 0; i < M; ++i) a[i] = t[i / NV];
        } else add_lanes(a, s.width);
    }
    template <typename T, bool NT> __device__ __forceinline__ void load(gnn_strip<T, VEC, NT> (&x)[NV], const T *row, bool there) const {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            x[i].v = {};
            if (there && active[i]) x[i].load(row + col[i]);
        }
    }
    __device__ __forceinline__ void columns(const float *p, float otherwise, float (&f)[NV][VEC]) const {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) f[i][j] = otherwise;
            if (p && active[i]) Affine<VEC>::columns(p + col[i], f[i]);
        }
    }
};
// rows that a thread has vectors of at once
template <typename T> __host__ __device__ constexpr int rows_held(int nv, bool backward) {
    const int r = (backward ? 16 / gnn_rows<T>::VEC : 2) / nv;
    return r > 1 ? r : 1;
}

template <typename T, int ACT, int NV, bool NT>
__global__ void __launch_bounds__(kRowThreads) row_kernel(const T *__restrict__ X, int64_t ldx, const PerRow s, const float *__restrict__ gamma,
                                                          const float *__restrict__ beta, float eps, float *__restrict__ mean, float *__restrict__ rstd,
                                                          T *__restrict__ Y, int64_t ldy) {
    constexpr int VEC = gnn_rows<T>::VEC, R = rows_held<T>(NV, false);
    const RowPlace<VEC, NV> at(s);
    const int64_t r0 = workgroup() * (at.units * R) + at.unit;
    gnn_strip<T, VEC, NT> x[R][NV];
#pragma unroll
    for (int u = 0; u < R; ++u) at.load(x[u], X + (r0 + u * at.units) * ldx, r0 + u * at.units < s.N);
    float gm[NV][VEC], bt[NV][VEC];
    at.columns(gamma, 1.0f, gm);
    at.columns(beta, 0.0f, bt);
    const float inv = 1.0f / float(s.K);
    // The mean of the values as they are is off by its own rounding, units of its last place; their distances f from it (m) are not.  The distances' mean e
    // completes it, and their squares' mean gives the variance.  All rows' sums go together: their steps wait for each other's lanes.
    constexpr int M = R * NV;
    float f[M][VEC], m[M], e[2 * M], *const q = e + M;
#pragma unroll
    for (int i = 0; i < M; ++i) {
        x[i / NV][i % NV].get(f[i]);
        m[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < VEC; ++j) m[i] += j >= at.skip[i % NV] ? f[i][j] : 0.0f;
    }
    at.groups(s, m);
#pragma unroll
    for (int i = 0; i < M; ++i) {
        m[i] = product(m[i], inv);
        e[i] = q[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            f[i][j] -= m[i];
            e[i] += j >= at.skip[i % NV] ? f[i][j] : 0.0f;
            q[i] += j >= at.skip[i % NV] ? f[i][j] * f[i][j] : 0.0f;
        }
    }
    at.groups(s, e);
#pragma unroll
    for (int n = 0; n < M; ++n) {
        const int i = n % NV;
        const int64_t r = r0 + n / NV * at.units;
        if (r >= s.N || !at.active[i]) continue;
        e[n] = quotient(e[n], float(s.K), inv);
        const float var = q[n] * inv - e[n] * e[n], k = 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps);
        if ((at.lane & (s.width - 1)) == 0 && (i == 0 || s.G > 1)) {
            const int64_t p = r * s.G + at.col[i] / s.K;
            mean[p] = m[n] + e[n];
            rstd[p] = k;
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) f[n][j] = activate<ACT>((f[n][j] - e[n]) * (k * gm[i][j]) + bt[i][j]);
        gnn_store_row<T, VEC, NT>(Y + r * ldy + at.col[i], f[n]);
    }
}

// Workgroups walk over the rows where the parameters' gradients are asked for, with the column sums of 32 rows in registers and those of all in LDS, and leave
// them in their row of `part`.  (One after the other, the thousand rows that a thread has of 8 M x 256 are off by 1e-5.)
template <typename T, int ACT, int NV, bool NT>
__global__ void __launch_bounds__(kRowThreads) row_bwd_kernel(const T *__restrict__ X, int64_t ldx, const T *__restrict__ dY, int64_t ldy, const PerRow s,
                                                              const float *__restrict__ gamma, const float *__restrict__ beta,
                                                              const float *__restrict__ mean, const float *__restrict__ rstd, T *__restrict__ dX,
                                                              int64_t lddx, float2 *__restrict__ part) {
    extern __shared__ float2 row_lds[];
    constexpr int VEC = gnn_rows<T>::VEC, R = rows_held<T>(NV, true);
    const RowPlace<VEC, NV> at(s);
    float gm[NV][VEC], bt[NV][VEC];
    at.columns(gamma, 1.0f, gm);
    at.columns(beta, 0.0f, bt);
    float2 total[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) total[i][j] = make_float2(0.0f, 0.0f);
    constexpr int RUN = 32 / R;
    int walked = 0;
    const auto all = [&](int i, int j) -> float2 & { return row_lds[(i * VEC + j) * kRowThreads + int(threadIdx.x)]; };
    if (part)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) all(i, j) = make_float2(0.0f, 0.0f);
    const float inv = 1.0f / float(s.K);
    for (int64_t base = int64_t(blockIdx.x) * (at.units * R); base < s.N; base += int64_t(gridDim.x) * (at.units * R)) {
        const int64_t r0 = base + at.unit;
        gnn_strip<T, VEC, NT> x[R][NV], d[R][NV];
        float m[R][NV], k[R][NV];
#pragma unroll
        for (int u = 0; u < R; ++u) {
            const int64_t r = r0 + u * at.units;
            at.load(x[u], X + r * ldx, r < s.N);
            at.load(d[u], dY + r * ldy, r < s.N);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const bool there = r < s.N && at.active[i];
                const int64_t p = r * s.G + (s.G > 1 ? at.col[i] / s.K : 0);
                m[u][i] = there ? mean[p] : 0.0f;
                k[u][i] = there ? rstd[p] : 0.0f;
            }
        }
#pragma unroll
        for (int u = 0; u < R; ++u) {
            const int64_t r = r0 + u * at.units;
            float f[NV][VEC], g[NV][VEC], s1[NV], s2[NV];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                x[u][i].get(f[i]);
                d[u][i].get(g[i]);
                s1[i] = s2[i] = 0.0f;
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    f[i][j] = (f[i][j] - m[u][i]) * k[u][i];
                    g[i][j] *= slope<ACT>(f[i][j] * gm[i][j] + bt[i][j]);
                    total[i][j].x += g[i][j];
                    total[i][j].y += g[i][j] * f[i][j];
                    const float t = j >= at.skip[i] ? g[i][j] * gm[i][j] : 0.0f;
                    s1[i] += t;
                    s2[i] += j >= at.skip[i] ? t * f[i][j] : 0.0f;
                }
            }
            if (!dX) continue;  // the same for the whole launch
            at.groups(s, s1);
            at.groups(s, s2);
            if (r >= s.N) continue;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const float2 sum = make_float2(s1[i] * inv, s2[i] * inv);
#pragma unroll
                for (int j = 0; j < VEC; ++j) f[i][j] = gradient(g[i][j], gm[i][j], f[i][j], k[u][i], sum);
                if (at.active[i]) gnn_store_row<T, VEC, NT>(dX + r * lddx + at.col[i], f[i]);
            }
        }
        if (part && ++walked == RUN) {
            walked = 0;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    add_to(all(i, j), total[i][j]);
                    total[i][j] = make_float2(0.0f, 0.0f);
                }
        }
    }
    if (!part) return;  // the same for the whole launch
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) add_to(total[i][j], all(i, j));
    __syncthreads();
    // the rows of a wavefront, then the wavefronts
    const int width = NV * VEC * s.lanes, wave = int(threadIdx.x) >> 6;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            float2 &t = total[i][j];
            for (int e = s.lanes; e < 64; e <<= 1) {
                t.x += __shfl_xor(t.x, e);
                t.y += __shfl_xor(t.y, e);
            }
            if (wave && (threadIdx.x & 63) < unsigned(s.lanes)) row_lds[(wave - 1) * width + (i * s.lanes + at.lane) * VEC + j] = t;
        }
    __syncthreads();
    if (threadIdx.x >= unsigned(s.lanes)) return;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            if (j < at.skip[i]) continue;
            float2 t = total[i][j];
#pragma unroll
            for (int w = 0; w < kRowThreads / 64 - 1; ++w) add_to(t, row_lds[w * width + (i * s.lanes + at.lane) * VEC + j]);
            part[int64_t(blockIdx.x) * s.C + at.col[i] + j] = t;
        }
}

// ---------------------------------------------------------------- host

int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

struct Layout {
    int64_t tile_rows, tiles, parts, map_off, open_off, total_off, sums_off, table_off, exact_off, bytes;
    int threads;  // of a tile
    bool joined;  // one sample, few tiles: two launches
};

// One sample of up to 32 K values for each of the tiles whose partial
// sums every writing workgroup can join by itself saves a launch.
Layout layout_of(int64_t N, int64_t C, int64_t G, int64_t B, bool backward) {
    Layout L{};
    const int64_t few = kJoined / C < 32 ? kJoined / C : 32;
    L.joined = B == 1 && C <= 1024 && N * C <= few * 32768;
    L.threads = N * C < kLarge ? kThreads : kLargeThreads;
    const int64_t most = L.joined ? few : N * C < kLarge ? kTiles : kLargeTiles;
    int64_t tiles = (N * C + kTileValues - 1) / kTileValues;
    tiles = tiles < most ? tiles : most;
    L.tile_rows = (N + tiles - 1) / tiles;
    L.tiles = (N + L.tile_rows - 1) / L.tile_rows;
    // partial sums: of the tiles, or of the workgroups of small_bwd_kernel and row_bwd_kernel.  (A backward call's workspace does for the forward call, too.)
    const int64_t slots = B > 1 ? 2 * L.tiles : L.tiles, small = backward ? (B < kSmallParts ? B : kSmallParts) : 0;
    L.parts = slots > small ? slots : small;
    const int64_t moments = slots * C * int64_t(sizeof(double2)), sums = L.parts * C * int64_t(sizeof(float2));
    int64_t off = round_up(moments > sums ? moments : sums, 256);
    L.map_off = off;
    if (B > 1) off += round_up(N * 4, 256);
    L.open_off = off;
    if (B > 1 && C / G > kSlice) off += round_up(B * G * int64_t(sizeof(double2)), 256);
    L.table_off = off;
    if (B == 1) off += round_up(4 * C * 4, 256);
    L.exact_off = off;
    L.bytes = off + round_up(B * G * int64_t(sizeof(float2)), 256);
    if (backward) {
        L.total_off = off;
        if (B > 1) off += round_up(L.tiles * C * int64_t(sizeof(float2)), 256);
        L.sums_off = off;
        off += round_up(B * G * int64_t(sizeof(float2)), 256);
        L.bytes = off;
    }
    return L;
}

int check_norm(int64_t N, int64_t C, int64_t G, int64_t B, const void *sample_ptr, const gnn_norm_opts *opts, gnn_norm_opts &o) {
    if (!opts) return GNN_ERR_INVALID_ARG;
    o = *opts;
    if (o.dtype != GNN_F32 && o.dtype != GNN_BF16) return GNN_ERR_INVALID_ARG;
    if (o.act < GNN_ACT_NONE || o.act > GNN_ACT_SILU) return GNN_ERR_INVALID_ARG;
    if (N < 0 || C < 0 || B < 0 || G <= 0 || C > (1 << 24) || B > INT32_MAX || N > INT32_MAX) return GNN_ERR_INVALID_ARG;
    if (C % G) return GNN_ERR_INVALID_ARG;
    if (!(o.eps >= 0.0f)) return GNN_ERR_INVALID_ARG;
    if (N > 0 && (B == 0 || (!sample_ptr && N % B))) return GNN_ERR_INVALID_ARG;
    if (o.ldx == 0) o.ldx = C;
    if (o.ldy == 0) o.ldy = C;
    if (o.lddx == 0) o.lddx = C;
    if (o.ldx < C || o.ldy < C || o.lddx < C || o.max_sample_rows < 0) return GNN_ERR_INVALID_ARG;
    return GNN_OK;
}

struct Call {
    const void *X, *dY, *sample_ptr;
    const float *gamma, *beta;
    float *mean, *rstd;
    void *out;  // Y or dX
    float *dgamma, *dbeta;
    int64_t N, C, G, B;
    gnn_norm_opts o;
    Layout L;
    bool backward;
    bool past_caches;  // more data than the last-level cache keeps until it is read again
    Samples samples() const { return Samples{sample_ptr, o.ptr_is_64, sample_ptr ? 0 : N / B, B, N}; }
    hipStream_t stream() const { return static_cast<hipStream_t>(o.stream); }
    char *scratch(int64_t off) const { return static_cast<char *>(o.workspace) + off; }
};

// Rows of `cols` vectors that fill whole wavefronts best, in workgroups of up to kBlockMost threads.
int row_lanes_of(int cols) {
    int best = 1;
    double share = 0.0;
    for (int r = 1; r * cols <= kBlockMost || r == 1; ++r) {
        const double full = double(r * cols) / double(round_up(r * cols, 64));
        if (full >= share - 0.02) {
            best = r;
            if (full > share) share = full;
        }
    }
    return best;
}

Shape shape_of(const Call &c, int vec, int rows, dim3 *grid, dim3 *block) {  // rows > 0: of a kernel that writes results
    Shape s{};
    s.samples = c.samples();
    s.N = c.N;
    s.C = int(c.C);
    s.G = int(c.G);
    s.group_width = int(c.C / c.G);
    s.tile_rows = c.L.tile_rows;
    s.many = c.B > 1;
    s.sample_of = c.sample_ptr && c.B > 1 ? reinterpret_cast<int32_t *>(c.scratch(c.L.map_off)) : nullptr;
    s.open = reinterpret_cast<double2 *>(c.scratch(c.L.open_off));
    s.pieces = 1;
    const int64_t vecs = (c.C + vec - 1) / vec, K = c.C / c.G;
    int64_t chunks = (vecs + 255) / 256;
    s.cols = int((vecs + chunks - 1) / chunks);
    s.slice = s.cols * vec;
    if (!rows && s.many) {
        if (K > kSlice) {
            const int64_t pieces = (K + kSlice - 1) / kSlice;
            s.slice = int((K + pieces - 1) / pieces);
            s.pieces = int((K + s.slice - 1) / s.slice);
            chunks = c.G;
        } else {  // alike: a narrow last slice takes as many workgroups as a wide one
            const int64_t most = kSlice / K, slices = (c.G + most - 1) / most;
            s.slice = int((c.G + slices - 1) / slices * K);
            chunks = (c.C + s.slice - 1) / s.slice;
        }
        s.cols = (s.slice + vec - 1) / vec;
    }
    if (rows) {
        s.row_lanes = row_lanes_of(s.cols);
        *block = dim3(unsigned(s.cols), unsigned(s.row_lanes));
        *grid = spread((c.N + rows * s.row_lanes - 1) / (rows * s.row_lanes), unsigned(chunks), block->x);
    } else {
        s.row_lanes = c.L.threads / s.cols;
        for (s.join = 1; 2 * s.join * s.cols * vec <= c.L.threads && 16 * s.join <= s.row_lanes;) s.join *= 2;  // eight to one and more
        *block = dim3(unsigned(c.L.threads));
        *grid = dim3(unsigned(c.L.tiles), unsigned(chunks));
    }
    return s;
}

// PART, OUT: elements of a thread's vectors in the kernel that adds up and in the one that writes.
template <typename T, int PART, int OUT, int ACT, bool NT> int run_tiles(const Call &c) {
    dim3 grid, threads, out_grid, out_threads;
    const Shape s = shape_of(c, PART, 0, &grid, &threads), w = shape_of(c, OUT, rows_of<T>(c.backward), &out_grid, &out_threads);
    const T *X = static_cast<const T *>(c.X), *dY = static_cast<const T *>(c.dY);
    T *out = static_cast<T *>(c.out);
    hipStream_t stream = c.stream();
    float2 *part = reinterpret_cast<float2 *>(c.scratch(0));
    double2 *moments = reinterpret_cast<double2 *>(c.scratch(0));
    float *table = c.B == 1 ? reinterpret_cast<float *>(c.scratch(c.L.table_off)) : nullptr;
    const int64_t pairs = (c.B > c.L.tiles ? c.L.tiles : c.B) * c.G;
    const unsigned many = unsigned(pairs < 65536 ? pairs : 65536);
    size_t lds;
    const int64_t finish = s.many ? s.slice : 0;
    if (c.backward) lds = size_t(tile_values<float2>(threads.x, PART, 2, finish, s.group_width) + (s.many ? 4 * s.cols * PART : 0)) * sizeof(float);
    else lds = size_t(tile_values<double2>(threads.x, PART, 3, finish, s.group_width) + 2 * finish) * sizeof(float);
    // what join_tiles keeps: the sums of every row lane, and a sixteenth
    const size_t values = size_t(w.row_lanes) * size_t(c.C), join = (values + c.G * ((values / c.G + 15) / 16)) * (c.backward ? sizeof(float2) : sizeof(double2));
    if (!c.backward) {
        float2 *exact = reinterpret_cast<float2 *>(c.scratch(c.L.exact_off));
        if (c.L.joined) {
            norm_part_kernel<T, PART, false, kThreads, kOneSample><<<grid, threads, lds, stream>>>(X, c.o.ldx, s, moments, c.o.eps, c.mean, c.rstd, exact);
            norm_apply_kernel<T, OUT, ACT, false, kJoin><<<out_grid, out_threads, join, stream>>>(X, c.o.ldx, w, c.gamma, c.beta, c.mean, c.rstd, exact, out, c.o.ldy, moments, c.o.eps, nullptr);
        } else {
            auto *sum = c.L.threads == kThreads ? norm_part_kernel<T, PART, NT, kThreads, kManySamples> : norm_part_kernel<T, PART, NT, kLargeThreads, kManySamples>;
            if (c.B == 1) sum = c.L.threads == kThreads ? norm_part_kernel<T, PART, NT, kThreads, kOneSample> : norm_part_kernel<T, PART, NT, kLargeThreads, kOneSample>;
            else if (s.pieces > 1) sum = c.L.threads == kThreads ? norm_part_kernel<T, PART, NT, kThreads, kPieces> : norm_part_kernel<T, PART, NT, kLargeThreads, kPieces>;
            sum<<<grid, threads, lds, stream>>>(X, c.o.ldx, s, moments, c.o.eps, c.mean, c.rstd, exact);
            if (pairs <= 512) norm_stats_kernel<1024><<<unsigned(pairs), 1024, 0, stream>>>(moments, s, c.o.eps, c.mean, c.rstd, exact, c.gamma, c.beta, table);
            else if (pairs < 4096) norm_stats_kernel<256><<<unsigned(pairs), 256, 0, stream>>>(moments, s, c.o.eps, c.mean, c.rstd, exact, c.gamma, c.beta, table);
            else norm_stats_kernel<64><<<many, 64, 0, stream>>>(moments, s, c.o.eps, c.mean, c.rstd, exact, c.gamma, c.beta, table);
            auto *apply = c.B == 1 ? norm_apply_kernel<T, OUT, ACT, NT, kOne> : norm_apply_kernel<T, OUT, ACT, NT, kMany>;
            apply<<<out_grid, out_threads, 0, stream>>>(X, c.o.ldx, w, c.gamma, c.beta, c.mean, c.rstd, exact, out, c.o.ldy, nullptr, 0.0f, table);
        }
    } else {
        float2 *sums = c.out ? reinterpret_cast<float2 *>(c.scratch(c.L.sums_off)) : nullptr;
        float2 *total = c.B > 1 && (c.dgamma || c.dbeta) ? reinterpret_cast<float2 *>(c.scratch(c.L.total_off)) : nullptr;
        if (c.L.joined) {
            norm_bwd_part_kernel<T, PART, ACT, false, kThreads, kOneSample><<<grid, threads, lds, stream>>>(X, c.o.ldx, dY, c.o.ldy, s, c.gamma, c.beta, c.mean, c.rstd, part, nullptr, nullptr);
            if (c.dgamma || c.dbeta) norm_bwd_columns_kernel<<<unsigned((c.C + 15) / 16), 1024, 0, stream>>>(part, c.L.tiles, int(c.C), c.dgamma, c.dbeta);
            if (c.out)
                norm_bwd_apply_kernel<T, OUT, ACT, false, kJoin><<<out_grid, out_threads, join, stream>>>(X, c.o.ldx, dY, c.o.ldy, w, c.gamma, c.beta, c.mean, c.rstd,
                                                                                                     nullptr, out, c.o.lddx, part, nullptr);
        } else {
            auto *sum = c.L.threads == kThreads ? norm_bwd_part_kernel<T, PART, ACT, NT, kThreads, kManySamples> : norm_bwd_part_kernel<T, PART, ACT, NT, kLargeThreads, kManySamples>;
            if (c.B == 1)
                sum = c.L.threads == kThreads ? norm_bwd_part_kernel<T, PART, ACT, NT, kThreads, kOneSample> : norm_bwd_part_kernel<T, PART, ACT, NT, kLargeThreads, kOneSample>;
            else if (s.pieces > 1)
                sum = c.L.threads == kThreads ? norm_bwd_part_kernel<T, PART, ACT, NT, kThreads, kPieces> : norm_bwd_part_kernel<T, PART, ACT, NT, kLargeThreads, kPieces>;
            sum<<<grid, threads, lds, stream>>>(X, c.o.ldx, dY, c.o.ldy, s, c.gamma, c.beta, c.mean, c.rstd, part, total, sums);
            float *dgamma = c.B == 1 ? c.dgamma : nullptr, *dbeta = c.B == 1 ? c.dbeta : nullptr;
            if (sums || dgamma || dbeta) {
                if (pairs <= 512) norm_bwd_stats_kernel<1024><<<unsigned(pairs), 1024, 0, stream>>>(part, s, c.gamma, sums, dgamma, dbeta, c.mean, c.rstd, c.out ? table : nullptr);
                else if (pairs < 4096) norm_bwd_stats_kernel<256><<<unsigned(pairs), 256, 0, stream>>>(part, s, c.gamma, sums, dgamma, dbeta, c.mean, c.rstd, c.out ? table : nullptr);
                else norm_bwd_stats_kernel<64><<<many, 64, 0, stream>>>(part, s, c.gamma, sums, dgamma, dbeta, c.mean, c.rstd, c.out ? table : nullptr);
            }
            if (total) norm_bwd_columns_kernel<<<unsigned((c.C + 15) / 16), 1024, 0, stream>>>(total, c.L.tiles, int(c.C), c.dgamma, c.dbeta);
            if (c.out) {
                auto *apply = c.B == 1 ? norm_bwd_apply_kernel<T, OUT, ACT, NT, kOne> : norm_bwd_apply_kernel<T, OUT, ACT, NT, kMany>;
                apply<<<out_grid, out_threads, 0, stream>>>(X, c.o.ldx, dY, c.o.ldy, w, c.gamma, c.beta, c.mean, c.rstd, sums, out, c.o.lddx, nullptr, table);
            }
        }
    }
    GNN_HIP_TRY(hipGetLastError());
    return GNN_OK;
}

// Whether samples of up to `rows` rows fit a workgroup, and how.  With few samples a team has one group, or as many as make 16
// columns (64 bytes of a row), so that there are more workgroups; with many all groups that fit.
constexpr int64_t kTeam = 256;  // threads of a workgroup of small samples
struct SmallPlan {
    Small s;
    dim3 grid;
    int threads;
    size_t lds;
    Vectors how;
};
bool small_plan(const Call &c, int vec, int held, int most, SmallPlan &p) {
    const int64_t rows = c.sample_ptr ? c.o.max_sample_rows : c.N / c.B;
    if (rows <= 0) return false;
    const int64_t K = c.C / c.G;
    // many samples may have four times the rows that the registers of the largest workgroup hold: 612 graphs of 0 to 200 vertices x 128 bf16, 20 us, in
    // tiles 81, backward 47 and 65; sixteen times, 1,000 graphs of 0 to 800 x 64 backward, 148, in tiles 136
    auto fits = [&](int64_t groups) {
        const int64_t cols = (groups * K + vec - 1) / vec;
        return cols <= most && rows <= (c.B < 256 ? 1 : 4) * held * (most / cols);
    };
    int64_t groups = c.G;
    if (c.B < 256) {
        const int64_t least = (16 + K - 1) / K, even = (c.G * c.B + 255) / 256;  // 256 teams
        groups = least > even ? least : even;
        groups = groups < c.G ? groups : c.G;
    }
    while (groups > 1 && !fits(groups)) groups = (groups + 1) / 2;
    if (!fits(groups)) return false;
    // Slices of a row narrower than two 128-byte lines fetch lines that others fetch too: 100 samples of 1,000 rows, slices of 10 of 100 columns,
    // 50 us, in tiles 38.
    if (groups < c.G && groups * K * (16 / vec) < 256 && c.N * c.C > (64 << 10)) return false;
    const int64_t cols = (groups * K + vec - 1) / vec;
    int64_t lanes = (rows + held - 1) / held;
    // A workgroup of 64 to 512 threads with about seven vectors each of a mean sample; what does not stay in its registers is fetched again by the
    // later passes, from the caches.  More threads wait for each other at every sum, fewer have too long a way through their rows (us; 2,449 graphs
    // of 25 vertices, ragged, forward, 64, 128, 256 and 512 threads: 100 bf16 columns 21, 22, 29, 49; 100 fp32 29, 21, 29, 45; 256 fp32 57, 37, 32, 34.
    // 612 graphs of 100 x 128 fp32 51, 29, 19, 17).  Backward, with its column sums to join, 256 (100 fp32 128 threads 37, 256 32, 384 51).
    const int64_t mean = (c.N + c.B - 1) / c.B;
    int64_t wide = c.backward ? kTeam : 2 * kTeam;
    while (!c.backward && wide > 64 && cols <= wide / 2 && mean * cols <= wide / 2 * 7) wide /= 2;
    const int64_t room = cols <= wide ? wide : most;  // threads; wide rows take what a workgroup can have
    if (cols * lanes > room) lanes = room / cols;
    Small &s = p.s;
    s = Small{};
    s.samples = c.samples();
    s.C = int(c.C);
    s.G = int(c.G);
    s.K = int(K);
    s.groups = int(groups);
    s.cols = int(cols);
    s.lanes = int(lanes);
    s.team = int(round_up(cols * lanes, 16) < most ? round_up(cols * lanes, 16) : cols * lanes);
    s.teams = s.team < wide ? int(wide) / s.team : 1;
    const int64_t slices = (c.G + groups - 1) / groups;
    p.how = K % vec == 0 ? kInside : (c.G - (slices - 1) * groups) * K >= vec ? kAcross : kShort;
    s.len = int(lanes * (p.how == kInside ? K / vec : K));
    s.team_sums = int(groups) * (s.len + (s.len + 15) / 16) + int((groups + 1) / 2);  // the last: a value of every group
    p.threads = int(round_up(s.team * s.teams, 64));
    int64_t blocks = (c.B + s.teams - 1) / s.teams;
    if (blocks > most_workgroups(p.threads)) blocks = most_workgroups(p.threads);  // (workgroups walk over the samples)
    p.grid = dim3(unsigned(blocks), unsigned(slices));
    size_t pairs = size_t(s.teams) * s.team_sums;
    if (c.backward) {
        const size_t columns = size_t(s.teams) * s.lanes * s.cols * vec;
        pairs = pairs > columns ? pairs : columns;
    } else pairs += size_t(groups * K);
    p.lds = pairs * sizeof(float2);
    return p.grid.y <= 65535 && p.lds <= (160u << 10);
}

// Workgroups of small_bwd_kernel that are resident at once: wavefronts of its registers on the 256 CUs, and what fits their LDS.  More would be
// a second round with few of them (2,449 graphs of 25 vertices x 100, us: 768 workgroups 35, 1024 40, 2048 45, 4096 48).
template <typename T, int ACT, Vectors HOW> unsigned resident(const SmallPlan &p) {
    static const int waves = [] {
        int blocks = 0;
        const hipError_t err = hipOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, reinterpret_cast<const void *>(small_bwd_kernel<T, ACT, HOW>), int(kTeam), 0);
        if (err != hipSuccess) (void)hipGetLastError();
        return err == hipSuccess && blocks > 0 ? blocks * int(kTeam / 64) : 8;
    }();
    const int by_waves = waves / (p.threads / 64), by_lds = p.lds ? int((160u << 10) / p.lds) : by_waves;
    const int each = by_waves < by_lds ? by_waves : by_lds;
    return 256u * unsigned(each > 1 ? each : 1);
}

template <typename T, int ACT, Vectors HOW> int run_small(const Call &c, SmallPlan &p) {
    const T *X = static_cast<const T *>(c.X);
    hipStream_t stream = c.stream();
    if (c.backward) {
        const int64_t here = resident<T, ACT, HOW>(p), most = here < c.L.parts ? here : c.L.parts;
        if (p.grid.x > most) p.grid.x = unsigned(most);
    }
    if (!c.backward) {
        small_kernel<T, ACT, HOW><<<p.grid, p.threads, p.lds, stream>>>(X, c.o.ldx, p.s, c.gamma, c.beta, c.o.eps, c.mean, c.rstd, static_cast<T *>(c.out),
                                                                           c.o.ldy);
    } else {
        float2 *part = c.dgamma || c.dbeta ? reinterpret_cast<float2 *>(c.scratch(0)) : nullptr;
        small_bwd_kernel<T, ACT, HOW><<<p.grid, p.threads, p.lds, stream>>>(X, c.o.ldx, static_cast<const T *>(c.dY), c.o.ldy, p.s, c.gamma, c.beta, c.mean,
                                                                               c.rstd, static_cast<T *>(c.out), c.o.lddx, part);
        if (part) norm_bwd_columns_kernel<<<unsigned((c.C + 15) / 16), 1024, 0, stream>>>(part, p.grid.x, int(c.C), c.dgamma, c.dbeta);
    }
    GNN_HIP_TRY(hipGetLastError());
    return GNN_OK;
}

// Whether rows are samples whose groups are whole powers of two of lanes, and how: as few places for vectors as will do.
bool row_plan(const Call &c, int vec, PerRow &s, int &nv) {
    if (c.sample_ptr || c.N != c.B || c.C < vec) return false;
    const int64_t K = c.C / c.G, most = 16 / vec;
    s = PerRow{c.N, int(c.C), int(c.G), int(K), 0, 0, 0};
    for (int n = 1; n <= most; ++n) {
        int shift = 0;
        while (((c.C + vec - 1) / vec + n - 1) / n > int64_t(1) << shift) ++shift;
        if (shift > 6 || (s.lanes && (n << shift) >= nv * s.lanes)) continue;
        if (c.G > 1 && (K % vec || (K / vec & (K / vec - 1)) || K / vec > int64_t(1) << shift)) continue;
        s.lanes = 1 << shift;
        s.shift = shift;
        nv = n;
    }
    s.width = c.G > 1 ? int(K / vec) : s.lanes;
    return s.lanes > 0;
}

template <typename T, int ACT, int NV, bool NT> int run_rows(const Call &c, const PerRow &s) {
    const T *X = static_cast<const T *>(c.X);
    hipStream_t stream = c.stream();
    const int64_t each = (kRowThreads >> s.shift) * rows_held<T>(NV, c.backward), blocks = (c.N + each - 1) / each;
    if (!c.backward) {
        row_kernel<T, ACT, NV, NT><<<spread(blocks, 1, kRowThreads), kRowThreads, 0, stream>>>(X, c.o.ldx, s, c.gamma, c.beta, c.o.eps, c.mean, c.rstd, static_cast<T *>(c.out), c.o.ldy);
    } else {
        const bool sums = c.dgamma || c.dbeta;
        float2 *part = sums ? reinterpret_cast<float2 *>(c.scratch(0)) : nullptr;
        const int64_t rows = c.N * c.C < kLarge ? kRowParts / 2 : kRowParts, most = !sums ? most_workgroups(kRowThreads) : rows < c.L.parts ? rows : c.L.parts, grid = blocks < most ? blocks : most;
        const size_t lds = sums ? size_t(kRowThreads) * NV * gnn_rows<T>::VEC * sizeof(float2) : 0;  // (joined in less: three wavefronts' lanes)
        row_bwd_kernel<T, ACT, NV, NT><<<unsigned(grid), kRowThreads, lds, stream>>>(X, c.o.ldx, static_cast<const T *>(c.dY), c.o.ldy, s, c.gamma, c.beta, c.mean,
                                                                                     c.rstd, static_cast<T *>(c.out), c.o.lddx, part);
        if (part) norm_bwd_columns_kernel<<<unsigned((c.C + 15) / 16), 1024, 0, stream>>>(part, grid, int(c.C), c.dgamma, c.dbeta);
    }
    GNN_HIP_TRY(hipGetLastError());
    return GNN_OK;
}
template <typename T, int ACT, int NV> int run_rows(const Call &c, const PerRow &s) {
    return c.past_caches ? run_rows<T, ACT, NV, true>(c, s) : run_rows<T, ACT, NV, false>(c, s);
}

template <typename T, int ACT> int run_act(const Call &c) {
    constexpr int V = gnn_rows<T>::VEC;
    PerRow rows;
    int nv = 0;
    if (row_plan(c, V, rows, nv)) {
        if (nv == 1) return run_rows<T, ACT, 1>(c, rows);
        if (nv == 2) return run_rows<T, ACT, 2>(c, rows);
        if constexpr (V == 4) return nv == 3 ? run_rows<T, ACT, 3>(c, rows) : run_rows<T, ACT, 4>(c, rows);
    }
    SmallPlan p;
    if (small_plan(c, V, held<T>(), c.backward ? 512 : 1024, p))
        return p.how == kInside ? run_small<T, ACT, kInside>(c, p) : p.how == kAcross ? run_small<T, ACT, kAcross>(c, p) : run_small<T, ACT, kShort>(c, p);
    if (c.C < V) return run_tiles<T, 1, 1, ACT, false>(c);
    // The backward sums keep many values for every column: with eight bf16 columns a thread two or three of its wavefronts fit a SIMD, and half vectors are
    // faster (us, eight -> four; 400 K x 128 silu 121 -> 115, 1 M x 256 441 -> 430, 103 K x 141 52 -> 43, 3.5 M x 128 738 either way, 1.1 M x 351 identity
    // 744 -> 785).  Results are written as whole vectors (halves instead: 1.1 M x 351 859, 3.5 M x 128 757).
    if (c.backward) return c.past_caches ? run_tiles<T, 4, V, ACT, true>(c) : run_tiles<T, 4, V, ACT, false>(c);
    return c.past_caches ? run_tiles<T, V, V, ACT, true>(c) : run_tiles<T, V, V, ACT, false>(c);
}

template <typename T> int run(const Call &c) {
    (void)hipGetLastError();
    if (c.o.act == GNN_ACT_RELU) return run_act<T, GNN_ACT_RELU>(c);
    if (c.o.act == GNN_ACT_SILU) return run_act<T, GNN_ACT_SILU>(c);
    return run_act<T, GNN_ACT_NONE>(c);
}

int run(Call &c) {
    c.L = layout_of(c.N, c.C, c.G, c.B, c.backward);
    if (!c.o.workspace || c.o.workspace_bytes < c.L.bytes || reinterpret_cast<uintptr_t>(c.o.workspace) % 16) return GNN_ERR_INVALID_ARG;
    const int64_t size = c.o.dtype == GNN_F32 ? 4 : 2;
    c.past_caches = c.N * c.C * size > (int64_t(256) << 20);
    return c.o.dtype == GNN_F32 ? run<float>(c) : run<gnn_bf16>(c);
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
    Call c{};
    const int rc = check_norm(N, C, G, B, sample_ptr, opts, c.o);
    if (rc != GNN_OK) return rc;
    if (N == 0 || C == 0) return GNN_OK;
    if (!X || !Y || !mean || !rstd || X == Y) return GNN_ERR_INVALID_ARG;
    c.X = X;
    c.sample_ptr = sample_ptr;
    c.gamma = gamma;
    c.beta = beta;
    c.mean = mean;
    c.rstd = rstd;
    c.out = Y;
    c.N = N;
    c.C = C;
    c.G = G;
    c.B = B;
    return run(c);
}

extern "C" GNN_API int gnn_group_norm_bwd(const void *X, const float *gamma, const float *beta, const float *mean, const float *rstd, const void *dY,
                                          const void *sample_ptr, void *dX, float *dgamma, float *dbeta, int64_t N, int64_t C, int64_t G, int64_t B,
                                          const gnn_norm_opts *opts) {
    Call c{};
    const int rc = check_norm(N, C, G, B, sample_ptr, opts, c.o);
    if (rc != GNN_OK) return rc;
    if (C == 0 || (!dX && !dgamma && !dbeta)) return GNN_OK;
    if (N == 0) {
        (void)hipGetLastError();
        if (dgamma || dbeta) norm_zero_kernel<<<64, 256, 0, static_cast<hipStream_t>(opts->stream)>>>(dgamma, dbeta, C);
        GNN_HIP_TRY(hipGetLastError());
        return GNN_OK;
    }
    if (!X || !dY || !mean || !rstd || dX == X || dX == dY) return GNN_ERR_INVALID_ARG;
    c.X = X;
    c.dY = dY;
    c.sample_ptr = sample_ptr;
    c.gamma = gamma;
    c.beta = beta;
    c.mean = const_cast<float *>(mean);
    c.rstd = const_cast<float *>(rstd);
    c.out = dX;
    c.dgamma = dgamma;
    c.dbeta = dbeta;
    c.N = N;
    c.C = C;
    c.G = G;
    c.B = B;
    c.backward = true;
    return run(c);
}
