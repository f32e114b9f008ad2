// Orthogonalised updates of weight matrices: Newton-Schulz products, and the optimizer step that uses them.
//
// With X = U / (|U| + eps), m x n, m <= n (the transposed matrix where it is taller than wide), and per step
//     A = X X^T,   Q = a I + b A + c A A,   X = Q X,
// singular values s of X become a s + b s^3 + c s^5.  Three products a step, all of the form  C[i][j] = sum_k P[i][k] R[j][k]:  A from X and X, Q
// from A and A (A is symmetric), X from Q and X^T, which is kept beside X.  A and Q are symmetric: only the tiles on and below the diagonal
// are computed, and written to both places.
//
// Operands live in the workspace as the matrix cores take them: split into P numbers of 16 bits whose sum they are, in fragments of 32 rows x 16 k, 1 KB
// a fragment, the 16 bytes of lane 32 * (k / 8) + row one after the other; the fragments of the same k side by side, so that workgroups that walk along k
// together spread over the channels of the L2s.  So whatever fetches a fragment reads 1 KB in a row, nothing is split twice, and a product's epilogue, which
// has four neighbouring results of a column in a lane, writes 8 bytes a plane.  Rows and columns are filled up with zeros to whole tiles, which the
// products keep zero.
//
// P = 2: fp16 numbers.  The rest behind the first is at most 2^-11 of it, of which the second keeps 11 bits and a sign: 23 of the 24 bits of fp32,
// with X, A and Q multiplied by powers of two that take the largest number they can reach near the largest of fp16.  The second number is held 2^11 times as large as
// it is, so that it loses bits only where the first one does: steps end at 2^-49 of the largest number, and rows or columns down to some 10^-7 of the others are as
// close as in fp32 (100 x 256, ten rows 10^-5 of the others, by themselves: 2 10^-7; with second numbers as they are, which end at 2^-38, 9 10^-6, and 10^-3 at 10^-7).  So
// products with a second number have sums of their own: 2560 x 4000 fp32 1944 us instead of 1890.  Two numbers do where the coefficients keep the
// singular values small, as the usual ones do (at most 1.2); else P = 3: bf16 numbers, which have the range and all 24 bits of fp32, at twice the products (2900 us).
// Of the products of parts those that matter are formed (P = 2: three of four, the last is at most 2^-22 of the first, 2^-25 on average; P = 3: six of nine, 2^-23 and 2^-26),
// summed from zero over 32 k (P = 3 through LDS: 16), smallest first, and added to the result with one rounding: the matrix cores cut off what lies below a sum's
// last bit, so that long chains through them would be the worse sums (not of second numbers, which are 2^-11 of the others).  Over 64 k: as fast; over 16, where
// there are twice the additions: 2030 us instead of 1890.
//
// Small matrices: a workgroup has a tile of 32 x 32 and its four wavefronts a quarter of k each, straight from the caches; such a product is one latency.
// Large ones: tiles of 64 x 64 or 128 x 128 through LDS.  All matrices of a call of the same kind share the launches.
#include "common.h"
#include "rows.h"

#include <math.h>

namespace {

constexpr int kThreads = 256;
constexpr int kMats = 16;               // of a launch
constexpr int kNormBlocks = 1024;       // partial sums of squares of a matrix, at most
constexpr int kNormChunk = 4096;        // elements of a workgroup, at least
constexpr int64_t kMostSide = 65536, kMostSteps = 100;

typedef float float16v __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct Mat {
    uint16_t *x, *xt[2], *a, *q;        // planes: X (rows m, k n), X^T (rows n, k m) before and after a step, A and Q
    double *squares;                    // [norm_blocks]; then the logarithm of X's norm
    const void *in;                     // U, or the gradient
    void *out;                          // O, or the parameters
    float *momentum, *master;           // of a Muon step, or nullptr
    int64_t ld_in, ld_out;
    int32_t m, n, mp, np;               // m <= n, and filled up
    int32_t rows, cols;                 // of U
    int32_t norm_blocks, flags;         // kBf16, kTall
    float decay, rate;                  // 1 - lr weight_decay; lr update_scale
};
enum { kBf16 = 1, kTall = 2 };          // tall: rows > cols
enum Phase { kGram, kPolynomial, kUpdate, kLast };
enum Launch { kNorms, kPlanes, kSymmetric, kOthers, kLaunches };

struct Job {
    Mat mat[kMats];
    int32_t first[kLaunches][kMats];    // workgroup that begins a matrix; INT32_MAX behind the last
    int32_t muon, nesterov;
    float mu, a, b, c;                  // (a, b and c with the powers of two that the planes hold A and Q with)
    double eps;
    float growth;                       // P = 2: the logarithm, to base 2, of what a step can multiply X by
    const float *grad_scale;
};
static_assert(sizeof(Job) <= 4096, "kernel arguments");

// the last matrix that begins at this workgroup or before, and the workgroup's number in it
template <Launch L> __device__ __forceinline__ int matrix_of_block(const Job &j, int &number) {
    int k = -1;
#pragma unroll
    for (int i = 0; i < kMats; ++i) k += j.first[L][i] <= int(blockIdx.x) ? 1 : 0;
    number = int(blockIdx.x) - j.first[L][k];
    return k;
}

__device__ __forceinline__ float element(const void *p, int64_t i, bool bf16) {
    return bf16 ? gnn_rows<gnn_bf16>::get(static_cast<const gnn_bf16 *>(p) + i) : static_cast<const float *>(p)[i];
}

// ---- the update and its norm

// elements i .. i + 3
__device__ __forceinline__ void four(const void *p, int64_t i, bool bf16, float (&v)[4]) {
    if (bf16) gnn_load_row<gnn_bf16, 4>(static_cast<const gnn_bf16 *>(p) + i, v);
    else gnn_load_row<float, 4>(static_cast<const float *>(p) + i, v);
}

// The sums of squares are fp64: squares of fp32 numbers neither overflow nor vanish there.
__global__ void __launch_bounds__(kThreads) norm_kernel(const Job j) {
    int part;
    const Mat &t = j.mat[matrix_of_block<kNorms>(j, part)];
    const bool bf16 = t.flags & kBf16;
    double s = 0.0;
    if (t.ld_in == t.cols) {
        const int64_t total = int64_t(t.rows) * t.cols;
        const int64_t per = ((total + t.norm_blocks - 1) / t.norm_blocks + 3) / 4 * 4, begin = part * per, end = begin + per < total ? begin + per : total;
        const float gs = j.grad_scale ? *j.grad_scale : 1.0f;
        for (int64_t i = begin + 4 * int(threadIdx.x); i < end; i += 4 * kThreads) {
            float u[4] = {0.0f, 0.0f, 0.0f, 0.0f}, m[4];
            const int have = end - i < 4 ? int(end - i) : 4;
            if (have == 4) {
                four(t.in, i, bf16, u);
                if (j.muon) four(t.momentum, i, false, m);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < have) {
                        u[e] = element(t.in, i + e, bf16);
                        if (j.muon) m[e] = t.momentum[i + e];
                    }
            }
            if (j.muon) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float g = u[e] * gs;
                    m[e] = j.mu * m[e] + g;
                    u[e] = e < have ? (j.nesterov ? g + j.mu * m[e] : m[e]) : 0.0f;
                    if (have < 4 && e < have) t.momentum[i + e] = m[e];
                }
                if (have == 4) gnn_store_row<float, 4>(t.momentum + i, m);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s += double(u[e]) * double(u[e]);
        }
    } else {
        for (int r = part; r < t.rows; r += t.norm_blocks)
            for (int c = int(threadIdx.x); c < t.cols; c += kThreads) {
                const float u = element(t.in, r * t.ld_in + c, bf16);
                s += double(u) * double(u);
            }
    }
    __shared__ double sums[kThreads / 64];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) t.squares[part] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// ---- planes

// What an operand is made of.  P = 2: fp16 numbers, with X, A and Q taken by powers of two that put the largest number they can hold near the type's.
template <int P> struct Parts;
template <> struct Parts<2> {
    typedef f16x8 Eight;
    static constexpr int kXLog2 = 15, kALog2 = 14, kQLog2 = 13;
    static constexpr float kRest = 2048.0f;  // what the second number holds the rest times
    static __device__ __forceinline__ float part(float x) { return float(_Float16(x)); }
    static __device__ __forceinline__ uint32_t pair(float x, float y) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(gnn_f32x2{x, y}, f16x2)); }
    static __device__ __forceinline__ float get(uint32_t w, int i) { return float(__builtin_bit_cast(f16x2, w)[i]); }
    static __device__ __forceinline__ float16v product(f16x8 a, f16x8 b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct Parts<3> {
    typedef bf16x8 Eight;
    static constexpr int kXLog2 = 0, kALog2 = 0, kQLog2 = 0;
    static constexpr float kRest = 1.0f;
    static __device__ __forceinline__ float part(float x) { return float(__bf16(x)); }
    static __device__ __forceinline__ uint32_t pair(float x, float y) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(gnn_f32x2{x, y}, gnn_bf16x2)); }
    static __device__ __forceinline__ float get(uint32_t w, int i) { return __uint_as_float(i ? w & 0xFFFF0000u : w << 16); }
    static __device__ __forceinline__ float16v product(bf16x8 a, bf16x8 b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
// P = 2: a matrix whose norm is far below eps has an X as small, and gets another power of two: as many more as keep it below 1 in this step.  (A matters
// beside 1 and stays as it is.)
constexpr float kMostExponent = 1000.0f;  // (an X below 2^-1000 vanishes in fp32, whatever the steps)
template <int P> __device__ __forceinline__ int exponent(const Job &j, float log_norm, int step) {
    if constexpr (P == 3) return 0;
    const float e = -fmaf(float(step), j.growth, log_norm);
    return e > 0.0f ? int(fminf(e, kMostExponent)) : 0;
}
// What a sum of a phase is times 2 to, to be the number that the planes hold, or the result.
template <int P, Phase phase> __device__ __forceinline__ int shift(const Job &j, const Mat &t, int step) {
    typedef Parts<P> S;
    if (P == 3 || phase == kPolynomial) return 0;
    const float log_norm = float(t.squares[t.norm_blocks]);
    const int now = exponent<P>(j, log_norm, step);
    if constexpr (phase == kGram) return S::kALog2 - 2 * (S::kXLog2 + now);
    else if constexpr (phase == kUpdate) return exponent<P>(j, log_norm, step + 1) - now - S::kQLog2;
    else return -(S::kQLog2 + S::kXLog2 + now);
}

// x = the sum of P parts, exactly where P = 3
template <int P> __device__ __forceinline__ void split(float x, float (&part)[P]) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
        part[p] = Parts<P>::part(x);
        x = (x - part[p]) * Parts<P>::kRest;
    }
}

// Where element (row, k) of an operand of rows x depth lies in plane 0, in elements of 2 bytes; planes are rows * depth apart.
__device__ __forceinline__ int64_t place(int rows, int row, int k) {
    return (int64_t(k >> 4) * (rows >> 5) + (row >> 5)) * 512 + (((k >> 3) & 1) * 32 + (row & 31)) * 8 + (k & 7);
}
// four neighbouring k, the first a multiple of four
template <int P> __device__ __forceinline__ void put4(uint16_t *planes, int rows, int depth, int row, int k, const float (&v)[4]) {
    uint16_t *p = planes + place(rows, row, k);
    float part[4][P];
#pragma unroll
    for (int i = 0; i < 4; ++i) split<P>(v[i], part[i]);
#pragma unroll
    for (int q = 0; q < P; ++q)
        *reinterpret_cast<u32x2 *>(p + int64_t(q) * rows * depth) = u32x2{Parts<P>::pair(part[0][q], part[1][q]), Parts<P>::pair(part[2][q], part[3][q])};
}
// eight, the first a multiple of eight
template <int P> __device__ __forceinline__ void put8(uint16_t *planes, int rows, int depth, int row, int k, const float (&v)[8]) {
    uint16_t *p = planes + place(rows, row, k);
    float part[8][P];
#pragma unroll
    for (int i = 0; i < 8; ++i) split<P>(v[i], part[i]);
#pragma unroll
    for (int q = 0; q < P; ++q) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = Parts<P>::pair(part[2 * i][q], part[2 * i + 1][q]);
        *reinterpret_cast<u32x4 *>(p + int64_t(q) * rows * depth) = w;
    }
}
template <int P> __device__ __forceinline__ void get4(const uint16_t *planes, int rows, int depth, int row, int k, float (&v)[4]) {
    const uint16_t *p = planes + place(rows, row, k);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = 0.0f;
#pragma unroll
    for (int q = P - 1; q >= 0; --q) {  // smallest first: the sum is exact
        const u32x2 w = *reinterpret_cast<const u32x2 *>(p + int64_t(q) * rows * depth);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = fmaf(v[i], 1.0f / Parts<P>::kRest, Parts<P>::get(i < 2 ? w.x : w.y, i & 1));
    }
}

// X and X^T from U: a workgroup has a tile of 64 x 64 of U.
template <int P, typename T> __global__ void __launch_bounds__(kThreads) planes_kernel(const Job j) {
    int tile;
    const Mat &t = j.mat[matrix_of_block<kPlanes>(j, tile)];
    const bool tall = t.flags & kTall;
    constexpr bool bf16 = sizeof(T) == 2;
    const int rp = tall ? t.np : t.mp, cp = tall ? t.mp : t.np;  // filled up sides of U
    const int tiles = cp / 64;
    const int r0 = tile / tiles * 64, c0 = tile % tiles * 64;
    __shared__ float u[64][65];
    __shared__ double sums[kThreads / 64];
    const float gs = j.grad_scale ? *j.grad_scale : 1.0f;
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6, col = c0 + lane;
    // all of the tile is on its way before the norm is waited for
    constexpr int U = 16;
    float x[U], mo[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const int row = r0 + wave + 4 * k;
        x[k] = mo[k] = 0.0f;
        if (row < t.rows && col < t.cols) {
            x[k] = element(t.in, int64_t(row) * t.ld_in + col, bf16);
            if (j.muon) mo[k] = t.momentum[int64_t(row) * t.cols + col];
        }
    }
    double s = 0.0;
    for (int i = int(threadIdx.x); i < t.norm_blocks; i += kThreads) s += t.squares[i];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    if (lane == 0) sums[wave] = s;
    __syncthreads();
    const double norm = sqrt((sums[0] + sums[1]) + (sums[2] + sums[3]));
    const bool fits = norm <= 1.7e308;
    const double size = fits ? norm / (norm + j.eps) : 1.0;  // of X, which may be below what fp32 holds
    const float log_norm = log2f(float(__builtin_amdgcn_frexp_mant(size))) + float(__builtin_amdgcn_frexp_exp(size));
    if (tile == 0 && threadIdx.x == 0) t.squares[t.norm_blocks] = double(log_norm);
    // what is not finite reaches all of the matrix; of zeros nothing is divided by an eps whose reciprocal may not be finite
    const double inverse = !fits ? __builtin_nan("") : norm > 0.0 ? ldexp(1.0, Parts<P>::kXLog2 + exponent<P>(j, log_norm, 0)) / (norm + j.eps) : 0.0;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const int row = r0 + wave + 4 * k;
        if (j.muon) x[k] = j.nesterov ? x[k] * gs + j.mu * mo[k] : mo[k];
        u[wave + 4 * k][lane] = row < t.rows && col < t.cols ? float(double(x[k]) * inverse) : 0.0f;
    }
    __syncthreads();
    uint16_t *by_row = tall ? t.xt[0] : t.x, *by_col = tall ? t.x : t.xt[0];  // rows of U as rows; columns of U as rows
    for (int i = int(threadIdx.x); i < 64 * 8; i += kThreads) {
        const int r = i & 63, k = (i >> 6) * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = u[r][k + e];
        put8<P>(by_row, rp, cp, r0 + r, c0 + k, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = u[k + e][r];
        put8<P>(by_col, cp, rp, c0 + r, r0 + k, v);
    }
}

// ---- products

// The operands of a phase: C[i][j] = sum_k left[i][k] right[j][k]
struct Operands {
    const uint16_t *left, *right;
    int rows, cols, depth;
};
template <Phase phase> __device__ __forceinline__ Operands operands(const Mat &t, int step) {
    if constexpr (phase == kGram) return {t.x, t.x, t.mp, t.mp, t.np};
    else if constexpr (phase == kPolynomial) return {t.a, t.a, t.mp, t.mp, t.mp};
    else return {t.q, t.xt[step & 1], t.mp, t.np, t.mp};
}

// The tile of a workgroup; of symmetric results those on and below the diagonal, where a tile is as wide as one or two are high.  Workgroup b of a launch
// runs on XCD b % 8, each with an L2 of its own: an XCD gets tiles that lie side by side, in bands of kBand rows of tiles, so that it reads
// few rows of either operand.
constexpr int kBand = 8;
template <bool SYMMETRIC, int WIDE> __device__ __forceinline__ void tile_of(int number, int tiles, int tiles_across, int &ti, int &tj) {
    const int xcd = number & 7, rest8 = tiles & 7;
    number = xcd * (tiles >> 3) + (xcd < rest8 ? xcd : rest8) + (number >> 3);
    if constexpr (!SYMMETRIC) {
        const int down = tiles / tiles_across, band = number / (kBand * tiles_across), first = band * kBand;
        const int high = down - first < kBand ? down - first : kBand, rest = number - first * tiles_across;
        tj = rest / high;
        ti = first + rest - tj * high;
    } else {  // rows i * WIDE .. i * WIDE + WIDE - 1 have i + 1 tiles each
        auto before = [](int i) { return WIDE * (i * (i + 1) / 2); };
        int i = int((sqrtf(8.0f / WIDE * float(number) + 1.0f) - 1.0f) * 0.5f);
        while (before(i) > number) --i;
        while (before(i + 1) <= number) ++i;
        const int rest = number - before(i);
        ti = i * WIDE + rest % WIDE;
        tj = rest / WIDE;
    }
}

// The products of parts that matter, smallest first, onto the sums of N fragments of the right operand, in turn, so that no product waits for the one before.
// P = 2: those with a second number onto `low`, which is kRest times as large and goes on over all of k.
template <int P, int N> __device__ __forceinline__ void add_products(float16v (&sum)[N], float16v (&low)[P == 2 ? N : 1], const typename Parts<P>::Eight (&a)[P], const typename Parts<P>::Eight (&b)[N][P]) {
    if constexpr (P == 2) {
#pragma unroll
        for (int y = 0; y < N; ++y) low[y] = Parts<P>::product(a[0], b[y][1], low[y]);
#pragma unroll
        for (int y = 0; y < N; ++y) sum[y] = Parts<P>::product(a[0], b[y][0], sum[y]);
#pragma unroll
        for (int y = 0; y < N; ++y) low[y] = Parts<P>::product(a[1], b[y][0], low[y]);
    } else {
#pragma unroll
        for (int s = P - 1; s >= 0; --s)
#pragma unroll
            for (int p = 0; p <= s; ++p)
#pragma unroll
                for (int y = 0; y < N; ++y) sum[y] = Parts<P>::product(a[p], b[y][s - p], sum[y]);
    }
}
template <int TI, int TJ> __device__ __forceinline__ void clear(float16v (&sum)[TI][TJ]) {
#pragma unroll
    for (int x = 0; x < TI; ++x)
#pragma unroll
        for (int y = 0; y < TJ; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) sum[x][y][v] = 0.0f;
}
// with one rounding
template <int TI, int TJ> __device__ __forceinline__ void add(float16v (&to)[TI][TJ], const float16v (&sum)[TI][TJ], float times = 1.0f) {
#pragma unroll
    for (int x = 0; x < TI; ++x)
#pragma unroll
        for (int y = 0; y < TJ; ++y)
#pragma unroll
            for (int v = 0; v < 16; ++v) to[x][y][v] = fmaf(sum[x][y][v], times, to[x][y][v]);
}

// What a phase makes of four sums, rows row_i .. row_i + 3 of column row_c, or the same columns of that row: A is symmetric.
template <int P, Phase phase> __device__ __forceinline__ void finish(const Job &j, const Mat &t, int times_log2, int row_i, int row_c, float (&v)[4]) {
    if constexpr (phase != kPolynomial) {
        if constexpr (P == 2)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_ldexpf(v[i], times_log2);
        return;
    }
    float a[4];
    get4<P>(t.a, t.mp, t.mp, row_c, row_i, a);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = fmaf(j.c, v[i], j.b * a[i]) + (row_i + i == row_c && row_c < t.m ? j.a : 0.0f);
}

template <typename T> __device__ __forceinline__ void write_out(const Job &j, const Mat &t, int64_t r, int64_t c, float o) {
    constexpr bool bf16 = sizeof(T) == 2;
    const int64_t at = r * t.ld_out + c;
    if (j.muon) {
        const float p = t.master ? t.master[at] : element(t.out, at, bf16);
        o = p * t.decay - t.rate * o;
        if (t.master) t.master[at] = o;
    }
    if (bf16) gnn_rows<gnn_bf16>::set(static_cast<gnn_bf16 *>(t.out) + at, o);
    else static_cast<float *>(t.out)[at] = o;
}

// Rows row .. row + 3 of column col of a phase's result.
template <int P, Phase phase, typename T> __device__ __forceinline__ void write_down(const Job &j, const Mat &t, int step, int row, int col, const float (&v)[4]) {
    if (phase == kGram) put4<P>(t.a, t.mp, t.mp, col, row, v);
    else if (phase == kPolynomial) put4<P>(t.q, t.mp, t.mp, col, row, v);
    else if (phase == kUpdate) put4<P>(t.xt[(step + 1) & 1], t.np, t.mp, col, row, v);
    else if (!(t.flags & kTall)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (row + i < t.m && col < t.n) write_out<T>(j, t, row + i, col, v[i]);
    }
}
// Columns col .. col + 3 of row `row`.
template <int P, Phase phase, typename T> __device__ __forceinline__ void write_across(const Job &j, const Mat &t, int row, int col, const float (&v)[4]) {
    if (phase == kGram) put4<P>(t.a, t.mp, t.mp, row, col, v);
    else if (phase == kPolynomial) put4<P>(t.q, t.mp, t.mp, row, col, v);
    else if (phase == kUpdate) put4<P>(t.x, t.mp, t.np, row, col, v);
    else if (t.flags & kTall) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (row < t.m && col + i < t.n) write_out<T>(j, t, col + i, row, v[i]);
    }
}

// What lanes of a wavefront wrote to LDS is there for its other lanes: LDS keeps their order, the compiler has to.
__device__ __forceinline__ void within_wavefront() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// A fragment of results on its way out: rows row0 .. row0 + 31, columns col0 .. col0 + 31, to both places where `both`.  The loop is not unrolled: code that
// a wavefront goes through once is as slow as it is fetched.
template <int P, Phase phase, typename T> __device__ __forceinline__ void write_fragment(const Job &j, const Mat &t, int times_log2, int step, int row0, int col0, const float (&turn)[32][33], bool both) {
    const int lane = int(threadIdx.x) & 63, l32 = lane & 31, lk = lane >> 5;
#pragma unroll 1
    for (int g = 0; g < 4; ++g) {
        const int at = 8 * g + 4 * lk;
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = turn[at + i][l32];
        finish<P, phase>(j, t, times_log2, row0 + at, col0 + l32, v);
        write_down<P, phase, T>(j, t, step, row0 + at, col0 + l32, v);
        if (!both) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = turn[l32][at + i];
        finish<P, phase>(j, t, times_log2, col0 + at, row0 + l32, v);
        write_across<P, phase, T>(j, t, row0 + l32, col0 + at, v);
    }
}

// Tiles of (32 T)^2: each of four wavefronts has all of the tile and every fourth 16 of k, straight from the caches, and keeps SETS steps on their way.
// Nothing waits but for its own loads; the four sums are added in LDS.
template <int P, Phase phase, typename OUT, int T> __global__ void __launch_bounds__(kThreads) split_product_kernel(const Job j, int step) {
    constexpr bool symmetric = phase == kGram || phase == kPolynomial;
    constexpr int SETS = 2;  // 602-1000-1000-41 bf16 258 us, three 263, four 271; 100-256-256-47 fp32 80.8, 82.6, 81.3
    typedef typename Parts<P>::Eight Eight;
    int number, ti, tj;
    const Mat &t = j.mat[matrix_of_block<symmetric ? kSymmetric : kOthers>(j, number)];
    const Operands o = operands<phase>(t, step);
    const int times_log2 = shift<P, phase>(j, t, step);
    const int side = o.rows / (32 * T), across = o.cols / (32 * T);
    tile_of<symmetric, 1>(number, symmetric ? side * (side + 1) / 2 : side * across, across, ti, tj);
    const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int ks = o.depth / 16;
    const Eight *left = reinterpret_cast<const Eight *>(o.left) + int64_t(ti) * T * 64 + lane;
    const Eight *right = reinterpret_cast<const Eight *>(o.right) + int64_t(tj) * T * 64 + lane;
    const int64_t left_plane = int64_t(o.rows) * o.depth / 8, right_plane = int64_t(o.cols) * o.depth / 8;
    constexpr int LOW = P == 2 ? T : 1;
    float16v acc[T][T], low[LOW][LOW];
    clear<T, T>(acc);
    clear<LOW, LOW>(low);
    Eight a[SETS][T][P], b[SETS][T][P];
    auto load = [&](int set, int k) {  // behind the last step: that one again
        const int64_t at = k < ks ? k : ks - 1;
#pragma unroll
        for (int x = 0; x < T; ++x)
#pragma unroll
            for (int p = 0; p < P; ++p) {
                a[set][x][p] = left[p * left_plane + at * (o.rows * 2) + x * 64];
                b[set][x][p] = right[p * right_plane + at * (o.cols * 2) + x * 64];
            }
    };
#pragma unroll
    for (int u = 0; u < SETS; ++u) load(u, wave + 4 * u);
    for (int k = wave; k < ks; k += 4 * SETS) {
        float16v sum[T][T];
        clear<T, T>(sum);
#pragma unroll
        for (int u = 0; u < SETS; ++u) {
            if (k + 4 * u >= ks) break;
#pragma unroll
            for (int x = 0; x < T; ++x) add_products<P, T>(sum[x], low[P == 2 ? x : 0], a[u][x], b[u]);
            load(u, k + 4 * (u + SETS));
        }
        add<T, T>(acc, sum);
    }
    if constexpr (P == 2) add<T, T>(acc, low, 1.0f / Parts<P>::kRest);
    const int l32 = lane & 31, lk = lane >> 5;
    if constexpr (T == 1) {
        // a wavefront adds up and writes eight rows, and eight columns for the other place
        __shared__ float tile[4][32][33];
        const int at = 8 * wave + 4 * lk, row0 = ti * 32, col0 = tj * 32;
#pragma unroll
        for (int v = 0; v < 16; ++v) tile[wave][8 * (v / 4) + 4 * lk + v % 4][l32] = acc[0][0][v];
        __syncthreads();
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (tile[0][at + i][l32] + tile[1][at + i][l32]) + (tile[2][at + i][l32] + tile[3][at + i][l32]);
        finish<P, phase>(j, t, times_log2, row0 + at, col0 + l32, v);
        write_down<P, phase, OUT>(j, t, step, row0 + at, col0 + l32, v);
        if (symmetric && ti == tj) return;  // (a tile on the diagonal is computed whole)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (tile[0][l32][at + i] + tile[1][l32][at + i]) + (tile[2][l32][at + i] + tile[3][l32][at + i]);
        finish<P, phase>(j, t, times_log2, col0 + at, row0 + l32, v);
        write_across<P, phase, OUT>(j, t, row0 + l32, col0 + at, v);
    } else {
        // a wavefront adds up and writes one fragment of the tile
        static_assert(T == 2, "a fragment a wavefront");
        __shared__ union {
            float part[4][4][16][64];
            float turn[4][32][33];
        } lds;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int v = 0; v < 16; ++v) lds.part[wave][2 * x + y][v][lane] = acc[x][y][v];
        __syncthreads();
        float sum[16];
#pragma unroll
        for (int v = 0; v < 16; ++v)
            sum[v] = (lds.part[0][wave][v][lane] + lds.part[1][wave][v][lane]) + (lds.part[2][wave][v][lane] + lds.part[3][wave][v][lane]);
        __syncthreads();
#pragma unroll
        for (int v = 0; v < 16; ++v) lds.turn[wave][8 * (v / 4) + 4 * lk + v % 4][l32] = sum[v];
        within_wavefront();
        write_fragment<P, phase, OUT>(j, t, times_log2, step, (ti * 2 + (wave >> 1)) * 32, (tj * 2 + (wave & 1)) * 32, lds.turn[wave], !(symmetric && ti == tj));
    }
}

// Tiles of 64 TI x 64 TJ through LDS (64 x 128; 128 x 128 2150 us for 2560 x 4000 where these took 1890): four wavefronts of TI x TJ fragments each, 16 KS k at a time, the next ones in the other half of the LDS and two more
// such steps on their way in registers (P = 2: 182, so two workgroups a unit; sums of second numbers that are scaled in place leave room for three and take as long).
template <int P, int TI, int TJ, int KS, Phase phase, typename T> __global__ void __launch_bounds__(kThreads, P == 2 ? 2 : 3) product_kernel(const Job j, int step) {
    typedef typename Parts<P>::Eight Eight;
    constexpr int ROWS = 2 * (TI + TJ), FRAGS = ROWS * P * KS, MINE = (FRAGS + 3) / 4;  // 32 rows of an operand; fragments of a step, of a wavefront
    static_assert(TJ % TI == 0, "tiles of symmetric results");
    __shared__ union {
        u32x4 frag[2][FRAGS][64];
        float turn[4][32][33];
    } lds;
    constexpr bool symmetric = phase == kGram || phase == kPolynomial;
    int number, ti, tj;
    const Mat &t = j.mat[matrix_of_block<symmetric ? kSymmetric : kOthers>(j, number)];
    const Operands o = operands<phase>(t, step);
    const int times_log2 = shift<P, phase>(j, t, step);
    const int down = o.rows / (64 * TI), across = o.cols / (64 * TJ);
    tile_of<symmetric, TJ / TI>(number, symmetric ? TJ / TI * (across * (across + 1) / 2) : down * across, across, ti, tj);
    const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int steps = o.depth / (16 * KS);

    // fragment f of a step: its 16 k, then 32 rows (of the left operand, then of the right one), then plane.  Where they cannot be shared out evenly the last
    // one is fetched more than once: branches around single loads cost more (three parts, 2560 x 4000 3110 us, 2940 so).
    const u32x4 *from[MINE];
    int64_t apart[MINE];  // from a step to the next, in 16 bytes
#pragma unroll
    for (int f = 0; f < MINE; ++f) {
        const int g = wave * MINE + f < FRAGS ? wave * MINE + f : FRAGS - 1, kk = g / (ROWS * P), r = g / P % ROWS, p = g % P;
        const bool right = r >= 2 * TI;
        const int64_t high = right ? o.cols : o.rows, rb = right ? int64_t(tj) * 2 * TJ + r - 2 * TI : int64_t(ti) * 2 * TI + r;
        from[f] = reinterpret_cast<const u32x4 *>((right ? o.right : o.left) + p * high * o.depth) + (kk * (high / 32) + rb) * 64;
        apart[f] = high * 2 * KS;
    }
    u32x4 next[2][MINE];
    auto load = [&](int set, int k) {  // behind the last step: that one again
#pragma unroll
        for (int f = 0; f < MINE; ++f) {
            next[set][f] = from[f][lane];
            from[f] += k + 1 < steps ? apart[f] : 0;
        }
    };
    auto stage = [&](int half) {
#pragma unroll
        for (int f = 0; f < MINE; ++f) lds.frag[half][wave * MINE + f < FRAGS ? wave * MINE + f : FRAGS - 1][lane] = next[half][f];
    };
    const int wi = wave >> 1, wj = wave & 1;
    constexpr int LOW_I = P == 2 ? TI : 1, LOW_J = P == 2 ? TJ : 1;
    float16v acc[TI][TJ], low[LOW_I][LOW_J];
    clear<TI, TJ>(acc);
    clear<LOW_I, LOW_J>(low);
    auto multiply = [&](int half) {
        __builtin_amdgcn_s_setprio(1);  // ahead of the other workgroup's wavefronts, which are then free to fetch: 2560 x 4000 1990 -> 1880 us when there were three
        float16v sum[TI][TJ];
        clear<TI, TJ>(sum);
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) {
            Eight a[TI][P], b[TJ][P];
#pragma unroll
            for (int x = 0; x < TI; ++x)
#pragma unroll
                for (int p = 0; p < P; ++p) a[x][p] = __builtin_bit_cast(Eight, lds.frag[half][(kk * ROWS + wi * TI + x) * P + p][lane]);
#pragma unroll
            for (int y = 0; y < TJ; ++y)
#pragma unroll
                for (int p = 0; p < P; ++p) b[y][p] = __builtin_bit_cast(Eight, lds.frag[half][(kk * ROWS + 2 * TI + wj * TJ + y) * P + p][lane]);
#pragma unroll
            for (int x = 0; x < TI; ++x) add_products<P, TJ>(sum[x], low[P == 2 ? x : 0], a[x], b);
        }
        add<TI, TJ>(acc, sum);
        __builtin_amdgcn_s_setprio(0);
    };
    load(0, 0);
    load(1, 1);
    stage(0);
    load(0, 2);
    __syncthreads();
#pragma unroll 1
    for (int k = 0;; k += 2) {
        multiply(0);
        if (k + 1 >= steps) break;
        stage(1);
        load(1, k + 3);
        __syncthreads();
        multiply(1);
        if (k + 2 >= steps) break;
        stage(0);
        load(0, k + 4);
        __syncthreads();
    }
    __syncthreads();
    if constexpr (P == 2) add<TI, TJ>(acc, low, 1.0f / Parts<P>::kRest);

    const int l32 = lane & 31, lk = lane >> 5;
#pragma unroll 1
    for (int q = 0; q < TI * TJ; ++q) {
#pragma unroll
        for (int x = 0; x < TI; ++x)
#pragma unroll
            for (int y = 0; y < TJ; ++y)
                if (q == x * TJ + y)
#pragma unroll
                    for (int v = 0; v < 16; ++v) lds.turn[wave][8 * (v / 4) + 4 * lk + v % 4][l32] = acc[x][y][v];
        within_wavefront();
        const int row0 = ti * 64 * TI + (wi * TI + q / TJ) * 32, col0 = tj * 64 * TJ + (wj * TJ + q % TJ) * 32;
        // squares of as many rows as a tile is wide are computed whole on the diagonal
        write_fragment<P, phase, T>(j, t, times_log2, step, row0, col0, lds.turn[wave], !(symmetric && row0 / (64 * TJ) == tj));
        within_wavefront();
    }
}

// ---- host

bool misaligned(const void *p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % uintptr_t(to) != 0; }
int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// A matrix as both calls describe it.
struct Entry {
    const void *in;
    void *out;
    float *momentum, *master;
    int64_t rows, cols, ld_in, ld_out;
    int32_t dtype;
    float decay, rate;
    bool skip;
};

// How the products of a matrix are tiled: 0 tiles of 32 x 32, k shared out; 1 of 64 x 64, the same; 2 of 64 x 128 through LDS.  Us in fp32 and bf16 alike:
// 800 x 800 157, 194 and 364, 1000 x 1000 203, 208 and 398, 1500 x 1800 604, 531 and 616, 2048 x 2048 1192, 923 and 838.
int kind_of(int64_t rows, int64_t cols) {
    const double m = double(rows < cols ? rows : cols), n = double(rows < cols ? cols : rows), work = m * m * n;
    return work <= 1.0e9 ? 0 : work <= 6.0e9 ? 1 : 2;
}
int64_t tile_of_kind(int kind) { return kind == 0 ? 32 : kind == 1 ? 64 : 128; }

struct Sizes {
    int kind, parts;
    int64_t m, n, mp, np, bytes;
    int32_t norm_blocks;
};
Sizes sizes_of(int64_t rows, int64_t cols, int parts) {
    Sizes s;
    s.kind = kind_of(rows, cols);
    s.parts = parts;
    s.m = rows < cols ? rows : cols;
    s.n = rows < cols ? cols : rows;
    const int64_t to = tile_of_kind(s.kind) < 64 ? 64 : tile_of_kind(s.kind);  // the first planes are made in tiles of 64
    s.mp = up(s.m, to);
    s.np = up(s.n, to);
    const int64_t blocks = (s.m * s.n + kNormChunk - 1) / kNormChunk;
    s.norm_blocks = int32_t(blocks < kNormBlocks ? blocks : kNormBlocks);
    s.bytes = 2 * s.parts * (3 * s.mp * s.np + 2 * s.mp * s.mp) + up(8 * (s.norm_blocks + 1), 256);
    return s;
}

template <int P, Phase phase, typename T> int launch_products(const Job &j, int kind, int step, int64_t blocks, hipStream_t stream) {
    if (blocks > INT32_MAX / kThreads) return GNN_ERR_UNSUPPORTED;
    if (kind == 0) split_product_kernel<P, phase, T, 1><<<unsigned(blocks), kThreads, 0, stream>>>(j, step);
    else if (kind == 1) split_product_kernel<P, phase, T, 2><<<unsigned(blocks), kThreads, 0, stream>>>(j, step);
    else product_kernel<P, 1, 2, P == 3 ? 1 : 2, phase, T><<<unsigned(blocks), kThreads, 0, stream>>>(j, step);
    GNN_HIP_TRY(hipGetLastError());
    return GNN_OK;
}

template <int P, typename T> int launch_job(const Job &j, int kind, const int64_t (&blocks)[kLaunches], int steps, hipStream_t stream) {
    norm_kernel<<<unsigned(blocks[kNorms]), kThreads, 0, stream>>>(j);
    planes_kernel<P, T><<<unsigned(blocks[kPlanes]), kThreads, 0, stream>>>(j);
    GNN_HIP_TRY(hipGetLastError());
    for (int s = 0; s < steps; ++s) {  // (what stays in planes is the same for all types)
        int rc = launch_products<P, kGram, float>(j, kind, s, blocks[kSymmetric], stream);
        if (rc == GNN_OK) rc = launch_products<P, kPolynomial, float>(j, kind, s, blocks[kSymmetric], stream);
        if (rc == GNN_OK) rc = s + 1 < steps ? launch_products<P, kUpdate, float>(j, kind, s, blocks[kOthers], stream) : launch_products<P, kLast, T>(j, kind, s, blocks[kOthers], stream);
        if (rc != GNN_OK) return rc;
    }
    return GNN_OK;
}

// Whether X, A and Q stay within what two fp16 numbers hold with the powers of two of Parts<2>, and directions of small singular values do not shrink below it; a
// matrix far below eps, which a step multiplies by a, keeps its power of two only where nothing grows faster.
// Singular values of X begin within 0 .. 1, and the step takes s to s q(s^2), q(t) = a + b t + c t^2: both have their extremes at the ends or where their
// derivative is 0.
bool two_parts_do(double a, double b, double c, int steps, float &growth) {
    if (!(fabs(a) >= 1.0)) return false;
    double most = 1.0 + 1e-6;
    for (int k = 0; k < steps; ++k) {
        const double top = most * most;
        auto q = [&](double t) { return fabs(a + t * (b + t * c)); };
        double q_most = fmax(q(0.0), q(top)), next = most * q(top);
        if (c != 0.0) {
            const double t = -b / (2.0 * c), root = 9.0 * b * b - 20.0 * a * c;
            if (t > 0.0 && t < top) q_most = fmax(q_most, q(t));
            if (root >= 0.0)
                for (int sign = -1; sign <= 1; sign += 2) {
                    const double u = (-3.0 * b + sign * sqrt(root)) / (10.0 * c);
                    if (u > 0.0 && u < top) next = fmax(next, sqrt(u) * q(u));
                }
        } else if (b != 0.0) {
            const double u = -a / (3.0 * b);
            if (u > 0.0 && u < top) next = fmax(next, sqrt(u) * q(u));
        }
        most = next * (1.0 + 1e-4);  // (roundings of the products)
        if (!(most <= 1.9) || !(q_most <= 7.5) || q_most > fabs(a)) return false;
    }
    growth = float(log2(fabs(a)) + 1e-4);
    return true;
}

// Matrices of the same kind and type, kMats at a time.
int orthogonalize(Entry (*at)(const void *, int64_t), const void *list, int64_t count, Job &j, double a, double b, double c, int steps, uint8_t *room, hipStream_t stream) {
    const int parts = two_parts_do(a, b, c, steps, j.growth) ? 2 : 3;
    const double unit_a = parts == 2 ? ldexp(1.0, Parts<2>::kALog2) : 1.0, unit_q = parts == 2 ? ldexp(1.0, Parts<2>::kQLog2) : 1.0;
    j.a = float(a * unit_q);
    j.b = float(b * (unit_q / unit_a));
    j.c = float(c * (unit_q / (unit_a * unit_a)));
    for (int kind = 0; kind < 3; ++kind)
        for (int32_t dtype : {GNN_F32, GNN_BF16}) {
            int64_t blocks[kLaunches];
            int matrices = 0;
            auto clear = [&]() {
                matrices = 0;
                for (int i = 0; i < kLaunches; ++i) {
                    blocks[i] = 0;
                    for (int32_t &f : j.first[i]) f = INT32_MAX;
                }
            };
            auto flush = [&]() -> int {
                if (matrices == 0) return GNN_OK;
                const int rc = parts == 2 ? dtype == GNN_F32 ? launch_job<2, float>(j, kind, blocks, steps, stream) : launch_job<2, gnn_bf16>(j, kind, blocks, steps, stream)
                               : dtype == GNN_F32 ? launch_job<3, float>(j, kind, blocks, steps, stream) : launch_job<3, gnn_bf16>(j, kind, blocks, steps, stream);
                clear();
                return rc;
            };
            clear();
            for (int64_t k = 0; k < count; ++k) {
                const Entry e = at(list, k);
                if (e.skip || e.rows == 0 || e.cols == 0) continue;
                const Sizes s = sizes_of(e.rows, e.cols, parts);
                if (s.kind != kind || e.dtype != dtype) continue;
                const int64_t tile = tile_of_kind(kind), across = s.mp / tile;
                // (large ones: two tiles of half the height for each square one)
                const int64_t more[kLaunches] = {s.norm_blocks, s.mp / 64 * (s.np / 64), across * (across + 1) / (kind == 2 ? 1 : 2),
                                                 across * (s.np / tile) * (kind == 2 ? 2 : 1)};
                bool full = matrices == kMats;
                for (int i = 0; i < kLaunches; ++i) full |= blocks[i] + more[i] > INT32_MAX / kThreads;
                if (full) {
                    const int rc = flush();
                    if (rc != GNN_OK) return rc;
                }
                Mat &t = j.mat[matrices];
                t = Mat{};
                const int64_t xs = s.parts * s.mp * s.np, as = s.parts * s.mp * s.mp;
                uint16_t *p = reinterpret_cast<uint16_t *>(room);
                t.x = p;
                t.xt[0] = p + xs;
                t.xt[1] = p + 2 * xs;
                t.a = p + 3 * xs;
                t.q = t.a + as;
                t.squares = reinterpret_cast<double *>(t.q + as);
                room += s.bytes;
                t.in = e.in;
                t.out = e.out;
                t.momentum = e.momentum;
                t.master = e.master;
                t.ld_in = e.ld_in;
                t.ld_out = e.ld_out;
                t.m = int32_t(s.m);
                t.n = int32_t(s.n);
                t.mp = int32_t(s.mp);
                t.np = int32_t(s.np);
                t.rows = int32_t(e.rows);
                t.cols = int32_t(e.cols);
                t.norm_blocks = s.norm_blocks;
                t.flags = (e.dtype == GNN_BF16 ? kBf16 : 0) | (e.rows > e.cols ? kTall : 0);
                t.decay = e.decay;
                t.rate = e.rate;
                for (int i = 0; i < kLaunches; ++i) {
                    j.first[i][matrices] = int32_t(blocks[i]);
                    blocks[i] += more[i];
                }
                ++matrices;
            }
            const int rc = flush();
            if (rc != GNN_OK) return rc;
        }
    return GNN_OK;
}

bool sides_fit(int64_t rows, int64_t cols) { return rows >= 0 && cols >= 0 && rows <= kMostSide && cols <= kMostSide; }
bool known(int32_t dtype) { return dtype == GNN_F32 || dtype == GNN_BF16; }
int64_t size_of(int32_t dtype) { return dtype == GNN_F32 ? 4 : 2; }
bool is_finite(double x) { return x - x == 0.0; }

int check_matrix(const gnn_orthogonalize_matrix &t) {
    if (!sides_fit(t.rows, t.cols) || !known(t.dtype)) return GNN_ERR_INVALID_ARG;
    if ((t.ld_in && t.ld_in < t.cols) || (t.ld_out && t.ld_out < t.cols)) return GNN_ERR_INVALID_ARG;
    if (t.rows == 0 || t.cols == 0) return GNN_OK;
    if (!t.in || !t.out || misaligned(t.in, size_of(t.dtype)) || misaligned(t.out, size_of(t.dtype))) return GNN_ERR_INVALID_ARG;
    if (t.in == t.out && t.rows > 1 && (t.ld_in ? t.ld_in : t.cols) != (t.ld_out ? t.ld_out : t.cols)) return GNN_ERR_INVALID_ARG;
    return GNN_OK;
}
int check_matrix(const gnn_muon_matrix &t) {
    if (!sides_fit(t.rows, t.cols) || !known(t.dtype) || !(t.weight_decay >= 0.0f) || !is_finite(t.update_scale)) return GNN_ERR_INVALID_ARG;
    if (t.rows == 0 || t.cols == 0 || !t.grad) return GNN_OK;
    if (!t.param || !t.momentum || (t.master && t.dtype == GNN_F32)) return GNN_ERR_INVALID_ARG;
    if (misaligned(t.param, size_of(t.dtype)) || misaligned(t.grad, size_of(t.dtype)) || misaligned(t.momentum, 4) || misaligned(t.master, 4)) return GNN_ERR_INVALID_ARG;
    return GNN_OK;
}
bool leaves_alone(const gnn_orthogonalize_matrix &) { return false; }
bool leaves_alone(const gnn_muon_matrix &t) { return !t.grad; }

// -1: a matrix that the call refuses
template <typename M> int64_t room_of(const M *matrices, int64_t count) {
    if (count < 0 || (count > 0 && !matrices)) return -1;
    int64_t bytes = 0;
    for (int64_t k = 0; k < count; ++k) {
        if (check_matrix(matrices[k]) != GNN_OK) return -1;
        if (matrices[k].rows > 0 && matrices[k].cols > 0 && !leaves_alone(matrices[k])) bytes += sizes_of(matrices[k].rows, matrices[k].cols, 3).bytes;
    }
    return bytes;
}
bool coefficients_fit(double a, double b, double c, double eps, int32_t steps) {
    return is_finite(a) && is_finite(b) && is_finite(c) && eps > 0.0 && is_finite(eps) && steps >= 1 && steps <= kMostSteps;
}

}  // namespace

extern "C" GNN_API int64_t gnn_orthogonalize_workspace_bytes(const gnn_orthogonalize_matrix *matrices, int64_t n_matrices) {
    const int64_t bytes = room_of(matrices, n_matrices);
    return bytes < 0 ? 0 : bytes;
}

extern "C" GNN_API int gnn_orthogonalize(const gnn_orthogonalize_matrix *matrices, int64_t n_matrices, const gnn_orthogonalize_opts *opts) {
    if (!opts || !coefficients_fit(opts->a, opts->b, opts->c, opts->eps, opts->steps)) return GNN_ERR_INVALID_ARG;
    const gnn_orthogonalize_opts &o = *opts;
    const int64_t bytes = room_of(matrices, n_matrices);
    if (bytes < 0) return GNN_ERR_INVALID_ARG;
    if (bytes == 0) return GNN_OK;
    if (!o.workspace || misaligned(o.workspace, 256) || o.workspace_bytes < bytes) return GNN_ERR_INVALID_ARG;
    (void)hipGetLastError();
    Job j{};
    j.eps = o.eps;
    return orthogonalize(
        [](const void *list, int64_t k) {
            const gnn_orthogonalize_matrix &t = static_cast<const gnn_orthogonalize_matrix *>(list)[k];
            return Entry{t.in, t.out, nullptr, nullptr, t.rows, t.cols, t.ld_in ? t.ld_in : t.cols, t.ld_out ? t.ld_out : t.cols, t.dtype, 1.0f, 1.0f, false};
        },
        matrices, n_matrices, j, o.a, o.b, o.c, o.steps, static_cast<uint8_t *>(o.workspace), static_cast<hipStream_t>(o.stream));
}

extern "C" GNN_API int64_t gnn_muon_workspace_bytes(const gnn_muon_matrix *matrices, int64_t n_matrices) {
    const int64_t bytes = room_of(matrices, n_matrices);
    return bytes < 0 ? 0 : bytes;
}

extern "C" GNN_API int gnn_muon_step(const gnn_muon_matrix *matrices, int64_t n_matrices, const gnn_muon_opts *opts) {
    if (!opts || !coefficients_fit(opts->a, opts->b, opts->c, opts->eps, opts->steps)) return GNN_ERR_INVALID_ARG;
    const gnn_muon_opts &o = *opts;
    if (!(o.lr >= 0.0) || !is_finite(o.lr) || !(o.momentum >= 0.0 && o.momentum < 1.0) || (o.nesterov & ~1)) return GNN_ERR_INVALID_ARG;
    const int64_t bytes = room_of(matrices, n_matrices);
    if (bytes < 0) return GNN_ERR_INVALID_ARG;
    if (bytes == 0) return GNN_OK;
    if (!o.workspace || misaligned(o.workspace, 256) || o.workspace_bytes < bytes) return GNN_ERR_INVALID_ARG;
    (void)hipGetLastError();
    Job j{};
    j.muon = 1;
    j.nesterov = o.nesterov;
    j.mu = float(o.momentum);
    j.eps = o.eps;
    j.grad_scale = o.grad_scale;
    struct List { const gnn_muon_matrix *matrices; double lr; } list{matrices, o.lr};
    return orthogonalize(
        [](const void *p, int64_t k) {
            const List &l = *static_cast<const List *>(p);
            const gnn_muon_matrix &t = l.matrices[k];
            return Entry{t.grad, t.param, t.momentum, t.master, t.rows, t.cols, t.cols, t.cols, t.dtype, float(1.0 - l.lr * double(t.weight_decay)),
                      float(l.lr * double(t.update_scale)), t.grad == nullptr};
        },
        &list, n_matrices, j, o.a, o.b, o.c, o.steps, static_cast<uint8_t *>(o.workspace), static_cast<hipStream_t>(o.stream));
}
