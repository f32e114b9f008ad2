// Rows kept in 8 bits: e4m3 codes with an exponent for every 32 neighbouring columns, written and read by id.
//
//     value[c] = code[c] 2^(e - 127),   e = the least with max |x| 2^(127 - e) <= 448 = 1.75 * 2^8:
//     of max = 1.f * 2^x   e - 127 = x - 8, or x - 7 where 1.f > 1.75.
//
// The factor is a power of two, so that products with it are exact and the code is the only rounding: results do not depend on how the kernel
// is written.  A code has four significant bits wherever the block's largest value lies, so a power of two costs at most one of the 17 binary orders of
// magnitude that a block spans, and takes one byte where a factor in fp32 takes four.  Codes and exponents of a row lie side by side: a row that is
// read by id costs the lines of one place.
//
// Eight columns a thread, whole rows a workgroup; the four threads of a block find its largest value by lane permutations.  Of rows written with the same id
// the last one has to stay: a row is written only if no later position has its id.  Few positions are compared in every workgroup;
// else each position is entered at its id, then raised to the last one, in two small passes before the rows.
#include "common.h"
#include "rows.h"

namespace {

constexpr int kThreads = 256;
constexpr int kItems = 1024;           // pieces of eight columns of a workgroup
constexpr int kBlock = GNN_STORE_BLOCK;
constexpr int64_t kCompareHere = 4096; // positions up to which every workgroup compares its rows' ids with all of them
constexpr int kCompareRows = 16;       // rows of a workgroup then
constexpr int kStoreRows = kItems / (kBlock / 8), kLoadRows = kItems;  // of a workgroup at most
constexpr int kPartsLog2 = 3, kParts = 1 << kPartsLog2, kChunk = 512;
constexpr int64_t kMostRows = INT32_MAX, kMostColumns = 1 << 24;
constexpr unsigned kGridX = 1 << 20;   // workgroups in x: a launch has fewer than 2^32 threads a dimension

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));

struct Rows {
    const void *ids;       // or nullptr: row i is position i
    void *x;               // matrix of numbers
    uint8_t *store;
    int32_t *last;         // [v] the last position with this id, or nullptr
    int64_t v, n, ldx, lds;
    int32_t f, pieces, rows;  // columns; pieces of eight of a row; rows of a workgroup
    uint32_t reciprocal;      // ceil(2^32 / pieces): quotients of numbers below 2^16
    int32_t is_64;
    __device__ __forceinline__ int64_t id(int64_t i) const {
        if (!ids) return i;
        const int64_t t = is_64 ? static_cast<const int64_t *>(ids)[i] : int64_t(static_cast<const int32_t *>(ids)[i]);
        return uint64_t(t) < uint64_t(v) ? t : -1;
    }
    __device__ __forceinline__ int row_of(int t) const { return pieces == 1 ? t : rows > 1 ? int(__umulhi(uint32_t(t), reciprocal)) : 0; }
};

struct Place { int64_t store, x; };  // of a row, from the store's first and from the workgroup's first row of X

__device__ __forceinline__ int64_t block_number() { return int64_t(blockIdx.z) * kGridX + blockIdx.x; }

// ---- the last position of every id

// Workgroup b takes the ids that share lines of `last` with others of part b mod 8, of chunk b / 8 of the positions: workgroups of one part run on one
// XCD and begin in order, so that its L2 has whole lines and mostly the last position already when the first pass ends.
__device__ __forceinline__ bool mine(int64_t id) { return id >= 0 && ((id >> 5) & (kParts - 1)) == int(blockIdx.x & (kParts - 1)); }

__global__ void __launch_bounds__(kThreads) enter_kernel(const Rows a) {
    const int64_t i0 = (block_number() >> kPartsLog2) * kChunk + threadIdx.x;
    int64_t id[kChunk / kThreads];
#pragma unroll
    for (int u = 0; u < kChunk / kThreads; ++u) id[u] = i0 + u * kThreads < a.n ? a.id(i0 + u * kThreads) : -1;
#pragma unroll
    for (int u = 0; u < kChunk / kThreads; ++u)
        if (mine(id[u])) a.last[id[u]] = int32_t(i0 + u * kThreads);  // of several any one
}
__global__ void __launch_bounds__(kThreads) raise_kernel(const Rows a) {
    const int64_t i0 = a.n - 1 - ((block_number() >> kPartsLog2) * kChunk + threadIdx.x);
    int64_t id[kChunk / kThreads];
    int32_t last[kChunk / kThreads];
#pragma unroll
    for (int u = 0; u < kChunk / kThreads; ++u) id[u] = i0 - u * kThreads >= 0 ? a.id(i0 - u * kThreads) : -1;
#pragma unroll
    for (int u = 0; u < kChunk / kThreads; ++u) last[u] = mine(id[u]) ? a.last[id[u]] : INT32_MAX;
#pragma unroll
    for (int u = 0; u < kChunk / kThreads; ++u)
        if (last[u] < int32_t(i0 - u * kThreads)) atomicMax(&a.last[id[u]], int32_t(i0 - u * kThreads));
}

// ---- writing

// eight columns from c on, or as many as there are; the others are 0
template <typename T> __device__ __forceinline__ void load8(const T *p, int have, float (&x)[8]) {
    if (have == 8) {
        constexpr int W = gnn_rows<T>::VEC;
#pragma unroll
        for (int k = 0; k < 8 / W; ++k) {
            float t[W];
            gnn_load_row<T, W, true>(p + k * W, t);
#pragma unroll
            for (int j = 0; j < W; ++j) x[k * W + j] = t[j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = j < have ? gnn_rows<T>::get(p + j) : 0.0f;
    }
}

typedef short v2i16 __attribute__((ext_vector_type(2)));

// Four columns in 8 bits, over 2^(e - 127), given as the fp32 number of that exponent (2^-127 as 0): the conversion scales before it rounds, to the bit what a
// product with the factor followed by a conversion gives, for every finite value and exponent.
__device__ __forceinline__ uint32_t codes4(const float (&x)[8], int j, float scale) {
    v2i16 t = {0, 0};
    t = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(t, x[j], x[j + 1], scale, false);
    t = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(t, x[j + 2], x[j + 3], scale, true);
    return __builtin_bit_cast(uint32_t, t);
}

// Columns 8 q .. 8 q + 8 of a row in 8 bits, with those of the three threads beside this one.  PAST: past the caches, as many rows as they do not hold are
// (1.2 M rows x 256 bf16 with other inputs between 213 us, through the caches 237; written again and again to the same places 213 and 177).
template <bool PAST> __device__ __forceinline__ void write8(const Rows &a, int64_t offset, int q, const float (&x)[8]) {
    const int c = q * 8, left = a.f - c, have = left < 0 ? 0 : left < 8 ? left : 8;
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t b = __float_as_uint(x[j]) & 0x7FFFFFFFu;
        top = b > top ? b : top;
    }
    const bool odd = top >= 0x7F800000u;
    if (odd) {
        top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t b = __float_as_uint(x[j]) & 0x7FFFFFFFu;
            top = b < 0x7F800000u && b > top ? b : top;
        }
    }
    const uint32_t other = __float_as_uint(gnn_from_lane<0xB1>(__uint_as_float(top)));  // the other of a pair
    top = other > top ? other : top;
    const uint32_t pair = __float_as_uint(gnn_from_lane<0x4E>(__uint_as_float(top)));   // the other pair of four
    top = pair > top ? pair : top;
    int e = int((top + 0x1FFFFFu) >> 23) - 8;  // (a mantissa above 0x600000 carries)
    e = e > 0 ? e : 0;
    const float scale = __uint_as_float(uint32_t(e) << 23);
    uint32_t w[2] = {codes4(x, 0, scale), codes4(x, 4, scale)};
    if (odd)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if ((__float_as_uint(x[j]) & 0x7FFFFFFFu) >= 0x7F800000u) w[j / 4] |= 0x7Fu << (8 * (j % 4));
    uint8_t *to = a.store + offset;
    if (have == 8) {
        if constexpr (PAST) __builtin_nontemporal_store(u32x2_any{w[0], w[1]}, reinterpret_cast<u32x2_any *>(to + c));
        else *reinterpret_cast<u32x2_any *>(to + c) = u32x2_any{w[0], w[1]};
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < have) to[c + j] = uint8_t(w[j / 4] >> (8 * (j % 4)));
    }
    if ((q & 3) == 0) to[a.f + (q >> 2)] = uint8_t(e);
}

constexpr int kAtOnce = 4;  // pieces of a thread on their way

// Few positions: rows are fetched before their ids are compared (1,021 rows x 64 fp32 9.0 us in the kernel with the way below, 5.0 so).
template <typename T> __global__ void __launch_bounds__(kThreads) few_store_kernel(const Rows a) {
    const int row0 = int(blockIdx.x) * a.rows, n = int(a.n), rows = n - row0 < a.rows ? n - row0 : a.rows;
    __shared__ __attribute__((aligned(16))) int32_t ids[kCompareHere];
    __shared__ int again[kCompareRows];  // a later position has this row's id
    const T *x0 = static_cast<const T *>(a.x) + row0 * a.ldx;
    const int items = rows * a.pieces;
    int row[kAtOnce], q[kAtOnce];
    float x[kAtOnce][8];
    auto fetch = [&](int t0) {
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int t = t0 + u * kThreads < items ? t0 + u * kThreads : items - 1;
            row[u] = a.row_of(t);
            q[u] = t - row[u] * a.pieces;
            const int left = a.f - q[u] * 8, have = left < 0 ? 0 : left < 8 ? left : 8;
            load8<T>(x0 + row[u] * a.ldx + q[u] * 8, have, x[u]);
        }
    };
    const int fours = (n + 3) / 4 * 4;
    for (int j0 = row0 / 4 * 4 + int(threadIdx.x); j0 < fours; j0 += 4 * kThreads) {  // (positions before do not matter)
        int32_t v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = int32_t(a.id(j0 + u * kThreads < n ? j0 + u * kThreads : n - 1));
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (j0 + u * kThreads < fours) ids[j0 + u * kThreads] = j0 + u * kThreads < n ? v[u] : INT32_MIN;
    }
    fetch(int(threadIdx.x));
    if (threadIdx.x < kCompareRows) again[threadIdx.x] = 0;
    __syncthreads();
    // a thread a row and a sixteenth of the positions, four at a time
    const int r = int(threadIdx.x) % kCompareRows, i = row0 + r;
    if (r < rows) {
        const int32_t id = ids[i];
        bool found = false;
#pragma unroll 4
        for (int j = row0 / 4 * 4 + int(threadIdx.x) / kCompareRows * 4; j < n; j += kThreads / kCompareRows * 4) {
            const i32x4 t = *reinterpret_cast<const i32x4 *>(ids + j);
#pragma unroll
            for (int e = 0; e < 4; ++e) found |= t[e] == id && j + e > i;
        }
        if (found) again[r] = 1;
    }
    __syncthreads();
    for (int t0 = int(threadIdx.x); t0 < items;) {  // (pieces is a multiple of four: the threads of a block take part together)
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (t0 + u * kThreads >= items) continue;
            const int64_t id = ids[row0 + row[u]];
            if (id >= 0 && !again[row[u]]) write8<false>(a, id * a.lds, q[u], x[u]);
        }
        t0 += kThreads * kAtOnce;
        if (t0 < items) fetch(t0);
    }
}

template <typename T> __global__ void __launch_bounds__(kThreads) store_kernel(const Rows a) {
    const int64_t row0 = block_number() * a.rows;
    if (row0 >= a.n) return;
    const int rows = a.n - row0 < a.rows ? int(a.n - row0) : a.rows;
    __shared__ Place places[kStoreRows];
    __shared__ int written;
    if (threadIdx.x == 0) written = 0;
    __syncthreads();
    // the rows that are written, in any order
    for (int r = int(threadIdx.x); r < rows; r += kThreads) {
        const int64_t id = a.id(row0 + r);
        if (id >= 0 && (!a.last || a.last[id] == int32_t(row0 + r))) places[atomicAdd(&written, 1)] = {id * a.lds, r * a.ldx};
    }
    __syncthreads();
    const T *x0 = static_cast<const T *>(a.x) + row0 * a.ldx;
    const int items = written * a.pieces;
    constexpr int U = kAtOnce;
    for (int t0 = int(threadIdx.x); t0 < items; t0 += kThreads * U) {  // (pieces is a multiple of four: the threads of a block take part together)
        Place at[U];
        int q[U];
        float x[U][8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = t0 + u * kThreads < items ? t0 + u * kThreads : items - 1, row = a.row_of(t);
            q[u] = t - row * a.pieces;
            at[u] = places[row];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int left = a.f - q[u] * 8, have = left < 0 ? 0 : left < 8 ? left : 8;
            load8<T>(x0 + at[u].x + q[u] * 8, have, x[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (t0 + u * kThreads < items) write8<true>(a, at[u].store, q[u], x[u]);
    }
}

// ---- reading

__device__ __forceinline__ float decoded(uint32_t w, int j, int e) {
    float x;
    if (j == 0) x = __builtin_amdgcn_cvt_f32_fp8(int(w), 0);
    else if (j == 1) x = __builtin_amdgcn_cvt_f32_fp8(int(w), 1);
    else if (j == 2) x = __builtin_amdgcn_cvt_f32_fp8(int(w), 2);
    else x = __builtin_amdgcn_cvt_f32_fp8(int(w), 3);
    return __builtin_amdgcn_ldexpf(x, e - 127);
}
typedef float f32x2 __attribute__((ext_vector_type(2)));
// eight columns of one exponent below 255, as they lie in memory: two codes an instruction
__device__ __forceinline__ void put8(float *to, const uint32_t (&w)[2], float scale) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[k], scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[k], scale, true);
        __builtin_nontemporal_store(gnn_f32x4{lo.x, lo.y, hi.x, hi.y}, reinterpret_cast<gnn_f32x4 *>(to + 4 * k));
    }
}
__device__ __forceinline__ void put8(gnn_bf16 *to, const uint32_t (&w)[2], float scale) {
    gnn_u32x4 v;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        v[2 * k] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[k], scale, false));
        v[2 * k + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[k], scale, true));
    }
    __builtin_nontemporal_store(v, reinterpret_cast<gnn_u32x4 *>(to));
}

// E columns a thread: eight, or one of rows narrower than that
template <typename T, int E> __global__ void __launch_bounds__(kThreads) load_kernel(const Rows a) {
    constexpr int U = 4;
    const int64_t row0 = block_number() * a.rows;
    if (row0 >= a.n) return;
    const int rows = a.n - row0 < a.rows ? int(a.n - row0) : a.rows;
    __shared__ int64_t places[kLoadRows];  // where a row is in the store, -1: nowhere
    for (int r = int(threadIdx.x); r < rows; r += kThreads) {
        const int64_t id = a.id(row0 + r);
        places[r] = id < 0 ? -1 : id * a.lds;
    }
    __syncthreads();
    const int items = rows * a.pieces;
    T *y = static_cast<T *>(a.x) + row0 * a.ldx;
    for (int t0 = int(threadIdx.x); t0 < items; t0 += kThreads * U) {
        int64_t at[U];
        int row[U], col[U];
        u32x2_any w[U];
        uint8_t e[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // no branch between the loads: what lies behind the end repeats the last piece, and an id that names no row reads row 0
            const int t = t0 + u * kThreads < items ? t0 + u * kThreads : items - 1;
            row[u] = a.row_of(t);
            const int c = (t - row[u] * a.pieces) * E;
            col[u] = c < a.f - E ? c : a.f - E;  // the last piece ends with the row
            at[u] = places[row[u]];
        }
        if (a.v > 0)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint8_t *p = a.store + (at[u] < 0 ? 0 : at[u]);
                if constexpr (E == 8) w[u] = *reinterpret_cast<const u32x2_any *>(p + col[u]);
                else w[u].x = p[col[u]];
                e[u] = p[a.f + col[u] / kBlock];
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (t0 + u * kThreads >= items) break;
            T *to = y + row[u] * a.ldx + col[u];
            if constexpr (E == 1) {
                gnn_rows<T>::set(to, at[u] < 0 ? 0.0f : decoded(w[u].x, 0, e[u]));
            } else {
                const int first = kBlock - col[u] % kBlock;  // columns of the first block
                uint32_t c[2] = {w[u].x, w[u].y};
                int e0 = e[u];
                if (at[u] < 0) c[0] = c[1] = 0, e0 = 127;
                if ((first >= E || at[u] < 0) && e0 < 255) {
                    put8(to, c, __uint_as_float(uint32_t(e0) << 23));
                } else {  // the last piece reaches over a block's end, or an exponent whose power of two fp32 does not have
                    const int e1 = a.store[at[u] + a.f + (col[u] + E - 1) / kBlock];
#pragma unroll
                    for (int j = 0; j < E; ++j) gnn_rows<T>::set(to + j, decoded(c[j / 4], j % 4, j < first ? e0 : e1));
                }
            }
        }
    }
}

dim3 grid_of(int64_t blocks) {
    return blocks <= kGridX ? dim3(unsigned(blocks)) : dim3(kGridX, 1, unsigned((blocks + kGridX - 1) / kGridX));
}

bool misaligned(const void *p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % uintptr_t(to) != 0; }
int64_t used_bytes(int64_t F) { return F + (F + kBlock - 1) / kBlock; }

int check(const void *x, const void *ids, const void *store, int64_t V, int64_t n, int64_t F, const gnn_store_opts &o) {
    if (V < 0 || n < 0 || F < 0 || V > kMostRows || n > kMostRows || F > kMostColumns || (o.dtype != GNN_F32 && o.dtype != GNN_BF16)) return GNN_ERR_INVALID_ARG;
    if ((o.ids_is_64 & ~1) || (o.unique & ~1) || (o.ldx && o.ldx < F) || (o.lds && o.lds < used_bytes(F))) return GNN_ERR_INVALID_ARG;
    if (n == 0 || F == 0) return GNN_OK;
    if (!x || (V > 0 && !store) || (!ids && n > V) || (V > 0 && x == store)) return GNN_ERR_INVALID_ARG;
    if (misaligned(x, o.dtype == GNN_F32 ? 4 : 2) || misaligned(ids, o.ids_is_64 ? 8 : 4)) return GNN_ERR_INVALID_ARG;
    return GNN_OK;
}

Rows rows_of(const void *x, const void *ids, const void *store, int64_t V, int64_t n, int64_t F, int64_t pieces, int64_t most, const gnn_store_opts &o) {
    Rows a{};
    a.ids = ids;
    a.x = const_cast<void *>(x);
    a.store = static_cast<uint8_t *>(const_cast<void *>(store));
    a.v = V;
    a.n = n;
    a.ldx = o.ldx ? o.ldx : F;
    a.lds = o.lds ? o.lds : gnn_store_row_bytes(F);
    a.f = int32_t(F);
    a.is_64 = o.ids_is_64;
    a.pieces = int32_t(pieces);
    a.rows = int32_t(pieces >= kItems ? 1 : kItems / pieces);
    if (a.rows > most) a.rows = int32_t(most);
    a.reciprocal = pieces > 1 ? uint32_t(((uint64_t(1) << 32) + uint64_t(pieces) - 1) / uint64_t(pieces)) : 0;
    return a;
}

}  // namespace

extern "C" GNN_API int64_t gnn_store_row_bytes(int64_t F) { return F <= 0 || F > kMostColumns ? 0 : (used_bytes(F) + 15) / 16 * 16; }

extern "C" GNN_API int64_t gnn_store_rows_workspace_bytes(int64_t V, int64_t n) {
    return V <= 0 || n <= kCompareHere || V > kMostRows || n > kMostRows ? 0 : 4 * V;
}

extern "C" GNN_API int gnn_store_rows(const void *X, const void *ids, void *store, int64_t V, int64_t n, int64_t F, const gnn_store_opts *opts) {
    if (!opts) return GNN_ERR_INVALID_ARG;
    const gnn_store_opts &o = *opts;
    const int rc = check(X, ids, store, V, n, F, o);
    if (rc != GNN_OK || n == 0 || F == 0 || V == 0) return rc;
    const bool twice = ids && !o.unique;  // an id may come twice
    const bool compare = twice && n <= kCompareHere;
    if (twice && !compare && (!o.workspace || misaligned(o.workspace, 4) || o.workspace_bytes < 4 * V)) return GNN_ERR_INVALID_ARG;
    (void)hipGetLastError();
    Rows a = rows_of(X, ids, store, V, n, F, (F + kBlock - 1) / kBlock * (kBlock / 8), compare ? kCompareRows : kItems, o);
    hipStream_t stream = static_cast<hipStream_t>(o.stream);
    if (twice && !compare) {
        a.last = static_cast<int32_t *>(o.workspace);
        const dim3 grid = grid_of((n + kChunk - 1) / kChunk << kPartsLog2);
        enter_kernel<<<grid, kThreads, 0, stream>>>(a);
        raise_kernel<<<grid, kThreads, 0, stream>>>(a);
        GNN_HIP_TRY(hipGetLastError());
    }
    const dim3 grid = grid_of((n + a.rows - 1) / a.rows);
    if (o.dtype == GNN_F32) compare ? few_store_kernel<float><<<grid, kThreads, 0, stream>>>(a) : store_kernel<float><<<grid, kThreads, 0, stream>>>(a);
    else compare ? few_store_kernel<gnn_bf16><<<grid, kThreads, 0, stream>>>(a) : store_kernel<gnn_bf16><<<grid, kThreads, 0, stream>>>(a);
    GNN_HIP_TRY(hipGetLastError());
    return GNN_OK;
}

extern "C" GNN_API int gnn_load_rows(const void *store, const void *ids, void *Y, int64_t V, int64_t n, int64_t F, const gnn_store_opts *opts) {
    if (!opts) return GNN_ERR_INVALID_ARG;
    const gnn_store_opts &o = *opts;
    const int rc = check(Y, ids, store, V, n, F, o);
    if (rc != GNN_OK || n == 0 || F == 0) return rc;
    (void)hipGetLastError();
    const bool narrow = F < 8;
    const Rows a = rows_of(Y, ids, store, V, n, F, narrow ? F : (F + 7) / 8, kItems, o);
    hipStream_t stream = static_cast<hipStream_t>(o.stream);
    const dim3 grid = grid_of((n + a.rows - 1) / a.rows);
    if (o.dtype == GNN_F32) narrow ? load_kernel<float, 1><<<grid, kThreads, 0, stream>>>(a) : load_kernel<float, 8><<<grid, kThreads, 0, stream>>>(a);
    else narrow ? load_kernel<gnn_bf16, 1><<<grid, kThreads, 0, stream>>>(a) : load_kernel<gnn_bf16, 8><<<grid, kThreads, 0, stream>>>(a);
    GNN_HIP_TRY(hipGetLastError());
    return GNN_OK;
}
