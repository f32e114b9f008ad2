// Rows of a table by id, and the gradient of the table.
//
//     Y[i] = scale T[id_i]          dT[v] = scale sum of dY[i] over the i with id_i = v   (+ dT[v])
//
// Forward: a copy of rows.  A workgroup has some whole rows, their vectors side by side over its threads, four ids and four vectors of 16 bytes
// of a thread on their way at once, and ends with them.
//
// Gradient: the positions are sorted by id (stable, so that rows of equal ids keep their order), and the sorted list is cut into runs of
// kRun positions, whatever the ids: a group of lanes adds up its run's rows in registers and lets go of the sum where the id changes.  So every group
// does the same work, with eight rows on their way, whether an id comes once or a million times.  A sum whose positions all lie in one run is
// written by it; what crosses runs is joined in LDS, and what crosses workgroups by a second kernel, in fp64, in the order of the runs.  Rows
// that no id names are zeroed by further workgroups of the same launch, which look their ids up in the sorted list.
//
// Gradient of few positions: one launch, no list (4,096 x 64 of 1,021 positions 16.1 -> 5.0 us, of 2,048 22.5 -> 5.9, all of one id 25 -> 31).  A workgroup compares some positions with all, which gives a bit for every position of the same id; the
// position that comes first adds up the rows of them all, in fp64.
#include "common.h"
#include "rows.h"

namespace {

constexpr int kThreads = 256;
constexpr int kAtOnce = 4;        // vectors of a thread on their way, forward
// Sorted positions of a group of lanes, which are terms added one after the other in fp32: many where there are enough groups, else as many as are on
// their way at once.
constexpr int kRun = 32, kBatch = 8;
constexpr int64_t kLong = 1 << 17; // positions from which on runs are long
constexpr int64_t kRankHere = 6144; // positions up to which every workgroup finds the places of its ones among all (4,096 x 64 of 4,000: sorting 23 us, so 18; of 8,192: 24 and 29; of 300 K rows 43 and 41)
constexpr int kRankRows = 8;      // of a workgroup then (of 4,000: 32 rows 30 us, 8 rows 18)
constexpr int kFew = 2048;        // positions up to which there is one launch, if ids do not come more often than eight times on average
constexpr int kFewRows = 16;      // of a workgroup then
constexpr int kFewLanesLog2 = 4;  // lanes of a group then, at most
constexpr int kTogether = 32;     // positions of an id from which on all of the workgroup adds them up
constexpr int kZeroWide = 2048;   // rows of a workgroup that zeroes then, at most
constexpr int kZeroRows = 256;    // rows of a workgroup that zeroes, at most
constexpr int64_t kMostRows = INT32_MAX, kMostColumns = 1 << 24;
constexpr int64_t kMostSlices = 65535;  // workgroups in y: pieces of a row of as many vectors as a group has lanes
static_assert((kMostColumns / 4 + 127) / 128 <= kMostSlices, "the widest rows");
constexpr int64_t kCaches = 256 << 20;  // bytes
constexpr unsigned kGridX = 1 << 20;  // workgroups in x: a launch has fewer than 2^32 threads a dimension

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));  // (a vector type may stand for its elements in memory, a struct may not)

// E neighbouring elements in fp32
template <typename T, int E, bool NT = false> struct Vector {
    static constexpr int W = E < gnn_rows<T>::VEC ? E : gnn_rows<T>::VEC;
    static_assert(E % W == 0, "whole strips");
    gnn_strip<T, W, NT> s[E / W];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int k = 0; k < E / W; ++k) s[k].load(p + k * W);
    }
    __device__ __forceinline__ void get(float (&v)[E]) const {
#pragma unroll
        for (int k = 0; k < E / W; ++k) {
            float t[W];
            s[k].get(t);
#pragma unroll
            for (int j = 0; j < W; ++j) v[k * W + j] = t[j];
        }
    }
};
template <typename T, int E, bool NT> __device__ __forceinline__ void store_vector(T *p, const float (&v)[E]) {
    constexpr int W = Vector<T, E>::W;
#pragma unroll
    for (int k = 0; k < E / W; ++k) {
        float t[W];
#pragma unroll
        for (int j = 0; j < W; ++j) t[j] = v[k * W + j];
        gnn_store_row<T, W, NT>(p + k * W, t);
    }
}

struct Ids {
    const void *p;
    int is_64;
    int64_t rows;
    // the row that position i names, or -1
    __device__ __forceinline__ int64_t at(int64_t i) const {
        const int64_t v = is_64 ? static_cast<const int64_t *>(p)[i] : int64_t(static_cast<const int32_t *>(p)[i]);
        return uint64_t(v) < uint64_t(rows) ? v : -1;
    }
};

struct Lookup {
    const void *table;
    void *y;
    Ids ids;
    int64_t n, ldt, ldy;
    int32_t f, vectors, rows;   // columns; vectors of a row; rows of a workgroup
    uint32_t reciprocal;        // ceil(2^32 / vectors): quotients of numbers below 2^16
    float scale;
};

__device__ __forceinline__ int64_t block_number() { return int64_t(blockIdx.z) * kGridX + blockIdx.x; }

template <typename TT, typename TY, int E> __global__ void __launch_bounds__(kThreads) lookup_kernel(const Lookup a) {
    const int64_t row0 = block_number() * a.rows;
    if (row0 >= a.n) return;
    const int rows = a.n - row0 < a.rows ? int(a.n - row0) : a.rows;
    const int items = rows * a.vectors;
    const TT *table = static_cast<const TT *>(a.table);
    TY *y = static_cast<TY *>(a.y) + row0 * a.ldy;
    for (int t0 = int(threadIdx.x); t0 < items; t0 += kThreads * kAtOnce) {
        // no branch between the loads: what lies behind the end repeats the last vector, and an id that names no row reads row 0
        Vector<TT, E> v[kAtOnce];
        int64_t id[kAtOnce];
        int row[kAtOnce], col[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int t = t0 + u * kThreads < items ? t0 + u * kThreads : items - 1;
            row[u] = a.vectors == 1 ? t : a.rows > 1 ? int(__umulhi(uint32_t(t), a.reciprocal)) : 0;
            const int c = (t - row[u] * a.vectors) * E;
            col[u] = c < a.f - E ? c : a.f - E;  // the last vector ends with the row
            id[u] = a.ids.at(row0 + row[u]);
        }
        if (a.ids.rows > 0)
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) v[u].load(table + (id[u] < 0 ? 0 : id[u]) * a.ldt + col[u]);
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (t0 + u * kThreads >= items) break;
            float x[E];
            v[u].get(x);
#pragma unroll
            for (int j = 0; j < E; ++j) x[j] = id[u] < 0 ? 0.0f : x[j] * a.scale;
            store_vector<TY, E, true>(y + int64_t(row[u]) * a.ldy + col[u], x);
        }
    }
}

// ---- gradient

struct Grad {
    const void *dy;
    void *dtable;
    const uint32_t *key, *order;  // [n] ids sorted, `rows` where there is none; the positions they come from
    float *head, *tail;           // [blocks][f] what a workgroup has of the sum that began before it, and of the one that goes on behind it
    uint32_t *flags;              // [blocks]
    int64_t rows, n, ldt, ldy, sum_blocks, zero_blocks;
    int32_t f, vectors, lanes_log2, run;
    uint32_t reciprocal;          // ceil(2^32 / vectors)
    int32_t accumulate, zero_rows, whole_lines;  // rows of dY are such
    float scale;
};
enum : uint32_t { kHead = 1, kThrough = 2, kTail = 4 };  // a run has: the end of a sum that began before, nothing but the middle of one, the beginning of one that goes on

// Few positions: the place of each is the number of those that come before it.
__global__ void __launch_bounds__(kThreads) rank_kernel(const Ids ids, int n, uint32_t *__restrict__ key, uint32_t *__restrict__ order) {
    __shared__ __attribute__((aligned(16))) uint32_t all[kRankHere];
    __shared__ int before[kThreads];
    const int fours = (n + 3) / 4;
    for (int j0 = int(threadIdx.x); j0 < fours * 4; j0 += 4 * kThreads) {
        int64_t v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = ids.at(j0 + u * kThreads < n ? j0 + u * kThreads : n - 1);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = j0 + u * kThreads;
            if (j < fours * 4) all[j] = j >= n ? UINT32_MAX : uint32_t(v[u] < 0 ? ids.rows : v[u]);  // behind the last: after all others
        }
    }
    __syncthreads();
    // a thread a position and a 32nd of the others, four at a time
    const int i = int(blockIdx.x) * kRankRows + int(threadIdx.x) % kRankRows;
    int count = 0;
    if (i < n) {
        const uint32_t k = all[i];
#pragma unroll 4
        for (int j = int(threadIdx.x) / kRankRows * 4; j < n; j += kThreads / kRankRows * 4) {
            const u32x4 t = *reinterpret_cast<const u32x4 *>(all + j);
#pragma unroll
            for (int e = 0; e < 4; ++e) count += int(t[e] < k || (t[e] == k && j + e < i));
        }
    }
    before[threadIdx.x] = count;
    __syncthreads();
    if (int(threadIdx.x) >= kRankRows || i >= n) return;
    int place = 0;
#pragma unroll
    for (int p = 0; p < kThreads / kRankRows; ++p) place += before[p * kRankRows + threadIdx.x];
    key[place] = all[i];
    order[place] = uint32_t(i);
}

// first position of key[0 .. n) that is not below v
__device__ __forceinline__ int64_t first_not_below(const uint32_t *key, int64_t lo, int64_t hi, uint32_t v) {
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (key[mid] < v) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// sum * scale into row v (or onto it), columns c .. c + E; `own`: how many of them, the last ones, are no other lane's
template <typename TT, int E> __device__ __forceinline__ void write_sum(const Grad &a, int64_t v, int c, int own, const float (&sum)[E]) {
    TT *p = static_cast<TT *>(a.dtable) + v * a.ldt + c;
    float x[E];
#pragma unroll
    for (int j = 0; j < E; ++j) x[j] = sum[j] * a.scale;
    if (!a.accumulate) {
        store_vector<TT, E, true>(p, x);
    } else if (own == E) {
        Vector<TT, E> old;
        old.load(p);
        float o[E];
        old.get(o);
#pragma unroll
        for (int j = 0; j < E; ++j) x[j] += o[j];
        store_vector<TT, E, false>(p, x);
    } else {
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (j >= E - own) gnn_rows<TT>::set(p + j, gnn_rows<TT>::get(p + j) + x[j]);
    }
}

// rows v0 .. v0 + rows - 1, at most 256, where they are not named
template <typename TT, int E> __device__ __forceinline__ void zero_unnamed(const Grad &a, int64_t v0, int rows, const uint8_t *named) {
    TT *p = static_cast<TT *>(a.dtable) + v0 * a.ldt;
    const float zero[E] = {};
    // the rows' vectors side by side over the threads: stores of neighbouring rows meet in the same lines
    const int64_t items = int64_t(rows) * a.vectors;
    for (int64_t t = threadIdx.x; t < items; t += kThreads) {
        const int r = a.vectors == 1 ? int(t) : items < (1 << 16) ? int(__umulhi(uint32_t(t), a.reciprocal)) : int(t / a.vectors);
        if (named[r]) continue;
        const int q = int(t - int64_t(r) * a.vectors), c = q * E < a.f - E ? q * E : a.f - E;
        store_vector<TT, E, true>(p + r * a.ldt + c, zero);
    }
}

// rows of part b, at most 256, that no id names
template <typename TT, int E> __device__ __forceinline__ void zero_rows(const Grad &a, int64_t b) {
    static_assert(kZeroRows == kThreads, "a thread a row");
    __shared__ uint8_t named[kZeroRows];
    __shared__ int64_t range[2];
    const int64_t v0 = b * a.zero_rows;
    const int rows = a.rows - v0 < a.zero_rows ? int(a.rows - v0) : a.zero_rows;
    named[threadIdx.x] = 0;
    if (threadIdx.x < 2) range[threadIdx.x] = first_not_below(a.key, 0, a.n, uint32_t(v0 + (threadIdx.x ? rows : 0)));
    __syncthreads();
    const int64_t lo = range[0], hi = range[1];
    if (hi - lo <= 16 * kZeroRows) {
        for (int64_t j = lo + threadIdx.x; j < hi; j += kThreads) named[a.key[j] - uint32_t(v0)] = 1;
    } else if (int(threadIdx.x) < rows) {  // ids that come very often: one by one
        const uint32_t v = uint32_t(v0 + threadIdx.x);
        const int64_t j = first_not_below(a.key, lo, hi, v);
        named[threadIdx.x] = j < hi && a.key[j] == v;
    }
    __syncthreads();
    zero_unnamed<TT, E>(a, v0, rows, named);
}

// total += the rows of dY at positions `words` names words of `match` for: bit p of word w for position 32 w + p; B rows on their way
template <typename TY, int E, int B> __device__ __forceinline__ void add_positions(const TY *dy, int64_t ldy, const uint32_t *match, uint64_t words, double (&total)[E]) {
    uint32_t m = 0;
    int w = 0;
    for (;;) {
        int from[B];
#pragma unroll
        for (int u = 0; u < B; ++u) {
            if (m == 0 && words != 0) {  // (a word that is named has a bit)
                w = __builtin_ctzll(words);
                words &= words - 1;
                m = match[w];
            }
            from[u] = m ? w * 32 + __builtin_ctz(m) : -1;
            m &= m - 1;  // (0 stays 0)
        }
        if (from[0] < 0) return;
        Vector<TY, E> v[B];
#pragma unroll
        for (int u = 0; u < B; ++u) v[u].load(dy + int64_t(from[u] < 0 ? from[0] : from[u]) * ldy);
#pragma unroll
        for (int u = 0; u < B; ++u) {
            if (from[u] < 0) return;
            float x[E];
            v[u].get(x);
#pragma unroll
            for (int i = 0; i < E; ++i) total[i] += double(x[i]);
        }
    }
}

// At most kFew positions: workgroups of kFewRows of them, then those that zero.
template <typename TY, typename TT, int E> __global__ void __launch_bounds__(kThreads) few_grad_kernel(const Grad a, const Ids ids, int zero_wide) {
    static_assert(kFew == 64 * 32, "a bit a word");
    const int n = int(a.n);
    if (block_number() >= a.sum_blocks) {
        if (blockIdx.y > 0) return;
        __shared__ uint8_t named[kZeroWide];
        const int64_t number = block_number() - a.sum_blocks;
        if (number >= a.zero_blocks) return;
        const int64_t v0 = number * zero_wide;
        const int rows = a.rows - v0 < zero_wide ? int(a.rows - v0) : zero_wide;
        for (int r = int(threadIdx.x); r < rows; r += kThreads) named[r] = 0;
        __syncthreads();
        for (int j = int(threadIdx.x); j < n; j += kThreads) {
            const int64_t r = ids.at(j) - v0;
            if (r >= 0 && r < rows) named[r] = 1;
        }
        __syncthreads();
        for (int r = 0; r < rows; r += kZeroRows) zero_unnamed<TT, E>(a, v0 + r, rows - r < kZeroRows ? rows - r : kZeroRows, named + r);
        return;
    }
    __shared__ __attribute__((aligned(16))) uint32_t all[kFew];
    __shared__ uint32_t match[kFewRows][65];  // bit j of a row's: position j has its id
    __shared__ unsigned long long words[kFewRows];
    __shared__ int count[kFewRows];
    __shared__ double parts[kThreads][E];
    const int n_words = (n + 31) / 32, i0 = int(blockIdx.x) * kFewRows;
    for (int j0 = int(threadIdx.x); j0 < n_words * 32; j0 += 4 * kThreads) {
        int64_t v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = ids.at(j0 + u * kThreads < n ? j0 + u * kThreads : n - 1);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int j = j0 + u * kThreads;
            if (j < n_words * 32) all[j] = j >= n || v[u] < 0 ? UINT32_MAX : uint32_t(v[u]);
        }
    }
    if (threadIdx.x < kFewRows) {
        words[threadIdx.x] = 0;
        count[threadIdx.x] = 0;
    }
    __syncthreads();
    {
        const int r = int(threadIdx.x) % kFewRows;
        const uint32_t k = i0 + r < n ? all[i0 + r] : UINT32_MAX;
        if (k != UINT32_MAX)
            for (int w = int(threadIdx.x) / kFewRows; w < n_words; w += kThreads / kFewRows) {
                uint32_t m = 0;
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    const u32x4 t = *reinterpret_cast<const u32x4 *>(all + w * 32 + j);
#pragma unroll
                    for (int e = 0; e < 4; ++e) m |= uint32_t(t[e] == k) << (j + e);
                }
                match[r][w] = m;
                if (m) {
                    atomicOr(&words[r], 1ull << w);
                    atomicAdd(&count[r], __builtin_popcount(m));
                }
            }
    }
    __syncthreads();
    const int lanes = 1 << a.lanes_log2, lane = int(threadIdx.x) & (lanes - 1), group = int(threadIdx.x) >> a.lanes_log2, groups = kThreads >> a.lanes_log2;
    const int q = int(blockIdx.y) * lanes + lane;
    const bool mine = q < a.vectors;
    const int c = !mine ? 0 : q * E < a.f - E ? q * E : a.f - E;
    const int own = q * E < a.f - E ? E : a.f - q * E;
    const TY *dy = static_cast<const TY *>(a.dy) + c;
    auto first_of_its_id = [&](int r) {
        const int w = __builtin_ctzll(words[r]);
        return w * 32 + __builtin_ctz(match[r][w]) == i0 + r;
    };
    bool together = false;
    for (int r = 0; r < kFewRows; ++r) together |= count[r] >= kTogether;
    for (int r = group; r < kFewRows; r += groups) {
        if (count[r] == 0 || count[r] >= kTogether || !first_of_its_id(r)) continue;
        double total[E] = {};
        add_positions<TY, E, 4>(dy, a.ldy, match[r], words[r], total);
        float x[E];
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = float(total[i]);
        if (mine) write_sum<TT, E>(a, all[i0 + r], c, own, x);
    }
    if (!together) return;
    const uint64_t every = groups >= 64 ? (group < 64 ? 1ull << group : 0ull) : ~0ull / ((1ull << groups) - 1) << group;  // words group, group + groups, ...
    for (int r = 0; r < kFewRows; ++r) {
        if (count[r] < kTogether || !first_of_its_id(r)) continue;
        double total[E] = {};
        add_positions<TY, E, 8>(dy, a.ldy, match[r], words[r] & every, total);
#pragma unroll
        for (int i = 0; i < E; ++i) parts[threadIdx.x][i] = total[i];
        __syncthreads();
        if (group == 0 && mine) {
            float x[E];
            const int have = groups < 64 ? groups : 64;
            for (int g = 1; g < have; ++g)
#pragma unroll
                for (int i = 0; i < E; ++i) total[i] += parts[(g << a.lanes_log2) + lane][i];
#pragma unroll
            for (int i = 0; i < E; ++i) x[i] = float(total[i]);
            write_sum<TT, E>(a, all[i0 + r], c, own, x);
        }
        __syncthreads();
    }
}

template <typename TY, typename TT, int E, bool PAST> __global__ void __launch_bounds__(kThreads) grad_kernel(const Grad a) {
    // the workgroups that zero lie between those that add up, so that writes and reads go on beside each other
    const int64_t number = block_number(), all = a.sum_blocks + a.zero_blocks;
    if (number >= all) return;
    const int64_t block = number * a.sum_blocks / all;
    if ((number + 1) * a.sum_blocks / all == block) {
        if (blockIdx.y == 0) zero_rows<TT, E>(a, number - block);
        return;
    }
    __shared__ float parts[2][kThreads][E];  // what a group has of the sums that cross its ends
    __shared__ uint32_t flags[kThreads];
    const int lanes = 1 << a.lanes_log2, lane = int(threadIdx.x) & (lanes - 1), group = int(threadIdx.x) >> a.lanes_log2, groups = kThreads >> a.lanes_log2;
    const int q = int(blockIdx.y) * lanes + lane;
    const bool mine = q < a.vectors;
    const int c = !mine ? 0 : q * E < a.f - E ? q * E : a.f - E;
    const int own = q * E < a.f - E ? E : a.f - q * E;
    const uint32_t none = uint32_t(a.rows);
    const int64_t j0 = (block * groups + group) * a.run;
    const TY *dy = static_cast<const TY *>(a.dy) + c;

    float sum[E];
    uint32_t my_flags = 0, id = none;
    bool first = false;  // the sum began before this run
    if (j0 < a.n) {
#pragma unroll
        for (int j = 0; j < E; ++j) sum[j] = 0.0f;
        id = a.key[j0];
        first = j0 > 0 && id != none && a.key[j0 - 1] == id;
        if (first) my_flags = kHead;
        const int64_t end = j0 + a.run < a.n ? j0 + a.run : a.n;
#pragma unroll 1
        for (int64_t j = j0; j < end; j += kBatch) {
            if (id == none) break;  // the list ends with the positions whose id names no row (2.4 M x 256 bf16 of 47 ids, half of them none, 252 -> 156 us)
            // no branch between the loads: behind the end and for ids that name no row row 0 is read (both arrays end with a whole batch)
            uint32_t k[kBatch], from[kBatch];
            Vector<TY, E, PAST> v[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; u += 4) {
                const u32x4 ku = *reinterpret_cast<const u32x4 *>(a.key + j + u), pu = *reinterpret_cast<const u32x4 *>(a.order + j + u);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    k[u + e] = ku[e];
                    from[u + e] = pu[e];
                }
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) from[u] = j + u < end && k[u] != none ? from[u] : 0;
#pragma unroll
            for (int u = 0; u < kBatch; ++u) v[u].load(dy + int64_t(from[u]) * a.ldy);
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                if (j + u >= end) break;
                if (k[u] != id) {
                    if (first) {
#pragma unroll
                        for (int i = 0; i < E; ++i) parts[0][threadIdx.x][i] = sum[i];
                    } else if (id != none && mine) {
                        write_sum<TT, E>(a, id, c, own, sum);
                    }
                    first = false;
                    id = k[u];
#pragma unroll
                    for (int i = 0; i < E; ++i) sum[i] = 0.0f;
                }
                float x[E];
                v[u].get(x);
#pragma unroll
                for (int i = 0; i < E; ++i) sum[i] += x[i];  // (of ids that name no row: a sum that goes nowhere)
            }
        }
        const bool goes_on = id != none && end < a.n && a.key[end] == id;
        if (first) {
            if (goes_on) my_flags |= kThrough;
#pragma unroll
            for (int i = 0; i < E; ++i) parts[0][threadIdx.x][i] = sum[i];
        } else if (goes_on) {
            my_flags |= kTail;
#pragma unroll
            for (int i = 0; i < E; ++i) parts[1][threadIdx.x][i] = sum[i];
        } else if (id != none && mine) {
            write_sum<TT, E>(a, id, c, own, sum);
        }
    }
    flags[group] = my_flags;  // (all lanes of the group the same)
    __syncthreads();
    // sums that cross runs: the run where one begins adds up the rest, as far as the workgroup goes
    if (my_flags & kTail) {
        double total[E];
#pragma unroll
        for (int i = 0; i < E; ++i) total[i] = double(sum[i]);
        int g = group + 1;
        for (; g < groups; ++g) {
#pragma unroll
            for (int i = 0; i < E; ++i) total[i] += double(parts[0][(g << a.lanes_log2) + lane][i]);
            if (!(flags[g] & kThrough)) break;
        }
        float x[E];
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = float(total[i]);
        if (g < groups) {
            if (mine) write_sum<TT, E>(a, id, c, own, x);
        } else {
            if (mine) store_vector<float, E, false>(a.tail + block * a.f + c, x);
        }
    }
    // what began before this workgroup
    if (group == 0 && (my_flags & kHead)) {
        double total[E] = {};
        int g = 0;
        for (; g < groups; ++g) {
#pragma unroll
            for (int i = 0; i < E; ++i) total[i] += double(parts[0][(g << a.lanes_log2) + lane][i]);
            if (!(flags[g] & kThrough)) break;
        }
        float x[E];
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = float(total[i]);
        if (mine) store_vector<float, E, false>(a.head + block * a.f + c, x);
    }
    if (threadIdx.x == 0 && blockIdx.y == 0) {
        uint32_t all = flags[0] & kHead;
        int g = groups - 1;
        while (g >= 0 && (flags[g] & kThrough)) --g;
        if (g < 0) all |= kThrough;
        else if (flags[g] & kTail) all |= kTail;
        a.flags[block] = all;
    }
}

// The sums that cross workgroups: workgroup b joins the one that begins in runs of workgroup b.
template <typename TT, int E> __global__ void __launch_bounds__(kThreads) join_kernel(const Grad a) {
    const int64_t block = block_number();
    if (block >= a.sum_blocks || !(a.flags[block] & kTail)) return;
    __shared__ double parts[kThreads][E];
    __shared__ int last;
    const int lanes = 1 << a.lanes_log2, lane = int(threadIdx.x) & (lanes - 1), group = int(threadIdx.x) >> a.lanes_log2, groups = kThreads >> a.lanes_log2;
    const int64_t chunk = int64_t(groups) * a.run;
    // how many workgroups behind it have parts: up to the first that has more than the middle
    int64_t more = 1;
    if (a.flags[block + 1] & kThrough) {
        for (;; more += kThreads) {
            if (threadIdx.x == 0) last = kThreads;
            __syncthreads();
            const int64_t b = block + 1 + more + threadIdx.x;
            if (b >= a.sum_blocks || !(a.flags[b] & kThrough)) atomicMin(&last, int(threadIdx.x));
            __syncthreads();
            const int found = last;
            __syncthreads();
            if (found < kThreads) {
                more += found + 1;
                break;
            }
        }
    }
    const int q = int(blockIdx.y) * lanes + lane;
    const bool mine = q < a.vectors;
    const int c = !mine ? 0 : q * E < a.f - E ? q * E : a.f - E;
    const int own = q * E < a.f - E ? E : a.f - q * E;
    double total[E] = {};
    if (mine) {
        constexpr int U = 4;  // on their way at once
        for (int64_t k = group; k < more; k += U * groups) {
            Vector<float, E> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u].load(a.head + (block + 1 + (k + u * groups < more ? k + u * groups : k)) * a.f + c);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (k + u * groups >= more) break;
                float x[E];
                v[u].get(x);
#pragma unroll
                for (int i = 0; i < E; ++i) total[i] += double(x[i]);
            }
        }
    }
    if (more > 1) {
#pragma unroll
        for (int i = 0; i < E; ++i) parts[threadIdx.x][i] = total[i];
        __syncthreads();
    }
    if (group > 0 || !mine) return;
    if (more > 1) {
        const int64_t have = more < groups ? more : groups;
        for (int g = 1; g < have; ++g)
#pragma unroll
            for (int i = 0; i < E; ++i) total[i] += parts[(g << a.lanes_log2) + lane][i];
    }
    Vector<float, E> v;
    v.load(a.tail + block * a.f + c);
    float x[E];
    v.get(x);
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = float(total[i] + double(x[i]));
    // (the last position of a workgroup with others behind it is there)
    write_sum<TT, E>(a, a.key[(block + 1) * chunk - 1], c, own, x);
}

dim3 grid_of(int64_t blocks, int64_t slices = 1) {
    return blocks <= kGridX ? dim3(unsigned(blocks), unsigned(slices)) : dim3(kGridX, unsigned(slices), unsigned((blocks + kGridX - 1) / kGridX));
}

bool known(int32_t dtype) { return dtype == GNN_F32 || dtype == GNN_BF16; }
int64_t size_of(int32_t dtype) { return dtype == GNN_F32 ? 4 : 2; }
bool misaligned(const void *p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % uintptr_t(to) != 0; }

// Elements of a vector: 16 bytes of Y or dY; one of rows narrower than that.
int elements_of(bool eight, int64_t f) { return f >= (eight ? 8 : 4) ? (eight ? 8 : 4) : 1; }

struct Room {  // of the gradient, in words
    int lanes_log2, run;
    int64_t vectors, chunk, blocks, table, sums, padded, words;
};
Room room_of(int64_t V, int64_t n, int64_t F, bool eight) {
    Room r;
    const int e = elements_of(eight, F);
    r.vectors = (F + e - 1) / e;
    r.lanes_log2 = r.vectors > kMostSlices * 64 ? 7 : r.vectors >= 64 ? 6 : gnn_ilog2_ceil(r.vectors);
    r.run = n >= kLong ? kRun : kBatch;
    r.chunk = int64_t(kThreads >> r.lanes_log2) * r.run;
    r.blocks = (n + r.chunk - 1) / r.chunk;
    r.table = gnn_sort_table_elems(n);
    r.sums = gnn_sort_sums_elems(n);
    r.padded = (n + kBatch - 1) / kBatch * kBatch;
    r.words = 4 * r.padded + r.table + r.sums + r.blocks * (2 * F + 1);
    return r;
}

int check(const void *table, const void *ids, const void *y, int64_t V, int64_t n, int64_t F, const gnn_lookup_opts &o) {
    if (V < 0 || n < 0 || F < 0 || V > kMostRows || n > kMostRows || F > kMostColumns || !known(o.table_dtype) || !known(o.dtype)) return GNN_ERR_INVALID_ARG;
    if ((o.ids_is_64 & ~1) || (o.accumulate & ~1) || (o.ldt && o.ldt < F) || (o.ldy && o.ldy < F)) return GNN_ERR_INVALID_ARG;
    if (F == 0) return GNN_OK;
    if ((V > 0 && !table) || (n > 0 && (!ids || !y)) || (V > 0 && n > 0 && table == y)) return GNN_ERR_INVALID_ARG;
    if (misaligned(table, size_of(o.table_dtype)) || misaligned(y, size_of(o.dtype)) || misaligned(ids, o.ids_is_64 ? 8 : 4)) return GNN_ERR_INVALID_ARG;
    return GNN_OK;
}

template <typename TT, typename TY, int E> void launch_lookup(const Lookup &a, hipStream_t stream) {
    lookup_kernel<TT, TY, E><<<grid_of((a.n + a.rows - 1) / a.rows), kThreads, 0, stream>>>(a);
}
template <typename TT, typename TY> void lookup(Lookup &a, hipStream_t stream) {
    // 16 bytes of Y a thread, so that a wavefront's stores are whole lines (1.2 M rows x 256 bf16 into fp32 362 -> 305 us)
    constexpr bool eight = sizeof(TY) == 2;
    const int e = elements_of(eight, a.f);
    a.vectors = (a.f + e - 1) / e;
    a.rows = a.vectors >= kThreads * kAtOnce ? 1 : kThreads * kAtOnce / a.vectors;
    a.reciprocal = a.vectors > 1 ? uint32_t(((uint64_t(1) << 32) + uint64_t(a.vectors) - 1) / uint64_t(a.vectors)) : 0;
    if (e == 1) launch_lookup<TT, TY, 1>(a, stream);
    else launch_lookup<TT, TY, eight ? 8 : 4>(a, stream);
}

template <typename TY, typename TT, int E> int launch_grad(const Grad &a, int64_t slices, hipStream_t stream) {
    if (a.sum_blocks + a.zero_blocks == 0) return GNN_OK;
    const dim3 grid = grid_of(a.sum_blocks + a.zero_blocks, slices);
    if (E > 1 && a.whole_lines) grad_kernel<TY, TT, E, (E > 1)><<<grid, kThreads, 0, stream>>>(a);
    else grad_kernel<TY, TT, E, false><<<grid, kThreads, 0, stream>>>(a);
    GNN_HIP_TRY(hipGetLastError());
    if (a.sum_blocks > 1) {
        join_kernel<TT, E><<<grid_of(a.sum_blocks, slices), kThreads, 0, stream>>>(a);
        GNN_HIP_TRY(hipGetLastError());
    }
    return GNN_OK;
}
template <typename TY, typename TT, int E> int launch_few(Grad a, const Ids &ids, hipStream_t stream) {
    // groups of few lanes, so that a workgroup has many: 1,021 and 2,048 positions of one id x 602 52 and 184 us with 64 lanes, 21 and 60 so
    if (a.lanes_log2 > kFewLanesLog2 && a.vectors <= kMostSlices) a.lanes_log2 = kFewLanesLog2;
    const int64_t slices = (a.vectors + (int64_t(1) << a.lanes_log2) - 1) >> a.lanes_log2;
    // rows of a workgroup that zeroes: about 64 KB of fp32, several times the ids that it reads (4,096 x 602 of 1,021 positions in 16 workgroups 24 us, in 256 7.2)
    int wide = kZeroWide;
    while (wide > 16 && int64_t(wide) * a.f > 16384) wide /= 2;
    a.sum_blocks = (a.n + kFewRows - 1) / kFewRows;
    a.zero_blocks = a.accumulate ? 0 : (a.rows + wide - 1) / wide;
    few_grad_kernel<TY, TT, E><<<grid_of(a.sum_blocks + a.zero_blocks, slices), kThreads, 0, stream>>>(a, ids, wide);
    GNN_HIP_TRY(hipGetLastError());
    return GNN_OK;
}
template <typename TY, typename TT> int few(const Grad &a, const Ids &ids, hipStream_t stream) {
    constexpr int E = gnn_rows<TY>::VEC;
    return a.f < E ? launch_few<TY, TT, 1>(a, ids, stream) : launch_few<TY, TT, E>(a, ids, stream);
}
template <typename TY, typename TT> int grad(const Grad &a, int64_t slices, hipStream_t stream) {
    constexpr int E = gnn_rows<TY>::VEC;
    return a.f < E ? launch_grad<TY, TT, 1>(a, slices, stream) : launch_grad<TY, TT, E>(a, slices, stream);
}

}  // namespace

extern "C" GNN_API int gnn_lookup_fwd(const void *table, const void *ids, void *Y, int64_t V, int64_t n, int64_t F, const gnn_lookup_opts *opts) {
    if (!opts) return GNN_ERR_INVALID_ARG;
    const gnn_lookup_opts &o = *opts;
    const int rc = check(table, ids, Y, V, n, F, o);
    if (rc != GNN_OK || n == 0 || F == 0) return rc;
    (void)hipGetLastError();
    Lookup a{};
    a.table = table;
    a.y = Y;
    a.ids = {ids, o.ids_is_64, V};
    a.n = n;
    a.ldt = o.ldt ? o.ldt : F;
    a.ldy = o.ldy ? o.ldy : F;
    a.f = int32_t(F);
    a.scale = o.scale;
    hipStream_t stream = static_cast<hipStream_t>(o.stream);
    if (o.table_dtype == GNN_F32) o.dtype == GNN_F32 ? lookup<float, float>(a, stream) : lookup<float, gnn_bf16>(a, stream);
    else o.dtype == GNN_F32 ? lookup<gnn_bf16, float>(a, stream) : lookup<gnn_bf16, gnn_bf16>(a, stream);
    GNN_HIP_TRY(hipGetLastError());
    return GNN_OK;
}

extern "C" GNN_API int64_t gnn_lookup_workspace_bytes(int64_t V, int64_t n, int64_t F) {
    if (V <= 0 || n <= 0 || F <= 0 || V > kMostRows || n > kMostRows || F > kMostColumns) return 0;
    // Enough for every smaller call as well: a call's room falls only where its runs become long, at kLong positions, and where its vectors become wide, at 4 and 8 columns.
    int64_t words = 0;
    for (const bool eight : {false, true})
        for (const int64_t positions : {n, n < kLong ? n : kLong - 1}) {
            const int64_t wide = eight ? 8 : 4;
            for (const int64_t columns : {F, F < wide ? F : wide - 1}) {
                const int64_t w = room_of(V, positions, columns, eight).words;
                words = w > words ? w : words;
            }
        }
    return 4 * words;
}

extern "C" GNN_API int gnn_lookup_bwd(const void *ids, const void *dY, void *dtable, int64_t V, int64_t n, int64_t F, const gnn_lookup_opts *opts) {
    if (!opts) return GNN_ERR_INVALID_ARG;
    const gnn_lookup_opts &o = *opts;
    const int rc = check(dtable, ids, dY, V, n, F, o);
    if (rc != GNN_OK || V == 0 || F == 0 || (n == 0 && o.accumulate)) return rc;
    const bool eight = o.dtype == GNN_BF16;
    const Room r = room_of(V, n, F, eight);
    if (n > 0 && (!o.workspace || misaligned(o.workspace, 16) || o.workspace_bytes < 4 * r.words)) return GNN_ERR_INVALID_ARG;
    (void)hipGetLastError();
    hipStream_t stream = static_cast<hipStream_t>(o.stream);
    Grad a{};
    a.dy = dY;
    a.dtable = dtable;
    a.rows = V;
    a.n = n;
    a.ldt = o.ldt ? o.ldt : F;
    a.ldy = o.ldy ? o.ldy : F;
    a.f = int32_t(F);
    a.vectors = int32_t(r.vectors);
    a.reciprocal = r.vectors > 1 ? uint32_t(((uint64_t(1) << 32) + uint64_t(r.vectors) - 1) / uint64_t(r.vectors)) : 0;
    a.lanes_log2 = r.lanes_log2;
    a.run = r.run;
    a.accumulate = o.accumulate;
    // past the caches where no two rows share a line and they would not fit (2.4 M x 256 bf16 of 47 ids 298 -> 267 us; 1.2 M x 100 fp32, which share
    // lines, 462 -> 479, and 200 K x 128 fp32, 100 MB, 95 -> 116)
    a.whole_lines = F * size_of(o.dtype) % 128 == 0 && a.ldy * size_of(o.dtype) % 128 == 0 && !misaligned(dY, 128) && n * F * size_of(o.dtype) > kCaches;
    a.scale = o.scale;
    a.sum_blocks = r.blocks;
    // small tables: less rows a workgroup, so that there are 1,024 of them (4,096 x 602 of 5,000 positions 56 us with 256 rows, 41 with 16)
    a.zero_rows = kZeroRows;
    while (a.zero_rows > 16 && V < int64_t(a.zero_rows) * 1024) a.zero_rows /= 2;
    a.zero_blocks = o.accumulate ? 0 : (V + a.zero_rows - 1) / a.zero_rows;
    const Ids named{ids, o.ids_is_64, V};
    if (n > 0 && n <= kFew && n <= 8 * V) {
        if (o.dtype == GNN_F32) return o.table_dtype == GNN_F32 ? few<float, float>(a, named, stream) : few<float, gnn_bf16>(a, named, stream);
        return o.table_dtype == GNN_F32 ? few<gnn_bf16, float>(a, named, stream) : few<gnn_bf16, gnn_bf16>(a, named, stream);
    }
    if (n > 0) {
        uint32_t *next = static_cast<uint32_t *>(o.workspace);
        uint32_t *buf_k[2] = {next, next + r.padded}, *buf_v[2] = {next + 2 * r.padded, next + 3 * r.padded};
        next += 4 * r.padded;
        a.head = reinterpret_cast<float *>(next);
        next += r.blocks * F;
        a.tail = reinterpret_cast<float *>(next);
        next += r.blocks * F;
        a.flags = next;
        next += r.blocks;
        if (n <= kRankHere) {
            rank_kernel<<<unsigned((n + kRankRows - 1) / kRankRows), kThreads, 0, stream>>>(named, int(n), buf_k[0], buf_v[0]);
            GNN_HIP_TRY(hipGetLastError());
            a.key = buf_k[0];
            a.order = buf_v[0];
        } else {
            uint32_t *keys = nullptr, *order = nullptr;
            const int sorted = gnn_radix_sort_positions({ids, o.ids_is_64, V}, buf_k, buf_v, n, gnn_ilog2_ceil(V + 1), next, next + r.table, stream, &keys, &order);
            if (sorted != GNN_OK) return sorted;
            a.key = keys;
            a.order = order;
        }
    }
    const int64_t slices = (r.vectors + (int64_t(1) << r.lanes_log2) - 1) >> r.lanes_log2;
    if (o.dtype == GNN_F32) return o.table_dtype == GNN_F32 ? grad<float, float>(a, slices, stream) : grad<float, gnn_bf16>(a, slices, stream);
    return o.table_dtype == GNN_F32 ? grad<gnn_bf16, float>(a, slices, stream) : grad<gnn_bf16, gnn_bf16>(a, slices, stream);
}
