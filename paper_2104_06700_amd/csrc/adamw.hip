// One AdamW step over many tensors.
//
// Per element, with gradient g (times *grad_scale), step number t, decoupled weight decay wd:
//     m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2,
//     p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps).
//
// States are fp32, or 8 bits: e4m3 numbers (4 exponent bits, 3 mantissa bits, largest number 448) times an fp32 scale for every
// 256 neighbouring elements, scale = largest finite magnitude of the 256 / 448.  The step computes with the fp32 values of m and v; rounding
// to 8 bits is what the next step reads.  m is rounded to the nearest number (half a step is at most 1/16 of the value, less than a step of
// b1 = 0.9 takes off).  v is rounded up or down at random, with the probability that keeps its mean: with b2 = 0.999 one step moves
// v by far less than half a step of the code, so that to the nearest it would stand still beside the largest of its 256 (3000 steps over
// values of a wide spread with rare large gradients: sqrt(v) off by 0.39 rms and 17 % on average to the nearest, by 0.11 and 1 % at
// random).  The random bits are a hash of seed, step, tensor and element.  v > 0 is never held as 0, which would divide m by eps.
//
// The tensors' descriptors are kernel arguments: no copy of them, no allocation, at most kTensors per launch.  A workgroup has
// kChunk neighbouring elements of one tensor and ends with them; its loads are all issued before the first is waited for.  A
// scale's 256 elements are 64 lanes of four (fp32) or 32 of eight (bf16), whose maximum is formed by lane permutations.
//
// Bound by the memory: 245 M fp32 elements 1162 us with fp32 states (28 bytes an element, 5.9 TB/s), 677 with 8-bit states (16 bytes, 5.8); 140 M in bf16
// with a master copy and 8-bit states 431 (16 bytes, 5.2).  Workgroups that stay and walk reach 4.3 to 4.9 TB/s.  The 103 K elements of a model of
// eight tensors 3.8 us in chunks of 2,048.
#include "common.h"
#include "rows.h"

#include <math.h>

#pragma clang fp contract(off)  // the states' rounding to 8 bits is defined on products and sums that are rounded one by one

namespace {

constexpr int kThreads = 256;
constexpr int kBlock = 256;      // elements of a scale: four a lane
constexpr int kChunk = 4096, kShortChunk = 2048;  // elements of a workgroup
constexpr int kTensors = 40;     // of a launch; 4 KB of arguments at most
constexpr int64_t kShort = 4 << 20;  // elements below which chunks are short
constexpr float kTop = 448.0f;
constexpr float kTiny = 0x1p-118f;  // below it 448 / x would overflow: such a block is held as zeros

struct Tensor {
    void *param;
    const void *grad;
    void *m, *v;
    float *m_scale, *v_scale, *master;
    int64_t n;
    uint32_t salt;    // of the random bits
    float decay;      // 1 - lr wd
    int32_t first;    // workgroup that begins it
    int32_t flags;    // 1: bf16, 2: 8-bit states, 4: a master copy
};
struct Step {
    Tensor t[kTensors];
    int32_t first[kTensors];  // t[].first side by side
    int32_t count, chunk;
    float b1, c1, b2, c2, rate, root, eps;  // c = 1 - b, rate = lr / (1 - b1^t), root = 1 / sqrt(1 - b2^t)
    const float *grad_scale;
};
static_assert(sizeof(Step) <= 4096, "kernel arguments");

__device__ __forceinline__ uint32_t random_bits(uint64_t element, uint32_t salt) {  // 20 of them
    uint32_t h = uint32_t(element) * 0x9E3779B9u + uint32_t(element >> 32) * 0x6A09E667u + salt;
    h = (h ^ (h >> 16)) * 0x6A09E667u;
    h = (h ^ (h >> 15)) * 0xBB67AE85u;
    return h >> 12;
}

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// four numbers to the nearest; not finite ones become NaN (odd: there may be some)
__device__ __forceinline__ uint32_t code_nearest(const float (&x)[4], float factor, bool odd) {
    int w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * factor, x[1] * factor, w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] * factor, x[3] * factor, w, true);
    if (odd)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (!finite(x[j])) w |= 0x7F << (8 * j);
    return uint32_t(w);
}

// four numbers x >= 0, up or down by their random bits.  From 2^-6 on, the 20 bits are added to the 20 of the mantissa that go;
// below, numbers are multiples of 2^-9.
__device__ __forceinline__ uint32_t code_random(const float (&v)[4], float factor, uint64_t element, uint32_t salt, bool odd) {
    uint32_t w = 0;
    const uint32_t least = factor > 0.0f ? 1 : 0;  // for what is above 0
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float x = fminf(v[j] * factor, kTop);
        const uint32_t bits = random_bits(element + j, salt);
        uint32_t c = x >= 0x1p-6f ? ((__float_as_uint(x) + bits) >> 20) - (120u << 3) : uint32_t(x * 512.0f + float(bits) * 0x1p-20f);
        const uint32_t low = v[j] > 0.0f ? least : 0;
        c = c > low ? c : low;
        w |= c << (8 * j);
    }
    if (odd)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (!finite(v[j])) w = (w & ~(0xFFu << (8 * j))) | (0x7Fu << (8 * j));
    return w;
}

typedef uint32_t u32_any __attribute__((aligned(1)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t u32x2_half __attribute__((ext_vector_type(2), aligned(2)));

// four neighbouring elements
__device__ __forceinline__ void load4(const float *p, float (&v)[4]) { gnn_rows<float>::unpack(gnn_rows<float>::fetch(p), v); }
__device__ __forceinline__ void load4(const gnn_bf16 *p, float (&v)[4]) {
    const u32x2_half t = *reinterpret_cast<const u32x2_half *>(p);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        v[2 * i] = __uint_as_float(t[i] << 16);
        v[2 * i + 1] = __uint_as_float(t[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void store4(float *p, const float (&v)[4]) { gnn_rows<float>::put(p, gnn_rows<float>::pack(v)); }
__device__ __forceinline__ void store4(gnn_bf16 *p, const float (&v)[4]) {
    u32x2_half t;
#pragma unroll
    for (int i = 0; i < 2; ++i) t[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(gnn_f32x2{v[2 * i], v[2 * i + 1]}, gnn_bf16x2));
    *reinterpret_cast<u32x2_half *>(p) = t;
}

// Any four elements, or as many as the tensor has left.
template <typename T, bool EIGHT>
__device__ __forceinline__ void update(const Step &s, const Tensor &t, int64_t i, float gs) {
    // elements i .. i + 3 of the tensor, or as many of them as there are
    const int64_t left = t.n - i;
    const int have = left < 0 ? 0 : left < 4 ? int(left) : 4;
    const T *param = static_cast<const T *>(t.param);
    const T *grad = static_cast<const T *>(t.grad);
    float p[4], g[4], m[4], v[4];
    uint32_t mc = 0, vc = 0;
    const uint8_t *m8 = static_cast<const uint8_t *>(t.m), *v8 = static_cast<const uint8_t *>(t.v);
    const float *m32 = static_cast<const float *>(t.m), *v32 = static_cast<const float *>(t.v);
    if (have == 4) {
        load4(grad + i, g);
        if (t.master) load4(t.master + i, p);
        else load4(param + i, p);
        if constexpr (EIGHT) {
            mc = *reinterpret_cast<const u32_any *>(m8 + i);
            vc = *reinterpret_cast<const u32_any *>(v8 + i);
        } else {
            load4(m32 + i, m);
            load4(v32 + i, v);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            p[j] = g[j] = m[j] = v[j] = 0.0f;
            if (j >= have) continue;
            p[j] = t.master ? t.master[i + j] : gnn_rows<T>::get(param + i + j);
            g[j] = gnn_rows<T>::get(grad + i + j);
            if constexpr (EIGHT) {
                mc |= uint32_t(m8[i + j]) << (8 * j);
                vc |= uint32_t(v8[i + j]) << (8 * j);
            } else {
                m[j] = m32[i + j];
                v[j] = v32[i + j];
            }
        }
    }
    if constexpr (EIGHT) {
        const int64_t block = i / kBlock;
        const float ms = have ? t.m_scale[block] : 0.0f, vs = have ? t.v_scale[block] : 0.0f;
        m[0] = __builtin_amdgcn_cvt_f32_fp8(int(mc), 0) * ms;
        m[1] = __builtin_amdgcn_cvt_f32_fp8(int(mc), 1) * ms;
        m[2] = __builtin_amdgcn_cvt_f32_fp8(int(mc), 2) * ms;
        m[3] = __builtin_amdgcn_cvt_f32_fp8(int(mc), 3) * ms;
        v[0] = __builtin_amdgcn_cvt_f32_fp8(int(vc), 0) * vs;
        v[1] = __builtin_amdgcn_cvt_f32_fp8(int(vc), 1) * vs;
        v[2] = __builtin_amdgcn_cvt_f32_fp8(int(vc), 2) * vs;
        v[3] = __builtin_amdgcn_cvt_f32_fp8(int(vc), 3) * vs;
    }
    float m_top = 0.0f, v_top = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float gj = g[j] * gs;
        m[j] = m[j] * s.b1 + gj * s.c1;
        v[j] = v[j] * s.b2 + (gj * gj) * s.c2;
        p[j] = p[j] * t.decay - s.rate * (m[j] / (sqrtf(v[j]) * s.root + s.eps));
        if (finite(m[j])) m_top = fmaxf(m_top, fabsf(m[j]));
        if (finite(v[j])) v_top = fmaxf(v_top, v[j]);
    }
    if constexpr (EIGHT) {
        m_top = wave_max(m_top);
        v_top = wave_max(v_top);
        const float mf = m_top >= kTiny ? kTop / m_top : 0.0f, vf = v_top >= kTiny ? kTop / v_top : 0.0f;
        mc = code_nearest(m, mf, true);
        vc = code_random(v, vf, uint64_t(i), t.salt, true);
        if ((threadIdx.x & 63) == 0 && have) {
            t.m_scale[i / kBlock] = m_top >= kTiny ? m_top / kTop : 0.0f;
            t.v_scale[i / kBlock] = v_top >= kTiny ? v_top / kTop : 0.0f;
        }
    }
    if (have == 4) {
        store4(static_cast<T *>(t.param) + i, p);
        if (t.master) store4(t.master + i, p);
        if constexpr (EIGHT) {
            *reinterpret_cast<u32_any *>(static_cast<uint8_t *>(t.m) + i) = mc;
            *reinterpret_cast<u32_any *>(static_cast<uint8_t *>(t.v) + i) = vc;
        } else {
            store4(static_cast<float *>(t.m) + i, m);
            store4(static_cast<float *>(t.v) + i, v);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (j >= have) continue;
        gnn_rows<T>::set(static_cast<T *>(t.param) + i + j, p[j]);
        if (t.master) t.master[i + j] = p[j];
        if constexpr (EIGHT) {
            static_cast<uint8_t *>(t.m)[i + j] = uint8_t(mc >> (8 * j));
            static_cast<uint8_t *>(t.v)[i + j] = uint8_t(vc >> (8 * j));
        } else {
            static_cast<float *>(t.m)[i + j] = m[j];
            static_cast<float *>(t.v)[i + j] = v[j];
        }
    }
}

// ---- whole chunks

// the largest of 64 lanes' values (0 is the least); with HALF of lanes 0 - 31 and of 32 - 63
template <bool HALF> __device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
#define GNN_DPP_MAX(ctrl, rows)                                                                                    \
    {                                                                                                             \
        const uint32_t o = uint32_t(__builtin_amdgcn_update_dpp(0, int(v), ctrl, rows, 0xf, false));               \
        v = o > v ? o : v;                                                                                        \
    }
    GNN_DPP_MAX(0x111, 0xf)  // row_shr:1, 2, 4, 8: the last of 16 lanes has their largest
    GNN_DPP_MAX(0x112, 0xf)
    GNN_DPP_MAX(0x114, 0xf)
    GNN_DPP_MAX(0x118, 0xf)
    GNN_DPP_MAX(0x142, 0xa)  // row_bcast:15 into rows 1 and 3
    if constexpr (HALF) {
        const uint32_t lo = uint32_t(__builtin_amdgcn_readlane(int(v), 31)), hi = uint32_t(__builtin_amdgcn_readlane(int(v), 63));
        return (threadIdx.x & 32) ? hi : lo;
    } else {
        GNN_DPP_MAX(0x143, 0xc)  // row_bcast:31 into rows 2 and 3
        return uint32_t(__builtin_amdgcn_readlane(int(v), 63));
    }
#undef GNN_DPP_MAX
}

// E neighbouring fp32 values
template <int E> struct Floats {
    gnn_f32x4 v[E / 4];
    __device__ __forceinline__ void load(const float *p) {
#pragma unroll
        for (int k = 0; k < E / 4; ++k) v[k] = __builtin_nontemporal_load(reinterpret_cast<const gnn_f32x4 *>(p) + k);
    }
    __device__ __forceinline__ float get(int j) const { return v[j / 4][j % 4]; }
    __device__ __forceinline__ void set(int j, float x) { v[j / 4][j % 4] = x; }
    __device__ __forceinline__ void store(float *p) const {
#pragma unroll
        for (int k = 0; k < E / 4; ++k) __builtin_nontemporal_store(v[k], reinterpret_cast<gnn_f32x4 *>(p) + k);
    }
};
// E neighbouring bytes
template <int E> struct Codes {
    uint32_t w[E / 4];
    __device__ __forceinline__ void load(const void *at) {
        const uint8_t *p = static_cast<const uint8_t *>(at);
        if constexpr (E == 4) w[0] = __builtin_nontemporal_load(reinterpret_cast<const u32_any *>(p));
        else {
            const u32x2_any t = __builtin_nontemporal_load(reinterpret_cast<const u32x2_any *>(p));
            w[0] = t.x;
            w[1] = t.y;
        }
    }
    __device__ __forceinline__ void store(void *at) const {
        uint8_t *p = static_cast<uint8_t *>(at);
        if constexpr (E == 4) __builtin_nontemporal_store(w[0], reinterpret_cast<u32_any *>(p));
        else __builtin_nontemporal_store(u32x2_any{w[0], w[1]}, reinterpret_cast<u32x2_any *>(p));
    }
};
__device__ __forceinline__ void decode(uint32_t w, float scale, float (&x)[4]) {
    x[0] = __builtin_amdgcn_cvt_f32_fp8(int(w), 0) * scale;
    x[1] = __builtin_amdgcn_cvt_f32_fp8(int(w), 1) * scale;
    x[2] = __builtin_amdgcn_cvt_f32_fp8(int(w), 2) * scale;
    x[3] = __builtin_amdgcn_cvt_f32_fp8(int(w), 3) * scale;
}

// CHUNK elements from `begin` on, all inside the tensor.
template <int CHUNK, typename T, bool EIGHT, bool MASTER> __device__ __forceinline__ void update_chunk(const Step &s, const Tensor &t, int64_t begin, float gs) {
    constexpr int E = gnn_rows<T>::VEC, U = CHUNK / (kThreads * E);
    typedef typename gnn_rows<T>::raw raw;
    raw p[MASTER ? 1 : U], g[U];
    Floats<E> master[MASTER ? U : 1], m32[EIGHT ? 1 : U], v32[EIGHT ? 1 : U];
    Codes<E> m8[EIGHT ? U : 1], v8[EIGHT ? U : 1];
    float ms[U], vs[U];
    const int64_t i0 = begin + int64_t(threadIdx.x) * E;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = i0 + u * (kThreads * E);
        g[u] = __builtin_nontemporal_load(reinterpret_cast<const raw *>(static_cast<const T *>(t.grad) + i));
        if constexpr (MASTER) master[u].load(t.master + i);
        else p[u] = __builtin_nontemporal_load(reinterpret_cast<const raw *>(static_cast<const T *>(t.param) + i));
        if constexpr (EIGHT) {
            m8[u].load(static_cast<const uint8_t *>(t.m) + i);
            v8[u].load(static_cast<const uint8_t *>(t.v) + i);
            ms[u] = t.m_scale[i / kBlock];
            vs[u] = t.v_scale[i / kBlock];
        } else {
            m32[u].load(static_cast<const float *>(t.m) + i);
            v32[u].load(static_cast<const float *>(t.v) + i);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = i0 + u * (kThreads * E);
        float gf[E], pf[E], m[E], v[E];
        gnn_rows<T>::unpack(g[u], gf);
        if constexpr (!MASTER) gnn_rows<T>::unpack(p[u], pf);
        uint32_t m_top = 0, v_top = 0;
#pragma unroll
        for (int q = 0; q < E / 4; ++q) {
            float mo[4], vo[4];
            if constexpr (EIGHT) {
                decode(m8[u].w[q], ms[u], mo);
                decode(v8[u].w[q], vs[u], vo);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int j = 4 * q + r;
                if constexpr (!EIGHT) {
                    mo[r] = m32[u].get(j);
                    vo[r] = v32[u].get(j);
                }
                const float po = MASTER ? master[u].get(j) : pf[j];
                const float x = gf[j] * gs;
                m[j] = mo[r] * s.b1 + x * s.c1;
                v[j] = vo[r] * s.b2 + (x * x) * s.c2;
                // (both instructions are good to a unit in the last place, but for roots below 2^-63, which eps covers)
                pf[j] = po * t.decay - s.rate * (m[j] * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v[j]) * s.root + s.eps));
                if constexpr (EIGHT) {
                    const uint32_t mb = __float_as_uint(m[j]) & 0x7FFFFFFFu, vb = __float_as_uint(v[j]) & 0x7FFFFFFFu;
                    m_top = mb > m_top ? mb : m_top;
                    v_top = vb > v_top ? vb : v_top;
                }
            }
        }
        if constexpr (MASTER) {
#pragma unroll
            for (int j = 0; j < E; ++j) master[u].set(j, pf[j]);
            master[u].store(t.master + i);
        }
        __builtin_nontemporal_store(gnn_rows<T>::pack(pf), reinterpret_cast<raw *>(static_cast<T *>(t.param) + i));
        if constexpr (EIGHT) {
            m_top = lanes_max<E == 8>(m_top);
            v_top = lanes_max<E == 8>(v_top);
            const bool odd = m_top >= 0x7F800000u || v_top >= 0x7F800000u;  // something is not finite: the largest of the others counts
            if (odd) {
                m_top = v_top = 0;
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    const uint32_t mb = __float_as_uint(m[j]) & 0x7FFFFFFFu, vb = __float_as_uint(v[j]) & 0x7FFFFFFFu;
                    if (mb < 0x7F800000u && mb > m_top) m_top = mb;
                    if (vb < 0x7F800000u && vb > v_top) v_top = vb;
                }
            }
            if (__ballot(odd)) {  // (all lanes take part in the permutations; the others' values are what they have)
                const uint32_t mt = lanes_max<E == 8>(m_top), vt = lanes_max<E == 8>(v_top);
                m_top = mt;
                v_top = vt;
            }
            const float mt = __uint_as_float(m_top), vt = __uint_as_float(v_top);
            const float mf = mt >= kTiny ? kTop / mt : 0.0f, vf = vt >= kTiny ? kTop / vt : 0.0f;
#pragma unroll
            for (int q = 0; q < E / 4; ++q) {
                const float mq[4] = {m[4 * q], m[4 * q + 1], m[4 * q + 2], m[4 * q + 3]}, vq[4] = {v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
                m8[u].w[q] = code_nearest(mq, mf, odd);
                v8[u].w[q] = code_random(vq, vf, uint64_t(i + 4 * q), t.salt, odd);
            }
            m8[u].store(static_cast<uint8_t *>(t.m) + i);
            v8[u].store(static_cast<uint8_t *>(t.v) + i);
            if ((threadIdx.x & (kBlock / E - 1)) == 0) {
                t.m_scale[i / kBlock] = mt >= kTiny ? mt / kTop : 0.0f;
                t.v_scale[i / kBlock] = vt >= kTiny ? vt / kTop : 0.0f;
            }
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                m32[u].set(j, m[j]);
                v32[u].set(j, v[j]);
            }
            m32[u].store(static_cast<float *>(t.m) + i);
            v32[u].store(static_cast<float *>(t.v) + i);
        }
    }
}

template <typename T, bool EIGHT> __device__ __forceinline__ void update_rest(const Step &s, const Tensor &t, int64_t begin, float gs) {
    for (int k = 0; k < s.chunk && begin + k < t.n; k += kThreads * 4) update<T, EIGHT>(s, t, begin + k + int64_t(threadIdx.x) * 4, gs);
}

template <int CHUNK> __global__ void __launch_bounds__(kThreads) adamw_kernel(const Step s) {
    // the last tensor that begins at this workgroup or before
    const int lane = int(threadIdx.x & 63);
    const bool before = lane < s.count && s.first[lane < kTensors ? lane : 0] <= int(blockIdx.x);
    const int k = __popcll(__ballot(before)) - 1;
    const Tensor &t = s.t[k];
    const int64_t begin = int64_t(int(blockIdx.x) - t.first) * CHUNK;
    const float gs = s.grad_scale ? *s.grad_scale : 1.0f;
    // the last elements, and an eps so small that quotients near the ends of the range matter: one by one
    if (begin + CHUNK > t.n || s.eps < 0x1p-40f) {
        if ((t.flags & 3) == 0) update_rest<float, false>(s, t, begin, gs);
        else if ((t.flags & 3) == 1) update_rest<gnn_bf16, false>(s, t, begin, gs);
        else if ((t.flags & 3) == 2) update_rest<float, true>(s, t, begin, gs);
        else update_rest<gnn_bf16, true>(s, t, begin, gs);
        return;
    }
    switch (t.flags) {
        case 0: update_chunk<CHUNK, float, false, false>(s, t, begin, gs); break;
        case 1: update_chunk<CHUNK, gnn_bf16, false, false>(s, t, begin, gs); break;
        case 2: update_chunk<CHUNK, float, true, false>(s, t, begin, gs); break;
        case 3: update_chunk<CHUNK, gnn_bf16, true, false>(s, t, begin, gs); break;
        case 5: update_chunk<CHUNK, gnn_bf16, false, true>(s, t, begin, gs); break;
        default: update_chunk<CHUNK, gnn_bf16, true, true>(s, t, begin, gs); break;
    }
}

bool misaligned(const void *p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % uintptr_t(to) != 0; }

int check_tensor(const gnn_adamw_tensor &t) {
    if (t.n < 0 || (t.dtype != GNN_F32 && t.dtype != GNN_BF16) || (t.state_bits != 8 && t.state_bits != 32)) return GNN_ERR_INVALID_ARG;
    if (!(t.weight_decay >= 0.0f)) return GNN_ERR_INVALID_ARG;
    if (t.n == 0 || !t.grad) return GNN_OK;
    if (!t.param || !t.exp_avg || !t.exp_avg_sq) return GNN_ERR_INVALID_ARG;
    if (t.state_bits == 8 && (!t.scale || !t.scale_sq)) return GNN_ERR_INVALID_ARG;
    if (t.master && t.dtype == GNN_F32) return GNN_ERR_INVALID_ARG;
    const int size = t.dtype == GNN_F32 ? 4 : 2, state = t.state_bits == 8 ? 1 : 4;
    if (misaligned(t.param, size) || misaligned(t.grad, size) || misaligned(t.exp_avg, state) || misaligned(t.exp_avg_sq, state) ||
        misaligned(t.scale, 4) || misaligned(t.scale_sq, 4) || misaligned(t.master, 4))
        return GNN_ERR_INVALID_ARG;
    return GNN_OK;
}

}  // namespace

extern "C" GNN_API int gnn_adamw_step(const gnn_adamw_tensor *tensors, int64_t n_tensors, const gnn_adamw_opts *opts) {
    if (!opts || n_tensors < 0 || (n_tensors > 0 && !tensors)) return GNN_ERR_INVALID_ARG;
    const gnn_adamw_opts &o = *opts;
    if (o.step < 1 || !(o.lr >= 0.0) || !(o.beta1 >= 0.0 && o.beta1 < 1.0) || !(o.beta2 >= 0.0 && o.beta2 < 1.0) || !(o.eps >= 0.0)) return GNN_ERR_INVALID_ARG;
    int64_t blocks = 0, elements = 0;
    for (int64_t k = 0; k < n_tensors; ++k) {
        const int rc = check_tensor(tensors[k]);
        if (rc != GNN_OK) return rc;
        if (tensors[k].grad && tensors[k].n / kChunk > INT32_MAX / 4) return GNN_ERR_INVALID_ARG;
        if (tensors[k].grad) elements += tensors[k].n < (int64_t(1) << 40) ? tensors[k].n : 0;
    }
    (void)hipGetLastError();
    Step s{};
    s.b1 = float(o.beta1);
    s.c1 = float(1.0 - o.beta1);
    s.b2 = float(o.beta2);
    s.c2 = float(1.0 - o.beta2);
    s.rate = float(o.lr / (1.0 - pow(o.beta1, double(o.step))));
    s.root = float(1.0 / sqrt(1.0 - pow(o.beta2, double(o.step))));
    s.eps = float(o.eps);
    s.grad_scale = o.grad_scale;
    // few elements: shorter chunks, so that more workgroups share them
    s.chunk = elements < kShort ? kShortChunk : kChunk;
    auto flush = [&]() -> int {
        if (s.count == 0) return GNN_OK;
        auto *kernel = s.chunk == kChunk ? adamw_kernel<kChunk> : adamw_kernel<kShortChunk>;
        kernel<<<unsigned(blocks), kThreads, 0, static_cast<hipStream_t>(o.stream)>>>(s);
        s.count = 0;
        blocks = 0;
        GNN_HIP_TRY(hipGetLastError());
        return GNN_OK;
    };
    for (int64_t k = 0; k < n_tensors; ++k) {
        const gnn_adamw_tensor &d = tensors[k];
        if (d.n == 0 || !d.grad) continue;
        const int64_t more = (d.n + s.chunk - 1) / s.chunk;
        if (s.count == kTensors || blocks + more > INT32_MAX / 2) {
            const int rc = flush();
            if (rc != GNN_OK) return rc;
        }
        Tensor &t = s.t[s.count++];
        t.param = d.param;
        t.grad = d.grad;
        t.m = d.exp_avg;
        t.v = d.exp_avg_sq;
        t.m_scale = d.scale;
        t.v_scale = d.scale_sq;
        t.master = d.master;
        t.n = d.n;
        t.salt = uint32_t(o.seed) + uint32_t(o.step) * 0x3C6EF373u + uint32_t(k) * 0xBB67AE85u;
        t.decay = float(1.0 - o.lr * double(d.weight_decay));
        t.first = s.first[s.count - 1] = int32_t(blocks);
        t.flags = (d.dtype == GNN_BF16 ? 1 : 0) | (d.state_bits == 8 ? 2 : 0) | (d.master ? 4 : 0);
        blocks += more;
    }
    return flush();
}
