// Rows of vertex matrices in fp32 and bf16 for the kernels of norm.hip, loss.hip, adamw.hip, lookup.hip, store.hip and muon.hip: VEC elements at a time, in fp32
// registers, at the alignment of one element (global loads and stores of 16 bytes need no more).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

struct gnn_bf16 { uint16_t bits; };

typedef float gnn_f32x4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t gnn_u32x4 __attribute__((ext_vector_type(4), aligned(2)));
typedef float gnn_f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 gnn_bf16x2 __attribute__((ext_vector_type(2)));

template <typename T> struct gnn_rows;

template <> struct gnn_rows<float> {
    static constexpr int VEC = 4;
    typedef gnn_f32x4 raw;
    static __device__ __forceinline__ raw fetch(const float *p) { return *reinterpret_cast<const gnn_f32x4 *>(p); }
    static __device__ __forceinline__ void put(float *p, raw t) { *reinterpret_cast<gnn_f32x4 *>(p) = t; }
    static __device__ __forceinline__ void unpack(raw t, float (&v)[4]) { v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w; }
    static __device__ __forceinline__ raw pack(const float (&v)[4]) { return raw{v[0], v[1], v[2], v[3]}; }
    static __device__ __forceinline__ float get(const float *p) { return *p; }
    static __device__ __forceinline__ void set(float *p, float v) { *p = v; }
};

template <> struct gnn_rows<gnn_bf16> {
    static constexpr int VEC = 8;
    typedef gnn_u32x4 raw;
    static __device__ __forceinline__ raw fetch(const gnn_bf16 *p) { return *reinterpret_cast<const gnn_u32x4 *>(p); }
    static __device__ __forceinline__ void put(gnn_bf16 *p, raw t) { *reinterpret_cast<gnn_u32x4 *>(p) = t; }
    static __device__ __forceinline__ void unpack(raw t, float (&v)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(t[i] << 16);
            v[2 * i + 1] = __uint_as_float(t[i] & 0xFFFF0000u);
        }
    }
    // to the nearest, ties to even: one instruction for two elements
    static __device__ __forceinline__ raw pack(const float (&v)[8]) {
        raw t;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            t[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(gnn_f32x2{v[2 * i], v[2 * i + 1]}, gnn_bf16x2));
        return t;
    }
    static __device__ __forceinline__ float get(const gnn_bf16 *p) { return __uint_as_float(uint32_t(p->bits) << 16); }
    static __device__ __forceinline__ void set(gnn_bf16 *p, float v) { p->bits = __builtin_bit_cast(uint16_t, __bf16(v)); }
};

// VEC elements as they lie in memory: a whole vector, half a bf16 vector, or one element of rows narrower than that.  NT: data that is not
// read again soon goes past the caches (reads alone 6.2 -> 7.0 TB/s, copies 6.2 -> 6.5 TB/s at 2.5 GB).
template <typename T, int VEC, bool NT> struct gnn_strip {
    static_assert(VEC == gnn_rows<T>::VEC, "a whole vector");
    typedef typename gnn_rows<T>::raw raw;
    raw v;
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (NT) v = __builtin_nontemporal_load(reinterpret_cast<const raw *>(p));
        else v = gnn_rows<T>::fetch(p);
    }
    __device__ __forceinline__ void store(T *p) const {
        if constexpr (NT) __builtin_nontemporal_store(v, reinterpret_cast<raw *>(p));
        else gnn_rows<T>::put(p, v);
    }
    __device__ __forceinline__ void get(float (&f)[VEC]) const { gnn_rows<T>::unpack(v, f); }
    __device__ __forceinline__ void set(const float (&f)[VEC]) { v = gnn_rows<T>::pack(f); }
    // unpacked again from here on: elements that stay unpacked take twice the registers
    __device__ __forceinline__ void forget() { asm volatile("" : "+v"(v)); }
};
typedef uint32_t gnn_u32x2 __attribute__((ext_vector_type(2), aligned(2)));
template <bool NT> struct gnn_strip<gnn_bf16, 4, NT> {
    gnn_u32x2 v;
    __device__ __forceinline__ void load(const gnn_bf16 *p) {
        if constexpr (NT) v = __builtin_nontemporal_load(reinterpret_cast<const gnn_u32x2 *>(p));
        else v = *reinterpret_cast<const gnn_u32x2 *>(p);
    }
    __device__ __forceinline__ void store(gnn_bf16 *p) const {
        if constexpr (NT) __builtin_nontemporal_store(v, reinterpret_cast<gnn_u32x2 *>(p));
        else *reinterpret_cast<gnn_u32x2 *>(p) = v;
    }
    __device__ __forceinline__ void get(float (&f)[4]) const {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f[2 * i] = __uint_as_float(v[i] << 16);
            f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
        }
    }
    __device__ __forceinline__ void set(const float (&f)[4]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(gnn_f32x2{f[2 * i], f[2 * i + 1]}, gnn_bf16x2));
    }
};
template <typename T, bool NT> struct gnn_strip<T, 1, NT> {
    float v;
    __device__ __forceinline__ void load(const T *p) { v = gnn_rows<T>::get(p); }
    __device__ __forceinline__ void store(T *p) const { gnn_rows<T>::set(p, v); }
    __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = v; }
    __device__ __forceinline__ void set(const float (&f)[1]) { v = f[0]; }
};

// CTRL: a permutation of the 16 lanes of a row
template <int CTRL> __device__ __forceinline__ float gnn_from_lane(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

template <typename T, int VEC, bool NT = false> __device__ __forceinline__ void gnn_load_row(const T *p, float (&v)[VEC]) {
    gnn_strip<T, VEC, NT> t;
    t.load(p);
    t.get(v);
}
template <typename T, int VEC, bool NT = false> __device__ __forceinline__ void gnn_store_row(T *p, const float (&v)[VEC]) {
    gnn_strip<T, VEC, NT> t;
    t.set(v);
    t.store(p);
}
