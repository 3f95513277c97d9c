// Rows of binary32 or bfloat16 elements, 16 bytes of a row to a lane at a time.
#pragma once

#include "tc_internal.h"

namespace tc {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Elements of T in 16 bytes, and their conversions.
template <typename T>
struct Lane;
template <>
struct Lane<float> {
    static constexpr int kVec = 4;
    static __device__ __forceinline__ void widen(u32x4 v, float* f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
    }
    static __device__ __forceinline__ u32x4 narrow(const float* f) {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(f[i]);
        return v;
    }
    static __device__ __forceinline__ float get(uintptr_t a) { return gld<float>(a); }
    static __device__ __forceinline__ void put(uintptr_t a, float f) { gst<float>(a, f); }
};
// bfloat16: widened exactly, rounded to nearest even once, where a result is
// stored.
template <>
struct Lane<__bf16> {
    static constexpr int kVec = 8;
    static __device__ __forceinline__ void widen(u32x4 v, float* f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(v[i] << 16);
            f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ u32x4 narrow(const float* f) {
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            bf2 p = {static_cast<__bf16>(f[2 * i]), static_cast<__bf16>(f[2 * i + 1])};
            v[i] = __builtin_bit_cast(uint32_t, p);
        }
        return v;
    }
    static __device__ __forceinline__ float get(uintptr_t a) {
        return __uint_as_float(static_cast<uint32_t>(gld<uint16_t>(a)) << 16);
    }
    static __device__ __forceinline__ void put(uintptr_t a, float f) { gst<__bf16>(a, static_cast<__bf16>(f)); }
};

// Vector v of a row at address a: whole, or what the row has of it with zeros
// after the row's end.  EDGE: the row may end inside a vector.
template <typename T, bool EDGE>
__device__ __forceinline__ u32x4 load_vec(uintptr_t a, int v, int cols) {
    constexpr int V = Lane<T>::kVec;
    const int left = cols - v * V;
    if (left >= V) return gld_u<u32x4>(a + static_cast<uintptr_t>(v) * 16);
    u32x4 r = {0, 0, 0, 0};
    if (EDGE && left > 0) {
        float f[V];
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = i < left ? Lane<T>::get(a + static_cast<uintptr_t>(v) * 16 + i * sizeof(T)) : 0.0f;
        r = Lane<T>::narrow(f);
    }
    return r;
}

// The same where it is needed only later.  A load of single elements would be
// waited for at once, with all loads before it; so of the vector that the row
// ends inside, the row's last 16 bytes are loaded, which are in the row where
// it has that many, and `settle` moves their elements down to their places
// (12,764 rows of 8,513 bfloat16, forward: 188 us by elements, 109 so; two
// workers' 22,424 rows of 722, backward: 59 and 50).  Not for the long rows'
// kernels, whose lanes may have stored over the elements before by then.
// NT: past the caches.
template <typename T, bool EDGE, bool NT = false>
__device__ __forceinline__ u32x4 load_ahead(uintptr_t a, int v, int cols) {
    constexpr int V = Lane<T>::kVec;
    if ((!EDGE && !NT) || cols < V) return load_vec<T, EDGE>(a, v, cols);
    const int c = v * V;
    u32x4 r = {0, 0, 0, 0};
    const uintptr_t at = a + static_cast<uintptr_t>(c + V <= cols ? c : cols - V) * sizeof(T);
    if (c < cols) r = NT ? gld_u_nt<u32x4>(at) : gld_u<u32x4>(at);
    return r;
}
template <typename T, bool EDGE>
__device__ __forceinline__ void settle(float* f, int v, int cols) {
    constexpr int V = Lane<T>::kVec;
    if (!EDGE || cols < V || v != cols / V) return;
    const int by = V - cols % V;
#pragma unroll
    for (int m = V / 2; m > 0; m >>= 1)
        if (by & m)
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] = e + m < V ? f[e + m] : 0.0f;
}

template <typename T, bool EDGE, bool NT = false>
__device__ __forceinline__ void store_vec(uintptr_t a, int v, int cols, const float* f) {
    constexpr int V = Lane<T>::kVec;
    const int left = cols - v * V;
    if (left >= V) {
        if (NT)
            gst_u_nt<u32x4>(a + static_cast<uintptr_t>(v) * 16, Lane<T>::narrow(f));
        else
            gst_u<u32x4>(a + static_cast<uintptr_t>(v) * 16, Lane<T>::narrow(f));
    } else if (EDGE) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < left) Lane<T>::put(a + static_cast<uintptr_t>(v) * 16 + i * sizeof(T), f[i]);
    }
}

}  // namespace
}  // namespace tc
