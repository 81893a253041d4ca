// Element types of the layers that take 16-bit operands (linear attention, layer normalisation):
// loads widen to float32 exactly, stores round to nearest (ties to even) once.  Internal to
// libdeer, not part of the ABI.
#pragma once

#include "common.h"

namespace deer {

struct F32 {
    typedef float T;
    static __device__ __forceinline__ float up(T x) { return x; }
    static __device__ __forceinline__ T down(float x) { return x; }
};
struct Bf16 {
    typedef __bf16 T;
    static __device__ __forceinline__ float up(T x) { return (float)x; }
    static __device__ __forceinline__ T down(float x) { return (__bf16)x; }
};
struct F16 {
    typedef _Float16 T;
    static __device__ __forceinline__ float up(T x) { return (float)x; }
    static __device__ __forceinline__ T down(float x) { return (_Float16)x; }
};

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// 16 bytes of a row from element d0 on, zero beyond its width
template <class Ty>
__device__ __forceinline__ v4u load_unit(const typename Ty::T *row, int d0, int width, bool vec) {
    constexpr int E = 16 / sizeof(typename Ty::T);
    v4u u = {0, 0, 0, 0};
    if (d0 >= width) return u;
    if (vec) return *(const v4u *)(row + d0);
    typename Ty::T x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = d0 + e < width ? row[d0 + e] : typename Ty::T(0);
    __builtin_memcpy(&u, x, 16);
    return u;
}

template <class Ty>
__device__ __forceinline__ void unpack_unit(v4u u, float (&x)[16 / sizeof(typename Ty::T)]) {
    typename Ty::T y[16 / sizeof(typename Ty::T)];
    __builtin_memcpy(y, &u, 16);
#pragma unroll
    for (int e = 0; e < (int)(16 / sizeof(typename Ty::T)); ++e) x[e] = Ty::up(y[e]);
}

// the counterpart of load_unit, rounding once
template <class Ty>
__device__ __forceinline__ void store_unit(typename Ty::T *row, int d0, int width, bool vec,
                                           const float (&x)[16 / sizeof(typename Ty::T)]) {
    constexpr int E = 16 / sizeof(typename Ty::T);
    if (d0 >= width) return;
    typename Ty::T y[E];
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = Ty::down(x[e]);
    if (vec) {
        v4u u;
        __builtin_memcpy(&u, y, 16);
        *(v4u *)(row + d0) = u;
        return;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (d0 + e < width) row[d0 + e] = y[e];
}

inline bool dtype_ok(int d) { return d == DEER_F32 || d == DEER_BF16 || d == DEER_F16; }
inline size_t dtype_size(int d) { return d == DEER_F32 ? 4 : 2; }

// f(type tag) for a runtime type
template <class Fn>
int with_dtype(int d, Fn f) {
    if (d == DEER_F32) return f(F32{});
    if (d == DEER_BF16) return f(Bf16{});
    return f(F16{});
}

}  // namespace deer
