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
