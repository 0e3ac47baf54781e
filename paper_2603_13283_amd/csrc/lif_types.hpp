// lif_types.hpp -- the element types of the sequence and answer operators
// (float32, bfloat16, float16): conversion to and from float32, and loads and
// stores of several contiguous elements by one lane.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/lif.h"

namespace lif {

using bf16 = __bf16;
using f16 = _Float16;

template <typename T> __device__ __forceinline__ float to_f32(T v) { return (float)v; }

// One rounding to nearest even.
template <typename T> __device__ __forceinline__ T from_f32(float v) { return (T)v; }

// N contiguous elements at an address that is aligned to one element only:
// one wide access (the hardware takes unaligned ones), so that rows of any
// length and views with any offset are read alike.
template <typename T, int N> struct __attribute__((packed, aligned(sizeof(T)))) Elems {
    T v[N];
};
template <typename T, int N> __device__ __forceinline__ void load_elems(const T* p, T (&v)[N])
{
    const Elems<T, N> q = *reinterpret_cast<const Elems<T, N>*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = q.v[i];
}
template <typename T, int N> __device__ __forceinline__ void store_elems(T* p, const T (&v)[N])
{
    Elems<T, N> q;
#pragma unroll
    for (int i = 0; i < N; ++i) q.v[i] = v[i];
    *reinterpret_cast<Elems<T, N>*>(p) = q;
}

// Calls fn with a value of the element type that `dtype` names; false for a
// type there is none of.
template <typename Fn> bool with_dtype(int dtype, Fn&& fn)
{
    switch (dtype) {
        case LIF_F32: fn(float()); return true;
        case LIF_BF16: fn(bf16()); return true;
        case LIF_F16: fn(f16()); return true;
        default: return false;
    }
}

}  // namespace lif
